"""Host-side driver of the early-exit decoder: device buffers and the layer loop.

Everything numeric runs in libadept (binding.py); this module only owns
device memory (torch tensors), lays out the per-token bookkeeping (positions,
sequence ids, cache slots) and calls the C ABI in order:

    adept_embed -> adept_token_init -> adept_layer_step(i), i = 1..N
                -> adept_final_logits [-> adept_argmax]

(the LayerNorm family: adept_embed_positions and adept_final_logits_layernorm
in place of the embedding gather and the RMSNorm head).

A prefill runs the rows of a [B, T] prompt batch (row b*T + p); a decode
step runs one new token per sequence against the cache the prefill (and
earlier steps) filled, with generated entries for every skipped layer.

The cache is either a KVCache (s_max slots for each sequence) or a
PagedKVCache: pages that sequences take as they grow, share and give back, in
the model's type or in 8 bits.  Over either, a prompt can be run in pieces
(prefill with start), and drafted tokens can be verified (verify,
generate_drafted).
"""
from __future__ import annotations

import ctypes
import dataclasses
import math

import numpy as np
import torch

from . import binding as B

_TORCH_DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@dataclasses.dataclass
class KVCache:
    k: torch.Tensor       # [N, n_seq * s_max, H, hd]
    v: torch.Tensor
    n_seq: int
    s_max: int

    @property
    def n_slots(self):
        return self.n_seq * self.s_max


class PagedKVCache:
    """The K/V cache of n_seq sequences in n_pages pages of page_size token slots per layer
    (k, v [N, n_pages * page_size, H, hd]), each sequence up to max_pages of them; kv_dtype:
    "f32", "bf16" or "fp8" (e4m3 codes with a scale byte per slot and head, k_scale, v_scale).
    page_table [n_seq, max_pages] int32 on the device (-1: no page); which pages are free is
    known on the host.  One page more, which no table names, takes the K/V of tokens that have
    no place.  A pass over an "fp8" cache holds its own rows' K and V of all layers in the
    model's type beside it: long prompts are better run in pieces (prefill with start).  Its
    decode passes need the K/V generation inside the layers (kv_fused, bf16 models); without
    it they run as prompts do, their attention in tiles: right, and slower.

    Sequences may share pages (fork): a page goes back when the last of them gives it up, and a
    pass that writes into a shared one gets a copy of it first (reserve with start)."""

    def __init__(self, n_layers, n_heads, head_dim, n_seq, n_pages, page_size, max_pages, kv_dtype,
                 device):
        dims = (n_layers, (n_pages + 1) * page_size, n_heads, head_dim)
        tdt = torch.uint8 if kv_dtype == "fp8" else _TORCH_DT[kv_dtype]
        self.k = torch.empty(dims, dtype=tdt, device=device)
        self.v = torch.empty(dims, dtype=tdt, device=device)
        self.k_scale = self.v_scale = None
        if kv_dtype == "fp8":
            self.k_scale = torch.empty(dims[:3], dtype=torch.uint8, device=device)
            self.v_scale = torch.empty(dims[:3], dtype=torch.uint8, device=device)
        self.kv_dtype, self.n_seq, self.page_size, self.max_pages = (kv_dtype, n_seq, page_size,
                                                                     max_pages)
        self.page_table = torch.full((n_seq, max_pages), -1, dtype=torch.int32, device=device)
        self._free = list(range(n_pages - 1, -1, -1))
        self._pages = [[] for _ in range(n_seq)]
        self._users = [0] * n_pages        # sequences that a page belongs to
        self.shared_pages = 0              # pages that belong to several
        self.kv = self.layer_kv(1)

    @property
    def n_slots(self):
        return self.k.shape[1]

    @property
    def s_max(self):
        return self.max_pages * self.page_size

    @property
    def n_pages(self):
        return len(self._users)

    @property
    def free_pages(self):
        return len(self._free)

    def layer_kv(self, layer):
        """Descriptor of one layer (binding.paged_kv), for the operators of a single layer."""
        i = layer - 1
        scales = (None, None) if self.k_scale is None else (self.k_scale[i], self.v_scale[i])
        return B.paged_kv(self.k[i], self.v[i], self.page_size, *scales)

    def _check_sequence(self, seq):
        if not 0 <= seq < self.n_seq:
            raise ValueError(f"sequence {seq}: the cache has {self.n_seq}")

    def _take(self, n):
        pages = [self._free.pop() for _ in range(n)]
        for p in pages:
            self._users[p] = 1
        return pages

    def _give(self, pages):
        """Pages that a sequence no longer has; the ones that no other has are free."""
        for p in reversed(pages):
            self._users[p] -= 1
            if self._users[p] == 0:
                self._free.append(p)
            elif self._users[p] == 1:
                self.shared_pages -= 1

    def _write_table(self, seq):
        row = self._pages[seq]
        self.page_table[seq, :len(row)] = torch.tensor(row, dtype=torch.int32)

    def _copy(self, src, dst, n_tokens=None):
        """Pages of all layers (binding.paged_copy)."""
        if src:
            up = lambda x: torch.tensor(x, dtype=torch.int32, device=self.k.device)
            B.paged_copy(self.kv, self.k.shape[0], up(src), up(dst),
                         None if n_tokens is None else up(n_tokens))

    def _take_copies(self, src, n_tokens=None):
        """New pages with what the pages src hold; none are taken where the copy fails."""
        new = self._take(len(src))
        try:
            self._copy(src, new, n_tokens)
        except BaseException:
            self._give(new)
            raise
        return new

    def reserve(self, lengths, start=None):
        """Pages for lengths[b] tokens of sequence b (a dict or one number for all); start[b]: the
        position from which on they are going to be written (a dict or one number; None: behind
        the tokens that are shared), whose pages a sequence then gets for itself.  Raises
        ValueError, with nothing taken, where they do not fit."""
        if not isinstance(lengths, dict):
            lengths = {b: int(lengths) for b in range(self.n_seq)}
        for b in lengths:
            self._check_sequence(b)
        for b, n in lengths.items():
            if not 0 <= n <= self.s_max:
                raise ValueError(f"{n} tokens of sequence {b}: a sequence holds up to {self.s_max}")
        more = {b: -(-n // self.page_size) - len(self._pages[b]) for b, n in lengths.items()}
        need = sum(m for m in more.values() if m > 0)
        own = []                            # (sequence, which of its pages)
        if start is not None:
            users = list(self._users)
            for b, n in lengths.items():
                first = int(start.get(b, n) if isinstance(start, dict) else start)
                last = min(-(-n // self.page_size), len(self._pages[b]))
                for i in range(max(first, 0) // self.page_size, last):
                    if users[self._pages[b][i]] > 1:
                        users[self._pages[b][i]] -= 1
                        own.append((b, i))
        if need + len(own) > len(self._free):
            raise ValueError(f"{need + len(own)} more pages needed, {len(self._free)} free")
        new = self._take_copies([self._pages[b][i] for b, i in own])
        for (b, i), page in zip(own, new):
            self._give([self._pages[b][i]])
            self._pages[b][i] = page
            self.page_table[b, i] = page
        for b, m in more.items():
            if m > 0:
                new = self._take(m)
                at = len(self._pages[b])
                self._pages[b] += new
                self.page_table[b, at:at + m] = torch.tensor(new, dtype=torch.int32)

    def release(self, seq):
        """Gives the sequence's pages back (its tokens are gone)."""
        self.truncate(seq, 0)

    def truncate(self, seq, length):
        """Keeps the first `length` tokens of a sequence and gives back the pages behind them."""
        self._check_sequence(seq)
        if length < 0:
            raise ValueError(f"{length} tokens of sequence {seq}")
        keep = -(-length // self.page_size)
        self._give(self._pages[seq][keep:])
        self._pages[seq] = self._pages[seq][:keep]
        self.page_table[seq, keep:].fill_(-1)

    def fork(self, src, dst, length):
        """The sequences dst (one or several, without pages) continue from the first `length`
        tokens of sequence src: they share its full pages, and each gets a copy of what is
        used of the open one.  Raises ValueError, with nothing taken, where that does not fit."""
        dst = [int(b) for b in dst] if hasattr(dst, "__iter__") else [int(dst)]
        for b in (src, *dst):
            self._check_sequence(b)
        if src in dst or len(set(dst)) < len(dst) or any(self._pages[b] for b in dst):
            raise ValueError("a fork goes to other sequences, each without pages of its own")
        full, left = divmod(length, self.page_size)
        if length < 0 or full + (left > 0) > len(self._pages[src]):
            raise ValueError(f"{length} tokens: sequence {src} has pages for "
                             f"{len(self._pages[src]) * self.page_size}")
        if left and len(dst) > len(self._free):
            raise ValueError(f"{len(dst)} more pages needed, {len(self._free)} free")
        new = (self._take_copies([self._pages[src][full]] * len(dst), [left] * len(dst)) if left
               else [])
        for k, b in enumerate(dst):
            self._pages[b] = self._pages[src][:full] + new[k:k + 1]
            for p in self._pages[b][:full]:
                self._users[p] += 1
                self.shared_pages += self._users[p] == 2
            self._write_table(b)

    def _move(self, n_pages):
        """Pages from the n_pages-th on into free ones below; how many."""
        src = [p for p in range(n_pages, self.n_pages) if self._users[p]]
        holes = sorted(p for p in self._free if p < n_pages)[:len(src)]
        self._copy(src, holes)
        to = dict(zip(src, holes))
        for p, q in to.items():
            self._users[q], self._users[p] = self._users[p], 0
        for b, pages in enumerate(self._pages):
            if any(p in to for p in pages):
                self._pages[b] = [to.get(p, p) for p in pages]
                self._write_table(b)
        self._free = [p for p in range(self.n_pages - 1, -1, -1) if not self._users[p]]
        return len(src)

    def compact(self):
        """Moves the pages in use to the front of the cache; how many were moved."""
        return self._move(self.n_pages - len(self._free))

    def resize(self, n_pages):
        """Another number of pages: more of them, or memory given back after a peak (pages in use
        behind the new end are moved first).  The old tensors and the new ones are held together
        for the time of the call, and descriptors of the old ones are no longer the cache's.
        Raises ValueError where more pages are in use; what fails for want of memory leaves the
        cache as it was."""
        used = self.n_pages - len(self._free)
        if n_pages < used or n_pages < 1:
            raise ValueError(f"{n_pages} pages, {used} in use")
        held = {name: getattr(self, name) for name in ("k", "v", "k_scale", "v_scale")}
        new = {name: old if old is None else
               torch.empty((old.shape[0], (n_pages + 1) * self.page_size, *old.shape[2:]),
                           dtype=old.dtype, device=old.device) for name, old in held.items()}
        if n_pages < self.n_pages:
            self._move(n_pages)
        keep = min(n_pages, self.n_pages) * self.page_size
        for name, old in held.items():
            if old is not None:
                new[name][:, :keep] = old[:, :keep]
        for name, t in new.items():
            setattr(self, name, t)
        self._users = (self._users + [0] * (n_pages - self.n_pages))[:n_pages]
        self._free = [p for p in range(n_pages - 1, -1, -1) if not self._users[p]]
        self.kv = self.layer_kv(1)

    def slots(self, pos, seq):
        """Slots (int32) of tokens at pos of sequences seq, both int32 device tensors; the last
        slot of the cache where a sequence has no page, or is none of the cache's."""
        p, b = pos.long(), seq.long()
        at = (p // self.page_size).clamp(0, self.max_pages - 1)
        page = self.page_table[b.clamp(0, self.n_seq - 1), at]
        there = (page >= 0) & (p >= 0) & (p < self.s_max) & (b >= 0) & (b < self.n_seq)
        return torch.where(there, page * self.page_size + (p % self.page_size).to(torch.int32),
                           self.n_slots - 1).to(torch.int32)


@dataclasses.dataclass
class PassState:
    """Device buffers of one token pass (prefill batch or decode step)."""
    n_tok: int
    h: list                # two [n_tok, D] buffers (ping-pong)
    inertia: torch.Tensor  # [n_tok, D] f32
    pos: torch.Tensor
    seq: torch.Tensor
    slot: torch.Tensor
    active: list           # two [n_tok] int32
    counts: torch.Tensor   # int32 [4]: n_active[0], n_active[1], n_exited, spare
    exited: torch.Tensor
    exit_layer: torch.Tensor
    exit_flag: torch.Tensor
    sim_out: torch.Tensor
    force_layer: torch.Tensor | None
    q_buf: torch.Tensor
    attn_out: torch.Tensor
    ffn_act: torch.Tensor
    workspace: torch.Tensor | None = None
    # passes over an 8-bit cache: K and V of the pass's rows as computed, [N, n_tok, H, hd]
    new_k: torch.Tensor | None = None
    new_v: torch.Tensor | None = None
    cache_slot: torch.Tensor | None = None

    def final_h(self, row):
        """[D] final state of a row (state at exit, or after the last layer)."""
        el = int(self.exit_layer[row])
        return self.h[el & 1][row]


@dataclasses.dataclass
class PassResult:
    logits: torch.Tensor       # [n_rows, V] f32 for the requested rows
    rows: torch.Tensor         # token rows of the logits
    exit_layer: torch.Tensor   # [n_tok]
    state: PassState


class DecoderModel:
    """A pre-norm decoder held on the device in the library's layout.

    shape.family "llama": weights like adept_inputs.decoder_weights() (numpy,
    per layer) or adept_inputs.decoder_weights_torch() (stacked torch tensors
    on device).  "gpt2": like adept_inputs.gpt2_weights() or
    gpt2_weights_torch(); the LayerNorm gains and shifts are folded into the
    projections that follow them (w_qkv / b_qkv, w_fc / b_fc) and the LM
    head is the token embedding.
    """

    def __init__(self, shape, weights, dtype="bf16", device="cuda", rope_max_pos=4096,
                 hsm_weights=None, kv_fused=True, quant=False):
        self.shape = shape
        # the layers' matrices and the head in 4 bits (bf16): passes of at most 64 tokens read
        # those, larger ones the bf16 matrices, which then hold the same values
        self.quant, self._quant_struct = None, None
        if quant and dtype != "bf16":
            raise ValueError("weights in 4 bits go with a bf16 model")
        # decode passes in bf16: exited rows' K/V from the later layers' QKV
        # GEMMs (True) or one grouped generation after the last layer (False)
        self.kv_fused = kv_fused
        self.dtype = dtype
        self.tdt = _TORCH_DT[dtype]
        self.device = torch.device(device)
        self.gpt2 = getattr(shape, "family", "llama") == "gpt2"
        N, D, Dq, F = shape.n_layers, shape.d_model, shape.d_q, shape.d_ff
        dev, tdt = self.device, self.tdt

        def up(x):
            if isinstance(x, torch.Tensor):
                return x.to(dev, tdt).contiguous()
            return torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(dev).to(tdt)

        self.hsm, self._hsm_struct = None, None
        if self.gpt2:
            if dtype != "bf16" or hsm_weights is not None:
                raise ValueError("the LayerNorm family runs in bf16 without a mapper")
            self._init_gpt2(weights, up)
            if quant:
                self._quantise()
            return
        self.b_qkv = self.b_o = self.b_fc = self.b_proj = None
        if isinstance(weights.get("layers"), list):
            L = weights["layers"]
            stack = lambda k: up(np.stack([lw[k] for lw in L]))
            self.attn_norm, self.ffn_norm = stack("attn_norm"), stack("ffn_norm")
            self.w_qkv = up(np.stack([np.concatenate([lw["wq"], lw["wk"], lw["wv"]]) for lw in L]))
            self.w_o = stack("wo")
            self.w_gate, self.w_up, self.w_down = stack("w_gate"), stack("w_up"), stack("w_down")
        else:
            self.attn_norm, self.ffn_norm = up(weights["attn_norm"]), up(weights["ffn_norm"])
            self.w_qkv = torch.empty((N, 3 * Dq, D), dtype=tdt, device=dev)
            self.w_qkv[:, :Dq].copy_(weights["wq"])
            self.w_qkv[:, Dq:2 * Dq].copy_(weights["wk"])
            self.w_qkv[:, 2 * Dq:].copy_(weights["wv"])
            self.w_o = up(weights["wo"])
            self.w_gate, self.w_up, self.w_down = (up(weights["w_gate"]), up(weights["w_up"]),
                                                   up(weights["w_down"]))
        self.embed = up(weights["embed"])
        self.final_norm = up(weights["final_norm"])
        self.lm_head = up(weights["lm_head"])
        assert self.w_qkv.shape == (N, 3 * Dq, D) and self.w_down.shape == (N, D, F)
        # fold the pre-norm gains into the projections that consume the normalised
        # state (the library applies only the 1/rms row factor)
        B.fold_gain(self.w_qkv, self.attn_norm)
        B.fold_gain(self.w_gate, self.ffn_norm)
        B.fold_gain(self.w_up, self.ffn_norm)
        # optional hidden state mapper (Section 4.2) of the exiting rows: a dict
        # like adept_inputs.hsm_weights(); None keeps the identity mapper
        if hsm_weights is not None:
            self.hsm = {k: (v if k in ("conv", "conv_b") else up(v)) for k, v in hsm_weights.items()}
            self._hsm_struct = B.hsm_weights(self.hsm)
        self.rope_max_pos = rope_max_pos
        half = shape.head_dim // 2
        self.rope_cos = torch.empty((rope_max_pos, half), dtype=torch.float32, device=dev)
        self.rope_sin = torch.empty_like(self.rope_cos)
        B.rope_table(rope_max_pos, shape.head_dim, shape.rope_theta, self.rope_cos, self.rope_sin)
        if quant:
            self._quantise()

    def _quantise(self):
        """The matrices in 4 bits, and the bf16 ones rounded to what those hold."""
        self.quant = {}
        for name in ("w_qkv", "w_o", "w_gate", "w_up", "w_down"):
            w = getattr(self, name)
            if w is None:
                self.quant[name] = None
                continue
            q = self.quant[name] = B.quant_weights(w.shape[1], w.shape[2], self.device, w.shape[0])
            held = torch.empty_like(w)      # the given matrices keep their values
            for i in range(w.shape[0]):
                B.quant_pack(w[i], q, i)
                B.quant_unpack(q, held[i], i)
            setattr(self, name, held)
        head = self.quant["lm_head"] = B.quant_weights(*self.lm_head.shape, self.device)
        B.quant_pack(self.lm_head, head)
        self.lm_head = torch.empty_like(self.lm_head)
        B.quant_unpack(head, self.lm_head)

    def _init_gpt2(self, weights, up):
        s = self.shape
        N, D, Dq, F = s.n_layers, s.d_model, s.d_q, s.d_ff
        if isinstance(weights.get("layers"), list):
            L = weights["layers"]
            stack = lambda k: up(np.stack([lw[k] for lw in L]))
            cat = lambda ks: up(np.stack([np.concatenate([lw[k] for k in ks]) for lw in L]))
            ln1_g, ln1_b, ln2_g, ln2_b = (stack("ln1_g"), stack("ln1_b"), stack("ln2_g"),
                                          stack("ln2_b"))
            self.w_qkv, self.b_qkv = cat(("wq", "wk", "wv")), cat(("bq", "bk", "bv"))
            self.w_o, self.b_o = stack("wo"), stack("bo")
            self.w_gate, self.b_fc = stack("w_fc"), stack("b_fc")
            self.w_down, self.b_proj = stack("w_proj"), stack("b_proj")
        else:
            ln1_g, ln1_b = up(weights["ln1_g"]), up(weights["ln1_b"])
            ln2_g, ln2_b = up(weights["ln2_g"]), up(weights["ln2_b"])
            self.w_qkv = torch.cat([up(weights[k]) for k in ("wq", "wk", "wv")], 1).contiguous()
            self.b_qkv = torch.cat([up(weights[k]) for k in ("bq", "bk", "bv")], 1).contiguous()
            self.w_o, self.b_o = up(weights["wo"]), up(weights["bo"])
            self.w_gate, self.b_fc = up(weights["w_fc"]), up(weights["b_fc"])
            self.w_down, self.b_proj = up(weights["w_proj"]), up(weights["b_proj"])
        self.w_up = None
        self.embed, self.pos_embed = up(weights["embed"]), up(weights["pos_embed"])
        self.final_ln_g, self.final_ln_b = up(weights["final_ln_g"]), up(weights["final_ln_b"])
        self.lm_head = self.embed      # tied
        assert self.w_qkv.shape == (N, 3 * Dq, D) and self.b_qkv.shape == (N, 3 * Dq)
        assert self.w_down.shape == (N, D, F) and self.pos_embed.shape == (s.max_pos, D)
        # LayerNorm shift into the bias (on the unfolded weights), then the
        # gain into the weights: LN(x) W^T + b = xh (W diag g)^T + (b + W beta)
        B.fold_bias(self.w_qkv, ln1_b, self.b_qkv)
        B.fold_gain(self.w_qkv, ln1_g)
        B.fold_bias(self.w_gate, ln2_b, self.b_fc)
        B.fold_gain(self.w_gate, ln2_g)
        self.rope_cos = self.rope_sin = None
        self.rope_max_pos = s.max_pos     # the position table bounds the positions

    # ------------------------------------------------------------------ buffers
    def new_cache(self, n_seq, s_max, fill=None):
        s = self.shape
        dims = (s.n_layers, n_seq * s_max, s.n_heads, s.head_dim)
        if fill is None:
            k = torch.empty(dims, dtype=self.tdt, device=self.device)
            v = torch.empty(dims, dtype=self.tdt, device=self.device)
        else:
            k = torch.full(dims, fill, dtype=self.tdt, device=self.device)
            v = torch.full(dims, fill, dtype=self.tdt, device=self.device)
        return KVCache(k, v, n_seq, s_max)

    def new_paged_cache(self, n_seq, n_pages, page_size=64, max_pages=None, kv_dtype=None):
        """A PagedKVCache of this model's layers; kv_dtype "fp8" or (default) the model's type;
        max_pages: of one sequence (default: all)."""
        s = self.shape
        kv_dtype = self.dtype if kv_dtype is None else kv_dtype
        if kv_dtype not in (self.dtype, "fp8"):
            raise ValueError(f"a {self.dtype} model has a {self.dtype} or fp8 cache, not {kv_dtype}")
        return PagedKVCache(s.n_layers, s.n_heads, s.head_dim, n_seq, n_pages, page_size,
                            n_pages if max_pages is None else max_pages, kv_dtype, self.device)

    def new_state(self, n_tok, pos, seq, slot, force_layer=None):
        s, dev, tdt = self.shape, self.device, self.tdt
        i32 = dict(dtype=torch.int32, device=dev)
        st = PassState(
            n_tok=n_tok,
            h=[torch.empty((n_tok, s.d_model), dtype=tdt, device=dev) for _ in range(2)],
            inertia=torch.empty((n_tok, s.d_model), dtype=torch.float32, device=dev),
            pos=pos, seq=seq, slot=slot,
            active=[torch.empty(n_tok, **i32) for _ in range(2)],
            counts=torch.zeros(4, **i32),
            exited=torch.empty(n_tok, **i32),
            exit_layer=torch.empty(n_tok, **i32),
            exit_flag=torch.empty(max(n_tok, 4), dtype=torch.uint8, device=dev),
            sim_out=torch.empty(n_tok, dtype=torch.float64, device=dev),
            force_layer=force_layer,
            q_buf=torch.empty((n_tok, s.d_q), dtype=tdt, device=dev),
            attn_out=torch.empty((n_tok, s.d_q), dtype=tdt, device=dev),
            ffn_act=torch.empty((n_tok, s.d_ff), dtype=tdt, device=dev),
        )
        return st

    def layer_args(self, st, cache, cfg, attn_tiles):
        s = self.shape
        a = B.LayerArgs()
        a.dtype = B.dtype_code(self.dtype)
        a.n_layers, a.d_model, a.n_heads = s.n_layers, s.d_model, s.n_heads
        a.head_dim, a.d_ff = s.head_dim, s.d_ff
        a.rms_eps = s.ln_eps if self.gpt2 else s.rms_eps
        a.exit = cfg
        a.w_qkv, a.w_o, a.w_gate = B.ptr(self.w_qkv), B.ptr(self.w_o), B.ptr(self.w_gate)
        a.w_up, a.w_down = B.ptr(self.w_up), B.ptr(self.w_down)
        a.rope_cos, a.rope_sin, a.rope_max_pos = B.ptr(self.rope_cos), B.ptr(self.rope_sin), self.rope_max_pos
        a.family = B.FAMILY_GPT2 if self.gpt2 else B.FAMILY_LLAMA
        a.b_qkv, a.b_o = B.ptr(self.b_qkv), B.ptr(self.b_o)
        a.b_fc, a.b_proj = B.ptr(self.b_fc), B.ptr(self.b_proj)
        a.n_tok, a.max_active, a.n_seq, a.s_max = st.n_tok, st.n_tok, cache.n_seq, cache.s_max
        a.attn_tiles = int(attn_tiles)
        a.kv_fused = int(bool(self.kv_fused) and not attn_tiles and self.dtype == "bf16")
        a.h[0], a.h[1] = B.ptr(st.h[0]), B.ptr(st.h[1])
        a.inertia, a.pos, a.seq, a.slot = B.ptr(st.inertia), B.ptr(st.pos), B.ptr(st.seq), B.ptr(st.slot)
        a.active[0], a.active[1] = B.ptr(st.active[0]), B.ptr(st.active[1])
        cp = B.ptr(st.counts)
        a.n_active[0], a.n_active[1], a.n_exited = cp, cp + 4, cp + 8
        a.exited, a.exit_layer, a.exit_flag = B.ptr(st.exited), B.ptr(st.exit_layer), B.ptr(st.exit_flag)
        a.sim_out = B.ptr(st.sim_out)
        a.force_layer = B.ptr(st.force_layer)
        paged = isinstance(cache, PagedKVCache)
        if paged and cache.kv_dtype == "fp8":
            if not a.kv_fused:      # generated after each layer, where the next one finds them
                a.attn_tiles = 1
            if st.new_k is None:
                dims = (s.n_layers, st.n_tok, s.n_heads, s.head_dim)
                st.new_k = torch.empty(dims, dtype=self.tdt, device=self.device)
                st.new_v = torch.empty(dims, dtype=self.tdt, device=self.device)
                st.cache_slot = st.slot
                st.slot = torch.arange(st.n_tok, dtype=torch.int32, device=self.device)
                a.slot = B.ptr(st.slot)
            a.k_cache, a.v_cache, a.n_slots = B.ptr(st.new_k), B.ptr(st.new_v), st.n_tok
        else:
            a.k_cache, a.v_cache, a.n_slots = B.ptr(cache.k), B.ptr(cache.v), cache.n_slots
        a.q_buf, a.attn_out, a.ffn_act = B.ptr(st.q_buf), B.ptr(st.attn_out), B.ptr(st.ffn_act)
        a.hsm = ctypes.addressof(self._hsm_struct) if self._hsm_struct is not None else None
        if self.quant is not None:
            if self._quant_struct is None:
                self._quant_struct = B.quant_layers(a, *(self.quant[n] for n in (
                    "w_qkv", "w_o", "w_gate", "w_up", "w_down")))
            need = B.layer_quant_workspace_bytes(a, self._quant_struct, cache.kv if paged else None,
                                                 cache.max_pages if paged else 0)
        else:
            need = (B.layer_paged_workspace_bytes(a, cache.kv, cache.max_pages) if paged
                    else B.layer_workspace_bytes(a))
        if st.workspace is None or st.workspace.numel() < need:
            st.workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=self.device)
        a.workspace, a.workspace_bytes = B.ptr(st.workspace), st.workspace.numel()
        return a

    # ------------------------------------------------------------------ passes
    def _check_positions(self, pos, s_max, pos_max=None):
        """Positions must lie inside the rotary (or position) table and the cache; pos_max
        (a host int, when the caller knows it) avoids reading pos back."""
        pmax = pos_max if pos_max is not None else (int(pos.max()) if pos.numel() else 0)
        if pmax >= self.rope_max_pos or pmax >= s_max:
            raise ValueError(f"position {pmax} outside rotary table / cache")

    @staticmethod
    def _check_sequences(cache, n):
        if n > cache.n_seq:
            raise ValueError(f"{n} sequences, the cache has {cache.n_seq}")

    def token_pass(self, ids, pos, seq, cache, cfg, force_layer=None, attn_tiles=True,
                   logit_rows=None, on_layer=None):
        """Run token rows (ids/pos/seq: int32 device tensors [n]) through all layers.  Over a
        paged cache the rows' pages are reserved before (reserve); the K/V of a row without one
        are lost."""
        s = self.shape
        n = int(ids.shape[0])
        paged = isinstance(cache, PagedKVCache)
        slot = cache.slots(pos, seq) if paged else (seq * cache.s_max + pos).to(torch.int32)
        st = self.new_state(n, pos, seq, slot, force_layer)
        if self.gpt2:
            B.embed_positions(n, s.d_model, s.vocab, s.max_pos, ids, pos, self.embed,
                              self.pos_embed, st.h[0])
        else:
            B.embed(n, s.d_model, s.vocab, ids, self.embed, st.h[0])
        B.token_init(n, s.n_layers, s.d_model, st.active[0], st.counts, st.exit_layer, st.inertia)
        args = self.layer_args(st, cache, cfg, attn_tiles)
        for i in range(1, s.n_layers + 1):
            if self.quant is not None:
                B.layer_step_quant(args, self._quant_struct, i, cache.kv if paged else None,
                                   cache.page_table if paged else None, st.cache_slot)
            elif paged:
                B.layer_step_paged(args, cache.kv, cache.page_table, i, st.cache_slot)
            else:
                B.layer_step(args, i)
            if on_layer is not None:
                on_layer(i, st)
        if logit_rows is None:
            return PassResult(None, None, st.exit_layer, st)
        rows = logit_rows.to(torch.int32)
        return PassResult(self._head(st, rows), rows, st.exit_layer, st)

    def _head(self, st, rows):
        """Logits of the listed rows of a pass, from their states at their exits."""
        s, nr = self.shape, int(rows.shape[0])
        count = lambda n: torch.tensor([n], dtype=torch.int32, device=self.device)
        logits = torch.empty((nr, s.vocab), dtype=torch.float32, device=self.device)
        xn = torch.empty((nr, s.d_model), dtype=self.tdt, device=self.device)
        # (the bf16 GEMMs take a vocabulary that is a multiple of 64)
        if self.quant is not None and (nr <= 64 or s.vocab % 64):
            gain, bias = ((self.final_ln_g, self.final_ln_b) if self.gpt2
                          else (self.final_norm, None))
            most = B.quant_linear_max_rows(s.vocab)
            for i in range(0, nr, most):
                m = min(most, nr - i)
                B.final_logits_quant(s.d_model, s.vocab, s.ln_eps if self.gpt2 else s.rms_eps,
                                     st.h[0], st.h[1], st.exit_layer, rows[i:i + m], count(m), m,
                                     gain, bias, self.quant["lm_head"], xn[i:i + m],
                                     logits[i:i + m])
        elif self.gpt2:
            B.final_logits_layernorm(s.d_model, s.vocab, s.ln_eps, st.h[0], st.h[1],
                                     st.exit_layer, rows, count(nr), nr, self.final_ln_g,
                                     self.final_ln_b, self.lm_head, xn, logits)
        else:
            B.final_logits(s.d_model, s.vocab, s.rms_eps, st.h[0], st.h[1], st.exit_layer, rows,
                           count(nr), nr, self.final_norm, self.lm_head, xn, logits)
        return logits

    def prefill(self, ids, cfg, s_max=None, force_layer=None, logits="all", cache=None,
                on_layer=None, start=0):
        """ids: [B, T] (numpy or tensor).  logits: "all", "last" or None.  start: position of
        the first token, after the `start` tokens of each sequence that the (given) cache holds:
        a prompt can be run in pieces."""
        ids = torch.as_tensor(np.asarray(ids) if not isinstance(ids, torch.Tensor) else ids)
        Bn, T = ids.shape
        dev = self.device
        if start < 0 or (start > 0 and cache is None):
            raise ValueError(f"a prompt from position {start} on continues a cache")
        if cache is None:
            cache = self.new_cache(Bn, T if s_max is None else s_max)
        self._check_sequences(cache, Bn)
        pos = torch.arange(start, start + T, dtype=torch.int32, device=dev).repeat(Bn)
        seq = torch.arange(Bn, dtype=torch.int32, device=dev).repeat_interleave(T)
        self._check_positions(pos, cache.s_max, pos_max=start + T - 1)
        if isinstance(cache, PagedKVCache):
            cache.reserve({b: start + T for b in range(Bn)}, start)
        fl = None
        if isinstance(force_layer, torch.Tensor):
            fl = force_layer.reshape(-1).to(dev, torch.int32)
        elif force_layer is not None:
            fl = torch.as_tensor(np.asarray(force_layer).reshape(-1), dtype=torch.int32).to(dev)
        rows = None
        if logits == "all":
            rows = torch.arange(Bn * T, dtype=torch.int32, device=dev)
        elif logits == "last":
            rows = torch.arange(Bn, dtype=torch.int32, device=dev) * T + (T - 1)
        res = self.token_pass(ids.reshape(-1).to(dev, torch.int32), pos, seq, cache, cfg, fl,
                              True, rows, on_layer)
        return res, cache

    def decode_step(self, cache, ids, pos, cfg, force_layer=None, on_layer=None, pos_max=None):
        """One new token per sequence: ids, pos int32 device tensors [n_seq];
        pos_max: the largest position, when known on the host (no read-back;
        over a paged cache every sequence then gets the pages for it)."""
        dev = self.device
        n = int(ids.shape[0])
        seq = torch.arange(n, dtype=torch.int32, device=dev)
        self._check_sequences(cache, n)
        self._check_positions(pos, cache.s_max, pos_max)
        if isinstance(cache, PagedKVCache):
            self._reserve(cache, pos, pos_max, 1)
        rows = torch.arange(n, dtype=torch.int32, device=dev)
        return self.token_pass(ids.to(torch.int32), pos.to(torch.int32), seq, cache, cfg,
                               force_layer, False, rows, on_layer)

    @staticmethod
    def _reserve(cache, pos, pos_max, n):
        """Pages for n new tokens from pos[b] on (at most pos_max, where the host knows no more: it
        reads pos back only if a page might be shared)."""
        if pos_max is None or cache.shared_pages:
            at = {b: int(p) for b, p in enumerate(pos.tolist())}
            top = (lambda p: p) if pos_max is None else (lambda p: max(p, pos_max))
            cache.reserve({b: top(p) + n for b, p in at.items()}, at)
        else:
            cache.reserve({b: pos_max + n for b in range(int(pos.shape[0]))})

    # --------------------------------------------------------------- drafts
    def draw(self, logits, u, temperature=None):
        """A token of each row of logits [n, V] from random numbers u [n] in [0, 1); temperature [n]
        f32 (None: 1; 0: the largest)."""
        return self.verify_logits(logits[:, None], None, torch.empty(
            (logits.shape[0], 0), dtype=torch.int32, device=logits.device), u[:, None],
            temperature)[0][:, 0]

    def verify_logits(self, target, draft, tokens, u, temperature=None, n_draft=None):
        """binding.verify_drafts: (tokens [n, g+1], kept [n])."""
        n, rows, V = target.shape
        i32 = dict(dtype=torch.int32, device=target.device)
        out, kept = torch.empty((n, rows), **i32), torch.empty(n, **i32)
        ws = torch.empty(B.verify_drafts_workspace_bytes(n, rows - 1, V), dtype=torch.uint8,
                         device=target.device)
        B.verify_drafts(target, draft, tokens, u.contiguous(), out, kept, n_draft, temperature, ws)
        return out, kept

    def verify(self, cache, last, drafts, pos, cfg, u, draft_logits=None, temperature=None,
               pos_max=None):
        """One pass over each sequence's last token (at pos[b], not yet in the cache) and its drafts
        [n, g] behind it, and their verification: (tokens [n, g+1], kept [n], pass result).  The
        cache then holds the last token and the drafts; those that were not kept are written
        over by what comes next.  It stands for decode passes: every token decides for itself
        when it exits, also where cfg lets a prompt's last token decide.  draft_logits [n, g, V]
        f32 (None: the drafts have no probabilities); u [n, g+1]; temperature [n]; pos_max: the
        largest pos, when known on the host."""
        n, g = drafts.shape
        self._check_sequences(cache, n)
        top = pos_max if pos_max is not None else (int(pos.max()) if n else 0)
        self._check_positions(pos, cache.s_max, top + g)
        if isinstance(cache, PagedKVCache):
            self._reserve(cache, pos, pos_max, g + 1)
        i32 = dict(dtype=torch.int32, device=self.device)
        ids = torch.cat([last.to(torch.int32)[:, None], drafts.to(torch.int32)], 1)
        at = pos.to(torch.int32)[:, None] + torch.arange(g + 1, **i32)
        seq = torch.arange(n, **i32).repeat_interleave(g + 1)
        rows = torch.arange(n * (g + 1), **i32)
        each = B.ExitCfg(cfg.delta, cfg.min_exit_layer, cfg.n_layers, cfg.metric, 0)
        res = self.token_pass(ids.reshape(-1), at.reshape(-1), seq, cache, each, None, True, rows)
        out, kept = self.verify_logits(res.logits.view(n, g + 1, -1), draft_logits,
                                       drafts.to(torch.int32).contiguous(), u, temperature)
        return out, kept, res

    def generate_drafted(self, ids, n_steps, cfg, draft_cfg, n_draft=4, temperature=0.0,
                         generator=None, cache=None):
        """n_steps tokens of each prompt of ids [B, T], drafted by passes that leave early
        (draft_cfg) and verified n_draft at a time by one pass under cfg, whose distribution the
        tokens have (temperature 0: its largest logits).  generator: of the random numbers, on the
        model's device.  cache: an empty one of either kind with room for T + n_steps + n_draft
        tokens of each sequence.  Returns (tokens [B, n_steps], how many drafts were kept, how many
        were made, cache)."""
        if n_draft < 1 or n_steps < 0:
            raise ValueError(f"{n_steps} tokens, {n_draft} drafts at a time")
        ids_t = torch.as_tensor(np.asarray(ids) if not isinstance(ids, torch.Tensor) else ids)
        n, T = ids_t.shape
        dev = self.device
        i32 = dict(dtype=torch.int32, device=dev)
        end = T + n_steps - 1               # of the last token that is put into the cache
        if cache is None:
            cache = self.new_cache(n, T + n_steps + n_draft)
        self._check_positions(ids_t, cache.s_max, end + n_draft)
        temp = torch.full((n,), float(temperature), dtype=torch.float32, device=dev)
        rand = lambda *d: torch.rand(d, generator=generator, device=dev)
        res, _ = self.prefill(ids_t, cfg, logits="last", cache=cache)
        # the last column takes what a finished sequence still draws, and what was not kept
        out = torch.zeros((n, n_steps + n_draft + 1), **i32)
        out[:, 0] = self.draw(res.logits, rand(n), temp)
        have = torch.ones(n, **i32)         # tokens of each sequence
        kept_all, made, least, most = 0, 0, 1, 1
        i = torch.arange(n_draft + 1, device=dev)
        while least < n_steps:
            pos = T - 1 + have              # of the last token
            last = out.gather(1, have.long()[:, None] - 1)[:, 0]
            tok, drafts, logits = last, [], []
            for k in range(n_draft):
                step = self.decode_step(cache, tok, pos + k, draft_cfg,
                                        pos_max=T - 1 + most + k)
                tok = self.draw(step.logits, rand(n), temp)
                drafts.append(tok)
                logits.append(step.logits)
            toks, kept, _ = self.verify(cache, last, torch.stack(drafts, 1), pos, cfg,
                                        rand(n, n_draft + 1), torch.stack(logits, 1), temp,
                                        pos_max=T - 1 + most)
            at = have[:, None] + i
            out.scatter_(1, torch.where((i <= kept[:, None]) & (at < n_steps), at,
                                        n_steps + n_draft).long(), toks)
            live = have < n_steps
            kept_all += int((kept * live).sum())
            made += n_draft * int(live.sum())
            have = (have + kept + 1).clamp(max=n_steps)
            least, most = int(have.min()), int(have.max())
        return out[:, :n_steps], kept_all, made, cache

    def greedy(self, logits):
        n, V = logits.shape
        out = torch.empty(n, dtype=torch.int32, device=self.device)
        B.argmax(n, V, logits, out)
        return out

    def generate(self, ids, n_steps, cfg, force_layer=None):
        """Prefill then n_steps greedy steps; returns (prefill result, [step results], ids [B, n_steps])."""
        ids_t = torch.as_tensor(np.asarray(ids))
        Bn, T = ids_t.shape
        res, cache = self.prefill(ids_t, cfg, s_max=T + n_steps, force_layer=force_layer,
                                  logits="last")
        nxt = self.greedy(res.logits)
        steps, out = [], []
        for k in range(n_steps):
            out.append(nxt)
            pos = torch.full((Bn,), T + k, dtype=torch.int32, device=self.device)
            st = self.decode_step(cache, nxt, pos, cfg, pos_max=T + k)
            steps.append(st)
            nxt = self.greedy(st.logits)
        gen = torch.stack(out, dim=1) if out else torch.zeros((Bn, 0), dtype=torch.int32)
        return res, steps, gen, cache


@dataclasses.dataclass
class ClassifyOutput:
    logits: torch.Tensor          # [B, n_classes] f32, from each [CLS] row at its exit
    exit_layer: torch.Tensor      # [B*T] int32 (n_layers: never exited)
    cls_exit_layer: torch.Tensor  # [B]
    state: dict                   # device buffers of the pass (h, inertia, sims, ...)


class EncoderModel:
    """A BERT-style post-norm encoder classifier held on the device (bf16),
    run with token-level exit in classification mode:

        adept_encoder_embed -> adept_token_init -> adept_encoder_layer_step(i),
        i = 1..N -> adept_classify_head

    weights: a dict like adept_inputs.encoder_weights() (numpy, per layer) or
    the same keys stacked over layers as torch tensors.
    """

    def __init__(self, shape, weights, device="cuda"):
        self.shape = shape
        self.device = torch.device(device)
        dev, tdt = self.device, torch.bfloat16

        def up(x):
            if isinstance(x, torch.Tensor):
                return x.to(dev, tdt).contiguous()
            return torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(dev).to(tdt)

        L = weights["layers"]
        if isinstance(L, list):
            stack = lambda k: up(np.stack([lw[k] for lw in L]))
            self.w_qkv = up(np.stack([np.concatenate([lw["wq"], lw["wk"], lw["wv"]]) for lw in L]))
            self.b_qkv = up(np.stack([np.concatenate([lw["bq"], lw["bk"], lw["bv"]]) for lw in L]))
        else:
            stack = lambda k: up(L[k])
            self.w_qkv = up(torch.cat([L["wq"], L["wk"], L["wv"]], dim=1))
            self.b_qkv = up(torch.cat([L["bq"], L["bk"], L["bv"]], dim=1))
        self.w_o, self.b_o = stack("wo"), stack("bo")
        self.ln1_g, self.ln1_b = stack("ln1_g"), stack("ln1_b")
        self.w_in, self.b_in = stack("w_in"), stack("b_in")
        self.w_out, self.b_out = stack("w_out"), stack("b_out")
        self.ln2_g, self.ln2_b = stack("ln2_g"), stack("ln2_b")
        self.word = up(weights["word_embed"])
        self.pos_emb = up(weights["pos_embed"])
        self.type_emb = up(weights["type_embed"])
        self.eln_g, self.eln_b = up(weights["embed_ln_g"]), up(weights["embed_ln_b"])
        self.cls_w, self.cls_b = up(weights["cls_w"]), up(weights["cls_b"])

    def classify(self, ids, cfg, force_layer=None, state=None, on_layer=None, stop_at_cls=True):
        """ids [B, T] (numpy or tensor); cfg from binding.exit_cfg.  A state
        dict from an earlier call of the same shape is reused (no allocation).
        on_layer(i, state) is called after each layer step (read-back hook).
        stop_at_cls: a sequence's rows leave when its [CLS] row exits."""
        s, dev = self.shape, self.device
        ids = torch.as_tensor(np.asarray(ids) if not isinstance(ids, torch.Tensor) else ids)
        Bn, T = ids.shape
        n, D, Dq, F, N = Bn * T, s.d_model, s.d_q, s.d_ff, s.n_layers
        i32 = dict(dtype=torch.int32, device=dev)
        bf = dict(dtype=torch.bfloat16, device=dev)
        st = state
        if st is None or st["n"] != n:
            st = {
                "n": n,
                "h": [torch.empty((n, D), **bf) for _ in range(2)],
                "inertia": torch.empty((n, D), dtype=torch.float32, device=dev),
                "pos": torch.arange(T, **i32).repeat(Bn),
                "seq": torch.arange(Bn, **i32).repeat_interleave(T),
                "active": [torch.empty(n, **i32) for _ in range(2)],
                "counts": torch.zeros(4, **i32),
                "exited": torch.empty(n, **i32),
                "exit_layer": torch.empty(n, **i32),
                "exit_flag": torch.empty(max(n, 4), dtype=torch.uint8, device=dev),
                "sim_out": torch.empty(n, dtype=torch.float64, device=dev),
                "key_live": torch.empty(n, dtype=torch.uint8, device=dev),
                "key_len": torch.full((Bn,), T, **i32),
                "k_buf": torch.empty((n, Dq), **bf), "v_buf": torch.empty((n, Dq), **bf),
                "q_buf": torch.empty((n, Dq), **bf), "attn_out": torch.empty((n, Dq), **bf),
                "y_buf": torch.empty((n, D), **bf), "ffn_act": torch.empty((n, F), **bf),
                "logits": torch.empty((Bn, s.n_classes), dtype=torch.float32, device=dev),
                "workspace": None,
            }
        st["force"] = None
        if force_layer is not None:
            st["force"] = torch.as_tensor(np.asarray(force_layer).reshape(-1)
                                          if not isinstance(force_layer, torch.Tensor)
                                          else force_layer.reshape(-1)).to(dev, torch.int32)
        a = B.EncoderArgs()
        a.dtype, a.n_layers, a.d_model, a.n_heads = B.BF16, N, D, s.n_heads
        a.head_dim, a.d_ff, a.ln_eps, a.exit = s.head_dim, F, s.ln_eps, cfg
        for k in ("w_qkv", "b_qkv", "w_o", "b_o", "ln1_g", "ln1_b", "w_in", "b_in", "w_out",
                  "b_out", "ln2_g", "ln2_b"):
            setattr(a, k, B.ptr(getattr(self, k)))
        a.n_tok, a.n_seq, a.seq_len = n, Bn, T
        a.cls_stop = int(bool(stop_at_cls))
        a.h[0], a.h[1] = B.ptr(st["h"][0]), B.ptr(st["h"][1])
        a.inertia, a.pos, a.seq = B.ptr(st["inertia"]), B.ptr(st["pos"]), B.ptr(st["seq"])
        a.active[0], a.active[1] = B.ptr(st["active"][0]), B.ptr(st["active"][1])
        cp = B.ptr(st["counts"])
        a.n_active[0], a.n_active[1], a.n_exited = cp, cp + 4, cp + 8
        a.exited, a.exit_layer = B.ptr(st["exited"]), B.ptr(st["exit_layer"])
        a.exit_flag, a.sim_out = B.ptr(st["exit_flag"]), B.ptr(st["sim_out"])
        a.force_layer = B.ptr(st["force"])
        a.key_live, a.key_len = B.ptr(st["key_live"]), B.ptr(st["key_len"])
        for k in ("k_buf", "v_buf", "q_buf", "attn_out", "y_buf", "ffn_act"):
            setattr(a, k, B.ptr(st[k]))
        need = B.encoder_workspace_bytes(a)
        if st["workspace"] is None or st["workspace"].numel() < need:
            st["workspace"] = torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
        a.workspace, a.workspace_bytes = B.ptr(st["workspace"]), st["workspace"].numel()

        ids_d = ids.reshape(-1).to(dev, torch.int32)
        B.encoder_embed(n, D, s.vocab, s.max_pos, s.ln_eps, ids_d, st["pos"], self.word,
                        self.pos_emb, self.type_emb, self.eln_g, self.eln_b, st["h"][0])
        B.token_init(n, N, D, st["active"][0], st["counts"], st["exit_layer"], st["inertia"])
        st["key_live"].fill_(1)
        for i in range(1, N + 1):
            B.encoder_layer_step(a, i)
            if on_layer is not None:
                on_layer(i, st)
        B.classify_head(Bn, T, D, s.n_classes, st["h"][0], st["h"][1], st["exit_layer"],
                        self.cls_w, self.cls_b, st["logits"])
        return ClassifyOutput(st["logits"], st["exit_layer"], st["exit_layer"][::T], st)
