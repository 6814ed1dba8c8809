"""Measured cases of what a serving loop does around a pass: drafted tokens verified against
the model's probabilities, products of few rows with weights in 4 bits, and pages of a K/V cache
copied where sequences fork or the cache is compacted.

Kinds of case (sizes stand for ranges; draw() gives more of each):

  verify   `batch` sequences with up to `drafts` drafted tokens each over `vocab` tokens: how many
           are kept, and the token that follows them, from given random numbers
  linear   `rows` activation rows times a weight matrix [n][k] of e2m1 codes with one power of two
           for every 32 of a row
  pack     a weight matrix brought into that form and read back
  copy     `pages` pages of all `layers` layers of a cache copied to other pages; partial: of each
           only its first tokens

With own = False, run() computes the operators from elementary torch operations (the verification
in 64 bits: a token is the border between two sums); with own = True it makes the framework's
calls.
"""
from __future__ import annotations

import math
import random
import zlib

import torch

own = False

# layers, K/V heads and head width: of the 7B-class decoder and the GPT2-XL-shaped decoder of the
# benchmark, and of the small f32 decoder of the tests
CACHES = {"7b": (32, 32, 128), "gpt2xl": (48, 25, 64), "tiny": (4, 4, 64)}


def listed():
    return [
        # one user's generation, four tokens drafted: latency counts
        {"name": "verify_1x4_32000", "kind": "verify", "batch": 1, "drafts": 4, "vocab": 32000,
         "source": "f32", "draft_logits": True, "ragged": False, "temperature": "one"},
        # the benchmark's serving batch, sampled at each request's temperature
        {"name": "verify_64x8_32000", "kind": "verify", "batch": 64, "drafts": 8, "vocab": 32000,
         "source": "f32", "draft_logits": True, "ragged": False, "temperature": "mixed"},
        # drafts looked up, with no probabilities of their own; an odd vocabulary
        {"name": "verify_24x5_50257_lookup", "kind": "verify", "batch": 24, "drafts": 5,
         "vocab": 50257, "source": "bf16", "draft_logits": False, "ragged": True,
         "temperature": "one"},
        # a decode step's Q, K and V of one token
        {"name": "linear_1_12288x4096", "kind": "linear", "rows": 1, "n": 12288, "k": 4096,
         "out": "bf16"},
        # the down projection of a batch
        {"name": "linear_16_4096x11008", "kind": "linear", "rows": 16, "n": 4096, "k": 11008,
         "out": "bf16"},
        # the head over one sequence's drafts
        {"name": "linear_5_32000x4096", "kind": "linear", "rows": 5, "n": 32000, "k": 4096,
         "out": "f32"},
        # the narrow decoder's second MLP matrix, 24 sequences
        {"name": "linear_24_1600x6400", "kind": "linear", "rows": 24, "n": 1600, "k": 6400,
         "out": "bf16"},
        # the serving batch through the up projection
        {"name": "linear_64_11008x4096", "kind": "linear", "rows": 64, "n": 11008, "k": 4096,
         "out": "bf16"},
        # a matrix of the 7B-class decoder as it is loaded
        {"name": "pack_11008x4096", "kind": "pack", "n": 11008, "k": 4096, "source": "bf16"},
        # one sequence continued twice: what it wrote of its last page
        {"name": "copy_7b_1_partial", "kind": "copy", "cache": "7b", "type": "bf16", "page": 16,
         "pages": 1, "partial": True},
        # a batch of prompts forked, each with an open page, in 8 bits
        {"name": "copy_gpt2xl_fp8_24_partial", "kind": "copy", "cache": "gpt2xl", "type": "fp8",
         "page": 16, "pages": 24, "partial": True},
        # a cache after a peak of load: its last pages moved into the holes
        {"name": "copy_7b_40x32", "kind": "copy", "cache": "7b", "type": "bf16", "page": 32,
         "pages": 40, "partial": False},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["verify", "verify", "verify", "linear", "linear", "linear", "pack", "copy",
                       "copy"])
    if kind == "verify":
        vocab = rng.choice([1024, 32000, 50304, 50257, _log_int(rng, 200, 130000)])
        drafts = rng.choice([0, 1, 2, 3, 4, 5, 8, rng.randint(6, 16)])
        most = max(1, min(128, 64 * 17 * 32000 // ((2 * drafts + 1) * vocab)))
        return {"kind": kind, "batch": _log_int(rng, 1, most), "drafts": drafts, "vocab": vocab,
                "source": rng.choice(["f32", "f32", "bf16"]), "draft_logits": rng.random() < 0.7,
                "ragged": rng.random() < 0.5,
                "temperature": rng.choice(["one", "mixed", "mixed", "greedy"])}
    if kind == "linear":
        n, k = rng.choice([(12288, 4096), (4096, 4096), (11008, 4096), (4096, 11008), (32000, 4096),
                           (4800, 1600), (1600, 6400), (50304, 1600),
                           (_log_int(rng, 64, 12000), 8 * _log_int(rng, 8, 1400))])
        return {"kind": kind, "rows": rng.choice([1, _log_int(rng, 1, 64)]), "n": n, "k": k,
                "out": rng.choice(["bf16", "bf16", "f32"])}
    if kind == "pack":
        return {"kind": kind, "n": _log_int(rng, 64, 11008), "k": 8 * _log_int(rng, 8, 512),
                "source": rng.choice(["bf16", "f32"])}
    cache = rng.choice(["7b", "gpt2xl", "tiny"])
    page = rng.choice([8, 16, 32])
    layers, heads, hd = CACHES[cache]
    most = max(2, min(200, (40 * 32 * 32 * 32 * 128) // (page * layers * heads * hd)))
    return {"kind": kind, "cache": cache, "type": "f32" if cache == "tiny" and rng.random() < 0.5
            else rng.choice(["bf16", "fp8"]), "page": page, "pages": _log_int(rng, 1, most),
            "partial": rng.random() < 0.5}


# --------------------------------------------------------------------------
# inputs, from the seed alone
# --------------------------------------------------------------------------
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.uint8}


def _generator(seed, tag):
    g = torch.Generator(device="cuda")
    g.manual_seed((seed * 1000003 + zlib.crc32(tag.encode())) & 0x7FFFFFFFFFFFFFFF)
    return g


def _randn(seed, tag, *shape):
    return torch.randn(shape, generator=_generator(seed, tag), device="cuda")


def _rand(seed, tag, *shape):
    return torch.rand(shape, generator=_generator(seed, tag), device="cuda")


def _prepare_verify(case, seed):
    n, g, V = case["batch"], case["drafts"], case["vocab"]
    dtype = DTYPES[case["source"]]
    r = random.Random(seed)
    if case["temperature"] == "one":
        temp = [1.0] * n
    elif case["temperature"] == "greedy":
        temp = [0.0] * n
    else:
        temp = [r.choice([0.0, 0.6, 0.8, 1.0, 1.3]) for _ in range(n)]
    # a model's logits: a wide bulk and a few tokens that stand out; a drafter that mostly agrees
    target = _randn(seed, "target", n, g + 1, V).mul_(2.0)
    top = (_rand(seed, "top", n, g + 1, 8) * V).long().clamp_(max=V - 1)
    target.scatter_add_(2, top, 8 + 4 * _rand(seed, "height", n, g + 1, 8))
    draft = target[:, :g] + _randn(seed, "draft", n, g, V).mul_(0.7)
    target, draft = target.to(dtype), draft.to(dtype)
    state = {"case": case, "target": target, "draft": draft if case["draft_logits"] else None,
             "temperature": torch.tensor(temp, dtype=torch.float32, device="cuda"),
             "u": _rand(seed, "u", n, g + 1), "n_draft": None}
    # tokens as the drafter drew them
    warm = state["temperature"].clamp(min=1e-3)[:, None, None]
    noise = -torch.log(-torch.log(_rand(seed, "noise", n, g, V).clamp(1e-7, 1 - 1e-7)))
    noise *= (state["temperature"] > 0)[:, None, None]
    state["tokens"] = (draft.float() / warm + noise).argmax(-1).to(torch.int32)
    if case["ragged"]:
        state["n_draft"] = torch.tensor([r.randint(0, g) for _ in range(n)], dtype=torch.int32,
                                        device="cuda")
    state["out"] = torch.empty((n, g + 1), dtype=torch.int32, device="cuda")
    state["kept"] = torch.empty(n, dtype=torch.int32, device="cuda")
    return state


E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)     # codes 0 .. 7; 8 .. 15 the same, negative


def _power(exponent):
    """2^exponent, exactly, for integers -126 .. 127."""
    return ((exponent.to(torch.int32) + 127) << 23).view(torch.float32)


def _weights(seed, tag, n, k):
    """A trained matrix's values: normal, rows and some columns of other sizes."""
    w = _randn(seed, tag, n, k).mul_(0.02)
    w *= 0.5 + _rand(seed, tag + "_rows", n, 1)
    return w.mul_(1 + 3 * (_rand(seed, tag + "_columns", 1, k) < 0.03))


def _prepare_linear(case, seed):
    m, n, k = case["rows"], case["n"], case["k"]
    codes, scale = _quantise(_weights(seed, "w", n, k))
    x = _randn(seed, "x", m, k).mul_(1 + 5 * (_rand(seed, "wide", 1, k) < 0.01))
    return {"case": case, "codes": codes, "scale": scale, "x": x.to(torch.bfloat16),
            "y": torch.empty((m, n), dtype=DTYPES[case["out"]], device="cuda")}


def _prepare_copy(case, seed):
    layers, heads, hd = CACHES[case["cache"]]
    n, page = case["pages"], case["page"]
    total = 2 * n + 3
    dims = (layers, total * page, heads, hd)
    pool = {}
    for tag in ("k", "v"):
        g = _generator(seed, tag)
        if case["type"] == "fp8":
            # any codes but the two of NaN, any of a cache's scales
            pool[tag] = torch.randint(0, 127, dims, generator=g, device="cuda", dtype=torch.uint8)
            pool[tag + "_scale"] = torch.randint(110, 130, dims[:3], generator=g, device="cuda",
                                                 dtype=torch.uint8)
        else:
            pool[tag] = torch.empty(dims, dtype=DTYPES[case["type"]], device="cuda")
            for i in range(layers):
                pool[tag][i] = torch.randn(dims[1:], generator=g, device="cuda")
    order = torch.randperm(total, generator=_generator(seed, "pages"), device="cuda").to(torch.int32)
    state = {"case": case, "pool": pool, "src": order[:n].contiguous(),
             "dst": order[n:2 * n].contiguous(), "length": None}
    if case["partial"]:
        # the open pages of sequences of any length, at least one token in each
        state["length"] = 1 + (_rand(seed, "length", n) * (page - 1)).to(torch.int32)
    return state


def prepare(case, seed):
    kind = case["kind"]
    if kind == "verify":
        return _prepare_verify(case, seed)
    if kind == "linear":
        return _prepare_linear(case, seed)
    if kind == "copy":
        return _prepare_copy(case, seed)
    w = _weights(seed, "w", case["n"], case["k"]).to(DTYPES[case["source"]])
    return {"case": case, "w": w, "back": torch.empty_like(w)}


# --------------------------------------------------------------------------
# plain forms
# --------------------------------------------------------------------------
def _weights64(logits, temperature):
    """exp((l - max l) / T) and its sum over a row."""
    x = logits.double()
    x = ((x - x.amax(-1, keepdim=True)) / temperature).exp_()
    return x, x.sum(-1, keepdim=True)


def _first_best(logits):
    """The lowest index of each row's largest value."""
    at = torch.arange(logits.shape[-1], device=logits.device)
    return torch.where(logits == logits.amax(-1, keepdim=True), at, len(at)).amin(-1)


def _verify_plain(state):
    target, draft, tokens = state["target"], state["draft"], state["tokens"].long()
    n, rows, V = target.shape
    g = rows - 1
    dev = target.device
    u, temp = state["u"].double(), state["temperature"].double()
    greedy = temp <= 0
    warm = torch.where(greedy, 1.0, temp)[:, None, None]
    count = state["n_draft"]
    count = torch.full((n,), g, device=dev) if count is None else count.long()
    p, total = _weights64(target, warm)
    p /= total
    best = _first_best(target)
    at = tokens[..., None]
    px = p[:, :g].gather(2, at)[..., 0]
    if draft is None:
        q, qx = None, torch.ones_like(px)
    else:
        q, total = _weights64(draft, warm)
        q /= total
        qx = q.gather(2, at)[..., 0]
    kept = torch.where(greedy[:, None], tokens == best[:, :g], u[:, :g] * qx < px)
    kept &= torch.arange(g, device=dev) < count[:, None]
    kept = kept.long().cumprod(1).sum(1)
    # the row that the next token comes from, and what is left of it
    b = torch.arange(n, device=dev)
    row = p[b, kept]
    if g:
        last = kept.clamp(max=g - 1)
        if q is None:
            minus = torch.zeros_like(row).scatter_(1, tokens[b, last][:, None], 2.0)
        else:
            minus = q[b, last]
        rest = (row - minus).clamp_(min=0)
        rest = torch.where(rest.sum(1, keepdim=True) > 0, rest, row)
        row = torch.where((kept < count)[:, None], rest, row)
    sums = row.cumsum(1)
    nxt = (sums <= u[:, g:] * sums[:, -1:]).sum(1)
    nonzero = torch.where(row > 0, torch.arange(V, device=dev), 0).amax(1)
    nxt = torch.where(greedy, best[b, kept], torch.minimum(nxt, nonzero))
    i = torch.arange(rows, device=dev)
    out = torch.cat([tokens, nxt[:, None]], 1)
    out = torch.where(i == kept[:, None], nxt[:, None], out)
    out = torch.where(i <= kept[:, None], out, -1)
    return {"tokens": out.to(torch.int32), "kept": kept.to(torch.int32)}


def _quantise(w):
    """(codes, scale bytes) of w [n][k] in f32: for every 32 of a row the least power of two 2^E with
    which the largest magnitude is at most 7, E in -100 .. 100 and stored as 127 + E; the values
    divided by it, to the nearest e2m1 value (ties to the even code), at most 6."""
    n, k = w.shape
    pad = -k % 32
    x = torch.nn.functional.pad(w.float(), (0, pad)).view(n, -1, 32)
    bits = x.abs().amax(-1).view(torch.int32)
    exponent = (bits >> 23) - 127 - 2 + ((bits & 0x7fffff) > 0x600000).to(torch.int32)
    exponent = exponent.clamp(-100, 100)
    y = (x * _power(-exponent)[..., None]).abs()
    # steps of 1/2 below 2, of 1 below 4, of 2 above
    step = torch.where(y < 2, 0.5, torch.where(y < 4, 1.0, 2.0))
    y = ((y / step).round() * step).clamp(max=6)       # round(): ties to even
    mag = torch.where(y < 2, y * 2, torch.where(y < 4, y + 2, y / 2 + 4)).to(torch.uint8)
    codes = mag | (torch.signbit(x).to(torch.uint8) << 3)
    return codes.view(n, -1)[:, :k], (exponent + 127).to(torch.uint8)


def _values(codes, scale):
    """The f32 values of e2m1 codes [n][k] (one a byte) and their scale bytes [n][ceil(k / 32)]."""
    table = torch.tensor(E2M1, device=codes.device)
    x = table[(codes & 7).int()] * (1 - 2 * (codes >> 3).float())
    s = _power(scale.to(torch.int32) - 127)
    return x * s.repeat_interleave(32, 1)[:, :codes.shape[1]]


def _linear_plain(state):
    w = _values(state["codes"], state["scale"])
    return torch.matmul(state["x"].float(), w.t()).to(state["y"].dtype)


def _pack_plain(state):
    codes, scale = _quantise(state["w"])
    return _values(codes, scale).to(state["w"].dtype)


def _copy_plain(state):
    case, pool = state["case"], state["pool"]
    page = case["page"]
    j = torch.arange(page, device="cuda")
    src = state["src"].long()[:, None] * page + j
    dst = state["dst"].long()[:, None] * page + j
    if state["length"] is not None:
        used = j < state["length"][:, None]
        src, dst = src[used], dst[used]
    src, dst = src.flatten(), dst.flatten()
    for t in pool.values():
        t[:, dst] = t[:, src]
    return pool


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------
def _handle(state):
    """The laid-out weights, descriptor and workspace, which a program keeps beside the data."""
    from paper_2601_03700_amd import binding as B
    if "ready" not in state:
        case = state["case"]
        if case["kind"] == "verify":
            need = B.verify_drafts_workspace_bytes(case["batch"], case["drafts"], case["vocab"])
            state["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda")
        elif case["kind"] == "copy":
            pool = state["pool"]
            first = {tag: t[0] for tag, t in pool.items()}
            state["kv"] = B.paged_kv(first["k"], first["v"], case["page"], first.get("k_scale"),
                                     first.get("v_scale"))
        else:
            state["weights"] = B.quant_weights(case["n"], case["k"], "cuda")
            if case["kind"] == "linear":
                B.quant_pack(_values(state["codes"], state["scale"]), state["weights"])
        state["ready"] = True
    return B


def run(state):
    case = state["case"]
    kind = case["kind"]
    if not own:
        return {"verify": _verify_plain, "linear": _linear_plain, "pack": _pack_plain,
                "copy": _copy_plain}[kind](state)
    B = _handle(state)
    if kind == "verify":
        B.verify_drafts(state["target"], state["draft"], state["tokens"], state["u"], state["out"],
                        state["kept"], n_draft=state["n_draft"], temperature=state["temperature"],
                        workspace=state["workspace"])
        return {"tokens": state["out"], "kept": state["kept"]}
    if kind == "linear":
        B.quant_linear(state["x"], state["weights"], state["y"])
        return state["y"]
    if kind == "pack":
        B.quant_pack(state["w"], state["weights"])
        B.quant_unpack(state["weights"], state["back"])
        return state["back"]
    B.paged_copy(state["kv"], CACHES[case["cache"]][0], state["src"], state["dst"],
                 n_tokens=state["length"])
    return state["pool"]


# --------------------------------------------------------------------------
# the work a pass cannot do without
# --------------------------------------------------------------------------
def work(case):
    kind = case["kind"]
    if kind == "verify":
        n, g, V = case["batch"], case["drafts"], case["vocab"]
        if case["ragged"]:
            g = g / 2       # on average
        rows = n * (g + 1) + (n * g if case["draft_logits"] else 0)
        e = 4 if case["source"] == "f32" else 2
        # a difference, an exponential and a sum for each logit, on the vector units
        return {"bytes": int(rows * V * e + n * (g + 1) * 12), "flops": int(rows * V * 3)}
    if kind in ("linear", "pack"):
        n, k = case["n"], case["k"]
        held = n * -(-k // 2) + n * -(-k // 32)
        if kind == "pack":
            e = 4 if case["source"] == "f32" else 2
            return {"bytes": 2 * n * k * e + held, "flops": 4 * n * k}
        m = case["rows"]
        return {"bytes": held + 2 * m * k + m * n * (4 if case["out"] == "f32" else 2),
                "flops": 2 * m * n * k}
    layers, heads, hd = CACHES[case["cache"]]
    cell = {"f32": 4 * hd, "bf16": 2 * hd, "fp8": hd + 1}[case["type"]] * heads * 2
    tokens = case["pages"] * (case["page"] // 2 if case["partial"] else case["page"])
    return {"bytes": max(1, 2 * tokens * cell * layers), "flops": 0}


# --------------------------------------------------------------------------
# the operators' definitions in 64 bits
# --------------------------------------------------------------------------
def _exact_verify(state):
    """Sequence by sequence, draft by draft."""
    target, draft = state["target"], state["draft"]
    n, rows, V = target.shape
    tokens, u = state["tokens"].tolist(), state["u"].double().tolist()
    temp = state["temperature"].double().tolist()
    count = [rows - 1] * n if state["n_draft"] is None else state["n_draft"].tolist()
    out = torch.full((n, rows), -1, dtype=torch.int32)
    kept = torch.zeros(n, dtype=torch.int32)

    def law(logits, t):
        return torch.softmax(logits.double() / t, 0)

    def largest(logits):
        return int(torch.nonzero(logits == logits.max())[0])

    for b in range(n):
        i, rest = 0, None
        while i < count[b]:
            x = tokens[b][i]
            if temp[b] <= 0:
                if largest(target[b, i]) != x:
                    break
            else:
                p = law(target[b, i], temp[b])
                q = torch.zeros_like(p)
                if draft is None:
                    q[x] = 1.0
                else:
                    q = law(draft[b, i], temp[b])
                if not u[b][i] < float(p[x]) / float(q[x]):
                    rest = torch.relu(p - q)
                    break
            out[b, i] = x
            i += 1
        kept[b] = i
        if temp[b] <= 0:
            out[b, i] = largest(target[b, i])
            continue
        if rest is None or float(rest.sum()) == 0:
            rest = law(target[b, i], temp[b])
        sums = torch.cumsum(rest, 0)
        over = torch.nonzero(sums > u[b][-1] * sums[-1])
        out[b, i] = int(over[0] if len(over) else torch.nonzero(rest)[-1])
    return {"tokens": out.cuda(), "kept": kept.cuda()}


def _exact_values(codes, scale):
    x = torch.tensor([*E2M1, *(-v for v in E2M1)], dtype=torch.float64, device="cuda")[codes.long()]
    group = torch.arange(codes.shape[1], device="cuda") // 32
    return torch.ldexp(x, scale.long()[:, group] - 127)


def _exact_pack(w):
    """Every value against all that its group's power of two offers."""
    n, k = w.shape
    x = w.double()
    grid = torch.tensor(E2M1, dtype=torch.float64, device="cuda")
    out = torch.empty_like(x)
    for i in range(0, k, 32):
        part = x[:, i:i + 32]
        top = part.abs().amax(1)
        e = torch.ceil(torch.log2(top / 7))
        e = torch.where(top > 7 * torch.exp2(e), e + 1, e)           # log2's rounding
        e = torch.where(top <= 7 * torch.exp2(e - 1), e - 1, e).clamp(-100, 100)
        unit = torch.exp2(e)[:, None]
        far = (part.abs()[..., None] / unit[..., None] - grid).abs()
        # the nearest; of two as near the one with the even code
        far += torch.tensor([0.0, 1e-9] * 4, dtype=torch.float64, device="cuda")
        out[:, i:i + 32] = torch.copysign(grid[far.argmin(-1)] * unit, part)
    return out


def exact(case, seed):
    state = prepare(case, seed)
    kind = case["kind"]
    if kind == "verify":
        return _exact_verify(state)
    if kind == "linear":
        out = torch.empty(state["y"].shape, dtype=torch.float64, device="cuda")
        for i in range(0, case["n"], 4096):
            w = _exact_values(state["codes"][i:i + 4096], state["scale"][i:i + 4096])
            out[:, i:i + 4096] = state["x"].double() @ w.T
        return out
    if kind == "pack":
        return _exact_pack(state["w"])
    page, pool = case["page"], state["pool"]
    if case["type"] == "fp8" or sum(t.numel() for t in pool.values()) > 1 << 27:
        return None
    src, dst = state["src"].tolist(), state["dst"].tolist()
    length = [page] * len(src) if state["length"] is None else state["length"].tolist()
    out = {tag: t.double() for tag, t in pool.items()}
    for s, d, m in zip(src, dst, length):
        for tag in pool:
            out[tag][:, d * page:d * page + m] = pool[tag][:, s * page:s * page + m].double()
    return out
