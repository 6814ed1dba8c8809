"""Plain 64-bit forms of the paged cache's operators, on the CPU, and inputs for them."""
import math

import torch

DEV = "cuda"
TDT = {"f32": torch.float32, "bf16": torch.bfloat16}


def e4m3_values():
    """The value of each of the 256 codes."""
    out = []
    for c in range(256):
        s, e, m = -1.0 if c & 128 else 1.0, (c >> 3) & 15, c & 7
        out.append(math.nan if (e, m) == (15, 7) else
                   s * (m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)))
    return torch.tensor(out, dtype=torch.float64)


def power(e):
    """2^e in 64 bits, exactly, for integers e."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def exponents(x):
    """The least E in -100 .. 100 with max finite |x| <= 448 2^E, per row of the last dimension."""
    x = x.double()
    top = torch.where(torch.isfinite(x), x.abs(), 0.0).amax(-1)
    E = torch.full(top.shape, -100, dtype=torch.int64)
    for e in range(-100, 100):
        E = torch.where(top > 448.0 * 2.0 ** e, e + 1, E)
    return E


def quantised(x):
    """(values of the codes, E) for rows x: the nearest code to x / 2^E, ties to the even code,
    saturated at 448, NaN where x is not finite.  By a search over all 127 magnitudes."""
    E = exponents(x)
    y = (x.double() * power(-E).unsqueeze(-1)).clamp(-448, 448)
    mags = e4m3_values()[:127]
    at = torch.searchsorted(mags, y.abs().nan_to_num()).clamp(1, 126)
    lo, hi = mags[at - 1], mags[at]
    below, above = y.abs() - lo, hi - y.abs()
    up = (above < below) | ((above == below) & (at % 2 == 0))
    val = torch.where(up, hi, lo) * torch.sign(y)
    return torch.where(torch.isfinite(x.double()), val, math.nan), E


def cache_values(codes, scale_bytes):
    """f64 values of an 8-bit cache."""
    return e4m3_values()[codes.long()] * power(scale_bytes.long() - 127).unsqueeze(-1)


def attend(q, k, v, table, page, pos, seq, scale, causal=True, key_len=None, live=None):
    """For entries q [n, H, hd] at pos, seq [n], and k, v [n_slots, Hkv, hd], in 64 bits: the
    result, and for the tolerances the sums of |weight v| and, over the seen keys, the largest
    sum of |q k| scale.  On the tensors' device; an entry at a time."""
    n, H, hd = q.shape
    G, n_pages = H // k.shape[1], k.shape[0] // page
    f64 = dict(dtype=torch.float64, device=q.device)
    out = torch.zeros((n, H, hd), **f64)
    wv, qk = torch.zeros_like(out), torch.zeros((n, H, 1), **f64)
    pos, seq = pos.tolist(), seq.tolist()
    lens = None if key_len is None else key_len.tolist()
    for i in range(n):
        b = seq[i]
        if not 0 <= b < table.shape[0]:
            continue
        lim = table.shape[1] * page
        if causal:
            lim = min(lim, pos[i] + 1)
        if lens is not None:
            lim = min(lim, lens[b])
        t = torch.arange(max(lim, 0), device=q.device)
        pages = table[b].long()[t // page]
        slot = pages * page + t % page
        slot = slot[(pages >= 0) & (pages < n_pages)]
        if live is not None:
            slot = slot[live[slot] != 0]
        if not len(slot):
            continue
        kk = k[slot].double().permute(1, 2, 0).contiguous()       # [Hkv, hd, t]
        vv = v[slot].double().permute(1, 0, 2).contiguous()       # [Hkv, t, hd]
        x = q[i].double().view(-1, G, hd)
        w = torch.softmax(torch.matmul(x, kk) * scale, -1)
        out[i] = torch.matmul(w, vv).view(H, hd)
        wv[i] = torch.matmul(w, vv.abs()).view(H, hd)
        qk[i] = (torch.matmul(x.abs(), kk.abs()) * scale).amax(-1).view(H, 1)
    return out, wv, qk


def bound(dtype, ref, wv, qk):
    """How far a result may be off.  A score: hd products and sums in f32 and its two factors,
    each off by at most 2^-24 of sum |q k| scale; exp2 by 2^-22 of its value; so a weight by the
    share d = (hd + 4) 2^-24 qk + 2^-22.  The sums over up to some 10^4 keys run in partial sums
    of a tile and over the tiles, below 2^10 additions in a row: 2^-14 in all is generous.
    Numerator and normaliser: 2 (d + 2^-14) wv.  bf16 rounds by up to 2^-8: the weights in the
    numerator (wv) and in the normaliser (|out|), and the result (|out|)."""
    hd = ref.shape[-1]
    d = (hd + 4) * 2.0 ** -24 * qk + 2.0 ** -22 + 2.0 ** -14
    tol = 2 * d * wv + 2.0 ** -24 * ref.abs()
    if dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * (wv + 2 * ref.abs())
    return tol + 1e-30
