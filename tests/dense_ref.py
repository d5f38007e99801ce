"""Plain 64-bit forms of the dense path's operators (block tables, 8-bit append, attention), for its tests."""
import math

import torch

MAX_E4M3 = 448.0


def e4m3_values(device="cpu"):
    """Values of the 256 e4m3 codes."""
    c = torch.arange(256, device=device)
    e, m = (c >> 3) & 15, (c & 7).double()
    v = torch.where(e == 0, m * 2.0 ** -9, (1 + m / 8) * torch.exp2(e.double() - 7))
    v[(c & 127) == 127] = float("nan")
    return torch.where(c >= 128, -v, v)


def e4m3_codes(x):
    """Codes of the nearest e4m3 values (ties to even) of 64-bit x, |x| <= 448; what is not finite gives a NaN code, compared by value only."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def scale_of(amax: float) -> float:
    if amax == 0:
        return 2.0 ** -126
    e = math.ceil(math.log2(amax / MAX_E4M3) - 1e-9)
    while amax > MAX_E4M3 * 2.0 ** e:
        e += 1
    while amax <= MAX_E4M3 * 2.0 ** (e - 1):
        e -= 1
    return 2.0 ** max(e, -126)


def append(x, codes, scale, table, lens, cu, values):
    """What kv8_append leaves: (values of the codes [P][KV][PT][D], scales) in 64 bits.  `values`: the code pool's values before."""
    val, sc = values.clone(), scale.double().clone()
    KV, PT = codes.shape[1], codes.shape[2]
    x = x.double()
    for b in range(len(lens)):
        n = int(cu[b + 1] - cu[b])
        if int(lens[b]) < 0 or n == 0:
            continue
        past = int(lens[b]) - n
        for i in range(past // PT, -(-int(lens[b]) // PT)):
            page = int(table[b, i])
            lo, hi = max(past, i * PT), min(int(lens[b]), (i + 1) * PT)
            for h in range(KV):
                rows = x[h, int(cu[b]) + lo - past: int(cu[b]) + hi - past]
                fine = torch.isfinite(rows)
                least = scale_of(float(torch.where(fine, rows, 0.0).abs().max()))
                to = least if lo == i * PT else max(least, float(sc[page, h]))
                if lo > i * PT and to > float(sc[page, h]):
                    val[page, h] = e4m3_codes(val[page, h] * (float(sc[page, h]) / to))
                new = torch.where(fine, e4m3_codes(torch.where(fine, rows, 0.0) / to), float("nan"))
                val[page, h, lo - i * PT: hi - i * PT] = new
                sc[page, h] = to
    return val, sc


def attention(q, keys, values, cu, lens, frame, dtype):
    """(o, bound) in 64 bits for packed queries [H][T][D]; keys(b, kvh), values(b, kvh): the [len][D] rows of a sequence's key head, 64 bits.
    bound: how far an output may be from o.  With u half a step of the type: u |o| from rounding the output; probabilities rounded to the type and summed up
    as rounded change sum p v / sum p by at most u / (1 - u) (sum p |v| + |o|) / sum p; an error e of the logits by 2 e of the same; logits add up 128 products
    in fp32 (some 130 x 2^-24 < 2^-16 of sum |q k|), and the kernel for few rows keeps queries as fp16 relative to their row's largest (2^-24 of it);
    exponentials and sums in fp32 are within 2^-15."""
    H, T, D = q.shape
    u = torch.finfo(dtype).eps / 2
    q = q.double()
    o = torch.full_like(q, float("nan"))
    bound = torch.zeros_like(q)
    for b in range(len(lens)):
        t0, t1, L = int(cu[b]), int(cu[b + 1]), int(lens[b])
        if L < 0 or t1 == t0:
            continue
        pos = torch.arange(L - (t1 - t0), L, device=q.device)
        end = torch.full_like(pos, L) if frame == 0 else ((pos // frame + 1) * frame).clamp(max=L)
        hide = torch.arange(L, device=q.device)[None] >= end[:, None]
        for h in range(H):
            k, v = keys(b, h), values(b, h)
            qq = q[h, t0:t1]
            x = (qq @ k.T / math.sqrt(D)).masked_fill_(hide, float("-inf"))
            p = x.softmax(-1)
            # a key that is not seen has no part in the sum, whatever its value is
            vf = torch.where(torch.isfinite(v), v, 0.0)
            r = p @ vf
            bad = (~torch.isfinite(v)).double()
            touched = (~hide).double() @ bad > 0
            o[h, t0:t1] = torch.where(touched, float("nan"), r)
            mass = p @ vf.abs()
            e = ((qq.abs() @ torch.nan_to_num(k).abs().T).masked_fill(hide, 0).amax(-1) * 2.0 ** -16
                 + qq.abs().amax(-1) * torch.nan_to_num(k).abs().sum(-1).amax() * 2.0 ** -23) / math.sqrt(D)
            bound[h, t0:t1] = u * r.abs() + (1.01 * u + 2 * e[:, None] + 2.0 ** -15) * (mass + r.abs())
    return o, bound
