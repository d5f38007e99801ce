"""What the operators of the dense path are measured on: several rollouts (or prompts) served at once.

A program that serves rollouts runs, in the layers and denoising steps that are not sparsified, causal attention over the packed
conditioning tokens of all of them (`packed`), keeps their keys and values in a paged cache of 8-bit codes (`append`), attends to that
cache with one token, a few or a whole chunk of frames per rollout (`attend`), and makes the page tables for it on the GPU (`tables`).

Sizes are those of this repository's workloads: 12 heads of 128 and frames of 1560 tokens, chunks of three frames, 28080 cached keys, the
40-head layer, 8 heads of 64 or 128 and 4k to 64k keys of the length sweep, prompts of 32 to 512 tokens.  Keys and queries follow the cluster
model of `synth.py`: centroid + 0.1 noise, clusters coherent over neighbouring tokens; values are normal.
"""
import math
import random

import torch

own = False

_BASE = dict(op="", dtype="bf16", heads=12, kv_heads=12, dim=128, seqs=1, new_lo=1, new_hi=1, past_lo=0, past_hi=0, frame=1, page=128, lens_seed=1)


def _case(name, op, **kw):
    return dict(_BASE, name=name, op=op, **kw)


def listed():
    return [
        # one prompt of 32 tokens, the tiny step's: latency is everything
        _case("packed_32", "packed", new_lo=32, new_hi=32),
        # sixteen prompts of 1 to 512 tokens, four key heads for twelve query heads, fp16
        _case("packed_prompts", "packed", dtype="fp16", kv_heads=4, dim=64, seqs=16, new_lo=1, new_hi=512),
        # the first chunks of three rollouts of the 12-head layer: three frames of 1560 tokens each, causal by frames
        _case("packed_frames", "packed", seqs=3, new_lo=4680, new_hi=4680, frame=1560),
        # one long context of the length sweep, token-causal, grouped heads
        _case("packed_16384", "packed", heads=8, kv_heads=2, new_lo=16384, new_hi=16384),
        # one token of one rollout behind one frame of cached keys
        _case("attend_token", "attend", past_lo=1560, past_hi=1560),
        # one token each of 32 rollouts of ragged lengths, grouped heads
        _case("attend_ragged", "attend", heads=16, kv_heads=4, seqs=32, past_lo=1, past_hi=16383, page=64),
        # the 40-head layer's 65536 cached keys, eight rollouts, five query heads to a key head, one token each
        _case("attend_65536", "attend", heads=40, kv_heads=8, seqs=8, past_lo=65535, past_hi=65535),
        # a frame of 1560 queries over 28080 cached keys and itself, the 12-head layer's dense step
        _case("attend_frame", "attend", new_lo=1560, new_hi=1560, past_lo=28080, past_hi=28080, frame=1560),
        # one new token each of 32 rollouts goes into the cache
        _case("append_tokens", "append", kv_heads=8, heads=8, seqs=32, past_lo=0, past_hi=4680, page=64),
        # a chunk of three frames of the 12-head layer goes into the cache
        _case("append_chunk", "append", new_lo=4680, new_hi=4680, past_lo=1000, past_hi=1000),
        # a decoding step's tables for eight rollouts
        _case("tables_step", "tables", seqs=8, past_lo=0, past_hi=28080),
        # tables for 1024 requests, prompts and decoding tokens mixed
        _case("tables_1024", "tables", seqs=1024, new_lo=1, new_hi=512, past_lo=0, past_hi=4680, page=64),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))


def draw(rng):
    op = rng.choice(["packed", "packed", "attend", "attend", "attend", "append", "tables"])
    group = rng.choice([1, 1, 2, 3, 4, 5, 8])
    kv = rng.choice([1, 2, 3, 4, 8, 12])
    c = dict(_BASE, op=op, dtype=rng.choice(["bf16", "bf16", "fp16"]), heads=group * kv, kv_heads=kv, dim=rng.choice([64, 128]),
             page=rng.choice([64, 128]), lens_seed=rng.randrange(1 << 30))
    if op == "packed":
        c["seqs"] = _spread(rng, 1, 24)
        c["new_hi"] = _spread(rng, 1, 8192)
        c["new_lo"] = rng.choice([1, c["new_hi"]])
        c["frame"] = rng.choice([1, 1, 0, _spread(rng, 2, 1560)])
    elif op == "attend":
        few = rng.random() < 0.65
        c["seqs"] = _spread(rng, 1, 64 if few else 4)
        c["new_hi"] = rng.choice([1, 1, 1, 2, 4, 7]) if few else _spread(rng, 8, 1560)
        c["new_lo"] = rng.choice([1, c["new_hi"]])
        c["past_hi"] = _spread(rng, 1, 32768)
        c["past_lo"] = rng.choice([0, c["past_hi"]])
        c["frame"] = rng.choice([1, 1, 0, _spread(rng, 2, 1560)])
    elif op == "append":
        c["seqs"] = _spread(rng, 1, 64)
        c["new_hi"] = _spread(rng, 1, 4680)
        c["new_lo"] = rng.choice([1, c["new_hi"]])
        c["past_hi"] = _spread(rng, 1, 4680)
    else:
        c["seqs"] = _spread(rng, 1, 1024)
        c["new_hi"] = _spread(rng, 1, 512)
        c["past_hi"] = _spread(rng, 1, 28080)
    # no drawn case costs more than the largest listed one of its kind: fewer sequences, then shorter ones
    most = {"packed": 0.5e9, "attend": 0.55e9, "append": 7.2e6, "tables": 3e5}[op]
    while _cost(c) > most:
        if c["seqs"] > 1:
            c["seqs"] -= max(1, c["seqs"] // 8)
        else:
            c["new_hi"] = max(1, c["new_hi"] * 7 // 8)
            c["past_hi"] = c["past_hi"] * 7 // 8
            c["new_lo"] = min(c["new_lo"], c["new_hi"])
            c["past_lo"] = min(c["past_lo"], c["past_hi"])
    return c


def _cost(c):
    """What the plain form holds: logits of the padded batch and the padded keys, or the elements."""
    new, total = c["new_hi"], c["new_hi"] + c["past_hi"]
    if c["op"] in ("packed", "attend"):
        return c["seqs"] * (c["heads"] * new * total * (c["dim"] / 128) + c["kv_heads"] * total * 128)
    if c["op"] == "append":
        return c["seqs"] * new * c["kv_heads"] * c["dim"]
    return c["seqs"] * new


def _lengths(c):
    """(new, past) tokens of every sequence, from the case alone."""
    r = random.Random(c["lens_seed"])
    new = [r.randint(c["new_lo"], c["new_hi"]) for _ in range(c["seqs"])]
    past = [r.randint(c["past_lo"], c["past_hi"]) for _ in range(c["seqs"])]
    return new, past


def _dtype(c):
    return torch.float16 if c["dtype"] == "fp16" else torch.bfloat16


def _tokens(gen, heads, n, dim, centroids, noise):
    """[heads][n][dim] rows of the cluster model: runs of eight neighbouring tokens share a cluster."""
    dev = centroids.device
    which = torch.randint(0, centroids.shape[0], (heads, -(-n // 8)), generator=gen, device=dev).repeat_interleave(8, 1)[:, :n]
    return centroids[which] + noise * torch.randn(heads, n, dim, generator=gen, device=dev)


def prepare(case, seed):
    dev = torch.device("cuda", torch.cuda.current_device())
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    new, past = _lengths(case)
    B, T, PT, H, KV, D, dt = case["seqs"], sum(new), case["page"], case["heads"], case["kv_heads"], case["dim"], _dtype(case)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    s = dict(op=case["op"], frame=case["frame"], page=PT, max_new=max(new), max_len=max(n + p for n, p in zip(new, past)), total=T, cu=i32(cu))
    if case["op"] == "tables":
        # pages that the requests hold already come first, those on the free list are in no order
        held = [-(-p // PT) for p in past]
        width = max(-(-(n + p) // PT) for n, p in zip(new, past))
        need = sum(-(-(n + p) // PT) - h for n, p, h in zip(new, past, held))
        pages = torch.randperm(sum(held) + need, generator=gen, device=dev).to(torch.int32)
        at = torch.arange(width, device=dev)[None, :] < i32(held)[:, None]
        table = torch.full((B, width), -1, dtype=torch.int32, device=dev)
        table[at] = pages[: sum(held)]
        # now and then the free list is too short for the last requests
        free = pages[sum(held): sum(held) + max(1, need - seed % 3)].contiguous()
        s.update(held=i32(past), add=i32(new), table=table, free=free if free.numel() else i32([0]), first=i32([0]))
        return s
    centroids = torch.randn(256, D, generator=gen, device=dev)
    if case["op"] != "append":
        s["q"] = _tokens(gen, H, T, D, centroids, 0.1).to(dt)
    if case["op"] in ("packed", "append"):
        s["k"] = _tokens(gen, KV, T, D, centroids, 0.1).to(dt)
        s["v"] = torch.randn(KV, T, D, generator=gen, device=dev).to(dt)
    if case["op"] == "packed":
        return s
    # the paged cache: every sequence's pages lie anywhere in the pool
    total = [n + p for n, p in zip(new, past)]
    pages = [-(-t // PT) for t in total]
    width = max(pages)
    order = torch.randperm(sum(pages), generator=gen, device=dev).to(torch.int32)
    at = torch.arange(width, device=dev)[None, :] < i32(pages)[:, None]
    table = torch.full((B, width), -1, dtype=torch.int32, device=dev)
    table[at] = order
    P = sum(pages)
    s.update(table=table, lens=i32(total))
    for name in ("k", "v"):
        codes, scale = torch.empty(P, KV, PT, D, dtype=torch.uint8, device=dev), torch.empty(P, KV, dtype=torch.float32, device=dev)
        for p0 in range(0, P, 256):
            n = min(256, P - p0)
            x = _tokens(gen, n * KV, PT, D, centroids, 0.1) if name == "k" else torch.randn(n * KV, PT, D, generator=gen, device=dev)
            if case["op"] == "append":       # rows already in the cache are smaller in half of the pages, so that new ones raise their scale
                x = x * torch.randint(0, 2, (n * KV, 1, 1), generator=gen, device=dev).mul(0.9).add(0.1)
            x = x.to(dt).float().view(n, KV, PT, D)
            sc = _scale_of(x.abs().amax((2, 3)))
            codes[p0: p0 + n] = (x / sc[:, :, None, None]).to(torch.float8_e4m3fn).view(torch.uint8)
            scale[p0: p0 + n] = sc
        s[name + "_codes"], s[name + "_scale"] = codes, scale
    return s


def _scale_of(amax):
    """The least power of two by which values up to amax fit e4m3's 448."""
    m, e = torch.frexp(amax)
    e = (e - 9 + (m > 0.875).to(e.dtype)).clamp(min=-126)
    return torch.where(amax > 0, torch.ldexp(torch.ones_like(amax), e), torch.full_like(amax, 2.0 ** -126))


def run(state):
    return _RUN[state["op"]](state)


def _packed(s):
    if own:
        from paper_2602_01801_b200 import fastar
        return fastar.packed_attention(s["q"], s["k"], s["v"], s["cu"], s["max_new"], frame_len=s["frame"])
    q, k, v, cu = s["q"], s["k"].float(), s["v"].float(), s["cu"].long()
    n = cu[1:] - cu[:-1]
    i = torch.arange(s["max_new"], device=q.device)
    at = torch.where(i[None, :] < n[:, None], cu[:-1, None] + i[None, :], 0)                    # [B, n]
    kb, vb = k[:, at].transpose(0, 1), v[:, at].transpose(0, 1)                               # [B, KV, n, D]
    return _attend(q, kb, vb, cu, n, at, n, s["frame"])


def _attend(q, kb, vb, cu, n, at, lens, frame):
    """Attention of packed queries [H][T][D] over keys and values [B][KV][L][D] of the padded batch, in 32 bits; rounded at the end."""
    (H, T, D), (B, KV, L, _) = q.shape, kb.shape
    i, j = torch.arange(at.shape[1], device=q.device), torch.arange(L, device=q.device)
    pos = lens[:, None] - n[:, None] + i[None, :]
    end = lens[:, None].expand_as(pos) if frame == 0 else torch.minimum((pos // frame + 1) * frame, lens[:, None])
    qb = q.float()[:, at].transpose(0, 1).reshape(B, KV, (H // KV) * at.shape[1], D) / math.sqrt(D)
    x = (qb @ kb.transpose(2, 3)).view(B, KV, H // KV, at.shape[1], L)
    x.masked_fill_((j[None, None, :] >= end[:, :, None])[:, None, None], float("-inf"))
    x = (x - x.amax(-1, keepdim=True)).exp_()
    x /= x.sum(-1, keepdim=True)
    live = j[None, :] < lens[:, None]
    o = x.view(B, KV, -1, L) @ torch.where(live[:, None, :, None], vb, 0.0)
    o = o.view(B, H, at.shape[1], D)
    t = torch.arange(T, device=q.device)
    b = torch.searchsorted(cu, t, right=True) - 1
    return o[b, :, t - cu[b]].transpose(0, 1).to(q.dtype).contiguous()


def _kv8(s):
    if own:
        from paper_2602_01801_b200 import fastar
        return fastar.kv8_attention(s["q"], s["k_codes"], s["v_codes"], s["k_scale"], s["v_scale"], s["table"], s["lens"], s["cu"], s["max_new"], s["max_len"],
                                    frame_len=s["frame"])
    cu, lens = s["cu"].long(), s["lens"].long()
    n = cu[1:] - cu[:-1]
    i = torch.arange(s["max_new"], device=cu.device)
    at = torch.where(i[None, :] < n[:, None], cu[:-1, None] + i[None, :], 0)
    pages = s["table"].clamp(min=0).long()

    def rows(codes, scale):
        B, W = pages.shape
        _, KV, PT, D = codes.shape
        x = codes[pages].view(torch.float8_e4m3fn).float() * scale[pages][..., None, None]         # [B, W, KV, PT, D]
        return x.transpose(1, 2).reshape(B, KV, W * PT, D)
    return _attend(s["q"], rows(s["k_codes"], s["k_scale"]), rows(s["v_codes"], s["v_scale"]), cu, n, at, lens, s["frame"])


def _append(s):
    if own:
        from paper_2602_01801_b200 import fastar
        fastar.kv8_append(s["k"], s["v"], s["k_codes"], s["v_codes"], s["k_scale"], s["v_scale"], s["table"], s["lens"], s["cu"])
    else:
        cu, lens, PT = s["cu"].long(), s["lens"].long(), s["page"]
        t = torch.arange(s["total"], device=cu.device)
        b = torch.searchsorted(cu, t, right=True) - 1
        pos = lens[b] - (cu[b + 1] - t)
        page, row = s["table"][b, pos // PT].long(), pos % PT
        for x, codes, scale in ((s["k"], s["k_codes"], s["k_scale"]), (s["v"], s["v_codes"], s["v_scale"])):
            x = x.float().transpose(0, 1)                                                            # [T, KV, D]
            P = scale.shape[0]
            amax = torch.zeros_like(scale).scatter_reduce_(0, page[:, None].expand(-1, x.shape[1]), x.abs().amax(2), "amax")
            touched = torch.zeros(P, dtype=torch.bool, device=x.device).index_fill_(0, page, True)
            fresh = torch.zeros(P, dtype=torch.bool, device=x.device).index_fill_(0, page[row == 0], True)
            was = torch.where(fresh[:, None], torch.zeros_like(scale), scale)
            to = torch.where(touched[:, None], torch.maximum(was, _scale_of(amax)), scale)
            grown = (to > was) & touched[:, None] & ~fresh[:, None]
            which, head = grown.nonzero(as_tuple=True)
            old = codes[which, head].view(torch.float8_e4m3fn).float() * (was / to)[which, head, None, None]
            codes[which, head] = old.to(torch.float8_e4m3fn).view(torch.uint8)
            codes[page, :, row] = (x / to[page][..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
            scale.copy_(to)
    f8 = torch.float8_e4m3fn
    return {"k_codes": s["k_codes"].view(f8), "v_codes": s["v_codes"].view(f8), "k_scale": s["k_scale"], "v_scale": s["v_scale"]}


def _tables(s):
    if own:
        from paper_2602_01801_b200 import fastar
        r = fastar.block_tables(s["held"], s["add"], s["page"], s["free"], s["first"], s["table"], s["total"])
        return {"table": s["table"], "cu": r["cu"], "lens": r["lens"], "slots": r["slots"], "first": r["first"]}
    held, add, PT, table, free = s["held"].long(), s["add"].long(), s["page"], s["table"], s["free"]
    had, now = (held + PT - 1) // PT, (held + add + PT - 1) // PT
    fits = now <= table.shape[1]
    need = torch.where(fits, now - had, 0)
    upto = need.cumsum(0)
    ok = fits & ((need == 0) | (upto <= free.numel() - s["first"].long()))
    w = torch.arange(table.shape[1], device=table.device)
    new = ok[:, None] & (w[None, :] >= had[:, None]) & (w[None, :] < now[:, None])
    index = s["first"].long() + upto[:, None] - need[:, None] + w[None, :] - had[:, None]
    table.copy_(torch.where(new, free[index.clamp(0, free.numel() - 1)], table))
    cu = torch.cat([torch.zeros(1, dtype=torch.long, device=table.device), add.cumsum(0)])
    t = torch.arange(s["total"], device=table.device)
    b = torch.searchsorted(cu, t, right=True) - 1
    pos = held[b] + t - cu[b]
    slots = torch.where(ok[b], table[b, (pos // PT).clamp(max=table.shape[1] - 1)].long() * PT + pos % PT, -1)
    taken = torch.where(ok & (need > 0), upto, 0).amax()
    return {"table": table, "cu": cu.to(torch.int32), "lens": torch.where(ok, held + add, -1).to(torch.int32), "slots": slots, "first": (s["first"] + taken).to(torch.int32)}


_RUN = {"packed": _packed, "attend": _kv8, "append": _append, "tables": _tables}


def work(case):
    """Bytes and operations that the operator cannot do without."""
    new, past = _lengths(case)
    H, KV, D, PT, T = case["heads"], case["kv_heads"], case["dim"], case["page"], sum(new)
    if case["op"] == "tables":
        pages = sum(-(-(n + p) // PT) for n, p in zip(new, past))
        return {"bytes": 8 * case["seqs"] + 4 * case["seqs"] + 4 * (case["seqs"] + 1) + 8 * pages + 8 * T, "flops": 0}
    if case["op"] == "append":
        return {"bytes": 2 * KV * D * T * 3 + 8 * KV * sum(-(-(n + p) // PT) - p // PT for n, p in zip(new, past)), "flops": 0}
    f = case["frame"]
    seen = sum(sum(n + p if f == 0 else min(((p + i) // f + 1) * f, n + p) for i in range(n)) for n, p in zip(new, past))
    kv = sum(2 * KV * D * n * 2 for n in new) if case["op"] == "packed" else sum(2 * KV * (D * (n + p) + 4 * -(-(n + p) // PT)) for n, p in zip(new, past))
    return {"bytes": 2 * H * T * D * 2 + kv, "flops": 4 * H * D * seen}


def exact(case, seed):
    s = prepare(case, seed)
    new, past = _lengths(case)
    H, KV, D, PT, f = case["heads"], case["kv_heads"], case["dim"], case["page"], case["frame"]
    if case["op"] == "tables":
        return None
    if case["op"] == "append":
        out = {}
        for name in ("k", "v"):
            x, sc = s[name].double(), s[name + "_scale"].double()
            val = _e4m3_values(x.device)[s[name + "_codes"].long()]
            t0 = 0
            for b in range(case["seqs"]):
                for p in range(past[b] // PT, -(-(new[b] + past[b]) // PT) if new[b] else 0):
                    page = int(s["table"][b, p])
                    lo, hi = max(past[b], p * PT), min(past[b] + new[b], (p + 1) * PT)
                    rows = x[:, t0 + lo - past[b]: t0 + hi - past[b]]
                    least = torch.exp2(torch.ceil(torch.log2(rows.abs().amax((1, 2)).clamp(min=448 * 2.0 ** -126) / 448)))
                    to = least if lo == p * PT else torch.maximum(least, sc[page])
                    if lo > p * PT:
                        keep = _round_e4m3(val[page] * (sc[page] / to)[:, None, None])
                        val[page] = torch.where((to > sc[page])[:, None, None], keep, val[page])
                    val[page, :, lo - p * PT: hi - p * PT] = _round_e4m3(rows / to[:, None, None])
                    sc[page] = to
                t0 += new[b]
            out[name + "_codes"], out[name + "_scale"] = val, sc
        return out
    q = s["q"].double()
    o = torch.empty_like(q)
    t0 = 0
    for b in range(case["seqs"]):
        n, total = new[b], new[b] + past[b]
        pos = torch.arange(past[b], total, device=q.device)
        end = torch.full_like(pos, total) if f == 0 else ((pos // f + 1) * f).clamp(max=total)
        hide = torch.arange(total, device=q.device)[None, :] >= end[:, None]
        for h in range(KV):
            if case["op"] == "packed":
                k, v = s["k"][h, t0: t0 + n].double(), s["v"][h, t0: t0 + n].double()
            else:
                pages, values = s["table"][b, : -(-total // PT)].long(), _e4m3_values(q.device)
                k, v = ((values[s[m + "_codes"][pages, h].long()] * s[m + "_scale"][pages, h].double()[:, None, None]).reshape(-1, D)[:total] for m in ("k", "v"))
            for g in range(h * (H // KV), (h + 1) * (H // KV)):
                for r in range(0, n, 2048):
                    x = q[g, t0 + r: t0 + min(n, r + 2048)] @ k.T / math.sqrt(D)
                    o[g, t0 + r: t0 + min(n, r + 2048)] = x.masked_fill_(hide[r: r + 2048], float("-inf")).softmax(-1) @ v
        t0 += n
    return o


def _e4m3_values(device):
    """The values of the 256 codes: a sign, four exponent bits with bias 7, three mantissa bits; the last of each sign is no number."""
    c = torch.arange(256, device=device)
    e, m = (c >> 3) & 15, (c & 7).double()
    v = torch.where(e == 0, m * 2.0 ** -9, (8 + m) * torch.exp2(e.double() - 10))
    v = torch.where((c & 127) == 127, torch.full_like(v, float("nan")), v)
    return torch.where(c >= 128, -v, v)


def _round_e4m3(x):
    """The nearest e4m3 value, ties to even."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step
