"""The dense path at the ends of what scales, queries and weights may be."""
import pytest
import torch

from tests import test_gpu_dense as base
from tests.test_gpu_dense import clean_status, fastar  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------- key scales far below and far above the queries
def zero_key_pages(*which):
    def spoil(q, pool, table):
        for b, i in which:
            page = table[b, i].long()
            pool.codes[0][page] = 0
            pool.scale[0][page] = 2.0 ** -126
    return spoil


@pytest.mark.parametrize("tiny", [1e-7, 1e-20, 1e-37])
@pytest.mark.parametrize("n", [1, 5, 140])
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("fp16", 128)])
def test_zero_keys_and_small_queries(fastar, tiny, n, dtype, D):  # noqa: F811
    """Pages of zero keys have the least scale, 2^-126.  With queries that are small too their product leaves fp32, and keys that a row does not see must stay
    out all the same: what is seen has equal weights."""
    if dtype == "fp16" and tiny < 1e-7:
        tiny = 6e-8                                                             # the least number of the type
    base.paged(fastar, dtype, D, 4, 2, [n, n], [500, 37], std=tiny, spoil=zero_key_pages((0, 0), (0, (500 + n - 1) // 64), (1, 0), (1, (37 + n - 1) // 64)))


@pytest.mark.parametrize("past", [3, 6001])                    # an item of a cluster, and cut ones
@pytest.mark.parametrize("n", [1, 140])
def test_all_keys_zero(fastar, past, n):  # noqa: F811
    pages = range(-(-(past + n) // 64))
    base.paged(fastar, "bf16", 128, 2, 1, [n], [past], std=1e-7, spoil=zero_key_pages(*((0, i) for i in pages)))


@pytest.mark.parametrize("n", [1, 5, 140])
def test_large_queries_and_key_scales(fastar, n):  # noqa: F811
    """Zero codes in a page whose scale times the queries' leaves fp32 at the other end: their logits are 0 all the same."""
    def spoil(q, pool, table):
        for i in (0, 2):
            page = table[0, i].long()
            pool.codes[0][page] = 0
            pool.scale[0][page] = 2.0 ** 100
        for i in range(1, -(-(230 + n) // 64)):
            if i != 2:
                pool.scale[0][table[0, i].long()] = 2.0 ** -100                 # logits of up to some 2^12
    base.paged(fastar, "bf16", 128, 4, 2, [n], [230], std=2.0 ** 100, spoil=spoil)


# ------------------------------------------------------------------------------------- calls that follow on one another without a pause
@pytest.mark.parametrize("most", [3, 140])                     # new tokens: cut items of few rows, parts of many
def test_lengths_that_change_from_call_to_call(fastar, most):  # noqa: F811
    """Steps whose tables, attention and join run straight after one another, with lengths and prefix sums written where those of the step before lay: the
    bits of the same calls with the GPU idle in between."""
    g = base.gen(31)
    H, KV, D, PT, B, W, steps = 4, 2, 128, 64, 3, 130, 6
    pool = base.Pool(B * W, KV, PT, D)
    free = torch.randperm(B * W, generator=g, device=base.DEV).to(torch.int32)
    pool.fill(g, torch.arange(B * W, dtype=torch.int32, device=base.DEV).view(1, -1), [B * W * PT])
    adds = [base.i32([(i * 7 + 3 * s * s) % (most + 1) for i in range(B)]) for s in range(steps)]
    T = B * most
    qs = [base.rows(g, H, T, D, torch.bfloat16) for _ in range(steps)]
    held, first = torch.zeros(B, dtype=torch.int32, device=base.DEV), base.i32([0])
    zeros, empty = base.i32([0] * B), torch.full((B, W), -1, dtype=torch.int32, device=base.DEV)

    def run(outs, pause):
        table, h = empty.clone(), held
        f = fastar.block_tables(zeros, h, PT, free, first, table, 3 * 8000)["first"]
        for s in range(steps):
            t = fastar.block_tables(h, adds[s], PT, free, f, table, T)
            pause()
            fastar.kv8_attention(qs[s], *pool.args(), table, t["lens"], t["cu"], most, W * PT, out=outs[s])
            pause()
            h, f = t["lens"], t["first"]

    want, got = ([torch.zeros_like(q) for q in qs] for _ in range(2))
    graph = torch.cuda.CUDAGraph()
    run(got, lambda: None)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        run(got, lambda: None)
    for lens in ([5000, 1, 7000], [64, 6400, 3001], [0, 0, 7300], [7000, 5000, 127]):
        held.copy_(base.i32(lens))
        for o in (*want, *got):
            o.zero_()
        torch.cuda.synchronize()
        run(want, torch.cuda.synchronize)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert torch.equal(a, b)
        assert any(bool(w.any()) for w in want)


@pytest.mark.parametrize("search_bits", [16, 8, 1])
@pytest.mark.parametrize("probe", [False, True])
def test_outputs_straight_into_the_sparse_step(fastar, search_bits, probe):  # noqa: F811
    """What dense attention writes is the very next kernel's input, in a cache's update and in its attention: the bits of the same calls with the GPU idle
    in between."""
    if probe and search_bits == 1:
        pytest.skip("sign bits have no dot products for the probe")
    import numpy as np
    g = base.gen(41)
    H, D, n = 3, 128, 520
    lsh = np.random.default_rng(5).standard_normal((32, D)).astype(np.float32)
    q, k, v = (base.rows(g, H, n, D, torch.bfloat16) for _ in range(3))
    cu, kp = base.i32([0, n]), base.rows(g, H, 48, D, torch.bfloat16)

    def run(pause):
        cache = fastar.Cache(H, D, 4096, 64, lsh, max_tokens=2 * n, max_prompt_tokens=48, max_frames=2, search_bits=search_bits)
        cache.update(k, v, n, 2.0, outputs=False)
        a, b, c = (torch.zeros_like(q) for _ in range(3))
        found = []
        for i in range(6):
            fastar.packed_attention(q, k, v, cu, n, frame_len=1 + i, out=a)
            fastar.packed_attention(k, q, v, cu, n, frame_len=3 + i, out=b)
            fastar.packed_attention(v, k, q, cu, n, frame_len=1 + i, out=c)
            pause()
            found.append(cache.update(c, b, n, 0.9, probe=a if probe else None))
            pause()
            fastar.packed_attention(b, q, v, cu, n, frame_len=2 + i, out=a)
            pause()
            found.append(cache.annsa(a, 64, 5))
            pause()
            fastar.packed_attention(k, b, q, cu, n, frame_len=2 + i, out=a)
            pause()
            found.append(cache.annca(a, kp, kp, n, 8))
            pause()
        torch.cuda.synchronize()
        assert cache.status() == fastar.OK
        return found

    want = run(torch.cuda.synchronize)
    for _ in range(3):
        for x, y in zip(want, run(lambda: None)):
            assert x.keys() == y.keys()
            for name in x:
                assert torch.equal(x[name], y[name]), name


# ------------------------------------------------------------------------------------- tables
def test_tables_without_free_pages(fastar):  # noqa: F811
    """The free list is used up: who needs no page is served, who needs one is refused, and nothing else changes."""
    none = torch.empty(0, dtype=torch.int32, device=base.DEV)
    t = base.i32([[4, 2], [7, -1]])
    got = fastar.block_tables(base.i32([70, 10]), base.i32([3, 54]), 64, none, base.i32([0]), t, 57)
    assert got["lens"].tolist() == [73, 64] and got["cu"].tolist() == [0, 3, 57] and got["first"].tolist() == [0]
    assert got["slots"].tolist() == [2 * 64 + 6 + i for i in range(3)] + [7 * 64 + 10 + i for i in range(54)]
    assert fastar.dense_last_status() == 0
    got = fastar.block_tables(base.i32([70, 10]), base.i32([3, 55]), 64, none, base.i32([0]), t, 58)
    assert got["lens"].tolist() == [73, -1] and got["cu"].tolist() == [0, 3, 58] and got["first"].tolist() == [0]
    assert got["slots"].tolist() == [2 * 64 + 6 + i for i in range(3)] + [-1] * 55
    assert t.tolist() == [[4, 2], [7, -1]]
    assert fastar.dense_last_status() == fastar.ERR_CAPACITY


# ------------------------------------------------------------------------------------- many small weights beside a large one
# One key has a logit some 19.5 to 20.5 binary orders above all others' and a value of zero, so that an output is the sum of thousands of weights of 2^-20.
# A weight may be off by half a step of its type, not more, for the sum to stay within what the test's bound gives it.
ABOVE = 20.5


def sink_queries(g, H, T, D, dt):
    c = ABOVE / (D ** 0.5 * 1.4426950408889634)                # every column of q; the key's are 1
    return ((0.951 + 0.048 * torch.rand(H, T, 1, generator=g, device=base.DEV)) * c).to(dt).expand(H, T, D).contiguous()


@pytest.mark.parametrize("B,n,past,H,KV", [(100, 1, 2000, 8, 8), (60, 4, 2000, 8, 8), (1, 140, 4000, 2, 2)])
@pytest.mark.parametrize("dtype,D", [("fp16", 64), ("bf16", 128), ("fp16", 128)])
def test_paged_small_weights_add_up(fastar, B, n, past, H, KV, dtype, D):  # noqa: F811
    g, dt, PT = base.gen(51), base.TYPES[dtype], 64
    L = past + n
    W = -(-L // PT)
    pool = base.Pool(B * W, KV, PT, D)
    table = torch.randperm(B * W, generator=g, device=base.DEV).to(torch.int32).view(B, W)
    pool.codes[0].zero_()
    pool.codes[1].copy_(torch.randint(0x30, 0x40, pool.codes[1].shape, generator=g, device=base.DEV, dtype=torch.uint8))       # 0.5 to 1.875
    pool.scale[0].fill_(1.0)
    pool.scale[1].fill_(1.0)
    pool.codes[0][table[:, 0].long(), :, 0] = 0x38                             # 1.0
    pool.codes[1][table[:, 0].long(), :, 0] = 0
    q = sink_queries(g, H, B * n, D, dt)
    cu, lens = base.prefix([n] * B), [L] * B
    out = fastar.kv8_attention(q, *pool.args(), table, base.i32(lens), base.i32(cu), n, L)
    G = H // KV
    o, bound = base.R.attention(q, lambda b, h: pool.rows(0, table[b], L, h // G), lambda b, h: pool.rows(1, table[b], L, h // G), cu, lens, 1, dt)
    base.check(out, o, bound, cu)


@pytest.mark.parametrize("dtype,D", [("fp16", 64), ("fp16", 128), ("bf16", 128)])
def test_packed_small_weights_add_up(fastar, dtype, D):  # noqa: F811
    """(A row that sees few keys has an output below 2^-14, whose fp16 numbers are 2^-24 apart, so that rounding it is off by up to 2^-25 and not by u |o| only.)"""
    dt = base.TYPES[dtype]
    for H, KV, n, frame in ((2, 2, 3000, 0), (4, 2, 1500, 1)):
        g = base.gen(1)
        q, k, v = (base.rows(g, heads, n, D, dt) for heads in (H, KV, KV))
        q.copy_(sink_queries(base.gen(52), H, n, D, dt))
        k.zero_()
        k[:, 0] = 1.0
        v.copy_(v.abs() + 0.5)
        v[:, 0] = 0.0
        out = fastar.packed_attention(q, k, v, base.i32([0, n]), n, frame_len=frame)
        o, bound = base.R.attention(q, lambda b, h: k[h // (H // KV)].double(), lambda b, h: v[h // (H // KV)].double(), [0, n], [n], frame, dt)
        base.check(out, o, bound + (2.0 ** -25 if dtype == "fp16" else 0.0), [0, n])


# ------------------------------------------------------------------------------------- strides
@pytest.mark.parametrize("H,KV", [(4, 4), (4, 1), (1, 1)])
def test_one_token_out_of_wider_rows(fastar, H, KV):  # noqa: F811
    """A single token's queries, keys and values as views of one projection's output, into a contiguous output."""
    g, D, dt = base.gen(61), 64, torch.bfloat16
    wide = base.rows(g, 1, 1, (H + 2 * KV) * D, dt).view(1, H + 2 * KV, D).transpose(0, 1)     # [heads][1][D]
    q, k, v = wide[:H], wide[H: H + KV], wide[H + KV:].contiguous()
    out = torch.zeros(H, 1, D, dtype=dt, device=base.DEV)
    got = fastar.packed_attention(q, k, v, base.i32([0, 1]), 1, out=out)
    assert got is out and torch.equal(out, v.repeat_interleave(H // KV, 0))
    pool = base.Pool(1, KV, 64, D)
    table, lens, cu = base.i32([[0]]), base.i32([1]), base.i32([0, 1])
    fastar.kv8_append(k, v, *pool.args(), table, lens, cu)
    want = fastar.kv8_attention(q.contiguous(), *pool.args(), table, lens, cu, 1, 1)
    assert torch.equal(fastar.kv8_attention(q, *pool.args(), table, lens, cu, 1, 1, out=out), want)
    assert torch.equal(want.double(), pool_values(pool)[0, :, :1].repeat_interleave(H // KV, 0))


def pool_values(pool):
    """[pages][heads][rows][D] of the values, in 64 bits (exact in bf16)."""
    return base.R.e4m3_values(base.DEV)[pool.codes[1].long()] * pool.scale[1].double()[:, :, None, None]


# ------------------------------------------------------------------------------------- logits of minus infinity over codes
@pytest.mark.parametrize("past", [20, 6000])
@pytest.mark.parametrize("n", [1, 5, 140])
@pytest.mark.parametrize("dtype,big", [("bf16", 1e6), ("bf16", 3e38), ("fp16", 6e4)])
def test_paged_logits_of_minus_infinity(fastar, n, past, dtype, big):  # noqa: F811
    """A row with -inf against a column of positive keys sees only logits of -inf and gives zeros, whatever finite numbers stand beside it; against keys of both signs,
    or of zero, it gives no number.  Other rows are as they were."""
    g, dt, D, PT, KV, H = base.gen(71), base.TYPES[dtype], 128, 64, 2, 4
    L = past + n
    W = -(-L // PT)
    pool, table = base.Pool(W, KV, PT, D), torch.arange(W, dtype=torch.int32, device=base.DEV).view(1, W)
    pool.fill(g, table, [L])
    pool.codes[0][..., 0] &= 0x7F                                              # the first column is not negative ...
    pool.codes[0][..., 0] |= 0x08                                              # ... nor zero
    pool.codes[0][..., 0][pool.codes[0][..., 0] == 0x7F] = 0x38
    pool.codes[0][..., 1] = 0xB8                                               # and the second is -1
    pool.codes[0][..., 2] = 0x38
    pool.codes[0][:, 0, 0, 2] = 0                                              # but for one key of the first head's
    q = base.rows(g, H, n, D, dt)
    want = fastar.kv8_attention(q, *pool.args(), table, base.i32([L]), base.i32([0, n]), n, L)
    spoilt = q.clone()
    spoilt[0, -1, 0], spoilt[0, -1, 1] = -float("inf"), -big                   # -inf + a finite positive number
    spoilt[1, 0, 2], spoilt[1, 0, 1] = float("inf"), big                       # inf x 0 where its keys have one
    spoilt[3, 0, 0], spoilt[3, 0, 1], spoilt[3, 0, 5] = -float("inf"), -big, big
    out = fastar.kv8_attention(spoilt, *pool.args(), table, base.i32([L]), base.i32([0, n]), n, L)
    assert bool((out[0, -1] == 0).all()) and bool((out[3, 0] == 0).all())
    assert bool(torch.isnan(out[1, 0]).all())
    same = torch.ones(H, n, dtype=torch.bool, device=base.DEV)
    same[0, -1] = same[1, 0] = same[3, 0] = False
    assert torch.isfinite(want).all()
    assert torch.allclose(out[same].float(), want[same].float(), rtol=2.0 ** -7, atol=2.0 ** -7)


# ------------------------------------------------------------------------------------- the first call of a kind in a capture
def test_first_calls_in_a_capture(fastar):  # noqa: F811
    """A process whose first call is one of the tables may capture all others without having made them before."""
    import os
    import subprocess
    import sys
    code = """
import torch
from tests import test_gpu_dense as base
from paper_2602_01801_b200 import fastar
g = base.gen(1)
table = torch.full((2, 130), -1, dtype=torch.int32, device=base.DEV)
free = torch.arange(260, dtype=torch.int32, device=base.DEV)
t = fastar.block_tables(base.i32([0, 0]), base.i32([8000, 300]), 64, free, base.i32([0]), table, 8300)
k = base.rows(g, 2, 8300, 128, torch.bfloat16)
q = base.rows(g, 4, 8300, 128, torch.bfloat16)
few, many = base.i32([0, 1, 3]), base.i32([0, 200, 300])
pool = [base.Pool(260, 2, 64, 128) for _ in range(2)]
def calls(p):
    fastar.kv8_append(k, k, *p.args(), table, t["lens"], t["cu"])
    fastar.kv8_append(k[:, :3], k[:, :3], *p.args(), table, t["lens"], few)
    return [fastar.kv8_attention(q[:, :3].contiguous(), *p.args(), table, t["lens"], few, 2, 8320), fastar.kv8_attention(q[:, :300].contiguous(), *p.args(), table, t["lens"], many, 200, 8320),
            fastar.kv8_attention(q[:, :3].contiguous(), *p.args(), table, base.i32([30, 40]) if p is pool[1] else small, few, 2, 64), fastar.packed_attention(q[:, :300].contiguous(), k[:, :300].contiguous(), k[:, :300].contiguous(), many, 200)]
small = base.i32([30, 40])
graph = torch.cuda.CUDAGraph()
torch.cuda.synchronize()
with torch.cuda.graph(graph):
    got = calls(pool[0])
graph.replay()
want = calls(pool[1])
torch.cuda.synchronize()
for a, b, n in zip(got, want, (3, 300, 3, 300)):
    assert torch.equal(a[:, :n], b[:, :n])
assert fastar.dense_last_status() == 0
print("equal")
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "equal" in r.stdout, r.stderr[-2000:]


# ------------------------------------------------------------------------------------- prefix sums that are wrong in places
@pytest.mark.parametrize("B,n,L", [(5, 3, 9000), (70, 3, 3000), (5, 140, 6000), (3, 700, 3000)])
@pytest.mark.parametrize("wrong", [-1, -2 ** 31, 0, 10 ** 6, 2 ** 31 - 1])
def test_wrong_prefix_sums_reach_their_own_sequences_only(fastar, B, n, L, wrong):  # noqa: F811
    """One entry of cu is out of range, or below the ones before it: the two sequences that it bounds are passed over or get what the entry says (from 0 on: a range
    that other sequences have too is not asked about), all others what they get without it, also where their keys are cut and joined."""
    g = base.gen(81)
    H, KV, D, PT = 4, 2, 64, 64
    W = -(-L // PT)
    pool, table = base.Pool(W, KV, PT, D), torch.arange(W, dtype=torch.int32, device=base.DEV).view(1, W).expand(B, W).contiguous()
    pool.fill(g, table[:1], [L])
    q = base.rows(g, H, B * n, D, torch.bfloat16)
    cu, lens = base.prefix([n] * B), base.i32([L - b for b in range(B)])
    # (not bit for bit: where keys are cut depends on all sequences' lengths)
    o, bound = base.R.attention(q, lambda b, h: pool.rows(0, table[b], L - b, h // 2), lambda b, h: pool.rows(1, table[b], L - b, h // 2), cu, [L - b for b in range(B)], 1, q.dtype)
    for at in sorted({1, 2, B // 2, B - 1}):
        off = list(cu)
        off[at] = wrong
        if off[at] <= off[at + 1] <= B * n and off[at + 1] - off[at] <= n:      # (the entry makes a sequence of its own, over others' rows)
            continue
        out = torch.full_like(q, 2.0)
        fastar.kv8_attention(q, *pool.args(), table, lens, base.i32(off), n, L, out=out)
        assert fastar.dense_last_status() == fastar.ERR_BOUNDS
        for b in range(B):
            rows = slice(n * b, n * b + n)
            if b in (at - 1, at):
                assert bool((out[:, rows] == 2.0).all()), (at, b)
            else:
                assert bool(((out[:, rows].double() - o[:, rows]).abs() <= bound[:, rows]).all()), (at, b)


@pytest.mark.parametrize("past", [0, 20, 6000])
@pytest.mark.parametrize("n", [1, 5, 140])
def test_rows_of_minus_infinity_take_no_values(fastar, n, past):  # noqa: F811
    """A row that sees only logits of -inf gives zeros, also where the values that it sees are no numbers."""
    g, D, PT, KV, H = base.gen(91), 128, 64, 1, 2
    L = past + n
    W = -(-L // PT)
    pool, table = base.Pool(W, KV, PT, D), torch.arange(W, dtype=torch.int32, device=base.DEV).view(1, W)
    pool.fill(g, table, [L])
    pool.codes[0][..., 0] = 0x38                                               # 1
    pool.codes[1][..., 3] = 0x7F
    q = base.rows(g, H, n, D, torch.bfloat16)
    q[0, :, 0] = -float("inf")
    out = fastar.kv8_attention(q, *pool.args(), table, base.i32([L]), base.i32([0, n]), n, L)
    assert bool((out[0] == 0).all()) and bool(torch.isnan(out[1, :, 3]).all()) and bool(torch.isfinite(out[1, :, 4:]).all())
    k, v = base.rows(g, KV, L, D, torch.bfloat16), base.rows(g, KV, L, D, torch.bfloat16)
    k[..., 0], v[..., 3] = 1.0, float("nan")
    q = base.rows(g, H, L, D, torch.bfloat16)
    q[0, :, 0] = -float("inf")
    for frame in (0, 1, 7):
        out = fastar.packed_attention(q, k, v, base.i32([0, L]), L, frame_len=frame)
        assert bool((out[0] == 0).all()) and bool(torch.isnan(out[1, :, 3]).all()) and bool(torch.isfinite(out[1, :, 4:]).all())
