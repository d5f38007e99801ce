"""The dense path on the GPU against plain 64-bit forms: page tables, the way into the 8-bit pages, attention over them, packed attention."""
import pytest
import torch

from tests import dense_ref as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


@pytest.fixture(scope="module")
def fastar():
    from paper_2602_01801_b200 import fastar
    fastar.dense_last_status()
    return fastar


@pytest.fixture(autouse=True)
def clean_status(fastar):
    yield
    assert fastar.dense_last_status() == 0


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def prefix(ns, start=0):
    cu = [start]
    for n in ns:
        cu.append(cu[-1] + n)
    return cu


def rows(g, heads, n, d, dtype, layout="htd", std=1.0):
    """[heads][n][d] rows: contiguous, token-major, or part of wider rows."""
    x = torch.randn(heads, n, d, generator=g, device=DEV) * std
    x = x.to(dtype)
    if layout == "thd":
        return x.transpose(0, 1).contiguous().transpose(0, 1)
    if layout == "slice":
        wide = torch.full((heads, n, d + 24), float("nan"), device=DEV, dtype=dtype)
        wide[:, :, 8: 8 + d] = x
        return wide[:, :, 8: 8 + d]
    return x


def check(out, o, bound, cu, keep=None):
    """Every row of a sequence within its bound (no number where the reference has none); rows of none as they were (`keep`)."""
    live = torch.zeros(out.shape[1], dtype=torch.bool, device=out.device)
    live[cu[0]: cu[-1]] = True
    if keep is not None:
        assert torch.equal(out[:, ~live].view(torch.int16), keep[:, ~live].view(torch.int16))
    x = out[:, live].double()
    o, bound = o[:, live], bound[:, live]
    nan = torch.isnan(o)
    assert not torch.isfinite(x[nan]).any()
    far = ((x - o).abs() - bound)[~nan]
    assert torch.isfinite(x[~nan]).all()
    if far.numel():
        assert float(far.max()) <= 0, (float(far.max()), float((x - o)[~nan].abs().max()))


# ---------------------------------------------------------------------------------------------------- packed attention
def packed(fastar, dtype, D, H, KV, ns, frame, layout="htd", behind=0, start=0, std=1.0, seed=1, spoil=None, max_tokens=None):
    g = gen(seed)
    dt = TYPES[dtype]
    cu = prefix(ns, start)
    T = cu[-1] + behind
    q, k, v = rows(g, H, T, D, dt, layout, std), rows(g, KV, T, D, dt, layout, std), rows(g, KV, T, D, dt, layout)
    if spoil is not None:
        spoil(q, k, v, cu)
    out = torch.empty_strided(q.shape, q.stride(), dtype=dt, device=DEV)
    out.copy_(torch.randn(out.shape, generator=g, device=DEV))
    keep = out.clone()
    fastar.packed_attention(q, k, v, i32(cu), max_tokens or max(1, max(ns)), frame_len=frame, out=out)
    G = H // KV
    o, bound = R.attention(q, lambda b, h: k[h // G, cu[b]: cu[b + 1]].double(), lambda b, h: v[h // G, cu[b]: cu[b + 1]].double(), cu, ns, frame, dt)
    check(out, o, bound, cu, keep)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,KV", [(1, 1), (4, 4), (6, 2), (5, 1), (8, 1)])
@pytest.mark.parametrize("frame", [0, 1, 37])
def test_packed_ragged(fastar, dtype, D, H, KV, frame):
    packed(fastar, dtype, D, H, KV, [1, 37, 0, 128, 129, 2, 255, 513], frame)


@pytest.mark.parametrize("ns", [[1], [2], [31], [63], [64], [65], [127], [128], [256], [257], [383], [640], [1, 1, 1, 1], [0, 5, 0, 0, 7, 0]])
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("fp16", 64)])
def test_packed_lengths(fastar, ns, dtype, D):
    packed(fastar, dtype, D, 4, 2, ns, 1)


@pytest.mark.parametrize("layout", ["thd", "slice"])
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("fp16", 128)])
def test_packed_strides_and_rows_of_no_sequence(fastar, layout, dtype, D):
    packed(fastar, dtype, D, 6, 3, [100, 3, 260], 1, layout=layout, behind=29, start=13)


@pytest.mark.parametrize("std", [1e-3, 4.0, 12.0])
def test_packed_flat_and_peaked_rows(fastar, std):
    packed(fastar, "bf16", 128, 2, 1, [700, 90], 1, std=std)
    packed(fastar, "fp16", 64, 2, 1, [700, 90], 0, std=std)


def test_packed_rising_logits(fastar):
    # keys grow with their position: every tile raises the running maximum
    def spoil(q, k, v, cu):
        ramp = torch.linspace(0.1, 20, k.shape[1], device=DEV)[None, :, None]
        k.copy_((k.float().abs() * ramp).to(k.dtype))
        q.copy_(q.abs())
    packed(fastar, "bf16", 128, 2, 1, [1500], 1, spoil=spoil)
    packed(fastar, "bf16", 64, 2, 2, [1100], 0, spoil=spoil)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("fp16", 64)])
@pytest.mark.parametrize("H,KV", [(2, 2), (6, 2)])
def test_packed_values_that_are_not_seen_have_no_influence(fastar, bad, dtype, D, H, KV):
    # rows between and behind the sequences, and tokens that earlier rows of the same sequence must not see
    def spoil(q, k, v, cu):
        k[:, cu[-1]:], v[:, cu[-1]:], q[:, cu[-1]:] = bad, bad, bad
        v[:, cu[1] + 70, 3] = bad            # inside the second sequence
        k[:, cu[2] - 1] = bad                # its last token's key
        v[:, cu[3] - 40:cu[3]] = bad         # the end of the third
    packed(fastar, dtype, D, H, KV, [50, 200, 300, 5], 1, behind=140, spoil=spoil)
    packed(fastar, dtype, D, H, KV, [50, 200, 300, 5], 48, behind=3, spoil=spoil)


def test_packed_logits_of_minus_infinity(fastar):
    # keys whose logits are -inf weigh nothing; a row that sees no others gives zeros
    g = gen(3)
    q, k, v = (rows(g, 1, 200, 64, torch.bfloat16) for _ in range(3))
    q[:, :, 0] = 1.0
    k[:, 7, 0] = float("-inf")
    k[:, 0, 0] = float("-inf")
    out = fastar.packed_attention(q, k, v, i32([0, 200]), 200)
    x = (q.double() @ k.double().transpose(1, 2) / 8).masked_fill(torch.ones(200, 200, device=DEV).triu(1).bool(), float("-inf"))
    o = x[:, 1:].softmax(-1) @ v.double()
    assert torch.equal(out[:, 0], torch.zeros_like(out[:, 0]))
    assert float((out[:, 1:].double() - o).abs().max()) <= 3 * 2.0 ** -8 * float(v.abs().max())


def test_packed_long_frames(fastar):
    packed(fastar, "bf16", 128, 2, 1, [3120, 1000], 1560)


def test_packed_results_repeat_bit_for_bit(fastar):
    g = gen(5)
    q, k, v = rows(g, 4, 900, 128, torch.bfloat16), rows(g, 2, 900, 128, torch.bfloat16), rows(g, 2, 900, 128, torch.bfloat16)
    cu = i32([0, 333, 900])
    a = fastar.packed_attention(q, k, v, cu, 567)
    for _ in range(3):
        assert torch.equal(a, fastar.packed_attention(q, k, v, cu, 567))


# ---------------------------------------------------------------------------------------------------- 8-bit cache
class Pool:
    """Pools of `pages` pages, all bytes (NaN codes among them) and scales garbage until something is written."""

    def __init__(self, pages, KV, PT, D, seed=0):
        g = gen(1000 + seed)
        self.codes = [torch.randint(0, 256, (pages, KV, PT, D), generator=g, device=DEV, dtype=torch.uint8) for _ in range(2)]
        self.scale = [torch.full((pages, KV), float("nan"), device=DEV) for _ in range(2)]
        self.PT, self.D, self.KV, self.pages = PT, D, KV, pages

    def args(self):
        return (*self.codes, *self.scale)

    def rows(self, which, table_row, length, kvh):
        n = -(-length // self.PT)
        pages = table_row[:n].long()
        v = R.e4m3_values(DEV)[self.codes[which][pages, kvh].long()] * self.scale[which][pages, kvh].double()[:, None, None]
        return v.reshape(-1, self.D)[:length]

    def fill(self, g, table, lens, stds=(1.0, 1.0), flip=True):
        """Rows [0, lens) of every sequence: scales differ from page to page by up to 2^6."""
        for b, n in enumerate(lens):
            for i in range(-(-n // self.PT)):
                p = int(table[b, i])
                m = min(self.PT, n - i * self.PT)
                for w in range(2):
                    x = torch.randn(self.KV, m, self.D, generator=g, device=DEV).double()
                    s = 2.0 ** -7 * (2.0 ** int(torch.randint(-3, 4, (1,), generator=g, device=DEV)) if flip else 1.0)
                    val = R.e4m3_codes((x * stds[w] / s).clamp(-448, 448))
                    self.codes[w][p, :, :m] = val.to(torch.float8_e4m3fn).view(torch.uint8)
                    self.scale[w][p] = s


def paged(fastar, dtype, D, H, KV, ns, past, PT=64, frame=1, layout="htd", behind=0, start=0, std=1.0, seed=1, max_len=None, spoil=None, extra_width=2):
    g = gen(seed)
    dt = TYPES[dtype]
    cu, lens = prefix(ns, start), [n + p for n, p in zip(ns, past)]
    W = max(1, max(-(-n // PT) for n in lens)) + extra_width
    need = sum(-(-n // PT) for n in lens)
    order = torch.randperm(need + 3, generator=g, device=DEV)[:need].to(torch.int32)
    table, at = torch.full((len(ns), W), -7, dtype=torch.int32, device=DEV), 0
    for b, n in enumerate(lens):
        m = -(-n // PT)
        table[b, :m] = order[at: at + m]
        at += m
    pool = Pool(need + 3, KV, PT, D, seed)
    pool.fill(g, table, lens)
    q = rows(g, H, cu[-1] + behind, D, dt, layout, std)
    if spoil is not None:
        spoil(q, pool, table)
    out = torch.empty_strided(q.shape, q.stride(), dtype=dt, device=DEV)
    out.copy_(torch.randn(out.shape, generator=g, device=DEV))
    keep = out.clone()
    fastar.kv8_attention(q, *pool.args(), table, i32(lens), i32(cu), max(1, max(ns)), max_len or max(lens), frame_len=frame, out=out)
    G = H // KV
    o, bound = R.attention(q, lambda b, h: pool.rows(0, table[b], lens[b], h // G), lambda b, h: pool.rows(1, table[b], lens[b], h // G), cu, lens, frame, dt)
    check(out, o, bound, cu, keep)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("PT", [64, 128])
@pytest.mark.parametrize("H,KV", [(1, 1), (4, 4), (6, 2), (5, 1), (16, 1), (34, 2)])
def test_paged_single_tokens(fastar, dtype, D, PT, H, KV):
    paged(fastar, dtype, D, H, KV, [1] * 9, [0, 1, 30, 31, 63, 64, 127, 200, 1000], PT)


@pytest.mark.parametrize("dtype,D,PT", [("bf16", 128, 64), ("bf16", 64, 128), ("fp16", 128, 128), ("fp16", 64, 64)])
@pytest.mark.parametrize("ns", [[2, 3, 1, 4], [7, 7, 7, 7], [16, 1, 0, 20], [33, 1, 64, 5], [1, 130, 300, 2]])
@pytest.mark.parametrize("H,KV", [(2, 2), (6, 2), (8, 1)])
@pytest.mark.parametrize("frame", [0, 1, 24])
def test_paged_several_tokens(fastar, dtype, D, PT, ns, H, KV, frame):
    paged(fastar, dtype, D, H, KV, ns, [0, 100, 700, 63], PT, frame)


@pytest.mark.parametrize("past", [0, 1, 5, 31, 32, 33, 95, 127, 128, 129, 255, 511, 512, 513, 2047, 4095, 4100, 9001])
@pytest.mark.parametrize("D", [64, 128])
def test_paged_lengths(fastar, past, D):
    paged(fastar, "bf16", D, 4, 2, [1], [past], 64 if past % 2 else 128)


@pytest.mark.parametrize("layout", ["thd", "slice"])
@pytest.mark.parametrize("ns", [[1, 1, 1], [100, 1, 260]])
def test_paged_strides_and_rows_of_no_sequence(fastar, layout, ns):
    paged(fastar, "bf16", 128, 6, 3, ns, [300, 5, 64], layout=layout, behind=17, start=5)
    paged(fastar, "fp16", 64, 6, 3, ns, [300, 5, 64], layout=layout, behind=17, start=5)


@pytest.mark.parametrize("std", [1e-3, 3.0, 10.0])
@pytest.mark.parametrize("n", [1, 6, 150])
def test_paged_flat_and_peaked_rows(fastar, std, n):
    paged(fastar, "bf16", 128, 4, 2, [n, n], [2500, 90], std=std)
    paged(fastar, "fp16", 64, 4, 2, [n, n], [2500, 90], std=std)


@pytest.mark.parametrize("D,H,KV", [(64, 2, 1), (128, 3, 3)])
def test_paged_many_sequences(fastar, D, H, KV):
    # more sequences than a CTA has threads; some without new tokens; of few rows, and with one of many among them
    g = gen(21)
    past = torch.randint(0, 700, (290,), generator=g, device=DEV).tolist()
    past[17], past[200] = 5000, 9000
    ns = [0 if b % 11 == 3 else 1 + (b % 5 == 2) for b in range(290)]
    paged(fastar, "bf16", D, H, KV, ns, past)
    ns[130] = 90
    paged(fastar, "bf16", D, H, KV, ns, past)


def test_packed_many_sequences(fastar):
    packed(fastar, "bf16", 64, 2, 1, [(7 * b) % 6 for b in range(700)] + [300], 1)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,KV", [(64, 1), (130, 1), (96, 2)])
def test_paged_wide_groups(fastar, D, H, KV):
    # more query heads to a key head than the kernel for few rows has rows, and than a query tile has
    paged(fastar, "bf16", D, H, KV, [1, 3, 1], [500, 40, 2000], 64)


def test_packed_wide_groups(fastar):
    packed(fastar, "bf16", 128, 130, 1, [5, 1, 40], 1)
    packed(fastar, "fp16", 64, 96, 2, [5, 1, 40], 3)


@pytest.mark.parametrize("D", [64, 128])
def test_queries_that_are_no_numbers_stay_by_themselves(fastar, D):
    def bad_rows(q, *_):
        q[0, 3], q[1, 5, 7], q[1, 60] = float("nan"), float("nan"), float("nan")
    packed(fastar, "bf16", D, 2, 1, [70, 40], 1, spoil=lambda q, k, v, cu: bad_rows(q))
    packed(fastar, "fp16", D, 2, 2, [70, 40], 0, spoil=lambda q, k, v, cu: bad_rows(q))
    paged(fastar, "bf16", D, 2, 1, [70, 40], [300, 0], spoil=bad_rows)
    paged(fastar, "fp16", D, 2, 1, [7, 7], [300, 6000], spoil=lambda q, *_: q[0, 3].fill_(float("nan")))


def test_nothing_to_do(fastar):
    q = torch.zeros(4, 0, 64, dtype=torch.bfloat16, device=DEV)
    pool = Pool(2, 2, 64, 64)
    assert fastar.packed_attention(q, q[:2], q[:2], i32([0, 0]), 1).shape == (4, 0, 64)
    fastar.kv8_append(q[:2], q[:2], *pool.args(), i32([[0]]), i32([5]), i32([0, 0]))
    assert fastar.kv8_attention(q, *pool.args(), i32([[0]]), i32([5]), i32([0, 0]), 1, 64).shape == (4, 0, 64)
    t = fastar.block_tables(i32([5, 0]), i32([0, 0]), 64, i32([1]), i32([0]), i32([[0], [1]]), 0)
    assert t["cu"].tolist() == [0, 0, 0] and t["lens"].tolist() == [5, 0] and t["slots"].numel() == 0 and t["first"].tolist() == [0]
    # sequences without new tokens beside one that has some
    q = rows(gen(1), 4, 3, 64, torch.bfloat16)
    out = torch.full_like(q, 2.0)
    pool.fill(gen(2), i32([[0], [1]]), [64, 64])
    fastar.kv8_attention(q, *pool.args(), i32([[0], [1]]), i32([60, 64]), i32([0, 0, 0]), 1, 64, out=out)
    assert bool((out == 2.0).all())


@pytest.mark.parametrize("n", [1, 4, 200])
def test_paged_few_keys_in_a_large_bound(fastar, n):
    # the launch is sized for far more keys than there are
    paged(fastar, "bf16", 128, 4, 2, [n, n, n], [0, 3, 1300], extra_width=300, max_len=20000 - 800)


@pytest.mark.parametrize("past", [300, 6000])                  # of one cluster's or item's keys, and cut into parts
@pytest.mark.parametrize("n", [1, 5, 20, 140])
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("fp16", 64)])
def test_paged_codes_that_are_not_seen_have_no_influence(fastar, n, dtype, D, past):
    # NaN codes behind a row's own position (rows of the same call) reach only the rows that see them; bytes behind the end reach none
    def spoil(q, pool, table):
        last = past + n - 1
        page = int(table[1, last // 64])
        pool.codes[0][page, :, last % 64, 5] = 0x7F
        pool.codes[1][page, :, last % 64, 7] = 0xFF
    paged(fastar, dtype, D, 4, 2, [n, n, n], [70, past, 2], spoil=spoil)


@pytest.mark.parametrize("n", [1, 140])
def test_paged_scales_far_apart(fastar, n):
    # pages whose values are 2^40 times those of others, and pages of zeros: what the softmax picks out keeps its precision
    def spoil(q, pool, table):
        pool.scale[1][table[0, 0].long()] *= 2.0 ** 40
        pool.scale[1][table[0, 2].long()] *= 2.0 ** -30
        pool.codes[1][table[0, 1].long()] = 0
        pool.scale[1][table[0, 1].long()] = 2.0 ** -126
        pool.scale[0][table[0, 0].long()] *= 2.0 ** -60       # nearly equal weights for the first page's keys
    paged(fastar, "bf16", 128, 4, 2, [n], [500], spoil=spoil)


@pytest.mark.parametrize("n", [1, 140])
@pytest.mark.parametrize("down", [-14, -17, -18, -19])
def test_paged_scales_some_way_apart(fastar, n, down):
    # a page whose values are up to 2^18 below the others', and further; the first queries see almost only that page
    def spoil(q, pool, table):
        q[:, : q.shape[1] // 2] = q[:, : q.shape[1] // 2].abs()
        page = table[0, 2].long()
        pool.codes[0][page] = pool.codes[0][page] & 0x7F
        for p in (0, 1, 3):
            pool.scale[1][table[0, p].long()] = 2.0 ** -6
        pool.scale[1][page] = 2.0 ** (-6 + down)
    paged(fastar, "bf16", 128, 2, 2, [n], [230], spoil=spoil, std=3.0)


@pytest.mark.parametrize("n", [1, 3, 300])
def test_paged_results_repeat_bit_for_bit(fastar, n):
    g = gen(9)
    pool = Pool(80, 2, 64, 128)
    table = torch.randperm(80, generator=g, device=DEV).to(torch.int32).view(2, 40)
    pool.fill(g, table, [2500, 700])
    q = rows(g, 4, 2 * n, 128, torch.bfloat16)
    call = lambda: fastar.kv8_attention(q, *pool.args(), table, i32([2500, 700]), i32([0, n, 2 * n]), n, 2500)  # noqa: E731
    a = call()
    for _ in range(3):
        assert torch.equal(a, call())


def test_paged_offsets_past_32_bits(fastar):
    # pools of over 2^31 bytes: the pages in use lie at their end
    KV, PT, D = 8, 128, 128
    pages = (1 << 31) // (KV * PT * D) + 40
    codes = [torch.empty(pages, KV, PT, D, dtype=torch.uint8, device=DEV) for _ in range(2)]
    scale = [torch.full((pages, KV), 1.0, device=DEV) for _ in range(2)]
    g = gen(4)
    table = (pages - 1 - torch.arange(5, device=DEV, dtype=torch.int32))[None].contiguous()
    k, v = rows(g, KV, 600, D, torch.bfloat16), rows(g, KV, 600, D, torch.bfloat16)
    fastar.kv8_append(k, v, *codes, *scale, table, i32([600]), i32([0, 600]))
    small = Pool(5, KV, PT, D)
    near = torch.arange(5, device=DEV, dtype=torch.int32)[None].contiguous()
    fastar.kv8_append(k, v, *small.args(), near, i32([600]), i32([0, 600]))
    q = rows(g, 16, 601, D, torch.bfloat16)
    for n in (1, 600):
        a = fastar.kv8_attention(q[:, :n].contiguous(), *codes, *scale, table, i32([600]), i32([0, n]), n, 600)
        b = fastar.kv8_attention(q[:, :n].contiguous(), *small.args(), near, i32([600]), i32([0, n]), n, 600)
        assert torch.equal(a, b)


# ---------------------------------------------------------------------------------------------------- append
def run_append(fastar, dtype, D, KV, PT, steps, seed=1, layout="htd", scale_of_step=lambda s: 1.0, spoil=None):
    """Steps of (new tokens per sequence): every pool value and scale as the plain form has them, bit for bit."""
    g, dt = gen(seed), TYPES[dtype]
    B = len(steps[0])
    total = [sum(s[b] for s in steps) for b in range(B)]
    need = [-(-t // PT) for t in total]
    table, order, at = torch.full((B, max(need) + 1), -3, dtype=torch.int32, device=DEV), torch.randperm(sum(need) + 2, generator=g, device=DEV).to(torch.int32), 0
    for b in range(B):
        table[b, : need[b]] = order[at: at + need[b]]
        at += need[b]
    pool = Pool(sum(need) + 2, KV, PT, D, seed)
    lens = [0] * B
    values = R.e4m3_values(DEV)
    for s, ns in enumerate(steps):
        lens = [a + n for a, n in zip(lens, ns)]
        cu = prefix(ns)
        k, v = (rows(g, KV, cu[-1] + 3, D, dt, layout, scale_of_step(s)) for _ in range(2))
        if spoil is not None:
            spoil(s, k, v)
        before, was = [c.clone() for c in pool.codes], [c.clone() for c in pool.scale]
        want = [R.append(x, c, sc, table, lens, cu, values[c.long()]) for x, c, sc in zip((k, v), pool.codes, pool.scale)]
        fastar.kv8_append(k, v, *pool.args(), table, i32(lens), i32(cu))
        for w in range(2):
            got = values[pool.codes[w].long()]
            val, sc = want[w]
            assert torch.equal(torch.nan_to_num(pool.scale[w].double(), nan=-1.0), torch.nan_to_num(sc, nan=-1.0))
            assert torch.equal(torch.isnan(got), torch.isnan(val))
            assert torch.equal(torch.nan_to_num(got), torch.nan_to_num(val))
            # bytes of rows that hold nothing are as they were, but in a page that has been recoded
            mask = torch.ones(pool.pages, PT, dtype=torch.bool, device=DEV)
            for b in range(B):
                for i in range(-(-lens[b] // PT)):
                    mask[int(table[b, i]), : min(PT, lens[b] - i * PT)] = False
            mask[(pool.scale[w] != was[w]).any(1)] = False
            same = (pool.codes[w] == before[w]).all(-1).all(1)
            assert bool(same[mask].all())


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("D,PT", [(64, 64), (64, 128), (128, 64), (128, 128)])
def test_append_in_steps(fastar, dtype, D, PT):
    run_append(fastar, dtype, D, 3, PT, [[1, 0, 130, 64, 5], [1, 1, 1, 1, 1], [70, 2, 0, 128, 1], [1, 1, 1, 1, 1]], scale_of_step=lambda s: [1.0, 3.0, 0.2, 40.0][s])


@pytest.mark.parametrize("dtype,big,tiny", [("bf16", 3e38, 1e-39), ("fp16", 65504.0, 6e-8)])
def test_append_extremes(fastar, dtype, big, tiny):
    def spoil(s, k, v):
        if s == 0:
            k.zero_()                      # a page of zeros, then rows that raise its scale
            v.fill_(tiny)
        elif s == 1:
            k.fill_(big)
            v[:, :, ::2] = 448.0
        elif s == 2:
            k[:, 0, 3], k[:, 1, 4], v[:, 0, 1] = float("inf"), float("nan"), float("-inf")
    run_append(fastar, dtype, 64, 2, 64, [[3, 60], [2, 1], [5, 3], [1, 1]], spoil=spoil)


@pytest.mark.parametrize("layout", ["thd", "slice"])
def test_append_strides(fastar, layout):
    run_append(fastar, "bf16", 128, 4, 64, [[100, 3], [1, 1], [5, 200]], layout=layout)


def test_append_many_sequences(fastar):
    run_append(fastar, "bf16", 64, 1, 64, [[(7 * b) % 5 for b in range(300)], [1] * 300, [b % 2 for b in range(300)]])


def test_append_passes_over_refused_sequences(fastar):
    g = gen(2)
    pool = Pool(4, 2, 64, 64)
    before = [t.clone() for t in pool.args()]
    k = rows(g, 2, 30, 64, torch.bfloat16)
    table = i32([[0, 1], [2, 3]])
    fastar.kv8_append(k, k, *pool.args(), table, i32([-1, -1]), i32([0, 10, 30]))
    for a, b in zip(before, pool.args()):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    out = torch.full((4, 30, 64), 3.0, dtype=torch.bfloat16, device=DEV)
    fastar.kv8_attention(rows(g, 4, 30, 64, torch.bfloat16), *pool.args(), table, i32([-1, -1]), i32([0, 10, 30]), 20, 128, out=out)
    assert bool((out == 3.0).all())


# ---------------------------------------------------------------------------------------------------- tables
def plain_tables(held, add, PT, free, first, table, max_add):
    table, cu, lens, slots, spent, upto = table.copy(), [0], [], [], 0, 0
    for b, (h, n) in enumerate(zip(held, add)):
        had, now = -(-h // PT), -(-(h + n) // PT)
        fits = now <= table.shape[1]
        need = now - had if fits else 0
        ok = fits and (need == 0 or upto + need <= len(free) - first)
        if ok:
            for i in range(need):
                table[b, had + i] = free[first + upto + i]
            if need:
                spent = upto + need
        upto += need
        cu.append(cu[-1] + n)
        lens.append(h + n if ok else -1)
        slots += [int(table[b, p // PT]) * PT + p % PT if ok else -1 for p in range(h, h + n)]
    return table, cu, lens, slots + [-1] * (max_add - len(slots)), first + spent


@pytest.mark.parametrize("PT", [64, 128])
@pytest.mark.parametrize("B", [1, 2, 33, 1024, 1025, 2500])
@pytest.mark.parametrize("short", [0, 1, 7])
def test_tables(fastar, PT, B, short):
    import random
    r = random.Random(B * 10 + short)
    held = [r.choice([0, 1, PT - 1, PT, PT + 1, 3 * PT, r.randrange(5 * PT)]) for _ in range(B)]
    add = [r.choice([0, 1, 1, 2, PT, r.randrange(3 * PT)]) for _ in range(B)]
    W = 8 if short != 7 else 5
    ids = list(range(3, 3 + 20 * B))
    r.shuffle(ids)
    import numpy as np
    table = np.full((B, W), -5, dtype=np.int32)
    for b in range(B):
        for i in range(min(W, -(-held[b] // PT))):
            table[b, i] = ids.pop()
    need = sum(max(0, -(-(h + n) // PT) - -(-h // PT)) for h, n in zip(held, add))
    first, free = 2, ids[: max(2, 2 + need - short)]
    if short:
        free = free[: 2 + max(0, need - short)]
    max_add = sum(add) + 5
    want = plain_tables(held, add, PT, free, first, table, max_add)
    t = torch.from_numpy(table).to(DEV)
    got = fastar.block_tables(i32(held), i32(add), PT, i32(free), i32([first]), t, max_add)
    assert t.cpu().tolist() == want[0].tolist()
    assert got["cu"].tolist() == want[1]
    assert got["lens"].tolist() == want[2]
    assert got["slots"].tolist() == want[3]
    assert got["first"].tolist() == [want[4]]
    full = any(n == -1 for n in want[2])
    assert fastar.dense_last_status() == (fastar.ERR_CAPACITY if full else 0)


def test_tables_slots_past_32_bits(fastar):
    t = i32([[-1, -1]])
    got = fastar.block_tables(i32([0]), i32([65]), 64, i32([2 ** 31 - 1, 2 ** 30]), i32([0]), t, 65)
    assert got["slots"][0].item() == (2 ** 31 - 1) * 64 and got["slots"][64].item() == 2 ** 30 * 64


def test_tables_bad_lengths(fastar):
    t = torch.full((4, 3), -1, dtype=torch.int32, device=DEV)
    got = fastar.block_tables(i32([0, -4, 2 ** 31 - 1, 10]), i32([5, 3, 9, 100]), 64, i32([0, 1, 2, 3]), i32([0]), t, 50)
    assert got["lens"].tolist() == [5, -1, -1, -1]                 # the last: beyond max_add
    assert got["cu"].tolist() == [0, 5, 8, 17, 50]
    assert fastar.dense_last_status() == fastar.ERR_BOUNDS
    got = fastar.block_tables(i32([0]), i32([5]), 64, i32([0, 1]), i32([3]), t[:1], 5)       # the list's start lies behind its end
    assert got["lens"].tolist() == [-1] and got["first"].tolist() == [3]
    assert fastar.dense_last_status() == fastar.ERR_BOUNDS


# ---------------------------------------------------------------------------------------------------- device-side refusals
def test_sequences_out_of_range_are_passed_over(fastar):
    g = gen(6)
    pool = Pool(8, 2, 64, 64)
    table = torch.arange(8, dtype=torch.int32, device=DEV).view(4, 2)
    pool.fill(g, table, [100] * 4)
    q = rows(g, 4, 12, 64, torch.bfloat16)
    good = fastar.kv8_attention(q, *pool.args(), table, i32([100] * 4), i32([0, 3, 6, 9, 12]), 3, 128)
    for lens, cu, alive in (([100, 200, 100, 100], [0, 3, 6, 9, 12], [0, 2, 3]),       # longer than max_len
                            ([100, 2, 100, 100], [0, 3, 6, 9, 12], [0, 2, 3]),         # fewer keys than new tokens
                            ([100] * 4, [0, 3, 6, 9, 13], [0, 1, 2]),                  # a token behind the last
                            ([100] * 4, [-1, 3, 6, 9, 12], [1, 2, 3])):
        out = torch.full_like(q, 2.0)
        fastar.kv8_attention(q, *pool.args(), table, i32(lens), i32(cu), 3, 128, out=out)
        assert fastar.dense_last_status() == fastar.ERR_BOUNDS
        for b in range(4):
            rows_b = out[:, 3 * b: 3 * b + 3]
            assert torch.equal(rows_b, good[:, 3 * b: 3 * b + 3]) if b in alive else bool((rows_b == 2.0).all())
    k = rows(g, 4, 12, 64, torch.bfloat16)
    out = torch.full_like(q, 2.0)
    fastar.packed_attention(q, k, k, i32([0, 3, 12]), 5, out=out)                        # nine tokens where five are the most
    assert fastar.dense_last_status() == fastar.ERR_BOUNDS
    assert bool((out[:, 3:] == 2.0).all()) and not bool((out[:, :3] == 2.0).all())


def test_pages_that_do_not_exist(fastar):
    g = gen(6)
    pool = Pool(3, 1, 64, 64)
    table = i32([[1, 3], [0, -1]])
    pool.fill(g, i32([[1], [0]]), [64, 64])
    before = [t.clone() for t in pool.args()]
    k = rows(g, 1, 4, 64, torch.bfloat16)
    fastar.kv8_append(k, k, *pool.args(), table, i32([66, 66]), i32([0, 2, 4]))
    assert fastar.dense_last_status() == fastar.ERR_BOUNDS
    for a, b in zip(before, pool.args()):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    for n in (2, 66):
        q = rows(g, 1, 2 * n, 64, torch.bfloat16)
        fastar.kv8_attention(q, *pool.args(), table, i32([66, 66]), i32([0, n, 2 * n]), n, 128)
        assert fastar.dense_last_status() == fastar.ERR_BOUNDS


# ---------------------------------------------------------------------------------------------------- together
def test_prompts_then_tokens(fastar):
    """Tables, prompts through packed attention, their rows into the cache, then steps of one or a few tokens, in a captured graph too."""
    g = gen(11)
    H, KV, D, PT, B = 6, 2, 128, 64, 5
    free = torch.randperm(64, generator=g, device=DEV).to(torch.int32)
    table = torch.full((B, 12), -1, dtype=torch.int32, device=DEV)
    pool = Pool(64, KV, PT, D)
    held, first = i32([0] * B), i32([0])
    for step, ns in enumerate([[70, 1, 200, 64, 333], [1] * B, [1] * B, [4, 1, 2, 3, 130], [1] * B]):
        T = sum(ns)
        q, k, v = rows(g, H, T, D, torch.bfloat16), rows(g, KV, T, D, torch.bfloat16), rows(g, KV, T, D, torch.bfloat16)
        t = fastar.block_tables(held, i32(ns), PT, free, first, table, T)
        fastar.kv8_append(k, v, *pool.args(), table, t["lens"], t["cu"])
        cu, lens = t["cu"].tolist(), t["lens"].tolist()
        if step == 0:
            out = fastar.packed_attention(q, k, v, t["cu"], max(ns))
            o, bound = R.attention(q, lambda b, h: k[h // 3, cu[b]: cu[b + 1]].double(), lambda b, h: v[h // 3, cu[b]: cu[b + 1]].double(), cu, ns, 1, torch.bfloat16)
            check(out, o, bound, cu)
        out = fastar.kv8_attention(q, *pool.args(), table, t["lens"], t["cu"], max(ns), 12 * PT)
        o, bound = R.attention(q, lambda b, h: pool.rows(0, table[b], lens[b], h // 3), lambda b, h: pool.rows(1, table[b], lens[b], h // 3), cu, lens, 1, torch.bfloat16)
        check(out, o, bound, cu)
        # the slots say where the rows went
        codes = pool.codes[0].transpose(1, 2).reshape(-1, KV, D)[t["slots"]]
        scale = pool.scale[0][t["slots"] // PT]
        near = R.e4m3_values(DEV)[codes.long()] * scale.double()[..., None]
        assert float((near - k.transpose(0, 1).double()).abs().max()) <= 2.0 ** -4 * float(k.abs().max())
        held, first = t["lens"].clone(), t["first"].clone()


@pytest.mark.parametrize("n", [1, 3])
def test_a_captured_step_goes_on(fastar, n):
    """One step in a graph: lengths, free list and tables advance on the device, replay after replay."""
    g = gen(12)
    H, KV, D, PT, B = 4, 2, 64, 64, 3
    free = torch.randperm(40, generator=g, device=DEV).to(torch.int32)

    def state():
        return dict(table=torch.full((B, 8), -1, dtype=torch.int32, device=DEV), pool=Pool(40, KV, PT, D), held=i32([60, 0, 127]), first=i32([0]),
                    q=torch.zeros(H, B * n, D, dtype=torch.bfloat16, device=DEV), k=torch.zeros(KV, B * n, D, dtype=torch.bfloat16, device=DEV),
                    v=torch.zeros(KV, B * n, D, dtype=torch.bfloat16, device=DEV), out=torch.zeros(H, B * n, D, dtype=torch.bfloat16, device=DEV), add=i32([n] * B))

    def step(s):
        t = fastar.block_tables(s["held"], s["add"], PT, free, s["first"], s["table"], B * n)
        fastar.kv8_append(s["k"], s["v"], *s["pool"].args(), s["table"], t["lens"], t["cu"])
        fastar.kv8_attention(s["q"], *s["pool"].args(), s["table"], t["lens"], t["cu"], n, 8 * PT, out=s["out"])
        s["held"].copy_(t["lens"])
        s["first"].copy_(t["first"])

    def start(s):      # rows that are there already
        t = fastar.block_tables(i32([0] * B), s["held"], PT, free, s["first"], s["table"], 187)
        s["first"].copy_(t["first"])
        x = rows(gen(1), KV, 187, D, torch.bfloat16)
        fastar.kv8_append(x, x, *s["pool"].args(), s["table"], t["lens"], t["cu"])
        return s

    a, b = start(state()), start(state())
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        step(b)
    for r in range(20):
        for name in "qkv":
            x = rows(g, a[name].shape[0], B * n, D, torch.bfloat16)
            a[name].copy_(x)
            b[name].copy_(x)
        step(a)
        graph.replay()
        assert torch.equal(a["out"], b["out"]) and torch.equal(a["held"], b["held"]) and torch.equal(a["first"], b["first"])
    assert a["held"].tolist() == [60 + 20 * n, 20 * n, 127 + 20 * n]


def test_two_captured_calls_at_once(fastar):
    """Each captured call has a workspace of its own: two graphs replayed at the same time give what they give alone."""
    g = gen(13)
    pool = Pool(300, 2, 64, 128)
    table = torch.arange(300, dtype=torch.int32, device=DEV).view(2, 150)
    pool.fill(g, table, [9000, 8000])
    qs = [rows(g, 4, 2, 128, torch.bfloat16) for _ in range(2)]
    outs = [torch.zeros_like(q) for q in qs]
    lens, cu = i32([9000, 8000]), i32([0, 1, 2])
    call = lambda i: fastar.kv8_attention(qs[i], *pool.args(), table, lens, cu, 1, 9000, out=outs[i])  # noqa: E731
    for i in range(2):
        call(i)
    want = [o.clone() for o in outs]
    graphs, streams = [], [torch.cuda.Stream() for _ in range(2)]
    for i in range(2):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr, stream=streams[i]):
            for _ in range(20):
                call(i)
        graphs.append(gr)
    for o in outs:
        o.zero_()
    torch.cuda.synchronize()
    for _ in range(5):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                graphs[i].replay()
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert torch.equal(o, w)


@pytest.mark.parametrize("D", [64, 128])
def test_strides_that_are_not_used(fastar, D):
    """One token, or one head: whatever the stride over it says."""
    g = gen(15)
    x = rows(g, 1, 6, D, torch.bfloat16)
    one = [t.as_strided((2, 1, D), (D, 3, 1)) for t in (rows(g, 2, 1, D, torch.bfloat16) for _ in range(3))]
    head = [t.as_strided((1, 6, D), (5, D, 1)) for t in (x, rows(g, 1, 6, D, torch.bfloat16), rows(g, 1, 6, D, torch.bfloat16))]
    for q, k, v in (one, head):
        T = q.shape[1]
        out = torch.empty_like(q.contiguous()).as_strided(q.shape, q.stride())
        got = fastar.packed_attention(q, k, v, i32([0, T]), T, out=out)
        want = fastar.packed_attention(*(t.clone(memory_format=torch.contiguous_format) for t in (q, k, v)), i32([0, T]), T)
        assert torch.equal(got, want)


def test_on_another_stream(fastar):
    g = gen(14)
    q, k, v = (rows(g, 2, 700, 64, torch.bfloat16) for _ in range(3))
    want = fastar.packed_attention(q, k, v, i32([0, 700]), 700)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = fastar.packed_attention(q, k, v, i32([0, 700]), 700)
    s.synchronize()
    assert torch.equal(want, got)
