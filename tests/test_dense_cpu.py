"""The dense path without a GPU: argument checks of the C entries, of the Python functions, and the index arithmetic that the kernels share with the host."""
import ctypes as C
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    from paper_2602_01801_b200 import build, fastar
    build.build_library()
    return fastar.load_library()


@pytest.fixture()
def mem():
    buf = C.create_string_buffer(4096 + 64)
    return (C.addressof(buf) + 63) & ~63, buf


BIG = 1 << 20


def packed_args(p, **kw):
    a = dict(q=p, k=p, v=p, out=p + 2048, hs=BIG, ts=128, khs=BIG, kts=128, cu=p, seqs=2, total=10, max=5, H=4, KV=2, D=128, dtype=0, frame=1, stream=None)
    a.update(kw)
    return list(a.values())


def attend_args(p, **kw):
    a = dict(q=p, out=p + 2048, hs=BIG, ts=128, kc=p, vc=p, ks=p, vs=p, pages=4, PT=64, table=p, W=400, lens=p, cu=p, seqs=2, total=10, max_new=5, max_len=25600, H=4, KV=2, D=128,
             dtype=0, frame=1, work=p, bytes=1 << 40, stream=None)
    a.update(kw)
    return list(a.values())


def append_args(p, **kw):
    a = dict(k=p, v=p, hs=BIG, ts=128, kc=p, vc=p, ks=p, vs=p, pages=4, PT=64, table=p, W=4, lens=p, cu=p, seqs=2, total=10, KV=2, D=128, dtype=0, stream=None)
    a.update(kw)
    return list(a.values())


def table_args(p, **kw):
    a = dict(held=p, add=p, seqs=2, PT=64, free=p, num_free=3, first=p, table=p, W=4, cu=p, lens=p + 64, slots=p, max_add=8, first_out=p + 128, stream=None)
    a.update(kw)
    return list(a.values())


@pytest.mark.parametrize("bad,status", [
    (dict(q=None), -1), (dict(k=None), -1), (dict(v=None), -1), (dict(out=None), -1), (dict(cu=None), -1), (dict(seqs=0), -1), (dict(total=-1), -1), (dict(max=0), -1),
    (dict(H=3), -1), (dict(KV=0), -1), (dict(H=1), -1), (dict(D=96), -2), (dict(dtype=1), -1), (dict(dtype=3), -1), (dict(frame=-1), -1), (dict(ts=64), -1),
    (dict(kts=120), -1), (dict(hs=100), -1), (dict(max=2 ** 30 + 1), -2), (dict(seqs=2 ** 20 + 1), -2), (dict(total=2 ** 29), -2), (dict(ts=132), -1), (dict(khs=0), -1), (dict(hs=-BIG), -1)])
def test_packed_refusals(lib, mem, bad, status):
    assert lib.fastar_packed_attention(*packed_args(mem[0], **bad)) == status
    if "q" in bad:
        assert lib.fastar_packed_attention(*packed_args(mem[0], q=mem[0] + 2)) == -1
        assert lib.fastar_packed_attention(*packed_args(mem[0], cu=mem[0] + 2)) == -1
        for name in ("q", "k", "v"):                                            # in place
            assert lib.fastar_packed_attention(*packed_args(mem[0], **{name: mem[0] + 2048})) == -1


@pytest.mark.parametrize("bad,status", [
    (dict(q=None), -1), (dict(out=None), -1), (dict(kc=None), -1), (dict(vs=None), -1), (dict(table=None), -1), (dict(lens=None), -1), (dict(cu=None), -1), (dict(seqs=0), -1),
    (dict(total=-1), -1), (dict(max_new=0), -1), (dict(max_len=4), -1), (dict(max_len=25601), -1), (dict(pages=0), -1), (dict(W=0), -1), (dict(PT=32), -2), (dict(D=32), -2),
    (dict(dtype=1), -1), (dict(frame=-2), -1), (dict(H=5), -1), (dict(work=None), -7), (dict(bytes=0), -7), (dict(ts=64), -1), (dict(hs=9), -1)])
def test_paged_refusals(lib, mem, bad, status):
    assert lib.fastar_kv8_attention(*attend_args(mem[0], **bad)) == status
    if "q" in bad:
        assert lib.fastar_kv8_attention(*attend_args(mem[0], kc=mem[0] + 8)) == -1
        assert lib.fastar_kv8_attention(*attend_args(mem[0], work=mem[0] + 8)) == -7
        assert lib.fastar_kv8_attention(*attend_args(mem[0], out=mem[0])) == -1             # in place


@pytest.mark.parametrize("bad,status", [
    (dict(k=None), -1), (dict(v=None), -1), (dict(kc=None), -1), (dict(ks=None), -1), (dict(table=None), -1), (dict(lens=None), -1), (dict(cu=None), -1), (dict(seqs=0), -1),
    (dict(total=-1), -1), (dict(pages=0), -1), (dict(W=0), -1), (dict(PT=16), -2), (dict(KV=0), -1), (dict(D=80), -2), (dict(dtype=1), -1), (dict(ts=8), -1), (dict(hs=8), -1)])
def test_append_refusals(lib, mem, bad, status):
    assert lib.fastar_kv8_append(*append_args(mem[0], **bad)) == status


@pytest.mark.parametrize("bad,status", [
    (dict(held=None), -1), (dict(add=None), -1), (dict(free=None), -1), (dict(first=None), -1), (dict(table=None), -1), (dict(cu=None), -1), (dict(lens=None), -1),
    (dict(slots=None), -1), (dict(first_out=None), -1), (dict(seqs=0), -1), (dict(PT=100), -2), (dict(num_free=-1), -1), (dict(W=0), -1), (dict(max_add=-1), -1)])
def test_table_refusals(lib, mem, bad, status):
    p = mem[0]
    assert lib.fastar_block_tables(*table_args(p, **bad)) == status
    assert lib.fastar_block_tables(*table_args(p, lens=p)) == -1               # in place
    assert lib.fastar_block_tables(*table_args(p, first_out=p)) == -1
    assert lib.fastar_block_tables(*table_args(p, slots=p + 4)) == -1


@pytest.mark.parametrize("bad", [dict(max_add=2 ** 30 + 1), dict(max_add=2 ** 31 - 1), dict(seqs=2 ** 20 + 1), dict(seqs=2 ** 31 - 1)])
def test_table_limits(lib, mem, bad):
    """Slots and requests are counted in 32 bits, with room for a grid's step: as many as the other calls take."""
    assert lib.fastar_block_tables(*table_args(mem[0], cu=mem[0] + 192, **bad)) == -2


def test_tables_are_not_in_place(lib, mem):
    """Every CTA of the tables' kernel reads all requests by itself, so what one writes must lie apart from what the others read, and outputs apart from one another."""
    p = mem[0]
    at = dict(held=p, add=p + 64, free=p + 128, first=p + 192, table=p + 256, cu=p + 320, lens=p + 384, slots=p + 512, first_out=p + 640)
    size = dict(held=8, add=8, free=12, first=4, table=32, cu=12, lens=8, slots=64, first_out=4)
    outputs = ("table", "cu", "lens", "slots", "first_out")
    import torch
    if not torch.cuda.is_available():                                          # (there it would run with host pointers)
        assert lib.fastar_block_tables(*table_args(p, **at)) not in (-1, -2)
        assert lib.fastar_block_tables(*table_args(p, **dict(at, held=p, add=p, lens=p + 8, cu=p + 16, first_out=p + 28))) not in (-1, -2)      # side by side, one input twice
    for out in outputs:
        for other in at:
            if other != out:
                for place in (at[other], at[other] + (size[other] - 1) // 8 * 8, at[other] - (size[out] - 1) // 8 * 8):
                    assert lib.fastar_block_tables(*table_args(p, **dict(at, **{out: place}))) == -1, (out, other, place - at[other])


def test_empty_free_list_is_no_bad_argument(lib, mem):
    """A list without pages may be a null pointer (an empty tensor's is): requests that need no page are served without it.  (What follows the checks here is that
    there is no GPU.)"""
    import torch
    if torch.cuda.is_available():
        pytest.skip("would run with host pointers")
    p = mem[0]
    args = dict(add=p + 64, first=p + 128, table=p + 256, cu=p + 320, lens=p + 384, slots=p + 512, first_out=p + 640, free=None, num_free=0)
    assert lib.fastar_block_tables(*table_args(p, **args)) not in (-1, -2)
    assert lib.fastar_block_tables(*table_args(p, **args, max_add=-1)) == -1
    assert lib.fastar_block_tables(*table_args(p, **args, seqs=0)) == -1
    assert lib.fastar_block_tables(*table_args(p, **dict(args, num_free=1))) == -1


def test_arguments_as_words(lib, mem):
    """fastar_dense_call takes the calls' arguments as 64-bit words and answers as they do; a count or a 32-bit argument that is not theirs is refused."""
    from paper_2602_01801_b200 import fastar
    p = mem[0]
    for (call, pack, n), args, bad in ((fastar._TABLES, table_args, dict(PT=100)), (fastar._APPEND, append_args, dict(D=80)), (fastar._ATTENTION, attend_args, dict(PT=32)),
                                       (fastar._PACKED, packed_args, dict(D=96))):
        words = [0 if a is None else a for a in args(p, **bad)]
        assert len(words) == n
        assert lib.fastar_dense_call(call, pack(*words), n) == -2
        assert lib.fastar_dense_call(call, pack(*words), n - 1) == -1
        assert lib.fastar_dense_call(call, None, n) == -1
        for i in (i for i, v in enumerate(words) if 0 < v < 1000):
            wide = list(words)
            wide[i] += 1 << 32
            assert lib.fastar_dense_call(call, pack(*wide), n) in (-1, -2)
    assert lib.fastar_dense_call(4, b"", 0) == -1 and lib.fastar_dense_call(-1, b"", 0) == -1
    words = packed_args(p, seqs=2 + (1 << 32))
    words[-1] = 0
    assert lib.fastar_dense_call(3, fastar._PACKED[1](*words), 18) == -1


def test_workspace_sizes(lib):
    size = lib.fastar_kv8_attention_workspace_bytes
    assert size(1, 0, 1, 1, 1, 1, 64) >= 16
    for bad in ((0, 1, 1, 1, 1, 1, 64), (1, -1, 1, 1, 1, 1, 64), (1, 1, 0, 1, 1, 1, 64), (1, 1, 2, 1, 1, 1, 64), (1, 1, 1, 1, 3, 2, 64), (1, 1, 1, 1, 1, 1, 96), (1, 1, 1, 2 ** 30 + 1, 1, 1, 64), (1, 2 ** 29, 1, 1, 4, 1, 64), (2 ** 20 + 1, 1, 1, 1, 1, 1, 64), (2 ** 20, 1, 1, 2 ** 30, 60000, 60000, 64)):
        assert size(*bad) == 0
    # never beyond one part for every 128 keys and row, and two pieces of 32 rows for each of 592 CTAs
    for args in ((1, 1, 1, 65536, 40, 8, 128), (64, 64, 1, 16384, 16, 4, 64), (3, 4680, 1560, 32768, 12, 12, 128), (1, 1, 1, 2 ** 30, 1, 1, 128)):
        B, T, n, L, H, KV, D = args
        assert 16 <= size(*args) <= 16 + T * H * (D + 2) * 4 * (-(-L // 128)) + 1184 * 32 * (D + 2) * 4 + T * H * 8 + 256


def test_python_refusals():
    import torch
    from paper_2602_01801_b200 import fastar
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16)                             # not on a GPU
    with pytest.raises(fastar.FastarError):
        fastar.packed_attention(q, q, q, torch.zeros(2, dtype=torch.int32), 4)
    with pytest.raises(fastar.FastarError):
        fastar.kv8_append(q, q, None, None, None, None, None, None, None)
    with pytest.raises(fastar.FastarError):
        fastar.block_tables(torch.zeros(2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), 64, q, q, torch.zeros(2, 2, dtype=torch.int32), 4)


def test_index_arithmetic(tmp_path):
    """visible_end, check_seq, scale_exp_of and the bounds of the launches against plain loops, over small ranges and at the ends of 32 bits."""
    exe = tmp_path / "dense_indices"
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    r = subprocess.run([nvcc, "-std=c++17", "-O1", "-o", str(exe), os.path.join(ROOT, "tests", "dense_indices.cu")], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "ok" in r.stdout, r.stdout + r.stderr


def test_strides_over_one_head_or_token_do_not_count():
    """Outputs (and values beside keys) whose strides differ only where there is one head, one token or none are taken, others refused."""
    import torch
    from paper_2602_01801_b200 import fastar
    wide = torch.zeros(4, 3, 5, 64, dtype=torch.bfloat16)                      # queries, keys and values of five tokens in one tensor, by heads
    rows = torch.zeros(5, 12, 64, dtype=torch.bfloat16).transpose(0, 1)        # and by tokens
    for q in (rows[:4, :1], wide[:1, 1], wide[:1, 2, :1], rows[8:9, 4:], wide[:, 0, :0]):
        out = torch.zeros(q.shape, dtype=q.dtype)
        assert fastar._out_like(torch, q, q.stride(), out, "here") is out
        made = fastar._out_like(torch, q, q.stride(), None, "here")
        assert made.shape == q.shape and fastar._strides_fit(q.shape, made.stride(), q.stride())
    for q in (wide[:, 0, :2], wide[:, 0, :1], rows[:1]):
        with pytest.raises(fastar.FastarError):
            fastar._out_like(torch, q, q.stride(), torch.zeros(q.shape, dtype=q.dtype), "here")
    with pytest.raises(fastar.FastarError):
        fastar._out_like(torch, wide[:1, 0], wide[:1, 0].stride(), torch.zeros(1, 5, 128, dtype=q.dtype)[..., ::2], "here")      # columns apart
    assert fastar._strides_fit((4, 1, 64), (960, 7, 1), (960, 64, 1)) and not fastar._strides_fit((4, 2, 64), (960, 7, 1), (960, 64, 1))
