"""Paged cache: bad arguments are refused on the host, before anything is launched."""
import ctypes
import pathlib
import random
import subprocess
import sys

import pytest
import torch

from paper_2609_16450_amd import binding as B

ROOT = pathlib.Path(__file__).resolve().parents[1]


def _ragged(batch=1, T=4, maxb=4, S=20, maxp=20, cu_b=0x1000, cu_p=0x2000):
    return B.eb_ragged(batch, T, maxb, S, maxp, cu_b, cu_p)


def _kv(**change):
    f = dict(dtype=B.EB_BF16, hkv=2, head_dim=128, n_pages=4, page_size=16, max_pages=2,
             page_table=0x1000, k=0x100, v=0x200, k_scale=None, v_scale=None)
    f.update(change)
    return B.eb_paged_kv(*f.values())


def _write(r, kv, dt=B.EB_BF16, pos=None, k=0x100, v=0x200):
    return B.load().eb_kv_write(dt, ctypes.byref(r), ctypes.byref(kv), pos, k, v, None)


def _read(r, kv, dt=B.EB_BF16, k=0x100, v=0x200):
    return B.load().eb_kv_read(dt, ctypes.byref(r), ctypes.byref(kv), k, v, None)


def _attn(r, kv, dt=B.EB_BF16, hq=4, scale=0.1, q=0x100, k=0x100, v=0x100, out=0x100, ws=None, n=0):
    return B.load().eb_block_attn_paged(dt, ctypes.byref(r), ctypes.byref(kv), hq, scale, q, k, v,
                                        out, ws, n, None)


BAD = [
    (dict(dtype=7), B.EB_ERR_INVALID, "dtype"),
    (dict(hkv=0), B.EB_ERR_INVALID, "hkv"),
    (dict(n_pages=0), B.EB_ERR_INVALID, "n_pages"),
    (dict(max_pages=0), B.EB_ERR_INVALID, "max_pages"),
    (dict(head_dim=0), B.EB_ERR_INVALID, "head_dim"),
    (dict(head_dim=96), B.EB_ERR_UNSUPPORTED, "head_dim"),
    (dict(page_size=0), B.EB_ERR_INVALID, "page_size"),
    (dict(page_size=8), B.EB_ERR_UNSUPPORTED, "page_size"),
    (dict(page_size=48), B.EB_ERR_UNSUPPORTED, "page_size"),
    (dict(page_size=512), B.EB_ERR_UNSUPPORTED, "page_size"),
    (dict(page_size=0x7fffffff), B.EB_ERR_UNSUPPORTED, "page_size"),
    (dict(dtype=B.EB_F32), B.EB_ERR_UNSUPPORTED, "dtype"),
    (dict(page_table=None), B.EB_ERR_INVALID, "NULL"),
    (dict(k=None), B.EB_ERR_INVALID, "NULL"),
    (dict(v=0x208), B.EB_ERR_INVALID, "aligned"),
    (dict(dtype=B.EB_E4M3), B.EB_ERR_INVALID, "k_scale"),
    (dict(dtype=B.EB_E4M3, k_scale=0x100), B.EB_ERR_INVALID, "v_scale"),
    (dict(dtype=B.EB_E4M3, k_scale=0x100, v_scale=0x101), B.EB_ERR_INVALID, "aligned"),
]


@pytest.mark.parametrize("change,status,word", BAD)
def test_bad_cache(change, status, word):
    r, kv = _ragged(), _kv(**change)
    for call in (_write, _read, _attn):
        assert call(r, kv) == status
        assert word in B.eb_last_error()


def test_bad_rows():
    r, kv = _ragged(), _kv()
    # the rows' type: unknown, or an 8-bit type, which only caches have
    for dt in (5, B.EB_E4M3):
        assert _write(r, kv, dt) == _read(r, kv, dt) == _attn(r, kv, dt) == B.EB_ERR_INVALID
    # bf16 rows of an fp32 cache would be rounded, and the other way mixed
    assert _write(r, kv, B.EB_F32) == _read(r, kv, B.EB_F32) == B.EB_ERR_UNSUPPORTED
    assert _attn(r, kv, B.EB_F32) == B.EB_ERR_UNSUPPORTED
    for bad in (None, 0x101):
        assert _write(r, kv, k=bad) == _write(r, kv, v=bad) == B.EB_ERR_INVALID
        assert _read(r, kv, k=bad) == _read(r, kv, v=bad) == B.EB_ERR_INVALID
        assert _attn(r, kv, q=bad) == _attn(r, kv, out=bad) == B.EB_ERR_INVALID
    assert _attn(r, kv, hq=3) == _attn(r, kv, hq=0) == B.EB_ERR_INVALID
    assert _attn(r, kv, scale=-1.0) == _attn(r, kv, scale=float("nan")) == B.EB_ERR_INVALID


def test_bad_lengths():
    kv = _kv()
    long = _ragged(S=33, maxp=33)                       # two pages of 16 rows
    assert _read(long, kv) == _attn(long, kv) == B.EB_ERR_INVALID
    assert "max_prefix" in B.eb_last_error()
    for r in (_ragged(batch=0), _ragged(cu_p=None), _ragged(S=3, maxp=4), _ragged(S=-1, maxp=-1)):
        assert _read(r, kv) == _attn(r, kv) == _write(r, kv) == B.EB_ERR_INVALID
    assert _attn(_ragged(cu_b=None), kv) == _write(_ragged(cu_b=None), kv) == B.EB_ERR_INVALID
    assert _attn(_ragged(T=4, maxb=5), kv) == _write(_ragged(T=4, maxb=5), kv) == B.EB_ERR_INVALID
    lib = B.load()
    assert lib.eb_kv_write(B.EB_BF16, None, ctypes.byref(kv), None, 0x100, 0x100, None) == \
        B.EB_ERR_INVALID
    assert lib.eb_kv_read(B.EB_BF16, ctypes.byref(_ragged()), None, 0x100, 0x100, None) == \
        B.EB_ERR_INVALID


def test_workspace():
    lib = B.load()
    r, kv = _ragged(S=20, maxp=20), _kv(max_pages=1 << 12, n_pages=1 << 12)
    long = _ragged(S=60000, maxp=60000)

    def need(rr, kk, hq=4):
        return lib.eb_block_attn_paged_workspace(B.EB_BF16, ctypes.byref(rr), ctypes.byref(kk), hq)

    n = need(long, kv)
    assert n > 0
    assert _attn(long, kv, ws=0x100, n=n - 1) == B.EB_ERR_WORKSPACE
    assert _attn(long, kv, ws=None, n=n) == B.EB_ERR_WORKSPACE
    # queries with bad arguments
    assert need(r, kv, hq=3) == need(_ragged(batch=0), kv) == 0
    assert need(r, _kv(hkv=0)) == need(_ragged(T=0, maxb=0), kv) == 0
    assert need(r, _kv(page_size=0x7fffffff)) >= 0
    assert lib.eb_block_attn_paged_workspace(B.EB_BF16, None, ctypes.byref(kv), 4) == 0
    assert lib.eb_block_attn_paged_workspace(B.EB_BF16, ctypes.byref(r), None, 4) == 0


# (batch, rows, longest block, cached rows, longest prefix), query heads, K/V heads: a longest block
# or prefix beyond the totals, negative totals, and sizes whose products pass 64 bits
NO_BATCH = [((70, 1, 100, 1000000, 20000), 28, 4), ((1, 1, 1, -256, 5000), 28, 4),
            ((1, 1, 1, 4000, 5000), 28, 4), ((3, -5, -5, 100, 100), 4, 4),
            ((1, 4, 4, 100, -1), 4, 4)]
TOO_LARGE = [((1, 1 << 29, 1 << 29, 0, 0), 1 << 30, 1), ((1, 1 << 30, 1 << 30, 0, 0), 1 << 30, 2),
             ((65535, 1 << 30, 1 << 15, 0, 0), 0x7fffffff, 1)]


def test_sizes_that_no_plan_is_made_for():
    """The query returns 0 and the call is refused, before a plan divides or multiplies by them.  (In
    a child process, which a division by zero would end.)"""
    sizes = NO_BATCH + TOO_LARGE
    types = [(B.EB_F32, B.EB_F32), (B.EB_F32, B.EB_E4M3), (B.EB_BF16, B.EB_BF16),
             (B.EB_BF16, B.EB_E4M3)]
    code = (f"import ctypes, sys; sys.path.insert(0, {str(ROOT)!r})\n"
            "from paper_2609_16450_amd import binding as B\n"
            f"B._LIB_PATH = {B._LIB_PATH!r}\n"
            f"for size, hq, hkv in {sizes}:\n"
            f"  for dt, cache in {types}:\n"
            "    r = B.eb_ragged(*size, 0x1000, 0x2000)\n"
            "    kv = B.eb_paged_kv(cache, hkv, 128, 1 << 20, 256, 1 << 22, 0x1000, 0x100, 0x200,"
            " 0x300, 0x400)\n"
            "    a = dt, ctypes.byref(r), ctypes.byref(kv), hq\n"
            "    print(B.load().eb_block_attn_paged_workspace(*a), B.load().eb_block_attn_paged("
            "*a, 0.1, 0x100, 0x100, 0x100, 0x100, None, 0, None), flush=True)\n")
    res = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    want = [f"0 {B.EB_ERR_INVALID if s in NO_BATCH else B.EB_ERR_UNSUPPORTED}"
            for s in sizes for _ in types]
    assert (res.returncode, res.stdout.splitlines()) == (0, want), res.stderr[-500:]


def _need(blocks, cached, hq, hkv, head_dim, dt, cache):
    r = _ragged(len(blocks), sum(blocks), max(blocks), sum(cached), max(cached))
    kv = _kv(dtype=cache, hkv=hkv, head_dim=head_dim, n_pages=1 << 20, max_pages=1 << 20,
             k_scale=0x100, v_scale=0x100)
    return B.load().eb_block_attn_paged_workspace(dt, ctypes.byref(r), ctypes.byref(kv), hq)


# a block of 33 rows behind 600: 11 ranges; a long block among many short ones, which the host can
# not tell from blocks of 17 rows: 1024 partials of 128 rows
@pytest.mark.parametrize("blocks,cached,hq,hkv,most", [
    ([33], [600], 1, 1, 16), ([100], [600], 28, 4, 512), ([1] * 255 + [512], [2500] * 256, 28, 4, 1024),
    ([1] * 199 + [64], [2500] * 200, 16, 4, 1024), ([2] * 299 + [40], [2500] * 300, 16, 4, 1024)])
@pytest.mark.parametrize("cache", [B.EB_BF16, B.EB_E4M3])
def test_workspace_follows_the_call(cache, blocks, cached, hq, hkv, most):
    row = (128 + 2) * 4
    assert _need(blocks, cached, hq, hkv, 128, B.EB_BF16, cache) <= most * 128 * row + 4096


def test_largest_workspace():
    """The bound that eb.h gives, over sizes of all orders."""
    rng = random.Random(0)
    for _ in range(4000):
        n = int(2 ** rng.uniform(0, 10))
        lo, hi = sorted(int(2 ** rng.uniform(0, 12)) for _ in range(2))
        blocks = [rng.randint(lo, hi) if rng.random() < 0.5 else lo for _ in range(n)]
        longest = int(2 ** rng.uniform(0, 17))
        cached = [rng.randint(0, longest) for _ in range(n)]
        hkv, group = 2 ** rng.randint(0, 9), rng.randint(1, 16)
        for dt, cache in ((B.EB_F32, B.EB_F32), (B.EB_BF16, B.EB_BF16), (B.EB_BF16, B.EB_E4M3)):
            if sum(blocks) * hkv * group < 2 ** 31:
                assert _need(blocks, cached, hkv * group, hkv, 128, dt, cache) <= 137e6


def test_workspace_alignment():
    kv = _kv(max_pages=1 << 12, n_pages=1 << 12)
    long = _ragged(S=60000, maxp=60000)
    assert _attn(long, kv, ws=0x108, n=1 << 30) == B.EB_ERR_INVALID
    assert "workspace" in B.eb_last_error()


def test_too_much_for_one_launch():
    """Grids of 2^32 threads and more, each kernel's own."""
    kv = _kv(max_pages=1 << 12, n_pages=1 << 12, hkv=1 << 10)
    rows = dict(S=0, maxp=0)
    heads = dict(hq=1 << 10)
    # 65000 sequences x 1024 heads of single tokens; many more rows of one head
    assert _attn(_ragged(65000, 65000, 1, **rows), kv, **heads) == B.EB_ERR_UNSUPPORTED
    assert "launch" in B.eb_last_error()
    assert _attn(_ragged(60000, 1 << 28, 1 << 14, **rows), kv, **heads) == B.EB_ERR_UNSUPPORTED
    # the tiles of the longest block for every sequence, in fp32
    kv = _kv(dtype=B.EB_F32, hkv=1)
    assert _attn(_ragged(1, 1 << 29, 1 << 29, **rows), kv, B.EB_F32, hq=1) == B.EB_ERR_UNSUPPORTED


def test_too_much_for_one_call():
    kv = _kv(max_pages=1 << 27, n_pages=1 << 27)
    many = _ragged(T=1 << 28, maxb=1, S=1 << 28, maxp=1)
    assert _write(many, kv) == _read(many, kv) == B.EB_ERR_UNSUPPORTED
    assert _attn(_ragged(S=1 << 30, maxp=1 << 30), kv) == B.EB_ERR_UNSUPPORTED
    assert _attn(_ragged(batch=70000), kv) == B.EB_ERR_UNSUPPORTED


def test_empty_calls_need_no_rows():
    kv, r = _kv(), _ragged(T=0, maxb=0, S=0, maxp=0)
    assert _write(r, kv, k=None, v=None) == B.EB_OK
    assert _read(r, kv, k=None, v=None) == B.EB_OK
    assert _attn(r, kv, q=None, k=None, v=None, out=None) == B.EB_OK


def test_binding_refuses_what_is_no_cache():
    t = torch.zeros(1, 1, dtype=torch.int32)
    pool = torch.zeros(1, 1, 16, 64)
    with pytest.raises(ValueError, match="float8"):
        B.PagedKV(pool.half(), pool.half(), t)
    with pytest.raises(ValueError, match="shape"):
        B.PagedKV(pool[0], pool[0], t)
    with pytest.raises(ValueError, match="page_table"):
        B.PagedKV(pool, pool, t[0])
    with pytest.raises(ValueError, match="device"):
        B.PagedKV(pool, pool, t)
