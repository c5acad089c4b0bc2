"""eb_lmhead_logits, eb_sample, eb_kv_assign: bad arguments are refused on the host, before anything is
launched."""
import ctypes

import pytest
import torch

from paper_2609_16450_amd import binding as B

A = 0x100                                              # an address that is never read


def _ragged(**change):
    f = dict(batch=2, total_block=6, max_block=4, total_prefix=0, max_prefix=0, cu_block=A,
             cu_prefix=None)
    f.update(change)
    return B.eb_ragged(*f.values())


def _sample(r=None, dt=B.EB_F32, vocab=100, pitch=100, logits=A, uniform=A, params=None, token=A,
            ws=A, n=1 << 40):
    r = _ragged() if r is None else r
    return B.load().eb_sample(dt, ctypes.byref(r), vocab, pitch, logits, uniform, params, token, None,
                              None, ws, n, None)


@pytest.mark.parametrize("change,status,word", [
    (dict(dt=B.EB_E4M3), B.EB_ERR_INVALID, "dtype"),
    (dict(dt=-1), B.EB_ERR_INVALID, "dtype"),
    (dict(r=_ragged(batch=0)), B.EB_ERR_INVALID, "batch"),
    (dict(r=_ragged(max_block=7)), B.EB_ERR_INVALID, "block"),
    (dict(r=_ragged(total_block=-1)), B.EB_ERR_INVALID, "block"),
    (dict(r=_ragged(cu_block=None)), B.EB_ERR_INVALID, "cu_block"),
    (dict(vocab=0), B.EB_ERR_INVALID, "vocab"),
    (dict(pitch=99), B.EB_ERR_INVALID, "pitch"),
    (dict(pitch=-(1 << 40)), B.EB_ERR_INVALID, "pitch"),
    (dict(vocab=(1 << 21) + 1, pitch=1 << 22), B.EB_ERR_UNSUPPORTED, "vocab"),
    (dict(logits=None), B.EB_ERR_INVALID, "NULL"),
    (dict(uniform=None), B.EB_ERR_INVALID, "NULL"),
    (dict(token=None), B.EB_ERR_INVALID, "NULL"),
])
def test_sample_refuses(change, status, word):
    assert _sample(**change) == status
    assert word in B.eb_last_error()


def test_sample_workspace():
    q = B.load().eb_sample_workspace
    for dt in (B.EB_F32, B.EB_BF16):
        for vocab in (1, 1000, 2048, 152064, 1 << 21):
            sizes = [q(dt, n, vocab) for n in (1, 2, 3, 17, 64, 255, 256, 1000, 4096)]
            assert sizes == sorted(sizes) and all(s % 256 == 0 for s in sizes)
        assert q(dt, 0, 100) == q(dt, -1, 100) == q(dt, 4, 0) == q(dt, 4, (1 << 21) + 1) == 0
    need = q(B.EB_F32, 6, 100000)
    if need:
        args = dict(vocab=100000, pitch=100000)
        assert _sample(**args, n=need - 1) == B.EB_ERR_WORKSPACE
        assert _sample(**args, ws=None, n=need) == B.EB_ERR_WORKSPACE
        assert _sample(**args, ws=A + 8, n=need) == B.EB_ERR_INVALID


def _logits(dt=B.EB_BF16, rows=4, hidden=64, vocab=100, h=A, w=A, out=A):
    return B.load().eb_lmhead_logits(dt, rows, hidden, vocab, h, w, out, None)


@pytest.mark.parametrize("change,status,word", [
    (dict(dt=B.EB_E4M3), B.EB_ERR_INVALID, "dtype"),
    (dict(rows=-1), B.EB_ERR_INVALID, "n_rows"),
    (dict(hidden=0), B.EB_ERR_INVALID, "hidden"),
    (dict(vocab=0), B.EB_ERR_INVALID, "vocab"),
    (dict(hidden=96), B.EB_ERR_UNSUPPORTED, "hidden"),
    (dict(h=None), B.EB_ERR_INVALID, "NULL"),
    (dict(w=None), B.EB_ERR_INVALID, "NULL"),
    (dict(out=None), B.EB_ERR_INVALID, "NULL"),
    (dict(w=A + 2), B.EB_ERR_INVALID, "aligned"),
    (dict(dt=B.EB_F32, rows=65535 * 32 + 1), B.EB_ERR_UNSUPPORTED, "rows"),
])
def test_logits_refuse(change, status, word):
    assert _logits(**change) == status
    assert word in B.eb_last_error()


POOL = dict(n_pages=8, page_size=16, max_pages=4, page_table=A, free_pages=A, state=A, state_out=A)
ASSIGN = dict(batch=2, n_rows=4, cached=A, new_rows=A, done=None, shared=None, cu_block=A,
              cu_prefix=A, pos=A, slot=None, shorted=None)


def _assign(**change):
    pool = B.eb_page_pool(*[change.get(k, v) for k, v in POOL.items()])
    return B.load().eb_kv_assign(ctypes.byref(pool),
                                 *[change.get(k, v) for k, v in ASSIGN.items()], None)


@pytest.mark.parametrize("change,status,word", [
    (dict(batch=0), B.EB_ERR_INVALID, "batch"),
    (dict(n_rows=-1), B.EB_ERR_INVALID, "n_rows"),
    (dict(n_pages=0), B.EB_ERR_INVALID, "n_pages"),
    (dict(max_pages=0), B.EB_ERR_INVALID, "max_pages"),
    (dict(page_size=0), B.EB_ERR_INVALID, "page_size"),
    (dict(page_size=48), B.EB_ERR_UNSUPPORTED, "page_size"),
    (dict(page_size=512), B.EB_ERR_UNSUPPORTED, "page_size"),
    *[(dict([(k, None)]), B.EB_ERR_INVALID, "NULL") for k in
      ("page_table", "free_pages", "state", "state_out", "cached", "new_rows", "cu_block",
       "cu_prefix", "pos")],
])
def test_assign_refuses(change, status, word):
    assert _assign(**change) == status
    assert word in B.eb_last_error()


@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are never read without a GPU")
@pytest.mark.parametrize("rows", [1, 1024, 1025, (1 << 21) + 1, (1 << 31) - 1024, (1 << 31) - 1])
def test_assign_launch_shapes(rows):
    """Up to the largest number of rows the launch's shape is formed without overflow (which the
    build with sanitizers reports); here the launch itself finds no device."""
    assert _assign(n_rows=rows) == B.EB_ERR_HIP


def test_null_descriptors():
    lib = B.load()
    assert lib.eb_kv_assign(None, 2, 4, A, A, None, None, A, A, A, None, None, None) == \
        B.EB_ERR_INVALID
    assert lib.eb_sample(B.EB_F32, None, 100, 100, A, A, None, A, None, None, None, 0, None) == \
        B.EB_ERR_INVALID


def test_binding_takes_device_tensors_only():
    z = torch.zeros(2, 10)
    r = B.Ragged(1, 2, 2, 0, 0, torch.zeros(2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError, match="device tensor"):
        B.eb_sample(r, z, torch.zeros(2), torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError, match="device tensor"):
        B.eb_lmhead_logits(z, z, z)
    with pytest.raises(ValueError, match="device tensor"):
        B.PagePool(torch.zeros(3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError, match="n_pages"):
        B.PagePool(torch.zeros(0, dtype=torch.int32), torch.zeros(2, dtype=torch.int32))
    with pytest.raises(TypeError):
        B.eb_kv_assign(None, None, z, z, z, z, z)
