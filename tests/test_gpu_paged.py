"""Paged key/value cache on the GPU: rows into pages and back, byte for byte, and the attention over
them, against the fp64 oracle."""
import numpy as np
import pytest
import torch

from oracle import paged
from paper_2609_16450_amd import binding
from paper_2609_16450_amd import (EbError, PagedKV, Ragged, eb_block_attn, eb_block_attn_paged,
                                  eb_block_attn_paged_workspace, eb_decode_step, eb_kv_read,
                                  eb_kv_write, EB_BF16, StepBuffers)

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}


def _cu(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


def _f64(t):
    return t.double().cpu().numpy()


class Cache:
    """A pool whose every byte is garbage (NaN, scales of 2^128), pages handed out in no order, and
    its oracle copy.  spare: pages that no sequence owns."""

    def __init__(self, spans, hkv, page, d, cache, seed, spare=3):
        rng = np.random.default_rng(seed)
        need = [-(-n // page) for n in spans]
        n_pages = sum(need) + spare
        order = rng.permutation(n_pages)
        # entries behind a sequence's pages hold no page number at all
        self.table = np.full((len(spans), max(max(need), 1)), 2 ** 30, np.int32)
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
        self.kv = PagedKV.empty(n_pages, hkv, page, d, torch.from_numpy(self.table).cuda(),
                                TYPES[cache])
        self.e4m3 = cache == "e4m3"
        for t in (self.kv.k, self.kv.v, self.kv.k_scale, self.kv.v_scale):
            if t is not None:
                t.view(torch.uint8).fill_(0xFF)

    def values(self, which):
        """[n_pages, hkv, page, d] in 64 bits."""
        pool = getattr(self.kv, which)
        if not self.e4m3:
            return _f64(pool)
        return paged.dequantise(pool.view(torch.uint8).cpu().numpy(),
                                getattr(self.kv, which + "_scale").cpu().numpy())

    def fill(self, spans, rng, size=1.0):
        """N(0, size^2) values in the first spans[b] positions, set from the host; large caches
        repeat 9973 rows."""
        for which in "kv":
            pool = getattr(self.kv, which)
            n, hkv, page, d = pool.shape
            b_of = np.repeat(np.arange(len(spans)), spans)
            p_of = np.concatenate([np.arange(s) for s in spans] or [[]]).astype(int)
            if not len(b_of):
                continue
            pg, slot = self.table[b_of, p_of // page].astype(np.int64), p_of % page
            rows = rng.standard_normal((min(len(b_of), 9973), hkv, d)) * size
            again = torch.from_numpy(np.arange(len(b_of)) % len(rows)).cuda()
            at = (torch.from_numpy(pg).cuda(), slice(None), torch.from_numpy(slot).cuda())
            if self.e4m3:
                codes, s = paged.quantise(rows)
                pool.view(torch.uint8)[at] = torch.from_numpy(codes).cuda()[again]
                getattr(self.kv, which + "_scale")[at] = torch.from_numpy(s).cuda()[again]
            else:
                pool[at] = torch.from_numpy(rows).to(pool.dtype).cuda()[again]


def _special_rows(rows):
    """Rows where quantising can go wrong, over the first rows of x [T, hkv, d]."""
    x = rows.copy()
    d = x.shape[-1]
    ties = np.resize(np.concatenate([[1.75], 1 + np.arange(0.5, 8) / 8]), d)     # half way: 4 bits
    odd = [np.zeros(d), np.resize([-0.0, 1.0], d), np.resize([np.inf, 2.0, -np.inf, np.nan], d),
           np.full(d, np.nan), ties, np.resize([448.0, 448.1, 1e-3], d), np.resize([1e-38, 3e-39], d),
           np.resize([3.38e38, 1.0], d), np.resize([448 * 2.0 ** -100, 2.0 ** -110], d),
           np.resize([2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -11, 448.0], d)]
    for i, o in enumerate(odd[:len(x)]):
        x[i] = o
    return x


# One row, one block short of a page, several sequences with empty ones among them and pages that
# end inside a block; rows at positions of their own, some left out.
WRITES = [([1], [0]), ([1], [15]), ([37], [5]), ([0, 40, 0, 1, 300], [3, 0, 70, 255, 17]),
          ([3] * 70, list(range(70)))]


@pytest.mark.parametrize("head_dim,hkv", [(128, 3), (64, 1)])
@pytest.mark.parametrize("dtype,cache", [("f32", "f32"), ("bf16", "bf16"), ("f32", "e4m3"),
                                         ("bf16", "e4m3")])
@pytest.mark.parametrize("page", [16, 256])
@pytest.mark.parametrize("scatter", [False, True])
@pytest.mark.parametrize("blocks,cached", WRITES)
def test_write(blocks, cached, scatter, page, dtype, cache, head_dim, hkv):
    print(f"write {len(blocks)} {scatter} {page} {dtype} {cache} D={head_dim}", flush=True)
    rng = np.random.default_rng([len(blocks), page, head_dim, scatter])
    T = sum(blocks)
    spans = [c + 2 * n for n, c in zip(blocks, cached)]
    c = Cache(spans, hkv, page, head_dim, cache, 1)
    rows = [torch.from_numpy(_special_rows(rng.standard_normal((T, hkv, head_dim)))).to(
        TYPES[dtype]) for _ in "kv"]
    pos = None
    if scatter:
        pos = np.concatenate([p + rng.permutation(2 * n)[:n] for n, p in zip(blocks, cached)])
        pos = np.where(rng.random(T) < 0.3, -1 - rng.integers(0, 2 ** 31 - 1, T), pos).astype(np.int32)
    want = {}
    for which, x in zip("kv", rows):
        pool = getattr(c.kv, which)
        if cache == "e4m3":
            codes, s = paged.quantise(_f64(x))
            for name, t, new in ((which, pool.view(torch.uint8), codes),
                                 (which + "_scale", getattr(c.kv, which + "_scale"), s)):
                want[name] = t.cpu().numpy().copy()
                paged.kv_write(want[name], c.table, new, _cu(blocks), cached, pos)
        else:
            bits = torch.int32 if dtype == "f32" else torch.int16
            want[which] = pool.view(bits).cpu().numpy().copy()
            paged.kv_write(want[which], c.table, x.view(bits).numpy(), _cu(blocks), cached, pos)
    eb_kv_write(Ragged.from_lengths(blocks, cached), c.kv, *(x.cuda() for x in rows),
                pos=None if pos is None else torch.from_numpy(pos).cuda())
    for name, w in want.items():
        t = getattr(c.kv, name)
        t = (t if name.endswith("scale") else t.view(
            {"f32": torch.int32, "bf16": torch.int16, "e4m3": torch.uint8}[cache]))
        got = t.cpu().numpy()
        if cache == "e4m3" and not name.endswith("scale"):    # the sign of a NaN is not defined
            got = np.where(got & 0x7F == 0x7F, 0x7F, got)
            w = np.where(w & 0x7F == 0x7F, 0x7F, w)
        np.testing.assert_array_equal(got, w, err_msg=name)


@pytest.mark.parametrize("cache,dtype", [("f32", "f32"), ("bf16", "bf16"), ("e4m3", "f32"),
                                         ("e4m3", "bf16")])
def test_rows_without_a_page(cache, dtype):
    """Page numbers below 0 and from n_pages on, and positions past the table: rows written there
    are dropped, rows read from there are zeros."""
    rng = np.random.default_rng(7)
    c = Cache([64, 64], 2, 16, 128, cache, 2)
    c.fill([64, 64], rng)
    bad = c.table.copy()
    bad[0, 1], bad[0, 2], bad[1, 3] = -1, c.kv.n_pages, -2 ** 31
    c.kv.page_table.copy_(torch.from_numpy(bad))
    before = {n: getattr(c.kv, n).view(torch.uint8).cpu().numpy().copy() for n in "kv"}
    r = Ragged.from_lengths([0, 0], [64, 61])
    out = [torch.full((125, 2, 128), 7.0, dtype=TYPES[dtype], device="cuda") for _ in "kv"]
    eb_kv_read(r, c.kv, *out)
    for which, o in zip("kv", out):
        np.testing.assert_array_equal(_f64(o), paged.kv_read(c.values(which), bad, [64, 61]))
    rows = torch.ones(4, 2, 128, dtype=TYPES[dtype], device="cuda")
    pos = torch.tensor([20, 40, 50, 64], dtype=torch.int32, device="cuda")   # 64: past the table
    eb_kv_write(Ragged.from_lengths([2, 2], [0, 0]), c.kv, rows, rows, pos=pos)
    for n, w in before.items():
        np.testing.assert_array_equal(getattr(c.kv, n).view(torch.uint8).cpu().numpy(), w)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("byte", [0, 255])
def test_no_page_at_all(byte, head_dim, dtype):
    """Rows that have no page read as zeros whatever the pool's first row and its scale hold."""
    table = torch.full((1, 2), -1, dtype=torch.int32, device="cuda")
    kv = PagedKV.empty(1, 2, 16, head_dim, table, TYPES["e4m3"])
    for t in (kv.k, kv.v):
        t.view(torch.uint8).fill_(0x38)
    for t in (kv.k_scale, kv.v_scale):
        t.fill_(byte)
    out = [torch.full((20, 2, head_dim), 7.0, dtype=TYPES[dtype], device="cuda") for _ in "kv"]
    eb_kv_read(Ragged.from_lengths([0], [20]), kv, *out)
    for o in out:
        assert torch.equal(o, torch.zeros_like(o))
    # the attention: 20 keys of zeros and the block's own, of ones
    for rows in (1, 12, 100):
        one = torch.ones(rows, 2, head_dim, dtype=TYPES[dtype], device="cuda")
        q = torch.zeros(rows, 4, head_dim, dtype=TYPES[dtype], device="cuda")
        got = torch.empty_like(q)
        eb_block_attn_paged(Ragged.from_lengths([rows], [20]), kv, q, one, one, got)
        want = rows / (rows + 20)
        # weights of exactly 1, their sum exact: the division's and the output's rounding
        tol = want * (2.0 ** -8 + 2.0 ** -20 if dtype == "bf16" else 2.0 ** -20)
        assert (got.double() - want).abs().max().item() <= tol


@pytest.mark.parametrize("head_dim,hkv", [(128, 2), (64, 5)])
@pytest.mark.parametrize("cache,dtype", [("f32", "f32"), ("bf16", "bf16"), ("e4m3", "f32"),
                                         ("e4m3", "bf16")])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("cached", [[1], [0, 33, 0, 16, 200], [5] * 130, [1000]])
def test_read(cached, page, cache, dtype, head_dim, hkv):
    print(f"read {len(cached)} {page} {cache} {dtype} D={head_dim}", flush=True)
    c = Cache(cached, hkv, page, head_dim, cache, 3)
    c.fill(cached, np.random.default_rng(len(cached)))
    S = sum(cached)
    # the rows behind the last one stay as they are
    out = [torch.full((S + 2, hkv, head_dim), 7.0, dtype=TYPES[dtype], device="cuda") for _ in "kv"]
    eb_kv_read(Ragged.from_lengths([0] * len(cached), cached), c.kv, *(o[:S] for o in out))
    for which, o in zip("kv", out):
        np.testing.assert_array_equal(_f64(o[:S]), paged.kv_read(c.values(which), c.table, cached))
        assert (o[S:] == 7.0).all()


def test_every_scale_and_code():
    """All 256 codes under scales from 2^-117 to 2^119 (all of whose values are ordinary numbers)
    read back exactly, in fp32 and bf16."""
    table = torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    kv = PagedKV.empty(1, 2, 256, 128, table, torch.float8_e4m3fn)
    codes = torch.arange(256, dtype=torch.uint8).view(2, 1, 128).expand(2, 256, 128)
    scale = torch.arange(10, 10 + 237).repeat(2)[:256].to(torch.uint8).expand(2, 256)
    for pool, s in ((kv.k, kv.k_scale), (kv.v, kv.v_scale)):
        pool.view(torch.uint8)[0].copy_(codes)
        s[0].copy_(scale)
    want = paged.dequantise(codes.numpy(), scale.numpy()).transpose(1, 0, 2)
    for dtype in (torch.float32, torch.bfloat16):
        out = [torch.zeros(256, 2, 128, dtype=dtype, device="cuda") for _ in "kv"]
        eb_kv_read(Ragged.from_lengths([0], [256]), kv, *out)
        for o in out:
            np.testing.assert_array_equal(_f64(o), want)


# --------------------------------------------------------------------------------------------
# attention
# --------------------------------------------------------------------------------------------
def _attention(blocks, cached, page, cache, dtype, group, head_dim, hkv=2, size=1.0, seed=0,
               scale=None, stream=None):
    """Output of eb_block_attn_paged, the oracle's, and the oracle's with |v|."""
    rng = np.random.default_rng([len(blocks), sum(blocks), page, head_dim, group, seed])
    c = Cache(cached, hkv, page, head_dim, cache, seed)
    c.fill(cached, rng, size)
    T = sum(blocks)
    q, k, v = (torch.from_numpy(rng.standard_normal((T, h, head_dim)) * size).to(TYPES[dtype])
               for h in (hkv * group, hkv, hkv))
    # rows behind the last one stay as they are
    out = torch.full((T + 1, hkv * group, head_dim), 7.0, dtype=TYPES[dtype], device="cuda")
    r, x = Ragged.from_lengths(blocks, cached), (q.cuda(), k.cuda(), v.cuda())
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())
    eb_block_attn_paged(r, c.kv, *x, out[:T], scale=scale, stream=stream)
    if stream is not None:
        torch.cuda.current_stream().wait_stream(stream)
    assert (out[T:] == 7.0).all()
    kc, vc = c.values("k"), c.values("v")
    args = dict(table=c.table, cu_block=_cu(blocks), cached=cached, hq=hkv * group, hkv=hkv,
                scale=scale)
    ref = paged.paged_attention(_f64(q), _f64(k), _f64(v), kc, vc, **args)
    mag = paged.paged_attention(_f64(q), _f64(k), np.abs(_f64(v)), kc, np.abs(vc), **args)
    return _f64(out[:T]), ref, mag


def _close(got, ref, mag, dtype):
    if dtype == "f32":
        # scores of size |q||k| / sqrt(d) < 16 off by some 128 2^-24 16 / sqrt(128): 1e-5 in a weight
        np.testing.assert_allclose(got, ref, rtol=2e-5, atol=2e-5)
        return
    # A weight is rounded to bf16 (2^-8 of itself) and divided by a sum of weights, rounded or not
    # (2^-8 again): at most 2^-7 sum_j p_j |v_j|; the output is rounded to bf16 (2^-8 of itself).
    # Scores are exact products summed in fp32, 128 2^-24 sum_d |q_d k_d| scale < 128 2^-24 16 =
    # 1.2e-4 off, as much in a weight and twice that in a quotient: within the factor of 1.1.
    bound = 1.1 * (2.0 ** -7 * mag + 2.0 ** -8 * np.abs(ref)) + 1e-30
    assert np.isfinite(got).all()
    worst = (np.abs(got - ref) / bound).max(initial=0.0)
    assert worst <= 1.0, worst


COMBOS = [("f32", "f32"), ("e4m3", "f32"), ("bf16", "bf16"), ("e4m3", "bf16")]

# Single tokens; one cached row; stages of 16, 64 and 128 keys that end at, before and after the
# cached rows; query rows of a K/V head around 16, 32, 64 and 128; empty blocks and caches.
SHAPES = [([1], [0]), ([1], [1]), ([1], [16]), ([1], [129]), ([1], [700]),
          ([1, 1, 1, 1], [63, 64, 65, 0]), ([5, 0, 6], [3, 7, 300]), ([16, 11], [128, 127]),
          ([32, 1, 33], [0, 95, 250]), ([64], [31]), ([65, 2], [64, 1000]), ([130, 127], [17, 513])]


@pytest.mark.parametrize("head_dim,page", [(128, 64), (64, 16)])
@pytest.mark.parametrize("cache,dtype", COMBOS)
@pytest.mark.parametrize("group", [1, 3])
@pytest.mark.parametrize("blocks,cached", SHAPES)
def test_attention(blocks, cached, group, cache, dtype, head_dim, page):
    print(f"attn {blocks} {cached} G={group} {cache} {dtype} D={head_dim} page={page}", flush=True)
    _close(*_attention(blocks, cached, page, cache, dtype, group, head_dim), dtype)


@pytest.mark.parametrize("page", [16, 32, 128, 256])
@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("cache,dtype", COMBOS)
@pytest.mark.parametrize("blocks,cached,group", [([1, 1, 1], [1000, 17, 257], 7),
                                                 ([40, 90], [321, 640], 4)])
def test_attention_page_sizes(blocks, cached, group, cache, dtype, head_dim, page):
    print(f"attn {blocks} G={group} {cache} {dtype} D={head_dim} page={page}", flush=True)
    _close(*_attention(blocks, cached, page, cache, dtype, group, head_dim), dtype)


# Many sequences of one token, of very different lengths; many of a few rows; one long context (key
# ranges over many workgroups) for a token, a block and a chunk.
@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("cache,dtype", COMBOS)
@pytest.mark.parametrize("blocks,cached,group,hkv", [
    ([1] * 150, [(37 * i) % 500 for i in range(150)], 2, 1),
    ([3, 0, 2] * 30, [(91 * i) % 300 for i in range(90)], 7, 2),
    ([1], [9001], 7, 2), ([20, 1], [5000, 1], 1, 3), ([300], [2500], 2, 1)])
def test_attention_batches(blocks, cached, group, hkv, cache, dtype, head_dim):
    print(f"attn {len(blocks)} {max(cached)} G={group} {cache} {dtype} D={head_dim}", flush=True)
    _close(*_attention(blocks, cached, 32, cache, dtype, group, head_dim, hkv=hkv), dtype)


# Every key counts exactly once, however the keys are cut: with queries of zeros all weights are 1,
# and with values of 1 in column (position + 7 head) % D of a window of positions, 0 elsewhere, a
# column is a count of at most 32 keys over their number.  fp32 sums of whole numbers are exact; the
# division and the output's rounding are off by at most 2^-8 + 2^-20 of the result, a lost or doubled
# key by 2^-5.
COUNTS = [
    # few query rows: single sequences over many parts, ragged ones, sequences that stay whole
    ([1], [9001], 2, 7), ([20, 1], [5000, 1], 3, 1),
    ([1] * 64, [(509 * i) % 8192 for i in range(64)], 2, 3),
    ([3, 0, 2] * 30, [(91 * i) % 300 for i in range(90)], 2, 7), ([32, 16], [2100, 4000], 2, 1),
    # more: ranges by the workgroups, the last round cut, the host's ranges, counted items
    ([300], [2500], 1, 2), ([70], [5000], 1, 1),
    ([70, 0, 66, 90, 65], [5000, 77, 10, 700, 0], 2, 3),
    ([33 + i % 9 for i in range(40)], [1030 - 26 * i for i in range(40)], 16, 1),
    ([34 + i % 3 * (i % 7 > 0) - 34 * (i == 9) for i in range(70)],
     [(53 * i) % 900 for i in range(70)], 1, 2),
    ([40 - i % 6 for i in range(64)], [(53 * i) % 900 for i in range(64)], 1, 1),
    ([i % 4 for i in range(150)] + [500] + [2] * 130, [(91 * i) % 400 for i in range(281)], 4, 3),
    # 8 bits: two launches; and more blocks with items of their own than are cut into ranges
    ([1, 0, 3, 9] * 20 + [150], [(191 * i) % 3000 + 700 for i in range(81)], 4, 3),
    ([17, 1, 0, 1] * 100 + [70], [(191 * i) % 900 + 600 for i in range(401)], 4, 1),
    ([70] + [0, 1, 17, 1] * 100, [(191 * i) % 900 + 600 for i in range(401)], 4, 1)]


@pytest.mark.parametrize("head_dim,page", [(64, 64), (128, 16)])
@pytest.mark.parametrize("cache,dtype", [("bf16", "bf16"), ("e4m3", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("blocks,cached,hkv,group", COUNTS)
def test_every_key_counts_once(blocks, cached, hkv, group, cache, dtype, head_dim, page):
    print(f"count {len(blocks)} {max(cached)} G={group} {cache} D={head_dim}", flush=True)
    c = Cache(cached, hkv, page, head_dim, cache, 14)
    dt, S, T = TYPES[dtype], sum(cached), sum(blocks)
    g = torch.Generator(device="cuda").manual_seed(len(blocks))

    def places(lens, first):
        """Sequence and position of packed rows that begin at first[b] of their sequences."""
        lens, first = (torch.tensor(x, device="cuda") for x in (lens, first))
        seq = torch.repeat_interleave(torch.arange(len(lens), device="cuda"), lens)
        at = torch.arange(len(seq), device="cuda") - (torch.cumsum(lens, 0) - lens)[seq]
        return seq, at + first[seq]

    seq_s, pos_s = places(cached, [0] * len(cached))
    seq_t, pos_t = places(blocks, cached)
    head = torch.arange(hkv, device="cuda")

    def values(pos, lo, hi):
        col = ((pos[:, None] + 7 * head) % head_dim)[..., None]
        one = ((pos >= lo) & (pos < hi)).float()[:, None, None].expand(-1, hkv, 1)
        return torch.zeros(len(pos), hkv, head_dim, device="cuda").scatter_(2, col, one)

    k_s, k_t = (torch.randn(n, hkv, head_dim, generator=g, device="cuda").to(dt) for n in (S, T))
    q = torch.zeros(T, hkv * group, head_dim, dtype=dt, device="cuda")
    keys = (torch.tensor(blocks, device="cuda") + torch.tensor(cached, device="cuda")).double()
    r, window = Ragged.from_lengths(blocks, cached), 32 * head_dim
    for lo in range(0, int(keys.max()), window):
        v_s, v_t = values(pos_s, lo, lo + window), values(pos_t, lo, lo + window)
        eb_kv_write(Ragged.from_lengths(cached, [0] * len(cached)), c.kv, k_s, v_s.to(dt))
        out = torch.full_like(q, 7.0)
        eb_block_attn_paged(r, c.kv, q, k_t, v_t.to(dt), out)
        want = torch.zeros(len(blocks), hkv, head_dim, dtype=torch.float64, device="cuda")
        want.index_add_(0, seq_s, v_s.double()).index_add_(0, seq_t, v_t.double())
        assert want.max() <= 32
        want = (want / keys.clamp(min=1)[:, None, None])[seq_t].repeat_interleave(group, dim=1)
        tol = 2.0 ** -20 + (2.0 ** -8 if dtype == "bf16" else 0.0)
        bad = (out.double() - want).abs() > tol * want
        assert not bad.any(), (lo, torch.nonzero(bad)[:4].tolist())


# More sequences than one workgroup looks through (2048), single tokens and small blocks, some empty.
@pytest.mark.parametrize("cache,dtype", COMBOS)
def test_attention_many_sequences(cache, dtype):
    print(f"many {cache} {dtype}", flush=True)
    blocks = [(i % 5) % 4 for i in range(2300)]
    cached = [(i * 13) % 40 + (500 if i == 77 else 0) for i in range(2300)]
    _close(*_attention(blocks, cached, 16, cache, dtype, 2, 64, hkv=1), dtype)


# Few query rows per K/V head: probabilities to 2^-16, so that a result is off by its own rounding to
# bf16 (2^-8 of itself) and, as in _close, scores that are 1.2e-4 off (twice that in a quotient) and
# twice 2^-16 of sum_j p_j |v_j|.  Few keys, where one probability counts most.
@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("cache,blocks,cached,group", [
    *((cache, *shape) for cache in ("bf16", "e4m3") for shape in (
        ([1] * 100, [2 + i for i in range(100)], 7), ([2] * 50, list(range(50)), 8),
        ([1, 2], [3000, 5], 4))),
    ("bf16", [20, 32], [10, 30], 1)])
def test_few_rows_hold_probabilities(blocks, cached, group, cache, head_dim):
    got, ref, mag = _attention(blocks, cached, 16, cache, "bf16", group, head_dim)
    bound = 2.0 ** -8 * np.abs(ref) + 1.1 * (2.4e-4 + 2.0 ** -15) * mag
    assert (np.abs(got - ref) <= bound).all(), (np.abs(got - ref) / bound).max()


# The plans of the tile kernel: more sequences than a wave has lanes, cut by the host (70 of one tile);
# so many items that sequences stay whole, over more pages of 16 rows than a wave holds numbers of
# (64); lengths so different that only the longest are cut; one long block, whose tiles share keys.
@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("blocks,cached,hkv,group", [
    ([34 + i % 3 * (i % 7 > 0) - 34 * (i == 9) for i in range(70)],
     [(53 * i) % 900 for i in range(70)], 1, 2),
    ([33 + i % 9 for i in range(58)], [1030 + 3 * i for i in range(58)], 16, 1),
    # somewhat more items than workgroups that run at a time: the last ones cut, into more ranges
    # than the shortest has stages; row tiles of one block on both sides
    ([33 + i % 9 for i in range(40)], [1030 - 26 * i for i in range(40)], 16, 1),
    ([34] * 33, [640 + 11 * i for i in range(33)], 16, 1),
    ([300, 0, 200, 60], [700, 9, 300, 1500], 4, 32),
    ([70, 0, 66, 90, 65], [5000, 77, 10, 700, 0], 2, 3),
    ([777], [1500], 1, 2)])
def test_attention_plans(blocks, cached, hkv, group, cache, head_dim):
    print(f"plans {len(blocks)} {max(cached)} G={group} {cache} D={head_dim}", flush=True)
    _close(*_attention(blocks, cached, 16, cache, "bf16", group, head_dim, hkv=hkv), "bf16")


# Long blocks among many short ones: key ranges of counted items, whole sequences, a batch of more
# than 2048, the long one last, in the middle, and first; and few sequences of many heads.
@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("blocks,cached,hkv,group", [
    ([1] * 80 + [300], [(53 * i) % 900 for i in range(81)], 1, 2),
    ([i % 4 for i in range(150)] + [500] + [2] * 130, [(91 * i) % 400 for i in range(281)], 4, 3),
    ([200, 70] + [1] * 2300, [40, 600] + [(7 * i) % 50 for i in range(2300)], 1, 2),
    ([600] + [1] * 39, [1000] + [9 * i for i in range(39)], 32, 1),
    # 8 bits: the short ones (of up to 16 and 32 rows per K/V head, some of more, some empty) in a
    # launch of their own, of equal parts and whole
    ([1, 0, 3, 9] * 20 + [150], [(191 * i) % 3000 + 700 for i in range(81)], 4, 3),
    ([0, 5, 7, 2, 12] * 10 + [90], [(83 * i) % 4000 + 900 for i in range(51)], 3, 3),
    ([1] * 2100 + [70], [(7 * i) % 90 + 80 for i in range(2101)], 2, 2)])
def test_attention_mixed(blocks, cached, hkv, group, cache, head_dim):
    print(f"mixed {len(blocks)} {max(cached)} G={group} {cache} D={head_dim}", flush=True)
    _close(*_attention(blocks, cached, 16, cache, "bf16", group, head_dim, hkv=hkv), "bf16")


# Rows of a K/V head at the border between the kernels: 32 and 33 over bf16 pages, 64 and 65 over 8
# bits; 16 and 17 query rows per workgroup; sequences at the border of staying whole.
@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
@pytest.mark.parametrize("rows", [16, 17, 32, 33, 64, 65])
@pytest.mark.parametrize("cached", [[640, 5], [768, 3], [2000, 900]])
def test_attention_borders(rows, cached, cache):
    print(f"borders {rows} {cached} {cache}", flush=True)
    _close(*_attention([rows, rows // 2], cached, 64, cache, "bf16", 1, 128, hkv=3), "bf16")


@pytest.mark.parametrize("cache,dtype", COMBOS)
@pytest.mark.parametrize("blocks,cached,group", [([1, 1], [3000, 40], 2), ([50, 90], [900, 2500], 2),
                                                 ([20], [4000], 1)])
def test_workspace_is_enough(blocks, cached, group, cache, dtype):
    _guarded(blocks, cached, group, cache, dtype)


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_workspace_of_many_sequences(cache):
    _guarded([1] * 80 + [300], [10 * i for i in range(81)], 2, cache, "bf16")


def test_workspace_of_many_cut_sequences():
    """More blocks with items of their own than are cut into ranges; few keys of one block, whose
    workspace is that of its items."""
    _guarded([17, 1, 0, 1] * 100 + [70], [(191 * i) % 900 + 600 for i in range(401)], 1, "e4m3",
             "bf16")
    _guarded([33], [600], 1, "bf16", "bf16")


def _guarded(blocks, cached, group, cache, dtype):
    """Nothing behind the bytes that the query asks for is written, and one byte less is refused."""
    rng = np.random.default_rng(3)
    c = Cache(cached, 2, 32, 128, cache, 4)
    c.fill(cached, rng)
    r = Ragged.from_lengths(blocks, cached)
    dt = TYPES[dtype]
    q, k, v = (torch.from_numpy(rng.standard_normal((sum(blocks), h, 128))).to(dt).cuda()
               for h in (2 * group, 2, 2))
    need = eb_block_attn_paged_workspace(0 if dtype == "f32" else EB_BF16, r, c.kv, 2 * group)
    assert need > 0
    ws = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    out = torch.zeros_like(q)
    eb_block_attn_paged(r, c.kv, q, k, v, out, ws=ws[:need])
    assert (ws[need:] == 0xA5).all()
    with pytest.raises(EbError, match="WORKSPACE"):
        eb_block_attn_paged(r, c.kv, q, k, v, out, ws=ws[:need - 1])


@pytest.mark.parametrize("cache,dtype", COMBOS)
@pytest.mark.parametrize("blocks,cached", [([1], [300]), ([40], [200]), ([140], [90])])
def test_attention_scale(blocks, cached, cache, dtype):
    print(f"scale {blocks} {cache} {dtype}", flush=True)
    _close(*_attention(blocks, cached, 16, cache, dtype, 2, 128, scale=0.021), dtype)


def _handmade(cache, dtype, blocks, cached, head_dim, k, v, k_new, v_new, q, page=16):
    """Attention of given rows (arrays [n, 1, d]); the cache is written with eb_kv_write."""
    c = Cache([cached], 1, page, head_dim, cache, 5)
    dt = TYPES[dtype]

    def dev(x):
        return torch.from_numpy(np.asarray(x, np.float32)).to(dt).cuda()

    eb_kv_write(Ragged.from_lengths([cached], [0]), c.kv, dev(k), dev(v))
    out = torch.zeros(blocks, q.shape[1], head_dim, dtype=dt, device="cuda")
    eb_block_attn_paged(Ragged.from_lengths([blocks], [cached]), c.kv, dev(q), dev(k_new),
                        dev(v_new), out)
    return _f64(out)


@pytest.mark.parametrize("cache,dtype", COMBOS)
@pytest.mark.parametrize("blocks", [1, 20, 150])
def test_attention_infinities(blocks, cache, dtype):
    """Keys with scores of -inf weigh nothing, whole stages of them and the first ones among them;
    an infinite or NaN value reaches the rows that see it, and only its own column."""
    d, n = 128, 300
    q = np.zeros((blocks, 1, d))
    q[:, 0, 0] = 1e19
    k, v = np.zeros((n, 1, d)), np.ones((n, 1, d))
    k[:150, 0, 0] = -1e25           # scores of -1e44 / sqrt(128): -inf in fp32
    v[:150] = 5.0
    k_new, v_new = np.zeros((blocks, 1, d)), np.ones((blocks, 1, d))
    got = _handmade(cache, dtype, blocks, n, d, k, v, k_new, v_new, q)
    np.testing.assert_array_equal(got, 1.0)
    v_new[-1, 0, 7] = np.inf
    v[-1, 0, 9] = np.nan
    got = _handmade(cache, dtype, blocks, n, d, k, v, k_new, v_new, q)
    assert (got[:, 0, 7] == np.inf).all() and np.isnan(got[:, 0, 9]).all()
    others = np.delete(got, [7, 9], axis=-1)
    np.testing.assert_array_equal(others, 1.0)


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("cache,dtype", COMBOS)
@pytest.mark.parametrize("blocks,n", [(1, 3000), (20, 2500), (40, 900), (150, 1500), (150, 70)])
def test_attention_infinities_without_weight(blocks, n, cache, dtype, head_dim):
    """One key takes all of the softmax's weight in 32 bits; infinities (in 8 bits NaN) at keys
    before and behind it, in its stage, in others and in other key ranges, still leave their columns
    infinite or NaN, as 0 times infinity is, and no other column."""
    print(f"weightless {blocks} {n} {cache} {dtype} D={head_dim}", flush=True)
    d = head_dim
    at = np.unique(np.linspace(0, n + blocks - 1, d // 2).astype(int))
    for big in (1, n // 2, n - 1, n + blocks - 1):
        q, k, v = np.zeros((blocks, 1, d)), np.zeros((n + blocks, 1, d)), np.ones((n + blocks, 1, d))
        q[:, 0, 0] = 64.0
        k[big, 0, 0] = 64.0           # a score of 362 or more; the others are 0 and expf(-362) is 0
        v[at, 0, np.arange(len(at))] = np.inf
        got = _handmade(cache, dtype, blocks, n, d, k[:n], v[:n], k[n:], v[n:], q)
        assert not np.isfinite(got[..., :len(at)]).any(), big
        np.testing.assert_array_equal(got[..., len(at):], 1.0)


@pytest.mark.parametrize("cache,dtype", COMBOS)
@pytest.mark.parametrize("blocks,cached,group", [([1, 1], [300, 20], 2), ([30, 60], [100, 700], 3)])
def test_attention_rising_scores(blocks, cached, group, cache, dtype):
    """Scores that rise along the keys by far more than a weight's range (the running maximum moves
    again and again)."""
    rng = np.random.default_rng(11)
    c = Cache(cached, 1, 16, 128, cache, 6)
    for b, n in enumerate(cached):
        k = rng.standard_normal((n, 1, 128)) * np.linspace(0.1, 6, n)[:, None, None]
        v = rng.standard_normal((n, 1, 128))
        one = PagedKV(c.kv.k, c.kv.v, c.kv.page_table[b:b + 1].contiguous(), c.kv.k_scale,
                      c.kv.v_scale)
        eb_kv_write(Ragged.from_lengths([n], [0]), one,
                    *(torch.from_numpy(x).to(TYPES[dtype]).cuda() for x in (k, v)))
    T = sum(blocks)
    q, k, v = (torch.from_numpy(rng.standard_normal((T, h, 128)) * 2).to(TYPES[dtype])
               for h in (group, 1, 1))
    out = torch.zeros(T, group, 128, dtype=TYPES[dtype], device="cuda")
    eb_block_attn_paged(Ragged.from_lengths(blocks, cached), c.kv, q.cuda(), k.cuda(), v.cuda(), out)
    args = dict(table=c.table, cu_block=_cu(blocks), cached=cached, hq=group, hkv=1)
    ref = paged.paged_attention(_f64(q), _f64(k), _f64(v), c.values("k"), c.values("v"), **args)
    mag = paged.paged_attention(_f64(q), _f64(k), np.abs(_f64(v)), c.values("k"),
                                np.abs(c.values("v")), **args)
    if dtype == "f32":
        # sum_d |q_d k_d| / sqrt(d) up to 128 * 0.64 * 12 / 11.3 = 87, so a score is off by at most
        # 128 2^-24 87 = 6.6e-4 and a weight by twice that of itself; typically by a tenth
        np.testing.assert_allclose(_f64(out), ref, rtol=0, atol=2 * 6.6e-4 * mag.max())
    else:
        # the same in addition to the roundings to bf16 (_close): 1.4e-3 against 2^-7 = 7.8e-3
        bound = 1.1 * (2.0 ** -7 * mag + 2.0 ** -8 * np.abs(ref)) + 1.4e-3 * mag
        assert (np.abs(_f64(out) - ref) <= bound).all()


def test_long_pool():
    """Pages whose rows lie past 2^32 bytes and 2^31 values of the pool."""
    hkv, page, d, n_pages = 8, 256, 128, 9000
    table = torch.tensor([[8999, 1, 8500]], dtype=torch.int32, device="cuda")
    for cache in ("bf16", "e4m3"):
        kv = PagedKV.empty(n_pages, hkv, page, d, table, TYPES[cache])
        assert kv.k.numel() > 2 ** 31
        g = torch.Generator(device="cuda").manual_seed(3)
        k, v, kb, vb = (torch.randn(n, hkv, d, generator=g, device="cuda", dtype=torch.bfloat16)
                        for n in (700, 700, 40, 40))
        q = torch.randn(40, hkv, d, generator=g, device="cuda", dtype=torch.bfloat16)
        r = Ragged.from_lengths([700], [0])
        eb_kv_write(r, kv, k, v)
        after = Ragged.from_lengths([40], [700])
        back = [torch.zeros_like(k), torch.zeros_like(v)]
        eb_kv_read(after, kv, *back)
        for x, y in zip((k, v), back):
            if cache == "bf16":
                assert torch.equal(x, y)
            else:
                want = paged.dequantise(*paged.quantise(_f64(x)))
                np.testing.assert_array_equal(_f64(y), want)
        out = torch.zeros_like(q)
        eb_block_attn_paged(after, kv, q, kb, vb, out)
        args = (_f64(q), _f64(kb))
        pre = [_f64(y) for y in back]
        ref = paged.block_attention(*args, _f64(vb), *pre, [0, 40], [0, 700], hkv, hkv)
        mag = paged.block_attention(*args, np.abs(_f64(vb)), pre[0], np.abs(pre[1]), [0, 40],
                                    [0, 700], hkv, hkv)
        _close(_f64(out), ref, mag, "bf16")
        del kv


@pytest.mark.parametrize("cache,head_dim", [("e4m3", 128), ("e4m3", 64), ("bf16", 64)])
def test_long_pool_many_rows(cache, head_dim):
    """The same for the kernels of many query rows (the others of them: test_long_pool)."""
    hkv, page, n_pages, rows, cached = 8, 256, 9000 * 128 // head_dim, 100, 700
    table = torch.tensor([[n_pages - 1, 1, n_pages - 500]], dtype=torch.int32, device="cuda")
    kv = PagedKV.empty(n_pages, hkv, page, head_dim, table, TYPES[cache])
    assert kv.k.numel() > 2 ** 31
    g = torch.Generator(device="cuda").manual_seed(4)
    k, v, kb, vb, q = (torch.randn(n, hkv, head_dim, generator=g, device="cuda",
                                   dtype=torch.bfloat16)
                       for n in (cached, cached, rows, rows, rows))
    eb_kv_write(Ragged.from_lengths([cached], [0]), kv, k, v)
    out = torch.zeros_like(q)
    eb_block_attn_paged(Ragged.from_lengths([rows], [cached]), kv, q, kb, vb, out)
    pre = [paged.dequantise(*paged.quantise(_f64(x))) if cache == "e4m3" else _f64(x)
           for x in (k, v)]
    args = ([0, rows], [0, cached], hkv, hkv)
    ref = paged.block_attention(_f64(q), _f64(kb), _f64(vb), *pre, *args)
    mag = paged.block_attention(_f64(q), _f64(kb), np.abs(_f64(vb)), pre[0], np.abs(pre[1]), *args)
    _close(_f64(out), ref, mag, "bf16")


# --------------------------------------------------------------------------------------------
# as they are used
# --------------------------------------------------------------------------------------------
def test_long_line():
    """One context of 2^27 keys among 2047 empty ones: as many stages, counted for every sequence,
    as pass 31 bits.  None of its rows has a page, so all weights are 1 and all values but the
    block's own are zero."""
    keys, batch = 1 << 27, 2048
    table = torch.full((batch, keys // 256), -1, dtype=torch.int32, device="cuda")
    kv = PagedKV.empty(1, 1, 256, 64, table, TYPES["e4m3"])
    for t in (kv.k, kv.v, kv.k_scale, kv.v_scale):
        t.view(torch.uint8).fill_(0xFF)
    r = Ragged.from_lengths([1] * batch, [0] * 1000 + [keys] + [0] * 1047)
    q = torch.zeros(batch, 1, 64, dtype=torch.bfloat16, device="cuda")
    v = torch.from_numpy(np.random.default_rng(0).standard_normal((batch, 1, 64))).bfloat16().cuda()
    out = torch.full_like(q, 7.0)
    eb_block_attn_paged(r, kv, q, q, v, out)
    want = v.double()
    want[1000] /= keys + 1
    # the output's rounding, and some of the sum's and the division's in fp32
    assert ((out.double() - want).abs() <= want.abs() * (2.0 ** -8 + 2.0 ** -18)).all()


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_decoding_run(cache):
    """Blocks decoded one after another: attention over the pages, the block into the pages, and so
    on; a block with uncommitted rows; and the packed cache for the dense attention and the step."""
    rng = np.random.default_rng(12)
    hq, hkv, d, page = 6, 2, 128, 32
    spans = [150, 90]
    c = Cache(spans, hkv, page, d, cache, 8)
    cached = [0, 0]

    def x(n, h):
        return torch.from_numpy(rng.standard_normal((n, h, d))).to(torch.bfloat16).cuda()

    for blocks in ([40, 1], [33, 7], [1, 1], [16, 50]):
        T = sum(blocks)
        q, k, v = x(T, hq), x(T, hkv), x(T, hkv)
        r = Ragged.from_lengths(blocks, cached)
        out, dense = torch.zeros_like(q), torch.zeros_like(q)
        ws = torch.empty(max(1, eb_block_attn_paged_workspace(EB_BF16, r, c.kv, hq)),
                         dtype=torch.uint8, device="cuda")
        eb_block_attn_paged(r, c.kv, q, k, v, out, ws=ws)
        pre = [torch.zeros(sum(cached), hkv, d, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
        eb_kv_read(r, c.kv, *pre)
        eb_block_attn(r, q, k, v, *pre, dense)
        args = (_cu(blocks), _cu(cached), hq, hkv)
        ref = paged.block_attention(_f64(q), _f64(k), _f64(v), *map(_f64, pre), *args)
        mag = paged.block_attention(_f64(q), _f64(k), np.abs(_f64(v)), _f64(pre[0]),
                                    np.abs(_f64(pre[1])), *args)
        _close(_f64(out), ref, mag, "bf16")
        _close(_f64(dense), ref, mag, "bf16")
        # every second row of the first sequence is committed first, then the others
        half = np.concatenate([np.arange(b) + p for b, p in zip(blocks, cached)]).astype(np.int32)
        even = np.where(np.arange(T) % 2 == 0, half, -1)
        odd = np.where(np.arange(T) % 2 == 1, half, -1)
        for pos in (even, odd):
            eb_kv_write(r, c.kv, k, v, pos=torch.from_numpy(pos.astype(np.int32)).cuda())
        cached = [p + b for p, b in zip(cached, blocks)]
    # the whole step on the packed cache
    r = Ragged.from_lengths([5, 9], cached)
    pre = [torch.zeros(sum(cached), hkv, d, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    eb_kv_read(r, c.kv, *pre)
    T, hidden, vocab = 14, 128, 1000
    q, k, v = x(T, hq), x(T, hkv), x(T, hkv)
    h = torch.randn(T, hidden, device="cuda").to(torch.bfloat16)
    w = torch.randn(vocab, hidden, device="cuda").to(torch.bfloat16)
    f, i, u = (dict(device="cuda", dtype=t) for t in (torch.float32, torch.int32, torch.uint8))
    attn = torch.zeros_like(q)
    step = StepBuffers(r, q, k, v, *pre, attn, h, w, torch.zeros(T, **f), torch.zeros(T, **f),
                       torch.zeros(T, **i), torch.full((2,), 0.9, **f), torch.ones(T, **u),
                       torch.full((T,), -1, **i), torch.zeros(T, **u), torch.zeros(2, **i),
                       torch.zeros(2, **u))
    eb_decode_step(step)
    out = torch.zeros_like(q)
    eb_block_attn_paged(r, c.kv, q, k, v, out)
    args = (_cu([5, 9]), _cu(cached), hq, hkv)
    ref = paged.block_attention(_f64(q), _f64(k), _f64(v), *map(_f64, pre), *args)
    mag = paged.block_attention(_f64(q), _f64(k), np.abs(_f64(v)), _f64(pre[0]),
                                np.abs(_f64(pre[1])), *args)
    _close(_f64(out), ref, mag, "bf16")
    _close(_f64(attn), ref, mag, "bf16")


@pytest.mark.parametrize("cache,dtype", COMBOS)
@pytest.mark.parametrize("blocks,cached", [([1, 1, 1], [400, 60, 999]), ([33, 90], [500, 70]),
                                           ([1] * 64 + [80], [2100] * 65)])
def test_captured_and_replayed(blocks, cached, cache, dtype):
    """Write, attention and read captured into one graph, replayed with eager work in between; and
    every eager run gives the same bits."""
    print(f"graph {blocks} {cache} {dtype}", flush=True)
    rng = np.random.default_rng(13)
    hkv, d, dt = 2, 128, TYPES[dtype]
    after = [p + b for p, b in zip(cached, blocks)]
    c = Cache(after, hkv, 32, d, cache, 9)
    c.fill(cached, rng)
    T = sum(blocks)
    q, k, v = (torch.from_numpy(rng.standard_normal((T, h, d))).to(dt).cuda() for h in (4, 2, 2))
    r, r2 = Ragged.from_lengths(blocks, cached), Ragged.from_lengths(blocks, after)
    code = 0 if dtype == "f32" else EB_BF16
    ws = torch.empty(max(1, eb_block_attn_paged_workspace(code, r, c.kv, 4)), dtype=torch.uint8,
                     device="cuda")
    out = torch.zeros_like(q)
    rows = [torch.zeros(sum(after), hkv, d, dtype=dt, device="cuda") for _ in "kv"]

    def go():
        eb_block_attn_paged(r, c.kv, q, k, v, out, ws=ws)
        eb_kv_write(r, c.kv, k, v)
        eb_kv_read(r2, c.kv, *rows)

    go()
    torch.cuda.synchronize()
    first = [t.clone() for t in (out, *rows)]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        go()
    for i in range(3):
        for t in (out, *rows):
            t.zero_()
        ws.fill_(0xFF)
        (q.float() @ q.float().transpose(1, 2).contiguous()).sum().item()   # work of the program's own
        g.replay()
        torch.cuda.synchronize()
        for t, w in zip((out, *rows), first):
            assert torch.equal(t, w), i
        go()
        torch.cuda.synchronize()
        for t, w in zip((out, *rows), first):
            assert torch.equal(t, w), i


@pytest.mark.parametrize("cache,dtype", COMBOS)
def test_another_stream(cache, dtype):
    s = torch.cuda.Stream()
    _close(*_attention([1, 30], [2000, 77], 16, cache, dtype, 3, 128, stream=s), dtype)
    with torch.cuda.stream(s):
        _close(*_attention([1, 30], [2000, 77], 16, cache, dtype, 3, 128), dtype)


@pytest.mark.parametrize("cache", ["f32", "e4m3"])
def test_fp32_rows_at_any_float(cache):
    """fp32 rows need not be 16-byte aligned: every one of the calls' tensors one float further."""
    rng = np.random.default_rng(15)
    blocks, cached, hkv, hq, d = [3, 40], [70, 500], 2, 6, 64
    spans = [p + n for n, p in zip(blocks, cached)]
    c = Cache(spans, hkv, 16, d, cache, 10)

    def off(n, h, values=True):
        flat = torch.zeros(n * h * d + 1, device="cuda")
        if values:
            flat.copy_(torch.from_numpy(rng.standard_normal(len(flat))))
        return flat[1:].view(n, h, d)

    pre = [off(sum(cached), hkv) for _ in "kv"]
    q, k, v, out = off(43, hq), off(43, hkv), off(43, hkv), off(43, hq, False)
    eb_kv_write(Ragged.from_lengths(cached, [0, 0]), c.kv, *pre)
    r = Ragged.from_lengths(blocks, cached)
    eb_block_attn_paged(r, c.kv, q, k, v, out)
    eb_kv_write(r, c.kv, k, v)
    back = [off(sum(spans), hkv, False) for _ in "kv"]
    eb_kv_read(Ragged.from_lengths([0, 0], spans), c.kv, *back)
    for which, o in zip("kv", back):
        np.testing.assert_array_equal(_f64(o), paged.kv_read(c.values(which), c.table, spans))
    ref = paged.paged_attention(_f64(q), _f64(k), _f64(v), c.values("k"), c.values("v"), c.table,
                                _cu(blocks), cached, hq, hkv)
    _close(_f64(out), ref, None, "f32")


@pytest.mark.parametrize("cache,dtype", COMBOS)
@pytest.mark.parametrize("blocks", [[1, 1, 2], [40, 1, 90]])
def test_shared_pages(blocks, cache, dtype):
    """Sequences that read the same pages (a common beginning), and one that reads a page twice."""
    rng = np.random.default_rng(16)
    cached, page, hkv, group, d = [200, 150, 330], 16, 2, 3, 128
    c = Cache(cached, hkv, page, d, cache, 11)
    c.fill(cached, rng)
    c.table[1, :6] = c.table[0, :6]
    c.table[2, 3:9] = c.table[2, 10]
    c.kv.page_table.copy_(torch.from_numpy(c.table))
    q, k, v = (torch.from_numpy(rng.standard_normal((sum(blocks), h, d))).to(TYPES[dtype])
               for h in (hkv * group, hkv, hkv))
    out = torch.zeros(q.shape, dtype=TYPES[dtype], device="cuda")
    eb_block_attn_paged(Ragged.from_lengths(blocks, cached), c.kv, q.cuda(), k.cuda(), v.cuda(), out)
    args = dict(table=c.table, cu_block=_cu(blocks), cached=cached, hq=hkv * group, hkv=hkv)
    ref = paged.paged_attention(_f64(q), _f64(k), _f64(v), c.values("k"), c.values("v"), **args)
    mag = paged.paged_attention(_f64(q), _f64(k), np.abs(_f64(v)), c.values("k"),
                                np.abs(c.values("v")), **args)
    _close(_f64(out), ref, mag, dtype)


@pytest.mark.parametrize("cache,dtype", COMBOS)
@pytest.mark.parametrize("blocks,cached,hkv,group,head_dim", [
    ([1, 1], [700, 33], 1, 71, 64), ([2, 1], [100, 900], 1, 130, 128), ([1], [400], 40, 1, 128),
    ([1, 0, 3], [90, 5, 300], 17, 5, 64)])
def test_attention_head_layouts(blocks, cached, hkv, group, head_dim, cache, dtype):
    """One K/V head for many query heads (a token is then many rows), many K/V heads, odd numbers."""
    _close(*_attention(blocks, cached, 32, cache, dtype, group, head_dim, hkv=hkv), dtype)


@pytest.mark.parametrize("cache", ["bf16", "e4m3"])
def test_two_streams_at_once(cache):
    """Two calls on one cache in flight on two streams, each with its own workspace."""
    rng = np.random.default_rng(17)
    cached, hkv, hq, d = [3000, 41], 2, 8, 128
    c = Cache(cached, hkv, 64, d, cache, 12)
    c.fill(cached, rng)
    calls = []
    for blocks in ([1, 1], [70, 40]):
        r = Ragged.from_lengths(blocks, cached)
        x = [torch.from_numpy(rng.standard_normal((sum(blocks), h, d))).bfloat16().cuda()
             for h in (hq, hkv, hkv)]
        ws = torch.empty(max(1, eb_block_attn_paged_workspace(EB_BF16, r, c.kv, hq)),
                         dtype=torch.uint8, device="cuda")
        alone, out = torch.zeros_like(x[0]), torch.zeros_like(x[0])
        eb_block_attn_paged(r, c.kv, *x, alone, ws=ws)
        calls.append((r, x, ws, alone, out, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        for r, x, ws, _, out, s in calls:
            eb_block_attn_paged(r, c.kv, *x, out, ws=ws, stream=s)
    torch.cuda.synchronize()
    for _, _, _, alone, out, _ in calls:
        assert torch.equal(alone, out)


def test_temporary_workspace_lives_until_the_launch(monkeypatch):
    """A workspace that the binding allocates is still held when the library is called: given back
    before, another thread's tensor could take its memory and be overwritten by the kernels."""
    c = Cache([3000], 2, 16, 128, "bf16", 1)
    c.fill([3000], np.random.default_rng(0))
    r = Ragged.from_lengths([1], [3000])
    q, k = (torch.ones(1, h, 128, dtype=torch.bfloat16, device="cuda") for h in (4, 2))
    h, w = (torch.ones(n, 128, dtype=torch.bfloat16, device="cuda") for n in (4, 5000))
    pre = [torch.ones(3000, 2, 128, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    conf, entropy, gap = (torch.zeros(4, device="cuda") for _ in range(3))
    top, suffix = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (4, 2))
    out, lib, seen = torch.zeros_like(q), binding.load(), {}

    class Watched:
        """The library, noting what a workspace query answers and the memory in use at a call."""

        def __getattr__(self, name):
            def call(*args):
                if not name.endswith("_workspace"):
                    seen["in use"] = torch.cuda.memory_allocated()
                answer = getattr(lib, name)(*args)
                if name.endswith("_workspace"):
                    seen["need"] = answer
                return answer
            return call

    monkeypatch.setattr(binding, "load", Watched)
    for go in (lambda: eb_block_attn_paged(r, c.kv, q, k, k, out),
               lambda: eb_block_attn(r, q, k, k, *pre, out),
               lambda: binding.eb_block_attn_dual(r, suffix, 0, q, k, k, *pre, k[:0], k[:0], out),
               lambda: binding.eb_lmhead_confidence(h, w, conf, entropy, top),
               lambda: binding.eb_lmhead_features(h, w, conf, entropy, top, gap)):
        before = torch.cuda.memory_allocated()
        go()
        assert seen["need"] > 0 and seen["in use"] >= before + seen["need"], seen


def test_binding_refusals():
    c = Cache([40], 2, 16, 128, "bf16", 1)
    r = Ragged.from_lengths([3], [20])
    q = torch.zeros(3, 4, 128, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(3, 2, 128, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="shape"):
        eb_kv_write(r, c.kv, k[:2], k)
    with pytest.raises(ValueError, match="contiguous"):
        eb_kv_write(r, c.kv, torch.zeros(3, 3, 128, dtype=torch.bfloat16, device="cuda")[:, :2], k)
    with pytest.raises(ValueError, match="pos"):
        eb_kv_write(r, c.kv, k, k, pos=torch.zeros(3, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError, match="shape"):
        eb_kv_read(r, c.kv, k, k)
    with pytest.raises(EbError, match="UNSUPPORTED"):
        eb_kv_write(r, c.kv, k.float(), k.float())
    with pytest.raises(ValueError, match="out"):
        eb_block_attn_paged(r, c.kv, q, k, k, q.float())
    with pytest.raises(ValueError, match="rows"):
        eb_kv_write(Ragged.from_lengths([3, 0], [20, 0]), c.kv, k, k)
    with pytest.raises(EbError, match="max_prefix"):
        eb_block_attn_paged(Ragged.from_lengths([3], [49]), c.kv, q, k, k, q.clone())
    with pytest.raises(ValueError, match="k_scale|device tensor|torch.Tensor"):
        PagedKV(c.kv.k.to(torch.float8_e4m3fn), c.kv.v.to(torch.float8_e4m3fn), c.kv.page_table,
                k_scale=torch.zeros(1), v_scale=torch.zeros(1))
    with pytest.raises(ValueError, match="float8"):
        PagedKV(c.kv.k, c.kv.v, c.kv.page_table, k_scale=torch.zeros(1))
    with pytest.raises(TypeError):
        eb_kv_write(r, c.kv.k, k, k)
    with pytest.raises(AttributeError, match="fixed"):
        c.kv.page_table = torch.zeros(1, 3, dtype=torch.int32, device="cuda")


def test_debug_checks(monkeypatch):
    """EB_DEBUG_CHECKS: pages out of range, positions past the table, one row of a page twice."""
    monkeypatch.setenv("EB_DEBUG_CHECKS", "1")
    c = Cache([40, 40], 2, 16, 128, "bf16", 1)
    r = Ragged.from_lengths([2, 2], [20, 20])
    k = torch.zeros(4, 2, 128, dtype=torch.bfloat16, device="cuda")
    q = torch.zeros(4, 4, 128, dtype=torch.bfloat16, device="cuda")

    def pos(*p):
        return torch.tensor(p, dtype=torch.int32, device="cuda")

    eb_kv_write(r, c.kv, k, k)
    eb_kv_write(r, c.kv, k, k, pos=pos(3, -1, 3, -1))       # the same position of two sequences
    eb_block_attn_paged(r, c.kv, q, k, k, q.clone())
    with pytest.raises(EbError, match="two rows"):
        eb_kv_write(r, c.kv, k, k, pos=pos(3, 3, 1, 2))
    with pytest.raises(EbError, match="does not fit"):
        eb_kv_write(r, c.kv, k, k, pos=pos(1, 48, 1, 2))
    shared = c.table.copy()
    shared[1, 1] = shared[0, 1]                              # both append to one page
    c.kv.page_table.copy_(torch.from_numpy(shared))
    with pytest.raises(EbError, match="two rows"):
        eb_kv_write(r, c.kv, k, k)
    eb_block_attn_paged(r, c.kv, q, k, k, q.clone())         # reading it is fine
    shared[1, 1] = c.kv.n_pages
    c.kv.page_table.copy_(torch.from_numpy(shared))
    out = [torch.zeros(40, 2, 128, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    for call in (lambda: eb_kv_write(r, c.kv, k, k), lambda: eb_kv_read(r, c.kv, *out),
                 lambda: eb_block_attn_paged(r, c.kv, q, k, k, q.clone())):
        with pytest.raises(EbError, match="page_table"):
            call()
