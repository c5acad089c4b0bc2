"""eb_kv_assign against a host's allocator (oracle/assign.py), every integer that it writes; and a run of
it with the calls that use its pages, rows, logits and draws."""
import numpy as np
import pytest
import torch

from oracle import block_attention
from oracle.assign import assign
from oracle.sample import sample
from paper_2609_16450_amd import (EbError, PagedKV, PagePool, Ragged, eb_block_attn_paged,
                                  eb_kv_assign, eb_kv_write, eb_lmhead_logits, eb_sample,
                                  eb_unmask_select)

pytestmark = pytest.mark.gpu

SENTINEL = -77


def _dev(x, dtype=torch.int32):
    return torch.as_tensor(np.asarray(x)).to(dtype).cuda()


class Requests:
    """Sequences with held pages handed out in no order, a ring that begins anywhere, garbage in the
    table's other entries and the ring's other places."""

    def __init__(self, cached, new, page, free, wide=None, done=None, shared=None, seed=0,
                 n_rows=None, spare=2):
        rng = np.random.default_rng(seed)
        self.page, self.cached, self.new = page, np.array(cached), np.array(new)
        held = -(-self.cached // page)
        end = -(-(self.cached + self.new) // page)
        B = len(cached)
        wide = int(max(end.max(), held.max(), 1)) if wide is None else wide
        n_pages = int(held.sum()) + free + spare
        order = rng.permutation(n_pages).astype(np.int32)
        self.table = rng.integers(-5, 2 ** 31 - 1, (B, wide)).astype(np.int32)
        at = 0
        for b in range(B):
            n = min(held[b], wide)
            self.table[b, :n] = order[at:at + n]
            at += n
        head = int(rng.integers(n_pages))
        self.ring = rng.integers(-5, 2 ** 31 - 1, n_pages).astype(np.int32)
        for i in range(free):
            self.ring[(head + i) % n_pages] = order[at + i]
        self.state = np.array([head, free], np.int32)
        self.done = None if done is None else np.array(done, np.uint8)
        self.shared = None if shared is None else np.array(shared, np.int32)
        rows = int(sum(n for b, n in enumerate(new) if done is None or not done[b]))
        self.n_rows = rows if n_rows is None else n_rows

    def oracle(self):
        return assign(self.table, self.ring, self.state, self.cached, self.new, self.page,
                      self.n_rows, self.done, self.shared)

    def tensors(self):
        B = len(self.cached)

        def out(n, dtype=torch.int32):
            return torch.full((n,), SENTINEL % 200, dtype=dtype, device="cuda")

        kv = PagedKV.empty(len(self.ring), 1, self.page, 64, _dev(self.table))
        pool = PagePool(_dev(self.ring), _dev(self.state))
        ins = dict(cached=_dev(self.cached), new_rows=_dev(self.new))
        opt = dict(done=None if self.done is None else _dev(self.done, torch.uint8),
                   shared=None if self.shared is None else _dev(self.shared))
        outs = dict(cu_block=out(B + 1), cu_prefix=out(B + 1), pos=out(self.n_rows))
        more = dict(slot=out(self.n_rows, torch.int64), short=out(B, torch.uint8))
        return kv, pool, ins, opt, outs, more

    def check(self, in_place):
        kv, pool, ins, opt, outs, more = self.tensors()
        state = None if in_place else torch.zeros(2, dtype=torch.int32, device="cuda")
        ref = self.oracle()
        for _ in range(1 if in_place else 2):           # with a state of its own the call can be repeated
            eb_kv_assign(kv, pool, *ins.values(), *outs.values(), **more, **opt, state_out=state)
            torch.cuda.synchronize()
            got = dict(table=kv.page_table, ring=pool.free_pages,
                       state=pool.state if in_place else state, **outs, **more)
            for k, t in got.items():
                np.testing.assert_array_equal(t.cpu().numpy(), ref[k], err_msg=k)
            if not in_place:
                np.testing.assert_array_equal(pool.state.cpu().numpy(), self.state)
        return ref


def _random(B, new, cached, page, seed, free=1.0, done=0.0, **kw):
    rng = np.random.default_rng(seed)
    n = rng.integers(new[0], new[1] + 1, B)
    c = rng.integers(cached[0], cached[1] + 1, B)
    gone = rng.random(B) < done
    need = int((-(-(c + n) // page) - -(-c // page))[~gone].sum())
    held = -(-c // page)
    return Requests(c, n, page, int(need * free), done=gone, seed=seed,
                    shared=rng.integers(0, held + 2), **kw)


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("B,new,cached", [
    (1, (1, 1), (0, 0)), (1, (1, 1), (16, 16)), (1, (1, 1), (15, 4097)), (1, (3000, 3000), (5, 5)),
    (3, (0, 0), (0, 40)), (7, (0, 2), (0, 300)), (63, (1, 40), (0, 500)), (64, (0, 1), (255, 257)),
    (65, (16, 256), (1, 1000)), (1023, (0, 3), (0, 64)), (1024, (1, 1), (0, 600)),
    (1025, (1, 1), (0, 600)), (2500, (0, 9), (0, 100)), (40, (500, 900), (0, 3000)),
])
def test_assign(B, new, cached, page, in_place):
    print(f"assign {B} {new} {cached} page {page}", flush=True)
    _random(B, new, cached, page, seed=B + page).check(in_place)


@pytest.mark.parametrize("free", [0.0, 0.3, 0.9])
@pytest.mark.parametrize("B,new,cached", [(1, (20, 20), (3, 3)), (50, (0, 60), (0, 200)),
                                          (1500, (0, 30), (0, 90)), (9, (900, 2000), (0, 20))])
def test_too_few_pages(B, new, cached, free):
    ref = _random(B, new, cached, 16, seed=B, free=free).check(True)
    assert ref["short"].any()


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("B,new,cached,page", [(2, (1, 5), (30, 60), 16), (64, (1, 200), (0, 900), 32),
                                               (1400, (1, 9), (0, 500), 16),
                                               (3, (0, 3000), (4000, 9000), 16)])
def test_finished_sequences(B, new, cached, page, in_place):
    """Pages go back behind the free ones, the shared ones stay; the ring wraps round."""
    for seed in range(4):
        _random(B, new, cached, page, seed, done=0.5).check(in_place)
    _random(B, new, cached, page, 9, done=1.0).check(in_place)      # no row is left


def test_padded_batch():
    """Rows behind the last sequence's hold -1, over several workgroups."""
    for n_rows in (5, 6, 1024, 5000):
        Requests([3, 20], [2, 3], 16, 4, n_rows=n_rows).check(True)


def test_narrow_table():
    """A row of the table with too few columns for its sequence; the others are served."""
    ref = Requests([10, 40, 63], [60, 3, 1], 16, 9, wide=4).check(False)
    assert ref["short"].tolist() == [1, 0, 0]
    Requests([64, 0], [1, 65], 16, 9, wide=4).check(True)


def test_longest_sequence():
    """Positions next to 2^31: the last one that fits, and the first that does not."""
    top = 2 ** 31 - 1
    for new, short in ((1, 0), (2, 1)):
        kv = PagedKV.empty(40, 1, 256, 64, torch.zeros(1, 2 ** 23, dtype=torch.int32, device="cuda"))
        pool = PagePool.full(40)
        cu, cp = (torch.zeros(2, dtype=torch.int32, device="cuda") for _ in range(2))
        pos = torch.zeros(new, dtype=torch.int32, device="cuda")
        sh = torch.zeros(1, dtype=torch.uint8, device="cuda")
        kv.page_table[0, -1] = 7
        slot = torch.zeros(new, dtype=torch.int64, device="cuda")
        eb_kv_assign(kv, pool, _dev([top - 1]), _dev([new]), cu, cp, pos, slot=slot, short=sh)
        assert sh.tolist() == [short]
        assert pos.tolist() == ([top - 1] if not short else [-1, -1])
        assert slot.tolist() == ([7 * 256 + 254] if not short else [-1, -1])


def test_optional_outputs():
    req = _random(33, (0, 50), (0, 300), 32, 5, done=0.2)
    kv, pool, ins, opt, outs, _ = req.tensors()
    eb_kv_assign(kv, pool, *ins.values(), *outs.values(), **opt)
    ref = req.oracle()
    for k, t in dict(table=kv.page_table, ring=pool.free_pages, state=pool.state, **outs).items():
        np.testing.assert_array_equal(t.cpu().numpy(), ref[k], err_msg=k)


def test_another_stream():
    s = torch.cuda.Stream()
    req = _random(90, (0, 90), (0, 300), 16, 6, done=0.2)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        req.check(True)
    kv, pool, ins, opt, outs, more = req.tensors()
    torch.cuda.synchronize()
    eb_kv_assign(kv, pool, *ins.values(), *outs.values(), **more, **opt, stream=s)
    s.synchronize()
    np.testing.assert_array_equal(kv.page_table.cpu().numpy(), req.oracle()["table"])


def test_captured_and_replayed():
    """A graph that takes a row per sequence and goes on: each replay is the allocator's next step."""
    B, page = 70, 16
    req = Requests([5 + 7 * b % 40 for b in range(B)], [1] * B, page, 200, wide=8, spare=0)
    kv, pool, ins, _, outs, more = req.tensors()

    def go():
        eb_kv_assign(kv, pool, *ins.values(), *outs.values(), **more)
        ins["cached"].add_(ins["new_rows"])

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        go()
    for step in range(12):
        ref = req.oracle()
        if step % 3 == 2:
            go()
        else:
            g.replay()
        torch.cuda.synchronize()
        got = dict(table=kv.page_table, state=pool.state, **outs, **more)
        for k, t in got.items():
            np.testing.assert_array_equal(t.cpu().numpy(), ref[k], err_msg=f"{step} {k}")
        req.table, req.ring, req.state = ref["table"], ref["ring"], ref["state"]
        req.cached = req.cached + req.new


def test_binding_refusals():
    req = Requests([5, 9], [1, 1], 16, 4)
    kv, pool, ins, _, outs, more = req.tensors()
    cached, new = ins.values()
    cu, cp, pos = outs.values()
    with pytest.raises(ValueError, match="cached"):
        eb_kv_assign(kv, pool, cached.long(), new, cu, cp, pos)
    with pytest.raises(ValueError, match="new_rows"):
        eb_kv_assign(kv, pool, cached, new[:1], cu, cp, pos)
    with pytest.raises(ValueError, match="cu_prefix"):
        eb_kv_assign(kv, pool, cached, new, cu, cp[:2], pos)
    with pytest.raises((ValueError, TypeError), match="cu_block"):
        eb_kv_assign(kv, pool, cached, new, None, cp, pos)
    with pytest.raises(ValueError, match="pos"):
        eb_kv_assign(kv, pool, cached, new, cu, cp, pos.long())
    with pytest.raises(ValueError, match="slot"):
        eb_kv_assign(kv, pool, cached, new, cu, cp, pos, slot=pos)
    with pytest.raises(ValueError, match="done"):
        eb_kv_assign(kv, pool, cached, new, cu, cp, pos, done=new)
    with pytest.raises(ValueError, match="ring"):
        eb_kv_assign(kv, PagePool.full(3), cached, new, cu, cp, pos)
    with pytest.raises(ValueError, match="state_out"):
        eb_kv_assign(kv, pool, cached, new, cu, cp, pos, state_out=cu)


def test_pool_attributes_are_fixed():
    """A tensor set behind the checks of the constructor would reach the kernel unchecked."""
    pool = PagePool.full(8)
    ring, state = pool.free_pages, pool.state
    for name, t in (("state", torch.zeros(1, dtype=torch.int32)), ("free_pages", ring.long())):
        with pytest.raises(AttributeError, match="fixed"):
            setattr(pool, name, t)
    assert pool.free_pages is ring and pool.state is state
    assert ring.tolist() == list(range(8)) and state.tolist() == [0, 8]


def test_debug_checks(monkeypatch):
    monkeypatch.setenv("EB_DEBUG_CHECKS", "1")

    def call(**change):
        req = Requests([5, 20], [1, 30], 16, 4, spare=0, wide=4, done=[1, 0])
        for k, v in change.items():
            getattr(req, k)[...] = v
        kv, pool, ins, opt, outs, more = req.tensors()
        eb_kv_assign(kv, pool, *ins.values(), *outs.values(), **more, **opt)

    call()
    with pytest.raises(EbError, match="negative"):
        call(new=[1, -1])
    with pytest.raises(EbError, match="do not fit"):
        call(cached=[5, 65])
    with pytest.raises(EbError, match="new rows"):
        call(new=[1, 31])
    with pytest.raises(EbError, match="state"):
        call(state=[7, 4])
    with pytest.raises(EbError, match="given back"):
        call(state=[0, 7], ring=np.arange(7))
    with pytest.raises(EbError, match="free_pages"):
        call(ring=7)
    with pytest.raises(EbError, match="page_table"):
        call(table=-1)


def test_serving_run():
    """Blocks of several requests, step after step: pages for the block's rows, the rows into them,
    attention over the pages, logits, a draw per row, the commit; a request that ends gives its pages
    back and another takes its place.  Every step against the oracles."""
    rng = np.random.default_rng(3)
    B, page, wide, hq, hkv, d, hidden, V = 3, 16, 5, 4, 2, 64, 64, 300
    n_pages = 7                                         # fewer than three long requests take
    kv = PagedKV.empty(n_pages, hkv, page, d, torch.full((B, wide), -1, dtype=torch.int32,
                                                         device="cuda"), torch.float32)
    pool = PagePool.full(n_pages)
    w = rng.standard_normal((V, hidden)).astype(np.float32)
    cached, keys = [0] * B, [[np.zeros((0, hkv, d))] * 2 for _ in range(B)]
    temp, top_k, top_p, min_p = [0.8, 0.0, 1.3], [0, 5, 40], [0.9, 1.0, 0.95], [0.0, 0.0, 0.01]
    ring, state = np.arange(n_pages, dtype=np.int32), np.array([0, n_pages], np.int32)
    table = np.full((B, wide), -1, np.int32)
    seen_short = ended = 0
    for step in range(14):
        new = [int(x) for x in rng.integers(1, 14, B)]
        done = [int(c > 40) for c in cached]
        live = [0 if x else n for x, n in zip(done, new)]
        pre = [0 if x else c for x, c in zip(done, cached)]
        T = sum(live)
        ref = assign(table, ring, state, cached, new, page, T, done)
        r = Ragged.from_lengths(live, pre)
        cu, cp = torch.zeros_like(r.cu_block), torch.zeros_like(r.cu_block)
        pos = torch.zeros(T, dtype=torch.int32, device="cuda")
        short = torch.zeros(B, dtype=torch.uint8, device="cuda")
        eb_kv_assign(kv, pool, _dev(cached), _dev(new), cu, cp, pos, done=_dev(done, torch.uint8),
                     short=short)
        r.cu_block, r.cu_prefix = cu, cp                # the device's offsets from here on
        k, v, q = (rng.standard_normal((T, n, d)).astype(np.float32) for n in (hkv, hkv, hq))
        h = rng.standard_normal((T, hidden)).astype(np.float32)
        u = rng.random(T).astype(np.float32)
        out = torch.zeros(T, hq, d, device="cuda")
        z = torch.zeros(T, V, device="cuda")
        token = torch.zeros(T, dtype=torch.int32, device="cuda")
        prob, conf = torch.zeros(T, device="cuda"), torch.zeros(T, device="cuda")
        f = lambda x: torch.from_numpy(x).cuda()  # noqa: E731
        eb_block_attn_paged(r, kv, f(q), f(k), f(v), out)
        eb_kv_write(r, kv, f(k), f(v), pos=pos)
        eb_lmhead_logits(f(h), f(w), z)
        eb_sample(r, z, f(u), token, prob=prob, conf=conf, temperature=_dev(temp, torch.float32),
                  top_k=_dev(top_k), top_p=_dev(top_p, torch.float32),
                  min_p=_dev(min_p, torch.float32))
        masked = torch.ones(T, dtype=torch.uint8, device="cuda")
        tokens = torch.full((T,), -1, dtype=torch.int32, device="cuda")
        unmask = torch.zeros_like(masked)
        nc, res = (torch.zeros(B, dtype=t, device="cuda") for t in (torch.int32, torch.uint8))
        eb_unmask_select(r, conf, token, torch.full((B,), 0.02, device="cuda"), masked, tokens,
                         unmask, nc, res)
        torch.cuda.synchronize()
        table, ring, state = ref["table"], ref["ring"], ref["state"]
        for name, t in dict(table=kv.page_table, ring=pool.free_pages, state=pool.state, cu_block=cu,
                            cu_prefix=cp, pos=pos, short=short).items():
            np.testing.assert_array_equal(t.cpu().numpy(), ref[name], err_msg=f"{step} {name}")
        at, zz = 0, z.double().cpu().numpy()
        np.testing.assert_allclose(zz, h.astype(np.float64) @ w.astype(np.float64).T, rtol=0,
                                   atol=1e-3)
        kk = [np.concatenate([keys[b][i] if not done[b] else keys[b][i][:0] for b in range(B)])
              for i in range(2)]
        att = block_attention(q, k, v, kk[0], kk[1], ref["cu_block"], ref["cu_prefix"], hq, hkv)
        np.testing.assert_allclose(out.cpu().numpy(), att, rtol=2e-5, atol=2e-5)
        for b in range(B):
            if done[b]:
                keys[b], cached[b] = [np.zeros((0, hkv, d))] * 2, 0
                ended += 1
                continue
            rows = slice(at, at + live[b])
            for i in range(at, at + live[b]):
                want = sample(zz[i], u[i], temp[b], top_k[b], np.float32(top_p[b]),
                              np.float32(min_p[b]))
                assert int(token[i]) == want[0], (step, i)
                assert float(prob[i]) == pytest.approx(want[1], rel=1e-6)
                assert int(tokens[i]) == (want[0] if int(unmask[i]) else -1)
            if not ref["short"][b]:
                keys[b] = [np.concatenate([keys[b][0], k[rows]]), np.concatenate([keys[b][1], v[rows]])]
                cached[b] += live[b]
            seen_short += int(ref["short"][b])
            at += live[b]
    assert seen_short and ended


@pytest.mark.parametrize("cached,new,dtype", [([5, 70, 33], [9, 1, 20], torch.float32),
                                              ([0, 400, 129, 31], [32, 16, 64, 1], torch.bfloat16)])
def test_step_captured_and_replayed(cached, new, dtype):
    """A whole step in one graph: pages for its rows, attention over the pages, the rows into them,
    logits, a draw, the commit.  The lengths are the capture's; every replay takes other pages, until
    there are too few, and other values, and leaves what the same calls leave eagerly, bit for bit."""
    page, hq, hkv, d, hidden, V = 16, 4, 2, 64, 64, 300
    B, T = len(cached), sum(new)
    held, wide = [-(-c // page) for c in cached], 40
    takes = sum(-(-(c + n) // page) for c, n in zip(cached, new)) - sum(held)
    replays = 4
    n_pages = sum(held) + takes * (replays + 1)         # an eager run, then all replays but one
    table = torch.full((B, wide), -1, dtype=torch.int32)
    for b in range(B):
        table[b, :held[b]] = torch.arange(sum(held[:b]), sum(held[:b + 1]))
    u8, f32, i32 = torch.uint8, torch.float32, torch.int32
    w = torch.randn(V, hidden, device="cuda").to(dtype)

    class Side:
        """All that one side of the comparison reads and writes."""

        def __init__(self):
            self.kv = PagedKV.empty(n_pages, hkv, page, d, table.cuda(), dtype)
            for t in (self.kv.k, self.kv.v):
                t.copy_(torch.randn(t.shape, generator=torch.Generator().manual_seed(5)))
            self.pool = PagePool(torch.arange(sum(held), sum(held) + n_pages, device="cuda",
                                              dtype=i32) % n_pages,
                                 _dev([0, n_pages - sum(held)]))
            z = lambda shape, dt: torch.zeros(shape, dtype=dt, device="cuda")  # noqa: E731
            self.cu, self.cp, self.pos = z(B + 1, i32), z(B + 1, i32), z(T, i32)
            self.short = z(B, u8)
            self.q, self.k, self.v = (z((T, n, d), dtype) for n in (hq, hkv, hkv))
            self.h, self.u, self.out = z((T, hidden), dtype), z(T, f32), z((T, hq, d), dtype)
            self.logits, self.token = z((T, V), f32), z(T, i32)
            self.prob, self.conf = z(T, f32), z(T, f32)
            self.masked, self.tokens, self.unmask = z(T, u8), z(T, i32), z(T, u8)
            self.nc, self.res = z(B, i32), z(B, u8)
            self.ragged = Ragged.from_lengths(new, cached)
            self.ragged.cu_block, self.ragged.cu_prefix = self.cu, self.cp
            self.ins = (_dev(cached), _dev(new))
            self.limits = dict(temperature=_dev([0.8] * B, f32), top_p=_dev([0.9] * B, f32))
            self.tau = torch.full((B,), 0.02, device="cuda")

        def fill(self, seed):
            g = torch.Generator().manual_seed(seed)
            for t in (self.q, self.k, self.v, self.h):
                t.copy_(torch.randn(t.shape, generator=g))
            self.u.copy_(torch.rand(T, generator=g))
            self.masked.fill_(1)
            self.tokens.fill_(-1)

        def step(self):
            eb_kv_assign(self.kv, self.pool, *self.ins, self.cu, self.cp, self.pos,
                         short=self.short)
            eb_block_attn_paged(self.ragged, self.kv, self.q, self.k, self.v, self.out)
            eb_kv_write(self.ragged, self.kv, self.k, self.v, pos=self.pos)
            eb_lmhead_logits(self.h, w, self.logits)
            eb_sample(self.ragged, self.logits, self.u, self.token, prob=self.prob, conf=self.conf,
                      **self.limits)
            eb_unmask_select(self.ragged, self.conf, self.token, self.tau, self.masked, self.tokens,
                             self.unmask, self.nc, self.res)

        def results(self):
            return dict(table=self.kv.page_table, state=self.pool.state, k=self.kv.k, v=self.kv.v,
                        cu=self.cu, cp=self.cp, pos=self.pos, short=self.short, out=self.out,
                        logits=self.logits, token=self.token, prob=self.prob, conf=self.conf,
                        masked=self.masked, tokens=self.tokens, unmask=self.unmask, nc=self.nc,
                        res=self.res)

    captured, eager = Side(), Side()
    for x in (captured, eager):
        x.fill(0)
        x.step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        captured.step()
    print(f"step captured {cached} {new}", flush=True)
    short = []
    for i in range(1, replays + 2):
        captured.fill(i)
        g.replay()
        torch.cuda.synchronize()
        (w.float() @ w.float().t()).sum().item()
        eager.fill(i)
        eager.step()
        torch.cuda.synchronize()
        for (name, a), b in zip(captured.results().items(), eager.results().values()):
            assert torch.equal(a, b), (i, name)
        short.append(int(captured.short.sum()))
    assert not any(short[:-1]) and short[-1]
