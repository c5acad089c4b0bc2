"""Measured cases of drawing tokens from a step's logits and of handing out the cache's pages: what a
serving program built on the library calls between two passes of its model, in plain torch
(own = False) or through the package's entry points (own = True).

  logits  eb_lmhead_logits: z = W h for every row, written out
  sample  eb_sample: a token per row from its logits and a given random number, with a temperature,
          top-k, top-p and min-p of its sequence
  assign  eb_kv_assign: from the sequences' lengths, their offsets, the pages that their new rows
          need, the rows' positions and slots; pages of finished sequences go back

A case holds sizes only.  Ragged lengths come from the case's own "lens" number, so that the work of
a case is known without a GPU; every value comes from the seed given to prepare().
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

SIZES = {"f32": 4, "bf16": 2}
LIFTED = 64  # tokens of a row that stand out of its bulk


def _logits(name, dtype, rows, hidden, vocab):
    return dict(name=name, kind="logits", dtype=dtype, rows=rows, hidden=hidden, vocab=vocab)


def _sample(name, dtype, batch, block, vocab, pitch, params, lens):
    return dict(name=name, kind="sample", dtype=dtype, batch=batch, block_lo=block[0],
                block_hi=block[1], vocab=vocab, pitch=pitch, params=params, lens=lens)


def _assign(name, batch, new, cached, page, lens, done=0.0, short=False):
    return dict(name=name, kind="assign", batch=batch, new_lo=new[0], new_hi=new[1],
                cached_lo=cached[0], cached_hi=cached[1], page=page, lens=lens, done=done,
                short=short)


def listed():
    return [
        # One user's block through the 8B model's head: W from memory for a handful of rows.
        _logits("logits_llada_t32", "bf16", 32, 4096, 126464),
        # A batch of blocks through the same head: a large product, and half a gigabyte of logits.
        _logits("logits_llada_t1024", "bf16", 1024, 4096, 126464),
        # An odd number of rows over an odd vocabulary, as a small model with added tokens has.
        _logits("logits_odd_t201", "bf16", 201, 2048, 32003),
        # The toy model in fp32, as in unit tests and debugging.
        _logits("logits_tiny_f32", "f32", 32, 256, 2048),
        # One user, one token: the usual chat setting.
        _sample("sample_token_b1", "f32", 1, (1, 1), 152064, 152064, "chat", 1),
        # One user's block of 32, top-p alone: wide nuclei where the model is unsure.
        _sample("sample_block_topp", "f32", 1, (32, 32), 126464, 126464, "topp", 2),
        # A served batch of single tokens, bf16 logits of another program's head, min-p.
        _sample("sample_tokens_b64_minp", "bf16", 64, (1, 1), 152064, 152064, "minp", 3),
        # A batch of blocks, every sequence with settings of its own.
        _sample("sample_batch_mixed", "f32", 16, (16, 128), 126464, 126464, "mixed", 4),
        # A small odd vocabulary in rows padded to a multiple of 64, temperature alone.
        _sample("sample_odd_temp", "f32", 7, (1, 1), 32003, 32064, "temp", 5),
        # One sequence, one token behind a long context: the smallest step.
        _assign("assign_token_b1", 1, (1, 1), (4096, 4096), 64, 6),
        # A full batch of blocks, some sequences finished, the pool too small for the last ones.
        _assign("assign_blocks_b64", 64, (16, 256), (1, 4096), 64, 7, done=0.15, short=True),
        # Many users, tokens beside long chunks of prompts, small pages.
        _assign("assign_prompts_b1024", 1024, (1, 400), (0, 3000), 16, 8, done=0.1),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _span(rng, lo, hi):
    a = _log_int(rng, lo, hi)
    return (a, a) if rng.random() < 0.4 else (max(lo, a // rng.choice((2, 4, 8))), a)


# no drawn case moves more, computes more or has more logits or rows than the largest listed ones
MOST_BYTES, MOST_FLOPS, MOST_LOGITS, MOST_ROWS = 1.5e9, 1.06e12, 1.2e8, 200000


def _draw_logits(rng):
    if rng.random() < 0.2:
        return _logits(None, "f32", _log_int(rng, 1, 64), _log_int(rng, 17, 512),
                       _log_int(rng, 1000, 8000))
    case = _logits(None, "bf16", _log_int(rng, 1, 1024), 64 * _log_int(rng, 1, 64),
                   _log_int(rng, 1000, 160000))
    while work(case)["bytes"] > MOST_BYTES or work(case)["flops"] > MOST_FLOPS:
        case["rows"] = (case["rows"] + 1) // 2
    return case


def _draw_sample(rng):
    batch, vocab = _log_int(rng, 1, 64), _log_int(rng, 1000, 160000)
    block = (1, 1) if rng.random() < 0.35 else _span(rng, 2, 128)
    while batch > 1 and batch * block[1] * vocab > MOST_LOGITS:
        batch = (batch + 1) // 2
    return _sample(None, rng.choice(("f32", "f32", "bf16")), batch, block, vocab,
                   vocab if rng.random() < 0.6 else (vocab + 63) // 64 * 64,
                   rng.choice(("chat", "topp", "minp", "temp", "mixed", "mixed")),
                   rng.randrange(1 << 20))


def _draw_assign(rng):
    batch, new = _log_int(rng, 1, 1024), _span(rng, 1, 400)
    while batch > 1 and batch * new[1] > MOST_ROWS:
        batch = (batch + 1) // 2
    return _assign(None, batch, new, (0, _log_int(rng, 1, 8000)),
                   rng.choice((16, 32, 64, 128, 256)), rng.randrange(1 << 20),
                   done=rng.choice((0.0, 0.1, 0.3)), short=rng.random() < 0.3)


def draw(rng):
    case = rng.choice((_draw_logits, _draw_sample, _draw_sample, _draw_assign))(rng)
    del case["name"]
    return case


# --------------------------------------------------------------------------------------------
# sizes and work
# --------------------------------------------------------------------------------------------
def _blocks(case):
    rng = random.Random(case["lens"])
    return [rng.randint(case["block_lo"], case["block_hi"]) for _ in range(case["batch"])]


def _requests(case):
    """New rows, cached rows and whether it is finished, of every sequence; the pages that the pool
    has free (all that are needed and some, or too few)."""
    rng = random.Random(case["lens"])
    new = [rng.randint(case["new_lo"], case["new_hi"]) for _ in range(case["batch"])]
    cached = [rng.randint(case["cached_lo"], case["cached_hi"]) for _ in range(case["batch"])]
    done = [rng.random() < case["done"] for _ in range(case["batch"])]
    ps = case["page"]
    need = sum((c + n + ps - 1) // ps - (c + ps - 1) // ps
               for n, c, d in zip(new, cached, done) if not d)
    return new, cached, done, max(need - need // 16 - 1, 0) if case["short"] else need + 3


def work(case):
    if case["kind"] == "logits":
        t, d, v, e = case["rows"], case["hidden"], case["vocab"], SIZES[case["dtype"]]
        return {"bytes": (t + v) * d * e + 4 * t * v, "flops": 2 * t * d * v}
    if case["kind"] == "sample":
        t = sum(_blocks(case))
        # logits in; a random number, a token, its probability and its confidence per row.  An
        # exponential counts as one operation, beside a difference and a sum.
        return {"bytes": t * (case["vocab"] * SIZES[case["dtype"]] + 16),
                "flops": 3 * t * case["vocab"]}
    new, cached, done, free = _requests(case)
    ps, rows, taken = case["page"], 0, 0
    for n, c, d in zip(new, cached, done):
        if not d:
            rows += n
            taken += (c + n + ps - 1) // ps - (c + ps - 1) // ps
    # lengths and flags in, offsets out; a page number from the ring into the table; position and
    # slot of a row
    return {"bytes": 21 * case["batch"] + 8 * min(taken, free) + 12 * rows, "flops": 0}


# --------------------------------------------------------------------------------------------
# inputs (plain torch; shared by prepare() and exact())
# --------------------------------------------------------------------------------------------
def _dtype(name):
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def _settings(case, seed):
    """Temperature, top-k, top-p and min-p of every sequence (None: the case does without)."""
    rng = random.Random(seed * 7919 + case["lens"])
    kind, batch = case["params"], case["batch"]

    def column(pick, dtype):
        return torch.tensor([pick() for _ in range(batch)], dtype=dtype, device="cuda")

    f32, i32 = torch.float32, torch.int32
    if kind == "chat":
        return (column(lambda: rng.uniform(0.6, 1.0), f32), column(lambda: rng.choice((20, 50)), i32),
                column(lambda: rng.uniform(0.8, 0.98), f32), None)
    if kind == "topp":
        return None, None, column(lambda: rng.uniform(0.85, 0.98), f32), None
    if kind == "minp":
        return (column(lambda: rng.uniform(0.8, 1.5), f32), None, None,
                column(lambda: rng.uniform(0.02, 0.1), f32))
    if kind == "temp":
        return column(lambda: rng.uniform(0.5, 1.2), f32), None, None, None
    # settings of many programs side by side; 0 is greedy, no top-k, no min-p, 1 is no top-p
    return (column(lambda: rng.choice((0.0, 0.7, 1.0, 1.0, rng.uniform(0.4, 1.5))), f32),
            column(lambda: rng.choice((0, 0, 1, 20, 50, 1000, 40000)), i32),
            column(lambda: rng.choice((1.0, 0.9, 0.95, rng.uniform(0.3, 1.0))), f32),
            column(lambda: rng.choice((0.0, 0.0, 0.05, 0.2)), f32))


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape, dtype=torch.float32):
        return torch.randn(*shape, generator=g, device="cuda", dtype=dtype)

    if case["kind"] == "logits":
        # h and W as a trained head has them: rows of W of length about 1, a few rows of h that
        # point at a token
        dt = _dtype(case["dtype"])
        t, d, v = case["rows"], case["hidden"], case["vocab"]
        w = (randn(v, d) / math.sqrt(d)).to(dt)
        h = randn(t, d)
        ids = torch.randint(v, ((t + 1) // 2,), generator=g, device="cuda")
        h[::2] += 12.0 * w[ids].float()
        return dict(h=h.to(dt), w=w)
    if case["kind"] == "sample":
        # A row's bulk is normal, between as wide as an unsure row's and three times that; some
        # tokens stand out, the first by 2 to 20, the others less and less
        t, v, pitch = sum(_blocks(case)), case["vocab"], case["pitch"]
        z = torch.full((t, pitch), float("nan"), device="cuda")
        for r in range(0, t, 128):
            n = min(128, t - r)
            width = 1 + 2 * torch.rand(n, 1, generator=g, device="cuda")
            row = randn(n, v) * width
            first = 2 + 18 * torch.rand(n, 1, generator=g, device="cuda")
            rank = torch.arange(1, LIFTED + 1, device="cuda", dtype=torch.float32)
            lift = torch.clamp(first - 1.5 * torch.log(rank), min=0.0)
            ids = torch.randint(v, (n, LIFTED), generator=g, device="cuda")
            row.scatter_add_(1, ids, lift)
            z[r:r + n, :v] = row
        return dict(z=z.to(_dtype(case["dtype"])),
                    u=torch.rand(t, generator=g, device="cuda"),
                    params=_settings(case, seed))
    new, cached, done, free = _requests(case)
    ps, batch = case["page"], case["batch"]
    have = [(c + ps - 1) // ps for c in cached]
    # a third of the sequences share their first pages with the one before, as prompts that begin
    # alike do
    rng = random.Random(seed * 104729 + case["lens"])
    shared = [0] * batch
    for b in range(1, batch):
        if rng.random() < 1 / 3:
            shared[b] = min(have[b - 1], have[b]) // 2
    n_pages = sum(have) + free + 5
    wide = max((c + n + ps - 1) // ps for n, c in zip(new, cached)) + 1
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32).tolist()
    table = [[-1] * wide for _ in range(batch)]
    at = 0
    for b in range(batch):
        for j in range(have[b]):
            if j < shared[b]:
                table[b][j] = table[b - 1][j]
            else:
                table[b][j] = order[at]
                at += 1
    # a sequence's own pages go back with it; those that the next one shares stay
    keep = [max(shared[b], shared[b + 1] if b + 1 < batch else 0) for b in range(batch)]
    head = rng.randrange(n_pages)
    ring = [-1] * n_pages
    for i in range(free):
        ring[(head + i) % n_pages] = order[at + i]

    def i32(x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")

    return dict(new=i32(new), cached=i32(cached), shared=i32(keep),
                done=torch.tensor(done, dtype=torch.uint8, device="cuda"), table=i32(table),
                ring=i32(ring), state=i32([head, free]))


# --------------------------------------------------------------------------------------------
# prepare / run
# --------------------------------------------------------------------------------------------
def prepare(case, seed):
    x = _inputs(case, seed)
    s = dict(case=case, x=x)

    def out(*shape, dtype=torch.float32):
        return torch.zeros(*shape, dtype=dtype, device="cuda")

    if case["kind"] == "logits":
        if own:
            s["z"] = out(case["rows"], case["vocab"])
    elif case["kind"] == "sample":
        s["blocks"] = _blocks(case)
        t = sum(s["blocks"])
        if own:
            import paper_2609_16450_amd as eb

            s["r"] = eb.Ragged.from_lengths(s["blocks"], [0] * case["batch"])
            s["token"] = out(t, dtype=torch.int32)
            s["prob"], s["conf"] = out(t), out(t)
            need = eb.eb_sample_workspace(eb.EB_F32 if case["dtype"] == "f32" else eb.EB_BF16, t,
                                          case["vocab"])
            s["ws"] = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
    else:
        new, _, done, _ = _requests(case)
        s["rows"] = sum(n for n, d in zip(new, done) if not d)
        batch = case["batch"]
        if own:
            import paper_2609_16450_amd as eb

            s["kv"] = eb.PagedKV.empty(x["ring"].numel(), 1, case["page"], 64, x["table"])
            s["pool"] = eb.PagePool(x["ring"], x["state"])
            s["state_out"] = out(2, dtype=torch.int32)
            s["cu_block"], s["cu_prefix"] = (out(batch + 1, dtype=torch.int32) for _ in range(2))
            s["pos"] = out(s["rows"], dtype=torch.int32)
            s["slot"] = out(s["rows"], dtype=torch.int64)
            s["short"] = out(batch, dtype=torch.uint8)
    if own:
        import paper_2609_16450_amd as eb

        s["eb"] = eb
    return s


def run(s):
    kind, x = s["case"]["kind"], s["x"]
    if not own:
        return {"logits": _plain_logits, "sample": _plain_sample, "assign": _plain_assign}[kind](s)
    eb = s["eb"]
    if kind == "logits":
        eb.eb_lmhead_logits(x["h"], x["w"], s["z"])
        return s["z"]
    if kind == "sample":
        temperature, top_k, top_p, min_p = x["params"]
        eb.eb_sample(s["r"], x["z"], x["u"], s["token"], prob=s["prob"], conf=s["conf"],
                     temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p,
                     vocab=s["case"]["vocab"], ws=s["ws"])
        return s["token"], s["prob"], s["conf"]
    # the state goes to a tensor of its own, so that the same call can be made again
    eb.eb_kv_assign(s["kv"], s["pool"], x["cached"], x["new"], s["cu_block"], s["cu_prefix"],
                    s["pos"], slot=s["slot"], done=x["done"], shared=x["shared"],
                    short=s["short"], state_out=s["state_out"])
    return (x["table"], x["ring"], s["state_out"], s["cu_block"], s["cu_prefix"], s["pos"],
            s["slot"], s["short"])


def _plain_logits(s):
    x = s["x"]
    return x["h"].float() @ x["w"].float().t()


def _per_row(s, column, dtype, default):
    """A sequence's setting for each of its rows, [T, 1]."""
    n = torch.tensor(s["blocks"], device="cuda")
    if column is None:
        return torch.full((sum(s["blocks"]), 1), default, dtype=dtype, device="cuda")
    return torch.repeat_interleave(column.to(dtype), n)[:, None]


def _plain_sample(s):
    x, case = s["x"], s["case"]
    v, f64 = case["vocab"], torch.float64
    temperature, top_k, top_p, min_p = x["params"]
    temp = _per_row(s, temperature, f64, 1.0)
    k = _per_row(s, top_k, torch.int64, 0)
    p = _per_row(s, top_p, f64, 1.0)
    least = _per_row(s, min_p, f64, 0.0)
    rank = torch.arange(v, device="cuda")[None]
    tokens, probs, confs = [], [], []
    for r in range(0, len(k), 128):  # 128 rows at a time: several values of 8 bytes per logit
        rows = slice(r, r + 128)
        z = x["z"][rows, :v].to(f64)
        m = z.amax(1, keepdim=True)
        greedy = temp[rows] <= 0
        w = torch.exp((z - m) / torch.where(greedy, torch.ones_like(m), temp[rows]))
        order = torch.sort(z, dim=1, descending=True, stable=True).indices
        ws = w.gather(1, order)
        n_k = torch.where(k[rows] <= 0, torch.full_like(k[rows], v), k[rows])
        n_k = torch.where(greedy, torch.ones_like(n_k), n_k)
        keep = rank < n_k
        below = torch.cumsum(torch.where(keep, ws, torch.zeros_like(ws)), dim=1)
        before = torch.cat([torch.zeros_like(m), below[:, :-1]], dim=1)
        keep &= (before < p[rows] * below[:, -1:]) | (p[rows] >= 1) | (rank == 0)
        keep &= ws >= least[rows]
        kept = torch.zeros_like(w).scatter_(1, order, torch.where(keep, ws, torch.zeros_like(ws)))
        total = torch.cumsum(kept, dim=1)
        drawn = (total > x["u"][rows, None].to(f64) * total[:, -1:]).to(torch.int32).argmax(1)[:, None]
        tokens.append(drawn)
        probs.append(kept.gather(1, drawn) / total[:, -1:])
        e = torch.exp(z - m)
        confs.append(e.gather(1, drawn) / e.sum(1, keepdim=True))
    return (torch.cat(tokens)[:, 0].to(torch.int32), torch.cat(probs)[:, 0].float(),
            torch.cat(confs)[:, 0].float())


def _plain_assign(s):
    x, ps = s["x"], s["case"]["page"]
    table, ring, n_pages = x["table"], x["ring"], x["ring"].numel()
    batch, wide = table.shape
    live = 1 - x["done"].long()
    new, cached = x["new"].long() * live, x["cached"].long()
    held = (cached + ps - 1) // ps
    want = (cached + new + ps - 1) // ps
    need = torch.where(want <= wide, (want - held) * live, torch.zeros_like(want))
    reach = torch.cumsum(need, 0)
    head, free = x["state"].long()
    served = (want <= wide) & ((need == 0) | (reach <= free))
    back = (held - x["shared"].long()).clamp(min=0) * (1 - live)
    zero = torch.zeros(1, dtype=torch.int64, device="cuda")
    cu_block = torch.cat([zero, torch.cumsum(new, 0)])
    cu_prefix = torch.cat([zero, torch.cumsum(cached * live, 0)])

    # the table: column j of a sequence that gets pages
    column = torch.arange(wide, device="cuda")[None]
    fresh = (column >= held[:, None]) & (column < want[:, None]) & (live[:, None] > 0)
    from_ring = ring[(head + (reach - need)[:, None] + column - held[:, None]) % n_pages]
    minus = torch.full_like(table, -1)
    full = torch.where(fresh, torch.where(served[:, None], from_ring, minus), table)

    # pages of finished sequences go behind the free ones
    gone = (column >= x["shared"].long()[:, None]) & (column < held[:, None]) & (live[:, None] == 0)
    pages = table[gone]
    rings = ring.clone()
    rings[(head + free + torch.arange(len(pages), device="cuda")) % n_pages] = pages

    taken = (need * served).sum()
    state = torch.stack([(head + taken) % n_pages, free - taken + back.sum()])

    seq = torch.repeat_interleave(torch.arange(batch, device="cuda"), new, output_size=s["rows"])
    pos = cached[seq] + torch.arange(s["rows"], device="cuda") - cu_block[seq]
    page = full[seq, (pos // ps).clamp(max=wide - 1)].long()
    ok = served[seq] & (page >= 0)
    none = torch.full_like(pos, -1)
    slot = torch.where(ok, page * ps + pos % ps, none)
    pos = torch.where(served[seq], pos, none)
    i32 = torch.int32
    return (full, rings, state.to(i32), cu_block.to(i32), cu_prefix.to(i32), pos.to(i32), slot,
            (~served).to(torch.uint8))


# --------------------------------------------------------------------------------------------
# the definition in 64 bits, apart from the above
# --------------------------------------------------------------------------------------------
def exact(case, seed):
    x = _inputs(case, seed)
    return {"logits": _exact_logits, "sample": _exact_sample,
            "assign": _exact_assign}[case["kind"]](case, x)


def _exact_logits(case, x):
    h = x["h"].double()
    z = torch.empty(case["rows"], case["vocab"], dtype=torch.float64, device="cuda")
    for v in range(0, case["vocab"], 16384):
        w = x["w"][v:v + 16384].double()
        z[:, v:v + len(w)] = torch.mm(h, w.t().contiguous())
    return z


def _exact_sample(case, x):
    """Row by row, walking the order: how long its kept prefix is, then which id is drawn."""
    v = case["vocab"]
    settings = [None if c is None else c.tolist() for c in x["params"]]
    u = x["u"].tolist()
    tokens, probs, confs = [], [], []
    row = 0
    for b, rows in enumerate(_blocks(case)):
        temp, k, p, least = (d if c is None else c[b] for c, d in zip(settings, (1.0, 0, 1.0, 0.0)))
        for _ in range(rows):
            z = x["z"][row, :v].double()
            top = z.max()
            soft = torch.exp(z - top)
            order = torch.argsort(-z, stable=True)
            if temp <= 0:
                token, prob = int(order[0]), 1.0
            else:
                w = torch.exp((z - top) / temp)
                falling = w[order]
                n = k if 0 < k < v else v
                sums = torch.cumsum(falling[:n], 0)
                if p < 1:
                    first = int(torch.searchsorted(sums, p * sums[-1:])[0])
                    n = min(n, max(first, 0) + 1)
                if least > 0:
                    n = min(n, int((falling >= least).sum()))
                ids = torch.sort(order[:n]).values
                sums = torch.cumsum(w[ids], 0)
                at = min(int(torch.searchsorted(sums, u[row] * sums[-1:], right=True)[0]), n - 1)
                token = int(ids[at])
                prob = float(w[token] / sums[-1])
            tokens.append(token)
            probs.append(prob)
            confs.append(float(soft[token] / soft.sum()))
            row += 1
    return (torch.tensor(tokens, dtype=torch.int32, device="cuda"),
            torch.tensor(probs, dtype=torch.float64, device="cuda"),
            torch.tensor(confs, dtype=torch.float64, device="cuda"))


def _exact_assign(case, x):
    """Sequence after sequence, as a host's allocator would go about it."""
    ps = case["page"]
    table, ring = x["table"].cpu().numpy().copy(), x["ring"].cpu().numpy().copy()
    new, cached, done, shared = (x[n].tolist() for n in ("new", "cached", "done", "shared"))
    head, free = x["state"].tolist()
    n_pages, (batch, wide) = len(ring), table.shape
    taken, demand, back = 0, 0, 0
    cu_block, cu_prefix, pos, slot = [0], [0], [], []
    short = np.zeros(batch, np.uint8)
    for b in range(batch):
        if done[b]:
            for j in range(shared[b], -(-cached[b] // ps)):
                ring[(head + free + back) % n_pages] = table[b, j]
                back += 1
            cu_block.append(cu_block[-1])
            cu_prefix.append(cu_prefix[-1])
            continue
        first, end = -(-cached[b] // ps), -(-(cached[b] + new[b]) // ps)
        fits = end <= wide
        if fits:
            demand += end - first
        if fits and (end == first or demand <= free):
            for j in range(first, end):
                table[b, j] = ring[(head + taken) % n_pages]
                taken += 1
        else:
            short[b] = 1
            table[b, first:end] = -1
        for i in range(new[b]):
            at = cached[b] + i
            pos.append(-1 if short[b] else at)
            page = -1 if short[b] else int(table[b, at // ps])
            slot.append(-1 if page < 0 else page * ps + at % ps)
        cu_block.append(cu_block[-1] + new[b])
        cu_prefix.append(cu_prefix[-1] + cached[b])

    def out(a, dtype=torch.int32):
        return torch.as_tensor(np.asarray(a), device="cuda").to(dtype)

    return (out(table), out(ring), out([(head + taken) % n_pages, free - taken + back]),
            out(cu_block), out(cu_prefix), out(pos), out(slot, torch.int64),
            out(short, torch.uint8))
