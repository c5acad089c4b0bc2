"""Measured cases of the paged key/value cache: what a serving program built on the library calls
for it, in plain torch (own = False) or through the package's entry points (own = True).

  write  eb_kv_write: rows of a block go into the cache's pages; an 8-bit cache is read back with
         eb_kv_read in the same pass, so that what it holds comes out as values
  read   eb_kv_read: the cached rows of every sequence, packed, as the dense attention takes them
  attn   eb_block_attn_paged: queries of a block against the cached rows and the block's own

A case holds sizes only.  Ragged lengths come from the case's own "lens" number, so that the work of
a case is known without a GPU; every value comes from the seed given to prepare().
"""
from __future__ import annotations

import math
import random

import torch

own = False

# Attention heads of the shapes that the workloads name, of a small model with 64-wide heads and of
# the toy model of the fp32 tests.
LLADA = dict(hq=32, hkv=32, head_dim=128)
DREAM = dict(hq=28, hkv=4, head_dim=128)
SMALL_HEADS = dict(hq=16, hkv=4, head_dim=64)
TINY = dict(hq=4, hkv=4, head_dim=64)

SIZES = {"f32": 4, "bf16": 2, "e4m3": 1}


def _case(name, kind, heads, dtype, cache, page, batch, block, prefix, lens, **more):
    return dict(name=name, kind=kind, dtype=dtype, cache=cache, page=page, batch=batch,
                block_lo=block[0], block_hi=block[1], prefix_lo=prefix[0], prefix_hi=prefix[1],
                lens=lens, **heads, **more)


def listed():
    return [
        # One user, one token at a time behind a long context: latency is everything.
        _case("attn_token_b1", "attn", DREAM, "bf16", "bf16", 64, 1, (1, 1), (4096, 4096), 1),
        # A served batch, one token each, contexts of very different lengths, 8-bit cache.
        _case("attn_token_b64_e4m3", "attn", DREAM, "bf16", "e4m3", 64, 64, (1, 1), (501, 8192), 2),
        # Ragged blocks of the 8B model: a K/V head per query head, so the cache is read for a
        # handful of queries each; small pages.
        _case("attn_block_llada_b32", "attn", LLADA, "bf16", "bf16", 16, 32, (8, 128),
              (2048, 2048), 3),
        # The base block of 32 behind odd contexts, 8-bit cache.
        _case("attn_block_llada_b16_e4m3", "attn", LLADA, "bf16", "e4m3", 32, 16, (32, 32),
              (1001, 4096), 4),
        # A full batch of blocks of very different lengths, grouped heads.
        _case("attn_block_dream_b64", "attn", DREAM, "bf16", "bf16", 64, 64, (16, 256),
              (4096, 4096), 5),
        # A prompt taken in chunks: many new rows behind a long, odd context, 8-bit cache.
        _case("attn_chunk_dream_e4m3", "attn", DREAM, "bf16", "e4m3", 128, 2, (1000, 2048),
              (7001, 12000), 6),
        # The toy model in fp32, as in unit tests and debugging.
        _case("attn_tiny_f32", "attn", TINY, "f32", "f32", 16, 1, (32, 32), (96, 96), 7),
        # One block goes into the cache once it is done: the smallest write.
        _case("write_block_b1", "write", DREAM, "bf16", "bf16", 64, 1, (32, 32), (512, 512), 8,
              scatter=False),
        # The committed rows of a full batch of blocks, at their positions, the others left out.
        _case("write_commit_b64", "write", DREAM, "bf16", "bf16", 64, 64, (16, 256), (1, 300), 9,
              scatter=True),
        # Prompts into an 8-bit cache, and back as values.
        _case("write_prompt_llada_e4m3", "write", LLADA, "bf16", "e4m3", 64, 8, (501, 2048), (0, 0),
              10, scatter=False),
        # One user's bf16 cache, packed for the dense step.
        _case("read_llada_b1", "read", LLADA, "bf16", "bf16", 32, 1, (0, 0), (512, 512), 11),
        # A full batch's 8-bit cache, packed for the dense step.
        _case("read_dream_b64_e4m3", "read", DREAM, "bf16", "e4m3", 64, 64, (0, 0), (1001, 4096),
              12),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _span(rng, lo, hi):
    a = _log_int(rng, lo, hi)
    return (a, a) if rng.random() < 0.4 else (max(lo, a // rng.choice((2, 4, 8))), a)


# no drawn case reads more or computes more than the largest listed ones
MOST_BYTES, MOST_FLOPS = 1.0e9, 0.55e12


def draw(rng):
    kind = rng.choice(("attn", "attn", "attn", "write", "read"))
    f32 = rng.random() < 0.15
    dtype = "f32" if f32 else "bf16"
    heads = rng.choice((TINY, SMALL_HEADS)) if f32 else rng.choice((LLADA, DREAM, DREAM,
                                                                    SMALL_HEADS))
    case = dict(kind=kind, dtype=dtype, cache=rng.choice((dtype, "e4m3")),
                page=rng.choice((16, 32, 64, 128, 256)), batch=_log_int(rng, 1, 4 if f32 else 64),
                lens=rng.randrange(1 << 20), **heads)
    if kind == "read":
        block, prefix = (0, 0), _span(rng, 1, 512 if f32 else 8192)
    elif kind == "write":
        block, prefix = _span(rng, 1, 256 if f32 else 2048), _span(rng, 1, 512)
        case["scatter"] = rng.random() < 0.5
    else:
        block = (1, 1) if rng.random() < 0.35 else _span(rng, 2, 64 if f32 else 1024)
        prefix = _span(rng, 1, 1024 if f32 else 16384)
    case.update(block_lo=block[0], block_hi=block[1], prefix_lo=prefix[0], prefix_hi=prefix[1])
    while case["batch"] > 1:
        w = work(case)
        if w["bytes"] <= MOST_BYTES and w["flops"] <= MOST_FLOPS:
            break
        case["batch"] = (case["batch"] + 1) // 2
    return case


# --------------------------------------------------------------------------------------------
# sizes and work
# --------------------------------------------------------------------------------------------
def _lens(case):
    """New rows and cached rows of every sequence (fixed by the case)."""
    rng = random.Random(case["lens"])
    block = [rng.randint(case["block_lo"], case["block_hi"]) for _ in range(case["batch"])]
    prefix = [rng.randint(case["prefix_lo"], case["prefix_hi"]) for _ in range(case["batch"])]
    return block, prefix


def _after(case):
    """Rows that each sequence's cache spans after a write: rows at given positions leave gaps."""
    block, prefix = _lens(case)
    return [p + (2 * b if case["scatter"] else b) for b, p in zip(block, prefix)]


def work(case):
    block, prefix = _lens(case)
    rows, cached = sum(block), sum(prefix)
    e, hq, hkv, d = SIZES[case["dtype"]], case["hq"], case["hkv"], case["head_dim"]
    row = hkv * d * e                                                  # a row of K or of V
    held = hkv * (d * SIZES[case["cache"]] + (case["cache"] == "e4m3"))  # the same in the cache

    def pages(lens):
        return 4 * sum((n + case["page"] - 1) // case["page"] for n in lens)

    if case["kind"] == "read":
        return {"bytes": 2 * cached * (held + row) + pages(prefix), "flops": 0}
    if case["kind"] == "write":
        pos = 4 * rows if case["scatter"] else 0
        moved = 2 * rows * (row + held) + pos + pages(block)
        if case["cache"] == "e4m3":  # and read back
            moved += 2 * sum(_after(case)) * (held + row) + pages(_after(case))
        return {"bytes": moved, "flops": 0}
    return {"bytes": 2 * rows * e * d * hq + 2 * rows * row + 2 * cached * held + pages(prefix),
            "flops": 4 * hq * d * sum(b * (b + p) for b, p in zip(block, prefix))}


# --------------------------------------------------------------------------------------------
# inputs (plain torch; shared by prepare() and exact())
# --------------------------------------------------------------------------------------------
def _dtype(name):
    return {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}[name]


def _pow2(e):
    """2^e for whole e in fp32, by its bits: a power function may be off by a bit, and the values
    next to it are often ties."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _inputs(case, seed):
    """Keys, values and queries about N(0, 1), the heads' channels of different sizes (a few of the
    keys' channels stand out in trained models); the pool's pages handed out in no order."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    block, prefix = _lens(case)
    hq, hkv, d, ps = case["hq"], case["hkv"], case["head_dim"], case["page"]
    dt = _dtype(case["dtype"])
    size = torch.exp(0.5 * torch.randn(2, hkv, 1, d, generator=g, device="cuda"))

    def rows(n, heads, which):
        x = torch.randn(n, heads, d, generator=g, device="cuda")
        return x if which is None else x * size[which].squeeze(1)

    spans = _after(case) if case["kind"] == "write" else prefix
    need = [(n + ps - 1) // ps for n in spans]
    n_pages, wide = sum(need) + 3, max(max(need), 1)
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((case["batch"], wide), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    x = dict(table=table)
    for i, name in enumerate("kv"):
        wide_dt = dt if case["cache"] == "f32" else torch.bfloat16
        pool = torch.randn(n_pages, hkv, ps, d, generator=g, device="cuda", dtype=wide_dt)
        pool = pool.mul_(size[i].to(wide_dt))
        if case["cache"] == "e4m3":
            # as a writer leaves a pool: the largest value of a row lies in (224, 448] 2^e
            e = torch.ceil(torch.log2(pool.abs().amax(-1, keepdim=True).float() / 448.0))
            x[name + "_scale"] = (e.squeeze(-1) + 127).to(torch.uint8)
            x[name + "_pool"] = (pool * _pow2(-e)).to(_dtype("e4m3"))
        else:
            x[name + "_pool"] = pool
    if case["kind"] != "read":
        x["k"], x["v"] = (rows(sum(block), hkv, i).to(dt) for i in range(2))
    if case["kind"] == "attn":
        x["q"] = rows(sum(block), hq, None).to(dt)
    if case["kind"] == "write" and case["scatter"]:
        # positions in order with gaps behind the cached rows; a third of the rows stay uncommitted
        pos = []
        r = torch.rand(2, sum(block), generator=g, device="cuda").cpu()
        i = 0
        for b, p in zip(block, prefix):
            for j in range(b):
                pos.append(p + 2 * j + int(r[0, i] < 0.5) if r[1, i] > 1 / 3 else -1)
                i += 1
        x["pos"] = torch.tensor(pos, dtype=torch.int32, device="cuda")
    return x


# --------------------------------------------------------------------------------------------
# prepare / run
# --------------------------------------------------------------------------------------------
def prepare(case, seed):
    x = _inputs(case, seed)
    block, prefix = _lens(case)
    s = dict(case=case, x=x, block=block, prefix=prefix)
    if case["kind"] == "write":
        s["spans"] = _after(case)
    if own:
        import paper_2609_16450_amd as eb

        s["eb"] = eb
        s["r"] = eb.Ragged.from_lengths(block, prefix)
        s["kv"] = eb.PagedKV(x["k_pool"], x["v_pool"], x["table"], k_scale=x.get("k_scale"),
                             v_scale=x.get("v_scale"))
        total = sum(s["spans"] if case["kind"] == "write" else prefix)
        if case["kind"] == "attn":
            s["out"] = torch.zeros_like(x["q"])
            need = eb.eb_block_attn_paged_workspace(
                eb.EB_F32 if case["dtype"] == "f32" else eb.EB_BF16, s["r"], s["kv"], case["hq"])
            s["ws"] = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
        elif case["kind"] == "read" or case["cache"] == "e4m3":
            s["rows"] = [torch.zeros(total, case["hkv"], case["head_dim"],
                                     dtype=_dtype(case["dtype"]), device="cuda") for _ in "kv"]
            s["r_read"] = (s["r"] if case["kind"] == "read" else
                           eb.Ragged.from_lengths([0] * case["batch"], s["spans"]))
    return s


def run(s):
    kind, x = s["case"]["kind"], s["x"]
    if not own:
        return {"attn": _plain_attn, "write": _plain_write, "read": _plain_read}[kind](s)
    eb = s["eb"]
    if kind == "attn":
        eb.eb_block_attn_paged(s["r"], s["kv"], x["q"], x["k"], x["v"], s["out"], ws=s["ws"])
        return s["out"]
    if kind == "write":
        eb.eb_kv_write(s["r"], s["kv"], x["k"], x["v"], pos=x.get("pos"))
        if s["case"]["cache"] != "e4m3":
            return x["k_pool"], x["v_pool"]
    eb.eb_kv_read(s["r_read"], s["kv"], *s["rows"])
    return tuple(s["rows"])


def _plain_rows(s, name, b, n):
    """The first n cached rows of sequence b as values: [hkv, n, d] in fp32."""
    x, ps = s["x"], s["case"]["page"]
    page = x["table"][b, :(n + ps - 1) // ps].long()
    pool = x[name + "_pool"][page]                                     # [pages, hkv, ps, d]
    rows = pool.float()
    if name + "_scale" in x:
        rows = rows * _pow2(x[name + "_scale"][page].int() - 127)[..., None]
    _, hkv, _, d = rows.shape
    return rows.transpose(0, 1).reshape(hkv, -1, d)[:, :n]


def _plain_read(s, spans=None):
    spans = s["prefix"] if spans is None else spans
    dt = _dtype(s["case"]["dtype"])
    return tuple(torch.cat([_plain_rows(s, name, b, n).transpose(0, 1).to(dt)
                            for b, n in enumerate(spans)]) for name in "kv")


def _plain_write(s):
    case, x, ps = s["case"], s["x"], s["case"]["page"]
    dev = x["table"].device
    n = torch.tensor(s["block"], device=dev)
    seq = torch.repeat_interleave(torch.arange(case["batch"], device=dev), n)
    if "pos" in x:
        pos = x["pos"].long()
    else:
        first = torch.cumsum(n, 0) - n
        pos = torch.arange(len(seq), device=dev) - first[seq] + torch.tensor(s["prefix"],
                                                                             device=dev)[seq]
    keep = torch.nonzero(pos >= 0).squeeze(1)
    seq, pos = seq[keep], pos[keep]
    page, slot = x["table"][seq, pos // ps].long(), pos % ps
    for name in "kv":
        rows = x[name][keep]
        if case["cache"] != "e4m3":
            x[name + "_pool"][page, :, slot] = rows
            continue
        y = rows.float()
        # the power of two that brings the row's largest value into (224, 448]
        mant, expo = torch.frexp(y.abs().amax(-1))                     # a = mant 2^expo, [1/2, 1)
        e = torch.clamp(expo - 9 + (mant > 0.875).int(), -100, 120)
        y = y * _pow2(-e)[..., None]
        x[name + "_pool"].view(torch.uint8)[page, :, slot] = y.to(_dtype("e4m3")).view(torch.uint8)
        x[name + "_scale"][page, :, slot] = (e + 127).to(torch.uint8)
    if case["cache"] != "e4m3":
        return x["k_pool"], x["v_pool"]
    return _plain_read(s, s["spans"])


def _plain_attn(s):
    case, x = s["case"], s["x"]
    hq, hkv, d = case["hq"], case["hkv"], case["head_dim"]
    out, at = [], 0
    for b, (n, p) in enumerate(zip(s["block"], s["prefix"])):
        k, v = (torch.cat([_plain_rows(s, name, b, p),
                           x[name][at:at + n].float().transpose(0, 1)], dim=1) for name in "kv")
        q = x["q"][at:at + n].float().reshape(n, hkv, hq // hkv, d).permute(1, 0, 2, 3)
        q = q.reshape(hkv, -1, d)
        got = []
        for g in range(hkv):
            z = (q[g] @ k[g].t().contiguous()) * d ** -0.5
            w = torch.exp(z - z.amax(-1, keepdim=True))
            got.append((w @ v[g].contiguous()) / w.sum(-1, keepdim=True))
        o = torch.stack(got).reshape(hkv, n, hq // hkv, d).permute(1, 0, 2, 3)
        out.append(o.reshape(n, hq, d))
        at += n
    return torch.cat(out).to(_dtype(case["dtype"]))


# --------------------------------------------------------------------------------------------
# the same outputs in 64 bits, from the definitions
# --------------------------------------------------------------------------------------------
def _exact_pow2(e):
    """2^e for whole e in 64 bits, by its bits."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_values(x, name):
    """What the pool holds, [pages, hkv, ps, d] in 64 bits."""
    pool = x[name + "_pool"]
    if name + "_scale" not in x:
        return pool.double()
    bits = pool.view(torch.uint8).to(torch.int64)
    sign, expo, frac = bits >> 7, (bits >> 3) & 15, (bits & 7).double()
    mag = torch.where(expo > 0, (8.0 + frac) * _exact_pow2(expo - 10), frac * 2.0 ** -9)
    value = torch.where(sign > 0, -mag, mag)
    return value * _exact_pow2(x[name + "_scale"].long() - 127).unsqueeze(-1)


def _exact_e4m3(rows):
    """Rows [n, d] rounded as the 8-bit cache holds them: 2^e times a multiple of the step of the
    value's binade (steps of 2^-9 below 2^-6), ties to even."""
    rows = rows.double()
    most = torch.clamp(rows.abs().amax(-1, keepdim=True), min=1e-60)
    e = torch.round(torch.log2(most / 448.0)).long()                   # to a whole number or one off
    e = torch.where(most > 448.0 * _exact_pow2(e), e + 1, e)
    e = torch.where(most <= 448.0 * _exact_pow2(e - 1), e - 1, e).clamp(-100, 120)
    y = rows / _exact_pow2(e)
    mag = torch.clamp(y.abs(), min=2.0 ** -6)
    binade = torch.round(torch.log2(mag)).long()
    binade = torch.where(_exact_pow2(binade) > mag, binade - 1, binade)
    step = _exact_pow2(binade - 3)
    return torch.round(y / step) * step * _exact_pow2(e)


def exact(case, seed):
    x = _inputs(case, seed)
    block, prefix = _lens(case)
    ps, hq, hkv, d = case["page"], case["hq"], case["hkv"], case["head_dim"]
    host = x["table"].cpu()
    held = {name: _exact_values(x, name) for name in "kv"}

    def cached(name, b, n):                                            # [n, hkv, d]
        if n == 0:
            return held[name].new_zeros(0, hkv, d)
        return torch.cat([held[name][int(host[b, j])].transpose(0, 1)
                          for j in range((n + ps - 1) // ps)])[:n]

    if case["kind"] == "write":
        pos = x["pos"].cpu().tolist() if "pos" in x else None
        for name in "kv":
            new = x[name].double()
            if case["cache"] == "e4m3":
                new = _exact_e4m3(new.reshape(-1, d)).reshape(new.shape)
            i = 0
            src, page, slot = [], [], []
            for b, (n, p) in enumerate(zip(block, prefix)):
                for j in range(n):
                    at = p + j if pos is None else pos[i]
                    if at >= 0:
                        src.append(i)
                        page.append(int(host[b, at // ps]))
                        slot.append(at % ps)
                    i += 1
            if src:
                held[name][page, :, slot] = new[src]
        if case["cache"] != "e4m3":
            return held["k"], held["v"]
    if case["kind"] != "attn":
        spans = _after(case) if case["kind"] == "write" else prefix
        return tuple(torch.cat([cached(name, b, n) for b, n in enumerate(spans)]) for name in "kv")
    out, at = torch.zeros(x["q"].shape, dtype=torch.float64, device="cuda"), 0
    for b, n in enumerate(block):
        rows = slice(at, at + n)
        at += n
        k, v = (torch.cat([cached(name, b, prefix[b]), x[name][rows].double()]) for name in "kv")
        q = x["q"][rows].double()
        for h in range(hq):
            g = h // (hq // hkv)
            z = q[:, h] @ k[:, g].t().contiguous() / math.sqrt(d)
            out[rows, h] = torch.softmax(z, dim=-1) @ v[:, g].contiguous()
    return out
