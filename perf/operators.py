"""What the speed of the 4-bit paged cache's operators is measured on: planning a step's blocks and slots from request
lengths, writing rows of K and V into the cache (and reading them back), and attention over it.

A case is a dict of plain values:
  kind       "plan" | "append" | "attend"
  heads, kv_heads, head_dim, block   head layout of the cache and positions per block
  dtype      "bf16" | "f32": what K, V and Q come in
  seqs, ctx_lo, ctx_hi   requests and the range of positions they hold after the step (spread evenly over the batch)
  rows       most new rows of a request: 1 = a plain decode step, a few = decode with deferred tokens, many = a prompt's chunk
  ragged     the requests bring 1..rows rows (a spread), some of them none; else all bring `rows`
  short      (plan) the pool holds fewer free blocks than the requests ask for
  fused      K, V and Q are column ranges of one Q|K|V matrix, as a fused projection leaves them
  lse        (attend) the log-sum-exp of each row and head is returned too
  window     (attend) each row sees that many of the latest positions (0: all)

Lengths follow from the case; the seed deals them to the requests and draws the values and the order of the free blocks.

The cache's 4 bits: a group is 32 neighbouring elements of one head's vector.  It shares a power of two 2^e, e the least
integer from -111 to 125 with max|x| <= 7 * 2^e, and each element is held as the nearest of +-{0, 0.5, 1, 1.5, 2, 3, 4, 6}
times it, a tie going to the value with the even index, larger ones to 6.
"""
import random

import numpy as np
import torch

own = False

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
E_MIN, E_MAX = -111, 125

HEADS = [  # heads, kv_heads, head_dim: the widths of the framework's own workloads, then layouts with shared heads
    (4, 4, 32), (12, 12, 64), (16, 16, 128), (32, 32, 128), (52, 52, 128), (32, 8, 128), (16, 2, 64), (28, 4, 128), (8, 1, 128), (20, 4, 64),
]


def listed():
    return [
        # the step of a batch of 16 chats with a few deferred tokens: launch latency
        dict(name="plan_step16", kind="plan", block=64, seqs=16, ctx_lo=256, ctx_hi=2048, rows=4, ragged=True, short=False),
        # a full server's step, some requests finished, some idle, small blocks
        dict(name="plan_step1000", kind="plan", block=16, seqs=1000, ctx_lo=1, ctx_hi=16000, rows=16, ragged=True, short=False),
        # prompts admitted at once, more than the pool holds
        dict(name="plan_admit", kind="plan", block=32, seqs=200, ctx_lo=40, ctx_hi=4096, rows=2048, ragged=True, short=True),
        # K and V of one decode step of the 7B-shaped model's ragged batch, out of the fused projection
        dict(name="append_step16", kind="append", heads=32, kv_heads=32, head_dim=128, block=64, dtype="bf16", seqs=16, ctx_lo=256, ctx_hi=2048,
             rows=3, ragged=True, fused=True),
        # an fp32 model's prompt of an odd length, small heads
        dict(name="append_f32", kind="append", heads=12, kv_heads=12, head_dim=64, block=16, dtype="f32", seqs=1, ctx_lo=777, ctx_hi=777, rows=777,
             ragged=False, fused=False),
        # prompts of a batch, shared heads
        dict(name="append_prompts", kind="append", heads=32, kv_heads=8, head_dim=128, block=64, dtype="bf16", seqs=8, ctx_lo=2000, ctx_hi=8192,
             rows=8192, ragged=False, fused=True),
        # one user of the 1.3B-shaped model: nothing but latency
        dict(name="attend_1b3", kind="attend", heads=16, kv_heads=16, head_dim=128, block=64, dtype="bf16", seqs=1, ctx_lo=513, ctx_hi=513, rows=1,
             ragged=False, fused=True, lse=False, window=0),
        # 16 users of the 7B-shaped model with ragged contexts and deferred tokens
        dict(name="attend_7b_ragged16", kind="attend", heads=32, kv_heads=32, head_dim=128, block=64, dtype="bf16", seqs=16, ctx_lo=256, ctx_hi=2048,
             rows=4, ragged=True, fused=True, lse=False, window=0),
        # a full batch of long chats, shared heads
        dict(name="attend_gqa64", kind="attend", heads=32, kv_heads=8, head_dim=128, block=64, dtype="bf16", seqs=64, ctx_lo=500, ctx_hi=16384, rows=1,
             ragged=False, fused=True, lse=False, window=0),
        # one user with a book in the context and one deferred token; the parts are joined with others', so the log-sum-exp too
        dict(name="attend_long", kind="attend", heads=32, kv_heads=8, head_dim=128, block=64, dtype="bf16", seqs=1, ctx_lo=131071, ctx_hi=131071,
             rows=2, ragged=False, fused=True, lse=True, window=0),
        # an fp32 model, small heads, small blocks, a few ragged requests and a window
        dict(name="attend_f32_window", kind="attend", heads=12, kv_heads=4, head_dim=64, block=16, dtype="f32", seqs=7, ctx_lo=30, ctx_hi=1500, rows=5,
             ragged=True, fused=False, lse=False, window=700),
        # the last chunk of a long prompt
        dict(name="attend_chunk", kind="attend", heads=32, kv_heads=8, head_dim=128, block=64, dtype="bf16", seqs=1, ctx_lo=8192, ctx_hi=8192,
             rows=1024, ragged=False, fused=True, lse=False, window=0),
    ]


def _span(rng, lo, hi):
    v = int(round(lo * (hi / lo) ** rng.random()))
    v += rng.choice((0, 0, 1, -1)) if lo < v < hi else 0
    return v + 1 if v == 3072 else v  # (no workload of the framework has that size)


def _draw(rng):
    kind = rng.choice(("plan", "append", "append", "attend", "attend", "attend", "attend"))
    block = rng.choice((16, 32, 64, 128))
    if kind == "plan":
        lo = _span(rng, 1, 4096)
        return dict(kind=kind, block=block, seqs=_span(rng, 1, 1000), ctx_lo=lo, ctx_hi=max(lo, _span(rng, 16, 16000)), rows=_span(rng, 1, 2048),
                    ragged=True, short=rng.random() < 0.3)
    heads, kv_heads, head_dim = rng.choice(HEADS)
    c = dict(kind=kind, heads=heads, kv_heads=kv_heads, head_dim=head_dim, block=block, dtype=rng.choice(("bf16", "bf16", "f32")))
    if kind == "append":
        rows = _span(rng, 1, 8192)
        lo = _span(rng, 1, 4096)
        c.update(seqs=_span(rng, 1, 32), ctx_lo=lo, ctx_hi=max(lo, _span(rng, 1, 8192)), rows=rows, ragged=rng.random() < 0.5, fused=rng.random() < 0.6)
        return c
    shape = rng.choice(("step", "step", "deferred", "long", "chunk"))
    if shape == "long":
        n = _span(rng, 16384, 131072)
        c.update(seqs=1, ctx_lo=n, ctx_hi=n, rows=rng.choice((1, 1, 2, 3)))
    elif shape == "chunk":
        n = _span(rng, 64, 8192)
        c.update(seqs=rng.choice((1, 1, 2, 3)), ctx_lo=n, ctx_hi=max(n, _span(rng, 64, 8192)), rows=_span(rng, 17, 1024))
    else:
        lo = _span(rng, 1, 4096)
        c.update(seqs=_span(rng, 1, 64), ctx_lo=lo, ctx_hi=max(lo, _span(rng, 16, 16384)), rows=1 if shape == "step" else _span(rng, 2, 16))
    c.update(ragged=rng.random() < 0.5, fused=rng.random() < 0.6, lse=False, window=_span(rng, 64, 4096) if rng.random() < 0.2 else 0)
    return c


def draw(rng):
    most = [work(c) for c in listed()]
    while True:
        c = _draw(rng)
        w = work(c)
        if w["bytes"] <= max(m["bytes"] for m in most) and w["flops"] <= max(m["flops"] for m in most):
            return c


# ---------------------------------------------------------------- lengths

def _lengths(case):
    """(held, start, end) per request, in an order of the case's own: held positions before the step; rows start..end-1 are
    the step's, and end is what the request holds afterwards."""
    n, lo, hi = case["seqs"], case["ctx_lo"], case["ctx_hi"]
    held, start, end = [], [], []
    for i in range(n):
        e = lo + (hi - lo) * i // max(1, n - 1) if n > 1 else hi
        r = min(e, case["rows"])
        if case["ragged"]:
            r = min(e, 1 + (case["rows"] - 1) * ((i * 5) % 8) // 7)
            if i % 8 == 5 and n > 4:
                r = 0  # a request that waits
        s, h = e - r, e - r
        if case["kind"] == "plan":
            if i % 8 == 7:  # a request that has ended gives its blocks back
                h, s, e = e, 0, 0
            elif i % 8 == 3:  # the step before held more: what it held beyond is taken back
                h = e + case["rows"] // 2 + 1
            elif i % 8 == 2:  # the step feeds positions again that the cache holds already
                h = s + r // 2
        held.append(h), start.append(s), end.append(e)
    return held, start, end


def _dealt(case, seed):
    held, start, end = _lengths(case)
    order = list(range(len(held)))
    random.Random(seed * 1000003 + 17).shuffle(order)
    return tuple(np.array([a[i] for i in order], dtype=np.int32) for a in (held, start, end))


def _blocks(tokens, block):
    return (np.asarray(tokens, dtype=np.int64) + block - 1) // block


def _pool(case):
    """Blocks of the pool, positions a request may reach."""
    held, _, end = _lengths(case)
    b = case["block"]
    had, need = _blocks(held, b), _blocks(end, b)
    if case["kind"] == "plan" and case["short"]:
        wanted = int(np.maximum(need - had, 0).sum())
        return int(had.sum()) + max(1, wanted // 2), max(max(end), max(held))
    return int(np.maximum(had, need).sum()) + 8, max(max(end), max(held), 1)


def work(case):
    held, start, end = (np.array(a, dtype=np.int64) for a in _lengths(case))
    rows = int((end - start).sum())
    n = case["seqs"]
    if case["kind"] == "plan":
        moved = int(np.abs(_blocks(end, case["block"]) - _blocks(held, case["block"])).sum())
        return {"bytes": 12 * n + 8 * moved + rows * 16 + 12 * n + 4, "flops": 0}
    es = 2 if case["dtype"] == "bf16" else 4
    hd, kvh, nh = case["head_dim"], case["kv_heads"], case["heads"]
    if case["kind"] == "append":
        # floats in, 4 bits out; read back: 4 bits in, floats out; the slots twice
        return {"bytes": rows * kvh * hd * 2 * (es + 17 / 32) * 2 + rows * 16, "flops": 0}
    w = case["window"] or (1 << 30)
    seen, read = 0, 0
    for s, e in zip(start, end):
        if e > s:
            p = np.arange(s, e)
            seen += int(np.minimum(p + 1, w).sum())
            read += int(e - max(0, s + 1 - w))
    out = rows * nh * hd * es + (rows * nh * 4 if case["lse"] else 0)
    return {"bytes": read * kvh * hd * 17 / 16 + rows * nh * hd * es + out + 4 * read // case["block"] + 16 * n, "flops": 4 * hd * nh * seen}


# ---------------------------------------------------------------- inputs

def _gen(seed, what):
    return torch.Generator(device=DEV).manual_seed((seed * 7919 + what) % (1 << 62))


def _channel_gains(case, seed):
    """Keys have a few loud channels, the same at every position."""
    g = _gen(seed, 3)
    z = torch.randn(case["kv_heads"], case["head_dim"], device=DEV, generator=g)
    return torch.exp(0.5 * z)


def _kv(case, seed, what, n):
    """K and V of n positions, [n][kv_heads][head_dim] each, or (fused) column ranges of one matrix."""
    hd, kvh, nh = case["head_dim"], case["kv_heads"], case["heads"]
    dt, g = DTYPES[case["dtype"]], _gen(seed, what)
    if case["fused"]:
        m = torch.randn(n, nh + 2 * kvh, hd, device=DEV, generator=g).to(dt)
        k, v = m[:, nh:nh + kvh], m[:, nh + kvh:]
    else:
        k = torch.randn(n, kvh, hd, device=DEV, generator=g).to(dt)
        v = torch.randn(n, kvh, hd, device=DEV, generator=g).to(dt)
    k.mul_(_channel_gains(case, seed).to(dt))
    return k, v


def _q(case, seed, rows):
    hd, kvh, nh = case["head_dim"], case["kv_heads"], case["heads"]
    dt, g = DTYPES[case["dtype"]], _gen(seed, 5)
    if case["fused"]:
        return torch.randn(rows, nh + 2 * kvh, hd, device=DEV, generator=g).to(dt)[:, :nh]
    return torch.randn(rows, nh, hd, device=DEV, generator=g).to(dt)


def _order(n_blocks, seed):
    """The free blocks' order in a pool that has been in use for a while."""
    return torch.randperm(n_blocks, device=DEV, generator=_gen(seed, 7)).to(torch.int32)


def _dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def _own_cache(case, max_rows, seed):
    import paper_2312_04916_amd as ee
    n_blocks, max_positions = _pool(case)
    cache = ee.Kv4Cache(1, case.get("heads", 1), case.get("kv_heads", 1), case.get("head_dim", 32), case["block"], n_blocks, case["seqs"],
                        max_positions, max_rows, case.get("dtype", "bf16"))
    cache.free.copy_(_order(n_blocks, seed))
    return cache


def prepare(case, seed):
    held, start, end = _dealt(case, seed)
    n = case["seqs"]
    n_rows = int((end - start).sum())
    n_blocks, max_positions = _pool(case)
    s = dict(case=case, n_rows=n_rows, most=int((end - start).max()), held=_dev(held), start=_dev(start), end=_dev(end))
    before = held if case["kind"] == "plan" else start if case["kind"] == "append" else end
    n_before = int(before.sum()) if case["kind"] == "attend" else 0
    zero = torch.zeros(n, dtype=torch.int32, device=DEV)
    if own:
        s["cache"] = cache = _own_cache(case, max(n_rows, n_before, 1), seed)
        # the requests as they stand before the pass hold their blocks already
        cache.plan(zero, zero if n_before else _dev(before), _dev(before), n_before)
        slots = cache.slots[:n_before].clone()
    else:
        s["table"] = torch.zeros(n, int(_blocks(max_positions, case["block"])), dtype=torch.int32, device=DEV)
        s["free"] = _order(n_blocks, seed)
        p = _plain_plan(case, zero, zero if n_before else _dev(before), _dev(before), s["table"], s["free"], n_before)
        s["table"], s["free"], slots = p["table"], p["free"], p["slots"]
    if case["kind"] == "plan":
        if own:  # (the plan's arrays stay where they are: a program takes their parts once)
            s["arrays"] = (cache.table, cache.slots[:n_rows], cache.positions[:n_rows], cache.row_seq[:n_rows], cache.row_start[:n + 1],
                           cache.served[:n], cache.held_next[:n], cache.n_free)
        return s
    hd, kvh = case["head_dim"], case["kv_heads"]
    if not own:
        size = n_blocks * case["block"]
        s["pool"] = {"k": torch.zeros(size, kvh, hd // 2, dtype=torch.uint8, device=DEV), "v": torch.zeros(size, kvh, hd // 2, dtype=torch.uint8, device=DEV),
                     "ks": torch.zeros(size, kvh, hd // 32, dtype=torch.uint8, device=DEV), "vs": torch.zeros(size, kvh, hd // 32, dtype=torch.uint8, device=DEV)}
    if case["kind"] == "append":
        s["k"], s["v"] = _kv(case, seed, 11, n_rows)
        if own:
            cache.plan(s["start"], s["start"], s["end"], n_rows)
            s["slots"] = cache.slots[:n_rows]
        else:
            p = _plain_plan(case, s["start"], s["start"], s["end"], s["table"], s["free"], n_rows)
            s["table"], s["free"], s["slots"] = p["table"], p["free"], p["slots"]
        return s
    at = 0
    for i in range(n):
        m = int(end[i])
        if m:
            k, v = _kv(case, seed, 100 + i, m)
            if own:
                cache.append(0, k, v, slots[at:at + m])
            else:
                _plain_append(s["pool"], k, v, slots[at:at + m])
        at += m
    s["q"] = _q(case, seed, n_rows)
    if own:
        cache.plan(s["end"], s["start"], s["end"], n_rows, s["most"])
    else:
        s["lengths"] = [(int(a), int(b)) for a, b in zip(start, end)]
    return s


# ---------------------------------------------------------------- the plain forms

def _plain_plan(case, held, start, end, table, free, n_rows):
    b = case["block"]
    n, per = table.shape
    n_blocks = free.numel()
    held, start, end = held.long(), start.long(), end.long()
    had, need = (held + b - 1) // b, (end + b - 1) // b
    give, take = (had - need).clamp_min(0), (need - had).clamp_min(0)
    left = n_blocks - had.sum()
    have = left + give.sum()
    served = (take == 0) | (take.cumsum(0) <= have)
    take_ok = torch.where(served, take, torch.zeros_like(take))
    # blocks that are given back go on the stack last request first, each request's last block first
    j = torch.arange(per, device=DEV)
    gone = (j >= need[:, None]) & (j < had[:, None])
    back = torch.flip(table, (0, 1))[torch.flip(gone, (0, 1))]
    free = free.clone()
    free[left + torch.arange(back.numel(), device=DEV)] = back
    # and are taken from its top in the requests' order
    new = (j >= had[:, None]) & (j < (had + take_ok)[:, None])
    rank = (take_ok.cumsum(0) - take_ok)[:, None] + j - had[:, None]
    table = torch.where(new, free[(have - 1 - rank).clamp(0, n_blocks - 1)], table)
    fresh = end - start
    row_start = torch.cat([torch.zeros(1, dtype=torch.long, device=DEV), fresh.cumsum(0)])
    row = torch.arange(n_rows, device=DEV)
    seq = torch.searchsorted(row_start[1:], row, right=True).clamp_max(n - 1)
    pos = start[seq] + row - row_start[seq]
    slots = table[seq, (pos // b).clamp(0, per - 1)].long() * b + pos % b
    ok = served[seq]
    return dict(table=table, free=free, n_free=(have - take_ok.sum()).to(torch.int32), slots=torch.where(ok, slots, torch.full_like(slots, -1)),
                positions=torch.where(ok, pos, torch.full_like(pos, -1)).to(torch.int32), row_seq=seq.to(torch.int32), row_start=row_start.to(torch.int32),
                served=served.to(torch.int32), held_next=torch.where(served, end, held).to(torch.int32))


def _plain_codes(x):
    """x [..., head_dim] -> codes [..., head_dim / 2] (two a byte, the even element in the low half) and exponents + 127."""
    g = x.float().reshape(*x.shape[:-1], -1, 32)
    top = g.abs().amax(-1)
    m, e = torch.frexp(top)
    e = torch.where(top == 0, torch.full_like(e, E_MIN), e - 3 + (m > 0.875).to(e.dtype)).clamp(E_MIN, E_MAX)
    a = torch.ldexp(g.abs(), -e[..., None])
    c = ((a > 0.25).int() + (a >= 0.75).int() + (a > 1.25).int() + (a >= 1.75).int() + (a > 2.5).int() + (a >= 3.5).int() + (a > 5.0).int())
    c = (c + 8 * (g < 0).int()).to(torch.uint8).reshape(*x.shape[:-1], -1, 2)
    return c[..., 0] | (c[..., 1] << 4), (e + 127).to(torch.uint8)


def _plain_values(codes, exponents):
    lut = torch.tensor(LEVELS + tuple(-v for v in LEVELS), device=DEV)
    c = torch.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], -1, 32)
    return torch.ldexp(lut[c.long()], exponents.int()[..., None] - 127).reshape(*codes.shape[:-1], -1)


def _plain_append(pool, k, v, slots):
    for name, x in (("k", k), ("v", v)):
        c, e = _plain_codes(x)
        pool[name][slots] = c
        pool[name + "s"][slots] = e


def _plain_read(pool, slots, dtype):
    return _plain_values(pool["k"][slots], pool["ks"][slots]).to(dtype), _plain_values(pool["v"][slots], pool["vs"][slots]).to(dtype)


def _plain_attend(s):
    case = s["case"]
    q, b = s["q"], case["block"]
    nh, kvh, hd = case["heads"], case["kv_heads"], case["head_dim"]
    out = torch.zeros(q.shape[0], nh, hd, dtype=q.dtype, device=DEV)
    lse = torch.full((q.shape[0], nh), -torch.inf, device=DEV)
    at = 0
    for i, (lo, hi) in enumerate(s["lengths"]):
        r = hi - lo
        if r == 0:
            continue
        first = max(0, lo + 1 - case["window"]) if case["window"] else 0
        key = torch.arange(first, hi, device=DEV)
        slots = s["table"][i, key // b].long() * b + key % b
        k, v = _plain_read(s["pool"], slots, torch.float32)
        qs = q[at:at + r].float().reshape(r, kvh, nh // kvh, hd).permute(1, 0, 2, 3).reshape(kvh, -1, hd)
        z = torch.matmul(qs, k.permute(1, 2, 0).contiguous()) * hd ** -0.5
        pos = torch.arange(lo, hi, device=DEV).repeat_interleave(nh // kvh)
        hide = key[None, :] > pos[:, None]
        if case["window"]:
            hide |= key[None, :] <= pos[:, None] - case["window"]
        z.masked_fill_(hide, -torch.inf)
        top = z.amax(-1, keepdim=True)
        p = torch.exp(z - top)
        total = p.sum(-1, keepdim=True)
        o = torch.matmul(p, v.permute(1, 0, 2).contiguous()) / total
        out[at:at + r] = o.reshape(kvh, r, nh // kvh, hd).permute(1, 0, 2, 3).reshape(r, nh, hd).to(q.dtype)
        lse[at:at + r] = (top + torch.log(total)).reshape(kvh, r, nh // kvh).permute(1, 0, 2).reshape(r, nh)
        at += r
    return (out, lse) if case["lse"] else (out,)


PLAN_OUT = ("table", "slots", "positions", "row_seq", "row_start", "served", "held_next", "n_free")


def run(s):
    case = s["case"]
    if case["kind"] == "plan":
        if own:
            s["cache"].plan(s["held"], s["start"], s["end"], s["n_rows"], s["most"])
            return s["arrays"]
        p = _plain_plan(case, s["held"], s["start"], s["end"], s["table"], s["free"], s["n_rows"])
        return tuple(p[k] if k != "n_free" else p[k].reshape(1) for k in PLAN_OUT)
    if case["kind"] == "append":
        if own:
            c = s["cache"]
            c.append(0, s["k"], s["v"])
            return c.read(0, s["slots"])
        _plain_append(s["pool"], s["k"], s["v"], s["slots"])
        return _plain_read(s["pool"], s["slots"], s["k"].dtype)
    if own:
        o = s["cache"].attend(0, s["q"], window=case["window"], lse=case["lse"])
        return o if case["lse"] else (o,)
    return _plain_attend(s)


# ---------------------------------------------------------------- the definitions in 64 bits

def _exact_plan(case, seed):
    """One request after the other, as a list of free blocks and a table would be kept by hand."""
    held, start, end = (a.tolist() for a in _dealt(case, seed))
    b = case["block"]
    n_blocks, max_positions = _pool(case)
    stack = _order(n_blocks, seed).tolist()
    table = np.zeros((case["seqs"], -(-max_positions // b)), dtype=np.int64)

    def step(held, start, end):
        had, need = [-(-h // b) for h in held], [-(-e // b) for e in end]
        for i in reversed(range(len(held))):
            for j in reversed(range(need[i], had[i])):
                stack.append(int(table[i, j]))
        asked, have, served = 0, len(stack), []
        for i in range(len(held)):
            asked += max(0, need[i] - had[i])
            served.append(need[i] <= had[i] or asked <= have)
            if served[i]:
                for j in range(had[i], need[i]):
                    table[i, j] = stack.pop()
        return served

    step([0] * len(held), held, held)
    served = step(held, start, end)
    slots, positions, row_seq, row_start = [], [], [], [0]
    for i, ok in enumerate(served):
        p = np.arange(start[i], end[i])
        slots.append(table[i, p // b] * b + p % b if ok else np.full(p.shape, -1))
        positions.append(p if ok else np.full(p.shape, -1))
        row_seq.append(np.full(p.shape, i))
        row_start.append(row_start[-1] + len(p))
    held_next = [e if ok else h for ok, e, h in zip(served, end, held)]
    whole = [table, np.concatenate(slots), np.concatenate(positions), np.concatenate(row_seq), row_start, [int(x) for x in served], held_next, [len(stack)]]
    return tuple(_dev(np.asarray(a, dtype=np.int64)) for a in whole)


def _exact_held(x):
    """What x stands for once it is held in 4 bits, from the definition, in 64 bits."""
    g = x.double().reshape(*x.shape[:-1], -1, 32)
    top = g.abs().amax(-1, keepdim=True)
    unit = torch.full_like(top, 2.0 ** E_MIN)
    for step in (128, 64, 32, 16, 8, 4, 2, 1):  # the least power of two with top <= 7 units
        more = unit * 2.0 ** step
        unit = torch.where(top > 7 * (more / 2), more, unit)
    unit = unit.clamp_max(2.0 ** E_MAX)
    a = g.abs() / unit
    near = torch.where(a < 2, torch.round(a * 2) / 2, torch.where(a < 4, torch.round(a), 2 * torch.round(a / 2))).clamp_max(6.0)
    return (torch.sign(g) * near * unit).reshape(x.shape)


def exact(case, seed):
    if case["kind"] == "plan":
        return _exact_plan(case, seed)
    held, start, end = _dealt(case, seed)
    n_rows = int((end - start).sum())
    if case["kind"] == "append":
        return tuple(_exact_held(x) for x in _kv(case, seed, 11, n_rows))
    nh, kvh, hd = case["heads"], case["kv_heads"], case["head_dim"]
    q = _q(case, seed, n_rows).double()
    out = torch.zeros(n_rows, nh, hd, dtype=torch.float64, device=DEV)
    lse = torch.full((n_rows, nh), -torch.inf, dtype=torch.float64, device=DEV)
    at = 0
    for i in range(case["seqs"]):
        lo, hi = int(start[i]), int(end[i])
        r = hi - lo
        if r == 0:
            continue
        k, v = _kv(case, seed, 100 + i, hi)
        key = torch.arange(hi, device=DEV)
        dist = torch.arange(lo, hi, device=DEV)[:, None] - key[None, :]
        seen = (dist >= 0) & (dist < (case["window"] or 1 << 30))
        for h in range(kvh):
            kh, vh = _exact_held(k[:, h].contiguous()), _exact_held(v[:, h].contiguous())
            for f in range(h * nh // kvh, (h + 1) * nh // kvh):
                z = torch.where(seen, (q[at:at + r, f] / hd ** 0.5) @ kh.T, -torch.inf)
                lse[at:at + r, f] = torch.logsumexp(z, -1)
                out[at:at + r, f] = torch.exp(z - lse[at:at + r, f, None]) @ vh
        at += r
    return (out, lse) if case["lse"] else (out,)
