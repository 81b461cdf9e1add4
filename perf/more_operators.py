"""What the speed of two operators of a decode step is measured on: products with weights held in 8 bits, and the choice of the
next token from logits and given random numbers.

A case is a dict of plain values:
  kind     "f8" | "sample"
  f8       rows m of x times a weight [n][k]
    m, n, k
    x, y     "bf16" | "f32": what x comes in and what the result is
    pair     a gate and an up weight of n rows each: the result is silu(x Wg^T) * (x Wu^T)
    add      rows of the result's shape are added (the residual stream)
  sample   rows of logits
    rows, vocab
    dtype    "bf16" | "f32"
    params   "plain": temperature alone; "nucleus": temperature and top-p; "mixed": each row with its own temperature (some 0),
             top-k, top-p and min-p, some of them off
    masked   part of the tokens is masked with -inf, in some rows all of them
    scores   the log-probability of the token and the largest probability are returned too

The 8 bits: a group is 128 neighbouring elements of a row of x, or a block of 128 x 128 of a weight (the last ones may be
smaller).  It shares a power of two 2^e, e the least integer from -110 to 120 with max|x| <= 448 * 2^e, and each element is held as
the nearest value that e4m3 has times 2^e, ties going to the even code.  Sums of products are not rounded before the result.

Sampling: tokens are ordered by logit z, the largest first, equal ones by index; a token's weight is exp((z - z_max) / temperature).
Kept are the first top_k (0: all); of these the shortest run from the start whose weights reach top_p of theirs (1: all); of
these the ones with z_max - z <= -ln(min_p) * temperature (0: all).  The token is the first one, by index, at which the running sum of
the kept weights exceeds u times their total.  Temperature 0: the first of the order.  A row with nothing above -inf: -1, with
log-probability -inf and confidence 0.
"""
import math

import torch

own = False

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
E_MIN, E_MAX, TOP = -110, 120, 448.0

SHAPES = [(2048, 5504), (4096, 11008), (6656, 17920)]  # widths of the framework's own workloads: d, d_ff
VOCAB = 50304


def _f8(name, m, n, k, x="bf16", y="bf16", pair=False, add=False):
    return dict(name=name, kind="f8", m=m, n=n, k=k, x=x, y=y, pair=pair, add=add)


def listed():
    return [
        # one user of the 1.3B-shaped model, the fused Q|K|V projection: nothing but latency
        _f8("f8_step1_qkv", 1, 3 * 2048, 2048),
        # one user of the 7B-shaped model, the output matrix of an exit: the widest weight that a step streams
        _f8("f8_step1_head", 1, VOCAB, 4096, y="f32"),
        # a batch of 16 of the 7B-shaped model, gate and up
        _f8("f8_step16_swiglu", 16, 11008, 4096, pair=True),
        # the same batch with its deferred tokens, the MLP's way back to the residual stream
        _f8("f8_rows61_down", 61, 4096, 11008, add=True),
        # a large ragged step of the 30B-shaped model, the output projection
        _f8("f8_rows203_oproj", 203, 6656, 6656, add=True),
        # a prompt's Q|K|V
        _f8("f8_prompt_qkv", 1024, 3 * 4096, 4096),
        # several prompts at once, gate and up: the most work that a call does
        _f8("f8_prompts_swiglu", 4096, 11008, 4096, pair=True),
        # an fp32 model of odd sizes
        _f8("f8_odd_f32", 777, 1001, 1003, x="f32", y="f32"),
        # one user: a token from the logits of one head
        dict(name="sample_1", kind="sample", rows=1, vocab=VOCAB, dtype="f32", params="nucleus", masked=False, scores=True),
        # a batch of 16, each with its own settings
        dict(name="sample_16", kind="sample", rows=16, vocab=VOCAB, dtype="bf16", params="mixed", masked=False, scores=True),
        # the largest step, some requests under a grammar's mask
        dict(name="sample_64", kind="sample", rows=64, vocab=VOCAB, dtype="f32", params="mixed", masked=True, scores=True),
        # a full server's step, temperature alone
        dict(name="sample_512", kind="sample", rows=512, vocab=VOCAB, dtype="f32", params="plain", masked=False, scores=False),
    ]


def _span(rng, lo, hi):
    v = int(round(lo * (hi / lo) ** rng.random()))
    return v + rng.choice((0, 0, 1, -1)) if lo < v < hi else v


def _draw(rng):
    if rng.random() < 0.6:
        d, f = rng.choice(SHAPES)
        n, k, pair, add = rng.choice([(3 * d, d, False, False), (d, d, False, True), (f, d, True, False), (d, f, False, True), (VOCAB, d, False, False)]
                                     + 4 * [(_span(rng, 1, 20000), _span(rng, 1, 12000), rng.random() < 0.3, rng.random() < 0.3)])
        y = rng.choice(("bf16", "bf16", "bf16", "f32"))
        return dict(kind="f8", m=_span(rng, 1, 4096), n=n, k=k, x=rng.choice(("bf16", y)), y=y, pair=pair, add=add)
    return dict(kind="sample", rows=_span(rng, 1, 512), vocab=rng.choice((VOCAB, _span(rng, 1, 200000))), dtype=rng.choice(("bf16", "f32")),
                params=rng.choice(("plain", "nucleus", "mixed", "mixed")), masked=rng.random() < 0.3, scores=rng.random() < 0.5)


def draw(rng):
    while True:
        c = _draw(rng)
        w = work(c)
        most = [work(m) for m in listed() if m["kind"] == c["kind"]]
        if c in [{a: b for a, b in m.items() if a != "name"} for m in listed()]:
            continue
        if w["bytes"] <= max(m["bytes"] for m in most) and w["flops"] <= max(m["flops"] for m in most):
            return c


def _size(name):
    return 2 if name == "bf16" else 4


def work(case):
    if case["kind"] == "sample":
        rows = case["rows"]
        return {"bytes": rows * (case["vocab"] * _size(case["dtype"]) + 20 + 4 + (8 if case["scores"] else 0)), "flops": 0}
    m, n, k = case["m"], case["n"], case["k"]
    w = 2 if case["pair"] else 1
    blocks = -(-n // 128) * -(-k // 128)
    return {"bytes": w * (n * k + blocks) + m * k * _size(case["x"]) + m * n * _size(case["y"]) * (2 if case["add"] else 1), "flops": 2 * w * m * n * k}


# ---------------------------------------------------------------- inputs

def _gen(seed, what):
    return torch.Generator(device=DEV).manual_seed((seed * 7919 + what) % (1 << 62))


def _weight(case, seed, what):
    """Rows of a trained weight differ in their norm, and so do its columns."""
    g, n, k = _gen(seed, what), case["n"], case["k"]
    w = torch.randn(n, k, device=DEV, generator=g) * (0.7 / math.sqrt(k))
    w *= torch.exp(0.3 * torch.randn(n, 1, device=DEV, generator=g))
    w *= torch.exp(0.3 * torch.randn(1, k, device=DEV, generator=g))
    return w.to(DTYPES["bf16" if case["x"] == "bf16" else "f32"])


def _rows(case, seed):
    """Normalised rows with a few loud channels, the same in every row."""
    g, m, k = _gen(seed, 3), case["m"], case["k"]
    x = torch.randn(m, k, device=DEV, generator=g)
    x *= torch.exp(0.7 * torch.randn(k, device=DEV, generator=g))
    return x.to(DTYPES[case["x"]])


def _added(case, seed):
    return torch.randn(case["m"], case["n"], device=DEV, generator=_gen(seed, 4)).to(DTYPES[case["y"]])


def _logits(case, seed):
    """A head's logits: a broad bulk, and a few dozen candidates above it, more of them in some rows than in others."""
    g, rows, vocab = _gen(seed, 5), case["rows"], case["vocab"]
    z = torch.randn(rows, vocab, device=DEV, generator=g) * 2.0
    n = min(vocab, 40)
    at = torch.randint(0, vocab, (rows, n), device=DEV, generator=g)
    lift = 4.0 + 6.0 * torch.rand(rows, 1, device=DEV, generator=g) + 1.5 * torch.randn(rows, n, device=DEV, generator=g)
    z.scatter_add_(1, at, lift)
    if case["masked"]:
        part = torch.rand(rows, 1, device=DEV, generator=g)
        z.masked_fill_(torch.rand(rows, vocab, device=DEV, generator=g) < part, -torch.inf)
        z.masked_fill_((torch.arange(rows, device=DEV) % 11 == 7)[:, None], -torch.inf)
    return z.to(DTYPES[case["dtype"]])


def _settings(case, seed):
    """u, temperature, top_k, top_p, min_p per row."""
    g, rows = _gen(seed, 6), case["rows"]
    u = torch.rand(rows, device=DEV, generator=g)
    r = torch.rand(4, rows, device=DEV, generator=g)
    t = 0.5 + 0.7 * r[0]
    if case["params"] == "plain":
        return u, t, None, None, None
    if case["params"] == "nucleus":
        return u, t, None, 0.8 + 0.19 * r[2], None
    i = torch.arange(rows, device=DEV)
    t = torch.where(i % 8 == 5, torch.zeros_like(t), t)
    top_k = torch.where(i % 4 == 1, torch.zeros_like(i), (1 + 200 * r[1] ** 2).long()).to(torch.int32)
    top_p = torch.where(i % 5 == 2, torch.ones_like(t), 0.7 + 0.29 * r[2])
    min_p = torch.where(i % 3 == 0, torch.zeros_like(t), 0.1 * r[3])
    return u, t, top_k, top_p, min_p


def prepare(case, seed):
    if case["kind"] == "sample":
        return dict(case=case, z=_logits(case, seed), settings=_settings(case, seed))
    s = dict(case=case, x=_rows(case, seed), add=_added(case, seed) if case["add"] else None)
    ws = [_weight(case, seed, 1)] + ([_weight(case, seed, 2)] if case["pair"] else [])
    # a program lays its weights out once
    if own:
        import paper_2312_04916_amd as ee
        s["w"] = ee.F8Weight(ws[0], up=ws[1]) if case["pair"] else ee.F8Weight(ws[0])
    else:
        s["w"] = [_plain_held_weight(w) for w in ws]
    return s


# ---------------------------------------------------------------- the plain forms

def _plain_held(g):
    """Groups in the last dimension -> the values that stand for them."""
    top = g.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(top)
    e = torch.where(top == 0, torch.full_like(e, E_MIN), e - 9 + (m > 0.875).to(e.dtype)).clamp(E_MIN, E_MAX)
    return torch.ldexp(torch.ldexp(g, -e).to(torch.float8_e4m3fn).float(), e)


def _plain_held_rows(x):
    m, k = x.shape
    p = torch.nn.functional.pad(x.float(), (0, -k % 128))
    return _plain_held(p.view(m, -1, 128)).view(m, -1)[:, :k]


def _plain_held_weight(w):
    n, k = w.shape
    p = torch.nn.functional.pad(w.float(), (0, -k % 128, 0, -n % 128))
    a, b = p.shape[0] // 128, p.shape[1] // 128
    g = p.view(a, 128, b, 128).permute(0, 2, 1, 3).reshape(a, b, -1)
    return _plain_held(g).view(a, b, 128, 128).permute(0, 2, 1, 3).reshape(p.shape)[:n, :k].contiguous()


def _plain_f8(s):
    case = s["case"]
    x = _plain_held_rows(s["x"])
    y = torch.matmul(x, s["w"][0].t())
    if case["pair"]:
        y = y / (1 + torch.exp(-y)) * torch.matmul(x, s["w"][1].t())
    if case["add"]:
        y = y + s["add"].float()
    return y.to(DTYPES[case["y"]])


def _plain_sample(s):
    z, (u, t, top_k, top_p, min_p) = s["z"].double(), s["settings"]
    rows, vocab = z.shape
    t = t.double()[:, None]
    zs, order = torch.sort(z, dim=-1, descending=True, stable=True)
    best = zs[:, :1]
    some = best[:, 0] > -torch.inf
    below = torch.where(zs > -torch.inf, best - zs, torch.inf)
    w = torch.exp(-below / torch.where(t > 0, t, torch.ones_like(t)))
    at = torch.arange(vocab, device=DEV)
    kept = torch.ones_like(w, dtype=torch.bool)
    if top_k is not None:
        k = torch.where(top_k > 0, top_k.long(), vocab)[:, None]
        kept &= at < k
        w = w * kept
    if top_p is not None:
        p = top_p.double()[:, None]
        run = w.cumsum(-1)
        before = torch.cat([torch.zeros_like(best), run[:, :-1]], -1)
        kept &= (before < p * run[:, -1:]) | (p >= 1) | (at == 0)
    if min_p is not None:
        m = min_p.double()[:, None]
        kept &= below <= torch.where(m > 0, -torch.log(m) * t, torch.inf)
    kept &= (t > 0) | (at == 0)
    chosen = torch.zeros_like(w).scatter_(1, order, w * kept)
    run = chosen.cumsum(-1)
    token = (run <= u.double()[:, None] * run[:, -1:]).sum(-1).clamp_max(vocab - 1)
    token = torch.where(some, token, -1)
    if not s["case"]["scores"]:
        return token.to(torch.int32)
    total = torch.exp(-below).sum(-1)
    mine = z.gather(1, token.clamp_min(0)[:, None])[:, 0]
    logprob = torch.where(some, mine - best[:, 0] - torch.log(total), -torch.inf)
    return token.to(torch.int32), logprob.float(), torch.where(some, 1 / total, 0.0).float()


def run(s):
    case = s["case"]
    if not own:
        return _plain_f8(s) if case["kind"] == "f8" else _plain_sample(s)
    if case["kind"] == "f8":
        return s["w"].matmul(s["x"], add=s["add"], dtype=DTYPES[case["y"]])
    import paper_2312_04916_amd as ee
    u, t, top_k, top_p, min_p = s["settings"]
    return ee.sample(s["z"], u, temperature=t, top_k=top_k, top_p=top_p, min_p=min_p, scores=case["scores"])


# ---------------------------------------------------------------- the definitions in 64 bits

def _exact_held(x, rows):
    """What x stands for in 8 bits, from the definition; groups of `rows` x 128."""
    x = x.double()
    n, k = x.shape
    top = torch.zeros(-(-n // rows) * rows, -(-k // 128) * 128, dtype=torch.float64, device=DEV)
    top[:n, :k] = x.abs()
    top = top.view(-1, rows, top.shape[1] // 128, 128).amax((1, 3))
    unit = torch.full_like(top, 2.0 ** E_MIN)
    for step in (128, 64, 32, 16, 8, 4, 2, 1):  # the least power of two with top <= 448 units
        unit = torch.where(top > TOP * unit * 2.0 ** (step - 1), unit * 2.0 ** step, unit)
    unit = unit.clamp_max(2.0 ** E_MAX).repeat_interleave(rows, 0)[:n].repeat_interleave(128, 1)[:, :k]
    a = x.abs() / unit
    # steps of an eighth of the power of two below, 2^-9 at least
    grain = torch.full_like(a, 2.0 ** -9)
    for p in range(-5, 9):
        grain = torch.where(a >= 2.0 ** p, torch.full_like(a, 2.0 ** (p - 3)), grain)
    return torch.sign(x) * torch.round(a / grain) * grain * unit


def _exact_f8(case, seed):
    x = _exact_held(_rows(case, seed), 1)
    y = x @ _exact_held(_weight(case, seed, 1), 128).T
    if case["pair"]:
        y = y * torch.sigmoid(y) * (x @ _exact_held(_weight(case, seed, 2), 128).T)
    return y + _added(case, seed).double() if case["add"] else y


def _exact_row(z, u, t, k, p, m):
    """One row, from a list of its tokens in order."""
    live = torch.nonzero(z > -torch.inf)[:, 0]
    if not live.numel():
        return -1, -math.inf, 0.0
    live = live[torch.argsort(z[live], descending=True, stable=True)]
    top = z[live[0]]
    total = torch.exp(z[live] - top).sum()
    if t > 0:
        w = torch.softmax(z[live] / t, 0)
        n = min(k, live.numel()) if k else live.numel()
        if p < 1:
            run = w[:n].cumsum(0)
            n = min(n, int((run < p * run[-1]).sum()) + 1)
        if m > 0:
            n = int((z[live[:n]] >= top + math.log(m) * t).sum())
        index, back = torch.sort(live[:n])
        run = w[:n][back].cumsum(0)
        token = index[min(n - 1, int((run <= u * run[-1]).sum()))]
    else:
        token = live[0]
    return int(token), float(z[token] - top - torch.log(total)), float(1 / total)


def _exact_sample(case, seed):
    z, settings = _logits(case, seed).double(), _settings(case, seed)
    rows = case["rows"]
    off = (None, None, 0, 1.0, 0.0)
    u, t, k, p, m = (torch.full((rows,), o).tolist() if a is None else a.double().tolist() for a, o in zip(settings, off))
    got = [_exact_row(z[i], u[i], t[i], int(k[i]), p[i], m[i]) for i in range(rows)]
    token = torch.tensor([a for a, _, _ in got], device=DEV)
    if not case["scores"]:
        return token
    return token, torch.tensor([b for _, b, _ in got], dtype=torch.float64, device=DEV), torch.tensor([c for _, _, c in got], dtype=torch.float64, device=DEV)


def exact(case, seed):
    return _exact_f8(case, seed) if case["kind"] == "f8" else _exact_sample(case, seed)
