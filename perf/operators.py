"""The operators of a long-context, distilled training run whose speed is kept track of:
rotary positions, attention with a sliding window and sinks, and distillation from a
teacher's top logits, each through the package's public entry points (`own`) or as
elementary torch operations in 32 bits.

A case is a dict of plain values.  Its "kind" says what one pass is:

  rotary     the rotation of q and k (and of the gradients that come back, "grad")
  attention  the attention of lq queries over lk keys, forward (and backward, "grad");
             lk > lq: the queries are the last positions of a cache, of another length
             for each sequence where "ragged"
  distill    the loss of a student's logits against a teacher's top logits (and targets),
             and with "grad" the gradient of the logits

Everything is drawn on the GPU from the seed.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
IGNORE = -100
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # generation with LLaMA-350M's heads, one token for each of 8 sequences: latency
        dict(name="rope-step", kind="rotary", b=8, l=1, heads=16, kv=16, hd=64, dims=64, layout="half", scaling="none",
             factor=1, start=700, dtype="bf16", grad=False),
        # pretraining: a LLaMA-350M micro-batch of 32 x 256 tokens, q and k and their gradients
        dict(name="rope-350m", kind="rotary", b=32, l=256, heads=16, kv=16, hd=64, dims=64, layout="half",
             scaling="none", factor=1, start=0, dtype="bf16", grad=True),
        # fine-tuning in fp32 on long odd-length sequences: half of a head of 128 rotated, neighbours paired, grouped
        # heads, frequencies scaled by parts to eight times the trained length
        dict(name="rope-long-f32", kind="rotary", b=2, l=12001, heads=32, kv=8, hd=128, dims=64, layout="interleaved",
             scaling="parts", factor=8, start=0, dtype="f32", grad=True),
        # generation: one token of each of 16 sequences over caches of up to 4096 keys, a window of 1024 and 4 sinks
        dict(name="attn-step", kind="attention", b=16, lq=1, lk=4096, heads=16, kv=16, hd=64, window=1024, sinks=4,
             ragged=True, packed=False, grad=False),
        # generation from long contexts: grouped heads of 128, all keys visible, four ragged caches of up to 70000
        dict(name="attn-step-long", kind="attention", b=4, lq=1, lk=70000, heads=32, kv=8, hd=128, window=0, sinks=0,
             ragged=True, packed=False, grad=False),
        # pretraining: LLaMA-60M's heads over 32 sequences of 256, q, k, v in one buffer as the projection writes them
        dict(name="attn-60m", kind="attention", b=32, lq=256, lk=256, heads=8, kv=8, hd=64, window=128, sinks=4,
             ragged=False, packed=True, grad=True),
        # pretraining on long sequences: LLaMA-350M's heads, 4 x 4096 tokens
        dict(name="attn-350m-4k", kind="attention", b=4, lq=4096, lk=4096, heads=16, kv=16, hd=64, window=1024, sinks=4,
             ragged=False, packed=True, grad=True),
        # a ragged fine-tuning batch: odd length, heads of 80 that share keys by fives, an odd window
        dict(name="attn-odd", kind="attention", b=3, lq=1531, lk=1531, heads=10, kv=2, hd=80, window=301, sinks=1,
             ragged=False, packed=False, grad=True),
        # the largest: a 16384-token document, grouped heads of 128, a window of 4096
        dict(name="attn-16k", kind="attention", b=1, lq=16384, lk=16384, heads=16, kv=4, hd=128, window=4096, sinks=16,
             ragged=False, packed=False, grad=True),
        # a small fp32 student (odd vocabulary), eight teacher entries a token
        dict(name="distill-small", kind="distill", rows=200, V=1003, K=8, temperature=2.0, weight=0.5, targets=True,
             dtype="f32", grad=True),
        # LLaMA-350M's vocabulary over 32 x 256 tokens, 64 teacher entries beside the targets
        dict(name="distill-32k", kind="distill", rows=8192, V=32000, K=64, temperature=2.0, weight=0.5, targets=True,
             dtype="bf16", grad=True),
        # a large vocabulary, the teacher alone
        dict(name="distill-131k", kind="distill", rows=4096, V=131072, K=128, temperature=1.0, weight=1.0, targets=False,
             dtype="bf16", grad=True),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _heads(rng, most):
    kv = rng.choice((1, 2, 3, 4, 8, 16))
    return min(most, kv * rng.choice((1, 1, 2, 4, 5))) // kv * kv or kv, kv


def draw(rng):
    kind = rng.choice(("rotary", "attention", "attention", "attention", "distill"))
    if kind == "rotary":
        heads, kv = _heads(rng, 32)
        hd = rng.choice((32, 64, 64, 80, 96, 128))
        b = _log_int(rng, 1, 32)
        dtype, grad = rng.choice(("bf16", "bf16", "f32")), rng.random() < 0.7
        cap = 120_000_000 // (heads + kv) // hd // b
        l = 1 if rng.random() < 0.2 else _log_int(rng, 2, min(12001, cap))
        return dict(kind=kind, b=b, l=l, heads=heads, kv=kv, hd=hd, dims=rng.choice((hd, hd, hd // 2, hd // 4)),
                    layout=rng.choice(("half", "interleaved")),
                    scaling=rng.choice(("none", "linear", "ntk", "parts")), factor=rng.choice((2, 4, 8)),
                    start=rng.choice((0, _log_int(rng, 1, 100_000))), dtype=dtype, grad=grad and l > 1)
    if kind == "attention":
        heads, kv = _heads(rng, 32)
        hd = rng.choice((32, 64, 64, 64, 80, 96, 128, 128))
        window = rng.choice((0, _log_int(rng, 16, 4096), _log_int(rng, 16, 4096)))
        sinks = rng.choice((0, 1, 4, rng.randint(0, 64))) if window else 0
        c = dict(kind=kind, heads=heads, kv=kv, hd=hd, window=window, sinks=sinks)
        if rng.random() < 0.4:  # over a cache: single tokens, a few drafted ones, a chunk of a prompt
            lk = _log_int(rng, 64, 70000)
            lq = min(lk, rng.choice((1, 1, rng.randint(2, 8), _log_int(rng, 16, 1024))))
            b = min(_log_int(rng, 1, 32), max(1, 280_000 // lk * 8 // kv), max(1, (1 << 31) // (heads * lq * lk)))
            return dict(c, b=b, lq=lq, lk=lk, ragged=rng.random() < 0.7, packed=False, grad=False)
        pairs = 16 * 16384 * 3500  # of the largest listed case
        l = min(_log_int(rng, 33, 12000), math.isqrt(2 * pairs // heads))
        b = max(1, min(_log_int(rng, 1, 32), pairs // (heads * l * min(l // 2, (window or l) + sinks)), 85_000_000 // (l * heads * hd)))
        return dict(c, b=b, lq=l, lk=l, ragged=False, packed=heads == kv and rng.random() < 0.6, grad=rng.random() < 0.75)
    V = _log_int(rng, 500, 131072)
    dtype = rng.choice(("bf16", "bf16", "f32"))
    rows = min(_log_int(rng, 16, 16384), 1_000_000_000 // (V * DTYPES[dtype].itemsize))
    weight = rng.choice((1.0, 0.5, 0.9))
    return dict(kind=kind, rows=rows, V=V, K=min(V // 2, _log_int(rng, 2, 256)), temperature=rng.choice((1.0, 2.0, 3.0)),
                weight=weight, targets=weight < 1 or rng.random() < 0.5, dtype=dtype,
                grad=rng.random() < 0.8)


# ------------------------------- inputs ------------------------------------

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _randn(g, *shape, dtype=torch.bfloat16, scale=1.0):
    return torch.randn(*shape, generator=g, device=DEV).mul_(scale).to(dtype)


def _rotary_inputs(case, seed):
    g, dtype = _gen(seed), DTYPES[case["dtype"]]
    b, l, hd = case["b"], case["l"], case["hd"]
    s = dict(q=_randn(g, b, l, case["heads"], hd, dtype=dtype), k=_randn(g, b, l, case["kv"], hd, dtype=dtype))
    # every sequence at its own place, up to `start` past the beginning
    first = torch.randint(case["start"] + 1, (b, 1), generator=g, device=DEV)
    s["positions"] = first + torch.arange(l, device=DEV)
    if case["grad"]:
        s.update(dq=_randn(g, b, l, case["heads"], hd, dtype=dtype, scale=0.01),
                 dk=_randn(g, b, l, case["kv"], hd, dtype=dtype, scale=0.01))
    return s


def _attention_inputs(case, seed):
    g = _gen(seed)
    b, lq, lk, heads, kv, hd = (case[n] for n in ("b", "lq", "lk", "heads", "kv", "hd"))
    if case["packed"]:
        q, k, v = _randn(g, b, lq, 3, heads, hd).unbind(2)
    else:
        q, k, v = _randn(g, b, lq, heads, hd), _randn(g, b, lk, kv, hd), _randn(g, b, lk, kv, hd)
    s = dict(zip("qkv", (t.transpose(1, 2) for t in (q, k, v))))
    s["lengths"] = None
    if case["ragged"]:
        s["lengths"] = torch.randint(max(lq, lk // 2), lk + 1, (b,), generator=g, device=DEV, dtype=torch.int32)
    if case["grad"]:
        s["do"] = _randn(g, b, lq, heads, hd, scale=0.01).transpose(1, 2)
    return s


def _distill_inputs(case, seed):
    g, dtype = _gen(seed), DTYPES[case["dtype"]]
    rows, V, K = case["rows"], case["V"], case["K"]
    x = _randn(g, rows, V, dtype=dtype, scale=2.0)
    # distinct ids spread over the vocabulary, falling logits with gaps of a trained teacher's kind
    step = V // K
    ids = torch.arange(K, device=DEV) * step + torch.randint(step, (rows, K), generator=g, device=DEV)
    ids = ids.gather(1, torch.rand(rows, K, generator=g, device=DEV).argsort(1))
    gaps = -torch.log1p(-torch.rand(rows, K, generator=g, device=DEV)) / (1.0 + torch.arange(K, device=DEV))
    top = (12.0 - 2.0 * gaps.cumsum(1)).to(dtype)
    # a student that has learnt some of it
    x.scatter_(1, ids, (0.5 * top.float() + _randn(g, rows, K, dtype=torch.float32)).to(dtype))
    ids[torch.rand(rows, generator=g, device=DEV) < 0.05, K - K // 2:] = -1  # some tokens came with half the entries
    s = dict(x=x, top=top, ids=ids, targets=None)
    if case["targets"]:
        s["targets"] = torch.where(torch.rand(rows, generator=g, device=DEV) < 0.9, ids[:, 0],
                                   torch.randint(V, (rows,), generator=g, device=DEV))
        s["targets"][torch.rand(rows, generator=g, device=DEV) < 0.05] = IGNORE
        s["targets"][0] = 0
    return s


_INPUTS = {"rotary": _rotary_inputs, "attention": _attention_inputs, "distill": _distill_inputs}
_LEAVES = {"rotary": "qk", "attention": "qkv", "distill": "x"}
PARTS = dict(original_length=2048, low=1.0, high=32.0)


def prepare(case, seed):
    s = _INPUTS[case["kind"]](case, seed)
    s["case"] = case
    if own:
        from paper_2410_15352_amd import functional
        s["functional"] = functional
        if case["kind"] == "rotary":
            s["rope"] = functional.Rotary(case["dims"], layout=case["layout"], scaling=case["scaling"],
                                          factor=case["factor"], **PARTS)
        if case["grad"]:
            for name in _LEAVES[case["kind"]]:
                s[name] = s[name].detach().requires_grad_(True)
    return s


# -------------------------------- a pass -----------------------------------

def run(s):
    case = s["case"]
    return (_own if own else _plain)[case["kind"]](s, case)


def _own_rotary(s, case):
    q, k = s["rope"](s["q"], s["k"], positions=s["positions"])
    if not case["grad"]:
        return [q, k]
    return [q.detach(), k.detach(), *torch.autograd.grad((q, k), (s["q"], s["k"]), (s["dq"], s["dk"]))]


def _own_attention(s, case):
    o = s["functional"].window_attention(s["q"], s["k"], s["v"], window=case["window"] or None, sinks=case["sinks"],
                                         lengths=s["lengths"])
    if not case["grad"]:
        return [o]
    return [o.detach(), *torch.autograd.grad(o, (s["q"], s["k"], s["v"]), s["do"])]


def _own_distill(s, case):
    loss = s["functional"].distill_loss(s["x"], s["top"], s["ids"], targets=s["targets"], temperature=case["temperature"],
                                        weight=case["weight"])
    if not case["grad"]:
        return [loss]
    return [loss.detach(), *torch.autograd.grad(loss, s["x"])]


_own = {"rotary": _own_rotary, "attention": _own_attention, "distill": _own_distill}


# --------------------------- the plain forms --------------------------------

def _frequencies(case, dtype=torch.float64):
    """Radians per position of each pair, and the factor on the rotated values."""
    D, s, base = case["dims"], float(case["factor"]), 10000.0
    i = torch.arange(0, D, 2, device=DEV, dtype=dtype)
    if case["scaling"] == "ntk":
        base = base * s ** (D / (D - 2))
    f = base ** (-i / D)
    if case["scaling"] == "linear":
        return f / s, 1.0
    if case["scaling"] == "parts":
        turns = PARTS["original_length"] * f / (2 * math.pi)
        keep = ((turns - PARTS["low"]) / (PARTS["high"] - PARTS["low"])).clamp(0, 1)
        return f * (keep + (1 - keep) / s), 0.1 * math.log(s) + 1
    return f, 1.0


def _rotate(x, cos, sin, layout):
    """x (b, l, heads, hd) in 32 bits, the first 2 P elements of a head rotated by the P angles of its token."""
    D = 2 * cos.shape[-1]
    cos, sin, rest = cos.unsqueeze(2), sin.unsqueeze(2), x[..., D:]
    a, b = (x[..., :D // 2], x[..., D // 2:D]) if layout == "half" else (x[..., 0:D:2], x[..., 1:D:2])
    ya, yb = a * cos - b * sin, b * cos + a * sin
    y = torch.cat((ya, yb), -1) if layout == "half" else torch.stack((ya, yb), -1).flatten(-2)
    return torch.cat((y, rest), -1)


def _plain_rotary(s, case):
    f, m = _frequencies(case)
    # the angle alone in 64 bits: in 32, a product of 100 000 positions is off by a hundredth of a radian
    angle = s["positions"].unsqueeze(-1).double() * f
    cos, sin = (m * torch.cos(angle)).float(), (m * torch.sin(angle)).float()
    out = [_rotate(s[n].float(), cos, sin, case["layout"]).to(s[n].dtype) for n in "qk"]
    if case["grad"]:
        out += [_rotate(s[n].float(), cos, -sin, case["layout"]).to(s[n].dtype) for n in ("dq", "dk")]
    return out


def _chunks(case, elements):
    """Query rows at a time: about `elements` scores."""
    return max(16, min(case["lq"], elements // (case["b"] * case["heads"] * min(case["lk"], (case["window"] or case["lk"]) + 1024))))


def _plain_attention(s, case):
    b, lq, lk, heads, kv, hd = (case[n] for n in ("b", "lq", "lk", "heads", "kv", "hd"))
    window, sinks, G = case["window"] or lk, case["sinks"], heads // kv
    scale = hd ** -0.5
    q = s["q"].float().reshape(b, kv, G, lq, hd)
    k, v = s["k"].float(), s["v"].float()
    lengths = s["lengths"] if s["lengths"] is not None else torch.full((b,), lk, device=DEV)
    shortest = 0 if s["lengths"] is not None else lk
    o = torch.empty(b, kv, G, lq, hd, device=DEV)
    if case["grad"]:
        do = s["do"].float().reshape(b, kv, G, lq, hd)
        dq, dk, dv = torch.empty_like(q), torch.zeros_like(k), torch.zeros_like(v)
    step = _chunks(case, 1 << 28)
    for i0 in range(0, lq, step):
        i1 = min(lq, i0 + step)
        n = i1 - i0
        # the keys that some row of the chunk sees
        lo = max(0, shortest - lq + i0 - window + 1) if shortest else 0
        keys = torch.cat((torch.arange(min(sinks, lo), device=DEV), torch.arange(lo, min(lk, lk - lq + i1), device=DEV)))
        kc, vc = (k, v) if len(keys) == lk else (k[:, :, keys], v[:, :, keys])
        p = (lengths.view(b, 1) - lq + torch.arange(i0, i1, device=DEV)).view(b, 1, 1, n, 1)
        seen = (keys <= p) & ((p - keys < window) | (keys < sinks))
        S = torch.matmul(q[:, :, :, i0:i1].reshape(b, kv, G * n, hd), kc.transpose(2, 3)).view(b, kv, G, n, -1).mul_(scale)
        S.masked_fill_(~seen, -math.inf)
        top = S.amax(-1, keepdim=True)
        S.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
        S.div_(S.sum(-1, keepdim=True).clamp(min=1e-37))  # a row without a key: zero
        P = S.view(b, kv, G * n, -1)
        oc = torch.matmul(P, vc)
        o[:, :, :, i0:i1] = oc.view(b, kv, G, n, hd)
        if case["grad"]:
            doc = do[:, :, :, i0:i1].reshape(b, kv, G * n, hd)
            dvc = torch.matmul(P.transpose(2, 3), doc)
            dS = torch.matmul(doc, vc.transpose(2, 3))
            dS.sub_((doc * oc).sum(-1, keepdim=True)).mul_(P).mul_(scale)
            dq[:, :, :, i0:i1] = torch.matmul(dS, kc).view(b, kv, G, n, hd)
            dk.index_add_(2, keys, torch.matmul(dS.transpose(2, 3), q[:, :, :, i0:i1].reshape(b, kv, G * n, hd)))
            dv.index_add_(2, keys, dvc)
    out = [o.view(b, heads, lq, hd)]
    if case["grad"]:
        out += [dq.view(b, heads, lq, hd), dk, dv]
    return [t.to(torch.bfloat16) for t in out]


def _plain_distill(s, case):
    T, w, rows = case["temperature"], case["weight"], case["rows"]
    x = s["x"].float()
    there = s["ids"] >= 0
    ids = s["ids"].clamp(min=0)
    t = (s["top"].float() / T).masked_fill(~there, -math.inf)
    logp = t - torch.logsumexp(t, -1, keepdim=True)
    p = logp.exp()
    lse_t = torch.logsumexp(x / T, -1, keepdim=True)
    logq = x.gather(1, ids) / T - lse_t
    loss = w * T * T * torch.where(p > 0, p * (logp - logq), 0.0).sum(-1)
    counts, target = torch.ones(rows, dtype=torch.bool, device=DEV), None
    if case["targets"]:
        counts = s["targets"] != IGNORE
        target = s["targets"].clamp(min=0).unsqueeze(1)
        lse = torch.logsumexp(x, -1, keepdim=True)
        loss = loss + (1 - w) * (lse - x.gather(1, target)).squeeze(1)
    N = counts.sum()
    out = [torch.where(counts, loss, 0.0).sum() / N]
    if case["grad"]:
        dx = torch.exp(x / T - lse_t).mul_(w * T)
        dx.scatter_add_(1, ids, -w * T * p)
        if case["targets"]:
            dx.add_(torch.exp(x - lse), alpha=1 - w)
            dx.scatter_add_(1, target, torch.full((rows, 1), w - 1.0, device=DEV))
        dx.mul_(torch.where(counts, 1.0 / N, 0.0).unsqueeze(1))
        out.append(dx.to(s["x"].dtype))
    return out


_plain = {"rotary": _plain_rotary, "attention": _plain_attention, "distill": _plain_distill}


# ------------------------- what a pass cannot avoid ------------------------

def _pairs(case, lengths):
    """Visible pairs of a query row and a key, and the keys that some row sees, for one head of all sequences."""
    lq, w, s = case["lq"], case["window"] or case["lk"], case["sinks"]
    pairs = keys = 0
    for L in lengths:
        p0, p1 = L - lq, L - 1
        pairs += sum(min(p + 1, w + min(s, max(0, p + 1 - w))) for p in range(max(0, p0), p1 + 1))
        lo = max(0, p0 - w + 1)
        keys += p1 + 1 - lo + min(s, lo)
    return pairs, keys


def work(case):
    kind = case["kind"]
    if kind == "rotary":
        n = case["b"] * case["l"] * (case["heads"] + case["kv"])
        size = DTYPES[case["dtype"]].itemsize
        passes = 2 if case["grad"] else 1
        return dict(bytes=passes * 2.0 * size * n * case["hd"] + 8.0 * case["b"] * case["l"],
                    flops=passes * 3.0 * n * case["dims"])
    if kind == "attention":
        b, lq, lk, heads, kv, hd = (case[n] for n in ("b", "lq", "lk", "heads", "kv", "hd"))
        # ragged: lengths spread evenly over their range
        lo = max(lq, lk // 2)
        lengths = [lk - (lk - lo) * (2 * i + 1) // (2 * b) for i in range(b)] if case["ragged"] else [lk] * b
        pairs, keys = _pairs(case, lengths)
        q, kvs = 2.0 * b * heads * lq * hd, 2.0 * kv * keys * hd
        # forward q, k, v -> o; backward q, k, v, o, do -> dq, dk, dv
        return dict(bytes=2 * q + 2 * kvs + (4 * q + 4 * kvs if case["grad"] else 0),
                    flops=heads * pairs * hd * (14.0 if case["grad"] else 4.0))
    rows, V, K, size = case["rows"], case["V"], case["K"], DTYPES[case["dtype"]].itemsize
    return dict(bytes=(2.0 if case["grad"] else 1.0) * rows * V * size + rows * K * (size + 8.0) + 8.0 * rows * case["targets"],
                flops=(8.0 if case["grad"] else 4.0) * rows * V)


# ------------------------- the same in 64 bits ------------------------------

def exact(case, seed):
    with torch.no_grad():
        return _exact[case["kind"]](case, _INPUTS[case["kind"]](case, seed))


def _exact_rotary(case, s):
    D, pairs, n = case["dims"], case["dims"] // 2, float(case["factor"])
    b, l = s["positions"].shape
    # the definition pair by pair, as a complex product
    f = [10000.0 ** (-2.0 * i / D) for i in range(pairs)]
    m = 1.0
    if case["scaling"] == "linear":
        f = [v / n for v in f]
    elif case["scaling"] == "ntk":
        f = [(10000.0 * n ** (D / (D - 2.0))) ** (-2.0 * i / D) for i in range(pairs)]
    elif case["scaling"] == "parts":
        m = 1.0 + math.log(n) / 10.0
        for i, v in enumerate(f):
            g = (PARTS["original_length"] / (2.0 * math.pi / v) - PARTS["low"]) / (PARTS["high"] - PARTS["low"])
            g = min(1.0, max(0.0, g))
            f[i] = (1.0 - g) * v / n + g * v
    angle = s["positions"].to(torch.float64).view(b, l, 1, 1) * torch.tensor(f, dtype=torch.float64, device=DEV)
    turn = torch.polar(torch.full_like(angle, m), angle)

    def rotated(x, turn):
        y = x.double()
        first = slice(0, pairs) if case["layout"] == "half" else slice(0, D, 2)
        second = slice(pairs, D) if case["layout"] == "half" else slice(1, D, 2)
        z = torch.complex(y[..., first], y[..., second]) * turn
        y[..., first], y[..., second] = z.real, z.imag
        return y

    out = [rotated(s["q"], turn), rotated(s["k"], turn)]
    if case["grad"]:
        out += [rotated(s["dq"], turn.conj()), rotated(s["dk"], turn.conj())]
    return out


def _exact_attention(case, s):
    b, lq, lk, heads, kv, hd = (case[n] for n in ("b", "lq", "lk", "heads", "kv", "hd"))
    window, sinks = case["window"] or lk, case["sinks"]
    lengths = [lk] * b if s["lengths"] is None else s["lengths"].tolist()
    f64 = dict(dtype=torch.float64, device=DEV)
    o = torch.zeros(b, heads, lq, hd, **f64)
    grads = [torch.zeros(b, n, l, hd, **f64) for n, l in ((heads, lq), (kv, lk), (kv, lk))] if case["grad"] else []
    rows = max(1, min(lq, (1 << 26) // min(lk, window + sinks + 2048), 2048))
    for n in range(b):
        for h in range(heads):
            q, k, v = s["q"][n, h].double(), s["k"][n, h * kv // heads].double(), s["v"][n, h * kv // heads].double()
            for r in range(0, lq, rows):
                at = torch.arange(r, min(lq, r + rows), device=DEV) + (lengths[n] - lq)
                last = lengths[n] - lq + min(lq, r + rows)  # one past the chunk's last position
                first = max(0, lengths[n] - lq + r + 1 - window)
                at = at.unsqueeze(1)
                # the sinks before the window, then the window
                parts = [(c, d) for c, d in ((0, min(sinks, first)), (first, last)) if d > c]
                K, V = (torch.cat([t[c:d] for c, d in parts]) for t in (k, v))
                j = torch.cat([torch.arange(c, d, device=DEV) for c, d in parts]).unsqueeze(0)
                hidden = (j > at) | ((j <= at - window) & (j >= sinks))
                Q = q[r:r + rows]
                P = torch.softmax((Q @ K.T / math.sqrt(hd)).masked_fill_(hidden, -math.inf), 1)
                O = P @ V
                o[n, h, r:r + rows] = O
                if not grads:
                    continue
                dO = s["do"][n, h, r:r + rows].double()
                dP = dO @ V.T
                dS = P * (dP - (P * dP).sum(1, keepdim=True)) / math.sqrt(hd)
                grads[0][n, h, r:r + rows] = dS @ K
                dK, dV, e = dS.T @ Q, P.T @ dO, 0
                for c, d in parts:
                    grads[1][n, h * kv // heads, c:d] += dK[e:e + d - c]
                    grads[2][n, h * kv // heads, c:d] += dV[e:e + d - c]
                    e += d - c
    return [o, *grads]


def _exact_distill(case, s):
    T, w, rows, V = case["temperature"], case["weight"], case["rows"], case["V"]
    counts = s["targets"] != IGNORE if case["targets"] else torch.ones(rows, dtype=torch.bool, device=DEV)
    N = int(counts.sum())
    total = 0.0
    dx = torch.zeros(rows, V, dtype=torch.float64, device=DEV) if case["grad"] else None
    step = max(1, (1 << 26) // V)
    for r in range(0, rows, step):
        x, ids = s["x"][r:r + step].double(), s["ids"][r:r + step]
        # the teacher's distribution over the whole vocabulary
        e = torch.exp((s["top"][r:r + step].double() - s["top"][r:r + step].double().amax(1, keepdim=True)) / T) * (ids >= 0)
        p = torch.zeros_like(x).scatter_add_(1, ids.clamp(min=0), e / e.sum(1, keepdim=True))
        logq = torch.log_softmax(x / T, 1)
        row = w * T ** 2 * (torch.xlogy(p, p) - p * logq).sum(1)
        g = w * T * (torch.exp(logq) - p)
        if case["targets"]:
            logs = torch.log_softmax(x, 1)
            hot = torch.zeros_like(x).scatter_(1, s["targets"][r:r + step].clamp(min=0).unsqueeze(1), 1.0)
            row = row - (1 - w) * (hot * logs).sum(1)
            g += (1 - w) * (torch.exp(logs) - hot)
        c = counts[r:r + step]
        total += float(row[c].sum())
        if case["grad"]:
            dx[r:r + step] = g * c.unsqueeze(1) / N
    return [torch.tensor(total / N, dtype=torch.float64, device=DEV), *([dx] if case["grad"] else [])]


_exact = {"rotary": _exact_rotary, "attention": _exact_attention, "distill": _exact_distill}
