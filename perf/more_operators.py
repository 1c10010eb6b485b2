"""The operators of a fine-tuning run after pretraining whose speed is kept track of: attention
over sequences packed end to end, the tokens' log-probabilities, the loss of preference pairs,
the clipped policy loss and the clipping of the gradients' global norm, each through the
package's public entry points (`own`) or as elementary torch operations in 32 bits.

A case is a dict of plain values.  Its "kind" says what one pass is:

  packed      causal attention inside each of n sequences that lie end to end in `rows` rows (and
              `tail` rows behind the last one), forward (and backward, "grad")
  logprobs    the log-probability of each row's target (and the gradient of the logits)
  preference  the loss of n pairs of sequences against a reference, and the gradient of the logits
  policy      the clipped loss of n sampled sequences, with or without a KL term against a
              reference, and the gradient of the logits
  clip        the norm of all gradients of a model with compressed layers, and their scaling;
              where it is "clipped" a pass begins with new gradients, as a backward pass leaves them

Lengths of sequences: `spread` is the longest's ratio to the shortest's.  Everything is drawn
from the seed, on the GPU but for the lengths.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
IGNORE = -100
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
MAX_NORM = 1.0


def listed():
    return [
        # evaluation of a few short prompts in one call, LLaMA-60M's heads: latency
        dict(name="packed-short", kind="packed", rows=181, n=6, spread=12, tail=0, heads=8, kv=8, hd=64, window=0, sinks=0,
             one=True, grad=False),
        # the prompts of a batch of requests before generation, ragged, grouped heads of 128, a buffer of fixed size
        # that they do not fill
        dict(name="packed-prompts", kind="packed", rows=11900, n=31, spread=40, tail=388, heads=32, kv=8, hd=128, window=0,
             sinks=0, one=False, grad=False),
        # fine-tuning of LLaMA-350M's heads on documents of all lengths packed into 16384 rows, q, k, v in one buffer
        dict(name="packed-350m", kind="packed", rows=16384, n=24, spread=30, tail=0, heads=16, kv=16, hd=64, window=0,
             sinks=0, one=True, grad=True),
        # the largest: four long documents, grouped heads of 128, a window of 4096 and 16 sinks
        dict(name="packed-long", kind="packed", rows=32768, n=4, spread=5, tail=0, heads=16, kv=4, hd=128, window=4096,
             sinks=16, one=False, grad=True),
        # a small fp32 model's tokens (odd vocabulary), with the gradient
        dict(name="logprobs-small", kind="logprobs", rows=203, n=3, spread=3, V=1003, dtype="f32", grad=True),
        # the frozen reference's log-probabilities of 8192 tokens over LLaMA-350M's vocabulary
        dict(name="logprobs-32k", kind="logprobs", rows=8192, n=32, spread=4, V=32000, dtype="bf16", grad=False),
        # two preference pairs of a small fp32 model
        dict(name="preference-small", kind="preference", rows=155, n=2, spread=3, V=1003, dtype="f32", smoothing=0.0),
        # sixteen preference pairs in 8192 rows of LLaMA-350M's vocabulary
        dict(name="preference-32k", kind="preference", rows=8192, n=16, spread=5, V=32000, dtype="bf16", smoothing=0.1),
        # a policy step over 32 sampled answers, against a reference
        dict(name="policy-32k", kind="policy", rows=8192, n=32, spread=6, V=32000, dtype="bf16", low=0.2, high=0.2, kl=0.05),
        # a large vocabulary, the upper bound further off, no reference
        dict(name="policy-131k", kind="policy", rows=4096, n=16, spread=4, V=131072, dtype="bf16", low=0.2, high=0.28, kl=0.0),
        # LLaMA-60M at rank 128: a norm within its bound, as most steps' is
        dict(name="clip-60m", kind="clip", d=512, ffn=1376, layers=8, vocab=32000, rank=128, clipped=False),
        # LLaMA-350M at rank 128: a norm past its bound
        dict(name="clip-350m", kind="clip", d=1024, ffn=2736, layers=24, vocab=32000, rank=128, clipped=True),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("packed", "packed", "packed", "logprobs", "preference", "policy", "clip"))
    if kind == "packed":
        kv = rng.choice((1, 2, 3, 4, 8, 16))
        heads = kv * rng.choice([g for g in (1, 1, 2, 4, 5) if kv * g <= 32])
        hd = rng.choice((32, 64, 64, 64, 80, 96, 128, 128))
        rows = _log_int(rng, 8, min(32768, 67_108_864 // (heads * hd)))
        n = _log_int(rng, 1, min(256, rows))
        spread = rng.choice((1, 4, 30))
        window = rng.choice((0, 0, _log_int(rng, 16, 4096)))
        c = dict(kind=kind, rows=rows, n=n, spread=spread, tail=rng.choice((0, 0, rng.randint(1, 300))), heads=heads, kv=kv, hd=hd,
                 window=window, sinks=rng.choice((0, 1, 4, rng.randint(0, 64))) if window else 0,
                 one=heads == kv and rng.random() < 0.6, grad=rng.random() < 0.65)
        most = work(dict(listed()[3]))["flops"]
        while work(c)["flops"] > most:  # (long sequences without a window)
            c["n"] *= 2
        return c
    if kind == "clip":
        d = 8 * _log_int(rng, 8, 128)
        ffn, vocab, rank = int(d * rng.choice((2.67, 2.7, 4))), _log_int(rng, 300, 32000), rng.choice((d // 8, d // 4, d // 2))
        return dict(kind=kind, d=d, ffn=ffn, layers=rng.randint(1, 24 if rank <= d // 4 else 12), vocab=vocab, rank=rank,
                    clipped=rng.random() < 0.5)
    V = _log_int(rng, 500, 131072)
    dtype = rng.choice(("bf16", "bf16", "f32"))
    rows = min(_log_int(rng, 32, 16384), 1_000_000_000 // (V * DTYPES[dtype].itemsize))
    c = dict(kind=kind, rows=rows, n=_log_int(rng, 1, min(64, rows // 16)), spread=rng.choice((1, 3, 8)), V=V, dtype=dtype)
    if kind == "logprobs":
        return dict(c, grad=rng.random() < 0.5)
    if kind == "preference":
        return dict(c, smoothing=rng.choice((0.0, 0.1)))
    # (several sequences: the loss is a mean that must not lie near zero by chance)
    return dict(c, n=max(8, c["n"]) if rows >= 128 else 2, low=0.2, high=rng.choice((0.2, 0.28)), kl=rng.choice((0.0, 0.05)))


# ------------------------------- inputs ------------------------------------

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _randn(g, *shape, dtype=torch.bfloat16, scale=1.0):
    return torch.randn(*shape, generator=g, device=DEV).mul_(scale).to(dtype)


def _lengths(rows, n, spread):
    """n lengths of at least one row, `rows` together, spread evenly over their logarithm."""
    raw = [spread ** ((i + 0.5) / n) for i in range(n)]
    ends, total = [0], 0.0
    for x in raw:
        total += x
        ends.append(total)
    free = rows - n
    ends = [i + round(free * e / total) for i, e in enumerate(ends)]
    return [b - a for a, b in zip(ends, ends[1:])]


def _case_lengths(case):
    return _lengths(case["rows"], case["n"] * (2 if case["kind"] == "preference" else 1), case["spread"])


def _starts(case, seed):
    lengths = _case_lengths(case)
    random.Random(int(seed)).shuffle(lengths)
    ends = [0]
    for x in lengths:
        ends.append(ends[-1] + x)
    return lengths, torch.tensor(ends, dtype=torch.int32, device=DEV)


def _packed_inputs(case, seed):
    g = _gen(seed)
    rows, heads, kv, hd = case["rows"] + case["tail"], case["heads"], case["kv"], case["hd"]
    if case["one"]:
        q, k, v = _randn(g, rows, 3, heads, hd).unbind(1)
    else:
        q, k, v = _randn(g, rows, heads, hd), _randn(g, rows, kv, hd), _randn(g, rows, kv, hd)
    lengths, starts = _starts(case, seed)
    s = dict(q=q, k=k, v=v, lengths=lengths, starts=starts)
    if case["grad"]:
        s["do"] = _randn(g, rows, heads, hd, scale=0.01)
    return s


def _prompt(length):
    """Rows of a sequence that are its prompt's: their tokens do not count."""
    return 3 * length // 10


def _logit_inputs(case, seed):
    """A trained model's logits for the tokens that were sampled or written, prompts among them."""
    g, dtype = _gen(seed), DTYPES[case["dtype"]]
    rows, V = case["rows"], case["V"]
    lengths, starts = _starts(case, seed)
    x = _randn(g, rows, V, dtype=dtype, scale=2.0)
    targets = torch.randint(V, (rows,), generator=g, device=DEV)
    x.scatter_(1, targets.unsqueeze(1), (_randn(g, rows, 1, dtype=torch.float32, scale=2.0) + math.log(V) + 1.0).to(dtype))
    at = torch.arange(rows, device=DEV)
    seq = torch.searchsorted(starts[1:].contiguous(), at.to(torch.int32), right=True)
    first = torch.tensor([_prompt(n) for n in lengths], device=DEV)
    counts = at - starts[seq] >= first[seq]
    s = dict(x=x, targets=torch.where(counts, targets, IGNORE), lengths=lengths, starts=starts)
    if case["kind"] == "logprobs":
        if case["grad"]:
            s["dl"] = _randn(g, rows, dtype=torch.float32, scale=0.01)
        return s
    logp = torch.cat([torch.log_softmax(c.double(), 1).gather(1, t.unsqueeze(1)).squeeze(1)
                      for c, t in zip(x.split(1024), targets.split(1024))])
    noise = lambda scale: scale * torch.randn(rows, generator=g, device=DEV, dtype=torch.float64)
    if case["kind"] == "preference":
        # tuned for some steps: the first of a pair a little likelier than the reference has it
        s["reference"] = (logp + noise(0.15) - 0.02 * (1 - 2 * (seq % 2))).float()
        return s
    ratio = noise(0.12)  # of the policy that sampled: its logarithm
    for border in (1 - case["low"], 1 + case["high"]):  # none so near a border that its side is a matter of rounding
        ratio = torch.where((torch.exp(ratio) / border - 1).abs() < 1e-3, ratio + 0.004, ratio)
    s["old"] = (logp - ratio).float()
    # (rewards over a slow baseline: their mean is not zero)
    order = torch.rand(case["n"], generator=g, device=DEV).argsort()
    s["advantages"] = ((2.0 * order + 1.0) / case["n"] - 0.5)[seq]
    s["reference"] = (logp + noise(0.3)).float() if case["kl"] > 0 else None
    return s


def _shapes(case):
    """The gradients of a model with compressed layers: bf16 of the others, fp32 of the compressed ones."""
    d, ffn, rank, V = case["d"], case["ffn"], case["rank"], case["vocab"]
    dense, compressed = [(V, d)], []
    for _ in range(case["layers"]):
        dense += [(d,), (d,), (d, d)]
        compressed += [(rank, d)] * 3 + [(rank, ffn)] * 2 + [(ffn * rank // d, d)]
    return dense + [(d,), (d, V)], compressed


def _clip_inputs(case, seed):
    g = _gen(seed)
    groups, count = _shapes(case), 0
    s = dict(flats=[], kept=[], grads=[])
    for shapes, dtype in zip(groups, (torch.bfloat16, torch.float32)):
        at, total = [], 0
        for shape in shapes:
            at.append(total)
            total += -(-math.prod(shape) // 128) * 128  # (each on a boundary of its own)
        flat = torch.zeros(total, dtype=dtype, device=DEV)
        grads = [flat[a:a + math.prod(shape)].view(shape) for a, shape in zip(at, shapes)]
        s["flats"].append(flat)
        s["grads"] += grads
        count += sum(t.numel() for t in grads)
    scale = (4.0 if case["clipped"] else 0.4) * MAX_NORM / math.sqrt(count)
    for i, t in enumerate(s["grads"]):
        t.copy_(torch.randn(t.shape, generator=g, device=DEV).mul_(scale * (0.7 if i % 2 else 1.2)))
    s["kept"] = [t.clone() for t in s["flats"]] if case["clipped"] else []
    return s


def _inputs(case, seed):
    return {"packed": _packed_inputs, "clip": _clip_inputs}.get(case["kind"], _logit_inputs)(case, seed)


_LEAVES = {"packed": "qkv", "logprobs": "x", "preference": "x", "policy": "x", "clip": ""}


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        from paper_2410_15352_amd import finetune, functional
        s.update(functional=functional, finetune=finetune)
        if case.get("grad", True):
            for name in _LEAVES[case["kind"]]:
                s[name] = s[name].detach().requires_grad_(True)
    return s


# -------------------------------- a pass -----------------------------------

def run(s):
    case = s["case"]
    return (_own if own else _plain)[case["kind"]](s, case)


def _own_packed(s, case):
    o = s["functional"].packed_attention(s["q"], s["k"], s["v"], s["starts"], window=case["window"] or None, sinks=case["sinks"])
    if not case["grad"]:
        return [o]
    return [o.detach(), *torch.autograd.grad(o, (s["q"], s["k"], s["v"]), s["do"])]


def _own_logprobs(s, case):
    logp = s["finetune"].token_logprobs(s["x"], s["targets"])
    if not case["grad"]:
        return [logp]
    return [logp.detach(), *torch.autograd.grad(logp, s["x"], s["dl"])]


def _own_preference(s, case):
    loss, rewards = s["finetune"].preference_loss(s["x"], s["targets"], s["starts"], reference=s["reference"], beta=0.1,
                                                  smoothing=case["smoothing"])
    return [loss.detach(), rewards, *torch.autograd.grad(loss, s["x"])]


def _own_policy(s, case):
    loss, logp = s["finetune"].policy_loss(s["x"], s["targets"], s["old"], s["advantages"], reference=s["reference"],
                                           clip=(case["low"], case["high"]), kl=case["kl"])
    return [loss.detach(), logp, *torch.autograd.grad(loss, s["x"])]


def _own_clip(s, case):
    for flat, kept in zip(s["flats"], s["kept"]):
        flat.copy_(kept)
    return [s["finetune"].clip_grad_norm(s["grads"], MAX_NORM), *s["flats"]]


_own = {"packed": _own_packed, "logprobs": _own_logprobs, "preference": _own_preference, "policy": _own_policy, "clip": _own_clip}


# --------------------------- the plain forms --------------------------------

def _plain_packed(s, case):
    """The sequences as a padded batch (n, longest), the scores of about 2^28 pairs at a time."""
    rows, heads, kv, hd = case["rows"] + case["tail"], case["heads"], case["kv"], case["hd"]
    n, M, G = case["n"], max(s["lengths"]), heads // kv
    window, sinks, scale = case["window"] or M, case["sinks"], hd ** -0.5
    starts = s["starts"].long()
    i, r = torch.arange(M, device=DEV), torch.arange(rows, device=DEV)
    live = i < (starts[1:] - starts[:-1]).unsqueeze(1)
    at = torch.where(live, starts[:-1].unsqueeze(1) + i, 0)
    inside = (r < starts[-1]).view(rows, 1, 1)
    seq = torch.searchsorted(starts[1:].contiguous(), r, right=True).clamp(max=n - 1)
    pos = torch.where(inside.view(rows), r - starts[seq], 0)

    def padded(t):
        return torch.where(live.view(n, M, 1, 1), t.float()[at], 0.0).transpose(1, 2)

    def unpadded(t, h):
        return torch.where(inside, t.reshape(n, h, M, hd)[seq, :, pos], 0.0).to(torch.bfloat16)

    q, k, v = padded(s["q"]).reshape(n, kv, G, M, hd), padded(s["k"]).contiguous(), padded(s["v"]).contiguous()
    o = torch.empty(n, kv, G, M, hd, device=DEV)
    if case["grad"]:
        do = padded(s["do"]).reshape(n, kv, G, M, hd)
        dq, dk, dv = torch.empty_like(q), torch.zeros_like(k), torch.zeros_like(v)
    step = max(16, min(M, (1 << 28) // (n * heads * min(M, window + 1024))))
    for i0 in range(0, M, step):
        i1 = min(M, i0 + step)
        m, lo = i1 - i0, max(0, i0 - window + 1)
        keys = torch.cat((torch.arange(min(sinks, lo), device=DEV), torch.arange(lo, i1, device=DEV)))
        kc, vc = k[:, :, keys], v[:, :, keys]
        p = torch.arange(i0, i1, device=DEV).view(m, 1)
        seen = (keys <= p) & ((p - keys < window) | (keys < sinks))
        S = torch.matmul(q[:, :, :, i0:i1].reshape(n, kv, G * m, hd), kc.transpose(2, 3).contiguous()).view(n, kv, G, m, -1).mul_(scale)
        S.masked_fill_(~seen, -math.inf)
        S.sub_(S.amax(-1, keepdim=True)).exp_()
        S.div_(S.sum(-1, keepdim=True))
        P = S.view(n, kv, G * m, -1)
        oc = torch.matmul(P, vc)
        o[:, :, :, i0:i1] = oc.view(n, kv, G, m, hd)
        if case["grad"]:
            doc, qc = do[:, :, :, i0:i1].reshape(n, kv, G * m, hd), q[:, :, :, i0:i1].reshape(n, kv, G * m, hd)
            dv.index_add_(2, keys, torch.matmul(P.transpose(2, 3), doc))
            dS = torch.matmul(doc, vc.transpose(2, 3))
            dS.sub_((doc * oc).sum(-1, keepdim=True)).mul_(P).mul_(scale)
            dq[:, :, :, i0:i1] = torch.matmul(dS, kc).view(n, kv, G, m, hd)
            dk.index_add_(2, keys, torch.matmul(dS.transpose(2, 3), qc))
    return [unpadded(o, heads)] + ([unpadded(dq, heads), unpadded(dk, kv), unpadded(dv, kv)] if case["grad"] else [])


def _plain_rows(s):
    """Which rows count, their targets, exp(x - lse) and the log-probabilities."""
    x, counts = s["x"].float(), s["targets"] != IGNORE
    target = torch.where(counts, s["targets"], 0).unsqueeze(1)
    top = x.amax(1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(1, keepdim=True)
    logp = (x.gather(1, target) - top - torch.log(total)).squeeze(1)
    return counts, target, e.div_(total), torch.where(counts, logp, 0.0)


def _plain_grad(s, counts, target, p, g):
    """Of the logits, from the softmax p and the log-probabilities' gradient."""
    g = torch.where(counts, g, 0.0).unsqueeze(1)
    p.mul_(-g).scatter_add_(1, target, g)
    return p.to(s["x"].dtype)


def _plain_logprobs(s, case):
    counts, target, p, logp = _plain_rows(s)
    return [logp] + ([_plain_grad(s, counts, target, p, s["dl"])] if case["grad"] else [])


def _plain_preference(s, case):
    counts, target, p, logp = _plain_rows(s)
    n, beta, eps = case["n"], 0.1, case["smoothing"]
    r = torch.arange(case["rows"], device=DEV, dtype=torch.int32)
    seq = torch.searchsorted(s["starts"][1:].contiguous(), r, right=True)
    # (sums of hundreds of near numbers' differences: in 64 bits)
    rewards = beta * torch.zeros(2 * n, dtype=torch.float64, device=DEV).index_add_(
        0, seq, torch.where(counts, logp.double() - s["reference"].double(), 0.0))
    rewards = rewards.view(n, 2)
    delta = rewards[:, 0] - rewards[:, 1]
    softplus = lambda t: t.clamp(min=0) + torch.log(1 + torch.exp(-t.abs()))
    loss = ((1 - eps) * softplus(-delta) + eps * softplus(delta)).sum() / n
    slope = beta / n * (1 / (1 + torch.exp(-delta)) - (1 - eps))
    g = torch.stack((slope, -slope), 1).view(-1)[seq]
    return [loss.float(), rewards.float(), _plain_grad(s, counts, target, p, g.float())]


def _plain_policy(s, case):
    counts, target, p, logp = _plain_rows(s)
    A, N = s["advantages"], counts.sum()
    ratio = torch.exp(logp - s["old"])
    bounded = ratio.clamp(1 - case["low"], 1 + case["high"])
    rows = -torch.minimum(ratio * A, bounded * A)
    g = torch.where((A > 0) & (ratio > 1 + case["high"]) | (A < 0) & (ratio < 1 - case["low"]), 0.0, -A * ratio)
    if case["kl"] > 0:
        d = s["reference"] - logp
        rows = rows + case["kl"] * (torch.exp(d) - d - 1)
        g = g + case["kl"] * (1 - torch.exp(d))
    loss = torch.where(counts, rows, 0.0).double().sum() / N
    return [loss.float(), logp, _plain_grad(s, counts, target, p, g / N)]


def _plain_clip(s, case):
    for flat, kept in zip(s["flats"], s["kept"]):
        flat.copy_(kept)
    norm = torch.stack([t.float().square().sum() for t in s["grads"]]).sum().sqrt()
    factor = (MAX_NORM / (norm + 1e-6)).clamp(max=1.0)
    for t in s["grads"]:
        t.copy_(t.float() * factor)
    return [norm, *s["flats"]]


_plain = {"packed": _plain_packed, "logprobs": _plain_logprobs, "preference": _plain_preference, "policy": _plain_policy,
          "clip": _plain_clip}


# ------------------------- what a pass cannot avoid ------------------------

def _pairs(length, window, sinks):
    """Pairs of a row and a key that it sees."""
    w = min(window or length, length)
    late = length - w  # rows past the window
    few = min(sinks, late)
    # a late row sees w keys of its window and the sinks before it
    return w * (w + 1) // 2 + late * w + few * (few + 1) // 2 + (late - few) * few


def work(case):
    kind = case["kind"]
    if kind == "packed":
        rows, heads, kv, hd = case["rows"], case["heads"], case["kv"], case["hd"]
        pairs = sum(_pairs(n, case["window"], case["sinks"]) for n in _case_lengths(case))
        q, kvs, tail = 2.0 * rows * heads * hd, 2.0 * rows * kv * hd, 2.0 * case["tail"] * hd
        # forward q, k, v -> o; backward q, k, v, o, do -> dq, dk, dv
        return dict(bytes=2 * q + 2 * kvs + tail * heads + (4 * q + 4 * kvs + tail * (heads + 2 * kv) if case["grad"] else 0),
                    flops=heads * pairs * hd * (14.0 if case["grad"] else 4.0))
    if kind == "clip":
        dense, compressed = (sum(math.prod(x) for x in shapes) for shapes in _shapes(case))
        # read; and where it is clipped: copied, read and written again
        return dict(bytes=(5.0 if case["clipped"] else 1.0) * (2 * dense + 4 * compressed), flops=2.0 * (dense + compressed))
    rows, V, size = case["rows"], case["V"], DTYPES[case["dtype"]].itemsize
    live = rows - sum(_prompt(n) for n in _case_lengths(case))
    grad = case.get("grad", True)
    # the logits of the rows that count are read once (twice where the gradient needs all rows' sums first), the gradient written
    reads = 2.0 if kind == "preference" or kind == "logprobs" and grad else 1.0
    return dict(bytes=size * V * (reads * live + (rows if grad else 0)) + rows * 24.0, flops=(8.0 if grad else 4.0) * live * V)


# ------------------------- the same in 64 bits ------------------------------

def exact(case, seed):
    with torch.no_grad():
        return _exact[case["kind"]](case, _inputs(case, seed))


def _exact_packed(case, s):
    rows, heads, kv, hd = case["rows"] + case["tail"], case["heads"], case["kv"], case["hd"]
    f64 = dict(dtype=torch.float64, device=DEV)
    o = torch.zeros(rows, heads, hd, **f64)
    grads = [torch.zeros(rows, h, hd, **f64) for h in (heads, kv, kv)] if case["grad"] else []
    first = 0
    for length in s["lengths"]:
        here = slice(first, first + length)
        window = case["window"] or length
        chunk = max(1, min(length, (1 << 26) // length))
        for h in range(heads):
            g = h * kv // heads
            q, k, v = s["q"][here, h].double(), s["k"][here, g].double(), s["v"][here, g].double()
            for a in range(0, length, chunk):
                b = min(length, a + chunk)
                i, j = torch.arange(a, b, device=DEV).unsqueeze(1), torch.arange(b, device=DEV)
                hidden = (j > i) | ((j <= i - window) & (j >= case["sinks"]))
                P = torch.softmax((q[a:b] @ k[:b].T / math.sqrt(hd)).masked_fill_(hidden, -math.inf), 1)
                at = slice(first + a, first + b)
                o[at, h] = P @ v[:b]
                if grads:
                    do = s["do"][at, h].double()
                    dP = do @ v[:b].T
                    dS = P * (dP - (P * dP).sum(1, keepdim=True)) / math.sqrt(hd)
                    grads[0][at, h] = dS @ k[:b]
                    grads[1][first:first + b, g] += dS.T @ q[a:b]
                    grads[2][first:first + b, g] += P.T @ do
        first += length
    return [o, *grads]


def _exact_rows(case, s, slope):
    """The log-probabilities, and the logits' gradient where slope(them) gives theirs."""
    x, t = s["x"], s["targets"]
    counts = t >= 0
    step = max(1, (1 << 26) // case["V"])
    spans = [slice(a, min(case["rows"], a + step)) for a in range(0, case["rows"], step)]
    logp = torch.cat([torch.log_softmax(x[r].double(), 1).gather(1, t[r].clamp(min=0).unsqueeze(1)).squeeze(1) for r in spans])
    logp = torch.where(counts, logp, 0.0)
    if slope is None:
        return logp, None
    g = torch.where(counts, slope(logp), 0.0)
    dx = torch.empty(x.shape, dtype=torch.float64, device=DEV)
    for r in spans:
        hot = torch.zeros(x[r].shape, dtype=torch.float64, device=DEV).scatter_(1, t[r].clamp(min=0).unsqueeze(1), 1.0)
        dx[r] = g[r].unsqueeze(1) * (hot - torch.softmax(x[r].double(), 1))
    return logp, dx


def _exact_logprobs(case, s):
    logp, dx = _exact_rows(case, s, (lambda logp: s["dl"].double()) if case["grad"] else None)
    return [logp] + ([dx] if case["grad"] else [])


def _exact_preference(case, s):
    n, beta, eps, found = case["n"], 0.1, case["smoothing"], []

    def slope(logp):
        counts = s["targets"] >= 0
        gain = torch.where(counts, logp - s["reference"].double(), 0.0)
        sums = torch.stack([part.sum() for part in gain.split(s["lengths"])])
        delta = beta * (sums[0::2] - sums[1::2])
        loss = -((1 - eps) * torch.nn.functional.logsigmoid(delta) + eps * torch.nn.functional.logsigmoid(-delta)).mean()
        found.extend((loss, beta * sums.view(n, 2)))
        each = beta / n * (eps * torch.sigmoid(delta) - (1 - eps) * torch.sigmoid(-delta))
        return torch.repeat_interleave(torch.stack((each, -each), 1).view(-1), torch.tensor(s["lengths"], device=DEV))

    _, dx = _exact_rows(case, s, slope)
    return [*found, dx]


def _exact_policy(case, s):
    found = []

    def slope(logp):
        with torch.enable_grad():
            l = logp.clone().requires_grad_(True)
            r, A = torch.exp(l - s["old"].double()), s["advantages"].double()
            each = -torch.min(r * A, torch.clamp(r, 1 - case["low"], 1 + case["high"]) * A)
            if case["kl"] > 0:
                d = s["reference"].double() - l
                each = each + case["kl"] * (torch.expm1(d) - d)
            loss = each[s["targets"] >= 0].mean()
        found.append(loss.detach())
        return torch.autograd.grad(loss, l)[0]

    logp, dx = _exact_rows(case, s, slope)
    return [*found, logp, dx]


def _exact_clip(case, s):
    wide = [t.double() for t in s["flats"]]
    norm = sum((t * t).sum() for t in wide) ** 0.5
    factor = min(1.0, MAX_NORM / (float(norm) + 1e-6))
    return [norm, *(t * factor for t in wide)]


_exact = {"packed": _exact_packed, "logprobs": _exact_logprobs, "preference": _exact_preference, "policy": _exact_policy,
          "clip": _exact_clip}
