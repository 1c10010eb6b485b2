"""Operators of fine-tuning after pretraining, as functions of their own:

    token_logprobs    the log-probabilities of given tokens
    preference_loss   pairs of sequences, the first preferred, against a reference
    policy_loss       the clipped loss of sampled tokens, with a KL term against a reference
    clip_grad_norm    the norm of many gradients together, and their scaling to a bound

Logits are (rows, V), as distill_loss takes them, with one target a row; sequences lie end to end
in the rows, as packed_attention takes them.  On the current GPU they run the HIP kernels of
libcompact.so (csrc/finetune.hip, clip.hip) on the current stream, forward and backward, for bf16
and fp32 (dense logits on a 16-byte boundary; others are copied first).  Other types and places,
autocast, tracing and functorch take the torch expressions beside each function, and so does a
backward that is itself recorded or batched.  Arguments that no form takes are refused with
ValueError or TypeError."""
from __future__ import annotations

import ctypes
import math
import struct
from array import array
from itertools import chain

import torch

from . import _block_ops as ops
from . import _lib
from ._block_ops import IGNORE, _eager, _i64, _plain, _stream, _vp
from .functional import _block, _bounds, _device_now, _here, _tracked

__all__ = ["token_logprobs", "preference_loss", "policy_loss", "clip_grad_norm"]

_bf16, _f32 = torch.bfloat16, torch.float32
_Tensor = torch.Tensor

# The argument blocks of csrc/functional.hpp as native struct layouts, passed by address.
_token_pack = struct.Struct("@8Q3q2i").pack
_pair_pack = struct.Struct("@7Q3qi2f4x").pack
_policy_pack = struct.Struct("@11Q3q3i3f").pack

ops._SIGNATURES.update({
    "compact_token_logprobs": [_block, _vp],
    "compact_preference_pairs": [_block, _vp],
    "compact_policy": [_block, _vp],
    "compact_clip": [_vp, _i64, ctypes.c_double, ctypes.c_int, _vp, _i64, _vp, _vp],
})


def _at(t):
    return 0 if t is None else t.data_ptr()


def _dense(t):
    t = t if t.is_contiguous() else t.contiguous()
    return t if t.data_ptr() % 16 == 0 else t.clone()


def _check_logits(name, logits, targets):
    if not isinstance(logits, _Tensor) or not isinstance(targets, _Tensor):
        raise TypeError(f"{name}: logits and targets are tensors")
    if logits.dim() != 2 or logits.shape[0] < 1 or logits.shape[1] < 1 or targets.shape != logits.shape[:1]:
        raise ValueError(f"{name}: logits (rows, V) and targets (rows,), at least one of each")
    if not logits.is_floating_point() or targets.dtype != torch.int64:
        raise TypeError(f"{name}: floating logits and targets of int64")
    if targets.device != logits.device:
        raise ValueError(f"{name}: tensors of one device")


def _check_rows(name, logits, **tensors):
    for what, t in tensors.items():
        if t is None:
            continue
        if not isinstance(t, _Tensor) or not t.is_floating_point():
            raise TypeError(f"{name}: {what} is a floating tensor")
        if t.shape != logits.shape[:1] or t.device != logits.device:
            raise ValueError(f"{name}: {what} (rows,) on the logits' device")


def _check_number(name, what, x, least, most):
    x = float(x)
    if not least <= x <= most:
        raise ValueError(f"{name}: {what} in [{least}, {most}]")
    return x


def _rows_usable(logits, targets, *rows):
    """Dense logits and targets as the kernels take them, and fp32 numbers of each row."""
    return (logits.dtype in (_bf16, _f32) and 0 < logits.shape[0] < ops.MAX_ROWS and 0 < logits.shape[1] <= 1 << 28
            and _here(logits) and logits.is_contiguous() and logits.data_ptr() % 16 == 0
            and targets.dtype is torch.int64 and targets.shape == logits.shape[:1] and _here(targets) and targets.is_contiguous()
            and all(t is None or t.dtype is _f32 and t.shape == logits.shape[:1] and _here(t) and t.is_contiguous() for t in rows))


def _fp32_rows(*tensors):
    """Constants of each row: dense, of 32 bits."""
    return [t if t is None else t.detach().float().contiguous() for t in tensors]


def _wide(t):
    return torch.float64 if t.dtype == torch.float64 else _f32


# --------------------------- log-probabilities ------------------------------

def _logprobs_torch(logits, targets):
    """The log-probabilities as torch expressions, in fp32 (fp64 for fp64); which rows count."""
    V = logits.shape[1]
    counts = targets != IGNORE
    # (a row that does not count has no part, whatever it holds)
    x = torch.where(counts.unsqueeze(1), logits.to(_wide(logits)), 0.0)
    bad = counts & ((targets < 0) | (targets >= V))
    l = torch.log_softmax(x, 1).gather(1, torch.where(counts & ~bad, targets, 0).unsqueeze(1)).squeeze(1)
    return torch.where(counts, l * torch.where(bad, math.nan, 1.0), 0.0), counts


def _token_call(logits, targets, reference=None, out=None, stats=None, grad=None, dloss=None, dx=None):
    rows, V = logits.shape
    ops._call("compact_token_logprobs",
              _token_pack(logits.data_ptr(), targets.data_ptr(), _at(reference), _at(out), _at(stats), _at(grad), _at(dloss), _at(dx),
                          rows, V, IGNORE, logits.dtype == _f32, dx is not None), _stream(logits))


class _LogprobsFn(torch.autograd.Function):
    """Keeps the logits, and the maximum and the sum of exponentials of each row."""

    @staticmethod
    def forward(ctx, logits, targets):
        rows = logits.shape[0]
        out = torch.empty(rows, dtype=_f32, device=logits.device)
        stats = torch.empty(2 * rows, dtype=_f32, device=logits.device)
        _token_call(logits, targets, out=out, stats=stats)
        ctx.size = logits.dtype, logits.shape
        ctx.save_for_backward(logits, targets, stats)
        return out

    @staticmethod
    def backward(ctx, dl):
        logits, targets, stats = ctx.saved_tensors
        if (torch.is_grad_enabled() or not _eager() or not _plain(dl) or (logits.dtype, logits.shape) != ctx.size
                or not _rows_usable(logits, targets) or not ops._companion(stats, _f32, 2 * logits.shape[0])):
            return ops._torch_grad(lambda t: _logprobs_torch(t, targets.to(torch.int64))[0], logits, dl), None
        dx = torch.empty_like(logits)
        _token_call(logits, targets, stats=stats, grad=dl.float().contiguous(), dx=dx)
        return dx, None


def token_logprobs(logits, targets):
    """log softmax(logits) at the targets: fp32 (rows,) of logits (rows, V) and targets (rows,); fp64
    of fp64 logits.

    A row whose target is -100 gives 0 and passes no gradient, whatever it holds; a target past V
    makes its row NaN.

    Under torch.no_grad() these are what preference_loss and policy_loss take of a reference or of
    the policy that sampled."""
    _check_logits("token_logprobs", logits, targets)
    if _eager() and logits.is_cuda:
        dense, targets = _dense(logits), targets.contiguous()
        if _rows_usable(dense, targets):
            if _tracked(dense):
                return _LogprobsFn.apply(dense, targets)
            out = torch.empty(dense.shape[0], dtype=_f32, device=dense.device)
            _token_call(dense, targets, out=out)
            return out
    return _logprobs_torch(logits, targets)[0]


# --------------------------- preference pairs -------------------------------

def _preference_torch(logits, targets, starts, reference, beta, smoothing):
    """The loss and the rewards as torch expressions, in fp32 with sums in fp64 (fp64 for fp64)."""
    rows, pairs = logits.shape[0], (starts.shape[0] - 1) // 2
    e = _bounds(starts, rows)
    s = torch.searchsorted(e, torch.arange(rows, device=e.device), right=True)
    l, counts = _logprobs_torch(logits, torch.where((s > 0) & (s < len(e)), targets, IGNORE))
    gain = l.double()
    if reference is not None:
        gain = torch.where(counts, gain - reference.double(), 0.0)
    sums = torch.zeros(2 * pairs + 2, dtype=torch.float64, device=e.device).index_add(0, s, gain)[1:-1].view(pairs, 2)
    rewards = beta * sums
    delta = rewards[:, 0] - rewards[:, 1]
    loss = (1 - smoothing) * torch.nn.functional.softplus(-delta)
    if smoothing > 0:
        loss = loss + smoothing * torch.nn.functional.softplus(delta)
    wide = _wide(logits)
    return loss.mean().to(wide), rewards.detach().to(wide)


OWN_PAIRS = 2048  # more have the starts' running maximum formed before, by a launch of its own


class _PreferenceFn(torch.autograd.Function):
    """Keeps the logits and three fp32 numbers of each row."""

    @staticmethod
    def forward(ctx, logits, targets, starts, reference, beta, smoothing, tracked):
        rows, pairs = logits.shape[0], (starts.shape[0] - 1) // 2
        device = logits.device
        stats = torch.empty(2 * rows, dtype=_f32, device=device) if tracked else None
        gain, slope = torch.empty(rows, dtype=_f32, device=device), torch.empty(rows, dtype=_f32, device=device)
        loss, rewards = torch.empty((), dtype=_f32, device=device), torch.empty(pairs, 2, dtype=_f32, device=device)
        bounds = pairs > OWN_PAIRS
        each = torch.empty(pairs + (2 * pairs + 1) * bounds, dtype=_f32, device=device)  # scratch
        _token_call(logits, targets, reference=reference, out=gain, stats=stats)
        ops._call("compact_preference_pairs",
                  _pair_pack(gain.data_ptr(), starts.data_ptr(), rewards.data_ptr(), slope.data_ptr(), each.data_ptr(),
                             loss.data_ptr(), each.data_ptr() + 4 * pairs if bounds else 0, starts.stride(0), rows, pairs,
                             starts.dtype == torch.int64, beta, smoothing),
                  _stream(logits))
        if tracked:
            ctx.rule = beta, smoothing
            ctx.size = logits.dtype, logits.shape
            ctx.save_for_backward(logits, targets, starts, reference, stats, slope)
            ctx.mark_non_differentiable(rewards)
            ctx.set_materialize_grads(False)
        return loss, rewards

    @staticmethod
    def backward(ctx, dloss, _):
        none = (None,) * 6
        if dloss is None:
            return None, *none
        logits, targets, starts, reference, stats, slope = ctx.saved_tensors
        if (torch.is_grad_enabled() or not _eager() or not _plain(dloss) or (logits.dtype, logits.shape) != ctx.size
                or not _rows_usable(logits, targets) or not ops._companion(stats, _f32, 2 * logits.shape[0])
                or not ops._companion(slope, _f32, logits.shape[0])):
            beta, smoothing = ctx.rule
            return (ops._torch_grad(lambda t: _preference_torch(t, targets.to(torch.int64), starts, reference, beta, smoothing)[0],
                                    logits, dloss), *none)
        dx = torch.empty_like(logits)
        _token_call(logits, targets, stats=stats, grad=slope, dloss=dloss.float(), dx=dx)
        return dx, *none


def preference_loss(logits, targets, starts, reference=None, beta=0.1, smoothing=0.0):
    """(loss, rewards) of n pairs of sequences, of which the first is preferred to the second:

        S = sum over a sequence's rows of (log softmax(logits)_target - reference)
        D = beta (S_first - S_second)
        loss = mean over the pairs of (1 - smoothing) softplus(-D) + smoothing softplus(D)

    logits (rows, V), targets (rows,): a row whose target is -100, as a prompt's, has no part.
    starts (2 n + 1,), integers on the device, ascending: sequence s holds the rows starts[s] ..
    starts[s + 1] - 1; pair i is the sequences 2 i and 2 i + 1.  Rows of no sequence have no part.
    (A start below an earlier one, or past the rows, is taken as that one, or as the last row's end.)
    reference (rows,): token_logprobs of the same tokens under the model that tuning began with, a
    constant; None: zeros.  smoothing: the share of pairs that are thought to be the wrong way
    round, up to 0.5.  rewards (n, 2): beta S, without a gradient.  A target past V makes its
    pair, and the loss, NaN.

    fp32 results (fp64 of fp64 logits), sums over rows in fp64.  The kernels read the logits once for
    the loss and once for the gradient, which is formed in the backward."""
    _check_logits("preference_loss", logits, targets)
    _check_rows("preference_loss", logits, reference=reference)
    if not isinstance(starts, _Tensor):
        raise TypeError("preference_loss: starts is a tensor")
    if (starts.dim() != 1 or starts.shape[0] < 3 or starts.shape[0] % 2 == 0 or starts.device != logits.device
            or starts.dtype not in (torch.int32, torch.int64)):
        raise ValueError("preference_loss: starts (2 n + 1,), n >= 1, of int32 or int64 on the logits' device")
    beta, smoothing = float(beta), _check_number("preference_loss", "smoothing", smoothing, 0.0, 0.5)
    if not (beta > 0 and math.isfinite(beta)):
        raise ValueError("preference_loss: beta > 0")
    if _eager() and logits.is_cuda and 2.0 ** -60 < beta < 2.0 ** 60 and starts.shape[0] < 1 << 25:
        dense, goals = _dense(logits), targets.contiguous()
        (ref,) = _fp32_rows(reference)
        if _rows_usable(dense, goals, ref) and _here(starts):
            if _tracked(dense):
                return _PreferenceFn.apply(dense, goals, starts, ref, beta, smoothing, True)
            return _PreferenceFn.forward(None, dense, goals, starts, ref, beta, smoothing, False)
    reference = reference if reference is None else reference.detach()
    return _preference_torch(logits, targets, starts, reference, beta, smoothing)


# -------------------------------- policy ------------------------------------

def _policy_torch(logits, targets, old, advantages, reference, low, high, kl):
    """The loss and the log-probabilities as torch expressions, in fp32 (fp64 for fp64)."""
    wide = _wide(logits)
    l, counts = _logprobs_torch(logits, targets)
    # (rows that do not count have no part, whatever they hold)
    old, A = torch.where(counts, old.to(wide), 0.0), torch.where(counts, advantages.to(wide), 0.0)
    log_ratio = l - old
    with torch.no_grad():
        ratio = torch.exp(log_ratio)
        clamped = (A > 0) & (ratio > 1 + high) | (A < 0) & (ratio < 1 - low)
        idle = (A == 0) & ~ratio.isnan()
    # (not a minimum: past its bound, or without an advantage, the ratio may be infinite, and its gradient NaN)
    ratio = torch.exp(torch.where(clamped | idle, 0.0, log_ratio))
    each = -A * torch.where(clamped, torch.where(A > 0, A.new_full((), 1 + high), A.new_full((), 1 - low)), ratio)
    if reference is not None:
        away = torch.where(counts, reference.to(wide), 0.0) - l
        each = each + kl * (torch.expm1(away) - away)
    return (torch.where(counts, each, 0.0).double().sum() / counts.sum()).to(wide), l.detach()


def _policy_call(logits, targets, old, advantages, reference, rule, scratch, loss=None, logp=None, dx=None, dloss=None, unless_one=False):
    """scratch: the rows' losses and the count, the call's own or an earlier call's on the same targets."""
    rows, V = logits.shape
    ready = scratch is not None
    if not ready:
        scratch = torch.empty(rows + 1, dtype=_f32, device=logits.device)
    at = scratch.data_ptr()
    ops._call("compact_policy",
              _policy_pack(logits.data_ptr(), targets.data_ptr(), old.data_ptr(), advantages.data_ptr(), _at(reference),
                           at + 4 * rows, 0 if loss is None else at, _at(loss), _at(logp), _at(dx), _at(dloss), rows, V, IGNORE,
                           logits.dtype == _f32, unless_one, ready, *rule), _stream(logits))
    return scratch


class _PolicyFn(torch.autograd.Function):
    """The loss, and with it the gradient for dloss = 1, while a row is in registers: the
    backward finds dloss to be 1 on the GPU and leaves it, or forms it again.  (The gradient is
    held beside the logits till then, not as a saved tensor: what the backward returns must not
    be shared.)  A backward that is captured without its forward, or the other way round, forms its own."""

    @staticmethod
    def forward(ctx, logits, targets, old, advantages, reference, rule):
        loss = torch.empty((), dtype=_f32, device=logits.device)
        logp = torch.empty(logits.shape[0], dtype=_f32, device=logits.device)
        ctx.dx = torch.empty_like(logits)
        ctx.scratch = _policy_call(logits, targets, old, advantages, reference, rule, None, loss=loss, logp=logp, dx=ctx.dx)
        ctx.capture = ops._capture(_stream(logits))
        ctx.rule = rule
        ctx.size = logits.dtype, logits.shape
        ctx.save_for_backward(logits, targets, old, advantages, reference)
        ctx.mark_non_differentiable(logp)
        ctx.set_materialize_grads(False)
        return loss, logp

    @staticmethod
    def backward(ctx, dloss, _):
        none = (None,) * 5
        if dloss is None:
            return None, *none
        logits, targets, *rows = ctx.saved_tensors
        # (the gradient's buffer and the scratch are of the forward's types and sizes)
        if (torch.is_grad_enabled() or not _eager() or not _plain(dloss) or (logits.dtype, logits.shape) != ctx.size
                or not _rows_usable(logits, targets, *rows)):
            return ops._torch_grad(lambda t: _policy_torch(t, targets.to(torch.int64), *rows, *ctx.rule)[0], logits, dloss), *none
        dx, ctx.dx = ctx.dx, None
        # (a second backward over a retained graph forms its own, too)
        first = dx is not None and ctx.capture == ops._capture(_stream(logits))
        dx = dx if first else torch.empty_like(logits)
        _policy_call(logits, targets, *rows, ctx.rule, ctx.scratch, dx=dx, dloss=dloss.float(), unless_one=first)
        return dx, *none


def policy_loss(logits, targets, old, advantages, reference=None, clip=0.2, kl=0.0):
    """(loss, logprobs) of sampled tokens: with l = log softmax(logits)_target, r = exp(l - old) and
    the advantage A of each row, the mean over the rows that count of

        -min(r A, clamp(r, 1 - low, 1 + high) A) + kl (exp(d) - d - 1),    d = reference - l

    logits (rows, V), targets (rows,): the sampled tokens, -100 where a row does not count, as a
    prompt's.  old, advantages, reference (rows,): constants; old and reference are token_logprobs
    of the same tokens under the policy that sampled, and under the model that it is held to (needed
    where kl > 0).  clip: low and high, or one number for both; low at most 1.  logprobs (rows,):
    l, 0 where a row does not count, without a gradient.  A row that counts for none of it (r
    clamped away or A zero, no KL term) has a gradient of zero, also where r overflows; a target past V
    makes its row and the loss NaN.

    fp32 results (fp64 of fp64 logits).  The kernels form the gradient with the loss and hold it
    for the backward, as many bytes as the logits.  Of a loss that is multiplied before its backward,
    or whose forward and backward are not captured into one graph but into two, or one of them alone, it
    is formed a second time there."""
    _check_logits("policy_loss", logits, targets)
    if old is None or advantages is None:
        raise TypeError("policy_loss: old and advantages are tensors")
    _check_rows("policy_loss", logits, old=old, advantages=advantages, reference=reference)
    low, high = clip if isinstance(clip, (tuple, list)) and len(clip) == 2 else (clip, clip)
    low = _check_number("policy_loss", "the lower clip", low, 0.0, 1.0)
    high, kl = _check_number("policy_loss", "the upper clip", high, 0.0, 2.0 ** 60), _check_number("policy_loss", "kl", kl, 0.0, 2.0 ** 60)
    if kl > 0 and reference is None:
        raise ValueError("policy_loss: a KL term needs a reference")
    reference = reference if kl > 0 else None
    if _eager() and logits.is_cuda:
        dense, goals = _dense(logits), targets.contiguous()
        rows = _fp32_rows(old, advantages, reference)
        if _rows_usable(dense, goals, *rows):
            if _tracked(dense):
                return _PolicyFn.apply(dense, goals, *rows, (low, high, kl))
            loss = torch.empty((), dtype=_f32, device=dense.device)
            logp = torch.empty(dense.shape[0], dtype=_f32, device=dense.device)
            _policy_call(dense, goals, *rows, (low, high, kl), None, loss=loss, logp=logp)
            return loss, logp
    rows = [t if t is None else t.detach() for t in (old, advantages, reference)]
    return _policy_torch(logits, targets, *rows, low, high, kl)


# ------------------------------- clipping -----------------------------------

_CLIP_KINDS = {_bf16: 0, _f32: 1}


def _clip_torch(tensors, max_norm, device):
    """The norm, with sums in fp64, and the scaling as torch expressions."""
    total = torch.zeros((), dtype=torch.float64, device=device)
    for t in tensors:
        total = total + t.double().square().sum()
    norm = total.sqrt()
    if max_norm is not None:
        factor = (max_norm / (norm + 1e-6)).clamp(max=1.0)
        for t in tensors:
            t.copy_(torch.where(factor == 1.0, t, (t.to(_wide(t)) * factor.to(_wide(t))).to(t.dtype)))
    return norm.to(_f32)


def _clip_pieces(entries, n):
    fn = _fns.get("pieces")
    if fn is None:
        fn = _lib.load().compact_clip_pieces
        fn.restype, fn.argtypes = _i64, [_vp, _i64, _vp]
        _fns["pieces"] = fn  # (for other threads to find: complete)
    order = array("q", bytes(8 * n))
    return fn(entries, n, order.buffer_info()[0])


_fns = {}


# Asked of many tensors, by calls that map makes: a loop in Python takes three times as long.
_pointers, _numels, _devices, _dtypes, _dense_all = (
    _Tensor.data_ptr, _Tensor.numel, _Tensor.get_device, _Tensor.dtype.__get__, _Tensor.is_contiguous)


def _clip_entries(tensors):
    """Addresses, elements and kinds of dense bf16 and fp32 tensors of the current GPU; None of others."""
    if not set(map(type, tensors)).issubset(ops._TYPES):
        return None
    at = set(map(_devices, tensors))  # -1: the CPU
    if len(at) != 1 or min(at) < 0 or at != {_device_now()}:
        return None
    try:
        at, kinds = map(_pointers, tensors), [_CLIP_KINDS[d] for d in map(_dtypes, tensors)]
        entries = array("Q", chain.from_iterable(zip(at, map(_numels, tensors), kinds)))
    except (KeyError, RuntimeError):  # another type; a tensor that wraps another has no pointer
        return None
    return entries if all(map(_dense_all, tensors)) else None


def _clip_apply(entries, device, max_norm):
    at, n = entries.buffer_info()[0], len(entries) // 3
    pieces = _clip_pieces(at, n)
    if pieces == -2:
        raise ValueError("clip_grad_norm: two of the tensors overlap")
    if pieces < 0:
        return None
    scratch = torch.empty(pieces, dtype=torch.float64, device=device)
    out = torch.empty(2, dtype=_f32, device=device)  # (not a part of the scratch, which a norm that is kept would keep)
    ops._call("compact_clip", at, n, 0.0 if max_norm is None else max_norm, max_norm is not None, scratch.data_ptr(), pieces,
              out.data_ptr(), _stream(scratch))
    return out[0]


@torch.no_grad()
def clip_grad_norm(tensors, max_norm=None):
    """The norm sqrt(sum g^2) over all elements of the given tensors (fp32, on their device), and
    with a max_norm each of them multiplied, where it stands, by

        min(1, max_norm / (norm + 1e-6)).

    tensors: gradients of any shapes on one device, one or an iterable of them; None among them,
    as of a parameter without a gradient, is passed over, and one that is given twice, in whatever
    shape or order of its dimensions, counts once.  Tensors that share a part of their elements are
    refused, also where only the norm is asked for.  Of a norm that is infinite, finite gradients
    become 0; of one that is NaN, all become NaN.

    The kernels take dense bf16 and fp32 tensors, mixed, in any order of their dimensions; views of
    others that are not dense are copied, and back.  Squares are added in fp64.  Nothing is
    written where the norm is within its bound, and nothing is waited for."""
    given = [tensors] if isinstance(tensors, _Tensor) else list(tensors)
    given = [t for t in given if t is not None]
    if max_norm is not None:
        max_norm = float(max_norm)
        if not max_norm >= 0:
            raise ValueError("clip_grad_norm: max_norm >= 0")
        if math.isinf(max_norm):
            max_norm = None
    entries = _clip_entries(given) if given and _eager() else None
    if entries is not None:
        norm = _clip_apply(entries, given[0].device, max_norm)
        if norm is not None:
            if max_norm is not None:
                _changed(given)
            return norm
    for t in given:
        if not isinstance(t, _Tensor) or not t.is_floating_point() or t.layout != torch.strided:
            raise TypeError("clip_grad_norm: dense floating tensors")
    device = given[0].device if given else None
    if any(t.device != device for t in given):
        raise ValueError("clip_grad_norm: tensors of one device")
    given = [t for t in given if t.numel() > 0]
    if all(map(_plain, given)):
        given = _distinct(given)
    if max_norm is not None and any(not t.is_contiguous() and torch._debug_has_internal_overlap(t) == 1 for t in given):
        raise ValueError("clip_grad_norm: a tensor whose elements lie on one another is not scaled")
    if given and _eager():
        dense = [t if t.is_contiguous() else _flat(t) for t in given]
        entries = _clip_entries(dense)
        norm = None if entries is None else _clip_apply(entries, device, max_norm)
        if norm is not None:
            if max_norm is not None:
                for t, d in zip(given, dense):
                    if d.data_ptr() != t.data_ptr():
                        t.copy_(d)
                _changed(given)
            return norm
    return _clip_torch(given, max_norm, device)


def _memory(t):
    """Where a tensor's elements lie, whatever their order and shape: (address, an element's bytes, ((stride in bytes,
    count), ..)), the widest stride first, dimensions that continue one another joined."""
    size, dims = t.element_size(), []
    if t.is_contiguous():
        n = t.numel()
        return t.data_ptr(), size, ((size, n),) if n > 1 else ()
    for stride, n in sorted(((s * size, n) for s, n in zip(t.stride(), t.shape) if n > 1), reverse=True):
        if dims and dims[-1][0] == stride * n:
            dims[-1] = (stride, dims[-1][1] * n)
        else:
            dims.append((stride, n))
    return t.data_ptr(), size, tuple(dims)


def _extent(memory):
    """Bytes from the first element's to the last one's end."""
    _, size, dims = memory
    return size + sum(stride * (n - 1) for stride, n in dims)


def _apart(a, b):
    """No byte of one tensor is the other's."""
    if a[0] > b[0]:
        a, b = b, a
    ahead = b[0] - a[0]
    if ahead >= _extent(a):
        return True
    if all(not dims or len(dims) == 1 and dims[0][0] == size for _, size, dims in (a, b)):
        return False  # dense, both
    # slices of one tensor: the strides of the dimensions outside are multiples of g, and what lies inside
    # takes places of its own in every g bytes
    for least in {stride for _, _, dims in (a, b) for stride, _ in dims if stride > 0}:
        outside = [stride for _, _, dims in (a, b) for stride, _ in dims if stride >= least]
        g = math.gcd(*outside)
        inside = [_extent((at, size, [d for d in dims if d[0] < least])) for at, size, dims in (a, b)]
        if inside[0] <= ahead % g <= g - inside[1]:
            return True
    unit = math.gcd(ahead, a[1], b[1], *(stride for _, _, dims in (a, b) for stride, _ in dims))
    mark = torch.zeros(max(_extent(a), ahead + _extent(b)) // unit, dtype=torch.bool)
    places = []
    for first, (_, size, dims) in ((0, a), (ahead, b)):
        dims = [d for d in dims if d[0] > 0] + [(unit, size // unit)]
        places.append(mark.as_strided([n for _, n in dims], [stride // unit for stride, _ in dims], first // unit))
    places[0].fill_(True)
    return not places[1].any()


def _distinct(tensors):
    """The tensors, without those that hold an earlier one's elements."""
    found, live = {}, []
    nowhere = [t for t in tensors if t.data_ptr() == 0]  # (of the meta device, zeros without memory)
    for t in tensors:
        if t.data_ptr() != 0:
            found.setdefault((_memory(t), t.dtype), t)
    for memory, _ in sorted(found, key=lambda m: m[0][0]):
        live = [m for m in live if m[0] + _extent(m) > memory[0]]
        if not all(_apart(m, memory) for m in live):
            raise ValueError("clip_grad_norm: two of the tensors overlap")
        live.append(memory)
    return [*found.values(), *nowhere]


def _changed(tensors):
    """Whoever saved them is told."""
    torch.autograd.graph.increment_version([t for t in tensors if not t.is_inference()])


def _flat(t):
    """A dense tensor's own memory in its order of dimensions, or a copy."""
    order = sorted(range(t.dim()), key=lambda d: -t.stride(d) if t.shape[d] > 1 else 0)
    p = t.permute(order)
    if p.is_contiguous():
        return p
    return t.contiguous()
