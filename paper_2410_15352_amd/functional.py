"""Operators of long-context and distilled training, as functions and modules of their own:

    Rotary             rotary positions: half and interleaved layouts, a part of the head,
                       frequencies scaled for long contexts
    window_attention   attention with a sliding window and a few first tokens that stay
                       visible (sinks); training, prompts, and single tokens over a cache
    packed_attention   the same inside each of several sequences that lie end to end
    distill_loss       distillation from a teacher's top logits, beside the targets

On the current GPU they run the HIP kernels of libcompact.so (csrc/rotary.hip, attention.hip,
packed.hip, distill.hip) on the current stream, forward and backward: bf16 (Rotary and distill_loss fp32
too), any strides whose rows start on 16-byte boundaries (others are copied first).  Other
types and places, autocast, tracing and functorch take the torch expressions beside each
function, and so does a backward that is itself recorded or batched.  Arguments that no form
takes are refused with ValueError or TypeError."""
from __future__ import annotations

import contextlib
import ctypes
import math
import struct
from operator import index

import torch

from . import _block_ops as ops
from . import _lib
from ._block_ops import _eager, _i64, _plain, _stream, _vp

__all__ = ["Rotary", "window_attention", "packed_attention", "packed_positions", "distill_loss"]

_bf16 = torch.bfloat16

# The argument blocks of csrc/functional.hpp as native struct layouts (a ctypes.Structure
# costs ten times as much to fill), passed by address.
_ROTARY = struct.Struct("@" + 3 * "2Q6q2i" + "2Q4q8if").pack
_ATTN = "7Q12q8if2i2Q"
_attn_pack = struct.Struct("@" + _ATTN).pack
_attn_grad_pack = struct.Struct("@" + _ATTN + "5Q12qQ6i").pack
_distill_pack = struct.Struct("@11Q5q6i2f").pack
_block = ctypes.c_char_p

ops._SIGNATURES.update({
    "compact_rotary": [_block, _vp],
    "compact_attention_fwd": [_block, _vp],
    "compact_attention_bwd": [_block, _vp],
    "compact_packed_fwd": [_block, _vp, ctypes.c_int, _i64, ctypes.c_int, _vp, _vp],
    "compact_packed_bwd": [_block, ctypes.c_int, _vp, _vp],
    "compact_distill": [_block, _vp],
})


_TYPES = ops._TYPES
_device_now = torch._C._cuda_getDevice
_is_compiling = torch.compiler.is_compiling
_Tensor = torch.Tensor


def _here(t):
    """A tensor of its own storage on the current GPU."""
    return _plain(t) and t.is_cuda and t.get_device() == _device_now()


def _strides(t):
    """The strides of the first three dimensions; 0 where a dimension has one element."""
    x, y, z, _ = t.stride()
    b, c, d, _ = t.shape
    return (x if b > 1 else 0, y if c > 1 else 0, z if d > 1 else 0)


def _rows(t):
    """t (4-D), or a copy of it, whose last dimension is dense and whose every row is on a
    16-byte boundary, and its strides."""
    x, y, z, w = t.stride()
    b, c, d, _ = t.shape
    s = (x if b > 1 else 0, y if c > 1 else 0, z if d > 1 else 0)
    if w != 1 or (t.data_ptr() | (s[0] | s[1] | s[2]) * t.element_size()) % 16 != 0:
        t = t.contiguous()
        t = t if t.data_ptr() % 16 == 0 else t.clone()
        s = _strides(t)
    return t, s


LEAST_FACTOR, MOST_FACTOR = 2.0 ** -60, 2.0 ** 60  # scales and temperatures: their squares and inverses are fp32 numbers


def _tracked(*tensors):
    """A gradient of some tensor is wanted."""
    return torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors)


# ------------------------------- rotary -------------------------------------

def _rotary_frequencies(dims, base, scaling, factor, original_length, low, high):
    """Radians per position of each pair, and the factor on the rotated values."""
    if scaling == "ntk":
        base = base * factor ** (dims / (dims - 2))
    f = [base ** (-2 * i / dims) for i in range(dims // 2)]
    if scaling == "linear":
        return [x / factor for x in f], 1.0
    if scaling == "parts":
        def part(x):
            # 1: the pair turns at least `high` times over the trained length, and is kept; 0: at most `low` times
            keep = min(1.0, max(0.0, (original_length * x / (2 * math.pi) - low) / (high - low)))
            return x * (keep + (1 - keep) / factor)
        return [part(x) for x in f], 0.1 * math.log(factor) + 1
    return f, 1.0


MAX_POSITION = 1 << 53  # positions are fp64 factors


class Rotary(torch.nn.Module):
    """Rotary positions: pair i of the first `dims` elements of a head turns by position x
    base^(-2 i / dims), the rest of the head stays.

    layout: "half" (element i with i + dims / 2) or "interleaved" (2 i with 2 i + 1).
    scaling, for contexts `factor` times as long as the trained ones:
      "none"
      "linear"  every frequency divided by factor
      "ntk"     base raised by factor^(dims / (dims - 2)): the slowest pair as with "linear",
                the fastest as it was
      "parts"   by the turns that a pair makes over original_length: `high` and more keep the
                frequency, `low` and fewer divide it by factor, a ramp between; the rotated
                values are multiplied by 0.1 ln(factor) + 1 (in q and in k)

    rope(q, k, positions=...) rotates q (b, l, heads, hd) and, if given, k (b, l, kv, hd);
    positions: None (0, 1, ...), an int (the first one's), or integers of shape (l,) or (b, l),
    which the backward reads again: written in between, autograd refuses it.
    No parameters; the angles are exact for any position (fp64)."""

    def __init__(self, dims, base=10000.0, layout="half", scaling="none", factor=1.0, original_length=2048, low=1.0,
                 high=32.0):
        super().__init__()
        if dims < 2 or dims % 2 != 0:
            raise ValueError("rotary dims: an even number from 2 on")
        if layout not in ("half", "interleaved"):
            raise ValueError('rotary layout: "half" or "interleaved"')
        if scaling not in ("none", "linear", "ntk", "parts"):
            raise ValueError('rotary scaling: "none", "linear", "ntk" or "parts"')
        if (not (base > 0 and factor >= 1 and original_length > 0 and high > low) or scaling == "ntk" and dims == 2
                or not all(map(math.isfinite, (base, factor, original_length, low, high)))):
            raise ValueError("rotary: base > 0, factor >= 1, original_length > 0, high > low, and dims > 2 with ntk")
        self.dims, self.interleaved = dims, layout == "interleaved"
        f, self.magnitude = _rotary_frequencies(dims, float(base), scaling, float(factor), original_length, low, high)
        # (not a buffer: module.to(dtype) must not round it)
        self._revolutions = [x / (2 * math.pi) for x in f]
        self._turns = {}  # by device

    def turns(self, device):
        """Revolutions per position of each pair, fp64; kept for the device, but for what a
        transform or a tracer makes of them."""
        t = self._turns.get(device) if _eager() else None
        if t is not None:
            return t
        if device.type == "cuda" and not _is_compiling() and torch.cuda.is_current_stream_capturing():
            # a copy from the host is not captured; these are part of the graph and hold nothing before its replay
            t = torch.empty(len(self._revolutions), dtype=torch.float64, device=device)
            for i, x in enumerate(self._revolutions):
                t[i].fill_(x)
            return t
        with torch.inference_mode(False) if torch.is_inference_mode_enabled() else contextlib.nullcontext():
            t = torch.tensor(self._revolutions, dtype=torch.float64, device=device)
        if _eager() and _plain(t):
            self._turns[device] = t
        return t

    def forward(self, q, k=None, positions=None):
        self._check(q, k, positions)
        if not self._usable(q, k, positions):
            out = _rotary_torch(self, positions, False, q, k)
        elif _tracked(q, k):
            out = _RotaryFn.apply(self, positions, q, k)
        else:
            out = _rotary_apply(self, positions, 0, q, k)
        return out if k is not None else out[0]

    def _check(self, q, k, positions):
        for t in (q, k):
            if t is None:
                continue
            if not isinstance(t, _Tensor):
                raise TypeError("rotary: q and k are tensors")
            if t.dim() != 4 or t.shape[:2] != q.shape[:2] or t.shape[3] != q.shape[3]:
                raise ValueError("rotary: q (b, l, heads, hd) and k (b, l, kv, hd)")
            if not t.is_floating_point() or t.dtype != q.dtype or t.device != q.device:
                raise TypeError("rotary: q and k of one floating type on one device")
        if self.dims > q.shape[3]:
            raise ValueError(f"rotary: {self.dims} dims of heads of {q.shape[3]}")
        if isinstance(positions, torch.Tensor):
            if positions.dtype not in (torch.int64, torch.int32) or positions.device != q.device:
                raise TypeError("rotary positions: int64 or int32 on q's device")
            if positions.shape not in (q.shape[1:2], q.shape[:2]):
                raise ValueError("rotary positions: shape (l,) or (b, l)")
        elif positions is not None and not isinstance(positions, int):
            raise TypeError("rotary positions: None, an int or a tensor of integers")
        elif positions is not None and not -MAX_POSITION <= positions <= MAX_POSITION:
            raise ValueError("rotary positions: within 2^53")

    def _usable(self, *tensors_and_positions):
        if not _eager():
            return False
        q, k, positions = tensors_and_positions
        if not all(_here(t) for t in (q, k) if t is not None) or q.dtype not in (_bf16, torch.float32):
            return False
        b, l, heads, hd = q.shape
        n = 16 // q.element_size()
        return (hd % n == 0 and n <= hd <= 1024 and min(q.shape) > 0 and (k is None or k.shape[2] > 0)
                and (heads + (0 if k is None else k.shape[2])) * hd < 1 << 16 and b * l < ops.MAX_ROWS
                and (not isinstance(positions, torch.Tensor) or _plain(positions)))


_NO_TENSOR = (0,) * 10


def _rotary_call(rope, positions, inverse, x, fields, count):
    """fields: of each of `count` tensors like x (b, l, heads, hd), its source and destination,
    their strides, its heads and whether it is turned."""
    b, l, _, hd = x.shape
    at, pos_b, pos_l, offset, pos32 = 0, 0, 0, 0, 0
    if isinstance(positions, torch.Tensor):
        at, pos32 = positions.data_ptr(), positions.dtype == torch.int32
        pos_b, pos_l = (0, *positions.stride()) if positions.dim() == 1 else positions.stride()
    else:
        offset = positions or 0
    turns = rope._turns.get(x.device)
    turns = rope.turns(x.device) if turns is None else turns
    ops._call("compact_rotary",
              _ROTARY(*fields, *_NO_TENSOR * (3 - count), turns.data_ptr(), at, pos_b, pos_l, offset, b * l, l,
                      hd, rope.dims, count, rope.interleaved, inverse, pos32, x.dtype == torch.float32, rope.magnitude),
              _stream(x))


def _rotary_apply(rope, positions, inverse, *tensors):
    out, fields, kept = [], [], []
    for t in tensors:
        if t is None:
            continue
        src, strides = _rows(t)
        _, l, heads, hd = src.shape
        dst = torch.empty(src.shape, dtype=src.dtype, device=src.device)
        fields += (src.data_ptr(), dst.data_ptr(), *strides, l * heads * hd, heads * hd, hd, heads, 1)
        out.append(dst)
        kept.append(src)
    _rotary_call(rope, positions, inverse, kept[0], fields, len(out))
    return out


def _rotary_torch(rope, positions, inverse, *tensors):
    """The rotation as torch expressions, in fp32 (fp64 for fp64)."""
    x = tensors[0]
    b, l = x.shape[:2]
    if not isinstance(positions, torch.Tensor):
        positions = torch.arange(l, device=x.device) + (positions or 0)
    turn = positions.unsqueeze(-1).double() * rope.turns(x.device)
    angle = 2 * math.pi * (turn - turn.round())
    wide = torch.float64 if x.dtype == torch.float64 else torch.float32
    cos = (rope.magnitude * torch.cos(angle)).to(wide).unsqueeze(-2)
    sin = (rope.magnitude * torch.sin(angle)).to(wide).unsqueeze(-2)
    sin = -sin if inverse else sin
    out = []
    D = rope.dims
    for t in tensors:
        if t is None:
            out.append(None)
            continue
        y = t[..., :D].to(wide)
        a, c = (y[..., 0::2], y[..., 1::2]) if rope.interleaved else (y[..., :D // 2], y[..., D // 2:])
        pair = (a * cos - c * sin, c * cos + a * sin)
        y = torch.stack(pair, -1).flatten(-2) if rope.interleaved else torch.cat(pair, -1)
        out.append(torch.cat((y.to(t.dtype), t[..., D:]), -1))
    return tuple(out)


def _save_positions(ctx, positions):
    """A tensor as autograd keeps them: written again before the backward, it is refused there."""
    if isinstance(positions, torch.Tensor):
        ctx.positions = positions.dtype, positions.shape
        ctx.save_for_backward(positions)
    else:
        ctx.positions = positions


def _saved_positions(ctx, x):
    """(a saved-tensor hook may have given them another type, place or shape)"""
    if not isinstance(ctx.positions, tuple):
        return ctx.positions
    (positions,), (dtype, shape) = ctx.saved_tensors, ctx.positions
    if positions.dtype is dtype and positions.shape == shape and positions.device == x.device:
        return positions
    return positions.to(x.device, dtype).reshape(shape)


class _RotaryFn(torch.autograd.Function):
    """q and k turned; nothing is kept but the positions."""

    @staticmethod
    def forward(ctx, rope, positions, q, k):
        ctx.rope, ctx.pair = rope, k is not None
        _save_positions(ctx, positions)
        ctx.set_materialize_grads(False)
        out = _rotary_apply(rope, positions, 0, q, k)
        return tuple(out) if ctx.pair else (out[0], None)

    @staticmethod
    def backward(ctx, dq, dk):
        given = [t for t in (dq, dk) if t is not None]
        if not given:
            return None, None, None, None
        positions = _saved_positions(ctx, given[0])
        if torch.is_grad_enabled() or not ctx.rope._usable(given[0], given[-1], positions):
            out = iter(_rotary_torch(ctx.rope, positions, True, *given))
        else:
            out = iter(_rotary_apply(ctx.rope, positions, 1, *given))
        dq, dk = (None if t is None else next(out) for t in (dq, dk))
        return None, None, dq, dk


class _RotaryQkvFn(torch.autograd.Function):
    """q, k (turned in place) and v (b, heads, l, hd) as views of qkv (b, l, 3, heads, hd);
    the backward turns back and joins their gradients in one pass."""

    @staticmethod
    def forward(ctx, rope, positions, qkv):
        ctx.rope, ctx.shape = rope, qkv.shape
        _save_positions(ctx, positions)
        ctx.set_materialize_grads(False)
        q, k, v = qkv.unbind(2)
        _rotary_call(rope, positions, 0, q, [x for t in (q, k) for x in (t.data_ptr(), t.data_ptr(), *_strides(t), *_strides(t),
                                                                        t.shape[2], 1)], 2)
        torch.autograd.graph.increment_version(qkv)  # whoever saved it is told
        return tuple(t.transpose(1, 2) for t in (q, k, v))

    @staticmethod
    def backward(ctx, *grads):
        some = next((g for g in grads if g is not None), None)
        if some is None:
            return None, None, None
        grads = [torch.zeros_like(some) if g is None else g for g in grads]
        dq, dk, dv = (g.transpose(1, 2) for g in grads)
        positions = _saved_positions(ctx, dv)
        if torch.is_grad_enabled() or not _here(dv) or not ctx.rope._usable(dq, dk, positions):
            dq, dk = _rotary_torch(ctx.rope, positions, True, dq, dk)
            return None, None, torch.stack((dq, dk, dv), 2)
        out = torch.empty(ctx.shape, dtype=dq.dtype, device=dq.device)
        rows = [_rows(g) for g in (dq, dk, dv)]
        _rotary_call(ctx.rope, positions, 1, rows[0][0],
                     [x for (g, s), to, rotate in zip(rows, out.unbind(2), (1, 1, 0))
                      for x in (g.data_ptr(), to.data_ptr(), *s, *_strides(to), g.shape[2], rotate)], 3)
        return None, None, out


def rotary_split_qkv(qkv, rope, positions=None, in_place=True):
    """q, k (turned) and v (b, heads, l, hd) of qkv (b, l, 3, heads, hd), which a projection
    has just written: in_place, the kernel turns q and k where they stand, so the block keeps no
    more than without positions."""
    q, k, v = qkv.unbind(2)
    if not in_place:
        return tuple(t.transpose(1, 2) for t in (*rope(q, k, positions), v))
    rope._check(q, k, positions)
    if (rope._usable(q, k, positions) and qkv.is_contiguous() and qkv.data_ptr() % 16 == 0
            and not (qkv.is_leaf and qkv.requires_grad)):
        return _RotaryQkvFn.apply(rope, positions, qkv)
    q, k = _rotary_torch(rope, positions, False, q, k)
    return tuple(t.transpose(1, 2) for t in (q, k, v))


# ------------------------------ attention -----------------------------------

NO_WINDOW = 1 << 30
MAX_HD = 128
MAX_ROW_STRIDE = (1 << 24) - 512


def _visible(lq, lk, lengths, window, sinks, device):
    """(b or 1, 1, lq, lk): key j is seen from row i."""
    j = torch.arange(lk, device=device)
    L = torch.full((1,), lk, device=device) if lengths is None else lengths.to(torch.int64).clamp(0, lk)
    p = (torch.arange(lq, device=device) + (L.unsqueeze(-1) - lq)).unsqueeze(-1)
    seen = j <= p
    if window is not None:
        seen = seen & ((p - j < window) | (j < sinks))
    return seen.unsqueeze(1)


def _as_typed(t):
    """Outside autocast: products in the types that they are given."""
    kind = t.device.type
    return torch.autocast(kind, enabled=False) if kind in ("cuda", "cpu") else contextlib.nullcontext()


def _attention_torch(q, k, v, window, sinks, lengths, scale):
    """The attention as torch expressions, in fp32 (fp64 for fp64).  (Autocast would make its
    products bf16 ones, of batches with a transposed operand in the backward.)"""
    with _as_typed(q):
        return _attention_expressions(q, k, v, window, sinks, lengths, scale)


def _attention_expressions(q, k, v, window, sinks, lengths, scale):
    b, heads, lq, hd = q.shape
    kv, lk = k.shape[1:3]
    wide = torch.float64 if q.dtype == torch.float64 else torch.float32
    qw, kw, vw = (t.to(wide) for t in (q, k, v))
    if kv != heads:
        kw, vw = (t.repeat_interleave(heads // kv, 1) for t in (kw, vw))
    if lk == 0:  # (a maximum over nothing is refused; sums over nothing are zero)
        return torch.matmul(torch.matmul(qw, kw.transpose(2, 3)), vw).to(q.dtype)
    return _attend(qw, kw, vw, _visible(lq, lk, lengths, window, sinks, q.device), scale).to(q.dtype)


def _attend(qw, kw, vw, seen, scale):
    """softmax(scale q k^T) v over the keys seen."""
    # (what lies past a sequence, or before every window, may be anything; so may rows that see no key, and their gradient)
    used, some = seen.any(2).unsqueeze(-1), seen.any(-1, keepdim=True)
    qw, kw, vw = torch.where(some, qw, 0.0), torch.where(used, kw, 0.0), torch.where(used, vw, 0.0)
    s = torch.matmul(qw, kw.transpose(2, 3).contiguous()) * scale
    s = torch.where(seen, s, -math.inf)
    top = torch.where(some, s.detach().amax(-1, keepdim=True), 0.0)
    e = torch.exp(s - top)
    p = e / torch.where(some, e.sum(-1, keepdim=True), 1.0)
    return torch.where(some, torch.matmul(p, vw), 0.0)


FEW_ROWS = 32
MAX_JOINED = 1 << 24  # rows of a split call: a workgroup of 256 threads joins each


def attention_splits(b, heads, kv, lq, lk, window, sinks):
    """Ranges of keys that are worked on apart and joined (0: the rows alone fill the card).
    Up to FEW_ROWS rows a head (and MAX_JOINED in all): a wave takes 32 rows of the heads that share keys and
    a range, of at least 4 tiles of 32 keys, or 8 past 1024 waves, and 2048 waves at most.  More rows: a
    workgroup takes 128 of one head; ranges of at least 8 tiles of 64 keys where 256 workgroups
    are not reached.  us, waves / workgroups: 4 x 8192 keys, 32 heads on 8 of 128, 8 rows 35 / 66,
    32 rows 64 / 68, 64 rows 103 / 78; 8 x 4096 keys, 16 heads of 64, 32 rows 34 / 32, 64 rows
    55 / 41.
    One token, us by ranges (the rule's *), heads of 128: 4 sequences of up to 70000 keys, 8
    heads of k: 16 270, 32 196, 64* 192, 128 186; one sequence: 64 77, 128 66, 256* 72, 512 86;
    32 of 8192: 2 194, 8* 202, 16 213; heads of 64, 16 x 16 of 1028 keys: 2 18, 4* 19, 8 20, 16
    21.  1000 rows of 16 heads over 20000 keys: 1 508, 2 281, 4* 191, 8 204."""
    share = heads // kv * lq
    rows = b * heads * lq
    if lq <= FEW_ROWS and b * kv <= 65535 and share <= 32 * 65535 and rows < MAX_JOINED:
        blocks = b * kv * -(-share // 32)
        tiles = -(-min(lk, window + sinks + lq) // 32)
        splits = max(1, min(-(-2048 // blocks), tiles // 4))
        return splits if blocks * splits <= 1024 else min(splits, max(-(-1024 // blocks), tiles // 8))
    blocks = b * heads * -(-lq // 128)
    if blocks >= 256 or rows >= MAX_JOINED:
        return 0
    splits = min(512 // blocks, -(-min(lk, window + sinks + 128) // 64) // 8)
    return splits if splits > 1 else 0


def _attn_tensor(t):
    """A bf16 (b, heads, l, hd) tensor as the kernels take it, and its strides: rows that lie on
    one another, or so far apart that a tile of 64 passes 2^31 bytes, are copied too."""
    l, hd = t.shape[2:]
    if l > 1 and not hd <= t.stride(2) <= MAX_ROW_STRIDE:
        t = t.contiguous()
    return _rows(t)


def _attn_fields(q, k, v, o, stats, lengths, window, sinks, scale, splits=0, waves=0, part=0, part_lse=0):
    """q, k, v, o: (tensor, strides); stats: the rows' log-sums, and with room for it what o's
    rounding took off."""
    b, heads, lq, hd = q[0].shape
    _, kv, lk, _ = k[0].shape
    rows, lse = b * heads * lq, stats.data_ptr()
    return (q[0].data_ptr(), k[0].data_ptr(), v[0].data_ptr(), o[0].data_ptr(), lse,
            lse + -(-rows // 4) * 16 if stats.numel() > rows else 0, 0 if lengths is None else lengths.data_ptr(), *q[1], *k[1], *v[1],
            *o[1], b, heads, kv, lq, lk, hd, NO_WINDOW if window is None or window > NO_WINDOW else window,
            min(sinks, NO_WINDOW), scale, splits, waves, part, part_lse)


def _stats_count(shape, tracked):
    """Floats of a call's statistics: one a row, and a byte for each element of o."""
    b, heads, lq, hd = shape
    rows = b * heads * lq
    return -(-rows // 4) * 4 + rows * hd // 4 if tracked else rows


def _empty_heads(shape, device):
    """(b, heads, l, hd) that lies as (b, l, heads, hd), the layout the projections take, and
    its strides."""
    b, heads, l, hd = shape
    strides = (l * heads * hd, hd, heads * hd)
    return torch.empty_strided(shape, (*strides, 1), dtype=_bf16, device=device), strides


def _attn_scratch(block):
    fn = _fns.get("scratch")
    if fn is None:
        fn = _lib.load().compact_attention_bwd_scratch
        fn.restype, fn.argtypes = _i64, [_block]
        _fns["scratch"] = fn  # (for other threads to find: complete)
    return fn(block)


_fns = {}


def _attention_apply(q, k, v, window, sinks, lengths, scale, tracked=False):
    """q, k, v: as _attn_tensor gives them; (o, the statistics that a backward wants)"""
    shape, device = q[0].shape, q[0].device
    b, heads, lq, hd = shape
    _, kv, lk, _ = k[0].shape
    o = _empty_heads(shape, device)
    stats = torch.empty(_stats_count(shape, tracked), dtype=torch.float32, device=device)
    splits = attention_splits(b, heads, kv, lq, lk, NO_WINDOW if window is None else window, sinks)
    split = ()
    if splits > 0:
        rows = splits * b * heads * lq
        part = torch.empty(rows * (hd + 1), dtype=torch.float32, device=device)
        at = part.data_ptr()
        split = (splits, lq <= FEW_ROWS, at, at + 4 * rows * hd)
    ops._call("compact_attention_fwd", _attn_pack(*_attn_fields(q, k, v, o, stats, lengths, window, sinks, scale, *split)),
              _stream(stats))
    return o[0], stats


class _AttentionFn(torch.autograd.Function):
    """Keeps q, k, v, o, and beside o one fp32 number a row and a byte an element.  Its q, k and v
    lie as the kernels take them: a copy made in here would have no history for a recorded backward."""

    @staticmethod
    def forward(ctx, q, k, v, strides, window, sinks, lengths, scale):
        o, stats = _attention_apply(*zip((q, k, v), strides), window, sinks, lengths, scale, tracked=True)
        ctx.rule = window, sinks, scale
        ctx.shapes = q.shape, k.shape
        ctx.save_for_backward(q, k, v, o, stats, lengths)
        return o

    @staticmethod
    def backward(ctx, do):
        q, k, v, o, stats, lengths = ctx.saved_tensors
        window, sinks, scale = ctx.rule
        none = (None,) * 5
        shape, kv_shape = ctx.shapes
        if (torch.is_grad_enabled() or not _eager() or not _here(do)
                or not ops._companion(stats, torch.float32, _stats_count(shape, True))
                or lengths is not None and not ops._companion(lengths, torch.int32, shape[0])
                or not all(t.dtype is _bf16 and t.shape == s and _here(t)
                           for t, s in ((q, shape), (k, kv_shape), (v, kv_shape), (o, shape)))):
            recorded = torch.is_grad_enabled()
            lengths = lengths if lengths is None else lengths.to(q.device)
            with torch.enable_grad():
                # (aliases: of v = f(k), k's own gradient must not hold what reaches k through v)
                leaves = [x.view_as(x) if recorded and x.requires_grad else x.detach().requires_grad_(True) for x in (q, k, v)]
                y = _attention_torch(*leaves, window, sinks, lengths, scale)
                return (*torch.autograd.grad(y, leaves, do, create_graph=recorded), *none)
        do = _attn_tensor(do if do.dtype is _bf16 else do.to(_bf16))
        fields = _attn_fields(_attn_tensor(q), _attn_tensor(k), _attn_tensor(v), _attn_tensor(o), stats, lengths, window, sinks,
                              scale)
        rows, device = shape[:3].numel(), q.device
        dq, dq_strides = _empty_heads(shape, device)
        dk = dv = None
        outs, strides, floats = (0, 0), (0,) * 6, 0
        if ctx.needs_input_grad[1] or ctx.needs_input_grad[2]:
            (dk, dk_strides), (dv, _) = _empty_heads(k.shape, device), _empty_heads(k.shape, device)
            outs, strides = (dk.data_ptr(), dv.data_ptr()), dk_strides * 2
            floats = _attn_scratch(_attn_pack(*fields))
        scratch = torch.empty(-(-rows // 4) * 4 + floats, dtype=torch.float32, device=device)  # D, and sums in parts
        delta = scratch.data_ptr()
        ops._call("compact_attention_bwd",
                  _attn_grad_pack(*fields, do[0].data_ptr(), dq.data_ptr(), *outs, delta, *do[1], *dq_strides, *strides,
                                  delta + -(-rows // 4) * 16 if floats > 0 else 0, 0, 0, 0, 0, 0, 0), _stream(q))
        return dq, dk, dv, *none


def window_attention(q, k, v, window=None, sinks=0, lengths=None, scale=None):
    """softmax(scale q k^T) v over the keys that each row sees; q (b, heads, lq, hd), k and v
    (b, kv, lk, hd), heads a multiple of kv (query head h reads head h kv // heads).

    A sequence has L keys: lk, or lengths[b] of them (integers on the device, 0 .. lk; what lies
    past them is not read).  Its rows are its last lq positions: row i stands at p = i + L - lq
    and sees key j when j <= p and (p - j < window or j < sinks); window None: every j <= p.
    A row that sees no key (lq > L) gives zeros and passes no gradient; one that sees scores of
    -inf alone gives NaN.  A key that a row does not see has no part in it, whatever it holds.
    scale: 1 / sqrt(hd) if None.

    The kernels take bf16 with heads of up to 128 elements, a multiple of 8.  In the torch
    expressions an infinite or NaN key or value that some rows see makes the others NaN too.  A gradient of a row with NaN is NaN."""
    if not (isinstance(q, _Tensor) and isinstance(k, _Tensor) and isinstance(v, _Tensor)
            and (lengths is None or isinstance(lengths, _Tensor))):
        raise TypeError("window_attention: q, k, v and lengths are tensors")
    if q.dim() != 4 or k.dim() != 4 or v.dim() != 4 or q.shape[3] == 0:
        raise ValueError("window_attention: q (b, heads, lq, hd), k and v (b, kv, lk, hd), hd >= 1")
    if k.shape != v.shape or q.shape[0] != k.shape[0] or q.shape[3] != k.shape[3]:
        raise ValueError(f"window_attention: q {tuple(q.shape)}, k {tuple(k.shape)}, v {tuple(v.shape)}")
    if k.shape[1] == 0 or q.shape[1] % k.shape[1] != 0:
        raise ValueError(f"window_attention: {q.shape[1]} query heads over {k.shape[1]} of k and v")
    if not q.is_floating_point() or q.dtype != k.dtype or q.dtype != v.dtype or not q.device == k.device == v.device:
        raise TypeError("window_attention: q, k and v of one floating type on one device")
    window, sinks = None if window is None else index(window), index(sinks)
    if window is not None and window < 1 or sinks < 0:
        raise ValueError("window_attention: window >= 1 (or None) and sinks >= 0")
    if lengths is not None:
        if lengths.shape != q.shape[:1] or lengths.device != q.device or lengths.dtype not in (torch.int32, torch.int64):
            raise ValueError("window_attention: lengths (b,) of int32 or int64 on q's device")
    scale = q.shape[3] ** -0.5 if scale is None else float(scale)
    if not (scale > 0 and math.isfinite(scale)):
        raise ValueError("window_attention: scale > 0")
    tracked = torch.is_grad_enabled() and (q.requires_grad or k.requires_grad or v.requires_grad)
    if _eager() and LEAST_FACTOR < scale < MOST_FACTOR and _attention_usable(q, k, v, tracked):
        if lengths is not None:
            lengths = lengths.to(torch.int32).contiguous()
        if window is not None and window + sinks >= k.shape[2]:
            window, sinks = None, 0  # every earlier key is one or the other
        q, k, v = _attn_tensor(q), _attn_tensor(k), _attn_tensor(v)
        if tracked:
            return _AttentionFn.apply(q[0], k[0], v[0], (q[1], k[1], v[1]), window, sinks, lengths, scale)
        return _attention_apply(q, k, v, window, sinks, lengths, scale)[0]
    return _attention_torch(q, k, v, window, sinks, lengths, scale)


def _attention_usable(q, k, v, tracked):
    b, heads, lq, hd = q.shape
    kv, lk = k.shape[1:3]
    # a launch has under 2^32 threads; dk and dv take a workgroup for 128 keys and up to two for 128 sinks
    if tracked and 4 * b * kv * -(-lk // 128) * (512 if hd > 96 else 256) >= 1 << 32:
        return False
    return (q.dtype == _bf16 and hd % 8 == 0 and 8 <= hd <= MAX_HD and min(b, lq, lk) > 0 and max(lq, lk) <= 1 << 30
            and b * heads * -(-lq // 32) < 1 << 24 and b * kv * -(-lk // 32) < 1 << 24
            and _here(q) and _here(k) and _here(v))


# --------------------------- packed sequences -------------------------------

MOST_SEQUENCES = (1 << 24) - 1


def _bounds(starts, rows):
    """The running maximum of the starts, each within the rows."""
    return starts.to(torch.int64).clamp(0, rows).cummax(0).values


def packed_positions(starts, rows):
    """The position of each of `rows` rows in its sequence (int64; 0 for rows of none), for Rotary.
    starts (n + 1,): as packed_attention takes them."""
    if not isinstance(starts, _Tensor):
        raise TypeError("packed_positions: starts is a tensor")
    if starts.dim() != 1 or starts.shape[0] < 2 or starts.dtype not in (torch.int32, torch.int64):
        raise ValueError("packed_positions: starts (n + 1,), n >= 1, of int32 or int64")
    rows = rows if isinstance(rows, torch.SymInt) else index(rows)  # (a traced size stays one)
    if rows < 0:
        raise ValueError("packed_positions: rows >= 0")
    e, i = _bounds(starts, rows), torch.arange(rows, device=starts.device)
    s = torch.searchsorted(e, i, right=True)
    return torch.where((s > 0) & (s < len(e)), i - e[(s - 1).clamp(min=0)], 0)


def _packed_torch(q, k, v, starts, window, sinks, scale):
    """The attention as torch expressions, in fp32 (fp64 for fp64)."""
    rows, heads, kv = q.shape[0], q.shape[1], k.shape[1]
    wide = torch.float64 if q.dtype == torch.float64 else torch.float32
    e, i = _bounds(starts, rows), torch.arange(rows, device=q.device)
    s = torch.searchsorted(e, i, right=True)  # 0, or n + 1: no sequence
    p, j = i.unsqueeze(1), i
    seen = (s.unsqueeze(1) == s) & ((s > 0) & (s < len(e))).unsqueeze(1) & (j <= p)
    if window is not None:
        seen = seen & ((p - j < window) | (packed_positions(starts, rows) < sinks))
    with _as_typed(q):
        qw, kw, vw = (t.to(wide).transpose(0, 1).unsqueeze(0) for t in (q, k, v))
        if kv != heads:
            kw, vw = (t.repeat_interleave(heads // kv, 1) for t in (kw, vw))
        if rows == 0:
            return torch.matmul(torch.matmul(qw, kw.transpose(2, 3)), vw).squeeze(0).transpose(0, 1).to(q.dtype)
        return _attend(qw, kw, vw, seen.view(1, 1, rows, rows), scale).squeeze(0).transpose(0, 1).to(q.dtype)


def _packed_tensor(t):
    """A bf16 (rows, heads, hd) tensor as the kernels take it, and its strides: (0, head, row)."""
    rows, heads, hd = t.shape
    x, y, z = t.stride()
    x, y = x if rows > 1 else 0, y if heads > 1 else 0
    if z != 1 or (t.data_ptr() | 2 * (x | y)) % 16 != 0 or rows > 1 and not hd <= x <= MAX_ROW_STRIDE:
        t = t.contiguous()
        t = t if t.data_ptr() % 16 == 0 else t.clone()
        x, y = heads * hd if rows > 1 else 0, hd if heads > 1 else 0
    return t, (0, y, x)


def _packed_fields(q, k, v, o, stats, window, sinks, scale):
    """q, k, v, o: (tensor, strides); a padded batch of one sequence, but for the table of the rows."""
    rows, heads, hd = q[0].shape
    kv, lse = k[0].shape[1], stats.data_ptr()
    stat = rows * heads
    return (q[0].data_ptr(), k[0].data_ptr(), v[0].data_ptr(), o[0].data_ptr(), lse,
            lse + -(-stat // 4) * 16 if stats.numel() > stat else 0, 0, *q[1], *k[1], *v[1], *o[1], 1, heads, kv, rows, rows, hd,
            NO_WINDOW if window is None else min(window, NO_WINDOW), min(sinks, NO_WINDOW), scale, 0, 0, 0, 0)


OWN_SEQUENCES, OWN_GRID = 61, 512


def _packed_items(n, rows):
    """At most so many tiles of 128 rows: each sequence, and what lies before and behind them, begins its own."""
    return rows // 128 + min(n + 2, rows)


def _packed_table_words(n, rows):
    return 4 + 2 * (-(-(n + 3) // 4) * 4) + 4 * _packed_items(n, rows)


def packed_wants_table(n, rows, heads):
    """A forward alone of few sequences, whose workgroups all run at once, in whatever order, finds their
    rows without the table's launch: 14.9 us for 19.1 for six prompts in 181 rows, 8 heads of 64."""
    return n > OWN_SEQUENCES or _packed_items(n, rows) * heads > OWN_GRID


def _packed_scratch(block, n):
    fn = _fns.get("packed")
    if fn is None:
        fn = _lib.load().compact_packed_bwd_scratch
        fn.restype, fn.argtypes = _i64, [_block, ctypes.c_int]
        _fns["packed"] = fn
    return fn(block, n)


def _packed_apply(q, k, v, starts, window, sinks, scale, tracked=False):
    """q, k, v: as _packed_tensor gives them; (o, the statistics that a backward wants, the table of the rows)"""
    rows, heads, hd = q[0].shape
    device, n = q[0].device, starts.shape[0] - 1
    o = torch.empty(rows, heads, hd, dtype=_bf16, device=device)
    stats = torch.empty(_stats_count((1, heads, rows, hd), tracked), dtype=torch.float32, device=device)
    table, at = None, 0
    if tracked or packed_wants_table(n, rows, heads):
        table = torch.empty(_packed_table_words(n, rows), dtype=torch.int32, device=device)
        at = table.data_ptr()
    ops._call("compact_packed_fwd", _attn_pack(*_packed_fields(q, k, v, (o, (0, hd, heads * hd)), stats, window, sinks, scale)),
              starts.data_ptr(), starts.dtype == torch.int64, starts.stride(0), n, at, _stream(stats))
    return o, stats, table


class _PackedFn(torch.autograd.Function):
    """Keeps q, k, v, o, one fp32 number a row and a byte an element beside o, and the table that the
    forward made of the starts."""

    @staticmethod
    def forward(ctx, q, k, v, strides, starts, window, sinks, scale):
        o, stats, table = _packed_apply(*zip((q, k, v), strides), starts, window, sinks, scale, tracked=True)
        ctx.rule = window, sinks, scale
        ctx.shapes = q.shape, k.shape, starts.shape[0] - 1
        ctx.save_for_backward(q, k, v, o, stats, table)
        return o

    @staticmethod
    def backward(ctx, do):
        q, k, v, o, stats, table = ctx.saved_tensors
        window, sinks, scale = ctx.rule
        shape, kv_shape, n = ctx.shapes
        rows, heads, hd = shape
        none = (None,) * 5
        words = _packed_table_words(n, rows)
        if (torch.is_grad_enabled() or not _eager() or not _here(do)
                or not ops._companion(stats, torch.float32, _stats_count((1, heads, rows, hd), True))
                or not ops._companion(table, torch.int32, words)
                or not all(t.dtype is _bf16 and t.shape == s and _here(t)
                           for t, s in ((q, shape), (k, kv_shape), (v, kv_shape), (o, shape)))):
            recorded = torch.is_grad_enabled()
            starts = table.reshape(-1)[5:6 + n].to(q.device)
            with torch.enable_grad():
                # (aliases: of v = f(k), k's own gradient must not hold what reaches k through v)
                leaves = [x.view_as(x) if recorded and x.requires_grad else x.detach().requires_grad_(True) for x in (q, k, v)]
                y = _packed_torch(*leaves, starts, window, sinks, scale)
                return (*torch.autograd.grad(y, leaves, do, create_graph=recorded), *none)
        do = _packed_tensor(do if do.dtype is _bf16 else do.to(_bf16))
        fields = _packed_fields(_packed_tensor(q), _packed_tensor(k), _packed_tensor(v), _packed_tensor(o), stats, window, sinks, scale)
        device, stat = q.device, rows * heads
        dq = torch.empty(shape, dtype=_bf16, device=device)
        dk = dv = None
        outs, kv, floats = (0, 0), kv_shape[1], 0
        if ctx.needs_input_grad[1] or ctx.needs_input_grad[2]:
            dk, dv = torch.empty(kv_shape, dtype=_bf16, device=device), torch.empty(kv_shape, dtype=_bf16, device=device)
            outs = dk.data_ptr(), dv.data_ptr()
            floats = _packed_scratch(_attn_pack(*fields), n)
        scratch = torch.empty(-(-stat // 4) * 4 + floats, dtype=torch.float32, device=device)  # D, and sums in parts
        delta = scratch.data_ptr()
        ops._call("compact_packed_bwd",
                  _attn_grad_pack(*fields, do[0].data_ptr(), dq.data_ptr(), *outs, delta, *do[1], 0, hd, heads * hd,
                                  *(0, hd, kv * hd) * 2, delta + -(-stat // 4) * 16 if floats > 0 else 0, 0, 0, 0, 0, 0, n),
                  n, table.data_ptr(), _stream(q))
        return dq, dk, dv, *none


def packed_attention(q, k, v, starts, window=None, sinks=0, scale=None):
    """softmax(scale q k^T) v inside each of n sequences that lie end to end: q (rows, heads, hd), k
    and v (rows, kv, hd), heads a multiple of kv (query head h reads head h kv // heads).

    starts (n + 1,), integers on the device, ascending: sequence s holds the rows starts[s] ..
    starts[s + 1] - 1 (none where they are equal).  Row p of a sequence sees its key j when
    j <= p and (p - j < window or j < sinks); window None: every j <= p.  Rows of no sequence,
    before the first or behind the last, give zeros and pass no gradient.  (A start below an
    earlier one, or past the rows, is taken as that one, or as the last row's end.)
    scale: 1 / sqrt(hd) if None.

    The kernels take bf16 with heads of up to 128 elements, a multiple of 8; what a row does not
    see has no part in it, whatever it holds, and a row whose scores are all -inf gives NaN, as in
    window_attention.  (P is one bf16 factor, and dS is one, not two, where both the mean sequence and
    window + sinks are over 512: results are up to 1.2 times, gradients 1.4 times as far from the exact ones
    as their rounding.  The mean decides for short sequences beside long ones, too.)  In the torch expressions an
    infinite or NaN key or value that some rows see makes the others NaN too, those of other sequences among
    them, and the scores of every head are rows x rows numbers, whatever the sequences' lengths.
    packed_positions(starts, rows) gives Rotary its positions."""
    if not (isinstance(q, _Tensor) and isinstance(k, _Tensor) and isinstance(v, _Tensor) and isinstance(starts, _Tensor)):
        raise TypeError("packed_attention: q, k, v and starts are tensors")
    if q.dim() != 3 or k.dim() != 3 or v.dim() != 3 or q.shape[2] == 0:
        raise ValueError("packed_attention: q (rows, heads, hd), k and v (rows, kv, hd), hd >= 1")
    if k.shape != v.shape or q.shape[0] != k.shape[0] or q.shape[2] != k.shape[2]:
        raise ValueError(f"packed_attention: q {tuple(q.shape)}, k {tuple(k.shape)}, v {tuple(v.shape)}")
    if k.shape[1] == 0 or q.shape[1] % k.shape[1] != 0:
        raise ValueError(f"packed_attention: {q.shape[1]} query heads over {k.shape[1]} of k and v")
    if not q.is_floating_point() or q.dtype != k.dtype or q.dtype != v.dtype or not q.device == k.device == v.device:
        raise TypeError("packed_attention: q, k and v of one floating type on one device")
    if starts.dim() != 1 or starts.shape[0] < 2 or starts.device != q.device or starts.dtype not in (torch.int32, torch.int64):
        raise ValueError("packed_attention: starts (n + 1,), n >= 1, of int32 or int64 on q's device")
    window, sinks = None if window is None else index(window), index(sinks)
    if window is not None and window < 1 or sinks < 0:
        raise ValueError("packed_attention: window >= 1 (or None) and sinks >= 0")
    scale = q.shape[2] ** -0.5 if scale is None else float(scale)
    if not (scale > 0 and math.isfinite(scale)):
        raise ValueError("packed_attention: scale > 0")
    tracked = torch.is_grad_enabled() and (q.requires_grad or k.requires_grad or v.requires_grad)
    if _eager() and LEAST_FACTOR < scale < MOST_FACTOR and _packed_usable(q, k, v, starts, tracked):
        if window is not None and window + sinks >= q.shape[0]:
            window, sinks = None, 0  # every earlier key is one or the other
        q, k, v = _packed_tensor(q), _packed_tensor(k), _packed_tensor(v)
        if tracked:
            return _PackedFn.apply(q[0], k[0], v[0], (q[1], k[1], v[1]), starts, window, sinks, scale)
        return _packed_apply(q, k, v, starts, window, sinks, scale)[0]
    return _packed_torch(q, k, v, starts, window, sinks, scale)


def _packed_usable(q, k, v, starts, tracked):
    rows, heads, hd = q.shape
    kv, n = k.shape[1], starts.shape[0] - 1
    items = _packed_items(n, rows)
    # a launch has under 2^32 threads: dk and dv take a workgroup for each item, up to two for its sinks, and up to
    # 2^20 more in parts
    if tracked and (3 * items * kv + (1 << 20) + 1024) * (512 if hd > 96 else 256) >= 1 << 32:
        return False
    return (q.dtype == _bf16 and hd % 8 == 0 and 8 <= hd <= MAX_HD and 0 < rows <= 1 << 30 and n <= MOST_SEQUENCES and heads > 0
            and items * heads < 1 << 24 and heads * -(-rows // 32) < 1 << 24 and _here(q) and _here(k) and _here(v) and _here(starts))


# ----------------------------- distillation ---------------------------------

MAX_TOP = 1024


def _distill_torch(logits, top_logits, top_ids, targets, temperature, weight):
    """The loss as torch expressions, in fp32 (fp64 for fp64)."""
    rows, V = logits.shape
    T, w = temperature, weight
    wide = torch.float64 if logits.dtype == torch.float64 else torch.float32
    counts = targets != ops.IGNORE if targets is not None else torch.ones(rows, dtype=torch.bool, device=logits.device)
    # (a row that does not count has no part, whatever it holds)
    x = torch.where(counts.unsqueeze(-1), logits.to(wide), 0.0)
    there = (top_ids >= 0) & (top_ids < V)
    ids = torch.where(there, top_ids, 0).to(torch.int64)
    bad = (top_ids >= V).any(-1)
    t = torch.where(top_ids >= 0, top_logits.to(wide) / T, -math.inf)
    top = t.amax(-1, keepdim=True)
    e = torch.exp(t - torch.where(top == -math.inf, 0.0, top))
    s = e.sum(-1, keepdim=True)
    p = e / torch.where(s == 0, 1.0, s)
    logq = torch.log_softmax(x / T, -1).gather(1, ids)
    part = (p != 0) & there
    terms = torch.where(part, p, 1.0) * (torch.log(torch.where(part, p, 1.0)) - torch.where(part, logq, 0.0))
    loss = w * T * T * torch.where(part, terms, 0.0).sum(-1)
    if targets is not None and w != 1.0:
        out = counts & ((targets < 0) | (targets >= V))
        bad = bad | out
        hard = torch.log_softmax(x, -1).gather(1, torch.where(counts & ~out, targets, 0).unsqueeze(-1)).squeeze(-1)
        loss = loss - (1 - w) * hard
    loss = loss * torch.where(bad, math.nan, 1.0)
    return (torch.where(counts, loss, 0.0).sum() / counts.sum()).to(torch.float64 if wide == torch.float64 else torch.float32)


def _distill_call(logits, top, ids, targets, scratch, temperature, weight, loss=None, dx=None, dloss=None, unless_one=False):
    """`scratch`: the call's own, or an earlier call's on the same tensors, whose reading of the
    teacher it holds."""
    rows, V = logits.shape
    K = top.shape[1]
    ready = scratch is not None
    if not ready:  # per row K + 1 pairs and a pair, and the loss; the count
        scratch = torch.empty(rows * (2 * K + 5) + 1, dtype=torch.float32, device=logits.device)
    entries = scratch.data_ptr()
    stats = entries + 8 * rows * (K + 1)
    at = lambda x: 0 if x is None else x.data_ptr()
    ops._call("compact_distill",
              _distill_pack(logits.data_ptr(), top.data_ptr(), ids.data_ptr(), at(targets), stats + 12 * rows,
                            0 if loss is None else stats + 8 * rows, at(loss), at(dx), at(dloss), entries, stats, rows, V,
                            top.stride(0), ids.stride(0), ops.IGNORE, K, logits.dtype == torch.float32,
                            top.dtype == torch.float32, ids.dtype == torch.int32, unless_one, ready, temperature, weight),
              _stream(logits))
    return scratch


class _DistillFn(torch.autograd.Function):
    """The loss, and with it the gradient for dloss = 1, while a row is in registers: the
    backward finds dloss to be 1 on the GPU and leaves it, or forms it again.  (The gradient is
    held beside the logits till then, not as a saved tensor: what the backward returns must not
    be shared.)  A backward that is captured without its forward, or the other way round, forms its own."""

    @staticmethod
    def forward(ctx, logits, top, ids, targets, temperature, weight):
        loss = torch.empty((), dtype=torch.float32, device=logits.device)
        ctx.dx = torch.empty_like(logits)
        ctx.scratch = _distill_call(logits, top, ids, targets, None, temperature, weight, loss=loss, dx=ctx.dx)
        ctx.capture = ops._capture(_stream(logits))
        ctx.rule = temperature, weight
        ctx.size = logits.dtype, logits.shape, top.shape
        ctx.save_for_backward(logits, top, ids, targets)
        return loss

    @staticmethod
    def backward(ctx, dloss):
        logits, top, ids, targets = ctx.saved_tensors
        rule = ctx.rule
        # (the gradient's buffer and the scratch are of the forward's types and sizes)
        if (torch.is_grad_enabled() or not _eager() or not _plain(dloss) or not _distill_usable(logits, top, ids, targets)
                or (logits.dtype, logits.shape, top.shape) != ctx.size
                or targets is not None and (targets.dtype is not torch.int64 or targets.shape != logits.shape[:1])):
            targets = targets if targets is None else targets.to(torch.int64)
            return (ops._torch_grad(lambda t: _distill_torch(t, top, ids, targets, *rule), logits, dloss),
                    None, None, None, None, None)
        dx, ctx.dx = ctx.dx, None
        # (a second backward over a retained graph forms its own, too)
        first = dx is not None and ctx.capture == ops._capture(_stream(logits))
        dx = dx if first else torch.empty_like(logits)
        _distill_call(logits, top, ids, targets, ctx.scratch, *rule, dx=dx, dloss=dloss.float(), unless_one=first)
        return dx, None, None, None, None, None


def _distill_usable(logits, top, ids, targets):
    return (logits.dtype in (_bf16, torch.float32) and top.dtype in (_bf16, torch.float32)
            and all(_here(t) for t in (logits, top, ids)) and logits.is_contiguous() and logits.data_ptr() % 16 == 0
            and 0 < logits.shape[0] < ops.MAX_ROWS and 0 < logits.shape[1] <= 1 << 28 and 1 <= top.shape[1] <= MAX_TOP
            and top.stride(1) == 1 and ids.stride(1) == 1 and (targets is None or _here(targets) and targets.is_contiguous()))


def _distill_taken(temperature):
    return LEAST_FACTOR < temperature < MOST_FACTOR


def distill_loss(logits, top_logits, top_ids, targets=None, temperature=1.0, weight=1.0):
    """The mean over the rows of

        weight T^2 sum_k p_k (log p_k - log q_id_k) + (1 - weight) (-log softmax(logits)_target)

    for logits (rows, V), a teacher's K top logits of each row and their ids (rows, K), in any
    order: p = softmax(top_logits / T) over a row's entries, q = softmax(logits / T) over all V.
    An entry with a negative id, or a logit of -inf, is none; a row without entries has no first
    part.  With targets (rows,) rows whose target is -100 do not count, and they are needed where
    weight < 1.  An id or a target past V makes the loss, and its row's gradient, NaN.

    fp32 scalar.  The kernels take dense bf16 or fp32 logits and K up to 1024; they form the
    gradient with the loss and hold it for the backward, as many bytes as the logits.  Of a loss
    that is multiplied before its backward, or whose forward and backward are not captured into one
    graph but into two, or one of them alone, it is formed a second time there."""
    if not (isinstance(logits, _Tensor) and isinstance(top_logits, _Tensor) and isinstance(top_ids, _Tensor)
            and (targets is None or isinstance(targets, _Tensor))):
        raise TypeError("distill_loss: logits, top_logits, top_ids and targets are tensors")
    if logits.dim() != 2 or top_logits.dim() != 2 or top_logits.shape != top_ids.shape or top_logits.shape[0] != logits.shape[0]:
        raise ValueError("distill_loss: logits (rows, V), top_logits and top_ids (rows, K)")
    if top_logits.shape[1] < 1 or logits.shape[1] < 1:
        raise ValueError("distill_loss: at least one logit and one entry a row")
    if not logits.is_floating_point() or not top_logits.is_floating_point() or top_ids.dtype not in (torch.int64, torch.int32):
        raise TypeError("distill_loss: floating logits, int64 or int32 ids")
    if targets is not None and (targets.shape != logits.shape[:1] or targets.dtype != torch.int64):
        raise ValueError("distill_loss: targets (rows,) of int64")
    if any(t is not None and t.device != logits.device for t in (top_logits, top_ids, targets)):
        raise ValueError("distill_loss: tensors of one device")
    temperature, weight = float(temperature), float(weight)
    if not (temperature > 0 and math.isfinite(temperature)) or not 0 <= weight <= 1:
        raise ValueError("distill_loss: temperature > 0 and weight in [0, 1]")
    if targets is None and weight != 1:
        raise ValueError("distill_loss: a weight below 1 needs targets")
    if _eager() and logits.is_cuda and _distill_taken(temperature):
        dense = logits if logits.is_contiguous() else logits.contiguous()
        dense = dense if dense.data_ptr() % 16 == 0 else dense.clone()
        top, ids = (t.detach() if t.stride(1) == 1 else t.detach().contiguous() for t in (top_logits, top_ids))
        targets = targets if targets is None else targets.contiguous()
        if not (top_logits.requires_grad and torch.is_grad_enabled()) and _distill_usable(dense, top, ids, targets):
            if _tracked(dense):
                return _DistillFn.apply(dense, top, ids, targets, temperature, weight)
            loss = torch.empty((), dtype=torch.float32, device=dense.device)
            _distill_call(dense, top, ids, targets, None, temperature, weight, loss=loss)
            return loss
    return _distill_torch(logits, top_logits, top_ids, targets, temperature, weight)
