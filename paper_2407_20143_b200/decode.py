"""Decoding operators on torch tensors: rotary positions, the paged key-value cache and the attention of
one new token over it.  The C calls and their formulas are in include/bcp.h; this module has the handles and
defaults, csrc/binding.cpp checks the tensors and turns them into the calls' descriptors.

    table = RopeTable.build(rope_frequencies(128, base=500000.0), n_positions=8192)
    cache = KvCache.empty(n_pages=1024, n_heads=8, page_size=16, head_dim=128, dtype=torch.float8_e4m3fn)
    work = KvWorkspace(cache, n_q_heads=32, max_seqs=64)
    slots = cache.slots(block_table, sequences, positions)     # where each new token goes
    q = bcp_rope(q, table, positions)
    bcp_kv_write(cache, k, v, slots, rope=table, positions=positions)
    out, lse = bcp_kv_attend(cache, q, block_table, lengths, workspace=work)
    cache.check()                                               # raises if an index was out of range

rope() is differentiable; the bcp_ calls record no gradients and refuse tensors that require one (outside torch.no_grad()).
Head vectors are tensors [tokens, heads, head_dim] with any strides over tokens and heads.  `stream` is a torch
stream, a raw handle, or None for the current stream of the tensors' device; that device must be current.
Handles keep the tensors they were made from alive, and a call with a `stream` records its tensors on it, so that torch's
allocator does not hand out their memory before the work is done.  The order of work on different streams is the caller's:
what another stream writes (a new handle's status word is zeroed on the stream that is current then) must be done before `stream`
reads it.  Nothing here synchronises except check().
"""
from __future__ import annotations

import ctypes as C
import importlib.machinery
import importlib.util
import math
from typing import Optional, Sequence

import torch

from . import _lib as L
from . import build as _build
from .api import ERR_INVALID, BcpError, _check

F32, BF16, F16, E4M3, I8 = 1, 2, 3, 4, 5
ROPE_HALF, ROPE_PAIRS = 0, 1
BAD_POSITION, BAD_SLOT, BAD_PAGE, BAD_LENGTH = 1, 2, 4, 8
MAX_HEAD_DIM = 256
_LAYOUTS = {"half": ROPE_HALF, "pairs": ROPE_PAIRS}

_FORMATS = {torch.bfloat16: BF16, torch.float16: F16, torch.float8_e4m3fn: E4M3, torch.int8: I8}


def _load_binding():
    """The module built from csrc/binding.cpp (built now if it is missing or older than its source)."""
    path = _build.build_binding()
    loader = importlib.machinery.ExtensionFileLoader(__package__ + "._binding", path)
    module = importlib.util.module_from_spec(importlib.util.spec_from_file_location(loader.name, path, loader=loader))
    loader.exec_module(module)
    calls = ("bcp_rope", "bcp_kv_write", "bcp_kv_read", "bcp_kv_attend", "bcp_last_error")
    module.bind(BcpError, *(C.cast(getattr(L.lib(), name), C.c_void_p).value for name in calls))
    return module


_b = _load_binding()


def _invalid(message: str, code: int = ERR_INVALID) -> BcpError:
    return BcpError(code, message)


def _raw(stream):
    """What the binding takes: None (the current stream of the tensors' device) or a raw handle."""
    return stream if stream is None or isinstance(stream, int) else stream.cuda_stream


def _torch_stream(stream, device):
    return torch.cuda.ExternalStream(stream, device=device) if isinstance(stream, int) else stream


def _empty(like, shape, dtype, stream):
    """Memory for an output that work on `stream` fills: taken from that stream's pool, so that it is not reused too early."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=like.device)
    with torch.cuda.stream(_torch_stream(stream, like.device)):
        return torch.empty(shape, dtype=dtype, device=like.device)


def _record(stream, *tensors) -> None:
    """Memory of `tensors`, which may belong to other streams, is not reused before the work now on `stream` is done."""
    s = _torch_stream(stream, tensors[0].device)
    for t in tensors:
        if t is not None:
            t.record_stream(s)


def _check_status(status, stream) -> None:
    handle = _raw(torch.cuda.current_stream(status.device) if stream is None else stream)
    _check(L.lib().bcp_decode_status(status.data_ptr(), handle))


# ------------------------------------------------------------------ rotary positions
def rope_frequencies(rot_dim: int, base: float = 10000.0, *, scaling: Optional[str] = None, factor: float = 1.0,
                     trained: Optional[int] = None, low: float = 1.0, high: float = 4.0) -> Sequence[float]:
    """Angles per position of the rot_dim / 2 pairs: base^(-2i / rot_dim), scaled for contexts longer than `trained`:

    "linear"  every frequency divided by `factor` (positions are squeezed into the trained range)
    "base"    the base grows to base * factor^(rot_dim / (rot_dim - 2)): the slowest pair is divided by `factor`,
              the fastest is kept
    "bands"   a pair that turns at least `high` times over the trained length is kept, one that turns at most `low`
              times is divided by `factor`, those between are mixed in proportion to their turns
    """
    if rot_dim < 2 or rot_dim % 2 or rot_dim > MAX_HEAD_DIM:
        raise _invalid(f"rot_dim {rot_dim} is not an even number from 2 to {MAX_HEAD_DIM}")
    if not factor >= 1.0 or not base > 0.0:
        raise _invalid(f"factor {factor} and base {base}: at least 1 and above 0 expected")
    if scaling == "base" and rot_dim > 2:
        base = base * factor ** (rot_dim / (rot_dim - 2))
    f = [base ** (-2.0 * i / rot_dim) for i in range(rot_dim // 2)]
    if scaling in (None, "base"):
        return f
    if scaling == "linear":
        return [x / factor for x in f]
    if scaling == "bands":
        if not trained or not high > low > 0:
            raise _invalid("scaling 'bands' needs the trained length and 0 < low < high")
        keep = [min(1.0, max(0.0, (trained * x / (2 * math.pi) - low) / (high - low))) for x in f]
        return [x * k + x / factor * (1.0 - k) for x, k in zip(f, keep)]
    raise _invalid(f"scaling {scaling!r}: None, 'linear', 'base' or 'bands' expected")


class RopeTable:
    """Cosines and sines for bcp_rope and bcp_kv_write, over a float32 tensor [positions, 2, rot_dim / 2]."""

    def __init__(self, table, layout: str = "half"):
        if layout not in _LAYOUTS:
            raise _invalid(f"layout {layout!r}: 'half' or 'pairs' expected")
        if table.dtype != torch.float32 or table.dim() != 3 or table.shape[1] != 2 or not table.is_contiguous() or not table.is_cuda:
            raise _invalid("a rotation table is a contiguous float32 CUDA tensor [positions, 2, rot_dim / 2]")
        self.table, self.layout, self.device = table, layout, table.get_device()
        self.status = torch.zeros(1, dtype=torch.int32, device=table.device)
        self.tensors = (table, self.status)
        self.c = L.RopeTableC(table.data_ptr(), table.shape[0], 2 * table.shape[2], _LAYOUTS[layout], self.status.data_ptr())
        self.address = C.addressof(self.c)

    @classmethod
    def build(cls, frequencies: Sequence[float], n_positions: int, *, layout: str = "half", attention_factor: float = 1.0,
              device="cuda") -> "RopeTable":
        """Table of attention_factor * cos / sin of position * frequency, computed in 64 bits, rounded once."""
        f = torch.tensor(list(frequencies), dtype=torch.float64, device=device)
        angle = torch.arange(n_positions, dtype=torch.float64, device=device)[:, None] * f
        return cls((torch.stack([angle.cos(), angle.sin()], 1) * attention_factor).float(), layout)

    def check(self, stream=None) -> None:
        """Waits for `stream`; raises BcpError (ERR_BOUNDS) if a call met a position outside the table."""
        _check_status(self.status, stream)


def _rope(x, table: RopeTable, positions, out, transpose: bool, stream):
    if isinstance(x, torch.Tensor):
        if out is None:
            out = _empty(x, x.shape, x.dtype, stream)
        elif not isinstance(out, torch.Tensor):
            out, = out
        _b.rope(table.address, table.device, x, None, out, None, positions, transpose, _raw(stream))
        if stream is not None:
            _record(stream, x, out, positions, *table.tensors)
        return out
    if len(x) == 1:
        return (_rope(x[0], table, positions, out if out is None else out[0], transpose, stream),)
    q, k = x
    if out is None:
        out = (_empty(q, q.shape, q.dtype, stream), _empty(k, k.shape, k.dtype, stream))
    _b.rope(table.address, table.device, q, k, out[0], out[1], positions, transpose, _raw(stream))
    if stream is not None:
        _record(stream, q, k, *out, positions, *table.tensors)
    return out


def bcp_rope(x, table: RopeTable, positions, out=None, stream=None):
    """x [tokens, heads, head_dim], or a pair (queries, keys), rotated by the tokens' positions (int64 [tokens]; negative:
    zeros).  `out` may be x itself.  Returns the output, or the pair of them."""
    return _rope(x, table, positions, out, False, stream)


def bcp_rope_backward(grad, table: RopeTable, positions, out=None, stream=None):
    """The gradient of bcp_rope: the transposed rotation of the outputs' gradient."""
    return _rope(grad, table, positions, out, True, stream)


class _Rope(torch.autograd.Function):
    @staticmethod
    def forward(ctx, table, positions, transpose, *xs):
        ctx.table, ctx.transpose = table, transpose
        ctx.save_for_backward(positions)
        ctx.set_materialize_grads(False)
        return _rope(xs, table, positions, None, transpose, None)

    @staticmethod
    def backward(ctx, *grads):
        positions, = ctx.saved_tensors
        wanted = [i for i, g in enumerate(grads) if g is not None and ctx.needs_input_grad[3 + i]]
        out = [None] * len(grads)
        if wanted:
            # an expanded gradient (of a sum, say) has no contiguous vectors
            given = [g if g.stride(-1) == 1 else g.contiguous() for g in (grads[i] for i in wanted)]
            # the gradient of a linear map is its transpose: through this function again, so that it has gradients itself
            for i, g in zip(wanted, _Rope.apply(ctx.table, positions, not ctx.transpose, *given)):
                out[i] = g
        return (None, None, None, *out)


def rope(x, table: RopeTable, positions):
    """bcp_rope as a differentiable function of x (a tensor, or a pair) on the current stream; its gradients are differentiable
    too."""
    if isinstance(x, torch.Tensor):
        return _Rope.apply(table, positions, False, x)[0]
    return _Rope.apply(table, positions, False, *x)


# ------------------------------------------------------------------ cache
class KvCache:
    """A paged cache over tensors k, v [pages, heads, page_size, head_dim] (bfloat16, float16, float8_e4m3fn or int8; any
    strides over the first three dimensions, the same for both) and, for the 8-bit types, contiguous float32 scales
    [pages, heads, page_size]."""

    def __init__(self, k, v, k_scale=None, v_scale=None):
        fmt = _FORMATS.get(k.dtype)
        if fmt is None or v.dtype != k.dtype:
            raise _invalid(f"a cache of {k.dtype} and {v.dtype}; bfloat16, float16, float8_e4m3fn or int8 expected, the same for both")
        if k.dim() != 4 or v.shape != k.shape or v.stride() != k.stride() or (k.stride(3) != 1 and k.shape[3] > 1):
            raise _invalid("k and v must be [pages, heads, page_size, head_dim] with the same strides and contiguous vectors")
        if not k.is_cuda or v.get_device() != k.get_device():
            raise _invalid("k and v must be on one CUDA device")
        device = k.get_device()
        if (fmt in (E4M3, I8)) != (k_scale is not None) or (k_scale is None) != (v_scale is None):
            raise _invalid("8-bit caches have k_scale and v_scale, the others have none")
        for s, name in ((k_scale, "k_scale"), (v_scale, "v_scale")):
            if s is not None and (s.dtype != torch.float32 or s.shape != k.shape[:3] or not s.is_contiguous() or s.get_device() != device):
                raise _invalid(f"{name} must be a contiguous float32 tensor {tuple(k.shape[:3])} beside the cache")
        self.k, self.v, self.k_scale, self.v_scale, self.device = k, v, k_scale, v_scale, device
        self.n_pages, self.n_heads, self.page_size, self.head_dim = k.shape
        self.status = torch.zeros(1, dtype=torch.int32, device=k.device)
        self.tensors = (k, v, k_scale, v_scale, self.status)
        # a dimension of one element may carry any stride: what the kernels get is that of a dense tensor
        strides, dense = [], self.head_dim
        for i in (2, 1, 0):
            strides.insert(0, k.stride(i) if k.shape[i] > 1 else dense)
            dense = max(dense, strides[0] * k.shape[i])
        self.c = L.KvCacheC(k.data_ptr(), v.data_ptr(), k_scale.data_ptr() if k_scale is not None else None,
                            v_scale.data_ptr() if v_scale is not None else None, *strides, self.n_pages, self.page_size, self.n_heads,
                            self.head_dim, fmt, 0, self.status.data_ptr())
        self.address = C.addressof(self.c)

    @classmethod
    def empty(cls, n_pages: int, n_heads: int, page_size: int, head_dim: int, dtype=None, device="cuda") -> "KvCache":
        """A cache of zeros."""
        dtype = torch.bfloat16 if dtype is None else dtype
        k, v = (torch.zeros((n_pages, n_heads, page_size, head_dim), dtype=dtype, device=device) for _ in range(2))
        if _FORMATS.get(dtype) in (E4M3, I8):
            return cls(k, v, *(torch.zeros((n_pages, n_heads, page_size), dtype=torch.float32, device=device) for _ in range(2)))
        return cls(k, v)

    def slots(self, block_table, sequences, positions):
        """Slots (int64) of tokens at `positions` of `sequences` (rows of block_table), all on the device.  -1, which the calls
        skip, for a negative position and where the table's page is negative; a slot past the cache, which they skip and
        report, for a position past the table's width or a sequence that is no row of it."""
        rows, width = block_table.shape
        positions = positions.long()
        page = torch.div(positions, self.page_size, rounding_mode="floor")
        # the table as one line: what lies before or behind it, or behind its row, is past the table
        if isinstance(sequences, int):
            place = page + range(rows)[sequences] * width
        else:
            place = torch.add(page, torch.as_tensor(sequences, device=block_table.device), alpha=width)
        slot = torch.remainder(positions, self.page_size)
        if block_table.numel():  # else there is nothing to look up
            there = place.clamp(0, rows * width - 1)
            first = block_table.take(there)
            slot = torch.add(slot, first, alpha=self.page_size).masked_fill_(first < 0, -1)
            past = (page >= width).logical_or(place != there)
        else:
            slot, past = slot + 0 * place, torch.ones_like(place, dtype=torch.bool)
        return slot.masked_fill_(past, self.n_pages * self.page_size).masked_fill_(positions < 0, -1)

    def check(self, stream=None) -> None:
        """Waits for `stream`; raises BcpError (ERR_BOUNDS) if a call met a slot, page, length or position out of range."""
        _check_status(self.status, stream)


def bcp_kv_write(cache: KvCache, k, v, slots, rope: Optional[RopeTable] = None, positions=None, stream=None) -> None:
    """k, v [tokens, heads, head_dim] into their slots (int64 [tokens]; negative: skipped); with `rope`, the keys are rotated
    by positions (int64 [tokens]) on the way."""
    if rope is None:
        _b.kv_write(cache.address, cache.device, k, v, slots, None, cache.device, positions, _raw(stream), cache.k, cache.v)
    else:
        _b.kv_write(cache.address, cache.device, k, v, slots, rope.address, rope.device, positions, _raw(stream), cache.k, cache.v)
    if stream is not None:
        _record(stream, k, v, slots, positions, *cache.tensors, *(() if rope is None else rope.tensors))


def bcp_kv_read(cache: KvCache, slots, out=None, dtype=None, stream=None):
    """Keys and values [tokens, heads, head_dim] at `slots` (int64 [tokens]; negative: zeros), in `dtype` (default bfloat16, or
    the cache's own 16-bit type) or into out = (k, v)."""
    if out is None:
        dtype = dtype or (cache.k.dtype if cache.k_scale is None else torch.bfloat16)
        out = tuple(_empty(slots, (slots.numel(), cache.n_heads, cache.head_dim), dtype, stream) for _ in range(2))
    k, v = out
    _b.kv_read(cache.address, cache.device, slots, k, v, _raw(stream))
    if stream is not None:
        _record(stream, slots, k, v, *cache.tensors)
    return k, v


class KvWorkspace:
    """Scratch memory of bcp_kv_attend for up to max_seqs sequences, zeroed on `stream`: a first use on another stream has to
    be ordered behind that.  It serves one call at a time: calls that may overlap on the GPU (other streams without
    ordering) need a workspace each."""

    def __init__(self, cache: KvCache, n_q_heads: int, max_seqs: int, stream=None):
        n = C.c_uint64()
        _check(L.lib().bcp_kv_attend_workspace(cache.address, n_q_heads, max_seqs, C.byref(n)))
        with torch.cuda.stream(_torch_stream(stream, cache.k.device)):  # None: the current one
            self.memory = torch.zeros(n.value, dtype=torch.uint8, device=cache.k.device)
        self.address, self.bytes, self.device = self.memory.data_ptr(), n.value, cache.device


def bcp_kv_attend(cache: KvCache, q, block_table, lengths, scale: Optional[float] = None, window: int = 0, out=None, lse=None,
                  workspace: Optional[KvWorkspace] = None, stream=None):
    """Attention of q [sequences, query heads, head_dim] over the first lengths[b] (int32) tokens of each sequence, or the last
    `window` of them, whose pages are block_table[b] (int32 [sequences, width]).  scale defaults to head_dim^-0.5.
    Returns (out, lse); lse [sequences, query heads] is the natural logarithm of the sum of exponentials, -inf where a
    sequence has no tokens (its output is zeros)."""
    if out is None:
        out = _empty(q, q.shape, q.dtype, stream)
    if lse is None:
        lse = _empty(q, q.shape[:2], torch.float32, stream)
    if workspace is None:
        workspace = KvWorkspace(cache, q.shape[1], q.shape[0], stream)
    _b.kv_attend(cache.address, cache.device, q, out, lse, block_table, lengths, cache.head_dim ** -0.5 if scale is None else scale, window,
                 workspace.address, workspace.bytes, workspace.device, _raw(stream))
    if stream is not None:
        _record(stream, q, out, lse, block_table, lengths, workspace.memory, *cache.tensors)
    return out, lse

