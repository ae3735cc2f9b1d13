"""Decoding operators on torch tensors: rotary positions, the paged key-value cache and the attention of
one new token over it.  The C calls and their formulas are in include/bcp.h; this module checks and
marshals their arguments.

    table = RopeTable.build(rope_frequencies(128, base=500000.0), n_positions=8192)
    cache = KvCache.empty(n_pages=1024, n_heads=8, page_size=16, head_dim=128, dtype=torch.float8_e4m3fn)
    work = KvWorkspace(cache, n_q_heads=32, max_seqs=64)
    slots = cache.slots(block_table, sequences, positions)     # where each new token goes
    q, = bcp_rope((q,), table, positions)
    bcp_kv_write(cache, k, v, slots, rope=table, positions=positions)
    out, lse = bcp_kv_attend(cache, q, block_table, lengths, workspace=work)
    cache.check()                                               # raises if an index was out of range

Head vectors are tensors [tokens, heads, head_dim] with any strides over tokens and heads.  `stream` is a torch
stream, a raw handle, or None for the current stream of the tensors' device; that device must be current.
Handles keep the tensors they were made from alive.  Nothing here synchronises except check().
"""
from __future__ import annotations

import ctypes as C
import math
from typing import Optional, Sequence, Tuple

import torch

from . import _lib as L
from .api import ERR_INVALID, ERR_MISMATCH, BcpError, _check

F32, BF16, F16, E4M3, I8 = 1, 2, 3, 4, 5
ROPE_HALF, ROPE_PAIRS = 0, 1
BAD_POSITION, BAD_SLOT, BAD_PAGE, BAD_LENGTH = 1, 2, 4, 8
MAX_HEAD_DIM = 256
_LAYOUTS = {"half": ROPE_HALF, "pairs": ROPE_PAIRS}

_TYPES = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}
_FORMATS = {torch.bfloat16: BF16, torch.float16: F16, torch.float8_e4m3fn: E4M3, torch.int8: I8}


def _invalid(message: str, code: int = ERR_INVALID) -> BcpError:
    return BcpError(code, message)


def _raw_stream(stream, device: int) -> int:
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(device)
    return stream if isinstance(stream, int) else stream.cuda_stream


def _empty(like, shape, dtype, stream):
    """Memory for an output that work on `stream` fills: taken from that stream's pool, so that it is not reused too early."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=like.device)
    with torch.cuda.stream(torch.cuda.ExternalStream(stream, device=like.device) if isinstance(stream, int) else stream):
        return torch.empty(shape, dtype=dtype, device=like.device)


def _device(t, name: str) -> int:
    """Index of the tensor's device, which has to be the current one."""
    if not t.is_cuda:
        raise _invalid(f"{name} is not on a CUDA device")
    d = t.get_device()
    if d != torch._C._cuda_getDevice():
        raise _invalid(f"{name} is on cuda:{d}, but cuda:{torch._C._cuda_getDevice()} is the current device")
    return d


def _heads(t, name: str, device: int, tokens: int, dim: int) -> L.HeadsC:
    if t.dim() != 3:
        raise _invalid(f"{name} has {t.dim()} dimensions; [tokens, heads, head_dim] expected")
    n, h, d = t.shape
    ts, hs, es = t.stride()
    typ = _TYPES.get(t.dtype)
    if typ is None:
        raise _invalid(f"{name} is {t.dtype}; float32, bfloat16 or float16 expected")
    if t.get_device() != device:
        raise _invalid(f"{name} is on another device")
    if n != tokens or d != dim:
        raise _invalid(f"{name} has shape {tuple(t.shape)}; {tokens} tokens and vectors of {dim} expected", ERR_MISMATCH)
    if es != 1 and d > 1:
        raise _invalid(f"the elements of {name}'s vectors are not contiguous")
    return L.HeadsC(t.data_ptr(), ts, hs, h, typ)


def _index(t, name: str, device: int, dtype, shape: Tuple[int, ...]) -> int:
    if t.dtype != dtype or t.get_device() != device:
        raise _invalid(f"{name} must be {dtype} on cuda:{device}")
    if t.shape != shape or not t.is_contiguous():
        raise _invalid(f"{name} has shape {tuple(t.shape)}; a contiguous {tuple(shape)} expected", ERR_MISMATCH)
    return t.data_ptr()


def _check_status(status, stream) -> None:
    _check(L.lib().bcp_decode_status(status.data_ptr(), _raw_stream(stream, status.get_device())))


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


def _rope(xs, table: RopeTable, positions, out, transpose: int, stream):
    single = isinstance(xs, torch.Tensor)
    xs = (xs,) if single else tuple(xs)
    if not 1 <= len(xs) <= 2:
        raise _invalid(f"{len(xs)} tensors: one, or queries and keys, expected")
    device = _device(xs[0], "x")
    if table.device != device:
        raise _invalid("the table is on another device")
    if out is None:
        outs = tuple(_empty(x, x.shape, x.dtype, stream) for x in xs)
    else:
        outs = (out,) if isinstance(out, torch.Tensor) else tuple(out)
    if len(outs) != len(xs):
        raise _invalid(f"{len(outs)} outputs for {len(xs)} inputs")
    if xs[0].dim() != 3:
        raise _invalid(f"x has {xs[0].dim()} dimensions; [tokens, heads, head_dim] expected")
    n, _, d = xs[0].shape
    c = [_heads(t, name, device, n, d) for x, o in zip(xs, outs) for t, name in ((x, "x"), (o, "out"))]
    where = [C.addressof(h) for h in c] + [None, None]
    p = _index(positions, "positions", device, torch.int64, (n,))
    _check(L.lib().bcp_rope(where[0], where[1], where[2], where[3], d, n, table.address, p, transpose, _raw_stream(stream, device)))
    return outs[0] if single and isinstance(outs[0], torch.Tensor) else outs


def bcp_rope(x, table: RopeTable, positions, out=None, stream=None):
    """x [tokens, heads, head_dim], or a pair (queries, keys), rotated by the tokens' positions (int64 [tokens]; negative:
    zeros).  `out` may be x itself.  Returns the output, or the tuple of them."""
    return _rope(x, table, positions, out, 0, stream)


def bcp_rope_backward(grad, table: RopeTable, positions, out=None, stream=None):
    """The gradient of bcp_rope: the transposed rotation of the outputs' gradient."""
    return _rope(grad, table, positions, out, 1, stream)


class _Rope(torch.autograd.Function):
    @staticmethod
    def forward(ctx, table, positions, *xs):
        ctx.table = table
        ctx.save_for_backward(positions)
        return _rope(xs, table, positions, None, 0, None)

    @staticmethod
    def backward(ctx, *grads):
        positions, = ctx.saved_tensors
        # an expanded gradient (of a sum, say) has no contiguous vectors
        grads = [g if g.stride(-1) == 1 else g.contiguous() for g in grads]
        return (None, None) + tuple(_rope(grads, ctx.table, positions, None, 1, None))


def rope(x, table: RopeTable, positions):
    """bcp_rope as a differentiable function of x (a tensor, or a pair) on the current stream."""
    if isinstance(x, torch.Tensor):
        return _Rope.apply(table, positions, x)[0]
    return _Rope.apply(table, positions, *x)


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
        device = _device(k, "k")
        if v.get_device() != device:
            raise _invalid("v is on another device")
        if (fmt in (E4M3, I8)) != (k_scale is not None) or (k_scale is None) != (v_scale is None):
            raise _invalid("8-bit caches have k_scale and v_scale, the others have none")
        for s, name in ((k_scale, "k_scale"), (v_scale, "v_scale")):
            if s is not None and (s.dtype != torch.float32 or s.shape != k.shape[:3] or not s.is_contiguous() or s.get_device() != device):
                raise _invalid(f"{name} must be a contiguous float32 tensor {tuple(k.shape[:3])} beside the cache")
        self.k, self.v, self.k_scale, self.v_scale, self.device = k, v, k_scale, v_scale, device
        self.n_pages, self.n_heads, self.page_size, self.head_dim = k.shape
        self.status = torch.zeros(1, dtype=torch.int32, device=k.device)
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
        """Slots (int64) of tokens at `positions` of `sequences` (rows of block_table), all on the device."""
        page = torch.div(positions, self.page_size, rounding_mode="floor")
        return block_table[sequences, page].long() * self.page_size + (positions - page * self.page_size)

    def check(self, stream=None) -> None:
        """Waits for `stream`; raises BcpError (ERR_BOUNDS) if a call met a slot, page, length or position out of range."""
        _check_status(self.status, stream)


def bcp_kv_write(cache: KvCache, k, v, slots, rope: Optional[RopeTable] = None, positions=None, stream=None) -> None:
    """k, v [tokens, heads, head_dim] into their slots (int64 [tokens]; negative: skipped); with `rope`, the keys are rotated
    by positions (int64 [tokens]) on the way."""
    device = _device(k, "k")
    if cache.device != device or (rope is not None and rope.device != device):
        raise _invalid("the cache or the table is on another device")
    n = k.shape[0]
    kc, vc = _heads(k, "k", device, n, cache.head_dim), _heads(v, "v", device, n, cache.head_dim)
    s = _index(slots, "slots", device, torch.int64, (n,))
    if (rope is None) != (positions is None):
        raise _invalid("rope and positions go together")
    p = _index(positions, "positions", device, torch.int64, (n,)) if rope is not None else None
    _check(L.lib().bcp_kv_write(cache.address, C.addressof(kc), C.addressof(vc), s, n, rope.address if rope is not None else None, p,
                                _raw_stream(stream, device)))


def bcp_kv_read(cache: KvCache, slots, out=None, dtype=None, stream=None):
    """Keys and values [tokens, heads, head_dim] at `slots` (int64 [tokens]; negative: zeros), in `dtype` (default bfloat16, or
    the cache's own 16-bit type) or into out = (k, v)."""
    device = _device(slots, "slots")
    if cache.device != device:
        raise _invalid("the cache is on another device")
    if slots.dim() != 1:
        raise _invalid(f"slots has {slots.dim()} dimensions; one expected")
    n = slots.shape[0]
    if out is None:
        dtype = dtype or (cache.k.dtype if cache.k_scale is None else torch.bfloat16)
        out = tuple(_empty(slots, (n, cache.n_heads, cache.head_dim), dtype, stream) for _ in range(2))
    k, v = out
    kc, vc = _heads(k, "k", device, n, cache.head_dim), _heads(v, "v", device, n, cache.head_dim)
    s = _index(slots, "slots", device, torch.int64, (n,))
    _check(L.lib().bcp_kv_read(cache.address, s, n, C.addressof(kc), C.addressof(vc), _raw_stream(stream, device)))
    return k, v


class KvWorkspace:
    """Scratch memory of bcp_kv_attend for up to max_seqs sequences.  It serves one call at a time: calls that may overlap
    on the GPU (other streams without ordering) need a workspace each."""

    def __init__(self, cache: KvCache, n_q_heads: int, max_seqs: int):
        n = C.c_uint64()
        _check(L.lib().bcp_kv_attend_workspace(cache.address, n_q_heads, max_seqs, C.byref(n)))
        self.memory = torch.zeros(n.value, dtype=torch.uint8, device=cache.k.device)
        self.address, self.bytes, self.device = self.memory.data_ptr(), n.value, cache.device


def bcp_kv_attend(cache: KvCache, q, block_table, lengths, scale: Optional[float] = None, window: int = 0, out=None, lse=None,
                  workspace: Optional[KvWorkspace] = None, stream=None):
    """Attention of q [sequences, query heads, head_dim] over the first lengths[b] (int32) tokens of each sequence, or the last
    `window` of them, whose pages are block_table[b] (int32 [sequences, width]).  scale defaults to head_dim^-0.5.
    Returns (out, lse); lse [sequences, query heads] is the natural logarithm of the sum of exponentials, -inf where a
    sequence has no tokens (its output is zeros)."""
    device = _device(q, "q")
    if cache.device != device:
        raise _invalid("the cache is on another device")
    if q.dim() != 3:
        raise _invalid(f"q has {q.dim()} dimensions; [sequences, heads, head_dim] expected")
    n, h, _ = q.shape
    if out is None:
        out = _empty(q, q.shape, q.dtype, stream)
    if lse is None:
        lse = _empty(q, (n, h), torch.float32, stream)
    if workspace is None:
        workspace = _new_workspace(cache, h, n, stream)
    elif workspace.device != device:
        raise _invalid("the workspace is on another device")
    qc, oc = _heads(q, "q", device, n, cache.head_dim), _heads(out, "out", device, n, cache.head_dim)
    if block_table.dim() != 2 or block_table.shape[0] != n or block_table.dtype != torch.int32 or block_table.get_device() != device or (
            block_table.shape[1] > 1 and block_table.stride(1) != 1):
        raise _invalid(f"block_table must be an int32 tensor [{n}, width] on cuda:{device} with contiguous rows")
    if window < 0:
        raise _invalid(f"window {window} is negative")
    lens = _index(lengths, "lengths", device, torch.int32, (n,))
    sums = _index(lse, "lse", device, torch.float32, (n, h))
    width = block_table.shape[1]
    _check(L.lib().bcp_kv_attend(cache.address, C.addressof(qc), C.addressof(oc), sums, n, block_table.data_ptr(),
                                 block_table.stride(0) if n > 1 else width, width, lens, cache.head_dim ** -0.5 if scale is None else scale,
                                 min(window, 0x7fffffff), workspace.address, workspace.bytes, _raw_stream(stream, device)))
    return out, lse


def _new_workspace(cache: KvCache, n_q_heads: int, max_seqs: int, stream) -> KvWorkspace:
    """A workspace zeroed on the stream that will use it."""
    if stream is None:
        return KvWorkspace(cache, n_q_heads, max_seqs)
    with torch.cuda.stream(torch.cuda.ExternalStream(stream, device=cache.k.device) if isinstance(stream, int) else stream):
        return KvWorkspace(cache, n_q_heads, max_seqs)
