"""ctypes binding of the paged cache: page pools, block tables, rotary positions, appended tokens, stored compressed
caches and attention over pages.  Argument marshalling only, every step runs in the HIP kernels."""
from __future__ import annotations

import ctypes
from typing import Optional, Tuple

import torch

from ._lib import (CompressedCache, MedaAppendParams, MedaError, MedaPagedParams, MedaPagePool, MedaPageParams,
                   MedaRotaryParams, MedaStoreParams, _check, _DTYPES, load_library)

ROTARY_INTERLEAVED = 1
ROTARY_INVERSE = 2
PAGE_SIZES = (16, 32, 64, 128, 256)
_E4M3 = 2
# Rows that a kernel writes count as changed in place: a graph that has kept them for its backward pass then says so.
_written = torch.autograd.graph.increment_version


def _p(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _call(fn, device: int, stream, *args):
    """Launches on the current device: the one where the tensors are."""
    if torch._C._cuda_getDevice() == device:
        status = fn(*args, torch._C._cuda_getCurrentRawStream(device) if stream is None else stream.cuda_stream)
    else:
        with torch.cuda.device(device):
            status = fn(*args, (torch.cuda.current_stream(device) if stream is None else stream).cuda_stream)
    if status != 0:
        _check(status)


def _empty(shape, dtype, device, stream):
    """New memory for a call on ``stream``: taken from that stream's memory, which nothing else on its way uses."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _no_graph(*tensors):
    """The kernels record nothing for a backward pass: a tensor that needs one is refused, not cut off in silence."""
    for t in tensors:
        if t is not None and t.requires_grad:
            raise ValueError("a tensor requires grad: gradients are not recorded here, call under torch.no_grad() or with detached "
                             "tensors (the gradient of meda_rotary is the same call with inverse=True)")


class _Kept:
    """Memory that an object keeps from call to call.  The allocator knows the stream where it was made; it has to hear of
    every other one that works with it, or it would give the memory away, once the object is gone, while kernels of that
    stream still use it."""

    def __init__(self, device: int, tensors):
        self._device, self._tensors = device, tensors
        self._streams = {torch._C._cuda_getCurrentRawStream(device)}

    def used_on(self, stream) -> None:
        raw = torch._C._cuda_getCurrentRawStream(self._device) if stream is None else stream.cuda_stream
        if raw not in self._streams:
            for t in self._tensors:
                t.record_stream(torch.cuda.current_stream(self._device) if stream is None else stream)
            self._streams.add(raw)


def _lend(device: int, stream, *tensors) -> None:
    """The tensors of a call on a stream that is not the current one: dropped after the call, their memory is not given away
    before that stream is done with it."""
    if stream.cuda_stream != torch._C._cuda_getCurrentRawStream(device):
        for t in tensors:
            if t is not None:
                t.record_stream(stream)


# A call of a kind that was checked before (the same shapes, strides, types and devices) is not checked again: half of the
# time of a small call went into it.  What an entry holds depends on nothing else, addresses least of all.  (Keys of the
# calls of every layer are spelled out: with a function per tensor an append of 64 tokens took 0.3 us more, a step of attention
# 0.7 more on the host.)
_checked: dict = {}


def _remember(key, entry):
    if len(_checked) >= 1024:
        _checked.clear()
    _checked[key] = entry
    return entry


def _kind(t):
    return None if t is None else (t.shape, t.stride(), t.dtype, t.get_device())


def _want(name, t, shape, dtype, device):
    """A contiguous tensor of this shape, type and device."""
    if (not isinstance(t, torch.Tensor) or t.dtype != dtype or tuple(t.shape) != tuple(shape) or t.device != device
            or not t.is_contiguous()):
        raise ValueError(f"{name}: expected a contiguous {dtype} tensor of shape {tuple(shape)} on {device}")


def _want_rows(name, t, shape, dtype, device):
    """Rows [tokens][heads][d] by strides: only the last dimension has to be contiguous."""
    if (not isinstance(t, torch.Tensor) or t.dtype != dtype or tuple(t.shape) != tuple(shape) or t.device != device
            or (t.numel() > 0 and t.stride(-1) != 1)):
        raise ValueError(f"{name}: expected a {dtype} tensor of shape {tuple(shape)} with contiguous rows on {device}")
    step = 16 // t.element_size()
    if t.numel() > 0 and any(n > 1 and s % step for n, s in zip(t.shape[:-1], t.stride()[:-1])):
        raise ValueError(f"{name}: rows must start at multiples of 16 bytes")


def _strides(t: torch.Tensor):
    """{token, head} strides; those of dimensions of one entry do not matter."""
    return (ctypes.c_int64 * 2)(t.stride(0) if t.shape[0] > 1 else 0, t.stride(1) if t.shape[1] > 1 else 0)


def _extent(t, dims):
    """Bytes from the first element of these dimensions to behind the last."""
    return (sum((t.shape[i] - 1) * t.stride(i) for i in dims) + 1) * t.element_size() if t.numel() else 0


def _want_no_overlap(name, out, other_name, other, may_be_same):
    """Rows of outputs [tokens][heads][d] lie apart from those of inputs, or are them (same memory, same strides)."""
    if out.numel() == 0 or other.numel() == 0:
        return
    a, b, size = out.data_ptr(), other.data_ptr(), out.element_size()
    if may_be_same and a == b and out.shape == other.shape and all(
            n == 1 or s == r for n, s, r in zip(out.shape, out.stride(), other.stride())):
        return
    if a + _extent(out, (0, 1, 2)) <= b or b + _extent(other, (0, 1, 2)) <= a:
        return
    # interleaved views of one buffer, as q and k of a fused projection: equally far apart in one dimension, and inside
    # that distance next to each other
    for i in (0, 1):
        step = out.stride(i) * size
        if step == other.stride(i) * size and step > 0 and (b - a) % step >= _extent(out, (1 - i, 2)) and (
                (a - b) % step >= _extent(other, (1 - i, 2))):
            return
    raise ValueError(f"{name} overlaps {other_name}")


def _pages_apart(k, v):
    """Whether no page of k shares memory with one of v: all of one behind the other's, or in the gaps between them."""
    a, b, size = k.data_ptr(), v.data_ptr(), k[0].numel() * k.element_size()
    step = k.stride(0) * k.element_size()
    extent = (k.shape[0] - 1) * step + size
    return a + extent <= b or b + extent <= a or (k.shape[0] > 1 and (b - a) % step >= size and (a - b) % step >= size)


class PagePool:
    """Pages of K and V [n_pages][n_kv_heads][page_size][head_dim] (any distance from page to page, the same for both),
    for 8-bit pages (uint8 codes) with one scale per row [n_pages][n_kv_heads][page_size]."""

    def __init__(self, k_pages: torch.Tensor, v_pages: torch.Tensor, k_scales: Optional[torch.Tensor] = None,
                 v_scales: Optional[torch.Tensor] = None):
        if k_pages.dim() != 4 or k_pages.dtype not in (torch.float32, torch.bfloat16, torch.uint8):
            raise ValueError("k_pages: expected a float32, bfloat16 or uint8 tensor [n_pages][n_kv_heads][page_size][head_dim] on the GPU")
        n, heads, page, d = k_pages.shape
        if n < 1 or heads < 1:
            raise ValueError("k_pages: expected at least one page and one head")
        for name, t in (("k_pages", k_pages), ("v_pages", v_pages)):
            if (t.shape != k_pages.shape or t.dtype != k_pages.dtype or t.device != k_pages.device
                    or not t[0].is_contiguous() or (n > 1 and t.stride(0) != k_pages.stride(0))):
                raise ValueError(f"{name}: expected {k_pages.dtype} {tuple(k_pages.shape)} on {k_pages.device}, every page "
                                 "contiguous, K and V pages the same distance apart")
        # (a page that is repeated has a distance of 0, which the library takes for that of pages next to each other)
        if n > 1 and k_pages.stride(0) < heads * page * d:
            raise ValueError(f"k_pages, v_pages: pages of {heads * page * d} elements lie {k_pages.stride(0)} apart")
        if page not in PAGE_SIZES:
            raise ValueError(f"page_size {page}: expected one of {PAGE_SIZES}")
        if k_pages.dtype == torch.uint8:
            for name, t in (("k_scales", k_scales), ("v_scales", v_scales)):
                _want(name, t, (n, heads, page), torch.float32, k_pages.device)
        elif k_scales is not None or v_scales is not None:
            raise ValueError("scales belong to uint8 pages")
        if not _pages_apart(k_pages, v_pages) or (k_scales is not None and not _pages_apart(k_scales, v_scales)):
            raise ValueError("k_pages and v_pages, k_scales and v_scales: must not share memory")
        _no_graph(k_pages, v_pages, k_scales, v_scales)
        if not k_pages.is_cuda:
            raise ValueError("k_pages, v_pages: expected tensors on the GPU")
        self.k_pages, self.v_pages, self.k_scales, self.v_scales = k_pages, v_pages, k_scales, v_scales
        self.tensors = (k_pages, v_pages) if k_scales is None else (k_pages, v_pages, k_scales, v_scales)
        self.device, self.page_size, self.n_kv_heads, self.head_dim, self.n_pages = k_pages.device, page, heads, d, n
        # the type of the rows that are written to the pages and of the queries that read them
        self.row_dtype = torch.float32 if k_pages.dtype == torch.float32 else torch.bfloat16
        code = _E4M3 if k_pages.dtype == torch.uint8 else _DTYPES[k_pages.dtype]
        self.desc = MedaPagePool(n, k_pages.stride(0) if n > 1 else 0, heads, d, page, code, _p(k_pages), _p(v_pages),
                                 _p(k_scales), _p(v_scales))
        self.ref = ctypes.byref(self.desc)
        self.index = self.device.index
        self.key = (n, heads, page, d, code, self.index)

    @classmethod
    def empty(cls, n_pages, n_kv_heads, page_size, head_dim, dtype=torch.bfloat16, device="cuda:0") -> "PagePool":
        """A new pool; ``dtype`` torch.uint8 (or torch.float8_e4m3fn) for 8-bit pages."""
        if dtype == torch.float8_e4m3fn:
            dtype = torch.uint8
        shape = (n_pages, n_kv_heads, page_size, head_dim)
        k, v = (torch.empty(shape, dtype=dtype, device=device) for _ in range(2))
        if dtype != torch.uint8:
            return cls(k, v)
        return cls(k, v, *(torch.empty(shape[:3], dtype=torch.float32, device=device) for _ in range(2)))


class RotaryPlan:
    """Frequencies of the pairs (float64 [rot_dim / 2] on the GPU), the position axis of every pair (uint8, None for one
    axis), and whether pairs are neighbours (2p, 2p + 1) or halves (p, p + rot_dim / 2)."""

    def __init__(self, inv_freq: torch.Tensor, axis: Optional[torch.Tensor] = None, n_axes: int = 1, interleaved: bool = False):
        if inv_freq.dim() != 1 or inv_freq.dtype != torch.float64 or not inv_freq.is_cuda or not inv_freq.is_contiguous() or inv_freq.numel() < 1:
            raise ValueError("inv_freq: expected a contiguous float64 vector on the GPU")
        if not 1 <= n_axes <= 4 or (axis is None and n_axes != 1):
            raise ValueError("n_axes: expected 1 to 4, and the axis of every pair with more than one")
        if axis is not None:
            _want("axis", axis, inv_freq.shape, torch.uint8, inv_freq.device)
        self.inv_freq, self.axis, self.n_axes, self.interleaved = inv_freq, axis, n_axes, interleaved
        self.rot_dim, self.device = 2 * inv_freq.numel(), inv_freq.device
        self.flags = ROTARY_INTERLEAVED if interleaved else 0
        self.key = (self.rot_dim, n_axes, axis is None, interleaved, self.device.index)

    def _positions(self, positions, n_tokens, device):
        """The stride from one axis' positions to the next."""
        if positions is None or positions.dtype != torch.int32 or positions.device != device or self.device != device:
            raise ValueError(f"positions: expected int32 on {device}, where the plan is")
        shape = tuple(positions.shape)
        if shape != (self.n_axes, n_tokens) and not (self.n_axes == 1 and shape == (n_tokens,)):
            raise ValueError(f"positions: expected int32 [{self.n_axes}][{n_tokens}]")
        if n_tokens > 1 and positions.stride(-1) != 1:
            raise ValueError("positions: those of an axis must be contiguous")
        if positions.dim() == 2 and self.n_axes > 1:
            if positions.stride(0) < 1 and n_tokens > 0:
                raise ValueError("positions: axes must lie apart")
            return positions.stride(0)
        return 0


def meda_rotary(q: torch.Tensor, k: Optional[torch.Tensor], positions: torch.Tensor, rope: RotaryPlan,
                q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None, inverse: bool = False,
                stream=None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """Rotary positions of q [T][Hq][d] and k [T][Hk][d] (any strides with contiguous rows; ``x.transpose(0, 1)`` of an
    [H][T][d] array is such a view).  The outputs may be the inputs; without them new ones are made.  ``inverse`` turns
    back: the gradient of the rotation (it is not recorded: tensors that require grad are refused where grad mode is on)."""
    if torch.is_grad_enabled():
        _no_graph(q, k, q_out, k_out)
    key = ("rotary", None if rope is None else rope.key, inverse, q.shape, q.stride(), q.dtype, q.get_device(),
           positions if positions is None else (positions.shape, positions.stride(), positions.dtype, positions.get_device()),
           k if k is None else (k.shape, k.stride(), k.dtype, k.get_device()),
           q_out if q_out is None else (q_out.shape, q_out.stride(), q_out.dtype, q_out.get_device()),
           k_out if k_out is None else (k_out.shape, k_out.stride(), k_out.dtype, k_out.get_device()))
    plan = _checked.get(key)
    if plan is None:
        plan = _remember(key, _plan_rotary(q, k, positions, rope, q_out, k_out, inverse))
    params, dev, new_q, new_k, ext = plan
    if new_q is not None:
        q_out = _empty(new_q, q.dtype, q.device, stream)
    if new_k is not None:
        k_out = _empty(new_k, k.dtype, k.device, stream)
    pq, pk, po, pko = q.data_ptr(), _p(k), q_out.data_ptr(), _p(k_out)
    for name, out, a, n in (("q_out", q_out, po, ext[2]), ("k_out", k_out, pko, ext[3])):
        if out is not None:
            if a < pq + ext[0] and pq < a + n:
                _want_no_overlap(name, out, "q", q, name == "q_out")
            if pk is not None and a < pk + ext[1] and pk < a + n:
                _want_no_overlap(name, out, "k", k, name == "k_out")
    if pko is not None and po < pko + ext[3] and pko < po + ext[2]:
        _want_no_overlap("q_out", q_out, "k_out", k_out, False)
    if new_q is None:
        _written(q_out)
    if new_k is None and k_out is not None:
        _written(k_out)
    if stream is not None:
        _lend(dev, stream, q, k, positions, rope.inv_freq, rope.axis, q_out, k_out)
    _call(load_library().meda_rotary, dev, stream, params, pq, pk, positions.data_ptr(), rope.inv_freq.data_ptr(), _p(rope.axis), po, pko)
    return q_out, k_out


def _plan_rotary(q, k, positions, rope, q_out, k_out, inverse):
    """The checks of a call, its parameters, the shapes of the outputs to make, and the extents of q, k and the outputs."""
    if q.dim() != 3 or q.dtype not in _DTYPES or not q.is_cuda:
        raise ValueError("q: expected a float32 or bfloat16 tensor [tokens][heads][head_dim] on the GPU")
    T, Hq, d = q.shape
    if rope is None or rope.rot_dim > d:
        raise ValueError("a plan of the rotation is needed" if rope is None else f"the plan turns {rope.rot_dim} elements, a row has {d}")
    dt, dev = q.dtype, q.device
    _want_rows("q", q, (T, Hq, d), dt, dev)
    if q_out is not None:
        _want_rows("q_out", q_out, (T, Hq, d), dt, dev)
    qo = _strides(q_out) if q_out is not None else (ctypes.c_int64 * 2)(Hq * d, d)
    Hk, ks, ko = 0, (ctypes.c_int64 * 2)(0, 0), (ctypes.c_int64 * 2)(0, 0)
    if k is not None:
        if k.dim() != 3:
            raise ValueError("k: expected [tokens][heads][head_dim]")
        Hk = k.shape[1]
        _want_rows("k", k, (T, Hk, d), dt, dev)
        if k_out is not None:
            _want_rows("k_out", k_out, (T, Hk, d), dt, dev)
        ks, ko = _strides(k), (_strides(k_out) if k_out is not None else (ctypes.c_int64 * 2)(Hk * d, d))
    elif k_out is not None:
        raise ValueError("k_out without k")
    params = MedaRotaryParams(T, _strides(q), qo, ks, ko, rope._positions(positions, T, dev), Hq, Hk, d, rope.rot_dim, rope.n_axes,
                              _DTYPES[dt], rope.flags | (ROTARY_INVERSE if inverse else 0))
    size, dims = q.element_size(), (0, 1, 2)
    ext = (_extent(q, dims), 0 if k is None else _extent(k, dims), T * Hq * d * size if q_out is None else _extent(q_out, dims),
           0 if k is None else (T * Hk * d * size if k_out is None else _extent(k_out, dims)))
    return (ctypes.byref(params), dev.index, (T, Hq, d) if q_out is None else None,
            (T, Hk, d) if k is not None and k_out is None else None, ext)


def meda_paged_append(pool: PagePool, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor,
                      q: Optional[torch.Tensor] = None, positions: Optional[torch.Tensor] = None,
                      rope: Optional[RotaryPlan] = None, q_out: Optional[torch.Tensor] = None,
                      stream=None) -> Optional[torch.Tensor]:
    """Writes k, v [M][Hkv][d] of new tokens to their ``slots`` (int64 [M], -1: none), k rotated where a plan is given;
    returns q [M][Hq][d] rotated alike (``q_out``, which may be q)."""
    if torch.is_grad_enabled() and (k.requires_grad or v.requires_grad or (q is not None and q.requires_grad)
                                    or (q_out is not None and q_out.requires_grad)):
        _no_graph(k, v, q, q_out)
    key = ("append", pool.key, None if rope is None else rope.key, k.shape, k.stride(), k.dtype, k.get_device(),
           v.shape, v.stride(), v.dtype, v.get_device(), slots.shape, slots.stride(), slots.dtype, slots.get_device(),
           q if q is None else (q.shape, q.stride(), q.dtype, q.get_device()),
           positions if positions is None else (positions.shape, positions.stride(), positions.dtype, positions.get_device()),
           q_out if q_out is None else (q_out.shape, q_out.stride(), q_out.dtype, q_out.get_device()))
    plan = _checked.get(key)
    if plan is None:
        plan = _remember(key, _plan_append(pool, k, v, slots, q, positions, rope, q_out))
    params, new_q, ext = plan
    if new_q is not None:
        q_out = _empty(new_q, q.dtype, q.device, stream)
    po = _p(q_out)
    if po is not None:
        for name, t, n in (("q", q, ext[0]), ("k", k, ext[1]), ("v", v, ext[2])):
            a = t.data_ptr()
            if po < a + n and a < po + ext[3]:
                _want_no_overlap("q_out", q_out, name, t, name == "q")
    if new_q is None and q_out is not None:
        _written(q_out)
    if stream is not None:
        _lend(pool.index, stream, k, v, slots, q, q_out, *pool.tensors)
        if rope is not None:
            _lend(pool.index, stream, positions, rope.inv_freq, rope.axis)
    turn = (None, None, None) if rope is None else (positions.data_ptr(), rope.inv_freq.data_ptr(), _p(rope.axis))
    _call(load_library().meda_paged_append, pool.index, stream, pool.ref, params, _p(q), k.data_ptr(), v.data_ptr(), *turn, slots.data_ptr(), po)
    return q_out


def _plan_append(pool, k, v, slots, q, positions, rope, q_out):
    """The checks of a call, its parameters, the shape of the output to make, and the extents of q, k, v and the output."""
    dev, dt, d = pool.device, pool.row_dtype, pool.head_dim
    if slots.dim() != 1 or slots.dtype != torch.int64 or slots.device != dev:
        raise ValueError(f"slots: expected an int64 vector on {dev}")
    M = slots.shape[0]
    if M > 1 and slots.stride(0) < 1:
        raise ValueError("slots: every token needs an entry of its own")
    _want_rows("k", k, (M, pool.n_kv_heads, d), dt, dev)
    _want_rows("v", v, (M, pool.n_kv_heads, d), dt, dev)
    zero = (ctypes.c_int64 * 2)(0, 0)
    Hq, qs, qo = 0, zero, zero
    if q is not None:
        if q.dim() != 3:
            raise ValueError("q: expected [tokens][heads][head_dim]")
        Hq = q.shape[1]
        _want_rows("q", q, (M, Hq, d), dt, dev)
        if q_out is not None:
            _want_rows("q_out", q_out, (M, Hq, d), dt, dev)
        qs, qo = _strides(q), (_strides(q_out) if q_out is not None else (ctypes.c_int64 * 2)(Hq * d, d))
    elif q_out is not None:
        raise ValueError("q_out without q")
    rot, axes, flags, pos_stride = 0, 1, 0, 0
    if rope is not None:
        if rope.rot_dim > d:
            raise ValueError(f"the plan turns {rope.rot_dim} elements, a row has {d}")
        rot, axes, flags, pos_stride = rope.rot_dim, rope.n_axes, rope.flags, rope._positions(positions, M, dev)
    elif positions is not None:
        raise ValueError("positions without a plan of the rotation")
    params = MedaAppendParams(M, qs, qo, _strides(k), _strides(v), pos_stride, slots.stride(0) if M > 1 else 1, Hq, rot, axes,
                              _DTYPES[dt], flags)
    dims = (0, 1, 2)
    ext = (0 if q is None else _extent(q, dims), _extent(k, dims), _extent(v, dims),
           0 if q is None else (M * Hq * d * k.element_size() if q_out is None else _extent(q_out, dims)))
    return ctypes.byref(params), (M, Hq, d) if q is not None and q_out is None else None, ext


def _want_table(table, lens, device):
    """Rows, blocks and the strides of a block table and its rows' lengths."""
    if table.dim() != 2 or table.dtype != torch.int32 or table.device != device or table.shape[1] < 1 or (
            table.shape[1] > 1 and table.stride(1) != 1):
        raise ValueError(f"table: expected int32 [rows][blocks] with contiguous rows on {device}")
    R, blocks = table.shape
    if lens.dim() != 1 or lens.dtype != torch.int32 or lens.device != device or lens.shape[0] != R:
        raise ValueError(f"lens: expected an int32 vector with one entry per row of the table on {device}")
    if R > 1 and (table.stride(0) < blocks or lens.stride(0) < 1):
        raise ValueError("table, lens: rows must lie apart")
    return R, blocks, (table.stride(0) if R > 1 else blocks), (lens.stride(0) if R > 1 else 1)


def meda_paged_store(pool: PagePool, cache: CompressedCache, table: torch.Tensor, lens: torch.Tensor, stream=None) -> None:
    """Moves the caches that a call of meda_compress returned to pages: row n * L + l of ``table`` and ``lens`` (the lengths
    that meda_page_update granted) belongs to layer l of sequence n."""
    if torch.is_grad_enabled():
        _no_graph(cache.k_out, cache.v_out)
    key = ("store", pool.key, cache.n_kv_heads, _kind(cache.k_out), _kind(cache.v_out), _kind(cache.layer_len), _kind(cache.layer_off),
           _kind(table), _kind(lens))
    params = _checked.get(key)
    if params is None:
        params = _remember(key, _plan_store(pool, cache, table, lens))
    if stream is not None:
        _lend(pool.index, stream, cache.k_out, cache.v_out, cache.layer_len, cache.layer_off, table, lens, *pool.tensors)
    _call(load_library().meda_paged_store, pool.index, stream, pool.ref, params, cache.k_out.data_ptr(), cache.v_out.data_ptr(),
          cache.layer_len.data_ptr(), cache.layer_off.data_ptr(), lens.data_ptr(), table.data_ptr())


def _plan_store(pool, cache, table, lens):
    dev, dt, d = pool.device, pool.row_dtype, pool.head_dim
    if cache.layer_len.dim() not in (1, 2):
        raise ValueError("layer_len: expected [layers] or [sequences][layers]")
    N, L = (1, cache.layer_len.shape[0]) if cache.layer_len.dim() == 1 else cache.layer_len.shape
    batch = () if cache.layer_len.dim() == 1 else (N,)
    _want("layer_len", cache.layer_len, batch + (L,), torch.int32, dev)
    _want("layer_off", cache.layer_off, batch + (L + 1,), torch.int64, dev)
    if cache.n_kv_heads != pool.n_kv_heads:
        raise ValueError(f"the cache has {cache.n_kv_heads} kv heads, the pool {pool.n_kv_heads}")
    rows = cache.k_out.shape[0]
    _want("k_out", cache.k_out, (rows, d), dt, dev)
    _want("v_out", cache.v_out, (rows, d), dt, dev)
    R, blocks, ts, ls = _want_table(table, lens, dev)
    if R != N * L:
        raise ValueError(f"table: expected {N * L} rows, one per sequence and layer")
    if R * -(-blocks * pool.page_size // 16) * pool.n_kv_heads >= 1 << 31:
        raise ValueError(f"table: {R} rows of {blocks * pool.page_size} positions in {pool.n_kv_heads} heads are more than 2^34 together")
    return ctypes.byref(MedaStoreParams(rows, ts, ls, N, L, blocks, _DTYPES[dt]))


class PagedDecoder:
    """Holds the workspace and the output rows for attention over pages with a fixed number of rows and blocks.  Calls, and
    graphs that captured them, share both: on several streams at once use a decoder for each."""

    def __init__(self, pool: PagePool, n_rows: int, n_q_heads: int, max_blocks: int, dtype=None, softmax_scale: float = 0.0):
        self.pool, self.n_rows, self.n_q_heads, self.max_blocks = pool, n_rows, n_q_heads, max_blocks
        dt = pool.row_dtype if dtype is None else dtype
        self.params = MedaPagedParams(0, 0, 0, 0, n_rows, n_q_heads, max_blocks, _DTYPES.get(dt, -1), softmax_scale)
        need = int(load_library().meda_paged_workspace_bytes(pool.ref, ctypes.byref(self.params)))
        if need == 0:
            raise MedaError(1, "invalid or unsupported parameters of the paged step")
        self.dtype = dt
        self.workspace, self._workspace_bytes = torch.empty(need, dtype=torch.uint8, device=pool.device), need
        self._calls: dict = {}     # parameters of calls by the shapes and strides of their tensors, as in _checked
        self.out = torch.empty((n_rows, n_q_heads, pool.head_dim), dtype=dt, device=pool.device)
        self._kept = _Kept(pool.index, (self.workspace, self.out))

    def __call__(self, q: torch.Tensor, table: torch.Tensor, lens: torch.Tensor, out: Optional[torch.Tensor] = None,
                 stream=None) -> torch.Tensor:
        """q [rows][Hq][d] (rows any distance apart) over the pages of ``table`` [rows][blocks]; ``lens`` [rows].  Without
        ``out`` the result lies in a buffer that the next call overwrites."""
        out = self.out if out is None else out
        if torch.is_grad_enabled() and (q.requires_grad or out.requires_grad):
            _no_graph(q, out)
        key = (q.shape, q.stride(), q.dtype, q.get_device(), table.shape, table.stride(), table.dtype, table.get_device(),
               lens.shape, lens.stride(), lens.dtype, lens.get_device(), out.shape, out.stride(), out.dtype, out.get_device())
        call = self._calls.get(key)
        if call is None:
            if len(self._calls) >= 64:
                self._calls.clear()
            call = self._calls[key] = self._plan(q, table, lens, out)
        params, q_bytes, out_bytes = call
        pool, pq, po = self.pool, q.data_ptr(), out.data_ptr()
        if pq < po + out_bytes and po < pq + q_bytes:
            _want_no_overlap("out", out, "q", q, False)
        _written(out)
        self._kept.used_on(stream)
        if stream is not None:
            _lend(pool.index, stream, q, table, lens, out, *pool.tensors)
        _call(load_library().meda_paged_attention, pool.index, stream, pool.ref, params, pq, table.data_ptr(), lens.data_ptr(), po,
              self.workspace.data_ptr(), self._workspace_bytes)
        return out

    def _plan(self, q, table, lens, out):
        """The checks of a call, its parameters, and the extents of q and out."""
        pool, shape = self.pool, (self.n_rows, self.n_q_heads, self.pool.head_dim)
        for name, t in (("q", q), ("out", out)):
            _want_rows(name, t, shape, self.dtype, pool.device)
            if shape[1] > 1 and t.stride(1) != shape[2]:
                raise ValueError(f"{name}: the heads of a row must be contiguous")
            if shape[0] > 1 and t.stride(0) < shape[1] * shape[2]:
                raise ValueError(f"{name}: rows must lie apart")
        R, blocks, ts, ls = _want_table(table, lens, pool.device)
        if R != self.n_rows or blocks != self.max_blocks:
            raise ValueError(f"table: expected {self.n_rows} rows of {self.max_blocks} blocks")
        p, row = self.params, shape[1] * shape[2]
        params = MedaPagedParams(q.stride(0) if R > 1 else row, out.stride(0) if R > 1 else row, ts, ls, R, shape[1], blocks, p.dtype,
                                 p.softmax_scale)
        return ctypes.byref(params), _extent(q, (0, 1, 2)), _extent(out, (0, 1, 2))


def meda_page_update_workspace_bytes(n_rows: int) -> int:
    return int(load_library().meda_page_update_workspace_bytes(n_rows))


def meda_page_update(lens: torch.Tensor, n_new: torch.Tensor, table: torch.Tensor, free_ring: torch.Tensor,
                     free_state: torch.Tensor, page_size: int, lens_out: Optional[torch.Tensor] = None,
                     free_state_out: Optional[torch.Tensor] = None, slots: Optional[torch.Tensor] = None,
                     granted: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None,
                     rows_per_seq: int = 1) -> None:
    """Room for ``n_new`` positions per row (negative: the row has ended), from the free pages.  ``table`` [R][blocks] and
    ``free_ring`` [n_pages] are updated in place, lens [R] and free_state [2] too unless outputs for them are given;
    ``slots`` [R][max_new] and ``granted`` [R] receive the slots and what each row got.  ``rows_per_seq`` consecutive rows
    are granted together: all that they ask for, or nothing."""
    lens_out = lens if lens_out is None else lens_out
    free_state_out = free_state if free_state_out is None else free_state_out
    key = ("pages", _kind(lens), _kind(n_new), _kind(table), _kind(free_ring), _kind(free_state), page_size, _kind(lens_out),
           _kind(free_state_out), _kind(slots), _kind(granted), _kind(workspace), rows_per_seq)
    plan = _checked.get(key)
    if plan is None:
        plan = _remember(key, _plan_update(lens, n_new, table, free_ring, free_state, page_size, lens_out, free_state_out, slots, granted,
                                           workspace, rows_per_seq))
    params, dev, max_new, need = plan
    if workspace is None:
        workspace = _empty(need, torch.uint8, table.device, stream)
    if stream is not None:
        _lend(dev, stream, lens, n_new, table, free_ring, free_state, lens_out, free_state_out, slots, granted, workspace)
    _call(load_library().meda_page_update, dev, stream, params, lens.data_ptr(), n_new.data_ptr(), table.data_ptr(), free_ring.data_ptr(),
          free_state.data_ptr(), lens_out.data_ptr(), free_state_out.data_ptr(), slots.data_ptr() if max_new else None, _p(granted),
          workspace.data_ptr(), workspace.shape[0])


def _plan_update(lens, n_new, table, free_ring, free_state, page_size, lens_out, free_state_out, slots, granted, workspace, rows_per_seq):
    """The checks of a call, its parameters, the columns of slots, the workspace's size."""
    dev = table.device
    if not table.is_cuda:
        raise ValueError("table: expected a tensor on the GPU")
    if table.dim() != 2 or table.shape[0] < 1 or table.shape[1] < 1:
        raise ValueError("table: expected [rows][blocks]")
    R, blocks = table.shape
    if page_size not in PAGE_SIZES:
        raise ValueError(f"page_size {page_size}: expected one of {PAGE_SIZES}")
    if rows_per_seq < 1 or R % rows_per_seq:
        raise ValueError(f"rows_per_seq {rows_per_seq}: {R} rows are no multiple of it")
    for name, t, shape, dtype in (("lens", lens, (R,), torch.int32), ("n_new", n_new, (R,), torch.int32),
                                  ("table", table, (R, blocks), torch.int32), ("lens_out", lens_out, (R,), torch.int32),
                                  ("free_state", free_state, (2,), torch.int64),
                                  ("free_state_out", free_state_out, (2,), torch.int64)):
        _want(name, t, shape, dtype, dev)
    if free_ring.dim() != 1 or free_ring.shape[0] < 1:
        raise ValueError("free_ring: expected one entry per page")
    _want("free_ring", free_ring, free_ring.shape, torch.int32, dev)
    max_new = 0
    if slots is not None:
        if slots.dim() != 2:
            raise ValueError("slots: expected [rows][new positions]")
        max_new = slots.shape[1]
        _want("slots", slots, (R, max_new), torch.int64, dev)
    if granted is not None:
        _want("granted", granted, (R,), torch.int32, dev)
    if workspace is not None and (workspace.dim() != 1 or workspace.device != dev or workspace.dtype != torch.uint8
                                  or not workspace.is_contiguous()):
        raise ValueError(f"workspace: expected a contiguous uint8 vector on {dev}")
    return (ctypes.byref(MedaPageParams(free_ring.shape[0], R, blocks, page_size, max_new, rows_per_seq)), dev.index, max_new,
            meda_page_update_workspace_bytes(R))


class PagedCache:
    """The paged caches of up to ``n_seqs`` sequences with ``n_layers`` layers each, served together: page pool, block
    tables, lengths and free pages, and the calls of a serving loop.

    ::

        cache.admit(0, compressed)                       # the result of meda_compress becomes sequence 0 (and following)
        cache.step(active)                               # room for one token per active sequence, in every layer
        for layer in range(n_layers):
            q = cache.append(layer, k, v, q, positions)  # rotate, write k and v
            out = cache.attend(layer, q)
        cache.release([0])

    Row ``s * n_layers + l`` of ``table``, ``lens``, ``slots`` and ``granted`` belongs to layer l of sequence s.  No call
    synchronises, so the loop's body can be captured into a graph.  ``granted`` says after ``admit`` and ``step`` what each
    row got; what these return are views of it, which the next ``admit``, ``step`` or ``release`` overwrites.  Where the pages
    do not suffice for all layers of a sequence, none of them gets any (0) and the sequence is left as it was: release others
    and ask again for it, or release it.  Calls share the workspaces: use one stream, or order the streams."""

    def __init__(self, n_seqs: int, n_layers: int, n_q_heads: int, n_kv_heads: int, head_dim: int, max_len: int, n_pages: int,
                 page_size: int = 64, dtype=torch.bfloat16, rope: Optional[RotaryPlan] = None, softmax_scale: float = 0.0,
                 device="cuda:0"):
        if n_seqs < 1 or n_layers < 1 or max_len < 1 or page_size not in PAGE_SIZES:
            raise ValueError(f"expected sequences, layers, a length and a page size of {PAGE_SIZES}")
        if max_len > 1 << 29 or n_seqs * n_layers > 65536 or n_seqs * n_layers * -(-max_len // page_size) > 1 << 30:
            raise ValueError("more than 2^29 positions, 65536 layers of sequences, or 2^30 blocks of them")
        self.pool = PagePool.empty(n_pages, n_kv_heads, page_size, head_dim, dtype, device)
        dev = self.pool.device
        self.n_seqs, self.n_layers, self.n_q_heads, self.rope = n_seqs, n_layers, n_q_heads, rope
        rows, self.max_blocks = n_seqs * n_layers, (max_len + page_size - 1) // page_size
        self.table = torch.full((rows, self.max_blocks), -1, dtype=torch.int32, device=dev)
        self.lens = torch.zeros(rows, dtype=torch.int32, device=dev)
        self.granted = torch.zeros(rows, dtype=torch.int32, device=dev)
        self.slots = torch.full((rows, 1), -1, dtype=torch.int64, device=dev)
        self.free_ring = torch.arange(n_pages, dtype=torch.int32, device=dev)
        self.free_state = torch.tensor([0, n_pages], dtype=torch.int64, device=dev)
        self._new = torch.zeros((n_seqs, n_layers), dtype=torch.int32, device=dev)
        self._workspace = torch.empty(meda_page_update_workspace_bytes(rows), dtype=torch.uint8, device=dev)
        self.decoder = PagedDecoder(self.pool, n_seqs, n_q_heads, self.max_blocks, None, softmax_scale)
        self._kept = _Kept(self.pool.index, self.pool.tensors + (self.table, self.lens, self.granted, self.slots, self.free_ring,
                                                                 self.free_state, self._new, self._workspace))

    def _update(self, slots=None):
        meda_page_update(self.lens, self._new.view(-1), self.table, self.free_ring, self.free_state, self.pool.page_size,
                         slots=slots, granted=self.granted, workspace=self._workspace, rows_per_seq=self.n_layers)

    def admit(self, first: int, cache: CompressedCache) -> torch.Tensor:
        """The sequences of a compressed cache become the sequences first, first + 1, ..; what these held is released.
        Returns the positions granted, [N][L], in a buffer that the next call overwrites."""
        layer_len = cache.layer_len if cache.layer_len.dim() == 2 else cache.layer_len[None]
        n, layers = layer_len.shape
        if layers != self.n_layers or first < 0 or first + n > self.n_seqs:
            raise ValueError(f"expected {self.n_layers} layers and sequences below {self.n_seqs}")
        rows = slice(first * layers, (first + n) * layers)
        table, lens = self.table[rows], self.lens[rows]
        _plan_store(self.pool, cache, table, lens)      # (a cache that the store would not take is refused before anything changes)
        if cache.k_out.data_ptr() % 16 or cache.v_out.data_ptr() % 16:
            raise ValueError("k_out, v_out: expected memory aligned to 16 bytes")
        if torch.is_grad_enabled():
            _no_graph(cache.k_out, cache.v_out)
        self.release(range(first, first + n))
        self._new.zero_()
        self._new[first:first + n].copy_(layer_len)
        self._update()
        meda_paged_store(self.pool, cache, table, lens)
        return self.granted.view(self.n_seqs, layers)[first:first + n]

    def step(self, active: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Room for one token per active sequence (int32 or bool [n_seqs]; all without it); returns what was granted,
        [n_seqs][n_layers], in a buffer that the next call overwrites."""
        self._kept.used_on(None)
        if active is None:
            self._new.fill_(1)
        else:
            if tuple(active.shape) != (self.n_seqs,) or active.device != self.pool.device:
                raise ValueError(f"active: expected one entry per sequence on {self.pool.device}")
            self._new.copy_((active != 0)[:, None])
        self._update(self.slots)
        return self.granted.view(self.n_seqs, self.n_layers)

    def _rows(self, layer: int):
        if not 0 <= layer < self.n_layers:
            raise ValueError(f"layer {layer}: expected one of {self.n_layers}")
        step = self.n_layers
        return self.table[layer::step], self.lens[layer::step], self.slots[layer::step, 0]

    def append(self, layer: int, k: torch.Tensor, v: torch.Tensor, q: Optional[torch.Tensor] = None,
               positions: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
        """k, v [n_seqs][Hkv][d] of the step's tokens enter the layer; returns q [n_seqs][Hq][d].  k and q are rotated by
        ``positions`` where the cache has a plan of the rotation; without one they are taken as they are."""
        self._kept.used_on(None)
        return meda_paged_append(self.pool, k, v, self._rows(layer)[2], q, positions, self.rope, q_out)

    def attend(self, layer: int, q: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Attention of q [n_seqs][Hq][d] over the layer's positions, the step's own included (without ``out`` the result
        lies in a buffer that the next call overwrites)."""
        self._kept.used_on(None)
        table, lens, _ = self._rows(layer)
        return self.decoder(q, table, lens, out)

    def release(self, seqs) -> None:
        """The sequences' pages go back to the pool, their lengths become 0.  A slot that the last step gave them is theirs no
        longer: what is appended for them before the next step is not written."""
        seqs = list(seqs)
        for s in seqs:
            if not 0 <= s < self.n_seqs:
                raise ValueError(f"sequence {s}: expected one of {self.n_seqs}")
        self._kept.used_on(None)
        self._new.zero_()
        slots = self.slots.view(self.n_seqs, self.n_layers)
        for s in seqs:
            self._new[s].fill_(-1)
            slots[s].fill_(-1)
        self._update()
