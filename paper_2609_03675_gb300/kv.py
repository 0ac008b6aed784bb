"""Answering from the selected frames: rotary positions, a paged key/value
cache of 16-bit values, bytes or 4-bit codes, and attention over it.

    from paper_2609_03675_gb300 import KVCache, Rotary
    rotary = Rotary(128, base=1e6)
    cache = KVCache(n_pages, 64, 32, 8, 128, bits=4, rotary=rotary)
    q = cache.append(k, v, table, lengths, offsets, positions=positions, q=q)
    out, lse = cache.attend(q, table, lengths, offsets, max_new=longest_question)
    out, lse = cache.attend_shared(q, table, lengths, offsets, prefix_table=stream, prefix_lengths=n)  # questions about one stream

Thin binding of the entry points that include/cofie_kv.h declares (the layout
of pages and codes is described there); every value is computed in the
library's CUDA kernels.
"""
from __future__ import annotations

import contextlib
import ctypes
import struct

import torch

from . import _abi
from ._abi import NGFFError

__all__ = ["KVCache", "Rotary"]

_DTYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}
_LAYOUTS = {"half": 0, "interleaved": 1}
_SCALINGS = {"none": 0, "linear": 1, "base": 2, "yarn": 3}
_BITS = {16: (16, 16), "int8": (8, 0x108), 4: (4, 4)}  # of a value, and as the library takes it
_get_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)


class _RotaryParams(ctypes.Structure):
    _fields_ = [("head_dim", ctypes.c_uint32), ("rotary_dim", ctypes.c_uint32), ("layout", ctypes.c_uint32),
                ("scaling", ctypes.c_uint32), ("base", ctypes.c_double), ("factor", ctypes.c_double),
                ("original_len", ctypes.c_double), ("beta_fast", ctypes.c_double), ("beta_slow", ctypes.c_double),
                ("n_axes", ctypes.c_uint32), ("axes", ctypes.c_char_p)]


class _Rows(ctypes.Structure):
    _fields_ = [("src", ctypes.c_void_p), ("out", ctypes.c_void_p), ("heads", ctypes.c_uint32), ("in_token", ctypes.c_int64),
                ("in_head", ctypes.c_int64), ("out_token", ctypes.c_int64), ("out_head", ctypes.c_int64)]


class _KVParams(ctypes.Structure):
    _fields_ = [("n_pages", ctypes.c_uint32), ("page_size", ctypes.c_uint32), ("n_heads", ctypes.c_uint32),
                ("n_kv_heads", ctypes.c_uint32), ("head_dim", ctypes.c_uint32), ("dtype", ctypes.c_uint32),
                ("bits", ctypes.c_uint32), ("device", ctypes.c_int32), ("k_pages", ctypes.c_void_p),
                ("v_pages", ctypes.c_void_p), ("k_scales", ctypes.c_void_p), ("v_scales", ctypes.c_void_p)]


class _Batch(ctypes.Structure):
    _fields_ = [("n_seqs", ctypes.c_uint32), ("n_tokens", ctypes.c_uint32), ("max_new", ctypes.c_uint32),
                ("table_stride", ctypes.c_uint32), ("table", ctypes.c_void_p), ("lengths", ctypes.c_void_p),
                ("offsets", ctypes.c_void_p)]


class _Prefix(ctypes.Structure):
    _fields_ = [("n_groups", ctypes.c_uint32), ("max_new", ctypes.c_uint32), ("table_stride", ctypes.c_uint32),
                ("table", ctypes.c_void_p), ("lengths", ctypes.c_void_p), ("groups", ctypes.c_void_p), ("mask", ctypes.c_void_p),
                ("mask_stride", ctypes.c_uint64)]


# The calls' structs, packed in one go into a buffer that the handle keeps (a
# ctypes field costs the host more than a tensor's stride; a step of single
# tokens is bound by the host).
_ROWS = struct.Struct("=QQI4xqqqq")
_BATCH = struct.Struct("=IIIIQQQ")
_PREFIX = struct.Struct("=III4xQQQQQ")
assert _ROWS.size == ctypes.sizeof(_Rows) and _BATCH.size == ctypes.sizeof(_Batch) and _PREFIX.size == ctypes.sizeof(_Prefix)
_PREFIX_AT = _BATCH.size + 3 * _ROWS.size

# Every symbol include/cofie_kv.h declares.
EXPORTS = ("cofie_rotary_create", "cofie_rotary_destroy", "cofie_rotary_run", "cofie_rotary_last_error", "cofie_kv_create",
           "cofie_kv_destroy", "cofie_kv_append", "cofie_kv_read", "cofie_kv_attend", "cofie_kv_attend_shared", "cofie_kv_status",
           "cofie_kv_last_error")

_bound = None


def _load():
    global _bound
    lib = _abi.load()
    if _bound is lib:
        return lib
    vp, u32, u64, P = ctypes.c_void_p, ctypes.c_uint32, ctypes.c_uint64, ctypes.POINTER
    for name, res, args in (
            ("cofie_rotary_create", ctypes.c_int, [P(_RotaryParams), P(vp)]),
            ("cofie_rotary_destroy", None, [vp]),
            ("cofie_rotary_run", ctypes.c_int, [vp, vp, u32, u32, vp, u32, ctypes.c_int, vp]),
            ("cofie_rotary_last_error", ctypes.c_char_p, [vp]),
            ("cofie_kv_create", ctypes.c_int, [P(_KVParams), P(vp)]),
            ("cofie_kv_destroy", None, [vp]),
            ("cofie_kv_append", ctypes.c_int, [vp, vp, vp, vp, vp, vp, vp, vp]),
            ("cofie_kv_read", ctypes.c_int, [vp, vp, vp, vp, vp]),
            ("cofie_kv_attend", ctypes.c_int, [vp, vp, vp, vp, vp, u64, ctypes.c_int, ctypes.c_float, vp]),
            ("cofie_kv_attend_shared", ctypes.c_int, [vp, vp, vp, vp, vp, vp, u64, ctypes.c_int, ctypes.c_float, vp]),
            ("cofie_kv_status", ctypes.c_int, [vp, vp]),
            ("cofie_kv_last_error", ctypes.c_char_p, [vp])):
        f = getattr(lib, name)
        f.restype, f.argtypes = res, args
    _bound = lib
    return lib


def _stream_of(cuda_stream, index):
    if cuda_stream is None:
        return _raw_stream(index)
    return cuda_stream.cuda_stream if isinstance(cuda_stream, torch.cuda.Stream) else int(cuda_stream)


def _allocating(cuda_stream, index):
    """Outputs made for a call on another stream than the current one belong to that stream."""
    if cuda_stream is None:
        return contextlib.nullcontext()
    if not isinstance(cuda_stream, torch.cuda.Stream):
        cuda_stream = torch.cuda.ExternalStream(int(cuda_stream), device=index)
    return torch.cuda.stream(cuda_stream)


def _heads(x, dtype, index, what, shape):
    """Refuses a tensor that is not of this shape, [tokens, heads, head_dim], as the call wants it; its strides."""
    if x.shape != shape or x.dtype is not dtype or x.get_device() != index:
        raise ValueError(f"{what} must be a {dtype} tensor {list(shape)} on cuda:{index}")
    st = x.stride()
    if st[2] != 1:
        raise ValueError(f"{what}: a head's values must be contiguous")
    return st


def _int32(x, index, what, shape):
    if x.dtype is not torch.int32 or x.get_device() != index or not x.is_contiguous() or x.shape != shape:
        raise ValueError(f"{what} must be a contiguous int32 tensor {list(shape)} on cuda:{index}")
    return x.data_ptr()


class _Turned(torch.autograd.Function):
    """Rotary._run as a node of autograd's graph: its gradient is the rotation the other way round."""

    @staticmethod
    def forward(ctx, rotary, positions, transpose, cuda_stream, *xs):
        ctx.rotary, ctx.transpose = rotary, transpose
        ctx.save_for_backward(positions)
        ctx.set_materialize_grads(False)
        return rotary._run(xs, positions, None, transpose, cuda_stream)

    @staticmethod
    def backward(ctx, *grads):
        some = [i for i, g in enumerate(grads) if g is not None and ctx.needs_input_grad[4 + i]]
        back = [None] * len(grads)
        if some:
            gs = tuple(grads[i] if grads[i].stride(-1) == 1 else grads[i].contiguous() for i in some)
            for i, g in zip(some, ctx.rotary._run(gs, ctx.saved_tensors[0], None, 1 - ctx.transpose, None)):
                back[i] = g
        return (None, None, None, None, *back)


class Rotary:
    """Rotates heads to their positions.

    layout: "half" pairs x[i] with x[i + rotary_dim / 2], "interleaved" x[2 i] with x[2 i + 1]; what lies past rotary_dim
    passes through. scaling: "none", "linear", "base" or "yarn" (with original_len, the trained length), by ``factor``.
    axes: None, or one axis number for each pair, where positions have several axes (frame, row, column)."""

    def __init__(self, head_dim: int, *, rotary_dim: int | None = None, base: float = 10000.0, layout: str = "half",
                 scaling: str = "none", factor: float = 1.0, original_len: float = 0.0, beta_fast: float = 32.0,
                 beta_slow: float = 1.0, axes=None):
        if layout not in _LAYOUTS or scaling not in _SCALINGS:
            raise ValueError(f"layout is one of {sorted(_LAYOUTS)}, scaling one of {sorted(_SCALINGS)}")
        rotary_dim = head_dim if rotary_dim is None else rotary_dim
        if axes is not None:
            axes = bytes(axes)
            if len(axes) != rotary_dim // 2:
                raise ValueError("axes has one entry for each of the rotary_dim / 2 pairs")
        self.head_dim, self.rotary_dim, self.layout = head_dim, rotary_dim, layout
        self.n_axes = max(axes) + 1 if axes else 1
        lib = _load()
        p = _RotaryParams(head_dim, rotary_dim, _LAYOUTS[layout], _SCALINGS[scaling], base, factor, original_len, beta_fast,
                          beta_slow, self.n_axes, axes)
        h = ctypes.c_void_p()
        rc = lib.cofie_rotary_create(ctypes.byref(p), ctypes.byref(h))
        if rc != _abi.OK:
            raise NGFFError(rc, lib.cofie_rotary_last_error(None).decode())
        self._lib, self._h = lib, h.value  # an integer: quicker to pass
        self._buf = ctypes.create_string_buffer(4 * _ROWS.size)
        self._at = ctypes.addressof(self._buf)

    def _positions(self, positions, n, index):
        return _int32(positions, index, "positions", (n,) if self.n_axes == 1 and positions.dim() == 1 else (self.n_axes, n))

    def _run(self, x, positions, out, transpose, cuda_stream):
        xs = (x,) if isinstance(x, torch.Tensor) else x
        k = len(xs)
        if not 1 <= k <= 4:
            raise ValueError("one to four tensors of the same tokens")
        for y in xs:
            if y.requires_grad and torch.is_grad_enabled():
                if out is not None:
                    raise ValueError("out does not go with tensors that require a gradient")
                outs = _Turned.apply(self, positions, transpose, cuda_stream, *xs)
                return outs[0] if xs is not x else outs
        first = xs[0]
        index, dtype, n = first.get_device(), first.dtype, first.shape[0]
        code = _DTYPES.get(dtype)
        if index < 0 or code is None:
            raise ValueError("the tensors must be bfloat16, float16 or float32, on a CUDA device")
        if out is None:
            with _allocating(cuda_stream, index):
                outs = tuple(torch.empty(y.shape, dtype=dtype, device=y.device) for y in xs)
        else:
            outs = (out,) if isinstance(out, torch.Tensor) else out
            if len(outs) != k:
                raise ValueError("out has a tensor for each input")
        d, buf, at = self.head_dim, self._buf, 0
        for y, o in zip(xs, outs):
            shape = (n, y.shape[1], d) if y.dim() == 3 else (n, 1, d)
            a, b = _heads(y, dtype, index, "x", shape), _heads(o, dtype, index, "out", shape)
            _ROWS.pack_into(buf, at, y.data_ptr(), o.data_ptr(), shape[1], a[0], a[1], b[0], b[1])
            at += 56
        where = self._positions(positions, n, index)
        stream = _raw_stream(index) if cuda_stream is None else _stream_of(cuda_stream, index)
        if index == _get_device():
            rc = self._lib.cofie_rotary_run(self._h, self._at, k, n, where, code, transpose, stream)
        else:
            with torch.cuda.device(index):
                rc = self._lib.cofie_rotary_run(self._h, self._at, k, n, where, code, transpose, stream)
        if rc:
            raise NGFFError(rc, self._lib.cofie_rotary_last_error(self._h).decode())
        return outs[0] if xs is not x else outs

    def apply(self, x, positions, *, out=None, cuda_stream=None):
        """x (a tensor [tokens, heads, head_dim], or up to four of the same tokens) rotated; positions int32 [tokens], or
        [axes, tokens]. ``out`` may be x itself. Tensors that require a gradient get it through autograd (without ``out``)."""
        return self._run(x, positions, out, 0, cuda_stream)

    def backward(self, grad, positions, *, out=None, cuda_stream=None):
        """The gradient of apply()'s input, from that of its output: the transposed rotation."""
        return self._run(grad, positions, out, 1, cuda_stream)

    def close(self):
        if getattr(self, "_h", None):
            self._lib.cofie_rotary_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:  # noqa: BLE001 -- interpreter shutdown
            pass


class KVCache:
    """Paged keys and values of one layer, n_pages pages of page_size tokens.

    bits: 16 (values of the cache's type), "int8" (bytes with a power of two for 64 of them: half the memory, values 0.6 to
    1.2 % of their standard deviation off) or 4 (codes, 10 % off). An 8 alone is refused: it names no one format.
    The pages are k_pages, v_pages (and k_scales, v_scales for less than 16 bits), made here unless given. Sequence s of a batch holds
    lengths[s] tokens; token i lies in page table[s, i // page_size]. A batch's new tokens are rows offsets[s] to
    offsets[s + 1] of every per-token argument, the last of the sequence's lengths[s] (offsets=None: one each).
    A cache has no gradient: tensors that require one are refused, unless under torch.no_grad()."""

    def __init__(self, n_pages: int, page_size: int, n_heads: int, n_kv_heads: int, head_dim: int, *,
                 dtype: torch.dtype = torch.bfloat16, bits: int | str = 16, rotary: Rotary | None = None, device: int | None = None,
                 k_pages=None, v_pages=None, k_scales=None, v_scales=None):
        lib = _load()
        if dtype not in (torch.bfloat16, torch.float16) or bits not in _BITS:
            raise ValueError("dtype is bfloat16 or float16, bits 16, 'int8' or 4")
        bits, kind = _BITS[bits]
        index = device if device is not None else k_pages.get_device() if k_pages is not None else torch.cuda.current_device()
        self.device = torch.device("cuda", index)
        lead = (n_pages, n_kv_heads, page_size)
        row, scale, of = (lead + (head_dim,), None, dtype) if bits == 16 else \
            (lead + (head_dim * bits // 8,), lead + (head_dim // 64,), torch.uint8)

        def pages(x, shape, dt):
            if shape is None:
                return None
            if x is None:
                return torch.zeros(shape, dtype=dt, device=self.device)
            if x.dtype != dt or tuple(x.shape) != shape or not x.is_contiguous() or x.get_device() != index:
                raise ValueError(f"pages must be contiguous {dt} of shape {shape} on cuda:{index}")
            return x

        self.k_pages, self.v_pages = pages(k_pages, row, of), pages(v_pages, row, of)
        self.k_scales, self.v_scales = pages(k_scales, scale, torch.int16), pages(v_scales, scale, torch.int16)
        ptr = lambda x: x.data_ptr() if x is not None else None  # noqa: E731
        p = _KVParams(n_pages, page_size, n_heads, n_kv_heads, head_dim, _DTYPES[dtype], kind, index, ptr(self.k_pages),
                      ptr(self.v_pages), ptr(self.k_scales), ptr(self.v_scales))
        h = ctypes.c_void_p()
        rc = lib.cofie_kv_create(ctypes.byref(p), ctypes.byref(h))
        if rc != _abi.OK:
            raise NGFFError(rc, lib.cofie_kv_last_error(None).decode())
        self._lib, self._h, self._index = lib, h.value, index
        self.n_pages, self.page_size, self.n_heads, self.n_kv_heads, self.head_dim = n_pages, page_size, n_heads, n_kv_heads, head_dim
        self.dtype, self.bits, self.rotary = dtype, bits, rotary
        # a batch, up to three tensors' rows, and the prefixes
        self._buf = ctypes.create_string_buffer(_PREFIX_AT + _PREFIX.size)
        self._at = ctypes.addressof(self._buf)

    def _check(self, rc):
        if rc:
            raise NGFFError(rc, self._lib.cofie_kv_last_error(self._h).decode())

    def _batch(self, table, lengths, offsets, n, max_new):
        index = self._index
        if table.dtype is not torch.int32 or table.get_device() != index or table.dim() != 2 or not table.is_contiguous():
            raise ValueError(f"table must be a contiguous int32 tensor [sequences, pages] on cuda:{index}")
        seqs, width = table.shape
        lengths, offsets = _int32(lengths, index, "lengths", (seqs,)), 0 if offsets is None else _int32(offsets, index, "offsets", (seqs + 1,))
        try:
            _BATCH.pack_into(self._buf, 0, seqs, n, max_new, width, table.data_ptr(), lengths, offsets)
        except struct.error:
            raise ValueError("max_new must be a whole number in [0, 2^32), and the batch's sizes below 2^32") from None

    def _rows(self, i, x, heads, what, n=None, out=None):
        """Packs tensor i of the call; returns where."""
        shape = (x.shape[0] if n is None else n, heads, self.head_dim)
        a = _heads(x, self.dtype, self._index, what, shape)
        at = 40 + 56 * i
        if out is None:
            _ROWS.pack_into(self._buf, at, x.data_ptr(), 0, heads, a[0], a[1], 0, 0)
        else:
            b = _heads(out, self.dtype, self._index, "out", shape)
            _ROWS.pack_into(self._buf, at, x.data_ptr(), out.data_ptr(), heads, a[0], a[1], b[0], b[1])
        return self._at + at

    def append(self, k, v, table, lengths, offsets=None, *, positions=None, q=None, q_out=None, cuda_stream=None):
        """Puts the batch's new keys (rotated, where the cache has a rotary) and values into their pages; lengths count them
        already. With q, its rotated copy is returned (in q_out, which may be q)."""
        n, rotary, index = k.shape[0], self.rotary, self._index
        if (k.requires_grad or v.requires_grad or (q is not None and q.requires_grad)) and torch.is_grad_enabled():
            raise ValueError("a cache has no gradient: detach k, v and q, or append under torch.no_grad()")
        kr, vr = self._rows(0, k, self.n_kv_heads, "k"), self._rows(1, v, self.n_kv_heads, "v", n)
        self._batch(table, lengths, offsets, n, 0)
        if (rotary is None) != (positions is None):
            raise ValueError("positions go with a cache that has a rotary")
        qr = at = handle = None
        if rotary is not None:
            handle, at = rotary._h, rotary._positions(positions, n, index)
            if not handle:
                raise ValueError("the cache's rotary is closed")
        if q is not None:
            if rotary is None:
                raise ValueError("q goes with a cache that has a rotary")
            if q_out is None:
                with _allocating(cuda_stream, index):
                    q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
            qr = self._rows(2, q, self.n_heads, "q", n, q_out)
        stream = _raw_stream(index) if cuda_stream is None else _stream_of(cuda_stream, index)
        self._check(self._lib.cofie_kv_append(self._h, self._at, kr, vr, qr, handle, at, stream))
        return q_out if q is not None else None

    def read(self, table, lengths, offsets=None, *, n_tokens=None, out=None, cuda_stream=None):
        """(keys, values) [tokens, kv heads, head_dim] as the cache holds them at the batch's new tokens. With offsets, which
        lie on the device, the count of tokens is the caller's to say: n_tokens, or that of ``out`` (a pair of tensors)."""
        index = self._index
        if out is None:
            if n_tokens is None and offsets is not None:
                raise ValueError("n_tokens or out goes with offsets")
            n = n_tokens if n_tokens is not None else table.shape[0]
            with _allocating(cuda_stream, index):
                out = tuple(torch.empty((n, self.n_kv_heads, self.head_dim), dtype=self.dtype, device=self.device) for _ in range(2))
        k, v = out
        n = k.shape[0]
        for x in (k, v):
            if x.dtype is not self.dtype or x.shape != (n, self.n_kv_heads, self.head_dim) or not x.is_contiguous() or x.get_device() != index:
                raise ValueError(f"out must be contiguous {self.dtype} [tokens, {self.n_kv_heads}, {self.head_dim}] on cuda:{index}")
        self._batch(table, lengths, offsets, n, 0)
        stream = _raw_stream(index) if cuda_stream is None else _stream_of(cuda_stream, index)
        self._check(self._lib.cofie_kv_read(self._h, self._at, k.data_ptr(), v.data_ptr(), stream))
        return k, v

    def attend(self, q, table, lengths, offsets=None, *, max_new=0, mask=None, causal=True, scale=0.0, out=None, lse=None,
               cuda_stream=None):
        """(out, lse) of the batch's new queries over their sequences' cached tokens; out like q, lse fp32 [tokens, heads].
        max_new: at least the largest count of new tokens. It chooses the kernel (with offsets and 0, all tokens are taken
        for one sequence's, and many short sequences run the kernel of long questions). mask: uint8
        [sequences, >= the longest], nonzero where a cached token may be seen. scale 0: head_dim ** -0.5."""
        rows, out, lse = self._asked(q, table, lengths, offsets, max_new, out, lse, cuda_stream)
        at, stride = (None, 0) if mask is None else self._mask(mask, table.shape[0], "mask")
        stream = _raw_stream(self._index) if cuda_stream is None else _stream_of(cuda_stream, self._index)
        rc = self._lib.cofie_kv_attend(self._h, self._at, rows, lse.data_ptr(), at, stride, causal, scale, stream)
        if rc:
            self._check(rc)
        return out, lse

    def _asked(self, q, table, lengths, offsets, max_new, out, lse, cuda_stream):
        """What attend and attend_shared check and pack alike."""
        n, index = q.shape[0], self._index
        if q.requires_grad and torch.is_grad_enabled():
            raise ValueError("attention over a cache has no gradient: detach q, or attend under torch.no_grad()")
        if out is None or lse is None:
            with _allocating(cuda_stream, index):
                out = torch.empty(q.shape, dtype=q.dtype, device=q.device) if out is None else out
                lse = torch.empty((n, self.n_heads), dtype=torch.float32, device=q.device) if lse is None else lse
        r = self._rows(0, q, self.n_heads, "q", None, out)
        self._batch(table, lengths, offsets, n, 1 if offsets is None else max_new)
        if lse.dtype is not torch.float32 or lse.shape != (n, self.n_heads) or not lse.is_contiguous() or lse.get_device() != index:
            raise ValueError(f"lse must be a contiguous float32 tensor [{n}, {self.n_heads}] on cuda:{index}")
        return r, out, lse

    def _mask(self, mask, seqs, what):
        if mask.dtype not in (torch.uint8, torch.bool) or mask.dim() != 2 or mask.shape[0] != seqs or not mask.is_contiguous() \
                or mask.get_device() != self._index:
            raise ValueError(f"{what} must be a contiguous uint8 or bool tensor [{seqs}, tokens] on cuda:{self._index}")
        # a mask of no tokens, which hides them all, may have no address; nothing is read at the one it gets here
        return mask.data_ptr() or self.k_pages.data_ptr(), mask.shape[1]

    def attend_shared(self, q, table, lengths, offsets=None, *, prefix_table, prefix_lengths, groups=None, max_new=0, max_shared=0,
                      mask=None, prefix_mask=None, causal=True, scale=0.0, out=None, lse=None, cuda_stream=None):
        """As attend(), for sequences that share prefixes, each read once for all of them: the answers or questions about
        one stream. table, lengths, mask and causal are those of a sequence's own cached tokens, which come behind its prefix.
        Group g is sequences groups[g] to groups[g + 1] (int32 [groups + 1]; None: one group of all), and its prefix the
        prefix_lengths[g] tokens in the pages prefix_table[g]; sequences of no group have no prefix. max_shared: at least the
        largest count of a group's new tokens together (0: all); it chooses the kernel. prefix_mask: uint8
        [sequences, >= the longest prefix], nonzero where a sequence may see a token of its prefix (its own evidence)."""
        index = self._index
        rows, out, lse = self._asked(q, table, lengths, offsets, max_new, out, lse, cuda_stream)
        at, stride = (None, 0) if mask is None else self._mask(mask, table.shape[0], "mask")
        if prefix_table.dtype is not torch.int32 or prefix_table.get_device() != index or prefix_table.dim() != 2 or not prefix_table.is_contiguous():
            raise ValueError(f"prefix_table must be a contiguous int32 tensor [groups, pages] on cuda:{index}")
        n, width = prefix_table.shape
        if groups is None and n != 1:
            raise ValueError("without groups prefix_table has one row")
        mask_at, mask_stride = (0, 0) if prefix_mask is None else self._mask(prefix_mask, table.shape[0], "prefix_mask")
        prefix_lengths, groups = _int32(prefix_lengths, index, "prefix_lengths", (n,)), 0 if groups is None else _int32(groups, index, "groups", (n + 1,))
        try:
            _PREFIX.pack_into(self._buf, _PREFIX_AT, n, max_shared, width, prefix_table.data_ptr(), prefix_lengths, groups, mask_at, mask_stride)
        except struct.error:
            raise ValueError("max_shared must be a whole number in [0, 2^32)") from None
        stream = _raw_stream(index) if cuda_stream is None else _stream_of(cuda_stream, index)
        rc = self._lib.cofie_kv_attend_shared(self._h, self._at, self._at + _PREFIX_AT, rows, lse.data_ptr(), at, stride, causal, scale, stream)
        if rc:
            self._check(rc)
        return out, lse

    def status(self, cuda_stream=None):
        """Synchronises and raises NGFFError if a kernel met a page, a length or an offset out of range."""
        self._check(self._lib.cofie_kv_status(self._h, _stream_of(cuda_stream, self._index)))

    def close(self):
        if getattr(self, "_h", None):
            self._lib.cofie_kv_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:  # noqa: BLE001 -- interpreter shutdown
            pass
