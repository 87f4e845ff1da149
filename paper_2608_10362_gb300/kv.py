"""A layer's cache and what reads and writes it: KVCache, op_kv_append, op_kv_read,
op_attention (memspec_ops.h).  Beside op_linear these make up a layer up to its O projection.

As in engine.py the wrappers look their arguments over in one expression, and only where that
is not satisfied piece by piece for the error.
"""
from __future__ import annotations

import ctypes as C
import functools

import torch

from . import _lib
from .engine import _BF16, _F32, _I32, _call_on, _check, _cuda_arg, _new, _new_result, _rows_arg, _used_on

_I8 = torch.int8


def _strides(t: torch.Tensor) -> tuple:
    """Strides of the first three dimensions, with 0 where there is but one place."""
    return tuple(s if n > 1 else 0 for n, s in zip(t.shape[:3], t.stride()))


class KVCache:
    """Keys and values of one layer, [sequences][kv heads][positions][head_dim] (64 or 128;
    the last dimension without gaps, the others at any stride of 16 bytes): bf16, or int8
    codes with fp32 scales [sequences][kv heads][positions] of k and of v.  The tensors are
    the caller's, the object keeps them; a slice of some sequences is a KVCache of its own."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, k_scale: torch.Tensor | None = None,
                 v_scale: torch.Tensor | None = None):
        codes = k_scale is not None
        if codes != (v_scale is not None):
            raise ValueError("a cache has scales of both k and v, or of none")
        kinds = [("k", k, _I8 if codes else _BF16, 4), ("v", v, _I8 if codes else _BF16, 4)]
        if codes:
            kinds += [("k_scale", k_scale, _F32, 3), ("v_scale", v_scale, _F32, 3)]
        for name, t, dtype, dims in kinds:
            _cuda_arg(name, t, dtype, like=k)
            if t.dim() != dims or t.numel() == 0:
                raise ValueError(f"{name} must have {dims} dimensions and not be empty, not {list(t.shape)}")
            if tuple(t.shape) != tuple(k.shape[:dims]):
                raise ValueError(f"{name} must be {list(k.shape[:dims])}, not {list(t.shape)}")
            if max(t.shape) >= 1 << 31:
                raise ValueError(f"{name} is too large: {list(t.shape)}")
        if k.stride(3) != 1 or v.stride(3) != 1:
            raise ValueError("the elements of a vector of k and v must be contiguous")
        if _strides(k) != _strides(v) or codes and _strides(k_scale) != _strides(v_scale):
            raise ValueError("k and v must have the same strides, and so must their scales")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.codes, self.device, self.dev = codes, k.device, k.get_device()
        self.n_seq, self.n_heads, self.max_pos, self.head_dim = k.shape
        self.tensors = (k, v, k_scale, v_scale)
        self.c = _lib.Kv(k.data_ptr(), v.data_ptr(), k_scale.data_ptr() if codes else None,
                         v_scale.data_ptr() if codes else None, *_strides(k),
                         *(_strides(k_scale) if codes else (0, 0, 0)), *k.shape)
        self.ref, self.pointer = C.byref(self.c), C.pointer(self.c)
        self.sizes = (*k.shape, codes)

    @classmethod
    def zeros(cls, n_seq: int, n_heads: int, max_pos: int, head_dim: int, dtype=_BF16, device="cuda") -> "KVCache":
        """A new cache of bf16, or (dtype int8) of codes."""
        if dtype not in (_BF16, _I8):
            raise ValueError(f"a cache is of bfloat16 or int8, not {dtype}")
        shape = (n_seq, n_heads, max_pos, head_dim)
        make = lambda *a, **kw: torch.zeros(*a, device=device, **kw)
        kv = [make(shape, dtype=dtype), make(shape, dtype=dtype)]
        return cls(*kv, *([make(shape[:3]), make(shape[:3])] if dtype is _I8 else []))


def op_rope_table(positions: int, head_dim: int, base: float = 10000.0, device="cuda",
                  stream: torch.cuda.Stream | None = None) -> torch.Tensor:
    """cos and sin of pos * base^(-2i/head_dim): fp32 [2][positions][head_dim/2], angles in 64 bits."""
    lib = _lib.load()
    device = torch.device(device)
    if device.type != "cuda":
        raise ValueError(f"the table is made on a CUDA device, not {device}")
    if not 1 <= positions < 1 << 31 or not 2 <= head_dim <= 1024 or head_dim % 2:
        raise ValueError("positions must be at least 1, head_dim even in 2..1024")
    table = _new_result(stream, 2, positions, head_dim // 2, dtype=_F32, device=device)
    st = _call_on(table.get_device(), stream, lib.memspec_op_rope_table, positions, head_dim, base, table.data_ptr())
    if st:
        _check(lib, st)
    return table


def _batch(starts: torch.Tensor, lens: torch.Tensor, cache: KVCache, rows: int) -> _lib.Batch:
    if not isinstance(cache, KVCache):
        raise ValueError("cache must be a KVCache")
    n, dev = lens.numel() if isinstance(lens, torch.Tensor) else 0, cache.dev
    if not (isinstance(starts, torch.Tensor) and 0 < n <= cache.n_seq and starts.numel() == n + 1 and starts.dtype is _I32
            and lens.dtype is _I32 and starts.get_device() == dev and lens.get_device() == dev and starts.dim() == 1
            and lens.dim() == 1 and starts.is_contiguous() and lens.is_contiguous() and 0 < rows < 1 << 31):
        _cuda_arg("lens", lens, _I32, (n,), cache.k)
        _cuda_arg("starts", starts, _I32, (n + 1,), cache.k)
        raise ValueError(f"{n} sequences of {rows} rows for a cache of {cache.n_seq}")
    return _lib.Batch(starts.data_ptr(), lens.data_ptr(), n, rows)


def op_kv_append(qkv: torch.Tensor, cache: KVCache, starts: torch.Tensor, lens: torch.Tensor, n_heads: int,
                 rope: torch.Tensor | None = None, offsets: torch.Tensor | None = None, prefix_len: int = 0,
                 q_gain: torch.Tensor | None = None, k_gain: torch.Tensor | None = None, eps: float = 1e-5,
                 q: torch.Tensor | None = None, stream: torch.cuda.Stream | None = None) -> torch.Tensor:
    """The rows of a Q/K/V projection (fp32 or bf16 [rows][n_heads + 2 kv heads, of head_dim]) into
    queries (the result, bf16 [rows][n_heads][head_dim]) and into the cache, at the end of each
    sequence: rows starts[b]..starts[b+1]-1 (int32 [sequences + 1]) take the last slots of lens[b]
    (int32).  q and k are normalised with gains (bf16 [head_dim], None: not) and rotated with
    op_rope_table's table (None: not) at position prefix_len + first own slot + offset (int32 [rows];
    None: the row's place), see memspec_op_kv_append."""
    lib = _lib.load()
    if not isinstance(qkv, torch.Tensor) or qkv.dtype is not _F32 and qkv.dtype is not _BF16:
        raise ValueError("qkv must be a float32 or bfloat16 tensor")
    rows = qkv.shape[0] if qkv.dim() == 2 else 0
    b = _batch(starts, lens, cache, rows)
    dev, hd, width = cache.dev, cache.head_dim, (n_heads + 2 * cache.n_heads) * cache.head_dim
    if qkv.is_contiguous() and qkv.get_device() == dev:
        ld = width
    else:
        ld = _rows_arg("qkv", qkv, qkv.dtype, cache.k)
    if n_heads < 1 or qkv.shape[1] != width:
        raise ValueError(f"qkv must have {n_heads} + 2 * {cache.n_heads} heads of {hd}, not {qkv.shape[1]} columns")
    positions = 0
    if rope is not None:
        positions = rope.shape[1] if isinstance(rope, torch.Tensor) and rope.dim() == 3 else 0
        if not (0 < positions < 1 << 31 and rope.numel() == positions * hd and rope.shape[0] == 2 and rope.dtype is _F32
                and rope.get_device() == dev and rope.is_contiguous()):
            if not 0 < positions < 1 << 31:
                raise ValueError("rope must be op_rope_table's")
            _cuda_arg("rope", rope, _F32, (2, positions, hd // 2), qkv)
    if offsets is not None:
        _cuda_arg("offsets", offsets, _I32, (rows,), qkv)
    if (q_gain is None) != (k_gain is None):
        raise ValueError("gains of both q and k, or of none")
    if q_gain is not None:
        _cuda_arg("q_gain", q_gain, _BF16, (hd,), qkv)
        _cuda_arg("k_gain", k_gain, _BF16, (hd,), qkv)
    if not 0 <= prefix_len < 1 << 31:
        raise ValueError(f"prefix_len must be from 0 to 2^31 - 1, not {prefix_len!r}")
    if q is None:
        q = _new_result(stream, rows, n_heads, hd, dtype=_BF16, device=cache.device)
    else:
        _cuda_arg("q", q, _BF16, (rows, n_heads, hd), qkv)
    if stream is not None:
        _used_on(stream, qkv, *cache.tensors, starts, lens, rope, offsets, q_gain, k_gain, q)
    a = _lib.Append(qkv.data_ptr(), _lib.F32 if qkv.dtype is _F32 else _lib.BF16, n_heads, ld,
                    None if rope is None else rope.data_ptr(), positions, prefix_len,
                    None if offsets is None else offsets.data_ptr(), None if q_gain is None else q_gain.data_ptr(),
                    None if k_gain is None else k_gain.data_ptr(), eps, q.data_ptr())
    st = _call_on(dev, stream, lib.memspec_op_kv_append, C.byref(b), cache.ref, C.byref(a))
    if st:
        _check(lib, st)
    return q


def op_kv_read(cache: KVCache, starts: torch.Tensor, lens: torch.Tensor, rows: int, k: torch.Tensor | None = None,
               v: torch.Tensor | None = None, stream: torch.cuda.Stream | None = None):
    """(k, v), bf16 [rows][kv heads][head_dim] each: what the cache holds at the rows' slots (as in
    op_kv_append).  With starts = 0, lens a whole sequence is read."""
    lib = _lib.load()
    b = _batch(starts, lens, cache, rows)
    if rows < 1:
        raise ValueError(f"rows must be at least 1, not {rows!r}")
    shape = (rows, cache.n_heads, cache.head_dim)
    if k is None:
        k = _new_result(stream, *shape, dtype=_BF16, device=cache.device)
    else:
        _cuda_arg("k", k, _BF16, shape, cache.k)
    if v is None:
        v = _new_result(stream, *shape, dtype=_BF16, device=cache.device)
    else:
        _cuda_arg("v", v, _BF16, shape, cache.k)
    if stream is not None:
        _used_on(stream, *cache.tensors, starts, lens, k, v)
    st = _call_on(cache.dev, stream, lib.memspec_op_kv_read, C.byref(b), cache.ref, k.data_ptr(), v.data_ptr())
    if st:
        _check(lib, st)
    return k, v


def _of_sizes(sizes: tuple) -> _lib.Kv:
    """A cache of these sizes, with addresses that only a size's check looks at."""
    n_seq, n_heads, max_pos, hd, codes = sizes
    at = 1 << 8
    return _lib.Kv(at, at, at if codes else None, at if codes else None, 0, 0, hd, 0, 0, 1, n_seq, n_heads, max_pos, hd)


@functools.lru_cache(maxsize=512)
def _attention_scratch_bytes(sizes: tuple, n_seq: int, rows: int, n_heads: int, max_rows: int, prefix: tuple | None,
                             prefix_len: int) -> int:
    lib = _lib.load()
    at, nb = 1 << 8, C.c_size_t()
    kv, b = _of_sizes(sizes), _lib.Batch(at, at, n_seq, rows)
    p = None if prefix is None else C.pointer(_of_sizes(prefix))
    a = _lib.Attention(at, 0, at, 0, n_heads, 1.0, None, p, prefix_len, max_rows)
    _check(lib, lib.memspec_op_attention_scratch_bytes(C.byref(b), C.byref(kv), C.byref(a), C.byref(nb)))
    return nb.value


def _heads_arg(name: str, t: torch.Tensor, like: torch.Tensor) -> int:
    """bf16 [rows][heads][head_dim] with whole rows without gaps; the row stride."""
    _cuda_arg(name, t, _BF16, like=like)
    if t.dim() != 3 or t.numel() == 0:
        raise ValueError(f"{name} must be [rows][heads][head_dim] and not empty, not {list(t.shape)}")
    rows, heads, hd = t.shape
    if (hd > 1 and t.stride(2) != 1) or (heads > 1 and t.stride(1) != hd) or rows > 1 and t.stride(0) < heads * hd:
        raise ValueError(f"{name}'s rows must be contiguous and not overlap (strides {t.stride()})")
    return t.stride(0) if rows > 1 else heads * hd


def op_attention(q: torch.Tensor, cache: KVCache, starts: torch.Tensor, lens: torch.Tensor, max_rows: int | None = None,
                 scale: float | None = None, tree: torch.Tensor | None = None, prefix: KVCache | None = None,
                 prefix_len: int | None = None, out: torch.Tensor | None = None, scratch: torch.Tensor | None = None,
                 stream: torch.cuda.Stream | None = None) -> torch.Tensor:
    """Attention of the rows of q (bf16 [rows][heads][head_dim], rows at any stride of 8) over the
    cache: bf16 [rows][heads][head_dim].  Row j of sequence b (starts and lens as in op_kv_append,
    the rows' own keys already in the cache) sees the slots up to its own; with `tree` (int32 [rows])
    those before the sequence's rows and, of the rows', those whose bit is set.  `prefix` is a cache
    whose first sequence, up to prefix_len (default: all of it), is before every sequence's slots; it is
    read once for the whole batch.  scale: of q . k, 1 / sqrt(head_dim) by default; max_rows: the
    most rows that a sequence has (default: all rows).  It chooses the kernel, and with it roundings; name it for a batch
    of short sequences, which the kernel for many rows serves at up to twice the time.
    ``scratch`` (any content) of memspec_op_attention_scratch_bytes bytes saves an allocation."""
    lib = _lib.load()
    if not isinstance(q, torch.Tensor) or q.dim() != 3:
        raise ValueError("q must be a CUDA tensor [rows][heads][head_dim]")
    rows, n_heads, hd = q.shape
    b = _batch(starts, lens, cache, rows)
    dev = cache.dev
    if q.is_contiguous() and q.dtype is _BF16 and q.get_device() == dev:
        ldq = n_heads * hd
    else:
        ldq = _heads_arg("q", q, cache.k)
    if hd != cache.head_dim or n_heads < 1 or n_heads % cache.n_heads:
        raise ValueError(f"q's heads must be of {cache.head_dim}, a multiple of {cache.n_heads}, not {list(q.shape)}")
    if max_rows is None:
        max_rows = rows
    if not 1 <= max_rows <= rows:
        raise ValueError(f"max_rows must be in 1..{rows}, not {max_rows!r}")
    if tree is not None:
        _cuda_arg("tree", tree, _I32, (rows,), cache.k)
    if prefix is None:
        if prefix_len:
            raise ValueError("prefix_len without a prefix")
    elif not isinstance(prefix, KVCache) or prefix.dev != dev:
        raise ValueError(f"prefix must be a KVCache on {cache.device}")
    elif prefix_len is None:
        prefix_len = prefix.max_pos
    elif not 0 <= prefix_len <= prefix.max_pos:
        raise ValueError(f"prefix_len must be in 0..{prefix.max_pos}, not {prefix_len!r}")
    if out is None:
        out = _new_result(stream, rows, n_heads, hd, dtype=_BF16, device=cache.device)
        ldo = n_heads * hd
    else:
        ldo = _heads_arg("out", out, cache.k)
        if out.shape != q.shape:
            raise ValueError(f"out must be {list(q.shape)}, not {list(out.shape)}")
    a = _lib.Attention(q.data_ptr(), ldq, out.data_ptr(), ldo, n_heads, hd ** -0.5 if scale is None else scale,
                       None if tree is None else tree.data_ptr(), None if prefix is None else prefix.pointer,
                       prefix_len or 0, max_rows)
    if scratch is None:
        nb = _attention_scratch_bytes(cache.sizes, b.n_seq, rows, n_heads, max_rows,
                                      None if prefix is None else prefix.sizes, prefix_len or 0)
        scratch = _new(stream, torch.empty, nb, dtype=torch.uint8, device=cache.device)
    elif not isinstance(scratch, torch.Tensor) or scratch.get_device() != dev or not scratch.is_contiguous():
        raise ValueError(f"scratch must be contiguous on {q.device}")
    if stream is not None:
        _used_on(stream, q, *cache.tensors, starts, lens, tree, *(() if prefix is None else prefix.tensors), out, scratch)
    st = _call_on(dev, stream, lib.memspec_op_attention, C.byref(b), cache.ref, C.byref(a), scratch.data_ptr(),
                  scratch.nbytes)
    if st:
        _check(lib, st)
    return out
