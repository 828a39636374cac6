"""Operators of a decoder's step between the sparse products: rotary positions, a paged cache
with a summary for each block, the choice of blocks by it, attention over the chosen blocks, and
products with 4-bit weights.  A ctypes binding over the entry points of
``include/sdnn_decode.h``, which states the mathematics, layouts and limits; as with ``Plan``,
outputs are the caller's tensors and there is no fallback path.

    rope = Rope(128, base=10000.0)
    cache = BlockCache.empty(pages, kv_heads, 128, block=64, dtype=torch.bfloat16)
    cache.append(k, v, pos, seq, table, rope=rope, q=q, q_out=q)    # rotate, store, summarise
    cache.select(q, pos, seq, table, chosen, sink=1, local=2)       # blocks for each token
    cache.attend(q, out, pos, seq, table, chosen)
    Q4Plan(packed, scales, K=K, group=64).matvec(x, y, bias, "gelu")
"""
from __future__ import annotations

import ctypes
import math
import struct

import numpy as np

from . import EPI, SdnnError, _torch_mod, lib

LAYOUTS = {"half": 0, "interleaved": 1}

# The structs of sdnn_decode.h, packed in native layout.
_CACHE = struct.Struct("@PPPPqiiii")
_TOKENS = struct.Struct("@PPPiiii")
_HEADS = struct.Struct("@Pqqii")
_ROTATION = struct.Struct("@Piid")

# Set with the library, at the first call: its handle, the types' codes, torch's types and accessors (each call of
# these operators is a few microseconds: looked up by name they would be a good part of it).
_bound = _codes = _INT32 = _FLOAT32 = _raw_stream = _device = None


def _lib():
    """libsdnn.so with the argument types of these entry points set."""
    global _bound, _codes, _INT32, _FLOAT32, _raw_stream, _device
    if _bound is None:
        L, torch = lib(), _torch_mod()
        _codes = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
        _INT32, _FLOAT32 = torch.int32, torch.float32
        _raw_stream, _device = torch._C._cuda_getCurrentRawStream, torch.cuda.current_device
        if hasattr(torch._C, "_cuda_getDevice"):  # what current_device calls once the GPU is in use
            _device = torch._C._cuda_getDevice
        p, s, i32, i64 = ctypes.c_void_p, ctypes.c_char_p, ctypes.c_int32, ctypes.c_int64
        L.sdnn_rope.argtypes = [s, s, i32, i32, i32, p, s, i32, p]
        L.sdnn_cache_append.argtypes = [s, s, s, s, s, s, s, p]
        L.sdnn_block_select.argtypes = [s, s, s, i32, i32, i32, p, p]
        L.sdnn_block_attend.argtypes = [s, s, s, s, p, i32, ctypes.c_float, p, p, i64, p]
        L.sdnn_block_attend_floats.argtypes = [s, i32, i32, i32]
        L.sdnn_block_attend_floats.restype = i64
        L.sdnn_block_attend_shared.argtypes = [s, s, s, s, i32, ctypes.c_float, p, p, i64, p]
        L.sdnn_block_attend_shared.restype = ctypes.c_int
        L.sdnn_block_attend_shared_floats.argtypes = [s, i32, i32, i32, i32]
        L.sdnn_block_attend_shared_floats.restype = i64
        L.sdnn_qmat_create.argtypes = [p, p, i32, p, i32, i32, i32, p, ctypes.POINTER(p)]
        L.sdnn_qmat_apply.argtypes = [p, p, i64, i64, p, i64, i64, i32, i32, p, i32, p]
        L.sdnn_qmat_destroy.argtypes = [p]
        L.sdnn_qmat_destroy.restype = None
        for fn in ("sdnn_rope", "sdnn_cache_append", "sdnn_block_select", "sdnn_block_attend",
                   "sdnn_qmat_create", "sdnn_qmat_apply"):
            getattr(L, fn).restype = ctypes.c_int
        _bound = L
    return _bound


def _stream_handle(stream) -> int:
    """The raw hipStream_t of `stream` (default: the current stream)."""
    return _raw_stream(_device()) if stream is None else stream.cuda_stream


def _dtype_code(dtype, name: str) -> int:
    """sdnn_dtype of a torch dtype."""
    code = _codes.get(dtype)
    if code is None:
        raise TypeError(f"{name} must be float32, float16 or bfloat16, not {dtype}")
    return code


def _on_gpu(t, name: str):
    if not isinstance(t, _torch_mod().Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA/HIP torch tensor")


def _dense(t, name: str, dtype, shape) -> int:
    """Device address of a contiguous tensor of the given type and shape (checked on a fast path;
    the slow path only builds the error message)."""
    try:
        if t.is_cuda and t.dtype is dtype and t.shape == shape and t.is_contiguous():
            return t.data_ptr()
    except AttributeError:
        pass
    _on_gpu(t, name)
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, not {t.dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    raise ValueError(f"{name} must be contiguous")


def _rows(t, name: str, dtype, tokens: int, heads, head_dim: int) -> bytes:
    """sdnn_heads of a (tokens, heads, head_dim) tensor; any strides but the last's."""
    try:
        T, H, D = t.shape
        by_token, by_head, by_value = t.stride()
        if t.is_cuda and t.dtype is dtype and T == tokens and D == head_dim and (heads is None or heads == H) and \
                (by_value == 1 or D == 1):
            return _HEADS.pack(t.data_ptr(), by_token, by_head, H, 0)
    except (AttributeError, ValueError):
        pass
    _on_gpu(t, name)
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, not {t.dtype}")
    want = (tokens, "heads" if heads is None else heads, head_dim)
    if t.dim() != 3 or t.shape[0] != tokens or t.shape[2] != head_dim or heads not in (None, t.shape[1]):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {want}")
    raise ValueError(f"{name}: the values of a head must be contiguous")


def _check(code: int, where: str):
    if code:
        raise SdnnError(code, where)


def _workspace(workspace, need, like, stream):
    """(tensor, address, floats) of a call's workspace, a contiguous float32 tensor; with None need() floats are
    allocated.  The caller keeps the tensor until its kernels are launched."""
    if workspace is None:
        n = need()
        if not n:
            return None, None, 0
        # of the memory of the stream that uses it: that of the current stream may still be in use there
        torch = _torch_mod()
        with torch.cuda.stream(stream):  # (None: the current stream)
            workspace = torch.empty(n, dtype=torch.float32, device=like.device)
    n = workspace.numel()
    return workspace, _dense(workspace, "workspace", _FLOAT32, (n,)), n


def rope_frequencies(rotated: int, base: float = 10000.0, scaling: str | None = None,
                     factor: float = 1.0, length: int = 0, turns=(1.0, 32.0)) -> np.ndarray:
    """Radians per position of the rotated / 2 pairs: base ** (-2 i / rotated), scaled for
    contexts `factor` times as long as the `length` positions a model was trained on:
      "linear": every frequency divided by factor (positions are squeezed),
      "base":   base * factor ** (rotated / (rotated - 2)) in base's place (the slowest pair is
                divided by factor, the fastest is kept),
      "bands":  a pair that makes fewer than turns[0] turns over `length` is divided by factor,
                one that makes more than turns[1] is kept, a linear mix between."""
    if rotated < 2 or rotated % 2:
        raise ValueError("rotated must be an even number of values, at least 2")
    if factor <= 0 or base <= 0:
        raise ValueError("base and factor must be positive")
    i = np.arange(0, rotated, 2, dtype=np.float64) / rotated
    if scaling == "base":
        if rotated == 2:
            raise ValueError("scaling by the base needs at least two pairs")
        base = base * factor ** (rotated / (rotated - 2))
    freq = base ** -i
    if scaling == "linear":
        return freq / factor
    if scaling == "bands":
        lo, hi = turns
        if length <= 0 or not lo < hi:
            raise ValueError("scaling in bands needs the trained length and turns = (low, high)")
        keep = np.clip((length * freq / (2 * math.pi) - lo) / (hi - lo), 0.0, 1.0)
        return freq * (keep + (1.0 - keep) / factor)
    if scaling not in (None, "base"):
        raise ValueError(f"unknown scaling {scaling!r}")
    return freq


class Rope:
    """A rotation of the first `rotated` values of every head.  `frequencies` (radians per
    position, a tensor or array of rotated / 2) replaces what rope_frequencies gives."""

    def __init__(self, rotated: int | None = None, base: float = 10000.0, layout: str = "half",
                 scaling: str | None = None, factor: float = 1.0, length: int = 0,
                 turns=(1.0, 32.0), amplitude: float = 1.0, frequencies=None, device="cuda"):
        torch = _torch_mod()
        if frequencies is None:
            if rotated is None:
                raise ValueError("rotated or frequencies is required")
            frequencies = rope_frequencies(rotated, base, scaling, factor, length, turns)
        freq = torch.as_tensor(frequencies, dtype=torch.float64, device=device).contiguous()
        if freq.dim() != 1 or (rotated is not None and freq.numel() * 2 != rotated):
            raise ValueError("frequencies must hold one value for each rotated pair")
        _on_gpu(freq, "frequencies")  # (the kernels read them)
        self._freq, self._layout = freq, layout
        self._packed = _ROTATION.pack(freq.data_ptr(), freq.numel(), LAYOUTS[layout], float(amplitude))

    # What the calls use is fixed with the object (another rotation is another Rope).
    freq = property(lambda self: self._freq, doc="The frequencies (float64, on the device).")
    layout = property(lambda self: self._layout)

    def apply(self, x, y, pos, inverse: bool = False, stream=None):
        """y = x (tokens, heads, head_dim) rotated to the positions pos (tokens, int32); by the
        negative angles with inverse (which is also the gradient).  y may be x."""
        L, d, shape = _lib(), x.dtype, x.shape
        if len(shape) != 3:
            raise ValueError("x must be 3-d (tokens, heads, head_dim)")
        T, H, D = shape
        code = L.sdnn_rope(_rows(x, "x", d, T, H, D), _rows(y, "y", d, T, H, D), _dtype_code(d, "x"), T, D,
                           _dense(pos, "pos", _INT32, (T,)), self._packed, 1 if inverse else 0,
                           _stream_handle(stream))
        if code:
            raise SdnnError(code, "sdnn_rope")
        return y


class BlockCache:
    """Keys and values of many sequences in pages of `block` tokens, with an 8-bit mean of the
    keys of every full block.  The tensors are the caller's:
        k_pages (pages, kv_heads, block, head_dim), v_pages (pages, kv_heads, head_dim, block),
        means (pages, kv_heads, head_dim) int8, mean_scales (pages, kv_heads) float32;
    those a program's calls do not use may be None; a cache on other tensors is another
    BlockCache.  Every call takes the tokens' positions
    pos and sequences seq (tokens, int32) and the block table (sequences, blocks, int32): the
    page of each sequence's blocks.  A token with pos < 0 is a filler: nothing is stored for it
    and its outputs are zero.  Kernels are chosen by a call's sizes: prompts and single tokens
    belong in calls of their own, a prompt's with its own sequences' rows of the table alone."""

    def __init__(self, k_pages=None, v_pages=None, means=None, mean_scales=None, block: int | None = None):
        torch = _torch_mod()
        if k_pages is not None:
            pages, heads, blk, dim = k_pages.shape
            if block not in (None, blk):
                raise ValueError(f"k_pages holds blocks of {blk} tokens, not {block}")
        elif means is not None and block is not None:
            (pages, heads, dim), blk = means.shape, block
        else:
            raise ValueError("k_pages, or means and block, is required")
        self.pages, self.kv_heads, self.block, self.head_dim = pages, heads, int(blk), dim
        self.dtype = None if k_pages is None else k_pages.dtype
        if (k_pages is None) != (v_pages is None) or (means is None) != (mean_scales is None):
            raise ValueError("k_pages and v_pages, means and mean_scales come together")
        at = [0, 0, 0, 0]
        if k_pages is not None:
            at[0] = _dense(k_pages, "k_pages", self.dtype, (pages, heads, blk, dim))
            at[1] = _dense(v_pages, "v_pages", self.dtype, (pages, heads, dim, blk))
        if means is not None:
            at[2] = _dense(means, "means", torch.int8, (pages, heads, dim))
            at[3] = _dense(mean_scales, "mean_scales", torch.float32, (pages, heads))
        self._tensors = k_pages, v_pages, means, mean_scales
        self._at, self._packed = at, {}

    # The calls use the tensors' addresses, which are taken once: the tensors cannot be replaced.
    k_pages = property(lambda self: self._tensors[0])
    v_pages = property(lambda self: self._tensors[1])
    means = property(lambda self: self._tensors[2])
    mean_scales = property(lambda self: self._tensors[3])

    @classmethod
    def empty(cls, pages: int, kv_heads: int, head_dim: int, block: int = 64, dtype=None, device="cuda"):
        """A cache on fresh tensors (their contents are whatever memory held)."""
        torch = _torch_mod()
        dtype = torch.bfloat16 if dtype is None else dtype
        return cls(torch.empty((pages, kv_heads, block, head_dim), dtype=dtype, device=device),
                   torch.empty((pages, kv_heads, head_dim, block), dtype=dtype, device=device),
                   torch.zeros((pages, kv_heads, head_dim), dtype=torch.int8, device=device),
                   torch.zeros((pages, kv_heads), dtype=torch.float32, device=device))

    def _struct(self, dtype) -> bytes:
        s = self._packed.get(dtype)
        if s is None:
            s = self._packed[dtype] = _CACHE.pack(*self._at, self.pages, self.kv_heads, self.head_dim,
                                                  self.block, _dtype_code(dtype, "the cache"))
        return s

    def _tokens(self, pos, seq, table) -> bytes:
        T = pos.shape[0]
        S, blocks = table.shape
        return _TOKENS.pack(_dense(pos, "pos", _INT32, (T,)), _dense(seq, "seq", _INT32, (T,)),
                            _dense(table, "table", _INT32, (S, blocks)), T, S, blocks, 0)

    def _need(self, what: str):
        if getattr(self, what) is None:
            raise ValueError(f"the cache was made without {what}")

    def append(self, k, v, pos, seq, table, rope: Rope | None = None, q=None, q_out=None, stream=None):
        """Stores keys and values (tokens, kv_heads, head_dim), the keys rotated by `rope`, and
        the mean of every block that a token fills; with q, rotates the queries into q_out (which
        may be q).  The tokens of one sequence are consecutive and ascend."""
        self._need("k_pages")
        L, T, d = _lib(), pos.shape[0], self.dtype
        pk = _rows(k, "k", d, T, self.kv_heads, self.head_dim)
        pv = _rows(v, "v", d, T, self.kv_heads, self.head_dim)
        pq = po = None
        if q is not None:
            pq = _rows(q, "q", d, T, None, self.head_dim)
            po = _rows(q_out, "q_out", d, T, q.shape[1], self.head_dim)
        _check(L.sdnn_cache_append(self._struct(d), self._tokens(pos, seq, table), pk, pv,
                                   None if rope is None else rope._packed, pq, po,
                                   _stream_handle(stream)), "sdnn_cache_append")

    def select(self, q, pos, seq, table, chosen, sink: int = 1, local: int = 1, stream=None):
        """Writes to chosen (tokens, kv_heads, blocks; int32) the blocks that each token's queries
        (tokens, heads, head_dim) attend to: the first `sink`, the last `local` and those with the
        largest scores, ascending, then -1."""
        self._need("means")
        L, d = _lib(), q.dtype if self.dtype is None else self.dtype
        T, blocks = pos.shape[0], chosen.shape[-1]
        pq = _rows(q, "q", d, T, None, self.head_dim)
        pc = _dense(chosen, "chosen", _INT32, (T, self.kv_heads, blocks))
        _check(L.sdnn_block_select(self._struct(d), self._tokens(pos, seq, table), pq, blocks,
                                   int(sink), int(local), pc, _stream_handle(stream)), "sdnn_block_select")
        return chosen

    def workspace_floats(self, tokens: int, heads: int, blocks: int, shared: int = 0) -> int:
        """Floats of workspace that attend needs (blocks: of a token, chosen.shape[2], or
        table.shape[1] without chosen)."""
        if shared:
            return _lib().sdnn_block_attend_shared_floats(self._struct(self.dtype), int(tokens), int(heads), int(blocks),
                                                          int(shared))
        return _lib().sdnn_block_attend_floats(self._struct(self.dtype), int(tokens), int(heads), int(blocks))

    def attend(self, q, out, pos, seq, table, chosen=None, scale: float | None = None, lse=None,
               workspace=None, stream=None, shared: int = 0):
        """out = attention of q (tokens, heads, head_dim) over the cached positions up to each
        token's own, in its chosen blocks (None: all it sees).  scale: 1 / sqrt(head_dim) by
        default; lse: float32 (tokens, heads), receives the logarithm of the sums of exponentials;
        workspace: a float32 tensor of workspace_floats(...) (allocated here when None); shared: the
        first blocks of every sequence that are the same pages, which are read once for all (looked up
        in the table's first row; not with chosen)."""
        self._need("k_pages")
        L, T, d = _lib(), pos.shape[0], self.dtype
        pq = _rows(q, "q", d, T, None, self.head_dim)
        H = q.shape[1]
        po = _rows(out, "out", d, T, H, self.head_dim)
        blocks = table.shape[1]
        pc = None
        if chosen is not None:
            if shared:
                raise ValueError("a shared prefix is attended to whole: chosen must be None")
            blocks = chosen.shape[-1]
            pc = _dense(chosen, "chosen", _INT32, (T, self.kv_heads, blocks))
        pl = None if lse is None else _dense(lse, "lse", _FLOAT32, (T, H))
        cache = self._struct(d)
        if shared:
            return self._attend_shared(cache, pq, po, q, out, pos, seq, table, int(shared), scale, pl, workspace, stream)
        workspace, pw, nw = _workspace(workspace, lambda: L.sdnn_block_attend_floats(cache, T, H, blocks), q, stream)
        _check(L.sdnn_block_attend(cache, self._tokens(pos, seq, table), pq, po, pc, blocks,
                                   1.0 / math.sqrt(self.head_dim) if scale is None else scale, pl,
                                   pw, nw, _stream_handle(stream)), "sdnn_block_attend")
        return out

    def _attend_shared(self, cache, pq, po, q, out, pos, seq, table, shared, scale, pl, workspace, stream):
        L = _bound
        T, H, blocks = pos.shape[0], q.shape[1], table.shape[1]
        workspace, pw, nw = _workspace(workspace, lambda: L.sdnn_block_attend_shared_floats(cache, T, H, blocks, shared),
                                       q, stream)
        _check(L.sdnn_block_attend_shared(cache, self._tokens(pos, seq, table), pq, po, shared,
                                          1.0 / math.sqrt(self.head_dim) if scale is None else scale, pl, pw, nw,
                                          _stream_handle(stream)), "sdnn_block_attend_shared")
        return out


class Q4Plan:
    """A matrix of 4-bit weights W[m][k] = scales[m][k // group] * (n - z), laid out once for
    the device; z is 8, or zeros[m][k // group].  packed (M, (K + 1) // 2) uint8 holds column
    2 i in the low half of byte i; scales (M, ceil(K / group)) float32, float16 or bfloat16; zeros
    the same shape, uint8.  All are on the GPU and may be freed afterwards."""

    def __init__(self, packed, scales, zeros=None, K: int | None = None, group: int = 64, stream=None):
        torch = _torch_mod()
        _on_gpu(packed, "packed")
        self.M = packed.shape[0]
        self.K = 2 * packed.shape[1] if K is None else int(K)
        self.group = int(group)
        groups = -(-self.K // self.group) if self.group > 0 else 0
        pp = _dense(packed, "packed", torch.uint8, (self.M, (self.K + 1) // 2))
        _on_gpu(scales, "scales")
        ps = _dense(scales, "scales", scales.dtype, (self.M, groups))
        pz = None if zeros is None else _dense(zeros, "zeros", torch.uint8, (self.M, groups))
        self._h = None
        self._lib = _lib()
        h = ctypes.c_void_p()
        _check(self._lib.sdnn_qmat_create(pp, ps, _dtype_code(scales.dtype, "scales"), pz, self.M, self.K,
                                          self.group, _stream_handle(stream), ctypes.byref(h)),
               "sdnn_qmat_create")
        self._h = h

    @property
    def handle(self):
        if self._h is None:
            raise RuntimeError("plan is closed")
        return self._h

    def matvec(self, x, y, bias=None, epi: str = "none", stream=None):
        """y (M, N) = epi(W @ x + bias) for x (K, N) of the same type, N few; any strides (rows of
        tokens are x.t(), y.t()).  bias: float32 (M,)."""
        d, shape = x.dtype, x.shape
        K, N = shape if len(shape) == 2 else (None, None)
        if K != self.K:
            raise ValueError(f"x has shape {tuple(x.shape)}, expected ({self.K}, N)")
        if y.shape != (self.M, N):
            raise ValueError(f"y has shape {tuple(y.shape)}, expected {(self.M, N)}")
        if y.dtype is not d:
            raise TypeError(f"y must be {d}, not {y.dtype}")
        if not (x.is_cuda and y.is_cuda):
            raise TypeError("x and y must be CUDA/HIP torch tensors")
        pb = None if bias is None else _dense(bias, "bias", _FLOAT32, (self.M,))
        (xf, xc), (yf, yc) = x.stride(), y.stride()
        code = self._lib.sdnn_qmat_apply(self.handle, x.data_ptr(), xf, xc, y.data_ptr(), yf, yc, N,
                                         _dtype_code(d, "x"), pb, EPI[epi], _stream_handle(stream))
        if code:
            raise SdnnError(code, "sdnn_qmat_apply")
        return y

    def close(self):
        if getattr(self, "_h", None) is not None:
            self._lib.sdnn_qmat_destroy(self._h)
            self._h = None

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
