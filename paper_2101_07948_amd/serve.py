"""Operators that a serving decoder's step needs beside those of ``decode``: norms of queries and
keys with the rotation in the same pass, a cache in 8 bits, attention of a batch that shares a long
prefix (``shared`` of ``BlockCache.attend`` and ``Q8Cache.attend``), and the choice of the next
token.  A ctypes binding over the entry points of ``include/sdnn_serve.h``, which states the
mathematics, layouts and limits; outputs are the caller's tensors and there is no fallback path.

    norm = HeadNorm(q_weight, k_weight, eps=1e-6)
    cache = Q8Cache.empty(pages, kv_heads, 128, block=64)
    cache.append(k, v, pos, seq, table, rope=rope, norm=norm, q=q, q_out=q)
    cache.attend(q, out, pos, seq, table, shared=blocks_in_common)
    sample(logits, u, token, temperature, top_k, top_p, min_p)
"""
from __future__ import annotations

import ctypes
import math
import struct

from . import SdnnError, _torch_mod, decode
from .decode import _check, _dense, _dtype_code, _on_gpu, _rows, _stream_handle, _workspace

# The structs of sdnn_serve.h, packed in native layout.
_NORM = struct.Struct("@PPiid")
_Q8 = struct.Struct("@PPPPPPqiiii")
_SAMPLING = struct.Struct("@PPPP")

_bound = None


def _lib():
    """libsdnn.so with the argument types of these entry points set."""
    global _bound
    if _bound is None:
        L = decode._lib()
        p, s, i32, i64, f32 = ctypes.c_void_p, ctypes.c_char_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
        L.sdnn_norm_rope.argtypes = [s, s, s, s, i32, i32, i32, p, s, s, p]
        L.sdnn_q8_append.argtypes = [s, s, i32, s, s, s, s, s, s, p]
        L.sdnn_q8_read.argtypes = [s, s, i32, s, s, p]
        L.sdnn_q8_attend.argtypes = [s, s, i32, s, s, p, i32, i32, f32, p, p, i64, p]
        L.sdnn_sample.argtypes = [p, i64, i32, i32, i32, p, s, p, p, p, i64, p]
        L.sdnn_q8_attend_floats.argtypes = [s, i32, i32, i32, i32]
        L.sdnn_sample_floats.argtypes = [i32, i32]
        for fn in ("sdnn_norm_rope", "sdnn_q8_append", "sdnn_q8_read", "sdnn_q8_attend", "sdnn_sample"):
            getattr(L, fn).restype = ctypes.c_int
        for fn in ("sdnn_q8_attend_floats", "sdnn_sample_floats"):
            getattr(L, fn).restype = i64
        _bound = L
    return _bound


def _weight(w, name: str):
    """(address, heads or 0 for a row for all heads, head_dim) of a norm's weights."""
    if w is None:
        return 0, 0, None
    torch = _torch_mod()
    _on_gpu(w, name)
    if w.dim() not in (1, 2) or 0 in w.shape:
        raise ValueError(f"{name} has shape {tuple(w.shape)}, expected (head_dim,) or (heads, head_dim)")
    return _dense(w, name, torch.float32, tuple(w.shape)), w.shape[0] if w.dim() == 2 else 0, w.shape[-1]


class HeadNorm:
    """Norms of queries and keys, each head by its root mean square:
    x / sqrt(mean(x ** 2) + eps) * weight, in 32 bits (the mean in 64).  Weights: float32 (head_dim,)
    for all heads or (heads, head_dim); None for 1."""

    def __init__(self, q_weight=None, k_weight=None, eps: float = 1e-6):
        if not 0.0 <= eps < math.inf:
            raise ValueError("eps must be finite and not negative")
        self._weights, self.eps = (q_weight, k_weight), float(eps)
        (pq, self._q_heads, dq), (pk, self._k_heads, dk) = _weight(q_weight, "q_weight"), _weight(k_weight, "k_weight")
        if None not in (dq, dk) and dq != dk:
            raise ValueError(f"weights of heads of {dq} and of {dk} values")
        self._dim = dq if dk is None else dk
        self._packed = _NORM.pack(pq, pk, dq if self._q_heads else 0, dk if self._k_heads else 0, self.eps)

    # What the calls use is fixed with the object (other weights are another HeadNorm).
    q_weight = property(lambda self: self._weights[0])
    k_weight = property(lambda self: self._weights[1])

    def _for(self, head_dim: int, q_heads, k_heads) -> bytes:
        """sdnn_head_norm for rows of these heads."""
        if self._dim not in (None, head_dim):
            raise ValueError(f"the norm's weights are of heads of {self._dim} values, not {head_dim}")
        if self._q_heads and q_heads not in (None, self._q_heads):
            raise ValueError(f"q_weight is of {self._q_heads} heads, not {q_heads}")
        if self._k_heads and k_heads not in (None, self._k_heads):
            raise ValueError(f"k_weight is of {self._k_heads} heads, not {k_heads}")
        return self._packed

    def apply(self, q, q_out, k=None, k_out=None, pos=None, rope=None, stream=None):
        """q_out = q normed, and with `rope` rotated to the positions pos (tokens, int32); the same of
        k with its weights.  Rows (tokens, heads, head_dim); outputs may be their inputs."""
        L, d = _lib(), q.dtype
        if q.dim() != 3:
            raise ValueError("q must be 3-d (tokens, heads, head_dim)")
        T, H, D = q.shape
        pq, po = _rows(q, "q", d, T, H, D), _rows(q_out, "q_out", d, T, H, D)
        pk = pko = kv = None
        if k is not None:
            kv = k.shape[1] if k.dim() == 3 else None
            pk, pko = _rows(k, "k", d, T, kv, D), _rows(k_out, "k_out", d, T, kv, D)
        elif k_out is not None:
            raise ValueError("k_out without k")
        if rope is not None and pos is None:
            raise ValueError("a rotation needs pos")
        code = L.sdnn_norm_rope(pq, po, pk, pko, _dtype_code(d, "q"), T, D,
                                None if pos is None else _dense(pos, "pos", decode._INT32, (T,)), self._for(D, H, kv),
                                None if rope is None else rope._packed, _stream_handle(stream))
        if code:
            raise SdnnError(code, "sdnn_norm_rope")
        return q_out


class Q8Cache:
    """Keys and values of many sequences in pages of `block` tokens, in 8 bits with a scale for every
    token and head.  The tensors are the caller's:
        k_codes (pages, kv_heads, block, head_dim), v_codes (pages, kv_heads, head_dim, block) int8,
        k_scales, v_scales (pages, kv_heads, block) float32,
        means (pages, kv_heads, head_dim) int8, mean_scales (pages, kv_heads) float32, or both None
    (as in BlockCache, for select).  A row with a value that is not finite has the scale NaN: it is read back as
    NaN, and NaN is what tokens that see it get.  Every call takes positions, sequences and the block table as
    BlockCache's do; rows may be of any of the three types, another in each call."""

    def __init__(self, k_codes, v_codes, k_scales, v_scales, means=None, mean_scales=None):
        torch = _torch_mod()
        _on_gpu(k_codes, "k_codes")
        if k_codes.dim() != 4:
            raise ValueError(f"k_codes has shape {tuple(k_codes.shape)}, expected (pages, kv_heads, block, head_dim)")
        pages, heads, block, dim = k_codes.shape
        if (means is None) != (mean_scales is None):
            raise ValueError("means and mean_scales come together")
        self.pages, self.kv_heads, self.block, self.head_dim = pages, heads, block, dim
        at = [_dense(k_codes, "k_codes", torch.int8, (pages, heads, block, dim)),
              _dense(v_codes, "v_codes", torch.int8, (pages, heads, dim, block)),
              _dense(k_scales, "k_scales", torch.float32, (pages, heads, block)),
              _dense(v_scales, "v_scales", torch.float32, (pages, heads, block)), 0, 0]
        self._summaries = None
        if means is not None:
            at[4] = _dense(means, "means", torch.int8, (pages, heads, dim))
            at[5] = _dense(mean_scales, "mean_scales", torch.float32, (pages, heads))
            self._summaries = decode.BlockCache(means=means, mean_scales=mean_scales, block=block)
        self._tensors = k_codes, v_codes, k_scales, v_scales, means, mean_scales
        self._packed = _Q8.pack(*at, pages, heads, dim, block, 0)

    # The calls use the tensors' addresses, which are taken once: the tensors cannot be replaced.
    k_codes = property(lambda self: self._tensors[0])
    v_codes = property(lambda self: self._tensors[1])
    k_scales = property(lambda self: self._tensors[2])
    v_scales = property(lambda self: self._tensors[3])
    means = property(lambda self: self._tensors[4])
    mean_scales = property(lambda self: self._tensors[5])

    @classmethod
    def empty(cls, pages: int, kv_heads: int, head_dim: int, block: int = 64, means: bool = True, device="cuda"):
        """A cache on fresh tensors (their contents are whatever memory held)."""
        torch = _torch_mod()
        i8, f32 = dict(dtype=torch.int8, device=device), dict(dtype=torch.float32, device=device)
        return cls(torch.empty((pages, kv_heads, block, head_dim), **i8),
                   torch.empty((pages, kv_heads, head_dim, block), **i8),
                   torch.empty((pages, kv_heads, block), **f32), torch.empty((pages, kv_heads, block), **f32),
                   torch.zeros((pages, kv_heads, head_dim), **i8) if means else None,
                   torch.zeros((pages, kv_heads), **f32) if means else None)

    _tokens = decode.BlockCache._tokens

    def append(self, k, v, pos, seq, table, rope=None, norm=None, q=None, q_out=None, stream=None):
        """Stores keys and values (tokens, kv_heads, head_dim) in 8 bits, the keys normed by `norm`
        and rotated by `rope` before, and the mean of every block that a token fills; with q, its
        norm and rotation into q_out (which may be q).  The tokens of one sequence are consecutive
        and ascend."""
        L, T, d, D = _lib(), pos.shape[0], k.dtype, self.head_dim
        pk, pv = _rows(k, "k", d, T, self.kv_heads, D), _rows(v, "v", d, T, self.kv_heads, D)
        pq = po = heads = None
        if q is not None:
            pq = _rows(q, "q", d, T, None, D)
            heads = q.shape[1]
            po = _rows(q_out, "q_out", d, T, heads, D)
        _check(L.sdnn_q8_append(self._packed, self._tokens(pos, seq, table), _dtype_code(d, "k"), pk, pv,
                                None if norm is None else norm._for(D, heads, self.kv_heads),
                                None if rope is None else rope._packed, pq, po, _stream_handle(stream)),
               "sdnn_q8_append")

    def read(self, pos, seq, table, k=None, v=None, stream=None):
        """Reads the tokens' keys and values back into k and v (tokens, kv_heads, head_dim; either may
        be None): number times scale, zeros where nothing is."""
        L, T = _lib(), pos.shape[0]
        some = v if k is None else k
        if some is None:
            raise ValueError("k or v is required")
        d = some.dtype
        pk = None if k is None else _rows(k, "k", d, T, self.kv_heads, self.head_dim)
        pv = None if v is None else _rows(v, "v", d, T, self.kv_heads, self.head_dim)
        _check(L.sdnn_q8_read(self._packed, self._tokens(pos, seq, table), _dtype_code(d, "k or v"), pk, pv,
                              _stream_handle(stream)), "sdnn_q8_read")

    def select(self, q, pos, seq, table, chosen, sink: int = 1, local: int = 1, stream=None):
        """The blocks that each token's queries attend to, as BlockCache.select."""
        if self._summaries is None:
            raise ValueError("the cache was made without means")
        return self._summaries.select(q, pos, seq, table, chosen, sink, local, stream)

    def workspace_floats(self, tokens: int, heads: int, blocks: int, shared: int = 0) -> int:
        """Floats of workspace that attend needs (blocks: of a token, chosen.shape[2], or
        table.shape[1] without chosen)."""
        return _lib().sdnn_q8_attend_floats(self._packed, int(tokens), int(heads), int(blocks), int(shared))

    def attend(self, q, out, pos, seq, table, chosen=None, scale: float | None = None, lse=None, workspace=None,
               stream=None, shared: int = 0):
        """out = attention of q (tokens, heads, head_dim) over the cached positions up to each
        token's own, in its chosen blocks (None: all it sees).  scale, lse, workspace, shared: as
        BlockCache.attend, whose order they are in."""
        L, T, d = _lib(), pos.shape[0], q.dtype
        pq = _rows(q, "q", d, T, None, self.head_dim)
        H = q.shape[1]
        po = _rows(out, "out", d, T, H, self.head_dim)
        blocks, pc, shared = table.shape[1], None, int(shared)
        if chosen is not None:
            if shared:
                raise ValueError("a shared prefix is attended to whole: chosen must be None")
            blocks = chosen.shape[-1]
            pc = _dense(chosen, "chosen", decode._INT32, (T, self.kv_heads, blocks))
        pl = None if lse is None else _dense(lse, "lse", decode._FLOAT32, (T, H))
        workspace, pw, nw = _workspace(workspace, lambda: L.sdnn_q8_attend_floats(self._packed, T, H, blocks, shared), q, stream)
        _check(L.sdnn_q8_attend(self._packed, self._tokens(pos, seq, table), _dtype_code(d, "q"), pq, po, pc, blocks,
                                shared, 1.0 / math.sqrt(self.head_dim) if scale is None else scale, pl,
                                pw, nw, _stream_handle(stream)), "sdnn_q8_attend")
        return out


def sample_workspace_floats(rows: int, vocab: int) -> int:
    """Floats of workspace that sample needs."""
    return _lib().sdnn_sample_floats(int(rows), int(vocab))


def sample(logits, u, token, temperature=None, top_k=None, top_p=None, min_p=None, logprob=None, workspace=None,
           stream=None):
    """token (rows, int32) = a token drawn for each row of logits (rows, vocab; rows may lie apart) by
    u (rows, float32, from [0, 1)): the first whose probability, summed by index over the tokens that
    the limits keep, exceeds u.  For each row: temperature (float32; 0: the largest logit), top_k (int32;
    0: all), top_p and min_p (float32; 1 and 0: all), None for all rows the same way.  logprob (rows,
    float32) receives the logarithm of the token's probability among those kept; a row without a finite
    logit gets token -1.  workspace: a float32 tensor of sample_workspace_floats(...) (allocated here
    when None)."""
    L = _lib()
    try:
        rows, vocab = logits.shape
        by_row, by_token = logits.stride()
    except (AttributeError, ValueError):
        _on_gpu(logits, "logits")
        raise ValueError(f"logits has shape {tuple(logits.shape)}, expected (rows, vocab)") from None
    _on_gpu(logits, "logits")
    if by_token != 1 and vocab > 1:
        raise ValueError("logits: the values of a row must be contiguous")
    f32, i32 = decode._FLOAT32, decode._INT32
    at = [0 if t is None else _dense(t, name, dtype, (rows,)) for t, name, dtype in
          ((temperature, "temperature", f32), (top_k, "top_k", i32), (top_p, "top_p", f32), (min_p, "min_p", f32))]
    pu, pt = _dense(u, "u", f32, (rows,)), _dense(token, "token", i32, (rows,))
    pl = None if logprob is None else _dense(logprob, "logprob", f32, (rows,))
    workspace, pw, nw = _workspace(workspace, lambda: L.sdnn_sample_floats(rows, vocab), logits, stream)
    _check(L.sdnn_sample(logits.data_ptr(), by_row, _dtype_code(logits.dtype, "logits"), rows, vocab, pu,
                         _SAMPLING.pack(*at), pt, pl, pw, nw, _stream_handle(stream)), "sdnn_sample")
    return token
