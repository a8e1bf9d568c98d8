"""Torch-facing binding of libeva: marshals device tensors and the current HIP
stream into the C ABI.  Every computation runs in the library's HIP kernels;
this module only checks shapes, allocates outputs with torch and forwards
pointers.  Tensors must live on a ROCm device; there is no CPU path.
"""
import ctypes
import math

import torch

from . import _lib

_DTYPES = {torch.bfloat16: _lib.EVA_BF16, torch.float32: _lib.EVA_F32}


def _dtype_code(t: torch.Tensor) -> int:
    try:
        return _DTYPES[t.dtype]
    except KeyError:
        raise TypeError(f"unsupported dtype {t.dtype}; use bfloat16 or float32") from None


def _require_device(*ts):
    for t in ts:
        if not t.is_cuda:
            raise RuntimeError("EVA kernels run on the GPU only: tensors must be on a ROCm device")
        if not t.is_contiguous():
            raise ValueError("tensors must be contiguous")


def _stream():
    """Handle of the current device's current stream (without the Stream
    object torch.cuda.current_stream() makes: 0.3 us instead of 3)."""
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _ptr(t):
    return t.data_ptr() if t is not None else None


def build_summaries(K: torch.Tensor, V: torch.Tensor, C: int, out=None):
    """Chunk summaries. K, V: [B, Hkv, L, d] -> (Ksum, Vsum): [B, Hkv, L // C, d].
    `out` = (Ksum, Vsum) preallocated, else allocated here."""
    _require_device(K, V)
    B, Hkv, L, d = K.shape
    if out is None:
        Ks = torch.empty(B, Hkv, L // C, d, dtype=K.dtype, device=K.device)
        Vs = torch.empty_like(Ks)
    else:
        Ks, Vs = out
        _require_device(Ks, Vs)
        if tuple(Ks.shape) != (B, Hkv, L // C, d) or Vs.shape != Ks.shape or Ks.dtype != K.dtype:
            raise ValueError("summary buffers must be [B, Hkv, L // C, d] in the input dtype")
    lib = _lib.load()
    _lib.check("eva_build_summaries",
               lib.eva_build_summaries(_ptr(K), _ptr(V), _ptr(Ks), _ptr(Vs), B, Hkv, L, d, C, _dtype_code(K),
                                       _stream()))
    return Ks, Vs


def build_summaries_rf(K: torch.Tensor, V: torch.Tensor, eps: torch.Tensor, C: int, lam: float = 0.1, out=None):
    """Stochastic random-feature summaries.  K, V: [B, Hkv, L, d]; eps: fp32
    [B, Hkv, L // C, d] standard normal draws (one per chunk) -> (Ksum, Vsum)."""
    _require_device(K, V, eps)
    B, Hkv, L, d = K.shape
    if eps.dtype != torch.float32 or tuple(eps.shape) != (B, Hkv, L // C, d):
        raise ValueError("eps must be float32 [B, Hkv, L // C, d]")
    if out is None:
        Ks = torch.empty(B, Hkv, L // C, d, dtype=K.dtype, device=K.device)
        Vs = torch.empty_like(Ks)
    else:
        Ks, Vs = out
    lib = _lib.load()
    _lib.check("eva_build_summaries_rf",
               lib.eva_build_summaries_rf(_ptr(K), _ptr(V), _ptr(eps), float(lam), _ptr(Ks), _ptr(Vs), B, Hkv, L, d,
                                          C, _dtype_code(K), _stream()))
    return Ks, Vs


def rf_noise(B, Hkv, n_chunks, d, seed, device="cuda"):
    """Counter-based standard normal draws for the stochastic summaries:
    fp32 [B, Hkv, n_chunks, d], chunk c of (b, g) depending only on
    (seed, b * Hkv + g, c) (eva_rf_noise); the draws a cache with the same
    seed uses for the chunks its appends complete."""
    eps = torch.empty(B, Hkv, n_chunks, d, dtype=torch.float32, device=device)
    _require_device(eps)
    _lib.check("eva_rf_noise", _lib.load().eva_rf_noise(_ptr(eps), B, Hkv, n_chunks, d, int(seed), _stream()))
    return eps


class Cache:
    """Window + summary decode cache in device memory (see eva_cache in eva.h).

    k_ring [B, Hkv, R, d], vt_ring [B, Hkv, R // 8, d, 8] (values transposed
    per 8-slot tile), k_sum [B, Hkv, S_max, d], vt_sum [B, Hkv, S_max // 8, d, 8].
    The ring holds the
    last R positions (R >= W + C - 1, a multiple of 32); S_max bounds the number
    of chunk summaries, i.e. the tokens the cache can ever absorb.
    """

    def __init__(self, B, H, Hkv, d, W, C, max_tokens, dtype=torch.bfloat16, device="cuda", R=None,
                 fill=None, window=_lib.EVA_WINDOW_SLIDING, rf_lambda=None, rf_seed=0):
        if R is None:
            R = -(-(W + C - 1) // 32) * 32
        S_max = max(32, -(-(max_tokens // C + 1) // 32) * 32)
        mk = (lambda *s: torch.full(s, fill, dtype=dtype, device=device)) if fill is not None else \
            (lambda *s: torch.empty(*s, dtype=dtype, device=device))
        self.k_ring = mk(B, Hkv, R, d)
        self.vt_ring = mk(B, Hkv, R // 8, d, 8)
        self.k_sum = mk(B, Hkv, S_max, d)
        self.vt_sum = mk(B, Hkv, S_max // 8, d, 8)
        self.dtype = dtype
        self.struct = _lib.EvaCacheStruct(B=B, H=H, H_kv=Hkv, d=d, W=W, C=C, dtype=_DTYPES[dtype], window=window,
                                          R=R, S_max=S_max, n_tok=0, k_ring=self.k_ring.data_ptr(),
                                          vt_ring=self.vt_ring.data_ptr(), k_sum=self.k_sum.data_ptr(),
                                          vt_sum=self.vt_sum.data_ptr(), rf=int(rf_lambda is not None),
                                          rf_lambda=float(rf_lambda or 0.0), rf_seed=int(rf_seed))
        self._ws = None

    @property
    def n_tok(self) -> int:
        return int(self.struct.n_tok)

    @property
    def R(self) -> int:
        return int(self.struct.R)

    @property
    def S_max(self) -> int:
        return int(self.struct.S_max)

    def workspace(self):
        """Decode split workspace for the current length (cached, grown on demand)."""
        n = _lib.load().eva_decode_workspace_bytes(ctypes.byref(self.struct))
        if n == 0:
            return None
        if self._ws is None or self._ws.numel() * 4 < n:
            self._ws = torch.empty((n + 3) // 4, dtype=torch.float32, device=self.k_ring.device)
        return self._ws


def prefill(Q, K, V, W: int, C: int, cache: Cache = None, return_summaries: bool = False,
            window: int = _lib.EVA_WINDOW_SLIDING, out=None, summaries=None):
    """EVA prefill. Q [B, H, L, d]; K, V [B, Hkv, L, d] -> O [B, H, L, d].
    `window`: one of the EVA_WINDOW_* variants.  `out` (O) and `summaries`
    ((Ks, Vs), [B, Hkv, L // C, d]) may be preallocated."""
    _require_device(Q, K, V)
    B, H, L, d = Q.shape
    Hkv = K.shape[1]
    if K.shape != (B, Hkv, L, d) or V.shape != K.shape or Q.dtype != K.dtype or V.dtype != K.dtype:
        raise ValueError("Q [B,H,L,d], K and V [B,Hkv,L,d] of one dtype expected")
    n_chunks = L // C
    if out is None:
        O = torch.empty_like(Q)
    else:
        O = out
        _require_device(O)
        if O.shape != Q.shape or O.dtype != Q.dtype:
            raise ValueError("out must be [B, H, L, d] in the dtype of Q")
    if summaries is None:
        Ks = torch.empty(B, Hkv, n_chunks, d, dtype=Q.dtype, device=Q.device)
        Vs = torch.empty_like(Ks)
    else:
        Ks, Vs = summaries
        _require_device(Ks, Vs)
        if tuple(Ks.shape) != (B, Hkv, n_chunks, d) or Vs.shape != Ks.shape or Ks.dtype != Q.dtype:
            raise ValueError("summaries must be [B, Hkv, L // C, d] in the dtype of Q")
    lib = _lib.load()
    cref = ctypes.byref(cache.struct) if cache is not None else None
    _lib.check("eva_prefill_ex",
               lib.eva_prefill_ex(_ptr(Q), _ptr(K), _ptr(V), _ptr(O), B, H, Hkv, L, d, W, C, _dtype_code(Q), window,
                                  _ptr(Ks) if n_chunks else None, _ptr(Vs) if n_chunks else None, cref, _stream()))
    if return_summaries:
        return O, Ks, Vs
    return O


def prefill_attention(Q, K, V, Ks, Vs, W: int, C: int, out=None, window: int = _lib.EVA_WINDOW_SLIDING):
    """The fused window + summary attention alone, given summaries from
    build_summaries(K, V, C). Q [B, H, L, d] -> O [B, H, L, d]."""
    _require_device(Q, K, V)
    B, H, L, d = Q.shape
    Hkv = K.shape[1]
    if K.shape != (B, Hkv, L, d) or V.shape != K.shape or Q.dtype != K.dtype or V.dtype != K.dtype:
        raise ValueError("Q [B,H,L,d], K and V [B,Hkv,L,d] of one dtype expected")
    if Ks is not None and (tuple(Ks.shape) != (B, Hkv, L // C, d) or Vs.shape != Ks.shape):
        raise ValueError("summaries must be [B, Hkv, L // C, d]")
    O = torch.empty_like(Q) if out is None else out
    _require_device(O)
    _lib.check("eva_prefill_attention_ex",
               _lib.load().eva_prefill_attention_ex(_ptr(Q), _ptr(K), _ptr(V), _ptr(Ks), _ptr(Vs), _ptr(O), B, H,
                                                    Hkv, L, d, W, C, _dtype_code(Q), window, _stream()))
    return O


def cache_fill(cache: Cache, K, V, Ks, Vs):
    """Load the cache from a prefilled sequence (K, V [B, Hkv, L, d] and its
    summaries); n_tok becomes L."""
    _require_device(K, V)
    s = cache.struct
    B, Hkv, L, d = K.shape
    if (B, Hkv, d) != (s.B, s.H_kv, s.d) or K.dtype != cache.dtype or V.shape != K.shape:
        raise ValueError("K, V must be [B, Hkv, L, d] matching the cache")
    _lib.check("eva_cache_fill",
               _lib.load().eva_cache_fill(ctypes.byref(s), _ptr(K), _ptr(V), _ptr(Ks), _ptr(Vs), L, _stream()))


def cache_append(cache: Cache, k_new, v_new):
    """Append one token per sequence: k_new, v_new [B, Hkv, d]."""
    _require_device(k_new, v_new)
    s = cache.struct
    if tuple(k_new.shape) != (s.B, s.H_kv, s.d) or v_new.shape != k_new.shape or k_new.dtype != cache.dtype:
        raise ValueError("k_new, v_new must be [B, Hkv, d] in the cache dtype")
    _lib.check("eva_cache_append",
               _lib.load().eva_cache_append(ctypes.byref(s), _ptr(k_new), _ptr(v_new), _stream()))


def append_decode(cache: Cache, q, k_new, v_new, use_workspace: bool = True, out=None):
    """Fused cache_append(k_new, v_new) + decode_step(q) in one launch."""
    _require_device(q, k_new, v_new)
    s = cache.struct
    if tuple(q.shape) != (s.B, s.H, s.d) or q.dtype != cache.dtype:
        raise ValueError("q must be [B, H, d] in the cache dtype")
    if tuple(k_new.shape) != (s.B, s.H_kv, s.d) or v_new.shape != k_new.shape or k_new.dtype != cache.dtype:
        raise ValueError("k_new, v_new must be [B, Hkv, d] in the cache dtype")
    o = torch.empty_like(q) if out is None else out
    ws = cache.workspace() if use_workspace else None
    nbytes = ws.numel() * 4 if ws is not None else 0
    _lib.check("eva_append_decode",
               _lib.load().eva_append_decode(ctypes.byref(s), _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(o), _ptr(ws),
                                             nbytes, _stream()))
    return o


def append_decode_noalloc(cache: Cache, q, k_new, v_new, out=None):
    """append_decode without a workspace: split partials go to the library's
    fixed device array (eva_append_decode_noalloc).  With `out` given the
    call allocates nothing."""
    _require_device(q, k_new, v_new)
    s = cache.struct
    if tuple(q.shape) != (s.B, s.H, s.d) or q.dtype != cache.dtype:
        raise ValueError("q must be [B, H, d] in the cache dtype")
    if tuple(k_new.shape) != (s.B, s.H_kv, s.d) or v_new.shape != k_new.shape or k_new.dtype != cache.dtype:
        raise ValueError("k_new, v_new must be [B, Hkv, d] in the cache dtype")
    o = torch.empty_like(q) if out is None else out
    _require_device(o)
    _lib.check("eva_append_decode_noalloc",
               _lib.load().eva_append_decode_noalloc(ctypes.byref(s), _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(o),
                                                     _stream()))
    return o


def decode_step(cache: Cache, q, use_workspace: bool = True, out=None):
    """Attention output of the last appended position: q [B, H, d] -> o [B, H, d]."""
    _require_device(q)
    s = cache.struct
    if tuple(q.shape) != (s.B, s.H, s.d) or q.dtype != cache.dtype:
        raise ValueError("q must be [B, H, d] in the cache dtype")
    o = torch.empty_like(q) if out is None else out
    ws = cache.workspace() if use_workspace else None
    nbytes = ws.numel() * 4 if ws is not None else 0
    _lib.check("eva_decode_step",
               _lib.load().eva_decode_step(ctypes.byref(s), _ptr(q), _ptr(o), _ptr(ws), nbytes, _stream()))
    return o


class RaggedCache:
    """Decode cache whose sequences hold different numbers of tokens (see
    eva_rcache in eva.h).  Same arrays as Cache; the per-sequence token counts
    `n_tok` [B] (int32) and the library's arrival counters live on the device,
    so steps need no host-side state.  `max_tokens` bounds every sequence."""

    def __init__(self, B, H, Hkv, d, W, C, max_tokens, dtype=torch.bfloat16, device="cuda", R=None, fill=None,
                 window=_lib.EVA_WINDOW_SLIDING, rf_lambda=None, rf_seed=0):
        if R is None:
            R = -(-(W + C - 1) // 32) * 32
        S_max = max(32, -(-(max_tokens // C + 1) // 32) * 32)
        mk = (lambda *s: torch.full(s, fill, dtype=dtype, device=device)) if fill is not None else \
            (lambda *s: torch.empty(*s, dtype=dtype, device=device))
        self.k_ring = mk(B, Hkv, R, d)
        self.vt_ring = mk(B, Hkv, R // 8, d, 8)
        self.k_sum = mk(B, Hkv, S_max, d)
        self.vt_sum = mk(B, Hkv, S_max // 8, d, 8)
        self.n_tok = torch.zeros(B, dtype=torch.int32, device=device)
        self.arrive = torch.zeros(B, dtype=torch.int32, device=device)
        self.dtype = dtype
        self.struct = _lib.EvaRCacheStruct(B=B, H=H, H_kv=Hkv, d=d, W=W, C=C, dtype=_DTYPES[dtype], window=window,
                                           R=R, S_max=S_max, max_tok=max_tokens, n_tok=self.n_tok.data_ptr(),
                                           arrive=self.arrive.data_ptr(), k_ring=self.k_ring.data_ptr(),
                                           vt_ring=self.vt_ring.data_ptr(), k_sum=self.k_sum.data_ptr(),
                                           vt_sum=self.vt_sum.data_ptr(), rf=int(rf_lambda is not None),
                                           rf_lambda=float(rf_lambda or 0.0), rf_seed=int(rf_seed))
        n = _lib.load().eva_rdecode_workspace_bytes(ctypes.byref(self.struct))
        self.ws = torch.empty((n + 3) // 4, dtype=torch.float32, device=device) if n else None

    @property
    def R(self) -> int:
        return int(self.struct.R)

    @property
    def S_max(self) -> int:
        return int(self.struct.S_max)

    def _ws_args(self, use_workspace):
        if use_workspace and self.ws is not None:
            return _ptr(self.ws), self.ws.numel() * 4
        return None, 0


def _active_ptr(active):
    if active is None:
        return None
    _require_device(active)
    if active.dtype != torch.int32:
        raise ValueError("active must be an int32 device tensor [B]")
    return _ptr(active)


def rcache_fill(cache: RaggedCache, K, V, Ks, Vs, lens):
    """Load a ragged cache from a right-padded prefill: K, V [B, Hkv, L, d] and
    their summaries; lens (int32 device [B]) are the valid lengths."""
    _require_device(K, V, lens)
    s = cache.struct
    B, Hkv, L, d = K.shape
    if (B, Hkv, d) != (s.B, s.H_kv, s.d) or K.dtype != cache.dtype or V.shape != K.shape:
        raise ValueError("K, V must be [B, Hkv, L, d] matching the cache")
    if lens.dtype != torch.int32 or tuple(lens.shape) != (B,):
        raise ValueError("lens must be an int32 device tensor [B]")
    _lib.check("eva_rcache_fill",
               _lib.load().eva_rcache_fill(ctypes.byref(s), _ptr(K), _ptr(V), _ptr(Ks), _ptr(Vs), L, _ptr(lens),
                                           _stream()))


def rcache_append(cache: RaggedCache, k_new, v_new, active=None):
    """Append one token to each active sequence: k_new, v_new [B, Hkv, d]."""
    _require_device(k_new, v_new)
    s = cache.struct
    if tuple(k_new.shape) != (s.B, s.H_kv, s.d) or v_new.shape != k_new.shape or k_new.dtype != cache.dtype:
        raise ValueError("k_new, v_new must be [B, Hkv, d] in the cache dtype")
    _lib.check("eva_rcache_append",
               _lib.load().eva_rcache_append(ctypes.byref(s), _ptr(k_new), _ptr(v_new), _active_ptr(active),
                                             _stream()))


def rdecode_step(cache: RaggedCache, q, active=None, out=None, use_workspace=True):
    """Output of each active sequence's last appended position: q [B, H, d].
    Rows of inactive or empty sequences keep the contents of `out`."""
    _require_device(q)
    s = cache.struct
    if tuple(q.shape) != (s.B, s.H, s.d) or q.dtype != cache.dtype:
        raise ValueError("q must be [B, H, d] in the cache dtype")
    o = torch.zeros_like(q) if out is None else out
    ws, nbytes = cache._ws_args(use_workspace)
    _lib.check("eva_rdecode_step",
               _lib.load().eva_rdecode_step(ctypes.byref(s), _ptr(q), _ptr(o), _active_ptr(active), ws, nbytes,
                                            _stream()))
    return o


def rappend_decode(cache: RaggedCache, q, k_new, v_new, active=None, out=None, use_workspace=True):
    """Fused rcache_append + rdecode_step of every active sequence in one launch."""
    _require_device(q, k_new, v_new)
    s = cache.struct
    if tuple(q.shape) != (s.B, s.H, s.d) or q.dtype != cache.dtype:
        raise ValueError("q must be [B, H, d] in the cache dtype")
    if tuple(k_new.shape) != (s.B, s.H_kv, s.d) or v_new.shape != k_new.shape or k_new.dtype != cache.dtype:
        raise ValueError("k_new, v_new must be [B, Hkv, d] in the cache dtype")
    o = torch.zeros_like(q) if out is None else out
    ws, nbytes = cache._ws_args(use_workspace)
    _lib.check("eva_rappend_decode",
               _lib.load().eva_rappend_decode(ctypes.byref(s), _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(o),
                                              _active_ptr(active), ws, nbytes, _stream()))
    return o


def generate(cache: RaggedCache, q, k, v, active=None, out=None, use_workspace=True):
    """T generation steps: q [T, B, H, d], k, v [T, B, Hkv, d] -> o [T, B, H, d]
    (token t of every active sequence appended, then decoded)."""
    _require_device(q, k, v)
    s = cache.struct
    T = q.shape[0]
    if tuple(q.shape) != (T, s.B, s.H, s.d) or tuple(k.shape) != (T, s.B, s.H_kv, s.d) or v.shape != k.shape:
        raise ValueError("q [T, B, H, d], k and v [T, B, Hkv, d] expected")
    if q.dtype != cache.dtype or k.dtype != cache.dtype or v.dtype != cache.dtype:
        raise ValueError("q, k, v must be in the cache dtype")
    o = torch.zeros_like(q) if out is None else out
    ws, nbytes = cache._ws_args(use_workspace)
    _lib.check("eva_generate",
               _lib.load().eva_generate(ctypes.byref(s), _ptr(q), _ptr(k), _ptr(v), _ptr(o), T, _active_ptr(active),
                                        ws, nbytes, _stream()))
    return o


def prefill_forward(Q, K, V, W: int, C: int, residual: bool = False, window: int = _lib.EVA_WINDOW_SLIDING):
    """Training forward under window variant `window` (EVA_WINDOW_*):
    summaries, O and the per-row log-sum-exp.  Returns (O, lse, Ks, Vs); lse
    is fp32 [B, H, L].  With `residual` (bf16) also the output's rounding
    residual O_lo: (O, lse, Ks, Vs, O_lo)."""
    _require_device(Q, K, V)
    B, H, L, d = Q.shape
    Hkv = K.shape[1]
    Ks, Vs = build_summaries(K, V, C)
    O = torch.empty_like(Q)
    O_lo = torch.empty_like(Q) if residual else None
    lse = torch.empty(B, H, L, dtype=torch.float32, device=Q.device)
    n_chunks = L // C
    _lib.check("eva_prefill_forward_ex",
               _lib.load().eva_prefill_forward_ex(_ptr(Q), _ptr(K), _ptr(V), _ptr(Ks) if n_chunks else None,
                                                  _ptr(Vs) if n_chunks else None, _ptr(O), _ptr(lse), _ptr(O_lo), B, H,
                                                  Hkv, L, d, W, C, _dtype_code(Q), window, _stream()))
    if residual:
        return O, lse, Ks, Vs, O_lo
    return O, lse, Ks, Vs


def prefill_backward(Q, K, V, Ks, Vs, O, lse, dO, W: int, C: int, workspace=None, O_lo=None,
                     window: int = _lib.EVA_WINDOW_SLIDING):
    """Gradients (dQ, dK, dV) of the EVA prefill for the output gradient dO
    (bf16, window variant `window`), from the training forward's O, lse and
    summaries under the same variant (and, if it kept one, its output
    residual O_lo)."""
    _require_device(Q, K, V, O, lse, dO)
    if O_lo is not None:
        _require_device(O_lo)
        if O_lo.shape != O.shape or O_lo.dtype != O.dtype:
            raise ValueError("O_lo must match O")
    B, H, L, d = Q.shape
    Hkv = K.shape[1]
    if dO.shape != Q.shape or O.shape != Q.shape or tuple(lse.shape) != (B, H, L) or lse.dtype != torch.float32:
        raise ValueError("O, dO [B, H, L, d] and fp32 lse [B, H, L] expected")
    lib = _lib.load()
    need = lib.eva_prefill_backward_workspace_bytes(B, H, Hkv, L, d, C)
    ws = workspace
    if ws is None or ws.numel() * ws.element_size() < need:
        ws = torch.empty((need + 3) // 4, dtype=torch.float32, device=Q.device)
    dQ = torch.empty_like(Q)
    dK = torch.empty_like(K)
    dV = torch.empty_like(V)
    n_chunks = L // C
    _lib.check("eva_prefill_backward_ex",
               lib.eva_prefill_backward_ex(_ptr(Q), _ptr(K), _ptr(V), _ptr(Ks) if n_chunks else None,
                                           _ptr(Vs) if n_chunks else None, _ptr(O), _ptr(O_lo), _ptr(dO), _ptr(lse),
                                           _ptr(dQ), _ptr(dK), _ptr(dV), _ptr(ws), ws.numel() * ws.element_size(), B,
                                           H, Hkv, L, d, W, C, _dtype_code(Q), window, _stream()))
    return dQ, dK, dV


# ---- head norms with rotation ----------------------------------------------
_functions = {}


def _call(dev, name, *args):
    """Call lib.<name>(*args, stream) on the current stream of device `dev` (its
    index), with that device current."""
    if dev < 0:  # (operands on the device of a cache in host memory)
        raise RuntimeError("EVA kernels run on the GPU only: tensors must be on a ROCm device")
    fn = _functions.get(name)
    if fn is None:
        fn = _functions[name] = getattr(_lib.load(), name)
    if dev == torch._C._cuda_getDevice():
        status = fn(*args, torch._C._cuda_getCurrentRawStream(dev))
    else:
        with torch.cuda.device(dev):
            status = fn(*args, torch._C._cuda_getCurrentRawStream(dev))
    if status != _lib.EVA_OK:
        raise _lib.EvaError(name, status)


def _expect(t, what, shape, dtype, dev):
    """Address of an operand (None: no operand): contiguous, of this shape (a
    tuple) and dtype, on device `dev`."""
    if t is None:
        return None
    if t.shape != shape or t.dtype is not dtype:
        raise ValueError(f"{what} must be {dtype} {list(shape)}")
    if t.get_device() != dev:
        raise RuntimeError(f"{what} must be on the same ROCm device as the others")
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    return t.data_ptr()


def rope_turns(rot: int, base: float = 10000.0, inv_freq=None, device="cuda") -> torch.Tensor:
    """Frequencies of qk_norm_rope, int64 [rot / 2]: base^(-2i / rot), or the
    `inv_freq` given (rot / 2 radians per position), in 2^-64 turns."""
    if inv_freq is None:
        inv_freq = [float(base) ** (-2.0 * i / rot) for i in range(rot // 2)]
    inv_freq = [float(f) for f in inv_freq]
    if len(inv_freq) != rot // 2:
        raise ValueError("inv_freq must hold rot / 2 frequencies")
    t = [round(f / (2 * math.pi) * 2 ** 64) % 2 ** 64 for f in inv_freq]
    return torch.tensor([x - 2 ** 64 if x >= 2 ** 63 else x for x in t], dtype=torch.int64, device=device)


def _norm_rope_args(x, H, Hkv, turns, q_weight, k_weight, eps, start, offsets, interleaved):
    """The arguments both directions share, and (device, B, L, d)."""
    dev = x.get_device()
    if dev < 0:
        raise RuntimeError("EVA kernels run on the GPU only: tensors must be on a ROCm device")
    if x.dim() != 3 or H < 1 or Hkv < 1 or x.shape[2] % (H + 2 * Hkv) != 0:
        raise ValueError("x must be [B, L, (H + 2 Hkv) * d]")
    B, L, d = x.shape
    d //= H + 2 * Hkv
    sb, sl, sf = x.stride()
    if sf != 1:
        raise ValueError("the features of x must be contiguous")
    rot = 0 if turns is None else 2 * turns.numel()
    # the stride of a single row is never used, and may be any number
    return (x.data_ptr(), sb if B > 1 else 0, sl if L > 1 else 0, _expect(q_weight, "q_weight", (d,), x.dtype, dev),
            _expect(k_weight, "k_weight", (d,), x.dtype, dev), _expect(turns, "turns", (rot // 2,), torch.int64, dev),
            rot, 1 if interleaved else 0, _expect(start, "start", (B,), torch.int32, dev),
            _expect(offsets, "offsets", (B, L), torch.int32, dev), eps), dev, B, L, d


def qk_norm_rope(x, H: int, Hkv: int, turns=None, q_weight=None, k_weight=None, eps: float = 1e-6, start=None,
                 offsets=None, interleaved: bool = False, out=None):
    """Head norms with rotation: x [B, L, (H + 2 Hkv) * d], a projection's
    output (its rows may be strided), -> Q [B, H, L, d], K, V [B, Hkv, L, d].

    `q_weight`, `k_weight` [d]: weights of the root-mean-square norms (None:
    no norm).  `turns`: rope_turns' frequencies (None: no rotation).  The
    token's position is start[b] (int32 [B], a ragged cache's n_tok for one;
    None: 0) + offsets[b, l] (int32 [B, L]; None: l).  `out` = (Q, K, V)
    preallocated.  The outputs carry no autograd history:
    qk_norm_rope_backward gives the gradients."""
    args, dev, B, L, d = _norm_rope_args(x, H, Hkv, turns, q_weight, k_weight, eps, start, offsets, interleaved)
    code = _dtype_code(x)
    if out is None:
        Q, K = x.new_empty((B, H, L, d)), x.new_empty((B, Hkv, L, d))
        V = torch.empty_like(K)
        q, k, v = Q.data_ptr(), K.data_ptr(), V.data_ptr()
    else:
        Q, K, V = out
        q = _expect(Q, "Q", (B, H, L, d), x.dtype, dev)
        k, v = (_expect(t, "K and V", (B, Hkv, L, d), x.dtype, dev) for t in (K, V))
    if B > 0 and L > 0:
        _call(dev, "eva_qk_norm_rope", *args, q, k, v, B, H, Hkv, L, d, code)
    return Q, K, V


def qk_norm_rope_backward(x, dQ, dK, dV, turns=None, q_weight=None, k_weight=None, eps: float = 1e-6, start=None,
                          offsets=None, interleaved: bool = False):
    """Gradients of qk_norm_rope: dQ [B, H, L, d], dK, dV [B, Hkv, L, d] ->
    (dx [B, L, (H + 2 Hkv) * d], dq_weight, dk_weight), the weights' in fp32
    (None where there is no weight)."""
    if dQ.dim() != 4 or dK.dim() != 4:
        raise ValueError("dQ [B, H, L, d], dK and dV [B, Hkv, L, d] expected")
    H, Hkv = dQ.shape[1], dK.shape[1]
    args, dev, B, L, d = _norm_rope_args(x, H, Hkv, turns, q_weight, k_weight, eps, start, offsets, interleaved)
    code = _dtype_code(x)
    grads = (_expect(dQ, "dQ", (B, H, L, d), x.dtype, dev), _expect(dK, "dK", (B, Hkv, L, d), x.dtype, dev),
             _expect(dV, "dV", (B, Hkv, L, d), x.dtype, dev))
    dx = x.new_empty(x.shape)
    none = B == 0 or L == 0
    dg = [None if w is None else (x.new_zeros if none else x.new_empty)(d, dtype=torch.float32)
          for w in (q_weight, k_weight)]
    if none:
        return (dx, *dg)
    n = ws = 0
    if q_weight is not None or k_weight is not None:
        n = _lib.load().eva_qk_norm_rope_backward_workspace_bytes(B, L, d)
        ws = x.new_empty(n, dtype=torch.uint8)
    _call(dev, "eva_qk_norm_rope_backward", *args, *grads, dx.data_ptr(), _ptr(dg[0]), _ptr(dg[1]),
          ws.data_ptr() if n else None, n, B, H, Hkv, L, d, code)
    return (dx, *dg)


# ---- 8-bit cache -------------------------------------------------------------
class QuantCache:
    """Ragged decode cache of e4m3 rows with a power of two each (see
    eva_qcache in eva.h): k_ring [B, Hkv, R, d], vt_ring [B, Hkv, R // 16, d, 16],
    k_sum, vt_sum likewise over S_max, and each row's exponent byte in *_exp.
    Queries, keys, values and outputs are bf16.  Entries that are not finite, or
    above 3.08e38, are held as NaN.  `max_tokens` bounds every sequence."""

    dtype = torch.bfloat16  # of the rows outside

    def __init__(self, B, H, Hkv, d, W, C, max_tokens, device="cuda", R=None, fill=None,
                 window=_lib.EVA_WINDOW_SLIDING):
        if R is None:
            R = -(-(W + C - 1) // 64) * 64
        S_max = max(64, -(-(max_tokens // C + 1) // 64) * 64)
        code = None if fill is None else int(torch.tensor(float(fill)).to(torch.float8_e4m3fn).view(torch.uint8))

        def mk(*s, value=code):
            t = torch.empty(*s, dtype=torch.uint8, device=device)
            return t if code is None else t.fill_(value)

        self.k_ring = mk(B, Hkv, R, d).view(torch.float8_e4m3fn)
        self.vt_ring = mk(B, Hkv, R // 16, d, 16).view(torch.float8_e4m3fn)
        self.k_sum = mk(B, Hkv, S_max, d).view(torch.float8_e4m3fn)
        self.vt_sum = mk(B, Hkv, S_max // 16, d, 16).view(torch.float8_e4m3fn)
        self.k_ring_exp, self.v_ring_exp = mk(B, Hkv, R, value=127), mk(B, Hkv, R, value=127)
        self.k_sum_exp, self.v_sum_exp = mk(B, Hkv, S_max, value=127), mk(B, Hkv, S_max, value=127)
        self.n_tok = torch.zeros(B, dtype=torch.int32, device=device)
        self.arrive = torch.zeros(B, dtype=torch.int32, device=device)
        names = ("n_tok", "arrive", "k_ring", "vt_ring", "k_sum", "vt_sum", "k_ring_exp", "v_ring_exp", "k_sum_exp",
                 "v_sum_exp")
        self.struct = _lib.EvaQCacheStruct(B=B, H=H, H_kv=Hkv, d=d, W=W, C=C, window=window, R=R, S_max=S_max,
                                           max_tok=max_tokens, **{n: getattr(self, n).data_ptr() for n in names})

    @property
    def R(self) -> int:
        return int(self.struct.R)

    @property
    def S_max(self) -> int:
        return int(self.struct.S_max)


def _rows_out(q, out, whole, dev):
    """The output of q's shape: `out`, or a new one (zeros where the call may
    leave rows unwritten); and its address."""
    if out is None:
        out = torch.empty_like(q) if whole else torch.zeros_like(q)
        return out, out.data_ptr()
    return out, _expect(out, "out", q.shape, q.dtype, dev)


def _scratch(q, n):
    """A workspace of n bytes of the call's own (None: none needed)."""
    return q.new_empty(n, dtype=torch.uint8) if n else None


def qcache_fill(cache: QuantCache, K, V, Ks, Vs, lens):
    """rcache_fill into an 8-bit cache: K, V [B, Hkv, L, d] and their summaries,
    quantised; lens (int32 [B]) are the valid lengths."""
    s, dev, dt = cache.struct, cache.n_tok.get_device(), cache.dtype
    if K.dim() != 4:
        raise ValueError("K must be [B, Hkv, L, d]")
    L = K.shape[2]
    shape, sums = (s.B, s.H_kv, L, s.d), (s.B, s.H_kv, L // s.C, s.d)
    _call(dev, "eva_qcache_fill", ctypes.byref(s), _expect(K, "K", shape, dt, dev), _expect(V, "V", shape, dt, dev),
          _expect(Ks, "Ks", sums, dt, dev), _expect(Vs, "Vs", sums, dt, dev), L,
          _expect(lens, "lens", (s.B,), torch.int32, dev))


def qcache_append(cache: QuantCache, k_new, v_new, active=None):
    """Append one token to each active sequence: k_new, v_new [B, Hkv, d]."""
    s, dev, dt = cache.struct, cache.n_tok.get_device(), cache.dtype
    row = (s.B, s.H_kv, s.d)
    _call(dev, "eva_qcache_append", ctypes.byref(s), _expect(k_new, "k_new", row, dt, dev),
          _expect(v_new, "v_new", row, dt, dev), _expect(active, "active", (s.B,), torch.int32, dev))


def qcache_read(cache: QuantCache, to: RaggedCache) -> RaggedCache:
    """Copy the 8-bit cache's rows and token counts into the bf16 ragged cache
    `to` of the same geometry, which can then go on with them."""
    if to.n_tok.device != cache.n_tok.device:
        raise RuntimeError("both caches must be on one device")
    _call(cache.n_tok.get_device(), "eva_qcache_read", ctypes.byref(cache.struct), ctypes.byref(to.struct))
    return to


def _qdecode(cache, name, q, new, active, out, use_workspace):
    s, dev, dt = cache.struct, cache.n_tok.get_device(), cache.dtype
    args = [_expect(q, "q", (s.B, s.H, s.d), dt, dev)]
    args += [_expect(t, "k_new and v_new", (s.B, s.H_kv, s.d), dt, dev) for t in new]
    on = _expect(active, "active", (s.B,), torch.int32, dev)
    o, po = _rows_out(q, out, active is None, dev)
    n = _lib.load().eva_qdecode_workspace_bytes(ctypes.byref(s)) if use_workspace else 0
    ws = _scratch(q, n)
    _call(dev, name, ctypes.byref(s), *args, po, on, _ptr(ws), n)
    return o


def qdecode_step(cache: QuantCache, q, active=None, out=None, use_workspace=True):
    """rdecode_step over an 8-bit cache: q [B, H, d] -> o [B, H, d].  Rows of
    inactive sequences keep the contents of `out`, those of empty ones are
    zeros."""
    return _qdecode(cache, "eva_qdecode_step", q, (), active, out, use_workspace)


def qappend_decode(cache: QuantCache, q, k_new, v_new, active=None, out=None, use_workspace=True):
    """qcache_append(k_new, v_new), then qdecode_step(q)."""
    return _qdecode(cache, "eva_qappend_decode", q, (k_new, v_new), active, out, use_workspace)


# ---- drafted trees -----------------------------------------------------------
def tree_attention(cache, q, k, v, parents, n_nodes=None, active=None, out=None, use_workspace=True):
    """Rows of a tree of drafted tokens for every sequence of a RaggedCache or
    QuantCache, which is left as it is: q [B, H, T, d], k, v [B, Hkv, T, d] ->
    o [B, H, T, d].

    parents (int32 [B, T]): the earlier node that node t continues, or -1: the
    sequence itself.  n_nodes (int32 [B]): each tree's size, T if None.  Node t's
    position is n_tok[b] + its depth.  T is at most 64 and W.  Rows of inactive
    sequences and absent nodes keep the contents of `out`."""
    s, dev, dt = cache.struct, cache.n_tok.get_device(), cache.dtype
    if q.dim() != 4:
        raise ValueError("q must be [B, H, T, d]")
    T, B, d = q.shape[2], s.B, s.d
    row = (B, s.H_kv, T, d)
    args = (_expect(q, "q", (B, s.H, T, d), dt, dev), _expect(k, "k", row, dt, dev), _expect(v, "v", row, dt, dev),
            _expect(parents, "parents", (B, T), torch.int32, dev), _expect(n_nodes, "n_nodes", (B,), torch.int32, dev))
    on = _expect(active, "active", (B,), torch.int32, dev)
    o, po = _rows_out(q, out, n_nodes is None and active is None, dev)
    ref, lib = ctypes.byref(s), _lib.load()
    if isinstance(cache, QuantCache):
        name, size = "eva_qtree_attention", lib.eva_qtree_workspace_bytes
    else:
        name, size = "eva_rtree_attention", lib.eva_rtree_workspace_bytes
    n = size(ref, T) if use_workspace else 0
    ws = _scratch(q, n)
    _call(dev, name, ref, *args, po, T, on, _ptr(ws), n)
    return o


def append_path(cache, k, v, path=None, counts=None, active=None):
    """Append an accepted path to every active sequence of a RaggedCache or
    QuantCache: the tokens path[b, :counts[b]] (int32 [B, T], [B]; by default
    all T in their order) of k, v [B, Hkv, T, d]."""
    s, dev, dt = cache.struct, cache.n_tok.get_device(), cache.dtype
    if k.dim() != 4:
        raise ValueError("k must be [B, Hkv, T, d]")
    T, B = k.shape[2], s.B
    row = (B, s.H_kv, T, s.d)
    _call(dev, "eva_qappend_path" if isinstance(cache, QuantCache) else "eva_rappend_path", ctypes.byref(s),
          _expect(k, "k", row, dt, dev), _expect(v, "v", row, dt, dev), _expect(path, "path", (B, T), torch.int32, dev),
          _expect(counts, "counts", (B,), torch.int32, dev), T, _expect(active, "active", (B,), torch.int32, dev))


# ---- paged cache ---------------------------------------------------------------
_LONGEST = 1 << 30  # tokens, slots and list entries; the C interface's ints would wrap beyond 2^31


class PageTable:
    """Which pages of a pool the sequences of a batch have (see eva_page_table in
    eva.h), shared by all layers' PagedCaches: n_tok [B], table [B, max_pages],
    the stack free_pages [n_pages] with n_free [1], all int32 on the device.
    `page`: tokens of a page (16, 32, 64, 128 or 256); `max_tokens` bounds every
    sequence.  `storage` = (n_tok, table, free_pages, n_free) takes arrays that there
    are already, as they stand; else every page is free."""

    def __init__(self, B, page, n_pages, max_tokens, device="cuda", storage=None):
        if page not in (16, 32, 64, 128, 256):
            raise ValueError("a page holds 16, 32, 64, 128 or 256 tokens")
        rows = -(-max_tokens // page)
        if max(B, B * rows, n_pages * page, rows * page) > _LONGEST:
            raise ValueError("a table has up to 2^30 entries, its pool and each of its rows up to 2^30 tokens")
        if storage is None:
            self.n_tok = torch.zeros(B, dtype=torch.int32, device=device)
            self.table = torch.full((B, rows), -1, dtype=torch.int32, device=device)
            # the lowest pages on top
            self.free_pages = torch.arange(n_pages - 1, -1, -1, dtype=torch.int32, device=device)
            self.n_free = torch.full((1,), n_pages, dtype=torch.int32, device=device)
        else:
            self.n_tok, self.table, self.free_pages, self.n_free = storage
            dev = self.n_tok.get_device()
            for t, what, shape in ((self.n_tok, "n_tok", (B,)), (self.table, "table", (B, rows)),
                                   (self.free_pages, "free_pages", (n_pages,)), (self.n_free, "n_free", (1,))):
                _expect(t, what, shape, torch.int32, dev)
        self.struct = _lib.EvaPageTableStruct(B=B, P=page, n_pages=n_pages, max_pages=rows,
                                              **{n: getattr(self, n).data_ptr()
                                                 for n in ("n_tok", "table", "free_pages", "n_free")})
        self.ref = ctypes.byref(self.struct)


class PagedCache:
    """A layer's rows in the pages of `table` (see eva_pcache in eva.h): k
    [n_pages, Hkv, page, d], vt [n_pages, Hkv, page // 8, d, 8] and, unless
    `means` is false, k_mean [n_pages, Hkv, d] (fp32), which paged_select needs.
    `storage` = (k, vt, k_mean or None) takes arrays that there are already."""

    def __init__(self, table: PageTable, H, Hkv, d, dtype=torch.bfloat16, means=True, fill=None, storage=None):
        t, dev = table.struct, table.n_tok.device
        if max(H, Hkv, d) > _LONGEST:
            raise ValueError("H, Hkv and d are at most 2^30")
        shapes = ((t.n_pages, Hkv, t.P, d), (t.n_pages, Hkv, t.P // 8, d, 8), (t.n_pages, Hkv, d))
        if storage is None:
            mk = (lambda s, dt: torch.full(s, fill, dtype=dt, device=dev)) if fill is not None else \
                (lambda s, dt: torch.empty(s, dtype=dt, device=dev))
            self.k, self.vt = mk(shapes[0], dtype), mk(shapes[1], dtype)
            self.k_mean = mk(shapes[2], torch.float32) if means else None
        else:
            self.k, self.vt, self.k_mean = storage
            for x, what, shape, dt in zip(storage, ("k", "vt", "k_mean"), shapes, (dtype, dtype, torch.float32)):
                _expect(x, what, shape, dt, table.n_tok.get_device())
        self.table, self.dtype = table, dtype
        self.struct = _lib.EvaPCacheStruct(H=H, H_kv=Hkv, d=d, dtype=_DTYPES[dtype], P=t.P, n_pages=t.n_pages,
                                           k=self.k.data_ptr(), vt=self.vt.data_ptr(), k_mean=_ptr(self.k_mean))
        self.ref = ctypes.byref(self.struct)
        self._sizes = {}  # workspace bytes by (call, length of the page list)

    def _ws_bytes(self, name, S):
        n = self._sizes.get((name, S))
        if n is None:
            n = self._sizes[name, S] = getattr(_lib.load(), name)(self.ref, self.table.ref, S)
        return n


def page_extend(table: PageTable, T: int = 1, counts=None):
    """Pages and slots for counts[b] (int32 [B], at most T; None: T) new tokens of
    every sequence: (slots [B, T], start [B], granted [B]), int32.  A sequence that the
    free pages or its row of the table do not suffice for is granted none.  One that the
    free pages do not suffice for holds up the later ones that need pages in this call, also
    where it asks for more than the pool has: set its count to 0 to let them pass."""
    s, dev = table.struct, table.n_tok.get_device()
    if not 1 <= T <= _LONGEST:
        raise ValueError("T must be at least 1 and at most 2^30")
    B, n_tok = s.B, table.n_tok
    c = _expect(counts, "counts", (B,), torch.int32, dev)
    slots, start = n_tok.new_empty((B, T)), torch.empty_like(n_tok)
    granted = torch.empty_like(start)
    _call(dev, "eva_page_extend", table.ref, c, T, slots.data_ptr(), start.data_ptr(), granted.data_ptr())
    return slots, start, granted


def page_truncate(table: PageTable, lens):
    """Sequence b keeps its first lens[b] (int32 [B]) tokens; pages that none is left
    in become free.  0: the sequence leaves."""
    dev = table.n_tok.get_device()
    _call(dev, "eva_page_truncate", table.ref, _expect(lens, "lens", (table.struct.B,), torch.int32, dev))


def paged_append(cache: PagedCache, k, v, slots):
    """Write new tokens' keys and values [B, Hkv, T, d] (or [B, Hkv, d]) into page_extend's
    slots [B, T]; pages that they complete get their mean key."""
    s, dev, dt = cache.struct, cache.k.get_device(), cache.dtype
    if slots.dim() != 2:
        raise ValueError("slots must be [B, T]")
    B, T = slots.shape
    row = (B, s.H_kv, s.d) if k.dim() == 3 and T == 1 else (B, s.H_kv, T, s.d)
    args = (_expect(k, "k", row, dt, dev), _expect(v, "v", row, dt, dev), _expect(slots, "slots", (B, T), torch.int32, dev))
    if B > 0 and T > 0:
        _call(dev, "eva_paged_append", cache.ref, *args, B, T)


def paged_select(cache: PagedCache, q, n_pages: int, first: int = 1, last: int = 1):
    """The pages that each kv head's queries choose by the pages' mean keys: q
    [B, H, d] -> int32 [B, Hkv, n_pages], ascending, then -1; the `first` first and the
    `last` last pages of a sequence are always among them."""
    s, dev, t = cache.struct, cache.k.get_device(), cache.table
    B = t.struct.B
    pq = _expect(q, "q", (B, s.H, s.d), cache.dtype, dev)
    if not 1 <= n_pages <= _LONGEST:
        raise ValueError("n_pages must be at least 1 and at most 2^30")
    if first < 0 or last < 1 or first + last > n_pages:
        raise ValueError("first must be at least 0, last at least 1, and both together at most n_pages")
    pages = t.n_tok.new_empty((B, s.H_kv, n_pages))
    n = cache._ws_bytes("eva_paged_select_workspace_bytes", n_pages)
    ws = _scratch(q, n)
    _call(dev, "eva_paged_select", cache.ref, t.ref, pq, n_pages, first, last, pages.data_ptr(), _ptr(ws), n)
    return pages


def paged_decode(cache: PagedCache, q, pages=None, active=None, out=None, use_workspace=True):
    """Attention of one query a sequence, that of its last token, over all its
    tokens, or over those of its kv heads' `pages` (int32 [B, Hkv, S], paged_select's):
    q [B, H, d] -> o [B, H, d].  Several new tokens are appended and attended one by one.
    Rows of sequences without tokens are zeros, those of inactive ones keep the contents
    of `out`."""
    s, dev, t = cache.struct, cache.k.get_device(), cache.table
    B, S = t.struct.B, 0
    pq = _expect(q, "q", (B, s.H, s.d), cache.dtype, dev)
    if pages is not None:
        if pages.dim() != 3 or pages.shape[2] < 1:
            raise ValueError("pages must be [B, Hkv, S]")
        S = pages.shape[2]
        if S > _LONGEST:
            raise ValueError("a list of pages has at most 2^30 entries")
    pp = _expect(pages, "pages", (B, s.H_kv, S), torch.int32, dev)
    on = _expect(active, "active", (B,), torch.int32, dev)
    o, po = _rows_out(q, out, active is None, dev)
    n = cache._ws_bytes("eva_paged_decode_workspace_bytes", S) if use_workspace else 0
    ws = _scratch(q, n)
    _call(dev, "eva_paged_decode", cache.ref, t.ref, pq, po, pp, S, on, _ptr(ws), n)
    return o
