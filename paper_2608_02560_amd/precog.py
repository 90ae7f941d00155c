"""Python binding of libprecog (the C ABI in include/precog.h).

Argument marshalling only: every step of the computation runs in the gfx950
kernels of libprecog.so.  PyTorch supplies device memory and the current
HIP stream.  There is no fallback: if the library is missing or the device is
not a gfx950, the calls raise.
"""
from __future__ import annotations

import contextlib
import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# Always the in-tree build: tests, smoke and bench measure the library built
# from this tree's sources.
LIB_PATH = os.path.join(_HERE, "libprecog.so")

F32, BF16, F16 = 0, 1, 2
_DT = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}

STATUS = {0: "PRECOG_OK", 1: "PRECOG_ERR_NULL", 2: "PRECOG_ERR_SHAPE", 3: "PRECOG_ERR_DTYPE",
          4: "PRECOG_ERR_STRIDE", 5: "PRECOG_ERR_ALIGN", 6: "PRECOG_ERR_WORKSPACE",
          7: "PRECOG_ERR_ARCH", 8: "PRECOG_ERR_HIP"}

EXPORTS = ("precog_scan_workspace_bytes", "precog_scan_encode", "precog_scan_encode_indexed",
           "precog_scan_trajectory",
           "precog_scan_complex", "precog_scan_complex_workspace_bytes",
           "precog_retrieve_workspace_bytes", "precog_retrieve_top1",
           "precog_retrieve_top1_noalloc",
           "precog_retrieve_topk", "precog_retrieve_index_bytes", "precog_retrieve_prepare",
           "precog_retrieve_topk_prepared", "precog_query_workspace_bytes",
           "precog_query_top1_prefill", "precog_inject_gather", "precog_inject_compose",
           "precog_inject_fuse",
           "precog_smc_route", "precog_smc_consolidate", "precog_delta_workspace_bytes",
           "precog_delta_encode",
           "precog_delta_step", "precog_conv_encode", "precog_conv_step",
           "precog_score_workspace_bytes", "precog_score_tokens", "precog_status_string")


class PrecogError(RuntimeError):
    def __init__(self, fn: str, status: int):
        self.status = status
        super().__init__("%s failed: %s (%s)" % (fn, STATUS.get(status, status),
                                                 status_string(status)))


class ScanDesc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("seqlen", ctypes.c_int64),
                ("dim", ctypes.c_int64), ("dstate", ctypes.c_int64),
                ("in_dtype", ctypes.c_int), ("out_dtype", ctypes.c_int),
                ("state_dtype", ctypes.c_int),
                ("h0_batch_stride", ctypes.c_int64), ("hT_batch_stride", ctypes.c_int64),
                ("chunk", ctypes.c_int64)]


class DeltaDesc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("seqlen", ctypes.c_int64),
                ("k_heads", ctypes.c_int64), ("v_heads", ctypes.c_int64),
                ("k_dim", ctypes.c_int64), ("v_dim", ctypes.c_int64),
                ("q_stride", ctypes.c_int64), ("k_stride", ctypes.c_int64),
                ("v_stride", ctypes.c_int64), ("h0_batch_stride", ctypes.c_int64),
                ("hT_batch_stride", ctypes.c_int64), ("in_dtype", ctypes.c_int),
                ("out_dtype", ctypes.c_int), ("state_dtype", ctypes.c_int),
                ("qk_norm", ctypes.c_int32), ("eps", ctypes.c_float), ("scale", ctypes.c_float)]


class ConvDesc(ctypes.Structure):
    _fields_ = [("batch", ctypes.c_int64), ("seqlen", ctypes.c_int64), ("dim", ctypes.c_int64),
                ("width", ctypes.c_int64), ("x_stride", ctypes.c_int64),
                ("in_dtype", ctypes.c_int), ("out_dtype", ctypes.c_int), ("silu", ctypes.c_int32)]


_lib = None


def lib():
    """The loaded libprecog.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libprecog.so is not built (%s); run "
                               "`python -m paper_2608_02560_amd.build`" % LIB_PATH)
        L = ctypes.CDLL(LIB_PATH)
        vp, i64, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t
        L.precog_scan_workspace_bytes.argtypes = [ctypes.POINTER(ScanDesc)]
        L.precog_scan_workspace_bytes.restype = sz
        L.precog_scan_encode.argtypes = [ctypes.POINTER(ScanDesc)] + [vp] * 11 + [sz, vp]
        L.precog_scan_encode.restype = ctypes.c_int
        L.precog_scan_encode_indexed.argtypes = [ctypes.POINTER(ScanDesc)] + [vp] * 8 + \
            [i64, vp, vp, i64, ctypes.c_double, vp, vp, vp, sz, vp]
        L.precog_scan_encode_indexed.restype = ctypes.c_int
        L.precog_scan_trajectory.argtypes = [ctypes.POINTER(ScanDesc)] + [vp] * 11 + \
            [i64, vp, sz, vp]
        L.precog_scan_trajectory.restype = ctypes.c_int
        L.precog_scan_complex.argtypes = [ctypes.POINTER(ScanDesc)] + [vp] * 12 + [sz, vp]
        L.precog_scan_complex.restype = ctypes.c_int
        L.precog_scan_complex_workspace_bytes.argtypes = [ctypes.POINTER(ScanDesc)]
        L.precog_scan_complex_workspace_bytes.restype = sz
        L.precog_retrieve_workspace_bytes.argtypes = [i64, i64, i64]
        L.precog_retrieve_workspace_bytes.restype = sz
        L.precog_retrieve_top1.argtypes = [vp, vp, i64, i64, i64, vp, vp, sz, vp]
        L.precog_retrieve_top1.restype = ctypes.c_int
        L.precog_retrieve_top1_noalloc.argtypes = [vp, vp, i64, i64, i64, vp, vp]
        L.precog_retrieve_top1_noalloc.restype = ctypes.c_int
        L.precog_retrieve_topk.argtypes = [vp, vp, i64, i64, i64, i64, vp, vp, vp, sz, vp]
        L.precog_retrieve_topk.restype = ctypes.c_int
        L.precog_retrieve_index_bytes.argtypes = [i64, i64]
        L.precog_retrieve_index_bytes.restype = sz
        L.precog_retrieve_prepare.argtypes = [vp, i64, i64, vp, sz, vp]
        L.precog_retrieve_prepare.restype = ctypes.c_int
        L.precog_retrieve_topk_prepared.argtypes = [vp, vp, vp, sz, i64, i64, i64, i64, vp, vp, vp,
                                                    sz, vp]
        L.precog_retrieve_topk_prepared.restype = ctypes.c_int
        L.precog_query_workspace_bytes.argtypes = [ctypes.POINTER(ScanDesc), i64, i64]
        L.precog_query_workspace_bytes.restype = sz
        L.precog_query_top1_prefill.argtypes = [ctypes.POINTER(ScanDesc), vp, vp, vp, sz, i64, i64,
                                                vp, vp] + [vp] * 9 + [vp, sz, vp]
        L.precog_query_top1_prefill.restype = ctypes.c_int
        L.precog_inject_gather.argtypes = [vp, ctypes.c_int, i64, i64, vp, i64, vp,
                                           ctypes.c_int, vp]
        L.precog_inject_gather.restype = ctypes.c_int
        L.precog_inject_compose.argtypes = [vp, ctypes.c_int, i64, i64, vp, vp, i64, i64,
                                            ctypes.c_double, vp, ctypes.c_int, vp]
        L.precog_inject_compose.restype = ctypes.c_int
        L.precog_inject_fuse.argtypes = [vp, i64, vp, vp, i64, vp, i64, vp, vp, i64, ctypes.c_int,
                                         i64, i64, i64, ctypes.c_double, vp, vp, i64,
                                         ctypes.c_double, vp, ctypes.c_int, vp]
        L.precog_inject_fuse.restype = ctypes.c_int
        L.precog_smc_route.argtypes = [vp, i64, i64, vp, i64, vp, i64, vp, vp, vp, vp]
        L.precog_smc_route.restype = ctypes.c_int
        L.precog_smc_consolidate.argtypes = [vp, ctypes.c_int, i64, i64, vp, ctypes.c_int, vp, i64,
                                             ctypes.c_double, vp]
        L.precog_smc_consolidate.restype = ctypes.c_int
        L.precog_delta_workspace_bytes.argtypes = [ctypes.POINTER(DeltaDesc), ctypes.c_int]
        L.precog_delta_workspace_bytes.restype = sz
        L.precog_delta_encode.argtypes = [ctypes.POINTER(DeltaDesc)] + [vp] * 7 + [i64] + [vp] * 4 + \
            [sz, vp]
        L.precog_delta_encode.restype = ctypes.c_int
        L.precog_delta_step.argtypes = [ctypes.POINTER(DeltaDesc)] + [vp] * 6 + [i64] + [vp] * 3
        L.precog_delta_step.restype = ctypes.c_int
        L.precog_conv_encode.argtypes = [ctypes.POINTER(ConvDesc)] + [vp] * 5 + [i64] + [vp] * 4
        L.precog_conv_encode.restype = ctypes.c_int
        L.precog_conv_step.argtypes = [ctypes.POINTER(ConvDesc)] + [vp] * 4 + [i64] + [vp] * 3
        L.precog_conv_step.restype = ctypes.c_int
        L.precog_score_workspace_bytes.argtypes = [i64, i64, i64]
        L.precog_score_workspace_bytes.restype = sz
        L.precog_score_tokens.argtypes = [vp, ctypes.c_int, i64, i64, i64, vp, i64] + [vp] * 5 + \
            [sz, vp]
        L.precog_score_tokens.restype = ctypes.c_int
        L.precog_status_string.argtypes = [ctypes.c_int]
        L.precog_status_string.restype = ctypes.c_char_p
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().precog_status_string(int(status)).decode()


def _ptr(t):
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream(stream):
    if stream is None:
        # the current stream's handle as an integer: building torch's Stream
        # object for it takes 2.8 us a call, these two queries 0.2
        if torch.cuda.is_initialized():
            return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _row_elems(t):
    """Elements of one row of t, without a view of it; no row: t[0]'s IndexError."""
    return t.numel() // t.shape[0] if t.shape[0] else t[0].numel()


def _check(fn, st):
    if st != 0:
        raise PrecogError(fn, st)


def scan_desc(batch, seqlen, dim, dstate, in_dtype=BF16, out_dtype=F32, state_dtype=F32,
              h0_batch_stride=0, hT_batch_stride=0, chunk=0) -> ScanDesc:
    return ScanDesc(batch, seqlen, dim, dstate, in_dtype, out_dtype, state_dtype,
                    h0_batch_stride, hT_batch_stride, chunk)


def scan_workspace_bytes(desc: ScanDesc) -> int:
    return int(lib().precog_scan_workspace_bytes(ctypes.byref(desc)))


def scan_encode(desc: ScanDesc, x, dt, A, B, C=None, z=None, Dskip=None, h0=None, y=None,
                hT=None, workspace=None, workspace_bytes=0, stream=None):
    """precog_scan_encode on device tensors (or raw device pointers)."""
    st = lib().precog_scan_encode(ctypes.byref(desc), _ptr(x), _ptr(dt), _ptr(A), _ptr(B),
                                  _ptr(C), _ptr(z), _ptr(Dskip), _ptr(h0), _ptr(y), _ptr(hT),
                                  _ptr(workspace), int(workspace_bytes), _stream(stream))
    _check("precog_scan_encode", st)


def scan_encode_indexed(desc: ScanDesc, x, dt, A, B, C=None, z=None, Dskip=None, store=None,
                        store_rows=0, h0_idx=None, y=None, hT=None, workspace=None,
                        workspace_bytes=0, stream=None, h0_score=None, k=1, tau=1.0):
    """precog_scan_encode_indexed on device tensors (or raw device pointers)."""
    st = lib().precog_scan_encode_indexed(ctypes.byref(desc), _ptr(x), _ptr(dt), _ptr(A), _ptr(B),
                                          _ptr(C), _ptr(z), _ptr(Dskip), _ptr(store),
                                          int(store_rows), _ptr(h0_idx), _ptr(h0_score), int(k),
                                          float(tau), _ptr(y), _ptr(hT), _ptr(workspace),
                                          int(workspace_bytes), _stream(stream))
    _check("precog_scan_encode_indexed", st)


def scan_trajectory(desc: ScanDesc, x, dt, A, B, C=None, z=None, Dskip=None, h0=None, y=None,
                    hT=None, traj=None, every=1, workspace=None, workspace_bytes=0, stream=None):
    """precog_scan_trajectory on device tensors (or raw device pointers)."""
    st = lib().precog_scan_trajectory(ctypes.byref(desc), _ptr(x), _ptr(dt), _ptr(A), _ptr(B),
                                      _ptr(C), _ptr(z), _ptr(Dskip), _ptr(h0), _ptr(y), _ptr(hT),
                                      _ptr(traj), int(every), _ptr(workspace),
                                      int(workspace_bytes), _stream(stream))
    _check("precog_scan_trajectory", st)


def scan_complex_workspace_bytes(desc: ScanDesc) -> int:
    return int(lib().precog_scan_complex_workspace_bytes(ctypes.byref(desc)))


def scan_complex_raw(desc: ScanDesc, x, dt, A_re, A_im, B, C=None, z=None, Dskip=None, h0=None,
                     y=None, hT=None, workspace=None, workspace_bytes=0, stream=None):
    """precog_scan_complex on device tensors (or raw device pointers)."""
    st = lib().precog_scan_complex(ctypes.byref(desc), _ptr(x), _ptr(dt), _ptr(A_re), _ptr(A_im),
                                   _ptr(B), _ptr(C), _ptr(z), _ptr(Dskip), _ptr(h0), _ptr(y),
                                   _ptr(hT), _ptr(workspace), int(workspace_bytes),
                                   _stream(stream))
    _check("precog_scan_complex", st)


def retrieve_workspace_bytes(Q, M, E) -> int:
    return int(lib().precog_retrieve_workspace_bytes(Q, M, E))


def retrieve_top1(query, index, idx, workspace, workspace_bytes=None, stream=None):
    Q, E = query.shape
    M = index.shape[0]
    if workspace_bytes is None:
        workspace_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    st = lib().precog_retrieve_top1(_ptr(query), _ptr(index), Q, M, E, _ptr(idx),
                                    _ptr(workspace), int(workspace_bytes), _stream(stream))
    _check("precog_retrieve_top1", st)


def retrieve_top1_noalloc(query, index, idx, stream=None):
    """precog_retrieve_top1_noalloc: top-1 with the library's fixed device
    array as workspace (nothing allocated)."""
    Q, E = query.shape
    M = index.shape[0]
    st = lib().precog_retrieve_top1_noalloc(_ptr(query), _ptr(index), Q, M, E, _ptr(idx),
                                            _stream(stream))
    _check("precog_retrieve_top1_noalloc", st)


NOALLOC_SCRATCH_BYTES = 32 << 20


def retrieve_topk(query, index, k, idx, score, workspace, workspace_bytes=None, stream=None):
    Q, E = query.shape
    M = index.shape[0]
    if workspace_bytes is None:
        workspace_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    st = lib().precog_retrieve_topk(_ptr(query), _ptr(index), Q, M, E, int(k), _ptr(idx),
                                    _ptr(score), _ptr(workspace), int(workspace_bytes),
                                    _stream(stream))
    _check("precog_retrieve_topk", st)


def retrieve_index_bytes(M, E) -> int:
    return int(lib().precog_retrieve_index_bytes(M, E))


def retrieve_prepare(index, prepared, stream=None):
    """precog_retrieve_prepare: the prepared form of index [M, E] into `prepared`."""
    M, E = index.shape
    nbytes = prepared.numel() * prepared.element_size()
    st = lib().precog_retrieve_prepare(_ptr(index), M, E, _ptr(prepared), int(nbytes),
                                       _stream(stream))
    _check("precog_retrieve_prepare", st)


def retrieve_topk_prepared(query, index, prepared, k, idx, score, workspace, workspace_bytes=None,
                           stream=None):
    Q, E = query.shape
    M = index.shape[0]
    if workspace_bytes is None:
        workspace_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    pbytes = prepared.numel() * prepared.element_size()
    st = lib().precog_retrieve_topk_prepared(_ptr(query), _ptr(index), _ptr(prepared), int(pbytes),
                                             Q, M, E, int(k), _ptr(idx), _ptr(score),
                                             _ptr(workspace), int(workspace_bytes),
                                             _stream(stream))
    _check("precog_retrieve_topk_prepared", st)


def query_workspace_bytes(desc: ScanDesc, M, E) -> int:
    return int(lib().precog_query_workspace_bytes(ctypes.byref(desc), int(M), int(E)))


def query_top1_prefill(desc: ScanDesc, query, index, store, idx, x, dt, A, B, C=None, z=None,
                       Dskip=None, y=None, hT=None, workspace=None, workspace_bytes=None,
                       prepared=None, stream=None):
    """precog_query_top1_prefill: exact top-1 of each query, then the prefill
    of batch row b from store row idx[b] (one call)."""
    M, E = index.shape
    if workspace_bytes is None:
        workspace_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    pbytes = prepared.numel() * prepared.element_size() if prepared is not None else 0
    st = lib().precog_query_top1_prefill(ctypes.byref(desc), _ptr(query), _ptr(index),
                                         _ptr(prepared), int(pbytes), int(M), int(E), _ptr(store),
                                         _ptr(idx), _ptr(x), _ptr(dt), _ptr(A), _ptr(B), _ptr(C),
                                         _ptr(z), _ptr(Dskip), _ptr(y), _ptr(hT), _ptr(workspace),
                                         int(workspace_bytes), _stream(stream))
    _check("precog_query_top1_prefill", st)


def inject_compose(store, idx, score, tau, h0, stream=None):
    M = store.shape[0]
    S = _row_elems(store) if M > 0 else _row_elems(h0)
    Q, k = idx.shape
    st = lib().precog_inject_compose(_ptr(store), _DT[store.dtype], M, S, _ptr(idx), _ptr(score),
                                     Q, k, float(tau), _ptr(h0), _DT[h0.dtype], _stream(stream))
    _check("precog_inject_compose", st)


def inject_gather(store, idx, h0, stream=None):
    M = store.shape[0]
    S = _row_elems(store) if M > 0 else _row_elems(h0)
    st = lib().precog_inject_gather(_ptr(store), _DT[store.dtype], M, S, _ptr(idx),
                                    idx.shape[0], _ptr(h0), _DT[h0.dtype], _stream(stream))
    _check("precog_inject_gather", st)


def inject_fuse(episodic_store, episodic_idx, episodic_score, corpus_store, corpus_idx,
                corpus_score, k, tau, h0, semantic=None, semantic_row=None, lam=1.0,
                stream=None):
    """precog_inject_fuse: stores [M, ...] (same dtype), candidate lists
    [Q, k_e] / [Q, k_c] (int32 rows, fp64 scores), h0 [Q, ...]."""
    Q = h0.shape[0]
    S = _row_elems(h0) if Q > 0 else 0
    ke = episodic_idx.shape[1] if episodic_idx is not None else 0
    kc = corpus_idx.shape[1] if corpus_idx is not None else 0
    st = lib().precog_inject_fuse(_ptr(episodic_store), episodic_store.shape[0],
                                  _ptr(episodic_idx), _ptr(episodic_score), ke,
                                  _ptr(corpus_store), corpus_store.shape[0], _ptr(corpus_idx),
                                  _ptr(corpus_score), kc, _DT[episodic_store.dtype], S, Q, int(k),
                                  float(tau), _ptr(semantic), _ptr(semantic_row),
                                  semantic.shape[0] if semantic is not None else 0, float(lam),
                                  _ptr(h0), _DT[h0.dtype], _stream(stream))
    _check("precog_inject_fuse", st)


def smc_route(emb, domain_protos, sub_protos, domain_out, sub_out, flat_out=None, stream=None):
    C, E = emb.shape
    st = lib().precog_smc_route(_ptr(emb), C, E, _ptr(domain_protos), domain_protos.shape[0],
                                _ptr(sub_protos), sub_protos.shape[1], _ptr(domain_out),
                                _ptr(sub_out), _ptr(flat_out), _stream(stream))
    _check("precog_smc_route", st)


def smc_consolidate(states, contrib, target, alpha, stream=None):
    R = states.shape[0]
    S = _row_elems(states) if R > 0 else 0
    C = target.shape[0]
    st = lib().precog_smc_consolidate(_ptr(states), _DT[states.dtype], R, S, _ptr(contrib),
                                      _DT[contrib.dtype], _ptr(target), C, float(alpha),
                                      _stream(stream))
    _check("precog_smc_consolidate", st)


def delta_desc(batch, seqlen, k_heads, v_heads, k_dim, v_dim, in_dtype=BF16, out_dtype=F32,
               state_dtype=F32, q_stride=0, k_stride=0, v_stride=0, h0_batch_stride=0,
               hT_batch_stride=0, qk_norm=False, eps=1e-6, scale=0.0) -> DeltaDesc:
    return DeltaDesc(batch, seqlen, k_heads, v_heads, k_dim, v_dim, q_stride, k_stride, v_stride,
                     h0_batch_stride, hT_batch_stride, in_dtype, out_dtype, state_dtype,
                     1 if qk_norm else 0, eps, scale)


def delta_workspace_bytes(desc: DeltaDesc, packed=False) -> int:
    return int(lib().precog_delta_workspace_bytes(ctypes.byref(desc), int(bool(packed))))


def delta_encode(desc: DeltaDesc, q, k, v, g=None, beta=None, starts=None, h0=None, h0_rows=0,
                 h0_idx=None, o=None, hT=None, workspace=None, workspace_bytes=0, stream=None):
    """precog_delta_encode on device tensors (or raw device pointers)."""
    st = lib().precog_delta_encode(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _ptr(g),
                                   _ptr(beta), _ptr(starts), _ptr(h0), int(h0_rows), _ptr(h0_idx),
                                   _ptr(o), _ptr(hT), _ptr(workspace), int(workspace_bytes),
                                   _stream(stream))
    _check("precog_delta_encode", st)


def delta_step_raw(desc: DeltaDesc, q, k, v, g, beta, states, state_rows, slots, o=None,
                   stream=None):
    """precog_delta_step on device tensors (or raw device pointers)."""
    st = lib().precog_delta_step(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _ptr(g),
                                 _ptr(beta), _ptr(states), int(state_rows), _ptr(slots), _ptr(o),
                                 _stream(stream))
    _check("precog_delta_step", st)


def conv_desc(batch, seqlen, dim, width, in_dtype=BF16, out_dtype=BF16, x_stride=0,
              silu=True) -> ConvDesc:
    return ConvDesc(batch, seqlen, dim, width, x_stride, in_dtype, out_dtype, 1 if silu else 0)


def conv_encode(desc: ConvDesc, x, w, bias=None, starts=None, tail0=None, tail_rows=0,
                tail_idx=None, y=None, tailT=None, stream=None):
    """precog_conv_encode on device tensors (or raw device pointers)."""
    st = lib().precog_conv_encode(ctypes.byref(desc), _ptr(x), _ptr(w), _ptr(bias), _ptr(starts),
                                  _ptr(tail0), int(tail_rows), _ptr(tail_idx), _ptr(y),
                                  _ptr(tailT), _stream(stream))
    _check("precog_conv_encode", st)


def conv_step_raw(desc: ConvDesc, x, w, bias, tails, tail_rows, slots, y=None, stream=None):
    """precog_conv_step on device tensors (or raw device pointers)."""
    st = lib().precog_conv_step(ctypes.byref(desc), _ptr(x), _ptr(w), _ptr(bias), _ptr(tails),
                                int(tail_rows), _ptr(slots), _ptr(y), _stream(stream))
    _check("precog_conv_step", st)


def score_workspace_bytes(T, V, top) -> int:
    return int(lib().precog_score_workspace_bytes(int(T), int(V), int(top)))


def score_tokens_raw(logits, logits_dtype, T, V, row_stride, token, top, logprob, entropy=None,
                     top_id=None, top_logprob=None, workspace=None, workspace_bytes=0,
                     stream=None):
    """precog_score_tokens on device tensors (or raw device pointers)."""
    st = lib().precog_score_tokens(_ptr(logits), int(logits_dtype), int(T), int(V),
                                   int(row_stride), _ptr(token), int(top), _ptr(logprob),
                                   _ptr(entropy), _ptr(top_id), _ptr(top_logprob),
                                   _ptr(workspace), int(workspace_bytes), _stream(stream))
    _check("precog_score_tokens", st)


# ----------------------------------------------------------------------------
# Convenience wrappers that allocate outputs and workspace with torch.
# ----------------------------------------------------------------------------
def scan(x, dt, A, B, C=None, z=None, Dskip=None, h0=None, *, out_dtype=torch.float32,
         state_dtype=torch.float32, want_y=True, want_hT=True, chunk=0, hT=None,
         hT_batch_stride=0, h0_batch_stride=0, stream=None):
    """Runs the scan; returns (y, hT) (None where not requested)."""
    Bt, L, D = x.shape
    N = A.shape[1]
    desc = scan_desc(Bt, L, D, N, _DT[x.dtype], _DT[out_dtype], _DT[state_dtype],
                     h0_batch_stride, hT_batch_stride, chunk)
    y = torch.empty((Bt, L, D), dtype=out_dtype, device=x.device) if want_y else None
    if want_hT and hT is None:
        hT = torch.empty((Bt, D, N), dtype=state_dtype, device=x.device)
    nbytes = scan_workspace_bytes(desc)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=x.device) if nbytes else None
    scan_encode(desc, x, dt, A, B, C, z, Dskip, h0, y, hT if want_hT else None, ws, nbytes,
                stream)
    return y, (hT if want_hT else None)


def scan_from_store(x, dt, A, B, store, idx, C=None, z=None, Dskip=None, *, score=None, tau=1.0,
                    out_dtype=torch.float32, want_y=True, want_hT=True, chunk=0, stream=None):
    """Runs the scan with batch row b starting from store[idx[b]] (store
    [M, D, N] in the state dtype, idx [B] int32), or, with score [B, k] fp64
    and idx [B, k], from the softmax composition of those k rows; returns
    (y, hT)."""
    Bt, L, D = x.shape
    N = A.shape[1]
    state_dtype = store.dtype
    desc = scan_desc(Bt, L, D, N, _DT[x.dtype], _DT[out_dtype], _DT[state_dtype], 0, 0, chunk)
    y = torch.empty((Bt, L, D), dtype=out_dtype, device=x.device) if want_y else None
    hT = torch.empty((Bt, D, N), dtype=state_dtype, device=x.device) if want_hT else None
    nbytes = scan_workspace_bytes(desc)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=x.device) if nbytes else None
    k = 1 if score is None else score.shape[1]
    scan_encode_indexed(desc, x, dt, A, B, C, z, Dskip, store, store.shape[0], idx, y, hT, ws,
                        nbytes, stream, h0_score=score, k=k, tau=tau)
    return y, hT


def query_prefill(query, index, store, x, dt, A, B, C=None, z=None, Dskip=None, *,
                  prepared=None, out_dtype=torch.float32, want_y=True, want_hT=True, chunk=0,
                  stream=None):
    """The query-time path in one call: idx = exact top-1 of each query row
    over index, then the scan of batch row b from store[idx[b]] (store
    [M, D, N] in the state dtype); returns (idx, y, hT)."""
    Bt, L, D = x.shape
    N = A.shape[1]
    M, E = index.shape
    desc = scan_desc(Bt, L, D, N, _DT[x.dtype], _DT[out_dtype], _DT[store.dtype], 0, 0, chunk)
    idx = torch.empty(Bt, dtype=torch.int32, device=x.device)
    y = torch.empty((Bt, L, D), dtype=out_dtype, device=x.device) if want_y else None
    hT = torch.empty((Bt, D, N), dtype=store.dtype, device=x.device) if want_hT else None
    nbytes = query_workspace_bytes(desc, M, E)
    ws = torch.empty(max(nbytes, 16), dtype=torch.uint8, device=x.device)
    query_top1_prefill(desc, query, index, store, idx, x, dt, A, B, C, z, Dskip, y, hT, ws, nbytes,
                       prepared, stream)
    return idx, y, hT


def trajectory(x, dt, A, B, every, C=None, z=None, Dskip=None, h0=None, *,
               out_dtype=torch.float32, state_dtype=torch.float32, want_y=False, want_hT=False,
               chunk=0, stream=None):
    """Runs the scan keeping every `every`-th state; returns (traj, y, hT)."""
    Bt, L, D = x.shape
    N = A.shape[1]
    desc = scan_desc(Bt, L, D, N, _DT[x.dtype], _DT[out_dtype], _DT[state_dtype], 0, 0, chunk)
    # every < 1 is left to the library to reject
    traj = torch.empty((Bt, L // every if every >= 1 else 0, D, N), dtype=state_dtype,
                       device=x.device)
    y = torch.empty((Bt, L, D), dtype=out_dtype, device=x.device) if want_y else None
    hT = torch.empty((Bt, D, N), dtype=state_dtype, device=x.device) if want_hT else None
    nbytes = scan_workspace_bytes(desc)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=x.device) if nbytes else None
    scan_trajectory(desc, x, dt, A, B, C, z, Dskip, h0, y, hT, traj, every, ws, nbytes, stream)
    return traj, y, hT


def scan_complex(x, dt, A_re, A_im, B, C=None, z=None, Dskip=None, h0=None, *,
                 out_dtype=torch.float32, state_dtype=torch.float32, want_y=True, want_hT=True,
                 chunk=0, stream=None):
    """Complex-A scan; returns (y, hT) with hT [Bt, D, N, 2] (None where not requested)."""
    Bt, L, D = x.shape
    N = A_re.shape[1]
    desc = scan_desc(Bt, L, D, N, _DT[x.dtype], _DT[out_dtype], _DT[state_dtype], chunk=chunk)
    y = torch.empty((Bt, L, D), dtype=out_dtype, device=x.device) if want_y else None
    hT = torch.empty((Bt, D, N, 2), dtype=state_dtype, device=x.device) if want_hT else None
    nbytes = scan_complex_workspace_bytes(desc)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=x.device) if nbytes else None
    scan_complex_raw(desc, x, dt, A_re, A_im, B, C, z, Dskip, h0, y, hT, ws, nbytes, stream)
    return y, hT


def top1(query, index, stream=None):
    Q, E = query.shape
    M = index.shape[0]
    idx = torch.empty(Q, dtype=torch.int32, device=query.device)
    nbytes = retrieve_workspace_bytes(Q, M, E)
    ws = torch.empty(max(nbytes, 16), dtype=torch.uint8, device=query.device)
    retrieve_top1(query, index, idx, ws, nbytes, stream)
    return idx


def topk(query, index, k, stream=None):
    """Exact top-k: returns (idx int32 [Q, k], score fp64 [Q, k])."""
    Q, E = query.shape
    M = index.shape[0]
    idx = torch.empty((Q, k), dtype=torch.int32, device=query.device)
    score = torch.empty((Q, k), dtype=torch.float64, device=query.device)
    nbytes = retrieve_workspace_bytes(Q, M, E)
    ws = torch.empty(max(nbytes, 16), dtype=torch.uint8, device=query.device)
    retrieve_topk(query, index, k, idx, score, ws, nbytes, stream)
    return idx, score


def prepare_index(index, stream=None):
    """The prepared form of index [M, E] (a uint8 device tensor)."""
    M, E = index.shape
    prepared = torch.empty(max(retrieve_index_bytes(M, E), 16), dtype=torch.uint8,
                           device=index.device)
    retrieve_prepare(index, prepared, stream)
    return prepared


def topk_prepared(query, index, prepared, k, want_score=True, stream=None):
    """Exact top-k over a prepared index: (idx int32 [Q, k], score fp64 [Q, k] or None)."""
    Q, E = query.shape
    M = index.shape[0]
    idx = torch.empty((Q, k), dtype=torch.int32, device=query.device)
    score = torch.empty((Q, k), dtype=torch.float64, device=query.device) if want_score else None
    nbytes = retrieve_workspace_bytes(Q, M, E)
    ws = torch.empty(max(nbytes, 16), dtype=torch.uint8, device=query.device)
    retrieve_topk_prepared(query, index, prepared, k, idx, score, ws, nbytes, stream)
    return idx, score


def compose(store, idx, score, tau=1.0, out_dtype=None, stream=None):
    out_dtype = out_dtype or store.dtype
    h0 = torch.empty((idx.shape[0],) + tuple(store.shape[1:]), dtype=out_dtype,
                     device=store.device)
    inject_compose(store, idx, score, tau, h0, stream)
    return h0


def route(emb, domain_protos, sub_protos, stream=None):
    """Two-stage routing: returns (domain int32 [C], sub int32 [C], flat int32 [C])."""
    C = emb.shape[0]
    outs = [torch.empty(C, dtype=torch.int32, device=emb.device) for _ in range(3)]
    smc_route(emb, domain_protos, sub_protos, *outs, stream=stream)
    return tuple(outs)


def gather(store, idx, out_dtype=None, stream=None):
    out_dtype = out_dtype or store.dtype
    h0 = torch.empty((idx.shape[0],) + tuple(store.shape[1:]), dtype=out_dtype,
                     device=store.device)
    inject_gather(store, idx, h0, stream)
    return h0


# The gated-delta layer and token scoring.  These wrappers check what the
# library cannot see (types, shapes, strides and devices of the tensors).  They
# have no backward pass, and refuse tensors whose gradient they would lose.
def _forward_only(*tensors):
    if torch.is_grad_enabled():
        for t in tensors:
            if t is not None and t.requires_grad:
                raise ValueError("there is no backward pass: call under torch.no_grad(), or with "
                                 "detached tensors")


def _same(name, t, dtype, shape, device, contiguous=True):
    """t is a tensor of that type, shape and device (and contiguous), or a ValueError."""
    if t.dtype is dtype and t.shape == shape and t.get_device() == device and \
            (not contiguous or t.is_contiguous()):
        return
    raise ValueError("%s must be %s%s %s on cuda:%d, not %s %s with strides %s on %s"
                     % (name, "contiguous " if contiguous else "", dtype, list(shape), device,
                        t.dtype, list(t.shape), list(t.stride()), t.device))


def _code(name, dtype, allowed):
    if dtype not in allowed:
        raise ValueError("%s must be one of %s, not %s" % (name, ", ".join(map(str, allowed)), dtype))
    return _DT[dtype]


_IO = (torch.float32, torch.bfloat16)
_STATE = (torch.float32, torch.float16)


def _device_of(t):
    """Number of t's device, which must be the current one: the library launches there."""
    if not t.is_cuda:
        raise ValueError("tensors must be on the GPU, not on %s" % t.device)
    device = t.get_device()
    if device != torch._C._cuda_getDevice():
        raise ValueError("tensors are on cuda:%d but the current device is cuda:%d"
                         % (device, torch._C._cuda_getDevice()))
    return device


def _token_stride(name, t, lead):
    """Elements between tokens of t (0: it is dense), whose first `lead` axes are
    the tokens' (a [B, L] batch, or one packed axis) and whose others are one
    token, which has to be dense: a slice of a wider tensor's last axis is."""
    if t.is_contiguous():
        return 0
    shape, strides, inner = t.shape, t.stride(), 1
    for i in range(len(shape) - 1, lead - 1, -1):
        if shape[i] != 1 and strides[i] != inner:
            raise ValueError("%s: the elements of one token must be contiguous" % name)
        inner *= shape[i]
    stride = strides[lead - 1]
    if lead == 2 and shape[0] > 1:
        if shape[1] == 1:
            stride = strides[0]
        elif strides[0] != stride * shape[1]:
            raise ValueError("%s: the rows of a batch must follow one another" % name)
    elif shape[lead - 1] == 1:
        return 0
    if stride < inner:
        raise ValueError("%s: tokens must not overlap" % name)
    return stride


_CURRENT_STREAM = contextlib.nullcontext()


def _own_stream(stream):
    """Context in which torch allocates from the stream that the kernels run on."""
    if stream is None:
        return _CURRENT_STREAM
    return torch.cuda.stream(torch.cuda.ExternalStream(stream) if isinstance(stream, int)
                             else stream)


def _at(t):
    return None if t is None else t.data_ptr()


def _handle(stream, device):
    return torch._C._cuda_getCurrentRawStream(device) if stream is None else _stream(stream)


def _delta_args(q, k, v, g, beta, lead, out_dtype, state_dtype):
    dev = _device_of(k)
    _forward_only(q, k, v, g, beta)
    if k.dim() != lead + 2 or v.dim() != lead + 2:
        raise ValueError("k and v must have %d axes" % (lead + 2))
    dtype = k.dtype
    code = _code("k", dtype, _IO)
    tokens, (Hk, K), (Hv, V) = k.shape[:lead], k.shape[lead:], v.shape[lead:]
    if q is not None:
        _same("q", q, dtype, k.shape, dev, False)
    _same("v", v, dtype, tokens + (Hv, V), dev, False)
    gates = tokens + (Hv,)
    if g is not None:
        _same("g", g, torch.float32, gates, dev)
    if beta is not None:
        _same("beta", beta, torch.float32, gates, dev)
    strides = (0 if q is None else _token_stride("q", q, lead), _token_stride("k", k, lead),
               _token_stride("v", v, lead))
    return dev, (Hk, Hv, K, V), (code, _code("out_dtype", out_dtype, _IO),
                                 _code("state_dtype", state_dtype, _STATE)), strides


def delta(q, k, v, g=None, beta=None, h0=None, *, starts=None, h0_idx=None, qk_norm=False,
          eps=1e-6, scale=0.0, out_dtype=torch.float32, state_dtype=None, want_o=True,
          want_hT=True, hT=None, stream=None):
    """The gated delta rule over whole sequences; returns (o, hT) (None where
    not wanted).

    q, k [B, L, Hk, K] and v [B, L, Hv, V], or with starts [B + 1] (int32) the
    packed [T, Hk, K] and [T, Hv, V]; g (log decay) and beta [..., Hv] fp32;
    h0 [B, Hv, K, V] or, with h0_idx [B] int32, a store [rows, Hv, K, V] whose
    rows h0_idx names the sequences start from.  q None with want_o False: the
    states only.  hT: a tensor for the states (h0 itself: in place).  Rows of o
    whose token is in none of starts' sequences are not written."""
    lead = 2 if starts is None else 1
    if q is None and want_o:
        raise ValueError("o needs q")
    state_dtype = state_dtype or (h0.dtype if h0 is not None else torch.float32)
    dev, (Hk, Hv, K, V), codes, strides = _delta_args(q, k, v, g, beta, lead, out_dtype,
                                                      state_dtype)
    if starts is not None:
        if starts.dim() != 1 or starts.shape[0] < 1:
            raise ValueError("starts must have B + 1 entries")
        _same("starts", starts, torch.int32, starts.shape, dev)
        B, L = starts.shape[0] - 1, k.shape[0]
    else:
        B, L = k.shape[0], k.shape[1]
    if h0_idx is not None:
        _same("h0_idx", h0_idx, torch.int32, (B,), dev)
        if h0 is None:
            raise ValueError("h0_idx needs a store h0")
    if h0 is not None:
        _forward_only(h0)
        rows = h0.shape[0] if h0_idx is not None else B
        _same("h0", h0, state_dtype, (rows, Hv, K, V), dev)
    if hT is not None:
        _same("hT", hT, state_dtype, (B, Hv, K, V), dev)
    desc = DeltaDesc(B, L, Hk, Hv, K, V, *strides, 0, 0, *codes, 1 if qk_norm else 0, eps, scale)
    ref, so = ctypes.byref(desc), lib()
    with _own_stream(stream):
        o = torch.empty(v.shape, dtype=out_dtype, device=dev) if want_o else None
        if want_hT and hT is None:
            hT = torch.empty((B, Hv, K, V), dtype=state_dtype, device=dev)
        nbytes = so.precog_delta_workspace_bytes(ref, 0 if starts is None else 1)
        ws = torch.empty(nbytes, dtype=torch.uint8, device=dev) if nbytes else None
    _check("precog_delta_encode", so.precog_delta_encode(
        ref, _at(q), k.data_ptr(), v.data_ptr(), _at(g), _at(beta), _at(starts), _at(h0),
        0 if h0 is None else h0.shape[0], _at(h0_idx), _at(o), _at(hT), _at(ws), nbytes,
        _handle(stream, dev)))
    return o, hT


def delta_step(q, k, v, g, beta, states, slots, *, qk_norm=False, eps=1e-6, scale=0.0,
               out_dtype=torch.float32, want_o=True, stream=None):
    """One token of each of n sessions: q, k [n, Hk, K], v [n, Hv, V], g and
    beta [n, Hv] fp32 or None; row i's state is states[slots[i]] (states
    [rows, Hv, K, V], slots int32), updated in place.  Returns o [n, Hv, V]; the
    rows of o whose slot is outside the states are not written."""
    dev, (Hk, Hv, K, V), codes, strides = _delta_args(q, k, v, g, beta, 1, out_dtype, states.dtype)
    if q is None and want_o:
        raise ValueError("o needs q")
    n = k.shape[0]
    _forward_only(states)
    _same("states", states, states.dtype, (states.shape[0], Hv, K, V), dev)
    _same("slots", slots, torch.int32, (n,), dev)
    desc = DeltaDesc(n, 1, Hk, Hv, K, V, *strides, 0, 0, *codes, 1 if qk_norm else 0, eps, scale)
    with _own_stream(stream):
        o = torch.empty((n, Hv, V), dtype=out_dtype, device=dev) if want_o else None
    _check("precog_delta_step", lib().precog_delta_step(
        ctypes.byref(desc), _at(q), k.data_ptr(), v.data_ptr(), _at(g), _at(beta),
        states.data_ptr(), states.shape[0], slots.data_ptr(), _at(o), _handle(stream, dev)))
    return o


def _conv_args(x, w, bias, lead, out_dtype):
    dev = _device_of(x)
    _forward_only(x, w, bias)
    if x.dim() != lead + 1 or w.dim() != 2:
        raise ValueError("x must have %d axes and w two" % (lead + 1))
    D, W = x.shape[-1], w.shape[1]
    _same("w", w, torch.float32, (D, W), dev)
    if bias is not None:
        _same("bias", bias, torch.float32, (D,), dev)
    return dev, D, W, (_code("x", x.dtype, _IO), _code("out_dtype", out_dtype, _IO)), \
        _token_stride("x", x, lead)


def conv(x, w, bias=None, tail0=None, *, starts=None, tail_idx=None, silu=True, out_dtype=None,
         want_y=True, want_tail=True, tailT=None, stream=None):
    """The short causal convolution; returns (y, tailT).  x [B, L, D], or with
    starts [B + 1] (int32) the packed [T, D]; w [D, W] and bias [D] fp32; tail0
    [B, W - 1, D], or with tail_idx [B] int32 a store of tails.  tailT: a tensor
    for the tails (tail0 itself: in place).  Rows of y whose token is in none of
    starts' sequences are not written."""
    lead = 2 if starts is None else 1
    out_dtype = out_dtype or x.dtype
    dev, D, W, codes, stride = _conv_args(x, w, bias, lead, out_dtype)
    if starts is not None:
        if starts.dim() != 1 or starts.shape[0] < 1:
            raise ValueError("starts must have B + 1 entries")
        _same("starts", starts, torch.int32, starts.shape, dev)
        B, L = starts.shape[0] - 1, x.shape[0]
    else:
        B, L = x.shape[0], x.shape[1]
    if tail_idx is not None:
        _same("tail_idx", tail_idx, torch.int32, (B,), dev)
        if tail0 is None:
            raise ValueError("tail_idx needs a store tail0")
    if tail0 is not None:
        _forward_only(tail0)
        rows = tail0.shape[0] if tail_idx is not None else B
        _same("tail0", tail0, x.dtype, (rows, W - 1, D), dev)
    if tailT is not None:
        _same("tailT", tailT, x.dtype, (B, W - 1, D), dev)
    desc = ConvDesc(B, L, D, W, stride, *codes, 1 if silu else 0)
    with _own_stream(stream):
        y = torch.empty(x.shape, dtype=out_dtype, device=dev) if want_y else None
        if want_tail and tailT is None:
            tailT = torch.empty((B, max(W - 1, 0), D), dtype=x.dtype, device=dev)
    _check("precog_conv_encode", lib().precog_conv_encode(
        ctypes.byref(desc), x.data_ptr(), w.data_ptr(), _at(bias), _at(starts), _at(tail0),
        0 if tail0 is None else tail0.shape[0], _at(tail_idx), _at(y), _at(tailT),
        _handle(stream, dev)))
    return y, tailT


def conv_step(x, w, bias, tails, slots, *, silu=True, out_dtype=None, stream=None):
    """One token of each of n sessions: x [n, D]; row i's tail is tails[slots[i]]
    (tails [rows, W - 1, D], slots int32), moved on in place.  Returns y [n, D];
    the rows of y whose slot is outside the tails are not written."""
    out_dtype = out_dtype or x.dtype
    dev, D, W, codes, stride = _conv_args(x, w, bias, 1, out_dtype)
    n = x.shape[0]
    _forward_only(tails)
    _same("tails", tails, x.dtype, (tails.shape[0], W - 1, D), dev)
    _same("slots", slots, torch.int32, (n,), dev)
    desc = ConvDesc(n, 1, D, W, stride, *codes, 1 if silu else 0)
    with _own_stream(stream):
        y = torch.empty((n, D), dtype=out_dtype, device=dev)
    _check("precog_conv_step", lib().precog_conv_step(
        ctypes.byref(desc), x.data_ptr(), w.data_ptr(), _at(bias), tails.data_ptr(),
        tails.shape[0], slots.data_ptr(), y.data_ptr(), _handle(stream, dev)))
    return y


def score_tokens(logits, token=None, top=0, *, want_entropy=True, stream=None):
    """Log probabilities of token [T] (int32) under logits [T, V] (fp32, bf16 or
    fp16; rows may be strided), with the entropies and the `top` alternatives:
    (logprob [T], entropy [T], top_id [T, top], top_logprob [T, top]), None where
    not wanted."""
    dev = _device_of(logits)
    _forward_only(logits)
    if logits.dim() != 2:
        raise ValueError("logits must be [T, V]")
    T, V = logits.shape
    code = _code("logits", logits.dtype, (torch.float32, torch.bfloat16, torch.float16))
    if V > 1 and logits.stride(1) != 1:
        raise ValueError("logits: the elements of a row must be contiguous")
    stride = logits.stride(0) if T > 1 else V
    if stride < V:
        raise ValueError("logits: rows must not overlap")
    if not 0 <= top <= 64:
        raise ValueError("top must be 0..64, not %d" % top)
    if token is not None:
        _same("token", token, torch.int32, (T,), dev)
    L = lib()
    nbytes = L.precog_score_workspace_bytes(T, V, top)
    with _own_stream(stream):
        logprob = torch.empty(T, dtype=torch.float32, device=dev) if token is not None else None
        entropy = torch.empty(T, dtype=torch.float32, device=dev) if want_entropy else None
        top_id = torch.empty((T, top), dtype=torch.int32, device=dev) if top else None
        top_logprob = torch.empty((T, top), dtype=torch.float32, device=dev) if top else None
        ws = torch.empty(nbytes, dtype=torch.uint8, device=dev) if nbytes else None
    _check("precog_score_tokens", L.precog_score_tokens(
        logits.data_ptr(), code, T, V, stride, _at(token), top, _at(logprob), _at(entropy),
        _at(top_id), _at(top_logprob), _at(ws), nbytes, _handle(stream, dev)))
    return logprob, entropy, top_id, top_logprob
