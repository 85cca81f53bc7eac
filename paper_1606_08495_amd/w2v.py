"""Thin ctypes binding over libw2v_shard.so -- same names as include/w2v_shard.h.

Argument marshalling only: every step of the shard path runs in the library's HIP kernels.
PyTorch supplies device memory (``tensor.data_ptr()``) and the stream.  There is no fallback: if
the library has not been built, or a call fails, an exception is raised.
"""
import contextlib
import ctypes
import os

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("W2V_LIB", os.path.join(_HERE, "libw2v_shard.so"))
_lib = None

PHASES = ["neg", "dot", "coeff", "sort", "uside", "wside", "apply", "pairs"]
K_MAX, D_MAX, S_MAX = 64, 1024, 32
NORM_D_MAX = 16384
NOALLOC_SCRATCH_U32 = 1 << 21

UNBOUNDED = 0xFFFFFFFF
HEAD_MAX, SINKS_MAX, SPAN_MAX, BUCKETS_MAX = 128, 64, 1023, 1024

c_u32, c_u64, c_vp = ctypes.c_uint32, ctypes.c_uint64, ctypes.c_void_p

_SIGNATURES = {
    "w2v_last_error": (ctypes.c_char_p, []),
    "w2v_shard_create": (ctypes.c_int, [c_u32, c_u32, c_u64, ctypes.POINTER(c_vp)]),
    "w2v_shard_create_ex": (ctypes.c_int, [c_u32, c_u32, c_u32, c_u32, c_u64, ctypes.c_int,
                                           ctypes.POINTER(c_vp)]),
    "w2v_shard_destroy": (ctypes.c_int, [c_vp]),
    "w2v_shard_set_counts": (ctypes.c_int, [c_vp, c_vp, ctypes.c_double]),
    "w2v_shard_get_tables": (ctypes.c_int, [c_vp, c_vp, c_vp, c_vp]),
    "w2v_shard_get_rows": (ctypes.c_int, [c_vp, ctypes.c_int, c_vp, c_u32, c_vp, c_vp]),
    "w2v_shard_set_rows": (ctypes.c_int, [c_vp, ctypes.c_int, c_vp, c_u32, c_vp, c_vp]),
    "w2v_shard_status": (ctypes.c_int, [c_vp, c_vp]),
    "w2v_negatives": (ctypes.c_int, [c_vp, c_vp, c_u32, c_u32, c_u64, c_vp, c_vp]),
    "w2v_dotprod": (ctypes.c_int, [c_vp, c_vp, c_vp, c_u32, c_u32, c_u64, c_vp, c_vp]),
    "w2v_dotprod_noalloc": (ctypes.c_int, [c_vp, c_vp, c_vp, c_u32, c_u32, c_u64, c_vp, c_vp]),
    "w2v_prefetch_cancel": (ctypes.c_int, [c_vp]),
    "w2v_coeffs": (ctypes.c_int, [c_vp, ctypes.POINTER(c_vp), c_u32, c_u32, c_u32, c_vp, c_vp, c_vp]),
    "w2v_adjust": (ctypes.c_int, [c_vp, c_vp, c_vp, c_u32, c_u32, c_u64, c_vp, ctypes.c_float, c_vp]),
    "w2v_train_minibatch": (ctypes.c_int, [ctypes.POINTER(c_vp), c_u32, c_vp, c_vp, c_u32, c_u32,
                                           c_u64, ctypes.c_float, c_vp, c_vp]),
    "w2v_step_graph_create": (ctypes.c_int, [c_vp, c_u32, c_u32, c_vp, ctypes.POINTER(c_vp)]),
    "w2v_step_graph_run": (ctypes.c_int, [c_vp, c_vp, c_vp, c_u64, ctypes.c_float, c_vp]),
    "w2v_step_graph_destroy": (ctypes.c_int, [c_vp]),
    "w2v_prefetch_minibatch": (ctypes.c_int, [c_vp, c_vp, c_vp, c_u32, c_u32, c_u64, c_vp]),
    "w2v_cbow_prefetch_minibatch": (ctypes.c_int, [c_vp, c_vp, c_vp, c_u32, c_vp, c_u32, c_u32, c_u64,
                                                   c_vp]),
    "w2v_make_pairs": (ctypes.c_int, [c_vp, c_vp, c_vp, c_u32, c_u32, c_u64, c_u32, c_u64, c_u32,
                                      c_vp, c_vp, c_u64, ctypes.POINTER(c_u64), c_vp]),
    "w2v_make_pairs_interleaved": (ctypes.c_int, [c_vp, c_vp, c_vp, c_u32, c_u32, c_u64, c_u32, c_u64,
                                                  c_u32, c_vp, c_vp, c_u64, ctypes.POINTER(c_u64),
                                                  c_vp]),
    "w2v_cbow_dotprod": (ctypes.c_int, [c_vp, c_vp, c_vp, c_u32, c_vp, c_u32, c_u32, c_u64, c_vp, c_vp]),
    "w2v_cbow_adjust": (ctypes.c_int, [c_vp, c_vp, c_vp, c_u32, c_vp, c_u32, c_u32, c_u64, c_vp,
                                       ctypes.c_float, c_vp]),
    "w2v_cbow_train_minibatch": (ctypes.c_int, [ctypes.POINTER(c_vp), c_u32, c_vp, c_vp, c_u32, c_vp,
                                                c_u32, c_u32, c_u64, ctypes.c_float, c_vp, c_vp]),
    "w2v_make_cbow_examples": (ctypes.c_int, [c_vp, c_vp, c_vp, c_u32, c_u32, c_u64, c_u32, c_u64,
                                              c_u32, c_vp, c_vp, c_vp, c_u64, c_u64,
                                              ctypes.POINTER(c_u64), ctypes.POINTER(c_u64), c_vp]),
    "w2v_export_rows": (ctypes.c_int, [ctypes.POINTER(c_vp), c_u32, ctypes.c_int, c_vp, c_u32, c_vp, c_vp]),
    "w2v_topk_cosine_workspace": (ctypes.c_size_t, [c_u32, c_u32, c_u32]),
    "w2v_topk_cosine": (ctypes.c_int, [c_vp, c_u32, c_vp, c_u32, c_u32, c_u32, ctypes.c_float, c_vp,
                                       c_vp, c_vp, c_vp, ctypes.c_size_t, c_vp]),
    "w2v_layer_norm": (ctypes.c_int, [ctypes.c_int, c_vp, c_u64, c_u64, c_u32, c_vp, c_vp, ctypes.c_float,
                                      c_vp, c_u64, c_vp, c_vp, c_vp]),
    "w2v_layer_norm_backward_workspace": (ctypes.c_size_t, [ctypes.c_int, c_u64, c_u32]),
    "w2v_layer_norm_backward": (ctypes.c_int, [ctypes.c_int, c_vp, c_u64, c_vp, c_u64, c_u64, c_u32, c_vp,
                                               c_vp, c_vp, c_vp, c_u64, c_vp, c_vp, c_vp, ctypes.c_size_t,
                                               c_vp]),
    "w2v_relative_buckets": (ctypes.c_int, [c_u32, c_u32, c_vp]),
    "w2v_attend": (ctypes.c_int, [c_vp, c_vp, c_vp, c_vp, c_vp, c_u32, c_u32, c_vp, c_vp, c_vp, c_vp]),
    "w2v_attend_backward_workspace": (ctypes.c_size_t, [c_vp, c_u32]),
    "w2v_attend_backward": (ctypes.c_int, [c_vp] * 6 + [c_vp, c_vp, c_u32, c_u32, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp,
                                                        ctypes.c_size_t, c_vp]),
    "w2v_attend_step_workspace": (ctypes.c_size_t, [c_vp, c_u32, c_u32]),
    "w2v_attend_step": (ctypes.c_int, [c_vp, c_vp, c_vp, c_vp, c_vp, c_u32, c_u32, c_vp, c_vp, c_vp, ctypes.c_size_t,
                                       c_vp]),
    "w2v_minibatch_seed": (c_u64, [c_u64, c_u64]),
    "w2v_shard_timing_enable": (ctypes.c_int, [c_vp, ctypes.c_int]),
    "w2v_shard_timing_read": (ctypes.c_int, [c_vp, c_vp, c_vp]),
}
EXPORTS = sorted(_SIGNATURES)


class W2VError(RuntimeError):
    def __init__(self, code, text):
        super().__init__("w2v error %d: %s" % (code, text))
        self.code = code


def lib():
    """Opens the built library; a missing library is an error (run paper_1606_08495_amd.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                "%s is missing: build it with `python -m paper_1606_08495_amd.build`" % LIB_PATH)
        L = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


def _check(rc):
    if rc != 0:
        raise W2VError(rc, lib().w2v_last_error().decode("utf-8", "replace"))


def _stream(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return c_vp(stream.cuda_stream)


def _dev(t, dtype, name):
    if t is None:
        return c_vp(0)
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == dtype and t.is_contiguous()):
        raise TypeError("%s must be a contiguous CUDA tensor of %s" % (name, dtype))
    return c_vp(t.data_ptr())


def _room(t, device):
    """(pointer, bytes) of a workspace that the caller keeps."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.is_contiguous()):
        raise TypeError("workspace must be a contiguous CUDA tensor")
    if t.device != device:
        raise ValueError("workspace must be on %s" % device)
    return t.data_ptr(), t.numel() * t.element_size()


# uint32 index arrays are carried in int32 tensors (torch has no arithmetic on uint32; the bit
# patterns are what the library reads).
IDX = torch.int32


def as_index_tensor(a, device="cuda"):
    """numpy uint32/int array -> int32 device tensor with the same bit pattern."""
    a = np.ascontiguousarray(a, dtype=np.uint32)
    return torch.from_numpy(a.view(np.int32)).to(device)


def index_to_numpy(t):
    return t.detach().cpu().numpy().view(np.uint32)


def minibatch_seed(master_seed, h):
    return int(lib().w2v_minibatch_seed(c_u64(master_seed), c_u64(h)))


class Shard:
    """One column shard (w2v_shard).  Methods mirror the C entry points one to one."""

    def __init__(self, V, d_slice, seed, d_total=None, col_begin=0, init_mode=0):
        self.V, self.d_slice = int(V), int(d_slice)
        self.d_total = int(d_slice if d_total is None else d_total)
        self.col_begin = int(col_begin)
        h = c_vp(0)
        _check(lib().w2v_shard_create_ex(self.V, self.d_total, self.col_begin, self.d_slice,
                                         int(seed), int(init_mode), ctypes.byref(h)))
        self.h = h

    def destroy(self):
        if getattr(self, "h", None):
            lib().w2v_shard_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    # -- tables ------------------------------------------------------------------------------
    def set_counts(self, counts, subsample_t=0.0):
        counts = np.ascontiguousarray(counts, dtype=np.uint64)
        if counts.size != self.V:
            raise ValueError("counts must have V entries")
        _check(lib().w2v_shard_set_counts(self.h, c_vp(counts.ctypes.data), float(subsample_t)))

    def get_tables(self):
        th = np.empty(self.V, np.uint32)
        al = np.empty(self.V, np.uint32)
        kp = np.empty(self.V, np.uint64)
        _check(lib().w2v_shard_get_tables(self.h, c_vp(th.ctypes.data), c_vp(al.ctypes.data),
                                          c_vp(kp.ctypes.data)))
        return th, al, kp

    # -- rows ----------------------------------------------------------------------------------
    def get_rows(self, which, rows, stream=None):
        out = torch.empty((rows.numel(), self.d_slice), dtype=torch.float32, device=rows.device)
        _check(lib().w2v_shard_get_rows(self.h, int(which), _dev(rows, IDX, "rows"), rows.numel(),
                                        _dev(out, torch.float32, "dst"), _stream(stream)))
        return out

    def set_rows(self, which, rows, src, stream=None):
        if src.shape != (rows.numel(), self.d_slice):
            raise ValueError("src must be [m, d_slice]")
        _check(lib().w2v_shard_set_rows(self.h, int(which), _dev(rows, IDX, "rows"), rows.numel(),
                                        _dev(src, torch.float32, "src"), _stream(stream)))

    def status(self, stream=None):
        _check(lib().w2v_shard_status(self.h, _stream(stream)))

    # -- the calls of the paper ------------------------------------------------------------------
    def negatives(self, out_idx, k, seed, stream=None):
        n = out_idx.numel()
        neg = torch.empty((n, k), dtype=IDX, device=out_idx.device)
        _check(lib().w2v_negatives(self.h, _dev(out_idx, IDX, "out_idx"), n, int(k), int(seed),
                                   _dev(neg, IDX, "neg"), _stream(stream)))
        return neg

    def dotprod(self, in_idx, out_idx, k, seed, out=None, stream=None):
        n = in_idx.numel()
        if out is None:
            out = torch.empty((n, k + 1), dtype=torch.float32, device=in_idx.device)
        _check(lib().w2v_dotprod(self.h, _dev(in_idx, IDX, "in_idx"), _dev(out_idx, IDX, "out_idx"),
                                 n, int(k), int(seed), _dev(out, torch.float32, "partial_dots"),
                                 _stream(stream)))
        return out

    def dotprod_noalloc(self, in_idx, out_idx, k, seed, out, stream=None):
        """w2v_dotprod_noalloc: `out` ([n, k+1] float32) must be given; the library allocates nothing."""
        _check(lib().w2v_dotprod_noalloc(self.h, _dev(in_idx, IDX, "in_idx"),
                                         _dev(out_idx, IDX, "out_idx"), in_idx.numel(), int(k),
                                         int(seed), _dev(out, torch.float32, "partial_dots"),
                                         _stream(stream)))
        return out

    def prefetch_cancel(self):
        _check(lib().w2v_prefetch_cancel(self.h))

    def coeffs(self, partials, k, want_loss=False, out=None, stream=None):
        S = len(partials)
        n = partials[0].shape[0]
        arr = (c_vp * S)(*[p.data_ptr() for p in partials])
        for p in partials:
            _dev(p, torch.float32, "partials")
        if out is None:
            out = torch.empty((n, k + 1), dtype=torch.float32, device=partials[0].device)
        loss = torch.zeros(1, dtype=torch.float64, device=out.device) if want_loss else None
        _check(lib().w2v_coeffs(self.h, arr, S, n, int(k), _dev(out, torch.float32, "coeffs"),
                                _dev(loss, torch.float64, "loss"), _stream(stream)))
        return (out, loss) if want_loss else out

    def adjust(self, in_idx, out_idx, k, seed, coeffs, alpha, stream=None):
        n = in_idx.numel()
        _check(lib().w2v_adjust(self.h, _dev(in_idx, IDX, "in_idx"), _dev(out_idx, IDX, "out_idx"),
                                n, int(k), int(seed), _dev(coeffs, torch.float32, "coeffs"),
                                float(alpha), _stream(stream)))

    def prefetch_minibatch(self, in_idx, out_idx, k, seed, stream=None):
        """Index work of the next minibatch, queued beside the current one (w2v_prefetch_minibatch)."""
        _check(lib().w2v_prefetch_minibatch(self.h, _dev(in_idx, IDX, "in_idx"),
                                            _dev(out_idx, IDX, "out_idx"), in_idx.numel(), int(k),
                                            int(seed), _stream(stream)))

    def make_pairs(self, tokens, sent_off, token_base, epoch, corpus_seed, B, in_idx, out_idx,
                   stream=None, interleaved=False):
        """tokens int32[n] (uint32 bits), sent_off int64[m+1] on the device; fills in_idx/out_idx
        (capacity = their length) and returns the full pair count.  ``interleaved`` calls
        w2v_make_pairs_interleaved instead of w2v_make_pairs."""
        cnt = c_u64(0)
        fn = lib().w2v_make_pairs_interleaved if interleaved else lib().w2v_make_pairs
        _check(fn(self.h, _dev(tokens, IDX, "tokens"),
                                    _dev(sent_off, torch.int64, "sent_off"), sent_off.numel() - 1,
                                    tokens.numel(), int(token_base), int(epoch), int(corpus_seed),
                                    int(B), _dev(in_idx, IDX, "in_idx"), _dev(out_idx, IDX, "out_idx"),
                                    min(in_idx.numel(), out_idx.numel()), ctypes.byref(cnt),
                                    _stream(stream)))
        return int(cnt.value)

    # -- continuous bag of words -----------------------------------------------------------------
    def cbow_dotprod(self, ctx_off, ctx_idx, out_idx, k, seed, out=None, stream=None):
        """ctx_off int32[n+1], ctx_idx int32[m], out_idx int32[n] (uint32 bits) on the device."""
        n = out_idx.numel()
        if out is None:
            out = torch.empty((n, k + 1), dtype=torch.float32, device=out_idx.device)
        _check(lib().w2v_cbow_dotprod(self.h, _dev(ctx_off, IDX, "ctx_off"),
                                      _dev(ctx_idx, IDX, "ctx_idx"), ctx_idx.numel(),
                                      _dev(out_idx, IDX, "out_idx"), n, int(k), int(seed),
                                      _dev(out, torch.float32, "partial_dots"), _stream(stream)))
        return out

    def cbow_adjust(self, ctx_off, ctx_idx, out_idx, k, seed, coeffs, alpha, stream=None):
        _check(lib().w2v_cbow_adjust(self.h, _dev(ctx_off, IDX, "ctx_off"),
                                     _dev(ctx_idx, IDX, "ctx_idx"), ctx_idx.numel(),
                                     _dev(out_idx, IDX, "out_idx"), out_idx.numel(), int(k), int(seed),
                                     _dev(coeffs, torch.float32, "coeffs"), float(alpha),
                                     _stream(stream)))

    def cbow_prefetch_minibatch(self, ctx_off, ctx_idx, out_idx, k, seed, stream=None):
        """Index work of a later bag-of-words minibatch, queued beside the calls that follow."""
        _check(lib().w2v_cbow_prefetch_minibatch(self.h, _dev(ctx_off, IDX, "ctx_off"),
                                                 _dev(ctx_idx, IDX, "ctx_idx"), ctx_idx.numel(),
                                                 _dev(out_idx, IDX, "out_idx"), out_idx.numel(),
                                                 int(k), int(seed), _stream(stream)))

    def make_cbow_examples(self, tokens, sent_off, token_base, epoch, corpus_seed, B, ctx_off, ctx_idx,
                           out_idx, stream=None):
        """Fills ctx_off (length cap+1), ctx_idx and out_idx (length cap) on the device; returns
        the full (number of examples, number of context entries)."""
        n_ex, n_ctx = c_u64(0), c_u64(0)
        cap = min(out_idx.numel(), ctx_off.numel() - 1)
        _check(lib().w2v_make_cbow_examples(
            self.h, _dev(tokens, IDX, "tokens"), _dev(sent_off, torch.int64, "sent_off"),
            sent_off.numel() - 1, tokens.numel(), int(token_base), int(epoch), int(corpus_seed), int(B),
            _dev(ctx_off, IDX, "ctx_off"), _dev(ctx_idx, IDX, "ctx_idx"), _dev(out_idx, IDX, "out_idx"),
            cap, ctx_idx.numel(), ctypes.byref(n_ex), ctypes.byref(n_ctx), _stream(stream)))
        return int(n_ex.value), int(n_ctx.value)

    # -- timing ----------------------------------------------------------------------------------
    def timing_enable(self, on=True):
        _check(lib().w2v_shard_timing_enable(self.h, int(bool(on))))

    def timing_read(self):
        ms = np.zeros(len(PHASES), np.float64)
        cnt = np.zeros(len(PHASES), np.uint64)
        _check(lib().w2v_shard_timing_read(self.h, c_vp(ms.ctypes.data), c_vp(cnt.ctypes.data)))
        return {PHASES[i]: (float(ms[i]), int(cnt[i])) for i in range(len(PHASES))}


class StepGraph:
    """w2v_step_graph: w2v_train_minibatch on one shard for a fixed (n, k), prepared once."""

    def __init__(self, shard, n, k, loss=None):
        self.n, self.k, self.shard, self.loss = int(n), int(k), shard, loss
        h = c_vp(0)
        _check(lib().w2v_step_graph_create(shard.h, self.n, self.k, _dev(loss, torch.float64, "loss"),
                                           ctypes.byref(h)))
        self.h = h

    def run(self, in_idx, out_idx, seed, alpha, stream=None):
        if in_idx.numel() != self.n or out_idx.numel() != self.n:
            raise ValueError("the graph was captured for %d pairs" % self.n)
        _check(lib().w2v_step_graph_run(self.h, _dev(in_idx, IDX, "in_idx"), _dev(out_idx, IDX, "out_idx"),
                                        int(seed), float(alpha), _stream(stream)))

    def destroy(self):
        if getattr(self, "h", None):
            lib().w2v_step_graph_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def train_minibatch(shards, in_idx, out_idx, k, seed, alpha, loss=None, stream=None):
    """One client step over the given shards (w2v_train_minibatch).  ``loss``: optional float64
    device tensor of one element that receives the minibatch loss."""
    S = len(shards)
    arr = (c_vp * S)(*[s.h.value for s in shards])
    n = in_idx.numel()
    _check(lib().w2v_train_minibatch(arr, S, _dev(in_idx, IDX, "in_idx"),
                                     _dev(out_idx, IDX, "out_idx"), n, int(k), int(seed),
                                     float(alpha), _dev(loss, torch.float64, "loss"),
                                     _stream(stream)))


def cbow_train_minibatch(shards, ctx_off, ctx_idx, out_idx, k, seed, alpha, loss=None, stream=None):
    """One client step of the bag-of-words variant over the given shards
    (w2v_cbow_train_minibatch)."""
    S = len(shards)
    arr = (c_vp * S)(*[s.h.value for s in shards])
    _check(lib().w2v_cbow_train_minibatch(arr, S, _dev(ctx_off, IDX, "ctx_off"),
                                          _dev(ctx_idx, IDX, "ctx_idx"), ctx_idx.numel(),
                                          _dev(out_idx, IDX, "out_idx"), out_idx.numel(), int(k),
                                          int(seed), float(alpha), _dev(loss, torch.float64, "loss"),
                                          _stream(stream)))


def export_rows(shards, which, rows, out=None, stream=None):
    """Whole vectors [m, d_total] of the listed rows, joined from the column shards
    (w2v_export_rows)."""
    S = len(shards)
    arr = (c_vp * S)(*[s.h.value for s in shards])
    m = rows.numel()
    if out is None:
        out = torch.empty((m, shards[0].d_total), dtype=torch.float32, device=rows.device)
    _check(lib().w2v_export_rows(arr, S, int(which), _dev(rows, IDX, "rows"), m,
                                 _dev(out, torch.float32, "dst"), _stream(stream)))
    return out


def topk_cosine(queries, cands, K, tau=-2.0, round_candidates=32768, workspace=None, stream=None):
    """(idx int32[Q, K] (uint32 bits), score float32[Q, K], count int32[Q]) of w2v_topk_cosine.
    ``workspace``: optional uint8 device tensor to reuse; otherwise one for rounds of
    ``round_candidates`` candidates is allocated here."""
    Q, d = queries.shape
    N = cands.shape[0]
    if cands.shape[1] != d:
        raise ValueError("queries and candidates differ in width")
    if workspace is None:
        need = int(lib().w2v_topk_cosine_workspace(Q, N, int(round_candidates)))
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=queries.device)
    at, size = _room(workspace, queries.device)
    idx = torch.empty((Q, K), dtype=IDX, device=queries.device)
    score = torch.empty((Q, K), dtype=torch.float32, device=queries.device)
    count = torch.empty(Q, dtype=IDX, device=queries.device)
    _check(lib().w2v_topk_cosine(_dev(queries, torch.float32, "queries"), Q,
                                 _dev(cands, torch.float32, "cands"), N, d, int(K), float(tau),
                                 _dev(idx, IDX, "out_idx"), _dev(score, torch.float32, "out_score"),
                                 _dev(count, IDX, "out_count"), c_vp(at), size, _stream(stream)))
    return idx, score, count


# -- vectors in context ------------------------------------------------------------------------------
# These calls record no graph for torch's automatic differentiation, whatever their inputs require: gradients come from the
# backward calls.
TYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}


_AS_IT_IS = contextlib.nullcontext()
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _on(stream, t):
    """What is allocated for a call belongs to the stream the call runs on, and to the tensor's device."""
    if not t.is_cuda:
        raise TypeError("a CUDA tensor is wanted")
    if stream is not None:
        return torch.cuda.stream(stream)
    return _AS_IT_IS if t.device.index == torch.cuda.current_device() else torch.cuda.device(t.device)


def _rows(t, like, name):
    """A matrix of rows that lie anywhere, their elements side by side: (pointer, elements from row to row)."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype in TYPES and t.dim() == 2):
        raise TypeError("%s must be a CUDA matrix of float32, float16 or bfloat16" % name)
    if like is not None and (t.shape != like.shape or t.dtype != like.dtype or t.device != like.device):
        raise ValueError("%s differs in shape, type or device" % name)
    (m, d), (a, b) = t.shape, t.stride()
    if b != 1 and d > 1 and m > 0:
        raise ValueError("%s: the elements of a row must lie side by side" % name)
    return t.data_ptr(), a if m > 1 else d


def _vec(t, n, device, name):
    if t is None:
        return None
    if t.shape != (n,) or t.device != device:
        raise ValueError("%s must have %d entries on %s" % (name, n, device))
    return _dev(t, torch.float32, name)


def layer_norm(x, gain=None, offset=None, eps=1e-5, out=None, stream=None):
    """(y, mean, rstd) of w2v_layer_norm for the rows of x [m, d]; gain and offset are float32 [d].  Not differentiable by
    torch: layer_norm_backward."""
    xp, xs = _rows(x, None, "x")
    m, d = x.shape
    with _on(stream, x):
        st = _raw_stream(x.device.index)
        y = x.new_empty((m, d)) if out is None else out
        stats = x.new_empty((2, m), dtype=torch.float32)
        yp, ys = _rows(y, x, "out")
        at = stats.data_ptr()
        _check(lib().w2v_layer_norm(TYPES[x.dtype], xp, xs, m, d, _vec(gain, d, x.device, "gain"),
                                    _vec(offset, d, x.device, "offset"), float(eps), yp, ys, at, at + 4 * m, st))
    mean, rstd = stats.unbind(0)
    return y, mean, rstd


def layer_norm_backward(dy, x, gain, mean, rstd, out=None, workspace=None, stream=None):
    """(dx, dgain, doffset) of w2v_layer_norm_backward; gain may be None.  ``workspace``: optional uint8
    device tensor to reuse."""
    xp, xs = _rows(x, None, "x")
    gp, gs = _rows(dy, x, "dy")
    m, d = x.shape
    with _on(stream, x):
        st = _raw_stream(x.device.index)
        dx = x.new_empty((m, d)) if out is None else out
        columns = x.new_empty((2, d), dtype=torch.float32)
        if workspace is None:
            workspace = x.new_empty(int(lib().w2v_layer_norm_backward_workspace(TYPES[x.dtype], m, d)),
                                    dtype=torch.uint8)
        at, size = _room(workspace, x.device)
        op, os_ = _rows(dx, x, "out")
        _check(lib().w2v_layer_norm_backward(TYPES[x.dtype], gp, gs, xp, xs, m, d, _vec(gain, d, x.device, "gain"),
                                             _vec(mean, m, x.device, "mean"), _vec(rstd, m, x.device, "rstd"), op,
                                             os_, columns.data_ptr(), columns.data_ptr() + 4 * d,
                                             at, size, st))
    dgain, doffset = columns.unbind(0)
    return dx, dgain, doffset


class Heads(ctypes.Structure):
    """w2v_heads: rows of heads, element c of head h of token i at p[i token_stride + h head_stride + c]."""
    _fields_ = [("p", c_vp), ("token_stride", c_u64), ("head_stride", c_u64)]


class Cache(ctypes.Structure):
    """w2v_cache: element c of head h of word j of text b at p[b text_stride + j token_stride + h head_stride + c]."""
    _fields_ = [("p", c_vp), ("text_stride", c_u64), ("token_stride", c_u64), ("head_stride", c_u64)]


class AttendSpec(ctypes.Structure):
    """w2v_attend_spec."""
    _fields_ = [("type", ctypes.c_int32), ("heads", c_u32), ("kv_heads", c_u32), ("width", c_u32), ("left", c_u32),
                ("right", c_u32), ("sinks", c_u32), ("skip_self", c_u32), ("scale", ctypes.c_float),
                ("n_buckets", c_u32), ("span", c_u32), ("bias_dev", c_vp), ("bucket_dev", c_vp)]


def _number(x, name):
    """A count as the library takes it: what lies past 32 bits is past every limit too."""
    x = int(x)
    if x < 0:
        raise ValueError("%s = %d is negative" % (name, x))
    return min(x, UNBOUNDED)


def relative_buckets(n_buckets, span, device="cuda"):
    """The bucket of every distance -span..span (w2v_relative_buckets), int32 [2 span + 1] on the device: one half for words
    before, one for words after, whether or not these are shown."""
    n_buckets, span = _number(n_buckets, "n_buckets"), _number(span, "span")
    m = np.empty(2 * min(span, SPAN_MAX) + 1, np.uint32)      # (a longer span is refused)
    _check(lib().w2v_relative_buckets(n_buckets, span, c_vp(m.ctypes.data)))
    return as_index_tensor(m, device)


def _heads(t, like, rows, heads, name):
    """[rows, heads, width], the elements of a head side by side."""
    width = like.shape[2]
    if not isinstance(t, torch.Tensor) or t.dtype is not like.dtype or t.device != like.device or \
            t.shape != (rows, heads, width):
        raise TypeError("%s must be a CUDA tensor [%d, %d, %d] of %s" % (name, rows, heads, width, like.dtype))
    a, b, c = t.stride()
    if (c != 1 and width > 1) or a < 0 or b < 0:
        raise ValueError("%s: the elements of a head must lie side by side" % name)
    return Heads(t.data_ptr(), a, b)


def _dense(t, heads, width):
    """A dense [rows, heads, width] of this module's own making."""
    return Heads(t.data_ptr(), heads * width, width)


def _spec(q, kv_heads, left, right, sinks, skip_self, scale, bias, buckets):
    if q.dtype not in TYPES:
        raise TypeError("q must be float32, float16 or bfloat16")
    heads, width = q.shape[1], q.shape[2]
    s = AttendSpec(TYPES[q.dtype], heads, kv_heads, width, UNBOUNDED if left is None else _number(left, "left"),
                   UNBOUNDED if right is None else _number(right, "right"), _number(sinks, "sinks"), 1 if skip_self else 0,
                   width ** -0.5 if scale is None else float(scale))
    if bias is not None:
        if bias.dim() != 2 or bias.shape[0] != heads or bias.device != q.device:
            raise ValueError("bias must be [heads, buckets]")
        if buckets is None or buckets.dim() != 1 or buckets.numel() % 2 == 0 or buckets.device != q.device:
            raise ValueError("buckets must give the bucket of the distances -span..span")
        s.n_buckets, s.span = bias.shape[1], buckets.numel() // 2
        s.bias_dev, s.bucket_dev = _dev(bias, torch.float32, "bias"), _dev(buckets, IDX, "buckets")
    return s


def _texts(sent_off, keep, q):
    if sent_off.device != q.device or (keep is not None and (keep.device != q.device or keep.shape != (q.shape[0],))):
        raise ValueError("sent_off and keep [tokens] must be on the device of q")
    return (_dev(sent_off, torch.int64, "sent_off"), max(sent_off.numel() - 1, 0), q.shape[0],
            _dev(keep, torch.uint8, "keep"))


def attend(q, k, v, sent_off, left=None, right=None, sinks=0, skip_self=False, scale=None, keep=None, bias=None,
           buckets=None, out=None, stream=None):
    """(out, lse) of w2v_attend: q [tokens, heads, width], k and v [tokens, kv_heads, width], texts as sent_off
    int64 [n + 1].  left, right: words shown on either side (None: all).  scale: width^-1/2 unless given.  keep:
    uint8 [tokens], 0 where a word is not to be seen.  bias float32 [heads, buckets] with the map ``buckets`` (relative_buckets).
    Not differentiable by torch: attend_backward."""
    if q.dim() != 3 or k.dim() != 3:
        raise TypeError("q, k and v must be [tokens, heads, width]")
    T, H, d = q.shape
    G = k.shape[1]
    with _on(stream, q):
        st, r = _raw_stream(q.device.index), ctypes.byref
        if out is None:
            out = q.new_empty(q.shape)
            into = _dense(out, H, d)
        else:
            into = _heads(out, q, T, H, "out")
        lse = q.new_empty((H, T), dtype=torch.float32)
        spec = _spec(q, G, left, right, sinks, skip_self, scale, bias, buckets)
        off, n, t, kp = _texts(sent_off, keep, q)
        _check(lib().w2v_attend(r(spec), r(_heads(q, q, T, H, "q")), r(_heads(k, q, T, G, "k")),
                                r(_heads(v, q, T, G, "v")), off, n, t, kp, r(into), lse.data_ptr(), st))
    return out, lse


def attend_backward(dout, q, k, v, out, lse, sent_off, left=None, right=None, sinks=0, skip_self=False, scale=None,
                    keep=None, bias=None, buckets=None, workspace=None, stream=None):
    """(dq, dk, dv, dbias) of w2v_attend_backward, for the arguments and results of ``attend``; dbias is None without
    a bias.  ``workspace``: optional uint8 device tensor to reuse."""
    if q.dim() != 3 or k.dim() != 3:
        raise TypeError("q, k and v must be [tokens, heads, width]")
    T, H, d = q.shape
    G = k.shape[1]
    if lse.shape != (H, T) or lse.device != q.device:
        raise ValueError("lse must be [heads, tokens]")
    with _on(stream, q):
        st = _raw_stream(q.device.index)
        dq, dk, dv = q.new_empty(q.shape), q.new_empty(k.shape), q.new_empty(k.shape)
        dbias = None if bias is None else bias.new_empty(bias.shape)
        spec = _spec(q, G, left, right, sinks, skip_self, scale, bias, buckets)
        if workspace is None:
            need = int(lib().w2v_attend_backward_workspace(ctypes.byref(spec), T))
            workspace = q.new_empty(max(need, 256), dtype=torch.uint8)
        at, size = _room(workspace, q.device)
        off, n, t, kp = _texts(sent_off, keep, q)
        r = ctypes.byref
        _check(lib().w2v_attend_backward(
            r(spec), r(_heads(dout, q, T, H, "dout")), r(_heads(q, q, T, H, "q")), r(_heads(k, q, T, G, "k")),
            r(_heads(v, q, T, G, "v")), r(_heads(out, q, T, H, "out")), _dev(lse, torch.float32, "lse"), off, n, t, kp,
            r(_dense(dq, H, d)), r(_dense(dk, G, d)), r(_dense(dv, G, d)),
            _dev(dbias, torch.float32, "dbias"), at, size, st))
    return dq, dk, dv, dbias


def _cache(t, like, shape, name):
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == like.dtype and t.device == like.device and
            t.shape == shape):
        raise TypeError("%s must be a CUDA tensor %s of %s" % (name, list(shape), like.dtype))
    s = t.stride()
    if (s[3] != 1 and shape[3] > 1) or min(s) < 0:
        raise ValueError("%s: the elements of a head must lie side by side" % name)
    return Cache(t.data_ptr(), s[0], s[1], s[2])


def attend_step(q, k, v, n, left=None, sinks=0, skip_self=False, scale=None, keep=None, bias=None, buckets=None, out=None,
                workspace=None, stream=None):
    """out [texts, heads, width] of w2v_attend_step: the newest word's q [texts, heads, width] over the caches k and
    v [texts, room, kv_heads, width], of which text b has filled n[b] (int32, the newest word's among them).  keep: uint8
    [texts, room].  ``workspace``: optional uint8 device tensor to reuse.  Other arguments as for ``attend``."""
    if q.dim() != 3 or k.dim() != 4:
        raise TypeError("q must be [texts, heads, width], k and v [texts, room, heads, width]")
    B, H, d = q.shape
    room, G = k.shape[1], k.shape[2]
    if n.shape != (B,) or n.device != q.device or (keep is not None and (keep.shape != (B, room) or keep.device != q.device)):
        raise ValueError("n must be [texts] and keep [texts, room] on the device of q")
    with _on(stream, q):
        st = _raw_stream(q.device.index)
        if out is None:
            out = q.new_empty(q.shape)
        spec = _spec(q, G, left, 0, sinks, skip_self, scale, bias, buckets)
        r = ctypes.byref
        if workspace is None:
            need = int(lib().w2v_attend_step_workspace(r(spec), B, room))
            workspace = q.new_empty(max(need, 256), dtype=torch.uint8)
        at, size = _room(workspace, q.device)
        shape = torch.Size((B, room, G, d))
        _check(lib().w2v_attend_step(r(spec), r(_heads(q, q, B, H, "q")), r(_cache(k, q, shape, "k")),
                                     r(_cache(v, q, shape, "v")), _dev(n, IDX, "n"), B, room, _dev(keep, torch.uint8, "keep"),
                                     r(_heads(out, q, B, H, "out")), at, size, st))
    return out
