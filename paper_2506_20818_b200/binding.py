"""Thin ctypes binding of the C ABI in include/lp.h.

Argument marshalling only: every step of the path runs inside liblp_b200.so.  torch is used
for device memory and streams.  There is no CPU fall-back: if the library is missing or no
B200 is present, calls raise.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from typing import Optional, Sequence

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "liblp_b200.so")

LP_OK = 0
LP_GCN, LP_SAGE_MEAN = 0, 1
LP_FP32, LP_BF16 = 0, 1
LP_NEG_PER_SOURCE, LP_NEG_GLOBAL_PAIR = 0, 1
LP_MAX_LAYERS = 4

STATUS_NAMES = {0: "LP_OK", -1: "LP_EINVAL", -2: "LP_ESTATE", -3: "LP_ENOMEM", -4: "LP_ECUDA",
                -5: "LP_EUNSUPPORTED", -6: "LP_ETIMEOUT"}

EXPORTS = [
    "lp_create", "lp_destroy", "lp_last_error", "lp_load_graph", "lp_get_structure", "lp_set_model",
    "lp_param_count", "lp_set_candidates", "lp_sample_negatives", "lp_train_step", "lp_train_step_host",
    "lp_adam_step", "lp_score", "lp_get_embeddings", "lp_get_output_gradient", "lp_get_block",
    "lp_get_stats", "lp_op_aggregate", "lp_op_gather_ceiling", "lp_op_linear", "lp_op_weight_grad", "lp_profile_begin", "lp_profile_end", "lp_profile_sample_every",
    "lp_weight_grad_static", "lp_sparsify", "lp_get_sparsified",
    "lp_worker_view", "lp_get_worker_view", "lp_hits_at_k", "lp_get_predictor_activations",
    "lp_invalidate_embeddings", "lp_set_wait_limit",
    "lp_embed", "lp_embed_grad", "lp_orthogonalize", "lp_muon_step",
    "lp_dropout", "lp_residual_norm", "lp_residual_norm_grad", "lp_grouped_linear", "lp_grouped_weight_grad",
]

PROF_CATEGORIES = ["agg_fwd", "agg_bwd", "gemm_fwd", "gemm_dgrad", "gemm_wgrad", "score", "incidence", "scatter",
                   "negatives", "blocks", "adam"]


class LpError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {message}")
        self.status = status


class ModelDesc(C.Structure):
    _fields_ = [("arch", C.c_int32), ("n_layers", C.c_int32), ("dims", C.c_int32 * (LP_MAX_LAYERS + 1)),
                ("prec", C.c_int32), ("fanout", C.c_int32 * LP_MAX_LAYERS), ("reject_edges", C.c_int32),
                ("max_attempts", C.c_int32), ("cache_input_aggregation", C.c_int32), ("predictor", C.c_int32),
                ("pred_hidden", C.c_int32)]


class Stats(C.Structure):
    _fields_ = [("negatives_exhausted", C.c_int64), ("block_nodes", C.c_int64 * (LP_MAX_LAYERS + 1)),
                ("block_edges", C.c_int64 * LP_MAX_LAYERS), ("workspace_bytes", C.c_int64),
                ("kernel_launches", C.c_int64)]


class ViewStats(C.Structure):
    _fields_ = [("own_entries", C.c_int64), ("foreign_entries", C.c_int64), ("foreign_rows", C.c_int64), ("own_nodes", C.c_int64)]


class Profile(C.Structure):
    _fields_ = [("ms", C.c_double * 11), ("bytes", C.c_double * 11), ("flops", C.c_double * 11), ("spans", C.c_int64 * 11)]


class Matrix(C.Structure):
    _fields_ = [("offset", C.c_int64), ("rows", C.c_int32), ("cols", C.c_int32)]


class MuonDesc(C.Structure):
    _fields_ = [("grad_scale", C.c_double), ("lr", C.c_double), ("momentum", C.c_double), ("weight_decay", C.c_double),
                ("coeffs", C.c_double * 3), ("eps", C.c_double), ("adam_lr", C.c_double), ("adam_beta1", C.c_double),
                ("adam_beta2", C.c_double), ("adam_eps", C.c_double), ("nesterov", C.c_int32), ("steps", C.c_int32)]


class ResidualDesc(C.Structure):
    _fields_ = [("rows", C.c_int64), ("width", C.c_int32), ("stream_prec", C.c_int32), ("prec", C.c_int32), ("pre_norm", C.c_int32),
                ("post_norm", C.c_int32), ("eps", C.c_double), ("scale", C.c_double), ("p", C.c_double), ("seed", C.c_uint64), ("step", C.c_uint64),
                ("row_base", C.c_int64), ("pre", C.c_void_p), ("pre_bias", C.c_void_p), ("post", C.c_void_p), ("post_bias", C.c_void_p),
                ("gate", C.c_void_p), ("ld_gate", C.c_int64)]


LP_NO_PADDING = -(1 << 31)
LP_NORM_NONE, LP_NORM_RMS, LP_NORM_LAYER = 0, 1, 2
_NORMS = {None: LP_NORM_NONE, "rms": LP_NORM_RMS, "layer": LP_NORM_LAYER}
_RESIDUAL = struct.Struct("qiiiii4xdddQQqQQQQQq")  # ResidualDesc, packed in one go: the fields of a Structure one by one take longer than the kernel

# argument types of the calls whose latency counts: ctypes converts plain Python numbers by them
_ARGTYPES = {
    "lp_embed": [C.c_void_p, C.c_int32, C.c_void_p, C.c_int64, C.c_int32, C.c_int64, C.c_void_p, C.c_int64, C.c_int32, C.c_double, C.c_int32,
                 C.c_void_p, C.c_int64],
    "lp_embed_grad": [C.c_void_p, C.c_int32, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_int32, C.c_double, C.c_int64, C.c_int32, C.c_int32,
                      C.c_void_p, C.c_int64, C.c_int32],
    "lp_orthogonalize": [C.c_void_p, C.c_int32, C.c_int64, C.c_int32, C.c_int32, C.c_void_p, C.c_int64, C.c_int64, C.c_int32, C.c_void_p, C.c_double,
                         C.c_void_p, C.c_int64, C.c_int64],
    "lp_muon_step": [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p,
                     C.c_void_p, C.c_void_p],
    "lp_dropout": [C.c_void_p, C.c_int32, C.c_int64, C.c_int32, C.c_void_p, C.c_int64, C.c_double, C.c_uint64, C.c_uint64, C.c_int64, C.c_void_p, C.c_int64],
    "lp_residual_norm": [C.c_void_p, C.c_void_p] + [C.c_void_p, C.c_int64] * 4,
    "lp_grouped_linear": [C.c_void_p, C.c_int32, C.c_int64, C.c_int32, C.c_int32, C.c_int64, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_int32, C.c_void_p,
                          C.c_int32, C.c_void_p, C.c_int64],
    "lp_grouped_weight_grad": [C.c_void_p, C.c_int32, C.c_int64, C.c_int32, C.c_int32, C.c_int64, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_int32,
                               C.c_void_p, C.c_void_p],
    "lp_residual_norm_grad": [C.c_void_p, C.c_void_p] + [C.c_void_p, C.c_int64] * 7 + [C.c_void_p] * 4 + [C.c_int32],
}

_lib = None


def load_library() -> C.CDLL:
    """dlopen the in-tree library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise FileNotFoundError(f"{_LIB_PATH} is missing: build it with paper_2506_20818_b200.build.build()")
        lib = C.CDLL(_LIB_PATH)
        lib.lp_last_error.restype = C.c_char_p
        lib.lp_last_error.argtypes = [C.c_void_p]
        lib.lp_destroy.restype = None
        lib.lp_destroy.argtypes = [C.c_void_p]
        for name in EXPORTS:
            if name not in ("lp_last_error", "lp_destroy"):
                getattr(lib, name).restype = C.c_int
        for name, types in _ARGTYPES.items():
            getattr(lib, name).argtypes = types
        _lib = lib
    return _lib


def _ptr(t):
    """Device (or host) address of a torch tensor / numpy array, or None."""
    if t is None:
        return None
    if hasattr(t, "data_ptr"):
        assert t.is_contiguous()
        return C.c_void_p(t.data_ptr())
    assert t.flags["C_CONTIGUOUS"]
    return C.c_void_p(t.ctypes.data)


class Context:
    """One lp_ctx: one graph, one model, one CUDA stream."""

    def __init__(self, device: int = 0, stream=None):
        import torch

        self._torch = torch
        self.lib = load_library()
        self.device = device
        self.stream = stream if stream is not None else torch.cuda.current_stream(device)
        h = C.c_void_p()
        st = self.lib.lp_create(C.byref(h), C.c_int32(device), C.c_void_p(self.stream.cuda_stream))
        if st != LP_OK:
            raise LpError(st, self.lib.lp_last_error(None).decode())
        self.h = h
        self.n = self.nnz = self.f = 0
        self.n_params = 0
        self._precs = {torch.float32: LP_FP32, torch.bfloat16: LP_BF16}
        self._f32, self._empty_like = torch.float32, torch.empty_like
        self._raw_stream = self.stream.cuda_stream
        self.desc: Optional[ModelDesc] = None

    def close(self):
        if getattr(self, "h", None):
            self.lib.lp_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _ck(self, st: int):
        if st != LP_OK:
            raise LpError(st, self.lib.lp_last_error(self.h).decode())

    # ---- graph
    def load_graph(self, n, rowptr, col, w, X, on_device: bool = False):
        """rowptr int64 [n+1], col int32 [nnz], w float32 [nnz] or None, X float32 [n, f]
        (numpy / CPU tensors, or CUDA tensors with on_device=True)."""
        nnz = int(col.shape[0])
        f = int(X.shape[1])
        self._ck(self.lib.lp_load_graph(self.h, C.c_int64(n), C.c_int64(nnz), _ptr(rowptr), _ptr(col), _ptr(w), _ptr(X),
                                        C.c_int32(f), C.c_int32(1 if on_device else 0)))
        self.n, self.nnz, self.f = int(n), nnz, f

    def get_structure(self):
        t = self._torch
        dev = f"cuda:{self.device}"
        colptr = t.empty(self.n + 1, dtype=t.int64, device=dev)
        rowidx = t.empty(max(self.nnz, 1), dtype=t.int32, device=dev)
        perm = t.empty(max(self.nnz, 1), dtype=t.int64, device=dev)
        self._ck(self.lib.lp_get_structure(self.h, _ptr(colptr), _ptr(rowidx), _ptr(perm)))
        return colptr, rowidx[: self.nnz], perm[: self.nnz]

    def sparsify(self, alpha: float, seed: int):
        """Algorithm 1's sparsification of the loaded (symmetric) graph: (rowptr int64, col int32, w float32) on the device."""
        t = self._torch
        dev = f"cuda:{self.device}"
        nnz = C.c_int64()
        self._ck(self.lib.lp_sparsify(self.h, C.c_double(alpha), C.c_uint64(seed), C.byref(nnz)))
        k = int(nnz.value)
        rowptr = t.empty(self.n + 1, dtype=t.int64, device=dev)
        col = t.empty(max(k, 1), dtype=t.int32, device=dev)
        w = t.empty(max(k, 1), dtype=t.float32, device=dev)
        self._ck(self.lib.lp_get_sparsified(self.h, _ptr(rowptr), _ptr(col), _ptr(w)))
        return rowptr, col[:k], w[:k]

    def worker_view(self, part, worker: int, keep_cross_edges: bool = True, foreign_mode: int = 1):
        """Graph that `worker` trains on (Section III): (rowptr int64, col int32, stats dict) on the device.
        foreign_mode 0 = no sharing, 1 = sparsified rows of the last sparsify(), 2 = full rows."""
        t = self._torch
        dev = f"cuda:{self.device}"
        nnz, st = C.c_int64(), ViewStats()
        self._ck(self.lib.lp_worker_view(self.h, _ptr(part), C.c_int32(worker), C.c_int32(int(keep_cross_edges)), C.c_int32(foreign_mode),
                                         C.byref(nnz), C.byref(st)))
        k = int(nnz.value)
        rowptr = t.empty(self.n + 1, dtype=t.int64, device=dev)
        col = t.empty(max(k, 1), dtype=t.int32, device=dev)
        self._ck(self.lib.lp_get_worker_view(self.h, _ptr(rowptr), _ptr(col)))
        return rowptr, col[:k], {"own_entries": st.own_entries, "foreign_entries": st.foreign_entries,
                                 "foreign_rows": st.foreign_rows, "own_nodes": st.own_nodes}

    # ---- model
    def set_model(self, arch: str, dims: Sequence[int], prec: str = "fp32", fanout: Optional[Sequence[int]] = None,
                  reject_edges: bool = True, max_attempts: int = 8, max_batch: int = 65536, max_k: int = 1,
                  cache_input_aggregation: bool = False, pred_hidden: int = 0):
        """pred_hidden = 0: dot-product predictor; > 0: 3-layer MLP predictor with that hidden width."""
        d = ModelDesc()
        d.arch = LP_GCN if arch == "gcn" else LP_SAGE_MEAN
        d.n_layers = len(dims) - 1
        for i, v in enumerate(dims):
            d.dims[i] = int(v)
        d.prec = LP_BF16 if prec == "bf16" else LP_FP32
        for i, v in enumerate(fanout or []):
            d.fanout[i] = int(v)
        d.reject_edges = int(bool(reject_edges))
        d.max_attempts = int(max_attempts)
        d.cache_input_aggregation = int(bool(cache_input_aggregation))
        d.predictor = 1 if pred_hidden > 0 else 0
        d.pred_hidden = int(pred_hidden)
        self._ck(self.lib.lp_set_model(self.h, C.byref(d), C.c_int64(max_batch), C.c_int32(max_k)))
        np_ = C.c_int64()
        self._ck(self.lib.lp_param_count(self.h, C.byref(np_)))
        self.n_params = int(np_.value)
        self.desc = d
        self.dims = list(dims)
        self.K = len(dims) - 1
        return self.n_params

    # ---- sampling
    def set_candidates(self, cand):
        self._ck(self.lib.lp_set_candidates(self.h, _ptr(cand), C.c_int64(0 if cand is None else cand.numel())))

    def sample_negatives(self, seed: int, step: int, k: int, pos_src, mode: int = LP_NEG_PER_SOURCE, edge_index_base: int = 0,
                         want_src: bool = False):
        t = self._torch
        B = int(pos_src.numel())
        neg_dst = t.empty(B * k, dtype=t.int32, device=pos_src.device)
        neg_src = t.empty(B * k, dtype=t.int32, device=pos_src.device) if (want_src or mode == LP_NEG_GLOBAL_PAIR) else None
        self._ck(self.lib.lp_sample_negatives(self.h, C.c_uint64(seed), C.c_uint64(step), C.c_int32(k), C.c_int32(mode), _ptr(pos_src),
                                              C.c_int64(B), C.c_int64(edge_index_base), _ptr(neg_src), _ptr(neg_dst)))
        return neg_src, neg_dst

    # ---- step
    def train_step(self, params, pos_src, pos_dst, neg_src, neg_dst, k: int, loss, grads, seed: int = 0, step: int = 0,
                   accumulate: bool = False):
        self._ck(self.lib.lp_train_step(self.h, _ptr(params), _ptr(pos_src), _ptr(pos_dst), C.c_int64(pos_src.numel()), _ptr(neg_src),
                                        _ptr(neg_dst), C.c_int32(k), C.c_uint64(seed), C.c_uint64(step), _ptr(loss), _ptr(grads),
                                        C.c_int32(int(accumulate))))

    def train_step_host(self, params, pos_src_host, pos_dst_host, k: int, seed: int, step: int, edge_index_base: int = 0,
                        adam_m=None, adam_v=None, adam_t: int = 1, loss_host=None, grads_host=None):
        self._ck(self.lib.lp_train_step_host(self.h, _ptr(params), _ptr(pos_src_host), _ptr(pos_dst_host), C.c_int64(pos_src_host.shape[0]),
                                             C.c_int32(k), C.c_uint64(seed), C.c_uint64(step), C.c_int64(edge_index_base), _ptr(adam_m),
                                             _ptr(adam_v), C.c_int64(adam_t), _ptr(loss_host), _ptr(grads_host)))

    def adam_step(self, params, m, v, grads, t: int, grad_scale: float = 1.0, lr: float = 1e-3, beta1: float = 0.9, beta2: float = 0.999,
                  eps: float = 1e-8):
        self._ck(self.lib.lp_adam_step(self.h, _ptr(params), _ptr(m), _ptr(v), _ptr(grads), C.c_double(grad_scale), C.c_double(lr),
                                       C.c_double(beta1), C.c_double(beta2), C.c_double(eps), C.c_int64(t)))

    def score(self, params, src, dst, seed: int = 0, step: int = 0):
        t = self._torch
        out = t.empty(src.numel(), dtype=t.float32, device=src.device)
        self._ck(self.lib.lp_score(self.h, _ptr(params), _ptr(src), _ptr(dst), C.c_int64(src.numel()), C.c_uint64(seed), C.c_uint64(step),
                                   _ptr(out)))
        return out

    def invalidate_embeddings(self):
        """Tell the library that the weights changed outside its own calls (see lp_score)."""
        self._ck(self.lib.lp_invalidate_embeddings(self.h))

    def set_wait_limit(self, limit_ns: int, overdeclare_bytes: int = 0):
        """Bound of the device-side waits of the tensor-core kernels; overdeclare_bytes > 0 makes the next such
        launch run into that bound (self-test of the LP_ETIMEOUT path)."""
        self._ck(self.lib.lp_set_wait_limit(self.h, C.c_uint64(limit_ns), C.c_int32(overdeclare_bytes)))

    def hits_at_k(self, pos_scores, neg_scores, k: int) -> float:
        """Hits@K of device score vectors (float32)."""
        out = C.c_double()
        self._ck(self.lib.lp_hits_at_k(self.h, _ptr(pos_scores), C.c_int64(pos_scores.numel()), _ptr(neg_scores), C.c_int64(neg_scores.numel()),
                                       C.c_int64(k), C.byref(out)))
        return float(out.value)

    # ---- learned node features (the checks are written for speed: a small call takes longer to make than to run)
    def _refuse(self, message: str):
        raise LpError(-1, message)

    def _prec(self, dtype, who: str) -> int:
        p = self._precs.get(dtype)
        if p is None:
            self._refuse(f"{who}: float32 or bfloat16 expected, got {dtype}")
        return p

    def _padding(self, padding_id, who: str) -> int:
        if padding_id is None:
            return LP_NO_PADDING
        if not -(1 << 31) <= padding_id < 1 << 31:  # ctypes would keep the low 32 bits, which are another id
            self._refuse(f"{who}: padding_id {padding_id} is no 32-bit id")
        return padding_id

    def _steps(self, steps, who: str) -> int:
        if not 1 <= steps <= 64:
            self._refuse(f"{who}: steps must be in [1, 64]")
        return steps

    def _rows(self, x, who: str):
        """(rows, width, row pitch) of a CUDA matrix whose rows are contiguous."""
        if x.get_device() != self.device or x.dim() != 2:
            self._refuse(f"{who}: expected a matrix on cuda:{self.device}")
        rows, width = x.shape
        ld, step = x.stride()
        if step != 1 and width > 1:
            self._refuse(f"{who}: the elements of a row must be contiguous")
        return rows, width, ld if rows > 1 or ld > width else width

    def _ids(self, ids, who: str):
        if ids.dtype is not self._torch.int32 or ids.get_device() != self.device or not ids.is_contiguous():
            self._refuse(f"{who}: ids must be a contiguous int32 tensor on cuda:{self.device}")

    def _enter(self, *tensors):
        """Work goes to the context's stream.  Called from another current stream, it waits for what that stream has
        enqueued so far, and the tensors are kept from reuse until it is done; returns the stream to hand back to."""
        t = self._torch
        if t._C._cuda_getCurrentRawStream(self.device) == self._raw_stream:
            return None
        cur = t.cuda.current_stream(self.device)
        self.stream.wait_stream(cur)
        for x in tensors:
            if x is not None:
                x.record_stream(self.stream)
        return cur

    def _leave(self, cur):
        if cur is not None:
            cur.wait_stream(self.stream)

    def embed(self, table, ids, scale: float = 1.0, padding_id: Optional[int] = None, out_dtype=None, out=None):
        """scale * table[ids] (ids int32, any shape; rows of zeros for padding_id); see lp_embed."""
        self._ids(ids, "embed")
        V, D, ldt = self._rows(table, "embed: table")
        N = ids.numel()
        if out is None:
            shape = (N, D) if ids.dim() == 1 else (*ids.shape, D)
            out = table.new_empty(shape) if out_dtype is None else table.new_empty(shape, dtype=out_dtype)
            ldo = D
        else:
            n, d, ldo = self._rows(out, "embed: out")
            if n != N or d != D or (out_dtype is not None and out.dtype != out_dtype):
                self._refuse(f"embed: out must be [{N}, {D}] of the requested type")
        cur = self._enter(table, ids, out)
        rc = self.lib.lp_embed(self.h, self._prec(table.dtype, "embed: table"), table.data_ptr(), V, D, ldt, ids.data_ptr(), N,
                               self._padding(padding_id, "embed"), scale, self._prec(out.dtype, "embed: out"), out.data_ptr(), ldo)
        if rc:
            self._ck(rc)
        if cur is not None:
            self._leave(cur)
        return out

    def embed_grad(self, dout, ids, rows: int, scale: float = 1.0, padding_id: Optional[int] = None, grad=None, grad_dtype=None, accumulate: bool = False):
        """Gradient [rows, width] of the table of embed(); see lp_embed_grad.  accumulate adds to `grad`."""
        self._ids(ids, "embed_grad")
        N, D, ldd = self._rows(dout, "embed_grad: dout")
        if ids.numel() != N:
            self._refuse(f"embed_grad: {ids.numel()} ids for {N} rows of dout")
        if grad is None:
            if accumulate:
                self._refuse("embed_grad: accumulate needs a gradient to add to")
            grad = dout.new_empty((rows, D), dtype=grad_dtype or self._torch.float32)
            ldg = D
        else:
            n, d, ldg = self._rows(grad, "embed_grad: grad")
            if n != rows or d != D or (grad_dtype is not None and grad.dtype != grad_dtype):
                self._refuse(f"embed_grad: grad must be [{rows}, {D}] of the requested type")
        cur = self._enter(dout, ids, grad)
        rc = self.lib.lp_embed_grad(self.h, self._prec(dout.dtype, "embed_grad: dout"), dout.data_ptr(), ldd, ids.data_ptr(), N,
                                    self._padding(padding_id, "embed_grad"), scale, rows, D, self._prec(grad.dtype, "embed_grad: grad"),
                                    grad.data_ptr(), ldg, accumulate)
        if rc:
            self._ck(rc)
        if cur is not None:
            self._leave(cur)
        return grad

    # ---- orthogonalised updates
    def orthogonalize(self, U, steps: int = 5, coeffs: Optional[Sequence[float]] = None, eps: float = 1e-7, out=None):
        """Newton-Schulz orthogonalisation of U [..., rows, cols] (float32 or bfloat16); see lp_orthogonalize."""
        if U.dim() < 2:
            self._refuse("orthogonalize: expected matrices")
        shape = U.shape
        U3 = U if U.dim() <= 3 else U.reshape(-1, shape[-2], shape[-1])
        if U3.get_device() != self.device or (shape[-1] > 1 and U3.stride(-1) != 1):
            self._refuse(f"orthogonalize: expected matrices with contiguous rows on cuda:{self.device}")
        if out is None:
            out = U.new_empty(shape)
        elif out.shape != shape or out.dtype != U.dtype or out.get_device() != self.device or out.dim() > 3 or (shape[-1] > 1 and out.stride(-1) != 1):
            self._refuse("orthogonalize: out must have the shape, type and device of U, with contiguous rows, and at most three dimensions")
        O3 = out if out.dim() <= 3 else out.view(-1, shape[-2], shape[-1])
        rows, cols = shape[-2], shape[-1]
        batch = U3.shape[0] if U3.dim() == 3 else 1
        ld_u, ld_o = (U3.stride(-2), O3.stride(-2)) if rows > 1 else (cols, cols)
        stride_u, stride_o = (U3.stride(0), O3.stride(0)) if batch > 1 else (rows * ld_u, rows * ld_o)
        c = (C.c_double * 3)(*coeffs) if coeffs is not None else None
        cur = self._enter(U, U3, out)
        self._ck(self.lib.lp_orthogonalize(self.h, self._prec(U.dtype, "orthogonalize"), batch, rows, cols, U3.data_ptr(), ld_u, stride_u,
                                           self._steps(steps, "orthogonalize"), c, eps, O3.data_ptr(), ld_o, stride_o))
        self._leave(cur)
        return out

    def muon_step(self, params, momentum, adam_v, grads, t: int, matrices=None, lr: float = 0.02, mu: float = 0.95, nesterov: bool = True,
                  weight_decay: float = 0.0, steps: int = 5, coeffs: Optional[Sequence[float]] = None, ns_eps: float = 1e-7, grad_scale: float = 1.0,
                  adam_lr: float = 1e-3, beta1: float = 0.9, beta2: float = 0.999, adam_eps: float = 1e-8, out=None):
        """Orthogonalised-momentum update of the weight matrices, Adam for the rest of the flat vector; see lp_muon_step.
        matrices: (offset, rows, cols) triples, or None for the matrices of the model.  Updates in place, or writes the new
        (params, momentum, adam_v) to `out`.  Returns (params, momentum, adam_v)."""
        f32 = self._torch.float32
        n = params.numel()
        new = (params, momentum, adam_v) if out is None else tuple(out)
        for x in (params, momentum, adam_v, grads, *new):
            if x is not None and (not x.is_cuda or x.device.index != self.device or x.dtype != f32 or x.numel() != n or not x.is_contiguous()):
                self._refuse(f"muon_step: expected contiguous float32 vectors of {n} elements on cuda:{self.device}")
        d = MuonDesc(grad_scale, lr, mu, weight_decay, (C.c_double * 3)(*(coeffs or (0.0, 0.0, 0.0))), ns_eps, adam_lr, beta1, beta2, adam_eps, int(nesterov),
                     self._steps(steps, "muon_step"))
        mats = None
        if matrices is not None:
            if any(not -(1 << 31) <= size < 1 << 31 for mat in matrices if not isinstance(mat, Matrix) for size in mat[1:3]):
                self._refuse("muon_step: a matrix has 1 to 2^17 rows and columns")
            mats = (Matrix * max(len(matrices), 1))(*matrices)
        p = [x.data_ptr() if x is not None else None for x in (params, momentum, adam_v, grads, *new)]
        cur = self._enter(params, momentum, adam_v, grads, *new)
        self._ck(self.lib.lp_muon_step(self.h, C.byref(d), mats, 0 if matrices is None else len(matrices), n, p[0], p[1], p[2], p[3], t, p[4], p[5], p[6]))
        self._leave(cur)
        return new

    # ---- residual blocks
    def dropout(self, x, p: float, seed: int, step: int, row_base: int = 0, out=None):
        """Dropout of a matrix (float32 or bfloat16); the gradient is the same call on the gradient.  See lp_dropout."""
        shape = x.shape
        prec = self._precs.get(x.dtype)
        if len(shape) != 2 or prec is None:
            self._refuse(f"dropout: expected a float32 or bfloat16 matrix on cuda:{self.device}")
        if not (0 <= seed < 1 << 64 and 0 <= step < 1 << 64 and 0 <= row_base < 1 << 62):
            self._refuse("dropout: seed and step are 64-bit numbers, row_base a number of rows")
        if shape[1] >= 1 << 31:
            self._refuse("dropout: width must be in [1, 2^20]")
        if out is None:
            out = self._empty_like(x)
        a, lda = self._matrix(x, shape, x.dtype, "dropout", "x")
        b, ldb = self._matrix(out, shape, x.dtype, "dropout", "out")
        cur = None
        if self._torch._C._cuda_getCurrentRawStream(self.device) != self._raw_stream:
            cur = self._enter(x, out)
        rc = self.lib.lp_dropout(self.h, prec, shape[0], shape[1], a, lda, p, seed, step, row_base, b, ldb)
        if rc:
            self._ck(rc)
        if cur is not None:
            self._leave(cur)
        return out

    def _column(self, v, width: int, who: str, name: str) -> int:
        """Address of a vector of the columns, 0 for None."""
        if v is None:
            return 0
        if v.dtype is not self._f32 or v.get_device() != self.device or v.numel() != width or not v.is_contiguous():
            self._refuse(f"{who}: {name} must be a contiguous float32 vector of {width} elements on cuda:{self.device}")
        return v.data_ptr()

    def _matrix(self, v, shape, dtype, who: str, name: str):
        """(address, row pitch) of a matrix that must have this shape and type; (None, width) for None."""
        if v is None:
            return None, shape[1]
        if v.shape != shape or v.dtype is not dtype or v.get_device() != self.device:
            self._refuse(f"{who}: {name} must be [{shape[0]}, {shape[1]}] of {dtype} on cuda:{self.device}")
        ld, step = v.stride()
        if step != 1 and shape[1] > 1:
            self._refuse(f"{who}: the elements of a row must be contiguous")
        return v.data_ptr(), ld if shape[0] > 1 or ld > shape[1] else shape[1]

    def _residual(self, who, like, dtype, pre_norm, pre, pre_bias, post_norm, post, post_bias, gate, scale, p, seed, step, row_base, eps):
        """The descriptor (lp_residual_desc as bytes) and the shape of the call's matrices."""
        shape = like.shape
        if len(shape) != 2 or like.get_device() != self.device:
            self._refuse(f"{who}: expected a matrix on cuda:{self.device}")
        if pre_norm not in _NORMS or post_norm not in _NORMS:
            self._refuse(f"{who}: norms are 'rms', 'layer' or None")
        if not (0 <= seed < 1 << 64 and 0 <= step < 1 << 64 and 0 <= row_base < 1 << 62):
            self._refuse(f"{who}: seed and step are 64-bit numbers, row_base a number of rows")
        rows, width = shape
        if width >= 1 << 31:
            self._refuse(f"{who}: width must be in [1, 8192]")
        g = ldg = 0
        if gate is not None:
            if gate.dim() == 1:
                g = self._column(gate, width, who, "gate")
            else:
                g, ldg = self._matrix(gate, shape, dtype, who, "gate")
        prec_s, prec_d = self._precs.get(like.dtype), self._precs.get(dtype)
        if prec_s is None or prec_d is None:
            self._refuse(f"{who}: float32 or bfloat16 expected, got {like.dtype} and {dtype}")
        return shape, _RESIDUAL.pack(rows, width, prec_s, prec_d, _NORMS[pre_norm], _NORMS[post_norm], eps, scale, p, seed, step, row_base,
                                     pre is not None and self._column(pre, width, who, "pre"), pre_bias is not None and self._column(pre_bias, width, who, "pre_bias"),
                                     post is not None and self._column(post, width, who, "post"), post_bias is not None and self._column(post_bias, width, who, "post_bias"),
                                     g, ldg)

    def residual_norm(self, x, h=None, pre_norm: Optional[str] = "rms", pre=None, pre_bias=None, post_norm: Optional[str] = None, post=None, post_bias=None,
                      gate=None, scale: float = 1.0, p: float = 0.0, seed: int = 0, step: int = 0, row_base: int = 0, eps: float = 1e-6, y=None, n=None, dtype=None):
        """y = x + scale * gate * dropout(post(h)) and n = pre(y); returns (y, n).  Without h only the norm is taken and y is x;
        without pre_norm n is None.  dtype: type of n where there is no h to say it.  See lp_residual_norm."""
        if h is not None:
            dtype = h.dtype
        elif dtype is None:
            dtype = n.dtype if n is not None else x.dtype
        shape, desc = self._residual("residual_norm", x, dtype, pre_norm, pre, pre_bias, post_norm, post, post_bias, gate, scale, p, seed, step, row_base, eps)
        if h is None:
            if y is not None and y is not x:
                self._refuse("residual_norm: without h there is no y to write")
            y = x
        elif y is None:
            y = self._empty_like(x)
        if pre_norm is None:
            if n is not None:
                self._refuse("residual_norm: without pre_norm there is no n to write")
        elif n is None:
            n = self._empty_like(x if h is None else h, dtype=dtype)
        a, lda = self._matrix(x, shape, x.dtype, "residual_norm", "x")
        b, ldb = self._matrix(h, shape, dtype, "residual_norm", "h")
        c, ldc = self._matrix(y, shape, x.dtype, "residual_norm", "y")
        d, ldd = self._matrix(n, shape, dtype, "residual_norm", "n")
        cur = None
        if self._torch._C._cuda_getCurrentRawStream(self.device) != self._raw_stream:
            cur = self._enter(x, h, y, n, pre, pre_bias, post, post_bias, gate)
        rc = self.lib.lp_residual_norm(self.h, desc, a, lda, b, ldb, c, ldc, d, ldd)
        if rc:
            self._ck(rc)
        if cur is not None:
            self._leave(cur)
        return y, n

    def residual_norm_grad(self, dy, dn, y, h=None, pre_norm: Optional[str] = "rms", pre=None, pre_bias=None, post_norm: Optional[str] = None, post=None,
                           post_bias=None, gate=None, scale: float = 1.0, p: float = 0.0, seed: int = 0, step: int = 0, row_base: int = 0, eps: float = 1e-6,
                           accumulate: bool = False, dx=None, dh=None, dgate=None, dpre=None, dpre_bias=None, dpost=None, dpost_bias=None):
        """Gradients of residual_norm: dx, dh, dgate and those of the norms' parameters that were given, as a dict.  dy may be None
        (zero) where there is a pre_norm; dn is None exactly where there is none.  Results may be given (accumulate adds to the vectors
        among them).  See lp_residual_norm_grad."""
        who = "residual_norm_grad"
        like = y if y is not None else dy
        if like is None:
            self._refuse(f"{who}: neither y nor dy")
        dtype = h.dtype if h is not None else dn.dtype if dn is not None else like.dtype
        shape, desc = self._residual(who, like, dtype, pre_norm, pre, pre_bias, post_norm, post, post_bias, gate, scale, p, seed, step, row_base, eps)
        width = shape[1]
        out = {"dx": dx if dx is not None else self._empty_like(like)}
        if h is not None:
            out["dh"] = dh if dh is not None else self._empty_like(like, dtype=dtype)
        elif dh is not None:
            self._refuse(f"{who}: a gradient of h is wanted and there is no h")
        gate_column = False
        if gate is not None and h is not None:
            gate_column = gate.dim() == 1
            if not gate_column:
                out["dgate"] = dgate if dgate is not None else self._empty_like(like, dtype=dtype)
        elif dgate is not None:
            self._refuse(f"{who}: a gradient of the gate is wanted and there is no gate")
        columns = [0, 0, 0, 0, 0]
        if pre_norm is None:
            pre = pre_bias = None  # residual_norm does not look at the parameters of a norm that is not taken
        if post_norm is None or h is None:
            post = post_bias = None
        for i, (name, param, given) in enumerate((("dpre", pre, dpre), ("dpre_bias", pre_bias, dpre_bias), ("dpost", post, dpost), ("dpost_bias", post_bias, dpost_bias),
                                                  ("dgate", gate if gate_column else None, dgate if gate_column else None))):
            if given is None:
                if param is None:
                    continue
                if accumulate:
                    self._refuse(f"{who}: accumulate needs a {name} to add to")
                given = like.new_empty(width, dtype=self._f32)
            out[name] = given
            columns[i] = self._column(given, width, who, name)
        a = (*self._matrix(dy, shape, like.dtype, who, "dy"), *self._matrix(dn, shape, dtype, who, "dn"), *self._matrix(y, shape, like.dtype, who, "y"),
             *self._matrix(h, shape, dtype, who, "h"), *self._matrix(out["dx"], shape, like.dtype, who, "dx"), *self._matrix(out.get("dh"), shape, dtype, who, "dh"))
        a += (columns[4], width) if gate_column else self._matrix(out.get("dgate"), shape, dtype, who, "dgate")
        cur = None
        if self._torch._C._cuda_getCurrentRawStream(self.device) != self._raw_stream:
            cur = self._enter(dy, dn, y, h, pre, pre_bias, post, post_bias, gate, *out.values())
        rc = self.lib.lp_residual_norm_grad(self.h, desc, *a, *columns[:4], accumulate)
        if rc:
            self._ck(rc)
        if cur is not None:
            self._leave(cur)
        return out

    # ---- products by group
    def _offsets(self, offsets, who: str) -> int:
        if offsets.dtype is not self._torch.int32 or offsets.get_device() != self.device or not offsets.is_contiguous() or offsets.dim() != 1 or offsets.numel() < 1:
            self._refuse(f"{who}: offsets must be a contiguous int32 vector on cuda:{self.device} of one more element than there are groups")
        return offsets.numel() - 1

    def grouped_linear(self, A, offsets, B, bias=None, relu: bool = False, trans_b: bool = False, out=None):
        """act(A[r] B[g] + bias[g]) for the rows offsets[g] <= r < offsets[g + 1]; B [groups, K, N], or [groups, N, K] with trans_b.
        Rows outside the groups are left as they are in `out`.  See lp_grouped_linear."""
        who = "grouped_linear"
        M, K, lda = self._rows(A, who)
        groups = self._offsets(offsets, who)
        if B.dim() != 3 or B.get_device() != self.device or B.dtype != A.dtype or not B.is_contiguous() or B.shape[0] != groups or B.shape[2 if trans_b else 1] != K:
            self._refuse(f"{who}: B must be {f'[{groups}, N, {K}]' if trans_b else f'[{groups}, {K}, N]'}, contiguous, of the type of A and on its device")
        N = B.shape[1 if trans_b else 2]
        if K >= 1 << 31 or N >= 1 << 31:
            self._refuse(f"{who}: widths must be in [1, 2^20]")
        if bias is not None and (bias.dtype is not self._torch.float32 or bias.get_device() != self.device or bias.shape != (groups, N) or not bias.is_contiguous()):
            self._refuse(f"{who}: bias must be a contiguous float32 matrix [{groups}, {N}] on cuda:{self.device}")
        prec = self._prec(A.dtype, who)
        if out is None:
            out, ldc = A.new_empty((M, N)), N
        else:
            r, d, ldc = self._rows(out, who)
            if r != M or d != N or out.dtype != A.dtype:
                self._refuse(f"{who}: out must be [{M}, {N}] of the type of A")
        cur = None
        if self._torch._C._cuda_getCurrentRawStream(self.device) != self._raw_stream:
            cur = self._enter(A, offsets, B, bias, out)
        rc = self.lib.lp_grouped_linear(self.h, prec, M, N, K, groups, offsets.data_ptr(), A.data_ptr(), lda, B.data_ptr(), trans_b,
                                        None if bias is None else bias.data_ptr(), relu, out.data_ptr(), ldc)
        if rc:
            self._ck(rc)
        if cur is not None:
            self._leave(cur)
        return out

    def grouped_weight_grad(self, A, dZ, offsets, bias: bool = False, accumulate: bool = False, dW=None, dbias=None):
        """Weight gradients of grouped_linear: dW[g] = A_g^T dZ_g, [groups, K, N] float32, and with bias=True (or a given dbias)
        (dW, column sums of dZ_g).  See lp_grouped_weight_grad."""
        who = "grouped_weight_grad"
        M, K, lda = self._rows(A, who)
        m, N, ldz = self._rows(dZ, who)
        groups = self._offsets(offsets, who)
        if m != M or dZ.dtype != A.dtype or K >= 1 << 31 or N >= 1 << 31:
            self._refuse(f"{who}: dZ must have {M} rows of the type of A")
        f32 = self._torch.float32
        bias = bias or dbias is not None
        if accumulate and (dW is None or (bias and dbias is None)):
            self._refuse(f"{who}: accumulate needs gradients to add to")
        for x, shape in ((dW, (groups, K, N)), (dbias, (groups, N))):
            if x is not None and (x.dtype is not f32 or x.get_device() != self.device or x.shape != shape or not x.is_contiguous()):
                self._refuse(f"{who}: gradients must be contiguous float32 tensors {(groups, K, N)} and {(groups, N)} on cuda:{self.device}")
        prec = self._prec(A.dtype, who)
        if dW is None:
            dW = A.new_empty((groups, K, N), dtype=f32)
        if bias and dbias is None:
            dbias = A.new_empty((groups, N), dtype=f32)
        cur = None
        if self._torch._C._cuda_getCurrentRawStream(self.device) != self._raw_stream:
            cur = self._enter(A, dZ, offsets, dW, dbias)
        rc = self.lib.lp_grouped_weight_grad(self.h, prec, M, N, K, groups, offsets.data_ptr(), A.data_ptr(), lda, dZ.data_ptr(), ldz, accumulate, dW.data_ptr(),
                                             None if dbias is None else dbias.data_ptr())
        if rc:
            self._ck(rc)
        if cur is not None:
            self._leave(cur)
        return (dW, dbias) if bias else dW

    # ---- inspection
    def stats(self) -> Stats:
        s = Stats()
        self._ck(self.lib.lp_get_stats(self.h, C.byref(s)))
        return s

    def embeddings(self, layer: int, rows: Optional[int] = None):
        t = self._torch
        rows = self.n if rows is None else rows
        out = t.empty((rows, self.dims[layer]), dtype=t.float32, device=f"cuda:{self.device}")
        self._ck(self.lib.lp_get_embeddings(self.h, C.c_int32(layer), _ptr(out)))
        return out

    def predictor_activations(self, layer: int, E: int):
        t = self._torch
        out = t.empty((E, int(self.desc.pred_hidden)), dtype=t.float32, device=f"cuda:{self.device}")
        self._ck(self.lib.lp_get_predictor_activations(self.h, C.c_int32(layer), C.c_int64(E), _ptr(out)))
        return out

    def output_gradient(self, rows: Optional[int] = None):
        t = self._torch
        rows = self.n if rows is None else rows
        out = t.empty((rows, self.dims[-1]), dtype=t.float32, device=f"cuda:{self.device}")
        self._ck(self.lib.lp_get_output_gradient(self.h, _ptr(out)))
        return out

    def block(self, hop: int):
        """(frontier F_hop or None for the outermost hop, blk_ptr, blk_col) of the last sampled step."""
        t = self._torch
        dev = f"cuda:{self.device}"
        s = self.stats()
        frontier = None
        if hop < self.K:
            frontier = t.empty(int(s.block_nodes[hop]), dtype=t.int32, device=dev)
        ptr = col = None
        if hop >= 1:
            ptr = t.empty(int(s.block_nodes[hop - 1]) + 1, dtype=t.int64, device=dev)
            col = t.empty(max(int(s.block_edges[hop - 1]), 1), dtype=t.int32, device=dev)
        self._ck(self.lib.lp_get_block(self.h, C.c_int32(hop), _ptr(frontier), _ptr(ptr), _ptr(col)))
        if col is not None:
            col = col[: int(s.block_edges[hop - 1])]
        return frontier, ptr, col

    # ---- per-kernel timing
    def profile_begin(self, categories=None):
        mask = 0
        for c in (categories if categories is not None else PROF_CATEGORIES):
            mask |= 1 << PROF_CATEGORIES.index(c)
        self._ck(self.lib.lp_profile_begin(self.h, C.c_uint32(mask)))

    def profile_sample_every(self, n: int):
        self._ck(self.lib.lp_profile_sample_every(self.h, C.c_uint32(n)))

    def profile_end(self):
        p = Profile()
        self._ck(self.lib.lp_profile_end(self.h, C.byref(p)))
        return {name: {"ms": p.ms[i], "bytes": p.bytes[i], "flops": p.flops[i], "spans": int(p.spans[i])}
                for i, name in enumerate(PROF_CATEGORIES)}

    # ---- single operators
    def op_aggregate(self, arch: str, H, transpose: bool = False):
        t = self._torch
        M = t.empty_like(H)
        self._ck(self.lib.lp_op_aggregate(self.h, C.c_int32(LP_GCN if arch == "gcn" else LP_SAGE_MEAN), C.c_int32(int(transpose)),
                                          C.c_int32(int(H.dtype == t.bfloat16)), _ptr(H), C.c_int32(H.shape[1]), _ptr(M)))
        return M

    def op_gather_ceiling(self, H, transpose: bool = False):
        """XOR folds of the rows of H named by every run of 64 stored entries (see lp_op_gather_ceiling)."""
        t = self._torch
        row_bytes = H.shape[1] * H.element_size()
        runs = (self.nnz + 63) // 64
        folds = t.empty((runs, row_bytes // 4), dtype=t.int32, device=H.device)
        self._ck(self.lib.lp_op_gather_ceiling(self.h, C.c_int32(int(transpose)), _ptr(H), C.c_int32(row_bytes), _ptr(folds)))
        return folds

    def op_linear(self, A, B, bias=None, relu: bool = False, trans_b: bool = False):
        t = self._torch
        M, K = A.shape
        N = B.shape[0] if trans_b else B.shape[1]
        Cout = t.empty((M, N), dtype=A.dtype, device=A.device)
        prec = LP_BF16 if A.dtype == t.bfloat16 else LP_FP32
        self._ck(self.lib.lp_op_linear(self.h, C.c_int32(prec), C.c_int64(M), C.c_int32(N), C.c_int32(K), _ptr(A), _ptr(B),
                                       C.c_int32(int(trans_b)), _ptr(bias), C.c_int32(int(relu)), _ptr(Cout)))
        return Cout

    def op_weight_grad(self, A, dZ):
        t = self._torch
        M, K = A.shape
        N = dZ.shape[1]
        dW = t.empty((K, N), dtype=t.float32, device=A.device)
        prec = LP_BF16 if A.dtype == t.bfloat16 else LP_FP32
        self._ck(self.lib.lp_op_weight_grad(self.h, C.c_int32(prec), C.c_int64(M), C.c_int32(N), C.c_int32(K), _ptr(A), _ptr(dZ), _ptr(dW)))
        return dW


def weight_grad_static(A, dZ, stream=None):
    """dW = A^T dZ (float32 CUDA tensors) through the allocation-free entry point.  The output
    tensor is allocated HERE, by torch, before the call: the library call itself allocates nothing.
    For callers that cannot allocate at call time (allocator-free loops, pre-pooled memory)."""
    import torch

    lib = load_library()
    M, K = A.shape
    N = dZ.shape[1]
    dW = torch.empty((K, N), dtype=torch.float32, device=A.device)
    st = stream if stream is not None else torch.cuda.current_stream(A.device)
    rc = lib.lp_weight_grad_static(C.c_int32(A.device.index or 0), C.c_void_p(st.cuda_stream), C.c_int64(M), C.c_int32(N), C.c_int32(K),
                                   _ptr(A), _ptr(dZ), _ptr(dW))
    if rc != LP_OK:
        raise LpError(rc, lib.lp_last_error(None).decode())
    return dW
