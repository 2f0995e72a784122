"""ctypes binding of the C ABI in include/distshap.h.

Every method of `Context` is one call of the function of the same name
(`Context.explain` -> `ds_explain`, ...): it only allocates output tensors,
passes device pointers, and turns a non-zero status into `DistShapError`.
There is no fallback: without the built library every call raises.
"""
import ctypes as C
import os
from typing import Any, NamedTuple

DS_OK, DS_EINVAL, DS_ECAPACITY, DS_ENOMEM, DS_ENOTCONV, DS_EDEVICE, DS_ESINGULAR, DS_EINTERNAL = range(8)
DS_F32, DS_BF16_IN_F32_ACC = 0, 1
DS_SCORE_PROB, DS_SCORE_LOGIT = 0, 1
DS_SOLVER_AUTO, DS_SOLVER_GRAM_CHOL, DS_SOLVER_CGLS = 0, 1, 2
DS_WEIGHT_CLASS_MASS, DS_WEIGHT_UNIFORM = 0, 1
DS_ELEM_F32, DS_ELEM_BF16, DS_ELEM_F16 = 0, 1, 2

EXPORTED_SYMBOLS = [
    "ds_create", "ds_destroy", "ds_last_error", "ds_set_tuning", "ds_set_graph", "ds_set_features", "ds_set_gcn", "ds_set_gat",
    "ds_explain", "ds_explain_cgraph", "ds_explain_batch", "ds_extract", "ds_cgraph_get_info", "ds_cgraph_edges",
    "ds_cgraph_nodes", "ds_cgraph_first_transform", "ds_cgraph_free", "ds_sample_plan", "ds_sample",
    "ds_plan_tables", "ds_plan_tables_ex", "ds_sample_ex", "ds_sample_range", "ds_eval", "ds_eval_pairs", "ds_eval_noalloc", "ds_solve", "ds_fidelity", "ds_copy_probe", "ds_version",
    "ds_layer_norm", "ds_layer_norm_backward_workspace", "ds_layer_norm_backward", "ds_dropout", "ds_group_rows_workspace",
    "ds_group_rows", "ds_grouped_mm", "ds_grouped_mm_backward_workspace", "ds_grouped_mm_backward",
    "ds_embed", "ds_embed_backward_workspace", "ds_embed_backward", "ds_route_workspace", "ds_route", "ds_route_backward",
    "ds_pack_rows", "ds_unpack_rows", "ds_grouped_mm_backward_packed_workspace", "ds_grouped_mm_backward_packed",
]


class Options(C.Structure):
    _fields_ = [("hops", C.c_int32), ("directed", C.c_int32), ("score", C.c_int32),
                ("solver", C.c_int32), ("tol", C.c_double), ("max_iter", C.c_int32),
                ("batch_rows", C.c_int32), ("paired", C.c_int32), ("weighting", C.c_int32),
                ("saturate", C.c_int32)]


class Tuning(C.Structure):
    _fields_ = [("batch_workers", C.c_int32), ("gram_sparse_div", C.c_int32), ("gram_dense_fraction", C.c_float),
                ("sampler_window", C.c_int32), ("eval_path", C.c_int32), ("cgls_dense_div", C.c_int32),
                ("pair_lists", C.c_int32)]


class Report(C.Structure):
    _fields_ = [("num_players", C.c_int64), ("num_nodes", C.c_int64), ("num_entries", C.c_int64),
                ("num_rows", C.c_int64), ("enumerated", C.c_int32), ("pred_class", C.c_int32),
                ("solver_used", C.c_int32), ("cgls_iterations", C.c_int32),
                ("cgls_rel_residual", C.c_double), ("f_empty", C.c_double), ("f_full", C.c_double),
                ("ms_extract", C.c_float), ("ms_sample", C.c_float), ("ms_eval", C.c_float),
                ("ms_solve", C.c_float), ("ms_total", C.c_float),
                ("ms_k_eval", C.c_float), ("ms_k_gram", C.c_float), ("ms_k_chol", C.c_float),
                ("ms_k_cgls", C.c_float),
                ("num_pairs", C.c_int64), ("bytes_sample", C.c_double), ("bytes_eval", C.c_double),
                ("bytes_solve", C.c_double), ("ms_k_stream", C.c_float)]

    def as_dict(self):
        return {name: getattr(self, name) for name, _ in self._fields_}


class CGraphInfo(C.Structure):
    _fields_ = [("num_players", C.c_int64), ("num_nodes", C.c_int64), ("num_entries", C.c_int64),
                ("target", C.c_int64), ("hops", C.c_int32), ("directed", C.c_int32),
                ("ball", C.c_int64 * 8)]


class Packed(NamedTuple):
    """Rows held in 8 bits: x ~ codes * 2^(scales - 127), one scale for 32 neighbouring columns (`Context.pack_rows`)."""
    codes: Any    # float8_e4m3fn[rows, cols]
    scales: Any   # uint8[rows, ceil(cols / 32)]


class DistShapError(RuntimeError):
    def __init__(self, code, message):
        super().__init__(f"distshap status {code}: {message}")
        self.code = code


_no_gradient_class = None


def _no_gradient():
    """The autograd function of a call whose gradient is a call of its own: its backward pass is an error."""
    global _no_gradient_class
    if _no_gradient_class is None:
        import torch

        class NoGradient(torch.autograd.Function):
            @staticmethod
            def forward(ctx, call, outputs, *inputs):
                ctx.call = call
                return outputs

            @staticmethod
            def backward(ctx, *grads):
                raise DistShapError(DS_EINVAL, f"autograd cannot go through {ctx.call}: its gradient is a call of its own (*_backward; dropout of the gradient)")

        _no_gradient_class = NoGradient
    return _no_gradient_class


def library_path():
    return os.path.join(os.path.dirname(os.path.abspath(__file__)), "libdistshap_hip.so")


_lib = None


def load_library():
    """Load the built library (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    # PyTorch ships its own HIP runtime: it has to be the one already in the process when this
    # library (linked against libamdhip64) is loaded, or two runtimes end up side by side
    import torch  # noqa: F401
    path = library_path()
    if not os.path.exists(path):
        raise FileNotFoundError(f"{path} is missing: run `python -m paper_2506_22668_amd.build` first")
    lib = C.CDLL(path)
    p, i32, i64, u64, u32, dbl = C.c_void_p, C.c_int32, C.c_int64, C.c_uint64, C.c_uint32, C.c_double
    sigs = {
        "ds_create": [C.POINTER(p), C.c_int, p],
        "ds_destroy": [p],
        "ds_set_tuning": [p, C.POINTER(Tuning)],
        "ds_set_graph": [p, i64, p, p],
        "ds_set_features": [p, p, i32, i32],
        "ds_set_gcn": [p, i32, C.POINTER(i32), C.POINTER(p), C.POINTER(p), i32],
        "ds_set_gat": [p, i32, C.POINTER(i32), C.POINTER(i32), C.POINTER(p), C.POINTER(p), C.POINTER(p), C.POINTER(p),
                       C.c_float],
        "ds_explain": [p, i64, i64, u64, C.POINTER(Options), p, C.POINTER(i64), p, p, C.POINTER(Report)],
        "ds_explain_cgraph": [p, p, i64, u64, C.POINTER(Options), p, C.POINTER(i64), p, p, C.POINTER(Report)],
        "ds_explain_batch": [p, C.POINTER(i64), i32, i64, u64, C.POINTER(Options), p, C.POINTER(i64),
                             C.POINTER(i64), p, p, i64, C.POINTER(Report)],
        "ds_extract": [p, i64, C.POINTER(Options), C.POINTER(p)],
        "ds_cgraph_get_info": [p, C.POINTER(CGraphInfo)],
        "ds_cgraph_edges": [p, p, p, p],
        "ds_cgraph_nodes": [p, p, p, p],
        "ds_cgraph_first_transform": [p, p, p],
        "ds_cgraph_free": [p, p],
        "ds_sample_plan": [i64, i64, C.POINTER(i64), C.POINTER(i32)],
        "ds_sample": [p, i64, i64, u64, u32, p, p, p, C.POINTER(i64)],
        "ds_plan_tables": [i64, i64, p, p],
        "ds_plan_tables_ex": [i64, i64, C.POINTER(Options), p, p, C.POINTER(i64)],
        "ds_sample_ex": [p, i64, i64, u64, u32, C.POINTER(Options), p, p, p, C.POINTER(i64)],
        "ds_sample_range": [p, i64, i64, u64, u32, i64, i64, p, p, p],
        "ds_eval": [p, p, p, i64, i32, p, C.POINTER(i32)],
        "ds_eval_pairs": [p, p, p, i64, i32, p, C.POINTER(i32)],
        "ds_eval_noalloc": [p, p, p, i64, i32, p],
        "ds_solve": [p, i64, i64, p, p, p, C.POINTER(Options), p, C.POINTER(Report)],
        "ds_copy_probe": [p, p, p, i64],
        "ds_fidelity": [p, p, p, C.POINTER(i64), i32, i32, C.POINTER(C.c_float), C.POINTER(C.c_float), p],
        "ds_layer_norm": [p, i32, i64, i64, p, i64, p, p, C.c_float, p, i64, p, p],
        "ds_layer_norm_backward_workspace": [i64, i64, C.POINTER(i64)],
        "ds_layer_norm_backward": [p, i32, i64, i64, p, i64, p, i64, p, p, p, p, i64, p, p, p, i64],
        "ds_dropout": [p, i32, i64, i64, p, i64, p, i64, dbl, u64, u32, p, i64],
        "ds_group_rows_workspace": [i64, i64, C.POINTER(i64)],
        "ds_group_rows": [p, p, i64, i64, p, p, p, i64],
        "ds_grouped_mm": [p, i32, i64, i64, i64, i64, p, i64, p, p, p, p, i32, p, i64],
        "ds_grouped_mm_backward_workspace": [i32, i64, i64, i64, i64, C.POINTER(i64)],
        "ds_grouped_mm_backward": [p, i32, i64, i64, i64, i64, p, i64, p, i64, p, p, p, p, i64, p, i64, p, p, p, i64],
        "ds_embed": [p, i32, i32, i64, i64, i64, p, i64, p, C.c_float, p, i64],
        "ds_embed_backward_workspace": [i64, i64, i64, C.POINTER(i64)],
        "ds_embed_backward": [p, i32, i32, i64, i64, i64, p, i64, p, C.c_float, p, i64, p, i64],
        "ds_route_workspace": [i64, i64, C.POINTER(i64)],
        "ds_route": [p, i32, i64, i64, i64, i32, p, i64, p, p, p, p, p, p, i64],
        "ds_route_backward": [p, i32, i64, i64, i64, i32, p, i64, p, p, p, p, p, p, i64],
        "ds_pack_rows": [p, i32, i64, i64, p, i64, p, i64, p, i64],
        "ds_unpack_rows": [p, i32, i64, i64, p, i64, p, i64, p, i64],
        "ds_grouped_mm_backward_packed_workspace": [i32, i64, i64, i64, i64, C.POINTER(i64)],
        "ds_grouped_mm_backward_packed": [p, i32, i64, i64, i64, i64, p, i64, p, i64, p, i64, p, p, p, p, i64, p, i64, p, p, p, i64],
    }
    for name, args in sigs.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = C.c_int
    lib.ds_last_error.argtypes = [p]
    lib.ds_last_error.restype = C.c_char_p
    lib.ds_version.argtypes = []
    lib.ds_version.restype = C.c_char_p
    _lib = lib
    return lib


def sample_plan(n, n_samples):
    """(k, enumerated) for n players and a sample budget (host-only call)."""
    lib = load_library()
    k, e = C.c_int64(), C.c_int32()
    rc = lib.ds_sample_plan(n, n_samples, C.byref(k), C.byref(e))
    if rc != DS_OK:
        raise DistShapError(rc, "ds_sample_plan: bad arguments")
    return k.value, bool(e.value)


def plan_tables(n, n_samples, options=None):
    """(b int64[H+1], wtab float32[H+1]) of the sampling plan (host-only call); with `options` also the number of
    enumerated size classes (ds_plan_tables_ex)."""
    import numpy as np
    lib = load_library()
    H = n // 2
    b = np.zeros(H + 1, dtype=np.int64)
    wtab = np.zeros(H + 1, dtype=np.float32)
    if options is None:
        rc = lib.ds_plan_tables(n, n_samples, b.ctypes.data_as(C.c_void_p), wtab.ctypes.data_as(C.c_void_p))
        if rc != DS_OK:
            raise DistShapError(rc, "ds_plan_tables: bad arguments")
        return b, wtab
    upto = C.c_int64()
    rc = lib.ds_plan_tables_ex(n, n_samples, C.byref(options), b.ctypes.data_as(C.c_void_p),
                               wtab.ctypes.data_as(C.c_void_p), C.byref(upto))
    if rc != DS_OK:
        raise DistShapError(rc, "ds_plan_tables_ex: bad arguments")
    return b, wtab, upto.value


def _ptr(t):
    return C.c_void_p(t.data_ptr()) if t is not None else C.c_void_p(0)


class Context:
    """One ds_ctx on a torch device; keeps the tensors registered with ds_set_* alive."""

    def __init__(self, device="cuda:0", stream=None):
        import torch
        self.torch = torch
        self.lib = load_library()
        self.device = torch.device(device)
        idx = self.device.index if self.device.index is not None else 0
        self._stream = stream
        handle = C.c_void_p()
        sptr = C.c_void_p(stream.cuda_stream) if stream is not None else C.c_void_p(0)
        rc = self.lib.ds_create(C.byref(handle), idx, sptr)
        if rc != DS_OK:
            raise DistShapError(rc, "ds_create failed")
        self.h = handle
        self._keep = {}
        self._index = idx
        self._raw_stream = stream.cuda_stream if stream is not None else 0
        # the handle of torch's current stream (a seventh of a small call's time as the attribute of a Stream object made for it)
        self._current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)
        self._elements = {torch.float32: DS_ELEM_F32, torch.bfloat16: DS_ELEM_BF16, torch.float16: DS_ELEM_F16}

    def close(self):
        if getattr(self, "h", None):
            self.lib.ds_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, rc, allow=()):
        if rc != DS_OK and rc not in allow:
            raise DistShapError(rc, self.lib.ds_last_error(self.h).decode())
        return rc

    def _sync_inputs(self):
        # inputs were produced on torch's current stream; the library runs on its own
        self.torch.cuda.current_stream(self.device).synchronize()

    def set_tuning(self, tuning=None):
        self._check(self.lib.ds_set_tuning(self.h, C.byref(tuning) if tuning is not None else None))

    # -- registration --------------------------------------------------------
    def set_graph(self, row_ptr, col):
        t = self.torch
        rp = t.as_tensor(row_ptr, dtype=t.int64).to(self.device).contiguous()
        ci = t.as_tensor(col, dtype=t.int32).to(self.device).contiguous()
        self._sync_inputs()
        self._check(self.lib.ds_set_graph(self.h, rp.numel() - 1, _ptr(rp), _ptr(ci)))
        self._keep["graph"] = (rp, ci)

    def set_features(self, X):
        t = self.torch
        X = t.as_tensor(X, dtype=t.float32).to(self.device).contiguous()
        self._sync_inputs()
        self._check(self.lib.ds_set_features(self.h, _ptr(X), X.shape[1], DS_F32))
        self._keep["X"] = X

    def set_gcn(self, weights, biases=None, transform_dtype=DS_F32):
        t = self.torch
        Ws = [t.as_tensor(w, dtype=t.float32).to(self.device).contiguous() for w in weights]
        L = len(Ws)
        dims = [Ws[0].shape[0]] + [w.shape[1] for w in Ws]
        Bs = None
        if biases is not None:
            Bs = [None if b is None else t.as_tensor(b, dtype=t.float32).to(self.device).contiguous() for b in biases]
        self._sync_inputs()
        dims_c = (C.c_int32 * (L + 1))(*dims)
        W_c = (C.c_void_p * L)(*[w.data_ptr() for w in Ws])
        B_c = None
        if Bs is not None:
            B_c = (C.c_void_p * L)(*[(b.data_ptr() if b is not None else 0) for b in Bs])
        self._check(self.lib.ds_set_gcn(self.h, L, dims_c, W_c, B_c, transform_dtype))
        self._keep["model"] = (Ws, Bs)
        self.dims = dims
        self.first_width = dims[1]

    def set_gat(self, weights, att_src, att_dst, heads, biases=None, negative_slope=0.2):
        """weights[l]: [in_l, heads_l * width_l]; att_src[l], att_dst[l]: [heads_l, width_l]."""
        t = self.torch
        dev = lambda a: t.as_tensor(a, dtype=t.float32).to(self.device).contiguous()
        Ws, As, Ad = [dev(w) for w in weights], [dev(a) for a in att_src], [dev(a) for a in att_dst]
        L = len(Ws)
        heads = [int(h) for h in heads]
        head_dims = [Ws[0].shape[0]] + [Ws[l].shape[1] // heads[l] for l in range(L)]
        Bs = None
        if biases is not None:
            Bs = [None if b is None else dev(b) for b in biases]
        self._sync_inputs()
        arr = lambda ts: (C.c_void_p * L)(*[(x.data_ptr() if x is not None else 0) for x in ts])
        self._check(self.lib.ds_set_gat(self.h, L, (C.c_int32 * (L + 1))(*head_dims), (C.c_int32 * L)(*heads),
                                        arr(Ws), arr(As), arr(Ad), None if Bs is None else arr(Bs),
                                        C.c_float(negative_slope)))
        self._keep["model"] = (Ws, As, Ad, Bs)
        self.dims = [head_dims[0]] + [heads[l] * head_dims[l + 1] for l in range(L - 1)] + [head_dims[L]]
        self.first_width = heads[0] * head_dims[1]

    # -- one-shot --------------------------------------------------------------
    def explain(self, target, n_samples, seed, options=None, capacity=None, want_edges=True,
                allow_not_converged=False):
        t = self.torch
        opts = options or Options()
        target, n_samples, seed = int(target), int(n_samples), C.c_uint64(int(seed))
        cg = None
        if capacity is None:  # the buffers are sized by the extracted graph, which the explanation then takes over
            cg = self.extract(target, opts)
        try:
            capacity = int(capacity) if cg is None else self.cgraph_info(cg).num_players
            cap = max(capacity, 1)
            phi = t.empty(cap, dtype=t.float32, device=self.device)
            es = t.empty(cap, dtype=t.int64, device=self.device) if want_edges else None
            ed = t.empty(cap, dtype=t.int64, device=self.device) if want_edges else None
            m = C.c_int64(capacity)
            rep = Report()
            self._sync_inputs()
            args = (n_samples, seed, C.byref(opts), _ptr(phi), C.byref(m), _ptr(es), _ptr(ed), C.byref(rep))
        except BaseException:  # (no memory for the buffers, say: the graph has not been handed over)
            if cg is not None:
                self.lib.ds_cgraph_free(self.h, cg)
            raise
        if cg is not None:
            rc = self.lib.ds_explain_cgraph(self.h, cg, *args)
        else:
            rc = self.lib.ds_explain(self.h, target, *args)
        self._check(rc, allow=(DS_ENOTCONV,) if allow_not_converged else ())
        n = m.value
        return phi[:n], (es[:n] if want_edges else None), (ed[:n] if want_edges else None), rep, rc

    def explain_batch(self, targets, n_samples, seed, options=None, capacity=0):
        t = self.torch
        opts = options or Options()
        T = len(targets)
        cap = max(int(capacity), 1)
        phi = t.empty(cap, dtype=t.float32, device=self.device)
        es = t.empty(cap, dtype=t.int64, device=self.device)
        ed = t.empty(cap, dtype=t.int64, device=self.device)
        tg = (C.c_int64 * T)(*[int(x) for x in targets])
        M = (C.c_int64 * T)()
        off = (C.c_int64 * (T + 1))()
        reps = (Report * T)()
        self._sync_inputs()
        rc = self._check(self.lib.ds_explain_batch(self.h, tg, T, int(n_samples), C.c_uint64(int(seed)),
                                                   C.byref(opts), _ptr(phi), M, off, _ptr(es), _ptr(ed),
                                                   int(capacity), reps), allow=(DS_ECAPACITY, DS_ENOTCONV))
        return phi, list(M), list(off), es, ed, list(reps), rc

    # -- stage-wise --------------------------------------------------------------
    def extract(self, target, options=None):
        opts = options or Options()
        cg = C.c_void_p()
        self._sync_inputs()
        self._check(self.lib.ds_extract(self.h, int(target), C.byref(opts), C.byref(cg)))
        return cg

    def cgraph_info(self, cg):
        info = CGraphInfo()
        self._check(self.lib.ds_cgraph_get_info(cg, C.byref(info)))
        return info

    def cgraph_edges(self, cg):
        t = self.torch
        n = self.cgraph_info(cg).num_players
        es = t.empty(max(n, 1), dtype=t.int64, device=self.device)
        ed = t.empty(max(n, 1), dtype=t.int64, device=self.device)
        self._check(self.lib.ds_cgraph_edges(self.h, cg, _ptr(es), _ptr(ed)))
        return es[:n], ed[:n]

    def cgraph_nodes(self, cg):
        t = self.torch
        V = self.cgraph_info(cg).num_nodes
        gid = t.empty(V, dtype=t.int64, device=self.device)
        hop = t.empty(V, dtype=t.int32, device=self.device)
        self._check(self.lib.ds_cgraph_nodes(self.h, cg, _ptr(gid), _ptr(hop)))
        return gid, hop

    def cgraph_first_transform(self, cg):
        t = self.torch
        V = self.cgraph_info(cg).num_nodes
        out = t.empty((V, self.first_width), dtype=t.float32, device=self.device)
        self._check(self.lib.ds_cgraph_first_transform(self.h, cg, _ptr(out)))
        return out

    def cgraph_free(self, cg):
        self._check(self.lib.ds_cgraph_free(self.h, cg))

    def sample(self, n, n_samples, seed, tag, options=None):
        """ds_sample, or ds_sample_ex when `options` is given."""
        t = self.torch
        k, _ = sample_plan(n, n_samples)
        W = (n + 63) // 64
        Z = t.empty((max(k, 1), max(W, 1)), dtype=t.int64, device=self.device)
        w = t.empty(max(k, 1), dtype=t.float32, device=self.device)
        sz = t.empty(max(k, 1), dtype=t.int32, device=self.device)
        kout = C.c_int64()
        if options is None:
            self._check(self.lib.ds_sample(self.h, int(n), int(n_samples), C.c_uint64(int(seed)),
                                           C.c_uint32(int(tag) & 0xFFFFFFFF), _ptr(Z), _ptr(w), _ptr(sz),
                                           C.byref(kout)))
        else:
            self._check(self.lib.ds_sample_ex(self.h, int(n), int(n_samples), C.c_uint64(int(seed)),
                                              C.c_uint32(int(tag) & 0xFFFFFFFF), C.byref(options), _ptr(Z), _ptr(w),
                                              _ptr(sz), C.byref(kout)))
        assert kout.value == k
        return Z[:k], w[:k], sz[:k]

    def sample_range(self, n, n_samples, seed, tag, pair_begin, pair_end):
        t = self.torch
        rows = 2 * (pair_end - pair_begin)
        W = (n + 63) // 64
        Z = t.empty((max(rows, 1), max(W, 1)), dtype=t.int64, device=self.device)
        w = t.empty(max(rows, 1), dtype=t.float32, device=self.device)
        sz = t.empty(max(rows, 1), dtype=t.int32, device=self.device)
        self._check(self.lib.ds_sample_range(self.h, int(n), int(n_samples), C.c_uint64(int(seed)),
                                             C.c_uint32(int(tag) & 0xFFFFFFFF), int(pair_begin),
                                             int(pair_end), _ptr(Z), _ptr(w), _ptr(sz)))
        return Z[:rows], w[:rows], sz[:rows]

    def eval(self, cg, Z, score=DS_SCORE_PROB, pairs=False):
        """ds_eval, or ds_eval_pairs when `pairs` (rows 2r, 2r+1 complementary)."""
        t = self.torch
        Z = Z.contiguous()
        k = Z.shape[0]
        y = t.empty(max(k, 1), dtype=t.float32, device=self.device)
        pc = C.c_int32()
        self._sync_inputs()
        fn = self.lib.ds_eval_pairs if pairs else self.lib.ds_eval
        self._check(fn(self.h, cg, _ptr(Z), k, score, _ptr(y), C.byref(pc)))
        return y[:k], pc.value

    def eval_noalloc(self, cg, Z, y, score=DS_SCORE_PROB):
        """ds_eval_noalloc into the caller's y (float32[k]); queued on the context's stream, no synchronisation."""
        self._sync_inputs()
        self._check(self.lib.ds_eval_noalloc(self.h, cg, _ptr(Z), Z.shape[0], score, _ptr(y)))

    def synchronize(self):
        """Wait for the library's stream (the one given at creation, else the default stream)."""
        if self._stream is not None:
            self._stream.synchronize()
        else:
            self.torch.cuda.synchronize(self.device)

    def fidelity(self, cg, phi, ks, score=DS_SCORE_PROB, want_masks=False):
        """(fid_plus, fid_minus[, masks]) for the top-k sub-graphs, k in ks."""
        t = self.torch
        T = len(ks)
        n = self.cgraph_info(cg).num_players
        phi = phi.contiguous()
        kk = (C.c_int64 * T)(*[int(x) for x in ks])
        fp, fm = (C.c_float * T)(), (C.c_float * T)()
        masks = t.empty((2 * T, max((n + 63) // 64, 1)), dtype=t.int64, device=self.device) if want_masks else None
        self._sync_inputs()
        self._check(self.lib.ds_fidelity(self.h, cg, _ptr(phi), kk, T, score, fp, fm, _ptr(masks)))
        out = (list(fp), list(fm))
        return out + (masks,) if want_masks else out

    def copy_probe(self, nbytes):
        """Plain device copy of nbytes (calibration of profiler byte counters)."""
        t = self.torch
        src = t.zeros(nbytes // 8, dtype=t.int64, device=self.device)
        dst = t.empty_like(src)
        self._sync_inputs()
        self._check(self.lib.ds_copy_probe(self.h, _ptr(dst), _ptr(src), int(nbytes)))

    def solve(self, n, Z, w, y, options=None, allow_not_converged=False):
        t = self.torch
        opts = options or Options()
        Z, w, y = Z.contiguous(), w.contiguous(), y.contiguous()
        phi = t.empty(n, dtype=t.float32, device=self.device)
        rep = Report()
        self._sync_inputs()
        rc = self._check(self.lib.ds_solve(self.h, int(n), Z.shape[0], _ptr(Z), _ptr(w), _ptr(y),
                                           C.byref(opts), _ptr(phi), C.byref(rep)),
                         allow=(DS_ENOTCONV,) if allow_not_converged else ())
        return phi, rep, rc

    # -- operators on rows of features ---------------------------------------------
    # Queued on the context's stream, which is ordered behind torch's current stream and in front of what that stream
    # does next; nothing waits on the host. Under graph capture the context has to be one made for the captured stream. Gradients are calls of their own
    # (`*_backward`; dropout is its own): autograd does not know them, and an error says so where it is asked to go through one.
    def _queue(self, fn, *args):
        t = self.torch
        if self._current_stream(self._index) == self._raw_stream:
            self._check(fn(self.h, *args))
            return
        current = t.cuda.current_stream(self._index)
        if t.cuda.is_current_stream_capturing():
            raise DistShapError(DS_EINVAL, "the stream being captured is not the context's")
        own = self._stream if self._stream is not None else t.cuda.default_stream(self._index)
        own.wait_stream(current)
        try:
            self._check(fn(self.h, *args))
        finally:
            current.wait_stream(own)

    def _refuse(self, message):
        raise DistShapError(DS_EINVAL, message)

    def _outputs(self, call, outputs, a, b=None, c=None):
        """The outputs; where autograd follows an input, they take part in its graph, so that its backward pass fails and leaves no gradient out."""
        if (a.requires_grad or b is not None and b.requires_grad or c is not None and c.requires_grad) and self.torch.is_grad_enabled():
            return _no_gradient().apply(call, outputs, *[i for i in (a, b, c) if i is not None])
        return outputs

    def _rows(self, a, name, shape=None, dtype=None):
        """(tensor, its rows' distance): rows may lie apart, columns have to be neighbours (copied if they are not)."""
        if a.dim() != 2 or (shape is not None and tuple(a.shape) != shape):
            self._refuse(f"{name} has shape {tuple(a.shape)}, {'two dimensions are' if shape is None else f'{shape} is'} needed")
        if a.dtype not in self._elements or (dtype is not None and a.dtype != dtype):
            self._refuse(f"{name} is {a.dtype}, {'float32, bfloat16 or float16' if dtype is None else dtype} is needed")
        if a.get_device() != self._index:
            self._refuse(f"{name} is not on {self.device}")
        step, inner = a.stride()
        if inner != 1 and a.shape[1] > 1:
            a = a.contiguous()
            step = a.shape[1]
        return a, step

    def _values(self, a, name, shape, dtype):
        """A contiguous tensor of the given shape and type, or None; its address."""
        if a is None:
            return None, None
        if tuple(a.shape) != shape or a.dtype != dtype:
            self._refuse(f"{name} is {a.dtype} of shape {tuple(a.shape)}, {dtype} of shape {shape} is needed")
        if a.get_device() != self._index:
            self._refuse(f"{name} is not on {self.device}")
        a = a.contiguous()
        return a, a.data_ptr()

    def _workspace(self, fn, *args):
        need = C.c_int64()
        rc = fn(*args, C.byref(need))
        if rc != DS_OK:
            raise DistShapError(rc, "sizes out of range")
        if need.value == 0:
            return None, None, 0
        ws = self.torch.empty(need.value, dtype=self.torch.uint8, device=self.device)
        return ws, ws.data_ptr(), need.value

    def layer_norm(self, x, weight=None, bias=None, eps=1e-5, want_stats=False):
        """y = (x - mean) rstd weight + bias over the columns of each row; with `want_stats` (y, mean, rstd), the
        last two for layer_norm_backward. x: [rows, cols] in fp32, bf16 or fp16, cols <= 4096; the others fp32."""
        t = self.torch
        x, xs = self._rows(x, "x")
        rows, cols = x.shape
        weight, wp = self._values(weight, "weight", (cols,), t.float32)
        bias, bp = self._values(bias, "bias", (cols,), t.float32)
        y = x.new_empty((rows, cols))
        mean = rstd = mp = rp = None
        if want_stats:
            mean, rstd = t.empty((2, rows), dtype=t.float32, device=x.device)
            mp, rp = mean.data_ptr(), rstd.data_ptr()
        self._queue(self.lib.ds_layer_norm, self._elements[x.dtype], rows, cols, x.data_ptr(), xs, wp, bp, eps, y.data_ptr(),
                    cols, mp, rp)
        y = self._outputs("layer_norm", y, x, weight, bias)
        return (y, mean, rstd) if want_stats else y

    def layer_norm_backward(self, dy, x, mean, rstd, weight=None):
        """(dx, dweight, dbias) of layer_norm; mean and rstd are what it gave for x."""
        t = self.torch
        x, xs = self._rows(x, "x")
        rows, cols = x.shape
        dy, dys = self._rows(dy, "dy", (rows, cols), x.dtype)
        if mean is None or rstd is None:
            self._refuse("mean and rstd of the forward pass are needed")
        mean, mp = self._values(mean, "mean", (rows,), t.float32)
        rstd, rp = self._values(rstd, "rstd", (rows,), t.float32)
        weight, wp = self._values(weight, "weight", (cols,), t.float32)
        dx = x.new_empty((rows, cols))
        dweight, dbias = t.empty((2, cols), dtype=t.float32, device=x.device)
        ws, wsp, wsn = self._workspace(self.lib.ds_layer_norm_backward_workspace, rows, cols)
        self._queue(self.lib.ds_layer_norm_backward, self._elements[x.dtype], rows, cols, dy.data_ptr(), dys, x.data_ptr(), xs, mp,
                    rp, wp, dx.data_ptr(), cols, dweight.data_ptr(), dbias.data_ptr(), wsp, wsn)
        return self._outputs("layer_norm_backward", (dx, dweight, dbias), dy, x, weight)

    def dropout(self, x, p, seed, tag=0, residual=None):
        """residual + dropout(x): the mask is a function of (row, column, seed, tag) and never stored, so the gradient is
        `dropout(dy, p, seed, tag)`."""
        t = self.torch
        x, xs = self._rows(x, "x")
        rows, cols = x.shape
        rp, rs = None, 0
        if residual is not None:
            residual, rs = self._rows(residual, "residual", (rows, cols), x.dtype)
            rp = residual.data_ptr()
        y = x.new_empty((rows, cols))
        self._queue(self.lib.ds_dropout, self._elements[x.dtype], rows, cols, x.data_ptr(), xs, rp, rs, p, int(seed),
                    int(tag) & 0xFFFFFFFF, y.data_ptr(), cols)
        return self._outputs("dropout", y, x, residual)

    def group_rows(self, ids, groups):
        """(offsets int64[groups + 1], order int32[rows]): the rows by group, ascending within each, those whose id
        (int32[rows]) is outside of [0, groups) last."""
        t = self.torch
        if ids is None or ids.dim() != 1:
            self._refuse("ids: one for every row")
        rows = ids.shape[0]
        ids, ip = self._values(ids, "ids", (rows,), t.int32)
        groups = int(groups)
        ws, wsp, wsn = self._workspace(self.lib.ds_group_rows_workspace, rows, groups)
        offsets = t.empty(groups + 1, dtype=t.int64, device=ids.device)
        order = ids.new_empty(rows)
        self._queue(self.lib.ds_group_rows, ip, rows, groups, offsets.data_ptr(), order.data_ptr(), wsp, wsn)
        return offsets, order

    def _grouped(self, x, w, offsets, order):
        t = self.torch
        x, xs = self._rows(x, "x")
        if w is None or w.dim() != 3 or w.shape[1] != x.shape[1]:
            self._refuse(f"w is [groups, {x.shape[1]}, outer] for rows of {x.shape[1]} columns")
        w, wp = self._values(w, "w", tuple(w.shape), x.dtype)
        if offsets is None:
            self._refuse("offsets are needed")
        offsets, op = self._values(offsets, "offsets", (w.shape[0] + 1,), t.int64)
        order, rp = self._values(order, "order", (x.shape[0],), t.int32)
        return x, xs, w, wp, (offsets, order), op, rp

    def grouped_mm(self, x, w, offsets, order=None, bias=None, relu=False):
        """y[r] = x[r] @ w[g] + bias[g] (then ReLU) for the rows of every group g (see group_rows; order None: rows sorted by
        group), zeros for rows of no group. x: [rows, inner], w: [groups, inner, outer] of x's type, bias fp32."""
        t = self.torch
        x, xs, w, wp, keep, op, rp = self._grouped(x, w, offsets, order)
        (rows, inner), (groups, _, outer) = x.shape, w.shape
        bias, bp = self._values(bias, "bias", (groups, outer), t.float32)
        y = x.new_empty((rows, outer))
        self._queue(self.lib.ds_grouped_mm, self._elements[x.dtype], rows, inner, outer, groups, x.data_ptr(), xs, wp, op, rp, bp,
                    int(bool(relu)), y.data_ptr(), outer)
        return self._outputs("grouped_mm", y, x, w, bias)

    def grouped_mm_backward(self, dy, x, w, offsets, order=None, gate=None):
        """(dx, dw, dbias fp32) of grouped_mm without its ReLU; dx is 0 where `gate` (rows like x) is not above 0. x may be rows that
        pack_rows holds in 8 bits; a gate is then one too."""
        t = self.torch
        if isinstance(x, Packed):
            return self._grouped_backward_packed(dy, x, w, offsets, order, gate)
        if isinstance(gate, Packed):
            self._refuse("a gate that is held in 8 bits is one of rows that are")
        x, xs, w, wp, keep, op, rp = self._grouped(x, w, offsets, order)
        (rows, inner), (groups, _, outer) = x.shape, w.shape
        dy, dys = self._rows(dy, "dy", (rows, outer), x.dtype)
        gp, gs = None, 0
        if gate is not None:
            gate, gs = self._rows(gate, "gate", (rows, inner), x.dtype)
            gp = gate.data_ptr()
        dx = x.new_empty((rows, inner))
        dw = x.new_empty((groups, inner, outer))
        db = t.empty((groups, outer), dtype=t.float32, device=x.device)
        element = self._elements[x.dtype]
        ws, wsp, wsn = self._workspace(self.lib.ds_grouped_mm_backward_workspace, element, rows, inner, outer, groups)
        self._queue(self.lib.ds_grouped_mm_backward, element, rows, inner, outer, groups, dy.data_ptr(), dys, x.data_ptr(), xs, wp, op,
                    rp, gp, gs, dx.data_ptr(), inner, dw.data_ptr(), db.data_ptr(), wsp, wsn)
        return self._outputs("grouped_mm_backward", (dx, dw, db), dy, x, w)

    def _packed(self, a, name, shape=None):
        """The codes and scales of rows held in 8 bits, and for both the distance of rows."""
        t = self.torch
        if not isinstance(a, Packed):
            self._refuse(f"{name} is not held in 8 bits (pack_rows)")
        codes, scales = a
        if codes.dtype != t.float8_e4m3fn or scales.dtype != t.uint8:
            self._refuse(f"{name} is {codes.dtype} with scales of {scales.dtype}, float8_e4m3fn and uint8 are needed")
        if codes.dim() != 2 or (shape is not None and tuple(codes.shape) != shape):
            self._refuse(f"{name} has shape {tuple(codes.shape)}, {'two dimensions are' if shape is None else f'{shape} is'} needed")
        if tuple(scales.shape) != (codes.shape[0], (codes.shape[1] + 31) // 32):
            self._refuse(f"{name}: scales of shape {tuple(scales.shape)} for codes of shape {tuple(codes.shape)}")
        if codes.get_device() != self._index or scales.get_device() != self._index:
            self._refuse(f"{name} is not on {self.device}")
        if codes.stride(1) != 1 and codes.shape[1] > 1:
            codes = codes.contiguous()
        if scales.stride(1) != 1 and scales.shape[1] > 1:
            scales = scales.contiguous()
        return codes, codes.stride(0), scales, scales.stride(0)

    def _grouped_backward_packed(self, dy, x, w, offsets, order, gate):
        t = self.torch
        codes, cs, scales, ss = self._packed(x, "x")
        rows, inner = codes.shape
        if w is None or w.dim() != 3 or w.shape[1] != inner:
            self._refuse(f"w is [groups, {inner}, outer] for rows of {inner} columns")
        groups, _, outer = w.shape
        if w.dtype not in self._elements:
            self._refuse(f"w is {w.dtype}, float32, bfloat16 or float16 is needed")
        w, wp = self._values(w, "w", tuple(w.shape), w.dtype)
        if offsets is None:
            self._refuse("offsets are needed")
        offsets, op = self._values(offsets, "offsets", (groups + 1,), t.int64)
        order, rp = self._values(order, "order", (rows,), t.int32)
        dy, dys = self._rows(dy, "dy", (rows, outer), w.dtype)
        gp, gs = None, 0
        if gate is not None:
            gate, gs, _, _ = self._packed(gate, "gate", (rows, inner))
            gp = gate.data_ptr()
        dx = w.new_empty((rows, inner))
        dw = w.new_empty((groups, inner, outer))
        db = t.empty((groups, outer), dtype=t.float32, device=w.device)
        element = self._elements[w.dtype]
        ws, wsp, wsn = self._workspace(self.lib.ds_grouped_mm_backward_packed_workspace, element, rows, inner, outer, groups)
        self._queue(self.lib.ds_grouped_mm_backward_packed, element, rows, inner, outer, groups, dy.data_ptr(), dys, codes.data_ptr(), cs, scales.data_ptr(), ss,
                    wp, op, rp, gp, gs, dx.data_ptr(), inner, dw.data_ptr(), db.data_ptr(), wsp, wsn)
        return self._outputs("grouped_mm_backward", (dx, dw, db), dy, codes, w)

    def pack_rows(self, x):
        """The rows of x in 8 bits, as `Packed`: what a training step keeps of an activation, half of 16 bits. Zeros stay zeros, and nothing else becomes
        one; an infinity becomes NaN."""
        t = self.torch
        given, (x, xs) = x, self._rows(x, "x")
        rows, cols = x.shape
        codes = t.empty((rows, cols), dtype=t.float8_e4m3fn, device=x.device)
        scales = t.empty((rows, (cols + 31) // 32), dtype=t.uint8, device=x.device)
        self._queue(self.lib.ds_pack_rows, self._elements[x.dtype], rows, cols, x.data_ptr(), xs, codes.data_ptr(), cols, scales.data_ptr(), scales.shape[1])
        return Packed(*self._outputs("pack_rows", (codes, scales), given))

    def unpack_rows(self, packed, dtype=None):
        """The rows that `packed` stands for, in `dtype` (float32 if none is given)."""
        t = self.torch
        codes, cs, scales, ss = self._packed(packed, "packed")
        dtype = t.float32 if dtype is None else dtype
        if dtype not in self._elements:
            self._refuse(f"rows are float32, bfloat16 or float16, not {dtype}")
        y = t.empty(tuple(codes.shape), dtype=dtype, device=codes.device)
        self._queue(self.lib.ds_unpack_rows, self._elements[dtype], *y.shape, codes.data_ptr(), cs, scales.data_ptr(), ss, y.data_ptr(), y.shape[1])
        return self._outputs("unpack_rows", y, codes)

    def _ids(self, ids):
        if ids is None or ids.dim() != 1:
            self._refuse("ids: one for every row")
        return self._values(ids, "ids", (ids.shape[0],), self.torch.int32)

    def embed(self, table, ids, scale=1.0, dtype=None):
        """y[r] = scale * table[ids[r]], zeros where the id (int32[rows]) is outside of the table. table: [vocab, cols]; y is of `dtype`: the
        table's (if none is given), or any where the table is fp32."""
        given, (table, ts) = table, self._rows(table, "table")
        vocab, cols = table.shape
        ids, ip = self._ids(ids)
        dtype = table.dtype if dtype is None else dtype
        if dtype not in self._elements:
            self._refuse(f"rows are float32, bfloat16 or float16, not {dtype}")
        y = table.new_empty((ids.shape[0], cols), dtype=dtype)
        self._queue(self.lib.ds_embed, self._elements[dtype], self._elements[table.dtype], ids.shape[0], cols, vocab, table.data_ptr(), ts, ip, scale,
                    y.data_ptr(), cols)
        return self._outputs("embed", y, given)

    def embed_backward(self, dy, ids, vocab, scale=1.0, dtype=None):
        """dtable [vocab, cols] of embed, in `dtype`: dy's (if none is given), or fp32. Its rows are summed by sorted ids, in fp32."""
        t = self.torch
        ids, ip = self._ids(ids)
        given = dy
        if dy.dim() != 2:
            self._refuse(f"dy has shape {tuple(dy.shape)}, two dimensions are needed")
        dy, dys = self._rows(dy, "dy", (ids.shape[0], dy.shape[1]))
        (rows, cols), vocab = dy.shape, int(vocab)
        dtype = dy.dtype if dtype is None else dtype
        if dtype not in self._elements:
            self._refuse(f"a table is float32, bfloat16 or float16, not {dtype}")
        ws, wsp, wsn = self._workspace(self.lib.ds_embed_backward_workspace, rows, cols, vocab)
        dtable = dy.new_empty((vocab, cols), dtype=dtype)
        self._queue(self.lib.ds_embed_backward, self._elements[dy.dtype], self._elements[dtype], rows, cols, vocab, dy.data_ptr(), dys, ip, scale,
                    dtable.data_ptr(), cols, wsp, wsn)
        return self._outputs("embed_backward", dtable, given)

    def route(self, scores, k=1, renorm=False):
        """(ids int32[k, rows], weights fp32[k, rows], counts int64[experts + 1], loss, lse fp32[rows]): every row's experts of the k highest scores, ties to
        the lowest (ids[j] is what group_rows takes; -1: none, a score of -inf closes an expert to a row); their softmax, or with `renorm` each's share of the
        chosen; how often each was chosen, then the rows that have one; a balance loss, 1 where all are used alike; and what route_backward needs. scores:
        [rows, experts], at most 1,024 experts and k of 8."""
        t = self.torch
        given, (x, xs) = scores, self._rows(scores, "scores")
        (rows, experts), k = x.shape, int(k)
        ws, wsp, wsn = self._workspace(self.lib.ds_route_workspace, rows, experts)
        if not 1 <= k <= min(8, experts):
            self._refuse(f"{k} experts to a row out of range [1, {min(8, experts)}]")
        ids = x.new_empty((k, rows), dtype=t.int32)
        weights = x.new_empty((k, rows), dtype=t.float32)
        counts = x.new_empty(experts + 1, dtype=t.int64)
        lse = x.new_empty(rows, dtype=t.float32)
        loss = x.new_empty((), dtype=t.float32)
        self._queue(self.lib.ds_route, self._elements[x.dtype], rows, experts, k, int(bool(renorm)), x.data_ptr(), xs, ids.data_ptr(), weights.data_ptr(),
                    counts.data_ptr(), loss.data_ptr(), lse.data_ptr(), wsp, wsn)
        return self._outputs("route", (ids, weights, counts, loss, lse), given)

    def route_backward(self, scores, lse, ids, counts, dweights=None, dloss=None, renorm=False):
        """The scores' gradient, of their type, from the weights' (fp32[k, rows]) and the loss' (a fp32 tensor of one element), one of them at
        least. lse, ids and counts are what route gave for the scores, `renorm` what it was called with."""
        t = self.torch
        given, (x, xs) = scores, self._rows(scores, "scores")
        rows, experts = x.shape
        if ids is None or ids.dim() != 2 or lse is None or counts is None:
            self._refuse("lse, ids and counts of the forward pass are needed")
        k = ids.shape[0]
        lse, lp = self._values(lse, "lse", (rows,), t.float32)
        ids, ip = self._values(ids, "ids", (k, rows), t.int32)
        counts, cp = self._values(counts, "counts", (experts + 1,), t.int64)
        dweights, wp = self._values(dweights, "dweights", (k, rows), t.float32)
        if dloss is not None and dloss.numel() != 1:
            self._refuse(f"dloss has shape {tuple(dloss.shape)}, one element is needed")
        dloss, dp = self._values(dloss, "dloss", () if dloss is None else tuple(dloss.shape), t.float32)
        dx = x.new_empty((rows, experts))
        self._queue(self.lib.ds_route_backward, self._elements[x.dtype], rows, experts, k, int(bool(renorm)), x.data_ptr(), xs, lp, ip, cp, wp, dp,
                    dx.data_ptr(), experts)
        return self._outputs("route_backward", dx, given, dweights, dloss)
