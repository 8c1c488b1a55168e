"""ctypes binding of include/sjd.h.  Same names as the C ABI; torch is used for device memory and streams only."""
import ctypes as C
import functools
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libsjd.so")
_lib = None

F32, BF16, FP8 = 0, 1, 2
KERNELS_REFERENCE, NO_GRAPH, KERNELS_ROWGROUPS, ATTENTION_CHUNKED, KERNELS_TILES, NO_L2_WARM, TILES_256_ROWS, NO_ROW_SPLIT, NO_MIXED_WIDTH, NO_K_ROTATION = 1, 2, 4, 8, 16, 32, 64, 128, 256, 512
KEEP_LOGITS, NO_HEAD_FUSION = 1024, 2048
OK, EINVAL, ENOMEM, ESTATE, EDEVICE, ECAPACITY = 0, -1, -2, -3, -4, -5


class SjdError(RuntimeError):
    def __init__(self, code, message):
        super().__init__(f"sjd error {code}: {message}")
        self.code = code


class ModelDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "d_model", "n_heads", "n_kv_heads", "d_ff", "vocab",
                                         "sample_lo", "sample_hi")] + \
               [("rms_eps", C.c_float), ("rope_theta", C.c_float)] + \
               [(n, C.c_int32) for n in ("dtype", "max_seqs", "max_ctx", "window", "kv_page_tokens", "kernel_flags")]


class KvCacheDesc(C.Structure):
    _fields_ = [("pages", C.c_void_p), ("page_table", C.c_void_p)] + \
               [(n, C.c_int32) for n in ("n_pages", "page_tokens", "n_kv_heads", "head_dim", "dtype", "n_seqs", "pages_per_seq")]


_VPP = C.POINTER(C.c_void_p)


class Weights(C.Structure):
    _fields_ = [("tok_emb", C.c_void_p), ("final_norm", C.c_void_p), ("lm_head", C.c_void_p)] + \
               [(n, _VPP) for n in ("attn_norm", "wq", "wk", "wv", "wo", "mlp_norm", "w_gate", "w_up", "w_down")]


class Sampling(C.Structure):
    _fields_ = [("cfg_scale", C.c_float), ("temperature", C.c_float), ("top_k", C.c_int32), ("reuse_tau", C.c_float),
                ("seed", C.c_uint64), ("init_mode", C.c_int32), ("row_width", C.c_int32)]


class StepResult(C.Structure):
    _fields_ = [("n_accepted", C.c_int32), ("n_finalized", C.c_int32), ("reject_index", C.c_int32), ("done", C.c_int32)]


class TraceEntry(C.Structure):
    _fields_ = [("name", C.c_char_p), ("launches", C.c_int64), ("total_ms", C.c_double)]


def library_path():
    return _LIB_PATH


def lib():
    """Loads libsjd.so (built by paper_2512_07503_amd/build.py).  There is no fallback: a missing library is an error."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise SjdError(EDEVICE, f"{_LIB_PATH} is not built; run `python -m paper_2512_07503_amd.build`")
        L = C.CDLL(_LIB_PATH)
        IP, IPP = C.POINTER(C.c_int32), C.POINTER(C.POINTER(C.c_int32))
        L.sjd_create.argtypes = [C.POINTER(ModelDesc), C.POINTER(Weights), C.POINTER(Sampling), C.c_void_p, _VPP]
        L.sjd_prefill.argtypes = [C.c_void_p, C.c_int32, IPP, IP, IPP, IP, IP]
        L.sjd_step.argtypes = [C.c_void_p, C.POINTER(StepResult)]
        L.sjd_destroy.argtypes = [C.c_void_p]
        L.sjd_destroy.restype = None
        L.sjd_get_tokens.argtypes = [C.c_void_p, C.c_int32, IP, C.c_int32, IP]
        L.sjd_get_window.argtypes = [C.c_void_p, C.c_int32, IP, IP, IP]
        L.sjd_last_error.argtypes = [C.c_void_p]
        L.sjd_last_error.restype = C.c_char_p
        L.sjd_debug_copy_logits.argtypes = [C.c_void_p, C.POINTER(C.c_float)]
        L.sjd_debug_step_from_logits.argtypes = [C.c_void_p, C.POINTER(C.c_float), C.POINTER(StepResult)]
        L.sjd_snapshot_size.argtypes = [C.c_void_p, C.POINTER(C.c_uint64)]
        L.sjd_snapshot_save.argtypes = [C.c_void_p, C.c_void_p, C.c_uint64, C.POINTER(C.c_uint64)]
        L.sjd_snapshot_restore.argtypes = [C.c_void_p, C.c_void_p, C.c_uint64]
        L.sjd_trace_enable.argtypes = [C.c_void_p, C.c_int32]
        L.sjd_trace_reset.argtypes = [C.c_void_p]
        L.sjd_trace_read.argtypes = [C.c_void_p, C.POINTER(TraceEntry), C.c_int32, IP]
        L.sjd_op_gemm.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32,
                                  C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.POINTER(C.c_float)]
        L.sjd_op_gemm_static.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32,
                                         C.c_int32, C.c_int32, C.c_int32]
        L.sjd_op_window_attention.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p,
                                              C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32,
                                              C.c_int32, C.c_int32, C.POINTER(C.c_float)]
        L.sjd_op_sampling_rows.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32,
                                           C.c_int32, C.c_float, C.c_float, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p,
                                           C.c_void_p, C.c_int32, C.POINTER(C.c_float)]
        L.sjd_set_token_ranges.argtypes = [C.c_void_p, C.c_int32, IP, IP, C.c_int32]
        L.sjd_op_philox.argtypes = [C.c_void_p, C.c_uint64, C.c_uint32, C.c_uint32, C.c_void_p, C.c_int32]
        P, I, I64, CP, U64P = C.c_void_p, C.c_int32, C.c_int64, C.POINTER(KvCacheDesc), C.POINTER(C.c_uint64)
        L.sjd_cache_page_bytes.argtypes = [CP, U64P]
        L.sjd_op_cache_write.argtypes = [P, CP, I, P, I64, P, I64, P, P, I]
        L.sjd_op_cache_read.argtypes = [P, CP, I, P, P, P, P, I]
        L.sjd_op_cache_compact.argtypes = [P, CP, P, P, P, I]
        L.sjd_rope_table.argtypes = [I, C.c_double, I, C.c_double, C.c_double, C.c_double, C.c_double, P]
        L.sjd_op_rotary.argtypes = [P, I, I, P, I, C.c_float, P, I, I, P, I64, P, I64, I, P, I64, P, I64, I]
        L.sjd_tree_masks.argtypes = [P, I, I, P, P]
        L.sjd_op_tree_attention_workspace.argtypes = [CP, I, I, I, U64P]
        L.sjd_op_tree_attention.argtypes = [P, CP, I, P, I64, P, I64, P, P, P, I, I, I, C.c_float, I, I, P, C.c_uint64]
        L.sjd_op_tree_verify_workspace.argtypes = [I, I, I, U64P]
        L.sjd_op_tree_verify.argtypes = [P, P, P, P, P, I64, P, I64, P, P, P, P, P, I, I, I, I, I, P, C.c_uint64]
        L.sjd_op_norm_rotary.argtypes = [P, I, I, C.c_float, I, I, P, I, C.c_float, P, I, I, P, I64, P, P, P, I64, I, P, I64, P, P, P, I64, I]
        L.sjd_op_prompt_attention_workspace.argtypes = [I, I, I, I, I, I, I, I, U64P]
        L.sjd_op_prompt_attention.argtypes = [P, I, P, I64, P, I64, P, I64, P, I64, P, P, I, I, I, I, I, I, C.c_float, I, I, P, C.c_uint64]
        L.sjd_op_token_logprobs_workspace.argtypes = [I, I, I, U64P]
        L.sjd_op_token_logprobs.argtypes = [P, I, P, I64, P, P, P, P, P, P, I, I, I, P, C.c_uint64]
        _lib = L
    return _lib


def _check(rc, ctx=None):
    if rc != OK:
        msg = lib().sjd_last_error(ctx)
        raise SjdError(rc, msg.decode() if msg else "")


def _stream_ptr():
    import torch
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


_PER_LAYER = ("attn_norm", "wq", "wk", "wv", "wo", "mlp_norm", "w_gate", "w_up", "w_down")


class Decoder:
    """sjd_create / sjd_prefill / sjd_step / sjd_destroy on device tensors.

    weights: dict of torch CUDA tensors (float32 for dtype "f32", bfloat16 for "bf16"): tok_emb, final_norm,
    lm_head and per-layer lists attn_norm, wq, wk, wv, wo, mlp_norm, w_gate, w_up, w_down."""

    def __init__(self, arch, weights, dtype, window, max_ctx, max_seqs=1, cfg_scale=3.0, temperature=1.0, top_k=2000,
                 reuse_tau=0.5, seed=0, kv_page_tokens=0, kernel_flags=0, init_mode=0, row_width=0):
        import torch
        want = torch.float32 if dtype == "f32" else torch.bfloat16
        tensors = [weights[n] for n in ("tok_emb", "final_norm", "lm_head")] + [t for n in _PER_LAYER for t in weights[n]]
        for t in tensors:
            if not (t.is_cuda and t.dtype == want and t.is_contiguous()):
                raise SjdError(EINVAL, "weights must be contiguous CUDA tensors of the model dtype")
        self.md = ModelDesc(arch["n_layers"], arch["d_model"], arch["n_heads"], arch["n_kv_heads"], arch["d_ff"],
                            arch["vocab"], arch["sample_lo"], arch["sample_hi"], arch.get("rms_eps", 1e-5),
                            arch.get("rope_theta", 10000.0), F32 if dtype == "f32" else BF16, max_seqs, max_ctx, window,
                            kv_page_tokens, kernel_flags)
        w = Weights()
        for n in ("tok_emb", "final_norm", "lm_head"):
            setattr(w, n, weights[n].data_ptr())
        keep = []
        for n in _PER_LAYER:
            arr = (C.c_void_p * arch["n_layers"])(*[t.data_ptr() for t in weights[n]])
            keep.append(arr)
            setattr(w, n, C.cast(arr, _VPP))
        sp = Sampling(cfg_scale, temperature, top_k, reuse_tau, seed, init_mode, row_width)
        self.ctx = C.c_void_p()
        self.L, self.Vs, self.n_seqs = window, arch["sample_hi"] - arch["sample_lo"], 0
        self.sparse_rows = True   # rows of the sampling distribution are stored as kept (id, weight) pairs
        # The context runs on the caller's current stream, unless that is the default stream: the library can only
        # capture its step into a HIP graph on an ordinary stream, so it then gets one of its own (default priority).
        # Either way the weights must be complete before sjd_create reads them.
        cur = torch.cuda.current_stream()
        cur.synchronize()
        self._stream = cur if cur.cuda_stream != 0 else torch.cuda.Stream()
        _check(lib().sjd_create(C.byref(self.md), C.byref(w), C.byref(sp), C.c_void_p(self._stream.cuda_stream), C.byref(self.ctx)))

    def close(self):
        if getattr(self, "ctx", None):
            lib().sjd_destroy(self.ctx)
            self.ctx = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def prefill(self, cond, uncond, n_image_tokens):
        S = len(cond)
        IP = C.POINTER(C.c_int32)
        conds = [np.ascontiguousarray(c, dtype=np.int32) for c in cond]
        unconds = [np.ascontiguousarray(c, dtype=np.int32) for c in uncond]
        cp = (IP * S)(*[a.ctypes.data_as(IP) for a in conds])
        up = (IP * S)(*[a.ctypes.data_as(IP) for a in unconds])
        cl = (C.c_int32 * S)(*[len(a) for a in conds])
        ul = (C.c_int32 * S)(*[len(a) for a in unconds])
        ni = (C.c_int32 * S)(*[int(n) for n in n_image_tokens])
        rc = lib().sjd_prefill(self.ctx, S, cp, cl, up, ul, ni)
        if rc == OK:
            self.n_seqs = S
        return rc

    @staticmethod
    def _results(arr):
        return [dict(n_accepted=r.n_accepted, n_finalized=r.n_finalized, reject_index=r.reject_index, done=r.done)
                for r in arr]

    def step(self):
        res = (StepResult * max(self.n_seqs, 1))()
        _check(lib().sjd_step(self.ctx, res), self.ctx)
        return self._results(res)

    def step_raw(self, res):
        """sjd_step into a preallocated (StepResult * n) array; returns the status code."""
        return lib().sjd_step(self.ctx, res)

    def step_from_logits(self, logits):
        lg = np.ascontiguousarray(logits, dtype=np.float32)
        assert lg.size == self.n_seqs * 2 * self.L * self.Vs
        res = (StepResult * self.n_seqs)()
        _check(lib().sjd_debug_step_from_logits(self.ctx, lg.ctypes.data_as(C.POINTER(C.c_float)), res), self.ctx)
        return self._results(res)

    def logits(self):
        out = np.zeros((self.n_seqs, 2, self.L, self.Vs), dtype=np.float32)
        _check(lib().sjd_debug_copy_logits(self.ctx, out.ctypes.data_as(C.POINTER(C.c_float))), self.ctx)
        return out

    def set_token_ranges(self, seq, first_id, end_id):
        """sjd_set_token_ranges: position i of sequence seq may only take ids in [first_id[i], end_id[i])."""
        IP = C.POINTER(C.c_int32)
        lo = np.ascontiguousarray(first_id, dtype=np.int32)
        hi = np.ascontiguousarray(end_id, dtype=np.int32)
        assert lo.shape == hi.shape and lo.ndim == 1
        return lib().sjd_set_token_ranges(self.ctx, seq, lo.ctypes.data_as(IP), hi.ctypes.data_as(IP), len(lo))

    def tokens(self, seq=0):
        n = C.c_int32(0)
        _check(lib().sjd_get_tokens(self.ctx, seq, None, 0, C.byref(n)), self.ctx)
        out = np.zeros(max(n.value, 1), dtype=np.int32)
        _check(lib().sjd_get_tokens(self.ctx, seq, out.ctypes.data_as(C.POINTER(C.c_int32)), n.value, C.byref(n)), self.ctx)
        return out[:n.value]

    def window(self, seq=0):
        IP = C.POINTER(C.c_int32)
        toks, refs, n = np.zeros(self.L, dtype=np.int32), np.zeros(self.L, dtype=np.int32), C.c_int32(0)
        _check(lib().sjd_get_window(self.ctx, seq, toks.ctypes.data_as(IP), refs.ctypes.data_as(IP), C.byref(n)), self.ctx)
        return toks, refs, n.value

    def snapshot(self):
        """The decoding state of the current batch as a uint8 array (sjd_snapshot_size + sjd_snapshot_save)."""
        n = C.c_uint64(0)
        _check(lib().sjd_snapshot_size(self.ctx, C.byref(n)), self.ctx)
        buf = np.zeros(n.value, dtype=np.uint8)
        w = C.c_uint64(0)
        _check(lib().sjd_snapshot_save(self.ctx, buf.ctypes.data_as(C.c_void_p), n.value, C.byref(w)), self.ctx)
        return buf[:w.value]

    def restore(self, buf):
        buf = np.ascontiguousarray(buf, dtype=np.uint8)
        _check(lib().sjd_snapshot_restore(self.ctx, buf.ctypes.data_as(C.c_void_p), buf.size), self.ctx)
        # the batch size travels with the snapshot
        self.n_seqs = int(np.frombuffer(buf[:32].tobytes(), dtype=np.int32)[5])

    def decode(self, max_steps=1 << 30):
        hist = []
        for _ in range(max_steps):
            r = self.step()
            hist.append(r)
            if all(x["done"] for x in r):
                break
        return hist

    def trace(self, on):
        _check(lib().sjd_trace_enable(self.ctx, 1 if on else 0), self.ctx)

    def trace_reset(self):
        _check(lib().sjd_trace_reset(self.ctx), self.ctx)

    def trace_read(self):
        n = C.c_int32(0)
        arr = (TraceEntry * 64)()
        _check(lib().sjd_trace_read(self.ctx, arr, 64, C.byref(n)), self.ctx)
        return {arr[i].name.decode(): (int(arr[i].launches), float(arr[i].total_ms)) for i in range(n.value)}


def _dtype_code(t):
    import torch
    return F32 if t.dtype == torch.float32 else BF16


def op_gemm(A, W, flags=0, splits=0, repeat=1):
    """C = A @ W.T through sjd_op_gemm; A [M,K], W [N,K] CUDA tensors (float32 or bfloat16). Returns (C, avg_ms)."""
    import torch
    M, K = A.shape
    N = W.shape[0]
    Cout = torch.empty((M, N), dtype=torch.float32, device=A.device)
    ms = C.c_float(0)
    _check(lib().sjd_op_gemm(_stream_ptr(), _dtype_code(A), flags, A.data_ptr(), W.data_ptr(), Cout.data_ptr(), M, N, K,
                             splits, repeat, C.byref(ms)))
    return Cout, ms.value


def op_gemm_static(A, W, flags=0, splits=0):
    """C = A @ W.T through sjd_op_gemm_static (no allocation inside the library); returns the status code and C."""
    import torch
    M, K = A.shape
    N = W.shape[0]
    Cout = torch.empty((M, N), dtype=torch.float32, device=A.device)
    rc = lib().sjd_op_gemm_static(_stream_ptr(), _dtype_code(A), flags, A.data_ptr(), W.data_ptr(), Cout.data_ptr(), M, N, K,
                                  splits)
    return rc, Cout


def op_window_attention(q, k, v, ctx, page_tokens=64, flags=0, repeat=1):
    """q [n,H,hd], k/v [ctx+n,Hkv,hd] -> out [n,H,hd] float32 through sjd_op_window_attention."""
    import torch
    n, H, hd = q.shape
    Hkv = k.shape[1]
    out = torch.empty((n, H, hd), dtype=torch.float32, device=q.device)
    ms = C.c_float(0)
    _check(lib().sjd_op_window_attention(_stream_ptr(), _dtype_code(q), flags, q.data_ptr(), k.data_ptr(), v.data_ptr(),
                                         out.data_ptr(), n, ctx, H, Hkv, hd, page_tokens, repeat, C.byref(ms)))
    return out, ms.value


def op_sampling_rows(logits_c, logits_u, cfg_scale, temperature, top_k, repeat=1, allow_lo=None, allow_hi=None, kept=False):
    """float32 CUDA [rows,V] x2 -> (e float32 [rows,V], Z int64-viewed uint64 [rows], avg_ms); with kept=True also the
    stored form of the rows: (kept_ids int32 [rows,V], kept_cnt int32 [rows]).  allow_lo / allow_hi: int32 CUDA [rows]."""
    import torch
    rows, V = logits_c.shape
    e = torch.empty((rows, V), dtype=torch.float32, device=logits_c.device)
    Z = torch.zeros(rows, dtype=torch.int64, device=logits_c.device)
    ids = torch.zeros((rows, V), dtype=torch.int32, device=logits_c.device) if kept else None
    cnt = torch.zeros(rows, dtype=torch.int32, device=logits_c.device) if kept else None
    ms = C.c_float(0)
    _check(lib().sjd_op_sampling_rows(_stream_ptr(), logits_c.data_ptr(), logits_u.data_ptr(), e.data_ptr(), Z.data_ptr(),
                                      rows, V, cfg_scale, temperature, top_k,
                                      allow_lo.data_ptr() if allow_lo is not None else None,
                                      allow_hi.data_ptr() if allow_hi is not None else None,
                                      ids.data_ptr() if kept else None, cnt.data_ptr() if kept else None, repeat, C.byref(ms)))
    if kept:
        return e, Z, ms.value, ids, cnt
    return e, Z, ms.value


def op_philox(seed, row, seq, n):
    import torch
    out = torch.zeros(4 * n, dtype=torch.int32, device="cuda")
    _check(lib().sjd_op_philox(_stream_ptr(), seed, row, seq, out.data_ptr(), n))
    return out.cpu().numpy().view(np.uint32).reshape(n, 4)


# ---- operators of a step of tree speculation.  They enqueue their work on the current stream of their tensors' device and return.  A
# decoding step makes a handful of such calls a layer, of a few microseconds of work each: what is looked up or allocated here counts
# (torch.cuda.current_stream() alone takes 2.9 us, the raw handle 0.1).

_CACHE_DTYPES = {"f32": F32, "bf16": BF16, "fp8": FP8}
_SCALINGS = {"none": 0, "linear": 1, "base": 2, "parts": 3}


def _refuse(message):
    raise SjdError(EINVAL, message)


def _device_of(first, *others):
    """Index of the device of `first`; the other tensors (None: not given) have to be there too."""
    d = first.get_device()
    if d < 0:
        _refuse("tensors must be on a GPU")
    for t in others:
        if t is not None and t.get_device() != d:
            _refuse("tensors are on different devices")
    return d


def _enqueue(device, function, *args):
    """function(current stream of the device, *args) with the device current; its errors are raised."""
    import torch
    if torch._C._cuda_getDevice() == device:
        rc = function(torch._C._cuda_getCurrentRawStream(device), *args)
    else:
        with torch.cuda.device(device):
            rc = function(torch._C._cuda_getCurrentRawStream(device), *args)
    if rc:
        _check(rc)


def _vector(t, n, dtype, name):
    if t.dtype is not dtype or t.dim() != 1 or (n is not None and t.shape[0] != n) or not t.is_contiguous():
        _refuse(f"{name} must be a contiguous vector of {dtype}" + ("" if n is None else f" with {n} elements"))
    return t.data_ptr()


def _row_code(t, name):
    import torch
    if t.dtype is torch.bfloat16:
        return BF16
    return F32 if t.dtype is torch.float32 else _refuse(f"{name} must be float32 or bfloat16")


def _row_stride(x, heads, hd, name):
    """Row stride of x [rows, heads, hd], whose heads have to be contiguous within a row."""
    shape, stride = x.shape, x.stride()
    if len(shape) != 3 or shape[1] != heads or shape[2] != hd:
        _refuse(f"{name} must be [rows, {heads}, {hd}]")
    if (stride[2] != 1 and hd != 1) or (stride[1] != hd and heads != 1):
        _refuse(f"{name}: the heads of a row must be contiguous")
    return stride[0] if shape[0] > 1 else heads * hd


class KvCache:
    """A paged key/value cache ("f32", "bf16" or "fp8") and its page table, int32 CUDA [n_seqs, pages_per_seq]; entries outside
    [0, n_pages) are unused.  Owns its pages (zeroed); the table is the caller's, and its contents may change between calls.  Either tensor stays
    the one that it is: calls take the addresses that the cache was made with."""

    def __init__(self, dtype, n_pages, page_tokens, n_kv_heads, head_dim, page_table):
        import torch
        if dtype not in _CACHE_DTYPES:
            _refuse("dtype must be f32, bf16 or fp8")
        if not (page_table.is_cuda and page_table.dtype is torch.int32 and page_table.dim() == 2 and page_table.is_contiguous()):
            _refuse("page_table must be a contiguous int32 CUDA matrix")
        if n_pages < 1:
            _refuse("n_pages must be positive")
        self.dtype, self.n_kv_heads, self.head_dim, self._page_table = dtype, n_kv_heads, head_dim, page_table
        self.n_seqs, self.device = page_table.shape[0], page_table.device
        self.desc = KvCacheDesc(None, page_table.data_ptr(), n_pages, page_tokens, n_kv_heads, head_dim, _CACHE_DTYPES[dtype], *page_table.shape)
        self.ref = C.byref(self.desc)
        n = C.c_uint64(0)
        _check(lib().sjd_cache_page_bytes(self.ref, C.byref(n)))
        self._pages = torch.zeros(n_pages * n.value, dtype=torch.uint8, device=self.device)
        self.desc.pages = self._pages.data_ptr()
        self.sizes = _CACHE_DTYPES[dtype], page_tokens, n_kv_heads, head_dim, self.n_seqs

    @property
    def pages(self):
        return self._pages

    @property
    def page_table(self):
        return self._page_table


def op_cache_write(cache, k, v, row_start, first_pos):
    """Writes k and v [rows, n_kv_heads, head_dim] (float32 or bfloat16; rows may be strided) to positions first_pos[b] + i of sequence b =
    rows row_start[b] + i.  row_start int32 [n_seqs + 1], first_pos int32 [n_seqs]."""
    import torch
    device = _device_of(cache._page_table, k, v, row_start, first_pos)
    code, n = _row_code(k, "k"), k.shape[0]
    ks, vs = _row_stride(k, cache.n_kv_heads, cache.head_dim, "k"), _row_stride(v, cache.n_kv_heads, cache.head_dim, "v")
    if v.dtype is not k.dtype or v.shape[0] != n:
        _refuse("k and v must have one dtype and number of rows")
    _enqueue(device, lib().sjd_op_cache_write, cache.ref, code, k.data_ptr(), ks, v.data_ptr(), vs, _vector(row_start, cache.n_seqs + 1, torch.int32, "row_start"),
             _vector(first_pos, cache.n_seqs, torch.int32, "first_pos"), n)


def op_cache_read(cache, row_start, first_pos, n_rows, dtype=None, out=None):
    """-> (k, v) [n_rows, n_kv_heads, head_dim] of `dtype` (bfloat16 unless given): what is stored at positions first_pos[b] + i of sequence
    b, in rows row_start[b] + i, and zeros for what is outside the cache.  out: a pair of such tensors to write to.  Rows of no sequence are not
    written."""
    import torch
    device = _device_of(cache._page_table, row_start, first_pos, *(out or ()))
    shape = (n_rows, cache.n_kv_heads, cache.head_dim)
    if out is None:
        if n_rows < 0:
            _refuse("n_rows must not be negative")
        k = torch.empty(shape, dtype=dtype or torch.bfloat16, device=cache.device)
        out = k, torch.empty_like(k)
    elif any(t.shape != shape or t.dtype is not (dtype or out[0].dtype) or not t.is_contiguous() for t in out):
        _refuse("out must be two contiguous tensors of the result's shape and dtype")
    _enqueue(device, lib().sjd_op_cache_read, cache.ref, _row_code(out[0], "dtype"), out[0].data_ptr(), out[1].data_ptr(),
             _vector(row_start, cache.n_seqs + 1, torch.int32, "row_start"), _vector(first_pos, cache.n_seqs, torch.int32, "first_pos"), n_rows)
    return out


def op_cache_compact(cache, first_pos, path, path_len):
    """Moves the entries at positions first_pos[b] + path[b, j] to first_pos[b] + j, j < path_len[b].  path int32 [n_seqs, max_path]."""
    import torch
    device = _device_of(cache._page_table, first_pos, path, path_len)
    if path.dtype is not torch.int32 or path.dim() != 2 or path.shape[0] != cache.n_seqs or not path.is_contiguous():
        _refuse("path must be a contiguous int32 [n_seqs, max_path]")
    _enqueue(device, lib().sjd_op_cache_compact, cache.ref, _vector(first_pos, cache.n_seqs, torch.int32, "first_pos"), path.data_ptr(),
             _vector(path_len, cache.n_seqs, torch.int32, "path_len"), path.shape[1])


def rope_table(rotary_dim, theta=10000.0, scaling="none", factor=1.0, trained_ctx=0.0, low_turns=1.0, high_turns=32.0, device="cuda"):
    """Frequencies for op_rotary (sjd_rope_table) on the device, as the bits of an int64 tensor [rotary_dim / 2].  scaling: "none",
    "linear", "base" or "parts"."""
    import torch
    if scaling not in _SCALINGS:
        _refuse("scaling must be none, linear, base or parts")
    table = np.zeros(max(rotary_dim // 2, 1), dtype=np.uint64)
    _check(lib().sjd_rope_table(rotary_dim, theta, _SCALINGS[scaling], factor, trained_ctx, low_turns, high_turns, table.ctypes.data))
    return torch.from_numpy(table.view(np.int64)).to(device)


def op_rotary(q, k, positions, table, interleaved=False, magnitude=1.0, out=None):
    """Turns q [rows, heads, hd] and k [rows, kv_heads, hd] (or None) by their rows' positions (int32) -> (q', k').  out: tensors to write to, which may
    be q and k themselves."""
    import torch
    device = _device_of(q, k, positions, table, *(out or ()))
    code, shape = _row_code(q, "q"), q.shape
    if len(shape) != 3:
        _refuse("q must be [rows, heads, head_dim]")
    rows, heads, hd = shape
    if out is None:
        # (new tensors are contiguous, whatever the strides of q and k)
        q_out, k_out = q.new_empty(shape), None if k is None else k.new_empty(k.shape)
    else:
        q_out, k_out = out[0], out[1] if len(out) > 1 else None
        if (k_out is None) != (k is None) or q_out.dtype is not q.dtype or q_out.shape[0] != rows or (k is not None and (k_out.dtype is not q.dtype or k_out.shape != k.shape)):
            _refuse("out must have the shapes and dtype of q and k")
    if k is None:
        keys = (None, 0, None, 0, 0)
    else:
        if k.dtype is not q.dtype or k.shape[0] != rows or k.dim() != 3:
            _refuse("k must have q's dtype and number of rows")
        n = k.shape[1]
        keys = (k.data_ptr(), _row_stride(k, n, hd, "k"), k_out.data_ptr(), n * hd if out is None else _row_stride(k_out, n, hd, "out"), n)
    _enqueue(device, lib().sjd_op_rotary, code, 1 if interleaved else 0, _vector(table, None, torch.int64, "table"), 2 * table.shape[0], magnitude,
             _vector(positions, rows, torch.int32, "positions"), rows, hd, q.data_ptr(), _row_stride(q, heads, hd, "q"), q_out.data_ptr(),
             heads * hd if out is None else _row_stride(q_out, heads, hd, "out"), heads, *keys)
    return q_out, k_out


def tree_masks(parents, mask_words=None):
    """Host: parents (ints; negative: a root) -> (mask uint32 [n, mask_words], depth int32 [n]): bit j of row i is node i or an ancestor of it."""
    parents = np.ascontiguousarray(parents, dtype=np.int32)
    n = len(parents)
    words = -(-n // 32) if mask_words is None else mask_words
    mask, depth = np.zeros((n, words), dtype=np.uint32), np.zeros(n, dtype=np.int32)
    _check(lib().sjd_tree_masks(parents.ctypes.data, n, words, mask.ctypes.data, depth.ctypes.data))
    return mask, depth


def _workspace(given, need, like):
    """-> (pointer, bytes, what to keep until the call is enqueued)"""
    import torch
    if given is None:
        if not need:
            return None, 0, None
        given = torch.empty(need, dtype=torch.uint8, device=like.device)
        return given.data_ptr(), need, given
    if not given.is_contiguous():
        _refuse("the workspace must be contiguous")
    return given.data_ptr(), given.numel() * given.element_size(), given


@functools.lru_cache(maxsize=256)
def _attention_bytes(sizes, heads, max_rows, max_ctx):
    """Of op_tree_attention's workspace, for KvCache.sizes."""
    dtype, page_tokens, n_kv_heads, head_dim, n_seqs = sizes
    n = C.c_uint64(0)
    _check(lib().sjd_op_tree_attention_workspace(C.byref(KvCacheDesc(None, None, 0, page_tokens, n_kv_heads, head_dim, dtype, n_seqs, 0)), heads, max_rows, max_ctx, C.byref(n)))
    return n.value


def op_tree_attention(q, cache, row_start, ctx_len, mask=None, max_rows=None, max_ctx=None, scale=0.0, out=None, workspace=None):
    """Attention of q [rows, heads, head_dim] over the cache: row row_start[b] + i (position ctx_len[b] + i) sees positions [0, ctx_len[b])
    and the nodes whose bits are set in its row of mask, int32 or uint32 [rows, words]; without a mask nodes 0 .. i.  max_rows: no tree has more
    (default: all rows); max_ctx: what ctx_len is expected to reach (default: what the page table holds).  The work is divided by these two: for several
    sequences the defaults launch for more than is there, so say them.  -> out like q; rows of no sequence are not written."""
    import torch
    device = _device_of(cache._page_table, q, row_start, ctx_len, mask, out, workspace)
    code, shape, hd = _row_code(q, "q"), q.shape, cache.head_dim
    if len(shape) != 3:
        _refuse("q must be [rows, heads, head_dim]")
    rows, heads = shape[0], shape[1]
    stride = _row_stride(q, heads, hd, "q")
    mask_ptr, words = None, 0
    if mask is not None:
        if mask.dtype not in (torch.int32, torch.uint32) or mask.dim() != 2 or mask.shape[0] != rows or not mask.is_contiguous():
            _refuse("mask must be a contiguous int32 or uint32 [rows, words]")
        if rows and not mask.shape[1]:
            _refuse("a mask needs a word a row (its pointer would be null, as a window's is)")
        mask_ptr, words = mask.data_ptr(), mask.shape[1]
    if out is None:
        out, out_stride = q.new_empty(shape), heads * hd
    else:
        if out.dtype is not q.dtype or out.shape != shape:
            _refuse("out must be like q")
        out_stride = _row_stride(out, heads, hd, "out")
    if max_rows is None:
        max_rows = max(rows, 1)
    if max_ctx is None:
        max_ctx = cache.desc.pages_per_seq * cache.desc.page_tokens
    at, size, keep = _workspace(workspace, _attention_bytes(cache.sizes, heads, max_rows, max_ctx), q)
    _enqueue(device, lib().sjd_op_tree_attention, cache.ref, code, q.data_ptr(), stride, out.data_ptr(), out_stride,
             _vector(row_start, cache.n_seqs + 1, torch.int32, "row_start"), _vector(ctx_len, cache.n_seqs, torch.int32, "ctx_len"), mask_ptr, words, rows, heads, scale,
             max_rows, max_ctx, at, size)
    return out


@functools.lru_cache(maxsize=256)
def _verify_bytes(rows, seqs, vocab):
    n = C.c_uint64(0)
    _check(lib().sjd_op_tree_verify_workspace(rows, seqs, vocab, C.byref(n)))
    return n.value


def op_tree_verify(tokens, parents, row_start, p, q, accept_words, draw_words, max_rows=None, max_path=None, workspace=None):
    """Verifies trees of drafted tokens: tokens, parents int32 [rows]; p (and q, or None) float32 [rows, vocab], rows may be strided; accept_words
    [rows], the bits of 32-bit words (int32 or uint32); draw_words [n_seqs], of 64-bit words.  -> (path int32 [n_seqs, max_path], path_len int32
    [n_seqs], next_token int32 [n_seqs]).  max_rows: no tree has more (default: all rows, at most 1024, with a workgroup launched for each of every sequence);
    max_path: nodes that a path has room for (default: max_rows)."""
    import torch
    device = _device_of(p, tokens, parents, row_start, q, accept_words, draw_words, workspace)
    rows, seqs, shape = tokens.shape[0], row_start.shape[0] - 1, p.shape
    for t in (p,) if q is None else (p, q):
        if t.dtype is not torch.float32 or t.dim() != 2 or t.shape != shape or shape[0] != rows or (shape[1] != 1 and t.stride(1) != 1):
            _refuse("p and q must be float32 [rows, vocab] with contiguous rows")
    if max_rows is None:
        max_rows = min(max(rows, 1), 1024)
    if max_path is None:
        max_path = max_rows
    if max_path < 1:
        _refuse("max_path must be positive")
    path = torch.empty((seqs, max_path), dtype=torch.int32, device=p.device)
    path_len = path.new_empty(seqs)
    token = path.new_empty(seqs)
    at, size, keep = _workspace(workspace, _verify_bytes(rows, seqs, shape[1]), p)
    _enqueue(device, lib().sjd_op_tree_verify, _vector(tokens, rows, torch.int32, "tokens"), _vector(parents, rows, torch.int32, "parents"),
             _vector(row_start, seqs + 1, torch.int32, "row_start"), p.data_ptr(), p.stride(0) if rows > 1 else shape[1], None if q is None else q.data_ptr(),
             0 if q is None else q.stride(0) if rows > 1 else shape[1],
             _vector(accept_words, rows, torch.uint32 if accept_words.dtype is torch.uint32 else torch.int32, "accept_words"),
             _vector(draw_words, seqs, torch.uint64 if draw_words.dtype is torch.uint64 else torch.int64, "draw_words"), path.data_ptr(), path_len.data_ptr(),
             token.data_ptr(), rows, seqs, shape[1], max_rows, max_path, at, size)
    return path, path_len, token


# ---- operators of scoring and prefilling prompts

_NORMS = {"rms": 0, "layer": 1}


def _head_vector(t, like, heads, hd, name):
    """-> (pointer, 0: one for all heads or 1: one for each) of a gain or bias."""
    shape = t.shape
    if t.dtype is not like.dtype or shape[-1:] != (hd,) or len(shape) > 2 or (len(shape) == 2 and shape[0] != heads) or not t.is_contiguous():
        _refuse(f"{name} must be a contiguous [{hd}] or [{heads}, {hd}] of the rows' dtype")
    return t.data_ptr(), len(shape) - 1


def op_norm_rotary(q, k, positions, table, q_gain, k_gain=None, q_bias=None, k_bias=None, norm="rms", eps=1e-5, interleaved=False, magnitude=1.0, out=None):
    """op_rotary of heads that are normalised first: norm "rms" or "layer" (the mean is taken off), gains and biases (a bias may be None) of q's dtype,
    [hd] for all heads or [heads, hd], all of them alike.  q [rows, heads, hd], k [rows, kv_heads, hd] or None -> (q', k').  out: tensors to write to, which may
    be q and k themselves."""
    import torch
    if norm not in _NORMS:
        _refuse("norm must be rms or layer")
    device = _device_of(q, k, positions, table, q_gain, k_gain, q_bias, k_bias, *(out or ()))
    code, shape = _row_code(q, "q"), q.shape
    if len(shape) != 3:
        _refuse("q must be [rows, heads, head_dim]")
    rows, heads, hd = shape
    if out is None:
        q_out, k_out = q.new_empty(shape), None if k is None else k.new_empty(k.shape)
    else:
        q_out, k_out = out[0], out[1] if len(out) > 1 else None
        if (k_out is None) != (k is None) or q_out.dtype is not q.dtype or q_out.shape[0] != rows or (k is not None and (k_out.dtype is not q.dtype or k_out.shape != k.shape)):
            _refuse("out must have the shapes and dtype of q and k")
    gain, per_head = _head_vector(q_gain, q, heads, hd, "q_gain")
    bias, kinds = None, {per_head}
    if q_bias is not None:
        bias, kind = _head_vector(q_bias, q, heads, hd, "q_bias")
        kinds.add(kind)
    if k is None:
        if k_gain is not None or k_bias is not None:
            _refuse("a gain or a bias without k")
        keys = (None, 0, None, None, None, 0, 0)
    else:
        if k.dtype is not q.dtype or k.shape[0] != rows or k.dim() != 3:
            _refuse("k must have q's dtype and number of rows")
        if k_gain is None:
            _refuse("k_gain is missing")
        n, k_bias_ptr = k.shape[1], None
        k_gain_ptr, kind = _head_vector(k_gain, q, n, hd, "k_gain")
        kinds.add(kind)
        if k_bias is not None:
            k_bias_ptr, kind = _head_vector(k_bias, q, n, hd, "k_bias")
            kinds.add(kind)
        keys = (k.data_ptr(), _row_stride(k, n, hd, "k"), k_gain_ptr, k_bias_ptr, k_out.data_ptr(), n * hd if out is None else _row_stride(k_out, n, hd, "out"), n)
    if len(kinds) > 1:
        _refuse("gains and biases must all be [hd] or all [heads, hd]")
    _enqueue(device, lib().sjd_op_norm_rotary, code, _NORMS[norm], eps, per_head, 1 if interleaved else 0, _vector(table, None, torch.int64, "table"), 2 * table.shape[0],
             magnitude, _vector(positions, rows, torch.int32, "positions"), rows, hd, q.data_ptr(), _row_stride(q, heads, hd, "q"), gain, bias, q_out.data_ptr(),
             heads * hd if out is None else _row_stride(q_out, heads, hd, "out"), heads, *keys)
    return q_out, k_out


@functools.lru_cache(maxsize=256)
def _prompt_bytes(*sizes):
    n = C.c_uint64(0)
    _check(lib().sjd_op_prompt_attention_workspace(*sizes, C.byref(n)))
    return n.value


def op_prompt_attention(q, k, v, row_start, kv_start=None, max_rows=None, max_kv=None, scale=0.0, out=None, workspace=None):
    """Causal attention of packed prompts: q [rows, heads, head_dim], k and v [kv_rows, kv_heads, head_dim] (rows may be strided).  Sequence b's queries are rows
    row_start[b] .. row_start[b + 1] - 1, its keys rows kv_start[b] .. (the same rows without a kv_start), the last of which are its queries' own: query i of n sees the
    first i + 1 + t - n of t keys.  row_start, kv_start int32 [n_seqs + 1].  max_kv: what a sequence's keys are expected to reach (default: all rows; say it where
    sequences are much shorter than all of them together); it only chooses how the work is divided.  max_rows, the same of its queries, changes nothing.  -> out like q; rows of no sequence are not written."""
    import torch
    device = _device_of(q, k, v, row_start, kv_start, out, workspace)
    code, shape = _row_code(q, "q"), q.shape
    if len(shape) != 3 or k.dim() != 3 or v.shape != k.shape:
        _refuse("q must be [rows, heads, head_dim], k and v [rows, kv_heads, head_dim]")
    if k.dtype is not q.dtype or v.dtype is not q.dtype:
        _refuse("q, k and v must have one dtype")
    (rows, heads, hd), (kv_rows, kv_heads, _), seqs = shape, k.shape, row_start.shape[0] - 1
    if kv_start is None and kv_rows != rows:
        _refuse("without kv_start k and v have q's rows")
    strides = _row_stride(q, heads, hd, "q"), _row_stride(k, kv_heads, hd, "k"), _row_stride(v, kv_heads, hd, "v")
    if out is None:
        out, out_stride = q.new_empty(shape), heads * hd
    else:
        if out.dtype is not q.dtype or out.shape != shape:
            _refuse("out must be like q")
        out_stride = _row_stride(out, heads, hd, "out")
    if max_rows is None:
        max_rows = rows
    if max_kv is None:
        max_kv = kv_rows
    at, size, keep = _workspace(workspace, _prompt_bytes(code, rows, seqs, heads, kv_heads, hd, 0, max_kv), q)      # (max_rows does not change it)
    _enqueue(device, lib().sjd_op_prompt_attention, code, q.data_ptr(), strides[0], k.data_ptr(), strides[1], v.data_ptr(), strides[2], out.data_ptr(), out_stride,
             _vector(row_start, seqs + 1, torch.int32, "row_start"), None if kv_start is None else _vector(kv_start, seqs + 1, torch.int32, "kv_start"), rows, kv_rows, seqs,
             heads, kv_heads, hd, scale, max_rows, max_kv, at, size)
    return out


@functools.lru_cache(maxsize=256)
def _logprob_bytes(rows, vocab, n_top):
    n = C.c_uint64(0)
    _check(lib().sjd_op_token_logprobs_workspace(rows, vocab, n_top, C.byref(n)))
    return n.value


def op_token_logprobs(logits, tokens, n_top=0, workspace=None):
    """Log probabilities of tokens int32 [rows] under logits [rows, vocab] (float32 or bfloat16, rows may be strided; -inf masks an id) -> (logprob float32 [rows], rank
    int32 [rows], entropy float32 [rows], top_ids int32 [rows, n_top], top_logprobs float32 [rows, n_top]).  rank: number of likelier ids, of equal ones those that are lower.
    n_top <= 64.  A token outside the vocabulary has -inf and rank -1; alternatives that there are not, -1 and -inf; rows with a NaN or +inf, NaN."""
    import torch
    device = _device_of(logits, tokens, workspace)
    code, shape = _row_code(logits, "logits"), logits.shape
    if len(shape) != 2 or (shape[1] != 1 and logits.stride(1) != 1):
        _refuse("logits must be [rows, vocab] with contiguous rows")
    rows, vocab = shape
    tokens_ptr, need = _vector(tokens, rows, torch.int32, "tokens"), _logprob_bytes(rows, vocab, n_top)
    logprob, rank = torch.empty(rows, dtype=torch.float32, device=logits.device), tokens.new_empty(rows)
    entropy, ids, top = logprob.new_empty(rows), rank.new_empty((rows, n_top)), logprob.new_empty((rows, n_top))
    at, size, keep = _workspace(workspace, need, logits)
    _enqueue(device, lib().sjd_op_token_logprobs, code, logits.data_ptr(), logits.stride(0) if rows > 1 else vocab, tokens_ptr, logprob.data_ptr(), rank.data_ptr(),
             entropy.data_ptr(), ids.data_ptr(), top.data_ptr(), rows, vocab, n_top, at, size)
    return logprob, rank, entropy, ids, top
