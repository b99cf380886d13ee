"""Thin Python binding of libspatvit (argument marshalling only).

Every step of the path runs inside the CUDA library; PyTorch is used for device memory and
streams.  The library must have been built (`python -m paper_2601_12150_b200.build` or
`__graft_entry__.build()`); importing the compute entry points without it raises.
There is no CPU fallback.
"""
import ctypes as C
import os
import struct

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libspatvit.so")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_CUDA, ERR_TIMEOUT, ERR_ALIGNMENT, ERR_STATIC_LIMIT = range(8)
FILTER_STATIC_BYTES = 2 << 20
TOKENS_ROW_MAJOR, TOKENS_BLOCK_MAJOR = 0, 1
MLP_GELU, MLP_SWIGLU = 0, 1
ATTN_DENSE, ATTN_SPARSE = 0, 1
KV_INT8, KV_E4M3 = 0, 1
BF16, FP16, FP32 = 0, 1, 2
EPI_BIAS, EPI_BIAS_GELU, EPI_BIAS_SILU, EPI_BIAS_MUL, EPI_BIAS_SCALE_RESID, EPI_BIAS_ADDROW = range(6)

EXPORTS = ["spv_create", "spv_destroy", "spv_status_string", "spv_check", "spv_last_wait_site", "spv_launch_count",
           "spv_attn_workspace_size", "spatial_block_attention",
           "spv_filter_keep_count", "spv_filter_workspace_size", "cls_score_topk_filter",
           "cls_score_topk_filter_static",
           "spv_vit_workspace_size", "vit_forward", "spv_gemm_bf16", "spv_layernorm",
           "kv_cache_append", "spv_kv_attention_workspace_size", "kv_cache_attention",
           "spv_kv_evict_workspace_size", "kv_cache_evict", "kv_cache_read",
           "spv_profile_enable", "spv_profile_read", "spv_microbench", "spv_selftest_wait"]


class SpvError(RuntimeError):
    def __init__(self, status, what):
        self.status = status
        super().__init__(f"{what}: status {status} ({status_string(status)})")


class AttnDesc(C.Structure):
    _fields_ = [("batch", C.c_int32), ("grid_h", C.c_int32), ("grid_w", C.c_int32),
                ("block", C.c_int32), ("radius", C.c_int32), ("n_global", C.c_int32),
                ("heads", C.c_int32), ("head_dim", C.c_int32), ("softmax_scale", C.c_float),
                ("n_patch", C.c_int32), ("patch_pos", C.c_void_p), ("token_order", C.c_int32),
                ("stride_b", C.c_int64), ("stride_tok", C.c_int64), ("stride_head", C.c_int64)]


class FilterDesc(C.Structure):
    _fields_ = [("batch", C.c_int32), ("heads", C.c_int32), ("n_patch", C.c_int32),
                ("n_global", C.c_int32), ("dim", C.c_int32), ("keep_ratio", C.c_double),
                ("in_stride_b", C.c_int64), ("out_stride_b", C.c_int64)]


class VitConfig(C.Structure):
    _fields_ = [("layers", C.c_int32), ("dim", C.c_int32), ("heads", C.c_int32),
                ("mlp_hidden", C.c_int32), ("mlp_kind", C.c_int32), ("patch", C.c_int32),
                ("n_global", C.c_int32), ("has_layerscale", C.c_int32), ("ln_eps", C.c_float),
                ("attn_mode", C.c_int32), ("block", C.c_int32), ("radius", C.c_int32),
                ("filter_layer", C.c_int32), ("keep_ratio", C.c_double),
                ("n_filters", C.c_int32), ("filter_layers", C.c_int32 * 4), ("keep_ratios", C.c_double * 4),
                ("unfused_filter", C.c_int32)]


LAYER_FIELDS = ["ln1_g", "ln1_b", "w_qkv", "b_qkv", "w_o", "b_o", "ls1", "ln2_g", "ln2_b",
                "w_fc1", "b_fc1", "w_fc3", "b_fc3", "w_fc2", "b_fc2", "ls2"]


class LayerWeights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in LAYER_FIELDS]


class VitWeights(C.Structure):
    _fields_ = [("w_pe", C.c_void_p), ("b_pe", C.c_void_p), ("cls", C.c_void_p),
                ("pos", C.c_void_p), ("lnf_g", C.c_void_p), ("lnf_b", C.c_void_p),
                ("layer", C.c_void_p)]


KERNEL_CLASSES = ["gemm", "attn_patch", "attn_global", "attn_plan", "layernorm", "filter_select",
                  "filter_gather", "misc", "kv_cache", "kv_attn"]


class KernelStat(C.Structure):
    _fields_ = [("launches", C.c_int64), ("ms", C.c_double), ("work", C.c_double)]


class GemmDesc(C.Structure):
    _fields_ = [("m", C.c_int32), ("n", C.c_int32), ("k", C.c_int32),
                ("lda", C.c_int64), ("ldw", C.c_int64), ("ldo", C.c_int64),
                ("epilogue", C.c_int32), ("bias", C.c_void_p), ("aux", C.c_void_p),
                ("ldaux", C.c_int64), ("scale", C.c_void_p), ("addrow", C.c_void_p),
                ("ldadd", C.c_int64), ("rows_per_image", C.c_int32)]


class KvCacheStruct(C.Structure):
    _fields_ = [("pages", C.c_int32), ("kv_heads", C.c_int32), ("head_dim", C.c_int32), ("block", C.c_int32),
                ("format", C.c_int32), ("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p),
                ("v_scale", C.c_void_p)]


class KvSeqs(C.Structure):
    _fields_ = [("batch", C.c_int32), ("columns", C.c_int32), ("table_stride", C.c_int64),
                ("page_table", C.c_void_p), ("lengths", C.c_void_p), ("max_length", C.c_int32)]


class KvAppendDesc(C.Structure):
    _fields_ = [("tokens", C.c_int32), ("dtype", C.c_int32), ("stride_b", C.c_int64), ("stride_tok", C.c_int64),
                ("stride_head", C.c_int64), ("counts", C.c_void_p)]


class KvAttnDesc(C.Structure):
    _fields_ = [("tokens", C.c_int32), ("heads", C.c_int32), ("dtype", C.c_int32), ("causal", C.c_int32),
                ("softmax_scale", C.c_float),
                ("q_stride_b", C.c_int64), ("q_stride_tok", C.c_int64), ("q_stride_head", C.c_int64),
                ("o_stride_b", C.c_int64), ("o_stride_tok", C.c_int64), ("o_stride_head", C.c_int64),
                ("w_stride_b", C.c_int64), ("w_stride_head", C.c_int64), ("counts", C.c_void_p)]


class KvEvictDesc(C.Structure):
    _fields_ = [("budget", C.c_int32), ("keep_first", C.c_int32), ("keep_last", C.c_int32),
                ("w_stride_b", C.c_int64), ("w_stride_head", C.c_int64), ("dst_table", C.c_void_p),
                ("dst_stride", C.c_int64)]


class KvReadDesc(C.Structure):
    _fields_ = [("rows", C.c_int32), ("dtype", C.c_int32), ("stride_b", C.c_int64), ("stride_tok", C.c_int64),
                ("stride_head", C.c_int64), ("first", C.c_void_p)]


# the same five as native layouts for struct.pack_into
_KV_SEQS = struct.Struct("@iiqPPi4x")
_KV_APPEND = struct.Struct("@iiqqqP")
_KV_ATTN = struct.Struct("@iiiif4x8qP")
_KV_EVICT = struct.Struct("@iii4xqqPq")
_KV_READ = struct.Struct("@iiqqqP")
assert [s.size for s in (_KV_SEQS, _KV_APPEND, _KV_ATTN, _KV_EVICT, _KV_READ)] == \
    [C.sizeof(t) for t in (KvSeqs, KvAppendDesc, KvAttnDesc, KvEvictDesc, KvReadDesc)]


MICROBENCH_KINDS = {"ex2": 0, "softmax_body": 1, "mma_ss": 2, "mma_ts": 3, "l2_tma": 4}


class MicrobenchDesc(C.Structure):
    _fields_ = [("kind", C.c_int32), ("ctas_per_sm", C.c_int32), ("threads", C.c_int32), ("iters", C.c_int32),
                ("m", C.c_int32), ("n", C.c_int32), ("box_rows", C.c_int32), ("stages", C.c_int32),
                ("poly_per_8", C.c_int32), ("accumulators", C.c_int32),
                ("issue_mode", C.c_int32), ("issuers", C.c_int32)]


class MicrobenchResult(C.Structure):
    _fields_ = [("ms", C.c_double), ("cycles", C.c_double), ("units", C.c_double), ("sm_count", C.c_int32)]


_lib = None


def lib():
    """The loaded C-ABI library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build the CUDA library first "
                               "(python -m paper_2601_12150_b200.build); there is no fallback path")
        L = C.CDLL(LIB_PATH)
        L.spv_status_string.restype = C.c_char_p
        L.spv_status_string.argtypes = [C.c_int32]
        L.spv_launch_count.restype = C.c_int64
        L.spv_launch_count.argtypes = [C.c_void_p]
        L.spv_last_wait_site.restype = C.c_uint32
        L.spv_last_wait_site.argtypes = [C.c_void_p]
        L.spv_create.argtypes = [C.POINTER(C.c_void_p), C.c_int32]
        L.spv_destroy.argtypes = [C.c_void_p]
        L.spv_check.argtypes = [C.c_void_p, C.c_void_p]
        L.spv_filter_keep_count.argtypes = [C.c_int32, C.c_double, C.POINTER(C.c_int32)]
        L.spv_filter_workspace_size.argtypes = [C.POINTER(FilterDesc), C.POINTER(C.c_size_t)]
        L.cls_score_topk_filter.argtypes = [C.c_void_p, C.POINTER(FilterDesc)] + [C.c_void_p] * 8 + \
            [C.c_size_t, C.c_void_p]
        L.cls_score_topk_filter_static.argtypes = [C.POINTER(FilterDesc)] + [C.c_void_p] * 8
        L.spv_attn_workspace_size.argtypes = [C.POINTER(AttnDesc), C.POINTER(C.c_size_t)]
        L.spatial_block_attention.argtypes = [C.c_void_p, C.POINTER(AttnDesc)] + [C.c_void_p] * 6 + \
            [C.c_size_t, C.c_void_p]
        L.spv_vit_workspace_size.argtypes = [C.POINTER(VitConfig), C.c_int32, C.c_int32, C.c_int32,
                                             C.POINTER(C.c_size_t)]
        L.vit_forward.argtypes = [C.c_void_p, C.POINTER(VitConfig), C.POINTER(VitWeights), C.c_void_p,
                                  C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p,
                                  C.c_void_p, C.c_size_t, C.c_void_p]
        L.spv_gemm_bf16.argtypes = [C.c_void_p, C.POINTER(GemmDesc), C.c_void_p, C.c_void_p, C.c_void_p,
                                    C.c_void_p]
        L.spv_layernorm.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_int32, C.c_void_p, C.c_void_p,
                                    C.c_float, C.c_void_p, C.c_void_p, C.c_void_p]
        # the cache calls' descriptors are passed by address (struct.pack_into is faster than building a Structure)
        p = C.c_void_p
        L.kv_cache_append.argtypes = [p] * 7
        L.spv_kv_attention_workspace_size.argtypes = [p, p, p, C.c_int32, C.POINTER(C.c_size_t)]
        L.kv_cache_attention.argtypes = [p] * 10 + [C.c_size_t, p]
        L.spv_kv_evict_workspace_size.argtypes = [p, p, p, C.POINTER(C.c_size_t)]
        L.kv_cache_evict.argtypes = [p] * 9 + [C.c_size_t, p]
        L.kv_cache_read.argtypes = [p] * 7
        L.spv_profile_enable.argtypes = [C.c_void_p, C.c_int32]
        L.spv_profile_read.argtypes = [C.c_void_p, C.POINTER(KernelStat)]
        L.spv_selftest_wait.argtypes = [C.c_void_p, C.c_uint32, C.c_void_p]
        L.spv_microbench.argtypes = [C.c_void_p, C.POINTER(MicrobenchDesc), C.c_void_p, C.c_size_t, C.c_void_p,
                                     C.POINTER(MicrobenchResult)]
        _lib = L
    return _lib


def status_string(status):
    return lib().spv_status_string(int(status)).decode()


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream(stream=None):
    import torch
    s = torch.cuda.current_stream() if stream is None else stream
    return C.c_void_p(s.cuda_stream)


def _raw_stream(device):
    """The current stream of a device as an address, without making a torch.cuda.Stream of it where torch allows that."""
    import torch
    get = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return get(device) if get else torch.cuda.current_stream(device).cuda_stream


def _raise(status, what):
    if status != OK:
        raise SpvError(status, what)


def _need(ok, what):
    """Argument checks of what the library cannot see (types, shapes, devices of the tensors behind the pointers)."""
    if not ok:
        raise SpvError(ERR_INVALID_ARG, what)


def _apart(strides, shape):
    """Whether an output's strides are those of a view in which the elements do not overlap."""
    reach = 1
    for stride, n in zip(reversed(strides), reversed(shape)):      # the usual order: every dimension beyond those after it
        if n > 1 and stride < reach:
            break
        reach = max(reach, stride * n)
    else:
        return True
    reach = 0
    for stride, n in sorted(zip(strides, shape)):
        if n > 1:
            if stride <= reach:
                return False
            reach += stride * (n - 1)
    return True


def filter_keep_count(n_patch, keep_ratio):
    k = C.c_int32(0)
    _raise(lib().spv_filter_keep_count(int(n_patch), float(keep_ratio), C.byref(k)), "spv_filter_keep_count")
    return k.value


def cls_score_topk_filter_static(scores, tokens_in, tokens_out, kept_idx, n_global=1, keep_ratio=0.5,
                                 mean_scores=None, pos_in=None, pos_out=None, stream=None):
    """The token filter through the entry point that allocates nothing: no context, no workspace
    (its scratch is a 2 MiB array built into the library), and this wrapper creates no tensor
    either -- every output is the caller's.  For callers that run under a fixed device-memory
    plan or inside a loop where an allocation would stall the device.  Works on the current CUDA
    device; calls that may overlap on the GPU must be ordered by the caller (shared scratch).
    scores fp32 [B, h, n_patch]; tokens_in / tokens_out bf16 [B, G+n_patch, dim] / [B, G+k, dim] or
    both None; kept_idx int32 [B, k]."""
    import torch
    B, H, NP = scores.shape
    dim = 0 if tokens_in is None else tokens_in.shape[-1]
    d = FilterDesc(B, H, NP, n_global, dim, float(keep_ratio), 0, 0)
    # the library writes k rows / indices per image into the caller's buffers: a buffer of another size, type or
    # device would be written out of bounds, so check them here (the count fails below if the ratio is invalid)
    kc = C.c_int32(0)
    if lib().spv_filter_keep_count(NP, float(keep_ratio), C.byref(kc)) == OK:
        k = kc.value
        dev = scores.device
        assert scores.dtype == torch.float32 and scores.is_contiguous()
        assert kept_idx.dtype == torch.int32 and kept_idx.is_contiguous() and tuple(kept_idx.shape) == (B, k)
        assert kept_idx.device == dev
        if tokens_in is not None:
            assert tokens_out is not None and tokens_in.dtype == tokens_out.dtype == torch.bfloat16
            assert tokens_in.is_contiguous() and tokens_out.is_contiguous()
            assert tuple(tokens_in.shape) == (B, n_global + NP, dim) and tuple(tokens_out.shape) == (B, n_global + k, dim)
            assert tokens_in.device == dev and tokens_out.device == dev
        if mean_scores is not None:
            assert mean_scores.dtype == torch.float32 and mean_scores.is_contiguous() and tuple(mean_scores.shape) == (B, NP)
        if pos_in is not None:
            assert pos_out is not None and pos_in.dtype == pos_out.dtype == torch.int32
            assert tuple(pos_in.shape) == (B, NP) and tuple(pos_out.shape) == (B, k)
            assert pos_in.is_contiguous() and pos_out.is_contiguous()
    with torch.cuda.device(scores.device):
        st = lib().cls_score_topk_filter_static(C.byref(d), _ptr(scores), _ptr(tokens_in), _ptr(tokens_out),
                                                _ptr(kept_idx), _ptr(mean_scores), _ptr(pos_in), _ptr(pos_out),
                                                _stream(stream))
    _raise(st, "cls_score_topk_filter_static")
    return tokens_out, kept_idx


class KvCache:
    """An 8-bit key/value cache: a pool of pages of `block` tokens and one scale for each page and key head
    (spv_kv_cache in include/spatvit.h).  The tensors are the caller's and are kept alive:
    k, v int8 or float8_e4m3fn [pages, kv_heads, block, head_dim]; k_scale, v_scale fp32 [pages, kv_heads]."""

    def __init__(self, k, v, k_scale, v_scale):
        import torch
        fmt = {torch.int8: KV_INT8, torch.float8_e4m3fn: KV_E4M3}.get(k.dtype)
        _need(fmt is not None and k.dim() == 4 and k.is_contiguous(), "k: contiguous int8 or float8_e4m3fn, 4-D")
        _need(v.dtype == k.dtype and v.shape == k.shape and v.is_contiguous(), "v: as k")
        for s in (k_scale, v_scale):
            _need(s.dtype == torch.float32 and s.shape == k.shape[:2] and s.is_contiguous(),
                  "scales: contiguous fp32 [pages, kv_heads]")
        _need(k.is_cuda and all(t.device == k.device for t in (v, k_scale, v_scale)), "one CUDA device")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.device, self.device_index = k.device, k.get_device()
        self.pages, self.kv_heads, self.block, self.head_dim = k.shape
        self.struct = KvCacheStruct(self.pages, self.kv_heads, self.head_dim, self.block, fmt, k.data_ptr(),
                                    v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr())
        self.address = C.addressof(self.struct)

    @classmethod
    def empty(cls, pages, kv_heads, head_dim, block=64, format=KV_INT8, device="cuda"):
        """A pool of its own; nothing in it is defined until it is appended."""
        import torch
        dt = {KV_INT8: torch.int8, KV_E4M3: torch.float8_e4m3fn}[format]
        shape = (pages, kv_heads, block, head_dim)
        return cls(torch.empty(shape, dtype=dt, device=device), torch.empty(shape, dtype=dt, device=device),
                   torch.empty(shape[:2], dtype=torch.float32, device=device),
                   torch.empty(shape[:2], dtype=torch.float32, device=device))


class Context:
    """Owns an spv_ctx for one CUDA device and the workspaces it hands to the library."""

    def __init__(self, device=0):
        import torch
        self._torch = torch
        self.device = torch.device("cuda", device)
        h = C.c_void_p()
        with torch.cuda.device(self.device):
            _raise(lib().spv_create(C.byref(h), device), "spv_create")
        self.handle = h
        self._ws = None
        self._index = device
        self._kv_types = {torch.bfloat16: BF16, torch.float16: FP16, torch.float32: FP32}
        self._seqs, self._desc, self._size = C.create_string_buffer(_KV_SEQS.size), C.create_string_buffer(128), C.c_size_t(0)
        self._seqs_at, self._desc_at = C.addressof(self._seqs), C.addressof(self._desc)

    def close(self):
        if self.handle:
            lib().spv_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def workspace(self, nbytes):
        """A cached device workspace of at least `nbytes` (grown on demand, 256-byte aligned)."""
        torch = self._torch
        if self._ws is None or self._ws.numel() < nbytes:
            self._ws = None
            self._ws = torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=self.device)
        return self._ws

    def check(self, stream=None):
        st = lib().spv_check(self.handle, _stream(stream))
        if st == ERR_TIMEOUT:
            raise SpvError(st, "spv_check (wait site 0x%x)" % lib().spv_last_wait_site(self.handle))
        _raise(st, "spv_check")

    def launch_count(self):
        return int(lib().spv_launch_count(self.handle))

    def profile(self, enable=True):
        """Start (and clear) or stop the per-kernel-class event timing."""
        _raise(lib().spv_profile_enable(self.handle, 1 if enable else 0), "spv_profile_enable")

    def profile_read(self):
        """{class: dict(launches, ms, work)} accumulated since the last read; waits for the events."""
        arr = (KernelStat * len(KERNEL_CLASSES))()
        _raise(lib().spv_profile_read(self.handle, arr), "spv_profile_read")
        return {n: dict(launches=int(a.launches), ms=float(a.ms), work=float(a.work))
                for n, a in zip(KERNEL_CLASSES, arr)}

    def microbench(self, kind, ctas_per_sm=1, threads=128, iters=1000, m=128, n=64, box_rows=64, stages=4,
                   poly_per_8=0, accumulators=1, issue_mode=0, issuers=1, stream=None):
        """One hardware rate probe (spv_microbench); returns dict(ms, cycles, units, sm_count)."""
        d = MicrobenchDesc(MICROBENCH_KINDS[kind], ctas_per_sm, threads, iters, m, n, box_rows, stages, poly_per_8,
                           accumulators, issue_mode, issuers)
        nbytes = (32 << 20) + (64 << 10) if kind == "l2_tma" else (64 << 10)
        buf = self.workspace(nbytes)
        r = MicrobenchResult()
        _raise(lib().spv_microbench(self.handle, C.byref(d), _ptr(buf), buf.numel(), _stream(stream), C.byref(r)),
               "spv_microbench")
        return dict(ms=r.ms, cycles=r.cycles, units=r.units, sm_count=r.sm_count)

    # -- Sec. 3.3 ---------------------------------------------------------------------------
    def cls_score_topk_filter(self, scores, tokens_in=None, n_global=1, keep_ratio=0.5,
                              tokens_out=None, kept_idx=None, mean_scores=None, pos_in=None,
                              pos_out=None, workspace=None, stream=None):
        """scores fp32 [B, h, n_patch]; tokens_in bf16 [B, G+n_patch, dim] or None.
        Returns (tokens_out | None, kept_idx int32 [B, k])."""
        torch = self._torch
        B, H, NP = scores.shape
        k = filter_keep_count(NP, keep_ratio)
        dim = 0 if tokens_in is None else tokens_in.shape[-1]
        d = FilterDesc(B, H, NP, n_global, dim, float(keep_ratio), 0, 0)
        if kept_idx is None:
            kept_idx = torch.empty((B, k), dtype=torch.int32, device=scores.device)
        if tokens_in is not None and tokens_out is None:
            tokens_out = torch.empty((B, n_global + k, dim), dtype=tokens_in.dtype, device=scores.device)
        if workspace is None:
            need = C.c_size_t(0)
            _raise(lib().spv_filter_workspace_size(C.byref(d), C.byref(need)), "spv_filter_workspace_size")
            workspace = self.workspace(need.value)
        st = lib().cls_score_topk_filter(self.handle, C.byref(d), _ptr(scores), _ptr(tokens_in),
                                         _ptr(tokens_out), _ptr(kept_idx), _ptr(mean_scores), _ptr(pos_in),
                                         _ptr(pos_out), _ptr(workspace), workspace.numel(), _stream(stream))
        _raise(st, "cls_score_topk_filter")
        return tokens_out, kept_idx

    # -- Sec. 3.2 ---------------------------------------------------------------------------
    def attn_desc(self, q, grid_h, grid_w, block, radius, n_global=1, patch_pos=None, scale=0.0,
                  token_order=TOKENS_ROW_MAJOR):
        B, N, H, E = q.shape
        sb, st, sh, se = q.stride()
        assert se == 1
        return AttnDesc(B, grid_h, grid_w, block, radius, n_global, H, E, float(scale), N - n_global,
                        None if patch_pos is None else patch_pos.data_ptr(), token_order, sb, st, sh)

    def spatial_block_attention(self, q, k, v, grid_h, grid_w, block, radius, n_global=1, patch_pos=None,
                                scale=0.0, token_order=TOKENS_ROW_MAJOR, out=None, want_scores=False,
                                workspace=None, stream=None):
        """q, k, v bf16 [B, N, h, 64] views with identical strides.  Returns (o, cls_scores | None)."""
        torch = self._torch
        assert q.stride() == k.stride() == v.stride()
        d = self.attn_desc(q, grid_h, grid_w, block, radius, n_global, patch_pos, scale, token_order)
        if out is None:
            out = torch.empty_strided(q.shape, q.stride(), dtype=q.dtype, device=q.device)
        assert out.stride() == q.stride()
        sc = None
        if want_scores:
            sc = torch.empty((q.shape[0], q.shape[2], q.shape[1] - n_global), dtype=torch.float32,
                             device=q.device)
        if workspace is None:
            need = C.c_size_t(0)
            _raise(lib().spv_attn_workspace_size(C.byref(d), C.byref(need)), "spv_attn_workspace_size")
            workspace = self.workspace(need.value)
        st = lib().spatial_block_attention(self.handle, C.byref(d), _ptr(q), _ptr(k), _ptr(v), _ptr(out),
                                           _ptr(sc), _ptr(workspace), workspace.numel(), _stream(stream))
        _raise(st, "spatial_block_attention")
        return out, sc

    # -- 8-bit key/value cache ------------------------------------------------------------------
    # A decoder's step is a few microseconds of GPU work, so these methods keep the host's part short: every argument is
    # checked, by the cheapest expression that tells, and descriptors are packed into buffers of the context.
    def _kv_seqs(self, cache, page_table, lengths, max_length=0):
        """Packs spv_kv_seqs; returns the batch."""
        B, cols = page_table.shape
        rows, inner = page_table.stride()
        i32, dev = self._torch.int32, self._index
        _need(cache.device_index == dev and page_table.get_device() == dev and page_table.dtype is i32 and inner == 1 and
              (rows >= cols or B == 1), "page_table: int32 [batch, columns], rows apart, on the context's device, as the cache")
        _need(lengths.dtype is i32 and lengths.shape == (B,) and lengths.is_contiguous() and lengths.get_device() == dev,
              "lengths: int32 [batch]")
        _KV_SEQS.pack_into(self._seqs, 0, B, cols, rows if B > 1 else 0, page_table.data_ptr(), lengths.data_ptr(), max_length)
        return B

    def _kv_vector(self, t, B, what):
        if t is None:
            return 0
        _need(t.dtype is self._torch.int32 and t.shape == (B,) and t.is_contiguous() and t.get_device() == self._index,
              what + ": int32 [batch]")
        return t.data_ptr()

    def _kv_scratch(self, nbytes, workspace, stream):
        """The caller's workspace, or one from torch's allocator in the order of the call's stream: a captured
        graph then owns its own, and calls on two streams do not share one."""
        if workspace is not None:
            _need(workspace.dtype is self._torch.uint8 and workspace.is_contiguous() and workspace.get_device() == self._index,
                  "workspace: contiguous uint8 on the context's device")
            return workspace
        if nbytes == 0:
            return None
        return self._kv_new(self._torch.empty, nbytes, self._torch.uint8, stream)

    def _kv_new(self, make, shape, dtype, stream):
        """A tensor made in the order of the call's stream."""
        if stream is None:
            return make(shape, dtype=dtype, device=self.device)
        with self._torch.cuda.stream(stream):
            return make(shape, dtype=dtype, device=self.device)

    def _kv_stream(self, stream):
        if stream is not None:
            return stream.cuda_stream
        return _raw_stream(self._index)

    def _kv_dtype(self, t):
        dt = self._kv_types.get(t.dtype)
        _need(dt is not None and t.dim() == 4 and t.stride(3) == 1 and t.get_device() == self._index,
              "bf16, fp16 (or, of kv_cache_read, fp32) [batch, tokens, heads, head_dim], head_dim contiguous, on the "
              "context's device")
        return dt

    def _kv_weights(self, cache, w, B):
        _need(w.dtype is self._torch.float32 and w.dim() == 3 and w.shape[:2] == (B, cache.kv_heads) and
              w.stride(2) == 1 and w.get_device() == self._index, "weights: fp32 [batch, kv_heads, slots], slots contiguous")

    def kv_cache_append(self, cache, k, v, page_table, lengths, counts=None, stream=None):
        """Quantise new tokens' keys and values into the cache, behind the `lengths` that each sequence holds.
        k, v: bf16 or fp16 [B, tokens, kv_heads, head_dim] views with the same strides; counts: int32 [B], new
        tokens of each sequence (default: all).  `lengths` is not changed: add the counts to it afterwards."""
        dt = self._kv_dtype(k)
        shape, strides = k.shape, k.stride()
        B, n, h, d = shape
        _need(v.dtype is k.dtype and v.shape == shape and v.stride() == strides and v.get_device() == self._index, "v: as k")
        _need(h == cache.kv_heads and d == cache.head_dim and self._kv_seqs(cache, page_table, lengths) == B,
              "k: the cache's heads and head_dim, the table's batch")
        _KV_APPEND.pack_into(self._desc, 0, n, dt, *strides[:3], self._kv_vector(counts, B, "counts"))
        _raise(lib().kv_cache_append(self.handle, cache.address, self._seqs_at, self._desc_at, k.data_ptr(), v.data_ptr(),
                                     self._kv_stream(stream)), "kv_cache_append")

    def kv_cache_attention(self, cache, q, page_table, lengths, counts=None, causal=True, scale=0.0, out=None, lse=None,
                           weights_in=None, weights_out=None, max_length=None, workspace=None, stream=None):
        """Attention of q (bf16 or fp16 [B, tokens, heads, head_dim] view) over the cache; `lengths` include the
        queries' own tokens.  counts: int32 [B], queries of each sequence (default: all; rows behind them are not
        written).  lse: optional fp32 [B, tokens, heads] to fill.  weights_out: optional fp32 [B, kv_heads, slots]:
        weights_in (default 0; may be weights_out itself) plus the attention weight that every kept token received.
        max_length: no sequence is longer (default: what the table and the weights have room for; the workspace grows
        with it, and few or short sequences take one launch less when it is close).  Returns out."""
        torch = self._torch
        dt = self._kv_dtype(q)
        shape = q.shape
        B, n, H, d = shape
        if out is None:
            out = self._kv_new(torch.empty, shape, q.dtype, stream)
        o_strides = out.stride()
        _need(out.dtype is q.dtype and out.shape == shape and o_strides[3] == 1 and out.get_device() == self._index and
              (out.is_contiguous() or _apart(o_strides, shape)), "out: as q, no two elements at one place")
        limit = page_table.shape[1] * cache.block
        wb = wh = w_in_at = w_out_at = lse_at = 0
        if weights_out is not None:
            self._kv_weights(cache, weights_out, B)
            wb, wh, _ = weights_out.stride()
            limit = min(limit, weights_out.shape[2])
            _need(weights_out.is_contiguous() or _apart((wb, wh, 1), weights_out.shape), "weights_out: no two elements at one place")
            w_out_at = weights_out.data_ptr()
        if weights_in is not None:
            _need(weights_out is not None, "weights_in: only with weights_out")
            if weights_in is not weights_out:
                self._kv_weights(cache, weights_in, B)
                _need(weights_in.shape == weights_out.shape and weights_in.stride() == (wb, wh, 1), "weights_in: as weights_out")
            w_in_at = weights_in.data_ptr()
        if max_length is not None:
            _need(1 <= max_length <= limit, "max_length: 1 .. what the table and the weights have room for")
            limit = max_length
        if lse is not None:
            _need(lse.dtype is torch.float32 and lse.shape == (B, n, H) and lse.is_contiguous() and
                  lse.get_device() == self._index, "lse: fp32 [batch, tokens, heads]")
            lse_at = lse.data_ptr()
        _need(d == cache.head_dim and self._kv_seqs(cache, page_table, lengths, limit) == B,
              "q: [batch, tokens, heads, the cache's head_dim], the table's batch")
        _KV_ATTN.pack_into(self._desc, 0, n, H, dt, 1 if causal else 0, scale, *q.stride()[:3], *o_strides[:3], wb, wh,
                           self._kv_vector(counts, B, "counts"))
        L, need = lib(), self._size
        _raise(L.spv_kv_attention_workspace_size(cache.address, self._seqs_at, self._desc_at, 1 if w_out_at else 0, need),
               "spv_kv_attention_workspace_size")
        ws = self._kv_scratch(need.value, workspace, stream)
        _raise(L.kv_cache_attention(self.handle, cache.address, self._seqs_at, self._desc_at, q.data_ptr(), out.data_ptr(),
                                    lse_at, w_in_at, w_out_at, 0 if ws is None else ws.data_ptr(),
                                    0 if ws is None else ws.numel(), self._kv_stream(stream)), "kv_cache_attention")
        return out

    def kv_cache_evict(self, cache, weights, page_table, lengths, budget, keep_first=0, keep_last=0, dst_table=None,
                       kept=None, weights_out=None, new_lengths=None, max_length=None, workspace=None, stream=None):
        """Keep min(length, budget) tokens of every sequence and key head: the first keep_first, the last keep_last
        and of the others those of the largest weight (fp32 [B, kv_heads, slots]); moved together, in order, onto
        dst_table's pages (int32 [B, columns]; none of them a page of page_table), or, without one, onto the
        sequence's own.  Returns (kept int32 [B, kv_heads, budget], new_lengths int32 [B], weights_out fp32
        [B, kv_heads, budget])."""
        torch = self._torch
        B, h = page_table.shape[0], cache.kv_heads
        self._kv_weights(cache, weights, B)
        limit = min(page_table.shape[1] * cache.block, weights.shape[2])
        if max_length is not None:
            _need(1 <= max_length <= limit, "max_length: 1 .. what the table and the weights have room for")
            limit = max_length
        self._kv_seqs(cache, page_table, lengths, limit)
        _need(budget >= 1, "budget: 1 or more")
        shape, dev = (B, h, budget), self._index
        if kept is None:
            kept = self._kv_new(torch.empty, shape, torch.int32, stream)
        if weights_out is None:
            weights_out = self._kv_new(torch.zeros, shape, torch.float32, stream)
        if new_lengths is None:
            new_lengths = self._kv_new(torch.empty, (B,), torch.int32, stream)
        _need(kept.dtype is torch.int32 and kept.shape == shape and kept.is_contiguous() and kept.get_device() == dev,
              "kept: int32 [batch, kv_heads, budget]")
        _need(weights_out.dtype is torch.float32 and weights_out.shape == shape and weights_out.is_contiguous() and
              weights_out.get_device() == dev, "weights_out: fp32 [batch, kv_heads, budget]")
        nl = self._kv_vector(new_lengths, B, "new_lengths")
        dst = stride = 0
        if dst_table is not None:
            rows, cols = dst_table.stride(0), dst_table.shape[1]
            _need(dst_table.dtype is torch.int32 and dst_table.dim() == 2 and dst_table.shape[0] == B and
                  dst_table.stride(1) == 1 and cols * cache.block >= budget and (B == 1 or rows >= cols) and
                  dst_table.get_device() == dev, "dst_table: int32 [batch, budget / block or more], rows apart")
            dst, stride = dst_table.data_ptr(), rows if B > 1 else 0
        _KV_EVICT.pack_into(self._desc, 0, budget, keep_first, keep_last, weights.stride(0), weights.stride(1), dst, stride)
        L, nbytes = lib(), 0
        if dst_table is None:
            need = self._size
            _raise(L.spv_kv_evict_workspace_size(cache.address, self._seqs_at, self._desc_at, need),
                   "spv_kv_evict_workspace_size")
            nbytes = need.value
        ws = self._kv_scratch(nbytes, workspace, stream)
        _raise(L.kv_cache_evict(self.handle, cache.address, self._seqs_at, self._desc_at, weights.data_ptr(), kept.data_ptr(),
                                weights_out.data_ptr(), nl, 0 if ws is None else ws.data_ptr(), 0 if ws is None else ws.numel(),
                                self._kv_stream(stream)), "kv_cache_evict")
        return kept, new_lengths, weights_out

    def kv_cache_read(self, cache, page_table, counts, first=None, k_out=None, v_out=None, rows=None, dtype=None,
                      stream=None):
        """The values of slots first[b] (default 0) .. first[b] + counts[b] - 1 as rows 0 .. of k_out, v_out
        [B, rows, kv_heads, head_dim] (bf16, fp16 or fp32 views with the same strides; rows behind counts[b] are left
        as they were).  Without outputs, zeroed ones of `rows` rows and `dtype` (default bf16) are made; a single
        output may be given for only that half.  Returns (k_out, v_out)."""
        if k_out is None and v_out is None:
            torch = self._torch
            rows = page_table.shape[1] * cache.block if rows is None else rows
            made = (page_table.shape[0], rows, cache.kv_heads, cache.head_dim)
            k_out, v_out = (self._kv_new(torch.zeros, made, dtype or torch.bfloat16, stream) for _ in range(2))
        o = k_out if k_out is not None else v_out
        dt = self._kv_dtype(o)
        shape, strides = o.shape, o.stride()
        B = self._kv_seqs(cache, page_table, counts)
        _need(shape[0] == B and shape[2] == cache.kv_heads and shape[3] == cache.head_dim and
              (o.is_contiguous() or _apart(strides, shape)),
              "outputs: [batch, rows, kv_heads, head_dim], no two elements at one place")
        if k_out is not None and v_out is not None:
            _need(v_out.dtype is o.dtype and v_out.shape == shape and v_out.stride() == strides and
                  v_out.get_device() == self._index, "v_out: as k_out")
        _KV_READ.pack_into(self._desc, 0, shape[1], dt, *strides[:3], self._kv_vector(first, B, "first"))
        _raise(lib().kv_cache_read(self.handle, cache.address, self._seqs_at, self._desc_at,
                                   0 if k_out is None else k_out.data_ptr(), 0 if v_out is None else v_out.data_ptr(),
                                   self._kv_stream(stream)), "kv_cache_read")
        return k_out, v_out

    # -- building blocks ----------------------------------------------------------------------
    def gemm_bf16(self, a, w, out, epilogue=EPI_BIAS, bias=None, aux=None, scale=None, addrow=None,
                  rows_per_image=0, stream=None):
        """out = epilogue(a [M, K] @ w [N, K]^T); see spv_gemm_desc in include/spatvit.h."""
        M, K = a.shape
        N = w.shape[0]
        d = GemmDesc(M, N, K, a.stride(0), w.stride(0), out.stride(0), epilogue,
                     None if bias is None else bias.data_ptr(),
                     None if aux is None else aux.data_ptr(), 0 if aux is None else aux.stride(0),
                     None if scale is None else scale.data_ptr(),
                     None if addrow is None else addrow.data_ptr(),
                     0 if addrow is None else addrow.stride(0), rows_per_image)
        _raise(lib().spv_gemm_bf16(self.handle, C.byref(d), _ptr(a), _ptr(w), _ptr(out), _stream(stream)),
               "spv_gemm_bf16")
        return out

    def layernorm(self, x, gamma, beta, eps=1e-6, out=None, out_row=None, stream=None):
        torch = self._torch
        rows, dim = x.shape
        if out is None:
            out = torch.empty((rows, dim), dtype=torch.bfloat16, device=x.device)
        _raise(lib().spv_layernorm(self.handle, _ptr(x), rows, dim, _ptr(gamma), _ptr(beta), float(eps),
                                   _ptr(out), _ptr(out_row), _stream(stream)), "spv_layernorm")
        return out

    # -- Sec. 3 / 4.1 ---------------------------------------------------------------------------
    def make_vit_weights(self, weights):
        """Upload a dict of numpy fp32 weights (synth.vit_weights layout): matrices as bf16, vectors
        as fp32.  Returns an object holding the device tensors and the C structs."""
        return VitWeightsOnDevice(self, weights)

    def vit_forward(self, cfg, dev_weights, image, grid_h, grid_w, forced_keep=None, want_kept=True,
                    out=None, workspace=None, stream=None):
        """cfg: dict with the spv_vit_config fields; `filters`: optional list of (layer, keep_ratio) stages
        in place of filter_layer / keep_ratio.  image fp32 device [B, 3, H*p, W*p].  forced_keep: int32
        device [B, k_1 + ... + k_S] (the layout of the returned kept array).
        Returns (out_tokens bf16 [B, G+k, dim], kept int32 [B, k_1 + ... + k_S] | None)."""
        torch = self._torch
        stages = vit_filter_stages(cfg)
        multi = bool(cfg.get("filters"))
        fl = (C.c_int32 * 4)(*([l for l, _ in stages] + [0] * (4 - len(stages)))) if multi else (C.c_int32 * 4)()
        kr = (C.c_double * 4)(*([r for _, r in stages] + [0.0] * (4 - len(stages)))) if multi else (C.c_double * 4)()
        c = VitConfig(cfg["layers"], cfg["dim"], cfg["heads"], cfg["mlp_hidden"], cfg["mlp_kind"],
                      cfg["patch"], cfg["n_global"], cfg.get("has_layerscale", 0), cfg.get("ln_eps", 1e-6),
                      cfg["attn_mode"], cfg.get("block", 8), cfg.get("radius", 1),
                      0 if multi else cfg.get("filter_layer", 0), 1.0 if multi else cfg.get("keep_ratio", 1.0),
                      len(stages) if multi else 0, fl, kr, int(cfg.get("unfused_filter", 0)))
        B = image.shape[0]
        npatch = grid_h * grid_w
        counts, cur = [], npatch
        for _, ratio in stages:
            cur = filter_keep_count(cur, ratio)
            counts.append(cur)
        k = counts[-1] if counts else npatch
        if out is None:
            out = torch.empty((B, cfg["n_global"] + k, cfg["dim"]), dtype=torch.bfloat16, device=image.device)
        kept = torch.empty((B, sum(counts)), dtype=torch.int32, device=image.device) if (counts and want_kept) else None
        if forced_keep is not None:
            assert forced_keep.dtype == torch.int32 and forced_keep.is_contiguous()
            assert tuple(forced_keep.shape) == (B, sum(counts)), "forced_keep: one row of k_1 + ... + k_S per image"
        if workspace is None:
            need = C.c_size_t(0)
            _raise(lib().spv_vit_workspace_size(C.byref(c), B, grid_h, grid_w, C.byref(need)),
                   "spv_vit_workspace_size")
            workspace = self.workspace(need.value)
        st = lib().vit_forward(self.handle, C.byref(c), C.byref(dev_weights.struct), _ptr(image), B, grid_h,
                               grid_w, _ptr(out), _ptr(kept), _ptr(forced_keep), _ptr(workspace),
                               workspace.numel(), _stream(stream))
        _raise(st, "vit_forward")
        return out, kept

    def selftest_wait(self, limit_ns=200000, stream=None):
        """Launch the library's one-CTA kernel that waits on a barrier nobody arrives on; the wait gives up
        after limit_ns and the next check() reports the expired wait."""
        _raise(lib().spv_selftest_wait(self.handle, int(limit_ns), _stream(stream)), "spv_selftest_wait")


def vit_filter_stages(cfg):
    """[(layer, keep_ratio), ...] of a config dict."""
    if cfg.get("filters"):
        return [(int(l), float(r)) for l, r in cfg["filters"]]
    if cfg.get("filter_layer", 0) > 0:
        return [(int(cfg["filter_layer"]), float(cfg["keep_ratio"]))]
    return []


class VitWeightsOnDevice:
    MATRICES = {"w_pe", "w_qkv", "w_o", "w_fc1", "w_fc2", "w_fc3"}

    def __init__(self, ctx, weights):
        import numpy as np
        import torch
        self.tensors = []

        def up(name, a):
            if a is None:
                return None
            t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(ctx.device)
            if name in self.MATRICES:
                t = t.to(torch.bfloat16)
            t = t.contiguous()
            self.tensors.append(t)
            return t.data_ptr()

        n = len(weights["layers"])
        self.layers = (LayerWeights * n)()
        for i, lw in enumerate(weights["layers"]):
            for f in LAYER_FIELDS:
                setattr(self.layers[i], f, up(f, lw.get(f)))
        self.struct = VitWeights(up("w_pe", weights["w_pe"]), up("b_pe", weights["b_pe"]),
                                 up("cls", weights["cls"]), up("pos", weights["pos"]),
                                 up("lnf_g", weights["lnf_g"]), up("lnf_b", weights["lnf_b"]),
                                 C.cast(self.layers, C.c_void_p))
