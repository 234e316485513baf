"""Python binding of libhq.so: argument marshalling only.

Every entry point has the name of the C function it calls (include/hq.h).
PyTorch provides device memory and the current HIP stream; all codec work
runs in the library's gfx950 kernels.  There is no fallback: if libhq.so is
missing or fails to load, every call raises.
"""
import ctypes as C
import os

import numpy as np
import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libhq.so")

HQ_OK = 0
HQ_E8, HQ_D4, HQ_A2, HQ_Z = 0, 1, 2, 3
HQ_BF16, HQ_FP32, HQ_FP16, HQ_INT8, HQ_E4M3, HQ_MXFP4 = 0, 1, 2, 3, 4, 5
HQ_ROT_NONE, HQ_ROT_SIGNS, HQ_ROT_QJL = 0, 1, 2
LATTICES = {"E8": HQ_E8, "D4": HQ_D4, "A2": HQ_A2, "Z": HQ_Z}
STATUS = {0: "HQ_OK", -1: "HQ_ERR_INVALID_ARG", -2: "HQ_ERR_UNSUPPORTED", -3: "HQ_ERR_CAPACITY",
          -4: "HQ_ERR_OVERFLOW", -5: "HQ_ERR_HIP", -6: "HQ_ERR_CORRUPT",
          -7: "HQ_ERR_NO_CALIBRATION"}


class HQError(RuntimeError):
    def __init__(self, fn, status):
        super().__init__(f"{fn} failed: {STATUS.get(status, status)}")
        self.status = status


class Options(C.Structure):
    _fields_ = [("rotation", C.c_int32), ("dither", C.c_int32), ("rot_seed", C.c_uint64),
                ("dither_seed", C.c_uint64), ("norm_dtype", C.c_int32), ("substream", C.c_int32),
                ("use_snr", C.c_int32), ("reserved0", C.c_int32), ("snr_db", C.c_double),
                ("qjl", C.c_void_p)]


class PlanInfo(C.Structure):
    _fields_ = [("alpha", C.c_float), ("snr_db", C.c_float), ("tile", C.c_int32),
                ("lattice", C.c_int32), ("substream", C.c_int32), ("rice_k", C.c_int32),
                ("cols", C.c_int64), ("tiles_per_row", C.c_int64), ("subs_per_row", C.c_int64),
                ("max_words_per_substream", C.c_int64), ("max_words_per_row", C.c_int64)]


class Stats(C.Structure):
    _fields_ = [("payload_bits", C.c_uint64), ("pad_bits", C.c_uint64), ("status", C.c_uint32),
                ("overflow_tiles", C.c_uint32), ("corrupt_substreams", C.c_uint32),
                ("clamps", C.c_uint32)]


STATS_BYTES = C.sizeof(Stats)


class StreamStruct(C.Structure):
    _fields_ = [("payload", C.c_void_p), ("capacity_words", C.c_int64), ("offsets", C.c_void_p),
                ("kparam", C.c_void_p), ("norms", C.c_void_p), ("rows_capacity", C.c_int64),
                ("rows", C.c_int64), ("scan", C.c_void_p), ("scan_bytes", C.c_int64),
                ("stats", C.c_void_p)]


class CacheStruct(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("scales", C.c_void_p), ("blocks", C.c_int64),
                ("block_tokens", C.c_int32), ("heads", C.c_int32), ("format", C.c_int32),
                ("reserved0", C.c_int32), ("stats", C.c_void_p)]


class RotaryStruct(C.Structure):
    _fields_ = [("table", C.c_void_p), ("positions", C.c_int64), ("dims", C.c_int32),
                ("interleaved", C.c_int32), ("axes", C.c_int32), ("reserved0", C.c_int32),
                ("axis", C.c_void_p), ("stats", C.c_void_p)]


_lib = None


def lib():
    """Load libhq.so (built in-tree by paper_2606_23406_amd.build)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                           "`python -m paper_2606_23406_amd.build`")
    L = C.CDLL(LIB_PATH)
    p, i32, i64, u64, f32 = C.c_void_p, C.c_int32, C.c_int64, C.c_uint64, C.c_float
    L.hq_plan.restype = i32
    L.hq_plan.argtypes = [i32, i32, f32, u64, i32, i64, p, p, p]
    L.hq_plan_destroy.restype = i32
    L.hq_plan_destroy.argtypes = [p]
    L.hq_plan_get_info.restype = i32
    L.hq_plan_get_info.argtypes = [p, p]
    L.hq_scan_bytes.restype = C.c_size_t
    L.hq_scan_bytes.argtypes = [p, i64]
    L.hq_encode.restype = i32
    L.hq_encode.argtypes = [p, p, i32, i64, i64, p, i32, p]
    L.hq_encode_noalloc.restype = i32
    L.hq_encode_noalloc.argtypes = [p, p, i32, i64, i64, p, i32, p]
    L.hq_decode.restype = i32
    L.hq_decode.argtypes = [p, p, i64, i64, p, i32, i64, p]
    L.hq_encode_group.restype = i32
    L.hq_encode_group.argtypes = [p, p, i32, p, p, p, i32, p]
    L.hq_decode_group.restype = i32
    L.hq_decode_group.argtypes = [p, p, p, i32, p, i32, p]
    L.hq_decode_int8.restype = i32
    L.hq_decode_int8.argtypes = [p, p, i64, i64, p, i64, p, p]
    L.hq_act_prep.restype = i32
    L.hq_act_prep.argtypes = [p, p, i64, i64, p, p, p]
    L.hq_gemm_int8_blockscaled.restype = i32
    L.hq_gemm_int8_blockscaled.argtypes = [p, p, p, i64, p, p, i64, p, i32, p]
    L.hq_decode_fp8.restype = i32
    L.hq_decode_fp8.argtypes = [p, p, i64, i64, p, i64, p, p]
    L.hq_act_prep_fp8.restype = i32
    L.hq_act_prep_fp8.argtypes = [p, p, i64, i64, p, p, p]
    L.hq_gemm_fp8_blockscaled.restype = i32
    L.hq_gemm_fp8_blockscaled.argtypes = [p, p, p, i64, p, p, i64, p, i32, p]
    L.hq_decode_mxfp4.restype = i32
    L.hq_decode_mxfp4.argtypes = [p, p, i64, i64, p, p, p]
    L.hq_act_prep_mxfp4.restype = i32
    L.hq_act_prep_mxfp4.argtypes = [p, p, i64, i64, p, p, p]
    L.hq_gemm_mxfp4_blockscaled.restype = i32
    L.hq_gemm_mxfp4_blockscaled.argtypes = [p, p, p, i64, p, p, i64, p, i32, p]
    L.hq_gemm_workspace_bytes.restype = C.c_size_t
    L.hq_gemm_workspace_bytes.argtypes = [p, i64, i64]
    L.hq_dequant_gemm_int8.restype = i32
    L.hq_dequant_gemm_int8.argtypes = [p, p, i64, p, i64, p, i32, p, C.c_size_t, p]
    L.hq_gemv_workspace_bytes.restype = C.c_size_t
    L.hq_gemv_workspace_bytes.argtypes = [p]
    L.hq_decode_gemv.restype = i32
    L.hq_decode_gemv.argtypes = [p, p, i64, i64, p, i32, p, i32, p, C.c_size_t, p]
    L.hq_attention_workspace_bytes.restype = C.c_size_t
    L.hq_attention_workspace_bytes.argtypes = [p, i64, i32, i64]
    L.hq_decode_attention.restype = i32
    L.hq_decode_attention.argtypes = [p, p, p, p, p, i32, i64, i32, C.c_float, p, i32, i32, p, p,
                                      p, i32, i32, p, i32, p, C.c_size_t, p]
    L.hq_cache_write.restype = i32
    L.hq_cache_write.argtypes = [p, p, i64, p, p, p, i64, p, i32, i64, p, p]
    L.hq_cache_read.restype = i32
    L.hq_cache_read.argtypes = [p, p, p, i64, p, i32, i64, p]
    L.hq_cache_attention_workspace_bytes.restype = C.c_size_t
    L.hq_cache_attention_workspace_bytes.argtypes = [p, i64, i32, i32]
    L.hq_cache_attention.restype = i32
    L.hq_cache_attention.argtypes = [p, p, p, p, p, i32, i64, i32, f32, p, i32, p, p, i32, p,
                                     C.c_size_t, p]
    L.hq_rope_table.restype = i32
    L.hq_rope_table.argtypes = [p, i32, i64, f32, p, p]
    L.hq_rope.restype = i32
    L.hq_rope.argtypes = [p, p, i32, i64, i64, i32, p, i32, p, i32, i64, p]
    L.hq_cache_append.restype = i32
    L.hq_cache_append.argtypes = [p, p, i64, p, p, p, i64, p, i32, i64, p, p, p, p, i64, i32, p, i32, i64, p]
    L.hq_cache_window_workspace_bytes.restype = C.c_size_t
    L.hq_cache_window_workspace_bytes.argtypes = [p, i64, i32, i32, i32, i32]
    L.hq_cache_window_attention.restype = i32
    L.hq_cache_window_attention.argtypes = [p, p, p, p, p, i32, i64, i32, f32, p, i32, p, i32, i32, p, i32,
                                            p, C.c_size_t, p]
    L.hq_cache_tree_workspace_bytes.restype = C.c_size_t
    L.hq_cache_tree_workspace_bytes.argtypes = [p, i64, i32, i32, i32, i32, i32]
    L.hq_cache_tree_attention.restype = i32
    L.hq_cache_tree_attention.argtypes = [p, p, p, p, p, i32, i64, i32, f32, p, p, i64, i32, p, i32, p, i32,
                                          i32, p, i32, p, C.c_size_t, p]
    for fn in (L.hq_rmsnorm_act_prep, L.hq_rmsnorm_act_prep_fp8):
        fn.restype = i32
        fn.argtypes = [p, p, i64, p, i64, p, i32, f32, i64, p, i64, p, p, p]
    L.hq_rice_kstar.restype = i32
    L.hq_rice_kstar.argtypes = [i64, i64]
    L.hq_calibrated_snr.restype = i32
    L.hq_calibrated_snr.argtypes = [i32, i32, f32, C.POINTER(C.c_double)]
    L.hq_status_string.restype = C.c_char_p
    L.hq_status_string.argtypes = [i32]
    _lib = L
    return L


def _check(fn, status):
    if status != HQ_OK:
        raise HQError(fn, status)


# the current stream's handle alone, in a torch that gives it: building the Stream object
# around it takes 2.7 us
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_handle(stream=None):
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


def _dtype_code(dt):
    if dt is torch.bfloat16:
        return HQ_BF16
    if dt is torch.float32:
        return HQ_FP32
    raise ValueError(f"unsupported dtype {dt}")


class Plan:
    """An hq_plan handle and its derived values."""

    def __init__(self, handle, info: PlanInfo, options: Options):
        self.handle = handle
        self.info = info
        self.options = options

    @property
    def cols(self):
        return self.info.cols

    def __del__(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.hq_plan_destroy(self.handle)
            self.handle = None


def hq_plan(tile=128, lattice=HQ_E8, bps=4.0, rht_seed=0, rice_k=-1, cols=4096, *, rotation=0,
            dither=False, rot_seed=0, dither_seed=0, norm_fp16=False, snr_db=None, substream=0,
            qjl=None):
    """hq_plan of include/hq.h; snr_db bypasses the calibration table; qjl: the
    tile x tile orthogonal S of rotation HQ_ROT_QJL (host array, copied)."""
    L = lib()
    S = None
    if qjl is not None:
        S = np.ascontiguousarray(np.asarray(qjl, dtype=np.float32))
        assert S.shape == (tile, tile)
    o = Options(rotation, int(bool(dither)), rot_seed & (2**64 - 1), dither_seed & (2**64 - 1),
                HQ_FP16 if norm_fp16 else HQ_FP32, substream, 0 if snr_db is None else 1, 0,
                0.0 if snr_db is None else float(snr_db),
                None if S is None else S.ctypes.data_as(C.c_void_p))
    h = C.c_void_p()
    info = PlanInfo()
    st = L.hq_plan(tile, lattice, C.c_float(bps), rht_seed & (2**64 - 1), rice_k, cols, C.byref(o),
                   C.byref(h), C.byref(info))
    _check("hq_plan", st)
    o.qjl = None  # the plan holds its own device copy of S
    plan = Plan(h, info, o)
    plan.qjl = S
    return plan


class EncodedStream:
    """Device buffers of one encoded matrix (hq_stream), allocated with torch."""

    def __init__(self, plan: Plan, rows_capacity: int, device="cuda", capacity_words=None,
                 stats=True):
        info = plan.info
        self.plan = plan
        self.device = torch.device(device)
        cap = capacity_words if capacity_words is not None else rows_capacity * info.max_words_per_row
        self.payload = torch.zeros(max(int(cap), 1), dtype=torch.int32, device=device)
        nsub = rows_capacity * info.subs_per_row
        self.offsets = torch.zeros(nsub + 1, dtype=torch.int32, device=device)
        self.kparam = torch.zeros(max(nsub, 1), dtype=torch.uint8, device=device)
        ndt = torch.float16 if plan.options.norm_dtype == HQ_FP16 else torch.float32
        self.norms = torch.zeros(max(rows_capacity * info.tiles_per_row, 1), dtype=ndt,
                                 device=device)
        scan_bytes = lib().hq_scan_bytes(plan.handle, rows_capacity)
        self.scan = torch.zeros((scan_bytes + 7) // 8, dtype=torch.int64, device=device)
        self.stats = torch.zeros(STATS_BYTES // 4, dtype=torch.int32, device=device) if stats else None
        self.c = StreamStruct(self.payload.data_ptr(), int(cap), self.offsets.data_ptr(),
                              self.kparam.data_ptr(), self.norms.data_ptr(), rows_capacity, 0,
                              self.scan.data_ptr(), self.scan.numel() * 8,
                              self.stats.data_ptr() if stats else None)

    @property
    def rows(self):
        return self.c.rows

    def read_stats(self):
        if self.stats is None:
            return None
        raw = self.stats.cpu().numpy().tobytes()
        s = Stats.from_buffer_copy(raw)
        return {f: getattr(s, f) for f, _ in Stats._fields_}

    def reset_stats(self):
        if self.stats is not None:
            self.stats.zero_()

    def end_words(self):
        return int(self.offsets[self.rows * self.plan.info.subs_per_row].item()) & 0xFFFFFFFF


def hq_encode(plan: Plan, x: torch.Tensor, s: EncodedStream, append=False, stream=None):
    assert x.dim() == 2 and x.is_cuda
    rows = x.shape[0]
    ld = x.stride(0)
    assert x.stride(1) == 1
    st = lib().hq_encode(plan.handle, C.c_void_p(x.data_ptr()), _dtype_code(x.dtype), rows, ld,
                         C.byref(s.c), int(bool(append)), _stream_handle(stream))
    _check("hq_encode", st)
    return s


def hq_encode_noalloc(plan: Plan, x: torch.Tensor, s: EncodedStream, append=False, stream=None):
    """hq_encode_noalloc: hq_encode with the library's fixed look-back scratch
    (s.scan is not used)."""
    assert x.dim() == 2 and x.is_cuda
    rows = x.shape[0]
    ld = x.stride(0)
    assert x.stride(1) == 1
    st = lib().hq_encode_noalloc(plan.handle, C.c_void_p(x.data_ptr()), _dtype_code(x.dtype), rows,
                                 ld, C.byref(s.c), int(bool(append)), _stream_handle(stream))
    _check("hq_encode_noalloc", st)
    return s


def hq_decode(plan: Plan, s: EncodedStream, row0=0, rows=None, out_dtype=torch.bfloat16, out=None,
              stream=None):
    rows = s.rows - row0 if rows is None else rows
    if out is None:
        out = torch.empty((rows, plan.cols), dtype=out_dtype, device=s.device)
    st = lib().hq_decode(plan.handle, C.byref(s.c), row0, rows, C.c_void_p(out.data_ptr()),
                         _dtype_code(out.dtype), out.stride(0), _stream_handle(stream))
    _check("hq_decode", st)
    return out


def hq_encode_group(plans, xs, streams, stream=None):
    """hq_encode_group: encode xs[i] with plans[i] into streams[i] (whole
    matrices, as hq_encode with append = 0), several per launch."""
    n = len(plans)
    assert len(xs) == n and len(streams) == n and n > 0
    dt = _dtype_code(xs[0].dtype)
    for x in xs:
        assert x.dim() == 2 and x.is_cuda and x.stride(1) == 1 and _dtype_code(x.dtype) == dt
    ph = (C.c_void_p * n)(*[pl.handle for pl in plans])
    xp = (C.c_void_p * n)(*[x.data_ptr() for x in xs])
    rows = (C.c_int64 * n)(*[x.shape[0] for x in xs])
    lds = (C.c_int64 * n)(*[x.stride(0) for x in xs])
    sp = (C.c_void_p * n)(*[C.addressof(s.c) for s in streams])
    st = lib().hq_encode_group(ph, xp, dt, rows, lds, sp, n, _stream_handle(stream))
    _check("hq_encode_group", st)
    return streams


def hq_decode_group(plans, streams, outs, stream=None):
    """hq_decode_group: decode every row of streams[i] with plans[i] into
    outs[i] (bf16 or fp32, one dtype for the group), several per launch."""
    n = len(plans)
    assert len(streams) == n and len(outs) == n and n > 0
    dt = _dtype_code(outs[0].dtype)
    for y in outs:
        assert y.is_cuda and y.stride(1) == 1 and _dtype_code(y.dtype) == dt
    ph = (C.c_void_p * n)(*[pl.handle for pl in plans])
    sp = (C.c_void_p * n)(*[C.addressof(s.c) for s in streams])
    yp = (C.c_void_p * n)(*[y.data_ptr() for y in outs])
    lds = (C.c_int64 * n)(*[y.stride(0) for y in outs])
    st = lib().hq_decode_group(ph, sp, yp, dt, lds, n, _stream_handle(stream))
    _check("hq_decode_group", st)
    return outs


def hq_decode_int8(plan: Plan, s: EncodedStream, row0=0, rows=None, stream=None):
    rows = s.rows - row0 if rows is None else rows
    codes = torch.empty((rows, plan.cols), dtype=torch.int8, device=s.device)
    g = torch.empty((rows, plan.info.tiles_per_row), dtype=torch.float32, device=s.device)
    st = lib().hq_decode_int8(plan.handle, C.byref(s.c), row0, rows, C.c_void_p(codes.data_ptr()),
                              codes.stride(0), C.c_void_p(g.data_ptr()), _stream_handle(stream))
    _check("hq_decode_int8", st)
    return codes, g


def hq_decode_mxfp4(plan: Plan, s: EncodedStream, row0=0, rows=None, stream=None):
    """hq_decode_mxfp4: E2M1 code pairs (uint8, cols / 2 per row) and E8M0
    scale bytes (cols / 32 per row) of the reconstruction."""
    rows = s.rows - row0 if rows is None else rows
    codes = torch.empty((rows, plan.cols // 2), dtype=torch.uint8, device=s.device)
    scales = torch.empty((rows, plan.cols // 32), dtype=torch.uint8, device=s.device)
    st = lib().hq_decode_mxfp4(plan.handle, C.byref(s.c), row0, rows, C.c_void_p(codes.data_ptr()),
                               C.c_void_p(scales.data_ptr()), _stream_handle(stream))
    _check("hq_decode_mxfp4", st)
    return codes, scales


def hq_act_prep_mxfp4(plan: Plan, a: torch.Tensor, stream=None):
    """hq_act_prep_mxfp4: MXFP4 of the rotated activations (codes, scales)."""
    assert a.dim() == 2 and a.dtype == torch.bfloat16 and a.stride(1) == 1
    M = a.shape[0]
    xq = torch.empty((M, plan.cols // 2), dtype=torch.uint8, device=a.device)
    xs = torch.empty((M, plan.cols // 32), dtype=torch.uint8, device=a.device)
    st = lib().hq_act_prep_mxfp4(plan.handle, C.c_void_p(a.data_ptr()), M, a.stride(0),
                                 C.c_void_p(xq.data_ptr()), C.c_void_p(xs.data_ptr()),
                                 _stream_handle(stream))
    _check("hq_act_prep_mxfp4", st)
    return xq, xs


def hq_gemm_mxfp4_blockscaled(plan: Plan, xq, xs, codes, ws, out_dtype=torch.bfloat16, out=None,
                              stream=None):
    M, N = xq.shape[0], codes.shape[0]
    if out is None:
        out = torch.empty((M, N), dtype=out_dtype, device=xq.device)
    st = lib().hq_gemm_mxfp4_blockscaled(plan.handle, C.c_void_p(xq.data_ptr()),
                                         C.c_void_p(xs.data_ptr()), M, C.c_void_p(codes.data_ptr()),
                                         C.c_void_p(ws.data_ptr()), N, C.c_void_p(out.data_ptr()),
                                         _dtype_code(out.dtype), _stream_handle(stream))
    _check("hq_gemm_mxfp4_blockscaled", st)
    return out


def hq_decode_fp8(plan: Plan, s: EncodedStream, row0=0, rows=None, stream=None):
    """hq_decode_fp8: E4M3 code bytes (uint8) and the per-tile factors."""
    rows = s.rows - row0 if rows is None else rows
    codes = torch.empty((rows, plan.cols), dtype=torch.uint8, device=s.device)
    g = torch.empty((rows, plan.info.tiles_per_row), dtype=torch.float32, device=s.device)
    st = lib().hq_decode_fp8(plan.handle, C.byref(s.c), row0, rows, C.c_void_p(codes.data_ptr()),
                             codes.stride(0), C.c_void_p(g.data_ptr()), _stream_handle(stream))
    _check("hq_decode_fp8", st)
    return codes, g


def hq_act_prep_fp8(plan: Plan, a: torch.Tensor, stream=None):
    assert a.dtype == torch.bfloat16 and a.stride(1) == 1
    M = a.shape[0]
    xq = torch.empty((M, plan.cols), dtype=torch.uint8, device=a.device)
    sx = torch.empty((M,), dtype=torch.float32, device=a.device)
    st = lib().hq_act_prep_fp8(plan.handle, C.c_void_p(a.data_ptr()), M, a.stride(0),
                               C.c_void_p(xq.data_ptr()), C.c_void_p(sx.data_ptr()),
                               _stream_handle(stream))
    _check("hq_act_prep_fp8", st)
    return xq, sx


def hq_gemm_fp8_blockscaled(plan: Plan, xq, sx, codes, g, out_dtype=torch.bfloat16, out=None,
                            stream=None):
    M, N = xq.shape[0], codes.shape[0]
    if out is None:
        out = torch.empty((M, N), dtype=out_dtype, device=xq.device)
    st = lib().hq_gemm_fp8_blockscaled(plan.handle, C.c_void_p(xq.data_ptr()),
                                       C.c_void_p(sx.data_ptr()), M,
                                       C.c_void_p(codes.data_ptr()), C.c_void_p(g.data_ptr()), N,
                                       C.c_void_p(out.data_ptr()), _dtype_code(out.dtype),
                                       _stream_handle(stream))
    _check("hq_gemm_fp8_blockscaled", st)
    return out


def hq_act_prep(plan: Plan, a: torch.Tensor, stream=None):
    assert a.dtype == torch.bfloat16 and a.stride(1) == 1
    M = a.shape[0]
    xq = torch.empty((M, plan.cols), dtype=torch.int8, device=a.device)
    sx = torch.empty((M,), dtype=torch.float32, device=a.device)
    st = lib().hq_act_prep(plan.handle, C.c_void_p(a.data_ptr()), M, a.stride(0),
                           C.c_void_p(xq.data_ptr()), C.c_void_p(sx.data_ptr()),
                           _stream_handle(stream))
    _check("hq_act_prep", st)
    return xq, sx


def hq_gemm_int8_blockscaled(plan: Plan, xq, sx, codes, g, out_dtype=torch.bfloat16, out=None,
                             stream=None):
    M, N = xq.shape[0], codes.shape[0]
    if out is None:
        out = torch.empty((M, N), dtype=out_dtype, device=xq.device)
    st = lib().hq_gemm_int8_blockscaled(plan.handle, C.c_void_p(xq.data_ptr()),
                                        C.c_void_p(sx.data_ptr()), M,
                                        C.c_void_p(codes.data_ptr()), C.c_void_p(g.data_ptr()), N,
                                        C.c_void_p(out.data_ptr()), _dtype_code(out.dtype),
                                        _stream_handle(stream))
    _check("hq_gemm_int8_blockscaled", st)
    return out


def hq_gemm_workspace_bytes(plan: Plan, M, N):
    return lib().hq_gemm_workspace_bytes(plan.handle, M, N)


def hq_dequant_gemm_int8(plan: Plan, w: EncodedStream, a: torch.Tensor, out_dtype=torch.bfloat16,
                         workspace=None, out=None, stream=None):
    M, N = a.shape[0], w.rows
    nbytes = hq_gemm_workspace_bytes(plan, M, N)
    if workspace is None:
        workspace = torch.empty(nbytes, dtype=torch.uint8, device=a.device)
    if out is None:
        out = torch.empty((M, N), dtype=out_dtype, device=a.device)
    st = lib().hq_dequant_gemm_int8(plan.handle, C.byref(w.c), N, C.c_void_p(a.data_ptr()), M,
                                    C.c_void_p(out.data_ptr()), _dtype_code(out.dtype),
                                    C.c_void_p(workspace.data_ptr()), workspace.numel(),
                                    _stream_handle(stream))
    _check("hq_dequant_gemm_int8", st)
    return out


def hq_gemv_workspace_bytes(plan: Plan):
    return lib().hq_gemv_workspace_bytes(plan.handle)


def hq_decode_gemv(plan: Plan, s: EncodedStream, x: torch.Tensor, row0=0, rows=None,
                   out_dtype=torch.float32, workspace=None, out=None, stream=None):
    """hq_decode_gemv: y[r] = sum_k W^[row0 + r, k] x[k], the decoded rows
    never materialized.  x: plan.cols values (bf16 or fp32) on the device."""
    rows = s.rows - row0 if rows is None else rows
    assert x.is_cuda and x.dim() == 1 and x.stride(0) == 1 and x.numel() == plan.cols
    if workspace is None:
        workspace = torch.empty(hq_gemv_workspace_bytes(plan), dtype=torch.uint8, device=x.device)
    if out is None:
        out = torch.empty((rows,), dtype=out_dtype, device=x.device)
    st = lib().hq_decode_gemv(plan.handle, C.byref(s.c), row0, rows, C.c_void_p(x.data_ptr()),
                              _dtype_code(x.dtype), C.c_void_p(out.data_ptr()),
                              _dtype_code(out.dtype), C.c_void_p(workspace.data_ptr()),
                              workspace.numel(), _stream_handle(stream))
    _check("hq_decode_gemv", st)
    return out


def hq_attention_workspace_bytes(k_plan: Plan, batch, heads_q, max_tokens):
    return lib().hq_attention_workspace_bytes(k_plan.handle, batch, heads_q, max_tokens)


def hq_decode_attention(k_plan: Plan, k: EncodedStream, v_plan: Plan, v: EncodedStream,
                        q: torch.Tensor, block_table: torch.Tensor, seq_lens: torch.Tensor,
                        block_tokens, scale=None, out_dtype=torch.float32, workspace=None,
                        out=None, stream=None, window_k=None, window_v=None):
    """hq_decode_attention: q [batch, heads_q, 128] (bf16 or fp32) attends
    over the coded cache; block_table int32 [batch, max_blocks] and seq_lens
    int32 [batch] on the device.  window_k / window_v: optional residual
    window rings [batch, W, H_kv * 128] (bf16 or fp32, token t in slot t % W).
    Returns [batch, heads_q, 128]."""
    assert q.is_cuda and q.dim() == 3 and q.shape[2] == 128 and q.is_contiguous()
    assert block_table.dtype == torch.int32 and block_table.is_contiguous() and block_table.dim() == 2
    assert seq_lens.dtype == torch.int32 and seq_lens.is_contiguous()
    batch, heads_q = q.shape[0], q.shape[1]
    max_blocks = block_table.shape[1]
    scale = 128 ** -0.5 if scale is None else scale
    if workspace is None:
        nb = hq_attention_workspace_bytes(k_plan, batch, heads_q, max_blocks * block_tokens)
        workspace = torch.empty(max(nb, 16), dtype=torch.uint8, device=q.device)
    if out is None:
        out = torch.empty((batch, heads_q, 128), dtype=out_dtype, device=q.device)
    window, wk, wv, wt = 0, None, None, 0
    if window_k is not None:
        assert window_v is not None and window_k.shape == window_v.shape and window_k.dim() == 3
        assert window_k.is_contiguous() and window_v.is_contiguous() and window_k.dtype == window_v.dtype
        window, wt = window_k.shape[1], _dtype_code(window_k.dtype)
        wk, wv = C.c_void_p(window_k.data_ptr()), C.c_void_p(window_v.data_ptr())
    st = lib().hq_decode_attention(k_plan.handle, C.byref(k.c), v_plan.handle, C.byref(v.c),
                                   C.c_void_p(q.data_ptr()), _dtype_code(q.dtype), batch, heads_q,
                                   C.c_float(scale), C.c_void_p(block_table.data_ptr()),
                                   max_blocks, block_tokens, C.c_void_p(seq_lens.data_ptr()),
                                   wk, wv, wt, window,
                                   C.c_void_p(out.data_ptr()), _dtype_code(out.dtype),
                                   C.c_void_p(workspace.data_ptr()), workspace.numel(),
                                   _stream_handle(stream))
    _check("hq_decode_attention", st)
    return out


def _dense(t, dtype, shape, dev, name):
    """The address of a contiguous tensor of one type, shape and (the current) device."""
    if t.dtype is dtype and t.shape == shape and t.is_contiguous() and t.get_device() == dev:
        return t.data_ptr()
    raise ValueError(f"{name} must be a contiguous {dtype} {list(shape)} on cuda:{dev}, not "
                     f"{t.dtype} {list(t.shape)} of strides {t.stride()} on {t.device}")


def _rows(t, dtype, shape, dev, name):
    """Address and row stride of a [rows, width] tensor whose rows are contiguous."""
    if t.dtype is dtype and t.shape == shape and t.get_device() == dev:
        if t.is_contiguous():
            return t.data_ptr(), shape[1]
        ld, step = t.stride()
        if step == 1:
            return t.data_ptr(), ld if shape[0] > 1 else shape[1]
    raise ValueError(f"{name} must be {dtype} {list(shape)} with contiguous rows on cuda:{dev}, not "
                     f"{t.dtype} {list(t.shape)} of strides {t.stride()} on {t.device}")


def _empty(shape, dtype, dev, stream):
    """New memory of the stream that the call goes to."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=dev)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=dev)


class Cache:
    """A fixed-rate key or value cache (hq_cache) of `blocks` blocks of
    `block_tokens` slots in HQ_INT8, HQ_E4M3 or HQ_MXFP4.  heads: KV heads (the
    plan's cols / 128 by default).  codes / scales: tensors to use instead of
    new, zeroed ones (one byte a code, [blocks, heads, block_tokens, 128], and
    fp32 [blocks, heads, block_tokens]; MXFP4 [..., 64] and bytes [..., 4])."""

    def __init__(self, plan: Plan, blocks, block_tokens, format=HQ_INT8, heads=None, device="cuda",
                 codes=None, scales=None, stats=True):
        self.plan = plan
        self.heads = plan.cols // 128 if heads is None else heads
        self.blocks, self.block_tokens, self.format = blocks, block_tokens, format
        if format not in (HQ_INT8, HQ_E4M3, HQ_MXFP4):
            raise ValueError(f"unsupported cache format {format}")
        mx = format == HQ_MXFP4
        shape = (blocks, self.heads, block_tokens)
        cshape, sshape = shape + (64 if mx else 128,), shape + ((4,) if mx else ())
        sdt = torch.uint8 if mx else torch.float32
        if codes is None:
            codes = torch.zeros(cshape, dtype=torch.int8 if format == HQ_INT8 else torch.uint8, device=device)
        if scales is None:
            scales = torch.zeros(sshape, dtype=sdt, device=codes.device)
        for t, want, what in ((codes, cshape, "codes"), (scales, sshape, "scales")):
            if tuple(t.shape) != want or not t.is_contiguous() or not t.is_cuda:
                raise ValueError(f"{what} must be a contiguous device tensor of shape {want}")
        if codes.element_size() != 1 or scales.dtype != sdt or scales.device != codes.device:
            raise ValueError(f"codes of one byte and scales of {sdt} on one device")
        self.codes, self.scales, self.device = codes, scales, codes.device
        self.stats = torch.zeros(STATS_BYTES // 4, dtype=torch.int32, device=codes.device) if stats else None
        self.c = CacheStruct(codes.data_ptr(), scales.data_ptr(), blocks, block_tokens, self.heads,
                             format, 0, self.stats.data_ptr() if stats else None)
        self.ref = C.byref(self.c)

    def read_stats(self):
        if self.stats is None:
            return None
        s = Stats.from_buffer_copy(self.stats.cpu().numpy().tobytes())
        return {f: getattr(s, f) for f, _ in Stats._fields_}

    def reset_stats(self):
        if self.stats is not None:
            self.stats.zero_()


def hq_cache_write(k_plan: Plan, k: torch.Tensor, k_cache: Cache, v_plan, v, v_cache,
                   slots: torch.Tensor, stream=None):
    """hq_cache_write: k and v [rows, heads * 128] (bf16 or fp32) into the slots
    (int64 [rows], negative: skipped) of their caches; v_plan, v and v_cache
    None: k alone."""
    dev, dt = torch.cuda.current_device(), k.dtype
    shape = (k.shape[0], k_cache.heads * 128)
    kp, ldk = _rows(k, dt, shape, dev, "k")
    if k_cache.device.index != dev:
        raise ValueError(f"a cache on {k_cache.device} in a call on cuda:{dev}")
    if v is None:
        if v_plan is not None or v_cache is not None:
            raise ValueError("v_plan, v and v_cache come together")
        vh = vp = vc = None
        ldv = 0
    else:
        vp, ldv = _rows(v, dt, shape, dev, "v")
        if v_cache.device.index != dev:
            raise ValueError(f"a cache on {v_cache.device} in a call on cuda:{dev}")
        vh, vc = v_plan.handle, C.byref(v_cache.c)
    st = lib().hq_cache_write(k_plan.handle, kp, ldk, C.byref(k_cache.c), vh, vp, ldv, vc,
                              _dtype_code(dt), shape[0],
                              _dense(slots, torch.int64, shape[:1], dev, "slots"), _stream_handle(stream))
    _check("hq_cache_write", st)


def hq_cache_read(plan: Plan, cache: Cache, slots: torch.Tensor, out_dtype=torch.bfloat16, out=None,
                  stream=None):
    """hq_cache_read: the rows of the slots (int64, negative: zeros), [rows, heads * 128]."""
    dev = torch.cuda.current_device()
    shape = (slots.shape[0], cache.heads * 128)
    if cache.device.index != dev:
        raise ValueError(f"a cache on {cache.device} in a call on cuda:{dev}")
    if out is None:
        out = _empty(shape, out_dtype, dev, stream)
    dt = out.dtype
    op, ld = _rows(out, dt, shape, dev, "out")
    st = lib().hq_cache_read(plan.handle, C.byref(cache.c),
                             _dense(slots, torch.int64, shape[:1], dev, "slots"), shape[0], op,
                             _dtype_code(dt), ld, _stream_handle(stream))
    _check("hq_cache_read", st)
    return out


def hq_cache_attention_workspace_bytes(k_cache: Cache, batch, heads_q, max_blocks):
    return lib().hq_cache_attention_workspace_bytes(C.byref(k_cache.c), batch, heads_q, max_blocks)


def _attention_caches(k, v, dev):
    if k.device.index != dev or v.device.index != dev:
        raise ValueError(f"caches on {k.device} and {v.device} in a call on cuda:{dev}")


def _workspace(workspace, nbytes, dev, stream):
    """The caller's workspace or a new one, as a tensor."""
    if workspace is None:
        return _empty((max(nbytes(), 16),), torch.uint8, dev, stream)
    if not workspace.is_contiguous() or workspace.get_device() != dev:
        raise ValueError(f"workspace must be contiguous on cuda:{dev}")
    return workspace


def hq_cache_attention(k_plan: Plan, k: Cache, v_plan: Plan, v: Cache, q: torch.Tensor,
                       block_table: torch.Tensor, seq_lens: torch.Tensor, scale=None,
                       out_dtype=torch.float32, workspace=None, out=None, stream=None):
    """hq_cache_attention: q [batch, heads_q, 128] (bf16 or fp32) attends over
    the caches' blocks block_table int32 [batch, max_blocks], seq_lens int32
    [batch] tokens each.  Returns [batch, heads_q, 128]."""
    dev = torch.cuda.current_device()
    _attention_caches(k, v, dev)
    if q.dim() != 3 or block_table.dim() != 2:
        raise ValueError("q must be [batch, heads_q, 128] and block_table [batch, max_blocks]")
    batch, heads_q, max_blocks = q.shape[0], q.shape[1], block_table.shape[1]
    shape, qt = (batch, heads_q, 128), q.dtype
    qp = _dense(q, qt, shape, dev, "q")
    tp = _dense(block_table, torch.int32, (batch, max_blocks), dev, "block_table")
    lp = _dense(seq_lens, torch.int32, (batch,), dev, "seq_lens")
    if out is None:
        out = _empty(shape, out_dtype, dev, stream)
    ot = out.dtype
    workspace = _workspace(workspace, lambda: hq_cache_attention_workspace_bytes(k, batch, heads_q, max_blocks),
                           dev, stream)
    st = lib().hq_cache_attention(k_plan.handle, k.ref, v_plan.handle, v.ref, qp,
                                  _dtype_code(qt), batch, heads_q,
                                  128 ** -0.5 if scale is None else scale, tp, max_blocks, lp,
                                  _dense(out, ot, shape, dev, "out"), _dtype_code(ot),
                                  workspace.data_ptr(), workspace.nbytes, _stream_handle(stream))
    _check("hq_cache_attention", st)
    return out


class Rope:
    """Rotary positions (hq_rotary): `table` fp32 [positions, 2, dims / 2] (hq_rope_table
    makes one), the axis of each pair (a list of dims / 2 numbers; None: one axis), pairs
    (i, i + dims / 2) or, interleaved, (2 i, 2 i + 1).  axes: positions of a row, 1 to 4 (by
    default as many as the pairs use)."""

    def __init__(self, table: torch.Tensor, interleaved=False, axis=None, stats=True, axes=None):
        if table.dim() != 3 or table.shape[1] != 2 or table.dtype != torch.float32 or not table.is_contiguous() \
                or not table.is_cuda:
            raise ValueError("table must be a contiguous fp32 device tensor [positions, 2, dims / 2]")
        pairs = table.shape[2]
        axis = [0] * pairs if axis is None else [int(a) for a in axis]
        if len(axis) != pairs or not all(0 <= a < 4 for a in axis):
            raise ValueError(f"axis must be {pairs} numbers from 0 to 3")
        self.table, self.axis, self.device = table, axis, table.device
        self.axes = max(axis, default=0) + 1 if axes is None else int(axes)
        if not max(axis, default=0) < self.axes <= 4:
            raise ValueError(f"{self.axes} axes for pairs of axis {max(axis, default=0)}")
        self._axis = (C.c_uint8 * pairs)(*axis)
        self.stats = torch.zeros(STATS_BYTES // 4, dtype=torch.int32, device=table.device) if stats else None
        self.c = RotaryStruct(table.data_ptr(), table.shape[0], 2 * pairs, int(bool(interleaved)), self.axes, 0,
                              C.addressof(self._axis), self.stats.data_ptr() if stats else None)
        self.ref = C.byref(self.c)

    read_stats = Cache.read_stats
    reset_stats = Cache.reset_stats


def hq_rope_table(freqs: torch.Tensor, positions, factor=1.0, out=None, stream=None):
    """hq_rope_table: cosines and sines of positions 0 .. positions - 1 at freqs (fp64
    [pairs], radians a position), fp32 [positions, 2, pairs]."""
    dev, pairs = torch.cuda.current_device(), freqs.shape[0]
    shape = (positions, 2, pairs)
    fp = _dense(freqs, torch.float64, (pairs,), dev, "freqs")
    if out is None:
        out = _empty(shape, torch.float32, dev, stream)
    st = lib().hq_rope_table(fp, pairs, positions, factor, _dense(out, torch.float32, shape, dev, "out"),
                             _stream_handle(stream))
    _check("hq_rope_table", st)
    return out


def _positions(rope, positions, rows, dev):
    if rope.device.index != dev:
        raise ValueError(f"a table on {rope.device} in a call on cuda:{dev}")
    if rope.axes == 1 and positions.dim() == 1:
        return _dense(positions, torch.int32, (rows,), dev, "positions")
    return _dense(positions, torch.int32, (rows, rope.axes), dev, "positions")


def hq_rope(rope: Rope, x: torch.Tensor, positions: torch.Tensor, transposed=False, out_dtype=None, out=None,
            stream=None):
    """hq_rope: x [rows, heads * 128] (bf16 or fp32) turned by positions int32 [rows, axes]
    (of one axis also [rows]); transposed: the gradient.  out may be x.  Without an out, rows
    of padding (a negative first position) are zeros."""
    dev, dt, shape = torch.cuda.current_device(), x.dtype, x.shape
    if len(shape) != 2 or shape[1] % 128:
        raise ValueError(f"x must be [rows, heads * 128], not {list(shape)}")
    xp, ldx = _rows(x, dt, shape, dev, "x")
    pp = _positions(rope, positions, shape[0], dev)
    if out is None:
        out = _empty(shape, dt if out_dtype is None else out_dtype, dev, stream)
        with torch.cuda.stream(stream):
            out.zero_()
    ot = out.dtype
    op, ldo = _rows(out, ot, shape, dev, "out")
    st = lib().hq_rope(rope.ref, xp, _dtype_code(dt), ldx, shape[0], shape[1] // 128, pp, int(bool(transposed)),
                       op, _dtype_code(ot), ldo, _stream_handle(stream))
    _check("hq_rope", st)
    return out


def hq_cache_append(k_plan: Plan, k: torch.Tensor, k_cache: Cache, v_plan, v, v_cache, slots: torch.Tensor,
                    rope: Rope, positions: torch.Tensor, q=None, q_out=None, stream=None):
    """hq_cache_append: hq_cache_write with k turned by positions int32 [rows, axes] on the
    way; q [rows, heads_q * 128] turned into q_out, which may be q and is returned (a new
    tensor of q's type without one, zeros in rows of padding)."""
    dev, dt = torch.cuda.current_device(), k.dtype
    shape = (k.shape[0], k_cache.heads * 128)
    kp, ldk = _rows(k, dt, shape, dev, "k")
    if k_cache.device.index != dev:
        raise ValueError(f"a cache on {k_cache.device} in a call on cuda:{dev}")
    if v is None:
        if v_plan is not None or v_cache is not None:
            raise ValueError("v_plan, v and v_cache come together")
        vh = vp = vc = None
        ldv = 0
    else:
        vp, ldv = _rows(v, dt, shape, dev, "v")
        if v_cache.device.index != dev:
            raise ValueError(f"a cache on {v_cache.device} in a call on cuda:{dev}")
        vh, vc = v_plan.handle, v_cache.ref
    sp = _dense(slots, torch.int64, shape[:1], dev, "slots")
    pp = _positions(rope, positions, shape[0], dev)
    if q is None:
        if q_out is not None:
            raise ValueError("q and q_out come together")
        qp = op = None
        ldq = ldo = heads_q = ot = 0
    else:
        qshape = (shape[0], q.shape[1])
        if qshape[1] % 128:
            raise ValueError(f"q must be [rows, heads_q * 128], not {list(q.shape)}")
        qp, ldq = _rows(q, dt, qshape, dev, "q")
        if q_out is None:
            q_out = _empty(qshape, dt, dev, stream)
            with torch.cuda.stream(stream):
                q_out.zero_()
        op, ldo = _rows(q_out, q_out.dtype, qshape, dev, "q_out")
        heads_q, ot = qshape[1] // 128, _dtype_code(q_out.dtype)
    st = lib().hq_cache_append(k_plan.handle, kp, ldk, k_cache.ref, vh, vp, ldv, vc, _dtype_code(dt), shape[0],
                               sp, rope.ref, pp, qp, ldq, heads_q, op, ot, ldo, _stream_handle(stream))
    _check("hq_cache_append", st)
    return q_out


def _tokens(n):
    """A number of tokens for an int32 argument, which would keep a larger one's low bits: no sequence
    has more than 2^30."""
    return n if -1 <= n < 1 << 30 else 1 << 30 if n > 0 else -1


def hq_cache_window_workspace_bytes(k_cache: Cache, batch, heads_q, max_blocks, window, sinks=0):
    return lib().hq_cache_window_workspace_bytes(k_cache.ref, batch, heads_q, max_blocks, _tokens(window), _tokens(sinks))


def hq_cache_window_attention(k_plan: Plan, k: Cache, v_plan: Plan, v: Cache, q: torch.Tensor,
                              block_table: torch.Tensor, seq_lens: torch.Tensor, window, sinks=0, scale=None,
                              out_dtype=torch.float32, workspace=None, out=None, stream=None):
    """hq_cache_window_attention: hq_cache_attention over the last `window` tokens of each
    sequence and its first `sinks`."""
    dev = torch.cuda.current_device()
    _attention_caches(k, v, dev)
    if q.dim() != 3 or block_table.dim() != 2:
        raise ValueError("q must be [batch, heads_q, 128] and block_table [batch, max_blocks]")
    batch, heads_q, max_blocks = q.shape[0], q.shape[1], block_table.shape[1]
    shape, qt = (batch, heads_q, 128), q.dtype
    qp = _dense(q, qt, shape, dev, "q")
    tp = _dense(block_table, torch.int32, (batch, max_blocks), dev, "block_table")
    lp = _dense(seq_lens, torch.int32, (batch,), dev, "seq_lens")
    if out is None:
        out = _empty(shape, out_dtype, dev, stream)
    ot = out.dtype
    workspace = _workspace(
        workspace, lambda: hq_cache_window_workspace_bytes(k, batch, heads_q, max_blocks, window, sinks), dev, stream)
    st = lib().hq_cache_window_attention(k_plan.handle, k.ref, v_plan.handle, v.ref, qp,
                                         _dtype_code(qt), batch, heads_q, 128 ** -0.5 if scale is None else scale, tp,
                                         max_blocks, lp, _tokens(window), _tokens(sinks),
                                         _dense(out, ot, shape, dev, "out"),
                                         _dtype_code(ot), workspace.data_ptr(), workspace.nbytes,
                                         _stream_handle(stream))
    _check("hq_cache_window_attention", st)
    return out


def hq_cache_tree_workspace_bytes(k_cache: Cache, batch, heads_q, max_blocks, max_tree, window=0, sinks=0):
    return lib().hq_cache_tree_workspace_bytes(k_cache.ref, batch, heads_q, max_blocks, max_tree, _tokens(window),
                                               _tokens(sinks))


def hq_cache_tree_attention(k_plan: Plan, k: Cache, v_plan: Plan, v: Cache, q: torch.Tensor, masks: torch.Tensor,
                            starts: torch.Tensor, max_tree, block_table: torch.Tensor, seq_lens: torch.Tensor,
                            window=0, sinks=0, scale=None, out_dtype=torch.float32, workspace=None, out=None,
                            stream=None):
    """hq_cache_tree_attention: q [rows, heads_q, 128] (bf16 or fp32), the drafted tokens of all
    sequences, sequence b's rows starts[b] .. starts[b + 1] - 1 (int32 [batch + 1], max_tree of
    them at most), the last tokens of its seq_lens; masks int64 or uint64 [rows]: bit j for the
    tree's token j.  Returns [rows, heads_q, 128]; without an out, rows of no sequence are zeros."""
    dev = torch.cuda.current_device()
    _attention_caches(k, v, dev)
    if q.dim() != 3 or block_table.dim() != 2:
        raise ValueError("q must be [rows, heads_q, 128] and block_table [batch, max_blocks]")
    rows, heads_q, (batch, max_blocks) = q.shape[0], q.shape[1], block_table.shape
    shape, qt, mt = (rows, heads_q, 128), q.dtype, masks.dtype
    if mt not in (torch.int64, torch.uint64):
        raise ValueError(f"masks must be int64 or uint64, not {mt}")
    qp = _dense(q, qt, shape, dev, "q")
    mp = _dense(masks, mt, (rows,), dev, "masks")
    sp = _dense(starts, torch.int32, (batch + 1,), dev, "starts")
    tp = _dense(block_table, torch.int32, (batch, max_blocks), dev, "block_table")
    lp = _dense(seq_lens, torch.int32, (batch,), dev, "seq_lens")
    if out is None:
        out = _empty(shape, out_dtype, dev, stream)
        with torch.cuda.stream(stream):
            out.zero_()
    ot = out.dtype
    workspace = _workspace(
        workspace, lambda: hq_cache_tree_workspace_bytes(k, batch, heads_q, max_blocks, max_tree, window, sinks), dev,
        stream)
    st = lib().hq_cache_tree_attention(k_plan.handle, k.ref, v_plan.handle, v.ref, qp, _dtype_code(qt),
                                       rows, heads_q, 128 ** -0.5 if scale is None else scale, mp, sp, batch, max_tree,
                                       tp, max_blocks, lp, _tokens(window), _tokens(sinks),
                                       _dense(out, ot, shape, dev, "out"), _dtype_code(ot), workspace.data_ptr(), workspace.nbytes,
                                       _stream_handle(stream))
    _check("hq_cache_tree_attention", st)
    return out


def _rmsnorm_act_prep(fn, code, plan, x, weight, eps, residual, h, xq, sx, stream):
    dev, bf16 = torch.cuda.current_device(), torch.bfloat16
    shape = (x.shape[0], plan.info.cols)
    xp, ldx = _rows(x, bf16, shape, dev, "x")
    wt = weight.dtype
    if residual is None:
        rp, ldr = None, 0
    else:
        rp, ldr = _rows(residual, bf16, shape, dev, "residual")
        if h is None:
            h = _empty(shape, bf16, dev, stream)
    hp, ldh = (None, 0) if h is None else _rows(h, bf16, shape, dev, "h")
    if xq is None:
        xq = _empty(shape, code, dev, stream)
    if sx is None:
        sx = _empty(shape[:1], torch.float32, dev, stream)
    st = getattr(lib(), fn)(plan.handle, xp, ldx, rp, ldr, _dense(weight, wt, shape[1:], dev, "weight"),
                            _dtype_code(wt), eps, shape[0], hp, ldh, _dense(xq, code, shape, dev, "xq"),
                            _dense(sx, torch.float32, shape[:1], dev, "sx"), _stream_handle(stream))
    _check(fn, st)
    return (xq, sx) if residual is None else (xq, sx, h)


def hq_rmsnorm_act_prep(plan: Plan, x: torch.Tensor, weight: torch.Tensor, eps=1e-5, residual=None,
                        h=None, xq=None, sx=None, stream=None):
    """hq_rmsnorm_act_prep: h = x + residual, then the int8 activation prep of
    its RMS norm.  Returns (xq, sx), with a residual (xq, sx, h); h may be
    residual or x itself."""
    return _rmsnorm_act_prep("hq_rmsnorm_act_prep", torch.int8, plan, x, weight, eps, residual, h, xq,
                             sx, stream)


def hq_rmsnorm_act_prep_fp8(plan: Plan, x: torch.Tensor, weight: torch.Tensor, eps=1e-5,
                            residual=None, h=None, xq=None, sx=None, stream=None):
    """hq_rmsnorm_act_prep_fp8: the same in E4M3 (bytes)."""
    return _rmsnorm_act_prep("hq_rmsnorm_act_prep_fp8", torch.uint8, plan, x, weight, eps, residual, h,
                             xq, sx, stream)


def hq_rice_kstar(count, total):
    return lib().hq_rice_kstar(int(count), int(total))


def hq_calibrated_snr(lattice, rice_k, bps):
    v = C.c_double()
    st = lib().hq_calibrated_snr(lattice, rice_k, C.c_float(bps), C.byref(v))
    _check("hq_calibrated_snr", st)
    return v.value


EXPORTED = ["hq_plan", "hq_plan_destroy", "hq_plan_get_info", "hq_scan_bytes", "hq_encode",
            "hq_encode_noalloc",
            "hq_decode", "hq_encode_group", "hq_decode_group", "hq_decode_int8", "hq_act_prep", "hq_gemm_int8_blockscaled",
            "hq_gemm_workspace_bytes", "hq_dequant_gemm_int8", "hq_gemv_workspace_bytes",
            "hq_decode_gemv", "hq_attention_workspace_bytes", "hq_decode_attention",
            "hq_decode_fp8", "hq_act_prep_fp8", "hq_gemm_fp8_blockscaled",
            "hq_decode_mxfp4", "hq_act_prep_mxfp4", "hq_gemm_mxfp4_blockscaled",
            "hq_cache_write", "hq_cache_read", "hq_cache_attention_workspace_bytes",
            "hq_cache_attention", "hq_rope_table", "hq_rope", "hq_cache_append",
            "hq_cache_window_workspace_bytes", "hq_cache_window_attention",
            "hq_cache_tree_workspace_bytes", "hq_cache_tree_attention", "hq_rmsnorm_act_prep", "hq_rmsnorm_act_prep_fp8",
            "hq_rice_kstar",
            "hq_calibrated_snr", "hq_status_string"]
