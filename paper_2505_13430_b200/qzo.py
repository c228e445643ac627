"""Thin Python binding of the C-ABI library (libqzo.so): argument marshalling only.

Every function has the name of the C entry point it calls and takes torch CUDA tensors
where the C function takes device pointers.  PyTorch is used for device memory and
streams; every step of the path runs in the library's kernels.  There is no fallback:
if the shared library is missing or fails to load, importing this module raises.
"""
import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libqzo.so")

QZO_OK = 0
ERR_BAD_ARG, ERR_UNSUPPORTED_DEVICE, ERR_WORKSPACE, ERR_NONFINITE = -1, -2, -3, -4
ERR_DEVICE_TIMEOUT, ERR_CUDA, ERR_MISSING_TENSOR = -5, -6, -7
ARCH = {"llama": 0, "opt": 1}
DTYPE = {torch.bfloat16: 0, torch.float32: 1, torch.int32: 3}
DTYPE_U32 = 2

EXPORTS = (
    "qzo_strerror", "qzo_last_cuda_error", "qzo_philox_words", "qzo_normals", "qzo_quantize_int4",
    "qzo_unpack_int4", "qzo_repacked_bytes", "qzo_repack_int4", "qzo_unpack_kernel_layout",
    "qzo_gemm_workspace_bytes", "qzo_perturbed_gemm", "qzo_perturbed_gemm_noalloc", "qzo_update_scales_flat", "qzo_num_scales",
    "qzo_scale_layout", "qzo_workspace_bytes", "qzo_init_model", "qzo_free_model", "qzo_forward_loss",
    "qzo_update_scales", "qzo_step", "qzo_step_host", "qzo_debug_set_capture", "qzo_debug_layer_output",
    "qzo_device_status", "qzo_launch_count", "qzo_profile_gemms", "qzo_profile_read",
    "qzo_step_begin", "qzo_step_finish", "qzo_get_scales", "qzo_set_scales", "qzo_debug_set_status", "qzo_use_recorded_steps", "qzo_recorded_step_count", "qzo_perturbed_gemm_codebook16_channelwise",
    "qzo_joint_workspace_bytes", "qzo_enable_joint_spsa", "qzo_perturbed_gemm_table16", "qzo_debug_gemm_wait_expiry",
    "qzo_gemv_int4", "qzo_rope_table", "qzo_qk_norm_rope_cache", "qzo_paged_attention_workspace_bytes", "qzo_paged_attention",
    "qzo_assign_slots", "qzo_decode", "qzo_decode_requests",
    "qzo_beam_select_workspace_bytes", "qzo_beam_select", "qzo_fork_requests", "qzo_compact_blocks", "qzo_copy_blocks",
    "qzo_shared_prefix_attention_workspace_bytes", "qzo_shared_prefix_attention", "qzo_debug_prefix_path", "qzo_decode_groups",
)


class QzoError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        msg = _lib.qzo_strerror(status).decode()
        if status == ERR_CUDA:
            msg += f" [cudaError {_lib.qzo_last_cuda_error()}]"
        super().__init__(f"{where}: {msg} ({status})")


class ModelDesc(ctypes.Structure):
    _fields_ = [("arch", ctypes.c_int), ("n_layers", ctypes.c_int), ("d_model", ctypes.c_int),
                ("n_heads", ctypes.c_int), ("d_ffn", ctypes.c_int), ("vocab", ctypes.c_int),
                ("max_seq", ctypes.c_int), ("group_size", ctypes.c_int),
                ("norm_eps", ctypes.c_float), ("rope_theta", ctypes.c_float)]


class Tensor(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char_p), ("dptr", ctypes.c_void_p), ("dtype", ctypes.c_int),
                ("shape", ctypes.c_int64 * 2)]


class KvCacheDesc(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("dtype", ctypes.c_int), ("n_blocks", ctypes.c_int),
                ("block_size", ctypes.c_int), ("n_kv_heads", ctypes.c_int), ("head_dim", ctypes.c_int),
                ("k_scale", ctypes.c_float), ("v_scale", ctypes.c_float)]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with paper_2505_13430_b200/build.py "
                          "(there is no fallback path)")
    lib = ctypes.CDLL(LIB_PATH)
    vp, u64, i64, ci, cf, sz = (ctypes.c_void_p, ctypes.c_uint64, ctypes.c_int64, ctypes.c_int,
                                ctypes.c_float, ctypes.c_size_t)
    P = ctypes.POINTER
    sig = {
        "qzo_strerror": (ctypes.c_char_p, [ci]),
        "qzo_last_cuda_error": (ci, []),
        "qzo_launch_count": (i64, []),
        "qzo_philox_words": (ci, [u64, u64, i64, vp, vp, vp]),
        "qzo_normals": (ci, [u64, u64, i64, vp, vp]),
        "qzo_quantize_int4": (ci, [vp, ci, ci, vp, vp, vp]),
        "qzo_unpack_int4": (ci, [vp, ci, ci, vp, vp]),
        "qzo_repacked_bytes": (ci, [ci, ci, P(sz)]),
        "qzo_repack_int4": (ci, [vp, ci, ci, vp, sz, vp]),
        "qzo_unpack_kernel_layout": (ci, [vp, ci, ci, vp, vp]),
        "qzo_gemm_workspace_bytes": (ci, [ci, ci, ci, P(sz)]),
        "qzo_perturbed_gemm": (ci, [vp, vp, vp, vp, vp, ci, ci, ci, u64, u64, ci, cf, vp, sz, vp, vp]),
        "qzo_perturbed_gemm_table16": (ci, [vp, vp, vp, P(cf), vp, vp, ci, ci, ci, u64, u64, ci, cf, vp, sz, vp, vp]),
        "qzo_perturbed_gemm_codebook16_channelwise": (ci, [vp, vp, vp, P(cf), vp, vp, ci, ci, ci, u64, u64, ci, cf, vp, sz, vp, vp]),
        "qzo_debug_gemm_wait_expiry": (ci, [vp, vp, vp, vp, ci, ci, ci, ci, i64, vp, vp]),
        "qzo_perturbed_gemm_noalloc": (ci, [vp, vp, vp, vp, vp, ci, ci, ci, u64, u64, ci, cf, vp, vp]),
        "qzo_update_scales_flat": (ci, [vp, i64, u64, u64, cf, cf, cf, vp]),
        "qzo_num_scales": (ci, [P(ModelDesc), P(i64), P(i64)]),
        "qzo_scale_layout": (ci, [P(ModelDesc), ci, ci, P(i64), P(ci), P(ci)]),
        "qzo_workspace_bytes": (ci, [P(ModelDesc), ci, P(sz)]),
        "qzo_init_model": (ci, [P(ModelDesc), P(Tensor), ci, vp, sz, ci, vp, P(vp)]),
        "qzo_free_model": (ci, [vp]),
        "qzo_forward_loss": (ci, [vp, vp, vp, ci, ci, u64, ci, cf, vp]),
        "qzo_update_scales": (ci, [vp, u64, cf, cf, cf]),
        "qzo_step": (ci, [vp, vp, vp, ci, ci, u64, cf, cf, cf, vp]),
        "qzo_step_host": (ci, [vp, vp, vp, ci, ci, u64, cf, cf, cf, vp]),
        "qzo_step_begin": (ci, [vp, vp, vp, ci, ci, u64, cf, vp]),
        "qzo_step_finish": (ci, [vp, vp, u64, cf, cf, cf, vp]),
        "qzo_get_scales": (ci, [vp, ci, vp, sz]),
        "qzo_set_scales": (ci, [vp, ci, vp, sz]),
        "qzo_debug_set_status": (ci, [vp, ci]),
        "qzo_use_recorded_steps": (ci, [vp, ci]),
        "qzo_recorded_step_count": (ci, [vp, vp]),
        "qzo_joint_workspace_bytes": (ci, [P(ModelDesc), P(sz)]),
        "qzo_enable_joint_spsa": (ci, [vp, vp, sz, cf]),
        "qzo_debug_set_capture": (ci, [vp, ci]),
        "qzo_debug_layer_output": (ci, [vp, ci, ci, vp, sz]),
        "qzo_device_status": (ci, [vp, P(ci)]),
        "qzo_gemv_int4": (ci, [vp, ci, vp, vp, vp, vp, ci, ci, ci, ci, vp]),
        "qzo_rope_table": (ci, [vp, ci, ci, cf, vp]),
        "qzo_qk_norm_rope_cache": (ci, [vp, ci, vp, ci, vp, ci, vp, vp, cf, vp, ci, vp, vp, vp, ci, P(KvCacheDesc), ci, ci, vp, vp]),
        "qzo_paged_attention_workspace_bytes": (ci, [ci, ci, ci, ci, ci, P(sz)]),
        "qzo_paged_attention": (ci, [vp, ci, P(KvCacheDesc), vp, ci, ci, vp, vp, cf, vp, ci, ci, ci, vp, sz, vp, vp]),
        "qzo_assign_slots": (ci, [vp, vp, ci, vp, ci, ci, vp, ci, vp, ci, vp, vp, vp, vp, vp, vp, vp]),
        "qzo_decode_requests": (ci, [vp, P(KvCacheDesc), vp, vp, vp, ci, vp, ci, vp, ci, vp, ci, vp, vp, vp]),
        "qzo_decode": (ci, [vp, P(KvCacheDesc), vp, vp, vp, vp, ci, vp, ci, ci, vp]),
        "qzo_beam_select_workspace_bytes": (ci, [ci, ci, ci, P(sz)]),
        "qzo_beam_select": (ci, [vp, i64, ci, vp, vp, vp, ci, vp, cf, ci, ci, ci, vp, vp, vp, vp, vp, sz, vp, vp]),
        "qzo_fork_requests": (ci, [vp, vp, ci, vp, ci, ci, ci, vp, ci, vp, vp, vp, vp, vp, vp, vp, vp]),
        "qzo_compact_blocks": (ci, [vp, ci, vp, ci, ci, ci, ci, vp, vp, ci, vp, vp, ci, vp, vp, vp]),
        "qzo_shared_prefix_attention_workspace_bytes": (ci, [ci, ci, ci, ci, ci, ci, P(sz)]),
        "qzo_debug_prefix_path": (ci, [ci]),
        "qzo_shared_prefix_attention": (ci, [vp, ci, P(KvCacheDesc), vp, ci, ci, vp, vp, vp, vp, vp, ci, cf, vp, ci, ci, ci, vp, sz, vp, vp]),
        "qzo_copy_blocks": (ci, [P(KvCacheDesc), ci, vp, vp, ci, vp, vp]),
        "qzo_decode_groups": (ci, [vp, P(KvCacheDesc), vp, vp, vp, vp, ci, vp, ci, ci, vp, vp, vp, ci, vp]),
        "qzo_profile_gemms": (ci, [vp, ci]),
        "qzo_profile_read": (ci, [vp, P(i64), P(ctypes.c_double), P(ctypes.c_double)]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = res, args
    return lib


_lib = _load()


def _check(status, where):
    if status != QZO_OK:
        raise QzoError(status, where)


def _stream():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _ptr(t):
    return ctypes.c_void_p(t.data_ptr()) if t is not None else ctypes.c_void_p(0)


def _cuda(t, dtype=None):
    assert t.is_cuda and t.is_contiguous(), "expects a contiguous CUDA tensor"
    if dtype is not None:
        assert t.dtype == dtype, f"expects {dtype}, got {t.dtype}"
    return t


def qzo_launch_count():
    return int(_lib.qzo_launch_count())


def qzo_philox_words(seed, block_base, n_blocks, with_uniforms=True):
    """-> (int32 [n_blocks][4] holding the uint32 words, float32 [n_blocks][4] uniforms or None)."""
    words = torch.empty((n_blocks, 4), dtype=torch.int32, device="cuda")
    uni = torch.empty((n_blocks, 4), dtype=torch.float32, device="cuda") if with_uniforms else None
    _check(_lib.qzo_philox_words(seed, block_base, n_blocks, _ptr(words), _ptr(uni), _stream()), "qzo_philox_words")
    return words, uni


def qzo_normals(seed, index_base, count):
    z = torch.empty((count,), dtype=torch.float32, device="cuda")
    _check(_lib.qzo_normals(seed, index_base, count, _ptr(z), _stream()), "qzo_normals")
    return z


def qzo_quantize_int4(w):
    """float32 [K][N] -> (int32 [K/8][N] interchange words, bf16 [G][N] scales)."""
    _cuda(w, torch.float32)
    K, N = w.shape
    packed = torch.empty((K // 8, N), dtype=torch.int32, device=w.device)
    scales = torch.empty(((K + 127) // 128, N), dtype=torch.bfloat16, device=w.device)
    _check(_lib.qzo_quantize_int4(_ptr(w), K, N, _ptr(packed), _ptr(scales), _stream()), "qzo_quantize_int4")
    return packed, scales


def qzo_unpack_int4(packed, K, N):
    _cuda(packed, torch.int32)
    q = torch.empty((K, N), dtype=torch.int8, device=packed.device)
    _check(_lib.qzo_unpack_int4(_ptr(packed), K, N, _ptr(q), _stream()), "qzo_unpack_int4")
    return q


def qzo_repacked_bytes(K, N):
    out = ctypes.c_size_t(0)
    _check(_lib.qzo_repacked_bytes(K, N, ctypes.byref(out)), "qzo_repacked_bytes")
    return out.value


def qzo_repack_int4(packed, K, N):
    """interchange words -> kernel-layout bytes (uint8 tensor)."""
    _cuda(packed, torch.int32)
    nbytes = qzo_repacked_bytes(K, N)
    out = torch.empty((nbytes,), dtype=torch.uint8, device=packed.device)
    _check(_lib.qzo_repack_int4(_ptr(packed), K, N, _ptr(out), nbytes, _stream()), "qzo_repack_int4")
    return out


def qzo_unpack_kernel_layout(wq, K, N):
    _cuda(wq, torch.uint8)
    q = torch.empty((K, N), dtype=torch.int8, device=wq.device)
    _check(_lib.qzo_unpack_kernel_layout(_ptr(wq), K, N, _ptr(q), _stream()), "qzo_unpack_kernel_layout")
    return q


def qzo_gemm_workspace_bytes(M, K, N):
    out = ctypes.c_size_t(0)
    _check(_lib.qzo_gemm_workspace_bytes(M, K, N, ctypes.byref(out)), "qzo_gemm_workspace_bytes")
    return out.value


def qzo_perturbed_gemm(x, wq, scales, M, K, N, seed, scale_index_base, sign, eps, bias=None, y=None,
                       workspace=None, status=None):
    """Y = X W' with W' de-quantised from int4 and s' = s + sign*eps*z.  Returns bf16 [M][N]."""
    _cuda(x, torch.bfloat16), _cuda(wq, torch.uint8), _cuda(scales, torch.bfloat16)
    if y is None:
        y = torch.empty((M, N), dtype=torch.bfloat16, device=x.device)
    need = qzo_gemm_workspace_bytes(M, K, N)
    if workspace is None and need:
        workspace = torch.empty((need,), dtype=torch.uint8, device=x.device)
    ws_bytes = workspace.numel() if workspace is not None else 0
    _check(_lib.qzo_perturbed_gemm(_ptr(x), _ptr(wq), _ptr(scales), _ptr(bias), _ptr(y), M, K, N, seed,
                                   scale_index_base, sign, eps, _ptr(workspace), ws_bytes, _ptr(status), _stream()),
           "qzo_perturbed_gemm")
    return y


def qzo_perturbed_gemm_table16(x, codes_wq, scales, table16, M, K, N, seed, scale_index_base, sign, eps, bias=None, y=None,
                               workspace=None, status=None):
    """Y = X W' for 4-bit codes into a 16-entry table with one bf16 scale per block of 64 rows (NF4-style storage);
    codes_wq is qzo_repack_int4 of the codes packed like int4 nibbles; table16: 16 floats (any sequence)."""
    _cuda(x, torch.bfloat16), _cuda(codes_wq, torch.uint8), _cuda(scales, torch.bfloat16)
    assert scales.shape[0] == (K + 63) // 64
    if y is None:
        y = torch.empty((M, N), dtype=torch.bfloat16, device=x.device)
    need = qzo_gemm_workspace_bytes(M, K, N)
    if workspace is None and need:
        workspace = torch.empty((need,), dtype=torch.uint8, device=x.device)
    ws_bytes = workspace.numel() if workspace is not None else 0
    table = (ctypes.c_float * 16)(*[float(v) for v in table16])
    _check(_lib.qzo_perturbed_gemm_table16(_ptr(x), _ptr(codes_wq), _ptr(scales), table, _ptr(bias), _ptr(y), M, K, N, seed,
                                           scale_index_base, sign, eps, _ptr(workspace), ws_bytes, _ptr(status), _stream()),
           "qzo_perturbed_gemm_table16")
    return y


def qzo_perturbed_gemm_codebook16_channelwise(x, codes_wq, scales, table16, M, K, N, seed, scale_index_base, sign, eps,
                                              bias=None, y=None, workspace=None, status=None):
    """Y = X W' for 4-bit codes into a 16-entry table with ONE bf16 scale per output channel (scales: [N]);
    codes_wq as for qzo_perturbed_gemm_table16."""
    _cuda(x, torch.bfloat16), _cuda(codes_wq, torch.uint8), _cuda(scales, torch.bfloat16)
    assert scales.numel() == N
    if y is None:
        y = torch.empty((M, N), dtype=torch.bfloat16, device=x.device)
    need = qzo_gemm_workspace_bytes(M, K, N)
    if workspace is None and need:
        workspace = torch.empty((need,), dtype=torch.uint8, device=x.device)
    ws_bytes = workspace.numel() if workspace is not None else 0
    table = (ctypes.c_float * 16)(*[float(v) for v in table16])
    _check(_lib.qzo_perturbed_gemm_codebook16_channelwise(_ptr(x), _ptr(codes_wq), _ptr(scales), table, _ptr(bias), _ptr(y),
                                                          M, K, N, seed, scale_index_base, sign, eps, _ptr(workspace),
                                                          ws_bytes, _ptr(status), _stream()),
           "qzo_perturbed_gemm_codebook16_channelwise")
    return y


def qzo_debug_gemm_wait_expiry(x, wq, scales, y, M, K, N, skip_group, wait_limit_cycles, status):
    """Test entry: the GEMM with one group's copies withheld and a short wait limit; see include/qzo.h."""
    _cuda(x, torch.bfloat16), _cuda(wq, torch.uint8), _cuda(scales, torch.bfloat16), _cuda(y, torch.bfloat16)
    _check(_lib.qzo_debug_gemm_wait_expiry(_ptr(x), _ptr(wq), _ptr(scales), _ptr(y), M, K, N, skip_group, wait_limit_cycles,
                                           _ptr(status), _stream()), "qzo_debug_gemm_wait_expiry")


NOALLOC_SCRATCH_BYTES = 16 << 20


def qzo_perturbed_gemm_noalloc(x, wq, scales, y, M, K, N, seed, scale_index_base, sign, eps, bias=None, status=None):
    """qzo_perturbed_gemm for callers that cannot allocate: no workspace argument (the library's
    fixed scratch array is used) and the output tensor y is the caller's.  Nothing is allocated here."""
    _cuda(x, torch.bfloat16), _cuda(wq, torch.uint8), _cuda(scales, torch.bfloat16), _cuda(y, torch.bfloat16)
    _check(_lib.qzo_perturbed_gemm_noalloc(_ptr(x), _ptr(wq), _ptr(scales), _ptr(bias), _ptr(y), M, K, N, seed,
                                           scale_index_base, sign, eps, _ptr(status), _stream()),
           "qzo_perturbed_gemm_noalloc")
    return y


def qzo_update_scales_flat(scales, seed, index_base, lr, g, clip):
    _cuda(scales, torch.bfloat16)
    _check(_lib.qzo_update_scales_flat(_ptr(scales), scales.numel(), seed, index_base, lr, g, clip, _stream()),
           "qzo_update_scales_flat")
    return scales


# ---- serving operators ----

# limits of qzo_gemv_int4 (above, qzo_perturbed_gemm at sign 0) and qzo_assign_slots, for a program that divides its work by them
GEMV_MAX_ROWS = 16
MAX_REQUESTS = 4096
# of qzo_beam_select, and of the calls that read from the tables who holds a block
MAX_BEAMS = 32
MAX_POOL_BLOCKS = 524288


_BF16, _F32, _I32, _U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8
_raw_stream, _device_now = torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice

# A serving call takes a few microseconds on the device, so these wrappers look at every tensor once, in as few steps as
# possible.  Every tensor has to live on the current device: the launches go to that device's current stream.


def _ints(dev, n, *tensors):
    for t in tensors:
        assert t.dtype is _I32 and t.numel() >= n and t.is_contiguous() and t.get_device() == dev, \
            f"expects contiguous int32 of {n} entries on the current device"


def _heads(dev, t, what):
    """Row stride of a bf16 [T][heads][head_dim] tensor whose heads lie side by side (a view of a projection's rows)."""
    T, H, dh = t.shape
    ld, lh, one = t.stride()
    assert t.dtype is _BF16 and one == 1 and (lh == dh or H == 1) and t.get_device() == dev, \
        f"{what}: expects bf16 [T][heads][head_dim] on the current device, a row's heads side by side"
    return ld if T > 1 else H * dh


def _floats(dev, n, t, what):
    """Address of a contiguous float32 tensor of at least n entries, None for None."""
    if t is None:
        return None
    assert t.dtype is _F32 and t.numel() >= n and t.is_contiguous() and t.get_device() == dev, f"{what}: expects float32 [{n}] on the current device"
    return t.data_ptr()


def _status(dev, t):
    if t is None:
        return None
    _ints(dev, 1, t)
    return t.data_ptr()


def qzo_gemv_int4(x, wq, scales, K, N, bias=None, y=None):
    """y = x W for up to 16 rows: x bf16 [M][K] (any row stride that is a multiple of 8), wq from qzo_repack_int4, scales
    bf16 [ceil(K/128)][N], bias float32 [N] or None -> bf16 [M][N]."""
    dev = _device_now()
    M, k = x.shape
    ldx, one = x.stride()
    assert x.dtype is _BF16 and k == K and one == 1 and x.get_device() == dev, "x: expects bf16 [M][K] on the current device"
    assert wq.dtype is _U8 and wq.numel() >= (N + 127) // 128 * ((K + 63) // 64) * 4096 and wq.is_contiguous() and wq.get_device() == dev, \
        "wq: expects the uint8 of qzo_repack_int4 on the current device"
    assert scales.dtype is _BF16 and scales.numel() >= (K + 127) // 128 * N and scales.is_contiguous() and scales.get_device() == dev, \
        "scales: expects bf16 [ceil(K/128)][N] on the current device"
    if y is None:
        y, ldy = x.new_empty(M, N), N
    else:
        assert y.dtype is _BF16 and y.shape == (M, N) and y.stride(1) == 1 and y.get_device() == dev, "y: expects bf16 [M][N] on the current device"
        ldy = y.stride(0) if M > 1 else N
    rc = _lib.qzo_gemv_int4(x.data_ptr(), ldx if M > 1 else K, wq.data_ptr(), scales.data_ptr(),
                            None if bias is None else _floats(dev, N, bias, "bias"), y.data_ptr(), ldy, M, K, N, _raw_stream(dev))
    if rc:
        _check(rc, "qzo_gemv_int4")
    return y


class KvCache:
    """One layer's paged cache: k, v [n_blocks][n_kv_heads][block_size][head_dim], bf16 or float8_e4m3fn (value = code *
    scale).  Keeps the tensors alive."""

    def __init__(self, k, v, k_scale=1.0, v_scale=1.0):
        assert k.shape == v.shape and k.dim() == 4 and k.dtype == v.dtype, "k, v: [n_blocks][n_kv_heads][block_size][head_dim]"
        assert k.is_cuda and k.is_contiguous() and v.is_contiguous() and k.device == v.device, "expects contiguous CUDA tensors"
        kind = {torch.bfloat16: 0, torch.float8_e4m3fn: 4}[k.dtype]
        self.k, self.v, self.k_scale, self.v_scale = k, v, float(k_scale), float(v_scale)
        self.n_blocks, self.n_kv_heads, self.block_size, self.head_dim = k.shape
        self.device = k.get_device()
        self.desc = KvCacheDesc(k.data_ptr(), v.data_ptr(), kind, self.n_blocks, self.block_size, self.n_kv_heads, self.head_dim,
                                self.k_scale, self.v_scale)
        self._ref = ctypes.byref(self.desc)


def qzo_rope_table(max_pos, head_dim, theta=10000.0):
    """float32 [max_pos][head_dim/2][2]: cosine and sine of pos * theta**(-2i/head_dim)."""
    table = torch.empty((max_pos, head_dim // 2, 2), dtype=torch.float32, device="cuda")
    _check(_lib.qzo_rope_table(table.data_ptr(), max_pos, head_dim, theta, _raw_stream(table.get_device())), "qzo_rope_table")
    return table


def qzo_qk_norm_rope_cache(q, k, v, positions, slots, cache, q_gain=None, k_gain=None, norm_eps=1e-6, table=None, q_out=None,
                           status=None):
    """Head norms (where a gain is given), rotation (where a table is given) and cache write of T new rows; returns q_out
    bf16 [T][heads][head_dim].  q, k, v bf16 [T][heads][head_dim] views; positions, slots int32 [T], negative = padding."""
    dev = _device_now()
    T, H, dh = q.shape
    assert k.shape == v.shape == (T, cache.n_kv_heads, dh) and dh == cache.head_dim and cache.device == dev, \
        "k, v: expects [T][n_kv_heads][head_dim] of the cache, which is on the current device"
    ldq, ldk, ldv = _heads(dev, q, "q"), _heads(dev, k, "k"), _heads(dev, v, "v")
    if q_out is None:
        q_out, ldo = q.new_empty(T, H, dh), H * dh
    else:
        assert q_out.shape == (T, H, dh), "q_out: as q"
        ldo = _heads(dev, q_out, "q_out")
    _ints(dev, T, positions, slots)
    max_pos = 0
    if table is not None:
        max_pos, half, two = table.shape
        assert half == dh // 2 and two == 2, "table: [max_pos][head_dim/2][2]"
    rc = _lib.qzo_qk_norm_rope_cache(q.data_ptr(), ldq, k.data_ptr(), ldk, v.data_ptr(), ldv,
                                     None if q_gain is None else _floats(dev, dh, q_gain, "q_gain"),
                                     None if k_gain is None else _floats(dev, dh, k_gain, "k_gain"), norm_eps,
                                     None if table is None else _floats(dev, max_pos * dh, table, "table"), max_pos,
                                     positions.data_ptr(), slots.data_ptr(), q_out.data_ptr(), ldo, cache._ref, T, H,
                                     None if status is None else _status(dev, status), _raw_stream(dev))
    if rc:
        _check(rc, "qzo_qk_norm_rope_cache")
    return q_out


def qzo_paged_attention_workspace_bytes(R, n_heads, n_kv_heads, head_dim, max_len):
    out = ctypes.c_size_t(0)
    _check(_lib.qzo_paged_attention_workspace_bytes(R, n_heads, n_kv_heads, head_dim, max_len, ctypes.byref(out)),
           "qzo_paged_attention_workspace_bytes")
    return out.value


def qzo_paged_attention(q, cache, block_table, positions, row_seq=None, scale=None, out=None, workspace=None, status=None):
    """Attention of one new token per row over the paged cache: q bf16 [R][heads][head_dim], block_table int32
    [n_seqs][table_width], positions int32 [R] (negative = empty row, zeros), row_seq int32 [R] or None (row t is request t)
    -> bf16 [R][heads][head_dim]."""
    dev = _device_now()
    R, H, dh = q.shape
    ldq = _heads(dev, q, "q")
    assert dh == cache.head_dim and cache.device == dev, "q: expects the head_dim of the cache, which is on the current device"
    if out is None:
        out, ldo = q.new_empty(R, H, dh), H * dh
    else:
        assert out.shape == (R, H, dh), "out: as q"
        ldo = _heads(dev, out, "out")
    n_seqs, width = block_table.shape
    _ints(dev, 0, block_table)
    _ints(dev, R, positions)
    seqs = None
    if row_seq is not None:
        _ints(dev, R, row_seq)
        seqs = row_seq.data_ptr()
    if workspace is None:
        need = qzo_paged_attention_workspace_bytes(R, H, cache.n_kv_heads, dh, width * cache.block_size)
        workspace = q.new_empty(need, dtype=_U8) if need else None
    ws, ws_bytes = None, 0
    if workspace is not None:
        assert workspace.is_contiguous() and (workspace.get_device() == dev or workspace.numel() == 0), "workspace: contiguous, on the current device"
        ws, ws_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    rc = _lib.qzo_paged_attention(q.data_ptr(), ldq, cache._ref, block_table.data_ptr(), n_seqs, width, seqs, positions.data_ptr(),
                                  dh ** -0.5 if scale is None else scale, out.data_ptr(), ldo, R, H, ws, ws_bytes,
                                  None if status is None else _status(dev, status), _raw_stream(dev))
    if rc:
        _check(rc, "qzo_paged_attention")
    return out


def qzo_assign_slots(lens, new, block_table, free, free_count, block_size, max_rows, lens_out=None, free_count_out=None,
                     row_seq=None, positions=None, slots=None, status=None):
    """Blocks, rows and slots of a step (all int32): lens [B], new [B] (negative = finished), block_table [B][width], free =
    stack of free blocks, free_count [1].  Lengths and count are updated in place unless lens_out / free_count_out are
    given.  Returns (row_seq, positions, slots), each [max_rows], -1 behind the last row."""
    B, width = block_table.shape
    if lens_out is None:
        lens_out = lens
    if free_count_out is None:
        free_count_out = free_count
    dev = _device_now()
    _ints(dev, B, lens, new, lens_out)
    _ints(dev, 1, block_table, free, free_count, free_count_out)
    if row_seq is None and positions is None and slots is None:
        maps = lens.new_empty(3, max_rows)
        row_seq, positions, slots = maps.unbind()
        at = maps.data_ptr()
        rows_at = at, at + 4 * max_rows, at + 8 * max_rows
    else:
        assert row_seq is not None and positions is not None and slots is not None, "row_seq, positions, slots: all of them or none"
        _ints(dev, max_rows, row_seq, positions, slots)
        rows_at = row_seq.data_ptr(), positions.data_ptr(), slots.data_ptr()
    rc = _lib.qzo_assign_slots(lens.data_ptr(), new.data_ptr(), B, block_table.data_ptr(), width, block_size, free.data_ptr(),
                               free.numel(), free_count.data_ptr(), max_rows, *rows_at, lens_out.data_ptr(), free_count_out.data_ptr(),
                               None if status is None else _status(dev, status), _raw_stream(dev))
    if rc:
        _check(rc, "qzo_assign_slots")
    return row_seq, positions, slots


def qzo_shared_prefix_attention_workspace_bytes(R, n_groups, n_heads, n_kv_heads, head_dim, max_len):
    out = ctypes.c_size_t(0)
    _check(_lib.qzo_shared_prefix_attention_workspace_bytes(R, n_groups, n_heads, n_kv_heads, head_dim, max_len, ctypes.byref(out)),
           "qzo_shared_prefix_attention_workspace_bytes")
    return out.value


def qzo_debug_prefix_path(path):
    """For tests: 0 = as measured best, 1 = own tables, 2 = units of few queries, 3 = units of 128; see include/qzo.h."""
    _check(_lib.qzo_debug_prefix_path(path), "qzo_debug_prefix_path")


def qzo_shared_prefix_attention(q, cache, block_table, positions, group_rows, prefix_seq, prefix_len, row_seq=None, scale=None, out=None,
                                workspace=None, status=None):
    """qzo_paged_attention for groups of rows that share the beginning of their cache (int32): rows group_rows[i] .. group_rows[i + 1] - 1
    ([n + 1], ascending) have the first prefix_len[i] tokens of request prefix_seq[i] ([n] each) as the first tokens of their own
    requests.  The other arguments and the result are those of qzo_paged_attention."""
    dev = _device_now()
    R, H, dh = q.shape
    ldq = _heads(dev, q, "q")
    assert dh == cache.head_dim and cache.device == dev, "q: expects the head_dim of the cache, which is on the current device"
    if out is None:
        out, ldo = q.new_empty(R, H, dh), H * dh
    else:
        assert out.shape == (R, H, dh), "out: as q"
        ldo = _heads(dev, out, "out")
    n_seqs, width = block_table.shape
    n = prefix_seq.numel()
    _ints(dev, 0, block_table)
    _ints(dev, R, positions)
    _ints(dev, n, prefix_seq, prefix_len)
    _ints(dev, n + 1, group_rows)
    seqs = None
    if row_seq is not None:
        _ints(dev, R, row_seq)
        seqs = row_seq.data_ptr()
    if workspace is None:
        need = qzo_shared_prefix_attention_workspace_bytes(R, n, H, cache.n_kv_heads, dh, width * cache.block_size)
        workspace = q.new_empty(need, dtype=_U8) if need else None
    ws, ws_bytes = None, 0
    if workspace is not None:
        assert workspace.is_contiguous() and (workspace.get_device() == dev or workspace.numel() == 0), "workspace: contiguous, on the current device"
        ws, ws_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    rc = _lib.qzo_shared_prefix_attention(q.data_ptr(), ldq, cache._ref, block_table.data_ptr(), n_seqs, width, seqs, positions.data_ptr(),
                                          group_rows.data_ptr(), prefix_seq.data_ptr(), prefix_len.data_ptr(), n, dh ** -0.5 if scale is None else scale,
                                          out.data_ptr(), ldo, R, H, ws, ws_bytes, None if status is None else _status(dev, status), _raw_stream(dev))
    if rc:
        _check(rc, "qzo_shared_prefix_attention")
    return out


def qzo_beam_select_workspace_bytes(B, W, V):
    out = ctypes.c_size_t(0)
    _check(_lib.qzo_beam_select_workspace_bytes(B, W, V, ctypes.byref(out)), "qzo_beam_select_workspace_bytes")
    return out.value


def qzo_beam_select(logits, scores, rows=None, last_tokens=None, end_token=-1, lengths=None, length_power=0.0, parents=None, tokens=None,
                    scores_out=None, lengths_out=None, workspace=None, status=None):
    """The next beams of every request: logits float32 [rows][V] (any row stride), scores float32 [B][W] (-inf = no such beam), rows int32 [B][W]
    (the row of each beam, negative = none) or None (row b * W + w), last_tokens int32 [B][W] or None (beams that took end_token have
    ended), lengths int32 [B][W] or None -> (parents, tokens int32 [B][W], scores float32 [B][W], lengths int32 [B][W] or None), best first by
    score / length**length_power; -1, -1, -inf, 0 where there are no more candidates.  parents are numbers b * W + w."""
    dev = _device_now()
    B, W = scores.shape
    n_rows, V = logits.shape
    ldl, one = logits.stride()
    n = B * W
    assert logits.dtype is _F32 and (one == 1 or V == 1) and logits.get_device() == dev, "logits: expects float32 [rows][V] on the current device"
    scores_at = _floats(dev, n, scores, "scores")
    rows_at = last_at = lengths_at = lengths_out_at = None
    if rows is not None:
        _ints(dev, n, rows)
        rows_at = rows.data_ptr()
    if last_tokens is not None:
        _ints(dev, n, last_tokens)
        last_at = last_tokens.data_ptr()
    if lengths is not None:
        _ints(dev, n, lengths)
        lengths_at = lengths.data_ptr()
    if parents is None and tokens is None and lengths_out is None:       # one allocation for what is int32
        made = scores.new_empty(2 if lengths is None else 3, B, W, dtype=_I32)
        parents, tokens, *rest = made.unbind()
        at = made.data_ptr()
        parents_at, tokens_at = at, at + 4 * n
        if rest:
            lengths_out, lengths_out_at = rest[0], at + 8 * n
    else:
        parents = scores.new_empty(B, W, dtype=_I32) if parents is None else parents
        tokens = scores.new_empty(B, W, dtype=_I32) if tokens is None else tokens
        _ints(dev, n, parents, tokens)
        parents_at, tokens_at = parents.data_ptr(), tokens.data_ptr()
        if lengths is not None or lengths_out is not None:
            lengths_out = scores.new_empty(B, W, dtype=_I32) if lengths_out is None else lengths_out
            _ints(dev, n, lengths_out)
            lengths_out_at = lengths_out.data_ptr()
    if scores_out is None:
        scores_out = scores.new_empty(B, W)
        scores_out_at = scores_out.data_ptr()
    else:
        scores_out_at = _floats(dev, n, scores_out, "scores_out")
    if workspace is None:
        workspace = scores.new_empty(qzo_beam_select_workspace_bytes(B, W, V), dtype=_U8)
    assert workspace.is_contiguous() and workspace.get_device() == dev, "workspace: contiguous, on the current device"
    rc = _lib.qzo_beam_select(logits.data_ptr(), ldl if n_rows > 1 else V, n_rows, rows_at, scores_at, last_at, end_token, lengths_at, length_power, B, W, V,
                              parents_at, tokens_at, scores_out_at, lengths_out_at, workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                              None if status is None else _status(dev, status), _raw_stream(dev))
    if rc:
        _check(rc, "qzo_beam_select")
    return parents, tokens, scores_out, lengths_out


def qzo_fork_requests(lens, parents, block_table, free, free_count, block_size, n_blocks, table_out=None, lens_out=None, free_count_out=None,
                      copies=None, copy_count=None, status=None):
    """Requests go on as copies of one another (all int32): lens [B], parents [B] (any shape; negative = the request ends), block_table [B][width],
    free = stack of free blocks, free_count [1], n_blocks = blocks of the pool.  Lengths and count are new tensors unless given (they may be the
    inputs); the table is always another one.  -> (table_out, lens_out, free_count_out, copies [B][3], copy_count [1]); the copies are for
    qzo_copy_blocks."""
    dev = _device_now()
    B, width = block_table.shape
    _ints(dev, B, lens, parents)
    _ints(dev, 1, block_table, free, free_count)
    if table_out is None:
        table_out = torch.empty_like(block_table)
    else:
        assert table_out.shape == block_table.shape, "table_out: as block_table"
        _ints(dev, 1, table_out)
    if lens_out is None and free_count_out is None and copies is None and copy_count is None:       # one allocation for all of them
        made = lens.new_empty(4 * B + 2)
        lens_out, copies, free_count_out, copy_count = made.split_with_sizes((B, 3 * B, 1, 1))
        copies = copies.view(B, 3)
        at = made.data_ptr()
        lens_at, copies_at, free_count_at, count_at = at, at + 4 * B, at + 16 * B, at + 16 * B + 4
    else:
        lens_out = lens.new_empty(B) if lens_out is None else lens_out
        free_count_out = lens.new_empty(1) if free_count_out is None else free_count_out
        copies = lens.new_empty(B, 3) if copies is None else copies
        copy_count = lens.new_empty(1) if copy_count is None else copy_count
        _ints(dev, B, lens_out)
        _ints(dev, 1, free_count_out, copy_count)
        _ints(dev, 3 * B, copies)
        lens_at, copies_at, free_count_at, count_at = lens_out.data_ptr(), copies.data_ptr(), free_count_out.data_ptr(), copy_count.data_ptr()
    rc = _lib.qzo_fork_requests(lens.data_ptr(), parents.data_ptr(), B, block_table.data_ptr(), width, block_size, n_blocks, free.data_ptr(), free.numel(),
                                free_count.data_ptr(), lens_at, table_out.data_ptr(), free_count_at, copies_at, count_at,
                                None if status is None else _status(dev, status), _raw_stream(dev))
    if rc:
        _check(rc, "qzo_fork_requests")
    return table_out, lens_out, free_count_out, copies, copy_count


def qzo_compact_blocks(lens, block_table, free, block_size, n_blocks, keep, free_count=None, table_out=None, copies=None, copy_count=None, status=None):
    """The blocks that requests hold move to the front of the pool, which then has `keep` blocks (all int32): lens [B], block_table [B][width] (written in
    place unless table_out is given), free = the stack of free blocks, written anew, free_count [1] = its count, written too ->
    (table, free_count, copies [n][3], copy_count [1]); the copies are for qzo_copy_blocks."""
    dev = _device_now()
    B, width = block_table.shape
    if table_out is None:
        table_out = block_table
    assert table_out.shape == block_table.shape, "table_out: as block_table"
    if free_count is None:
        free_count = lens.new_full((1,), -1)
    if copies is None:
        copies = lens.new_empty(n_blocks, 3)
    if copy_count is None:
        copy_count = lens.new_empty(1)
    _ints(dev, B, lens)
    _ints(dev, 1, block_table, table_out, free, free_count, copies, copy_count)
    rc = _lib.qzo_compact_blocks(lens.data_ptr(), B, block_table.data_ptr(), width, block_size, n_blocks, keep, table_out.data_ptr(), free.data_ptr(),
                                 free.numel(), free_count.data_ptr(), copies.data_ptr(), copies.numel() // 3, copy_count.data_ptr(),
                                 None if status is None else _status(dev, status), _raw_stream(dev))
    if rc:
        _check(rc, "qzo_compact_blocks")
    return table_out, free_count, copies, copy_count


def qzo_copy_blocks(caches, copies, copy_count, status=None):
    """The listed copies of pages (int32 [n][3]: from, to, tokens; copy_count int32 [1]: how many) in every one of the caches (list of KvCache of
    one shape and type, as the layers of a model)."""
    dev = _device_now()
    assert len(caches) > 0, "caches: expects at least one"
    for c in caches:
        assert c.device == dev, "caches: expects KvCache on the current device"
    _ints(dev, 1, copies, copy_count)
    rc = _lib.qzo_copy_blocks((KvCacheDesc * len(caches))(*[c.desc for c in caches]), len(caches), copies.data_ptr(), copy_count.data_ptr(),
                              copies.numel() // 3, None if status is None else _status(dev, status), _raw_stream(dev))
    if rc:
        _check(rc, "qzo_copy_blocks")


def make_desc(cfg):
    return ModelDesc(ARCH[cfg["arch"]], cfg["n_layers"], cfg["d_model"], cfg["n_heads"], cfg["d_ffn"],
                     cfg["vocab"], cfg["max_seq"], 128, cfg["norm_eps"], cfg["rope_theta"])


def qzo_num_scales(cfg):
    flat, train = ctypes.c_int64(0), ctypes.c_int64(0)
    d = make_desc(cfg)
    _check(_lib.qzo_num_scales(ctypes.byref(d), ctypes.byref(flat), ctypes.byref(train)), "qzo_num_scales")
    return flat.value, train.value


def qzo_scale_layout(cfg, layer, linear):
    base, G, N = ctypes.c_int64(0), ctypes.c_int(0), ctypes.c_int(0)
    d = make_desc(cfg)
    _check(_lib.qzo_scale_layout(ctypes.byref(d), layer, linear, ctypes.byref(base), ctypes.byref(G),
                                 ctypes.byref(N)), "qzo_scale_layout")
    return base.value, G.value, N.value


def qzo_workspace_bytes(cfg, max_tokens):
    out = ctypes.c_size_t(0)
    d = make_desc(cfg)
    _check(_lib.qzo_workspace_bytes(ctypes.byref(d), max_tokens, ctypes.byref(out)), "qzo_workspace_bytes")
    return out.value


class Model:
    """Owns the device tensors of a model (allocated by torch) and the library handle.

    tensors: dict name -> CUDA tensor with the names qzo_init_model documents; "*.qweight"
    tensors are int32 holding the interchange words and may be dropped after construction.
    """

    def __init__(self, cfg, tensors, max_tokens):
        self.cfg = dict(cfg)
        self.max_tokens = max_tokens
        self.desc = make_desc(cfg)
        self.scales = tensors["scales"]
        self._keep = {k: v for k, v in tensors.items() if not k.endswith(".qweight")}
        nbytes = qzo_workspace_bytes(cfg, max_tokens)
        self.workspace = torch.empty((nbytes,), dtype=torch.uint8, device="cuda")
        arr = (Tensor * len(tensors))()
        for i, (name, t) in enumerate(tensors.items()):
            _cuda(t)
            dt = DTYPE_U32 if name.endswith(".qweight") else DTYPE[t.dtype]
            shape = (t.shape[0], t.shape[1] if t.dim() > 1 else 1)
            arr[i] = Tensor(name.encode(), t.data_ptr(), dt, (ctypes.c_int64 * 2)(*shape))
        handle = ctypes.c_void_p(0)
        self.stream = torch.cuda.current_stream()
        _check(_lib.qzo_init_model(ctypes.byref(self.desc), arr, len(tensors), _ptr(self.workspace), nbytes,
                                   max_tokens, ctypes.c_void_p(self.stream.cuda_stream), ctypes.byref(handle)),
               "qzo_init_model")
        self.handle = handle
        self.stream.synchronize()
        self._loss = torch.zeros((2,), dtype=torch.float32, device="cuda")

    def close(self):
        if self.handle:
            _lib.qzo_free_model(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def qzo_forward_loss(self, tokens, labels, seed, sign, eps, loss_out=None):
        _cuda(tokens, torch.int32), _cuda(labels, torch.int32)
        B, S = tokens.shape
        out = self._loss[:1] if loss_out is None else loss_out
        _check(_lib.qzo_forward_loss(self.handle, _ptr(tokens), _ptr(labels), B, S, seed, sign, eps, _ptr(out)),
               "qzo_forward_loss")
        return out

    def _decode_args(self, caches, R, logits):
        """Checks what the two decode calls share -> (device, cache descriptions, logits)."""
        dev = _device_now()
        assert _raw_stream(dev) == self.stream.cuda_stream, "expects the model's stream to be the current one"
        assert len(caches) == self.cfg["n_layers"] and all(c.device == dev for c in caches), "expects one cache per layer, on the current device"
        if logits is None:
            logits = torch.empty((R, self.cfg["vocab"]), dtype=torch.float32, device="cuda")
        assert logits.shape == (R, self.cfg["vocab"]), "logits: float32 [R][vocab]"
        _floats(dev, R, logits, "logits")
        return dev, (KvCacheDesc * len(caches))(*(c.desc for c in caches)), logits

    def qzo_decode(self, caches, tokens, row_seq, positions, slots, block_table, logits=None):
        """One answering step of R rows over the layers' caches (list of KvCache, one per layer); tokens, row_seq, positions,
        slots int32 [R], block_table int32 [n_seqs][width] -> float32 logits [R][vocab].  Runs on the stream the model was made on,
        which has to be the current one."""
        R = tokens.numel()
        dev, descs, logits = self._decode_args(caches, R, logits)
        _ints(dev, R, tokens, row_seq, positions, slots)
        n_seqs, width = block_table.shape
        _ints(dev, 1, block_table)
        _check(_lib.qzo_decode(self.handle, descs, tokens.data_ptr(), row_seq.data_ptr(), positions.data_ptr(), slots.data_ptr(), R,
                               block_table.data_ptr(), n_seqs, width, logits.data_ptr()), "qzo_decode")
        return logits

    def qzo_decode_groups(self, caches, tokens, row_seq, positions, slots, block_table, group_rows, prefix_seq, prefix_len, logits=None):
        """qzo_decode for rows that share the beginning of their caches (int32): rows group_rows[i] .. group_rows[i + 1] - 1 ([n + 1]) have the
        first prefix_len[i] tokens of request prefix_seq[i] ([n] each) as the first tokens of their own requests."""
        R, n = tokens.numel(), prefix_seq.numel()
        dev, descs, logits = self._decode_args(caches, R, logits)
        _ints(dev, R, tokens, row_seq, positions, slots)
        _ints(dev, n, prefix_seq, prefix_len)
        _ints(dev, n + 1, group_rows)
        n_seqs, width = block_table.shape
        _ints(dev, 1, block_table)
        _check(_lib.qzo_decode_groups(self.handle, descs, tokens.data_ptr(), row_seq.data_ptr(), positions.data_ptr(), slots.data_ptr(), R,
                                      block_table.data_ptr(), n_seqs, width, group_rows.data_ptr(), prefix_seq.data_ptr(), prefix_len.data_ptr(), n,
                                      logits.data_ptr()), "qzo_decode_groups")
        return logits

    def qzo_decode_requests(self, caches, tokens, lens, new, block_table, free, free_count, logits=None, status=None):
        """qzo_assign_slots (in place) and qzo_decode of its rows in one call: tokens int32 [R], the new tokens request by
        request -> (float32 logits [R][vocab], int32 [3][R]: row_seq, positions, slots)."""
        R = tokens.numel()
        dev, descs, logits = self._decode_args(caches, R, logits)
        B, width = block_table.shape
        _ints(dev, B, lens, new)
        _ints(dev, 1, tokens, block_table, free, free_count)
        maps = lens.new_empty(3, R)
        _check(_lib.qzo_decode_requests(self.handle, descs, tokens.data_ptr(), lens.data_ptr(), new.data_ptr(), B, block_table.data_ptr(),
                                        width, free.data_ptr(), free.numel(), free_count.data_ptr(), R, maps.data_ptr(),
                                        logits.data_ptr(), _status(dev, status)), "qzo_decode_requests")
        return logits, maps

    def qzo_update_scales(self, seed, lr, g, clip):
        _check(_lib.qzo_update_scales(self.handle, seed, lr, g, clip), "qzo_update_scales")

    def qzo_step(self, tokens, labels, seed, eps, lr, clip, read_back=True):
        _cuda(tokens, torch.int32), _cuda(labels, torch.int32)
        B, S = tokens.shape
        out = (ctypes.c_float * 4)() if read_back else None
        _check(_lib.qzo_step(self.handle, _ptr(tokens), _ptr(labels), B, S, seed, eps, lr, clip, out), "qzo_step")
        return tuple(out) if read_back else None

    def qzo_step_begin(self, tokens, labels, seed, eps, sums=None):
        """-> float32 CUDA tensor [4]: sum of token losses (+), the same (-), kept tokens (+), (-)."""
        _cuda(tokens, torch.int32), _cuda(labels, torch.int32)
        B, S = tokens.shape
        if sums is None:
            sums = torch.empty((4,), dtype=torch.float32, device="cuda")
        _check(_lib.qzo_step_begin(self.handle, _ptr(tokens), _ptr(labels), B, S, seed, eps, _ptr(sums)),
               "qzo_step_begin")
        return sums

    def qzo_step_finish(self, sums, seed, eps, lr, clip, read_back=True):
        _cuda(sums, torch.float32)
        out = (ctypes.c_float * 4)() if read_back else None
        _check(_lib.qzo_step_finish(self.handle, _ptr(sums), seed, eps, lr, clip, out), "qzo_step_finish")
        return tuple(out) if read_back else None

    def _linear_bytes(self, linear_id):
        if linear_id == -1:
            return self.scales.numel() * 2
        n_lin = 7 if self.cfg["arch"] == "llama" else 6
        _, G, N = qzo_scale_layout(self.cfg, linear_id // n_lin, linear_id % n_lin)
        return G * N * 2

    def qzo_get_scales(self, linear_id, out=None):
        """Copy of one linear's scales (bf16, flat [G*N]) or of the whole flat buffer (linear_id = -1)."""
        if out is None:
            out = torch.empty((self._linear_bytes(linear_id) // 2,), dtype=torch.bfloat16, device="cuda")
        _check(_lib.qzo_get_scales(self.handle, linear_id, _ptr(out), out.numel() * 2), "qzo_get_scales")
        return out

    def qzo_set_scales(self, linear_id, values):
        _cuda(values, torch.bfloat16)
        _check(_lib.qzo_set_scales(self.handle, linear_id, _ptr(values), values.numel() * 2), "qzo_set_scales")

    def qzo_enable_joint_spsa(self, lr_dense, on=True):
        """Joint mode: embed, lm_head and the norm vectors are perturbed and updated too (plain SPSA)."""
        if not on:
            _check(_lib.qzo_enable_joint_spsa(self.handle, None, 0, 0.0), "qzo_enable_joint_spsa")
            return
        need = ctypes.c_size_t(0)
        _check(_lib.qzo_joint_workspace_bytes(ctypes.byref(self.desc), ctypes.byref(need)), "qzo_joint_workspace_bytes")
        self._joint_ws = torch.empty((need.value,), dtype=torch.uint8, device="cuda")
        _check(_lib.qzo_enable_joint_spsa(self.handle, _ptr(self._joint_ws), need.value, lr_dense), "qzo_enable_joint_spsa")

    def tensor(self, name):
        """The caller-owned device tensor bound under `name` at construction (e.g. "embed", "L0.norm1_w")."""
        return self._keep[name]

    def qzo_debug_set_status(self, value):
        _check(_lib.qzo_debug_set_status(self.handle, value), "qzo_debug_set_status")

    def qzo_use_recorded_steps(self, on):
        _check(_lib.qzo_use_recorded_steps(self.handle, 1 if on else 0), "qzo_use_recorded_steps")

    def qzo_recorded_step_count(self):
        n = ctypes.c_int(0)
        _check(_lib.qzo_recorded_step_count(self.handle, ctypes.byref(n)), "qzo_recorded_step_count")
        return n.value

    def qzo_step_host(self, tokens_host, labels_host, seed, eps, lr, clip):
        assert not tokens_host.is_cuda and tokens_host.dtype == torch.int32 and tokens_host.is_contiguous()
        B, S = tokens_host.shape
        out = (ctypes.c_float * 4)()
        _check(_lib.qzo_step_host(self.handle, ctypes.c_void_p(tokens_host.data_ptr()),
                                  ctypes.c_void_p(labels_host.data_ptr()), B, S, seed, eps, lr, clip, out),
               "qzo_step_host")
        return tuple(out)

    def qzo_debug_set_capture(self, layer):
        _check(_lib.qzo_debug_set_capture(self.handle, layer), "qzo_debug_set_capture")

    def qzo_debug_layer_output(self, layer, which, T):
        if which == 0:
            out = torch.empty((T, self.cfg["d_model"]), dtype=torch.bfloat16, device="cuda")
        else:
            out = torch.empty((T, self.cfg["vocab"]), dtype=torch.float32, device="cuda")
        _check(_lib.qzo_debug_layer_output(self.handle, layer, which, _ptr(out), out.numel() * out.element_size()),
               "qzo_debug_layer_output")
        return out

    def qzo_device_status(self):
        st = ctypes.c_int(0)
        rc = _lib.qzo_device_status(self.handle, ctypes.byref(st))
        if rc not in (QZO_OK, ERR_DEVICE_TIMEOUT, ERR_BAD_ARG):
            _check(rc, "qzo_device_status")
        return st.value

    def qzo_profile_gemms(self, max_launches):
        _check(_lib.qzo_profile_gemms(self.handle, max_launches), "qzo_profile_gemms")

    def qzo_profile_read(self):
        """-> (launches, total_ms, total_flops) of the bracketed GEMM launches since the last read."""
        n, ms, fl = ctypes.c_int64(0), ctypes.c_double(0), ctypes.c_double(0)
        _check(_lib.qzo_profile_read(self.handle, ctypes.byref(n), ctypes.byref(ms), ctypes.byref(fl)),
               "qzo_profile_read")
        return n.value, ms.value, fl.value

    def scales_of(self, layer, linear):
        """View of one linear's scales [G][N] inside the flat buffer."""
        base, G, N = qzo_scale_layout(self.cfg, layer, linear)
        return self.scales[base:base + G * N].view(G, N)


def build_model_from_raw(raw, max_tokens, quantized=None):
    """Quantise (library kernel) and upload the seeded raw tensors of `inputs.raw_model_tensors`.

    quantized: optional dict (layer, name) -> (int32 words [K/8][N], bf16 scales [G][N]) to use instead
    of quantising here.  Returns Model.
    """
    from .inputs import linear_shapes
    cfg = raw["cfg"]
    flat, _ = qzo_num_scales(cfg)
    scales = torch.zeros((flat,), dtype=torch.bfloat16, device="cuda")
    t = {"embed": raw["embed"].cuda(), "lm_head": raw["lm_head"].cuda(),
         "final_norm_w": raw["final_norm_w"].float().cuda(), "scales": scales}
    if cfg["arch"] == "opt":
        t["pos_embed"] = raw["pos_embed"].cuda()
        t["final_norm_b"] = raw["final_norm_b"].float().cuda()
    for li, layer in enumerate(raw["layers"]):
        for k in ("norm1_w", "norm2_w", "norm1_b", "norm2_b"):
            if k in layer:
                t[f"L{li}.{k}"] = layer[k].float().cuda()
        for idx, (name, K, N) in enumerate(linear_shapes(cfg)):
            ent = layer["lin"][name]
            if quantized is not None:
                words, s = quantized[(li, name)]
                words, s = words.cuda(), s.cuda()
            else:
                words, s = qzo_quantize_int4(ent["w"].cuda().contiguous())
            base, G, Nn = qzo_scale_layout(cfg, li, idx)
            scales[base:base + G * Nn] = s.reshape(-1)
            t[f"L{li}.{name}.qweight"] = words
            if "bias" in ent:
                t[f"L{li}.{name}.bias"] = ent["bias"].float().cuda()
    return Model(cfg, t, max_tokens)


def build_random_model_gpu(cfg, max_tokens, seed=1000):
    """Random-init int4 model generated and quantised tensor by tensor on the device
    (fp32 N(0, 0.02) weights -> library quantiser), so that no full-precision copy of the
    model ever exists.  Used by the benchmark for the large configurations."""
    from .inputs import linear_shapes, normal_fp32
    flat, _ = qzo_num_scales(cfg)
    d, V = cfg["d_model"], cfg["vocab"]
    sid = [int(seed)]

    def nxt():
        sid[0] += 1
        return sid[0]

    scales = torch.zeros((flat,), dtype=torch.bfloat16, device="cuda")
    t = {"embed": normal_fp32((V, d), 0.02, nxt(), "cuda").bfloat16(),
         "lm_head": normal_fp32((V, d), 0.02, nxt(), "cuda").bfloat16(),
         "final_norm_w": torch.ones(d, device="cuda"), "scales": scales}
    opt = cfg["arch"] == "opt"
    if opt:
        t["pos_embed"] = normal_fp32((cfg["max_seq"], d), 0.02, nxt(), "cuda").bfloat16()
        t["final_norm_b"] = torch.zeros(d, device="cuda")
    for li in range(cfg["n_layers"]):
        t[f"L{li}.norm1_w"] = torch.ones(d, device="cuda")
        t[f"L{li}.norm2_w"] = torch.ones(d, device="cuda")
        if opt:
            t[f"L{li}.norm1_b"] = torch.zeros(d, device="cuda")
            t[f"L{li}.norm2_b"] = torch.zeros(d, device="cuda")
        for idx, (name, K, N) in enumerate(linear_shapes(cfg)):
            w = normal_fp32((K, N), 0.02, nxt(), "cuda")
            words, s = qzo_quantize_int4(w)
            del w
            base, G, Nn = qzo_scale_layout(cfg, li, idx)
            scales[base:base + G * Nn] = s.reshape(-1)
            t[f"L{li}.{name}.qweight"] = words
            if opt:
                t[f"L{li}.{name}.bias"] = normal_fp32((N,), 0.02, nxt(), "cuda")
    m = Model(cfg, t, max_tokens)
    del t
    torch.cuda.empty_cache()
    return m
