"""ctypes binding of libqspec.so: same names as the C ABI (include/qspec.h),
argument marshalling only.  Tensors are torch CUDA tensors; torch provides the
device memory and the stream, every computation runs in the HIP library.
There is no fallback: a missing library raises."""
from __future__ import annotations

import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libqspec.so")
GROUP = 128

OK, ERR_NULL, ERR_SHAPE, ERR_ALIGN, ERR_WORKSPACE, ERR_HIP, ERR_UNSUPPORTED = range(7)

EXPORTS = (
    "qspec_status_string", "qspec_version", "qspec_packed_weight_bytes", "qspec_workspace_bytes",
    "qspec_pack_weights", "qspec_unpack_weights", "qspec_quant_act", "qspec_gemm_w4a4",
    "qspec_gemm_w4a16", "qspec_gemm_w4a4_partials", "qspec_describe_kernel",
    "qspec_accept_workspace_bytes", "qspec_greedy_accept", "qspec_kv_overwrite",
    "qspec_rmsnorm_quant", "qspec_silu_mul_quant", "qspec_hadamard_quant",
    "qspec_reorder_quant", "qspec_debug_set_plan",
    "qspec_gemm_w4a16_noalloc", "qspec_mlp_draft", "qspec_mlp_draft_workspace_bytes",
    "qspec_w4a4_takes_wide", "qspec_quant_act_wide", "qspec_gemm_w4a4_wide",
    "qspec_kv4_page_bytes", "qspec_rope_kv4_append", "qspec_kv4_read", "qspec_attn_kv4_workspace_bytes", "qspec_attn_kv4",
    "qspec_sample_workspace_bytes", "qspec_sample",
    "qspec_attn_kv4_shared_workspace_bytes", "qspec_attn_kv4_shared", "qspec_kv4_bounds_bytes", "qspec_kv4_bounds", "qspec_kv4_bounds_read",
    "qspec_kv4_select_workspace_bytes", "qspec_kv4_select", "qspec_attn_kv4_blocks_workspace_bytes", "qspec_attn_kv4_blocks",
)


class QSpecError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


_lib = None


def lib() -> ctypes.CDLL:
    """Load libqspec.so (built by `python -m paper_2410_11305_amd.build`)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2410_11305_amd.build` "
            "(there is no CPU fallback)")
    L = ctypes.CDLL(LIB_PATH)
    vp, ci, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
    L.qspec_status_string.restype = ctypes.c_char_p
    L.qspec_status_string.argtypes = [ci]
    L.qspec_version.restype = ci
    L.qspec_version.argtypes = []
    L.qspec_packed_weight_bytes.restype = sz
    L.qspec_packed_weight_bytes.argtypes = [ci, ci, ci]
    L.qspec_workspace_bytes.restype = sz
    L.qspec_workspace_bytes.argtypes = [ci, ci, ci, ci]
    L.qspec_pack_weights.restype = ci
    L.qspec_pack_weights.argtypes = [vp, vp, ci, ci, ci, vp, vp]
    L.qspec_w4a4_takes_wide.restype = ci
    L.qspec_w4a4_takes_wide.argtypes = [ci, ci, ci, ci]
    L.qspec_quant_act_wide.restype = ci
    L.qspec_quant_act_wide.argtypes = [vp, ci, ci, ci, vp, vp, vp]
    L.qspec_gemm_w4a4_wide.restype = ci
    L.qspec_gemm_w4a4_wide.argtypes = [vp, vp, vp, ci, ci, ci, ci, vp, vp, sz, vp]
    L.qspec_unpack_weights.restype = ci
    L.qspec_unpack_weights.argtypes = [vp, ci, ci, ci, vp, vp, vp]
    L.qspec_quant_act.restype = ci
    L.qspec_quant_act.argtypes = [vp, ci, ci, ci, vp, vp, vp]
    L.qspec_gemm_w4a4.restype = ci
    L.qspec_gemm_w4a4.argtypes = [vp, vp, vp, ci, ci, ci, ci, vp, vp, sz, vp]
    L.qspec_gemm_w4a16.restype = ci
    L.qspec_gemm_w4a16.argtypes = [vp, vp, ci, ci, ci, ci, vp, vp, sz, vp]
    L.qspec_gemm_w4a4_partials.restype = ci
    L.qspec_gemm_w4a4_partials.argtypes = [vp, vp, ci, ci, ci, ci, ci, ci, vp, vp]
    L.qspec_describe_kernel.restype = ci
    L.qspec_describe_kernel.argtypes = [ci, ci, ci, ci, ci, ctypes.c_char_p, sz]
    L.qspec_accept_workspace_bytes.restype = sz
    L.qspec_accept_workspace_bytes.argtypes = [ci, ci, ci]
    L.qspec_greedy_accept.restype = ci
    L.qspec_greedy_accept.argtypes = [vp, vp, ci, ci, ci, vp, vp, vp, sz, vp]
    L.qspec_kv_overwrite.restype = ci
    L.qspec_kv_overwrite.argtypes = [vp, vp, vp, ci, ci, ci, ci, vp, vp]
    L.qspec_rmsnorm_quant.restype = ci
    L.qspec_rmsnorm_quant.argtypes = [vp, vp, ctypes.c_float, ci, ci, ci, ci, vp, vp, vp, vp]
    L.qspec_silu_mul_quant.restype = ci
    L.qspec_silu_mul_quant.argtypes = [vp, ci, ci, ci, ci, vp, vp, vp, vp]
    L.qspec_hadamard_quant.restype = ci
    L.qspec_hadamard_quant.argtypes = [vp, ci, ci, ci, vp, vp, vp, vp]
    L.qspec_reorder_quant.restype = ci
    L.qspec_reorder_quant.argtypes = [vp, vp, ci, ci, ci, ci, vp, vp, vp, vp]
    L.qspec_gemm_w4a16_noalloc.restype = ci
    L.qspec_gemm_w4a16_noalloc.argtypes = [vp, vp, ci, ci, ci, ci, vp, vp]
    L.qspec_mlp_draft_workspace_bytes.restype = sz
    L.qspec_mlp_draft_workspace_bytes.argtypes = [ci, ci, ci, ci]
    L.qspec_mlp_draft.restype = ci
    L.qspec_mlp_draft.argtypes = [vp, vp, vp, vp, ci, ci, ci, ci, vp, vp, vp, vp, vp, sz, vp, vp]
    L.qspec_kv4_page_bytes.restype = sz
    L.qspec_kv4_page_bytes.argtypes = [ci, ci, ci]
    L.qspec_rope_kv4_append.restype = ci
    L.qspec_rope_kv4_append.argtypes = [vp, vp, vp, vp, ci, ci, ci, ci, ci, ci, ci, ctypes.c_float, ci, ci, ci, vp, vp, vp]
    L.qspec_kv4_read.restype = ci
    L.qspec_kv4_read.argtypes = [vp, vp, vp, ci, ci, ci, ci, ci, ci, ci, vp, vp, vp]
    L.qspec_attn_kv4_workspace_bytes.restype = sz
    L.qspec_attn_kv4_workspace_bytes.argtypes = [ci, ci, ci, ci, ci]
    L.qspec_attn_kv4.restype = ci
    L.qspec_attn_kv4.argtypes = [vp, vp, vp, vp, ci, ci, ci, ci, ci, ci, ci, ci, ctypes.c_float, ci, ci, vp, vp, sz, vp]
    L.qspec_attn_kv4_shared_workspace_bytes.restype = sz
    L.qspec_attn_kv4_shared_workspace_bytes.argtypes = [ci, ci, ci, ci, ci, ci]
    L.qspec_attn_kv4_shared.restype = ci
    L.qspec_attn_kv4_shared.argtypes = [vp, vp, vp, vp, vp, ci, ci, ci, ci, ci, ci, ci, ci, ci, ctypes.c_float, vp, vp, sz, vp]
    L.qspec_kv4_bounds_bytes.restype = sz
    L.qspec_kv4_bounds_bytes.argtypes = [ci, ci]
    L.qspec_kv4_bounds.restype = ci
    L.qspec_kv4_bounds.argtypes = [vp, vp, vp, ci, ci, ci, ci, ci, ci, ci, vp, vp]
    L.qspec_kv4_bounds_read.restype = ci
    L.qspec_kv4_bounds_read.argtypes = [vp, vp, vp, ci, ci, ci, ci, ci, ci, ci, vp, vp, vp]
    L.qspec_kv4_select_workspace_bytes.restype = sz
    L.qspec_kv4_select_workspace_bytes.argtypes = [ci, ci, ci, ci, ci]
    L.qspec_kv4_select.restype = ci
    L.qspec_kv4_select.argtypes = [vp, vp, vp, vp, ci, ci, ci, ci, ci, ci, ci, ci, ci, ci, ci, vp, vp, sz, vp]
    L.qspec_attn_kv4_blocks_workspace_bytes.restype = sz
    L.qspec_attn_kv4_blocks_workspace_bytes.argtypes = [ci, ci, ci, ci, ci]
    L.qspec_attn_kv4_blocks.restype = ci
    L.qspec_attn_kv4_blocks.argtypes = [vp, vp, vp, vp, vp, ci, ci, ci, ci, ci, ci, ci, ci, ci, ctypes.c_float, vp, vp, sz, vp]
    L.qspec_sample_workspace_bytes.restype = sz
    L.qspec_sample_workspace_bytes.argtypes = [ci, ci, ci]
    L.qspec_sample.restype = ci
    L.qspec_sample.argtypes = [vp, vp, vp, vp, vp, vp, vp, ci, ci, ci, vp, vp, vp, sz, vp]
    L.qspec_debug_set_plan.restype = ci
    L.qspec_debug_set_plan.argtypes = [ctypes.c_char_p, ctypes.c_char_p]
    _lib = L
    return L


def status_string(status: int) -> str:
    return lib().qspec_status_string(int(status)).decode()


def version() -> int:
    return lib().qspec_version()


def packed_weight_bytes(N: int, K: int, group: int = GROUP) -> int:
    return lib().qspec_packed_weight_bytes(N, K, group)


def workspace_bytes(M: int, N: int, K: int, group: int = GROUP) -> int:
    return lib().qspec_workspace_bytes(M, N, K, group)


def debug_set_plan(name: str, value: str = None) -> None:
    """Force (value) or release (None) one of the library's kernel-plan overrides."""
    _check(lib().qspec_debug_set_plan(name.encode(), None if value is None else str(value).encode()),
           "qspec_debug_set_plan")


def describe_kernel(w4a4: bool, M: int, N: int, K: int, group: int = GROUP, wide: bool = False) -> str:
    """`wide`: the draft-mode product on widened codes."""
    buf = ctypes.create_string_buffer(128)
    _check(lib().qspec_describe_kernel(2 if wide else 1 if w4a4 else 0, M, N, K, group, buf, 128), "qspec_describe_kernel")
    return buf.value.decode()


def _dev(t: torch.Tensor, dtype, name: str) -> int:
    if not t.is_cuda:
        raise ValueError(f"{name} must live on the GPU")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


# The current stream's handle without building a torch.cuda.Stream object (1.3 us of the 8 that an
# eager call used to cost the host; the two functions are what torch.cuda.current_stream() itself asks).
_device = getattr(torch._C, "_cuda_getDevice", None)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream() -> int:
    if _raw_stream is None or _device is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(_device())


def _check(status: int, where: str) -> None:
    if status != OK:
        raise QSpecError(status, where)


def alloc_workspace(nbytes: int) -> torch.Tensor:
    """A workspace for the GEMM entry points.  Zero-filled: the head of a workspace
    holds arrival counters that must be zero before its first use (every call
    leaves them zero again, so one workspace serves any number of calls in turn)."""
    return torch.zeros(max(int(nbytes), 16), dtype=torch.uint8, device="cuda")


def _without_workspace(call, args, M, N, K, group) -> int:
    """The status of call(*args, workspace, its size, stream) with a workspace of its own if the call asks for
    one (convenience for tests: hot loops pass one from alloc_workspace instead)."""
    status = call(*args, None, 0, _stream())
    if status == ERR_WORKSPACE:
        workspace = alloc_workspace(workspace_bytes(M, N, K, group))
        status = call(*args, workspace.data_ptr(), workspace.numel(), _stream())
    return status


def pack_weights(codes: torch.Tensor, scales: torch.Tensor, packed: torch.Tensor = None,
                 group: int = GROUP) -> torch.Tensor:
    """codes int8 [N,K] in [-8,7], scales fp16 [N,K/128] -> uint8 blob."""
    N, K = codes.shape
    if packed is None:
        nbytes = packed_weight_bytes(N, K, group)
        if nbytes == 0:
            raise QSpecError(ERR_SHAPE, "qspec_pack_weights")
        packed = torch.empty(nbytes, dtype=torch.uint8, device=codes.device)
    _check(lib().qspec_pack_weights(_dev(codes, torch.int8, "codes"), _dev(scales, torch.float16, "scales"),
                                    N, K, group, _dev(packed, torch.uint8, "packed"), _stream()),
           "qspec_pack_weights")
    return packed


def unpack_weights(packed: torch.Tensor, N: int, K: int, group: int = GROUP):
    codes = torch.empty((N, K), dtype=torch.int8, device=packed.device)
    scales = torch.empty((N, K // group), dtype=torch.float16, device=packed.device)
    _check(lib().qspec_unpack_weights(_dev(packed, torch.uint8, "packed"), N, K, group,
                                      codes.data_ptr(), scales.data_ptr(), _stream()),
           "qspec_unpack_weights")
    return codes, scales


def quant_act(x: torch.Tensor, qa: torch.Tensor = None, sa: torch.Tensor = None, group: int = GROUP):
    """x fp16 [M,K] -> (qa uint8 [M,K/2], sa fp32 [M,K/128])."""
    M, K = x.shape
    if qa is None:
        qa = torch.empty((M, K // 2), dtype=torch.uint8, device=x.device)
    if sa is None:
        sa = torch.empty((M, max(K // group, 1)), dtype=torch.float32, device=x.device)
    _check(lib().qspec_quant_act(_dev(x, torch.float16, "x"), M, K, group,
                                 _dev(qa, torch.uint8, "qa"), _dev(sa, torch.float32, "sa"), _stream()),
           "qspec_quant_act")
    return qa, sa


def w4a4_takes_wide(M: int, N: int, K: int, group: int = GROUP) -> bool:
    """True when the widened activation format (quant_act_wide -> gemm_w4a4_wide) is the faster one for the
    draft-mode GEMM of this shape.  It is accepted from 25 tokens on either way."""
    return bool(lib().qspec_w4a4_takes_wide(M, N, K, group))


def quant_act_wide(x: torch.Tensor, qa8: torch.Tensor = None, sa: torch.Tensor = None, group: int = GROUP):
    """x fp16 [M,K] -> (qa8 int8 [M,K] in the widened device format, sa fp32 [M,K/128])."""
    M, K = x.shape
    if qa8 is None:
        qa8 = torch.empty((M, K), dtype=torch.int8, device=x.device)
    if sa is None:
        sa = torch.empty((M, max(K // group, 1)), dtype=torch.float32, device=x.device)
    _check(lib().qspec_quant_act_wide(_dev(x, torch.float16, "x"), M, K, group,
                                      _dev(qa8, torch.int8, "qa8"), _dev(sa, torch.float32, "sa"), _stream()),
           "qspec_quant_act_wide")
    return qa8, sa


def _quant_outputs(M, K, group, device, qa, sa, h, want_h, wide=False):
    if qa is None:
        qa = (torch.empty((M, K), dtype=torch.int8, device=device) if wide
              else torch.empty((M, K // 2), dtype=torch.uint8, device=device))
    if sa is None:
        sa = torch.empty((M, max(K // group, 1)), dtype=torch.float32, device=device)
    if h is None and want_h:
        h = torch.empty((M, K), dtype=torch.float16, device=device)
    return qa, sa, h


def rmsnorm_quant(x: torch.Tensor, weight: torch.Tensor, eps: float, qa: torch.Tensor = None,
                  sa: torch.Tensor = None, h: torch.Tensor = None, want_h: bool = False, rotate: bool = False,
                  group: int = GROUP, wide: bool = False):
    """RMSNorm (then, if `rotate`, the per-group Hadamard rotation) fused with the activation
    quantiser: x fp16 [M,K], weight fp16 [K] -> (qa uint8 [M,K/2], sa fp32 [M,K/128], h fp16 [M,K] or None);
    `wide`: qa int8 [M,K] in the widened format instead."""
    M, K = x.shape
    qa, sa, h = _quant_outputs(M, K, group, x.device, qa, sa, h, want_h, wide)
    _check(lib().qspec_rmsnorm_quant(_dev(x, torch.float16, "x"), _dev(weight, torch.float16, "weight"),
                                     float(eps), M, K, group, int(bool(rotate)) | (2 if wide else 0),
                                     _dev(qa, torch.int8 if wide else torch.uint8, "qa"),
                                     _dev(sa, torch.float32, "sa"),
                                     None if h is None else _dev(h, torch.float16, "h"), _stream()),
           "qspec_rmsnorm_quant")
    return qa, sa, h


def silu_mul_quant(gate_up: torch.Tensor, qa: torch.Tensor = None, sa: torch.Tensor = None,
                   h: torch.Tensor = None, want_h: bool = False, rotate: bool = False, group: int = GROUP,
                   wide: bool = False):
    """SiLU(gate) * up (then, if `rotate`, the per-group Hadamard rotation) fused with the activation
    quantiser: gate_up fp16 [M,2I] (gate first) -> (qa uint8 [M,I/2], sa fp32 [M,I/128], h fp16 [M,I] or None);
    `wide`: qa int8 [M,I] in the widened format instead."""
    M, I = gate_up.shape[0], gate_up.shape[1] // 2
    qa, sa, h = _quant_outputs(M, I, group, gate_up.device, qa, sa, h, want_h, wide)
    _check(lib().qspec_silu_mul_quant(_dev(gate_up, torch.float16, "gate_up"), M, I, group,
                                      int(bool(rotate)) | (2 if wide else 0),
                                      _dev(qa, torch.int8 if wide else torch.uint8, "qa"), _dev(sa, torch.float32, "sa"),
                                      None if h is None else _dev(h, torch.float16, "h"), _stream()),
           "qspec_silu_mul_quant")
    return qa, sa, h


def hadamard_quant(x: torch.Tensor, qa: torch.Tensor = None, sa: torch.Tensor = None,
                   h: torch.Tensor = None, want_h: bool = False, group: int = GROUP):
    """Every group of 128 features times H_128 / 8, then the activation quantiser: x fp16 [M,K] ->
    (qa uint8 [M,K/2], sa fp32 [M,K/128], h fp16 [M,K] or None)."""
    M, K = x.shape
    qa, sa, h = _quant_outputs(M, K, group, x.device, qa, sa, h, want_h)
    _check(lib().qspec_hadamard_quant(_dev(x, torch.float16, "x"), M, K, group,
                                      _dev(qa, torch.uint8, "qa"), _dev(sa, torch.float32, "sa"),
                                      None if h is None else _dev(h, torch.float16, "h"), _stream()),
           "qspec_hadamard_quant")
    return qa, sa, h


def reorder_quant(x: torch.Tensor, perm: torch.Tensor, n_outlier_groups: int, qa: torch.Tensor = None,
                  sa: torch.Tensor = None, h: torch.Tensor = None, want_h: bool = False, group: int = GROUP):
    """Reordering quantiser: x fp16 [M,K], perm int32 [K] -> (qa uint8 [M,K'/2], sa fp32 [M,K'/128],
    h fp16 [M,K'] or None) with K' = K + 128 * n_outlier_groups."""
    M, K = x.shape
    Kx = K + group * int(n_outlier_groups)
    qa, sa, h = _quant_outputs(M, Kx, group, x.device, qa, sa, h, want_h)
    _check(lib().qspec_reorder_quant(_dev(x, torch.float16, "x"), _dev(perm, torch.int32, "perm"), M, K, group,
                                     int(n_outlier_groups), _dev(qa, torch.uint8, "qa"),
                                     _dev(sa, torch.float32, "sa"),
                                     None if h is None else _dev(h, torch.float16, "h"), _stream()),
           "qspec_reorder_quant")
    return qa, sa, h


def gemm_w4a4(packed: torch.Tensor, qa: torch.Tensor, sa: torch.Tensor, N: int,
              y: torch.Tensor = None, workspace: torch.Tensor = None, group: int = GROUP) -> torch.Tensor:
    M, K = qa.shape[0], qa.shape[1] * 2
    if y is None:
        y = torch.empty((M, N), dtype=torch.float16, device=qa.device)
    if workspace is None:
        args = (_dev(packed, torch.uint8, "packed"), _dev(qa, torch.uint8, "qa"), _dev(sa, torch.float32, "sa"), M, N, K, group, _dev(y, torch.float16, "y"))
        status = _without_workspace(lib().qspec_gemm_w4a4, args, M, N, K, group)
    else:
        status = lib().qspec_gemm_w4a4(_dev(packed, torch.uint8, "packed"), _dev(qa, torch.uint8, "qa"), _dev(sa, torch.float32, "sa"),
                                       M, N, K, group, _dev(y, torch.float16, "y"),
                                       _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream())
    _check(status, "qspec_gemm_w4a4")
    return y


def gemm_w4a4_wide(packed: torch.Tensor, qa8: torch.Tensor, sa: torch.Tensor, N: int,
                   y: torch.Tensor = None, workspace: torch.Tensor = None, group: int = GROUP) -> torch.Tensor:
    M, K = qa8.shape
    if y is None:
        y = torch.empty((M, N), dtype=torch.float16, device=qa8.device)
    need = workspace_bytes(M, N, K, group) if workspace is None else 0
    if need:                              # (the call does not ask for one everywhere that it is faster with it)
        workspace = alloc_workspace(need)
    ws = (None, 0) if workspace is None else (_dev(workspace, torch.uint8, "workspace"), workspace.numel())
    _check(lib().qspec_gemm_w4a4_wide(_dev(packed, torch.uint8, "packed"), _dev(qa8, torch.int8, "qa8"), _dev(sa, torch.float32, "sa"),
                                      M, N, K, group, _dev(y, torch.float16, "y"), *ws, _stream()), "qspec_gemm_w4a4_wide")
    return y


def gemm_w4a16(packed: torch.Tensor, x: torch.Tensor, N: int, y: torch.Tensor = None,
               workspace: torch.Tensor = None, group: int = GROUP) -> torch.Tensor:
    M, K = x.shape
    if y is None:
        y = torch.empty((M, N), dtype=torch.float16, device=x.device)
    if workspace is None:
        args = (_dev(packed, torch.uint8, "packed"), _dev(x, torch.float16, "x"), M, N, K, group, _dev(y, torch.float16, "y"))
        status = _without_workspace(lib().qspec_gemm_w4a16, args, M, N, K, group)
    else:
        status = lib().qspec_gemm_w4a16(_dev(packed, torch.uint8, "packed"), _dev(x, torch.float16, "x"),
                                       M, N, K, group, _dev(y, torch.float16, "y"),
                                       _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream())
    _check(status, "qspec_gemm_w4a16")
    return y


NOALLOC_SCRATCH_BYTES = (32 << 20) + 16384


def gemm_w4a16_noalloc(packed: torch.Tensor, x: torch.Tensor, N: int, y: torch.Tensor,
                       group: int = GROUP) -> torch.Tensor:
    """qspec_gemm_w4a16 on the library's built-in scratch: the caller passes every buffer,
    nothing is allocated here or in the library."""
    M, K = x.shape
    _check(lib().qspec_gemm_w4a16_noalloc(_dev(packed, torch.uint8, "packed"), _dev(x, torch.float16, "x"),
                                          M, N, K, group, _dev(y, torch.float16, "y"), _stream()),
           "qspec_gemm_w4a16_noalloc")
    return y


def mlp_draft_workspace_bytes(M: int, H: int, I: int, group: int = GROUP) -> int:
    return lib().qspec_mlp_draft_workspace_bytes(M, H, I, group)


def mlp_draft(packed_gate_up: torch.Tensor, packed_down: torch.Tensor, qa_h: torch.Tensor, sa_h: torch.Tensor,
              H: int, I: int, workspace: torch.Tensor, status: torch.Tensor, gate_up: torch.Tensor = None,
              qa_i: torch.Tensor = None, sa_i: torch.Tensor = None, y: torch.Tensor = None, group: int = GROUP):
    """The draft-pass MLP of a block in one persistent launch.  workspace: zero-filled uint8 of
    mlp_draft_workspace_bytes; status: int32 [1] the caller zeroed (1 afterwards: the launch gave up).
    Returns (gate_up fp16 [M, 2I], qa_i, sa_i, y fp16 [M, H])."""
    M = qa_h.shape[0]
    dev = qa_h.device
    if gate_up is None:
        gate_up = torch.empty((M, 2 * I), dtype=torch.float16, device=dev)
    if qa_i is None:
        qa_i = torch.empty((M, I // 2), dtype=torch.uint8, device=dev)
    if sa_i is None:
        sa_i = torch.empty((M, I // group), dtype=torch.float32, device=dev)
    if y is None:
        y = torch.empty((M, H), dtype=torch.float16, device=dev)
    _check(lib().qspec_mlp_draft(_dev(packed_gate_up, torch.uint8, "packed_gate_up"), _dev(packed_down, torch.uint8, "packed_down"),
                                 _dev(qa_h, torch.uint8, "qa_h"), _dev(sa_h, torch.float32, "sa_h"), M, H, I, group,
                                 _dev(gate_up, torch.float16, "gate_up"), _dev(qa_i, torch.uint8, "qa_i"),
                                 _dev(sa_i, torch.float32, "sa_i"), _dev(y, torch.float16, "y"),
                                 _dev(workspace, torch.uint8, "workspace"), workspace.numel(),
                                 _dev(status, torch.int32, "status"), _stream()),
           "qspec_mlp_draft")
    return gate_up, qa_i, sa_i, y


def gemm_w4a4_partials(packed: torch.Tensor, qa: torch.Tensor, N: int, n0: int, n_count: int,
                       partials: torch.Tensor = None, group: int = GROUP) -> torch.Tensor:
    M, K = qa.shape[0], qa.shape[1] * 2
    if partials is None:
        partials = torch.empty((M, n_count, K // group), dtype=torch.int32, device=qa.device)
    _check(lib().qspec_gemm_w4a4_partials(_dev(packed, torch.uint8, "packed"), _dev(qa, torch.uint8, "qa"),
                                          M, N, K, group, n0, n_count,
                                          _dev(partials, torch.int32, "partials"), _stream()),
           "qspec_gemm_w4a4_partials")
    return partials


def accept_workspace_bytes(B: int, gamma: int, V: int) -> int:
    return lib().qspec_accept_workspace_bytes(B, gamma, V)


def greedy_accept(logits: torch.Tensor, draft: torch.Tensor, n_accept: torch.Tensor = None,
                  out_tokens: torch.Tensor = None, workspace: torch.Tensor = None):
    """logits fp16 [B, gamma+1, V], draft int32 [B, gamma] -> (n_accept int32 [B], out_tokens int32 [B, gamma+1])."""
    B, rows, V = logits.shape
    gamma = rows - 1
    if n_accept is None:
        n_accept = torch.empty((B,), dtype=torch.int32, device=logits.device)
    if out_tokens is None:
        out_tokens = torch.empty((B, rows), dtype=torch.int32, device=logits.device)
    if workspace is None:
        workspace = torch.empty(max(accept_workspace_bytes(B, gamma, V), 16), dtype=torch.uint8, device=logits.device)
    _check(lib().qspec_greedy_accept(_dev(logits, torch.float16, "logits"), _dev(draft, torch.int32, "draft"),
                                     B, gamma, V, _dev(n_accept, torch.int32, "n_accept"),
                                     _dev(out_tokens, torch.int32, "out_tokens"),
                                     _dev(workspace, torch.uint8, "workspace"), workspace.numel(), _stream()),
           "qspec_greedy_accept")
    return n_accept, out_tokens


def kv_overwrite(cache: torch.Tensor, kv_verify: torch.Tensor, n_accept: torch.Tensor, pos: torch.Tensor) -> torch.Tensor:
    """cache fp16 [B, S, D] (updated in place), kv_verify fp16 [B, gamma+1, D], n_accept / pos int32 [B]."""
    B, S, D = cache.shape
    gamma = kv_verify.shape[1] - 1
    _check(lib().qspec_kv_overwrite(_dev(kv_verify, torch.float16, "kv_verify"), _dev(n_accept, torch.int32, "n_accept"),
                                    _dev(pos, torch.int32, "pos"), B, gamma, D, S,
                                    _dev(cache, torch.float16, "cache"), _stream()),
           "qspec_kv_overwrite")
    return cache


# ---- the 4-bit key/value cache (layout: include/qspec.h), attention over it, sampling

def _shaped(t: torch.Tensor, dtype, shape, device: int, name: str) -> int:
    """_dev for a tensor of device number `device` whose sizes are given by the others: the kernels index by those sizes alone."""
    if t.get_device() != device or t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        if t.is_cuda and t.get_device() != device:
            raise ValueError(f"{name} must live on cuda:{device}, got {t.device}")
        _dev(t, dtype, name)
        raise ValueError(f"{name} must have the shape {tuple(shape)}, got {tuple(t.shape)}")
    return t.data_ptr()


def _here(t: torch.Tensor, name: str) -> int:
    """Device number of the tensor that stands for the call's: the launch goes to the current device's stream."""
    device = t.get_device()
    if device < 0:
        raise ValueError(f"{name} must live on the GPU")
    if device != (torch.cuda.current_device() if _device is None else _device()):
        raise ValueError(f"{name} lives on {t.device}, the current device is cuda:{torch.cuda.current_device()}")
    return device


def kv4_page_bytes(Hkv: int, D: int, page_size: int) -> int:
    return lib().qspec_kv4_page_bytes(Hkv, D, page_size)


def alloc_kv4_cache(n_pages: int, Hkv: int, D: int, page_size: int) -> torch.Tensor:
    """A cache of n_pages pages: uint8 [n_pages, kv4_page_bytes], zeroed (not that a row is read before it is written)."""
    nbytes = kv4_page_bytes(Hkv, D, page_size)
    if nbytes == 0:
        raise QSpecError(ERR_SHAPE, "qspec_kv4_page_bytes")
    return torch.zeros((n_pages, nbytes), dtype=torch.uint8, device="cuda")


_page_bytes = {}


def _kv4(cache, pos, page_table, Hkv, D, page_size, where):
    """(device number, cache, pos, table pointers, B, max_pages, n_pages) of a call's cache."""
    nbytes = _page_bytes.get((Hkv, D, page_size))
    if nbytes is None:
        nbytes = kv4_page_bytes(Hkv, D, page_size)
        if nbytes == 0:
            raise QSpecError(ERR_SHAPE, where)
        _page_bytes[Hkv, D, page_size] = nbytes
    n_pages, B = cache.shape[0], pos.shape[0]
    if B == 0 or n_pages == 0:
        raise QSpecError(ERR_SHAPE, where)
    device = _here(cache, "cache")
    table, max_pages = None, n_pages // B
    if page_table is not None:
        max_pages = page_table.shape[-1]
        table = _shaped(page_table, torch.int32, (B, max_pages), device, "page_table")
    return (device, _shaped(cache, torch.uint8, (n_pages, nbytes), device, "cache"), _shaped(pos, torch.int32, (B,), device, "pos"),
            table, B, max_pages, n_pages)


def rope_kv4_append(qkv: torch.Tensor, inv_freq: torch.Tensor, pos: torch.Tensor, cache: torch.Tensor, Hq: int, Hkv: int,
                    page_size: int, page_table: torch.Tensor = None, interleaved: bool = False, mscale: float = 1.0,
                    q: torch.Tensor = None) -> torch.Tensor:
    """qkv fp16 [B, T, (Hq + 2 Hkv) D], inv_freq float64 [rot/2] (rope.frequencies; None: no rotation), pos int32 [B], cache uint8
    [pages, kv4_page_bytes] (updated in place), page_table int32 [B, max_pages] or None -> rotated queries fp16 [B, T, Hq, D]."""
    B, T, width = qkv.shape
    heads = Hq + 2 * Hkv
    if heads < 1 or width % heads:
        raise QSpecError(ERR_SHAPE, "qspec_rope_kv4_append")
    D = width // heads
    device, c, at, table, Bp, max_pages, n_pages = _kv4(cache, pos, page_table, Hkv, D, page_size, "qspec_rope_kv4_append")
    x = _shaped(qkv, torch.float16, (Bp, T, width), device, "qkv")
    rot, freq = 0, None
    if inv_freq is not None:
        rot = 2 * inv_freq.numel()
        freq = _shaped(inv_freq, torch.float64, (rot // 2,), device, "inv_freq") if rot else None
    if q is None:
        q = torch.empty((B, T, Hq, D), dtype=torch.float16, device=cache.device)
    _check(lib().qspec_rope_kv4_append(x, freq, at, table, B, T, Hq, Hkv, D, rot, int(bool(interleaved)), mscale, page_size, max_pages,
                                       n_pages, _shaped(q, torch.float16, (B, T, Hq, D), device, "q"), c, _stream()),
           "qspec_rope_kv4_append")
    return q


def kv4_read(cache: torch.Tensor, pos: torch.Tensor, T: int, Hkv: int, D: int, page_size: int, page_table: torch.Tensor = None,
             k: torch.Tensor = None, v: torch.Tensor = None):
    """Values of rows pos[b] .. pos[b] + T - 1 of the cache: (k, v), fp16 [B, T, Hkv, D]; zeros for rows outside of it."""
    device, c, at, table, B, max_pages, n_pages = _kv4(cache, pos, page_table, Hkv, D, page_size, "qspec_kv4_read")
    if T < 1:
        raise QSpecError(ERR_SHAPE, "qspec_kv4_read")
    shape = (B, T, Hkv, D)
    k = torch.empty(shape, dtype=torch.float16, device=cache.device) if k is None else k
    v = torch.empty(shape, dtype=torch.float16, device=cache.device) if v is None else v
    _check(lib().qspec_kv4_read(c, at, table, B, T, Hkv, D, page_size, max_pages, n_pages, _shaped(k, torch.float16, shape, device, "k"),
                                _shaped(v, torch.float16, shape, device, "v"), _stream()), "qspec_kv4_read")
    return k, v


def attn_kv4_workspace_bytes(B: int, T: int, Hq: int, Hkv: int, D: int) -> int:
    return lib().qspec_attn_kv4_workspace_bytes(B, T, Hq, Hkv, D)


def attn_kv4(q: torch.Tensor, cache: torch.Tensor, pos: torch.Tensor, Hkv: int, page_size: int, page_table: torch.Tensor = None,
             scale: float = None, window: int = 0, sinks: int = 0, out: torch.Tensor = None,
             workspace: torch.Tensor = None) -> torch.Tensor:
    """Attention of q fp16 [B, T, Hq, D] (rows at positions pos[b] ..) over the 4-bit cache -> fp16 [B, T, Hq, D].  scale: 1 / sqrt(D)
    by default; window > 0: the last `window` tokens and the first `sinks`.  Hot loops pass out and a workspace."""
    B, T, Hq, D = q.shape
    device, c, at, table, Bp, max_pages, n_pages = _kv4(cache, pos, page_table, Hkv, D, page_size, "qspec_attn_kv4")
    x = _shaped(q, torch.float16, (Bp, T, Hq, D), device, "q")
    if out is None:
        out = torch.empty_like(q)
    if workspace is None:
        workspace = alloc_workspace(attn_kv4_workspace_bytes(B, T, Hq, Hkv, D))
    _check(lib().qspec_attn_kv4(x, c, at, table, B, T, Hq, Hkv, D, page_size, max_pages, n_pages, D ** -0.5 if scale is None else scale,
                                window, sinks, _shaped(out, torch.float16, q.shape, device, "out"),
                                _shaped(workspace, torch.uint8, (workspace.numel(),), device, "workspace"), workspace.numel(), _stream()),
           "qspec_attn_kv4")
    return out


def attn_kv4_shared_workspace_bytes(B: int, T: int, Hq: int, Hkv: int, D: int, groups: int) -> int:
    return lib().qspec_attn_kv4_shared_workspace_bytes(B, T, Hq, Hkv, D, groups)


def attn_kv4_shared(q: torch.Tensor, cache: torch.Tensor, pos: torch.Tensor, shared: torch.Tensor, Hkv: int, page_size: int,
                    page_table: torch.Tensor = None, scale: float = None, out: torch.Tensor = None,
                    workspace: torch.Tensor = None) -> torch.Tensor:
    """attn_kv4 for sequences that share beginnings: shared int32 [groups], the B sequences being that many sets of neighbours; the
    first shared[g] tokens of a set are read once, through the page table's row of its first sequence.  One sequence many times longer than the others, or few long
    ones over few key/value heads, are faster with attn_kv4.  Hot loops pass out and a workspace."""
    B, T, Hq, D = q.shape
    groups = shared.shape[0]
    device, c, at, table, Bp, max_pages, n_pages = _kv4(cache, pos, page_table, Hkv, D, page_size, "qspec_attn_kv4_shared")
    x = _shaped(q, torch.float16, (Bp, T, Hq, D), device, "q")
    if out is None:
        out = torch.empty_like(q)
    if workspace is None:
        workspace = alloc_workspace(attn_kv4_shared_workspace_bytes(B, T, Hq, Hkv, D, groups))
    _check(lib().qspec_attn_kv4_shared(x, c, at, table, _shaped(shared, torch.int32, (groups,), device, "shared"), B, T, Hq, Hkv, D, groups, page_size,
                                       max_pages, n_pages, D ** -0.5 if scale is None else scale, _shaped(out, torch.float16, q.shape, device, "out"),
                                       _shaped(workspace, torch.uint8, (workspace.numel(),), device, "workspace"), workspace.numel(), _stream()),
           "qspec_attn_kv4_shared")
    return out


def kv4_bounds_bytes(Hkv: int, D: int) -> int:
    return lib().qspec_kv4_bounds_bytes(Hkv, D)


def alloc_kv4_bounds(n_pages: int, Hkv: int, D: int) -> torch.Tensor:
    """Bounds for a cache of n_pages pages: uint8 [n_pages, kv4_bounds_bytes], zeroed."""
    nbytes = kv4_bounds_bytes(Hkv, D)
    if nbytes == 0:
        raise QSpecError(ERR_SHAPE, "qspec_kv4_bounds_bytes")
    return torch.zeros((n_pages, nbytes), dtype=torch.uint8, device="cuda")


def kv4_bounds(cache: torch.Tensor, pos: torch.Tensor, T: int, bounds: torch.Tensor, Hkv: int, D: int, page_size: int,
               page_table: torch.Tensor = None) -> torch.Tensor:
    """Bounds of the keys in the pages that rows pos[b] .. pos[b] + T - 1 lie in, from the tokens up to the last of them: bounds uint8 [pages,
    kv4_bounds_bytes], updated in place.  To be called behind each rope_kv4_append."""
    device, c, at, table, B, max_pages, n_pages = _kv4(cache, pos, page_table, Hkv, D, page_size, "qspec_kv4_bounds")
    _check(lib().qspec_kv4_bounds(c, at, table, B, T, Hkv, D, page_size, max_pages, n_pages,
                                  _shaped(bounds, torch.uint8, (n_pages, _kv4_bounds_bytes(Hkv, D)), device, "bounds"), _stream()), "qspec_kv4_bounds")
    return bounds


_bounds_bytes = {}


def _kv4_bounds_bytes(Hkv, D):
    nbytes = _bounds_bytes.get((Hkv, D))
    if nbytes is None:
        nbytes = _bounds_bytes[Hkv, D] = kv4_bounds_bytes(Hkv, D)
    return nbytes


def _kv4_bounds(bounds, pos, page_table, Hkv, D, where):
    """(device number, bounds, pos, table pointers, B, max_pages, n_pages) of a call that reads bounds."""
    n_pages, B = bounds.shape[0], pos.shape[0]
    nbytes = _kv4_bounds_bytes(Hkv, D)
    if B == 0 or n_pages == 0 or nbytes == 0:
        raise QSpecError(ERR_SHAPE, where)
    device = _here(bounds, "bounds")
    table, max_pages = None, n_pages // B
    if page_table is not None:
        max_pages = page_table.shape[-1]
        table = _shaped(page_table, torch.int32, (B, max_pages), device, "page_table")
    return (device, _shaped(bounds, torch.uint8, (n_pages, nbytes), device, "bounds"), _shaped(pos, torch.int32, (B,), device, "pos"),
            table, B, max_pages, n_pages)


def kv4_bounds_read(bounds: torch.Tensor, pos: torch.Tensor, T: int, Hkv: int, D: int, page_size: int, page_table: torch.Tensor = None,
                    upper: torch.Tensor = None, lower: torch.Tensor = None):
    """Bounds of the pages that rows pos[b] .. pos[b] + T - 1 lie in, as numbers: (upper, lower), fp32 [B, (T - 1) // page_size + 2, Hkv, D];
    zeros behind the last of them."""
    device, c, at, table, B, max_pages, n_pages = _kv4_bounds(bounds, pos, page_table, Hkv, D, "qspec_kv4_bounds_read")
    if T < 1 or page_size < 1:
        raise QSpecError(ERR_SHAPE, "qspec_kv4_bounds_read")
    shape = (B, (T - 1) // page_size + 2, Hkv, D)
    upper = torch.empty(shape, dtype=torch.float32, device=bounds.device) if upper is None else upper
    lower = torch.empty(shape, dtype=torch.float32, device=bounds.device) if lower is None else lower
    _check(lib().qspec_kv4_bounds_read(c, at, table, B, T, Hkv, D, page_size, max_pages, n_pages, _shaped(upper, torch.float32, shape, device, "upper"),
                                       _shaped(lower, torch.float32, shape, device, "lower"), _stream()), "qspec_kv4_bounds_read")
    return upper, lower


def kv4_select_workspace_bytes(B: int, T: int, Hq: int, Hkv: int, max_pages: int) -> int:
    return lib().qspec_kv4_select_workspace_bytes(B, T, Hq, Hkv, max_pages)


def kv4_select(q: torch.Tensor, bounds: torch.Tensor, pos: torch.Tensor, Hkv: int, page_size: int, count: int, page_table: torch.Tensor = None,
               first: int = 1, last: int = 1, blocks: torch.Tensor = None, workspace: torch.Tensor = None) -> torch.Tensor:
    """For every row of q fp16 [B, T, Hq, D] and key/value head the `count` pages that its attention is to read, int32 [B, T, Hkv, count] in
    ascending order (-1 behind the last): the first `first`, the last `last`, and the best of the others by their bounds."""
    B, T, Hq, D = q.shape
    device, c, at, table, Bp, max_pages, n_pages = _kv4_bounds(bounds, pos, page_table, Hkv, D, "qspec_kv4_select")
    x = _shaped(q, torch.float16, (Bp, T, Hq, D), device, "q")
    if count < 1:
        raise QSpecError(ERR_SHAPE, "qspec_kv4_select")
    if blocks is None:
        blocks = torch.empty((B, T, Hkv, count), dtype=torch.int32, device=q.device)
    if workspace is None:
        workspace = torch.empty(max(kv4_select_workspace_bytes(B, T, Hq, Hkv, max_pages), 16), dtype=torch.uint8, device=q.device)
    _check(lib().qspec_kv4_select(x, c, at, table, B, T, Hq, Hkv, D, page_size, max_pages, n_pages, first, last, count,
                                  _shaped(blocks, torch.int32, (B, T, Hkv, count), device, "blocks"),
                                  _shaped(workspace, torch.uint8, (workspace.numel(),), device, "workspace"), workspace.numel(), _stream()),
           "qspec_kv4_select")
    return blocks


def attn_kv4_blocks_workspace_bytes(B: int, T: int, Hq: int, Hkv: int, D: int) -> int:
    return lib().qspec_attn_kv4_blocks_workspace_bytes(B, T, Hq, Hkv, D)


def attn_kv4_blocks(q: torch.Tensor, cache: torch.Tensor, pos: torch.Tensor, blocks: torch.Tensor, Hkv: int, page_size: int,
                    page_table: torch.Tensor = None, scale: float = None, out: torch.Tensor = None,
                    workspace: torch.Tensor = None) -> torch.Tensor:
    """attn_kv4 over the pages that blocks int32 [B, T, Hkv, count] names for every row and key/value head (kv4_select writes
    such lists).  Hot loops pass out and a workspace."""
    B, T, Hq, D = q.shape
    device, c, at, table, Bp, max_pages, n_pages = _kv4(cache, pos, page_table, Hkv, D, page_size, "qspec_attn_kv4_blocks")
    x = _shaped(q, torch.float16, (Bp, T, Hq, D), device, "q")
    count = blocks.shape[-1]
    if out is None:
        out = torch.empty_like(q)
    if workspace is None:
        workspace = alloc_workspace(attn_kv4_blocks_workspace_bytes(B, T, Hq, Hkv, D))
    _check(lib().qspec_attn_kv4_blocks(x, c, at, table, _shaped(blocks, torch.int32, (B, T, Hkv, count), device, "blocks"), B, T, Hq, Hkv, D, count,
                                       page_size, max_pages, n_pages, D ** -0.5 if scale is None else scale,
                                       _shaped(out, torch.float16, q.shape, device, "out"),
                                       _shaped(workspace, torch.uint8, (workspace.numel(),), device, "workspace"), workspace.numel(), _stream()),
           "qspec_attn_kv4_blocks")
    return out


def sample_workspace_bytes(B: int, gamma: int, V: int) -> int:
    return lib().qspec_sample_workspace_bytes(B, gamma, V)


def sample(logits: torch.Tensor, u: torch.Tensor, temperature: torch.Tensor = None, top_k: torch.Tensor = None,
           top_p: torch.Tensor = None, min_p: torch.Tensor = None, draft: torch.Tensor = None, n_accept: torch.Tensor = None,
           out_tokens: torch.Tensor = None, workspace: torch.Tensor = None):
    """A token per row of logits fp16 [B, gamma+1, V] by the random numbers u fp32 [B, gamma+1]; temperature, top_p, min_p fp32 [B] and
    top_k int32 [B], each optional.  Returns (None, tokens int32 [B, gamma+1]), or with draft int32 [B, gamma] the acceptance of the
    drafts: (n_accept int32 [B], out_tokens int32 [B, gamma+1]), as greedy_accept does."""
    B, rows, V = logits.shape
    gamma, device = rows - 1, _here(logits, "logits")
    x = _shaped(logits, torch.float16, (B, rows, V), device, "logits")
    t = None if temperature is None else _shaped(temperature, torch.float32, (B,), device, "temperature")
    k = None if top_k is None else _shaped(top_k, torch.int32, (B,), device, "top_k")
    tp = None if top_p is None else _shaped(top_p, torch.float32, (B,), device, "top_p")
    mp = None if min_p is None else _shaped(min_p, torch.float32, (B,), device, "min_p")
    if out_tokens is None:
        out_tokens = torch.empty((B, rows), dtype=torch.int32, device=logits.device)
    drafts = accepted = ws = None
    nbytes = 0
    if draft is not None:
        if gamma == 0:
            raise QSpecError(ERR_SHAPE, "qspec_sample")
        if n_accept is None:
            n_accept = torch.empty((B,), dtype=torch.int32, device=logits.device)
        if workspace is None:
            workspace = torch.empty(max(sample_workspace_bytes(B, gamma, V), 16), dtype=torch.uint8, device=logits.device)
        drafts = _shaped(draft, torch.int32, (B, gamma), device, "draft")
        accepted = _shaped(n_accept, torch.int32, (B,), device, "n_accept")
        ws, nbytes = _shaped(workspace, torch.uint8, (workspace.numel(),), device, "workspace"), workspace.numel()
    _check(lib().qspec_sample(x, _shaped(u, torch.float32, (B, rows), device, "u"), t, k, tp, mp, drafts, B, gamma, V, accepted,
                              _shaped(out_tokens, torch.int32, (B, rows), device, "out_tokens"), ws, nbytes, _stream()), "qspec_sample")
    return (None if draft is None else n_accept), out_tokens
