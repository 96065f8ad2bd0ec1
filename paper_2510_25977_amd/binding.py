"""Thin ctypes binding of ``libsvdmlp.so`` (same names as ``include/svdmlp.h``).

Argument marshalling only: PyTorch supplies device memory and streams, every step of the forward
runs in the library's HIP kernels.  There is no CPU or PyTorch fallback: if the library is missing
or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import functools
from pathlib import Path
from typing import NamedTuple, Optional

import torch

HERE = Path(__file__).resolve().parent
LIB_PATH = HERE / "libsvdmlp.so"      # the in-tree build, nothing else
TENSORS_PATH = HERE / "_tensors.so"

SVDMLP_BF16, SVDMLP_F32 = 0, 1
SVDMLP_GATED, SVDMLP_LINEAR = 0, 1
SVDMLP_OK = 0
SVDMLP_INVALID_ARGUMENT, SVDMLP_UNSUPPORTED, SVDMLP_WORKSPACE_TOO_SMALL, SVDMLP_HIP_ERROR, SVDMLP_NO_DEVICE = -1, -2, -3, -4, -5
SVDMLP_SCRATCH_TOO_SMALL, SVDMLP_OUT_OF_HOST_MEMORY, SVDMLP_TIMED_OUT = -6, -7, -8
FLAG_FORCE_TILED, FLAG_FORCE_STREAM, FLAG_SKIP_ARCH_CHECK, FLAG_STREAM_ONE_KERNEL, FLAG_TILED_FUSED, FLAG_TILE_128 = 1, 2, 4, 8, 16, 32
FLAG_PLAN_ROOM = 64
FIRST_S1, FIRST_IN, OUT_256, OUT_128 = 1, 2, 1, 2
SVDMLP_F8 = 2
NORM_NONE, NORM_RMS, NORM_LAYER = 0, 1, 2
GATE_PLAIN, GATE_SIGMOID, GATE_TANH = 0, 1, 2
SCALE_BLOCK = 128

EXPORTS = ["svdmlp_workspace_bytes", "svdmlp_create", "svdmlp_forward", "svdmlp_destroy", "svdmlp_status_string",
           "svdmlp_last_hip_error", "svdmlp_last_path", "svdmlp_abi_version", "svdmlp_profile_begin",
           "svdmlp_profile_end", "svdmlp_profile_kernel_name", "svdmlp_describe", "svdmlp_rank_for_ratio",
           "svdmlp_forward_static_scratch", "svdmlp_static_scratch_bytes",
           "svdmlp_roof_read", "svdmlp_roof_mfma", "svdmlp_roof_mfma_operands", "svdmlp_roof_pingpong", "svdmlp_roof_empty", "svdmlp_roof_empty_chain", "svdmlp_force_plan", "svdmlp_roof_coexec", "svdmlp_check", "svdmlp_debug_set_poll_limit", "svdmlp_debug_preset_static_tickets",
           "svdmlp_quantize", "svdmlp_norm", "svdmlp_scaled_matmul", "svdmlp_scaled_matmul_workspace_bytes",
           "svdmlp_scaled_matmul_describe"]


class svdmlp_desc(ctypes.Structure):
    _fields_ = [
        ("kind", ctypes.c_int32), ("dtype", ctypes.c_int32),
        ("max_M", ctypes.c_int64), ("d", ctypes.c_int64), ("ffn", ctypes.c_int64), ("r", ctypes.c_int64),
        ("r_down", ctypes.c_int64),
        ("Ug", ctypes.c_void_p), ("Vg", ctypes.c_void_p), ("Uu", ctypes.c_void_p), ("Vu", ctypes.c_void_p),
        ("Ud", ctypes.c_void_p), ("Vd", ctypes.c_void_p),
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
        ("flags", ctypes.c_uint32),
    ]


class SvdMlpError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} ({status})")


_lib = None


def lib() -> ctypes.CDLL:
    """Load the built library (raises if it has not been built: ``python -m paper_2510_25977_amd.build``)."""
    global _lib
    if _lib is None:
        if not LIB_PATH.exists():
            raise FileNotFoundError(f"{LIB_PATH} not found: build it with `python -m paper_2510_25977_amd.build`")
        L = ctypes.CDLL(str(LIB_PATH))
        L.svdmlp_workspace_bytes.argtypes = [ctypes.POINTER(svdmlp_desc)]
        L.svdmlp_workspace_bytes.restype = ctypes.c_size_t
        L.svdmlp_create.argtypes = [ctypes.POINTER(svdmlp_desc), ctypes.POINTER(ctypes.c_void_p)]
        L.svdmlp_create.restype = ctypes.c_int
        L.svdmlp_forward.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p]
        L.svdmlp_forward.restype = ctypes.c_int
        L.svdmlp_forward_static_scratch.argtypes = L.svdmlp_forward.argtypes
        L.svdmlp_forward_static_scratch.restype = ctypes.c_int
        L.svdmlp_static_scratch_bytes.argtypes = []
        L.svdmlp_static_scratch_bytes.restype = ctypes.c_size_t
        L.svdmlp_roof_read.argtypes = [ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p]
        L.svdmlp_roof_read.restype = ctypes.c_int
        L.svdmlp_roof_mfma.argtypes = [ctypes.c_int, ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p]
        L.svdmlp_roof_mfma.restype = ctypes.c_int
        L.svdmlp_roof_mfma_operands.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p]
        L.svdmlp_roof_mfma_operands.restype = ctypes.c_int
        L.svdmlp_roof_pingpong.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p]
        L.svdmlp_roof_pingpong.restype = ctypes.c_int
        L.svdmlp_roof_coexec.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.c_void_p, ctypes.c_int, ctypes.c_void_p]
        L.svdmlp_roof_coexec.restype = ctypes.c_int
        L.svdmlp_roof_empty.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.c_void_p]
        L.svdmlp_roof_empty.restype = ctypes.c_int
        L.svdmlp_roof_empty_chain.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_void_p]
        L.svdmlp_roof_empty_chain.restype = ctypes.c_int
        L.svdmlp_debug_set_poll_limit.argtypes = [ctypes.c_void_p, ctypes.c_int32]
        L.svdmlp_debug_set_poll_limit.restype = ctypes.c_int
        L.svdmlp_debug_preset_static_tickets.argtypes = [ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p]
        L.svdmlp_debug_preset_static_tickets.restype = ctypes.c_int
        L.svdmlp_check.argtypes = [ctypes.c_void_p]
        L.svdmlp_check.restype = ctypes.c_int
        L.svdmlp_force_plan.argtypes = [ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, ctypes.c_int32]
        L.svdmlp_force_plan.restype = ctypes.c_int
        L.svdmlp_destroy.argtypes = [ctypes.c_void_p]
        L.svdmlp_destroy.restype = ctypes.c_int
        L.svdmlp_status_string.argtypes = [ctypes.c_int]
        L.svdmlp_status_string.restype = ctypes.c_char_p
        L.svdmlp_last_hip_error.argtypes = [ctypes.c_void_p]
        L.svdmlp_last_hip_error.restype = ctypes.c_int
        L.svdmlp_last_path.argtypes = [ctypes.c_void_p]
        L.svdmlp_last_path.restype = ctypes.c_int
        L.svdmlp_abi_version.restype = ctypes.c_int
        L.svdmlp_rank_for_ratio.argtypes = [ctypes.c_int64, ctypes.c_int64, ctypes.c_double, ctypes.c_int64, ctypes.c_double]
        L.svdmlp_rank_for_ratio.restype = ctypes.c_int64
        L.svdmlp_profile_begin.argtypes = [ctypes.c_void_p, ctypes.c_int]
        L.svdmlp_profile_begin.restype = ctypes.c_int
        L.svdmlp_profile_end.argtypes = [ctypes.c_void_p, ctypes.POINTER(ctypes.c_float), ctypes.POINTER(ctypes.c_int),
                                         ctypes.POINTER(ctypes.c_int)]
        L.svdmlp_profile_end.restype = ctypes.c_int
        L.svdmlp_profile_kernel_name.argtypes = [ctypes.c_void_p, ctypes.c_int]
        L.svdmlp_profile_kernel_name.restype = ctypes.c_char_p
        L.svdmlp_describe.argtypes = [ctypes.POINTER(svdmlp_desc), ctypes.c_int64, ctypes.c_char_p, ctypes.c_size_t]
        L.svdmlp_describe.restype = ctypes.c_int
        # packed argument structures go as bytes
        for name in ("svdmlp_quantize", "svdmlp_norm", "svdmlp_scaled_matmul"):
            getattr(L, name).argtypes = [ctypes.c_char_p, ctypes.c_void_p]
            getattr(L, name).restype = ctypes.c_int
        L.svdmlp_scaled_matmul_workspace_bytes.argtypes = [ctypes.c_int64, ctypes.c_int64, ctypes.c_int64, ctypes.c_int32]
        L.svdmlp_scaled_matmul_workspace_bytes.restype = ctypes.c_size_t
        L.svdmlp_scaled_matmul_describe.argtypes = [ctypes.c_int64, ctypes.c_int64, ctypes.c_int64, ctypes.c_int32, ctypes.c_int32,
                                                    ctypes.c_char_p, ctypes.c_size_t]
        L.svdmlp_scaled_matmul_describe.restype = ctypes.c_int
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().svdmlp_status_string(int(status)).decode()


def svdmlp_workspace_bytes(desc: svdmlp_desc) -> int:
    return int(lib().svdmlp_workspace_bytes(ctypes.byref(desc)))


def svdmlp_rank_for_ratio(k: int, n: int, ratio: float, block: int = 128, alpha: float = 0.5) -> int:
    r = lib().svdmlp_rank_for_ratio(int(k), int(n), float(ratio), int(block), float(alpha))
    if r < 0:
        raise SvdMlpError(SVDMLP_INVALID_ARGUMENT, "svdmlp_rank_for_ratio")
    return int(r)


def svdmlp_describe(desc: svdmlp_desc, M: int) -> str:
    buf = ctypes.create_string_buffer(4096)
    st = lib().svdmlp_describe(ctypes.byref(desc), int(M), buf, len(buf))
    if st != SVDMLP_OK:
        raise SvdMlpError(st, "svdmlp_describe")
    return buf.value.decode()


def svdmlp_create(desc: svdmlp_desc) -> ctypes.c_void_p:
    out = ctypes.c_void_p()
    st = lib().svdmlp_create(ctypes.byref(desc), ctypes.byref(out))
    if st != SVDMLP_OK:
        raise SvdMlpError(st, "svdmlp_create")
    return out


# The argument types of the forwards would also take bytes and str, by their host address: anything but plain integers goes
# through c_void_p, which takes integers and None.  (Integers as they are: 0.3 us less per call.)
def svdmlp_forward(ctx, X_ptr: int, M: int, Y_ptr: int, stream_ptr: int = 0) -> None:
    if not (type(X_ptr) is type(Y_ptr) is type(stream_ptr) is int):
        X_ptr, Y_ptr, stream_ptr = ctypes.c_void_p(X_ptr), ctypes.c_void_p(Y_ptr), ctypes.c_void_p(stream_ptr)
    st = lib().svdmlp_forward(ctx, X_ptr, int(M), Y_ptr, stream_ptr)
    if st != SVDMLP_OK:
        raise SvdMlpError(st, "svdmlp_forward")


def svdmlp_forward_static_scratch(ctx, X_ptr: int, M: int, Y_ptr: int, stream_ptr: int = 0) -> None:
    if not (type(X_ptr) is type(Y_ptr) is type(stream_ptr) is int):
        X_ptr, Y_ptr, stream_ptr = ctypes.c_void_p(X_ptr), ctypes.c_void_p(Y_ptr), ctypes.c_void_p(stream_ptr)
    st = lib().svdmlp_forward_static_scratch(ctx, X_ptr, int(M), Y_ptr, stream_ptr)
    if st != SVDMLP_OK:
        raise SvdMlpError(st, "svdmlp_forward_static_scratch")


def svdmlp_static_scratch_bytes() -> int:
    return int(lib().svdmlp_static_scratch_bytes())


def _check(st: int, where: str) -> None:
    if st != SVDMLP_OK:
        raise SvdMlpError(st, where)


def svdmlp_roof_read(buf_ptr: int, nbytes: int, sink_ptr: int, workgroups: int, stream_ptr: int = 0) -> None:
    _check(lib().svdmlp_roof_read(ctypes.c_void_p(buf_ptr), int(nbytes), ctypes.c_void_p(sink_ptr), int(workgroups),
                                  ctypes.c_void_p(stream_ptr)), "svdmlp_roof_read")


def svdmlp_roof_mfma(iters: int, sink_ptr: int, workgroups: int, stream_ptr: int = 0) -> None:
    _check(lib().svdmlp_roof_mfma(int(iters), ctypes.c_void_p(sink_ptr), int(workgroups), ctypes.c_void_p(stream_ptr)),
           "svdmlp_roof_mfma")


ROOF_OPERANDS_ZERO, ROOF_OPERANDS_CONSTANT, ROOF_OPERANDS_RANDOM = 0, 1, 2


def svdmlp_roof_mfma_operands(iters: int, operands: int, sink_ptr: int, workgroups: int, stream_ptr: int = 0) -> None:
    _check(lib().svdmlp_roof_mfma_operands(int(iters), int(operands), ctypes.c_void_p(sink_ptr), int(workgroups),
                                           ctypes.c_void_p(stream_ptr)), "svdmlp_roof_mfma_operands")


def svdmlp_roof_pingpong(steps: int, operands: int, sink_ptr: int, workgroups: int, stream_ptr: int = 0) -> None:
    _check(lib().svdmlp_roof_pingpong(int(steps), int(operands), ctypes.c_void_p(sink_ptr), int(workgroups),
                                      ctypes.c_void_p(stream_ptr)), "svdmlp_roof_pingpong")


def svdmlp_roof_coexec(mfma_iters: int, valu_iters: int, sink_ptr: int, workgroups: int, stream_ptr: int = 0) -> None:
    _check(lib().svdmlp_roof_coexec(int(mfma_iters), int(valu_iters), ctypes.c_void_p(sink_ptr), int(workgroups),
                                    ctypes.c_void_p(stream_ptr)), "svdmlp_roof_coexec")


def svdmlp_roof_empty(workgroups: int, threads: int, stream_ptr: int = 0) -> None:
    _check(lib().svdmlp_roof_empty(int(workgroups), int(threads), ctypes.c_void_p(stream_ptr)), "svdmlp_roof_empty")


def svdmlp_roof_empty_chain(launches: int, workgroups: int, threads: int, stream_ptr: int = 0) -> None:
    _check(lib().svdmlp_roof_empty_chain(int(launches), int(workgroups), int(threads), ctypes.c_void_p(stream_ptr)),
           "svdmlp_roof_empty_chain")


def svdmlp_force_plan(ctx, first_kernel: int = 0, first_ranges: int = 0, down_ranges: int = 0, out_kernel: int = 0) -> None:
    _check(lib().svdmlp_force_plan(ctx, int(first_kernel), int(first_ranges), int(down_ranges), int(out_kernel)),
           "svdmlp_force_plan")


def svdmlp_check(ctx) -> None:
    _check(lib().svdmlp_check(ctx), "svdmlp_check")


def svdmlp_destroy(ctx) -> None:
    lib().svdmlp_destroy(ctx)


def svdmlp_profile_begin(ctx, max_forwards: int) -> None:
    st = lib().svdmlp_profile_begin(ctx, int(max_forwards))
    if st != SVDMLP_OK:
        raise SvdMlpError(st, "svdmlp_profile_begin")


def svdmlp_profile_end(ctx):
    """Returns ({kernel name: average ms}, number of forwards averaged)."""
    ms = (ctypes.c_float * 8)()
    nk, nf = ctypes.c_int(), ctypes.c_int()
    st = lib().svdmlp_profile_end(ctx, ms, ctypes.byref(nk), ctypes.byref(nf))
    if st != SVDMLP_OK:
        raise SvdMlpError(st, "svdmlp_profile_end")
    names = [lib().svdmlp_profile_kernel_name(ctx, k).decode() for k in range(nk.value)]
    return {n: float(ms[k]) for k, n in enumerate(names)}, nf.value


# device index -> raw handle of the current stream there: torch's own function for it where there is one (0.1 us; a Stream
# object takes 2.3)
_current_raw_stream = (getattr(torch._C, "_cuda_getCurrentRawStream", None)
                       or (lambda device: torch.cuda.current_stream(device).cuda_stream))

_TORCH_DTYPE = {torch.bfloat16: SVDMLP_BF16, torch.float32: SVDMLP_F32}


class SvdMlp:
    """A context plus the torch tensors that back it (factors and workspace stay referenced here so
    the device memory outlives the context)."""

    def __init__(self, *, max_M: int, Ug: torch.Tensor, Vg: torch.Tensor, Uu: Optional[torch.Tensor] = None,
                 Vu: Optional[torch.Tensor] = None, Ud: Optional[torch.Tensor] = None, Vd: Optional[torch.Tensor] = None,
                 kind: int = SVDMLP_GATED, flags: int = 0, keep_factors: bool = True):
        self.kind = kind
        self.tensors = [t for t in (Ug, Vg, Uu, Vu, Ud, Vd) if t is not None]
        for t in self.tensors:
            if not (t.is_cuda and t.is_contiguous() and t.dtype == Ug.dtype):
                raise ValueError("factors must be contiguous device tensors of one dtype")
        self.dtype = Ug.dtype
        self.d, self.r = Ug.shape
        self.ffn = Vg.shape[1]
        self.r_down = Ud.shape[1] if Ud is not None else 0
        self.max_M = int(max_M)
        de = svdmlp_desc()
        de.kind, de.dtype = kind, _TORCH_DTYPE[self.dtype]
        de.max_M, de.d, de.ffn, de.r, de.r_down = self.max_M, self.d, self.ffn, self.r, self.r_down
        de.Ug, de.Vg = Ug.data_ptr(), Vg.data_ptr()
        for name, t in (("Uu", Uu), ("Vu", Vu), ("Ud", Ud), ("Vd", Vd)):
            setattr(de, name, t.data_ptr() if t is not None else None)
        de.flags = flags
        nbytes = svdmlp_workspace_bytes(de)
        if nbytes == 0:
            # let create report the precise reason
            de.workspace, de.workspace_bytes = None, 0
            svdmlp_create(de)
            raise SvdMlpError(SVDMLP_UNSUPPORTED, "svdmlp_workspace_bytes")
        self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=Ug.device)
        base = self.workspace.data_ptr()
        de.workspace = (base + 255) // 256 * 256
        de.workspace_bytes = nbytes
        self.workspace_bytes = nbytes
        self.desc = de
        torch.cuda.synchronize(Ug.device)
        self.ctx = svdmlp_create(de)
        if not keep_factors and self.dtype == torch.bfloat16:
            self.tensors = []       # bf16 contexts do not read the factor buffers again after create

    def out_features(self) -> int:
        return self.d if self.kind == SVDMLP_GATED else self.ffn

    def forward(self, X: torch.Tensor, Y: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None):
        if not (X.is_cuda and X.is_contiguous() and X.dtype == self.dtype and X.dim() == 2 and X.shape[1] == self.d):
            raise ValueError("X must be a contiguous [M, d] device tensor of the context's dtype")
        M = X.shape[0]
        if Y is None:
            shape = (M, self.out_features())
            # new_empty of a tensor type of the caller's own would return that type
            Y = X.new_empty(shape) if type(X) is torch.Tensor else torch.empty(shape, dtype=self.dtype, device=X.device)
        # The smallest forwards are bound by this call: the stream's raw handle, new_empty and plain integers for the pointers
        # bring it from 5.8 to 2.7 us beside 2.8 us per launch.
        s = _current_raw_stream(X.get_device()) if stream is None else stream.cuda_stream
        svdmlp_forward(self.ctx, X.data_ptr(), M, Y.data_ptr(), s)
        return Y

    __call__ = forward

    @property
    def last_path(self) -> int:
        return int(lib().svdmlp_last_path(self.ctx))

    def close(self):
        if getattr(self, "ctx", None):
            svdmlp_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---- operators around a factored layer in 8 bits -----------------------------------------------------------------------
# Forward only, as the rest of the binding: results carry no gradient, whatever their inputs require.
class Scaled(NamedTuple):
    """An 8-bit tensor: codes [R, C] (torch.float8_e4m3fn, rows starting on 16 bytes) times scales: activations bfloat16
    [ceil(C / 128), R], one per row and 128 columns; weights float32 [ceil(R / 128), ceil(C / 128)], one per 128 x 128."""
    codes: torch.Tensor
    scales: torch.Tensor

    def to_float(self) -> torch.Tensor:
        """The values it stands for, in float32 (for looking at; the operators take the codes)."""
        R, C = self.codes.shape
        if self.scales.dtype == torch.bfloat16:
            s = self.scales.t().float()
        else:
            s = self.scales.repeat_interleave(SCALE_BLOCK, 0)[:R]
        return self.codes.float() * s.repeat_interleave(SCALE_BLOCK, 1)[:, :C]


def empty_scaled(rows: int, cols: int, device, block_rows: int = 1) -> Scaled:
    """An uninitialised 8-bit tensor, rows of codes padded to 16 bytes."""
    blocks = -(-cols // SCALE_BLOCK)
    codes = torch.empty((rows, (cols + 15) // 16 * 16), dtype=torch.float8_e4m3fn, device=device)
    if cols % 16:
        codes = codes[:, :cols]
    if block_rows == 1:
        return Scaled(codes, torch.empty((blocks, rows), dtype=torch.bfloat16, device=device))
    return Scaled(codes, torch.empty((-(-rows // SCALE_BLOCK), blocks), dtype=torch.float32, device=device))


_F8, _BF16 = torch.float8_e4m3fn, torch.bfloat16


_checks = None


def _tensors():
    """The extension module that checks tensors and packs arguments (raises if it has not been built, or not for this torch)."""
    global _checks
    if _checks is None:
        how = "build it with `python -m paper_2510_25977_amd.build`"
        if not TENSORS_PATH.exists():
            raise FileNotFoundError(f"{TENSORS_PATH} not found: {how}")
        from . import _tensors
        from .build import tensors_for
        if _tensors.built_for != tensors_for():
            raise ImportError(f"{TENSORS_PATH} is built for {_tensors.built_for}, this is {tensors_for()}: {how}")
        _checks = _tensors
    return _checks


def _device_of(t: torch.Tensor, what: str) -> int:
    if not t.is_cuda or t.dim() != 2:
        raise ValueError(f"{what} must be a matrix on the GPU")
    return t.get_device()


_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _on(stream: torch.cuda.Stream, op, t, *args, **kw):
    """op(t, ...) with its launches on `stream`, and the results and workspaces that it makes `stream`'s as well: memory of the
    current stream may be freed memory that work on that stream still uses."""
    device = (t[0] if isinstance(t, tuple) else t).get_device()
    if stream.device_index != device:
        raise ValueError(f"the stream is one of cuda:{stream.device_index}, the tensors are on cuda:{device}")
    with torch.cuda.stream(stream):
        return op(t, *args, **kw)


def _run(name: str, args: Optional[bytes], device: int) -> None:
    if args is None:         # no rows
        return
    op = getattr(lib(), name)
    if device == _current_device():
        st = op(args, _current_raw_stream(device))
    else:                    # kernels are launched on the current device
        with torch.cuda.device(device):
            st = op(args, _current_raw_stream(device))
    if st != SVDMLP_OK:
        raise SvdMlpError(st, name)


def quantize(x: torch.Tensor, gate_with: Optional[torch.Tensor] = None, *, block_rows: int = 1, out=None,
             stream: Optional[torch.cuda.Stream] = None) -> Scaled:
    """x, or SiLU(x) * gate_with, as e4m3 codes with a scale per row and 128 columns (``block_rows=128``: weights, one per
    128 x 128).  x: [R, C] bfloat16 or float32."""
    if stream is not None:
        return _on(stream, quantize, x, gate_with, block_rows=block_rows, out=out)
    dev = _device_of(x, "x")
    if out is None:
        out = empty_scaled(*x.shape, x.device, block_rows)
    codes, scales = out
    _run("svdmlp_quantize", _tensors().quantize_args(dev, x, gate_with, block_rows, codes, scales), dev)
    return out if type(out) is Scaled else Scaled(codes, scales)


def _norm(x, branch, residual, weight, bias, kind, eps, weight_plus, residual_scale, branch_scale, gate, gate_rows, gate_act,
          next_weight, next_bias, next_kind, next_eps, h, out, scaled, want_h):
    """x: the residual, or the branch where there is none: of the residual stream's type"""
    dev = _device_of(x, "x")
    if h is None and want_h:
        h = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    if next_kind == NORM_NONE:
        if out is not None or scaled:
            raise ValueError("out is what the next norm makes, and there is none")
    elif out is None:
        if scaled:
            out = empty_scaled(*x.shape, x.device)
        else:
            of = next((t for t in (branch, weight, next_weight, bias, next_bias) if t is not None), x)
            out = torch.empty(x.shape, dtype=of.dtype, device=x.device)
    if isinstance(out, tuple):
        out = out if type(out) is Scaled else Scaled(*out)
        codes, scales = out
    elif scaled:
        raise ValueError("an 8-bit result goes to a Scaled, out is a plain tensor")
    else:
        codes, scales = out, None
    args = _tensors().norm_args(dev, branch, residual, weight, bias, kind, eps, weight_plus, residual_scale, branch_scale, gate,
                                gate_rows, gate_act, next_weight, next_bias, next_kind, next_eps, h, codes, scales)
    _run("svdmlp_norm", args, dev)
    return h, out


def norm_in(x: torch.Tensor, weight: Optional[torch.Tensor] = None, *, bias: Optional[torch.Tensor] = None,
            add: Optional[torch.Tensor] = None, kind: int = NORM_RMS, eps: float = 1e-6, weight_plus: float = 0.0,
            residual_scale: float = 1.0, h: Optional[torch.Tensor] = None, out=None, scaled: bool = False,
            stream: Optional[torch.cuda.Stream] = None):
    """The norm before a block: norm(residual_scale * x + add) * (weight + weight_plus) + bias, as a tensor of the weights'
    type or, with ``scaled`` (or a ``Scaled`` as ``out``), in 8 bits.  x is the residual stream, float32 or of the weights'
    type; ``add`` what the block before adds to it; the sum goes to ``h`` if that is given (x itself is allowed)."""
    args = (x, add, x, None, None, NORM_NONE, eps, weight_plus, residual_scale, None, None, 1, GATE_PLAIN, weight, bias, kind, eps, h,
            out, scaled, False)
    return (_norm(*args) if stream is None else _on(stream, _norm, *args))[1]


def norm_out(branch: torch.Tensor, residual: Optional[torch.Tensor] = None, weight: Optional[torch.Tensor] = None, *,
             bias: Optional[torch.Tensor] = None, kind: int = NORM_RMS, eps: float = 1e-6, weight_plus: float = 0.0,
             residual_scale: float = 1.0, branch_scale: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None,
             gate_rows: int = 1, gate_act: int = GATE_PLAIN, next_weight: Optional[torch.Tensor] = None,
             next_bias: Optional[torch.Tensor] = None, next_kind: Optional[int] = None, next_eps: Optional[float] = None,
             h: Optional[torch.Tensor] = None, out=None, scaled: bool = False, stream: Optional[torch.cuda.Stream] = None):
    """What follows a block: h = residual_scale * residual + [norm(branch) * (weight + weight_plus) + bias] * branch_scale *
    act(gate[row // gate_rows]).  With a next norm (next_kind, or any of next_weight, next_bias, out and scaled) also the norm
    before the next block, as ``norm_in`` makes it.  Returns (h, out or None); ``h`` may be ``residual``."""
    if next_kind is None:
        wanted = out is not None or scaled or next_weight is not None or next_bias is not None
        next_kind = NORM_RMS if wanted else NORM_NONE
    args = (branch if residual is None else residual, branch, residual, weight, bias, kind, eps, weight_plus, residual_scale,
            branch_scale, gate, gate_rows, gate_act, next_weight, next_bias, next_kind, eps if next_eps is None else next_eps, h, out,
            scaled, True)
    return _norm(*args) if stream is None else _on(stream, _norm, *args)


@functools.lru_cache(maxsize=4096)
def svdmlp_scaled_matmul_workspace_bytes(M: int, N: int, K: int, out_type: int) -> int:
    return int(lib().svdmlp_scaled_matmul_workspace_bytes(int(M), int(N), int(K), int(out_type)))


def svdmlp_scaled_matmul_describe(M: int, N: int, K: int, out_type: int, gated: bool = False) -> str:
    buf = ctypes.create_string_buffer(512)
    _check(lib().svdmlp_scaled_matmul_describe(int(M), int(N), int(K), int(out_type), int(gated), buf, len(buf)),
           "svdmlp_scaled_matmul_describe")
    return buf.value.decode()


def scaled_matmul(a, w, *, gated: bool = False, out=None, out_dtype: torch.dtype = torch.bfloat16,
                  stream: Optional[torch.cuda.Stream] = None):
    """a [M, K] times the transpose of w [N, K], both ``Scaled`` (or pairs of codes and scales): activations with a scale per
    row and 128 columns, weights with one per 128 x 128.  The result [M, N] is ``out`` or a new tensor of ``out_dtype``;
    torch.float8_e4m3fn (or a ``Scaled`` as ``out``) makes it the next product's activations.  ``gated``: the two halves of K
    (a multiple of 256) are a gate and an up product side by side, the result SiLU(gate) * up."""
    if stream is not None:
        return _on(stream, scaled_matmul, tuple(a), w, gated=gated, out=out, out_dtype=out_dtype)
    codes, scales = a
    w_codes, w_scales = w
    dev = _device_of(codes, "a")
    M, K = codes.shape
    if w_codes.dim() != 2:
        raise ValueError(f"w must be [N, {K}]")
    N = w_codes.shape[0]
    if out is None:
        if out_dtype is not _BF16 and out_dtype is not _F8:
            raise ValueError("out_dtype must be bfloat16 or float8_e4m3fn")
        out = empty_scaled(M, N, codes.device) if out_dtype is _F8 else torch.empty((M, N), dtype=_BF16, device=codes.device)
    if isinstance(out, tuple):
        out = out if type(out) is Scaled else Scaled(*out)
        c, c_scales = out
    elif out_dtype is _F8:
        raise ValueError("an 8-bit result goes to a Scaled, out is a plain tensor")
    else:
        c, c_scales = out, None
    need = 0 if gated else svdmlp_scaled_matmul_workspace_bytes(M, N, K, SVDMLP_BF16 if c_scales is None else SVDMLP_F8)
    space = torch.empty(need, dtype=torch.uint8, device=codes.device) if need else None
    args = _tensors().scaled_matmul_args(dev, M, N, K, codes, scales, w_codes, w_scales, c, c_scales, space, bool(gated))
    _run("svdmlp_scaled_matmul", args, dev)
    return out


class SvdMlpF8:
    """``SvdMlp`` in 8 bits: the factors are quantised once (a scale per 128 x 128), activations between the products carry a
    scale per row and 128 columns, the result is bfloat16.  ``kind`` and the factors are ``SvdMlp``'s (any strides; not needed
    afterwards); there is no context, no flags and no max_M: rows as many as the operators take.  On another stream than that of
    its construction the block may be called at once; it has to live until what it was called for there is done.

    Half the weight bytes for an error of about 0.09 of the result in the root mean square.  Faster than ``SvdMlp`` from about 100
    rows on, not below (4096 x 14336, rank 512, from codes, in a graph: 21.5 us, bfloat16 20.1, at one row; 46.7, 63.1 at 512; 183,
    234 at 4096); and slow at few rows where ffn is small beside the rank, since the gated product does not cut its contraction."""

    def __init__(self, *, Ug: torch.Tensor, Vg: torch.Tensor, Uu: Optional[torch.Tensor] = None, Vu: Optional[torch.Tensor] = None,
                 Ud: Optional[torch.Tensor] = None, Vd: Optional[torch.Tensor] = None, kind: int = SVDMLP_GATED):
        if kind not in (SVDMLP_GATED, SVDMLP_LINEAR):
            raise ValueError("kind must be SVDMLP_GATED or SVDMLP_LINEAR")
        if kind == SVDMLP_GATED and any(t is None for t in (Uu, Vu, Ud, Vd)):
            raise ValueError("a gated block has six factors")
        used = [Ug, Vg] if kind == SVDMLP_LINEAR else [Ug, Vg, Uu, Vu, Ud, Vd]
        for t in used:
            if not (t.is_cuda and t.dim() == 2 and t.dtype == Ug.dtype and t.device == Ug.device) or t.dtype not in _TORCH_DTYPE:
                raise ValueError("factors must be device matrices of one dtype, bfloat16 or float32")
        self.kind = kind
        self.d, self.r = Ug.shape
        self.ffn = Vg.shape[1]
        self.r_down = Ud.shape[1] if kind == SVDMLP_GATED else 0
        shapes = [(self.d, self.r), (self.r, self.ffn)] * (len(used) // 4 + 1)
        shapes = shapes[:len(used)] if kind == SVDMLP_LINEAR else shapes[:4] + [(self.ffn, self.r_down), (self.r_down, self.d)]
        if [tuple(t.shape) for t in used] != shapes:
            raise ValueError(f"factor shapes {[tuple(t.shape) for t in used]} do not make a block, expected {shapes}")

        def weights(*parts):
            """Products take weights as [columns, contraction]; a rank ends on a block of 128, zero columns behind it."""
            return quantize(torch.cat([p.t() for p in parts]), block_rows=SCALE_BLOCK)

        def ranked(U):
            return torch.nn.functional.pad(U, (0, -U.shape[1] % SCALE_BLOCK))

        def rank_rows(V):
            return torch.nn.functional.pad(V, (0, 0, 0, -V.shape[0] % SCALE_BLOCK))

        if kind == SVDMLP_LINEAR:
            self.first, self.last = weights(ranked(Ug)), weights(rank_rows(Vg))
        else:
            self.first = weights(ranked(Ug), ranked(Uu))
            self.gate_up = quantize(torch.cat([rank_rows(Vg).t(), rank_rows(Vu).t()], 1), block_rows=SCALE_BLOCK)
            self.down, self.last = weights(ranked(Ud)), weights(rank_rows(Vd))
        # A forward may run on another stream than this one, and nothing orders it after the quantiser: so, as SvdMlp's, its
        # operands are there when it is.  (A stream that is being captured cannot be waited for: the graph quantises.)
        with torch.cuda.device(Ug.device):
            if not torch.cuda.is_current_stream_capturing():
                torch.cuda.current_stream().synchronize()

    def out_features(self) -> int:
        return self.d if self.kind == SVDMLP_GATED else self.ffn

    def forward(self, X, out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
        """X: [M, d] bfloat16 or float32, or ``Scaled`` as ``norm_in`` makes it.  The result is ``out`` or a new tensor."""
        if stream is not None:
            return _on(stream, self.forward, X, out)
        if not isinstance(X, tuple):
            X = quantize(X)
        T = scaled_matmul(X, self.first, out_dtype=_F8)
        if self.kind == SVDMLP_GATED:
            H = scaled_matmul(T, self.gate_up, gated=True, out_dtype=_F8)
            T = scaled_matmul(H, self.down, out_dtype=_F8)
        return scaled_matmul(T, self.last, out=out)

    __call__ = forward
