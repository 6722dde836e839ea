"""ctypes binding of the C-ABI CUDA library (``include/sol_nvfp4.h``).

Argument marshalling only: torch supplies device memory and the current stream, every
compute step runs in the library's kernels.  There is no fallback: if the library is
missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import functools
import os
import struct
import types

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("SOL_NVFP4_LIB", os.path.join(_HERE, "libsol_nvfp4.so"))

SF_ROW_MAJOR = 0
SF_SWIZZLED_128x4 = 1

EXPORTS = [
    "sol_status_string", "sol_nvfp4_data_bytes", "sol_nvfp4_scale_bytes",
    "sol_nvfp4_linear_workspace_bytes", "sol_amax_bf16", "nvfp4_quantize", "nvfp4_quantize_weight",
    "nvfp4_linear", "bf16_linear", "nvfp4_quantize_linear", "sol_last_device_status",
    "sol_nvfp4_static_scratch_bytes", "nvfp4_quantize_linear_static", "nvfp4_quantize_linear_host",
    "nvfp4_requantize_lora", "nvfp4_requantize_lora_batch", "nvfp4_linear_quantized_out",
    "solrl_select_contrastive", "solrl_rank_consistency", "sol_mxfp4_scale_bytes", "mxfp4_quantize",
    "mxfp4_linear", "nvfp4_linear_split_out", "nvfp4_quantize_into",
    "nvfp4_quantize_linear_delayed", "sol_roll_tensor_scale", "nvfp4_layernorm_quantize", "sol_attention_bf16", "sol_attention_bf16_joint",
    "sol_attention_nvfp4_out", "mxfp4_linear_quantized_out", "sol_set_wait_limit_cycles", "sol_test_hold_loads",
    "mxfp4_linear_split_out", "mxfp4_quantize_into", "sol_qk_rotary", "sol_qk_rotary_backward",
    "sol_qk_rotary_backward_workspace_bytes", "sol_rotary_frequencies", "nvfp4_matvec", "mxfp4_matvec",
    "sol_matvec_workspace_bytes", "sol_select_blocks", "sol_select_blocks_workspace_bytes", "sol_attention_blocks",
    "sol_layernorm", "sol_layernorm_backward", "sol_layernorm_backward_workspace_bytes", "sol_adamw_step",
    "sol_lora_apply", "sol_lora_backward", "sol_lora_workspace_bytes",
]

_lib = None


class SolError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {status_string(code)} ({code})")


def lib() -> ctypes.CDLL:
    """Load the CUDA library; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2604_06916_b200.build` "
            "(there is no CPU or PyTorch fallback)")
    L = ctypes.CDLL(LIB_PATH)
    vp, i64, sz, i32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t, ctypes.c_int
    L.sol_status_string.restype, L.sol_status_string.argtypes = ctypes.c_char_p, [i32]
    L.sol_nvfp4_data_bytes.restype, L.sol_nvfp4_data_bytes.argtypes = sz, [i64, i64]
    L.sol_nvfp4_scale_bytes.restype, L.sol_nvfp4_scale_bytes.argtypes = sz, [i64, i64, i32]
    L.sol_nvfp4_linear_workspace_bytes.restype = sz
    L.sol_nvfp4_linear_workspace_bytes.argtypes = [i64, i64, i64]
    L.sol_amax_bf16.restype, L.sol_amax_bf16.argtypes = i32, [vp, i64, i64, i64, vp, vp]
    L.nvfp4_quantize.restype, L.nvfp4_quantize.argtypes = i32, [vp, i64, i64, i64, vp, vp, vp, i32, vp]
    L.nvfp4_quantize_weight.restype = i32
    L.nvfp4_quantize_weight.argtypes = [vp, i64, i64, i64, vp, vp, vp, i32, vp]
    L.nvfp4_linear.restype = i32
    L.nvfp4_linear.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, i64, i64, i64, i64, vp]
    L.bf16_linear.restype = i32
    L.bf16_linear.argtypes = [vp, vp, vp, vp, i64, i64, i64, i64, i64, i64, vp]
    L.nvfp4_quantize_linear.restype = i32
    L.nvfp4_quantize_linear.argtypes = [vp, i64, vp, vp, vp, vp, vp, i64, i64, i64, i64, vp, sz, vp]
    L.sol_nvfp4_static_scratch_bytes.restype, L.sol_nvfp4_static_scratch_bytes.argtypes = sz, []
    L.nvfp4_quantize_linear_static.restype = i32
    L.nvfp4_quantize_linear_static.argtypes = [vp, i64, vp, vp, vp, vp, vp, i64, i64, i64, i64, vp]
    L.nvfp4_quantize_linear_host.restype = i32
    L.nvfp4_quantize_linear_host.argtypes = [vp, i64, vp, vp, vp, vp, vp, i64, i64, i64, i64, vp, vp, vp, sz, vp]
    L.nvfp4_requantize_lora.restype = i32
    L.nvfp4_requantize_lora.argtypes = [vp, i64, vp, i64, vp, i64, i64, i64, i64, ctypes.c_float, vp, vp, vp, vp,
                                        i32, vp]
    L.nvfp4_requantize_lora_batch.restype = i32
    L.nvfp4_requantize_lora_batch.argtypes = [i64, vp, vp, vp, vp, vp, vp, i64, i64, i64, ctypes.c_float, vp, i64,
                                              i32, vp]
    L.nvfp4_linear_quantized_out.restype = i32
    L.nvfp4_linear_quantized_out.argtypes = [vp, vp, vp, vp, vp, vp, vp, i32, vp, vp, vp, vp, i64, i64, i64, vp]
    L.solrl_select_contrastive.restype = i32
    L.solrl_select_contrastive.argtypes = [vp, vp, i64, i64, i64, vp, vp, vp, vp]
    L.solrl_rank_consistency.restype = i32
    L.solrl_rank_consistency.argtypes = [vp, vp, i64, i64, i64, vp, vp, vp]
    L.sol_mxfp4_scale_bytes.restype, L.sol_mxfp4_scale_bytes.argtypes = sz, [i64, i64, i32]
    L.mxfp4_quantize.restype, L.mxfp4_quantize.argtypes = i32, [vp, i64, i64, i64, vp, vp, i32, vp]
    L.mxfp4_linear.restype, L.mxfp4_linear.argtypes = i32, [vp, vp, vp, vp, vp, vp, i64, i64, i64, i64, vp]
    L.nvfp4_linear_split_out.restype = i32
    L.nvfp4_linear_split_out.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, i64, i64, i32, vp, vp, vp, i64, i64, vp, i64,
                                         i64, i64, vp]
    L.nvfp4_quantize_into.restype = i32
    L.nvfp4_quantize_into.argtypes = [vp, i64, i64, i64, vp, vp, vp, i64, i64, vp]
    L.nvfp4_quantize_linear_delayed.restype = i32
    L.nvfp4_quantize_linear_delayed.argtypes = [vp, i64, vp, vp, vp, vp, vp, i64, i64, i64, i64, vp, vp, sz, vp]
    L.sol_roll_tensor_scale.restype, L.sol_roll_tensor_scale.argtypes = i32, [vp, vp]
    L.sol_attention_bf16_joint.restype = i32
    L.sol_attention_bf16_joint.argtypes = [ctypes.POINTER(AttentionStream), ctypes.POINTER(AttentionStream), i64, i64, i64, vp]
    L.mxfp4_linear_quantized_out.restype = i32
    L.mxfp4_linear_quantized_out.argtypes = [vp, vp, vp, vp, vp, i32, vp, vp, vp, i64, i64, i64, vp]
    L.sol_attention_nvfp4_out.restype = i32
    L.sol_attention_nvfp4_out.argtypes = [vp, vp, vp, i64, i64, i64, i64, i64, i64, i64, i64, vp, vp, vp, i64, i64, vp, vp]
    L.sol_attention_bf16.restype = i32
    L.sol_attention_bf16.argtypes = [vp, vp, vp, vp, i64, i64, i64, i64, i64, i64, i64, i64, i64, vp]
    L.nvfp4_layernorm_quantize.restype = i32
    L.nvfp4_layernorm_quantize.argtypes = [vp, i64, i64, i64, vp, vp, i64, ctypes.c_float, vp, vp, vp, vp, vp]
    L.mxfp4_linear_split_out.restype = i32
    L.mxfp4_linear_split_out.argtypes = [vp, vp, vp, vp, vp, vp, i64, i64, i32, vp, vp, i64, i64, vp, i64, i64, i64, vp]
    L.mxfp4_quantize_into.restype = i32
    L.mxfp4_quantize_into.argtypes = [vp, i64, i64, i64, vp, vp, i64, i64, vp]
    f32, f64 = ctypes.c_float, ctypes.c_double
    L.nvfp4_matvec.restype = L.mxfp4_matvec.restype = i32
    L.nvfp4_matvec.argtypes = [vp, i64, vp, vp, vp, vp, i32, vp, i64, i64, i64, i64, vp, sz, vp]
    L.mxfp4_matvec.argtypes = [vp, i64, vp, vp, vp, i32, vp, i64, i64, i64, i64, vp, sz, vp]
    L.sol_matvec_workspace_bytes.restype, L.sol_matvec_workspace_bytes.argtypes = sz, [i64, i64]
    L.sol_select_blocks_workspace_bytes.restype, L.sol_select_blocks_workspace_bytes.argtypes = sz, [i64] * 6
    L.sol_select_blocks.restype = i32
    L.sol_select_blocks.argtypes = [vp, vp] + [i64] * 10 + [vp, vp, vp, vp, vp, sz, vp]
    L.sol_attention_blocks.restype = i32
    L.sol_attention_blocks.argtypes = [vp, vp, vp, vp] + [i64] * 10 + [vp, vp, i64, vp, vp]
    L.sol_qk_rotary.restype = i32
    L.sol_qk_rotary.argtypes = [vp, vp, i64, i64, vp, f32, vp]
    L.sol_qk_rotary_backward.restype = i32
    L.sol_qk_rotary_backward.argtypes = [vp, vp, i64, i64, vp, f32, vp, sz, vp]
    L.sol_qk_rotary_backward_workspace_bytes.restype, L.sol_qk_rotary_backward_workspace_bytes.argtypes = sz, [i64]
    L.sol_rotary_frequencies.restype = i32
    L.sol_rotary_frequencies.argtypes = [i64, f64, i32, f64, f64, f64, f64, vp, vp]
    L.sol_layernorm.restype = i32
    L.sol_layernorm.argtypes = [vp, i64, i64, i64, vp, vp, i64, i64, f32, f32, vp, i64, vp, vp]
    L.sol_layernorm_backward.restype = i32
    L.sol_layernorm_backward.argtypes = [vp, i64, vp, i64, vp, vp, i64, i64, i64, i64, f32, vp, i64, vp, vp, vp, sz, vp]
    L.sol_layernorm_backward_workspace_bytes.restype = sz
    L.sol_layernorm_backward_workspace_bytes.argtypes = [i64, i64, i64]
    L.sol_adamw_step.restype, L.sol_adamw_step.argtypes = i32, [vp, i64, vp, vp, vp]
    L.sol_lora_workspace_bytes.restype, L.sol_lora_workspace_bytes.argtypes = sz, [i64] * 6 + [i32]
    L.sol_lora_apply.restype = i32
    L.sol_lora_apply.argtypes = [vp, i64, vp, vp, vp, vp, vp, i64, i64, vp, i64, vp, i64, i64, i64, i64, vp, sz, vp]
    L.sol_lora_backward.restype = i32
    L.sol_lora_backward.argtypes = [vp, i64, vp, i64, vp, vp, vp, vp, vp, vp, i64, i64, vp, i64, vp, vp, i64, i64, i64, i64, vp, sz, vp]
    L.sol_set_wait_limit_cycles.restype, L.sol_set_wait_limit_cycles.argtypes = i32, [i64]
    L.sol_test_hold_loads.restype, L.sol_test_hold_loads.argtypes = i32, [i32]
    L.sol_last_device_status.restype = i32
    L.sol_last_device_status.argtypes = [vp, ctypes.POINTER(ctypes.c_uint32)]
    _lib = L
    return L


def status_string(code: int) -> str:
    return lib().sol_status_string(int(code)).decode()


def _check(code: int, where: str) -> None:
    if code != 0:
        raise SolError(code, where)


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


# Guard bands (debugging aid, off unless SOL_NVFP4_GUARD=1): every output this module allocates sits between
# two 4 KB bands of a fixed byte, and after each call the device is synchronised and the bands are checked, so
# a kernel that writes outside its output is caught by the call that did it.  Callers' own `out=` buffers
# are theirs to guard.
GUARD_BYTES = 4096
GUARD_BYTE = 0xA5
_guard_pending: list = []
_guarding = False        # inside a guarded call


def guard_mode() -> bool:
    if "SOL_NVFP4_GUARD" not in os.environ or os.environ["SOL_NVFP4_GUARD"] in ("", "0"):
        return False
    # a capture records the bands' fills without running them, and must not be synchronised: nothing to check there
    return not (torch.cuda.is_available() and torch.cuda.is_current_stream_capturing())


def _empty(shape, dtype, device) -> torch.Tensor:
    """torch.empty, or (guard mode) a view between two guard bands of one larger allocation."""
    if not guard_mode():
        return torch.empty(shape, dtype=dtype, device=device)
    shape = (shape,) if isinstance(shape, int) else tuple(shape)
    n = 1
    for d in shape:
        n *= int(d)
    nbytes = n * torch.empty((), dtype=dtype).element_size()
    padded = (nbytes + 255) // 256 * 256          # the back band starts on a 256-byte boundary
    raw = torch.empty(2 * GUARD_BYTES + padded, dtype=torch.uint8, device=device)
    raw[:GUARD_BYTES].fill_(GUARD_BYTE)
    raw[GUARD_BYTES + nbytes:].fill_(GUARD_BYTE)
    _guard_pending.append((raw, nbytes))
    return raw[GUARD_BYTES:GUARD_BYTES + nbytes].view(dtype).view(shape)


def check_guards(where: str = "") -> None:
    """Verify and forget the guard bands of the outputs allocated since the last check."""
    pending, bad = list(_guard_pending), []
    _guard_pending.clear()
    if not pending:
        return
    if pending[0][0].is_cuda:
        torch.cuda.synchronize()
    for raw, nbytes in pending:
        front = bool((raw[:GUARD_BYTES] == GUARD_BYTE).all())
        back = bool((raw[GUARD_BYTES + nbytes:] == GUARD_BYTE).all())
        if not (front and back):
            bad.append(f"{nbytes}-byte output: {'front' if not front else 'back'} band overwritten")
    if bad:
        raise AssertionError(f"{where}: write outside an output buffer ({'; '.join(bad)})")


def _guarded(fn):
    @functools.wraps(fn)
    def call(*args, **kwargs):
        global _guarding
        if not guard_mode():
            return fn(*args, **kwargs)
        _guarding = True
        try:
            return fn(*args, **kwargs)
        finally:
            _guarding = False
            check_guards(fn.__name__)
    return call


def _on_device_of_first(fn):
    """Run `fn` with the device of its first argument current: its launches, its outputs and its stream (the
    current one of that device) are then that device's, whichever device the caller has current.  The guard bands are
    checked here as well, in one wrapper: these calls are a few microseconds of GPU work at their smallest."""
    guarded = _guarded(fn)
    name = fn.__code__.co_varnames[0]

    @functools.wraps(fn)
    def call(*args, **kwargs):
        if args:
            first = args[0]
        elif name in kwargs:
            first = kwargs[name]
        else:
            return fn(**kwargs)                   # raises: the message names what is missing
        index = first.get_device() if isinstance(first, torch.Tensor) else -1
        if index < 0:
            raise TypeError(f"{fn.__name__}: expected CUDA tensors")
        run = guarded if guard_mode() else fn
        if index == torch._C._cuda_getDevice():
            return run(*args, **kwargs)
        with torch.cuda.device(first.device):
            return run(*args, **kwargs)
    call._guards_itself = True
    return call


def _raw_stream(index: int) -> int:
    """Handle of the current stream of device `index` (no Stream object is built)."""
    return torch._C._cuda_getCurrentRawStream(index)


def _new(x: torch.Tensor, shape, dtype=None) -> torch.Tensor:
    """An output on x's device (of x's type unless one is given)."""
    if _guarding:
        return _empty(shape, x.dtype if dtype is None else dtype, x.device)
    return x.new_empty(shape) if dtype is None else x.new_empty(shape, dtype=dtype)


def _like(x: torch.Tensor) -> torch.Tensor:
    """A dense output of x's shape and type."""
    return _empty(tuple(x.shape), x.dtype, x.device) if _guarding else torch.empty_like(x, memory_format=torch.contiguous_format)


def _ptr(t) -> int | None:
    return None if t is None else t.data_ptr()


def data_bytes(rows: int, K: int) -> int:
    return lib().sol_nvfp4_data_bytes(rows, K)


def scale_bytes(rows: int, K: int, layout: int = SF_SWIZZLED_128x4) -> int:
    return lib().sol_nvfp4_scale_bytes(rows, K, layout)


def linear_workspace_bytes(M: int, N: int, K: int) -> int:
    return lib().sol_nvfp4_linear_workspace_bytes(M, N, K)


def _need_2d_bf16(x: torch.Tensor, name: str):
    if x.dtype != torch.bfloat16 or x.dim() != 2 or x.stride(1) != 1 or not x.is_cuda:
        raise TypeError(f"{name}: expected a 2-D CUDA bf16 tensor with contiguous rows")


def sol_amax_bf16(x: torch.Tensor, out: torch.Tensor | None = None) -> torch.Tensor:
    """Per-tensor scale T = max|x| / 2688 (1 for zeros) as a 1-element float32 device tensor."""
    _need_2d_bf16(x, "x")
    if out is None:
        out = _empty(1, torch.float32, x.device)
    _check(lib().sol_amax_bf16(_ptr(x), x.shape[0], x.shape[1], x.stride(0), _ptr(out), _stream()), "sol_amax_bf16")
    return out


def _alloc_q(rows: int, K: int, layout: int, device):
    nq, ns = data_bytes(rows, K), scale_bytes(rows, K, layout)
    if nq == 0 or ns == 0:
        raise SolError(2, "shape check")
    q = _empty((rows, K // 2), torch.uint8, device)
    sf = _empty(ns, torch.uint8, device)
    return q, sf


def nvfp4_quantize(x: torch.Tensor, tensor_scale: torch.Tensor, layout: int = SF_SWIZZLED_128x4,
                   out: tuple[torch.Tensor, torch.Tensor] | None = None):
    """BF16 [M, K] -> (packed nibbles uint8 [M, K/2], E4M3 scales uint8 flat buffer)."""
    _need_2d_bf16(x, "x")
    M, K = x.shape
    q, sf = out if out is not None else _alloc_q(M, K, layout, x.device)
    _check(lib().nvfp4_quantize(_ptr(x), M, K, x.stride(0), _ptr(tensor_scale), _ptr(q), _ptr(sf), layout,
                                _stream()), "nvfp4_quantize")
    return q, sf


def nvfp4_quantize_weight(w: torch.Tensor, layout: int = SF_SWIZZLED_128x4):
    """BF16 [N, K] -> (packed nibbles, scales, per-tensor scale T_w)."""
    _need_2d_bf16(w, "w")
    N, K = w.shape
    q, sf = _alloc_q(N, K, layout, w.device)
    ts = _empty(1, torch.float32, w.device)
    _check(lib().nvfp4_quantize_weight(_ptr(w), N, K, w.stride(0), _ptr(q), _ptr(sf), _ptr(ts), layout, _stream()),
           "nvfp4_quantize_weight")
    return q, sf, ts


def nvfp4_requantize_lora(w: torch.Tensor, lora_a: torch.Tensor, lora_b: torch.Tensor, scaling: float,
                          layout: int = SF_SWIZZLED_128x4, merged: torch.Tensor | None = None, out=None):
    """Merge adapters (W + scaling * B A, BF16) and quantize: (merged W', nibbles, scales, T).

    ``out`` = (q, sf, ts) supplies the output buffers; ts holds two floats (T and the entry
    point's scratch word), the returned T is a view of its first element.
    """
    _need_2d_bf16(w, "w")
    _need_2d_bf16(lora_a, "lora_a")
    _need_2d_bf16(lora_b, "lora_b")
    N, K = w.shape
    r = lora_a.shape[0]
    if lora_a.shape[1] != K or tuple(lora_b.shape) != (N, r):
        raise ValueError("shapes: w [N, K], lora_a [r, K], lora_b [N, r]")
    if merged is None:
        merged = _empty((N, K), torch.bfloat16, w.device)
    if out is None:
        q, sf = _alloc_q(N, K, layout, w.device)
        ts2 = _empty(2, torch.float32, w.device)
    else:
        q, sf, ts2 = out
        if ts2.numel() < 2:
            raise ValueError("ts must hold two floats")
    _check(lib().nvfp4_requantize_lora(_ptr(w), w.stride(0), _ptr(lora_a), lora_a.stride(0), _ptr(lora_b),
                                       lora_b.stride(0), N, K, r, float(scaling), _ptr(merged), _ptr(q),
                                       _ptr(sf), _ptr(ts2), layout, _stream()), "nvfp4_requantize_lora")
    return merged, q, sf, ts2[:1]


class LoraRefreshPlan:
    """Pointer lists for nvfp4_requantize_lora_batch, built once for a set of same-shaped matrices.

    ``items`` = [(w, lora_a, lora_b), ...]; the outputs (q, sf, ts) are allocated here and kept in
    ``outputs``; ``run()`` re-quantizes all of them with one call into the library, ``group``
    matrices per launch (the merged-weight scratch holds that many).
    """

    def __init__(self, items, scaling: float, layout: int = SF_SWIZZLED_128x4, group: int = 8):
        if not items:
            raise ValueError("no matrices")
        N, K = items[0][0].shape
        r = items[0][1].shape[0]
        for w, a, b in items:
            for t, name in ((w, "w"), (a, "lora_a"), (b, "lora_b")):
                _need_2d_bf16(t, name)
                if not t.is_contiguous():
                    raise ValueError(f"{name} must be dense")
            if tuple(w.shape) != (N, K) or tuple(a.shape) != (r, K) or tuple(b.shape) != (N, r):
                raise ValueError("all matrices of a plan share one shape")
        dev = items[0][0].device
        self.items = list(items)
        self.N, self.K, self.r, self.scaling, self.layout = N, K, r, float(scaling), layout
        self.group = max(1, min(group, len(items)))
        self.merged = _empty((self.group, N, K), torch.bfloat16, dev)
        self.outputs = []
        for _ in items:
            q, sf = _alloc_q(N, K, layout, dev)
            self.outputs.append((q, sf, _empty(2, torch.float32, dev)))
        n = len(items)
        arr = ctypes.c_void_p * n
        self._lists = [arr(*[t[i].data_ptr() for t in items]) for i in range(3)] + \
                      [arr(*[o[i].data_ptr() for o in self.outputs]) for i in range(3)]

    def run(self):
        _check(lib().nvfp4_requantize_lora_batch(len(self.items), *self._lists, self.N, self.K, self.r,
                                                 self.scaling, _ptr(self.merged), self.group, self.layout, _stream()),
               "nvfp4_requantize_lora_batch")
        return self.outputs


def nvfp4_linear(xq, xsf, x_tscale, wq, wsf, w_tscale, bias=None, out: torch.Tensor | None = None):
    """Y = dequant(X) . dequant(W)^T + bias in BF16 from quantized operands (swizzled scales)."""
    M, K = xq.shape[0], xq.shape[1] * 2
    N = wq.shape[0]
    if out is None:
        out = _empty((M, N), torch.bfloat16, xq.device)
    _check(lib().nvfp4_linear(_ptr(xq), _ptr(xsf), _ptr(x_tscale), _ptr(wq), _ptr(wsf), _ptr(w_tscale), _ptr(bias),
                              _ptr(out), M, N, K, out.stride(0), _stream()), "nvfp4_linear")
    return out


ACT_NONE, ACT_GELU_TANH, ACT_SILU = 0, 1, 2


def nvfp4_linear_split_out(xq, xsf, x_tscale, wq, wsf, w_tscale, bias, n_split: int, activation: int, out_tscale,
                           dest, dest_col0: int, y_out: torch.Tensor | None = None,
                           amax_out: torch.Tensor | None = None):
    """Columns below n_split -> BF16 `y_out`; the rest -> activation -> quantized into dest = (q [M, dest_K/2], sf)."""
    M, K = xq.shape[0], xq.shape[1] * 2
    N = wq.shape[0]
    hq, hsf = dest
    dest_K = hq.shape[1] * 2
    if y_out is None:
        y_out = _empty((M, n_split), torch.bfloat16, xq.device)
    _check(lib().nvfp4_linear_split_out(_ptr(xq), _ptr(xsf), _ptr(x_tscale), _ptr(wq), _ptr(wsf), _ptr(w_tscale),
                                        _ptr(bias), _ptr(y_out), y_out.stride(0), n_split, activation, _ptr(out_tscale),
                                        _ptr(hq), _ptr(hsf), dest_K, dest_col0, _ptr(amax_out), M, N, K, _stream()),
           "nvfp4_linear_split_out")
    return y_out


def nvfp4_quantize_into(x: torch.Tensor, tensor_scale: torch.Tensor, dest, dest_col0: int):
    """Quantize BF16 x [M, K] into columns [dest_col0, dest_col0 + K) of dest = (q [M, dest_K/2], sf)."""
    _need_2d_bf16(x, "x")
    M, K = x.shape
    hq, hsf = dest
    _check(lib().nvfp4_quantize_into(_ptr(x), M, K, x.stride(0), _ptr(tensor_scale), _ptr(hq), _ptr(hsf),
                                     hq.shape[1] * 2, dest_col0, _stream()), "nvfp4_quantize_into")


def nvfp4_quantize_linear_delayed(x, wq, wsf, w_tscale, bias, scale_state: torch.Tensor,
                                  workspace: torch.Tensor | None = None, out: torch.Tensor | None = None):
    """Fused quantize + NVFP4 linear with T = scale_state[0]; max|x| is accumulated into scale_state[1]."""
    _need_2d_bf16(x, "x")
    M, K = x.shape
    N = wq.shape[0]
    if workspace is None:
        workspace = _empty(linear_workspace_bytes(M, N, K), torch.uint8, x.device)
    if out is None:
        out = _empty((M, N), torch.bfloat16, x.device)
    _check(lib().nvfp4_quantize_linear_delayed(_ptr(x), x.stride(0), _ptr(wq), _ptr(wsf), _ptr(w_tscale), _ptr(bias),
                                               _ptr(out), M, N, K, out.stride(0), _ptr(scale_state), _ptr(workspace),
                                               workspace.numel(), _stream()), "nvfp4_quantize_linear_delayed")
    return out


def sol_roll_tensor_scale(scale_state: torch.Tensor):
    _check(lib().sol_roll_tensor_scale(_ptr(scale_state), _stream()), "sol_roll_tensor_scale")


def nvfp4_layernorm_quantize(x, scale, shift, rows_per_sample: int, tensor_scale, eps: float = 1e-6,
                             amax_out: torch.Tensor | None = None, out=None):
    """LN(x) * (1 + scale[sample]) + shift[sample], quantized for the next linear: (nibbles, swizzled scales)."""
    _need_2d_bf16(x, "x")
    _need_2d_bf16(scale, "scale")
    _need_2d_bf16(shift, "shift")
    M, K = x.shape
    if out is None:
        out = _alloc_q(M, K, SF_SWIZZLED_128x4, x.device)
    q, sf = out
    _check(lib().nvfp4_layernorm_quantize(_ptr(x), M, K, x.stride(0), _ptr(scale), _ptr(shift), rows_per_sample,
                                          float(eps), _ptr(tensor_scale), _ptr(q), _ptr(sf), _ptr(amax_out), _stream()),
           "nvfp4_layernorm_quantize")
    return q, sf


class AttentionStream(ctypes.Structure):
    """sol_attention_stream_t of the C header."""
    _fields_ = [("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("out", ctypes.c_void_p),
                ("seq", ctypes.c_int64), ("ld_q", ctypes.c_int64), ("ld_k", ctypes.c_int64), ("ld_v", ctypes.c_int64),
                ("ld_out", ctypes.c_int64)]


def _token_pitch(t: torch.Tensor) -> int:
    """Elements between consecutive tokens of a [B, S, H, D] view (a dimension of extent 1 has no meaningful stride)."""
    if t.shape[1] > 1:
        return t.stride(1)
    return t.stride(0) if t.shape[0] > 1 else t.shape[2] * t.shape[3]


def _check_attention_view(name: str, t: torch.Tensor):
    if t.dtype != torch.bfloat16 or t.dim() != 4 or t.shape[3] not in (64, 128):
        raise ValueError(f"{name} must be a [B, S, H, D] BF16 tensor with D = 64 or 128")
    if t.stride(3) != 1 or (t.shape[2] > 1 and t.stride(2) != t.shape[3]) or \
            (t.shape[0] > 1 and t.shape[1] > 1 and t.stride(0) != t.shape[1] * t.stride(1)):
        raise ValueError(f"{name}: heads and head dimension must be contiguous, batches stacked densely")


def sol_attention_bf16_joint(first, second, out=None):
    """Joint attention of two token streams: first = (q, k, v) of the stream whose tokens come first.

    Every tensor is a [B, S_stream, H, D] view as in sol_attention_bf16; S of the first stream is a
    multiple of 256.  Returns (out_first, out_second), each [B, S_stream, H, D].
    """
    streams = []
    outs = list(out) if out is not None else [None, None]
    for i, (q, k, v) in enumerate((first, second)):
        for name, t in (("q", q), ("k", k), ("v", v)):
            _check_attention_view(name, t)
        if q.shape != k.shape or q.shape != v.shape:
            raise ValueError("q, k and v of a stream must have one shape")
        if outs[i] is None:
            outs[i] = _empty(tuple(q.shape), torch.bfloat16, q.device)
        _check_attention_view("out", outs[i])
        streams.append(AttentionStream(_ptr(q), _ptr(k), _ptr(v), _ptr(outs[i]), q.shape[1], _token_pitch(q),
                                       _token_pitch(k), _token_pitch(v), _token_pitch(outs[i])))
    B_, _, H, D = first[0].shape
    if second[0].shape[0] != B_ or second[0].shape[2] != H or second[0].shape[3] != D:
        raise ValueError("both streams must share batch, heads and head dimension")
    _check(lib().sol_attention_bf16_joint(ctypes.byref(streams[0]), ctypes.byref(streams[1]), B_, H, D, _stream()),
           "sol_attention_bf16_joint")
    return outs[0], outs[1]


def sol_attention_bf16(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor | None = None):
    """softmax(q k^T / sqrt(D)) v per batch element and head, D = 64 or 128.

    q [B, Sq, H, D], k and v [B, Skv, H, D], BF16; the last two dimensions contiguous, the batch
    dimension densely on top of the token dimension (stride(0) == S * stride(1)) -- views into a fused
    projection output qualify.  Returns [B, Sq, H, D].
    """
    for name, t in (("q", q), ("k", k), ("v", v)):
        _check_attention_view(name, t)
    B, Sq, H, D = q.shape
    if k.shape != v.shape or k.shape[0] != B or k.shape[2] != H or k.shape[3] != D:
        raise ValueError("k and v must share [B, Skv, H, D] with q's batch, heads and head dimension")
    if out is None:
        out = _empty((B, Sq, H, D), torch.bfloat16, q.device)
    _check_attention_view("out", out)
    _check(lib().sol_attention_bf16(_ptr(q), _ptr(k), _ptr(v), _ptr(out), B, Sq, k.shape[1], H, D, _token_pitch(q),
                                    _token_pitch(k), _token_pitch(v), _token_pitch(out), _stream()), "sol_attention_bf16")
    return out


def sol_attention_nvfp4_out(q, k, v, out_tscale: torch.Tensor, dest, dest_col0: int = 0,
                            amax_out: torch.Tensor | None = None):
    """Attention whose output is quantized into columns [dest_col0, dest_col0 + H * D) of `dest`.

    dest = (nibbles [B * Sq, dest_K / 2] uint8, swizzled scales of a [B * Sq, dest_K] tensor); returns dest.
    """
    for name, t in (("q", q), ("k", k), ("v", v)):
        _check_attention_view(name, t)
    B, Sq, H, D = q.shape
    if k.shape != v.shape or k.shape[0] != B or k.shape[2] != H or k.shape[3] != D:
        raise ValueError("k and v must share [B, Skv, H, D] with q's batch, heads and head dimension")
    dq, dsf = dest
    if dq.dtype != torch.uint8 or dq.dim() != 2 or dq.shape[0] != B * Sq or not dq.is_contiguous():
        raise ValueError("dest nibbles must be a contiguous [B * Sq, dest_K / 2] uint8 tensor")
    _check(lib().sol_attention_nvfp4_out(_ptr(q), _ptr(k), _ptr(v), B, Sq, k.shape[1], H, D, _token_pitch(q), _token_pitch(k),
                                         _token_pitch(v), _ptr(out_tscale), _ptr(dq), _ptr(dsf), dq.shape[1] * 2, dest_col0,
                                         _ptr(amax_out), _stream()), "sol_attention_nvfp4_out")
    return dest


def matvec_workspace_bytes(M: int, K: int) -> int:
    return lib().sol_matvec_workspace_bytes(M, K)


def _matvec(entry, name: str, x, wq, wsf, w_tscale, bias, activation: int, out, workspace, scale_columns: int):
    """Checks and the call of a weight-only product; `scale_columns`: columns of K that a scale chunk spans."""
    index = x.get_device()
    if x.dtype is not torch.bfloat16 or x.dim() != 2 or x.stride(1) != 1:
        raise TypeError("x: expected a 2-D CUDA bf16 tensor with contiguous rows")
    if wq.dtype is not torch.uint8 or wq.dim() != 2 or not wq.is_contiguous() or wsf.dtype is not torch.uint8 or not wsf.is_contiguous():
        raise TypeError("weights: expected dense uint8 nibbles [N, K/2] and a dense uint8 scale buffer")
    (M, K), (N, packed) = x.shape, wq.shape
    if packed * 2 != K:
        raise ValueError(f"x has {K} columns, the weight {packed * 2}")
    if wsf.numel() < (N + 127) // 128 * ((K + scale_columns - 1) // scale_columns) * 512:
        raise ValueError("scale buffer too small for the weight's chunked scales")
    if wq.get_device() != index or wsf.get_device() != index:
        raise ValueError("the weight must be on x's device")
    if bias is not None and (bias.dtype is not torch.bfloat16 or bias.dim() != 1 or bias.shape[0] != N or not bias.is_contiguous()
                             or bias.get_device() != index):
        raise TypeError("bias: expected a dense [N] bf16 tensor on x's device")
    if out is None:
        out, ldy = _new(x, (M, N)), N
    elif out.dtype is not torch.bfloat16 or out.dim() != 2 or out.shape != (M, N) or out.stride(1) != 1 or out.get_device() != index:
        raise TypeError("out: expected a [M, N] bf16 tensor with contiguous rows on x's device")
    else:
        ldy = out.stride(0) if M > 1 else N      # a single row has no pitch of its own
    ws_ptr, ws_bytes = None, 0
    if workspace is None:
        ws_bytes = lib().sol_matvec_workspace_bytes(M, K)
        if ws_bytes:
            workspace = _new(wq, ws_bytes)
            ws_ptr = workspace.data_ptr()
    elif not workspace.is_contiguous() or workspace.get_device() != index:
        raise TypeError("workspace: expected a dense tensor on x's device")
    else:
        ws_ptr, ws_bytes = workspace.data_ptr(), workspace.nbytes
    tail = (None if bias is None else bias.data_ptr(), activation, out.data_ptr(), ldy, M, N, K, ws_ptr, ws_bytes, _raw_stream(index))
    ldx = x.stride(0) if M > 1 else K
    if w_tscale is None:
        code = entry(x.data_ptr(), ldx, wq.data_ptr(), wsf.data_ptr(), *tail)
    else:
        if w_tscale.dtype is not torch.float32 or w_tscale.numel() < 1 or w_tscale.get_device() != index:
            raise TypeError("w_tscale: expected a float32 tensor on x's device")
        code = entry(x.data_ptr(), ldx, wq.data_ptr(), wsf.data_ptr(), w_tscale.data_ptr(), *tail)
    if code:
        raise SolError(code, name)
    return out


@_on_device_of_first
def nvfp4_matvec(x, wq, wsf, w_tscale, bias=None, activation: int = ACT_NONE, out: torch.Tensor | None = None,
                 workspace: torch.Tensor | None = None):
    """Y = act(X) . dequant(W)^T + bias for a few BF16 rows: x is not quantized.  `activation`: ACT_NONE or ACT_SILU, on x."""
    if w_tscale is None:
        raise TypeError("w_tscale: expected a float32 tensor on x's device")
    return _matvec(lib().nvfp4_matvec, "nvfp4_matvec", x, wq, wsf, w_tscale, bias, activation, out, workspace, 64)


@_on_device_of_first
def mxfp4_matvec(x, wq, wsf, bias=None, activation: int = ACT_NONE, out: torch.Tensor | None = None,
                 workspace: torch.Tensor | None = None):
    """The same against an MXFP4 weight (no tensor scale)."""
    return _matvec(lib().mxfp4_matvec, "mxfp4_matvec", x, wq, wsf, None, bias, activation, out, workspace, 128)


ROTARY_INTERLEAVED, ROTARY_HALF = 0, 1
ROTARY_SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "yarn": 3}


# sol_rotary_t, sol_head_tensor_t and sol_head_grad_t of the C header, packed by the native rules: these calls are a few
# microseconds of GPU work for short streams, and a packed string costs a quarter of a ctypes structure.
_ROTARY = struct.Struct("@PPqqqqqqif")
_HEAD_TENSOR = struct.Struct("@PPPqqq")
_HEAD_GRAD = struct.Struct("@PPPPPqqqq")


def rotary_frequencies(axis_dims, theta: float = 10000.0, scaling: str = "none", factor: float = 1.0,
                       original_length: float = 0.0, beta_fast: float = 32.0, beta_slow: float = 1.0, device="cuda"):
    """Frequencies of the rotated pairs of all axes, side by side (FP64 on `device`), and the factor on cosine and sine.

    `scaling` = "none" | "linear" | "ntk" | "yarn" stretches them for contexts `factor` times longer than the
    model was trained on (`original_length` positions: "yarn").
    """
    if scaling not in ROTARY_SCALINGS:
        raise ValueError(f"scaling must be one of {sorted(ROTARY_SCALINGS)}")
    parts, scale = [], ctypes.c_double(1.0)
    for d in axis_dims:
        buf = (ctypes.c_double * max(1, d // 2))()
        _check(lib().sol_rotary_frequencies(d, float(theta), ROTARY_SCALINGS[scaling], float(factor), float(original_length),
                                            float(beta_fast), float(beta_slow), buf, ctypes.byref(scale)),
               "sol_rotary_frequencies")
        parts += list(buf)[:d // 2]
    if not parts:
        raise ValueError("no axes")
    return torch.tensor(parts, dtype=torch.float64, device=device), scale.value


def _head_pitch(name: str, t: torch.Tensor, index: int) -> int:
    """Checks a BF16 view [B, S, H, D] on CUDA device `index` and returns its token pitch."""
    if t.dtype is not torch.bfloat16 or t.dim() != 4:
        raise TypeError(f"{name}: expected a [B, S, H, D] bf16 tensor")
    if t.get_device() != index:
        raise ValueError(f"{name} is on {t.device}, the call's first tensor on cuda:{index}")
    b, s, h, d = t.shape
    sb, ss, sh, sd = t.stride()
    if sd != 1 or (sh != d and h > 1) or (b > 1 and s > 1 and sb != s * ss):
        raise ValueError(f"{name}: heads and head dimension must be contiguous, batches stacked densely")
    return ss if s > 1 else (sb if b > 1 else h * d)


def _head_view(name: str, t: torch.Tensor, shape, index: int) -> int:
    """The same for a view that must have the given shape."""
    if t.shape != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    return _head_pitch(name, t, index)


def _rotary_of(positions, freqs, axis_dims, layout, scale, rows: int, index: int):
    if positions is None:
        if freqs is not None:
            raise ValueError("freqs without positions")
        return None
    if positions.dtype is not torch.int64 or positions.dim() != 2 or not positions.is_contiguous():
        raise TypeError("positions: expected a dense [rows, axes] int64 tensor")
    if freqs is None or freqs.dtype is not torch.float64 or freqs.dim() != 1 or not freqs.is_contiguous():
        raise TypeError("freqs: expected a dense 1-D float64 tensor")
    if positions.get_device() != index or freqs.get_device() != index:
        raise ValueError(f"positions and freqs must be on the first tensor's device, cuda:{index}")
    pos_rows, axes = positions.shape
    columns = 2 * freqs.shape[0]
    dims = (columns,) if axis_dims is None else tuple(axis_dims)
    if len(dims) != axes or axes > 4 or sum(dims) != columns:
        raise ValueError("axis_dims must name each axis of positions and add up to twice the frequencies")
    if pos_rows == 0 or rows % pos_rows != 0:
        raise ValueError("the tokens must be a multiple of the rows of positions")
    return _ROTARY.pack(positions.data_ptr(), freqs.data_ptr(), pos_rows, axes, *dims, *(0,) * (4 - axes), layout, scale)


def _norm_weight(name: str, w, d: int, index: int) -> int:
    if w is None:
        return 0
    if w.dtype is not torch.bfloat16 or w.dim() != 1 or w.shape[0] != d or not w.is_contiguous() or w.get_device() != index:
        raise TypeError(f"{name}: expected a dense [head_dim] bf16 tensor on the first tensor's device")
    return w.data_ptr()


@_on_device_of_first
def sol_qk_rotary(q, k, positions, freqs, axis_dims=None, layout: int = ROTARY_INTERLEAVED, q_weight=None, k_weight=None,
                  eps: float = 1e-6, scale: float = 1.0, out=None):
    """RMS norm of every head of q [B, S, H, D] and k [B, S, Hk, D] (where a weight is given), then rotary positions.

    q and k may be views into a fused projection output; k may be None.  `positions` [R, axes] int64 holds the
    position of each token (token m of the B * S takes row m % R), or is None for the norm alone; `freqs`, `scale`
    as from rotary_frequencies; `axis_dims` the rotated columns of each axis (default: one axis).  Returns (q', k');
    `out` = (q_out, k_out) supplies the destinations, which may be q and k themselves.
    """
    index = q.get_device()
    ld = _head_pitch("q", q, index)
    b, s, h, d = q.shape
    rows = b * s
    rot = _rotary_of(positions, freqs, axis_dims, layout, scale, rows, index)
    if out is None:
        oq, ld_out = _like(q), h * d
    else:
        oq, ld_out = out[0], _head_view("q_out", out[0], q.shape, index)
    pq = _HEAD_TENSOR.pack(q.data_ptr(), oq.data_ptr(), _norm_weight("q_weight", q_weight, d, index), h, ld, ld_out)
    ok = pk = None
    if k is not None:
        ld = _head_pitch("k", k, index)
        bk, sk, hk, dk = k.shape
        if bk != b or sk != s or dk != d:
            raise ValueError("k must share q's batch, tokens and head dimension")
        if out is None:
            ok, ld_out = _like(k), hk * d
        else:
            ok, ld_out = out[1], _head_view("k_out", out[1], k.shape, index)
        pk = _HEAD_TENSOR.pack(k.data_ptr(), ok.data_ptr(), _norm_weight("k_weight", k_weight, d, index), hk, ld, ld_out)
    code = lib().sol_qk_rotary(pq, pk, rows, d, rot, eps, _raw_stream(index))
    if code:
        raise SolError(code, "sol_qk_rotary")
    return oq, ok


@_on_device_of_first
def sol_qk_rotary_backward(dq, dk, q, k, positions, freqs, axis_dims=None, layout: int = ROTARY_INTERLEAVED, q_weight=None,
                           k_weight=None, eps: float = 1e-6, scale: float = 1.0, out=None,
                           workspace: torch.Tensor | None = None):
    """Gradients of sol_qk_rotary from those of its outputs: (grad q, grad k, grad q_weight, grad k_weight).

    q and k are the forward call's inputs (needed where there is a weight, else they may be None); dk may be None.
    Weight gradients are FP32 [D], None without a weight.  `out` = (grad q, grad k) destinations, which may be
    dq and dk themselves.
    """
    index = dq.get_device()
    ld = _head_pitch("dq", dq, index)
    b, s, _, d = dq.shape
    rot = _rotary_of(positions, freqs, axis_dims, layout, scale, b * s, index)
    packed, dxs, dws = [None, None], [None, None], [None, None]
    for i, name, dy, x, w in ((0, "q", dq, q, q_weight), (1, "k", dk, k, k_weight)):
        if dy is None:
            continue
        if i:
            ld = _head_pitch("dk", dy, index)
            if dy.shape[0] != b or dy.shape[1] != s or dy.shape[3] != d:
                raise ValueError("dk must share dq's batch, tokens and head dimension")
        h = dy.shape[2]
        weight = _norm_weight(name + "_weight", w, d, index)
        x_ptr = ld_x = dw_ptr = 0
        if weight:
            if x is None:
                raise ValueError(f"{name}: the gradient of a norm needs the forward input")
            ld_x, x_ptr = _head_view(name, x, dy.shape, index), x.data_ptr()
            dws[i] = _new(dy, d, torch.float32)
            dw_ptr = dws[i].data_ptr()
        if out is None:
            dxs[i], ld_dx = _like(dy), h * d
        else:
            dxs[i], ld_dx = out[i], _head_view(name + "_grad", out[i], dy.shape, index)
        packed[i] = _HEAD_GRAD.pack(dy.data_ptr(), x_ptr, dxs[i].data_ptr(), weight, dw_ptr, h, ld, ld_x, ld_dx)
    ws_ptr = ws_bytes = 0
    if dws[0] is not None or dws[1] is not None:
        if workspace is None:
            workspace = _new(dq, max(1, lib().sol_qk_rotary_backward_workspace_bytes(d)), torch.uint8)
        elif workspace.get_device() != index or not workspace.is_contiguous():
            raise ValueError("workspace: expected a dense tensor on the first tensor's device")
        ws_ptr, ws_bytes = workspace.data_ptr(), workspace.nbytes
    code = lib().sol_qk_rotary_backward(packed[0], packed[1], b * s, d, rot, eps, ws_ptr, ws_bytes, _raw_stream(index))
    if code:
        raise SolError(code, "sol_qk_rotary_backward")
    return dxs[0], dxs[1], dws[0], dws[1]


def _rows_view(name: str, t: torch.Tensor, index: int, shape=None) -> int:
    """Checks a BF16 matrix [M, K] with contiguous rows on CUDA device `index` and returns its row pitch."""
    if t.dtype is not torch.bfloat16 or t.dim() != 2:
        raise TypeError(f"{name}: expected a 2-D bf16 tensor")
    if t.get_device() != index:
        raise ValueError(f"{name} is on {t.device}, the call's first tensor on cuda:{index}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    rows, cols = t.shape
    if cols > 1 and t.stride(1) != 1:
        raise ValueError(f"{name}: rows must be contiguous")
    return t.stride(0) if rows > 1 else cols


def _dense(name: str, t: torch.Tensor, dtype, shape, index: int) -> int:
    """Checks a dense tensor of the given type and shape on CUDA device `index` and returns its address."""
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous() or t.get_device() != index:
        raise TypeError(f"{name}: expected a dense {dtype} tensor of shape {tuple(shape)} on cuda:{index}")
    return t.data_ptr()


def _scratch(workspace, need: int, like: torch.Tensor, index: int):
    """A call's workspace: the caller's, or a new one of `need` bytes; (tensor or None, address, bytes)."""
    if workspace is None:
        if need == 0:
            return None, None, 0
        workspace = _new(like, need, torch.uint8)
    elif workspace.get_device() != index or not workspace.is_contiguous():
        raise TypeError("workspace: expected a dense tensor on the first tensor's device")
    return workspace, workspace.data_ptr(), workspace.nbytes


@_on_device_of_first
def sol_layernorm(x, scale=None, shift=None, rows_per_sample: int | None = None, eps: float = 1e-6, scale_offset: float = 1.0,
                  out: torch.Tensor | None = None, with_stats: bool = False):
    """LN(x) * (scale_offset + scale[sample]) + shift[sample] in BF16; scale_offset 1: modulation, 0: a weight and a bias.

    x [M, K] (a view with a row pitch will do); scale and shift [samples, K] or None (slices of one modulation tensor will do, both
    with its pitch; one vector expanded over the samples is refused), a sample being `rows_per_sample` rows (default: all).
    Returns y, or (y, stats) `with_stats`: FP32 [M, 2] mean and 1 / sqrt(var + eps) for sol_layernorm_backward.
    """
    index = x.get_device()
    ldx = _rows_view("x", x, index)
    M, K = x.shape
    rows = M if rows_per_sample is None else rows_per_sample
    samples = -(-M // rows) if rows > 0 else 0
    ld_scale = None if scale is None else _rows_view("scale", scale, index, (samples, K))
    ld_mod = ld_scale if shift is None else _rows_view("shift", shift, index, (samples, K))
    if ld_scale is not None and ld_scale != ld_mod:
        raise ValueError("scale and shift must have the same row pitch")
    if out is None:
        out, ldy = _like(x), K
    else:
        ldy = _rows_view("out", out, index, x.shape)
    stats = _new(x, (M, 2), torch.float32) if with_stats else None
    code = lib().sol_layernorm(x.data_ptr(), M, K, ldx, _ptr(scale), _ptr(shift), K if ld_mod is None else ld_mod, rows, scale_offset, eps, out.data_ptr(), ldy,
                               None if stats is None else stats.data_ptr(), _raw_stream(index))
    if code:
        raise SolError(code, "sol_layernorm")
    return (out, stats) if with_stats else out


@_on_device_of_first
def sol_layernorm_backward(dy, x, stats, scale=None, rows_per_sample: int | None = None, scale_offset: float = 1.0,
                           out: torch.Tensor | None = None, with_scale: bool = True, with_shift: bool = True,
                           workspace: torch.Tensor | None = None):
    """Gradients of sol_layernorm from that of its output: (grad x, grad scale, grad shift).

    x, stats and scale are the forward call's.  The gradients of scale and shift are FP32 [samples, K], summed over each
    sample's rows, None where not asked for.  `out` = grad x may be dy or x itself.
    """
    index = dy.get_device()
    ld_dy = _rows_view("dy", dy, index)
    M, K = dy.shape
    ldx = _rows_view("x", x, index, dy.shape)
    rows = M if rows_per_sample is None else rows_per_sample
    samples = -(-M // rows) if rows > 0 else 0
    stats_ptr = _dense("stats", stats, torch.float32, (M, 2), index)
    ld_scale = K if scale is None else _rows_view("scale", scale, index, (samples, K))
    if out is None:
        out, ld_dx = _like(dy), K
    else:
        ld_dx = _rows_view("out", out, index, dy.shape)
    dscale = _new(dy, (samples, K), torch.float32) if with_scale else None
    dshift = _new(dy, (samples, K), torch.float32) if with_shift else None
    need = lib().sol_layernorm_backward_workspace_bytes(M, K, rows) if workspace is None and (with_scale or with_shift) else 0
    workspace, ws_ptr, ws_bytes = _scratch(workspace, need, dy, index)
    code = lib().sol_layernorm_backward(dy.data_ptr(), ld_dy, x.data_ptr(), ldx, stats_ptr, _ptr(scale), ld_scale, M, K, rows, scale_offset,
                                        out.data_ptr(), ld_dx, _ptr(dscale), _ptr(dshift), ws_ptr, ws_bytes, _raw_stream(index))
    if code:
        raise SolError(code, "sol_layernorm_backward")
    return out, dscale, dshift


def _lora_stacks(lora_a, lora_b, scaling, offsets, ids, K: int, N: int, index: int):
    """Checks the adapters' stacks and the requests; returns (adapters, rank, requests) and the five addresses."""
    if lora_a.dim() != 3 or lora_b.dim() != 3:
        raise TypeError("lora_a, lora_b: expected [adapters, r, K] and [adapters, N, r] tensors")
    adapters, r = lora_a.shape[:2]
    requests = ids.shape[0] if ids.dim() == 1 else -1
    return (adapters, r, requests, _dense("lora_a", lora_a, torch.bfloat16, (adapters, r, K), index),
            _dense("lora_b", lora_b, torch.bfloat16, (adapters, N, r), index), _dense("scaling", scaling, torch.float32, (adapters,), index),
            _dense("offsets", offsets, torch.int32, (requests + 1,), index), _dense("ids", ids, torch.int32, (requests,), index))


@_on_device_of_first
def sol_lora_apply(x, lora_a, lora_b, scaling, offsets, ids, y, with_t: bool = False, workspace: torch.Tensor | None = None):
    """y += scaling[a] (x A_a^T) B_a^T in place for every request's rows, a being the request's adapter (or none); returns y.

    x [M, K], y [M, N] BF16 (views with a row pitch will do); lora_a [n, r, K], lora_b [n, N, r] BF16, scaling [n] FP32; request i is
    the rows offsets[i] .. offsets[i + 1] (int32, ascending) and has adapter ids[i] (int32), none outside 0 .. n - 1.  `with_t`
    returns (y, t) with t [M, 2 r], x A^T in two BF16 parts, for sol_lora_backward.
    """
    index = x.get_device()
    ldx, ldy = _rows_view("x", x, index), _rows_view("y", y, index)
    M, K = x.shape
    N = y.shape[1]
    if y.shape[0] != M:
        raise ValueError("x and y must have the same rows")
    n, r, requests, a_ptr, b_ptr, s_ptr, o_ptr, i_ptr = _lora_stacks(lora_a, lora_b, scaling, offsets, ids, K, N, index)
    t = _new(x, (M, 2 * r)) if with_t else None
    need = 0 if workspace is not None else lib().sol_lora_workspace_bytes(M, K, N, r, n, requests, 0)
    workspace, ws_ptr, ws_bytes = _scratch(workspace, need, x, index)
    code = lib().sol_lora_apply(x.data_ptr(), ldx, a_ptr, b_ptr, s_ptr, o_ptr, i_ptr, requests, n, y.data_ptr(), ldy, _ptr(t), M, K, N, r,
                                ws_ptr, ws_bytes, _raw_stream(index))
    if code:
        raise SolError(code, "sol_lora_apply")
    return (y, t) if with_t else y


@_on_device_of_first
def sol_lora_backward(dy, x, t, lora_a, lora_b, scaling, offsets, ids, dx: torch.Tensor | None = None,
                      workspace: torch.Tensor | None = None):
    """Gradients of sol_lora_apply: (grad lora_a, grad lora_b) in FP32, zeros for an adapter without rows.

    x, t and the stacks are the forward call's.  `dx` [M, K] BF16, the gradient that x has from the shared projection, gets the
    adapters' part added in place.
    """
    index = dy.get_device()
    ld_dy, ldx = _rows_view("dy", dy, index), _rows_view("x", x, index)
    M, N = dy.shape
    K = x.shape[1]
    if x.shape[0] != M:
        raise ValueError("dy and x must have the same rows")
    n, r, requests, a_ptr, b_ptr, s_ptr, o_ptr, i_ptr = _lora_stacks(lora_a, lora_b, scaling, offsets, ids, K, N, index)
    t_ptr = _dense("t", t, torch.bfloat16, (M, 2 * r), index)
    ld_dx = K if dx is None else _rows_view("dx", dx, index, x.shape)
    da, db = _new(dy, (n, r, K), torch.float32), _new(dy, (n, N, r), torch.float32)
    need = 0 if workspace is not None else lib().sol_lora_workspace_bytes(M, K, N, r, n, requests, 1)
    workspace, ws_ptr, ws_bytes = _scratch(workspace, need, dy, index)
    code = lib().sol_lora_backward(dy.data_ptr(), ld_dy, x.data_ptr(), ldx, t_ptr, a_ptr, b_ptr, s_ptr, o_ptr, i_ptr, requests, n, _ptr(dx), ld_dx,
                                   da.data_ptr(), db.data_ptr(), M, K, N, r, ws_ptr, ws_bytes, _raw_stream(index))
    if code:
        raise SolError(code, "sol_lora_backward")
    return da, db


# sol_adamw_tensor_t and sol_adamw_options_t of the C header, packed by the native rules.
_ADAMW_TENSOR = struct.Struct("@PPPPPPPq")
_ADAMW_OPTIONS = struct.Struct("@dddddPPQiiii")
_ADAMW_STATES = {32: (("m", torch.float32, 1), ("v", torch.float32, 1)),
                 8: (("m", torch.uint8, 1), ("v", torch.uint8, 1), ("m_scale", torch.uint8, 32), ("v_scale", torch.uint8, 32))}


class AdamWPlan:
    """Tensors of an AdamW step laid out once: parameters, gradients, states and the step counter (see sol_adamw_plan)."""

    def __init__(self, params, grads, copies, state_bits: int, states, step: int):
        params = list(params)
        if not params:
            raise ValueError("no parameters")
        if state_bits not in _ADAMW_STATES:
            raise ValueError("state_bits must be 32 or 8")
        if step < 0:
            raise ValueError("step: the steps that the states have behind them, 0 or more")
        self.index, self.state_bits, self.params = params[0].get_device(), state_bits, params
        if self.index < 0:
            raise TypeError("sol_adamw_plan: expected CUDA tensors")
        self.device = params[0].device
        self.param_dtype = params[0].dtype
        if self.param_dtype not in (torch.float32, torch.bfloat16):
            raise TypeError("params: expected float32 or bfloat16")
        for p in params:
            self._check("params", p, self.param_dtype, p.numel())
        if len({p.data_ptr() for p in params if p.numel()}) != sum(p.numel() > 0 for p in params):
            raise ValueError("params: the same tensor twice")
        if copies is not None:
            if self.param_dtype is not torch.float32:
                raise ValueError("copies: only beside float32 parameters")
            copies = list(copies)
            self._check_all("copies", copies, torch.bfloat16, 1)
        self.copies = copies
        for name, dtype, unit in _ADAMW_STATES[state_bits]:
            if states is None:
                # one buffer for all, every tensor's part on a 128-byte boundary
                sizes = [-(-p.numel() // unit) for p in params]
                each = [-(-n // 128) * 128 for n in sizes]
                flat = torch.zeros(sum(each), dtype=dtype, device=self.device)
                parts, at = [], 0
                for n, e in zip(sizes, each):
                    parts.append(flat[at:at + n])
                    at += e
            else:
                parts = list(states[name])
                self._check_all(name, parts, dtype, unit)
            setattr(self, name, parts)
        self.step = torch.tensor([step, 0], dtype=torch.int64, device=self.device)
        # a view of each: the memory stays as long as the plan, whatever the caller does to the tensors
        columns = [params, copies or [None] * len(params)] + [getattr(self, s[0]) for s in _ADAMW_STATES[state_bits]]
        self._memory = [[None if t is None else t.detach() for t in column] for column in columns]
        self._columns = [[0 if t is None else t.data_ptr() for t in column] for column in self._memory]
        self._sizes = [p.numel() for p in params]
        # what a step compares: where the tensors are that it writes, and where they were
        self._pointers = [t.data_ptr for t in (*params, *(copies or []))]
        self._addresses = [f() for f in self._pointers]
        self.set_grads(grads)

    def _check(self, name, t, dtype, numel):
        if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.numel() != numel or not t.is_contiguous() or t.get_device() != self.index:
            raise TypeError(f"{name}: expected a dense {dtype} tensor of {numel} elements on cuda:{self.index}")

    def _check_all(self, name, tensors, dtype, unit):
        if len(tensors) != len(self.params):
            raise ValueError(f"{name}: one for each parameter")
        for t, p in zip(tensors, self.params):
            self._check(name, t, dtype, -(-p.numel() // unit))

    def set_grads(self, grads) -> None:
        """Other gradient tensors for the following steps (None for a parameter that takes no step)."""
        grads = list(grads)
        if len(grads) != len(self.params):
            raise ValueError("grads: one for each parameter")
        dtypes = {g.dtype for g in grads if g is not None}
        if len(dtypes) > 1 or not dtypes <= {torch.float32, torch.bfloat16}:
            raise TypeError("grads: expected float32 or bfloat16, the same for all")
        for g, n in zip(grads, self._sizes):
            if g is not None:
                self._check("grads", g, g.dtype, n)
        self.grads = grads
        self.grad_bf16 = torch.bfloat16 in dtypes
        self._grads_memory = [None if g is None else g.detach() for g in grads]
        param, copy, m, v, *scales = self._columns
        m_scale, v_scale = scales or ([0] * len(param),) * 2
        grad = [0 if g is None else g.data_ptr() for g in grads]
        sizes = [0 if g is None else n for g, n in zip(grads, self._sizes)]
        self._packed = b"".join(map(_ADAMW_TENSOR.pack, param, copy, grad, m, v, m_scale, v_scale, sizes))

    def _refuse_moved(self) -> None:
        moved = next(i for i, (f, a) in enumerate(zip(self._pointers, self._addresses)) if f() != a)
        name = "params" if moved < len(self._sizes) else "copies"
        raise ValueError(f"{name}[{moved % len(self._sizes)}]: its memory is not that of the plan any more; make a plan of the tensors as they are")


def sol_adamw_plan(params, grads, copies=None, state_bits: int = 32, states=None, step: int = 0) -> AdamWPlan:
    """Lays out tensors for sol_adamw_step: dense FP32 or BF16 parameters and their FP32 or BF16 gradients.

    `copies`: BF16 tensors that receive the rounded FP32 parameters (what the linears read).  `state_bits` 32: FP32 moments;
    8: E4M3 and E5M2 codes under one power of two per 32 values.  The states are new and zero, or `states`' lists ("m", "v" and, in
    8 bits, "m_scale", "v_scale"); `step` is the number of steps that they have behind them.  The plan keeps the tensors and
    offers them as attributes: params, grads, copies, m, v, m_scale, v_scale, step ([0] on the device).  It is laid out for the memory
    that they have now: once the `data` of a parameter or a copy has been replaced a step is refused (a captured one cannot be, and
    goes on with the memory of before), and a gradient whose `data` has been replaced is given again with set_grads.  No two of the tensors may overlap.
    """
    return AdamWPlan(params, grads, copies, state_bits, states, step)


def sol_adamw_step(plan: AdamWPlan, lr: float, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8, weight_decay: float = 0.01,
                   seed: int | None = None, lr_scale: torch.Tensor | None = None, grad_scale: torch.Tensor | None = None) -> None:
    """One AdamW step of the plan's parameters, in place, from the gradients that its tensors hold now.

    With a `seed`, 8-bit states and BF16 parameters are rounded up or down by chance in proportion (other bits every step), without
    one to nearest.  `lr_scale` and `grad_scale` are one-element FP32 device tensors or None: factors read when the step runs.
    """
    if not isinstance(plan, AdamWPlan):
        raise TypeError("sol_adamw_step: expected a plan of sol_adamw_plan")
    index = plan.index
    scales = [0, 0]
    for i, (name, t) in enumerate((("lr_scale", lr_scale), ("grad_scale", grad_scale))):
        if t is not None:
            scales[i] = _dense(name, t.reshape(-1), torch.float32, (1,), index)
    if [f() for f in plan._pointers] != plan._addresses:
        plan._refuse_moved()
    options = _ADAMW_OPTIONS.pack(lr, beta1, beta2, eps, weight_decay, *scales, 0 if seed is None else seed & (2 ** 64 - 1), seed is not None,
                                  plan.param_dtype is torch.bfloat16, plan.grad_bf16, plan.state_bits)
    packed, count = plan._packed, len(plan._sizes)
    if index == torch._C._cuda_getDevice():
        code = lib().sol_adamw_step(packed, count, options, plan.step.data_ptr(), _raw_stream(index))
    else:
        with torch.cuda.device(index):
            code = lib().sol_adamw_step(packed, count, options, plan.step.data_ptr(), _raw_stream(index))
    if code:
        raise SolError(code, "sol_adamw_step")


QUERY_BLOCK, KEY_BLOCK = 256, 128


def _kv_of(q, k, index: int):
    """Shapes of q [B, Sq, H, D] and k [B, Skv, Hk, D] and their token pitches."""
    ld_q, ld_k = _head_pitch("q", q, index), _head_pitch("k", k, index)
    B_, Sq, H, D = q.shape
    b, Skv, Hk, d = k.shape
    if b != B_ or d != D or Hk == 0 or H % Hk != 0:
        raise ValueError("k must share q's batch and head dimension, and its heads must divide q's")
    return B_, Sq, Skv, H, Hk, D, ld_q, ld_k


def _lens_ptr(kv_lens, B_: int, index: int) -> int | None:
    if kv_lens is None:
        return None
    if kv_lens.dtype is not torch.int32 or kv_lens.shape != (B_,) or not kv_lens.is_contiguous() or kv_lens.get_device() != index:
        raise TypeError("kv_lens: expected a dense [B] int32 tensor on q's device")
    return kv_lens.data_ptr()


@_on_device_of_first
def sol_select_blocks(q, k, count: int, keep_first: int = 0, kv_lens=None, with_scores: bool = False,
                      workspace: torch.Tensor | None = None):
    """Key blocks (128 tokens) of highest mean-pooled score for each query block (256 tokens) of each head.

    q [B, Sq, H, D], k [B, Skv, Hk, D] (D = 64 or 128, Hk divides H).  Returns (blocks [B, H, ceil(Sq / 256), count]
    int32, ascending, -1 behind the last; counts [B, H, ceil(Sq / 256)] int32) and, `with_scores`, the chosen
    blocks' FP32 scores.  The first `keep_first` blocks are always kept; `kv_lens` [B] int32 limits the keys that exist.
    """
    index = q.get_device()
    B_, Sq, Skv, H, Hk, D, ld_q, ld_k = _kv_of(q, k, index)
    lens = _lens_ptr(kv_lens, B_, index)
    nq = (Sq + QUERY_BLOCK - 1) // QUERY_BLOCK
    if not 0 < count <= 8192:
        raise ValueError("count must be between 1 and 8192")
    blocks = _new(q, (B_, H, nq, count), torch.int32)
    counts = _new(q, (B_, H, nq), torch.int32)
    scores = _new(q, (B_, H, nq, count), torch.float32) if with_scores else None
    if workspace is None:
        workspace = _new(q, max(1, lib().sol_select_blocks_workspace_bytes(B_, Sq, Skv, H, Hk, D)), torch.uint8)
    elif workspace.get_device() != index or not workspace.is_contiguous():
        raise TypeError("workspace: expected a dense tensor on q's device")
    code = lib().sol_select_blocks(q.data_ptr(), k.data_ptr(), B_, Sq, Skv, H, Hk, D, ld_q, ld_k, count, keep_first, lens,
                                   blocks.data_ptr(), counts.data_ptr(), None if scores is None else scores.data_ptr(),
                                   workspace.data_ptr(), workspace.nbytes, _raw_stream(index))
    if code:
        raise SolError(code, "sol_select_blocks")
    return (blocks, counts, scores) if with_scores else (blocks, counts)


@_on_device_of_first
def sol_attention_blocks(q, k, v, blocks, counts, kv_lens=None, out: torch.Tensor | None = None):
    """Attention of each 256-query block of each head over its listed 128-key blocks (as from sol_select_blocks).

    q [B, Sq, H, D], k and v [B, Skv, Hk, D]; blocks [B, H, ceil(Sq / 256), n] int32, counts [B, H, ceil(Sq / 256)] int32.
    Entries that name no existing block are skipped; a query whose list names no key gets zeros.  Returns [B, Sq, H, D].
    """
    index = q.get_device()
    B_, Sq, Skv, H, Hk, D, ld_q, ld_k = _kv_of(q, k, index)
    ld_v = _head_view("v", v, k.shape, index)
    nq = (Sq + QUERY_BLOCK - 1) // QUERY_BLOCK
    if blocks.dtype is not torch.int32 or blocks.dim() != 4 or blocks.shape[:3] != (B_, H, nq) or not blocks.is_contiguous() \
            or blocks.get_device() != index:
        raise TypeError("blocks: expected a dense [B, H, ceil(Sq / 256), n] int32 tensor on q's device")
    if counts.dtype is not torch.int32 or counts.shape != (B_, H, nq) or not counts.is_contiguous() or counts.get_device() != index:
        raise TypeError("counts: expected a dense [B, H, ceil(Sq / 256)] int32 tensor on q's device")
    if out is None:
        out, ld_out = _like(q), H * D
    else:
        ld_out = _head_view("out", out, q.shape, index)
    code = lib().sol_attention_blocks(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), B_, Sq, Skv, H, Hk, D, ld_q, ld_k, ld_v,
                                      ld_out, blocks.data_ptr(), counts.data_ptr(), blocks.shape[3],
                                      _lens_ptr(kv_lens, B_, index), _raw_stream(index))
    if code:
        raise SolError(code, "sol_attention_blocks")
    return out


def mxfp4_scale_bytes(rows: int, K: int, layout: int = SF_SWIZZLED_128x4) -> int:
    return int(lib().sol_mxfp4_scale_bytes(rows, K, layout))


def mxfp4_quantize(x: torch.Tensor, layout: int = SF_SWIZZLED_128x4, out=None):
    """BF16 [rows, K] -> (packed nibbles [rows, K/2], E8M0 scales in the given layout)."""
    _need_2d_bf16(x, "x")
    rows, K = x.shape
    if out is None:
        nbytes = mxfp4_scale_bytes(rows, K, layout)
        if nbytes == 0:
            raise ValueError("bad shape for mxfp4_quantize")
        out = (_empty((rows, K // 2), torch.uint8, x.device),
               _empty(nbytes, torch.uint8, x.device))
    q, sf = out
    _check(lib().mxfp4_quantize(_ptr(x), rows, K, x.stride(0), _ptr(q), _ptr(sf), layout, _stream()), "mxfp4_quantize")
    return q, sf


def mxfp4_linear(xq, xsf, wq, wsf, bias=None, out: torch.Tensor | None = None):
    """Y = dequant(X) . dequant(W)^T + bias in BF16 from MXFP4 operands (chunked scales)."""
    M, K = xq.shape[0], xq.shape[1] * 2
    N = wq.shape[0]
    if out is None:
        out = _empty((M, N), torch.bfloat16, xq.device)
    _check(lib().mxfp4_linear(_ptr(xq), _ptr(xsf), _ptr(wq), _ptr(wsf), _ptr(bias), _ptr(out), M, N, K, out.stride(0),
                              _stream()), "mxfp4_linear")
    return out


def mxfp4_linear_split_out(xq, xsf, wq, wsf, bias, n_split: int, activation: int, dest, dest_col0: int,
                           y_out: torch.Tensor | None = None, amax_out: torch.Tensor | None = None):
    """Columns below n_split -> BF16 `y_out`; the rest -> activation -> MXFP4 into dest = (q [M, dest_K/2], sf)."""
    M, K = xq.shape[0], xq.shape[1] * 2
    N = wq.shape[0]
    hq, hsf = dest
    if y_out is None:
        y_out = _empty((M, n_split), torch.bfloat16, xq.device)
    _check(lib().mxfp4_linear_split_out(_ptr(xq), _ptr(xsf), _ptr(wq), _ptr(wsf), _ptr(bias), _ptr(y_out), y_out.stride(0),
                                        n_split, activation, _ptr(hq), _ptr(hsf), hq.shape[1] * 2, dest_col0,
                                        _ptr(amax_out), M, N, K, _stream()), "mxfp4_linear_split_out")
    return y_out


def mxfp4_quantize_into(x: torch.Tensor, dest, dest_col0: int):
    """Quantize BF16 x [M, K] into columns [dest_col0, dest_col0 + K) of the MXFP4 tensor dest = (q, sf)."""
    _need_2d_bf16(x, "x")
    M, K = x.shape
    hq, hsf = dest
    _check(lib().mxfp4_quantize_into(_ptr(x), M, K, x.stride(0), _ptr(hq), _ptr(hsf), hq.shape[1] * 2, dest_col0,
                                     _stream()), "mxfp4_quantize_into")


def solrl_select_contrastive(rewards: torch.Tensor, K: int, seeds: torch.Tensor | None = None,
                             with_advantages: bool = True):
    """[P, N] FP32 rewards -> (indices [P, K] int32, selected seeds or None, advantages [P, N] or None)."""
    if rewards.dtype != torch.float32 or rewards.dim() != 2 or not rewards.is_contiguous():
        raise ValueError("rewards must be a dense 2-D float32 tensor")
    P, N = rewards.shape
    idx = _empty((P, K), torch.int32, rewards.device)
    sel = None
    if seeds is not None:
        if seeds.dtype != torch.int64 or tuple(seeds.shape) != (P, N) or not seeds.is_contiguous():
            raise ValueError("seeds must be a dense [P, N] int64 tensor")
        sel = _empty((P, K), torch.int64, rewards.device)
    adv = torch.empty_like(rewards) if with_advantages else None
    _check(lib().solrl_select_contrastive(_ptr(rewards), _ptr(seeds), P, N, K, _ptr(idx), _ptr(sel), _ptr(adv),
                                          _stream()), "solrl_select_contrastive")
    return idx, sel, adv


def solrl_rank_consistency(ref: torch.Tensor, proxy: torch.Tensor, k: int):
    """Per prompt: exact counts [P, 4] int64 and (tau, rho, top-k match, bottom-k match) [P, 4] FP32."""
    for t in (ref, proxy):
        if t.dtype != torch.float32 or t.dim() != 2 or not t.is_contiguous():
            raise ValueError("rewards must be dense 2-D float32 tensors")
    if ref.shape != proxy.shape:
        raise ValueError("shapes differ")
    P, N = ref.shape
    counts = _empty((P, 4), torch.int64, ref.device)
    metrics = _empty((P, 4), torch.float32, ref.device)
    _check(lib().solrl_rank_consistency(_ptr(ref), _ptr(proxy), P, N, k, _ptr(counts), _ptr(metrics), _stream()),
           "solrl_rank_consistency")
    return counts, metrics


def nvfp4_linear_quantized_out(xq, xsf, x_tscale, wq, wsf, w_tscale, bias, activation: int, out_tscale,
                               amax_out: torch.Tensor | None = None, out=None):
    """NVFP4 linear whose output leaves as (nibbles [M, N/2], swizzled scales) for the next linear."""
    M, K = xq.shape[0], xq.shape[1] * 2
    N = wq.shape[0]
    if out is None:
        out = _alloc_q(M, N, SF_SWIZZLED_128x4, xq.device)
    hq, hsf = out
    _check(lib().nvfp4_linear_quantized_out(_ptr(xq), _ptr(xsf), _ptr(x_tscale), _ptr(wq), _ptr(wsf), _ptr(w_tscale),
                                            _ptr(bias), activation, _ptr(out_tscale), _ptr(hq), _ptr(hsf),
                                            _ptr(amax_out), M, N, K, _stream()), "nvfp4_linear_quantized_out")
    return hq, hsf


def mxfp4_linear_quantized_out(xq, xsf, wq, wsf, bias, activation: int, amax_out: torch.Tensor | None = None, out=None):
    """MXFP4 linear whose output leaves as (nibbles [M, N/2], swizzled E8M0 scales) for the next MXFP4 linear."""
    M, K = xq.shape[0], xq.shape[1] * 2
    N = wq.shape[0]
    if out is None:
        out = (_empty((M, N // 2), torch.uint8, xq.device),
               _empty(mxfp4_scale_bytes(M, N), torch.uint8, xq.device))
    hq, hsf = out
    _check(lib().mxfp4_linear_quantized_out(_ptr(xq), _ptr(xsf), _ptr(wq), _ptr(wsf), _ptr(bias), activation, _ptr(hq),
                                            _ptr(hsf), _ptr(amax_out), M, N, K, _stream()), "mxfp4_linear_quantized_out")
    return hq, hsf


def bf16_linear(x, w, bias=None, out: torch.Tensor | None = None):
    """Y = X . W^T + bias, BF16 in / BF16 out, FP32 accumulation."""
    _need_2d_bf16(x, "x")
    _need_2d_bf16(w, "w")
    M, K = x.shape
    N = w.shape[0]
    if out is None:
        out = _empty((M, N), torch.bfloat16, x.device)
    _check(lib().bf16_linear(_ptr(x), _ptr(w), _ptr(bias), _ptr(out), M, N, K, x.stride(0), w.stride(0),
                             out.stride(0), _stream()), "bf16_linear")
    return out


def nvfp4_quantize_linear(x, wq, wsf, w_tscale, bias=None, workspace: torch.Tensor | None = None,
                          out: torch.Tensor | None = None):
    """Dynamic per-tensor scale + quantize X + NVFP4 GEMM against pre-quantized W, one call."""
    _need_2d_bf16(x, "x")
    M, K = x.shape
    N = wq.shape[0]
    if workspace is None:
        workspace = _empty(linear_workspace_bytes(M, N, K), torch.uint8, x.device)
    if out is None:
        out = _empty((M, N), torch.bfloat16, x.device)
    _check(lib().nvfp4_quantize_linear(_ptr(x), x.stride(0), _ptr(wq), _ptr(wsf), _ptr(w_tscale), _ptr(bias),
                                       _ptr(out), M, N, K, out.stride(0), _ptr(workspace), workspace.numel(),
                                       _stream()), "nvfp4_quantize_linear")
    return out


def nvfp4_quantize_linear_host(x_host, wq, wsf, w_tscale, bias, y_host, x_dev, y_dev, workspace):
    """End-to-end form: host X (ideally pinned) -> device, fused quantize + NVFP4 linear, Y -> host."""
    M, K = x_host.shape
    N = wq.shape[0]
    _check(lib().nvfp4_quantize_linear_host(_ptr(x_host), x_host.stride(0), _ptr(wq), _ptr(wsf), _ptr(w_tscale),
                                            _ptr(bias), _ptr(y_host), M, N, K, y_host.stride(0), _ptr(x_dev),
                                            _ptr(y_dev), _ptr(workspace), workspace.numel(), _stream()),
           "nvfp4_quantize_linear_host")
    return y_host


def static_scratch_bytes() -> int:
    return lib().sol_nvfp4_static_scratch_bytes()


def nvfp4_quantize_linear_static(x, wq, wsf, w_tscale, bias=None, out: torch.Tensor | None = None):
    """nvfp4_quantize_linear for callers that may not allocate: the scratch is a fixed array inside
    the library (64 MiB, shared by every call on the device; overlapping calls race).  Only the output
    tensor is created here when `out` is not given -- pass `out` to allocate nothing at all."""
    _need_2d_bf16(x, "x")
    M, K = x.shape
    N = wq.shape[0]
    if out is None:
        out = _empty((M, N), torch.bfloat16, x.device)
    _check(lib().nvfp4_quantize_linear_static(_ptr(x), x.stride(0), _ptr(wq), _ptr(wsf), _ptr(w_tscale), _ptr(bias),
                                              _ptr(out), M, N, K, out.stride(0), _stream()),
           "nvfp4_quantize_linear_static")
    return out


def sol_last_device_status() -> int:
    """Synchronises the current stream; raises SolError if a bounded device wait ran out."""
    detail = ctypes.c_uint32(0)
    code = lib().sol_last_device_status(_stream(), ctypes.byref(detail))
    if code != 0:
        err = SolError(code, f"device status word 0x{detail.value:x}")
        err.detail = detail.value
        raise err
    return 0


def sol_set_wait_limit_cycles(cycles: int) -> None:
    """Limit of every bounded device-side wait on the current device, in SM cycles (<= 0: default)."""
    _check(lib().sol_set_wait_limit_cycles(int(cycles)), "sol_set_wait_limit_cycles")


def sol_test_hold_loads(on: bool) -> None:
    """Test hook: while on, the pair GEMM kernels issue no loads and their waits run into the limit."""
    _check(lib().sol_test_hold_loads(1 if on else 0), "sol_test_hold_loads")


# every public entry checks the guard bands of what it allocated (a no-op outside guard mode)
for _name, _fn in list(globals().items()):
    if (isinstance(_fn, types.FunctionType) and _fn.__module__ == __name__ and not _name.startswith("_")
            and _name not in ("lib", "guard_mode", "check_guards", "status_string") and not hasattr(_fn, "_guards_itself")):
        globals()[_name] = _guarded(_fn)
del _name, _fn
