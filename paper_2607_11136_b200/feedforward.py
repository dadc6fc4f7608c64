"""The feed-forward half of a gated layer on torch tensors: RMSNorm with the residual's addition, the gated
feed-forward with its gradients, and a projection with the adapters of many requests.

    out, scale, residual = rms_norm(x, gain, residual, out_dtype=torch.float8_e4m3fn)
    h = gated_ffn(out, w_gate, w_up, x_scale=scale, gate_scale=sg, up_scale=su)
    y = lora_linear(h, w_down, lora_a, lora_b, lora_scale, adapter)

Everything runs on the current stream of the tensors' device, without synchronising; results and workspaces come from
torch's allocator unless the caller gives the results.  Last dimensions are contiguous.  Between rows rms_norm takes any
stride; the products want rows on 16-byte boundaries (strides of 8 values, e4m3: 16) that do not lie over one another, so a dh that was expanded
from a scalar has to be made contiguous.  Arguments that
the operators do not take raise ValueError or XemaError before anything is launched; what a kernel finds out later (an adapter
index beyond the adapters, a wait that ran out) is raised by `check`.

The functions are not recorded by autograd: while gradients are on, operands that require one are refused.  In a training program they stand in a
torch.autograd.Function, or under torch.no_grad(), and gated_ffn_backward is the gradient of gated_ffn.  Forward-mode derivatives, vmap and tracers
(torch.jit.trace, make_fx) are refused; torch.compile runs its graphs around the calls.
"""
from __future__ import annotations

import ctypes
import os
import threading

import torch

from . import binding as xb
from .session import _current_device

_ACTIVATIONS = {"silu": xb.ACT_SILU, "gelu_tanh": xb.ACT_GELU_TANH}
_TYPES = {torch.bfloat16: False, torch.float8_e4m3fn: True}
_status = {}
_status_lock = threading.Lock()
_module = None


def _ops():
    """The compiled module, with the library's functions bound to it.  Raises if it was not built."""
    global _module
    if _module is None:
        lib = xb.lib()
        if not os.path.exists(os.path.join(os.path.dirname(os.path.abspath(__file__)), "_torch_ops.so")):
            raise ImportError("_torch_ops.so is not built: run `python -m paper_2607_11136_b200.build`")
        from . import _torch_ops
        _torch_ops.bind(*(ctypes.cast(getattr(lib, name), ctypes.c_void_p).value for name in (
            "xema_op_rms_norm", "xema_op_gated_ffn", "xema_op_gated_ffn_grad", "xema_op_lora", "xema_lora_work_bytes")))
        _module = _torch_ops
    return _module


def _status_of(t) -> int:
    """Address of the status word of the tensor's device (one for all calls; kernels only write it when something went wrong)."""
    index = t.get_device() if isinstance(t, torch.Tensor) else -1
    address = _status.get(index)
    if address is not None:
        return address[1]
    if index < 0:
        raise ValueError("want tensors on a CUDA device (there is no CPU fallback)")
    if torch.cuda.is_current_stream_capturing():
        raise RuntimeError("the first call on a device makes its status word: make one before the capture begins")
    with _status_lock, torch.inference_mode(False):       # (a word made in that mode could not be cleared outside)
        if index not in _status:
            word = torch.zeros(1, dtype=torch.int32, device="cuda:%d" % index)
            torch.cuda.current_stream(index).synchronize()      # (other streams may be the first to use it)
            _status[index] = (word, word.data_ptr())
        return _status[index][1]


def check(device=None) -> None:
    """Waits for the device (the current one, unless given) and raises XemaError if a kernel of this module reported a failure since
    the last check."""
    index = None if device is None else torch.device(device).index
    if index is None:
        index = _current_device()
    torch.cuda.synchronize(index)
    if index not in _status:
        return
    word = _status[index][0]
    value = int(word.item()) & 0xFFFFFFFF
    if value:
        word.zero_()
        if value == xb.DEVICE_STATUS_ADAPTER:
            raise xb.XemaError(xb.XEMA_EINVAL, "lora_linear: an adapter index lies beyond the adapters")
        raise xb.XemaError(xb.XEMA_ETIMEOUT, "device status 0x%08x" % value)


def _activation(name: str) -> int:
    code = _ACTIVATIONS.get(name)
    if code is None:
        raise ValueError("activation: want one of %s" % ", ".join(_ACTIVATIONS))
    return code


def rms_norm(x, gain, residual=None, *, eps: float = 1e-6, out_dtype=torch.bfloat16, out=None, residual_out=None):
    """v = x + residual; out = v / sqrt(mean(v^2) + eps) * gain per row -> (out, scale, residual_out).

    x: bf16 [rows, D] (or fp32 without a residual), residual: bf16 or fp32 of the same shape.  out_dtype
    bf16, or float8_e4m3fn: then scale is fp32 [rows] with out * scale the result, otherwise None.  residual_out holds v in the
    residual's type; give the residual itself to update it in place.  D up to 65536, any strides between rows."""
    e4m3 = _TYPES.get(out_dtype)
    if e4m3 is None:
        raise ValueError("out_dtype: want bfloat16 or float8_e4m3fn")
    r = (_module or _ops()).rms_norm(x, gain, residual, eps, e4m3, out, residual_out)
    if r.__class__ is int:
        raise xb.XemaError(r, "xema_op_rms_norm")
    return r


def gated_ffn(x, w_gate, w_up, *, activation: str = "silu", x_scale=None, gate_scale=None, up_scale=None, out=None,
              save: bool = False):
    """h = act(x w_gate^T) * (x w_up^T) in bf16, x [rows, width], weights [ffn, width]; -> h, or (h, saved) with save.

    bf16, or float8_e4m3fn operands with the fp32 factors x_scale [rows], gate_scale and up_scale [ffn] that their rows were
    divided by.  width is a multiple of 8 (e4m3: 16), ffn of 8.  `saved` (int16 [3, rows, ffn]: the bits of both
    projections in bf16, and a byte of each that bf16 leaves out) is what gated_ffn_backward takes; bf16 operands only."""
    r = (_module or _ops()).gated_ffn(x, w_gate, w_up, _activation(activation), x_scale, gate_scale, up_scale, out, save, _status_of(x))
    if r.__class__ is int:
        raise xb.XemaError(r, "xema_op_gated_ffn")
    return r


def gated_ffn_backward(dh, x, w_gate, w_up, saved, *, activation: str = "silu", want_x: bool = True, want_weights: bool = True,
                       reuse_saved: bool = False):
    """Gradients of gated_ffn from dh [rows, ffn] and what the forward call saved -> (dx, dw_gate, dw_up) in bf16; None for
    those that are not wanted.  reuse_saved: `saved` serves as the workspace and is overwritten."""
    r = (_module or _ops()).gated_ffn_backward(dh, x, w_gate, w_up, saved, _activation(activation), want_x, want_weights, reuse_saved,
                                               _status_of(x))
    if r.__class__ is int:
        raise xb.XemaError(r, "xema_op_gated_ffn_grad")
    return r


def lora_linear(x, weight, lora_a, lora_b, scale, adapter, *, bias=None, out=None):
    """out[b] = x[b] weight^T + bias + scale[a] (x[b] lora_a[a]^T) lora_b[a]^T with a = adapter[b], none where that is negative.

    x: bf16 [batch, rows, K], weight: bf16 [N, K], lora_a: bf16 [n, rank, K], lora_b: bf16 [n, N, rank], scale: fp32 [n],
    adapter: int32 [batch] on the device.  K, N and rank are multiples of 8, rank at most 128 (adapters of a lower rank
    are filled up with zeros).  An index of n or more counts as no adapter and is raised by `check`."""
    r = (_module or _ops()).lora_linear(x, weight, lora_a, lora_b, scale, adapter, bias, out, _status_of(x))
    if r.__class__ is int:
        raise xb.XemaError(r, "xema_op_lora")
    return r
