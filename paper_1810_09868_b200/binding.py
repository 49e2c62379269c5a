"""ctypes binding of libvgg19_b200.so: the same entry points as
include/vgg19_b200.h, with argument marshalling only.  Device tensors are
passed as torch CUDA tensors (or raw integer addresses), host buffers as
numpy arrays or torch CPU tensors.  Nothing here computes anything: if the
CUDA library is missing or fails to load, importing the symbols raises.
"""
from __future__ import annotations

import ctypes
import os

from . import build as _build

VGG19_OK = 0
VGG19_ERR_ARG, VGG19_ERR_SHAPE, VGG19_ERR_WORKSPACE = -1, -2, -3
VGG19_ERR_CUDA, VGG19_ERR_DEVICE_TIMEOUT, VGG19_ERR_UNSUPPORTED_ARCH, VGG19_ERR_RANGE = -4, -5, -6, -7
VGG19_FP32, VGG19_BF16 = 0, 1
VGG19_FLAG_NO_GRAPH, VGG19_FLAG_NO_TENSOR_CORES, VGG19_FLAG_NO_CTA_PAIRS, VGG19_FLAG_FIRST_FUSION = 1, 2, 4, 8
VGG19_FLAG_SPLIT_F16, VGG19_FLAG_DENSE_Q4 = 16, 32
VGG19_DENSE_Q4_GROUP = 64
VGG19_MODE_FORWARD, VGG19_MODE_BACKWARD, VGG19_MODE_TRAIN = 0, 1, 2

EXPORTS = (
    "vgg19_create", "vgg19_create_from_params", "vgg19_destroy", "vgg19_param_count", "vgg19_param_info",
    "vgg19_get_params", "vgg19_set_params", "vgg19_workspace_bytes", "vgg19_bind_workspace",
    "vgg19_forward", "vgg19_backward", "vgg19_sgd_step", "vgg19_train_step", "vgg19_train_steps",
    "vgg19_set_dense_grads_event", "vgg19_io_bytes", "vgg19_forward_host", "vgg19_forward_host_async", "vgg19_backward_host",
    "vgg19_conv_layer_forward", "vgg19_conv_layer_forward_ex", "vgg19_first_block_forward", "vgg19_conv_layer_backward", "vgg19_conv_layer_backward_ex", "vgg19_dense_layer_forward", "vgg19_dense_layer_backward", "vgg19_saved_tensor", "vgg19_conv_wgrad_static", "vgg19_sync_status", "vgg19_selftest_wait_timeout", "vgg19_launch_count",
    "vgg19_describe", "vgg19_last_error",
    "vgg19_logprobs", "vgg19_logprobs_backward", "vgg19_ops_status",
    "vgg19_q4_code_bytes", "vgg19_q4_scale_bytes", "vgg19_q4_pack", "vgg19_q4_linear",
    "vgg19_selftest_operator_timeout", "vgg19_muon_workspace_bytes", "vgg19_muon_update", "vgg19_muon_step_bytes", "vgg19_muon_step",
    "vgg19_dropout", "vgg19_dropout_backward", "vgg19_set_dropout",
    "vgg19_linear_cross_entropy_bytes", "vgg19_linear_cross_entropy", "vgg19_linear_cross_entropy_backward",
)
VGG19_NO_CLASS = -1
VGG19_LOGPROBS_MAX_TOP, VGG19_LOGPROBS_MAX_IDS = 32, 256
VGG19_SELFTEST_DENSE_Q4, VGG19_SELFTEST_UPDATE, VGG19_SELFTEST_UPDATE_STEPS = 0, 1, 2
VGG19_SELFTEST_LOSS = 4
VGG19_SELFTEST_BYTES = 1048576


class vgg19_config(ctypes.Structure):
    _fields_ = [("height", ctypes.c_int32), ("width", ctypes.c_int32), ("batch_max", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("flags", ctypes.c_uint32)]


class vgg19_muon_tensor(ctypes.Structure):
    _fields_ = [("w", ctypes.c_void_p), ("w_bf16", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("momentum", ctypes.c_void_p),
                ("rows", ctypes.c_int64), ("cols", ctypes.c_int64)]


class vgg19_linear_loss(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("ldx", ctypes.c_int64), ("w", ctypes.c_void_p), ("ldw", ctypes.c_int64), ("bias", ctypes.c_void_p),
                ("labels", ctypes.c_void_p), ("rows", ctypes.c_int64), ("in_", ctypes.c_int32), ("classes", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class Vgg19Error(RuntimeError):
    def __init__(self, code, text):
        super().__init__(f"vgg19 error {code}: {text}")
        self.code = code


_lib = None


def lib_path() -> str:
    return _build.LIB


def load():
    """Load the CUDA library; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    path = lib_path()
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with `python -c 'import __graft_entry__ as g; g.build()'` "
                           "(there is no CPU fallback)")
    L = ctypes.CDLL(path)
    vp, i32, i64, u64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64, ctypes.c_size_t
    f32 = ctypes.c_float
    cfgp = ctypes.POINTER(vgg19_config)
    sig = {
        "vgg19_create": ([cfgp, u64, ctypes.POINTER(vp)], ctypes.c_int),
        "vgg19_create_from_params": ([cfgp, vp, ctypes.POINTER(vp)], ctypes.c_int),
        "vgg19_destroy": ([vp], None),
        "vgg19_param_count": ([vp, ctypes.POINTER(i32), ctypes.POINTER(sz)], ctypes.c_int),
        "vgg19_param_info": ([vp, i32, ctypes.POINTER(sz), ctypes.POINTER(i32), ctypes.POINTER(ctypes.c_int64)], ctypes.c_int),
        "vgg19_get_params": ([vp, vp], ctypes.c_int),
        "vgg19_set_params": ([vp, vp], ctypes.c_int),
        "vgg19_workspace_bytes": ([vp, i32, i32], sz),
        "vgg19_bind_workspace": ([vp, vp, sz], ctypes.c_int),
        "vgg19_forward": ([vp, vp, i32, vp, vp, vp], ctypes.c_int),
        "vgg19_backward": ([vp, vp, vp, i32, vp, vp, vp, vp], ctypes.c_int),
        "vgg19_sgd_step": ([vp, vp, ctypes.c_float, vp], ctypes.c_int),
        "vgg19_train_step": ([vp, vp, vp, i32, ctypes.c_float, vp, vp], ctypes.c_int),
        "vgg19_train_steps": ([vp, vp, vp, i32, i32, ctypes.c_float, vp, vp], ctypes.c_int),
        "vgg19_set_dense_grads_event": ([vp, vp], ctypes.c_int),
        "vgg19_io_bytes": ([vp, i32, i32], sz),
        "vgg19_forward_host": ([vp, vp, i32, vp, vp, vp], ctypes.c_int),
        "vgg19_forward_host_async": ([vp, vp, i32, vp, vp, vp], ctypes.c_int),
        "vgg19_backward_host": ([vp, vp, vp, i32, vp, vp, vp], ctypes.c_int),
        "vgg19_conv_layer_forward": ([vp, i32, vp, i32, vp, vp, vp], ctypes.c_int),
        "vgg19_conv_layer_backward": ([vp, i32, vp, vp, i32, vp, vp, vp, vp], ctypes.c_int),
        "vgg19_conv_layer_forward_ex": ([vp, i32, vp, i32, vp, vp, vp, vp], ctypes.c_int),
        "vgg19_first_block_forward": ([vp, vp, i32, vp, vp, vp], ctypes.c_int),
        "vgg19_conv_layer_backward_ex": ([vp, i32, vp, vp, i32, vp, vp, vp, vp, vp, vp], ctypes.c_int),
        "vgg19_dense_layer_forward": ([vp, i32, vp, i32, vp, vp, vp], ctypes.c_int),
        "vgg19_dense_layer_backward": ([vp, i32, vp, vp, i32, vp, vp, vp, vp, vp], ctypes.c_int),
        "vgg19_saved_tensor": ([vp, i32, i32, i32, ctypes.POINTER(sz), ctypes.POINTER(ctypes.c_int64)], ctypes.c_int),
        "vgg19_conv_wgrad_static": ([vp, vp, i32, i32, i32, i32, i32, i32, vp, vp, ctypes.POINTER(sz), vp], ctypes.c_int),
        "vgg19_sync_status": ([vp, vp], ctypes.c_int),
        "vgg19_selftest_wait_timeout": ([vp, vp], ctypes.c_int),
        "vgg19_launch_count": ([vp, i32, ctypes.POINTER(i32)], ctypes.c_int),
        "vgg19_describe": ([vp, ctypes.c_char_p, sz], ctypes.c_int),
        "vgg19_last_error": ([vp], ctypes.c_char_p),
        "vgg19_logprobs": ([vp, i32, i64, i32, i64, vp, i32, i32, vp, vp, vp, vp, vp, vp], ctypes.c_int),
        "vgg19_logprobs_backward": ([vp, i32, i64, i32, i64, vp, i32, vp, vp, vp, vp, vp, i64, vp], ctypes.c_int),
        "vgg19_ops_status": ([vp], ctypes.c_int),
        "vgg19_selftest_operator_timeout": ([vp, i32, vp, sz, vp], ctypes.c_int),
        "vgg19_muon_workspace_bytes": ([vp, i32], sz),
        "vgg19_muon_update": ([vp, i32, f32, f32, f32, i32, i32, vp, sz, vp], ctypes.c_int),
        "vgg19_muon_step_bytes": ([vp], sz),
        "vgg19_muon_step": ([vp, vp, vp, f32, f32, f32, f32, i32, i32, vp, sz, vp], ctypes.c_int),
        "vgg19_dropout": ([vp, i32, i64, i32, i64, f32, u64, u64, vp, u64, vp, i64, vp], ctypes.c_int),
        "vgg19_dropout_backward": ([vp, i32, i64, i32, i64, f32, u64, u64, vp, u64, vp, i64, vp], ctypes.c_int),
        "vgg19_set_dropout": ([vp, f32, u64, u64], ctypes.c_int),
        "vgg19_linear_cross_entropy_bytes": ([vp, i32], sz),
        "vgg19_linear_cross_entropy": ([vp, vp, vp, vp, sz, vp], ctypes.c_int),
        "vgg19_linear_cross_entropy_backward": ([vp, vp, vp, vp, i64, vp, i32, i64, vp, vp, sz, vp], ctypes.c_int),
        "vgg19_q4_code_bytes": ([i32, i32], sz),
        "vgg19_q4_scale_bytes": ([i32, i32, i32], sz),
        "vgg19_q4_pack": ([vp, i32, i32, i32, i64, i32, vp, vp, vp], ctypes.c_int),
        "vgg19_q4_linear": ([vp, i32, i64, i32, i64, vp, vp, i32, i32, vp, i32, vp, vp, vp], ctypes.c_int),
    }
    for name, (args, res) in sig.items():
        fn = getattr(L, name)
        fn.argtypes = args
        fn.restype = res
    _lib = L
    return L


def _ptr(x):
    """Address of a torch tensor / numpy array / int / None."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    if hasattr(x, "data_ptr"):
        return x.data_ptr()
    if hasattr(x, "ctypes"):
        return x.ctypes.data
    raise TypeError(type(x))


def _stream(stream):
    if stream is None:
        return None
    return stream if isinstance(stream, int) else stream.cuda_stream


def _check(net, rc):
    if rc != VGG19_OK:
        raise Vgg19Error(rc, load().vgg19_last_error(net).decode())
    return rc


def vgg19_create(height, width, batch_max, dtype, seed, flags=0):
    cfg = vgg19_config(height, width, batch_max, dtype, flags)
    out = ctypes.c_void_p()
    _check(None, load().vgg19_create(ctypes.byref(cfg), seed, ctypes.byref(out)))
    return out.value


def vgg19_create_from_params(height, width, batch_max, dtype, host_params, flags=0):
    cfg = vgg19_config(height, width, batch_max, dtype, flags)
    out = ctypes.c_void_p()
    _check(None, load().vgg19_create_from_params(ctypes.byref(cfg), _ptr(host_params), ctypes.byref(out)))
    return out.value


def vgg19_destroy(net):
    load().vgg19_destroy(net)


def vgg19_param_count(net):
    n, e = ctypes.c_int32(), ctypes.c_size_t()
    _check(net, load().vgg19_param_count(net, ctypes.byref(n), ctypes.byref(e)))
    return n.value, e.value


def vgg19_param_info(net, i):
    off, rank = ctypes.c_size_t(), ctypes.c_int32()
    dims = (ctypes.c_int64 * 4)()
    _check(net, load().vgg19_param_info(net, i, ctypes.byref(off), ctypes.byref(rank), dims))
    return off.value, tuple(dims[:rank.value])


def vgg19_get_params(net, host_params):
    return _check(net, load().vgg19_get_params(net, _ptr(host_params)))


def vgg19_set_params(net, host_params):
    return _check(net, load().vgg19_set_params(net, _ptr(host_params)))


def vgg19_sgd_step(net, grads, lr, stream=None):
    return _check(net, load().vgg19_sgd_step(net, _ptr(grads), float(lr), _stream(stream)))


def vgg19_train_step(net, images, labels, batch, lr, loss=None, stream=None):
    return _check(net, load().vgg19_train_step(net, _ptr(images), _ptr(labels), batch, float(lr), _ptr(loss), _stream(stream)))


def vgg19_train_steps(net, images, labels, batch, steps, lr, losses=None, stream=None):
    return _check(net, load().vgg19_train_steps(net, _ptr(images), _ptr(labels), batch, steps, float(lr), _ptr(losses),
                                                 _stream(stream)))


def vgg19_set_dense_grads_event(net, event):
    """event: a torch.cuda.Event that has been recorded at least once (so that its handle exists), a raw
    cudaEvent_t as an integer, or None."""
    h = None if event is None else (event if isinstance(event, int) else event.cuda_event)
    return _check(net, load().vgg19_set_dense_grads_event(net, h))


def vgg19_workspace_bytes(net, batch, mode):
    return load().vgg19_workspace_bytes(net, batch, mode)


def vgg19_io_bytes(net, batch, mode):
    return load().vgg19_io_bytes(net, batch, mode)


def vgg19_bind_workspace(net, workspace, nbytes):
    return _check(net, load().vgg19_bind_workspace(net, _ptr(workspace), nbytes))


def vgg19_forward(net, images, batch, logits, probs=None, stream=None):
    return _check(net, load().vgg19_forward(net, _ptr(images), batch, _ptr(logits), _ptr(probs), _stream(stream)))


def vgg19_backward(net, images, labels, batch, grads, loss=None, logits=None, stream=None):
    return _check(net, load().vgg19_backward(net, _ptr(images), _ptr(labels), batch, _ptr(grads), _ptr(loss),
                                             _ptr(logits), _stream(stream)))


def vgg19_forward_host(net, host_images, batch, host_logits, host_probs=None, stream=None):
    return _check(net, load().vgg19_forward_host(net, _ptr(host_images), batch, _ptr(host_logits),
                                                  _ptr(host_probs), _stream(stream)))


def vgg19_forward_host_async(net, host_images, batch, host_logits, host_probs=None, stream=None):
    return _check(net, load().vgg19_forward_host_async(net, _ptr(host_images), batch, _ptr(host_logits),
                                                        _ptr(host_probs), _stream(stream)))


def vgg19_backward_host(net, host_images, host_labels, batch, host_grads, host_loss=None, stream=None):
    return _check(net, load().vgg19_backward_host(net, _ptr(host_images), _ptr(host_labels), batch,
                                                   _ptr(host_grads), _ptr(host_loss), _stream(stream)))


def vgg19_conv_layer_forward(net, layer, x, batch, y, pooled=None, stream=None):
    return _check(net, load().vgg19_conv_layer_forward(net, layer, _ptr(x), batch, _ptr(y), _ptr(pooled),
                                                        _stream(stream)))


def vgg19_conv_layer_backward(net, layer, x, dz, batch, dw, db, dx=None, stream=None):
    return _check(net, load().vgg19_conv_layer_backward(net, layer, _ptr(x), _ptr(dz), batch, _ptr(dw), _ptr(db),
                                                         _ptr(dx), _stream(stream)))


def vgg19_dense_layer_forward(net, layer, x, batch, y=None, y_f32=None, stream=None):
    return _check(net, load().vgg19_dense_layer_forward(net, layer, _ptr(x), batch, _ptr(y), _ptr(y_f32), _stream(stream)))


def vgg19_dense_layer_backward(net, layer, x, dy, batch, dw, db, dx=None, relu_mask=None, stream=None):
    return _check(net, load().vgg19_dense_layer_backward(net, layer, _ptr(x), _ptr(dy), batch, _ptr(dw), _ptr(db),
                                                          _ptr(dx), _ptr(relu_mask), _stream(stream)))


def vgg19_conv_layer_forward_ex(net, layer, x, batch, y, pooled=None, pool_code=None, stream=None):
    return _check(net, load().vgg19_conv_layer_forward_ex(net, layer, _ptr(x), batch, _ptr(y), _ptr(pooled),
                                                           _ptr(pool_code), _stream(stream)))


def vgg19_first_block_forward(net, images, batch, y2=None, pooled=None, stream=None):
    return _check(net, load().vgg19_first_block_forward(net, _ptr(images), batch, _ptr(y2), _ptr(pooled), _stream(stream)))


def vgg19_conv_layer_backward_ex(net, layer, x, dz, batch, dw=None, db=None, dx=None, relu_mask=None, pool_code=None,
                                 stream=None):
    return _check(net, load().vgg19_conv_layer_backward_ex(net, layer, _ptr(x), _ptr(dz), batch, _ptr(dw), _ptr(db),
                                                            _ptr(dx), _ptr(relu_mask), _ptr(pool_code), _stream(stream)))


def vgg19_saved_tensor(net, batch, mode, index):
    off = ctypes.c_size_t()
    dims = (ctypes.c_int64 * 4)()
    _check(net, load().vgg19_saved_tensor(net, batch, mode, index, ctypes.byref(off), dims))
    return off.value, tuple(dims)


VGG19_STATIC_SCRATCH_BYTES = 8 << 20


def vgg19_conv_wgrad_static(x, dz, batch, height, width, cin, cout, dtype, dw, db, stream=None):
    """Allocation-free filter/bias gradient; returns (status, scratch bytes the shape needs)."""
    need = ctypes.c_size_t()
    rc = load().vgg19_conv_wgrad_static(_ptr(x), _ptr(dz), batch, height, width, cin, cout, dtype, _ptr(dw), _ptr(db),
                                        ctypes.byref(need), _stream(stream))
    return rc, need.value


def vgg19_sync_status(net, stream=None):
    return _check(net, load().vgg19_sync_status(net, _stream(stream)))


def vgg19_selftest_wait_timeout(net, stream=None):
    return _check(net, load().vgg19_selftest_wait_timeout(net, _stream(stream)))


def vgg19_launch_count(net, mode):
    n = ctypes.c_int32()
    _check(net, load().vgg19_launch_count(net, mode, ctypes.byref(n)))
    return n.value


def vgg19_describe(net):
    need = load().vgg19_describe(net, None, 0)
    buf = ctypes.create_string_buffer(need + 1)
    load().vgg19_describe(net, buf, need + 1)
    return buf.value.decode()


def vgg19_last_error(net=None):
    return load().vgg19_last_error(net).decode()


# ---- operators without a handle -------------------------------------------------------------------------------
# They take torch CUDA tensors and read sizes, strides and types from them; a tensor that does not fit is refused here,
# before its address reaches the library.  They run on the tensors' device, whichever is current.  stream as above:
# None is the legacy default stream.  The ones a program calls once per answer go through _tensor_calls first
# (csrc/tensor_calls.cpp), which makes the same checks in a tenth of the time and answers None where one of them fails.

_tensor_calls = None


def _calls():
    global _tensor_calls
    if _tensor_calls is None:
        load()
        import importlib.util

        from .build import calls_path
        path = calls_path()  # (imports torch, whose libraries come first)
        try:
            spec = importlib.util.spec_from_file_location(__package__ + "._tensor_calls", path)
            module = importlib.util.module_from_spec(spec)
            spec.loader.exec_module(module)
        except ImportError as e:
            raise RuntimeError(f"{path}, the compiled calls for this torch and this Python, cannot be loaded: build them with "
                               "`python -c 'import __graft_entry__ as g; g.build()'`") from e
        _tensor_calls = module
    return _tensor_calls


def _answered(rc):
    return rc if rc == VGG19_OK else _check(None, rc)


_MOST = (1 << 31) - 1


def _refuse(code, text):
    raise Vgg19Error(code, text)


_types = None  # (storage types of the library, float32, bfloat16, int32, current_device), once torch is there


def _torch():
    global _types
    if _types is None:
        import torch
        _types = ({torch.float32: VGG19_FP32, torch.bfloat16: VGG19_BF16}, torch.float32, torch.bfloat16, torch.int32,
                  torch.cuda.current_device)
    return _types


def _tensor(t, name, dtype, shape, dev):
    """Address of a dense tensor of that type and shape on CUDA device `dev`; None stays None."""
    if t is None:
        return None
    if t.dtype is dtype and t.shape == shape and t.get_device() == dev and t.is_contiguous():
        return t.data_ptr()
    if t.dtype != dtype:
        _refuse(VGG19_ERR_ARG, f"{name} is {t.dtype}, not {dtype}")
    if tuple(t.shape) != shape:
        _refuse(VGG19_ERR_SHAPE, f"{name} is {tuple(t.shape)}, not {shape}")
    if not t.is_contiguous():
        _refuse(VGG19_ERR_ARG, f"{name} is not contiguous")
    _refuse(VGG19_ERR_ARG, f"{name} is on {t.device}, not on cuda:{dev}")


def _last(t):
    return t.shape[-1] if t.dim() else 0  # (what has no dimension is refused for its shape)


def _rows_of(t, name):
    """(storage type, rows, columns, row stride, CUDA device index) of a 2-d tensor whose rows are dense."""
    dtype = _torch()[0].get(t.dtype)
    if dtype is None:
        _refuse(VGG19_ERR_ARG, f"{name} is {t.dtype}, neither float32 nor bfloat16")
    if t.dim() != 2:
        _refuse(VGG19_ERR_SHAPE, f"{name} has {t.dim()} dimensions, not 2")
    rows, cols = t.shape
    if cols > _MOST:  # (a C int: beyond it the library would be told another size)
        _refuse(VGG19_ERR_SHAPE, f"{name} has {cols} columns, at most {_MOST} are possible")
    dev = t.get_device()
    if dev < 0:
        _refuse(VGG19_ERR_ARG, f"{name} is on {t.device}, not on a CUDA device")
    if t.is_contiguous():
        return dtype, rows, cols, cols, dev
    ld = t.stride(0) if rows > 1 else cols
    if (cols > 1 and t.stride(1) != 1) or ld < cols:
        _refuse(VGG19_ERR_ARG, f"{name}: strides {t.stride()}; a row has to be dense and rows must not overlap")
    return dtype, rows, cols, ld, dev


def _call(dev, fn, *args):
    """fn(*args) on the tensors' device."""
    if dev == _types[4]():
        rc = fn(*args)
    else:
        import torch
        with torch.cuda.device(dev):
            rc = fn(*args)
    return rc if rc == VGG19_OK else _check(None, rc)


def vgg19_logprobs(logits, ids=None, logprob=None, lse=None, entropy=None, top_id=None, top_logprob=None, stream=None):
    """logits [rows][classes] (a row stride is allowed), ids and logprob [rows][n_ids], lse and entropy [rows], top_id and
    top_logprob [rows][top_k]; what is None is left out."""
    rc = (_tensor_calls or _calls()).logprobs(logits, ids, logprob, lse, entropy, top_id, top_logprob, stream)
    if rc is not None:
        return _answered(rc)
    dtype, rows, classes, ld, dev = _rows_of(logits, "logits")
    _, f32, _, i32, _ = _types
    if (ids is None) != (logprob is None) or (top_id is None) != (top_logprob is None):
        _refuse(VGG19_ERR_ARG, "ids goes with logprob, and top_id with top_logprob")
    n_ids = 0 if ids is None else _last(ids)
    top_k = 0 if top_id is None else _last(top_id)
    given, top, each = (rows, n_ids), (rows, top_k), (rows,)
    return _call(dev, (_lib or load()).vgg19_logprobs, logits.data_ptr(), dtype, rows, classes, ld, _tensor(ids, "ids", i32, given, dev),
                 n_ids, top_k, _tensor(logprob, "logprob", f32, given, dev), _tensor(lse, "lse", f32, each, dev),
                 _tensor(entropy, "entropy", f32, each, dev), _tensor(top_id, "top_id", i32, top, dev),
                 _tensor(top_logprob, "top_logprob", f32, top, dev), _stream(stream))


def vgg19_logprobs_backward(logits, ids, lse, entropy, d_logprob, d_entropy, d_logits, stream=None):
    """The gradient at the logits; ids and d_logprob may be None together, and so may d_entropy (entropy then too).
    d_logits may be logits."""
    rc = (_tensor_calls or _calls()).logprobs_backward(logits, ids, lse, entropy, d_logprob, d_entropy, d_logits, stream)
    if rc is not None:
        return _answered(rc)
    dtype, rows, classes, ld, dev = _rows_of(logits, "logits")
    d_dtype, d_rows, d_classes, d_ld, d_dev = _rows_of(d_logits, "d_logits")
    if (d_dtype, d_rows, d_classes, d_dev) != (dtype, rows, classes, dev):
        _refuse(VGG19_ERR_SHAPE, "d_logits differs from logits in type, shape or device")
    _, f32, _, i32, _ = _types
    if (ids is None) != (d_logprob is None):
        _refuse(VGG19_ERR_ARG, "ids goes with d_logprob")
    if lse is None:
        _refuse(VGG19_ERR_ARG, "lse is needed")
    n_ids = 0 if ids is None else _last(ids)
    given, each = (rows, n_ids), (rows,)
    return _call(dev, (_lib or load()).vgg19_logprobs_backward, logits.data_ptr(), dtype, rows, classes, ld,
                 _tensor(ids, "ids", i32, given, dev), n_ids, _tensor(lse, "lse", f32, each, dev),
                 _tensor(entropy, "entropy", f32, each, dev), _tensor(d_logprob, "d_logprob", f32, given, dev),
                 _tensor(d_entropy, "d_entropy", f32, each, dev), d_logits.data_ptr(), d_ld, _stream(stream))


def vgg19_q4_code_bytes(out, in_):
    return load().vgg19_q4_code_bytes(out, in_)


def vgg19_q4_scale_bytes(out, in_, group):
    return load().vgg19_q4_scale_bytes(out, in_, group)


def _q4_buffers(codes, scales, out, in_, group, dev):
    lib = _lib or load()
    if not 0 < out <= _MOST or group not in (32, 64, 128):
        _refuse(VGG19_ERR_SHAPE if group in (32, 64, 128) else VGG19_ERR_ARG, f"{out} rows in groups of {group}")
    for t, name, need in ((codes, "codes", lib.vgg19_q4_code_bytes(out, in_)), (scales, "scales", lib.vgg19_q4_scale_bytes(out, in_, group))):
        if t.get_device() != dev or not t.is_contiguous():
            _refuse(VGG19_ERR_ARG, f"{name} is on {t.device}, or not contiguous")
        if t.numel() * t.element_size() < need:
            _refuse(VGG19_ERR_SHAPE, f"{name} holds {t.numel() * t.element_size()} bytes, {out} x {in_} in groups of {group} take {need}")
    return lib


def vgg19_q4_pack(w, group, codes, scales, stream=None):
    """w [out][in] (a row stride is allowed) into codes and scales, of vgg19_q4_code_bytes and vgg19_q4_scale_bytes."""
    dtype, out, in_, ld, dev = _rows_of(w, "w")
    lib = _q4_buffers(codes, scales, out, in_, group, dev)
    return _call(dev, lib.vgg19_q4_pack, w.data_ptr(), dtype, out, in_, ld, group, codes.data_ptr(), scales.data_ptr(), _stream(stream))


def vgg19_q4_linear(x, codes, scales, out, group, bias=None, relu=False, y=None, y_f32=None, stream=None):
    """x [rows][in] (a row stride is allowed); y [rows][out] in x's type and / or y_f32 in fp32."""
    rc = (_tensor_calls or _calls()).q4_linear(x, codes, scales, out, group, bias, relu, y, y_f32, stream)
    if rc is not None:
        return _answered(rc)
    dtype, rows, in_, ldx, dev = _rows_of(x, "x")
    f32 = _types[1]
    lib = _q4_buffers(codes, scales, out, in_, group, dev)
    shape = (rows, out)
    return _call(dev, lib.vgg19_q4_linear, x.data_ptr(), dtype, rows, in_, ldx, codes.data_ptr(), scales.data_ptr(), out, group,
                 _tensor(bias, "bias", f32, (out,), dev), 1 if relu else 0, _tensor(y, "y", x.dtype, shape, dev),
                 _tensor(y_f32, "y_f32", f32, shape, dev), _stream(stream))


class MuonTensors:
    """The tensors of an update as the library takes them, holding on to the torch tensors whose addresses it has."""

    def __init__(self, tensors):
        _, f32, b16, _, _ = _torch()
        self.tensors = [tuple(t) for t in tensors]
        self.count = len(self.tensors)
        self.array = (vgg19_muon_tensor * max(self.count, 1))()
        self.device = None
        for a, (w, w16, grad, momentum) in zip(self.array, self.tensors):
            dtype, rows, cols, ld, dev = _rows_of(w, "w")
            if self.device is None:
                self.device = dev
            a.w = _tensor(w, "w", f32, (rows, cols), self.device)
            a.w_bf16 = _tensor(w16, "w_bf16", b16, (rows, cols), self.device)
            a.grad = _tensor(grad, "grad", f32, (rows, cols), self.device)
            a.momentum = _tensor(momentum, "momentum", f32, (rows, cols), self.device)
            a.rows, a.cols = rows, cols


def vgg19_muon_tensors(tensors):
    """A list of (w, w_bf16 or None, grad, momentum), fp32 matrices of one shape each, for vgg19_muon_update; it may be kept and
    used again while those tensors live."""
    return MuonTensors(tensors)


def vgg19_muon_workspace_bytes(tensors):
    t = tensors if isinstance(tensors, MuonTensors) else MuonTensors(tensors)
    return load().vgg19_muon_workspace_bytes(t.array, t.count)


def _workspace(workspace, device):
    if workspace.get_device() != device:
        _refuse(VGG19_ERR_ARG, f"the workspace is on {workspace.device}, not on cuda:{device}")
    if not workspace.is_contiguous():
        _refuse(VGG19_ERR_ARG, "the workspace is not contiguous")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def vgg19_muon_update(tensors, lr, momentum, decay, steps, nesterov, workspace, stream=None):
    t = tensors if isinstance(tensors, MuonTensors) else MuonTensors(tensors)
    if t.count == 0:
        return VGG19_OK
    ptr, nbytes = _workspace(workspace, t.device)
    return _call(t.device, load().vgg19_muon_update, t.array, t.count, lr, momentum, decay, steps, int(nesterov), ptr, nbytes, _stream(stream))


def vgg19_muon_step_bytes(net):
    return load().vgg19_muon_step_bytes(net)


def vgg19_muon_step(net, grads, momentum_buffer, lr, momentum, decay, bias_lr, steps, nesterov, workspace, nbytes, stream=None):
    return _check(net, load().vgg19_muon_step(net, _ptr(grads), _ptr(momentum_buffer), lr, momentum, decay, bias_lr, steps, int(nesterov),
                                              _ptr(workspace), nbytes, _stream(stream)))


def _word64(v, what):
    if not 0 <= v < 1 << 64:
        _refuse(VGG19_ERR_ARG, f"{what} {v} is not an unsigned 64-bit number")
    if int(v) != v:
        _refuse(VGG19_ERR_ARG, f"{what} {v} is not a whole number")
    return int(v)


def _any_dropout(name, x, y, rate, seed, step, step_counter, first, stream):
    source, result = ("dy", "dx") if name.endswith("backward") else ("x", "y")
    dtype, rows, cols, ldx, dev = _rows_of(x, source)
    y_dtype, y_rows, y_cols, ldy, y_dev = _rows_of(y, result)
    if (y_dtype, y_rows, y_cols, y_dev) != (dtype, rows, cols, dev):
        _refuse(VGG19_ERR_SHAPE, f"{result} differs from {source} in type, shape or device")
    seed, step, first = _word64(seed, "seed"), _word64(step, "step"), _word64(first, "first")
    import torch
    counter = _tensor(step_counter, "step_counter", torch.int64, (1,), dev)
    return _call(dev, getattr(_lib or load(), "vgg19_" + name), x.data_ptr(), dtype, rows, cols, ldx, rate, seed, step, counter, first, y.data_ptr(), ldy,
                 _stream(stream))


def vgg19_dropout(x, y, rate, seed, step=0, step_counter=None, first=0, stream=None):
    """y = x with values dropped at `rate` and the others scaled up; [rows][cols], row strides are allowed, y may be x.
    step_counter: an int64 CUDA tensor of one element, added to step on the device."""
    rc = (_tensor_calls or _calls()).dropout(x, y, rate, seed, step, step_counter, first, stream)
    return _answered(rc) if rc is not None else _any_dropout("dropout", x, y, rate, seed, step, step_counter, first, stream)


def vgg19_dropout_backward(dy, dx, rate, seed, step=0, step_counter=None, first=0, stream=None):
    """dx from dy, with what vgg19_dropout was given for the mask; dx may be dy."""
    rc = (_tensor_calls or _calls()).dropout_backward(dy, dx, rate, seed, step, step_counter, first, stream)
    return _answered(rc) if rc is not None else _any_dropout("dropout_backward", dy, dx, rate, seed, step, step_counter, first, stream)


def _linear_loss(x, w, bias, labels):
    """(the layer as the library takes it, CUDA device index)"""
    dtype, rows, in_, ldx, dev = _rows_of(x, "x")
    w_dtype, classes, w_in, ldw, w_dev = _rows_of(w, "w")
    if (w_dtype, w_in, w_dev) != (dtype, in_, dev):
        _refuse(VGG19_ERR_SHAPE, "w differs from x in type, columns or device")
    if classes > _MOST:
        _refuse(VGG19_ERR_SHAPE, f"{classes} classes, at most {_MOST} are possible")
    _, f32, _, i32, _ = _types
    return vgg19_linear_loss(x.data_ptr(), ldx, w.data_ptr(), ldw, _tensor(bias, "bias", f32, (classes,), dev),
                             _tensor(labels, "labels", i32, (rows,), dev), rows, in_, classes, dtype), dev


def vgg19_linear_cross_entropy_bytes(x, w, backward):
    """Bytes of workspace for x [rows][in] and w [classes][in]; 0 for sizes that are refused.  backward: for the loss and for its gradients.
    Fewer rows may take more: a program with batches of several sizes asks for each."""
    layer, dev = _linear_loss(x, w, None, None)
    import torch
    with torch.cuda.device(dev):
        return load().vgg19_linear_cross_entropy_bytes(ctypes.byref(layer), 1 if backward else 0)


def vgg19_linear_cross_entropy(x, w, bias, labels, loss, lse, workspace, stream=None):
    """x [rows][in] and w [classes][in] (row strides are allowed), bias [classes] or None, labels int32 [rows]; loss and lse
    [rows], either may be None."""
    rc = (_tensor_calls or _calls()).linear_cross_entropy(x, w, bias, labels, loss, lse, workspace, stream)
    if rc is not None:
        return _answered(rc)
    layer, dev = _linear_loss(x, w, bias, labels)
    f32, each = _types[1], (layer.rows,)
    return _call(dev, (_lib or load()).vgg19_linear_cross_entropy, ctypes.byref(layer), _tensor(loss, "loss", f32, each, dev),
                 _tensor(lse, "lse", f32, each, dev), *_workspace(workspace, dev), _stream(stream))


def vgg19_linear_cross_entropy_backward(x, w, bias, labels, lse, d_loss, dx, dw, db, workspace, stream=None):
    """Gradients of sum(d_loss * loss): dx [rows][in] in x's type, dw [classes][in] in w's type or fp32 (row strides are allowed), db
    [classes]; any may be None."""
    rc = (_tensor_calls or _calls()).linear_cross_entropy_backward(x, w, bias, labels, lse, d_loss, dx, dw, db, workspace, stream)
    if rc is not None:
        return _answered(rc)
    layer, dev = _linear_loss(x, w, bias, labels)
    f32, each = _types[1], (layer.rows,)
    lddx = lddw = layer.in_
    dw_dtype = layer.dtype
    if dx is not None:
        dx_dtype, dx_rows, dx_cols, lddx, dx_dev = _rows_of(dx, "dx")
        if (dx_dtype, dx_rows, dx_cols, dx_dev) != (layer.dtype, layer.rows, layer.in_, dev):
            _refuse(VGG19_ERR_SHAPE, "dx differs from x in type, shape or device")
    if dw is not None:
        dw_dtype, dw_rows, dw_cols, lddw, dw_dev = _rows_of(dw, "dw")
        if (dw_rows, dw_cols, dw_dev) != (layer.classes, layer.in_, dev):
            _refuse(VGG19_ERR_SHAPE, "dw differs from w in shape or device")
    return _call(dev, (_lib or load()).vgg19_linear_cross_entropy_backward, ctypes.byref(layer), _tensor(lse, "lse", f32, each, dev),
                 _tensor(d_loss, "d_loss", f32, each, dev), _ptr(dx), lddx, _ptr(dw), dw_dtype, lddw,
                 _tensor(db, "db", f32, (layer.classes,), dev), *_workspace(workspace, dev), _stream(stream))


def vgg19_set_dropout(net, rate, seed, first_pass=0):
    return _check(net, load().vgg19_set_dropout(net, rate, _word64(seed, "seed"), _word64(first_pass, "first_pass")))


def vgg19_selftest_operator_timeout(net, which, workspace, stream=None):
    """net or None; workspace: a CUDA tensor of at least VGG19_SELFTEST_BYTES."""
    dev = workspace.get_device()
    if dev < 0:
        _refuse(VGG19_ERR_ARG, f"the workspace is on {workspace.device}, not on a CUDA device")
    _torch()
    return _call(dev, load().vgg19_selftest_operator_timeout, net, which, *_workspace(workspace, dev), _stream(stream))


def vgg19_ops_status(stream=None):
    """Waits for the stream; raises what the operators without a handle recorded on the current device."""
    return _check(None, load().vgg19_ops_status(_stream(stream)))
