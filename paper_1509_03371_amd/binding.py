"""ctypes binding of libsknet.so: the same entry points as include/sknet.h, argument marshalling
only.  Device buffers are torch CUDA tensors (used for memory and streams, nothing else); every
step of the path runs inside the library's HIP kernels.  There is no CPU fallback: if the library
is missing, importing this module raises.
"""
import ctypes as C
import functools
import os

import numpy as np
import torch  # noqa: F401  (imported first so that the library binds to the HIP runtime torch loaded)

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsknet.so")
if not os.path.exists(LIB_PATH):
    raise ImportError("libsknet.so is not built: run `python -m paper_1509_03371_amd.build` "
                      "(or __graft_entry__.build()) first")
lib = C.CDLL(LIB_PATH)

SK_F32, SK_BF16, SK_F16 = 0, 1, 2
SK_CONV, SK_MAXPOOL, SK_LAYERNORM, SK_DROPOUT = 0, 1, 2, 3
SK_ROWS, SK_MAPS = 0, 1
STATUS_NAMES = ["SK_OK", "SK_EINVAL", "SK_ESHAPE", "SK_ESTATE", "SK_ENOMEM", "SK_EDEVICE", "SK_EUNSUPPORTED"]
DTYPES = {"f32": SK_F32, "bf16": SK_BF16, "f16": SK_F16}


class SkLayer(C.Structure):
    _fields_ = [("kind", C.c_int32), ("c_out", C.c_int32), ("k", C.c_int32), ("d", C.c_int32),
                ("s", C.c_int32), ("relu", C.c_int32)]


class SwLayer(C.Structure):
    _fields_ = [("kind", C.c_int32), ("c_out", C.c_int32), ("k", C.c_int32), ("s", C.c_int32),
                ("relu", C.c_int32)]


class SkExtent(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("layout", C.c_int32), ("n", C.c_int64), ("c", C.c_int64), ("plane", C.c_int64)]


class SkView(C.Structure):
    _fields_ = [("data", C.c_void_p), ("stride_n", C.c_int64), ("stride_c", C.c_int64)]


class SkDrop(C.Structure):
    _fields_ = [("p", C.c_double), ("seed", C.c_uint64), ("offset", C.c_uint64), ("step_dev", C.c_void_p)]


class SknetError(RuntimeError):
    def __init__(self, status, message):
        self.status = status
        self.status_name = STATUS_NAMES[status] if 0 <= status < len(STATUS_NAMES) else str(status)
        super().__init__("%s: %s" % (self.status_name, message))


_vp, _i32, _fp, _ip = C.c_void_p, C.c_int32, C.POINTER(C.c_float), C.POINTER(C.c_int32)
_SIGS = {
    "sknet_convert_sw": [C.POINTER(SwLayer), _i32, _i32, C.POINTER(SkLayer), _ip],
    "sknet_create": [C.POINTER(SkLayer), _i32, _i32, _i32, _i32, _i32, C.POINTER(_vp)],
    "sknet_context": [_vp, _ip],
    "sknet_infer_shapes": [_vp, _i32, _i32, _i32, _ip],
    "sknet_num_convs": [_vp, _ip],
    "sknet_conv_shape": [_vp, _i32, _ip],
    "sknet_set_weights": [_vp, _i32, _fp, _fp],
    "sknet_get_weights": [_vp, _i32, _fp, _fp],
    "sknet_plan": [_vp, _i32, _i32, _i32, _i32, _i32],
    "sknet_forward": [_vp, _vp, _vp, _vp],
    "sknet_time_backward_step": [_vp, _vp, _i32, _i32, _i32, _vp, _fp],
    "sknet_backward_noalloc": [_vp, _vp, _vp, _vp],
    "sknet_backward": [_vp, _vp, _vp, _vp],
    "sknet_sgd_step": [_vp, C.c_float, C.c_float, C.c_float, _vp],
    "sknet_get_grad": [_vp, _i32, _fp, _fp],
    "sknet_get_activation_grad": [_vp, _i32, _vp, _fp],
    "sknet_get_activation": [_vp, _i32, _fp],
    "sknet_get_pool_argmax": [_vp, _i32, _ip],
    "sknet_num_steps": [_vp, _ip],
    "sknet_step_name": [_vp, _i32, C.c_char_p, _i32],
    "sknet_time_step": [_vp, _i32, _i32, _vp, _fp],
    "unet_create": [_i32, _i32, _i32, _i32, _i32, C.POINTER(_vp)],
    "unet_num_params": [_vp, _ip],
    "unet_param_shape": [_vp, _i32, _ip],
    "unet_set_weights": [_vp, _i32, _fp, _fp],
    "unet_output_size": [_vp, _i32, _i32, _ip, _ip],
    "unet_plan": [_vp, _i32, _i32, _i32],
    "unet_forward": [_vp, _vp, _vp, _vp],
    "unet_get_activation": [_vp, C.c_char_p, _fp, _ip],
    "usknet_create": [_i32, _i32, _i32, _i32, C.POINTER(_vp)],
    "unet_plan_training": [_vp, _i32, _i32, _i32],
    "unet_set_merge_backward": [_vp, _i32],
    "unet_backward": [_vp, _vp, _vp, _vp],
    "unet_get_grad": [_vp, _i32, _fp, _fp],
    "unet_param_kind": [_vp, _i32, _ip],
    "unet_sgd_step": [_vp, C.c_float, C.c_float, C.c_float, _vp],
    "unet_get_weights": [_vp, _i32, _fp, _fp],
    "sknet3d_create": [C.POINTER(SkLayer), _i32, _i32, _i32, C.POINTER(_vp)],
    "sknet3d_create_dtype": [C.POINTER(SkLayer), _i32, _i32, _i32, _i32, C.POINTER(_vp)],
    "sknet3d_context": [_vp, _ip],
    "sknet3d_infer_shapes": [_vp, _i32, _i32, _i32, _ip],
    "sknet3d_num_convs": [_vp, _ip],
    "sknet3d_conv_shape": [_vp, _i32, _ip],
    "sknet3d_set_weights": [_vp, _i32, _fp, _fp],
    "sknet3d_plan": [_vp, _i32, _i32, _i32, _i32],
    "sknet3d_forward": [_vp, _vp, _vp, _vp],
    "sknet3d_get_activation": [_vp, _i32, _fp],
    "sknet3d_backward": [_vp, _vp, _vp, _vp],
    "sknet3d_sgd_step": [_vp, C.c_float, C.c_float, C.c_float, _vp],
    "sknet3d_get_grad": [_vp, _i32, _fp, _fp],
    "sknet3d_get_weights": [_vp, _i32, _fp, _fp],
    "sknet3d_get_pool_argmax": [_vp, _i32, _ip],
    "sknet_num_norms": [_vp, _ip],
    "sknet_norm_size": [_vp, _i32, _ip],
    "sknet_set_norm": [_vp, _i32, _fp, _fp],
    "sknet_get_norm": [_vp, _i32, _fp, _fp],
    "sknet_get_norm_grad": [_vp, _i32, _fp, _fp],
    "sknet_set_dropout": [_vp, C.c_uint64, C.c_uint64],
    "sknet_get_dropout": [_vp, C.POINTER(C.c_uint64), C.POINTER(C.c_uint64)],
    "sknet_dropout": [_vp, _vp, _vp, _vp, _vp],
    "sknet_layer_norm": [_vp, _vp, _vp, _vp, _vp, _vp, C.c_float, _vp, _vp, _vp, _vp, _vp],
    "sknet_layer_norm_workspace": [_vp, C.POINTER(C.c_uint64)],
    "sknet_layer_norm_backward": [_vp] * 13 + [C.c_uint64, _vp],
    "sk_probe_mfma": [_i32, _i32, _i32, _vp, C.POINTER(C.c_double)],
    "sk_probe_copy": [_vp, _vp, C.c_uint64, _i32, _vp, C.POINTER(C.c_double)],
    "sk_probe_conv_path": [_i32] * 8 + [_ip],
    "sk_probe_pairs_path": [_i32] * 8 + [_ip],
}
for _name, _args in _SIGS.items():
    _f = getattr(lib, _name)
    _f.argtypes = _args
    _f.restype = C.c_int
lib.sknet_destroy.argtypes = [_vp]
lib.sknet_destroy.restype = None
lib.unet_destroy.argtypes = [_vp]
lib.unet_destroy.restype = None
lib.sknet3d_destroy.argtypes = [_vp]
lib.sknet3d_destroy.restype = None
lib.sknet_last_error.argtypes = []
lib.sknet_last_error.restype = C.c_char_p
lib.sknet_conv_flops.argtypes = [C.c_int64] * 4
lib.sknet_conv_flops.restype = C.c_int64

EXPORTED = sorted(list(_SIGS) + ["sknet_destroy", "unet_destroy", "sknet3d_destroy", "sknet_last_error", "sknet_conv_flops"])


def _check(status):
    if status != 0:
        raise SknetError(status, lib.sknet_last_error().decode())


def _f32(a):
    a = np.ascontiguousarray(a, dtype=np.float32)
    return a, a.ctypes.data_as(_fp)


def _stream(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return C.c_void_p(stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream))


def _dev_ptr(t, dtype, what):
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == dtype and t.is_contiguous()):
        raise TypeError("%s must be a contiguous CUDA tensor of %s" % (what, dtype))
    return C.c_void_p(t.data_ptr())


def layers_to_c(layers):
    """[{'type': 'conv'|'pool'|'norm'|'dropout', 'f_out', 'k', 'd', 's', 'relu', 'p'}] -> SkLayer array."""
    arr = (SkLayer * len(layers))()
    for i, l in enumerate(layers):
        if l["type"] == "conv":
            arr[i] = SkLayer(SK_CONV, l["f_out"], l["k"], l.get("d", 1), 1, int(l.get("relu", False)))
        elif l["type"] == "pool":
            arr[i] = SkLayer(SK_MAXPOOL, 0, l["k"], l.get("d", 1), l.get("s", 1), 0)
        elif l["type"] == "norm":
            arr[i] = SkLayer(SK_LAYERNORM, 0, 1, 1, 1, int(l.get("relu", False)))
        elif l["type"] == "dropout":
            if not 0.0 <= l["p"] <= 1.0:
                raise ValueError("layer %d: the rate must be in [0, 1]" % i)
            arr[i] = SkLayer(SK_DROPOUT, int(l["p"] * 65536.0 + 0.5), 1, 1, 1, 0)
        else:
            raise ValueError("unknown layer type %r" % (l["type"],))
    return arr


def sk_probe_mfma(dtype, iters=20000, stream=None, varied=False):
    """Sustained TFLOP/s of a bare MFMA issue loop of the shape used for dtype ('f32'|'bf16'|'f16');
    varied=True gives every MFMA operands of its own with hashed bit patterns (real-data switching activity)."""
    out = C.c_double(0.0)
    _check(lib.sk_probe_mfma(DTYPES[dtype], 1 if varied else 0, iters, _stream(stream), C.byref(out)))
    return out.value


def sk_probe_copy(src, dst, reps=10, stream=None):
    """GB/s (read + written) of a streaming copy between two equally sized CUDA tensors."""
    nbytes = src.numel() * src.element_size()
    if not (src.is_cuda and dst.is_cuda and src.is_contiguous() and dst.is_contiguous()
            and dst.numel() * dst.element_size() == nbytes):
        raise TypeError("sk_probe_copy: two contiguous CUDA tensors of the same byte size")
    out = C.c_double(0.0)
    _check(lib.sk_probe_copy(C.c_void_p(src.data_ptr()), C.c_void_p(dst.data_ptr()), nbytes, reps, _stream(stream), C.byref(out)))
    return out.value


def sk_probe_conv_path(k, d, maps_in, maps_out, n, h_out, w_out, data_gradient=False, planes=False, scratch=False):
    """(kernel, tile shape, split, loads) of a 16-bit convolution; host arithmetic, nothing runs."""
    out = (C.c_int32 * 4)()
    flags = (1 if data_gradient else 0) | (2 if planes else 0) | (4 if scratch else 0)
    _check(lib.sk_probe_conv_path(k, d, maps_in, maps_out, n, h_out, w_out, flags, out))
    return tuple(out)


def sk_probe_pairs_path(k, d, maps_in, maps_out, n, h_out, w_out, what=0):
    """Tile of an fp32 layer on pairs of fp16 (what: 0 convolution, 1 data gradient, 2 weight gradient), zeros if it is on the fp32 unit."""
    out = (C.c_int32 * 3)()
    _check(lib.sk_probe_pairs_path(k, d, maps_in, maps_out, n, h_out, w_out, what, out))
    return tuple(out)


def sknet_conv_flops(f_in, f_out, k, w_out):
    return int(lib.sknet_conv_flops(f_in, f_out, k, w_out))


def sknet_convert_sw(sw_layers, w0_sw):
    """Algorithm 1. sw_layers: [{'type': 'conv'|'pool'|'ip'|'other', ...}] -> SK layer dicts."""
    kinds = {"conv": 0, "pool": 1, "ip": 2, "other": 3}
    arr = (SwLayer * len(sw_layers))()
    for i, l in enumerate(sw_layers):
        arr[i] = SwLayer(kinds[l["type"]], l.get("f_out", 0), l.get("k", 1), l.get("s", 1), int(l.get("relu", False)))
    out = (SkLayer * len(sw_layers))()
    n_out = C.c_int32(0)
    _check(lib.sknet_convert_sw(arr, len(sw_layers), w0_sw, out, C.byref(n_out)))
    res = []
    for i in range(n_out.value):
        l = out[i]
        if l.kind == SK_CONV:
            res.append({"type": "conv", "f_out": l.c_out, "k": l.k, "d": l.d, "relu": bool(l.relu)})
        else:
            res.append({"type": "pool", "k": l.k, "d": l.d, "s": l.s})
    return res


# ---- operators on the caller's own tensors ------------------------------------------------------------------------

_OP_TYPES = {torch.float32: SK_F32, torch.bfloat16: SK_BF16, torch.float16: SK_F16}


@functools.lru_cache(maxsize=4096)
def _orders(shape, strides, axis):
    """{(layout, n, c, plane): (stride_n, stride_c)}: every way to see a tensor of these sizes and strides with its channels on
    `axis` as rows or as maps, rows and the largest planes first.  Positions count in the order of the other axes."""
    others = [(shape[a], strides[a]) for a in range(len(shape)) if a != axis]
    c, sc = shape[axis], strides[axis]

    def merged(parts):                             # axes as one: (length, stride), None if their strides do not allow it
        length, stride = 1, 0
        for size, step in reversed(parts):
            if size == 1:
                continue
            if length == 1:
                stride = step
            elif step != stride * length:
                return None
            length *= size
        return length, stride

    if any(size == 0 for size, _ in others):
        return {(SK_ROWS, 0, c, 1): (0, 0)}
    found = {}
    rows = merged(others) if c == 1 or sc == 1 else None
    if rows is not None:
        found[SK_ROWS, rows[0], c, 1] = rows[1], 0
    for cut in range(len(others) + 1):             # the axes from `cut` on are the plane
        outer, inner = merged(others[:cut]), merged(others[cut:])
        if outer is not None and inner is not None and (inner[0] == 1 or inner[1] == 1):
            found.setdefault((SK_MAPS, outer[0], c, inner[0]), (outer[1], sc))
    return found


@functools.lru_cache(maxsize=4096)
def _workspace(dtype, layout, n, c, plane):
    """Bytes of a backward call's workspace: a matter of the extent alone."""
    need = C.c_uint64()
    _check(lib.sknet_layer_norm_workspace(C.byref(SkExtent(dtype, layout, n, c, plane)), C.byref(need)))
    return need.value


class _Operator:
    """One call of an operator: its stream and device, and its tensors as views of one extent."""

    def __init__(self, x, axis, what, stream):
        if not (isinstance(x, torch.Tensor) and x.is_cuda and x.dtype in _OP_TYPES):
            raise TypeError("%s must be a CUDA tensor of float32, bfloat16 or float16" % what)
        if not -x.dim() <= axis < x.dim():
            raise ValueError("%s has no axis %d" % (what, axis))
        self.x, self.what, self.axis, self.device = x, what, axis % x.dim(), x.device
        self.views = {}
        self.scope = None
        elsewhere = self.device.index != torch.cuda.current_device()
        if stream is None and not elsewhere:       # the usual call: a stream object would take 2 us
            self.stream = torch._C._cuda_getCurrentRawStream(self.device.index)
            return
        if stream is None:
            stream = torch.cuda.current_stream(x.device)
        elif not hasattr(stream, "cuda_stream"):
            stream = torch.cuda.ExternalStream(int(stream), device=x.device)
        if stream.device != x.device:
            raise ValueError("the stream is not one of %s" % (x.device,))
        # the call runs, and what it allocates belongs, there
        self.scope = torch.cuda.stream(stream)
        self.stream = stream.cuda_stream

    def __enter__(self):
        if self.scope is not None:
            self.scope.__enter__()
        return self

    def __exit__(self, *exc):
        if self.scope is not None:
            self.scope.__exit__(*exc)

    def output(self):
        """A tensor for a result: x's sizes and order of axes, without its gaps."""
        return torch.empty_like(self.x, memory_format=torch.contiguous_format if self.x.is_contiguous() else torch.preserve_format)

    def place(self, **tensors):
        """Find the order that the tensors have in common; returns the extent, and their views by name (None for None)."""
        x, axis = self.x, self.axis
        choices = _orders(x.shape, x.stride(), axis)
        theirs = {}
        for name, t in tensors.items():
            if t is None or t is x:
                continue
            if not (isinstance(t, torch.Tensor) and t.device == self.device and t.dtype == x.dtype):
                raise TypeError("%s must be a tensor of %s on %s" % (name, x.dtype, self.device))
            if t.shape != x.shape:
                raise ValueError("%s has shape %s instead of %s" % (name, tuple(t.shape), tuple(x.shape)))
            theirs[name] = _orders(t.shape, t.stride(), axis)
        for order in choices:
            if all(order in o for o in theirs.values()):
                break
        else:
            raise ValueError("%s, strides %s, keep the channels of axis %d neither as rows nor as maps in common; make them contiguous" % (
                ", ".join([self.what] + sorted(theirs)), [x.stride()] + [tensors[n].stride() for n in sorted(theirs)], axis))
        layout, n, c, plane = order
        self.order = order
        self.extent = SkExtent(_OP_TYPES[x.dtype], layout, n, c, plane)
        out = [SkView(x.data_ptr(), *choices[order])]
        for name, t in tensors.items():
            out.append(None if t is None else out[0] if t is x else SkView(t.data_ptr(), *theirs[name][order]))
        self.held = out
        return [None if v is None else C.byref(v) for v in out]

    def values(self, t, count, name):
        """DEVICE pointer of `count` fp32 values, None for None."""
        if t is None:
            return None
        if not (isinstance(t, torch.Tensor) and t.device == self.device and t.dtype == torch.float32 and t.is_contiguous()):
            raise TypeError("%s must be a contiguous tensor of torch.float32 on %s" % (name, self.device))
        if t.numel() != count:
            raise ValueError("%s has %d values instead of %d" % (name, t.numel(), count))
        return t.data_ptr()

    def drop(self, p, seed, offset, step):
        if step is not None and not (isinstance(step, torch.Tensor) and step.device == self.device and step.dtype == torch.int64 and step.numel() == 1):
            raise TypeError("step must be one value of torch.int64 on %s" % (self.device,))
        if not (0 <= seed < 1 << 64 and 0 <= offset < 1 << 64):
            raise ValueError("seed and offset are unsigned 64-bit numbers")
        return C.byref(SkDrop(p, seed, offset, None if step is None else step.data_ptr()))


def dropout(x, p, seed, offset=0, axis=-1, out=None, step=None, stream=None):
    """x with the elements of the mask (seed, offset + step, p) zeroed and the others scaled; the gradient of x is the same call on
    the gradient of the result.  axis: the channels'; the mask belongs to the (position, channel) of an element, whatever the strides.  step:
    optional tensor of one int64, read when the call runs (a recorded graph can advance it)."""
    with _Operator(x, axis, "x", stream) as op:
        if out is None:
            out = op.output()
        xv, yv = op.place(out=out)
        _check(lib.sknet_dropout(C.byref(op.extent), xv, yv, op.drop(p, seed, offset, step), op.stream))
    return out


def layer_norm(x, gamma=None, beta=None, eps=1e-5, axis=-1, residual=None, p=0.0, seed=0, offset=0, step=None, out=None, sum_out=None, mean=None,
               rstd=None, stream=None):
    """(y, s, mean, rstd): y = (s - mean) * rstd * gamma + beta with the mean and 1 / sqrt(variance + eps) of s = residual +
    dropout(x) over the channels on `axis`.  s is x itself where nothing is added or dropped (p = 0); mean and rstd have x's axes without
    the channels'.  out, sum_out, mean, rstd: tensors to write to."""
    with _Operator(x, axis, "x", stream) as op:
        plain = residual is None and p == 0.0 and sum_out is None
        if out is None:
            out = op.output()
        if sum_out is None and not plain:
            sum_out = op.output()
        if mean is None or rstd is None:
            shape = x.shape[:op.axis] + x.shape[op.axis + 1:]
            mean = torch.empty(shape, dtype=torch.float32, device=x.device) if mean is None else mean
            rstd = torch.empty(shape, dtype=torch.float32, device=x.device) if rstd is None else rstd
        xv, rv, sv, yv = op.place(residual=residual, sum_out=sum_out, out=out)
        _, n, c, plane = op.order
        drop = None if p == 0.0 else op.drop(p, seed, offset, step)
        _check(lib.sknet_layer_norm(C.byref(op.extent), xv, rv, drop, op.values(gamma, c, "gamma"), op.values(beta, c, "beta"), eps, sv, yv,
                                    op.values(mean, n * plane, "mean"), op.values(rstd, n * plane, "rstd"), op.stream))
    return out, x if plain else sum_out, mean, rstd


def layer_norm_backward(dy, s, mean, rstd, gamma=None, axis=-1, dsum=None, p=0.0, seed=0, offset=0, step=None, residual=True, parameters=True,
                        dx=None, dresidual=None, dgamma=None, dbeta=None, stream=None):
    """(dx, dresidual, dgamma, dbeta) of layer_norm's y, with the s, mean, rstd it returned and its p, seed, offset and step.  dsum: the gradient that
    reaches s from elsewhere.  dresidual is the gradient of s, and dx dropout of it: one tensor if p = 0 (then leave
    dresidual out).  residual=False: no dresidual (None) where p > 0; parameters=False: no dgamma and dbeta (None)."""
    with _Operator(dy, axis, "dy", stream) as op:
        if dx is None:
            dx = op.output()
        if p == 0.0:
            if dresidual is not None and dresidual is not dx:
                raise ValueError("without dropout dx is the gradient of the residual too; leave dresidual out")
            dresidual = None
        elif dresidual is None and residual:
            dresidual = op.output()
        dyv, sv, dsv, dxv, drv = op.place(s=s, dsum=dsum, dx=dx, dresidual=dresidual)
        _, n, c, plane = op.order
        workspace, bytes_ = None, 0
        if parameters:
            dgamma = torch.empty(c, dtype=torch.float32, device=dy.device) if dgamma is None else dgamma
            dbeta = torch.empty(c, dtype=torch.float32, device=dy.device) if dbeta is None else dbeta
            bytes_ = _workspace(op.extent.dtype, *op.order)
            if bytes_:
                workspace = torch.empty(bytes_, dtype=torch.uint8, device=dy.device)
        elif dgamma is not None or dbeta is not None:
            raise ValueError("parameters=False leaves no gradients to write")
        drop = None if p == 0.0 else op.drop(p, seed, offset, step)
        _check(lib.sknet_layer_norm_backward(C.byref(op.extent), dyv, sv, op.values(mean, n * plane, "mean"), op.values(rstd, n * plane, "rstd"),
                                             op.values(gamma, c, "gamma"), dsv, drop, dxv, drv, op.values(dgamma, c, "dgamma"),
                                             op.values(dbeta, c, "dbeta"), None if workspace is None else workspace.data_ptr(), bytes_, op.stream))
    return dx, dx if p == 0.0 else dresidual, dgamma, dbeta


class SKNet:
    """Owner of one sknet_t handle; methods are the C entry points without the `sknet_` prefix."""

    def __init__(self, layers, c_in, n_classes, dtype="f32", pad_mode=0):
        self.layers = list(layers)
        self._h = _vp()
        arr = layers_to_c(layers)
        _check(lib.sknet_create(arr, len(layers), c_in, n_classes, DTYPES[dtype], pad_mode, C.byref(self._h)))
        self.c_in, self.n_classes = c_in, n_classes
        self._plan = None

    def close(self):
        if self._h:
            lib.sknet_destroy(self._h)
            self._h = _vp()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def context(self):
        v = C.c_int32()
        _check(lib.sknet_context(self._h, C.byref(v)))
        return v.value

    def infer_shapes(self, h, w, pad=True):
        out = (C.c_int32 * (3 * (len(self.layers) + 1)))()
        _check(lib.sknet_infer_shapes(self._h, h, w, int(pad), out))
        return [tuple(out[3 * i:3 * i + 3]) for i in range(len(self.layers) + 1)]

    def num_convs(self):
        c = C.c_int32()
        _check(lib.sknet_num_convs(self._h, C.byref(c)))
        return c.value

    def conv_shape(self, conv_idx):
        s = (C.c_int32 * 4)()
        _check(lib.sknet_conv_shape(self._h, conv_idx, s))
        return tuple(s)

    def set_weights(self, conv_idx, w, b=None):
        shape = self.conv_shape(conv_idx)
        w, wp = _f32(w)
        if w.shape != shape:
            raise ValueError("conv %d expects weights %s, got %s" % (conv_idx, shape, w.shape))
        if b is not None:
            b, bp = _f32(b)
            if b.shape != (shape[0],):
                raise ValueError("conv %d expects %d biases" % (conv_idx, shape[0]))
        else:
            bp = None
        _check(lib.sknet_set_weights(self._h, conv_idx, wp, bp))

    def get_weights(self, conv_idx):
        shape = self.conv_shape(conv_idx)
        w = np.empty(shape, np.float32)
        b = np.empty(shape[0], np.float32)
        _check(lib.sknet_get_weights(self._h, conv_idx, w.ctypes.data_as(_fp), b.ctypes.data_as(_fp)))
        return w, b

    def num_norms(self):
        c = C.c_int32()
        _check(lib.sknet_num_norms(self._h, C.byref(c)))
        return c.value

    def norm_size(self, norm_idx):
        c = C.c_int32()
        _check(lib.sknet_norm_size(self._h, norm_idx, C.byref(c)))
        return c.value

    def set_norm(self, norm_idx, gamma=None, beta=None):
        size = self.norm_size(norm_idx)
        ptrs = []
        for name, v in (("gammas", gamma), ("betas", beta)):
            v, p = (None, None) if v is None else _f32(v)
            if v is not None and v.shape != (size,):
                raise ValueError("norm %d expects %d %s" % (norm_idx, size, name))
            ptrs.append((v, p))
        _check(lib.sknet_set_norm(self._h, norm_idx, ptrs[0][1], ptrs[1][1]))

    def _norm_pair(self, fn, norm_idx):
        gamma, beta = (np.empty(self.norm_size(norm_idx), np.float32) for _ in range(2))
        _check(fn(self._h, norm_idx, gamma.ctypes.data_as(_fp), beta.ctypes.data_as(_fp)))
        return gamma, beta

    def get_norm(self, norm_idx):
        return self._norm_pair(lib.sknet_get_norm, norm_idx)

    def get_norm_grad(self, norm_idx):
        return self._norm_pair(lib.sknet_get_norm_grad, norm_idx)

    def set_dropout(self, seed, step=0):
        if not 0 <= seed < 1 << 64 or step < 0:
            raise ValueError("seed and step are unsigned")
        _check(lib.sknet_set_dropout(self._h, seed, step))

    def get_dropout(self):
        """(seed, step): with them a later run continues the masks of this one."""
        seed, step = C.c_uint64(), C.c_uint64()
        _check(lib.sknet_get_dropout(self._h, C.byref(seed), C.byref(step)))
        return seed.value, step.value

    def plan(self, n, h, w, pad=True, training=False, keep=False, fused_head=False):
        """mode 1 if training (3 with fused_head: the head and the loss as one kernel in each direction),
        else 2 if keep (inference, every layer kept), else 0 (inference, fused)."""
        mode = (3 if fused_head else 1) if training else (2 if keep else 0)
        _check(lib.sknet_plan(self._h, n, h, w, int(pad), mode))
        self._plan = (n, h, w, bool(pad), bool(training))
        self._shapes = self.infer_shapes(h, w, pad)

    def out_shape(self):
        n = self._plan[0]
        c, h, w = self._shapes[-1]
        return (n, c, h, w)

    def forward(self, image, prob=None, stream=None):
        n, h, w = self._plan[:3]
        if tuple(image.shape) != (n, self.c_in, h, w):
            raise ValueError("image shape %s does not match the plan %s" % (tuple(image.shape), (n, self.c_in, h, w)))
        if prob is None:
            prob = torch.empty(self.out_shape(), dtype=torch.float32, device=image.device)
        elif tuple(prob.shape) != self.out_shape():
            raise ValueError("prob shape %s does not match %s" % (tuple(prob.shape), self.out_shape()))
        _check(lib.sknet_forward(self._h, _dev_ptr(image, torch.float32, "image"),
                                 _dev_ptr(prob, torch.float32, "prob"), _stream(stream)))
        return prob

    def backward(self, labels, loss=None, stream=None, noalloc=False):
        """noalloc=True: sknet_backward_noalloc (scratch in the library's static device buffer); loss must then
        be given, so that nothing is allocated on the way."""
        n, _, h, w = self.out_shape()
        if tuple(labels.shape) != (n, h, w):
            raise ValueError("labels shape %s does not match %s" % (tuple(labels.shape), (n, h, w)))
        if loss is None:
            if noalloc:
                raise ValueError("noalloc needs a caller-provided loss tensor")
            loss = torch.empty(1, dtype=torch.float32, device=labels.device)
        fn = lib.sknet_backward_noalloc if noalloc else lib.sknet_backward
        _check(fn(self._h, _dev_ptr(labels, torch.int32, "labels"), _dev_ptr(loss, torch.float32, "loss"), _stream(stream)))
        return loss

    def sgd_step(self, lr, momentum=0.0, weight_decay=0.0, stream=None):
        _check(lib.sknet_sgd_step(self._h, lr, momentum, weight_decay, _stream(stream)))

    def get_grad(self, conv_idx):
        shape = self.conv_shape(conv_idx)
        dw = np.empty(shape, np.float32)
        db = np.empty(shape[0], np.float32)
        _check(lib.sknet_get_grad(self._h, conv_idx, dw.ctypes.data_as(_fp), db.ctypes.data_as(_fp)))
        return dw, db

    def get_activation(self, layer_idx):
        c, h, w = self._shapes[layer_idx + 1]
        out = np.empty((self._plan[0], c, h, w), np.float32)
        _check(lib.sknet_get_activation(self._h, layer_idx, out.ctypes.data_as(_fp)))
        return out

    def get_activation_grad(self, layer_idx, labels):
        """Error map of layer layer_idx (fp32 NCHW numpy), recomputed from the last forward with labels."""
        c, h, w = self._shapes[layer_idx + 1]
        out = np.empty((self._plan[0], c, h, w), np.float32)
        _check(lib.sknet_get_activation_grad(self._h, layer_idx, _dev_ptr(labels, torch.int32, "labels"), out.ctypes.data_as(_fp)))
        return out

    def get_pool_argmax(self, pool_idx):
        li = [i for i, l in enumerate(self.layers) if l["type"] == "pool"][pool_idx]
        c, h, w = self._shapes[li + 1]
        out = np.empty((self._plan[0], c, h, w), np.int32)
        _check(lib.sknet_get_pool_argmax(self._h, pool_idx, out.ctypes.data_as(_ip)))
        return out

    def num_steps(self):
        c = C.c_int32()
        _check(lib.sknet_num_steps(self._h, C.byref(c)))
        return c.value

    def step_name(self, step):
        buf = C.create_string_buffer(64)
        _check(lib.sknet_step_name(self._h, step, buf, 64))
        return buf.value.decode()

    def time_backward_step(self, labels, layer_idx, part, iters=10, stream=None):
        """Average ms of one piece of the backward pass: part 0 weight gradient, 1 input gradient, 2 loss."""
        ms = C.c_float()
        _check(lib.sknet_time_backward_step(self._h, _dev_ptr(labels, torch.int32, "labels"), layer_idx, part, iters, _stream(stream), C.byref(ms)))
        return ms.value

    def time_step(self, step, iters=10, stream=None):
        ms = C.c_float()
        _check(lib.sknet_time_step(self._h, step, iters, _stream(stream), C.byref(ms)))
        return ms.value


class UNet:
    """Owner of one unet_t handle."""

    def __init__(self, c_in, n_classes, depth=4, base_ch=64, dtype="f32"):
        self._h = _vp()
        self._create(c_in, n_classes, depth, base_ch, dtype)
        self.c_in, self.n_classes, self.depth = c_in, n_classes, depth
        self._plan = None

    def _create(self, c_in, n_classes, depth, base_ch, dtype):
        _check(lib.unet_create(c_in, n_classes, depth, base_ch, DTYPES[dtype], C.byref(self._h)))

    def close(self):
        if self._h:
            lib.unet_destroy(self._h)
            self._h = _vp()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def num_params(self):
        c = C.c_int32()
        _check(lib.unet_num_params(self._h, C.byref(c)))
        return c.value

    def param_shape(self, idx):
        s = (C.c_int32 * 4)()
        _check(lib.unet_param_shape(self._h, idx, s))
        return tuple(s)

    def set_weights(self, idx, w, b=None):
        shape = self.param_shape(idx)
        w, wp = _f32(w)
        if w.shape != shape:
            raise ValueError("parameter %d expects %s, got %s" % (idx, shape, w.shape))
        bp = None
        if b is not None:
            b, bp = _f32(b)
        _check(lib.unet_set_weights(self._h, idx, wp, bp))

    def output_size(self, h_in, w_in):
        ho, wo = C.c_int32(), C.c_int32()
        _check(lib.unet_output_size(self._h, h_in, w_in, C.byref(ho), C.byref(wo)))
        return ho.value, wo.value

    def plan(self, n, h_in, w_in, training=False):
        _check((lib.unet_plan_training if training else lib.unet_plan)(self._h, n, h_in, w_in))
        self._plan = (n, h_in, w_in)

    def set_merge_backward(self, mode):
        """0: MergeCrop backwards into the up path only (default); 1: into the skip map as well."""
        _check(lib.unet_set_merge_backward(self._h, int(mode)))

    def backward(self, labels, loss=None, stream=None):
        """labels: int32 CUDA tensor [n, h_out, w_out] (-1 = masked pixel); returns the loss (1-element CUDA tensor)."""
        n, h, w = self._plan
        ho, wo = self.output_size(h, w)
        if tuple(labels.shape) != (n, ho, wo):
            raise ValueError("labels shape %s does not match the plan" % (tuple(labels.shape),))
        if loss is None:
            loss = torch.zeros(1, dtype=torch.float32, device=labels.device)
        _check(lib.unet_backward(self._h, _dev_ptr(labels, torch.int32, "labels"), _dev_ptr(loss, torch.float32, "loss"), _stream(stream)))
        return loss

    def sgd_step(self, lr, momentum=0.0, weight_decay=0.0, stream=None):
        _check(lib.unet_sgd_step(self._h, lr, momentum, weight_decay, _stream(stream)))

    def get_weights(self, idx):
        shape = self.param_shape(idx)
        kind = C.c_int32()
        _check(lib.unet_param_kind(self._h, idx, C.byref(kind)))
        w = np.empty(shape, np.float32)
        b = np.empty((shape[1] if kind.value == 1 else shape[0],), np.float32)
        _check(lib.unet_get_weights(self._h, idx, w.ctypes.data_as(_fp), b.ctypes.data_as(_fp)))
        return w, b

    def get_grad(self, idx):
        shape = self.param_shape(idx)
        kind = C.c_int32()
        _check(lib.unet_param_kind(self._h, idx, C.byref(kind)))
        dw = np.empty(shape, np.float32)
        db = np.empty((shape[1] if kind.value == 1 else shape[0],), np.float32)
        _check(lib.unet_get_grad(self._h, idx, dw.ctypes.data_as(_fp), db.ctypes.data_as(_fp)))
        return dw, db

    def forward(self, image, prob=None, stream=None):
        n, h, w = self._plan
        if tuple(image.shape) != (n, self.c_in, h, w):
            raise ValueError("image shape %s does not match the plan" % (tuple(image.shape),))
        ho, wo = self.output_size(h, w)
        if prob is None:
            prob = torch.empty((n, self.n_classes, ho, wo), dtype=torch.float32, device=image.device)
        _check(lib.unet_forward(self._h, _dev_ptr(image, torch.float32, "image"),
                                _dev_ptr(prob, torch.float32, "prob"), _stream(stream)))
        return prob

    def get_activation(self, stage):
        dims = (C.c_int32 * 3)()
        _check(lib.unet_get_activation(self._h, stage.encode(), None, dims))
        out = np.empty((self._plan[0], dims[0], dims[1], dims[2]), np.float32)
        _check(lib.unet_get_activation(self._h, stage.encode(), out.ctypes.data_as(_fp), dims))
        return out


class USKNet(UNet):
    """USK-Net (usknet_create): the same handle type and calls as UNet."""

    def __init__(self, c_in, n_classes, base_ch=64, dtype="f32"):
        super().__init__(c_in, n_classes, 1, base_ch, dtype)

    def _create(self, c_in, n_classes, depth, base_ch, dtype):
        _check(lib.usknet_create(c_in, n_classes, base_ch, DTYPES[dtype], C.byref(self._h)))


class SKNet3D:
    """Owner of one sknet3d_t handle; methods are the C entry points without the `sknet3d_` prefix.
    Volumes are slice-major: [depth][maps][height][width]."""

    def __init__(self, layers, c_in, n_classes, dtype="f32"):
        self.layers = list(layers)
        self._h = _vp()
        _check(lib.sknet3d_create_dtype(layers_to_c(layers), len(layers), c_in, n_classes, DTYPES[dtype], C.byref(self._h)))
        self.c_in, self.n_classes = c_in, n_classes
        self._plan = None

    def close(self):
        if self._h:
            lib.sknet3d_destroy(self._h)
            self._h = _vp()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def context(self):
        v = C.c_int32()
        _check(lib.sknet3d_context(self._h, C.byref(v)))
        return v.value

    def infer_shapes(self, dz, h, w):
        """[(maps, depth, height, width)] for the input volume and every layer's output."""
        out = (C.c_int32 * (4 * (len(self.layers) + 1)))()
        _check(lib.sknet3d_infer_shapes(self._h, dz, h, w, out))
        return [tuple(out[4 * i:4 * i + 4]) for i in range(len(self.layers) + 1)]

    def num_convs(self):
        c = C.c_int32()
        _check(lib.sknet3d_num_convs(self._h, C.byref(c)))
        return c.value

    def conv_shape(self, conv_idx):
        s = (C.c_int32 * 5)()
        _check(lib.sknet3d_conv_shape(self._h, conv_idx, s))
        return tuple(s)

    def set_weights(self, conv_idx, w, b=None):
        shape = self.conv_shape(conv_idx)
        w, wp = _f32(w)
        if w.shape != shape:
            raise ValueError("conv %d expects weights %s, got %s" % (conv_idx, shape, w.shape))
        if b is not None:
            b, bp = _f32(b)
            if b.shape != (shape[0],):
                raise ValueError("conv %d expects %d biases" % (conv_idx, shape[0]))
        else:
            bp = None
        _check(lib.sknet3d_set_weights(self._h, conv_idx, wp, bp))

    def plan(self, dz, h, w, keep=False, training=False):
        """mode 1 if training, else 2 if keep (inference, every layer kept), else 0 (inference, fused head)."""
        _check(lib.sknet3d_plan(self._h, dz, h, w, 1 if training else (2 if keep else 0)))
        self._plan = (dz, h, w)
        self._shapes = self.infer_shapes(dz, h, w)

    def out_shape(self):
        """(depth, classes, height, width) of the probabilities."""
        c, dz, h, w = self._shapes[-1]
        return (dz, c, h, w)

    def forward(self, volume, prob=None, stream=None):
        dz, h, w = self._plan
        if tuple(volume.shape) != (dz, self.c_in, h, w):
            raise ValueError("volume shape %s does not match the plan %s" % (tuple(volume.shape), (dz, self.c_in, h, w)))
        if prob is None:
            prob = torch.empty(self.out_shape(), dtype=torch.float32, device=volume.device)
        elif tuple(prob.shape) != self.out_shape():
            raise ValueError("prob shape %s does not match %s" % (tuple(prob.shape), self.out_shape()))
        _check(lib.sknet3d_forward(self._h, _dev_ptr(volume, torch.float32, "volume"),
                                   _dev_ptr(prob, torch.float32, "prob"), _stream(stream)))
        return prob

    def get_activation(self, layer_idx):
        """Output of layer layer_idx as a numpy array [depth, maps, height, width]."""
        c, dz, h, w = self._shapes[layer_idx + 1]
        out = np.empty((dz, c, h, w), np.float32)
        _check(lib.sknet3d_get_activation(self._h, layer_idx, out.ctypes.data_as(_fp)))
        return out

    def backward(self, labels, loss=None, stream=None):
        dz, _, h, w = self.out_shape()
        if tuple(labels.shape) != (dz, h, w):
            raise ValueError("labels shape %s does not match %s" % (tuple(labels.shape), (dz, h, w)))
        if loss is None:
            loss = torch.empty((), dtype=torch.float32, device=labels.device)
        _check(lib.sknet3d_backward(self._h, _dev_ptr(labels, torch.int32, "labels"), _dev_ptr(loss, torch.float32, "loss"),
                                    _stream(stream)))
        return loss

    def sgd_step(self, lr, momentum=0.0, weight_decay=0.0, stream=None):
        _check(lib.sknet3d_sgd_step(self._h, lr, momentum, weight_decay, _stream(stream)))

    def get_grad(self, conv_idx):
        shape = self.conv_shape(conv_idx)
        dw = np.empty(shape, np.float32)
        db = np.empty(shape[0], np.float32)
        _check(lib.sknet3d_get_grad(self._h, conv_idx, dw.ctypes.data_as(_fp), db.ctypes.data_as(_fp)))
        return dw, db

    def get_weights(self, conv_idx):
        shape = self.conv_shape(conv_idx)
        w = np.empty(shape, np.float32)
        b = np.empty(shape[0], np.float32)
        _check(lib.sknet3d_get_weights(self._h, conv_idx, w.ctypes.data_as(_fp), b.ctypes.data_as(_fp)))
        return w, b

    def get_pool_argmax(self, pool_idx):
        """Winner offsets of max pool number pool_idx as int32 [depth, maps, height, width]."""
        pools = [i for i, l in enumerate(self.layers) if l["type"] == "pool"]
        c, dz, h, w = self._shapes[pools[pool_idx] + 1]
        out = np.empty((dz, c, h, w), np.int32)
        _check(lib.sknet3d_get_pool_argmax(self._h, pool_idx, out.ctypes.data_as(_ip)))
        return out
