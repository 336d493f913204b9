"""Binding of libdraco.so: argument marshalling only, by ctypes, and natively (``csrc/native.cpp``) for the calls of a training loop
where that module was built for the running interpreter.

Every function takes raw device pointers (``tensor.data_ptr()``) or torch
tensors and a CUDA stream handle; PyTorch is used by callers for device memory
and streams, never for arithmetic on the path.
"""
from __future__ import annotations

import ctypes as C
import importlib.util
import os
import sysconfig
import warnings

REP, CYC, CYC_PACKED = 0, 1, 2
ADV_REVGRAD, ADV_CONST, ADV_GAUSS = 0, 1, 2
OK, EINVAL, ECUDA, ETOOMANY, ENOMEM, EINTERNAL, ELIMIT, ENOMAJ, EUNSURE = 0, -1, -2, -3, -4, -5, -6, 1, 2
MAX_N = 128
F32, BF16, F16 = 0, 1, 2
NORM_2, NORM_MAX = 0, 1
MAX_TENSORS = 65536

_PKG = os.path.dirname(os.path.abspath(__file__))


class DracoError(RuntimeError):
    pass


class DracoInfo(C.Structure):
    _fields_ = [("status", C.c_int32), ("n_flagged", C.c_int32), ("locator_rank", C.c_int32),
                ("n_active", C.c_int32), ("no_majority", C.c_uint64), ("scale", C.c_double),
                ("max_syndrome", C.c_double), ("internal_error", C.c_int32), ("svd_sweeps", C.c_int32),
                ("locator_margin", C.c_double), ("im_residual", C.c_double), ("re_max", C.c_double)]

    def as_dict(self):
        return {k: getattr(self, k) for k, _ in self._fields_}


def library_path() -> str:
    return os.path.join(_PKG, "libdraco.so")


def _load() -> C.CDLL:
    path = library_path()
    if not os.path.exists(path):
        raise DracoError(f"{path} is missing: build it with `python -m paper_1803_09877_b200.build` "
                         "(there is no CPU fallback)")
    return C.CDLL(path)


lib = _load()

_TYPES = {"torch.float32": F32, "torch.bfloat16": BF16, "torch.float16": F16}

_vp, _i, _i64, _u64, _f = C.c_void_p, C.c_int, C.c_int64, C.c_uint64, C.c_float
_SIGS = {
    "draco_plan_create": ([_i, _i, _i64, _i, C.POINTER(_vp)], _i),
    "draco_plan_destroy": ([_vp], _i),
    "draco_plan_set_theta": ([_vp, C.c_double], _i),
    "draco_num_groups": ([_vp], _i),
    "draco_groups": ([_vp, C.POINTER(_i), C.POINTER(_i)], _i),
    "draco_cyc_W": ([_vp, C.POINTER(C.c_double)], _i),
    "draco_encode": ([_vp, _vp, _vp, _vp], _i),
    "draco_locate": ([_vp, _vp, _vp, _vp, _vp], _i),
    "draco_decode": ([_vp, _vp, _vp, _vp, _vp], _i),
    "draco_locate_decode": ([_vp, _vp, _vp, _vp, _vp, _vp], _i),
    "draco_decode_update": ([_vp, _vp, _vp, _vp, _f, _vp], _i),
    "draco_rep_vote": ([_vp, _vp, _vp, _vp, _vp, _vp], _i),
    "draco_cyc_project": ([_vp, _vp, _vp, _vp, _vp], _i),
    "draco_cyc_locate_from_projection": ([_vp, _vp, _vp, _vp], _i),
    "draco_cyc_project_noalloc": ([_i, _i64, _vp, _vp, _vp, _vp], _i),
    "draco_cyc_decode_vector": ([_vp, C.POINTER(C.c_double), _vp], _i),
    "draco_cyc_reads": ([_vp, C.POINTER(_i), _vp], _i),
    "draco_get_info": ([_vp, C.POINTER(DracoInfo), _vp], _i),
    "draco_pipeline_host": ([_vp, _vp, _vp, C.POINTER(_i), C.POINTER(_i), C.POINTER(_f), _i, _u64, _vp, _vp, _vp,
                             C.POINTER(DracoInfo)], _i),
    "draco_generate": ([_vp, _i, _i64, _i, _f, _f, _u64, _vp], _i),
    "draco_corrupt": ([_vp, _vp, C.POINTER(_i), C.POINTER(_i), C.POINTER(_f), _i, _u64, _vp], _i),
    "draco_layout_create": ([_i, C.POINTER(_i64), C.POINTER(_i), C.POINTER(_vp)], _i),
    "draco_layout_destroy": ([_vp], _i),
    "draco_layout_size": ([_vp], _i64),
    "draco_norm": ([_vp, C.POINTER(_vp), _i, _vp, _vp, _vp], _i),
    "draco_clip": ([_vp, C.POINTER(_vp), C.POINTER(_vp), _i, _f, _i, _vp, _vp, _vp], _i),
    "draco_pack": ([_vp, C.POINTER(_vp), _i, _f, _vp, _vp, _vp], _i),
    "draco_update": ([_vp, C.POINTER(_vp), _vp, _vp, _i, _f, _f, _vp, _vp], _i),
    "draco_strerror": ([_i], C.c_char_p),
    "draco_last_cuda_error": ([], C.c_char_p),
}
for _name, (_args, _res) in _SIGS.items():
    _fn = getattr(lib, _name)
    _fn.argtypes = _args
    _fn.restype = _res

EXPORTS = tuple(_SIGS)


def _check(rc: int) -> int:
    if rc < 0:
        msg = lib.draco_strerror(rc).decode()
        if rc == ECUDA:
            msg += ": " + lib.draco_last_cuda_error().decode()
        raise DracoError(f"libdraco: {msg} ({rc})")
    return rc


def _ptr(x):
    """Device / host address of a torch tensor, an int address, or None."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return x.data_ptr()


def _find_current_stream():
    """torch.cuda.current_stream().cuda_stream, without the Stream object that it builds on every call where torch offers the
    handle itself: 0.2 us instead of 3.3 us of the 8.1 us that a call of this module took (a launch is 3.9 us of it)."""
    global _current_stream
    import torch
    first = torch.cuda.current_stream().cuda_stream        # also sets CUDA up
    raw, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
    if raw and device:
        _native.set_current_stream(raw, device)
        _current_stream = lambda: raw(device())
    else:
        _current_stream = lambda: torch.cuda.current_stream().cuda_stream
    return first


_current_stream = _find_current_stream


def _stream(stream):
    if stream is None:
        return _current_stream()
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _wrote(*written):
    """Tells autograd of tensors and lists of tensors that a call has written, so that a graph which had saved one of them says so instead of
    taking its new values."""
    import torch
    tell = torch.autograd.graph.increment_version
    tensors = [t for x in written for t in (x if isinstance(x, (list, tuple)) else (x,)) if isinstance(t, torch.Tensor)]
    try:
        tell(tensors)
    except (TypeError, RuntimeError):   # a torch that takes one at a time
        for t in tensors:
            tell(t)


class _CtypesCalls:
    """The calls of csrc/native.cpp through ctypes."""

    @staticmethod
    def encode(plan, G, Z, stream):
        return _check(lib.draco_encode(plan, _ptr(G), _ptr(Z), _stream(stream)))

    @staticmethod
    def locate(plan, R, f, flags, stream):
        return _check(lib.draco_locate(plan, _ptr(R), _ptr(f), _ptr(flags), _stream(stream)))

    @staticmethod
    def decode(plan, R, flags, u, stream):
        return _check(lib.draco_decode(plan, _ptr(R), _ptr(flags), _ptr(u), _stream(stream)))

    @staticmethod
    def decode_update(plan, R, flags, w, scale, stream):
        return _check(lib.draco_decode_update(plan, _ptr(R), _ptr(flags), _ptr(w), scale, _stream(stream)))

    @staticmethod
    def locate_decode(plan, R, f, flags, u, stream):
        return _check(lib.draco_locate_decode(plan, _ptr(R), _ptr(f), _ptr(flags), _ptr(u), _stream(stream)))

    @staticmethod
    def norm(*_):                       # binding.py itself lists the addresses then
        return NotImplemented

    clip = pack = update = norm

    @staticmethod
    def set_current_stream(raw, device):
        pass

    @staticmethod
    def set_exchange(tensor, parameter, capsule):
        pass


def _load_module(name, path):
    spec = importlib.util.spec_from_file_location(f"{__package__}.{name}", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _load_native():
    """The module that was built for this interpreter, by its full name; without it ctypes makes the same calls."""
    path = os.path.join(_PKG, "_native" + sysconfig.get_config_var("EXT_SUFFIX"))
    if not os.path.exists(path):
        return _CtypesCalls
    try:
        module = _load_module("_native", path)
    except ImportError as e:
        warnings.warn(f"{path} cannot be loaded ({e}): ctypes makes its calls", RuntimeWarning)
        return _CtypesCalls
    module.set_functions(_check, _stream, _wrote)
    return module


_native = _load_native()


def _adv_arrays(adv_idx, adv_model, adv_param):
    k = len(adv_idx)
    return ((_i * k)(*[int(a) for a in adv_idx]), (_i * k)(*[int(a) for a in adv_model]),
            (_f * k)(*[float(a) for a in adv_param]), k)


def cyc_project_noalloc(n: int, d: int, R, f, e, stream=None):
    """draco_cyc_project_noalloc: e = f R with the library's built-in scratch; needs no plan and allocates nothing."""
    return _check(lib.draco_cyc_project_noalloc(n, d, _ptr(R), _ptr(f), _ptr(e), _stream(stream)))


def generate(out, rows: int, length: int, row0: int = 0, mean: float = 0.0, std: float = 1.0, seed: int = 0,
             stream=None):
    """draco_generate: fill device [rows][length] fp32 with the seeded generator."""
    _check(lib.draco_generate(_ptr(out), rows, length, row0, mean, std, seed & 0xFFFFFFFFFFFFFFFF, _stream(stream)))


class Plan:
    """draco_plan: tables and scratch for one (n, s, d, code) on the current device."""

    def __init__(self, n: int, s: int, d: int, code: int):
        self.n, self.s, self.d, self.code = n, s, d, code
        h = _vp()
        _check(lib.draco_plan_create(n, s, d, code, C.byref(h)))
        self._h = h
        self._address = h.value

    def close(self):
        if getattr(self, "_h", None):
            lib.draco_plan_destroy(self._h)
            self._h = None
            self._address = None

    __del__ = close

    def set_theta(self, theta: float):
        _check(lib.draco_plan_set_theta(self._h, theta))

    def groups(self):
        g = _check(lib.draco_num_groups(self._h))
        first, size = (_i * max(g, 1))(), (_i * max(g, 1))()
        if g:
            _check(lib.draco_groups(self._h, first, size))
        return [(first[k], size[k]) for k in range(g)]

    def cyc_W(self):
        import numpy as np
        buf = (C.c_double * (2 * self.n * self.n))()
        _check(lib.draco_cyc_W(self._h, buf))
        a = np.frombuffer(buf, dtype=np.float64).reshape(self.n, self.n, 2)
        return a[..., 0] + 1j * a[..., 1]

    def encode(self, G, Z, stream=None):
        return _native.encode(self._address, G, Z, stream)

    def locate(self, R, f, flags, stream=None):
        return _native.locate(self._address, R, f, flags, stream)

    def decode(self, R, flags, u, stream=None):
        return _native.decode(self._address, R, flags, u, stream)

    def decode_update(self, R, flags, w, scale: float, stream=None):
        return _native.decode_update(self._address, R, flags, w, scale, stream)

    def locate_decode(self, R, f, flags, u, stream=None):
        return _native.locate_decode(self._address, R, f, flags, u, stream)

    def rep_vote(self, R, u=None, maj=None, flags=None, stream=None):
        return _check(lib.draco_rep_vote(self._h, _ptr(R), _ptr(u), _ptr(maj), _ptr(flags), _stream(stream)))

    def cyc_project(self, R, f, e, stream=None):
        return _check(lib.draco_cyc_project(self._h, _ptr(R), _ptr(f), _ptr(e), _stream(stream)))

    def cyc_locate_from_projection(self, e, flags, stream=None):
        return _check(lib.draco_cyc_locate_from_projection(self._h, _ptr(e), _ptr(flags), _stream(stream)))

    def cyc_decode_vector(self, stream=None):
        import numpy as np
        buf = (C.c_double * (2 * self.n))()
        _check(lib.draco_cyc_decode_vector(self._h, buf, _stream(stream)))
        a = np.frombuffer(buf, dtype=np.float64).reshape(self.n, 2)
        return a[:, 0] + 1j * a[:, 1]

    def cyc_reads(self, stream=None) -> int:
        reads = _i()
        _check(lib.draco_cyc_reads(self._h, C.byref(reads), _stream(stream)))
        return reads.value

    def info(self, stream=None) -> dict:
        out = DracoInfo()
        _check(lib.draco_get_info(self._h, C.byref(out), _stream(stream)))
        return out.as_dict()

    def corrupt(self, R, adv_idx, adv_model, adv_param, seed: int = 0, stream=None):
        idx, model, param, k = _adv_arrays(adv_idx, adv_model, adv_param)
        return _check(lib.draco_corrupt(self._h, _ptr(R), idx, model, param, k, seed & 0xFFFFFFFFFFFFFFFF,
                                        _stream(stream)))

    def pipeline_host(self, G_host, f_host, adv_idx, adv_model, adv_param, adv_seed, Z, u_host, flags_host) -> dict:
        idx, model, param, k = _adv_arrays(adv_idx, adv_model, adv_param)
        out = DracoInfo()
        _check(lib.draco_pipeline_host(self._h, _ptr(G_host), _ptr(f_host), idx, model, param, k,
                                       adv_seed & 0xFFFFFFFFFFFFFFFF, _ptr(Z), _ptr(u_host), _ptr(flags_host),
                                       C.byref(out)))
        return out.as_dict()


class _Meta(C.Structure):
    """What the native calls compare a list of tensors with."""
    _fields_ = [("count", _i64), ("d", _i64), ("numels", C.POINTER(_i64)), ("types", C.POINTER(C.c_int32)), ("device", C.c_int32)]


_exchange_known = False


def _exchange(torch):
    """What tells the native calls of a tensor: the module that was built for this torch, or else torch's own table of DLPack functions, or None."""
    path = os.path.join(_PKG, f"_torch_tensors-{torch.__version__}" + sysconfig.get_config_var("EXT_SUFFIX"))
    if os.path.exists(path):
        try:
            return _load_module("_torch_tensors", path).exchange
        except ImportError as e:
            warnings.warn(f"{path} cannot be loaded ({e}): torch's own function takes its place", RuntimeWarning)
    return getattr(torch.Tensor, "__dlpack_c_exchange_api__", None)


def _find_exchange(torch):
    global _exchange_known
    if not _exchange_known:
        _exchange_known = True
        capsule = _exchange(torch)
        if capsule is not None:
            _native.set_exchange(torch.Tensor, torch.nn.Parameter, capsule)


def _order(t) -> list:
    """Sizes and strides, those of sizes of one apart, which say nothing."""
    return [(n, st if n != 1 else 0) for n, st in zip(t.shape, t.stride())]


def _dense(t) -> bool:
    """Whether the tensor's elements fill one piece of memory, in whatever order."""
    if t.is_contiguous():
        return True
    run = 1
    for stride, size in sorted((st, n) for st, n in zip(t.stride(), t.shape) if n != 1):
        if stride != run:
            return False
        run *= size
    return True


class Layout:
    """draco_layout: sizes and types of a list of tensors, on the current device.

    ``numels``: the numbers of elements.  ``types``: F32, BF16, F16 or torch's dtypes, one for each tensor or one for all.  The calls
    take the list itself (any iterable, ``model.parameters()`` too): tensors of these sizes and types on the layout's device, None for
    one that is absent, or raw addresses.
    ``norm`` and ``clip`` take tensors that are dense in any order of their dimensions, and add up in the order of their memory; ``pack`` and ``update``,
    whose flat vectors follow the order of the elements, take contiguous ones.  A layout has to live as long as a graph that has captured a call on it.

    To autograd the calls are writes in place under ``torch.no_grad()``: nothing is recorded, and a graph that had saved a tensor which a call has
    since written refuses its backward pass (raw addresses and the calls of Plan are not told of).
    """

    def __init__(self, numels, types):
        import torch
        self.numels = [int(n) for n in numels]
        one = isinstance(types, int) or str(types) in _TYPES
        self.types = [self._type(t) for t in ([types] * len(self.numels) if one else types)]
        if len(self.types) != len(self.numels):
            raise DracoError(f"{len(self.numels)} sizes, {len(self.types)} types")
        count = len(self.numels)
        h = _vp()
        _check(lib.draco_layout_create(count, (_i64 * count)(*self.numels), (_i * count)(*self.types), C.byref(h)))
        self._h = h
        self._address = h.value
        self.device = torch.cuda.current_device()
        self.d = lib.draco_layout_size(h)
        self._meta = _Meta(count, self.d, (_i64 * count)(*self.numels), (C.c_int32 * count)(*self.types), self.device)
        self._meta_address = C.addressof(self._meta)
        _find_exchange(torch)

    @classmethod
    def of(cls, tensors):
        """The layout of these tensors, on their device (which has to be the current one for the calls); of tensors elsewhere, on the current device."""
        import contextlib

        import torch
        tensors = list(tensors)
        devices = {t.get_device() for t in tensors if t.is_cuda}
        if len(devices) > 1:
            raise DracoError(f"tensors are on several devices: cuda:{', cuda:'.join(map(str, sorted(devices)))}")
        with torch.cuda.device(devices.pop()) if devices else contextlib.nullcontext():
            return cls([t.numel() for t in tensors], [t.dtype for t in tensors])

    @staticmethod
    def _type(t):
        if isinstance(t, int):
            return t
        if str(t) not in _TYPES:
            raise DracoError(f"{t}: tensors are float32, bfloat16 or float16")
        return _TYPES[str(t)]

    def close(self):
        if getattr(self, "_h", None) and lib is not None:       # None while the interpreter ends
            lib.draco_layout_destroy(self._h)
            self._h = None
            self._address = None

    __del__ = close

    def _here(self, x, numel, type_, what, ordered=True):
        """Address of a tensor of this size and type on the layout's device; ints and None as in the other calls."""
        if x is None or isinstance(x, int):
            return x
        if x.numel() != numel or _TYPES.get(str(x.dtype)) != type_:
            raise DracoError(f"{what}: {x.numel()} x {x.dtype}, not {numel} of type {type_}")
        if not x.is_cuda or x.get_device() != self.device:
            raise DracoError(f"{what} is on {x.device}, not on cuda:{self.device}")
        if not (x.is_contiguous() if ordered else _dense(x)):
            raise DracoError(f"{what} is not {'contiguous' if ordered else 'dense'}: strides {x.stride()}")
        if x.is_neg():
            raise DracoError(f"{what} is a negated view: its memory holds other values")
        address = x.data_ptr()
        if numel and not address:                              # a wrapper without memory of its own, not a tensor that is absent
            raise DracoError(f"{what} has no memory")
        return address

    @staticmethod
    def _sequence(tensors):
        return tensors if isinstance(tensors, (list, tuple)) else list(tensors)

    def _list(self, tensors, what, ordered):
        if len(tensors) != len(self.numels):
            raise DracoError(f"{what}: {len(tensors)} tensors, not {len(self.numels)}")
        a = (_vp * len(tensors))()
        for i, (x, n, t) in enumerate(zip(tensors, self.numels, self.types)):
            a[i] = self._here(x, n, t, f"{what}[{i}]", ordered)
        return a

    def norm(self, tensors, norm, each=None, kind: int = NORM_2, stream=None):
        """draco_norm: norm <- the norm of all tensors, each[t] <- that of tensor t."""
        tensors = self._sequence(tensors)
        rc = _native.norm(self._address, self._meta_address, tensors, norm, each, kind, stream)
        if rc is not NotImplemented:
            return rc
        rc = _check(lib.draco_norm(self._h, self._list(tensors, "tensors", False), kind, self._here(norm, 1, F32, "norm"),
                                   self._here(each, len(self.numels), F32, "each"), _stream(stream)))
        _wrote(norm, each)
        return rc

    def clip(self, tensors, max_norm: float, out=None, norm=None, each=None, separately: bool = False, kind: int = NORM_2, stream=None):
        """draco_clip: the tensors scaled so that their norm (separately: that of each) is at most max_norm, in place or to ``out``.

        An ``out`` tensor has the memory order of its input."""
        tensors, out = self._sequence(tensors), None if out is None else self._sequence(out)
        rc = _native.clip(self._address, self._meta_address, tensors, max_norm, out, norm, each, separately, kind, stream)
        if rc is not NotImplemented:
            return rc
        src = self._list(tensors, "tensors", False)
        dst = None
        if out is not None:
            dst = self._list(out, "out", False)
            for i, (x, y) in enumerate(zip(tensors, out)):
                if hasattr(x, "stride") and hasattr(y, "stride") and _order(x) != _order(y):
                    raise DracoError(f"out[{i}]: shape {tuple(y.shape)}, strides {y.stride()}, not {tuple(x.shape)}, {x.stride()}")
        rc = _check(lib.draco_clip(self._h, src, dst, kind, max_norm, bool(separately), self._here(norm, 1, F32, "norm"),
                                   self._here(each, len(self.numels), F32, "each"), _stream(stream)))
        _wrote(tensors if out is None else out, norm, each)
        return rc

    def pack(self, tensors, row, max_norm: float = float("inf"), norm=None, kind: int = NORM_2, stream=None):
        """draco_pack: the tensors one after the other in the fp32 row, clipped."""
        tensors = self._sequence(tensors)
        rc = _native.pack(self._address, self._meta_address, tensors, row, max_norm, norm, kind, stream)
        if rc is not NotImplemented:
            return rc
        rc = _check(lib.draco_pack(self._h, self._list(tensors, "tensors", True), kind, max_norm, self._here(row, self.d, F32, "row"),
                                   self._here(norm, 1, F32, "norm"), _stream(stream)))
        _wrote(row, norm)
        return rc

    def update(self, params, u, scale: float, max_norm: float = float("inf"), master=None, norm=None, kind: int = NORM_2, stream=None):
        """draco_update: params <- params - scale * c * u, by way of the fp32 master copy where there is one.

        c is from the norm of this u: where ranks hold slices of one vector, leave max_norm out and make their common factor part of scale."""
        params = self._sequence(params)
        rc = _native.update(self._address, self._meta_address, params, u, scale, max_norm, master, norm, kind, stream)
        if rc is not NotImplemented:
            return rc
        rc = _check(lib.draco_update(self._h, self._list(params, "params", True), self._here(u, self.d, F32, "u"),
                                     self._here(master, self.d, F32, "master"), kind, max_norm, scale, self._here(norm, 1, F32, "norm"),
                                     _stream(stream)))
        _wrote(params, master, norm)
        return rc
