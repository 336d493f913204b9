"""Lists of tensors: what is refused before anything runs (no compute: this runs without a GPU)."""
import ctypes

import pytest


def _binding():
    from paper_1803_09877_b200 import build
    build.build()
    from paper_1803_09877_b200 import binding
    return binding


@pytest.mark.parametrize("numels,types", [([], []), ([4, -1], [0, 0]), ([4], [3]), ([4], [-1])])
def test_layouts_that_are_refused(numels, types):
    b = _binding()
    h = ctypes.c_void_p(7)
    n = len(numels)
    rc = b.lib.draco_layout_create(n, (ctypes.c_int64 * max(n, 1))(*numels), (ctypes.c_int * max(n, 1))(*types), ctypes.byref(h))
    assert rc == b.EINVAL and not h.value


def test_too_many_tensors():
    b = _binding()
    n = b.MAX_TENSORS + 1
    h = ctypes.c_void_p()
    assert b.lib.draco_layout_create(n, (ctypes.c_int64 * n)(), (ctypes.c_int * n)(), ctypes.byref(h)) == b.ELIMIT


@pytest.mark.parametrize("numels", [[(1 << 40) + 1], [1 << 39, 1 << 39, 1], [(1 << 63) - 1, (1 << 63) - 1]])
def test_too_many_elements(numels):
    b = _binding()
    h, n = ctypes.c_void_p(), len(numels)
    assert b.lib.draco_layout_create(n, (ctypes.c_int64 * n)(*numels), (ctypes.c_int * n)(), ctypes.byref(h)) == b.ELIMIT


def test_null_arguments():
    b = _binding()
    lib, h = b.lib, ctypes.c_void_p()
    one, zero = (ctypes.c_int64 * 1)(4), (ctypes.c_int * 1)(0)
    assert lib.draco_layout_create(1, one, zero, None) == b.EINVAL
    assert lib.draco_layout_create(1, None, zero, ctypes.byref(h)) == b.EINVAL
    assert lib.draco_layout_create(1, one, None, ctypes.byref(h)) == b.EINVAL
    assert lib.draco_layout_size(None) == b.EINVAL
    assert lib.draco_layout_destroy(None) == b.OK
    tensors = (ctypes.c_void_p * 1)(4096)
    assert lib.draco_norm(None, tensors, 0, 4096, None, None) == b.EINVAL
    assert lib.draco_clip(None, tensors, None, 0, 1.0, 0, None, None, None) == b.EINVAL
    assert lib.draco_pack(None, tensors, 0, 1.0, 4096, None, None) == b.EINVAL
    assert lib.draco_update(None, tensors, 4096, None, 0, 1.0, 1.0, None, None) == b.EINVAL


def test_python_refuses_sizes_and_types_that_do_not_go_together():
    b = _binding()
    import torch
    with pytest.raises(b.DracoError, match="2 sizes, 1 types"):
        b.Layout([1, 2], [b.F32])
    with pytest.raises(b.DracoError, match="float64"):
        b.Layout([1], [torch.float64])
    with pytest.raises(b.DracoError, match="float64"):
        b.Layout.of([torch.zeros(3, dtype=torch.float64)])


def test_dense_tensors():
    """Elements that fill one piece of memory in whatever order: their sum of squares does not depend on it."""
    b = _binding()
    import torch
    x = torch.zeros(4, 6, 5)
    assert b._dense(x) and b._dense(x.permute(2, 0, 1)) and b._dense(torch.zeros(2, 3, 4, 5).to(memory_format=torch.channels_last))
    assert b._dense(x[1]) and b._dense(x[:, :1, :1][:1]) and b._dense(torch.zeros(0, 3))
    assert not b._dense(x[:, :, ::2]) and not b._dense(x[:, 1:]) and not b._dense(torch.zeros(3, 1).expand(3, 4)) and not b._dense(x[:, :1, :1])


def _native_arguments(call, layout, meta, tensors):
    return {"norm": (layout, meta, tensors, None, None, 0, 7), "clip": (layout, meta, tensors, 1.0, None, None, None, False, 0, 7),
            "pack": (layout, meta, tensors, None, 1.0, None, 0, 7), "update": (layout, meta, tensors, None, 1.0, 1.0, None, None, 0, 7)}[call]


@pytest.mark.parametrize("call", ["norm", "clip", "pack", "update"])
def test_native_calls_leave_what_is_unusual_to_python(call):
    b = _binding()
    import torch
    b._find_exchange(torch)
    meta = b._Meta(2, 9, (ctypes.c_int64 * 2)(4, 5), (ctypes.c_int32 * 2)(b.F32, b.BF16), 0)
    at, native = ctypes.addressof(meta), getattr(b._native, call)
    right = [torch.zeros(4), torch.zeros(5, dtype=torch.bfloat16)]             # but on the host
    for tensors in (right, right[:1], iter(right), [right[1], right[0]], [torch.zeros(4).to_sparse(), None], [object(), None], [4096, None], None):
        assert native(*_native_arguments(call, None, at, tensors)) is NotImplemented
        assert getattr(b._CtypesCalls, call)(*_native_arguments(call, None, at, tensors)) is NotImplemented
    if b._native is not b._CtypesCalls:
        for tensors in ([None, None], (None, None)):
            with pytest.raises(b.DracoError, match="invalid argument"):        # no layout, as after close()
                native(*_native_arguments(call, None, at, tensors))
        with pytest.raises(TypeError):
            native(None, at, right)
        with pytest.raises(TypeError):
            native(*[x if x != 0 or isinstance(x, bool) else "2-norm" for x in _native_arguments(call, None, at, [None, None])])


def test_any_torch_goes_without_its_module(monkeypatch, tmp_path):
    """Another torch's module is not taken, and one that cannot be loaded is told of; torch's own function takes its place."""
    b = _binding()
    import sysconfig
    import torch
    own = getattr(torch.Tensor, "__dlpack_c_exchange_api__", None)
    monkeypatch.setattr(b, "_PKG", str(tmp_path))
    assert b._exchange(torch) is own
    (tmp_path / (f"_torch_tensors-{torch.__version__}" + sysconfig.get_config_var("EXT_SUFFIX"))).write_bytes(b"not a module")
    with pytest.warns(RuntimeWarning, match="torch's own function"):
        assert b._exchange(torch) is own


class _DLTensor(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("device_type", ctypes.c_int32), ("device_id", ctypes.c_int32), ("ndim", ctypes.c_int32),
                ("code", ctypes.c_uint8), ("bits", ctypes.c_uint8), ("lanes", ctypes.c_uint16), ("shape", ctypes.c_void_p),
                ("strides", ctypes.c_void_p), ("byte_offset", ctypes.c_uint64)]


_READ = ctypes.PYFUNCTYPE(ctypes.c_int, ctypes.py_object, ctypes.POINTER(_DLTensor))
_capsule_name = ctypes.PYFUNCTYPE(ctypes.c_char_p, ctypes.py_object)(("PyCapsule_GetName", ctypes.pythonapi))
_capsule_pointer = ctypes.PYFUNCTYPE(ctypes.c_void_p, ctypes.py_object, ctypes.c_char_p)(("PyCapsule_GetPointer", ctypes.pythonapi))
_new_capsule = ctypes.PYFUNCTYPE(ctypes.py_object, ctypes.c_void_p, ctypes.c_char_p, ctypes.c_void_p)(("PyCapsule_New", ctypes.pythonapi))
_READERS = (5, 7)                                # places of functions that read a tensor, eight bytes each: DLPack's, and one behind its table


def _as_if_on_a_gpu(capsule, keep):
    """The exchange of this capsule, telling of host tensors as if they were on cuda:0."""
    name = _capsule_name(capsule)
    words = 8 if name != b"dlpack_exchange_api" else 7
    table = (ctypes.c_uint64 * 8)()
    ctypes.memmove(table, _capsule_pointer(capsule, name), 8 * words)
    for place in _READERS:
        if place < words and table[place]:
            def read(x, out, real=_READ(table[place])):
                rc = real(x, out)
                out.contents.device_type, out.contents.device_id = 2, 0
                return rc
            keep.append(_READ(read))
            table[place] = ctypes.cast(keep[-1], ctypes.c_void_p).value
    keep += [table, name]
    return _new_capsule(ctypes.addressof(table), name, None)


@pytest.fixture(params=["built", "torch's own"])
def exchange(request):
    """The binding with one of the two exchanges in place."""
    b = _binding()
    import torch
    if b._native is b._CtypesCalls:
        pytest.skip("no native calls")
    b._find_exchange(torch)
    own, usual, keep = getattr(torch.Tensor, "__dlpack_c_exchange_api__", None), b._exchange(torch), []
    chosen = own if request.param == "torch's own" else usual
    if chosen is None or (request.param == "built" and usual is own):
        pytest.skip("not there")
    b._native.set_exchange(torch.Tensor, torch.nn.Parameter, _as_if_on_a_gpu(chosen, keep))
    yield b
    b._native.set_exchange(torch.Tensor, torch.nn.Parameter, usual)


@pytest.mark.parametrize("call", ["norm", "clip", "pack", "update"])
def test_negated_views_are_left_to_python(exchange, call):
    """Their memory holds the other sign, whoever tells of it."""
    b = exchange
    import torch
    meta = b._Meta(1, 4, (ctypes.c_int64 * 1)(4), (ctypes.c_int32 * 1)(b.F32), 0)
    at, x = ctypes.addressof(meta), torch.ones(4)
    one = b._Meta(1, 1, (ctypes.c_int64 * 1)(1), (ctypes.c_int32 * 1)(b.F32), 0)
    with pytest.raises(b.DracoError, match="invalid argument"):                # taken: no layout
        getattr(b._native, call)(*_native_arguments(call, None, at, [x]))
    assert getattr(b._native, call)(*_native_arguments(call, None, at, [torch._neg_view(x)])) is NotImplemented
    part = torch.ones(1, dtype=torch.complex64).conj().imag
    assert part.is_neg()
    assert getattr(b._native, call)(*_native_arguments(call, None, ctypes.addressof(one), [part])) is NotImplemented
    for place, numel in {"norm": [(4, 1)], "clip": [(6, 1)], "pack": [(3, 4)], "update": [(3, 4), (6, 4)]}[call]:        # each, each, row, u and master
        args = list(_native_arguments(call, None, at, [x]))
        args[place] = torch._neg_view(torch.ones(numel))
        assert getattr(b._native, call)(*args) is NotImplemented


@pytest.mark.parametrize("call", ["norm", "clip", "clip to out", "pack", "update"])
def test_lazy_clones_get_memory_of_their_own_before_they_are_written(exchange, call):
    """And whose memory else a call writes would be the source's, too."""
    b = exchange
    import torch
    meta = b._Meta(1, 4, (ctypes.c_int64 * 1)(4), (ctypes.c_int32 * 1)(b.F32), 0)
    name, at = call.split()[0], ctypes.addressof(meta)
    sources = [torch.ones(4), torch.ones(1), torch.ones(4)]
    x, scalar, vector = (torch._lazy_clone(t) for t in sources)
    args = list(_native_arguments(name, None, at, [x]))
    written = [scalar]
    if call == "norm":
        args[3] = scalar
    elif call == "clip":
        args[5] = scalar
        written += [x]
    elif call == "clip to out":
        args[4], args[5] = [vector], scalar
        written += [vector]
    elif call == "pack":
        args[3], args[5] = vector, scalar
        written += [vector]
    else:
        args[6], args[7] = vector, scalar
        written += [x, vector]
    with pytest.raises(b.DracoError, match="invalid argument"):                # taken: no layout
        getattr(b._native, name)(*args)
    assert not any(torch._C._is_cow_tensor(t) for t in written)
    assert all(bool((t == 1.0).all()) for t in [x, scalar, vector] + sources)


def test_autograd_is_told_by_any_torch(monkeypatch):
    """Of lists at once, or tensor by tensor where torch takes no list."""
    b = _binding()
    import torch
    with torch.inference_mode():
        without = torch.zeros(1)
    for one_at_a_time in (False, True):
        if one_at_a_time:
            real = torch._C._increment_version
            monkeypatch.setattr(torch.autograd.graph, "increment_version", lambda t: real((t,)) if isinstance(t, torch.Tensor) else real(0))
        x = [torch.zeros(2) for _ in range(4)]
        before = [t._version for t in x]
        b._wrote([x[0], None, 4096, x[1], without], x[2], None)
        b._wrote(None, 4096, ())
        assert [t._version - v for t, v in zip(x, before)] == [1, 1, 1, 0]


class _Somewhere:
    """A tensor, as far as a layout asks."""

    def __init__(self, numel, dtype, device):
        self.count, self.dtype, self.device = numel, dtype, device
        self.is_cuda = device is not None

    def numel(self):
        return self.count

    def get_device(self):
        return self.device


def test_layouts_are_made_on_their_tensors_device(monkeypatch):
    b = _binding()
    import contextlib
    import torch
    current, made = [0], []

    @contextlib.contextmanager
    def device(index):
        before, current[0] = current[0], index
        yield
        current[0] = before

    class Layout(b.Layout):
        def __init__(self, numels, types):
            made.append((current[0], numels, types))

    monkeypatch.setattr(torch.cuda, "device", device)
    f32, bf16 = torch.float32, torch.bfloat16
    Layout.of([_Somewhere(3, f32, 1), _Somewhere(4, bf16, 1)])
    Layout.of(iter([_Somewhere(3, f32, 0)]))
    Layout.of([_Somewhere(3, f32, None), _Somewhere(4, bf16, 1)])
    Layout.of([_Somewhere(3, f32, None)])
    Layout.of([])
    assert made == [(1, [3, 4], [f32, bf16]), (0, [3], [f32]), (1, [3, 4], [f32, bf16]), (0, [3], [f32]), (0, [], [])] and current == [0]
    with pytest.raises(b.DracoError, match="cuda:0, cuda:2"):
        Layout.of([_Somewhere(3, f32, 2), _Somewhere(3, f32, 0)])
