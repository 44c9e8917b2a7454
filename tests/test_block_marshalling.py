"""The native half of the operators around attention (csrc/va_host_block.h), built for CPU tensors and bound to a function that only
notes what it is called with: it leaves to the Python half what that refuses, and calls the library with the same arguments."""
import ctypes
import importlib.machinery
import importlib.util
import os

import pytest
import torch

from paper_2605_08962_amd import binding, build
from tests import test_block_refusals as R
from tests.test_block_refusals import on_cpu  # noqa: F401

NAMES = ("rotary_positions", "rotary_fwd", "rotary_bwd", "act8_pack", "act8_unpack", "bwd_act8_workspace_bytes", "bwd_act8", "norm_fwd",
         "norm_bwd_workspace_bytes", "norm_bwd")
STRUCTS = {"rotary_fwd": binding.RotaryParams, "rotary_bwd": binding.RotaryParams, "norm_fwd": binding.NormParams,
           "norm_bwd": binding.NormParams, "bwd_act8": binding.Params}


@pytest.fixture(scope="module")
def module(tmp_path_factory):
    path = build.compile_host(os.path.join(R.__file__.rsplit(os.sep, 1)[0], "block_marshalling_check.cpp"),
                              str(tmp_path_factory.mktemp("host") / "block_marshalling_check.so"))
    loader = importlib.machinery.ExtensionFileLoader("block_marshalling_check", path)
    m = importlib.util.module_from_spec(importlib.util.spec_from_loader("block_marshalling_check", loader))
    loader.exec_module(m)
    return m


def _noted(name, args):
    """A call's arguments, the structures behind its first pointer read out; pointers of tensors the test cannot know by their being
    there."""
    args = list(args)
    if name in STRUCTS:
        p = ctypes.cast(args[0], ctypes.POINTER(STRUCTS[name])).contents
        args[0] = tuple(getattr(p, f) for f, _ in p._fields_)
    elif name.startswith("act8"):
        t = ctypes.cast(args[0], ctypes.POINTER(binding.Act8Tensor))
        args[0] = [(bool(x.values), bool(x.codes), bool(x.scales), x.total_tokens, x.rows_per_token, x.channels, x.stride)
                   for x in (t[i] for i in range(args[1]))]
    values = [getattr(x, "value", x) for x in args]
    return name, [bool(v) if isinstance(v, int) and abs(v) > 1 << 20 else v for v in values]


@pytest.fixture
def both(module, on_cpu, monkeypatch):  # noqa: F811
    """The binding on CPU tensors, `native(True)` through the native half, `native(False)` through the Python one; calls of both."""
    calls, keep, addresses = [], [], []
    real = ctypes.CDLL(binding.LIB_PATH)
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    types = {"rotary_positions": [i32] * 3 + [vp] * 5, "rotary_fwd": [vp] * 11, "rotary_bwd": [vp] * 11, "act8_pack": [vp, i32, i32, vp],
             "act8_unpack": [vp, i32, i32, vp], "bwd_act8": [vp, i32] + [vp] * 15 + [sz, vp], "norm_fwd": [vp] * 12,
             "norm_bwd": [vp] * 13 + [sz, vp]}
    assert all(hasattr(real, "varlen_attn_" + n) for n in NAMES)

    def make(name):
        if name.endswith("bytes"):
            return ctypes.CFUNCTYPE(sz, vp)(lambda p: 4096)
        return ctypes.CFUNCTYPE(ctypes.c_int, *types[name])(lambda *a: calls.append(_noted(name, a)) or status[0])
    status = [0]
    for n in NAMES:
        keep.append(make(n))
        addresses.append(ctypes.cast(keep[-1], vp).value)
    module.bind_block(*addresses, binding.Act8)
    module.set_current_stream(48)
    module.watch(False)

    class Lib:
        def __getattr__(self, name):
            f = keep[NAMES.index(name[len("varlen_attn_"):])]
            argtypes = types.get(name[len("varlen_attn_"):])
            return (lambda p: 4096) if argtypes is None else \
                lambda *a: f(*(ctypes.cast(x, vp) if not isinstance(x, (int, type(None), vp)) else x for x in a))

    monkeypatch.setattr(binding, "load", Lib)
    monkeypatch.setattr(binding, "status_string", str)

    def native(on):
        monkeypatch.setattr(binding, "_host", module if on else binding._PythonHalf)
        calls.clear()
    native.calls, native.status, native.module = calls, status, module
    yield native
    module.watch(False)


MORE = [(R._rotary_call, dict(q=R.bf(2 * R.T, R.HQ, R.D)[::2], q_out=R.bf(R.T, 9, R.D)[:, :R.HQ], v=None)),
        (lambda **o: lambda b: b.varlen_attn_rotary_bwd(R.bf(6, 4, 64), R.bf(6, 2, 64), R.i32(3, 6), torch.zeros(20), R.i32(20), interleaved=True), {}),
        (lambda **o: lambda b: b.varlen_attn_act8_pack([R.bf(3, 200), R.bf(5, 2, 64), R.bf(0, 8), R.bf(6, 32)[:, :16]], "e4m3"), {}),
        (lambda **o: lambda b: b.varlen_attn_act8_unpack([R._a8(3, 200), R._a8(5, 2, 64), R._a8(7, 8)]), {}),
        (R._bwd_call, dict(dx=R.bf(R.T, 200)[:, 8:104], dsummed=R.bf(R.T, 96))), (R._bwd_call, dict(x=R._a8(R.T, 96, code=torch.float8_e4m3fn))),
        (R._fwd_call, dict(weight=None, bias=None, residual=None, out=R.bf(R.T, 96)))]


@pytest.mark.parametrize("make,other", R.GOOD + MORE)
def test_the_native_half_calls_what_the_python_half_calls(both, make, other):
    call, results = make(**other), []
    for on in (False, True):
        both(on)
        r = call(binding)
        results.append((both.calls[:], r))
    (want, a), (got, b) = results
    assert len(want) == 1 and got == want
    flat = lambda r: [t for x in (r if isinstance(r, (list, tuple)) else [r]) for t in (x if isinstance(x, (list, tuple)) else [x])]  # noqa: E731
    assert type(a) is type(b) and len(flat(a)) == len(flat(b))
    for x, y in zip(flat(a), flat(b)):
        assert (x is None) == (y is None)
        if x is not None:
            assert x.shape == y.shape and x.dtype == y.dtype and x.stride() == y.stride()


@pytest.mark.parametrize("make,other,why", R.BAD)
def test_the_native_half_leaves_what_is_refused_to_the_python_half(both, make, other, why):
    both(True)
    with pytest.raises(ValueError, match=why):
        make(**other)(binding)
    assert not both.calls


def test_a_status_is_raised(both):
    both.status[0] = 2
    for make, other in R.GOOD + MORE:
        both(True)
        with pytest.raises(binding.VarlenAttnError) as e:
            make(**other)(binding)
        assert e.value.status == 2 and len(both.calls) == 1


def test_allocations_leave_the_interpreter_to_other_threads_and_run_out_as_torchs(both):
    for make, other in [(R._rotary_call, {}), (R._fwd_call, dict(save="int8")), (R._bwd_call, {}), (R._attn_call, {}), *MORE[1:4]]:
        both(True)
        both.module.watch(False)
        make(**other)(binding)
        with_lock, without_lock = both.module.watch(False)
        assert with_lock == 0 and without_lock >= 2
        call = make(**other)
        both.module.watch(True)
        with pytest.raises(torch.OutOfMemoryError, match="the test has no memory"):
            call(binding)
        both.module.watch(False)


def test_a_tensor_elsewhere_is_left_to_the_python_half(both):
    """On the device `meta` here, which stands for another GPU: the Python half names it."""
    meta = lambda t: t.to("meta")  # noqa: E731
    for make, other, why in [(R._rotary_call, dict(k=meta(R.bf(R.T, R.HKV, R.D))), "k must be on"),
                             (R._fwd_call, dict(bias=meta(R.bf(96))), "bias must be on"), (R._bwd_call, dict(mean=meta(torch.zeros(R.T))), "mean must be on"),
                             (R._attn_call, dict(cu=meta(R.i32(2))), "cu_seqlens must be on"), (R._pos_call, dict(first=meta(R.i32(2))), "first must be on")]:
        both(True)
        with pytest.raises(ValueError, match=why):
            make(**other)(binding)
        assert not both.calls
