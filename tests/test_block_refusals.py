"""What the operators around attention refuse, on the CPU: the library's checks of what the host can see (with pointers that are never
followed), and the binding's checks of tensors (with a library that notes its calls)."""
import contextlib
import ctypes
import types

import pytest
import torch

from paper_2605_08962_amd import binding

OK, NULL, SHAPE, UNSUPPORTED, SMALL, SCALE, MISALIGNED = 0, 1, 2, 3, 4, 5, 7


@pytest.fixture(scope="module")
def lib():
    return binding.load()


def test_structs_match_the_header():
    import os
    import re
    text = open(os.path.join(os.path.dirname(binding._HERE), "include", "varlen_attn.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    for name, cls in (("varlen_attn_rotary_params", binding.RotaryParams), ("varlen_attn_act8_tensor", binding.Act8Tensor),
                      ("varlen_attn_norm_params", binding.NormParams)):
        body = text[:text.index("} " + name + ";")]
        body = body[body.rindex("typedef struct {") + len("typedef struct {"):]
        fields = [n.strip(" *") for line in body.split(";") if line.strip() for n in line.strip().split(None, 1)[1].split(",")]
        assert fields == [f[0] for f in cls._fields_]
    assert (ctypes.sizeof(binding.RotaryParams), ctypes.sizeof(binding.Act8Tensor), ctypes.sizeof(binding.NormParams)) == (80, 48, 48)


def _rotary(lib, ptrs=None, inverse=False, **change):
    f = dict(total_tokens=8, num_q_heads=4, num_kv_heads=2, head_dim=64, num_pairs=32, num_axes=3, interleaved=0, q_stride=512,
             k_stride=512, v_stride=512, q_out_stride=256, k_out_stride=128, v_out_stride=128)
    f.update(change)
    p = binding.RotaryParams(*(f[n] for n, _ in binding.RotaryParams._fields_))
    a = dict(q=16, k=16, v=16, positions=16, inv_freq=16, pair_axis=16, q_out=16, k_out=16, v_out=16)
    a.update(ptrs or {})
    return (lib.varlen_attn_rotary_bwd if inverse else lib.varlen_attn_rotary_fwd)(ctypes.byref(p), *a.values(), None)


@pytest.mark.parametrize("inverse", [False, True])
def test_rotary_arguments(lib, inverse):
    call = lambda ptrs=None, **c: _rotary(lib, ptrs, inverse, **c)  # noqa: E731
    assert call(total_tokens=0) == OK and call({"q": None}, total_tokens=0) == OK
    for bad in (dict(total_tokens=-1), dict(num_q_heads=0), dict(num_kv_heads=0), dict(num_pairs=0), dict(num_pairs=33), dict(num_axes=0),
                dict(num_axes=9), dict(interleaved=2), dict(q_stride=255), dict(k_stride=127), dict(v_stride=127), dict(q_out_stride=255),
                dict(k_out_stride=0), dict(v_out_stride=-5), dict(num_q_heads=1 << 21, q_stride=1 << 40, q_out_stride=1 << 40)):
        assert call(**bad) == SHAPE, bad
    for d in (0, 1, 513):
        assert call(head_dim=d) == UNSUPPORTED
    for name in ("q", "k", "positions", "inv_freq", "pair_axis", "q_out", "k_out", "v", "v_out"):
        assert call({name: None}) == NULL, name
    for name in ("q", "k", "v", "q_out", "k_out", "v_out"):
        assert call({name: 17}) == MISALIGNED, name
    for name in ("positions", "inv_freq", "pair_axis"):
        assert call({name: 18}) == MISALIGNED, name
    assert lib.varlen_attn_rotary_fwd(None, *[16] * 9, None) == NULL


def test_position_arguments(lib):
    def call(T=8, S=2, m=1, cu=16, grids=16, first=16, out=16):
        return lib.varlen_attn_rotary_positions(T, S, m, cu, grids, first, out, None)
    assert call(T=0) == OK and call(T=0, cu=None, out=None) == OK
    assert call(T=-1) == SHAPE and call(S=-1) == SHAPE and call(m=0) == SHAPE and call(m=65) == SHAPE
    assert call(cu=None) == NULL and call(grids=None) == NULL and call(out=None) == NULL
    assert call(cu=18) == call(grids=18) == call(first=18) == call(out=18) == MISALIGNED


def _act8(lib, pack=True, num=1, fmt=0, **change):
    f = dict(values=16, codes=16, scales=16, total_tokens=8, rows_per_token=2, channels=64, stride=128)
    f.update(change)
    t = binding.Act8Tensor(*f.values())
    return (lib.varlen_attn_act8_pack if pack else lib.varlen_attn_act8_unpack)(ctypes.byref(t), num, fmt, None)


@pytest.mark.parametrize("pack", [False, True])
def test_act8_arguments(lib, pack):
    call = lambda **c: _act8(lib, pack, **c)  # noqa: E731
    assert call(num=0) == OK and call(total_tokens=0) == OK and call(total_tokens=0, values=None) == OK
    for bad in (dict(num=-1), dict(num=9), dict(fmt=2), dict(fmt=-1), dict(total_tokens=-1), dict(rows_per_token=0), dict(channels=0),
                dict(stride=127), dict(total_tokens=1 << 30, rows_per_token=1 << 10, stride=1 << 40)):
        assert call(**bad) == SHAPE, bad
    assert call(channels=16385, stride=1 << 20) == UNSUPPORTED
    assert call(values=None) == call(codes=None) == call(scales=None) == NULL
    assert call(values=17) == call(scales=18) == MISALIGNED
    assert lib.varlen_attn_act8_pack(None, 1, 0, None) == NULL


def test_act8_backward_arguments(lib):
    mk = binding.make_params
    call = lambda p, fmt=0, ptrs=(16,) * 15, n=1 << 30: lib.varlen_attn_bwd_act8(ctypes.byref(p), fmt, *ptrs, n, None)  # noqa: E731
    ok = mk(8, 1, 2, 2, 64, 0, 0.125)
    assert call(mk(0, 0, 2, 2, 64, 0, 0.125), ptrs=(None,) * 15, n=0) == OK
    assert call(mk(8, 1, 3, 2, 64, 0, 0.125)) == SHAPE and call(ok, fmt=2) == SHAPE
    assert call(mk(8, 1, 2, 2, 72, 0, 0.125)) == UNSUPPORTED and call(mk(8, 1, 2, 2, 64, 0, -1.0)) == SCALE
    for i in range(15):
        assert call(ok, ptrs=[None if j == i else 16 for j in range(15)]) == NULL, i
        wrong = {0: 24, 2: 18, 4: 18, 6: 18, 8: 18, 9: 18, 10: 18, 11: 24, 12: 24, 13: 24, 14: 24}.get(i)
        if wrong:  # (codes are bytes)
            assert call(ok, ptrs=[wrong if j == i else 16 for j in range(15)]) == MISALIGNED, i
    need = binding.bwd_act8_workspace_bytes(mk(8, 1, 2, 2, 64, 0, 0.125, 1))
    assert call(mk(8, 1, 2, 2, 64, 0, 0.125, 1), n=need - 1) == SMALL and call(ok, n=0) == SMALL
    assert need == binding.bwd_workspace_bytes(mk(8, 1, 2, 2, 64, 0, 0.125, 1)) + 4 * 8 * 2 * 64 * 2
    assert binding.bwd_act8_workspace_bytes(mk(8, 1, 2, 2, 72, 0, 0.1)) == 0


def _norm(lib, back=False, ptrs=None, n=1 << 30, **change):
    f = dict(total_tokens=8, rows_per_token=2, channels=64, weight_type=0, act8_format=0, eps=1e-5, x_stride=128, dy_stride=128,
             dx_stride=128)
    f.update(change)
    p = binding.NormParams(*f.values())
    if back:
        a = dict(dy=16, x=16, codes=None, scales=None, mean=16, rstd=16, weight=16, dsummed=16, dx=16, dweight=16, dbias=16, ws=16)
        a.update(ptrs or {})
        return lib.varlen_attn_norm_bwd(ctypes.byref(p), *a.values(), n, None)
    a = dict(x=16, residual=16, weight=16, bias=16, y=16, summed=16, mean=16, rstd=16, codes=16, scales=16)
    a.update(ptrs or {})
    return lib.varlen_attn_norm_fwd(ctypes.byref(p), *a.values(), None)


@pytest.mark.parametrize("back", [False, True])
def test_norm_arguments(lib, back):
    call = lambda ptrs=None, **c: _norm(lib, back, ptrs, **c)  # noqa: E731
    for bad in (dict(total_tokens=-1), dict(rows_per_token=0), dict(channels=0), dict(weight_type=2), dict(act8_format=2),
                dict(x_stride=127), dict(total_tokens=1 << 30, rows_per_token=1 << 11, x_stride=1 << 40, dy_stride=1 << 40, dx_stride=1 << 40)):
        assert call(**bad) == SHAPE, bad
    assert call(channels=16385, x_stride=1 << 20, dy_stride=1 << 20, dx_stride=1 << 20) == UNSUPPORTED
    for eps in (-1e-5, float("nan"), float("inf")):
        assert call(eps=eps) == SCALE
    names = ("dy", "mean", "rstd", "dx", "dweight", "dbias", "ws", "x") if back else \
        ("x", "y", "mean", "rstd", "residual", "summed", "codes", "scales", "weight")
    for name in names:
        assert call({name: None}) == NULL, name
    halves = ("dy", "x", "dsummed", "dx", "weight") if back else ("x", "residual", "y", "summed", "weight", "bias")
    for name in halves:
        assert call({name: 17}) == MISALIGNED, name
    for name in ("mean", "rstd", "dweight", "dbias", "ws") if back else ("mean", "rstd", "scales"):
        assert call({name: 18}) == MISALIGNED, name
    assert call({"weight": 18}, weight_type=1) == MISALIGNED
    if back:
        assert call(dy_stride=127) == SHAPE and call(dx_stride=127) == SHAPE
        assert call({"codes": 16, "scales": 16}) == NULL            # h twice
        assert call({"x": None, "codes": 16}) == NULL               # without its scales
        assert call(n=255) == SMALL
        assert call({"weight": None}, total_tokens=0) == OK
        assert lib.varlen_attn_norm_bwd(None, *[16] * 12, 64, None) == NULL
    else:
        assert call(total_tokens=0) == OK
        assert lib.varlen_attn_norm_fwd(None, *[16] * 10, None) == NULL
    assert binding.norm_bwd_workspace_bytes(binding.NormParams(8, 2, 64, 0, 0, 1e-5, 128, 128, 128)) % 256 == 0
    assert binding.norm_bwd_workspace_bytes(binding.NormParams(8, 2, 0, 0, 0, 1e-5, 128, 128, 128)) == 0


def test_tensors_on_the_cpu_are_refused_by_name():
    x, i = torch.zeros(4, 2, 64, dtype=torch.bfloat16), torch.zeros(3, 4, dtype=torch.int32)
    for call in (lambda: binding.varlen_attn_rotary_fwd(x, x, i, x, i), lambda: binding.varlen_attn_rotary_bwd(x, x, i, x, i),
                 lambda: binding.varlen_attn_rotary_positions(i[0], i, 4), lambda: binding.varlen_attn_act8_pack([x]),
                 lambda: binding.varlen_attn_norm_fwd(x), lambda: binding.varlen_attn_norm_bwd(x, x, x, x),
                 lambda: binding.varlen_attn_act8_unpack([binding.Act8(x.to(torch.int8), x)]),
                 lambda: binding.varlen_attn_bwd_act8(x, x, x, x, x, x, i, True, 0.1)):
        with pytest.raises(ValueError, match="on the GPU"):
            call()


# ---- the binding's own checks ----------------------------------------------------------------------------------------

def bf(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


T, HQ, HKV, D, P = 6, 4, 2, 64, 32


def _rotary_call(f=None, **o):
    a = dict(q=bf(T, HQ, D), k=bf(T, HKV, D), positions=i32(3, T), inv_freq=torch.zeros(P), pair_axis=i32(P), v=bf(T, HKV, D), q_out=None,
             k_out=None, v_out=None)
    a.update(o)
    return lambda b: b.varlen_attn_rotary_fwd(a["q"], a["k"], a["positions"], a["inv_freq"], a["pair_axis"], v=a["v"], q_out=a["q_out"],
                                              k_out=a["k_out"], v_out=a["v_out"])


def _pos_call(**o):
    a = dict(cu=i32(3), grids=i32(2, 3), total=T, first=i32(2), out=None)
    a.update(o)
    return lambda b: b.varlen_attn_rotary_positions(a["cu"], a["grids"], a["total"], first=a["first"], out=a["out"])


def _a8(*shape, code=torch.int8):
    return binding.Act8(torch.zeros(shape).to(code), torch.zeros(*shape[:-1], -(-shape[-1] // 128)))


def _fwd_call(**o):
    a = dict(x=bf(T, 96), weight=bf(96), bias=bf(96), residual=bf(T, 96), save=None, out=None, mean=None, summed=None, saved=None)
    a.update(o)
    return lambda b: b.varlen_attn_norm_fwd(a["x"], a["weight"], a["bias"], residual=a["residual"], save=a["save"], out=a["out"],
                                            mean=a["mean"], summed=a["summed"], saved=a["saved"])


def _bwd_call(**o):
    a = dict(dy=bf(T, 96), x=bf(T, 96), mean=torch.zeros(T), rstd=torch.zeros(T), weight=bf(96), dsummed=None, dx=None, dw=None, ws=None)
    a.update(o)
    return lambda b: b.varlen_attn_norm_bwd(a["dy"], a["x"], a["mean"], a["rstd"], a["weight"], dsummed=a["dsummed"], dx=a["dx"],
                                            dweight=a["dw"], workspace=a["ws"])


def _attn_call(**o):
    a = dict(dout=bf(T, HQ, D), q=_a8(T, HQ, D), k=_a8(T, HKV, D), v=_a8(T, HKV, D), out=_a8(T, HQ, D), lse=torch.zeros(HQ, T), cu=i32(2),
             dq=None, dk=None, ws=None)
    a.update(o)
    return lambda b: b.varlen_attn_bwd_act8(a["dout"], a["q"], a["k"], a["v"], a["out"], a["lse"], a["cu"], True, 0.1, dq=a["dq"],
                                            dk=a["dk"], workspace=a["ws"])


BAD = [
    (_rotary_call, dict(q=bf(T, HQ, D).float()), "q must be"), (_rotary_call, dict(q=bf(T, HQ * D)), "q must be"),
    (_rotary_call, dict(q=bf(T, D, HQ).transpose(1, 2)), "q must hold"), (_rotary_call, dict(q=bf(HQ, T, D).transpose(0, 1)), "q must hold"),
    (_rotary_call, dict(q=bf(1, HQ, D).expand(T, -1, -1)), "q must hold"), (_rotary_call, dict(q=bf(T, HQ, 2 * D)[..., ::2]), "q must hold"),
    (_rotary_call, dict(k=bf(T - 1, HKV, D)), "k must be"), (_rotary_call, dict(k=bf(T, HKV, 2 * D)), "k must be"),
    (_rotary_call, dict(v=bf(T, HQ, D)), "v must match"), (_rotary_call, dict(v=None, v_out=bf(T, HKV, D)), "v must be given"),
    (_rotary_call, dict(positions=i32(3, T - 1)), "positions must"), (_rotary_call, dict(positions=i32(3, T).long()), "positions must"),
    (_rotary_call, dict(positions=i32(T, 3).T), "positions must"), (_rotary_call, dict(pair_axis=i32(P - 1)), "pair_axis must"),
    (_rotary_call, dict(inv_freq=torch.zeros(P).double()), "inv_freq must"), (_rotary_call, dict(q_out=bf(T, HQ, D + 8)), "q_out must"),
    (_rotary_call, dict(k_out=bf(T, HQ, D)), "k_out must"), (_rotary_call, dict(v_out=bf(T, HKV, D).half()), "v_out must"),
    (_rotary_call, dict(q_out=bf(1, HQ, D).expand(T, -1, -1)), "q_out must hold"),
    (_pos_call, dict(grids=i32(3, 3)), "grids must"), (_pos_call, dict(grids=i32(2, 2)), "grids must"), (_pos_call, dict(cu=i32(3).long()), "cu_rows must"),
    (_pos_call, dict(first=i32(3)), "first must"), (_pos_call, dict(out=i32(3, T + 1)), "out must"), (_pos_call, dict(cu=i32(1, 3)), "grids must"),
    (lambda **o: lambda b: b.varlen_attn_act8_pack([bf(2, 8)], "int4"), {}, "format must"),
    (lambda **o: lambda b: b.varlen_attn_act8_pack([bf(2, 8), bf(8)]), {}, r"tensors\[1\] must"),
    (lambda **o: lambda b: b.varlen_attn_act8_pack([bf(2, 8)], out=[]), {}, "out must"),
    (lambda **o: lambda b: b.varlen_attn_act8_pack([bf(2, 8)], out=[_a8(2, 8, code=torch.float8_e4m3fn)]), {}, r"out\[0\] must match"),
    (lambda **o: lambda b: b.varlen_attn_act8_pack([bf(2, 8)], out=[_a8(2, 9)]), {}, r"out\[0\] must match"),
    (lambda **o: lambda b: b.varlen_attn_act8_unpack([bf(2, 8)]), {}, r"packed\[0\] must be an Act8"),
    (lambda **o: lambda b: b.varlen_attn_act8_unpack([_a8(2, 8), _a8(2, 8, code=torch.float8_e4m3fn)]), {}, "packed must be of one"),
    (lambda **o: lambda b: b.varlen_attn_act8_unpack([binding.Act8(torch.zeros(2, 8, dtype=torch.uint8), torch.zeros(2, 1))]), {}, "codes must"),
    (lambda **o: lambda b: b.varlen_attn_act8_unpack([binding.Act8(torch.zeros(2, 8, dtype=torch.int8), torch.zeros(2, 2))]), {}, "scales must"),
    (lambda **o: lambda b: b.varlen_attn_act8_unpack([_a8(2, 8)], out=[bf(2, 9)]), {}, r"out\[0\] must"),
    (_fwd_call, dict(x=bf(96)), "x must"), (_fwd_call, dict(x=bf(96, T).T), "x must hold"), (_fwd_call, dict(weight=None), "weight must be given"),
    (_fwd_call, dict(weight=bf(95)), "weight must"), (_fwd_call, dict(weight=bf(96).half()), "weight must"),
    (_fwd_call, dict(bias=torch.zeros(96)), "bias must have"), (_fwd_call, dict(residual=bf(T, 95)), "residual must"),
    (_fwd_call, dict(residual=bf(T, 192)[:, ::2]), "residual must"), (_fwd_call, dict(save="e5m2"), "save must"),
    (_fwd_call, dict(out=bf(T, 192)[:, :96]), "out must"), (_fwd_call, dict(out=bf(T + 1, 96)), "out must"),
    (_fwd_call, dict(mean=torch.zeros(T, 1)), "mean must"), (_fwd_call, dict(summed=bf(T, 97)), "summed must"),
    (_fwd_call, dict(residual=None, summed=bf(T, 96)), "residual must be given"), (_fwd_call, dict(saved=_a8(T, 96)), "saved must match"),
    (_fwd_call, dict(save="e4m3", saved=_a8(T, 96)), "saved must match"), (_bwd_call, dict(dw=torch.zeros(95)), "dweight must"),
    (_bwd_call, dict(dw=torch.zeros(96), weight=None), "weight must be given"),
    (_bwd_call, dict(x=bf(T, 95)), "x must match"), (_bwd_call, dict(x=_a8(T, 95)), "x must match"), (_bwd_call, dict(mean=torch.zeros(T + 1)), "mean must"),
    (_bwd_call, dict(rstd=torch.zeros(T).double()), "rstd must"), (_bwd_call, dict(dsummed=bf(T - 1, 96)), "dsummed must"),
    (_bwd_call, dict(dx=bf(T, 97)), "dx must"), (_bwd_call, dict(dx=bf(1, 96).expand(T, -1)), "dx must hold"),
    (_bwd_call, dict(ws=torch.zeros(64, dtype=torch.uint8)[::2]), "workspace must"), (_bwd_call, dict(weight=bf(2, 96)), "weight must"),
    (_attn_call, dict(q=_a8(T, HQ, D, code=torch.float8_e4m3fn)), "q, k, v and out must"), (_attn_call, dict(dout=bf(T, HKV, D)), "dout and out must"),
    (_attn_call, dict(out=_a8(T, HKV, D)), "dout and out must"), (_attn_call, dict(v=_a8(T, HQ, D)), "k and v must"),
    (_attn_call, dict(k=_a8(T - 1, HKV, D), v=_a8(T - 1, HKV, D)), "k and v must"), (_attn_call, dict(lse=torch.zeros(HQ, T - 1)), "lse must"),
    (_attn_call, dict(dq=bf(T, HKV, D)), "dq must"), (_attn_call, dict(dk=bf(T, HQ, D)[:, ::2]), "dk must"), (_attn_call, dict(k=bf(T, HKV, D)), "k must"),
    (_attn_call, dict(ws=torch.zeros(8, dtype=torch.uint8).expand(2, 8)), "workspace must"),
]
GOOD = [
    (_rotary_call, {}), (_rotary_call, dict(v=None)), (_rotary_call, dict(q=bf(T, HQ + 2 * HKV, D)[:, 1:5])), (_rotary_call, dict(q_out=bf(T, 9, D)[:, :HQ])),
    (_rotary_call, dict(q=bf(2 * T, HQ, D)[::2])), (_pos_call, {}), (_pos_call, dict(first=None)), (_fwd_call, {}), (_fwd_call, dict(save="e4m3", bias=None)),
    (_fwd_call, dict(x=bf(T, 3, 96)[:, 1:], residual=bf(T, 2, 96), weight=torch.zeros(96), bias=torch.zeros(96))), (_bwd_call, {}),
    (_fwd_call, dict(save="int8", saved=_a8(T, 96), mean=torch.zeros(T), summed=bf(T, 96))), (_bwd_call, dict(dw=torch.zeros(96))),
    (_bwd_call, dict(x=_a8(T, 96), weight=None)), (_attn_call, {}), (_attn_call, dict(ws=torch.zeros(1 << 20, dtype=torch.uint8), dq=bf(T * HQ * D))),
]


@pytest.fixture
def on_cpu(monkeypatch):
    """The binding with CPU tensors taken for GPU ones and a library that succeeds and notes its calls."""
    calls = []
    monkeypatch.setattr(binding, "_host", None)
    monkeypatch.setattr(binding, "_load_host", lambda: binding._PythonHalf)

    class Lib:
        def __getattr__(self, name):
            return (lambda *a: 4096) if name.endswith("bytes") else lambda *a: calls.append((name, a)) or 0

    monkeypatch.setattr(binding, "load", Lib)
    monkeypatch.setattr(torch.Tensor, "is_cuda", property(lambda t: True))
    monkeypatch.setattr(torch.cuda, "device", lambda d: contextlib.nullcontext())
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: types.SimpleNamespace(cuda_stream=48))
    return calls


@pytest.mark.parametrize("make,other,why", BAD)
def test_the_binding_refuses_by_name(on_cpu, make, other, why):
    with pytest.raises(ValueError, match=why):
        make(**other)(binding)
    assert not on_cpu


@pytest.mark.parametrize("make,other", GOOD)
def test_the_binding_takes(on_cpu, make, other):
    make(**other)(binding)
    assert len(on_cpu) == 1
    stream = on_cpu[0][1][-1]
    assert getattr(stream, "value", stream) == 48
