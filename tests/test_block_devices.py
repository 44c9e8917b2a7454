"""Everything that a call of the operators around attention is given is on one GPU, or the call is refused by the name of what is not:
on the CPU, where the device `meta` stands for another GPU."""
import pytest
import torch

from tests import test_block_refusals as R
from tests.test_block_marshalling import both, module  # noqa: F401
from tests.test_block_refusals import _a8, bf, i32, on_cpu  # noqa: F401
from paper_2605_08962_amd import binding

T, HQ, HKV, D, C = R.T, R.HQ, R.HKV, R.D, 96


def _scratch(n=1 << 16):
    return torch.zeros(n, dtype=torch.uint8)


# call -> (every tensor it can be given by name, the call made with them)
def _positions(a):
    return binding.varlen_attn_rotary_positions(a["cu_rows"], a["grids"], T, first=a["first"], out=a["out"])


def _rotary(a):
    return binding.varlen_attn_rotary_fwd(a["q"], a["k"], a["positions"], a["inv_freq"], a["pair_axis"], v=a["v"], q_out=a["q_out"],
                                          k_out=a["k_out"], v_out=a["v_out"])


def _norm_fwd(a):
    return binding.varlen_attn_norm_fwd(a["x"], a["weight"], a["bias"], residual=a["residual"], save="int8", out=a["out"], mean=a["mean"],
                                        rstd=a["rstd"], summed=a["summed"], saved=a["saved"])


def _norm_bwd(a):
    return binding.varlen_attn_norm_bwd(a["dy"], a["x"], a["mean"], a["rstd"], a["weight"], dsummed=a["dsummed"], dx=a["dx"],
                                        dweight=a["dweight"], dbias=a["dbias"], workspace=a["workspace"])


def _attn(a):
    return binding.varlen_attn_bwd_act8(a["dout"], a["q"], a["k"], a["v"], a["out"], a["lse"], a["cu_seqlens"], True, 0.1, dq=a["dq"],
                                        dk=a["dk"], dv=a["dv"], workspace=a["workspace"])


def _pack(a):
    return binding.varlen_attn_act8_pack([a["first"], a["tensors[1]"]], out=[_a8(T, C), a["out[1]"]])


def _unpack(a):
    return binding.varlen_attn_act8_unpack([a["first"], a["packed[1]"]], out=[bf(T, C), a["out[1]"]])


CALLS = {
    _positions: lambda: dict(cu_rows=i32(3), grids=i32(2, 3), first=i32(2), out=i32(3, T)),
    _rotary: lambda: dict(q=bf(T, HQ, D), k=bf(T, HKV, D), v=bf(T, HKV, D), positions=i32(3, T), inv_freq=torch.zeros(R.P), pair_axis=i32(R.P),
                          q_out=bf(T, HQ, D), k_out=bf(T, HKV, D), v_out=bf(T, HKV, D)),
    _norm_fwd: lambda: dict(x=bf(T, C), weight=bf(C), bias=bf(C), residual=bf(T, C), out=bf(T, C), mean=torch.zeros(T), rstd=torch.zeros(T),
                            summed=bf(T, C), saved=_a8(T, C)),
    _norm_bwd: lambda: dict(dy=bf(T, C), x=bf(T, C), mean=torch.zeros(T), rstd=torch.zeros(T), weight=bf(C), dsummed=bf(T, C), dx=bf(T, C),
                            dweight=torch.zeros(C), dbias=torch.zeros(C), workspace=_scratch()),
    _attn: lambda: dict(dout=bf(T, HQ, D), q=_a8(T, HQ, D), k=_a8(T, HKV, D), v=_a8(T, HKV, D), out=_a8(T, HQ, D), lse=torch.zeros(HQ, T),
                        cu_seqlens=i32(2), dq=bf(T, HQ, D), dk=bf(T, HKV, D), dv=bf(T, HKV, D), workspace=_scratch()),
    _pack: lambda: {"first": bf(T, C), "tensors[1]": bf(T, C), "out[1]": _a8(T, C)},
    _unpack: lambda: {"first": _a8(T, C), "packed[1]": _a8(T, C), "out[1]": bf(T, C)},
}
ONES = [(call, name) for call, make in CALLS.items() for name in list(make())[1:]]


def _elsewhere(t):
    return binding.Act8(t[0].to("meta"), t[1].to("meta")) if isinstance(t, binding.Act8) else t.to("meta")


@pytest.mark.parametrize("native", [False, True])
@pytest.mark.parametrize("call,name", ONES)
def test_a_tensor_on_another_gpu_is_named(both, call, name, native):  # noqa: F811
    both(native)
    given = CALLS[call]()
    call(given)
    assert len(both.calls) == 1
    both(native)
    given[name] = _elsewhere(given[name])
    with pytest.raises(ValueError, match=name.replace("[", r"\[").replace("]", r"\]") + r" must be on"):
        call(given)
    assert not both.calls


@pytest.mark.parametrize("call,names", [(_attn, ("dq", "dk", "dv", "workspace")), (_norm_bwd, ("workspace",))])
def test_buffers_in_pinned_host_memory_are_taken(both, monkeypatch, call, names):  # noqa: F811
    both(False)
    given = CALLS[call]()
    host = [given[n] for n in names]
    monkeypatch.setattr(torch.Tensor, "is_cuda", property(lambda t: not any(t is h for h in host)))
    monkeypatch.setattr(torch.Tensor, "is_pinned", lambda t: any(t is h for h in host))
    call(given)
    assert len(both.calls) == 1
