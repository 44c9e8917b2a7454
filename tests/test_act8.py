"""Activations in 8 bits on the GPU: codes and scales to the bit, what they come back as, and attention's backward pass from them."""
import pytest
import torch

from paper_2605_08962_amd import workloads as W
from tests import _block as B
from tests._util import upload

pytestmark = pytest.mark.gpu
FORMATS = pytest.mark.parametrize("fmt", ["int8", "e4m3"])


def _check(x, packed, fmt):
    codes, scales = B.act8(x, fmt)
    assert packed.codes.dtype == B.CODES[fmt] and packed.codes.shape == x.shape
    good = torch.isfinite(scales)
    assert torch.equal(packed.scales.cpu()[good], scales[good]) and torch.isnan(packed.scales.cpu()[~good]).all()
    here = good.repeat_interleave(B.BLOCK, dim=-1)[..., :x.shape[-1]]
    bits = lambda c: c.cpu().view(torch.int8)  # noqa: E731
    assert torch.equal(bits(packed.codes)[here], bits(codes)[here])


@FORMATS
@pytest.mark.parametrize("shape", [(1, 1), (3, 7), (5, 64), (2, 128), (9, 129), (4, 1280), (7, 1001), (1, 16384), (246, 2, 64),
                                   (31, 3, 80), (65, 4, 96), (1025, 8, 128), (10, 2, 200), (3, 5, 11)])
def test_there_and_back(shape, fmt):
    from paper_2605_08962_amd import binding
    print(shape, fmt, flush=True)
    x = B.bf(*shape, seed=3, scale=2.0)
    x.view(-1)[::17] *= 30
    packed = binding.varlen_attn_act8_pack([x], fmt)[0]
    _check(x, packed, fmt)
    back = binding.varlen_attn_act8_unpack([packed])[0]
    want = B.act8_values(packed.codes.cpu(), packed.scales.cpu())
    assert torch.equal(back.cpu(), want.to(torch.bfloat16))
    # within half a step of the format, and half a step of bf16; 2 roundings of the product in 32 bits on the way to the code
    s = packed.scales.cpu().double().repeat_interleave(B.BLOCK, dim=-1)[..., :shape[-1]]
    a = x.cpu().double().abs()
    step = s / 2 if fmt == "int8" else torch.maximum(a * 2.0 ** -4, s * 2.0 ** -10)
    B.assert_within("value", back.cpu(), x.cpu(), step * (1 + 2.0 ** -20) + (a + step) * B.HALF16)


@FORMATS
def test_several_tensors_of_different_shapes_and_strides(fmt):
    """More than one launch takes, empty ones among them, parts of wider tensors, rows off 16 bytes."""
    from paper_2605_08962_amd import binding
    xs = [B.bf(t, *rest, seed=i) for i, (t, *rest) in enumerate([(33, 2, 64), (0, 64), (100, 1280), (7, 3, 80), (5, 9), (1, 1, 128), (300, 96),
                                                             (2, 5, 24), (64, 2, 64), (3, 640)])]
    parts = [B.wider(x, *((8, 16) if i % 2 else (3, 2)))[0] if x.numel() else x for i, x in enumerate(xs)]
    packed = binding.varlen_attn_act8_pack(parts, fmt)
    for x, p in zip(xs, packed):
        _check(x, p, fmt)
    back = binding.varlen_attn_act8_unpack(packed)
    places = [B.wider(torch.zeros_like(x), *((8, 16) if i % 2 else (3, 2))) if x.numel() else (x, x) for i, x in enumerate(xs)]
    got = binding.varlen_attn_act8_unpack(packed, out=[p for p, _ in places])
    for i, (b, g, (part, whole), x) in enumerate(zip(back, got, places, xs)):
        assert g is part and torch.equal(part, b)
        if x.numel():
            before, after = (8, 16) if i % 2 else (3, 2)
            assert torch.isnan(whole[:, :before]).all() and torch.isnan(whole[:, -after:]).all()
    mine = [binding.Act8(torch.empty_like(p.codes), torch.empty_like(p.scales)) for p in packed]
    assert all(a is b for a, b in zip(binding.varlen_attn_act8_pack(parts, fmt, out=mine), mine))
    for a, b in zip(mine, packed):
        assert torch.equal(a.codes.view(torch.int8), b.codes.view(torch.int8)) and torch.equal(a.scales, b.scales)


@FORMATS
def test_extreme_blocks(fmt):
    """Zeros, the smallest and largest numbers, and blocks with an infinity or a NaN, which come back as NaN and leave their neighbours
    alone."""
    from paper_2605_08962_amd import binding
    x = B.bf(8, 3 * 128, seed=9)
    x[0, :128] = 0
    x[0, 128:256] = -0.0
    x[1] = x[1] * 2.0 ** -130
    x[2] = 2.0 ** -133
    x[3] = torch.finfo(torch.bfloat16).max
    x[4, 5], x[5, 200], x[6, 383] = float("inf"), float("-inf"), float("nan")
    x[7, :128] = 1.0
    packed = binding.varlen_attn_act8_pack([x], fmt)[0]
    _check(x, packed, fmt)
    back = binding.varlen_attn_act8_unpack([packed])[0]
    nan = torch.zeros(8, 3, dtype=torch.bool, device="cuda")
    nan[4, 0] = nan[5, 1] = nan[6, 2] = True
    assert torch.equal(torch.isnan(back).view(8, 3, 128).all(-1), nan) and torch.equal(torch.isnan(back).view(8, 3, 128).any(-1), nan)
    assert (back[0, :256] == 0).all() and torch.equal(back[7, :128], x[7, :128])
    # the floor of the scale: values below it are off by less than half a step of 2^-126
    assert ((back[1:3].double() - x[1:3].double()).abs() <= 2.0 ** -127).all()


@FORMATS
@pytest.mark.parametrize("D,hq,hkv,causal,lengths", [
    (64, 2, 2, False, [16, 37, 64, 129]), (80, 3, 3, True, [1, 300, 0, 65]), (96, 4, 1, False, [513]), (128, 8, 2, True, [700, 1, 129]),
    (128, 2, 2, True, [2500])])
def test_attention_backward_from_the_checkpoint(D, hq, hkv, causal, lengths, fmt):
    """The very gradients of varlen_attn_bwd on the unpacked tensors."""
    from paper_2605_08962_amd import binding
    w = W.make_custom(lengths, hq, hkv, D, causal, seed=40 + D, with_dout=True)
    print(lengths, D, hq, hkv, causal, fmt, flush=True)
    d = upload(w)
    o, lse = binding.varlen_attn_fwd(d["q"], d["k"], d["v"], d["cu"], causal, w.scale)
    kept = binding.varlen_attn_act8_pack([d["q"], d["k"], d["v"], o], fmt)
    hint = {"max_seqlen": max(lengths)}
    back = binding.varlen_attn_act8_unpack(kept)
    want = binding.varlen_attn_bwd(d["dout"], *back, lse, d["cu"], causal, w.scale, kv_splits=1, **hint)
    got = binding.varlen_attn_bwd_act8(d["dout"], *kept, lse, d["cu"], causal, w.scale, kv_splits=1, **hint)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    mine = [torch.empty_like(t) for t in want]
    p = binding.make_params(w.total_tokens, w.num_seqs, hq, hkv, D, causal, w.scale, 1, max(lengths))
    ws = torch.empty(binding.bwd_act8_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    binding.varlen_attn_bwd_act8(d["dout"], *kept, lse, d["cu"], causal, w.scale, dq=mine[0], dk=mine[1], dv=mine[2], workspace=ws,
                                 kv_splits=1, **hint)
    assert all(torch.equal(a, b) for a, b in zip(mine, want))
    with pytest.raises(binding.VarlenAttnError, match="workspace too small"):
        binding.varlen_attn_bwd_act8(d["dout"], *kept, lse, d["cu"], causal, w.scale, workspace=ws[:-512], kv_splits=1, **hint)
    # with chunks chosen by the call, and a workspace that holds none of them
    auto = binding.varlen_attn_bwd_act8(d["dout"], *kept, lse, d["cu"], causal, w.scale, **hint)
    least = binding.varlen_attn_bwd_act8(d["dout"], *kept, lse, d["cu"], causal, w.scale, workspace=ws, **hint)
    for a, b, c in zip(auto, want, least):
        assert float((a.double() - b.double()).norm()) <= 5e-3 * float(b.double().norm()) and torch.equal(b, c)


def test_attention_backward_from_an_empty_checkpoint():
    from paper_2605_08962_amd import binding
    q = torch.empty((0, 2, 64), dtype=torch.bfloat16, device="cuda")
    kept = binding.varlen_attn_act8_pack([q] * 4)
    cu = torch.zeros(1, dtype=torch.int32, device="cuda")
    grads = binding.varlen_attn_bwd_act8(q, *kept, torch.empty((2, 0), device="cuda"), cu, True, 0.1)
    assert [g.shape for g in grads] == [q.shape] * 3
