"""Activations in 8 bits at the ends of bf16's range on the GPU: every finite block comes back as code * scale, whatever it holds."""
import pytest
import torch

from tests import _block as B

pytestmark = pytest.mark.gpu
MOST, NEXT = 0x7f7f, 0x7f7e  # bf16's two largest numbers, as bits
LEAST = 0x0001


def _bits(*values):
    return torch.tensor(values, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)


def _rows(C):
    """Rows of C channels whose blocks hold the largest numbers of either sign, alone and beside ordinary, small and no values."""
    x = B.bf(10, C, seed=C, device="cpu")
    top, low, nxt = _bits(MOST, MOST | 0x8000, NEXT)
    x[0], x[1], x[2], x[3] = top, low, nxt, -nxt
    x[4, ::2], x[4, 1::2] = top, low
    x[5, C // 2] = low                                       # the usual value of a masked place
    x[6] = 0
    x[6, C - 1] = nxt
    x[7] = x[7] * 5e37
    x[7, 0], x[7, C // 3] = top, 0
    x[8], x[8, 1::3], x[8, 0] = _bits(LEAST)[0], -0.0, top
    x[9] = 2.0 ** 127                                        # just below
    return x


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("shape", [(384,), (1001,), (130,), (64,), (2, 64), (3, 80), (5, 30)])
def test_the_largest_numbers_come_back(shape, fmt):
    from paper_2605_08962_amd import binding
    x = _rows(torch.Size(shape).numel()).view(10, *shape)
    packed = binding.varlen_attn_act8_pack([x.cuda()], fmt)[0]
    codes, scales = B.act8(x, fmt)
    assert torch.equal(packed.scales.cpu(), scales) and torch.equal(packed.codes.cpu().view(torch.int8), codes.view(torch.int8))
    want = B.act8_values(codes, scales).to(torch.bfloat16)
    assert torch.isfinite(want).all()
    back = binding.varlen_attn_act8_unpack([packed])[0].cpu()
    assert torch.equal(back, want)
    # half a step of the format, and of bf16; 2 roundings of the product in 32 bits on the way to the code
    s = scales.double().repeat_interleave(B.BLOCK, dim=-1)[..., :shape[-1]]
    a = x.double().abs()
    step = s / 2 if fmt == "int8" else torch.maximum(a * 2.0 ** -4, s * 2.0 ** -10)
    B.assert_within("value", back, x, step * (1 + 2.0 ** -20) + (a + step) * B.HALF16)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_every_code_of_a_block_at_the_top_of_the_range(fmt):
    """All codes beside the largest scale, in every place of a thread's eight."""
    from paper_2605_08962_amd import binding
    n = torch.arange(256, dtype=torch.int32).to(torch.uint8)
    codes = torch.stack([n.roll(i) for i in range(8)]).view(torch.int8)
    codes[(codes == -128) if fmt == "int8" else ((codes & 0x7f) == 0x7f)] = 0  # (packing makes none; NaN)
    codes = codes.view(B.CODES[fmt])
    top = float(_bits(MOST)[0].float())
    scales = torch.full((8, 2), top, dtype=torch.float32) * torch.tensor(1.0 / B.MOST[fmt], dtype=torch.float32)
    back = binding.varlen_attn_act8_unpack([binding.Act8(codes.cuda(), scales.cuda())])[0].cpu()
    want = B.act8_values(codes, scales).to(torch.bfloat16)
    assert torch.isfinite(want).all() and torch.equal(back, want)
