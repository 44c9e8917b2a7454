"""Rotary positions on the GPU at far angles, to what the header promises of them."""
import pytest
import torch

from tests import _block as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("P,d", [(32, 64), (20, 80), (3, 7)])
@pytest.mark.parametrize("far", [31, 28, 24])
def test_angles_up_to_two_to_the_31(far, P, d, interleaved):
    """Positions of either sign up to 2^far at frequencies up to 2^(31 - far), whose 24 bits are all in use: angles right to 2^-20, and the
    reference's own, of products rounded to 53 bits, to 2^-22; the rest of 2^-19 is for the rotation in 32 bits."""
    from paper_2605_08962_amd import binding
    T = 500
    gen = torch.Generator().manual_seed(far)
    pos = torch.randint(-2 ** far, 2 ** far, (2, T), generator=gen)
    pos[:, 0], pos[:, 1] = 2 ** far - 1, -2 ** far
    freq = (1 - 0.5 * torch.rand(P, generator=gen)) * 2.0 ** (31 - far)
    axis = (torch.arange(P) % 2).int()
    turn = pos.int().cuda(), freq.cuda(), axis.cuda()
    assert float(pos.abs().max() * freq.max()) <= 2 ** 31
    q, k = B.bf(T, 2, d, seed=1), B.bf(T, 1, d, seed=2)
    for inverse, f in ((False, binding.varlen_attn_rotary_fwd), (True, binding.varlen_attn_rotary_bwd)):
        got = f(q, k, *turn, interleaved=interleaved)
        B.assert_within("q", got[0], *B.rotary(q, *turn, interleaved, inverse))
        B.assert_within("k", got[1], *B.rotary(k, *turn, interleaved, inverse))


@pytest.mark.parametrize("power", [3, 8, 16])
def test_angles_beyond(power):
    """Powers of two as frequencies, so that the reference's angles are exact: right to 2^-51 of themselves."""
    from paper_2605_08962_amd import binding
    T, P = 500, 32
    gen = torch.Generator().manual_seed(power)
    pos = torch.randint(-2 ** 31, 2 ** 31, (1, T), generator=gen).int().cuda()
    freq, axis = torch.full((P,), 2.0 ** power, device="cuda"), torch.zeros(P, dtype=torch.int32, device="cuda")
    q = B.bf(T, 1, 2 * P, seed=3)
    got = binding.varlen_attn_rotary_fwd(q, q, pos, freq, axis)[0]
    want, off = B.rotary(q, pos, freq, axis, False)
    pairs = q.double().abs().unflatten(-1, (2, P)).sum(-2).repeat(1, 1, 2)
    B.assert_within("q", got, want, off + 2.0 ** (31 + power - 51) * pairs)
