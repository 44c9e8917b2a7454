"""Layer norm's backward on the GPU where rows are far off zero or hardly vary, against its definition in 64 bits."""
import pytest
import torch

from tests import _block as B

pytestmark = pytest.mark.gpu


def _finite(*tensors):
    return all(bool(torch.isfinite(t).all()) for t in tensors if t is not None)


@pytest.mark.parametrize("weights", [torch.float32, None])
@pytest.mark.parametrize("shape", [(24, 192), (24, 1001), (24, 4096), (12, 2, 64)])
@pytest.mark.parametrize("eps", [0.0, 1e-30])
def test_rows_of_next_to_no_variance(shape, weights, eps):
    """Variances from 2^-124 to 2^-32, under gradients along the row itself: (g n)'s mean is as large as g."""
    from paper_2605_08962_amd import binding
    T, C = shape[0], shape[-1]
    far = (2.0 ** torch.linspace(-62, -16, T, device="cuda").round()).view(T, *[1] * (len(shape) - 1))
    x = (B.bf(*shape, seed=1).float() * far).to(torch.bfloat16)
    w = (1 + 0.1 * B.bf(C, seed=2).float()) if weights else None
    f = binding.varlen_attn_norm_fwd(x, w, eps=eps)
    dy = (64 * B.bf(*shape, seed=1).float() + B.bf(*shape, seed=3).float()).to(torch.bfloat16)
    got = binding.varlen_attn_norm_bwd(dy, x, f.mean, f.rstd, w)
    (dx, dx_off), (dw, dw_off), (db, db_off) = B.norm_bwd(dy, x, f.mean, f.rstd, w, None)
    assert _finite(f.mean, f.rstd, dx, *got)
    B.assert_within("dx", got[0], dx, dx_off)
    if w is not None:
        B.assert_within("dw", got[1], dw, dw_off)
        B.assert_within("db", got[2], db, db_off)


@pytest.mark.parametrize("weights", [torch.float32, None])
@pytest.mark.parametrize("shape", [(7, 8), (7, 40), (7, 128), (7, 200), (7, 1001), (7, 1537), (7, 2056), (7, 4104), (7, 8200), (5, 3, 80), (5, 3, 30)])
def test_constant_rows_beyond_the_range_of_mean_times_rstd(shape, weights):
    """h - mean is zero in every channel, and what lanes without channels hold in its place does not count."""
    from paper_2605_08962_amd import binding
    x = torch.full(shape, 3.5e25, device="cuda").to(torch.bfloat16)
    x[1], x[2], x[3] = -1e30, 1.0, 0.0
    w = (1 + 0.1 * B.bf(shape[-1], seed=2).float()) if weights else None
    f = binding.varlen_attn_norm_fwd(x, w, eps=1e-30)
    dy = B.bf(*shape, seed=4)
    got = binding.varlen_attn_norm_bwd(dy, x, f.mean, f.rstd, w)
    (dx, dx_off), _, (db, db_off) = B.norm_bwd(dy, x, f.mean, f.rstd, w, None)
    assert _finite(f.mean, f.rstd, *got)
    B.assert_within("dx", got[0], dx, dx_off)
    if w is not None:
        assert not got[1].any()
        B.assert_within("db", got[2], db, db_off)
