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


@pytest.mark.parametrize("weights", [torch.bfloat16, None])
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("C", [128, 192, 640, 1001, 2056, 4096, 16384])
@pytest.mark.parametrize("eps,values", [(1e-30, [3.5e23, -1e25, 1e30, 3.0]), (1e-5, [1.5e34, -2e34, 1e30, 3.0]), (1e20, [1e-30, 0.0, 5.0, -7e-20])])
def test_constant_rows_from_8_bits(eps, values, C, fmt, weights):
    """mean * rstd is beyond fp32 in some; h - mean is what the rounding of the code times the scale leaves (2^-24 of h), so that n is up
    to 3e37.  dx holds rstd n sum(g n) / C: a row where that is beyond fp32 has no dx (n = 1e31, rstd = 1e15 make 1e76), and a column no
    dweight where the rows' |dy n| are; those may be anything, and everything beside them is held to the definition."""
    from paper_2605_08962_amd import binding
    x = torch.tensor(values, device="cuda").repeat(3)[:, None].expand(-1, C).to(torch.bfloat16).contiguous()
    w = (1 + 0.1 * B.bf(C, seed=2).float()).to(weights) if weights else None
    f = binding.varlen_attn_norm_fwd(x, w, eps=eps, save=fmt)
    dy = B.bf(*x.shape, seed=4)
    got = binding.varlen_attn_norm_bwd(dy, f.saved, f.mean, f.rstd, w)
    # code * scale is exact in 64 bits
    h = f.saved.codes.float().double() * f.saved.scales.double().repeat_interleave(B.BLOCK, dim=-1)[:, :C]
    (dx, dx_off), (dw, dw_off), (db, db_off) = B.norm_bwd(dy, h, f.mean, f.rstd, w, None)
    assert _finite(f.mean, f.rstd)
    n = (h - f.mean.double()[:, None]) * f.rstd.double()[:, None]
    g = dy.double() * (1 if w is None else w.double())
    fits = (f.rstd.double()[:, None] * n.abs() * (g * n).abs().mean(-1, keepdim=True)).amax(-1) < 2.0 ** 126
    assert fits[3::4].all()
    B.assert_within("dx", got[0][fits], dx[fits], dx_off[fits])
    if w is not None:
        fits = (dy.double() * n).abs().sum(0) < 2.0 ** 126
        assert int(fits.sum()) > C // 2
        B.assert_within("dw", got[1][fits], dw[fits], dw_off[fits])
        B.assert_within("db", got[2], db, db_off)


@pytest.mark.parametrize("fmt,value", [("int8", 1.984375 * 2.0 ** 78), ("int8", -1.984375 * 2.0 ** 96), ("e4m3", 1.75 * 2.0 ** 78),
                                       ("e4m3", -1.96875 * 2.0 ** 90)])
@pytest.mark.parametrize("C", [128, 200, 1001, 2056, 16384])
def test_constant_rows_that_8_bits_hold(C, fmt, value):
    """Numbers that the largest code times the scale is: h - mean and n are zero, while mean * rstd is beyond fp32, and the gradients are
    those of any constant row."""
    from paper_2605_08962_amd import binding
    x = torch.full((6, C), value, device="cuda").to(torch.bfloat16)
    w = 1 + 0.1 * B.bf(C, seed=2).float()
    f = binding.varlen_attn_norm_fwd(x, w, eps=1e-30, save=fmt)
    dy = B.bf(*x.shape, seed=4)
    got = binding.varlen_attn_norm_bwd(dy, f.saved, f.mean, f.rstd, w)
    (dx, dx_off), _, (db, db_off) = B.norm_bwd(dy, x, f.mean, f.rstd, w, None)
    assert _finite(f.mean, f.rstd, *got) and not got[1].any()
    B.assert_within("dx", got[0], dx, dx_off)
    B.assert_within("db", got[2], db, db_off)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("shift", [1e2, 1e4, 1e6])
def test_rows_far_off_zero_from_8_bits(shift, fmt):
    """To the bounds of the definition, which know nothing of mean * rstd."""
    from paper_2605_08962_amd import binding
    x = (B.bf(50, 1280, seed=5).float() + shift).to(torch.bfloat16)
    f = binding.varlen_attn_norm_fwd(x, eps=1e-5, save=fmt)
    dy = B.bf(50, 1280, seed=6)
    h = f.saved.codes.float().double() * f.saved.scales.double().repeat_interleave(B.BLOCK, dim=-1)[:, :1280]
    (dx, dx_off), _, _ = B.norm_bwd(dy, h, f.mean, f.rstd, None, None)
    B.assert_within("dx", binding.varlen_attn_norm_bwd(dy, f.saved, f.mean, f.rstd)[0], dx, dx_off)
