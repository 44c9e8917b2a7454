"""Layer norm on the GPU, forward and backward, against its definition in 64 bits."""
import pytest
import torch

from tests import _block as B

pytestmark = pytest.mark.gpu
EPS = 1e-5


def _inputs(shape, weights, seed=1, shift=0.5):
    C = shape[-1]
    gen = torch.Generator().manual_seed(seed)
    size = torch.exp(0.5 * torch.randn(C, generator=gen))
    x = ((torch.randn(shape, generator=gen) + shift) * size).to(torch.bfloat16).cuda()
    w = (1 + 0.3 * torch.randn(C, generator=gen)).to(weights).cuda() if weights else None
    b = (0.2 * torch.randn(C, generator=gen)).to(weights).cuda() if weights else None
    return x, w, b, B.bf(*shape, seed=seed + 1)


def _check_forward(f, h, w, b):
    (y, y_off), (mean, mean_off), (rstd, rstd_off) = B.norm(h, w, b, EPS)
    B.assert_within("mean", f.mean, mean, mean_off)
    B.assert_within("rstd", f.rstd, rstd, rstd_off)
    B.assert_within("y", f.out, y, y_off)


def _check_backward(got, dy, h, f, w, dsummed=None):
    (dx, dx_off), (dw, dw_off), (db, db_off) = B.norm_bwd(dy, h, f.mean, f.rstd, w, dsummed)
    B.assert_within("dx", got[0], dx, dx_off)
    if w is None:
        assert got[1] is None and got[2] is None
    else:
        assert got[1].dtype == got[2].dtype == torch.float32
        B.assert_within("dw", got[1], dw, dw_off)
        B.assert_within("db", got[2], db, db_off)


# every number of threads a row, full and with a rest; one row and many; heads of tokens
SHAPES = [(1, 1), (1, 8), (3, 40), (700, 64), (2, 65), (513, 96), (5, 128), (1000, 130), (33, 256), (7, 257), (40, 511), (129, 512),
          (9, 1000), (2500, 1024), (11, 1280), (3, 1536), (10, 2000), (4, 2048), (5, 2056), (3, 4096), (130, 4104), (2, 8192),
          (2, 8200), (3, 16384), (1, 16383), (41, 3, 64), (1030, 8, 128), (6, 2, 80), (5, 7, 30)]


@pytest.mark.parametrize("weights", [torch.bfloat16, torch.float32, None])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward_and_backward(shape, weights):
    from paper_2605_08962_amd import binding
    print(shape, weights, flush=True)
    x, w, b, dy = _inputs(shape, weights)
    f = binding.varlen_attn_norm_fwd(x, w, b, eps=EPS)
    assert f.summed is None and f.saved is None
    _check_forward(f, x, w, b)
    _check_backward(binding.varlen_attn_norm_bwd(dy, x, f.mean, f.rstd, w), dy, x, f, w)


@pytest.mark.parametrize("save", [None, "int8", "e4m3"])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("shape", [(1, 3), (257, 64), (31, 200), (600, 1280), (19, 1001), (9, 4096), (4, 8200), (65, 3, 80), (70, 4, 128), (33, 2, 136)])
def test_residual_and_checkpoint(shape, residual, save):
    from paper_2605_08962_amd import binding
    print(shape, residual, save, flush=True)
    x, w, b, dy = _inputs(shape, torch.bfloat16, seed=5)
    r = B.bf(*shape, seed=8) if residual else None
    f = binding.varlen_attn_norm_fwd(x, w, b, eps=EPS, residual=r, save=save)
    h = (x.float() + r.float()).to(torch.bfloat16) if residual else x
    assert (f.summed is None) == (not residual) and (f.saved is None) == (save is None)
    if residual:
        assert torch.equal(f.summed, h)
    _check_forward(f, h, w, b)
    source, seen = h, h
    if save:
        alone = binding.varlen_attn_act8_pack([h], save)[0]
        assert torch.equal(alone.codes.view(torch.int8), f.saved.codes.view(torch.int8)) and torch.equal(alone.scales, f.saved.scales)
        source, seen = f.saved, B.act8_values(*f.saved)
    ds = B.bf(*shape, seed=9) if residual else None
    _check_backward(binding.varlen_attn_norm_bwd(dy, source, f.mean, f.rstd, w, dsummed=ds), dy, seen, f, w, ds)


@pytest.mark.parametrize("shape,before,after", [((50, 1024), 8, 8), ((50, 1024), 3, 6), ((300, 4, 64), 16, 128), ((77, 2, 80), 1, 0)])
def test_parts_of_wider_tensors(shape, before, after):
    """x, dy and dx with a stride between tokens, also one that puts rows off 16 bytes: the same bits, and nothing beside them written."""
    from paper_2605_08962_amd import binding
    x, w, b, dy = _inputs(shape, torch.float32, seed=3)
    xs, dys = B.wider(x, before, after)[0], B.wider(dy, before, after)[0]
    f, g = (binding.varlen_attn_norm_fwd(t, w, b, eps=EPS) for t in (x, xs))
    for a, c in zip(f[:3], g[:3]):
        assert torch.equal(a, c)
    place, whole = B.wider(torch.zeros_like(x), before, after)
    want = binding.varlen_attn_norm_bwd(dy, x, f.mean, f.rstd, w)
    got = binding.varlen_attn_norm_bwd(dys, xs, f.mean, f.rstd, w, dx=place)
    assert got[0] is place and all(torch.equal(a, c) for a, c in zip(got, want))
    n = whole.shape[1]
    assert torch.isnan(whole[:, :before]).all() and torch.isnan(whole[:, n - after:]).all()


def test_backward_is_the_gradient():
    """Of sum(y * dy), against central differences of the definition in 64 bits: x, weight and bias."""
    from paper_2605_08962_amd import binding
    C, T = 12, 3
    x, w, b, dy = _inputs((T, C), torch.float32, seed=7)
    f = binding.varlen_attn_norm_fwd(x, w, b, eps=EPS)
    dx, dw, db = binding.varlen_attn_norm_bwd(dy, x, f.mean, f.rstd, w)
    leaves = [t.double() for t in (x, w, b)]
    loss = lambda x, w, b: (B.norm(x, w, b, EPS)[0][0] * dy.double()).sum()  # noqa: E731
    h = 1e-5  # second-order error h^2 f'''/6: below 1e-8 for these sizes; 64-bit roundings 1e-11
    for i, (leaf, got) in enumerate(zip(leaves, (dx, dw, db))):
        for j in range(leaf.numel()):
            moved = []
            for sign in (1, -1):
                at = [t.clone() for t in leaves]
                at[i].view(-1)[j] += sign * h
                moved.append(float(loss(*at)))
            diff = (moved[0] - moved[1]) / (2 * h)
            # dx is rounded to bf16; fp32 sums of a dozen terms below 30 in the rest
            assert abs(float(got.view(-1)[j]) - diff) <= (B.HALF16 * abs(diff) if i == 0 else 0) + 1e-4, (i, j)


def test_constant_and_far_rows():
    """A row of one value has variance 0 (eps alone counts); a row far off zero keeps what bf16 holds of it."""
    from paper_2605_08962_amd import binding
    x = torch.full((4, 640), 3.0, dtype=torch.bfloat16, device="cuda")
    x[1] = 0
    x[2] = 1024 + 8 * B.bf(640, seed=2)
    x[3] = 1e30
    f = binding.varlen_attn_norm_fwd(x, eps=EPS)
    _check_forward(f, x, None, None)
    assert (f.out[:2] == 0).all() and torch.allclose(f.rstd[:2], torch.full((2,), EPS ** -0.5, device="cuda"), rtol=1e-6)
    dy = B.bf(4, 640, seed=4)
    _check_backward(binding.varlen_attn_norm_bwd(dy, x, f.mean, f.rstd), dy, x, f, None)


def test_rows_that_are_no_numbers_stay_by_themselves():
    from paper_2605_08962_amd import binding
    x, w, b, dy = _inputs((40, 96), torch.bfloat16, seed=6)
    clean = binding.varlen_attn_norm_fwd(x, w, b)
    y = x.clone()
    y[3, 7], y[20, 0] = float("nan"), float("inf")
    f = binding.varlen_attn_norm_fwd(y, w, b)
    bad = torch.zeros(40, dtype=torch.bool, device="cuda")
    bad[[3, 20]] = True
    assert torch.isnan(f.out[bad]).all() and torch.equal(f.out[~bad], clean.out[~bad])
    assert torch.isnan(f.mean[3]) and torch.isposinf(f.mean[20]) and torch.isnan(f.rstd[bad]).all()
    dx = binding.varlen_attn_norm_bwd(dy, y, f.mean, f.rstd, w)[0]
    want = binding.varlen_attn_norm_bwd(dy, x, clean.mean, clean.rstd, w)[0]
    assert torch.isnan(dx[bad]).all() and torch.equal(dx[~bad], want[~bad])


def test_no_rows():
    """The gradients of weight and bias are sums of nothing."""
    from paper_2605_08962_amd import binding
    x = torch.empty((0, 1280), dtype=torch.bfloat16, device="cuda")
    w = torch.ones(1280, device="cuda")
    f = binding.varlen_attn_norm_fwd(x, w, w, residual=x, save="int8")
    assert f.out.shape == x.shape and f.mean.shape == (0,)
    dx, dw, db = binding.varlen_attn_norm_bwd(x, f.saved, f.mean, f.rstd, w)
    assert dx.shape == x.shape and not dw.any() and not db.any()


def test_the_same_call_gives_the_same_bits():
    from paper_2605_08962_amd import binding
    x, w, b, dy = _inputs((5000, 768), torch.bfloat16)
    f = binding.varlen_attn_norm_fwd(x, w, b)
    first = binding.varlen_attn_norm_bwd(dy, x, f.mean, f.rstd, w)
    for _ in range(3):
        assert all(torch.equal(a, c) for a, c in zip(binding.varlen_attn_norm_bwd(dy, x, f.mean, f.rstd, w), first))


def test_results_go_where_the_caller_says():
    from paper_2605_08962_amd import binding
    x, w, b, dy = _inputs((70, 200), torch.float32, seed=9)
    f = binding.varlen_attn_norm_fwd(x, w, b, residual=dy, save="int8")
    mine = binding.NormForward(*(binding.Act8(*map(torch.zeros_like, t)) if isinstance(t, tuple) else torch.zeros_like(t) for t in f))
    got = binding.varlen_attn_norm_fwd(x, w, b, residual=dy, save="int8", **mine._asdict())
    assert all(a is m for a, m in zip(got, mine))
    for a, m in zip((*f[:4], *f.saved), (*mine[:4], *mine.saved)):
        assert torch.equal(a, m)
    want = binding.varlen_attn_norm_bwd(dy, f.saved, f.mean, f.rstd, w)
    outs = [torch.zeros_like(t) for t in want]
    ws = torch.empty(binding.norm_bwd_workspace_bytes(binding.NormParams(70, 1, 200, 1, 0, 0.0, 200, 200, 200)), dtype=torch.uint8, device="cuda")
    got = binding.varlen_attn_norm_bwd(dy, f.saved, f.mean, f.rstd, w, dx=outs[0], dweight=outs[1], dbias=outs[2], workspace=ws)
    assert all(a is m and torch.equal(a, t) for a, m, t in zip(got, outs, want))
    with pytest.raises(binding.VarlenAttnError, match="workspace too small"):
        binding.varlen_attn_norm_bwd(dy, f.saved, f.mean, f.rstd, w, workspace=ws[:-256])


@pytest.mark.parametrize("eps", [0.0, 1e-30, 1e-5, 1e20])
def test_statistics_at_the_ends_of_the_range(eps):
    """Variances from 2^-120 to 2^110, with and without an eps beside them."""
    from paper_2605_08962_amd import binding
    x = B.bf(60, 192, seed=4) * (2.0 ** torch.arange(-60, 60, 2, device="cuda"))[:, None]
    x = x.to(torch.bfloat16)
    f = binding.varlen_attn_norm_fwd(x, eps=eps)
    (y, y_off), (mean, mean_off), (rstd, rstd_off) = B.norm(x, None, None, float(torch.tensor(eps)))
    B.assert_within("mean", f.mean, mean, mean_off)
    B.assert_within("rstd", f.rstd, rstd, rstd_off)
    B.assert_within("y", f.out, y, y_off + 1e-37)  # (a bf16 below 2^-126 has fewer bits)
