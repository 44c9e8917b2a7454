"""Plain 64-bit forms of the operators around attention, for their tests; on whatever device the tensors are."""
import torch

U32 = 2.0 ** -24   # half a step of fp32, relative
HALF16 = 2.0 ** -8  # of bf16
BLOCK = 128
MOST = {"int8": 127.0, "e4m3": 448.0}
CODES = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}


def bf(*shape, seed=0, scale=1.0, shift=0.0, device="cuda"):
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=gen) * scale + shift).to(torch.bfloat16).to(device)


def wider(x, before=8, after=16):
    """x as a part of a wider tensor (the same values, the same shape, a stride between tokens)."""
    width = x[0].numel()
    whole = torch.full((x.shape[0], before + width + after), float("nan"), dtype=x.dtype, device=x.device)
    part = whole[:, before:before + width].unflatten(1, x.shape[1:])
    part.copy_(x)
    return part, whole


def positions(cu, grids, first, merge, total):
    """Token by token."""
    out = torch.zeros((3, total), dtype=torch.int64)
    for s, (t, h, w) in enumerate(grids):
        lo, hi, f = cu[s], cu[s + 1], first[s] if first is not None else 0
        for i in range(hi - lo):
            if h < 1 or w < 1:
                p = (i, i, i)
            else:
                r, m = i % (h * w), merge
                b, e = r // (m * m), r % (m * m)
                p = (i // (h * w), b // (w // m) * m + e // m, b % (w // m) * m + e % m)
            out[:, lo + i] = torch.tensor(p) + f
    return out.to(torch.int32)


def rotary(x, pos, inv_freq, pair_axis, interleaved, inverse=False):
    """(result in 64 bits, what may be off: half a step of bf16 and of the 32-bit rotation; angles are right to 2^-20)."""
    x, n = x.double(), inv_freq.numel()
    phi = (pos.double()[pair_axis.long()].T * inv_freq.double())[:, None]
    c, s = torch.cos(phi), torch.sin(phi) * (-1 if inverse else 1)
    y, size = x.clone(), torch.zeros_like(x)
    i0, i1 = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    a, b = x[..., i0], x[..., i1]
    y[..., i0], y[..., i1] = a * c - b * s, b * c + a * s
    size[..., i0] = size[..., i1] = a.abs() + b.abs()
    return y, HALF16 * y.abs() + 2.0 ** -19 * size


def norm(h, weight, bias, eps):
    """y, mean, rstd of rows h in 64 bits and what each may be off: sums of at most 50 additions one after the other in fp32 (a
    thread's 32 or fewer, the lanes', the waves'), and a rounding to bf16."""
    h = h.double()
    mean = h.mean(-1)
    d = h - mean[..., None]
    rstd = ((d * d).mean(-1) + eps) ** -0.5
    n = d * rstd[..., None]
    w = torch.ones_like(h[0]) if weight is None else weight.double()
    b = torch.zeros_like(w) if bias is None else bias.double()
    most = h.abs().amax(-1)
    y = n * w + b
    off = 64 * U32
    rel = off * (1 + most * rstd)
    return (y, HALF16 * y.abs() + w.abs() * (n.abs() * rel[..., None] + off * (most * rstd)[..., None]) + 4 * U32 * b.abs()), \
        (mean, off * most + 1e-45), (rstd, rel * rstd)


def norm_bwd(dy, h, mean, rstd, weight, dsummed):
    """dx, dweight, dbias in 64 bits from the statistics as given, and what each may be off."""
    dy, n = dy.double(), (h.double() - mean.double()[..., None]) * rstd.double()[..., None]
    g = dy * (1 if weight is None else weight.double())
    c0, c1 = g.mean(-1, keepdim=True), (g * n).mean(-1, keepdim=True)
    r = rstd.double()[..., None]
    dx = r * (g - c0 - n * c1)
    size = r * (g.abs() + g.abs().mean(-1, keepdim=True) + n.abs() * (g * n).abs().mean(-1, keepdim=True))
    if dsummed is not None:
        dx, size = dx + dsummed.double(), size + dsummed.double().abs()
    rows = lambda t: t.flatten(0, -2).sum(0)  # noqa: E731
    # at most 256 additions one after the other: rows of a thread, threads of a workgroup, workgroups' sums
    return (dx, HALF16 * dx.abs() + 128 * U32 * size), (rows(dy * n), 256 * U32 * rows((dy * n).abs()) + 1e-45), \
        (rows(dy), 256 * U32 * rows(dy.abs()) + 1e-45)


def act8(x, fmt):
    """(codes, scales) of the definition, whose numbers are 32-bit; on the CPU."""
    x = x.detach().cpu().float()
    c = x.shape[-1]
    b = torch.nn.functional.pad(x, (0, -c % BLOCK)).unflatten(-1, (-1, BLOCK))
    most = b.abs().amax(-1)
    scale = torch.clamp(most * torch.tensor(1.0 / MOST[fmt], dtype=torch.float32), min=2.0 ** -126)
    u = b * (torch.ones_like(scale) / scale)[..., None]
    codes = torch.round(u).to(torch.int8) if fmt == "int8" else u.to(torch.float8_e4m3fn)
    scale = torch.where(torch.isfinite(most), scale, torch.full_like(scale, float("nan")))
    return codes.flatten(-2)[..., :c], scale


def act8_values(codes, scales):
    """What codes and scales stand for, in fp32 (exact up to one rounding)."""
    c = codes.shape[-1]
    return codes.float() * scales.repeat_interleave(BLOCK, dim=-1)[..., :c]


def assert_within(name, got, ref, off):
    got, ref, off = got.double(), ref.double().to(got.device), off.double().to(got.device)
    bad = ~((got - ref).abs() <= off)
    assert not bad.any(), f"{name}: {int(bad.sum())} of {bad.numel()} off, worst {float((got - ref).abs()[bad].max()):.3e}" \
        f" where {float(off[bad].min()):.3e} is allowed"
