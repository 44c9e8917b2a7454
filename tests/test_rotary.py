"""Rotary positions on the GPU against their definition in 64 bits."""
import pytest
import torch

from tests import _block as B

pytestmark = pytest.mark.gpu


def _turn(P, axes, far, T, seed=1, device="cuda"):
    gen = torch.Generator().manual_seed(seed)
    pos = torch.randint(0, far, (axes, T), generator=gen, dtype=torch.int32)
    if T > 1:
        pos[:, 0], pos[:, 1] = far - 1, 0
    freq = 10000.0 ** (-torch.arange(P) / max(P, 1))
    axis = (torch.arange(P) * axes // P).to(torch.int32)
    return pos.to(device), freq.float().to(device), axis.to(device)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,hq,hkv,d,P,axes,far", [
    (1, 1, 1, 64, 32, 1, 10), (5, 2, 1, 80, 40, 2, 100), (246, 2, 2, 64, 32, 3, 1000), (37, 3, 3, 96, 48, 3, 1 << 20),
    (4099, 4, 1, 128, 64, 3, 1 << 30), (129, 8, 2, 128, 16, 2, 5000),    # a part of the channels turned
    (65, 2, 1, 80, 20, 2, 5000), (33, 2, 2, 64, 13, 2, 77), (9, 1, 1, 7, 3, 2, 50), (21, 2, 1, 66, 33, 1, 9),  # odd runs
    (6, 1, 2, 512, 256, 8, 100), (4100, 1, 1, 2, 1, 1, 100), (17, 2, 1, 64, 4, 2, 100), (300, 5, 5, 12, 4, 2, 40)])
def test_forward_and_backward(T, hq, hkv, d, P, axes, far, interleaved):
    from paper_2605_08962_amd import binding
    print(f"T={T} hq={hq} hkv={hkv} d={d} P={P} axes={axes} far={far} interleaved={interleaved}", flush=True)
    turn = _turn(P, axes, far, T)
    q, k, v = B.bf(T, hq, d, seed=1), B.bf(T, hkv, d, seed=2), B.bf(T, hkv, d, seed=3)
    for inverse, f in ((False, binding.varlen_attn_rotary_fwd), (True, binding.varlen_attn_rotary_bwd)):
        extra = {"dv": v} if inverse else {"v": v}
        got = f(q, k, *turn, interleaved=interleaved, **extra)
        assert all(g.is_contiguous() for g in got)
        for name, x, g in (("q", q, got[0]), ("k", k, got[1])):
            B.assert_within(name, g, *B.rotary(x, *turn, interleaved, inverse))
        assert torch.equal(got[2], v)
        two = f(q, k, *turn, interleaved=interleaved)
        assert len(two) == 2 and torch.equal(two[0], got[0]) and torch.equal(two[1], got[1])


@pytest.mark.parametrize("T,hq,hkv,d,odd", [(50, 4, 2, 64, 0), (4200, 4, 1, 128, 0), (50, 4, 2, 64, 4), (50, 2, 1, 80, 1)])
def test_parts_of_the_fused_projection(T, hq, hkv, d, odd):
    """q, k, v out of one tensor and their gradients back into one, whatever stands beside them stays; `odd` elements shift the
    rows off 16 and 8 bytes."""
    from paper_2605_08962_amd import binding
    turn = _turn(d // 2, 2, 1000, T)
    whole = B.bf(T, (hq + 2 * hkv) * d + 2 * odd, seed=4)
    part = lambda w, lo, h: w[:, odd + lo * d:odd + (lo + h) * d].unflatten(1, (h, d))  # noqa: E731
    q, k, v = part(whole, 0, hq), part(whole, hq, hkv), part(whole, hq + hkv, hkv)
    got = binding.varlen_attn_rotary_fwd(q, k, *turn, v=v)
    want = binding.varlen_attn_rotary_fwd(q.contiguous(), k.contiguous(), *turn, v=v.contiguous())
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    grads = torch.full_like(whole, 7.0)
    outs = part(grads, 0, hq), part(grads, hq, hkv), part(grads, hq + hkv, hkv)
    back = binding.varlen_attn_rotary_bwd(*got[:2], *turn, dv=got[2], dq_out=outs[0], dk_out=outs[1], dv_out=outs[2])
    assert all(a is b for a, b in zip(back, outs))
    plain = binding.varlen_attn_rotary_bwd(*got[:2], *turn, dv=got[2])
    assert all(torch.equal(a, b) for a, b in zip(outs, plain))
    assert (grads[:, :odd] == 7).all() and (grads[:, grads.shape[1] - odd:] == 7).all()


@pytest.mark.parametrize("interleaved", [False, True])
def test_in_place(interleaved):
    from paper_2605_08962_amd import binding
    T, hq, hkv, d = 777, 4, 2, 96
    turn = _turn(40, 3, 1000, T)
    whole = B.bf(T, hq + hkv, d, seed=5)
    q, k = whole[:, :hq], whole[:, hq:]
    want = binding.varlen_attn_rotary_fwd(q, k, *turn, interleaved=interleaved)
    binding.varlen_attn_rotary_fwd(q, k, *turn, interleaved=interleaved, q_out=q, k_out=k)
    assert torch.equal(whole, torch.cat(want, dim=1))


def test_backward_is_the_gradient():
    """Of sum(y * dy), against central differences of the definition in 64 bits."""
    from paper_2605_08962_amd import binding
    T, d, P = 3, 20, 8
    for interleaved in (False, True):
        pos, freq, axis = _turn(P, 2, 50, T)
        x, dy = B.bf(T, 1, d, seed=6), B.bf(T, 1, d, seed=7)
        got = binding.varlen_attn_rotary_bwd(dy, dy, pos, freq, axis, interleaved=interleaved)[0].double()
        f = lambda z: (B.rotary(z, pos, freq, axis, interleaved)[0] * dy.double()).sum()  # noqa: E731
        h = 1e-3  # (the function is linear: differences are exact but for 64-bit roundings)
        for i in range(x.numel()):
            e = torch.zeros(x.numel(), dtype=torch.float64, device="cuda")
            e[i] = h
            e = e.view(x.shape)
            diff = float(f(x.double() + e) - f(x.double() - e)) / (2 * h)
            # half a step of bf16, and of the rotation in 32 bits (|dy| < 4)
            assert abs(float(got.flatten()[i]) - diff) <= B.HALF16 * abs(diff) + 2.0 ** -16


def test_values_that_are_no_numbers_stay_with_their_pair():
    from paper_2605_08962_amd import binding
    T, d = 8, 64
    turn = _turn(32, 2, 1000, T)
    x = B.bf(T, 1, d, seed=8)
    clean = binding.varlen_attn_rotary_fwd(x, x, *turn)[0]
    y = x.clone()
    y[2, 0, 5], y[4, 0, 40] = float("nan"), float("inf")
    got = binding.varlen_attn_rotary_fwd(y, y, *turn)[0]
    hit = torch.zeros_like(got, dtype=torch.bool)
    hit[2, 0, [5, 37]] = hit[4, 0, [8, 40]] = True
    assert not torch.isfinite(got[hit]).any() and torch.equal(got[~hit], clean[~hit])


def test_an_axis_that_does_not_exist_is_the_nearest_one():
    from paper_2605_08962_amd import binding
    x, (pos, freq, axis) = B.bf(9, 2, 64), _turn(32, 2, 100, 9)
    wild, tame = axis.clone(), axis.clone()
    wild[:3] = torch.tensor([-5, 2, 1 << 30], dtype=torch.int32)
    tame[:3] = torch.tensor([0, 1, 1], dtype=torch.int32)
    a, b = (binding.varlen_attn_rotary_fwd(x, x, pos, freq, i) for i in (wild, tame))
    assert torch.equal(a[0], b[0])


@pytest.mark.parametrize("merge,grids", [
    (1, [(1, 3, 5), (0, 0, 0), (2, 4, 4), (0, 0, 0)]), (2, [(0, 0, 0), (3, 4, 6), (1, 2, 2), (0, 0, 0), (1, 8, 2)]),
    (4, [(1, 4, 8), (2, 8, 4)]), (2, [(0, 0, 0)])])
@pytest.mark.parametrize("based", [False, True])
def test_positions(merge, grids, based):
    from paper_2605_08962_amd import binding
    lens = [t * h * w if h else 7 + 3 * i for i, (t, h, w) in enumerate(grids)]
    lens.insert(1, 0)  # an empty segment
    grids = grids[:1] + [(1, merge, merge)] + grids[1:]
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    first = [11 * i - 5 for i in range(len(lens))] if based else None
    dev = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    for total in (cu[-1], cu[-1] + 3):  # (tokens behind the last segment are in none)
        out = torch.full((3, total), -1, dtype=torch.int32, device="cuda")
        got = binding.varlen_attn_rotary_positions(dev(cu), dev(grids), total, first=dev(first), merge=merge, out=out)
        assert got is out and torch.equal(got.cpu(), B.positions(cu, grids, first, merge, total))
        assert torch.equal(binding.varlen_attn_rotary_positions(dev(cu), dev(grids), total, first=dev(first), merge=merge), got)


@pytest.mark.parametrize("seed,segments,longest,empty", [(1, 70, 3, 0.9), (2, 500, 2, 0.95), (3, 64, 1, 0.0), (4, 65, 1, 0.0), (5, 300, 200, 0.3),
                                                          (6, 20000, 4, 0.5), (7, 4097, 1, 0.99), (8, 1, 700, 0.0), (9, 129, 64, 0.0)])
def test_positions_of_short_and_empty_segments(seed, segments, longest, empty):
    """Few and many of them to a wave of tokens, and a wave that no segment or every one ends in."""
    from paper_2605_08962_amd import binding
    gen = torch.Generator().manual_seed(seed)
    lens = torch.randint(1, longest + 1, (segments,), generator=gen)
    lens[torch.rand(segments, generator=gen) < empty] = 0
    cu = torch.cat([torch.zeros(1, dtype=torch.long), lens.cumsum(0)])
    first = torch.randint(0, 1000, (segments,), generator=gen)
    total = int(cu[-1]) + 70  # (and tokens behind the last)
    seg = torch.repeat_interleave(torch.arange(segments), lens)
    want = torch.zeros(total, dtype=torch.int32)
    want[:len(seg)] = (torch.arange(len(seg)) - cu[seg] + first[seg]).int()
    dev = lambda x: x.to(torch.int32).cuda()  # noqa: E731
    got = binding.varlen_attn_rotary_positions(dev(cu), torch.zeros((segments, 3), dtype=torch.int32, device="cuda"), total, first=dev(first))
    assert torch.equal(got.cpu(), want.expand(3, -1))


def test_positions_of_many_and_of_no_segments():
    from paper_2605_08962_amd import binding
    n = 5000
    cu = torch.arange(0, 3 * n + 1, 3, dtype=torch.int32, device="cuda")
    grids = torch.zeros((n, 3), dtype=torch.int32, device="cuda")
    got = binding.varlen_attn_rotary_positions(cu, grids, 3 * n)
    assert torch.equal(got, torch.arange(3, dtype=torch.int32, device="cuda").repeat(n).expand(3, -1))
    none = binding.varlen_attn_rotary_positions(cu[:1], grids[:0], 10)
    assert not none.any()
    assert binding.varlen_attn_rotary_positions(cu[:1], grids[:0], 0).shape == (3, 0)


def test_no_tokens():
    from paper_2605_08962_amd import binding
    q = torch.empty((0, 2, 64), dtype=torch.bfloat16, device="cuda")
    out = binding.varlen_attn_rotary_fwd(q, q, *_turn(32, 2, 10, 0), v=q)
    assert [t.shape for t in out] == [q.shape] * 3
