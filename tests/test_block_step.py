"""The operators around attention run together, as a training step runs them (bench.py's block): the attention half of a pre-norm
block, forward and backward, against the same block in 64 bits with gradients by autograd."""
import numpy as np
import pytest
import torch

import bench
from paper_2605_08962_amd import workloads as W
from tests import _block as B

pytestmark = pytest.mark.gpu

# Relative 2-norm of the error.  A rounding to bf16 leaves 1.7e-3 of a tensor, int8 at 64 to 128 channels a block 6e-3 to 7e-3 (a step
# of amax / 127, amax 2.5 to 2.9 standard deviations), e4m3 2.6e-2.  A result is behind up to 10 roundings to bf16 (5e-3), and a gradient
# of q and k behind the stored q, k, v and o: scores of unit size are off by sqrt(2) steps, P by as much, dP and Delta by one step
# each, and the product with k by another: 2.3 steps; twice that for what depends on the draw.
TOLERANCE = {None: 1e-2, "int8": 1e-2 + 2 * 2.3 * 7e-3, "e4m3": 1e-2 + 2 * 2.3 * 2.6e-2}


def _block64(p, x, r, cu, turn, causal, scale):
    hq, hkv = p["heads"]
    h = x + r
    d = h - h.mean(-1, keepdim=True)
    n = d * ((d * d).mean(-1, keepdim=True) + 1e-5) ** -0.5 * p["norm_w"] + p["norm_b"]
    qkv = (n @ p["w_qkv"].T).unflatten(1, (hq + 2 * hkv, -1))
    pos, freq, axis = turn
    phi = (pos.double()[axis.long()].T * freq.double())[:, None]

    def rotate(z):
        a, b = z.chunk(2, dim=-1)
        return torch.cat([a * phi.cos() - b * phi.sin(), b * phi.cos() + a * phi.sin()], dim=-1)
    q, k, v = rotate(qkv[:, :hq]), rotate(qkv[:, hq:hq + hkv]), qkv[:, hq + hkv:]
    outs = []
    for lo, hi in zip(cu[:-1], cu[1:]):
        heads = []
        for i in range(hq):
            s = scale * q[lo:hi, i] @ k[lo:hi, i // (hq // hkv)].T
            if causal:
                s = s.masked_fill(torch.ones_like(s, dtype=torch.bool).triu(1), float("-inf"))
            heads.append(torch.softmax(s, -1) @ v[lo:hi, i // (hq // hkv)])
        outs.append(torch.stack(heads, dim=1))
    return h, torch.cat(outs).flatten(1) @ p["w_out"].T


@pytest.mark.parametrize("save", [None, "int8", "e4m3"])
@pytest.mark.parametrize("lengths,hq,hkv,d,causal", [([16, 37, 64, 129], 2, 2, 64, False), ([300, 1, 77], 4, 2, 80, True),
                                                     ([513], 2, 1, 128, True)])
def test_forward_and_backward_of_the_attention_half(lengths, hq, hkv, d, causal, save):
    from paper_2605_08962_amd import binding
    w = W.make_custom(lengths, hq, hkv, d, causal, seed=5)
    print(lengths, hq, hkv, d, causal, save, flush=True)
    T, C = w.total_tokens, hq * d
    p = {"heads": (hq, hkv), "norm_w": 1 + B.bf(C, seed=1, scale=0.1), "norm_b": B.bf(C, seed=2, scale=0.1),
         "w_qkv": B.bf((hq + 2 * hkv) * d, C, seed=3, scale=C ** -0.5), "w_out": B.bf(C, C, seed=4, scale=C ** -0.5)}
    x, r, ds, dy = (B.bf(T, C, seed=10 + i) for i in range(4))
    cu, turn = bench.block_positions(torch, binding, w)
    call = (cu, turn, causal, w.scale, max(lengths))
    summed, y, saved = bench.block_forward(torch, binding, p, x, r, *call, save)
    got = bench.block_backward(torch, binding, p, ds, dy, saved, *call)

    leaves = {n: t.double().requires_grad_() for n, t in (("x", x), *((n, t) for n, t in p.items() if n != "heads"))}
    h64, y64 = _block64({**leaves, "heads": (hq, hkv)}, leaves["x"], r.double(), w.cu_seqlens.tolist(), turn, causal, w.scale)
    ((h64 * ds.double()).sum() + (y64 * dy.double()).sum()).backward()
    off = lambda a, b: float((a.double() - b).norm() / b.norm())  # noqa: E731
    assert torch.equal(summed, (x.float() + r.float()).to(torch.bfloat16)) and off(y, y64.detach()) <= TOLERANCE[None]
    for name, g in zip(("x", "norm_w", "norm_b", "w_qkv", "w_out"), got):
        assert off(g, leaves[name].grad) <= TOLERANCE[save], (name, off(g, leaves[name].grad))


def test_positions_of_the_images_are_their_lengths():
    from paper_2605_08962_amd import binding
    w = W.make(2, lengths_only=True)
    cu, (pos, freq, axis) = bench.block_positions(torch, binding, w)
    ends = np.asarray(w.cu_seqlens[1:]) - 1
    last = pos[:, torch.from_numpy(ends).long().cuda()].cpu().numpy()
    assert (last[0] == 0).all() and ((last[1] + 1) * (last[2] + 1) == w.lengths).all()
