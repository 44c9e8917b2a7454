"""The operators around attention at sizes that do not fit 31 or 32 bits somewhere on the way, on the GPU."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_norm_of_as_many_rows_a_token_as_there_can_be():
    """Rows of one channel, whose mean is that channel: two tokens of 2^31 - 1, a stride apart."""
    from paper_2605_08962_amd import binding
    n = 2 ** 31 - 1
    gen = torch.Generator(device="cuda").manual_seed(1)
    whole = torch.empty((2, n + 9), dtype=torch.bfloat16, device="cuda")
    for t in whole:
        t.normal_(generator=gen)
    x = whole[:, 3:3 + n].unsqueeze(-1)
    assert x.shape == (2, n, 1) and x.stride(0) > n
    f = binding.varlen_attn_norm_fwd(x)
    assert not f.out.any()
    for t in range(2):
        assert torch.equal(f.mean[t].to(torch.bfloat16), x[t, :, 0])


def test_rotation_by_more_workgroups_than_one_launch_takes():
    """Four tokens a workgroup of 256 threads: 2^26 tokens are the first that 2^32 threads do not cover."""
    from paper_2605_08962_amd import binding
    T, P = 2 ** 26 + 1003, 1
    gen = torch.Generator(device="cuda").manual_seed(2)
    x = torch.empty((T, 2, 2), dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    pos = torch.randint(0, 1000, (1, T), generator=gen, device="cuda", dtype=torch.int32)
    freq, axis = torch.rand(P, device="cuda"), torch.zeros(P, dtype=torch.int32, device="cuda")
    q, k = binding.varlen_attn_rotary_fwd(x[:, :1], x[:, 1:], pos, freq, axis)
    for at in range(0, T, 2 ** 25):
        s = slice(at, min(at + 2 ** 25, T))
        a, b = binding.varlen_attn_rotary_fwd(x[s, :1], x[s, 1:], pos[:, s].contiguous(), freq, axis)
        assert torch.equal(q[s], a) and torch.equal(k[s], b), at


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_packing_by_more_workgroups_than_one_launch_takes(fmt):
    """128 rows a workgroup: 2^31 rows are the first that 2^32 threads do not cover.  A second tensor starts behind them."""
    from paper_2605_08962_amd import binding
    T, h = 2 ** 16 + 1, 2 ** 15
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.empty((T, h, 1), dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    y = torch.empty((77, 3), dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    whole, small = binding.varlen_attn_act8_pack([x, y], fmt)
    back, small_back = binding.varlen_attn_act8_unpack([whole, small])
    bits = lambda c: c.view(torch.int8)  # noqa: E731
    parts = [slice(at, min(at + 2 ** 14, T)) for at in range(0, T, 2 ** 14)]
    for s in parts:
        want = binding.varlen_attn_act8_pack([x[s]], fmt)[0]
        assert torch.equal(bits(whole.codes[s]), bits(want.codes)) and torch.equal(whole.scales[s], want.scales), s
        assert torch.equal(back[s], binding.varlen_attn_act8_unpack([want])[0]), s
    want = binding.varlen_attn_act8_pack([y], fmt)[0]
    assert torch.equal(bits(small.codes), bits(want.codes)) and torch.equal(small_back, binding.varlen_attn_act8_unpack([want])[0])
