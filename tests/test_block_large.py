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
