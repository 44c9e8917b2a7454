"""Sizes at the ends of their types in the operators around attention, on the CPU: the library's checks (with pointers that are never
followed) and the binding's."""
import pytest
import torch

from tests import test_block_refusals as R
from tests.test_block_refusals import lib, on_cpu  # noqa: F401
from paper_2605_08962_amd import binding

INT_MAX = 2 ** 31 - 1


@pytest.mark.parametrize("inverse", [False, True])
def test_numbers_of_pairs_beyond_the_head(lib, inverse):  # noqa: F811
    """Their double does not fit the type they come in."""
    for pairs in (33, 1 << 29, 1 << 30, (1 << 30) + 32, INT_MAX):
        assert R._rotary(lib, None, inverse, num_pairs=pairs) == R.SHAPE, pairs
    for d in (2, 3, 65, 512):
        wide = dict(head_dim=d, q_stride=4 * d, k_stride=2 * d, v_stride=2 * d, q_out_stride=4 * d, k_out_stride=2 * d, v_out_stride=2 * d)
        assert R._rotary(lib, None, inverse, num_pairs=d // 2 + 1, **wide) == R.SHAPE
        assert R._rotary(lib, None, inverse, num_pairs=d // 2, total_tokens=0, **wide) == R.OK


WRAPPED = 2 ** 32 + 8  # eight, in 32 bits


def _big(*shape, dtype=torch.bfloat16):
    """Takes no memory: the checks come before anything is read."""
    return torch.empty(shape, dtype=dtype, device="meta")


def _big8(*shape):
    return binding.Act8(_big(*shape, dtype=torch.int8), _big(*shape[:-1], -(-shape[-1] // 128), dtype=torch.float32))


def _f32(*shape):
    return _big(*shape, dtype=torch.float32)


def _i32(*shape):
    return _big(*shape, dtype=torch.int32)


@pytest.mark.parametrize("call", [
    lambda b: b.varlen_attn_norm_fwd(_big(WRAPPED, 64)), lambda b: b.varlen_attn_norm_fwd(_big(1, WRAPPED, 64)),
    lambda b: b.varlen_attn_norm_fwd(_big(2, WRAPPED)),
    lambda b: b.varlen_attn_norm_bwd(_big(WRAPPED, 64), _big(WRAPPED, 64), _f32(WRAPPED), _f32(WRAPPED)),
    lambda b: b.varlen_attn_norm_bwd(_big(WRAPPED, 64), _big8(WRAPPED, 64), _f32(WRAPPED), _f32(WRAPPED)),
    lambda b: b.varlen_attn_act8_pack([_big(WRAPPED, 64)]), lambda b: b.varlen_attn_act8_pack([_big(3, 8), _big(4, WRAPPED, 64)]),
    lambda b: b.varlen_attn_act8_unpack([_big8(WRAPPED, 64)]), lambda b: b.varlen_attn_act8_unpack([_big8(1, WRAPPED)]),
    lambda b: b.varlen_attn_rotary_fwd(_big(WRAPPED, 1, 64), _big(WRAPPED, 1, 64), _i32(2, WRAPPED), _f32(32), _i32(32)),
    lambda b: b.varlen_attn_rotary_bwd(_big(1, WRAPPED, 64), _big(1, 1, 64), _i32(2, 1), _f32(32), _i32(32)),
    lambda b: b.varlen_attn_rotary_fwd(_big(1, 2, 64), _big(1, 1, 64), _i32(WRAPPED, 1), _f32(32), _i32(32)),
    lambda b: b.varlen_attn_rotary_fwd(_big(1, 2, 64), _big(1, 1, 64), _i32(2, 1), _f32(WRAPPED), _i32(WRAPPED)),
    lambda b: b.varlen_attn_rotary_positions(_i32(3), _i32(2, 3), WRAPPED), lambda b: b.varlen_attn_rotary_positions(_i32(3), _i32(2, 3), -WRAPPED),
    lambda b: b.varlen_attn_rotary_positions(_i32(3), _i32(2, 3), 10, merge=2 ** 32 + 2),
    lambda b: b.varlen_attn_rotary_positions(_i32(WRAPPED), _i32(WRAPPED - 1, 3), 10),
    lambda b: R._attn_call(cu=_i32(WRAPPED))(b), lambda b: R._attn_call(q=_big8(WRAPPED, 1, 64), dout=_big(WRAPPED, 1, 64))(b),
    lambda b: b.varlen_attn_bwd_act8(*R_ATTN, kv_splits=2 ** 32)])
def test_sizes_that_do_not_fit_are_refused_instead_of_cut(on_cpu, call):  # noqa: F811
    with pytest.raises(ValueError, match="must be below"):
        call(binding)
    assert not on_cpu


R_ATTN = (R.bf(6, 4, 64), R._a8(6, 4, 64), R._a8(6, 2, 64), R._a8(6, 2, 64), R._a8(6, 4, 64), torch.zeros(4, 6), R.i32(2), True, 0.1)


def test_the_largest_sizes_that_fit_are_taken(on_cpu):  # noqa: F811
    binding.varlen_attn_norm_fwd(_big(INT_MAX, 8))
    binding.varlen_attn_act8_pack([_big(INT_MAX, 8)])
    binding.varlen_attn_rotary_positions(_i32(3), _i32(2, 3), INT_MAX)
    assert len(on_cpu) == 3


@pytest.mark.parametrize("longest", [INT_MAX, 2 ** 31, 2 ** 32, 2 ** 32 + 1, 2 ** 40])
def test_a_promise_beyond_32_bits_stays_one(on_cpu, longest):  # noqa: F811
    """That no sample is longer than that: never that none is longer than its low half."""
    binding.varlen_attn_bwd_act8(*R_ATTN, max_seqlen=longest)
    (name, args), = on_cpu
    assert args[0]._obj.max_seqlen == INT_MAX
