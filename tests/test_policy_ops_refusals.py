"""Policy-network operators, host side: calls whose numbers or addresses the kernels could not work with are refused before anything is
enqueued (no GPU needed; what is accepted stops at the missing device)."""

import pytest
import torch

import test_policy_ops_host as base
from paper_2510_03515_b200 import binding as rb

ATTENTION = [base._attn_fwd, base._attn_bwd]


def _attn(**kw):
    return rb.make_attn_desc(4, 8, 4, 2, 64, **kw)


# ---- the factor of the scores ----------------------------------------------------------------------------------

FLT_MIN, FLT_MAX = torch.finfo(torch.float32).tiny, torch.finfo(torch.float32).max


@pytest.mark.parametrize("call", ATTENTION)
@pytest.mark.parametrize("scale", [1e39, 1e300, FLT_MAX, FLT_MAX / 1.44, 1e-39, 1e-50, 5e-324, FLT_MIN * 0.999])
def test_a_scale_that_is_no_float_is_refused(call, scale):
    """The kernels work with scale and scale * log2(e) in float: neither may be infinite, zero or subnormal."""
    assert call(_attn(scale=scale)) == base.INVALID


@base.no_gpu
@pytest.mark.parametrize("call", ATTENTION)
@pytest.mark.parametrize("scale", [FLT_MAX / 1.45, FLT_MIN, 1.0, 64 ** -0.5])
def test_any_other_scale_is_accepted(call, scale):
    assert call(_attn(scale=scale)) == rb.RAPID_ERR_CUDA
