"""Few rows, which more warps share the fewer they are: on both sides of every number of rows where that changes."""
import pytest
import torch

import test_gpu_losses as base

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("per_sm", [1, 2, 4, 8])
@pytest.mark.parametrize("more", [0, 1])
@pytest.mark.parametrize("v,dtype", [(1, BF), (300, F32), (4097, BF), (6911, F32), (13825, BF), (28161, BF)])
def test_rows_for_each_sm(per_sm, more, v, dtype):
    rows = per_sm * torch.cuda.get_device_properties(0).multi_processor_count + more
    shape = (rows, 1, v, dtype, None, [i % 7 > 0 for i in range(rows)])
    base.test_clip(shape)
    base.test_distill(shape, more == 1)
