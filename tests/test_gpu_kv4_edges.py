"""seq_tree_kv4_attention where its kernels hand things over: ranges that open or end with a piece of a unit."""
import numpy as np
import pytest
import torch

from tests.test_gpu_kv4_attention import Case

pytestmark = pytest.mark.gpu
BOTH = pytest.mark.parametrize("dt", [torch.float16, torch.bfloat16])


@BOTH
@pytest.mark.parametrize("R,seed", [(60, 0), (100, 1), (150, 2)])
def test_ranges_that_open_with_the_last_step_of_a_unit(R, seed, dt):
    """Many ragged units over all SMs: between 9 and 16 of the ranges begin with one step and go on with the next unit.  The two
    groups of threads that share a row of q have channels of different magnitudes, so that each needs what the other found."""
    lengths = np.random.default_rng(seed).integers(100, 700, R)
    c = Case(list(lengths), 20, 8, 2, 16, dt, seed=seed)
    piece = torch.arange(128) // 8 % 2
    size = 2.0 ** torch.randint(-6, 1, (R, 20, 8, 2), generator=torch.Generator().manual_seed(seed))
    c.q = (c.q.float() * size[..., piece]).to(dt)
    out, call = c.check(exact_keys=dt == torch.float16)
    assert call.workspace is not None  # ranges, not clusters
    out, lse = out.clone(), call.lse.clone()
    for _ in range(20):
        assert torch.equal(call.run(), out) and torch.equal(call.lse, lse)
