"""What calls of the policy's operators refuse, and what they do to the tensors that they are given, through the binding
(needs an MI355X)."""
import math

import numpy as np
import pytest
import torch

from paper_2408_12525_amd import binding, workloads as wl

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda", 0)


@pytest.fixture(scope="module")
def env():
    e = binding.Pcgrl(wl.workload("dungeon32", batch=8), 0)
    yield e
    e.close()


def test_a_top_k_beyond_32_bits(env):
    x, u = torch.randn((40, 9), device=DEV), torch.rand((40,), device=DEV)
    for k in (2**31, 2**32, 2**32 + 5, 10**30):
        with pytest.raises(binding.PcgrlError, match="top_k"):
            env.pcgrl_sample(x, u, top_k=k)
    want = env.pcgrl_sample(x, u)
    got = env.pcgrl_sample(x, u, top_k=2**31 - 1)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert torch.equal(env.pcgrl_sample(x, u, top_k=np.int64(1))[0], env.pcgrl_sample(x, u, top_k=1)[0])


def test_sizes_beyond_32_bits(env):
    """Sizes of tensors that would be others in the numbers of the C interface (none of these holds an element)."""
    e = lambda t, *s: torch.empty(s, dtype=t, device=DEV)  # noqa: E731
    f32 = torch.float32
    for V in (32769, 2**31 + 1, 2**32, 2**32 + 7):
        with pytest.raises(binding.PcgrlError):
            env.pcgrl_sample(e(f32, 0, V), e(f32, 0))
        with pytest.raises(binding.PcgrlError):
            env.pcgrl_policy_loss(e(f32, 0, V), e(torch.int32, 0), e(f32, 0))
    for T, n in ((2**32 + 3, 0), (2**31, 0), (2**20 + 1, 0)):
        with pytest.raises(binding.PcgrlError):
            env.pcgrl_advantages(e(f32, T, n), e(torch.uint8, T, n), e(f32, T + 1, n), .9, .9)
