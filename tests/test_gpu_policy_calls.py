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
