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


@pytest.mark.parametrize("v", [10**400, "1", None], ids=["large", "text", "none"])
def test_numbers_that_are_none(env, v):
    """One that no double holds, and what is no number."""
    x, u, a = torch.zeros((5, 7), device=DEV), torch.zeros((5,), device=DEV), torch.zeros((5,), dtype=torch.int32, device=DEV)
    r, d = torch.zeros((4, 3), device=DEV), torch.zeros((4, 3), dtype=torch.uint8, device=DEV)
    values = torch.zeros((5, 3), device=DEV)
    bad = pytest.raises(binding.PcgrlError, match="must be a number")
    for name in ("temperature", "top_p", "min_p"):
        with bad:
            env.pcgrl_sample(x, u, **{name: v})
    for name in ("temperature", "clip_low", "clip_high", "entropy_coef", "value_coef") + (("scale",) if v is not None else ()):
        with bad:
            env.pcgrl_policy_loss(x, a, u, **{name: v})
    for discount, trace in ((v, .9), (.9, v)):
        with bad:
            env.pcgrl_advantages(r, d, values, discount, trace)
