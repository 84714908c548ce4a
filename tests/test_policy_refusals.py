"""Host-only checks of what the policy's entry points refuse, before any GPU call, beyond test_policy_abi."""
import ctypes as C

import pytest

from paper_2408_12525_amd import binding

CTX = C.c_void_p(4096)          # (never followed: every call here ends before the context is looked at)
P = 1 << 20
OK, NULL, CONFIG = 0, -1, -2


def policy_loss(**more):
    d = dict(type=3, n_classes=7, n_rows=5, logits=P, logits_stride=7, mask_stride=7, actions=2 * P, advantages=2 * P, old_log_probs=2 * P, temperature=1.0,
             clip_low=.2, clip_high=.2, entropy_coef=.01, value_coef=.5, scale=1.0, grad_logits=3 * P, grad_stride=7, stats=4 * P, workspace=5 * P)
    loss = binding.PcgrlLoss(**dict(d, **more))
    return binding.load().pcgrl_policy_loss(CTX, C.byref(loss), None)


@pytest.mark.parametrize("more", [dict(scale=1e280, temperature=1e-30), dict(scale=-1e301), dict(scale=1e200, entropy_coef=1e101), dict(scale=1e-5, entropy_coef=-1e300, temperature=1e-10),
                                  dict(scale=1e200, value_coef=1e101), dict(scale=1e300, entropy_coef=1e300, value_coef=0.)])
def test_factors_beyond_64_bits_are_refused(more):
    """What gradients are multiplied by has to be a number, with room for a sum of products: also where there are no rows."""
    assert policy_loss(**more) == CONFIG and policy_loss(n_rows=0, stats=None, **more) == CONFIG


def test_large_factors_that_are_numbers_are_not():
    for more in (dict(scale=1e30, temperature=1e-30), dict(scale=1e-300, entropy_coef=1e300), dict(scale=0., entropy_coef=1e300, value_coef=1e300), dict(scale=-1e300)):
        assert policy_loss(n_rows=0, stats=None, **more) == OK


@pytest.mark.parametrize("k", [-1, 2**31, 2**32, 2**32 + 5, 10**30, 1.5, "5", None])
def test_a_top_k_that_is_no_32_bit_number_is_refused(k):
    """It would be another one in the structure of the C interface (no tensor is looked at before)."""
    import torch
    env = object.__new__(binding.Pcgrl)
    env.device = torch.device("cuda", 0)
    x = torch.zeros((3, 2))
    with pytest.raises(binding.PcgrlError, match="top_k"):
        env._sampling(x, torch.zeros(3), None, None, 1.0, k, 1.0, 0.0)
    with pytest.raises(binding.PcgrlError, match="logits must be a tensor on"):
        env._sampling(x, torch.zeros(3), None, None, 1.0, 2**31 - 1, 1.0, 0.0)


@pytest.mark.parametrize("v", [10**400, -10**400, "1", None, [1.0], 1j], ids=["large", "low", "text", "none", "list", "complex"])
def test_a_coefficient_that_is_no_number_is_refused(v):
    import torch
    env = object.__new__(binding.Pcgrl)
    env.device = torch.device("cuda", 0)
    x = torch.zeros((3, 2))
    for more in ((v, 0, 1.0, 0.0), (1.0, 0, v, 0.0), (1.0, 0, 1.0, v)):
        with pytest.raises(binding.PcgrlError, match="temperature|top_p|min_p"):
            env._sampling(x, torch.zeros(3), None, None, *more)


@pytest.mark.parametrize("rc,more", [(NULL, dict(grad_values=6 * P)), (CONFIG, dict(grad_values=6 * P + 2)), (OK, dict(n_rows=0, stats=None, grad_values=6 * P))])
def test_a_gradient_of_values_needs_values(rc, more):
    """It would be left as it was."""
    assert policy_loss(**more) == rc
