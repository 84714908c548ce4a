"""The policy's operators where their numbers are out of the ordinary, against plain 64-bit statements (needs an
MI355X): temperatures and coefficients over the whole range that the entry points take, ratios and advantages that
are infinite or no number, a great many rows, outputs left out.

Tolerances.  As for ordinary numbers: a result is rounded once to its type, half a step, and what is computed in 32
bits before that (the parts of a gradient) takes at most eight roundings of its size, 8 * 2^-24.  Everything else is
computed in 64 bits.  Two of those roundings, of a weight w <= 1 and of w times 1 / (sum of weights) <= 1, are of numbers that may lie
below 2^-126, where a step of 32 bits is 2^-149 and half of it no share of the number: each takes up to 2^-150, and what
the product is multiplied by after that is at most m = |scale / temperature| (|u| + |entropy_coef| (1 + |log p| + H)), so that
2^-149 m comes on top (and a p below 2^-150, which 32 bits have as 0, is off by p m, less than that)."""
import math

import numpy as np
import pytest
import torch

from paper_2408_12525_amd import binding, workloads as wl

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda", 0)
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF = {t: torch.finfo(t).eps / 2 for t in TYPES.values()}
TINY = {torch.float32: 2.**-149, torch.bfloat16: 2.**-133, torch.float16: 2.**-24}   # the smallest steps
# a row in a lane, in eight or sixteen lanes, in a wavefront, in 128 to 1024 threads
CLASSES = [2, 7, 40, 100, 200, 500, 1000, 2000, 4000, 6000, 12000, 28672]


@pytest.fixture(scope="module")
def env():
    e = binding.Pcgrl(wl.workload("dungeon32", batch=8), 0)
    yield e
    e.close()


def gpu(a, dtype=None):
    t = torch.as_tensor(np.ascontiguousarray(a))
    return t.to(DEV, dtype) if dtype else t.to(DEV)


def wide64(t):
    return t.detach().double().cpu().numpy()


def distribution(x, mask, T):
    """Which classes of each row may be chosen, and the probabilities and log-probabilities (0 where not) of all."""
    may = x != -np.inf if mask is None else (x != -np.inf) & (mask != 0)
    x = np.where(may, x, -np.inf)
    y = (x - x.max(1, keepdims=True)) / T
    p = np.exp(y)
    whole = p.sum(1, keepdims=True)
    return may, p / whole, np.where(may, y - np.log(whole), 0.)


def gradients(x, mask, actions, advantages, old=None, temperature=1., clip_low=.2, clip_high=.2, entropy_coef=.01, scale=1.):
    """Of the policy loss and the entropy bonus, for rows that all count, and what rounding their parts to 32 bits goes by.
    Where a probability is nothing in 64 bits so is the gradient."""
    n, V = x.shape
    may, p, logs = distribution(x, mask, temperature)
    with np.errstate(all="ignore"):
        some = p > 0
        h = -np.where(some, p * logs, 0.).sum(1, keepdims=True)
        now = logs[np.arange(n), actions][:, None]
        adv = np.asarray(advantages, np.float64)[:, None]
        r = np.ones((n, 1)) if old is None else np.exp(now - np.asarray(old, np.float64)[:, None])
        held = np.zeros((n, 1), bool) if old is None else ((adv > 0) & (r > 1 + clip_high)) | ((adv < 0) & (r < 1 - clip_low))
        u = np.where(held, 0., -adv * r)
        chosen = np.arange(V)[None] == np.asarray(actions)[:, None]
        bonus = np.where(some, entropy_coef * p * (logs + h), 0.)
        g = np.where(chosen, u * (1 - p), np.where(some, -u * p, 0.)) + bonus
        by = scale / temperature
        most = np.abs(u) + np.where(some, abs(entropy_coef) * (1 + np.abs(logs) + h), 0.)
        size = abs(by) * (np.where(chosen, np.abs(u), 0.) + most * (p + 2.**-149 / (8 * 2.**-24)))
    return np.where(may, g * by, 0.), np.where(may, size, 0.)


def check_gradient(got, want, size, dtype):
    """Element by element, with the type's infinity where the value is beyond it (either where it is within its rounding of that)."""
    got, most = wide64(got), torch.finfo(dtype).max
    assert np.array_equal(np.isnan(got), np.isnan(want))
    some = ~np.isnan(want)
    over = some & (np.abs(want) > most * (1 + 2 * HALF[dtype]))
    assert np.array_equal(got[over], np.sign(want[over]) * np.inf)
    near = some & ~over & (np.abs(want) < most * (1 - 2 * HALF[dtype]))
    with np.errstate(all="ignore"):
        far = np.abs(got - want) - (np.abs(want) * HALF[dtype] + size * 8 * 2.**-24 * (1 + HALF[dtype]) + TINY[dtype] / 2)
    assert far[near].max(initial=-1) <= 0, far[near].max()


def some_mask(rng, n, V, actions):
    mask = (rng.random((n, V)) < .7).astype(np.uint8)
    mask[np.arange(n), actions] = 1
    return mask


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", CLASSES)
def test_gradients_at_any_temperature(env, V, dtype):
    """From 1e-30 to 3e38, with logits of a policy and with logits of the temperature's size, by themselves and scaled so
    that gradients are of a size of 1."""
    rng, t = np.random.default_rng(V), TYPES[dtype]
    n = 9 if V <= 4096 else 3
    for T in (1e-30, 1e-25, 1e-22, 1e-20, 1e-10, 1e-3, 1e3, 1e10, 1e25, 3e38):
        for spread in (1.5, T / 4):
            if not 1e-3 < spread < 1e3 and t == torch.float16:
                continue
            x = gpu(np.clip(rng.normal(size=(n, V)) * spread, -3.3e38, 3.3e38), torch.float64).to(t)
            a = rng.integers(0, V, n)
            for scale, mask in ((1., None), (T, some_mask(rng, n, V, a)), (-T / 8, None)):
                if t == torch.float16 and scale == 1. and T < 1e-3:
                    continue
                adv, coef = rng.normal(size=n).astype(np.float32), .3
                got = env.pcgrl_policy_loss(x, gpu(a, torch.int32), gpu(adv), mask=None if mask is None else gpu(mask), temperature=T, scale=scale, entropy_coef=coef)
                want, size = gradients(wide64(x), mask, a, adv, temperature=T, scale=scale, entropy_coef=coef)
                check_gradient(got["grad_logits"], want, size, t)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", CLASSES)
def test_gradients_of_any_size(env, V, dtype):
    """Coefficients from 1e-30 to 1e30, and ratios up to e^300."""
    rng, t = np.random.default_rng(V), TYPES[dtype]
    n = 9 if V <= 4096 else 3
    x = gpu(rng.normal(size=(n, V)) * 1.5, t)
    a = rng.integers(0, V, n)
    mask = some_mask(rng, n, V, a)
    logs = distribution(wide64(x), mask, 1.)[2][np.arange(n), a]
    for coef, scale, up in ((1e30, 1., 0.), (1e-30, 1., 0.), (.01, 1e30, 0.), (.01, 1e-30, 0.), (1e30, 1e-30, 0.), (1e-30, 1e30, 0.), (-1e20, 1e-15, 0.), (.01, 1., 30.), (.01, 1., 95.),
                            (.01, 1e-40, 95.), (.01, 1., 300.), (.01, 1e-120, 300.), (0., 1., 95.)):
        adv = -np.abs(rng.normal(size=n)).astype(np.float32) - .1 if up else rng.normal(size=n).astype(np.float32)
        old = (logs - up + .01).astype(np.float32) if up else None
        got = env.pcgrl_policy_loss(x, gpu(a, torch.int32), gpu(adv), old_log_probs=None if old is None else gpu(old), mask=gpu(mask), scale=scale, entropy_coef=coef)
        want, size = gradients(wide64(x), mask, a, adv, old, scale=scale, entropy_coef=coef)
        check_gradient(got["grad_logits"], want, size, t)
        assert not bool((got["grad_logits"][gpu(mask) == 0] != 0).any())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", CLASSES)
def test_masked_classes_have_no_gradient_whatever_the_row_is_weighed_by(env, V, dtype):
    """Advantages and old log-probabilities that are infinite or no number, beside rows that are in order."""
    rng, t, inf, nan = np.random.default_rng(V), TYPES[dtype], math.inf, math.nan
    n = 12
    x = gpu(rng.normal(size=(n, V)), t)
    a = rng.integers(0, V, n)
    a[a == 0] = V - 1
    mask = some_mask(rng, n, V, a)
    mask[:, 0] = 1                                      # (two classes or more, so that none has all of the probability)
    logs = distribution(wide64(x), mask, 1.)[2][np.arange(n), a]
    adv, old = rng.normal(size=n).astype(np.float32), (logs + rng.choice([-.5, 0., .5], n)).astype(np.float32)
    adv[1], adv[3], adv[4] = nan, inf, -inf
    old[5], old[6], old[7], old[8], old[9], old[10] = nan, -inf, -inf, inf, inf, -150.
    adv[6], adv[7], adv[8], adv[9], adv[10] = -1., 1., 1., -1., -2.
    want, size = gradients(wide64(x), mask, a, adv, old)
    got = env.pcgrl_policy_loss(x, gpu(a, torch.int32), gpu(adv), old_log_probs=gpu(old), mask=gpu(mask), scale=1.)["grad_logits"]
    assert not bool((got[gpu(mask) == 0] != 0).any())
    assert bool(torch.isnan(got[5][gpu(mask[5]) != 0]).all()) and bool(torch.isinf(got[6][gpu(mask[6]) != 0]).all()) and bool(torch.isfinite(got[[0, 2, 7, 11]]).all())
    check_gradient(got, want, size, t)
    got = env.pcgrl_policy_loss(x, gpu(a, torch.int32), gpu(adv), mask=gpu(mask), scale=1.)["grad_logits"]
    assert not bool((got[gpu(mask) == 0] != 0).any())
    check_gradient(got, *gradients(wide64(x), mask, a, adv), t)
