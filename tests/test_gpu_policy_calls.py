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


def test_gradients_over_the_logits_where_autograd_needs_them(env):
    """A head that keeps its output for its own gradient may not find another tensor in its place: autograd says so. One that does
    not keep it goes on, and so do calls with results of their own."""
    g = torch.Generator(DEV).manual_seed(3)
    n, V, d = 60, 9, 16
    feats = torch.randn((n, d), generator=g, device=DEV)
    head = torch.randn((d, V), generator=g, device=DEV).mul_(.3).requires_grad_()
    act, adv = torch.randint(0, V, (n,), generator=g, device=DEV).int(), torch.randn((n,), generator=g, device=DEV)
    logits = feats @ head
    logits.backward(env.pcgrl_policy_loss(logits, act, adv)["grad_logits"])
    want, head.grad = head.grad, None
    logits = feats @ head
    logits.backward(env.pcgrl_policy_loss(logits, act, adv, grad_logits=logits)["grad_logits"])
    assert torch.equal(head.grad, want)
    kept = torch.tanh(feats @ head)
    with pytest.raises(binding.PcgrlError):
        env.pcgrl_policy_loss(kept, act, adv, grad_logits=kept, clip_low=2.)
    kept.sum().backward()                               # (a refused call writes nothing)
    kept = torch.tanh(feats @ head)
    got = env.pcgrl_policy_loss(kept, act, adv, grad_logits=kept)["grad_logits"]
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        kept.backward(got)
    values = torch.tanh(feats @ head[:, 0])
    got = env.pcgrl_policy_loss((feats @ head).detach(), act, adv, values=values, returns=adv, grad_values=values)["grad_values"]
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        values.backward(got)


def test_what_a_call_writes_counts_as_changed(env):
    """Every tensor of the caller's that a call writes, and none that it reads; through both call paths."""
    n, V, T = 20, 5, 6
    f = lambda *s: torch.zeros(s, device=DEV)  # noqa: E731
    x, u, a, lp = torch.randn((n, V), device=DEV), torch.rand((n,), device=DEV), torch.zeros((n,), dtype=torch.int32, device=DEV), f(n)
    steps = dict(reward=f(T, n), done=torch.zeros((T, n), dtype=torch.uint8, device=DEV), values=f(T + 1, n))
    outs = dict(grad_logits=f(n, V), grad_values=f(n), log_probs=f(n), entropies=f(n), stats=f(7), workspace=torch.zeros((1 << 20,), dtype=torch.uint8, device=DEV))
    adv, ret, values = f(T, n), f(T, n), f(n)

    class Float:                                        # (a number that the compiled path leaves to Python)
        def __float__(self):
            return 1.0

    for one in (1.0, Float()):
        for call, written, read in ((lambda: env.pcgrl_sample(x, u, temperature=one, actions=a, log_probs=lp), [a, lp], [x, u]),
                                    (lambda: env.pcgrl_advantages(*steps.values(), one, .9, advantages=adv, returns=ret), [adv, ret], list(steps.values())),
                                    (lambda: env.pcgrl_policy_loss(x, a, u, old_log_probs=lp, values=values, returns=u, temperature=one, **outs), list(outs.values()), [x, a, u, lp, values])):
            before = [t._version for t in written], [t._version for t in read]
            call()
            assert all(t._version > v for t, v in zip(written, before[0])) and [t._version for t in read] == before[1]
    with torch.inference_mode():
        y, b = torch.randn((n, V), device=DEV), torch.zeros((n,), dtype=torch.int32, device=DEV)
    env.pcgrl_sample(y, u, actions=b)                   # (those have no version)
    env.pcgrl_policy_loss(y, b, u, grad_logits=y)


def test_a_step_counts_as_a_change_of_its_actions():
    e = binding.Pcgrl(wl.workload("dungeon32", batch=8), 0)
    e.pcgrl_reset(1)
    x, u, a, lp = torch.zeros((8, 7), device=DEV), torch.rand((8,), device=DEV), torch.zeros((8,), dtype=torch.int32, device=DEV), torch.zeros((8,), device=DEV)
    before = a._version, lp._version
    e.pcgrl_step_logits(x, u, actions=a, log_probs=lp)
    assert a._version > before[0] and lp._version > before[1]
    e.close()


def test_a_gradient_of_values_needs_values(env):
    x, a, adv = torch.zeros((5, 7), device=DEV), torch.zeros((5,), dtype=torch.int32, device=DEV), torch.zeros((5,), device=DEV)
    with pytest.raises(binding.PcgrlError):
        env.pcgrl_policy_loss(x, a, adv, grad_values=torch.zeros((5,), device=DEV))


def test_step_logits_refuses_outputs_in_one_place():
    """The step would read actions where it writes; what the draw reads may be written by the step."""
    e, other = (binding.Pcgrl(wl.workload("dungeon32", batch=40), 0) for _ in range(2))
    size = math.prod(e.obs_shape)
    room = torch.zeros((size,), dtype=torch.uint8, device=DEV)
    g = torch.Generator(DEV).manual_seed(1)
    x, u = torch.randn((40, e.K), generator=g, device=DEV), torch.rand((40,), generator=g, device=DEV)
    for one in (e, other):
        one.pcgrl_reset(5)
    obs, at = room.view(e.obs_shape), (size - 160) // 4 * 4
    inside = room[at:at + 160]
    f = lambda n=40: torch.zeros((n,), device=DEV)  # noqa: E731
    ints, floats, flags = inside.view(torch.int32), inside.view(torch.float32), inside[:40]
    wide = f(60)
    for more in (dict(obs=obs, actions=ints), dict(obs=obs, log_probs=floats), dict(reward=floats, actions=ints), dict(done=flags, actions=ints), dict(done=inside[120:], log_probs=floats),
                 dict(reward=wide[20:], log_probs=wide[:40])):
        with pytest.raises(binding.PcgrlError, match="configuration field"):
            e.pcgrl_step_logits(x, u, **more)
    reward, done = f(), torch.zeros((40,), dtype=torch.uint8, device=DEV)
    want = e.pcgrl_step_logits(x, u, obs, reward, done)
    got = other.pcgrl_step_logits(x, u, reward=u)       # (the numbers have been read by then)
    assert all(torch.equal(p, q) for p, q in zip(got, want)) and torch.equal(u, reward)
    assert torch.equal(other.pcgrl_observe(), obs)
    for one in (e, other):
        one.close()
