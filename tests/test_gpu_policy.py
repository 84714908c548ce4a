"""The policy's operators on the GPU against the plain 64-bit statements of policy_oracle: actions drawn from
logits, advantages of rollouts, the policy loss and its gradients (needs an MI355X).

Tolerances.  A result is rounded once to its type: half a step, eps / 2 of the value.  What is computed in
32 bits before that (the parts of a gradient) takes at most eight roundings of its size, 8 * 2^-24.
Everything else is computed in 64 bits; the weights that actions are drawn by are rounded to 2^-39 of the
largest one, n of them to n * 2^-39 of their sum, and an action may differ only where its target is
that near to a border."""
import math

import numpy as np
import pytest
import torch

import oracle
import policy_oracle
from paper_2408_12525_amd import binding, workloads as wl

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda", 0)
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF = {t: torch.finfo(t).eps / 2 for t in TYPES.values()}
TINY = {torch.float32: 2.**-149, torch.bfloat16: 2.**-133, torch.float16: 2.**-24}   # the smallest steps
CLASSES = [1, 2, 3, 7, 8, 9, 31, 64, 65, 200, 512, 513, 1000, 2047, 2048, 2049, 4097, 8192, 8193, 16384, 16385, 28672, 32768]


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


def rows_for(V):
    return 37 if V <= 64 else 9 if V <= 4096 else 3


def make_logits(rng, n, V, dtype, pad=0, spread=1.5):
    store = gpu(rng.normal(size=(n, V + pad)) * spread, dtype)
    return store[:, :V]


def make_mask(rng, n, V):
    mask = (rng.random((n, V)) < .7).astype(np.uint8)
    mask[np.arange(n), rng.integers(0, V, n)] = 1
    mask[n // 2] = 0                                    # nothing may be chosen there
    return mask


def check_sample(env, logits, mask, u, settled=.6, **how):
    """Actions of rows whose target is `sure` to be inside its class, which more than `settled` of them have to be."""
    n, V = logits.shape
    actions, logps = env.pcgrl_sample(logits, gpu(u, torch.float32), mask=None if mask is None else gpu(mask), **how)
    want, want_lp, room = policy_oracle.sample(wide64(logits), mask, u, **how)
    actions, logps = actions.cpu().numpy(), wide64(logps)
    sure = room > V * 2.**-39 + 1e-12
    assert sure.mean() > settled
    assert np.array_equal(actions[sure], want[sure])
    lp = want_lp[sure]
    assert np.all(np.abs(logps[sure] - lp) <= np.abs(lp) * HALF[torch.float32] + V * 2.**-39 + 1e-12)
    return actions, logps


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", CLASSES)
def test_actions_drawn(env, V, dtype):
    rng = np.random.default_rng(V)
    n = rows_for(V)
    for masked, pad, how in [(False, 0, {}), (True, 3, dict(temperature=.7)), (True, 0, dict(top_k=max(1, V // 3), temperature=1.3)), (False, 5, dict(top_p=.8)),
                             (True, 0, dict(min_p=.05)), (False, 0, dict(top_k=5, top_p=.6, min_p=.01)), (True, 1, dict(temperature=0.)),
                             (False, 0, dict(top_k=V + 3, top_p=1.5)), (True, 0, dict(top_k=1))]:
        u = rng.random(n).astype(np.float32)
        u[0] = 0.
        u[-1] = 1 - 2.**-24
        check_sample(env, make_logits(rng, n, V, TYPES[dtype], pad), make_mask(rng, n, V) if masked else None, u, **how)


@pytest.mark.parametrize("V", [1, 2, 4, 8, 64, 128, 512, 1024, 4096, 16384, 32768])
def test_equal_logits_are_drawn_in_order(env, V):
    """Equal weights, and as many as a power of two: every border is a number that is held exactly, and the
    uniform numbers lie on them.  Ties of the truncations go to the lowest indices."""
    n = min(V, 64)
    u = (np.arange(n) / n).astype(np.float32)
    x = torch.full((n, V), -2.5, device=DEV)
    at = lambda **how: env.pcgrl_sample(x, gpu(u), **how)[0].cpu().numpy().tolist()  # noqa: E731
    assert at() == [int(v * V) for v in u]
    if V >= 4:
        for how in (dict(top_k=V // 4), dict(top_p=.25), dict(top_k=V // 2, top_p=.5), dict(top_k=V // 4, top_p=.999, min_p=1.)):
            kept = math.ceil(.999 * (V // 4)) if "min_p" in how else V // 4     # (the classes that it takes to reach the share)
            assert at(**how) == [int(v * kept) for v in u], how
    assert at(temperature=0.) == [0] * n
    # the larger half behind, two values
    if V >= 16:
        x[:, V // 2:] = 3.
        for how in (dict(top_k=V // 8), dict(top_p=2.**-3, temperature=.01), dict(temperature=.01, top_k=V // 4, top_p=.5)):
            assert at(**how) == [V // 2 + int(v * (V // 8 if how.get("top_p") != .125 else V // 16)) for v in u], how
        assert at(temperature=0.) == [V // 2] * n


@pytest.mark.parametrize("V", [1, 5, 8, 40, 300, 1500, 5000, 20000])
@pytest.mark.parametrize("how", [dict(), dict(temperature=0.), dict(top_k=2, top_p=.9, min_p=.01)], ids=["plain", "best", "cut"])
def test_rows_without_a_choice_and_odd_values(env, V, how):
    inf, nan = math.inf, math.nan
    x = torch.zeros((9, V), device=DEV)
    mask = torch.ones((9, V), dtype=torch.bool, device=DEV)
    mask[0] = False                                     # nothing allowed
    x[1] = -inf                                         # the same
    x[2, V - 1] = nan
    x[3, V // 2] = inf
    x[4], mask[4, 1:] = nan, False                      # NaN in masked places only
    x[4, 0] = 1.
    x[5, 1:], mask[5, 1:] = inf, False
    x[6] = torch.finfo(torch.float32).min               # the lowest value is a value
    x[7] = -inf                                         # one class left, the last
    x[7, -1] = -1e30
    x[8] = torch.finfo(torch.float32).max
    u = torch.full((9,), .25, device=DEV)
    a, lp = env.pcgrl_sample(x, u, mask=mask, **how)
    a, lp = a.cpu().tolist(), lp.cpu().tolist()
    kept = V if not how else 1 if "temperature" in how else min(2, V)
    assert a == [-1, -1, -1, -1, 0, 0, int(.25 * kept), V - 1, int(.25 * kept)]
    flat = -math.log(V) if how.get("temperature") != 0 else 0.
    assert lp[0] == lp[1] == 0 and math.isnan(lp[2]) and math.isnan(lp[3]) and lp[4] == lp[5] == lp[7] == 0
    assert abs(lp[6] - flat) <= 1e-6 * (1 + abs(flat)) and lp[6] == lp[8]


@pytest.mark.parametrize("V", [300, 1000, 1024, 2500, 8192, 20000, 32768])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_classes_close_together(env, V, dtype):
    """Truncations where a great many logits are equal or next to each other, beside few that are far away: values that
    are one step apart, down to the smallest there are, two values, a few values, zeros of both signs, huge ones."""
    rng = np.random.default_rng(V)
    t = TYPES[dtype]
    step = 2.**-23 if dtype == "f32" else 2.**-7
    rows = [1 + step * rng.integers(0, 2, V), 1 + step * rng.integers(0, 40, V), step * rng.integers(-3, 3, V), rng.integers(0, 3, V) * 1., np.where(rng.random(V) < .5, 0., -0.),
            rng.integers(0, 900, V) * 2.**-126, rng.integers(0, 5, V) * 2.**-130, np.where(rng.random(V) < .01, 9., 1 + step * rng.integers(0, 2, V)), 3e38 - 1e37 * rng.integers(0, 3, V),
            np.where(rng.random(V) < .5, -1e9, 0.), np.where(np.arange(V) == V // 2, 3e38, -3e38), np.full(V, -7.)]
    x = gpu(np.stack(rows), torch.float64).to(t)
    # The first numbers times 1000 are whole, so that with equal weights of 20 000 classes each target is a class's border to within the rounding of
    # the number to 32 bits (2^-25, below the 2^-24.7 that V 2^-39 is): such rows are no test of the action, only the others and the second numbers are.
    u = (np.arange(len(rows)) * .079 + .03).astype(np.float32)
    between = ((np.arange(len(rows)) + 1) * .6180339887 % 1).astype(np.float32)
    for how in (dict(top_k=V // 2), dict(top_k=40), dict(top_p=.6), dict(top_k=V - 1, top_p=.9), dict(top_k=V // 3, top_p=.5, min_p=.9), dict(temperature=1e6, top_p=.3), dict(temperature=1e-6, top_k=200)):
        check_sample(env, x, None, u, settled=-1, **how)
        check_sample(env, x, None, between, **how)


@pytest.mark.parametrize("V,n", [(200, 5000), (500, 3000), (1024, 900), (4100, 400), (8192, 400), (8193, 400), (15400, 400), (16384, 400), (30000, 400), (31000, 400),
                                 (600, 2**22 + 7), (1030, 2**20 + 5), (4100, 2**20 + 300)])
def test_a_row_is_drawn_alike_whatever_is_drawn_with_it(env, V, n):
    """However many rows there are, which decides on the threads that a row gets, and also where workgroups take several in turn."""
    g = torch.Generator(DEV).manual_seed(V)
    for dtype in TYPES.values() if n < 10000 else [torch.bfloat16]:
        x = torch.empty((n, V), dtype=dtype, device=DEV).normal_(0, 2, generator=g)
        u = torch.rand((n,), generator=g, device=DEV)
        for how in ({}, dict(top_p=.8), dict(top_k=30, top_p=.9), dict(top_k=V // 2, min_p=.01)):
            actions, logps = env.pcgrl_sample(x, u, **how)
            for rows in (slice(0, 5), slice(n // 2, n // 2 + 3), slice(n - 4, n)):
                few, their = env.pcgrl_sample(x[rows], u[rows], **how)
                assert torch.equal(actions[rows], few) and torch.equal(logps[rows], their)
            few = actions[-4:].cpu().numpy()
            want, _, room = policy_oracle.sample(wide64(x[-4:]), None, u[-4:].cpu().numpy(), **how)
            sure = room > V * 2.**-39 + 1e-12
            assert np.array_equal(few[sure], want[sure])


def test_uniform_numbers_outside_and_zeros_of_both_signs(env):
    x = torch.zeros((6, 4), device=DEV)
    u = torch.tensor([-1., 1., 2., math.nan, math.inf, -math.inf], device=DEV)
    assert env.pcgrl_sample(x, u)[0].tolist() == [0, 3, 3, 0, 3, 0]
    for V in (6, 60, 700):
        z = torch.zeros((4, V), device=DEV)
        z[:, 0] = -0.
        assert env.pcgrl_sample(z, None, temperature=0.)[0].tolist() == [0] * 4
        assert env.pcgrl_sample(z, torch.full((4,), .9, device=DEV), top_k=1)[0].tolist() == [0] * 4
        h = z.half()
        assert env.pcgrl_sample(h, torch.full((4,), .9, device=DEV), top_k=1)[0].tolist() == [0] * 4


def test_float16_order_down_to_the_smallest(env):
    x = torch.tensor([[6e-8, 1.2e-7, 0., -6e-8, 65504., -65504., 65472., 1.2e-7, 6e-8]], dtype=torch.float16, device=DEV)
    best = torch.argsort(-x[0].float(), stable=True).tolist()
    for k in range(1, 10):
        for dtype in (torch.float16, torch.float32):
            got = {int(env.pcgrl_sample(x.to(dtype), torch.tensor([u], device=DEV), top_k=k, temperature=1e9)[0]) for u in np.linspace(0, .999, 64, dtype=np.float32).tolist()}
            assert got == set(best[:k])


def test_many_rows_and_one_mask_for_all(env):
    rng = np.random.default_rng(1)
    for n, V in ((300001, 2), (70001, 9), (5000, 100)):
        x = make_logits(rng, n, V, torch.float32)
        u = rng.random(n).astype(np.float32)
        mask = np.ones(V, np.uint8)
        mask[V // 2] = 0
        a, lp = env.pcgrl_sample(x, gpu(u), mask=gpu(mask))
        b, lp2 = env.pcgrl_sample(x, gpu(u), mask=gpu(np.broadcast_to(mask, (n, V)).copy()))
        assert torch.equal(a, b) and torch.equal(lp, lp2) and not bool((a == V // 2).any())
        w = np.exp(wide64(x)) * mask
        c = w.cumsum(1)
        want = (c > (u * c[:, -1])[:, None]).argmax(1)
        assert (a.cpu().numpy() != want).mean() < 1e-5    # (a running sum of 64-bit weights, next to a border)
    assert env.pcgrl_sample(torch.empty((0, 5), device=DEV), torch.empty((0,), device=DEV))[0].shape == (0,)


@pytest.mark.parametrize("V", [2, 3, 7, 40, 100, 128, 129, 256, 300, 512, 700, 1024, 3000])
@pytest.mark.parametrize("dtype", TYPES)
def test_draws_do_not_depend_on_how_many_rows_there_are(env, V, dtype):
    """The kernel is chosen by the number of rows, too: the same rows in a large and in a small batch, one after the other and last."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(V)
    n = 9001 if V <= 1024 else 600
    x = (torch.randn((n, V), generator=gen, device=DEV) * 2).to(TYPES[dtype])
    u = torch.rand((n,), generator=gen, device=DEV)
    mask = (torch.rand((n, V), generator=gen, device=DEV) < .8).to(torch.uint8)
    for how in (dict(), dict(top_k=5), dict(top_p=.7, min_p=.01), dict(top_k=max(1, V // 2), top_p=.9), dict(temperature=0.)):
        a, lp = env.pcgrl_sample(x, u, mask=mask, **how)
        for at in (slice(0, 3), slice(n - 5, n), slice(100, 101)):
            b, lp2 = env.pcgrl_sample(x[at], u[at].contiguous(), mask=mask[at], **how)
            # (the logarithm of the same sum, which is rounded to float32 once)
            assert torch.equal(a[at], b) and torch.allclose(lp[at], lp2, rtol=2.**-23, atol=1e-9), how


def test_rows_beyond_32_bit_offsets(env):
    """Rows so far apart that the last ones lie more than 2^32 bytes and 2^31 elements behind the first."""
    n, V, stride = 70001, 33, 32768
    store = torch.empty((n, stride), dtype=torch.bfloat16, device=DEV)
    x = store[:, :V]
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1)
    close = torch.randn((n, V), generator=gen, device=DEV).bfloat16()
    x.copy_(close)
    u = torch.rand((n,), generator=gen, device=DEV)
    for how in (dict(), dict(top_k=3, top_p=.9)):
        got, want = env.pcgrl_sample(x, u, **how), env.pcgrl_sample(close, u, **how)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    act = want[0]
    adv = torch.randn((n,), generator=gen, device=DEV)
    want = env.pcgrl_policy_loss(close, act, adv)
    grads = torch.empty((n, stride), dtype=torch.bfloat16, device=DEV)[:, :V]
    got = env.pcgrl_policy_loss(x, act, adv, grad_logits=grads)
    assert torch.equal(got["stats"], want["stats"]) and torch.equal(got["grad_logits"], want["grad_logits"])


# ---- the loss

def make_loss(rng, n, V, dtype, masked=True, pad=0, clipped=True, critic=True):
    logits = make_logits(rng, n, V, dtype, pad)
    mask = make_mask(rng, n, V) if masked else None
    x, _ = policy_oracle.allowed_logits(wide64(logits), mask)
    actions, _, _ = policy_oracle.sample(wide64(logits), mask, rng.random(n))
    old = np.zeros(n)
    for r in range(n):
        if actions[r] >= 0:
            old[r] = x[r, actions[r]] - np.log(np.exp(x[r]).sum())
    s = dict(logits=logits, mask=mask, actions=actions, advantages=rng.normal(size=n).astype(np.float32),
             old=(old + rng.normal(size=n) * .25).astype(np.float32) if clipped else None)
    if critic:
        s["values"], s["returns"] = gpu(rng.normal(size=n) * 3, dtype), (rng.normal(size=n) * 3).astype(np.float32)
    return s


def run_loss(env, s, **how):
    up = lambda k: None if s.get(k) is None else s[k] if isinstance(s[k], torch.Tensor) else gpu(s[k])  # noqa: E731
    return env.pcgrl_policy_loss(s["logits"], up("actions"), up("advantages"), old_log_probs=up("old"), mask=up("mask"), values=up("values"), returns=up("returns"), **how)


def plain_loss(s, **how):
    return policy_oracle.loss(wide64(s["logits"]), s["mask"], s["actions"], s["advantages"], old=s["old"],
                              values=None if s.get("values") is None else wide64(s["values"]), returns=s.get("returns"), **how)


def check_gradient(got, want, size, dtype):
    far = np.abs(wide64(got) - want) - (np.abs(want) * HALF[dtype] + size * 8 * 2.**-24 * (1 + HALF[dtype]) + TINY[dtype] / 2)
    assert far.max(initial=-1) <= 0, far.max()


def check_loss(env, s, dtype, **how):
    n = len(s["actions"])
    lp, h = torch.full((n,), 7., device=DEV), torch.full((n,), 7., device=DEV)
    got = run_loss(env, s, log_probs=lp, entropies=h, **how)
    want = plain_loss(s, **dict(dict(scale=1 / max(n, 1)), **how))
    assert want["room"].min(initial=1) > 1e-9
    check_gradient(got["grad_logits"], want["grad_logits"], want["size"], dtype)
    if s.get("values") is not None:
        check_gradient(got["grad_values"], want["grad_values"], np.abs(want["grad_values"]), dtype)
    for t, w in ((lp, want["log_probs"]), (h, want["entropies"])):
        assert np.all(np.abs(wide64(t) - w) <= np.abs(w) * HALF[torch.float32] + 1e-11)
    sums = np.concatenate([[want["loss"]], want["sums"]])
    parts = np.concatenate([[want["loss_parts"]], want["parts"]])
    assert np.all(np.abs(wide64(got["stats"]) - sums) <= np.abs(sums) * HALF[torch.float32] + parts * 1e-12)
    return got


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", CLASSES)
def test_policy_loss(env, V, dtype):
    rng = np.random.default_rng(100 + V)
    n, t = rows_for(V), TYPES[dtype]
    for k, how in enumerate([dict(), dict(temperature=.7, entropy_coef=.2, scale=64.), dict(clip_low=.1, clip_high=.5, value_coef=0.), dict(entropy_coef=0., scale=-3.), dict(entropy_coef=-.5)]):
        check_loss(env, make_loss(rng, n, V, t, masked=k % 2 == 0, pad=(0, 3, 8, 1, 0)[k], clipped=k != 3, critic=k != 2), t, **how)


@pytest.mark.parametrize("V", [2, 7, 12, 90, 600])
def test_policy_gradients_are_the_differences_of_the_loss(env, V):
    """Against differences of the plain loss in 64 bits, which know nothing of the gradient's formula: second
    order in h = 2^-16, so within h^2 times a third derivative of below 8, and 2^-40 / h of rounding."""
    rng = np.random.default_rng(V)
    s = make_loss(rng, 5, V, torch.float32)
    how, h = dict(temperature=.8, entropy_coef=.3, value_coef=.6, scale=1.), 2.**-16
    got = run_loss(env, s, **how)
    x, v = wide64(s["logits"]), wide64(s["values"])
    f = lambda x, v: policy_oracle.loss(x, s["mask"], s["actions"], s["advantages"], old=s["old"], values=v, returns=s["returns"], **how)["loss"]  # noqa: E731
    size = plain_loss(s, **how)["size"]
    for i in range(5):
        for j in rng.permutation(V)[:20]:
            e = np.zeros_like(x)
            e[i, j] = h
            d = (f(x + e, v) - f(x - e, v)) / (2 * h)
            assert abs(d - float(got["grad_logits"][i, j])) <= 8 * h * h + 2.**-40 / h * 64 + (8 * size[i, j] + abs(d)) * 2.**-24
        e = np.zeros_like(v)
        e[i] = h
        d = (f(x, v + e) - f(x, v - e)) / (2 * h)
        assert abs(d - float(got["grad_values"][i])) <= 2.**-40 / h * 64 + abs(d) * 2.**-23


@pytest.mark.parametrize("V", [1, 5, 33, 300, 1500, 5000, 12000, 20000])
def test_rows_that_do_not_count(env, V):
    """Padded rows with anything in them, actions that are no class or may not be chosen, NaN where it is masked."""
    rng = np.random.default_rng(V)
    n, t = 10, torch.float32
    s = make_loss(rng, n, V, t, masked=False, clipped=True)
    s["mask"] = np.ones((n, V), np.uint8)
    s["actions"][:3] = -1, V, 2**31 - 1
    s["mask"][3, s["actions"][3]] = 0                   # its action may not be chosen
    s["mask"][4] = 0
    s["actions"][5] = -2**31
    s["logits"][0] = math.nan
    s["logits"][6], s["mask"][6] = math.nan, 0
    s["logits"][6, V // 2], s["mask"][6, V // 2], s["actions"][6] = 1., 1, V // 2
    s["logits"][7, :] = -math.inf
    for r in (0, 1, 2, 3, 4, 5, 7):
        s["advantages"][r], s["old"][r], s["returns"][r], s["values"][r] = math.nan, math.inf, math.nan, -math.inf
    out = torch.full((n, V + 4), 5., device=DEV)
    lp = torch.full((n,), 7., device=DEV)
    got = run_loss(env, s, grad_logits=out[:, :V], log_probs=lp, scale=1.)
    want = plain_loss(s, scale=1.)
    check_gradient(out[:, :V], want["grad_logits"], want["size"], t)
    check_gradient(got["grad_values"], want["grad_values"], np.abs(want["grad_values"]), t)
    assert bool((out[:, V:] == 5.).all())
    assert got["stats"][1] == 3 and not bool((out[[0, 1, 2, 3, 4, 5, 7], :V] != 0).any()) and not bool((lp[[0, 1, 2, 3, 4, 5, 7]] != 0).any())
    assert bool(torch.isfinite(got["stats"]).all())


@pytest.mark.parametrize("V", [3, 50, 400, 1100, 9000])
def test_nan_and_infinity_show_in_the_row_alone(env, V):
    rng = np.random.default_rng(V)
    for odd in (math.nan, math.inf):
        s = make_loss(rng, 6, V, torch.float32, masked=False)
        s["logits"][2, V - 1] = odd
        got = run_loss(env, s, scale=1.)
        bad = torch.isnan(got["grad_logits"])
        assert bool(bad[2].any()) and bool(bad[2, int(s["actions"][2])]) and not bool(bad[[0, 1, 3, 4, 5]].any()) and math.isnan(float(got["stats"][0]))


@pytest.mark.parametrize("V", [2, 7, 60, 500, 1200, 6000, 16000, 28672])
def test_loss_in_place_is_the_same_and_sums_repeat(env, V):
    rng = np.random.default_rng(V)
    n = 5000 if V < 10 else 200
    logits = gpu(rng.normal(size=(n, V)), torch.bfloat16)
    act, adv = gpu(rng.integers(0, V, n), torch.int32), gpu(rng.normal(size=n), torch.float32)
    old = gpu(rng.normal(-math.log(V), .3, size=n), torch.float32)
    val, ret = gpu(rng.normal(size=n), torch.bfloat16), gpu(rng.normal(size=n), torch.float32)
    call = lambda x, v, **more: env.pcgrl_policy_loss(x, act, adv, old_log_probs=old, values=v, returns=ret, **more)  # noqa: E731
    want, again = call(logits, val), call(logits, val)
    assert all(torch.equal(want[k], again[k]) for k in want)
    x, v = logits.clone(), val.clone()
    got = call(x, v, grad_logits=x, grad_values=v)
    assert got["grad_logits"] is x and torch.equal(x, want["grad_logits"]) and torch.equal(v, want["grad_values"]) and torch.equal(got["stats"], want["stats"])


def test_cross_entropy_and_scaled_gradients_in_autograd(env):
    """With advantages of one and no old policy it is the cross entropy, against torch's in float32 on the CPU; the
    gradient goes into a network through autograd."""
    rng = np.random.default_rng(4)
    n, V, d = 300, 70, 24
    feats, head = gpu(rng.normal(size=(n, d)), torch.float32), gpu(rng.normal(size=(d, V)) * .3, torch.float32).requires_grad_()
    act = gpu(rng.integers(0, V, n), torch.int32)
    logits = feats @ head
    got = env.pcgrl_policy_loss(logits, act, torch.ones(n, device=DEV), entropy_coef=0.)
    logits.backward(got["grad_logits"])
    h = head.detach().cpu().double().requires_grad_()
    want = torch.nn.functional.cross_entropy(feats.cpu().double() @ h, act.cpu().long())
    want.backward()
    assert abs(float(got["stats"][0]) - float(want)) < 1e-5 * float(want)
    assert (head.grad.cpu().double() - h.grad).abs().max() < 1e-6     # sums of 300 products of a size of 1/300 in 32 bits
    assert float(got["stats"][6]) == 0 and float(got["stats"][5]) == 0


def test_no_rows(env):
    e = lambda *s, t=torch.float32: torch.empty(s, dtype=t, device=DEV)  # noqa: E731
    got = env.pcgrl_policy_loss(e(0, 9), e(0, t=torch.int32), e(0))
    assert got["stats"].tolist() == [0.] * 7 and got["grad_logits"].shape == (0, 9)


# ---- advantages

@pytest.mark.parametrize("T,n", [(1, 1), (2, 1), (1, 300), (3, 5), (7, 64), (8, 65), (9, 63), (33, 17), (64, 16), (100, 1000), (257, 31), (1000, 3), (4096, 2), (513, 257), (31, 4100), (40, 20001),
                                 (10001, 1), (5000, 33), (4097, 64), (2049, 65), (2600, 700), (2100, 2100), (30000, 5), (64, 131073), (20, 32768), (1, 1), (130000, 1)])
def test_advantages(env, T, n):
    rng = np.random.default_rng(T * 1000 + n)
    for k, dtype in enumerate(TYPES.values()):
        reward = (rng.integers(-12, 13, (T, n)) * (rng.random((T, n)) < .5)).astype(np.float32)
        done = (rng.random((T, n)) < (.01, .3, 0.)[k]).astype(np.uint8) * 255
        values = gpu(rng.normal(size=(T + 1, n)) * 4 + 5, dtype)
        discount, trace = [(.99, .95), (1., 1.), (.9, 0.)][k]
        adv, ret = env.pcgrl_advantages(gpu(reward), gpu(done), values, discount, trace)
        want, back = policy_oracle.advantages(reward, done, wide64(values), discount, trace)
        room = 1e-13 * np.abs(want).max()              # of sums in 64 bits, in whatever order
        assert np.all(np.abs(wide64(adv) - want) <= np.abs(want) * HALF[torch.float32] + room)
        assert np.all(np.abs(wide64(ret) - back) <= np.abs(back) * HALF[torch.float32] + room)


@pytest.mark.parametrize("T,n", [(5, 3), (300, 40), (2000, 2)])
def test_nothing_passes_the_end_of_an_episode(env, T, n):
    """What stands behind the end of an episode does not count, NaN and infinity included."""
    rng = np.random.default_rng(T)
    reward, values = rng.normal(size=(T, n)).astype(np.float32), rng.normal(size=(T + 1, n)).astype(np.float32)
    done = np.zeros((T, n), np.uint8)
    cut = T // 2
    done[cut - 1] = 1
    want, back = env.pcgrl_advantages(gpu(reward), gpu(done), gpu(values), .99, .95)
    reward[cut:], values[cut:] = math.nan, math.inf
    got, got_back = env.pcgrl_advantages(gpu(reward), gpu(done).bool(), gpu(values), .99, .95)
    assert torch.equal(got[:cut], want[:cut]) and torch.equal(got_back[:cut], back[:cut]) and bool(torch.isfinite(got[:cut]).all())
    values[:], done[-1] = 1., 1
    values[T], reward[:] = math.nan, 1.
    assert bool(torch.isfinite(env.pcgrl_advantages(gpu(reward), gpu(done), gpu(values), .99, .95)[0]).all())


@pytest.mark.parametrize("T,n", [(5, 3), (40, 70), (300, 40), (2000, 2), (6000, 3), (33, 5000)])
@pytest.mark.parametrize("discount,trace", [(.99, .95), (.5, .5), (1., 0.), (0., 1.), (1e-200, 1.)])
def test_infinite_and_missing_rewards(env, T, n, discount, trace):
    """NaN and infinity reach every step before them in their episode, however far, and no others: with a trace of 0 too, as
    0 times infinity is NaN."""
    rng = np.random.default_rng(T)
    reward, values = rng.normal(size=(T, n)).astype(np.float32), rng.normal(size=(T + 1, n)).astype(np.float32)
    done = np.zeros((T, n), np.uint8)
    done[T // 3, ::2] = 1
    reward[T - 1, 0], reward[T - 2, 1 % n], values[T, 2 % n] = np.inf, np.nan, -np.inf
    reward[T // 2, n // 2] = -np.inf
    adv, ret = env.pcgrl_advantages(gpu(reward), gpu(done), gpu(values), discount, trace)
    with np.errstate(invalid="ignore"):
        want, back = policy_oracle.advantages(reward, done, values, discount, trace)
    for got, exact in ((wide64(adv), want), (wide64(ret), back)):
        plain = np.isfinite(exact)
        assert np.array_equal(got[~plain], exact[~plain], equal_nan=True) and (~plain).any()
        room = 1e-13 * np.abs(exact[plain]).max()
        assert np.all(np.abs(got[plain] - exact[plain]) <= np.abs(exact[plain]) * HALF[torch.float32] + room)


def test_no_steps_and_no_environments(env):
    for T, n in ((0, 4), (4, 0)):
        e = lambda t, steps=T: torch.empty((steps, n), dtype=t, device=DEV)  # noqa: E731
        assert env.pcgrl_advantages(e(torch.float32), e(torch.uint8), e(torch.float32, T + 1), .9, .9)[0].shape == (T, n)


# ---- together

def test_a_policy_in_the_loop(env):
    """Steps by a policy's logits, then advantages and the loss's gradient, as a training loop runs them: the
    environments agree with the oracle of the environments, the rest with the plain statements."""
    T, B = 12, 50
    cfg = wl.workload("dungeon32", batch=B, max_steps=7)
    gpu_env, cpu = binding.Pcgrl(cfg, 0), oracle.Oracle(cfg)
    K, rng = gpu_env.K, np.random.default_rng(8)
    obs = gpu_env.new_obs()
    gpu_env.pcgrl_reset(3, obs)
    cpu.reset(3)
    reward, done = torch.empty((T, B), device=DEV), torch.empty((T, B), dtype=torch.uint8, device=DEV)
    actions, logps = torch.empty((T, B), dtype=torch.int32, device=DEV), torch.empty((T, B), device=DEV)
    logits = torch.empty((T, B, K), dtype=torch.bfloat16, device=DEV)
    head = gpu(rng.normal(size=(obs[0].numel(), K)) * .2, torch.float32)
    mask = np.ones((B, K), np.uint8)
    mask[:, 2] = 0
    mask[4] = 0                                         # this level is left alone: action -1 is a bad action
    for t in range(T):
        logits[t] = (obs.reshape(B, -1).float() @ head).bfloat16()
        u = gpu(rng.random(B), torch.float32)
        got = gpu_env.pcgrl_step_logits(logits[t], u, obs, reward[t], done[t], mask=gpu(mask), temperature=1.2, top_p=.95, actions=actions[t], log_probs=logps[t])
        assert got[0].data_ptr() == actions[t].data_ptr()
        want, want_lp, room = policy_oracle.sample(wide64(logits[t]), mask, wide64(u), temperature=1.2, top_p=.95)
        sure = room > 1e-9
        assert np.array_equal(actions[t].cpu().numpy()[sure], want[sure])
        o, r, d = cpu.step(actions[t].cpu().numpy())
        assert np.array_equal(obs.cpu().numpy(), o) and np.array_equal(done[t].cpu().numpy(), d) and np.abs(reward[t].cpu().numpy() - r).max() <= 1e-6
    assert gpu_env.pcgrl_bad_action_count() == T
    values = gpu(rng.normal(size=(T + 1, B)), torch.bfloat16)
    adv, ret = gpu_env.pcgrl_advantages(reward, done, values, .99, .95)
    want, back = policy_oracle.advantages(wide64(reward), done.cpu().numpy(), wide64(values), .99, .95)
    assert np.all(np.abs(wide64(adv) - want) <= np.abs(want) * HALF[torch.float32] + 1e-12)
    adv = (adv / 40).contiguous()
    flat = lambda t: t.reshape((T * B,) + tuple(t.shape[2:])).contiguous()  # noqa: E731
    s = dict(logits=flat(logits), mask=np.tile(mask, (T, 1)), actions=flat(actions).cpu().numpy(), advantages=flat(adv).cpu().numpy(), old=flat(logps).cpu().numpy(),
             values=flat(values[:T]), returns=flat(ret).cpu().numpy())
    got = check_loss(gpu_env, s, torch.bfloat16, temperature=1.2)
    # the policy is still the one that acted: every ratio is 1 but for the rounding of the old one
    assert float(got["stats"][1]) == T * (B - 1) and float(got["stats"][6]) == 0 and abs(float(got["stats"][5])) < 1e-6
    gpu_env.close()


def test_step_logits_is_the_sample_and_the_step():
    cfg = wl.workload("maze16", batch=300)
    one, two = binding.Pcgrl(cfg, 0), binding.Pcgrl(cfg, 0)
    rng = np.random.default_rng(2)
    outs = [(e.new_obs(), torch.empty(300, device=DEV), torch.empty(300, dtype=torch.uint8, device=DEV)) for e in (one, two)]
    for e in (one, two):
        e.pcgrl_reset(5)
    for how in (dict(), dict(temperature=0.), dict(temperature=.5, top_k=2), dict(min_p=.2, top_p=.9)):
        x, u = gpu(rng.normal(size=(300, 6)), torch.float16)[:, :4], gpu(rng.random(300), torch.float32)
        a = one.pcgrl_step_logits(x, u, *outs[0], **how)
        b = two.pcgrl_sample(x, u, **how)
        two.pcgrl_step(b[0], *outs[1])
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and all(torch.equal(p, q) for p, q in zip(*outs))
    with pytest.raises(binding.PcgrlError, match="configuration field"):
        one.pcgrl_step_logits(gpu(rng.normal(size=(300, 5)), torch.float32), u)
    with pytest.raises(binding.PcgrlError, match="300 environments"):
        one.pcgrl_step_logits(gpu(rng.normal(size=(299, 4)), torch.float32), u)
    one.close()
    two.close()


def test_captured_replayed_and_on_other_streams(env):
    """All of it in one graph, replayed with other inputs and eager work in between; and at once on two streams."""
    rng = np.random.default_rng(6)
    shapes = [(700, 7), (64, 40), (33, 700), (9, 20000)]
    inputs = [(gpu(rng.normal(size=s), torch.bfloat16), gpu(rng.random(s[0]), torch.float32)) for s in shapes]
    reward, done, values = gpu(rng.normal(size=(2000, 8)), torch.float32), gpu(rng.random((2000, 8)) < .01).to(torch.uint8), gpu(rng.normal(size=(2001, 8)), torch.float32)

    def everything():
        out = []
        for x, u in inputs:
            a, lp = env.pcgrl_sample(x, u, temperature=.9, top_p=.9, top_k=30)
            l = env.pcgrl_policy_loss(x, a, u, old_log_probs=lp)
            out += [a, lp, l["stats"], l["grad_logits"]]
        return out + list(env.pcgrl_advantages(reward, done, values, .99, .95))

    everything()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = everything()
    for k in range(4):
        for x, u in inputs:
            x.copy_(gpu(rng.normal(size=tuple(x.shape)), torch.bfloat16))
            u.copy_(gpu(rng.random(len(u)), torch.float32))
        reward.copy_(gpu(rng.normal(size=(2000, 8)), torch.float32))
        graph.replay()
        want = everything()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(held, want)), k
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for s in streams:
        with torch.cuda.stream(s):
            for _ in range(3):
                outs.append(everything())
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for o in outs for p, q in zip(o, want))


def test_binding_refuses(env):
    x, u = torch.zeros((5, 7), device=DEV), torch.zeros((5,), device=DEV)
    act, adv = torch.zeros((5,), dtype=torch.int32, device=DEV), torch.zeros((5,), device=DEV)
    bad = pytest.raises(binding.PcgrlError)
    for args, more in [((x.double(), u), {}), ((x.cpu(), u), {}), ((x[0], u), {}), ((x.t(), u), {}), ((x.t()[:5, :5], u), {}), ((x[:1].expand(5, 7), u), {}), ((x, u[:4]), {}), ((x, None), {}), ((x, u.double()), {}),
                       ((x, u.cpu()), {}), ((x, u), dict(mask=torch.ones((5, 6), dtype=torch.uint8, device=DEV))), ((x, u), dict(mask=x)), ((x, u), dict(mask=torch.ones((5, 7), dtype=torch.uint8))),
                       ((x, u), dict(temperature=-1.)), ((x, u), dict(top_p=0.)), ((x, u), dict(min_p=2.)), ((x, u), dict(top_k=-1)), ((x, u), dict(actions=u)), ((x, u), dict(log_probs=act)),
                       ((x[:, :0], u), {})]:
        with bad:
            env.pcgrl_sample(*args, **more)
    for args, more in [((x, act.long(), adv), {}), ((x, act, adv.double()), {}), ((x, act[:3], adv), {}), ((x, act, adv), dict(values=adv)), ((x, act, adv), dict(values=adv.half(), returns=adv)),
                       ((x, act, adv), dict(grad_logits=x.half())), ((x, act, adv), dict(grad_logits=x[:, :6])), ((x, act, adv), dict(stats=adv)), ((x, act, adv), dict(workspace=act)), ((x, act, adv), dict(temperature=0.)),
                       ((x, act, adv), dict(clip_low=2.)), ((x, act, adv), dict(scale=math.nan)), ((x, act, adv), dict(old_log_probs=act)), ((x, act, adv), dict(log_probs=act)), ((x, act, adv), dict(grad_logits=x[:1].expand(5, 7)))]:
        with bad:
            env.pcgrl_policy_loss(*args, **more)
    r, d, v = torch.zeros((4, 3), device=DEV), torch.zeros((4, 3), dtype=torch.uint8, device=DEV), torch.zeros((5, 3), device=DEV)
    for args, more in [((r.double(), d, v), {}), ((r, d.int(), v), {}), ((r, d, v[:4]), {}), ((r, d, v.double()), {}), ((r[0], d, v), {}), ((r, d, v), dict(advantages=r)), ((r, d, v), dict(returns=v[:4])), ((r.t(), d, v), {})]:
        with bad:
            env.pcgrl_advantages(*args, .9, .9, **more)
    with bad:
        env.pcgrl_advantages(r, d, v, 1.1, .9)
    with bad:
        env.pcgrl_advantages(r, d, v, .9, -.1)
