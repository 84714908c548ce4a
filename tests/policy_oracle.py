"""Plain 64-bit numpy statements of the policy's operators, row by row, for the tests: actions drawn from
logits, advantages of a rollout, the policy loss and its gradients."""
import math

import numpy as np


def allowed_logits(logits, mask):
    """Logits in 64 bits, -infinity where a class may not be chosen; and whether a row has a NaN or +infinity left."""
    x = np.asarray(logits, np.float64).copy()
    if mask is not None:
        x[np.broadcast_to(np.asarray(mask) == 0, x.shape)] = -np.inf
    return x, (np.isnan(x) | (x == np.inf)).any(1)


def kept_classes(x, temperature, top_k, top_p, min_p):
    """The classes of one row (largest logit finite) that the truncations keep, in ascending order, and their weights."""
    top = x.max()
    order = sorted((i for i in range(len(x)) if x[i] > -math.inf), key=lambda i: (-x[i], i))
    if top_k:
        order = order[:top_k]
    w = {i: math.exp((x[i] - top) / temperature) for i in order}
    share = top_p * math.fsum(w.values())
    kept, before = [], 0.
    for i in order:
        if not (top_p >= 1 or before < share) or not w[i] >= min_p:
            break
        kept.append(i)
        before += w[i]
    return sorted(kept), w


def sample(logits, mask, uniform, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(actions, log-probabilities, how far each target is from the border of its class, as a share of the sum)."""
    x, odd = allowed_logits(logits, mask)
    n, V = x.shape
    actions, logps, room = np.full(n, -1, np.int32), np.zeros(n), np.full(n, np.inf)
    for r in range(n):
        if odd[r]:
            logps[r] = np.nan
            continue
        if x[r].max() == -np.inf:
            continue
        if temperature == 0:
            actions[r] = int(np.argmax(x[r]))
            continue
        if top_k or top_p < 1 or min_p:
            at, w = kept_classes(x[r], temperature, top_k, top_p, min_p)
            at, weights = np.array(at), np.array([w[i] for i in at])
        else:
            at = np.flatnonzero(x[r] > -np.inf)
            weights = np.exp((x[r][at] - x[r].max()) / temperature)
        running = np.cumsum(weights)
        target = min(max(float(uniform[r]), 0.), 1 - 2.**-24) * running[-1]
        first = int(np.flatnonzero(running > target)[0])
        actions[r] = at[first]
        borders = np.concatenate([running[:-1], [np.inf]])
        room[r] = np.abs(borders - target).min() / running[-1]
        finite = x[r][x[r] > -np.inf]
        logps[r] = (x[r][at[first]] - x[r].max()) / temperature - math.log(math.fsum(np.exp((finite - x[r].max()) / temperature)))
    return actions, logps, room


def advantages(reward, done, values, discount, trace):
    reward, values = np.asarray(reward, np.float64), np.asarray(values, np.float64)
    out, after = np.empty_like(reward), np.zeros(reward.shape[1])
    for t in range(len(reward) - 1, -1, -1):
        ends = np.asarray(done[t]) != 0
        error = reward[t] + np.where(ends, 0., discount * values[t + 1]) - values[t]
        after = error + np.where(ends, 0., discount * trace * after)
        out[t] = after
    return out, out + values[:-1]


def loss(logits, mask, actions, advantages, old=None, values=None, returns=None, temperature=1.0, clip_low=0.2, clip_high=0.2,
         entropy_coef=0.01, value_coef=0.5, scale=1.0):
    """A dict: `loss`, `sums` (as the library's stats behind the loss), `grad_logits`, `grad_values`, `log_probs`,
    `entropies`, `room` (how far each ratio is from where it is clipped) and `size`, what rounding a
    gradient's parts to 32 bits goes by."""
    x, _ = allowed_logits(logits, mask)
    n, V = x.shape
    out = dict(grad_logits=np.zeros((n, V)), grad_values=np.zeros(n), log_probs=np.zeros(n), entropies=np.zeros(n), room=np.full(n, np.inf), size=np.zeros((n, V)))
    sums, parts = np.zeros(6), np.zeros(6)
    for r in range(n):
        a = int(actions[r])
        if not 0 <= a < V or x[r, a] == -np.inf:
            continue
        if np.isnan(x[r]).any() or (x[r] == np.inf).any():
            out["grad_logits"][r] = np.where(x[r] == -np.inf, 0., np.nan)
            out["log_probs"][r] = out["entropies"][r] = np.nan
            sums += np.nan
            continue
        top = x[r].max()
        y = (x[r] - top) / temperature
        p = np.exp(y)
        whole = p.sum()
        p /= whole
        logs = np.where(p > 0, y - math.log(whole), 0.)
        h = -(p * logs).sum()
        adv = float(advantages[r])
        change = 0. if old is None else logs[a] - float(old[r])
        ratio = math.exp(change)
        if old is None:
            policy, pull, clipped = -adv * logs[a], -adv, False
        else:
            bounded = min(max(ratio, 1 - clip_low), 1 + clip_high)
            policy = -min(ratio * adv, bounded * adv)
            clipped = bounded * adv < ratio * adv
            pull = 0. if clipped else -adv * ratio
            out["room"][r] = min(abs(ratio - 1 + clip_low), abs(ratio - 1 - clip_high))
        chosen = np.arange(V) == a
        by = scale / temperature
        out["grad_logits"][r] = by * (pull * (chosen - p) + entropy_coef * p * (logs + h))
        out["size"][r] = abs(by) * (abs(pull) * (chosen + p) + abs(entropy_coef) * p * (1 + np.where(p > 0, -y, 0.) + abs(h - math.log(whole))))
        off = 0. if values is None else float(values[r]) - float(returns[r])
        out["grad_values"][r] = scale * value_coef * off
        out["log_probs"][r], out["entropies"][r] = logs[a], h
        one = np.array([1., policy, h, off * off / 2, ratio - 1 - change, float(clipped)])
        sums += one
        parts += np.abs(one) + np.array([0, 0, 0, 0, ratio + 1 + abs(change), 0])
    out["sums"], out["parts"] = sums, parts
    out["loss"] = scale * (sums[1] - entropy_coef * sums[2] + value_coef * sums[3])
    out["loss_parts"] = abs(scale) * (parts[1] + abs(entropy_coef) * parts[2] + abs(value_coef) * parts[3])
    return out
