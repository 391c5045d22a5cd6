"""Plain fp64 versions (numpy) of the operators on score maps (TEST INFRASTRUCTURE ONLY, like
the rest of ``oracle/``): a teacher's record, the divergence from it, log probabilities of decisions and the clipped policy loss. Scores are
[..., c] of which the first `classes` count; pixels are the leading axes of one image
each: [n, h, w, c]. Every function follows the operator's definition and shares nothing with
the library."""
import numpy as np


def lse(z):
    """log(sum(exp(z))) over the last axis; -inf where nothing is above -inf."""
    m = np.max(z, -1, initial=-np.inf)
    ref = np.where(np.isinf(m) & (m < 0), 0.0, m)
    with np.errstate(divide="ignore"):
        return ref + np.log(np.sum(np.exp(z - ref[..., None]), -1))


def top_scores(scores, classes, k, temperature):
    """(values, classes, rest): descending, the lower class first among equals."""
    z = np.asarray(scores, np.float64)[..., :classes]
    order = np.argsort(-z, axis=-1, kind="stable")
    value = np.take_along_axis(z, order, -1)
    return value[..., :k], order[..., :k].astype(np.int32), lse(value[..., k:] / temperature)


def distill(scores, classes, top, index, rest, temperature, weight, scale):
    """(loss per image, gradient, magnitude), pixel by pixel. The magnitude is the gradient's
    with the teacher's and the student's parts added instead of subtracted: what rounding
    errors are relative to."""
    scores = np.asarray(scores, np.float64)
    grad, size = np.zeros_like(scores), np.zeros_like(scores)
    loss = np.zeros(scores.shape[0])
    for at in np.ndindex(*scores.shape[:3]):
        w = 1.0 if weight is None else float(weight[at])
        if w == 0.0:
            continue
        z = scores[at][:classes] / temperature
        # the teacher's share of each class of the record, entries of one class together
        entries = [(int(i), float(t) / temperature) for i, t in zip(index[at], top[at]) if 0 <= i < classes]
        tt = np.array([t for _, t in entries] + [-np.inf if rest is None else float(rest[at])])
        norm, all_z = lse(tt), lse(z)
        if norm == -np.inf or all_z == -np.inf:
            continue
        p = np.exp(tt - norm)
        record = sorted({i for i, _ in entries})
        left = np.ones(classes, bool)
        left[record] = False
        others = np.flatnonzero(left)
        log_q = z - all_z
        log_rest = lse(log_q[others]) if len(others) else -np.inf
        kl = 0.0
        for (i, _), pi, t in zip(entries, p, tt):
            if pi > 0:
                kl += pi * ((t - norm) - log_q[i]) if log_q[i] > -np.inf else np.inf
        if p[-1] > 0:
            kl += p[-1] * ((tt[-1] - norm) - log_rest) if log_rest > -np.inf else np.inf
        loss[at[0]] += scale * w * kl
        g, sz, share = np.zeros(classes), np.zeros(classes), np.zeros(classes)
        for (i, _), pi in zip(entries, p):
            share[i] += pi
        q_rest = np.exp(log_rest)
        for j in record:
            g[j] = np.exp(log_q[j]) - share[j]
            sz[j] = np.exp(log_q[j]) + share[j]
        if len(others) and log_rest > -np.inf:
            g[others] = (q_rest - p[-1]) * np.exp(log_q[others] - log_rest)
            sz[others] = (q_rest + p[-1]) * np.exp(log_q[others] - log_rest)
        grad[at][:classes] = g * scale * w / temperature
        size[at][:classes] = sz * abs(scale * w) / temperature
    return loss, grad, size


def log_pi(scores, classes):
    """log probabilities of all actions: [..., classes], or [..., 2] for classes = 1."""
    z = np.asarray(scores, np.float64)[..., :classes]
    if classes == 1:
        return -np.logaddexp(0.0, np.concatenate([z, -z], -1))
    with np.errstate(invalid="ignore"):
        return z - lse(z)[..., None]


def log_probs(scores, classes, action):
    """(log pi(action), entropy)."""
    lp = log_pi(scores, classes)
    act = (np.asarray(action) != 0).astype(int) if classes == 1 else np.asarray(action)
    ok = (act >= 0) & (act < lp.shape[-1])
    picked = np.take_along_axis(lp, np.where(ok, act, 0)[..., None], -1)[..., 0]
    empty = np.all(np.asarray(scores, np.float64)[..., :classes] == -np.inf, -1) & (classes > 1)
    picked = np.where(ok, np.where(empty, -np.inf, picked), 0.0)
    with np.errstate(invalid="ignore"):
        pi = np.exp(lp)
        ent = -np.sum(np.where(pi > 0, pi * lp, np.where(np.isnan(pi), np.nan, 0.0)), -1)
    return picked, np.where(empty, 0.0, ent)


def clipped_loss(scores, classes, action, advantage, old, ref, weight, low, high, beta, scale):
    """(loss per image, gradient, divergence to the reference per image, magnitude): the
    magnitude is the gradient's with the two parts of its slope added."""
    scores = np.asarray(scores, np.float64)
    size = np.zeros_like(scores)
    lp = log_pi(scores, classes)
    picked, _ = log_probs(scores, classes, action)
    grad = np.zeros_like(scores)
    loss, kl = np.zeros(scores.shape[0]), np.zeros(scores.shape[0])
    for at in np.ndindex(*scores.shape[:3]):
        w = 1.0 if weight is None else float(weight[at])
        a = int(action[at] != 0) if classes == 1 else int(action[at])
        if w == 0.0 or not 0 <= a < lp.shape[-1] or picked[at] == -np.inf:
            continue
        l, adv = picked[at], float(advantage[at])
        r = np.exp(l - float(old[at]))
        kept, held = r * adv, min(max(r, 1.0 - low), 1.0 + high) * adv
        each, slope = -min(kept, held), (-kept if kept <= held else 0.0)
        steep = abs(slope)
        if ref is not None:
            d = float(ref[at]) - l
            k3 = np.expm1(d) - d
            each += beta * k3
            slope += beta * -np.expm1(d)
            steep += beta * (1.0 + np.exp(d))
            kl[at[0]] += scale * w * k3
        loss[at[0]] += scale * w * each
        g = -np.exp(lp[at])
        g[a] = -np.delete(g, a).sum()                             # 1 - pi(a)
        g = g[1:] if classes == 1 else g
        grad[at][:classes] = g * scale * w * slope
        size[at][:classes] = np.abs(g * scale * w) * steep
    return loss, grad, kl, size
