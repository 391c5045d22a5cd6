"""The operators on score maps that learning from a teacher and from a policy's own actions
needs, whose speed is measured, through the library's public entry points.

Score maps are channels-last, [n, h, w, c], of which the first `classes` channels count; a
batch of token rows is a map of one pixel row. Top scores: a teacher's k largest scores of
each pixel with their channels and the logarithm of what the others weigh. Distillation: the
divergence of a student's scores from such a record, with its gradient. Action log
probabilities: of the classes that a policy chose, with its entropy. Clipped policy loss:
the clipped ratio times the advantage, with a divergence to a reference, and its gradient.

The listed cases stand for
  top_frame        a teacher's scores of a sparse segmentation frame (38 of 128 blocks of a
                   2048x1024 frame at stride 4, 19 classes): the record of the executed blocks
  top_long         rows over a large vocabulary, the longest record
  top_odd_f32      fp32 rows whose length and number divide by nothing
  distill_frame    the student's whole segmentation map against such a record
  distill_long     long rows, many of them: the largest
  distill_one      a single row, in fp32 and without the rest: all latency
  logp_grid        the policy network's block decisions at 2048x1024 (execute or not): the
                   smallest call
  logp_long        a batch of long rows in fp16, with the entropy
  clip_grid        the policy network's update over one frame's blocks
  clip_long        eight sequences of token rows of unequal length, with a reference
  clip_odd_f32     fp32 rows of odd length, without a reference
  clip_few         a few very long rows: work split along the row
"""
import math
import random

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


# ------------------------------------------------------------------ the cases

def top_case(dtype, n, gh, gw, bh, bw, c, classes, k, t, active):
    """Maps of gh x gw blocks of bh x bw pixels; active 0: every block. t: temperature."""
    return dict(kind="top", dtype=dtype, n=n, gh=gh, gw=gw, bh=bh, bw=bw, c=c, classes=classes, k=k, t=t,
                active=active)


def distill_case(dtype, n, h, w, c, classes, k, t, rest, weighted):
    return dict(kind="distill", dtype=dtype, n=n, h=h, w=w, c=c, classes=classes, k=k, t=t, rest=rest,
                weighted=weighted)


def logp_case(dtype, n, h, w, c, classes, entropy):
    return dict(kind="logp", dtype=dtype, n=n, h=h, w=w, c=c, classes=classes, entropy=entropy)


def clip_case(dtype, n, h, w, c, classes, ref, weighted):
    return dict(kind="clip", dtype=dtype, n=n, h=h, w=w, c=c, classes=classes, ref=ref, weighted=weighted)


def listed():
    named = dict(
        top_frame=top_case("bf16", 1, 8, 16, 32, 32, 64, 19, 4, 2.0, 38),
        top_long=top_case("bf16", 1, 1, 1, 1, 2048, 65536, 65536, 64, 1.0, 0),
        top_odd_f32=top_case("f32", 1, 1, 1, 1, 513, 10007, 10007, 17, 1.5, 0),
        distill_frame=distill_case("bf16", 1, 256, 512, 64, 19, 4, 2.0, True, True),
        distill_long=distill_case("bf16", 1, 1, 4096, 131072, 131072, 64, 1.0, True, False),
        distill_one=distill_case("f32", 1, 1, 1, 32768, 32768, 16, 1.0, False, False),
        logp_grid=logp_case("bf16", 1, 8, 16, 64, 1, False),
        logp_long=logp_case("f16", 1, 1, 8192, 32768, 32768, True),
        clip_grid=clip_case("bf16", 1, 8, 16, 64, 1, True, False),
        clip_long=clip_case("bf16", 8, 1, 1024, 32768, 32768, True, True),
        clip_odd_f32=clip_case("f32", 3, 1, 173, 4099, 4099, False, False),
        clip_few=clip_case("bf16", 2, 1, 3, 150001, 150001, True, False),
    )
    return [dict(c, name=k) for k, c in named.items()]


def spread(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw_map(rng):
    """n, gh, gw, edge, c, classes of a segmentation-like map."""
    n, gh, gw = rng.randint(1, 2), rng.randint(2, 8), rng.randint(2, 16)
    edge = rng.choice((2, 3, 4, 8, 16, 32))
    c = rng.choice((8, 24, 37, 64, 64, 128))
    return n, gh, gw, edge, c, rng.randint(2, c)


def draw_rows(rng, most):
    """Rows and classes of a batch of token rows."""
    rows = spread(rng, 1, 16384)
    classes = spread(rng, 64, min(200000, max(64, most // rows)))
    return rows, classes if rng.random() < 0.4 else max(8, classes // 8 * 8)


def draw(rng):
    what = rng.choice(("top", "distill", "logp", "clip"))
    kind = rng.choice(("bf16", "bf16", "f16", "f32"))
    on_map = rng.random() < 0.4
    if on_map:
        n, gh, gw, edge, c, classes = draw_map(rng)
        h, w = gh * edge, gw * edge
    else:
        rows, classes = draw_rows(rng, 1 << 26 if what == "top" else 1 << 28)
        n = rng.choice((1, 1, 2, 5)) if what != "top" else 1
        gh, gw, edge, h, w, c = 1, 1, 1, 1, max(1, rows // n), classes
    k, t = spread(rng, 1, min(64, classes)), rng.choice((1.0, 1.5, 2.0, 4.0))
    if what == "top":
        if on_map:
            return top_case(kind, n, gh, gw, edge, edge, c, classes, k, t, max(1, n * gh * gw * rng.randint(5, 100) // 100))
        return top_case(kind, 1, 1, 1, 1, w, c, classes, k, t, 0)
    if what == "distill":
        return distill_case(kind, n, h, w, c, classes, k, t, rng.random() < 0.6, rng.random() < 0.5)
    if on_map and rng.random() < 0.5:
        classes = 1
    if what == "logp":
        return logp_case(kind, n, h, w, c, classes, rng.random() < 0.5)
    return clip_case(kind, n, h, w, c, classes, rng.random() < 0.6, rng.random() < 0.5)


def size_of(c):
    """n, h, w of a case's map."""
    return (c["n"], c["gh"] * c["bh"], c["gw"] * c["bw"]) if c["kind"] == "top" else (c["n"], c["h"], c["w"])


# what the clipped loss is called with
CLIP_LOW, CLIP_HIGH, BETA = 0.2, 0.28, 0.04


# ------------------------------------------------------------------ inputs

def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=DEV)

    n, h, w = size_of(case)
    c, classes, dt = case["c"], case["classes"], DTYPES[case["dtype"]]
    s = dict(case=case, kept={})
    # scores spread like a network's, channels with offsets of their own
    s["scores"] = (normal(n, h, w, c).mul_(2.0).add_(0.7 * normal(c))).to(dt)
    if case["kind"] == "top":
        k = case["k"]
        # the previous frame's record
        s["top"] = normal(n, h, w, k).to(dt)
        s["index"] = torch.randint(0, classes, (n, h, w, k), generator=gen, device=DEV, dtype=torch.int32)
        s["rest"] = normal(n, h, w)
        blocks = n * case["gh"] * case["gw"]
        s["idx"] = s["count"] = None
        if case["active"]:
            a = min(case["active"], blocks)
            s["idx"] = torch.zeros(blocks, dtype=torch.int32, device=DEV)
            s["idx"][:a] = torch.randperm(blocks, generator=gen, device=DEV)[:a].sort().values.to(torch.int32)
            s["count"] = torch.full((1,), a, dtype=torch.int32, device=DEV)
        return s
    rows = s["scores"][..., :classes].to(torch.float32, copy=True)
    s["weight"] = None
    if case.get("weighted"):
        # sequences end at lengths of their own; a map counts where the teacher is sure
        if h == 1:
            ends = torch.randint(1, w + 1, (n, 1, 1), generator=gen, device=DEV)
            s["weight"] = (torch.arange(w, device=DEV) < ends).float() / ends
        else:
            s["weight"] = normal(n, h, w).clamp_(min=0.0)
    if case["kind"] == "distill":
        k, t = case["k"], case["t"]
        teacher = rows.mul_(0.8).add_(normal(n, h, w, classes).mul_(1.2)).to(dt).float()
        top = torch.topk(teacher, k, dim=-1)
        s["index"], s["top"] = top.indices.to(torch.int32), top.values.to(dt)
        s["rest"] = None
        if case["rest"]:
            s["rest"] = torch.logsumexp(teacher.scatter_(-1, top.indices, -math.inf).div_(t), -1)
    elif classes == 1:
        lp = torch.nn.functional.logsigmoid(rows[..., 0])
        s["action"] = (normal(n, h, w) > 0).to(torch.uint8)
        lp = torch.where(s["action"] != 0, lp, lp - rows[..., 0])
    else:
        lse = torch.logsumexp(rows, -1)
        # classes drawn from among the likelier ones
        some = torch.randint(0, classes, (n, h, w, 16), generator=gen, device=DEV)
        best = rows.gather(-1, some).argmax(-1, keepdim=True)
        s["action"] = some.gather(-1, best)[..., 0].to(torch.int32)
        lp = rows.gather(-1, s["action"].long()[..., None])[..., 0] - lse
    if case["kind"] == "logp":
        s["logp"] = torch.empty((n, h, w), dtype=torch.float32, device=DEV)
        s["entropy"] = torch.empty_like(s["logp"]) if case["entropy"] else None
        return s
    if case["kind"] == "clip":
        s["advantage"] = normal(n, h, w)
        s["old"] = lp + 0.2 * normal(n, h, w)
        s["ref"] = s["old"] + 0.3 * normal(n, h, w) if case["ref"] else None
        s["kl"] = torch.empty(n, dtype=torch.float32, device=DEV) if case["ref"] else None
    s["scale"] = 1.0 if case.get("weighted") else 1.0 / (h * w)
    if dt is torch.float16:
        s["scale"] *= 1024.0                             # as training in fp16 scales its loss
    s["grad"] = torch.empty_like(s["scores"])
    s["loss"] = torch.empty(n, dtype=torch.float32, device=DEV)
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    kind = s["case"]["kind"]
    if own:
        return {"top": own_top, "distill": own_distill, "logp": own_logp, "clip": own_clip}[kind](s)
    return {"top": plain_top, "distill": plain_distill, "logp": plain_logp, "clip": plain_clip}[kind](s)


def kept_work(s, nbytes):
    """The workspace a program keeps beside its buffers."""
    if "work" not in s["kept"]:
        s["kept"]["work"] = torch.empty(nbytes(), dtype=torch.uint8, device=DEV)
    return s["kept"]["work"]


def own_top(s):
    from paper_2108_09376_amd import bc
    c = s["case"]
    work = kept_work(s, lambda: bc.bc_top_scores_work(s["scores"], c["classes"], c["k"]))
    bc.bc_top_scores(s["scores"], c["classes"], c["t"], s["top"], s["index"], s["rest"], (c["gh"], c["gw"]), s["idx"],
                     s["count"], work=work)
    return s["top"], s["index"], s["rest"]


def own_distill(s):
    from paper_2108_09376_amd import bc
    c = s["case"]
    work = kept_work(s, lambda: bc.bc_distill_loss_work(s["scores"], c["classes"], c["k"]))
    bc.bc_distill_loss(s["scores"], c["classes"], s["top"], s["index"], s["rest"], c["t"], s["weight"], s["scale"],
                       s["grad"], s["loss"], work=work)
    return s["grad"], s["loss"]


def own_logp(s):
    from paper_2108_09376_amd import bc
    c = s["case"]
    work = kept_work(s, lambda: bc.bc_action_log_probs_work(s["scores"], c["classes"]))
    bc.bc_action_log_probs(s["scores"], c["classes"], s["action"], s["logp"], s["entropy"], work=work)
    return s["logp"], s["entropy"]


def own_clip(s):
    from paper_2108_09376_amd import bc
    c = s["case"]
    work = kept_work(s, lambda: bc.bc_clipped_policy_loss_work(s["scores"], c["classes"]))
    bc.bc_clipped_policy_loss(s["scores"], c["classes"], s["action"], s["advantage"], s["old"], s["ref"], s["weight"],
                              (CLIP_LOW, CLIP_HIGH, BETA), s["scale"], s["grad"], s["loss"], s["kl"], work=work)
    return s["grad"], s["loss"], s["kl"]


def plain_top(s):
    c, t = s["case"], s["case"]["t"]
    blocks = (c["n"], c["gh"], c["bh"], c["gw"], c["bw"])
    at = None
    if s["idx"] is not None:
        i = s["idx"][:min(c["active"], c["n"] * c["gh"] * c["gw"])].long()
        at = (i // (c["gh"] * c["gw"]), i // c["gw"] % c["gh"], i % c["gw"])

    def of(x, *last):
        x = x.view(*blocks, *last)
        return x if at is None else x[at[0], at[1], :, at[2]]

    def put(x, v, *last):
        if at is None:
            x.view(*blocks, *last).copy_(v)
        else:
            x.view(*blocks, *last)[at[0], at[1], :, at[2]] = v.to(x.dtype)

    z = of(s["scores"], c["c"])[..., :c["classes"]].float()
    # order: the score, then the lower channel
    bits = (z + 0.0).view(torch.int32).long()
    keys = torch.where(bits >= 0, bits, -2147483648 - bits) * (1 << 32) - torch.arange(c["classes"], device=DEV)
    top = torch.topk(keys, c["k"], dim=-1).indices
    value = z.gather(-1, top)
    left = z.scatter(-1, top, -math.inf) / t
    m = left.amax(-1, keepdim=True).clamp(min=-1e38)
    rest = m[..., 0] + torch.log(torch.exp(left - m).sum(-1))
    put(s["top"], value, c["k"])
    put(s["index"], top, c["k"])
    put(s["rest"], rest)
    return s["top"], s["index"], s["rest"]


def plain_lse(z):
    m = z.amax(-1, keepdim=True)
    return m[..., 0] + torch.log(torch.exp(z - m).sum(-1))


def plain_distill(s):
    c, t = s["case"], s["case"]["t"]
    z = s["scores"][..., :c["classes"]].float()
    at = s["index"].long()
    left = z.scatter(-1, at, -math.inf) / t
    m = left.amax(-1, keepdim=True).clamp(min=-1e38)
    e = torch.exp(left - m)
    # a pixel's few outcomes in 64 bits: a small divergence is the difference of large terms
    weight = e.sum(-1, keepdim=True, dtype=torch.float64)
    zt, tt = z.gather(-1, at).double() / t, s["top"].double() / t
    others = m + torch.log(weight)
    log_q = torch.cat([zt, others], -1)
    log_q = log_q - plain_lse(log_q)[..., None]
    tt = torch.cat([tt, torch.full_like(others, -math.inf) if s["rest"] is None else s["rest"].double()[..., None]], -1)
    log_p = tt - plain_lse(tt)[..., None]
    p, q = torch.exp(log_p), torch.exp(log_q)
    # both sum to 1, so that p log(p / q) may be taken as p log(p / q) - p + q
    each = (torch.where(p > 0, p * (log_p - log_q), torch.zeros_like(p)) - p + q).sum(-1)
    wt = torch.full_like(each, s["scale"]) if s["weight"] is None else s["weight"].double() * s["scale"]
    dz = (q - p) * (wt[..., None] / t)
    share = dz[..., -1:] / weight.clamp(min=1e-300)      # of every e
    dz = (e * share.float()).scatter(-1, at, dz[..., :-1].float())
    s["grad"][..., :c["classes"]] = dz.to(s["grad"].dtype)
    s["grad"][..., c["classes"]:] = 0
    s["loss"].copy_((wt * each).sum((1, 2)))
    return s["grad"], s["loss"]


def plain_logp(s):
    c = s["case"]
    z = s["scores"][..., :c["classes"]].float()
    if c["classes"] == 1:
        # two actions with the scores z and 0
        z = torch.cat([torch.zeros_like(z), z], -1)
        action = (s["action"] != 0).long()
    else:
        action = s["action"].long()
    lse = plain_lse(z)
    s["logp"].copy_(z.gather(-1, action[..., None])[..., 0] - lse)
    if s["entropy"] is not None:
        lp = z - lse[..., None]
        s["entropy"].copy_(-(torch.exp(lp) * lp).sum(-1))
    return s["logp"], s["entropy"]


def plain_clip(s):
    c = s["case"]
    z = s["scores"][..., :c["classes"]].float()
    two = c["classes"] == 1
    if two:
        z = torch.cat([torch.zeros_like(z), z], -1)
        action = (s["action"] != 0).long()[..., None]
    else:
        action = s["action"].long()[..., None]
    m = z.amax(-1, keepdim=True)
    e = torch.exp(z - m)
    # a ratio next to the border of the clipped range is decided in 64 bits
    total = e.sum(-1, keepdim=True, dtype=torch.float64)
    lp = (z.gather(-1, action).double() - m - torch.log(total))[..., 0]
    ratio, adv = torch.exp(lp - s["old"]), s["advantage"].double()
    kept, held = ratio * adv, ratio.clamp(1.0 - CLIP_LOW, 1.0 + CLIP_HIGH) * adv
    each = -torch.minimum(kept, held)
    slope = torch.where(kept <= held, -kept, torch.zeros_like(kept))
    wt = torch.full_like(each, s["scale"]) if s["weight"] is None else s["weight"].double() * s["scale"]
    if s["ref"] is not None:
        d = s["ref"] - lp
        kl = torch.exp(d) - d - 1.0
        each = each + BETA * kl
        slope = slope + BETA * (1.0 - torch.exp(d))
        s["kl"].copy_((wt * kl).sum((1, 2)))
    g = (wt * slope).float()[..., None]
    dz = e * (-g / total.float())
    dz.scatter_add_(-1, action, g)
    dz = dz[..., 1:] if two else dz
    s["grad"][..., :c["classes"]] = dz.to(s["grad"].dtype)
    s["grad"][..., c["classes"]:] = 0
    s["loss"].copy_((wt * each).sum((1, 2)))
    return s["grad"], s["loss"], s["kl"]


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    n, h, w = size_of(case)
    rows, classes = n * h * w, case["classes"]
    if case["kind"] == "top":
        blocks = case["n"] * case["gh"] * case["gw"]
        rows = rows // blocks * (min(case["active"], blocks) or blocks)
        return dict(bytes=rows * (classes * es + case["k"] * (es + 4) + 4), flops=5.0 * rows * classes)
    if case["kind"] == "distill":
        per = classes * es + case["c"] * es + case["k"] * (es + 4) + 4 * bool(case["rest"]) + 4 * bool(case["weighted"])
        return dict(bytes=rows * per + 4 * n, flops=7.0 * rows * classes)
    action = 1 if classes == 1 else 4
    if case["kind"] == "logp":
        return dict(bytes=rows * (classes * es + action + 4 + 4 * bool(case["entropy"])),
                    flops=(6.0 if case["entropy"] else 4.0) * rows * classes)
    per = classes * es + case["c"] * es + action + 8 + 4 * bool(case["ref"]) + 4 * bool(case["weighted"])
    return dict(bytes=rows * per + 8 * n, flops=6.0 * rows * classes)


# ------------------------------------------------------------------ in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"top": exact_top, "distill": exact_distill, "logp": exact_logp, "clip": exact_clip}[case["kind"]](s)


def exact_top(s):
    c = s["case"]
    z = s["scores"][..., :c["classes"]].double()
    value, index = torch.sort(z, dim=-1, descending=True, stable=True)
    k = c["k"]
    rest = torch.full_like(value[..., 0], -math.inf)
    if k < c["classes"]:
        rest = torch.logsumexp(value[..., k:] / c["t"], -1)
    value, index = value[..., :k], index[..., :k].to(torch.int32)
    if s["idx"] is None:
        return value, index, rest
    grid = torch.zeros(c["n"] * c["gh"] * c["gw"], dtype=torch.bool, device=DEV)
    grid[s["idx"][:int(s["count"])].long()] = True
    on = grid.view(c["n"], c["gh"], c["gw"]).repeat_interleave(c["bh"], 1).repeat_interleave(c["bw"], 2)
    return (torch.where(on[..., None], value, s["top"].double()), torch.where(on[..., None], index, s["index"]),
            torch.where(on, rest, s["rest"].double()))


def exact_distill(s):
    """By the definition: a student's distribution over the record's classes (and over all the
    others as one), and the chain rule through its logarithms, by torch's own differentiation."""
    c = s["case"]
    at = s["index"].long()
    t = s["top"].double() / c["t"]
    others_too = s["rest"] is not None and c["k"] < c["classes"]
    if others_too:
        t = torch.cat([t, s["rest"].double()[..., None]], -1)
    p = torch.softmax(t, -1)
    log_p = torch.log_softmax(t, -1)
    wt = torch.ones_like(p[..., 0]) if s["weight"] is None else s["weight"].double()
    grad = torch.zeros(s["scores"].shape, dtype=torch.float64, device=DEV)
    loss = torch.zeros(c["n"], dtype=torch.float64, device=DEV)
    cuts = max(1, s["scores"].numel() >> 27)
    for i in range(c["n"]):
        for part in torch.arange(c["w"], device=DEV).chunk(cuts):
            x = s["scores"][i, :, part, :c["classes"]].double().requires_grad_(True)
            log_q = torch.log_softmax(x / c["t"], -1)
            mine = log_q.gather(-1, at[i, :, part])
            if others_too:
                others = torch.logsumexp(log_q.scatter(-1, at[i, :, part], -math.inf), -1, keepdim=True)
                mine = torch.cat([mine, others], -1)
            pp = p[i, :, part]
            each = (torch.xlogy(pp, torch.exp(log_p[i, :, part])) - torch.where(pp > 0, pp * mine, 0.0)).sum(-1)
            total = (each * wt[i, :, part]).sum() * s["scale"]
            grad[i, :, part, :c["classes"]] = torch.autograd.grad(total, x)[0]
            loss[i] += total.detach()
    return grad, loss


def exact_parts(s):
    """log probabilities of all actions, and which was taken."""
    z = s["scores"][..., :s["case"]["classes"]].double()
    if s["case"]["classes"] == 1:
        return torch.nn.functional.logsigmoid(torch.cat([-z, z], -1)), s["action"].long().clamp(max=1)[..., None]
    return torch.log_softmax(z, -1), s["action"].long()[..., None]


def exact_logp(s):
    log_pi, action = exact_parts(s)
    lp = torch.take_along_dim(log_pi, action, -1)[..., 0]
    if s["entropy"] is None:
        return lp, None
    return lp, torch.special.entr(log_pi.exp_()).sum(-1)


def exact_clip(s):
    log_pi, action = exact_parts(s)
    lp = torch.take_along_dim(log_pi, action, -1)[..., 0]
    lp.requires_grad_(True)
    r, a = torch.exp(lp - s["old"].double()), s["advantage"].double()
    # clipped from above where the advantage is positive, from below where it is not
    bound = torch.where(a >= 0, torch.full_like(a, 1.0 + CLIP_HIGH), torch.full_like(a, 1.0 - CLIP_LOW))
    inside = torch.where(a >= 0, r <= bound, r >= bound)
    each = -a * torch.where(inside, r, bound)
    wt = s["scale"] * (torch.ones_like(a) if s["weight"] is None else s["weight"].double())
    kl = None
    if s["ref"] is not None:
        d = s["ref"].double() - lp
        k3 = torch.expm1(d) - d
        kl = (wt * k3).sum((1, 2)).detach()
        each = each + BETA * k3
    loss = (wt * each).sum((1, 2))
    slope = torch.autograd.grad(loss.sum(), lp)[0]
    c = s["case"]
    pi = log_pi.exp_()
    grad = torch.zeros(s["scores"].shape, dtype=torch.float64, device=DEV)
    # log pi(a) changes with score j by [j = a] - pi(j)
    if c["classes"] == 1:
        grad[..., 0] = slope * (action[..., 0] - pi[..., 1])
    else:
        grad[..., :c["classes"]] = pi.mul_(-slope[..., None]).scatter_add_(-1, action, slope[..., None])
    return grad, loss.detach(), kl
