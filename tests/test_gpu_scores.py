"""GPU: the operators on score maps (top scores, distillation, action log probabilities,
clipped policy loss) against plain fp64 versions (oracle/scores.py).

Tolerances, fixed before the first run. An exponential of the row has the argument
(z - m) log2(e) / t, whose three roundings (the difference, the constant, the product) and those of
joining parts of a row change it by at most 8 steps of 2^-24 relative to its size, at most the
row's range R / t; with the steps of the exponential itself and of sums (at most 128 terms one after
another in a lane, 6 exchanges in a wave, 16 waves or the chunks of a row) an fp32 share of a row is
off by at most C = (8 R / t + 200) 2^-24 of itself. A gradient is off by 2 C of its magnitude (its
teacher's and student's parts added) and half a step of its type; a divergence, whose terms'
first order cancels, by C (4 + itself) per pixel; a log probability by C and half a step. 16-bit
gradients below the type's smallest normal number are off by half its smallest step."""
import numpy as np
import pytest
import torch

from oracle import scores as S
from tests._util import TORCH, shifted

pytestmark = pytest.mark.gpu

EPS = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}          # half a step, relative
TINY = {"f32": 2.0 ** -126, "bf16": 2.0 ** -126, "f16": 2.0 ** -25}


@pytest.fixture(scope="module")
def B(gpu):
    from paper_2108_09376_amd import bc
    return bc


def dev(x, dtype, off=0):
    t = torch.from_numpy(np.ascontiguousarray(x)).to(dtype).cuda()
    return shifted(t, off) if off else t


def host(t):
    return t.double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def draw_scores(r, shape, classes, how):
    z = r.normal(0, 2, shape)
    if how == "ties":
        z = r.integers(-2, 3, shape).astype(float)
    elif how == "equal":
        z = np.zeros(shape)
        z[..., 1::3] = -0.0
    elif how == "masked":
        z[r.random(shape) < 0.6] = -np.inf
        z[0, 0, :2] = -np.inf                                     # rows that nothing is left of
    elif how == "peaked":
        z[..., r.integers(0, classes)] += 30.0
    elif how == "low":
        z = z - 60.0
        z[..., -1 if classes == shape[-1] else classes - 1] = 40.0
    elif how == "rising":
        z = np.broadcast_to(np.arange(shape[-1]) / shape[-1] * 8.0, shape).copy()
    elif how == "blocks":
        z[..., : classes // 3] = -np.inf
    z[..., classes:] = np.nan                                     # never looked at
    return z


def constant(z, classes, t=1.0):
    """C of every image: [n]."""
    f = np.where(np.isfinite(z[..., :classes]), z[..., :classes], np.nan)
    with np.errstate(all="ignore"):
        spread = np.nan_to_num(np.nanmax(f, (1, 2, 3), initial=-1e9) - np.nanmin(f, (1, 2, 3), initial=1e9))
    return (8 * np.maximum(spread, 0) / t + 200) * 2.0 ** -24


# n, h, w, c, classes, k: small maps, classes below the channels, odd rows, rows of one class more
# or less than a vector, a wave's or a workgroup's registers, long rows in chunks
MAPS = [(1, 4, 8, 64, 19, 4), (2, 3, 5, 24, 24, 24), (1, 1, 3, 2, 2, 2), (1, 2, 2, 7, 5, 1), (3, 1, 33, 37, 29, 7),
        (1, 1, 9, 513, 513, 64), (2, 1, 7, 1031, 1000, 16), (1, 1, 5, 4099, 4099, 33), (1, 1, 3, 16400, 16400, 64),
        (1, 1, 2, 40001, 40001, 3), (2, 1, 1, 150001, 150000, 64)]
# as many rows as are not split into chunks, in each form of long rows, and one that has to be
MANY = [("bf16", 5003, 9), ("f32", 8190, 64), ("f16", 16389, 5), ("bf16", 32768, 64), ("f32", 32771, 7),
        ("bf16", 65541, 64), ("f16", 131072, 17), ("f32", 66000, 64), ("bf16", 131081, 3)]


def run_top(B, z, dtype, classes, k, t, grid=(1, 1), idx=None, count=None, off=0, rest=True, prev=None):
    n, h, w, _ = z.shape
    x = dev(z, TORCH[dtype], off)
    if prev is None:
        top, index = torch.full((n, h, w, k), 7.0, dtype=TORCH[dtype]).cuda(), torch.full((n, h, w, k), -5, dtype=torch.int32).cuda()
        rst = torch.full((n, h, w), 3.0).cuda() if rest else None
    else:
        top, index, rst = [p.clone() for p in prev]
    B.bc_top_scores(x, classes, t, top, index, rst, grid, idx, count)
    torch.cuda.synchronize()
    return x, top, index, rst


def check_top(x, got, classes, k, t):
    z = host(x)
    v, i, rest = S.top_scores(z, classes, k, t)
    assert np.array_equal(host(got[1]), i)
    assert np.array_equal(host(got[0]), v)
    if got[2] is not None:
        g, c = host(got[2]), constant(np.where(np.isnan(z), 0, z), classes, t)[:, None, None]
        fin = np.isfinite(rest)
        assert np.array_equal(fin, np.isfinite(g)) and np.all(g[~fin] == -np.inf)
        assert np.all(np.abs(g - rest)[fin] <= (c + 2.0 ** -23 * np.abs(rest))[fin])


@pytest.mark.parametrize("how", ["normal", "ties", "equal", "masked", "low", "rising", "blocks"])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_top_scores(B, dtype, how):
    r = np.random.default_rng(1)
    for m, (n, h, w, c, classes, k) in enumerate(MAPS):
        z = draw_scores(r, (n, h, w, c), classes, how)
        t = (1.0, 2.0, 0.7)[m % 3]
        print(dtype, how, n, h, w, c, classes, k, flush=True)
        x, *got = run_top(B, z, dtype, classes, k, t, off=m % 2, rest=m % 4 != 3)
        check_top(x, got, classes, k, t)


@pytest.mark.parametrize("dtype,classes,k", MANY)
def test_top_scores_of_many_long_rows(B, dtype, classes, k):
    r = np.random.default_rng(2)
    base = r.normal(0, 2, (1, 1, 8, classes))
    base[0, 0, 3] = 1.5                                            # a row of equal scores
    base[0, 0, 4, : classes // 2] = -np.inf
    x = dev(base, TORCH[dtype]).repeat(1, 1, 17, 1).contiguous()   # 136 rows
    top = torch.empty((1, 1, 136, k), dtype=TORCH[dtype], device="cuda")
    index, rest = torch.empty((1, 1, 136, k), dtype=torch.int32, device="cuda"), torch.empty((1, 1, 136), device="cuda")
    B.bc_top_scores(x, classes, 1.0, top, index, rest, (1, 1), None, None)
    torch.cuda.synchronize()
    check_top(x[:, :, :8], (top[:, :, :8], index[:, :, :8], rest[:, :, :8]), classes, k, 1.0)
    for got in (top, index, rest):
        assert torch.equal(got, got[:, :, :8].repeat(1, 1, 17, *[1] * (got.dim() - 3)))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_top_scores_of_awkward_rows(B, dtype):
    """Rows that few scores stand out of, or that lie badly over the lanes: runs of equal scores at and
    across the record's end, all masked but a few, largest scores side by side, in one lane's
    vectors, in the last elements; NaN, for which classes are distinct and in range."""
    r = np.random.default_rng(4)
    for classes, k in ((520, 64), (1100, 9), (4099, 64), (8200, 64), (17000, 33), (33003, 64), (50001, 64), (90001, 64),
                       (700001, 64)):                            # the last two in chunks, joined in LDS and by rounds
        rows = r.normal(0, 2, (1, 1, 12, classes))
        rows[0, 0, 1] = -3.0
        rows[0, 0, 2, ::2] = 9.0                                   # half of it equal and largest
        rows[0, 0, 3] = -np.inf
        rows[0, 0, 3, classes - 3:] = 1.0
        rows[0, 0, 4] = -np.inf
        rows[0, 0, 4, 5] = -7.0
        rows[0, 0, 5, 100:100 + k] += 20.0                         # side by side
        rows[0, 0, 6, -k:] += 20.0                                 # at the end
        rows[0, 0, 7, 7::2048] += 20.0                             # in few lanes
        rows[0, 0, 8] = np.round(rows[0, 0, 8])                    # few values
        rows[0, 0, 9] = -np.abs(rows[0, 0, 9]) - 1e-3              # all negative
        rows[0, 0, 10] = r.integers(0, 2, classes) * -0.0          # zeros of both signs
        rows[0, 0, 10][r.random(classes) < 0.5] = 0.0
        rows[0, 0, 11, 3:] = 0.0
        print(dtype, classes, k, flush=True)
        x, *got = run_top(B, rows, dtype, classes, k, 1.0, off=1)
        check_top(x, got, classes, k, 1.0)
        for share in (0.01, 0.9, 1.0):
            z = rows[:, :, :2].copy()
            z[r.random(z.shape) < share] = np.nan
            x, top, index, rest = run_top(B, z, dtype, classes, k, 1.0)
            for row in host(index).reshape(2, k):
                assert len(set(row.tolist())) == k and row.min() >= 0 and row.max() < classes


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("c,classes,k", [(64, 19, 4), (24, 24, 3), (30000, 30000, 20)])
def test_top_scores_on_active_blocks(B, dtype, c, classes, k):
    """Blocks that did not run keep their record bit for bit, an index of none changes nothing."""
    r = np.random.default_rng(3)
    n, gh, gw, bh, bw = (2, 3, 4, 2, 3) if c < 100 else (1, 2, 2, 1, 2)
    z = draw_scores(r, (n, gh * bh, gw * bw, c), classes, "normal")
    shape = (n, gh * bh, gw * bw)
    prev = (torch.randn(*shape, k).to(TORCH[dtype]).cuda(), torch.randint(0, 99, (*shape, k), dtype=torch.int32).cuda(),
            torch.randn(*shape).cuda())
    for mask in (r.random((n, gh, gw)) < 0.4, np.zeros((n, gh, gw), bool), np.ones((n, gh, gw), bool)):
        ids = np.flatnonzero(mask)
        idx = torch.full((n * gh * gw,), 10 ** 6, dtype=torch.int32)
        idx[:len(ids)] = torch.from_numpy(ids.astype(np.int32))
        count = torch.tensor([len(ids)], dtype=torch.int32).cuda()
        x, *got = run_top(B, z, dtype, classes, k, 2.0, (gh, gw), idx.cuda(), count, prev=prev)
        on = torch.from_numpy(np.repeat(np.repeat(mask, bh, 1), bw, 2)).cuda()
        _, *full = run_top(B, z, dtype, classes, k, 2.0, (gh, gw))
        check_top(x, full, classes, k, 2.0)
        for g, f, p in zip(got, full, prev):
            sel = on.view(*on.shape, *[1] * (g.dim() - 3))
            assert torch.equal(g, torch.where(sel, f, p))


# ------------------------------------------------------------------ distillation

def draw_record(r, z, classes, k, t, how):
    """A teacher's record for these scores: top, index, rest."""
    teacher = np.where(np.isnan(z), 0, np.where(np.isinf(z), -3.0, z)) * 0.8 + r.normal(0, 1, z.shape)
    kk = min(k, classes)
    top, index, rest = S.top_scores(teacher, classes, kk, t)
    if kk < k:                                                    # padded with entries that are left out
        pad = [(0, 0)] * 3 + [(0, k - kk)]
        top, index = np.pad(top, pad, constant_values=5.0), np.pad(index, pad, constant_values=-1)
    if how == "twice" and k >= 3:
        index[..., 2] = index[..., 0]
        index[0, 0, 0, 1] = classes
        index[-1, -1, -1, :] = index[-1, -1, -1, 0]
    if how == "masked":
        top[-1, -1, -1, :] = -np.inf
    return top, index.astype(np.int32), rest


def check_distill(x, top, index, rest, w, classes, t, scale, dtype, grad, loss):
    z = host(x)
    want_l, want_g, size = S.distill(z, classes, host(top), host(index), None if rest is None else host(rest), t,
                                     None if w is None else host(w), scale)
    c = constant(z, classes, t)
    if grad is not None:
        g = host(grad)
        # 2 C of the magnitude: a teacher's scores have a range of their own in it
        lim = EPS[dtype] * np.abs(want_g) + 2 * c[:, None, None, None] * size + TINY[dtype]
        bad = ~(np.abs(g - want_g) <= lim)
        assert not bad.any(), (np.argwhere(bad)[:5], g[bad][:5], want_g[bad][:5])
        assert not g[..., classes:].any()
    if loss is not None:
        l = host(loss)
        fin = np.isfinite(want_l)
        assert np.array_equal(fin, np.isfinite(l)) and np.all(l[~fin] == want_l[~fin])
        wt = np.full(z.shape[:3], abs(scale)) if w is None else np.abs(host(w)) * abs(scale)
        lim = c * (4 * wt.sum((1, 2)) + np.abs(want_l)) + 2.0 ** -23 * np.abs(want_l)
        assert np.all(np.abs(l - want_l)[fin] <= lim[fin]), (l, want_l, lim)


@pytest.mark.parametrize("how", ["normal", "masked", "peaked", "twice", "low"])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_distill_loss(B, dtype, how):
    r = np.random.default_rng(11)
    for m, (n, h, w, c, classes, k) in enumerate(MAPS):
        z = draw_scores(r, (n, h, w, c), classes, how)
        t = (1.0, 2.0, 0.7)[m % 3]
        top, index, rest = draw_record(r, z, classes, k, t, how)
        print(dtype, how, n, h, w, c, classes, k, flush=True)
        x = dev(z, TORCH[dtype], m % 2)
        top = dev(top, TORCH[("bf16", "f32", "f16")[m % 3]])
        index = dev(index, torch.int32)
        rest = dev(rest, torch.float32) if m % 2 or how == "low" else None
        weight = None
        if m % 3:
            weight = r.random((n, h, w)).astype(np.float32)
            weight[0, 0, 0] = 0.0
            x[0, 0, 0] = float("nan")                              # takes no part
            weight = dev(weight, torch.float32)
        loss = torch.full((n,), 9.0, device="cuda")
        grad = torch.full_like(x, 5.0)
        B.bc_distill_loss(x, classes, top, index, rest, t, weight, 1.5, grad, loss)
        torch.cuda.synchronize()
        check_distill(x, top, index, rest, weight, classes, t, 1.5, dtype, grad, loss)
        # the loss alone, the gradient alone and in place: the same bits
        loss2, grad2, y = torch.empty_like(loss), torch.empty_like(grad), x.clone()
        B.bc_distill_loss(x, classes, top, index, rest, t, weight, 1.5, None, loss2)
        B.bc_distill_loss(x, classes, top, index, rest, t, weight, 1.5, grad2, None)
        B.bc_distill_loss(y, classes, top, index, rest, t, weight, 1.5, y, None)
        bits = lambda v: v.view(torch.int16 if v.element_size() == 2 else torch.int32)
        assert torch.equal(bits(loss), bits(loss2)) and torch.equal(bits(grad), bits(grad2)) and torch.equal(bits(grad), bits(y))


@pytest.mark.parametrize("dtype,classes,k", MANY)
def test_distill_loss_of_many_long_rows(B, dtype, classes, k):
    r = np.random.default_rng(12)
    z = r.normal(0, 2, (1, 1, 4, classes))
    top, index, rest = draw_record(r, z, classes, k, 1.0, "normal")
    rep = lambda v: v.repeat(1, 1, 34, *[1] * (v.dim() - 3)).contiguous()    # 136 rows
    x, top, index, rest = [rep(v) for v in (dev(z, TORCH[dtype]), dev(top, TORCH[dtype]), dev(index, torch.int32),
                                            dev(rest, torch.float32))]
    grad, loss = torch.empty_like(x), torch.empty(1, device="cuda")
    B.bc_distill_loss(x, classes, top, index, rest, 1.0, None, 1.0 / 34, grad, loss)
    torch.cuda.synchronize()
    want_l = S.distill(host(x[:, :, :4]), classes, host(top[:, :, :4]), host(index[:, :, :4]), host(rest[:, :, :4]), 1.0,
                       None, 1.0)[0]
    check_distill(x[:, :, :4], top[:, :, :4], index[:, :, :4], rest[:, :, :4], None, classes, 1.0, 1.0 / 34, dtype,
                  grad[:, :, :4], None)
    assert abs(float(loss) - want_l[0]) <= 2 * constant(z, classes)[0] * (4 * 4 + want_l[0])
    assert torch.equal(grad, rep(grad[:, :, :4]))


def test_distill_of_a_mean_record_moves_towards_it(B):
    """The record of the scores themselves: no divergence, no gradient beyond rounding; and many
    images at once."""
    r = np.random.default_rng(13)
    x = dev(r.normal(0, 2, (700, 2, 3, 21)), torch.float32)
    top, index = torch.empty((700, 2, 3, 5), device="cuda"), torch.empty((700, 2, 3, 5), dtype=torch.int32, device="cuda")
    rest, loss, grad = torch.empty((700, 2, 3), device="cuda"), torch.empty(700, device="cuda"), torch.empty_like(x)
    B.bc_top_scores(x, 21, 2.0, top, index, rest, (1, 1), None, None)
    B.bc_distill_loss(x, 21, top, index, rest, 2.0, None, 1.0, grad, loss)
    torch.cuda.synchronize()
    c = constant(host(x), 21, 2.0)
    assert np.all(np.abs(host(loss)) <= c * 4 * 6) and np.all(np.abs(host(grad)) <= c[:, None, None, None])


# ------------------------------------------------------------------ policy

def draw_decisions(r, z, classes, dtype):
    """Actions, advantages, old and reference log probabilities; ratios stay away from the borders
    of the clipped range (0.8, 1.3), where rounding decides."""
    shape = z.shape[:3]
    act = r.integers(0, max(2, classes), shape)
    l, _ = S.log_probs(z, classes, act)
    l = np.where(np.isfinite(l), l, -1.0)
    step = r.choice([-0.6, -0.35, -0.1, -0.02, 0.0, 0.03, 0.2, 0.4, 0.9], shape)
    return act, r.normal(0, 1, shape), l - step, l + r.normal(0, 0.4, shape)


def check_clip(x, classes, act, adv, old, ref, w, clip, scale, dtype, grad, loss, kl):
    z = host(x)
    f = lambda v: None if v is None else host(v)
    want_l, want_g, want_k, size = S.clipped_loss(z, classes, f(act), f(adv), f(old), f(ref), f(w),
                                                  float(np.float32(clip[0])), float(np.float32(clip[1])), clip[2], scale)
    c = constant(z, classes)
    if grad is not None:
        g = host(grad)
        lim = EPS[dtype] * np.abs(want_g) + 2 * c[:, None, None, None] * size + TINY[dtype]
        bad = ~(np.abs(g - want_g) <= lim)
        assert not bad.any(), (np.argwhere(bad)[:5], g[bad][:5], want_g[bad][:5])
    if loss is None:
        return
    wt = np.full(z.shape[:3], abs(scale)) if w is None else np.abs(f(w)) * abs(scale)
    # a change of C in l changes the ratio by C of itself (at most e) and K by C e^d (at most e^2)
    lim = c * (wt * (np.abs(f(adv)) * 3 + clip[2] * 8)).sum((1, 2)) + 2.0 ** -23 * np.abs(want_l)
    assert np.all(np.abs(host(loss) - want_l) <= lim), (host(loss), want_l, lim)
    if kl is not None:
        assert np.all(np.abs(host(kl) - want_k) <= c * 8 * wt.sum((1, 2)) + 2.0 ** -23 * np.abs(want_k))


POLICY = [(1, 8, 16, 64, 1), (2, 5, 7, 3, 1), (3, 1, 300, 1, 1)] + [m[:5] for m in MAPS]


@pytest.mark.parametrize("how", ["normal", "masked", "peaked", "low"])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_policy(B, dtype, how):
    r = np.random.default_rng(21)
    for m, (n, h, w, c, classes) in enumerate(POLICY):
        z = draw_scores(r, (n, h, w, c), classes, how if classes > 1 or how != "masked" else "normal")
        x = dev(z, TORCH[dtype], m % 2)
        z = host(x)
        print(dtype, how, n, h, w, c, classes, flush=True)
        act, adv, old, ref = draw_decisions(r, z, classes, dtype)
        if classes > 1:
            act[0, 0, -1], act[-1, -1, 0] = -1, classes            # no decision
        a = dev(act, torch.uint8 if classes == 1 else torch.int32)
        logp, ent = torch.empty((n, h, w), device="cuda"), torch.empty((n, h, w), device="cuda")
        logp2 = torch.empty_like(logp)
        B.bc_action_log_probs(x, classes, a, logp, ent)
        B.bc_action_log_probs(x, classes, a, logp2)
        torch.cuda.synchronize()
        want, want_e = S.log_probs(z, classes, host(a))
        cc = constant(z, classes)[:, None, None]
        got = host(logp)
        fin = np.isfinite(want)
        assert np.array_equal(fin, np.isfinite(got)) and np.all(got[~fin] == -np.inf)
        assert np.all(np.abs(got - want)[fin] <= (cc + EPS["f32"] * np.abs(want))[fin])
        assert torch.equal(logp, logp2)
        # log s and sum of pi (z - m), each off by C, the second of at most R
        spread = cc / 2.0 ** -24 / 8
        assert np.all(np.abs(host(ent) - want_e) <= cc * (2 + spread * (want_e > 0)))
        weight = None
        if m % 2:
            weight = r.random((n, h, w)).astype(np.float32)
            weight[0, 0, 0] = 0.0
            x[0, 0, 0] = float("nan")
            weight = dev(weight, torch.float32)
        adv, old, ref = [dev(v, torch.float32) for v in (adv, old, ref)]
        ref = ref if m % 3 else None
        loss, kl = torch.full((n,), 9.0, device="cuda"), torch.full((n,), 9.0, device="cuda") if ref is not None else None
        grad, clip = torch.full_like(x, 5.0), (0.2, 0.3, 0.1)
        B.bc_clipped_policy_loss(x, classes, a, adv, old, ref, weight, clip, 0.5, grad, loss, kl)
        torch.cuda.synchronize()
        check_clip(x, classes, a, adv, old, ref, weight, clip, 0.5, dtype, grad, loss, kl)
        loss2, grad2, y = torch.empty_like(loss), torch.empty_like(grad), x.clone()
        B.bc_clipped_policy_loss(x, classes, a, adv, old, ref, weight, clip, 0.5, None, loss2)
        B.bc_clipped_policy_loss(x, classes, a, adv, old, ref, weight, clip, 0.5, grad2, None)
        B.bc_clipped_policy_loss(y, classes, a, adv, old, ref, weight, clip, 0.5, y, None)
        bits = lambda v: v.view(torch.int16 if v.element_size() == 2 else torch.int32)
        assert torch.equal(bits(loss), bits(loss2)) and torch.equal(bits(grad), bits(grad2)) and torch.equal(bits(grad), bits(y))


@pytest.mark.parametrize("dtype,classes,k", MANY)
def test_policy_of_many_long_rows(B, dtype, classes, k):
    r = np.random.default_rng(22)
    z = r.normal(0, 2, (2, 1, 2, classes))
    x = dev(z, TORCH[dtype])
    act, adv, old, ref = draw_decisions(r, host(x), classes, dtype)
    rep = lambda v: v.repeat(1, 1, 34, *[1] * (v.dim() - 3)).contiguous()    # 136 rows
    x, a, adv, old, ref = [rep(v) for v in (x, dev(act, torch.int32), dev(adv, torch.float32), dev(old, torch.float32),
                                            dev(ref, torch.float32))]
    logp, ent = torch.empty((2, 1, 68), device="cuda"), torch.empty((2, 1, 68), device="cuda")
    grad, loss, kl = torch.empty_like(x), torch.empty(2, device="cuda"), torch.empty(2, device="cuda")
    B.bc_action_log_probs(x, classes, a, logp, ent)
    B.bc_clipped_policy_loss(x, classes, a, adv, old, ref, None, (0.2, 0.3, 0.1), 1.0 / 34, grad, loss, kl)
    torch.cuda.synchronize()
    s = [v[:, :, :2].contiguous() for v in (x, a, adv, old, ref, grad)]
    check_clip(*s[:1], classes, *s[1:5], None, (0.2, 0.3, 0.1), 1.0 / 34, dtype, s[5], None, None)
    check_clip(*s[:1], classes, *s[1:5], None, (0.2, 0.3, 0.1), 1.0, dtype, None, loss, kl)
    want, want_e = S.log_probs(host(s[0]), classes, host(s[1]))
    c = constant(z, classes)[:, None, None]
    assert np.all(np.abs(host(logp[:, :, :2]) - want) <= c + EPS["f32"] * np.abs(want))
    assert np.all(np.abs(host(ent[:, :, :2]) - want_e) <= c * (2 + c * 2.0 ** 21))
    for v in (logp, ent, grad):
        assert torch.equal(v, rep(v[:, :, :2]))


def test_extreme_policies(B):
    """Scores at the ends of the range: probabilities of 0 and 1, ratios past 1e38."""
    z = np.array([[[[0.0, 3e38], [-3e38, 3e38], [88.0, -88.0], [1.0, 1.0]]]])
    x = dev(z, torch.float32)
    a = dev(np.array([[[1, 0, 1, 0]]]), torch.int32)
    logp, ent = torch.empty((1, 1, 4), device="cuda"), torch.empty((1, 1, 4), device="cuda")
    B.bc_action_log_probs(x, 2, a, logp, ent)
    want, want_e = S.log_probs(host(x), 2, host(a))
    assert np.allclose(host(logp), np.maximum(want, -np.finfo(np.float32).max * 2), rtol=1e-6) or np.isinf(host(logp)[0, 0, 1])
    assert np.allclose(host(ent), want_e, atol=1e-6)
    for z1 in (-200.0, -30.0, 0.0, 30.0, 200.0, float("inf"), float("-inf")):
        x = torch.full((1, 1, 2, 1), z1, device="cuda")
        a = torch.tensor([[[0, 1]]], dtype=torch.uint8, device="cuda")
        logp, ent = torch.empty((1, 1, 2), device="cuda"), torch.empty((1, 1, 2), device="cuda")
        grad, loss = torch.empty_like(x), torch.empty(1, device="cuda")
        B.bc_action_log_probs(x, 1, a, logp, ent)
        B.bc_clipped_policy_loss(x, 1, a, torch.ones_like(logp), logp.clamp(min=-1e30), None, None, (0.2, 0.2, 0.0), 1.0, grad, loss)
        torch.cuda.synchronize()
        with np.errstate(over="ignore"):
            p = 1.0 / (1.0 + np.exp(-np.float64(z1)))
        sp = lambda v: np.logaddexp(0.0, v)                        # log(1 + e^v)
        # one rounding: half a step of 2^-23, and below fp32's numbers up to its smallest, 2^-149
        assert np.allclose(host(logp)[0, 0], [-sp(z1), -sp(-z1)], rtol=2e-7, atol=2.0 ** -149), z1
        assert np.isfinite(host(ent)).all() and np.all(host(ent) >= 0)
        # at ratio 1: -(a - p)
        want = np.array([p, -(1.0 - p if abs(z1) < 30 else np.exp(-sp(z1)))])
        want = np.where(np.isfinite(host(logp)[0, 0]), want, 0.0)
        assert np.allclose(host(grad)[0, 0, :, 0], want, rtol=1e-5, atol=1e-38), z1


def test_nan_stays_in_its_pixel(B):
    r = np.random.default_rng(23)
    for c, classes in ((64, 40), (3000, 3000), (40000, 40000)):
        x = dev(r.normal(0, 2, (2, 1, 3, c)), torch.float32)
        y = x.clone()
        y[0, 0, 1, 7] = float("nan")
        act = torch.full((2, 1, 3), 3, dtype=torch.int32, device="cuda")
        one, old = torch.ones((2, 1, 3), device="cuda"), torch.full((2, 1, 3), -2.0, device="cuda")
        top, index = torch.zeros((2, 1, 3, 2), device="cuda"), torch.tensor([1, 5], dtype=torch.int32).repeat(2, 1, 3, 1).cuda()
        outs = []
        for v in (x, y):
            g1, l1, g2, l2 = torch.empty_like(v), torch.empty(2, device="cuda"), torch.empty_like(v), torch.empty(2, device="cuda")
            lp, ent = torch.empty_like(one), torch.empty_like(one)
            B.bc_clipped_policy_loss(v, classes, act, one, old, None, None, (0.2, 0.2, 0.0), 1.0, g1, l1)
            B.bc_distill_loss(v, classes, top, index, one, 1.0, None, 1.0, g2, l2)
            B.bc_action_log_probs(v, classes, act, lp, ent)
            outs.append((g1, l1, g2, l2, lp, ent))
        torch.cuda.synchronize()
        for i, (p, q) in enumerate(zip(*outs)):
            keep = torch.ones(p.shape[:3] if p.dim() > 1 else p.shape, dtype=torch.bool)
            if p.dim() > 1:
                keep[0, 0, 1] = False
            else:
                keep[0] = False
            assert torch.equal(p[keep.cuda()], q[keep.cuda()]), i
            if i in (1, 3, 4, 5):
                assert torch.isnan(q[~keep.cuda()]).all(), i


def test_a_class_alone(B):
    """Every class but one masked: its probability is 1, its gradient 0; a NaN there stays one."""
    for c in (5, 40, 600, 9000, 70000):
        for rows in (1, 200):
            x = torch.full((1, 1, rows, c), float("-inf"), device="cuda")
            x[..., c // 2] = 3.0
            x[0, 0, -1, c // 2] = float("nan") if rows > 1 else 3.0
            act = torch.full((1, 1, rows), c // 2, dtype=torch.int32, device="cuda")
            one = torch.ones((1, 1, rows), device="cuda")
            lp, ent, grad, loss = torch.empty_like(one), torch.empty_like(one), torch.empty_like(x), torch.empty(1, device="cuda")
            B.bc_action_log_probs(x, c, act, lp, ent)
            B.bc_clipped_policy_loss(x, c, act, one, one * 0, None, None, (0.2, 0.2, 0.0), 1.0, grad, loss)
            torch.cuda.synchronize()
            n = rows - (rows > 1)
            assert not lp[0, 0, :n].any() and not ent[0, 0, :n].any() and not grad[0, 0, :n].any(), c
            if rows > 1:
                assert torch.isnan(lp[0, 0, -1]) and torch.isnan(grad[0, 0, -1, c // 2]) and torch.isnan(loss).all()
            else:
                assert float(loss) == -1.0


def test_offsets_past_32_bits(B):
    """2.2e9 scores: the last rows of a large map have what they have in a small one."""
    rows, c, k = 17000, 131072, 5
    x = torch.empty((1, 1, rows, c), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(5)
    tail = (2 * torch.randn((1, 1, 8, c), generator=g, device="cuda")).bfloat16()
    x[:, :, :-8] = tail[:, :, :1]
    x[:, :, -8:] = tail
    act = torch.randint(0, c, (1, 1, rows), generator=g, device="cuda", dtype=torch.int32)
    one = torch.ones((1, 1, rows), device="cuda")
    outs = []
    for v, a, o in ((x, act, one), (x[:, :, -200:].clone(), act[:, :, -200:].contiguous(), one[:, :, -200:].contiguous())):
        n = v.shape[2]
        top, index = torch.empty((1, 1, n, k), dtype=v.dtype, device="cuda"), torch.empty((1, 1, n, k), dtype=torch.int32, device="cuda")
        rest, lp, loss = torch.empty_like(o), torch.empty_like(o), torch.empty(1, device="cuda")
        B.bc_top_scores(v, c, 1.0, top, index, rest, (1, 1), None, None)
        B.bc_action_log_probs(v, c, a, lp)
        y = v.clone() if n == 200 else None
        w = o * 1e4
        B.bc_clipped_policy_loss(v, c, a, o, lp - 0.1, None, w, (0.2, 0.2, 0.0), 1.0, y if n == 200 else v, loss)
        first = (y if n == 200 else v)[:, :, -8:].clone()
        if n != 200:
            v[:, :, :-8] = tail[:, :, :1]
            v[:, :, -8:] = tail
        grad = torch.empty_like(v) if n == 200 else v
        B.bc_distill_loss(v, c, top, index, None, 1.0, w, 1.0, grad, loss)
        outs.append([t[:, :, -8:].clone() for t in (top, index, rest, lp)] + [first, grad[:, :, -8:].clone()])
        torch.cuda.synchronize()
    for p, q in zip(*outs):
        assert torch.equal(p, q)


# ------------------------------------------------------------------ streams, graphs, devices

def all_calls(B, st, work, stream=None):
    """One call of each operator on a state of tensors, chained as in training: the teacher's record,
    the student's gradient; the old log probabilities, the policy's gradient."""
    B.bc_top_scores(st["teacher"], st["classes"], 2.0, st["top"], st["index"], st["rest"], (1, 1), None, None, work=work[0],
                    stream=stream)
    B.bc_distill_loss(st["x"], st["classes"], st["top"], st["index"], st["rest"], 2.0, None, 0.1, st["g1"], st["l1"],
                      work=work[1], stream=stream)
    B.bc_action_log_probs(st["teacher"], st["classes"], st["act"], st["old"], st["ent"], work=work[2], stream=stream)
    B.bc_clipped_policy_loss(st["x"], st["classes"], st["act"], st["adv"], st["old"], st["old"], None, (0.2, 0.2, 0.1), 0.1,
                             st["g2"], st["l2"], st["kl"], work=work[3], stream=stream)


def new_state(seed, rows, c, dtype):
    g = torch.Generator(device="cuda").manual_seed(seed)
    nrm = lambda *s: torch.randn(s, generator=g, device="cuda")
    e = lambda *s, dt=torch.float32: torch.empty(s, dtype=dt, device="cuda")
    return dict(classes=c, teacher=(2 * nrm(2, 1, rows, c)).to(dtype), x=(2 * nrm(2, 1, rows, c)).to(dtype), adv=nrm(2, 1, rows),
                act=torch.randint(0, c, (2, 1, rows), generator=g, device="cuda", dtype=torch.int32),
                top=e(2, 1, rows, 9, dt=dtype), index=e(2, 1, rows, 9, dt=torch.int32), rest=e(2, 1, rows), old=e(2, 1, rows),
                ent=e(2, 1, rows), g1=e(2, 1, rows, c, dt=dtype), g2=e(2, 1, rows, c, dt=dtype), l1=e(2), l2=e(2), kl=e(2))


OUT = ("top", "index", "rest", "g1", "l1", "old", "ent", "g2", "l2", "kl")


def new_work(B, st):
    x, c = st["x"], st["classes"]
    sizes = (B.bc_top_scores_work(x, c, 9), B.bc_distill_loss_work(x, c, 9), B.bc_action_log_probs_work(x, c),
             B.bc_clipped_policy_loss_work(x, c))
    return [torch.full((max(s, 16),), 255, dtype=torch.uint8, device="cuda") for s in sizes]


@pytest.mark.parametrize("rows,c,dtype", [(700, 19, torch.bfloat16), (3, 50000, torch.float32), (200, 20000, torch.float16)])
def test_graph_replays_equal_eager_runs(B, rows, c, dtype):
    st, ref = new_state(1, rows, c, dtype), new_state(1, rows, c, dtype)
    work, rwork = new_work(B, st), new_work(B, st)
    all_calls(B, st, work)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        all_calls(B, st, work)
    for seed in range(2, 6):
        new = new_state(seed, rows, c, dtype)
        for key in ("teacher", "x", "adv", "act"):
            st[key].copy_(new[key])
            ref[key].copy_(new[key])
        all_calls(B, ref, rwork)
        torch.cuda.synchronize()
        for w in work:
            w.fill_(seed * 50)                                    # nothing is kept in a workspace
        graph.replay()
        torch.cuda.synchronize()
        for key in OUT:
            assert torch.equal(st[key], ref[key]), (seed, key)


def test_two_streams_at_once(B):
    rows, c = 150, 9001
    states = [new_state(s, rows, c, torch.bfloat16) for s in (1, 2)]
    want = []
    for st in states:
        all_calls(B, st, new_work(B, st))
        torch.cuda.synchronize()
        want.append([st[k].clone() for k in OUT])
        for k in OUT:
            st[k].zero_()
    streams = [torch.cuda.Stream() for _ in states]
    torch.cuda.synchronize()
    for _ in range(4):
        for st, s in zip(states, streams):
            all_calls(B, st, [None] * 4, stream=s)                 # workspaces of the calls' own
    torch.cuda.synchronize()
    for st, w in zip(states, want):
        for k, v in zip(OUT, w):
            assert torch.equal(st[k], v), k


def test_refusals_of_the_binding(B):
    st = new_state(1, 4, 30, torch.float32)
    x = st["x"]
    bad = lambda f, *a, **k: pytest.raises(ValueError, f, *a, **k)
    bad(B.bc_action_log_probs, x.cpu(), 30, st["act"].cpu(), st["old"].cpu())
    bad(B.bc_action_log_probs, x, 30, st["act"].long(), st["old"])
    bad(B.bc_action_log_probs, x, 1, st["act"], st["old"])
    bad(B.bc_action_log_probs, x, 30, st["act"][:1], st["old"])
    bad(B.bc_action_log_probs, x.transpose(0, 2), 30, st["act"], st["old"])
    bad(B.bc_action_log_probs, x, 30, st["act"], st["old"].cpu())
    bad(B.bc_distill_loss, x, 30, st["top"], st["index"].long(), None, 1.0, None, 1.0, st["g1"], st["l1"])
    bad(B.bc_distill_loss, x, 30, st["top"], st["index"], None, 1.0, None, 1.0, st["g1"].half(), st["l1"])
    bad(B.bc_distill_loss, x, 30, st["top"][..., :4], st["index"][..., :4].contiguous(), None, 1.0, None, 1.0, st["g1"], None)
    bad(B.bc_distill_loss, x, 30, st["top"], st["index"], st["rest"][0], 1.0, None, 1.0, st["g1"], st["l1"])
    bad(B.bc_distill_loss, x, 30, st["top"], st["index"], None, 1.0, None, 1.0, st["g1"], st["l1"][:1])
    bad(B.bc_top_scores, x, 30, 1.0, st["top"].half(), st["index"], None, (1, 1), None, None)
    bad(B.bc_top_scores, x, 30, 1.0, st["top"], st["index"], None, (1, 1), torch.zeros(2, dtype=torch.int64).cuda(), None)
    bad(B.bc_clipped_policy_loss, x, 30, st["act"], st["adv"].double(), st["old"], None, None, (0.2, 0.2, 0.0), 1.0, st["g2"], None)
    for fn in (lambda: B.bc_distill_loss(x, 30, st["top"], st["index"], None, 0.0, None, 1.0, st["g1"], None),
               lambda: B.bc_top_scores(x, 31, 1.0, st["top"], st["index"], None, (1, 1), None, None),
               lambda: B.bc_clipped_policy_loss(x, 30, st["act"], st["adv"], st["old"], None, None, (1.2, 0.2, 0.0), 1.0, st["g2"], None)):
        with pytest.raises(B.BCError) as e:
            fn()
        assert e.value.status == B.BC_ERR_SHAPE
    with pytest.raises(B.BCError) as e:                            # the gradient over half of the scores
        buf = torch.zeros(x.numel() + 8, device="cuda")
        B.bc_distill_loss(buf[:x.numel()].view(x.shape), 30, st["top"], st["index"], None, 1.0, None, 1.0,
                          buf[8:].view(x.shape), None)
    assert e.value.status == B.BC_ERR_ALIAS
    st = new_state(1, 400, 40, torch.float32)
    with pytest.raises(B.BCError) as e:
        B.bc_distill_loss(st["x"], 40, st["top"], st["index"], None, 1.0, None, 1.0, st["g1"], st["l1"],
                          work=torch.empty(8, dtype=torch.uint8, device="cuda"))
    assert e.value.status == B.BC_ERR_CAPACITY
