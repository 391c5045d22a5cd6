"""CPU: the operators on score maps refuse invalid arguments with the documented status before
anything is enqueued, and say how much workspace they need."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def B():
    from paper_2108_09376_amd import bc
    return bc


# addresses that are never touched: every call below is refused first, and only where no GPU is
no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="fake device pointers are used only on machines without a GPU")
X, TOP, INDEX, REST, GRAD, LOSS, WORK = [i << 32 for i in range(1, 8)]
ACT, ADV, OLD, REF, WEIGHT, KL, IDX, COUNT = [i << 32 for i in range(8, 16)]
MAP = (2, 30, 4, 6, 0, 1)                                          # n, c, h, w, f32, NHWC
BIG = 1 << 30
NAN, INF = float("nan"), float("inf")


def top(B, x=X, m=MAP, classes=30, k=5, t=1.0, out=TOP, index=INDEX, rest=REST, grid=(2, 3), idx=IDX, count=COUNT, cap=12,
        work=WORK, nbytes=BIG):
    return B.raw().bc_top_scores(x, B.bc_tensor(*m), classes, k, t, out, index, rest, B.bc_grid(*grid), idx, count, cap, work,
                                 nbytes, None)


def distill(B, x=X, m=MAP, classes=30, tp=TOP, td=1, index=INDEX, k=5, rest=REST, t=1.0, weight=WEIGHT, scale=1.0, grad=GRAD,
            loss=LOSS, work=WORK, nbytes=BIG):
    return B.raw().bc_distill_loss(x, B.bc_tensor(*m), classes, tp, td, index, k, rest, t, weight, scale, grad, loss, work, nbytes,
                                   None)


def logp(B, x=X, m=MAP, classes=30, act=ACT, out=OLD, ent=REF, work=WORK, nbytes=BIG):
    return B.raw().bc_action_log_probs(x, B.bc_tensor(*m), classes, act, out, ent, work, nbytes, None)


def clip(B, x=X, m=MAP, classes=30, act=ACT, adv=ADV, old=OLD, ref=REF, weight=WEIGHT, c=(0.2, 0.2, 0.1), scale=1.0, grad=GRAD,
         loss=LOSS, kl=KL, work=WORK, nbytes=BIG):
    cc = ctypes.byref(B.bc_policy_clip(*c)) if c else None
    return B.raw().bc_clipped_policy_loss(x, B.bc_tensor(*m), classes, act, adv, old, ref, weight, cc, scale, grad, loss, kl, work,
                                          nbytes, None)


@no_gpu
def test_maps_and_classes(B):
    for call in (top, distill, logp, clip):
        assert call(B, x=None) == B.BC_ERR_NULL
        assert call(B, m=(2, 30, 4, 6, 0, 0)) == B.BC_ERR_LAYOUT
        assert call(B, m=(2, 30, 4, 6, 3, 1)) == B.BC_ERR_DTYPE
        assert call(B, m=(0, 30, 4, 6, 0, 1)) == B.BC_ERR_SHAPE
        assert call(B, m=(2, 2 ** 31 - 1, 4, 6, 0, 1)) == B.BC_ERR_SHAPE   # past 4e9 elements
        assert call(B, m=(1, (1 << 30) + 1, 1, 1, 0, 1)) == B.BC_ERR_UNSUPPORTED
        for classes in (0, -1, 31):
            assert call(B, classes=classes) == B.BC_ERR_SHAPE
    for call in (distill, clip):
        # an image of more pixels than a workgroup takes needs a workspace
        wide = dict(m=(2, 30, 40, 60, 0, 1))
        assert call(B, **wide, work=None) == B.BC_ERR_NULL
        assert call(B, **wide, work=WORK + 8) == B.BC_ERR_UNSUPPORTED
        assert call(B, **wide, nbytes=8) == B.BC_ERR_CAPACITY and call(B, **wide, nbytes=-1) == B.BC_ERR_CAPACITY
        assert call(B, grad=None, loss=None) == B.BC_ERR_NULL
        assert call(B, scale=NAN) == B.BC_ERR_SHAPE and call(B, scale=INF) == B.BC_ERR_SHAPE
        assert call(B, loss=GRAD + 4) == B.BC_ERR_ALIAS
        assert call(B, grad=X, weight=X) == B.BC_ERR_ALIAS         # in place over its weights
        assert call(B, grad=X + 4) == B.BC_ERR_ALIAS
        assert call(B, weight=GRAD) == B.BC_ERR_ALIAS
        assert call(B, loss=X) == B.BC_ERR_ALIAS and call(B, **wide, work=X) == B.BC_ERR_ALIAS
        assert call(B, **wide, loss=WORK) == B.BC_ERR_ALIAS
    for call in (top, logp):                                       # long rows are split: these need one too
        long = (1, 100000, 1, 1, 0, 1)
        more = dict(grid=(1, 1)) if call is top else {}
        assert call(B, m=long, classes=100000, work=None, **more) == B.BC_ERR_NULL
        assert call(B, m=long, classes=100000, nbytes=8, **more) == B.BC_ERR_CAPACITY
        assert call(B, m=long, classes=100000, work=WORK + 4, **more) == B.BC_ERR_UNSUPPORTED


@no_gpu
def test_records(B):
    for k in (0, -1, 65):
        assert top(B, m=(2, 300, 4, 6, 0, 1), classes=300, k=k) == B.BC_ERR_SHAPE
        assert distill(B, k=k) == B.BC_ERR_SHAPE
    assert top(B, k=31) == B.BC_ERR_SHAPE                          # more than the classes
    for t in (0.0, -1.0, NAN, INF, 1e-45, 3e-39, 5e-39):
        assert top(B, t=t) == B.BC_ERR_SHAPE and distill(B, t=t) == B.BC_ERR_SHAPE
    for key in ("out", "index"):
        assert top(B, **{key: None}) == B.BC_ERR_NULL
    for key in ("tp", "index"):
        assert distill(B, **{key: None}) == B.BC_ERR_NULL
    assert distill(B, td=5) == B.BC_ERR_DTYPE
    assert top(B, idx=None) == B.BC_ERR_NULL
    assert top(B, cap=11) == B.BC_ERR_CAPACITY
    assert top(B, grid=(3, 3)) == B.BC_ERR_NOT_DIVISIBLE
    assert top(B, grid=(0, 3)) == B.BC_ERR_SHAPE
    for a, b in (("out", X), ("index", TOP + 8), ("rest", INDEX), ("index", IDX), ("out", COUNT), ("rest", X + 64)):
        assert top(B, **{a: b}) == B.BC_ERR_ALIAS, (a, b)
    for a, b in (("grad", TOP), ("grad", INDEX + 4), ("loss", REST), ("grad", WEIGHT)):
        assert distill(B, **{a: b}) == B.BC_ERR_ALIAS, (a, b)


@no_gpu
def test_decisions(B):
    assert logp(B, act=None) == B.BC_ERR_NULL and logp(B, out=None) == B.BC_ERR_NULL
    for a, b in (("out", X), ("ent", OLD), ("out", ACT), ("ent", X + 400)):
        assert logp(B, **{a: b}) == B.BC_ERR_ALIAS, (a, b)
    for key in ("act", "adv", "old"):
        assert clip(B, **{key: None}) == B.BC_ERR_NULL
    assert clip(B, c=None) == B.BC_ERR_NULL
    assert clip(B, ref=None) == B.BC_ERR_NULL                      # with kl
    for c in ((-0.1, 0.2, 0.0), (1.1, 0.2, 0.0), (0.2, -0.1, 0.0), (0.2, INF, 0.0), (0.2, 0.2, -1.0), (NAN, 0.2, 0.0),
              (0.2, NAN, 0.0), (0.2, 0.2, NAN), (0.2, 0.2, INF)):
        assert clip(B, c=c) == B.BC_ERR_SHAPE, c
    for a, b in (("grad", ADV), ("kl", LOSS), ("loss", OLD), ("grad", ACT + 4), ("kl", REF)):
        assert clip(B, **{a: b}) == B.BC_ERR_ALIAS, (a, b)
    # decisions of one class are a byte each, of more an int
    small = dict(m=(1, 8, 1, 64, 0, 1), classes=1)
    assert logp(B, **small, out=ACT + 63) == B.BC_ERR_ALIAS
    assert logp(B, m=(1, 8, 1, 64, 0, 1), classes=2, out=ACT + 255) == B.BC_ERR_ALIAS


def test_workspaces(B):
    n = ctypes.c_int64(-1)
    t = B.bc_tensor(1, 64, 256, 512, 1, 1)
    lib = B.raw()
    assert lib.bc_top_scores_work(t, 19, 4, ctypes.byref(n)) == 0 and n.value == 0
    assert lib.bc_action_log_probs_work(t, 19, ctypes.byref(n)) == 0 and n.value == 0
    assert lib.bc_distill_loss_work(t, 19, 4, ctypes.byref(n)) == 0 and 16 <= n.value < 1 << 20
    assert lib.bc_clipped_policy_loss_work(t, 19, ctypes.byref(n)) == 0 and 16 <= n.value < 1 << 20
    for f in (lib.bc_action_log_probs_work, lib.bc_clipped_policy_loss_work):
        assert f(t, 19, None) == B.BC_ERR_NULL and f(t, 65, ctypes.byref(n)) == B.BC_ERR_SHAPE
    for f in (lib.bc_top_scores_work, lib.bc_distill_loss_work):
        assert f(t, 19, 4, None) == B.BC_ERR_NULL and f(t, 65, 4, ctypes.byref(n)) == B.BC_ERR_SHAPE
        assert f(t, 19, 65, ctypes.byref(n)) == B.BC_ERR_SHAPE
    x = torch.empty((2, 3, 4, 24))
    assert B.bc_distill_loss_work(x, 20, 3) == 0 == B.bc_clipped_policy_loss_work(x, 20)
    y = torch.empty((2, 1, 400, 40))
    assert B.bc_distill_loss_work(y, 40, 3) > 0 and B.bc_clipped_policy_loss_work(y, 40) > 0
    with pytest.raises(ValueError):
        B.bc_distill_loss_work(x.transpose(1, 2), 20, 3)
    with pytest.raises(ValueError):                                # not on a GPU: never handed on
        B.bc_action_log_probs(x, 20, torch.zeros((2, 3, 4), dtype=torch.int32), torch.zeros((2, 3, 4)))
