"""Orthogonalised updates on the device against the iteration in 64 bits.

Tolerances, fixed before the kernels ran. The operators promise fp32 accuracy, so the
measure is what plain fp32 arithmetic does on the same matrix: with e32 the relative error
(Frobenius norm) of the textbook iteration computed in fp32 on the CPU, the device's fp32
result may be off by 4 e32 + 2e-6 (4: other orders of summation and rounding; 2e-6: eight
fp32 roundings of the whole matrix, where e32 happens to vanish). A 16-bit result adds its
rounding. An optimiser's step scales that error by its rate."""
import math

import numpy as np
import pytest
import torch

import synth
from tests._util import TORCH, shifted

pytestmark = pytest.mark.gpu

COEF, EPS = (3.4445, -4.7750, 2.0315), 1e-7
ROUND = {"f32": 0.0, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}


@pytest.fixture(scope="module")
def bc(gpu):
    from paper_2108_09376_amd import bc
    return bc


def iterate(g, steps=5, coef=COEF, eps=EPS, dtype=torch.float64):
    g = g.detach().cpu().to(dtype)
    x = g / (torch.sqrt((g.double() ** 2).sum()).to(dtype) + eps)
    flip = x.shape[0] > x.shape[1]
    x = x.T.contiguous() if flip else x
    for _ in range(steps):
        a = x @ x.T
        x = coef[0] * x + (coef[1] * a + coef[2] * (a @ a)) @ x
    return x.T if flip else x


def bounds(g, dtype, **kw):
    want = iterate(g, **kw)
    e32 = ((iterate(g, dtype=torch.float32, **kw).double() - want).norm() / want.norm().clamp(min=1e-300)).item()
    return want, 4 * e32 + 2e-6 + ROUND[dtype]


def check(got, want, tol, dtype):
    got = got.detach().double().cpu()
    assert torch.isfinite(got).all()
    norm = want.norm().item()
    assert (got - want).norm().item() <= tol * norm + 1e-30, ((got - want).norm().item() / norm, tol)
    # no single element far off: within 64 times the bound of the mean element, plus its rounding
    rms = norm / math.sqrt(want.numel())
    assert ((got - want).abs() <= 64 * (tol - ROUND[dtype]) * rms + 2 * ROUND[dtype] * (want.abs() + 1e-6)).all()


def gradient(seed, m, n, kind="fall"):
    r = synth.rng(seed)
    k = max(1, min(m, n) // 2)
    if kind == "noise":
        g = r.standard_normal((m, n))
    elif kind == "rank":                                   # fewer directions than rows
        g = r.standard_normal((m, k)) @ r.standard_normal((k, n))
    else:
        g = (r.standard_normal((m, k)) * np.exp(-np.linspace(0, 3, k))) @ r.standard_normal((k, n)) / math.sqrt(k)
        g += 0.1 * r.standard_normal((m, n))
    return torch.from_numpy((1e-3 * g).astype(np.float32))


SIZES = [(1, 1), (1, 9), (9, 1), (3, 2), (8, 8), (63, 65), (64, 64), (65, 64), (64, 147), (64, 576), (100, 37), (128, 128),
         (129, 130), (128, 64), (127, 1152), (256, 256), (256, 129), (193, 301), (300, 257), (256, 1152), (320, 320),
         (512, 1000), (513, 77), (700, 641)]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("m,n", SIZES)
def test_sizes_and_formats(bc, dtype, m, n):
    g = gradient(m * 1000 + n, m, n).to(TORCH[dtype]).cuda()
    out = torch.full_like(g, float("nan"))
    bc.bc_orthogonalize(g, out)
    check(out, *bounds(g, dtype), dtype)
    again = torch.empty_like(out)
    bc.bc_orthogonalize(g, again)
    assert torch.equal(out, again)


@pytest.mark.parametrize("m,n", [(1800, 2000), (2000, 1800), (1700, 2300), (300, 4608), (4608, 300), (64, 4096), (512, 4608),
                                 (700, 2100)])
@pytest.mark.parametrize("kind", ["fall", "noise"])
def test_large_and_long(bc, m, n, kind):
    """Dense matrices of enough tiles for the large ones in every product, step by step and in
    spans (two jobs and two addends in a launch), and products long enough for ranges of K, whose
    sums meet in no fixed order of arrival: the same bits in every run."""
    g = gradient(m + n, m, n, kind)
    out, again = torch.empty_like(g, device="cuda"), torch.empty_like(g, device="cuda")
    g = g.cuda()
    bc.bc_orthogonalize(g, out)
    check(out, *bounds(g, "f32"), "f32")
    for _ in range(3):
        bc.bc_orthogonalize(g, again)
        assert torch.equal(out, again)


def test_batch_in_large_tiles(bc):
    """40 matrices of 193 x 301 take the large tiles, one of them the small ones: the same bits."""
    g = torch.stack([gradient(500 + i, 193, 301) for i in range(40)]).cuda()
    out, alone = torch.empty_like(g), torch.empty_like(g[0])
    bc.bc_orthogonalize(g, out)
    for i in (0, 1, 19, 39):
        bc.bc_orthogonalize(g[i], alone)
        assert torch.equal(out[i], alone)
        check(out[i], *bounds(g[i], "f32"), "f32")


@pytest.mark.parametrize("shapes", [[(1800, 2000), (600, 700), (64, 2304)],               # large tiles, 48 chunks and more whole
                                    [(300, 400)] * 40,                                    # large tiles, many matrices
                                    [(700, 5000), (400, 1200), (2304, 64), (128, 1152)]])  # in ranges beside short ones
def test_step_of_large_and_long(bc, shapes):
    """The step over many matrices against each by itself: to the bit up to 1408, else to rounding."""
    params = [(torch.zeros(s, device="cuda"), torch.zeros(s, device="cuda"), gradient(i + 600, *s).cuda(), None)
              for i, s in enumerate(shapes)]
    alone = [tuple(None if t is None else t.clone() for t in p) for p in params]
    again = [tuple(None if t is None else t.clone() for t in p) for p in params]
    bc.bc_muon_step_many(params, 1.0, 0.0, 0.0, nesterov=False)
    bc.bc_muon_step_many(again, 1.0, 0.0, 0.0, nesterov=False)
    for i, (p, a, b) in enumerate(zip(params, alone, again)):
        assert torch.equal(p[0], b[0])
        if i % 13 == 0 or len(shapes) < 13:
            bc.bc_muon_step_many([a], 1.0, 0.0, 0.0, nesterov=False)
            if max(shapes[i]) <= 1408:
                assert torch.equal(p[0], a[0])
            rate = math.sqrt(max(1.0, shapes[i][0] / shapes[i][1]))
            for w in (p[0], a[0]):
                check(w / -rate, *bounds(gradient(i + 600, *shapes[i]), "f32"), "f32")


@pytest.mark.parametrize("m,n", [(64, 64), (96, 512), (256, 256), (300, 90)])
@pytest.mark.parametrize("kind", ["noise", "rank"])
def test_spectra(bc, m, n, kind):
    g = gradient(5, m, n, kind).cuda()
    out = torch.empty_like(g)
    bc.bc_orthogonalize(g, out)
    check(out, *bounds(g, "f32"), "f32")


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 6, 7, 9])
@pytest.mark.parametrize("m,n", [(48, 80), (200, 140)])
def test_steps(bc, steps, m, n):
    g = gradient(7, m, n).cuda()
    out = torch.empty_like(g)
    bc.bc_orthogonalize(g, out, steps=steps)
    check(out, *bounds(g, "f32", steps=steps), "f32")


@pytest.mark.parametrize("coef", [(1.5, -0.5, 0.0), (1.875, -1.25, 0.375), (2.0, -1.5, 0.5), (1.0, 0.0, 0.0)])
def test_other_coefficients(bc, coef):
    g = gradient(8, 70, 150, "noise").cuda()
    out = torch.empty_like(g)
    bc.bc_orthogonalize(g, out, steps=4, coef=coef, eps=1e-6)
    check(out, *bounds(g, "f32", steps=4, coef=coef, eps=1e-6), "f32")


@pytest.mark.parametrize("coef", [COEF, (1.5, -0.5, 0.0), (1.875, -1.25, 0.375), (2.0, -1.5, 0.5)])
@pytest.mark.parametrize("steps", [2, 4, 5, 7, 8])
def test_other_coefficients_in_spans(bc, coef, steps):
    g = gradient(12, 400, 600, "noise").cuda()
    out = torch.empty_like(g)
    bc.bc_orthogonalize(g, out, steps=steps, coef=coef)
    check(out, *bounds(g, "f32", steps=steps, coef=coef), "f32")


def test_one_value_in_spans(bc):
    """One element, whose singular value is 1: the factors of a span are as large as the check of
    the coefficients counts them (2.19 three times, 10.5, in the first)."""
    coef = (0.45704228, -0.49950711, 1.04263144)
    g = torch.zeros(500, 1000, device="cuda")
    g[3, 5] = 1.0
    out = torch.empty_like(g)
    for steps in (3, 5, 6):
        bc.bc_orthogonalize(g, out, steps=steps, coef=coef, eps=0.0)
        s = 1.0
        for _ in range(steps):                             # an error grows less than fivefold a step, on the mean
            s = coef[0] * s + coef[1] * s ** 3 + coef[2] * s ** 5
        assert abs(out[3, 5].item() - s) <= 2e-6 * 5.0 ** steps * s
        out[3, 5] = 0.0
        assert not out.any()


@pytest.mark.parametrize("batch,m,n", [(1, 40, 50), (3, 65, 33), (12, 193, 301), (40, 17, 70), (300, 8, 16)])
def test_batches(bc, batch, m, n):
    """Each matrix by itself: a matrix of a batch has the bits it has alone; formats may
    differ; a NaN or zeros stay where they are."""
    g = torch.stack([gradient(100 + i, m, n) * 4.0 ** (i % 5 - 2) for i in range(batch)]).cuda()
    out = torch.empty_like(g)
    bc.bc_orthogonalize(g, out)
    for i in {0, batch // 2, batch - 1}:
        check(out[i], *bounds(g[i], "f32"), "f32")
        alone = torch.empty_like(g[i])
        bc.bc_orthogonalize(g[i], alone)
        assert torch.equal(alone, out[i])
    if batch >= 3:
        g[0], g[2, m // 2, n // 2] = 0.0, float("nan")
        half = torch.empty_like(g, dtype=torch.bfloat16)
        bc.bc_orthogonalize(g, half)
        assert (half[0] == 0).all() and torch.isnan(half[2]).all()
        assert torch.equal(half[1], out[1].bfloat16())


@pytest.mark.parametrize("m,n", [(140, 200), (193, 301), (256, 256), (256, 2304), (4000, 150), (320, 1000), (512, 512),
                                 (640, 512)])
@pytest.mark.parametrize("kind", ["fall", "noise", "rank"])
def test_no_further_off_than_fp32(bc, m, n, kind):
    """What is promised as fp32 accuracy is no worse than plain fp32 arithmetic: the mean
    difference to 64 bits over three matrices is at most that of the textbook form in fp32."""
    here = fp32 = 0.0
    for seed in (11, 12, 13):
        g = gradient(seed, m, n, kind)
        want = iterate(g)
        out = torch.empty_like(g, device="cuda")
        bc.bc_orthogonalize(g.cuda(), out)
        here += ((out.double().cpu() - want).norm() / want.norm()).item()
        fp32 += ((iterate(g, dtype=torch.float32).double() - want).norm() / want.norm()).item()
    assert here <= fp32, (here / 3, fp32 / 3)


def test_magnitudes(bc):
    """The result does not depend on G's scale, from values near fp32's largest to small
    ones (eps = 0), and eps takes part where the norm is near it."""
    g = gradient(9, 48, 90)
    for scale in (1e35, 1.0, 1e-30):
        s = (g * scale).cuda()
        out = torch.empty_like(s)
        bc.bc_orthogonalize(s, out, eps=0.0)
        check(out, *bounds(s.double(), "f32", eps=0.0), "f32")
    s = (g * 1e-6).cuda()
    out = torch.empty_like(s)
    bc.bc_orthogonalize(s, out, eps=1e-6)
    check(out, *bounds(s, "f32", eps=1e-6), "f32")


def test_in_place_and_unaligned(bc):
    for dtype in ("f32", "bf16", "f16"):
        g = gradient(10, 75, 131).to(TORCH[dtype]).cuda()
        want, over = torch.empty_like(g), g.clone()
        bc.bc_orthogonalize(g, want)
        bc.bc_orthogonalize(over, over)
        out = shifted(torch.zeros_like(g), 3)
        bc.bc_orthogonalize(shifted(g, 1), out)
        assert torch.equal(over, want) and torch.equal(out, want)


@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_step_many(bc, nesterov, dtype):
    shapes = [(64, 288), (64, 9, 64), (128, 64), (1, 5), (5, 1), (130, 3, 3, 20), (256, 129), (33, 70), (300, 40)]
    lr, mu, wd = 0.02, 0.95, 0.01
    params, copies = [], []
    for i, shape in enumerate(shapes):
        m, n = shape[0], math.prod(shape[1:])
        r = synth.rng(200 + i)
        w = torch.from_numpy((r.standard_normal(shape) * math.sqrt(2 / n)).astype(np.float32))
        copies.append((w, gradient(300 + i, m, n).view(shape) * 5, gradient(400 + i, m, n).view(shape)))
        p = [t.clone().cuda() for t in copies[-1]]
        params.append((*p, torch.empty(shape, dtype=TORCH[dtype], device="cuda") if i % 3 else None))
    bc.bc_muon_step_many(params, lr, mu, wd, nesterov=nesterov)
    for (w0, m0, g0), (w, m, g, w16) in zip(copies, params):
        rows, cols = w0.shape[0], w0[0].numel()
        m1 = mu * m0.double() + g0.double()
        assert ((m.double().cpu() - m1).abs() <= 2.0 ** -23 * (mu * m0.abs() + g0.abs() + m1.abs())).all()
        assert (g == 0).all()
        u = g0.double() + mu * m1 if nesterov else m1
        o, tol = bounds(u.float().view(rows, cols), "f32")
        rate = lr * math.sqrt(max(1.0, rows / cols))
        want = (1 - lr * wd) * w0.double() - rate * o.view(w0.shape)
        err = (w.double().cpu() - want).norm().item()
        # u itself is rounded to fp32 (as any fp32 form's is): one part in 2^23 more
        assert err <= rate * (tol + 2.0 ** -22) * o.norm().item() + 2.0 ** -23 * want.norm().item()
        if w16 is not None:
            assert torch.equal(w16, w.to(TORCH[dtype]))


def test_step_equals_its_parts(bc):
    """The step over many matrices takes each as bc_orthogonalize does, and a matrix does not
    depend on its neighbours."""
    shapes = [(64, 576), (128, 1152), (200, 31)]
    make = lambda: [(torch.zeros(s, device="cuda"), torch.zeros(s, device="cuda"), gradient(i, *s).cuda(), None)
                    for i, s in enumerate(shapes)]
    a, b = make(), make()
    outs = []
    for i, s in enumerate(shapes):
        outs.append(torch.empty(s, device="cuda"))
        bc.bc_orthogonalize(gradient(i, *s).cuda(), outs[-1])
    bc.bc_muon_step_many(a, 1.0, 0.0, 0.0, nesterov=False)
    for p in b:
        bc.bc_muon_step_many([p], 1.0, 0.0, 0.0, nesterov=False)
    for (w, *_), (w1, *_), o in zip(a, b, outs):
        assert torch.equal(w, w1)
        rate = math.sqrt(max(1.0, w.shape[0] / w.shape[1]))
        assert ((w + rate * o).abs() <= 2.0 ** -22 * rate * o.abs()).all()


@pytest.mark.parametrize("shapes,long", [([(64, 576), (128, 1152), (576, 64), (200, 1408)], (64, 2304)),
                                         ([(64, 1000), (1400, 130), (300, 900)], (4000, 100)),
                                         ([(64, 640), (150, 800)], (300, 4608))])
def test_step_beside_long_products(bc, shapes, long):
    """A product along more than 1408 elements may be summed in ranges. The matrices beside it have
    the bits they have alone; it agrees with itself to rounding."""
    make = lambda ss: [(gradient(i + 60, *s).cuda(), torch.zeros(s, device="cuda"), gradient(i, *s).cuda(), None)
                       for i, s in enumerate(ss)]
    together, alone = make(shapes + [long]), make(shapes + [long])
    before = [p[0].double().cpu() for p in alone]
    bc.bc_muon_step_many(together, 0.1, 0.9, 0.0)
    for p in alone:
        bc.bc_muon_step_many([p], 0.1, 0.9, 0.0)
    for i, (p, q) in enumerate(zip(together, alone)):
        if i < len(shapes):
            assert torch.equal(p[0], q[0]), shapes[i]
    g = gradient(len(shapes), *long)
    o, tol = bounds(g.double() * 1.9, "f32")
    rate = 0.1 * math.sqrt(max(1.0, long[0] / long[1]))
    for p in (together[-1], alone[-1]):
        err = (p[0].double().cpu() - (before[-1] - rate * o)).norm().item()
        assert err <= rate * (tol + 2.0 ** -22) * o.norm().item() + 2.0 ** -23 * before[-1].norm().item()


@pytest.mark.parametrize("nesterov", [False, True])
def test_small_matrices_alone_and_among_large(bc, nesterov):
    """Small matrices take one launch by themselves and the products' launches beside larger ones:
    the same result either way, to the bit."""
    shapes = [(1, 1), (5, 3), (64, 64), (64, 147), (147, 64), (30, 129), (64, 512), (500, 33), (128, 128), (65, 128), (128, 97)]
    def make():
        return [(gradient(i + 50, *s).cuda(), gradient(i + 20, *s).cuda(), gradient(i, *s, "noise").cuda(),
                 torch.empty(s, dtype=torch.bfloat16, device="cuda")) for i, s in enumerate(shapes)]
    large = lambda: [(torch.zeros(300, 400, device="cuda"), torch.zeros(300, 400, device="cuda"), gradient(9, 300, 400).cuda(), None)]
    among, together, alone = make(), make(), make()
    for _ in range(2):                                     # two steps: the momentum as well
        bc.bc_muon_step_many(among + large(), 0.1, 0.9, 0.01, nesterov=nesterov)
        bc.bc_muon_step_many(together, 0.1, 0.9, 0.01, nesterov=nesterov)
        for p in alone:
            bc.bc_muon_step_many([p], 0.1, 0.9, 0.01, nesterov=nesterov)
        for p, q, r, s in zip(among, together, alone, shapes):
            for x, y, z in zip(p, q, r):
                assert torch.equal(x, y) and torch.equal(x, z), s
            for x in (p, q, r):
                assert not x[2].any()                      # the gradient has been taken
                x[2].copy_(gradient(77, *s))


# Normal values (8 x 16 by seed) with two of them set so that the sum of squares lies where its
# last bit in 64 bits, that is the order of summation, decides on the norm's rounding to 32.
EDGES = [(0, "0x1.e7dab4p-1", "0x1.6ef872p-13"), (1, "0x1.d1f888p-1", "0x1.2a1f0cp-12"),
         (2, "0x1.ed6dc6p-1", "0x1.8cc1e0p-13"), (4, "0x1.0016c4p+0", "0x1.c7fd54p-13"),
         (9, "0x1.0a11d8p+0", "0x1.69c1a4p-13"), (12, "0x1.e3d394p-1", "0x1.0075cep-12"),
         (17, "0x1.0a327ep+0", "0x1.5b1508p-12"), (18, "0x1.e9e41ep-1", "0x1.441b9cp-12")]


@pytest.mark.parametrize("seed,first,last", EDGES)
def test_norm_in_one_order(bc, seed, first, last):
    """The norm's sum is taken in one order, whichever kernel takes it: the bits are the same alone
    and beside a larger matrix."""
    g = np.random.default_rng(seed).standard_normal((8, 16)).astype(np.float32)
    g[0, 0], g[7, 15] = float.fromhex(first), float.fromhex(last)
    make = lambda a: (torch.zeros(a.shape, device="cuda"), torch.zeros(a.shape, device="cuda"), torch.from_numpy(a).cuda(), None)
    alone, beside = make(g), make(g)
    bc.bc_muon_step_many([alone], 1.0, 0.0, 0.0, nesterov=False, eps=0.0)
    bc.bc_muon_step_many([beside, make(np.ones((300, 400), np.float32))], 1.0, 0.0, 0.0, nesterov=False, eps=0.0)
    assert torch.equal(alone[0], beside[0])


def test_streams_and_graph(bc):
    """On a stream of its own, and captured: replays equal eager calls on new gradients."""
    shapes = [(64, 576), (300, 200)]
    params = [(torch.zeros(s, device="cuda"), torch.zeros(s, device="cuda"), gradient(i, *s).cuda(), None)
              for i, s in enumerate(shapes)]
    work = torch.empty(bc.bc_muon_step_many_work(params), dtype=torch.uint8, device="cuda")
    step = lambda: bc.bc_muon_step_many(params, 0.1, 0.9, 0.0, work=work)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (20, 30, 40):
        before = [(w.clone(), m.clone()) for w, m, _, _ in params]
        fresh = [gradient(seed + i, *s).cuda() for i, s in enumerate(shapes)]

        def load():
            for (w, m, g, _), (w0, m0), f in zip(params, before, fresh):
                w.copy_(w0), m.copy_(m0), g.copy_(f)

        load()
        step()
        torch.cuda.synchronize()
        want = [(w.clone(), m.clone()) for w, m, _, _ in params]
        load()
        graph.replay()
        torch.cuda.synchronize()
        for (w, m, g, _), (w1, m1) in zip(params, want):
            assert torch.equal(w, w1) and torch.equal(m, m1) and (g == 0).all()


@pytest.mark.parametrize("by_handle", [False, True])
def test_workspace_belongs_to_the_stream(bc, monkeypatch, by_handle):
    """Calls on a stream that is not torch's current one and bring no workspace: what they take
    is not given to the current stream, whose work is not ordered with theirs, behind them."""
    made, real = [], bc._work

    def spy(*args):
        t = real(*args)
        made.append((t.data_ptr(), t.numel()))
        return t

    monkeypatch.setattr(bc, "_work", spy)
    g = gradient(11, 300, 400).cuda()
    params = [(g.clone(), g.clone(), g.clone(), None)]
    x, gamma = torch.randn(1, 32, 32, 4096, device="cuda"), torch.rand(4096, device="cuda")
    dx, dg = torch.empty_like(x), torch.empty_like(gamma)
    out, want = torch.empty_like(g), torch.empty_like(g)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    at = side.cuda_stream if by_handle else side
    for call in (lambda s: bc.bc_orthogonalize(g, out, stream=s),
                 lambda s: bc.bc_muon_step_many(params, 0.1, 0.9, 0.0, stream=s),
                 lambda s: bc.bc_layer_norm_grad(x, bc.BC_NHWC, gamma, None, x, 1e-5, dx, None, dg, None, stream=s)):
        torch.cuda.empty_cache()
        call(at)
        begin, size = made[-1]
        assert size > 1 << 20
        others = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(4)]
        assert all(t.data_ptr() >= begin + size or t.data_ptr() + size <= begin for t in others)
        side.synchronize()
    bc.bc_orthogonalize(g, want)
    assert torch.equal(out, want)


def test_handle_of_the_default_stream(bc, monkeypatch):
    """A handle of 0 names the default stream, also for the workspace that is made for it."""
    device = torch.device("cuda", torch.cuda.current_device())
    assert bc.torch_stream(0, device) == torch.cuda.default_stream(device)
    side, on = torch.cuda.Stream(), []
    assert bc.torch_stream(side, device) is side
    assert bc.torch_stream(side.cuda_stream, device).cuda_stream == side.cuda_stream
    g = gradient(11, 300, 400).cuda()
    out = torch.empty_like(g)
    real = torch.empty
    torch.cuda.synchronize()
    monkeypatch.setattr(torch, "empty", lambda *a, **k: on.append(torch.cuda.current_stream().cuda_stream) or real(*a, **k))
    with torch.cuda.stream(side):
        bc.bc_orthogonalize(g, out, stream=torch.cuda.default_stream().cuda_stream)
    monkeypatch.undo()
    torch.cuda.synchronize()
    assert on == [0]
    check(out, *bounds(g, "f32"), "f32")


def test_offsets_past_32_bits(bc):
    """A matrix whose X passes 2^32 bytes, with one element per row: its singular values are
    those elements, and each becomes what the iteration makes of it alone."""
    m, n = 300, 2 ** 22
    cols = [0, 1, 31, 32, n // 2 - 1, n // 2, n - 129, n - 64, n - 2, n - 1]
    g = torch.zeros(m, n, device="cuda")
    values = [0.3 + 0.05 * i for i in range(len(cols))]
    rows = [i * (m - 1) // (len(cols) - 1) for i in range(len(cols))]
    for r, c, v in zip(rows, cols, values):
        g[r, c] = v
    norm = math.sqrt(sum(float(np.float32(v)) ** 2 for v in values)) + EPS
    out = torch.full_like(g, float("nan"))
    bc.bc_orthogonalize(g, out)
    for r, c, v in zip(rows, cols, values):
        s = float(np.float32(v)) / norm
        for _ in range(5):
            s = COEF[0] * s + COEF[1] * s ** 3 + COEF[2] * s ** 5
        assert abs(out[r, c].item() - s) <= 1e-5 * abs(s), (r, c)
        out[r, c] = 0.0
    assert not out.any()


def test_batches_past_32_bits(bc):
    """More than 2^31 elements in a batch: the last matrices as by themselves."""
    g = torch.empty((66000, 64, 512), dtype=torch.float16, device="cuda")
    g.normal_(generator=torch.Generator(device="cuda").manual_seed(4))
    out = torch.full_like(g, float("nan"))
    bc.bc_orthogonalize(g, out)
    for i in (0, 65535, 65536, 65999):
        alone = torch.empty_like(out[i])
        bc.bc_orthogonalize(g[i], alone)
        assert torch.equal(alone, out[i]), i
    assert not out.isnan().any()
