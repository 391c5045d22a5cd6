"""Layer normalisation on the device, forward on active blocks and backward, against the
formulas in 64 bits, element by element.

Tolerances, fixed before the kernels ran: u = 2^-24, a sum of c values on the device adds at
most d = c / 8 + 16 of them after one another (eight lanes at least hold a row of 64 or more),
so a mean is off by at most d u mean|.|, and with it
  e_xhat = (d + 8) u (rstd mean|x| + |xhat|),
from which the bounds below follow term by term; the store adds half an ulp of the format.
Sums over rows: at most rows / 32 + 700 additions after one another."""
import numpy as np
import pytest
import torch

import synth
from tests._util import TORCH, shifted

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF_ULP = {"f32": U, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 2.0 ** -149, "bf16": 2.0 ** -133, "f16": 2.0 ** -24}
EPS = 1e-5


@pytest.fixture(scope="module")
def bc(gpu):
    from paper_2108_09376_amd import bc
    return bc


def maps(seed, shape, dtype, scale=1.0, mean=0.5):
    r = synth.rng(seed)
    x = scale * (r.standard_normal(shape) + mean * r.standard_normal(shape[-1]))
    return torch.from_numpy(x.astype(np.float32)).to(TORCH[dtype]).cuda()


def vectors(seed, c):
    r = synth.rng(seed)
    f = lambda a: torch.from_numpy(a.astype(np.float32)).cuda()
    return f(1 + 0.3 * r.standard_normal(c)), f(0.3 * r.standard_normal(c))


def stats64(x):
    x = x.double()
    c = x.shape[-1]
    mean = x.sum(-1, keepdim=True) / c
    d = x - mean
    rstd = 1 / torch.sqrt((d * d).sum(-1, keepdim=True) / c + EPS)
    xhat = d * rstd
    e_xhat = (c / 8 + 24) * U * (rstd * x.abs().mean(-1, keepdim=True) + xhat.abs())
    return xhat, rstd, e_xhat


def forward64(x, gamma, beta, res, relu):
    """(y, bound of the error before the store's rounding)."""
    xhat, _, e = stats64(x)
    ga = 1.0 if gamma is None else gamma.double()
    be = torch.zeros(x.shape[-1], dtype=torch.float64, device=x.device) if beta is None else beta.double()
    y = xhat * ga + be
    tol = e * abs(ga) + 4 * U * ((xhat * ga).abs() + be.abs())
    if res is not None:
        y = y + res.double()
        tol = tol + 2 * U * (y.abs() + res.double().abs())
    return (y.clamp(min=0) if relu else y), tol


def check(got, want, tol, dtype):
    got, want = got.double(), want.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    bound = tol + HALF_ULP[dtype] * (want.abs() + tol) + TINY[dtype]
    over = ((got - want).abs() / bound).nan_to_num(0.0)
    assert over.max().item() <= 1.0, f"{over.max().item():.3g} of the bound"


ROWS = [  # dtype, n, h, w, c: every form of a row, whole and ragged, one value to long rows
    ("bf16", 1, 1, 1, 1), ("f32", 1, 3, 5, 1), ("f16", 1, 1, 7, 3), ("f32", 1, 2, 2, 3), ("bf16", 2, 3, 5, 7),
    ("bf16", 1, 16, 32, 64), ("f16", 1, 5, 7, 65), ("f32", 1, 3, 3, 32), ("f32", 2, 3, 3, 37), ("bf16", 1, 9, 9, 128),
    ("bf16", 1, 9, 9, 100), ("f16", 1, 4, 4, 256), ("bf16", 1, 4, 5, 255), ("f32", 1, 4, 4, 256), ("f32", 1, 4, 4, 255),
    ("bf16", 1, 3, 5, 512), ("f16", 1, 3, 5, 509), ("bf16", 1, 3, 5, 1024), ("bf16", 1, 3, 5, 777),
    ("bf16", 1, 2, 5, 2048), ("f32", 1, 2, 5, 1001), ("f16", 1, 2, 5, 2001), ("f32", 1, 2, 3, 2048),
    ("f32", 1, 2, 3, 4096), ("bf16", 1, 2, 3, 4096), ("f16", 1, 2, 3, 4099), ("bf16", 1, 1, 3, 8192),
    ("f16", 1, 1, 3, 16384), ("f32", 1, 1, 3, 8192), ("f32", 1, 1, 3, 8001), ("bf16", 1, 1, 3, 16385),
    ("f32", 1, 1, 3, 9000), ("f16", 1, 1, 70, 20000),
]


@pytest.mark.parametrize("dtype,n,h,w,c", ROWS)
@pytest.mark.parametrize("form", ["plain", "residual_relu", "no_affine"])
def test_forward_every_pixel(bc, dtype, n, h, w, c, form):
    x = maps(1, (n, h, w, c), dtype)
    gamma, beta = vectors(2, c) if form != "no_affine" else (None, None)
    res = maps(3, (n, h, w, c), dtype) if form == "residual_relu" else None
    relu = form == "residual_relu"
    out = torch.full_like(x, float("nan"))
    bc.bc_sparse_layer_norm(x, bc.BC_NHWC, gamma, beta, res, EPS, relu, out, (1, 1), None, None)
    check(out, *forward64(x, gamma, beta, res, relu), dtype)


@pytest.mark.parametrize("dtype,c", [("bf16", 64), ("bf16", 77), ("f16", 256), ("f32", 40), ("bf16", 2048), ("f32", 4100)])
def test_forward_active_blocks(bc, dtype, c):
    """Active blocks only; every other block keeps its bits, and is not read (NaN there)."""
    n, gh, gw, bh, bw = 2, 3, 4, 2, 5
    shape = (n, gh * bh, gw * bw, c)
    gamma, beta = vectors(5, c)
    for pattern in ("none", "one", "some", "all"):
        mask = {"none": np.zeros((n, gh, gw)), "one": np.eye(1, n * gh * gw, 17).reshape(n, gh, gw),
                "some": synth.bernoulli_mask(synth.rng(6), n, gh, gw, 0.4), "all": np.ones((n, gh, gw))}[pattern]
        mask = torch.from_numpy(mask.astype(np.uint8)).cuda()
        on = mask.bool().repeat_interleave(bh, 1).repeat_interleave(bw, 2)[..., None].expand(shape)
        x, res, prev = maps(7, shape, dtype), maps(8, shape, dtype), maps(9, shape, dtype)
        x, res = torch.where(on, x, float("nan")), torch.where(on, res, float("nan"))
        idx = torch.empty(n * gh * gw, dtype=torch.int32, device="cuda")
        cnt = torch.empty(1, dtype=torch.int32, device="cuda")
        bc.bc_build_block_index(mask, n, (gh, gw), idx, cnt)
        out = prev.clone()
        bc.bc_sparse_layer_norm(x, bc.BC_NHWC, gamma, beta, res, EPS, True, out, (gh, gw), idx, cnt)
        want, tol = forward64(x, gamma, beta, res, True)
        check(torch.where(on, out, 0), torch.where(on, want, 0), torch.where(on, tol, 0), dtype)
        bits = torch.int32 if dtype == "f32" else torch.int16
        assert torch.equal(out.view(bits)[~on], prev.view(bits)[~on])


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("c", [5, 64, 100, 1001, 4096, 5001])
def test_forward_in_place_and_unaligned(bc, dtype, c):
    """The output over the input or the residual, tensors that start anywhere: equal bits."""
    x, res = maps(10, (1, 3, 7, c), dtype), maps(11, (1, 3, 7, c), dtype)
    gamma, beta = vectors(12, c)
    want = torch.empty_like(x)
    bc.bc_sparse_layer_norm(x, bc.BC_NHWC, gamma, beta, res, EPS, True, want, (3, 7), None, None)
    over_x, over_res = x.clone(), res.clone()
    bc.bc_sparse_layer_norm(over_x, bc.BC_NHWC, gamma, beta, res, EPS, True, over_x, (3, 7), None, None)
    bc.bc_sparse_layer_norm(x, bc.BC_NHWC, gamma, beta, over_res, EPS, True, over_res, (3, 7), None, None)
    a, b, out = shifted(x, 1), shifted(res, 3), shifted(torch.zeros_like(x), 5)
    bc.bc_sparse_layer_norm(a, bc.BC_NHWC, shifted(gamma, 1), shifted(beta, 2), b, EPS, True, out, (3, 7), None, None)
    for got in (over_x, over_res, out):
        assert torch.equal(got, want)


def test_forward_special_values(bc):
    """Constant rows, large means, infinities and NaN: each stays in its own pixel."""
    c = 72
    x = maps(13, (1, 1, 6, c), "f32")
    x[0, 0, 0] = 3.25                                     # variance 0: beta
    x[0, 0, 1] += 4096.0                                  # a mean far above the spread
    x[0, 0, 2, 5] = float("nan")
    x[0, 0, 3, 71] = float("inf")
    gamma, beta = vectors(14, c)
    out = torch.empty_like(x)
    bc.bc_sparse_layer_norm(x, bc.BC_NHWC, gamma, beta, None, EPS, True, out, (1, 1), None, None)
    want, tol = forward64(x, gamma, beta, None, True)
    assert torch.equal(out[0, 0, 0], beta.clamp(min=0))
    check(out[:, :, [0, 1, 4, 5]], want[:, :, [0, 1, 4, 5]], tol[:, :, [0, 1, 4, 5]], "f32")
    assert torch.isnan(out[0, 0, 2]).all() and torch.isnan(out[0, 0, 3]).all()


def grad64(x, gamma, y, dy):
    xhat, rstd, e = stats64(x)
    c, rows = x.shape[-1], x[..., 0].numel()
    dy = dy.double()
    if y is not None:
        dy = torch.where(y > 0, dy, torch.zeros_like(dy))
    g = dy * (1.0 if gamma is None else gamma.double())
    mean = lambda t: t.mean(-1, keepdim=True)
    m, mx = mean(g), mean(g * xhat)
    dx = rstd * (g - m - xhat * mx)
    E = (c / 8 + 28) * U
    M = mean((g * xhat).abs())
    tol = rstd * (E * (2 * g.abs() + mean(g.abs()) + 2 * xhat.abs() * M) + e * M + xhat.abs() * mean(g.abs() * e))
    tol = tol + E * dx.abs()
    flat = lambda t: t.reshape(-1, c).sum(0)
    depth = (rows / 32 + 700) * U
    tg = flat(dy.abs() * e) + depth * flat((dy * xhat).abs())
    return (dx, tol), dy, (flat(dy * xhat), tg), (flat(dy), depth * flat(dy.abs()))


@pytest.mark.parametrize("dtype,n,h,w,c", ROWS + [("bf16", 1, 64, 128, 64), ("f32", 1, 40, 101, 24), ("f16", 2, 31, 33, 300)])
@pytest.mark.parametrize("form", ["plain", "relu_residual", "no_affine"])
def test_backward(bc, dtype, n, h, w, c, form):
    x, dy = maps(20, (n, h, w, c), dtype), maps(21, (n, h, w, c), dtype, 0.1, 0.0)
    gamma = None if form == "no_affine" else vectors(22, c)[0]
    y = res = None
    if form == "relu_residual":
        y = maps(23, (n, h, w, c), dtype).clamp(min=0)
        dy = torch.where(y > 0, dy, float("nan"))          # masked gradients are not used
        res = torch.full_like(x, float("nan"))
    dx = torch.full_like(x, float("nan"))
    dgamma = torch.full((c,), float("nan"), device="cuda")
    dbeta = dgamma.clone()
    bc.bc_layer_norm_grad(x, bc.BC_NHWC, gamma, y, dy, EPS, dx, res, dgamma, dbeta)
    (wx, tx), wdy, (wg, tg), (wb, tb) = grad64(x, gamma, y, dy)
    check(dx, wx, tx, dtype)
    check(dgamma, wg, tg, "f32")
    check(dbeta, wb, tb, "f32")
    if res is not None:
        assert torch.equal(res.double(), wdy)
    # added to what is there, and only what is wanted; the same bits again
    acc, only = torch.ones(c, device="cuda"), torch.empty_like(dbeta)
    dx2 = torch.empty_like(dx)
    bc.bc_layer_norm_grad(x, bc.BC_NHWC, gamma, y, dy, EPS, dx2, None, acc, None, accumulate=True)
    bc.bc_layer_norm_grad(x, bc.BC_NHWC, gamma, y, dy, EPS, dx2, None, None, only)
    assert torch.equal(acc, dgamma + 1) and torch.equal(only, dbeta) and torch.equal(dx2, dx)
    bc.bc_layer_norm_grad(x, bc.BC_NHWC, gamma, y, dy, EPS, dx2, None, None, None)
    assert torch.equal(dx2, dx)


@pytest.mark.parametrize("dtype,c", [("bf16", 64), ("f32", 77), ("f16", 1001), ("bf16", 5000), ("f32", 9001)])
def test_backward_in_place_and_unaligned(bc, dtype, c):
    x, dy = maps(30, (1, 4, 9, c), dtype), maps(31, (1, 4, 9, c), dtype, 0.1)
    y, gamma = maps(32, (1, 4, 9, c), dtype).clamp(min=0), vectors(33, c)[0]
    new = lambda: (torch.empty_like(x), torch.empty_like(x), torch.empty(c, device="cuda"), torch.empty(c, device="cuda"))
    want = new()
    bc.bc_layer_norm_grad(x, bc.BC_NHWC, gamma, y, dy, EPS, *want)
    over, got = dy.clone(), new()
    bc.bc_layer_norm_grad(x, bc.BC_NHWC, gamma, y, over, EPS, over, *got[1:])
    assert torch.equal(over, want[0]) and all(torch.equal(a, b) for a, b in zip(got[1:], want[1:]))
    over, xx, got = dy.clone(), x.clone(), new()
    bc.bc_layer_norm_grad(xx, bc.BC_NHWC, gamma, y, over, EPS, xx, over, *got[2:])
    assert torch.equal(xx, want[0]) and torch.equal(over, want[1]) and torch.equal(got[2], want[2])
    got = tuple(shifted(t, k + 1) for k, t in enumerate(new()))
    bc.bc_layer_norm_grad(shifted(x, 1), bc.BC_NHWC, shifted(gamma, 3), shifted(y, 5), shifted(dy, 7), EPS, *got)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("c", [1, 7, 64, 100, 255, 1001, 4096, 20001])
@pytest.mark.parametrize("eps", [1e-5, 1e-12])
def test_backward_flat_rows(bc, dtype, c, eps):
    """Rows of one value each (of so few bits that their sums are exact): x - mean is 0, so they
    add exactly nothing to dgamma, and dx is (g - mean(g)) / sqrt(eps)."""
    values = [3.25, -100.0, 4160.0, 30720.0] + ([2.0 ** 120, -(2.0 ** 120)] if c <= 255 and dtype != "f16" else [])
    n = 7 * len(values)
    x = torch.tensor(values, device="cuda").repeat(7).view(1, n, 1, 1).expand(1, n, 1, c).to(TORCH[dtype]).contiguous()
    dy, gamma = maps(90, (1, n, 1, c), dtype, 2.0 ** -8), vectors(91, c)[0]
    dx = torch.full_like(x, float("nan"))
    dgamma, dbeta = torch.full((c,), float("nan"), device="cuda"), torch.full((c,), float("nan"), device="cuda")
    bc.bc_layer_norm_grad(x, bc.BC_NHWC, gamma, None, dy, eps, dx, None, dgamma, dbeta)
    assert (dgamma == 0).all()
    flat = dy.double().reshape(-1, c)
    assert ((dbeta.double() - flat.sum(0)).abs() <= (n / 32 + 700) * U * flat.abs().sum(0)).all()
    g = dy.double() * gamma.double()
    rstd = 1 / np.sqrt(np.float64(np.float32(eps)))
    tol = rstd * (c / 8 + 28) * U * (g.abs() + g.abs().mean(-1, keepdim=True))
    want = rstd * (g - g.mean(-1, keepdim=True))
    inside = want.abs() < torch.finfo(TORCH[dtype]).max / 2
    check(torch.where(inside, dx.double(), 0), torch.where(inside, want, 0), tol, dtype)


def test_backward_against_differences(bc):
    """Directional derivatives of the forward pass in fp32, with central differences in 64
    bits on the same formula: d/dt loss(x + t v) = sum grad_in v, likewise gamma and beta."""
    c = 48
    x, w = maps(40, (1, 5, 7, c), "f32"), maps(41, (1, 5, 7, c), "f32", 1.0, 0.0)
    res = maps(42, (1, 5, 7, c), "f32")
    gamma, beta = vectors(43, c)
    y = torch.empty_like(x)
    bc.bc_sparse_layer_norm(x, bc.BC_NHWC, gamma, beta, res, EPS, True, y, (1, 1), None, None)
    dx, dres = torch.empty_like(x), torch.empty_like(x)
    dg, db = torch.empty_like(gamma), torch.empty_like(beta)
    bc.bc_layer_norm_grad(x, bc.BC_NHWC, gamma, y, w, EPS, dx, dres, dg, db)

    def loss(x, gamma, beta, res):
        y, _ = forward64(x, gamma, beta, res, True)
        return (y * w.double()).sum().item()

    at = [t.double() for t in (x, gamma, beta, res)]
    for k, grad in enumerate((dx, dg, db, dres)):
        v = torch.from_numpy(synth.rng(50 + k).standard_normal(tuple(at[k].shape))).cuda()
        t = 1e-6
        hi, lo = list(at), list(at)
        hi[k], lo[k] = at[k] + t * v, at[k] - t * v
        slope = (loss(*hi) - loss(*lo)) / (2 * t)
        got = (grad.double() * v).sum().item()
        scale = (grad.double() * v).abs().sum().item()
        # the differences' own error is about t^2 and 1e-10 / t; ReLU kinks within t move it by t
        assert abs(got - slope) <= 1e-4 * scale, (k, got, slope)


def test_streams_and_graph(bc):
    """On a stream of its own, and captured: replays equal eager calls on new inputs."""
    c = 96
    x, dy, gamma, beta = maps(60, (1, 16, 8, c), "bf16"), maps(61, (1, 16, 8, c), "bf16"), *vectors(62, c)
    y, dx, dg, db = torch.empty_like(x), torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(beta)
    work = torch.empty(bc.bc_layer_norm_grad_work(x, bc.BC_NHWC), dtype=torch.uint8, device="cuda")

    def step():
        bc.bc_sparse_layer_norm(x, bc.BC_NHWC, gamma, beta, None, EPS, True, y, (2, 2), None, None)
        bc.bc_layer_norm_grad(x, bc.BC_NHWC, gamma, y, dy, EPS, dx, None, dg, db, work=work)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (70, 71, 72):
        x.copy_(maps(seed, (1, 16, 8, c), "bf16"))
        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in (y, dx, dg, db)]
        for t in (y, dx, dg, db):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((y, dx, dg, db), want))


def test_offsets_past_32_bits(bc):
    """A map of more than 2^31 elements, forward and backward: pixels at both ends and on both
    sides of 2^31 elements against the formulas in 64 bits."""
    h, w, c = 16400, 1024, 128                             # 2.15e9 elements, 4.3 GB a map
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.empty((1, h, w, c), dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    gy = torch.empty_like(x).normal_(generator=gen)
    gamma = torch.rand(c, device="cuda", generator=gen) + 0.5
    beta = torch.rand(c, device="cuda", generator=gen) - 0.5
    y, gx = torch.full_like(x, float("nan")), torch.full_like(x, float("nan"))
    bc.bc_sparse_layer_norm(x, bc.BC_NHWC, gamma, beta, None, 1e-5, True, y, (h // 8, w // 8), None, None)
    bc.bc_layer_norm_grad(x, bc.BC_NHWC, gamma, y, gy, 1e-5, gx, None, None, None)
    row = 2 ** 31 // (w * c)
    for r in (0, 1, row - 1, row, row + 1, h - 1):
        at = slice(r, r + 1)
        xd, gd, gm = x[0, at].double(), gy[0, at].double(), gamma.double()
        mean = xd.mean(-1, keepdim=True)
        rstd = ((xd - mean) ** 2).mean(-1, keepdim=True).add(1e-5).rsqrt()
        hat = (xd - mean) * rstd
        want = torch.relu(hat * gm + beta.double())
        assert ((y[0, at].double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-5).all(), r
        g = gd * (y[0, at] > 0) * gm
        want = (g - g.mean(-1, keepdim=True) - hat * (g * hat).mean(-1, keepdim=True)) * rstd
        assert ((gx[0, at].double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-4).all(), r
    assert not y.isnan().any() and not gx.isnan().any()


@pytest.mark.parametrize("rows,c", [(2, 2 ** 26 + 5), (1, 2 ** 30 + 9), (1, 2 ** 31 - 1)])
def test_backward_more_channels_than_threads(bc, rows, c):
    """The sums over pixels of 2^27 and 2^31 columns: more than a launch has threads, more than
    31 bits count. Values of -1 and 1 and small integers: every sum over channels is exact in
    fp32 but for the last additions (4 u), xhat = x / sqrt(var + eps) to 8 u."""
    i = torch.arange(c, device="cuda", dtype=torch.int32)
    x = torch.empty((1, 1, rows, c), dtype=torch.bfloat16, device="cuda")
    dy, dx = torch.empty_like(x), torch.full_like(x, float("nan"))
    for r in range(rows):
        x[0, 0, r] = 1 - 2 * ((i + r) & 1)
        dy[0, 0, r] = (i * 5 + r * 3 >> 2) % 4 - 1
    del i
    dgamma, dbeta = torch.full((c,), float("nan"), device="cuda"), torch.full((c,), float("nan"), device="cuda")
    bc.bc_layer_norm_grad(x, bc.BC_NHWC, None, None, dy, EPS, dx, None, dgamma, dbeta)
    means = []
    for r in range(rows):
        sx = sxg = sg = 0.0
        for a in range(0, c, 1 << 27):
            xr, gr = x[0, 0, r, a:a + (1 << 27)].double(), dy[0, 0, r, a:a + (1 << 27)].double()
            sx, sg, sxg = sx + xr.sum().item(), sg + gr.sum().item(), sxg + (gr * xr).sum().item()
        mean = sx / c
        rstd = (1 - mean * mean + EPS) ** -0.5
        means.append((mean, rstd, sg / c, (sxg / c - mean * sg / c) * rstd))
    for a in range(0, c, 1 << 27):
        at = slice(a, min(c, a + (1 << 27)))
        wg = wb = 0.0
        for r, (mean, rstd, mg, mgx) in enumerate(means):
            g, xhat = dy[0, 0, r, at].double(), (x[0, 0, r, at].double() - mean) * rstd
            wg, wb = wg + g * xhat, wb + g
            want = rstd * (g - mg - xhat * mgx)
            assert ((dx[0, 0, r, at].double() - want).abs() <= 2.0 ** -8 * want.abs() + 64 * U).all()
        assert ((dgamma[at].double() - wg).abs() <= 8 * U * 2 * rows).all()
        assert torch.equal(dbeta[at].double(), wb)


def test_forward_most_channels(bc):
    """A row of 2^31 - 1 channels, as many as a size can say: -1 and 1 in turn."""
    c = 2 ** 31 - 1
    x = torch.empty((1, 1, 1, c), dtype=torch.bfloat16, device="cuda")
    x.view(-1)[0::2], x.view(-1)[1::2] = 1.0, -1.0
    out = torch.full_like(x, float("nan"))
    bc.bc_sparse_layer_norm(x, bc.BC_NHWC, None, None, None, 0.5, False, out, (1, 1), None, None)
    want = (1 / 1.5 ** 0.5) * torch.tensor([1.0, -1.0], dtype=torch.float64, device="cuda")
    for k in (0, 1):                                       # the mean is 1 / c, the variance 1 - 1 / c^2
        assert ((out.view(-1)[k::2].float() - want[k]).abs() <= 2.0 ** -8 * want[k].abs() + 8 * U).all()
