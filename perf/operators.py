"""The training operators of the policy network and the backbones whose speed is measured,
through the library's public entry points.

Layer normalisation over the channels of a channels-last map, run on a frame's active
blocks or on every pixel, with its backward pass; and the orthogonalised update: the
momentum of a weight matrix pushed towards the nearest orthogonal matrix by Newton-Schulz
products, alone or as an optimiser's whole step over many weight matrices.

The listed cases stand for
  norm_head        the first head layer of the policy network at 2048x1024: the smallest
                   map that a frame normalises, all latency
  norm_frame_s4    a stride-4 bottleneck's output in a sparse frame (38 of 128 blocks): norm,
                   shortcut, ReLU in one pass over the executed blocks
  norm_rows_f32    fp32 rows whose length and number divide by nothing
  grad_stem        the backward pass behind the policy network's stem, ReLU and shortcut
                   gradient included
  grad_wide_f16    the backward pass of long rows over many of them: the largest sums
  grad_odd_f32     fp32 rows of odd length, without ReLU
  orth_stem_f16    one stem's momentum, 64 x 147, fp16: the smallest matrix
  orth_batch_odd   a dozen equal matrices of odd sizes in one call, fp32
  orth_wide_f32    the 3x3 weights of a ResNet-50 stage-4 bottleneck, 512 x 4608
  orth_square      one large square matrix in bf16
  step_policy      the optimiser's step over the policy network's weight matrices
  step_resnet50    the same over every convolution of ResNet-50

Where the calls write over their inputs (the step), each pass brings a new gradient first,
as a backward pass does.
"""
import math
import random

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
NORM_EPS = 1e-5
STEPS, COEF, ORTH_EPS = 5, (3.4445, -4.7750, 2.0315), 1e-7
LR, MOMENTUM, DECAY = 0.02, 0.95, 0.01


# ------------------------------------------------------------------ the cases

def norm_case(dtype, n, gh, gw, bh, bw, c, active, res, relu):
    """A forward pass over maps of gh x gw blocks of bh x bw pixels; active 0: every block."""
    return dict(kind="norm", dtype=dtype, n=n, gh=gh, gw=gw, bh=bh, bw=bw, c=c, active=active, res=res,
                relu=relu)


def grad_case(dtype, n, h, w, c, relu, res):
    return dict(kind="grad", dtype=dtype, n=n, h=h, w=w, c=c, relu=relu, res=res)


def orth_case(dtype, batch, rows, cols):
    return dict(kind="orth", dtype=dtype, batch=batch, rows=rows, cols=cols)


def step_case(dtype, net, matrices, width):
    return dict(kind="step", dtype=dtype, net=net, matrices=matrices, width=width)


def listed():
    named = dict(
        norm_head=norm_case("bf16", 1, 8, 16, 2, 2, 64, 0, False, True),
        norm_frame_s4=norm_case("bf16", 1, 8, 16, 32, 32, 256, 38, True, True),
        norm_rows_f32=norm_case("f32", 1, 1, 1, 1, 8191, 1001, 0, False, False),
        grad_stem=grad_case("bf16", 1, 128, 256, 64, True, True),
        grad_wide_f16=grad_case("f16", 1, 1, 16384, 4096, False, False),
        grad_odd_f32=grad_case("f32", 1, 29, 53, 777, False, False),
        orth_stem_f16=orth_case("f16", 1, 64, 147),
        orth_batch_odd=orth_case("f32", 12, 193, 301),
        orth_wide_f32=orth_case("f32", 1, 512, 4608),
        orth_square=orth_case("bf16", 1, 2048, 2048),
        step_policy=step_case("bf16", "policy", 0, 0),
        step_resnet50=step_case("bf16", "resnet50", 0, 0),
    )
    return [dict(c, name=k) for k, c in named.items()]


def spread(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    what = rng.choices(("norm", "rows", "grad", "orth", "step"), (3, 2, 5, 5, 3))[0]
    kind = rng.choice(("bf16", "bf16", "f16", "f32"))
    if what == "norm":
        n, gh, gw = rng.randint(1, 3), rng.randint(2, 8), rng.randint(3, 16)
        edge = rng.choice((2, 4, 5, 8, 16, 32))
        top = min(2048, (1 << 25) // (n * gh * gw * edge * edge))
        c = spread(rng, 8, max(8, top))
        c = c if rng.random() < 0.4 else max(8, c // 8 * 8)
        return norm_case(kind, n, gh, gw, edge, edge, c,
                         max(1, spread(rng, 5, 100) * n * gh * gw // 100), rng.random() < 0.5,
                         rng.random() < 0.7)
    if what == "rows":
        rows = spread(rng, 1, 32768)
        return norm_case(kind, 1, 1, 1, 1, rows, spread(rng, 2, min(16384, max(2, (1 << 25) // rows))), 0,
                         rng.random() < 0.3, rng.random() < 0.3)
    if what == "grad":
        rows = spread(rng, 1, 65536)
        c = spread(rng, 8, min(8192, max(8, (1 << 25) // rows)))
        c = c if rng.random() < 0.4 else max(8, c // 8 * 8)
        relu = rng.random() < 0.5
        h = rng.randint(1, min(rows, 16))
        return grad_case(kind, 1, h, max(1, rows // h), c, relu, relu and rng.random() < 0.5)
    if what == "orth":
        rows, cols = spread(rng, 8, 2048), spread(rng, 8, 2048)
        if rng.random() < 0.5:
            rows, cols = max(8, rows // 8 * 8), max(8, cols // 8 * 8)
        batch = spread(rng, 1, max(1, min(48, (1 << 21) // (rows * cols))))
        return orth_case(kind, batch, rows, cols)
    return step_case(rng.choice(("bf16", "f16")), "drawn", rng.randint(1, 24), rng.randint(1, 8) * 32)


def shapes_of(case):
    """The weight matrices of a step, [output channels, everything else]."""
    if case["net"] == "policy":
        return [(64, 288), (64, 576), (64, 576), (128, 64), (128, 576), (128, 1152), (256, 128), (256, 1152),
                (256, 2304), (64, 2304), (64, 576)]
    if case["net"] == "resnet50":
        out, ch = [(64, 147)], 64
        for stage, blocks in enumerate((3, 4, 6, 3)):
            width = 64 << stage
            for b in range(blocks):
                if b == 0:
                    out.append((4 * width, ch))
                out += [(width, ch), (width, 9 * width), (4 * width, width)]
                ch = 4 * width
        return out
    rng = random.Random(case["matrices"] * 1000 + case["width"])
    out = []
    for _ in range(case["matrices"]):
        m = max(8, case["width"] * rng.choice((1, 1, 2, 4)) // rng.choice((1, 1, 3)))
        n = max(8, case["width"] * rng.choice((1, 2, 9, 9)) // rng.choice((1, 1, 5)))
        out.append((m, n))
    return out


# ------------------------------------------------------------------ inputs

def matrix_gradient(gen, batch, m, n):
    """Gradients as a layer's backward pass sums them: output gradients times inputs, of
    fewer directions than the matrix has and of falling weight, over a floor of noise."""
    k = max(1, min(m, n) // 2)
    fall = torch.linspace(0.0, -3.0, k, device=DEV).exp()
    g = torch.randn((batch, m, k), generator=gen, device=DEV) * fall
    x = torch.randn((batch, k, n), generator=gen, device=DEV)
    floor = torch.randn((batch, m, n), generator=gen, device=DEV)
    return (torch.matmul(g, x) / math.sqrt(k) + 0.1 * floor) * 1e-3


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=DEV)

    dt = DTYPES[case["dtype"]]
    s = dict(case=case, kept={})
    if case["kind"] in ("norm", "grad"):
        c = case["c"]
        n = case["n"]
        h, w = (case["gh"] * case["bh"], case["gw"] * case["bw"]) if case["kind"] == "norm" else (case["h"], case["w"])
        # a convolution's output: channels with means of their own
        s["x"] = (normal(n, h, w, c) + 0.5 * normal(c)).to(dt)
        s["gamma"], s["beta"] = 1.0 + 0.2 * normal(c), 0.2 * normal(c)
    if case["kind"] == "norm":
        s["res"] = normal(n, h, w, c).to(dt) if case["res"] else None
        s["out"] = normal(n, h, w, c).relu().to(dt)            # the previous frame's
        blocks = n * case["gh"] * case["gw"]
        s["idx"] = s["count"] = None
        if case["active"]:
            a = min(case["active"], blocks)
            ids = torch.randperm(blocks, generator=gen, device=DEV)[:a].sort().values
            s["idx"] = torch.zeros(blocks, dtype=torch.int32, device=DEV)
            s["idx"][:a] = ids.to(torch.int32)
            s["count"] = torch.full((1,), a, dtype=torch.int32, device=DEV)
    elif case["kind"] == "grad":
        s["y"] = normal(n, h, w, c).relu().to(dt) if case["relu"] else None
        s["grad_out"] = (1e-2 * normal(n, h, w, c)).to(dt)
        s["grad_in"] = torch.empty_like(s["x"])
        s["grad_res"] = torch.empty_like(s["x"]) if case["res"] else None
        s["dgamma"] = torch.empty(c, dtype=torch.float32, device=DEV)
        s["dbeta"] = torch.empty(c, dtype=torch.float32, device=DEV)
    elif case["kind"] == "orth":
        s["g"] = matrix_gradient(gen, case["batch"], case["rows"], case["cols"]).to(dt)
        s["out"] = torch.empty_like(s["g"])
    else:
        shapes = shapes_of(case)
        total = sum(m * n for m, n in shapes)
        for key in ("w", "m", "grad", "new_grad"):
            s[key] = torch.empty(total, dtype=torch.float32, device=DEV)
        s["w16"] = torch.empty(total, dtype=dt, device=DEV)
        s["shapes"], s["views"], at = shapes, {k: [] for k in ("w", "m", "grad", "w16")}, 0
        for m, n in shapes:
            s["w"][at:at + m * n] = normal(m * n) * math.sqrt(2.0 / n)
            s["m"][at:at + m * n] = 8.0 * matrix_gradient(gen, 1, m, n).reshape(-1)
            s["new_grad"][at:at + m * n] = matrix_gradient(gen, 1, m, n).reshape(-1)
            for key, views in s["views"].items():
                views.append(s[key][at:at + m * n].view(m, n))
            at += m * n
        s["w16"].copy_(s["w"])
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    kind = s["case"]["kind"]
    if own:
        return {"norm": own_norm, "grad": own_grad, "orth": own_orth, "step": own_step}[kind](s)
    return {"norm": plain_norm, "grad": plain_grad, "orth": plain_orth, "step": plain_step}[kind](s)


def kept_work(s, nbytes):
    """The workspace a program keeps beside its buffers."""
    if "work" not in s["kept"]:
        s["kept"]["work"] = torch.empty(nbytes(), dtype=torch.uint8, device=DEV)
    return s["kept"]["work"]


def own_norm(s):
    from paper_2108_09376_amd import bc
    c = s["case"]
    bc.bc_sparse_layer_norm(s["x"], bc.BC_NHWC, s["gamma"], s["beta"], s["res"], NORM_EPS, c["relu"], s["out"],
                            (c["gh"], c["gw"]), s["idx"], s["count"])
    return s["out"]


def own_grad(s):
    from paper_2108_09376_amd import bc
    work = kept_work(s, lambda: bc.bc_layer_norm_grad_work(s["x"], bc.BC_NHWC))
    bc.bc_layer_norm_grad(s["x"], bc.BC_NHWC, s["gamma"], s["y"], s["grad_out"], NORM_EPS, s["grad_in"],
                          s["grad_res"], s["dgamma"], s["dbeta"], accumulate=False, work=work)
    return s["grad_in"], s["grad_res"], s["dgamma"], s["dbeta"]


def own_orth(s):
    from paper_2108_09376_amd import bc
    work = kept_work(s, lambda: bc.bc_orthogonalize_work(s["g"], STEPS))
    bc.bc_orthogonalize(s["g"], s["out"], steps=STEPS, coef=COEF, eps=ORTH_EPS, work=work)
    return s["out"]


def own_step(s):
    from paper_2108_09376_amd import bc
    v = s["views"]
    s["grad"].copy_(s["new_grad"])
    params = list(zip(v["w"], v["m"], v["grad"], v["w16"]))
    work = kept_work(s, lambda: bc.bc_muon_step_many_work(params, STEPS))
    bc.bc_muon_step_many(params, LR, MOMENTUM, DECAY, nesterov=True, steps=STEPS, coef=COEF, eps=ORTH_EPS, work=work)
    return s["w"], s["m"], s["w16"]


def plain_rows(x, gamma, beta):
    x = x.float()
    d = x - x.mean(-1, keepdim=True)
    rstd = 1.0 / torch.sqrt((d * d).mean(-1, keepdim=True) + NORM_EPS)
    return d * rstd * gamma + beta


def plain_norm(s):
    c = s["case"]
    blocks = (c["n"], c["gh"], c["bh"], c["gw"], c["bw"], c["c"])

    def of(t):
        t = t.view(blocks)
        return t if at is None else t[at[0], at[1], :, at[2]]

    at = None
    if s["idx"] is not None:
        i = s["idx"][:min(c["active"], c["n"] * c["gh"] * c["gw"])].long()
        at = (i // (c["gh"] * c["gw"]), i // c["gw"] % c["gh"], i % c["gw"])
    y = plain_rows(of(s["x"]), s["gamma"], s["beta"])
    if s["res"] is not None:
        y = y + of(s["res"]).float()
    if c["relu"]:
        y = y.clamp(min=0.0)
    out = s["out"].view(blocks)
    if at is None:
        out.copy_(y)
    else:
        out[at[0], at[1], :, at[2]] = y.to(out.dtype)
    return s["out"]


def plain_grad(s):
    x = s["x"].float()
    d = x - x.mean(-1, keepdim=True)
    rstd = 1.0 / torch.sqrt((d * d).mean(-1, keepdim=True) + NORM_EPS)
    xhat = d * rstd
    dy = s["grad_out"].float()
    if s["y"] is not None:
        dy = dy * (s["y"] > 0)
    g = dy * s["gamma"]
    s["grad_in"].copy_(rstd * (g - g.mean(-1, keepdim=True) - xhat * (g * xhat).mean(-1, keepdim=True)))
    if s["grad_res"] is not None:
        s["grad_res"].copy_(dy)
    s["dgamma"].copy_((dy * xhat).sum((0, 1, 2)))
    s["dbeta"].copy_(dy.sum((0, 1, 2)))
    return s["grad_in"], s["grad_res"], s["dgamma"], s["dbeta"]


def plain_newton_schulz(g):
    """g [..., rows, cols]; the products run on the shorter side."""
    x = g.float()
    x = x / (torch.sqrt((x * x).sum((-2, -1), keepdim=True)) + ORTH_EPS)
    tall = x.shape[-2] > x.shape[-1]
    if tall:
        x = x.transpose(-2, -1).contiguous()
    a, b, c = COEF
    for _ in range(STEPS):
        p = torch.matmul(x, x.transpose(-2, -1).contiguous())
        x = a * x + torch.matmul(b * p + c * torch.matmul(p, p), x)
    return x.transpose(-2, -1) if tall else x


def plain_orth(s):
    s["out"].copy_(plain_newton_schulz(s["g"]))
    return s["out"]


def plain_step(s):
    s["grad"].copy_(s["new_grad"])
    s["m"].mul_(MOMENTUM).add_(s["grad"])
    u = s["grad"] + MOMENTUM * s["m"]
    at = 0
    for (m, n), w in zip(s["shapes"], s["views"]["w"]):
        o = plain_newton_schulz(u[at:at + m * n].view(m, n))
        w.mul_(1.0 - LR * DECAY).sub_(LR * math.sqrt(max(1.0, m / n)) * o)
        at += m * n
    s["w16"].copy_(s["w"])
    s["grad"].zero_()
    return s["w"], s["m"], s["w16"]


# ------------------------------------------------------------------ what a pass cannot do without

def orth_flops(m, n):
    """The fewest products known to give the result: with A = X X^T on the shorter side
    (m), every step's factor and every later A are polynomials of A, all symmetric (half
    of a product each), and X is read twice: for A and for the last product."""
    m, n = min(m, n), max(m, n)
    by_gram = 2.0 * m * m * (1.5 * n + (2 * STEPS - 1.5) * m)
    by_step = 2.0 * m * m * STEPS * (1.5 * n + 0.5 * m)
    return min(by_gram, by_step)


def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "norm":
        blocks = case["n"] * case["gh"] * case["gw"]
        active = min(case["active"], blocks) or blocks
        elems = active * case["bh"] * case["bw"] * case["c"]
        return dict(bytes=elems * es * (3 if case["res"] else 2) + 8 * case["c"], flops=8.0 * elems)
    if case["kind"] == "grad":
        elems = case["n"] * case["h"] * case["w"] * case["c"]
        return dict(bytes=elems * es * (3 + bool(case["relu"]) + bool(case["res"])) + 12 * case["c"],
                    flops=16.0 * elems)
    if case["kind"] == "orth":
        return dict(bytes=2 * es * case["batch"] * case["rows"] * case["cols"],
                    flops=case["batch"] * orth_flops(case["rows"], case["cols"]))
    total = sum(m * n for m, n in shapes_of(case))
    # the new gradient's copy, then w, momentum, gradient read and written, the 16-bit copy
    return dict(bytes=total * (8 + 24 + 2), flops=sum(orth_flops(m, n) for m, n in shapes_of(case)))


# ------------------------------------------------------------------ in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": exact_norm, "grad": exact_grad, "orth": exact_orth, "step": exact_step}[case["kind"]](s)


def exact_stats(x):
    var, mean = torch.var_mean(x, dim=3, keepdim=True, correction=0)
    return mean, (var + NORM_EPS).rsqrt()


def exact_norm(s):
    c, x = s["case"], s["x"].double()
    mean, rstd = exact_stats(x)
    y = (x - mean) * rstd * s["gamma"].double() + s["beta"].double()
    if s["res"] is not None:
        y += s["res"].double()
    if c["relu"]:
        y = torch.where(y > 0, y, torch.zeros_like(y))
    if s["idx"] is None:
        return y
    grid = torch.zeros(c["n"] * c["gh"] * c["gw"], dtype=torch.bool, device=DEV)
    grid[s["idx"][:int(s["count"])].long()] = True
    grid = grid.view(c["n"], c["gh"], c["gw"]).repeat_interleave(c["bh"], 1).repeat_interleave(c["bw"], 2)
    return torch.where(grid[..., None], y, s["out"].double())


def exact_grad(s):
    x, dy, gamma = s["x"].double(), s["grad_out"].double(), s["gamma"].double()
    if s["y"] is not None:
        dy = torch.where(s["y"].double() > 0, dy, torch.zeros_like(dy))
    mean, rstd = exact_stats(x)
    c = x.shape[3]
    xhat = (x - mean) * rstd
    g = dy * gamma
    # y = xhat gamma + beta, xhat = (x - mean) rstd: the chain rule over both statistics
    sum_g, sum_gx = g.sum(3, keepdim=True), torch.linalg.vecdot(g, xhat, dim=3).unsqueeze(3)
    grad_in = (rstd / c) * (c * g - sum_g - xhat * sum_gx)
    dgamma = (xhat * dy).reshape(-1, c).sum(0)
    return grad_in, (dy if s["grad_res"] is not None else None), dgamma, dy.reshape(-1, c).sum(0)


def exact_newton_schulz(g):
    a, b, c = COEF
    g = g.double()
    x = g / (torch.linalg.norm(g) + ORTH_EPS)
    flip = x.shape[0] > x.shape[1]
    x = x.T.contiguous() if flip else x
    one = torch.eye(x.shape[0], dtype=torch.float64, device=x.device)
    for _ in range(STEPS):
        p = x @ x.T
        x = torch.linalg.multi_dot([a * one + (b * one + c * p) @ p, x])
    return x.T if flip else x


def exact_orth(s):
    return torch.stack([exact_newton_schulz(g) for g in s["g"]])


def exact_step(s):
    g = s["new_grad"].double()
    m = MOMENTUM * s["m"].double() + g
    u, w, at = g + MOMENTUM * m, s["w"].double(), 0
    for rows, cols in s["shapes"]:
        part = slice(at, at + rows * cols)
        o = exact_newton_schulz(u[part].view(rows, cols)).reshape(-1)
        w[part] -= LR * (DECAY * w[part] + math.sqrt(max(1.0, rows / cols)) * o)
        at += rows * cols
    return w, m, w
