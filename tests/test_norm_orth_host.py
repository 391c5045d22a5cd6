"""Argument checks of the layer normalisation and the orthogonalised updates, before anything
is enqueued: no GPU, fake device addresses (see test_abi_host.py)."""
import ctypes
import os
import shutil
import subprocess
import sys

import pytest
import torch

no_gpu = pytest.mark.skipif(torch.cuda.is_available(),
                            reason="fake device pointers are used only on machines without a GPU")
pytestmark = no_gpu

A, B_, C, D, E, F, W = (0x10000000 * k for k in range(1, 8))
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def B():
    from paper_2108_09376_amd import bc
    return bc


def test_layer_norm_refusals(B):
    lib = B.raw()

    def call(x=A, d=(1, 64, 16, 32, 1, 1), gamma=B_, beta=C, res=None, eps=1e-5, relu=0, out=D, grid=(8, 16),
             idx=E, cnt=F, cap=128):
        return lib.bc_sparse_layer_norm(x, B.bc_tensor(*d), gamma, beta, res, eps, relu, out, B.bc_grid(*grid), idx,
                                        cnt, cap, None)

    assert call(x=None) == call(out=None) == call(idx=None) == B.BC_ERR_NULL
    for bad in (dict(d=(1, 0, 16, 32, 1, 1)), dict(d=(-1, 64, 16, 32, 1, 1)), dict(relu=2), dict(eps=-1.0),
                dict(eps=NAN), dict(eps=INF), dict(grid=(0, 16)), dict(d=(4000, 4000, 16, 32, 1, 1))):
        assert call(**bad) == B.BC_ERR_SHAPE, bad
    assert call(d=(1, 64, 16, 32, 5, 1)) == B.BC_ERR_DTYPE
    assert call(d=(1, 64, 16, 32, 0, 0)) == call(d=(1, 64, 16, 32, 1, 7)) == B.BC_ERR_LAYOUT
    assert call(grid=(5, 16)) == B.BC_ERR_NOT_DIVISIBLE
    assert call(cap=127) == B.BC_ERR_CAPACITY
    nb = 64 * 16 * 32 * 2
    for bad in (dict(out=A + 2), dict(out=A - nb + 2), dict(res=D + 16), dict(gamma=D + 8), dict(beta=D + nb - 4),
                dict(idx=D), dict(cnt=D + 64)):
        assert call(**bad) == B.BC_ERR_ALIAS, bad


def test_layer_norm_grad_refusals(B):
    lib = B.raw()
    d = B.bc_tensor(1, 64, 16, 32, 1, 1)
    n = ctypes.c_int64()
    assert lib.bc_layer_norm_grad_work(d, None) == B.BC_ERR_NULL
    assert lib.bc_layer_norm_grad_work(B.bc_tensor(1, 64, 16, 32, 1, 0), ctypes.byref(n)) == B.BC_ERR_LAYOUT
    assert lib.bc_layer_norm_grad_work(B.bc_tensor(1, 64, 0, 32, 1, 1), ctypes.byref(n)) == B.BC_ERR_SHAPE
    assert lib.bc_layer_norm_grad_work(d, ctypes.byref(n)) == B.BC_OK and n.value > 0
    need = n.value

    def call(x=A, d=d, gamma=None, y=None, dy=B_, eps=1e-5, dx=C, dres=None, dg=D, db=E, acc=0, work=W, size=need):
        return lib.bc_layer_norm_grad(x, d, gamma, y, dy, eps, dx, dres, dg, db, acc, work, size, None)

    assert call(x=None) == call(dy=None) == call(dx=None) == call(work=None) == B.BC_ERR_NULL
    assert call(acc=2) == call(eps=-1.0) == B.BC_ERR_SHAPE
    assert call(d=B.bc_tensor(1, 64, 16, 32, 9, 1)) == B.BC_ERR_DTYPE
    assert call(d=B.bc_tensor(1, 64, 16, 32, 0, 0)) == B.BC_ERR_LAYOUT
    assert call(size=need - 1) == call(size=-1) == B.BC_ERR_CAPACITY
    assert call(work=W + 4) == B.BC_ERR_UNSUPPORTED
    for bad in (dict(dx=A + 2), dict(dx=B_ + 2), dict(y=C), dict(dres=A), dict(dres=C), dict(gamma=C + 64), dict(dg=A),
                dict(db=D + 4), dict(dg=W), dict(dx=W), dict(work=A), dict(dx=B_, dres=B_)):
        assert call(**bad) == B.BC_ERR_ALIAS, bad


def test_orthogonalize_refusals(B):
    lib = B.raw()
    n = ctypes.c_int64()
    for args in ((0, 64, 64, 5), (1, 0, 64, 5), (1, 64, -1, 5), (1, 64, 64, 0), (1, 64, 64, 65), (1, 20000, 20000, 5),
                 (1, 1 << 30, 8, 5), (1 << 25, 1, 1, 5), (2000, 2000, 2000, 5)):
        assert lib.bc_orthogonalize_work(*args, ctypes.byref(n)) == B.BC_ERR_SHAPE, args
    assert lib.bc_orthogonalize_work(1, 64, 64, 5, None) == B.BC_ERR_NULL
    assert lib.bc_orthogonalize_work(2, 64, 100, 5, ctypes.byref(n)) == B.BC_OK
    need = n.value
    good = (5, 3.4445, -4.7750, 2.0315, 1e-7)

    def call(g=A, dt=0, size=(2, 64, 100), ns=good, out=B_, odt=0, work=W, nb=need):
        return lib.bc_orthogonalize(g, dt, *size, None if ns is None else ctypes.byref(B.bc_newton_schulz(*ns)), out,
                                    odt, work, nb, None)

    assert call(g=None) == call(out=None) == call(work=None) == call(ns=None) == B.BC_ERR_NULL
    assert call(size=(0, 64, 100)) == call(ns=(0,) + good[1:]) == B.BC_ERR_SHAPE
    assert call(ns=good[:4] + (-1.0,)) == call(ns=good[:4] + (NAN,)) == B.BC_ERR_SHAPE
    assert call(dt=4) == call(odt=-1) == B.BC_ERR_DTYPE
    # not positive, not finite, growing without bound, past the entries' range in one step
    for c in ((0.0, -1.0, 1.0), (-1.0, 0.0, 0.0), (NAN, 0.0, 0.0), (1.0, INF, 0.0), (3.0, 0.0, 0.0), (3.0, 8.0, 8.0)):
        assert call(ns=(5, *c, 1e-7)) == B.BC_ERR_UNSUPPORTED, c
    assert call(nb=need - 1) == B.BC_ERR_CAPACITY
    assert call(work=W + 8) == B.BC_ERR_UNSUPPORTED
    for bad in (dict(out=A + 4), dict(out=A, odt=1), dict(work=A), dict(out=W + 256)):
        assert call(**bad) == B.BC_ERR_ALIAS, bad


def test_tiles_of_a_call(B):
    """As many matrices as the header promises, and not one more."""
    n = ctypes.c_int64()
    for most, rows, cols in ((2 ** 22 - 1, 1, 1), (2 ** 22 - 1, 30, 31), (127, 1, 2 ** 22), (127, 2 ** 22, 5)):
        assert B.raw().bc_orthogonalize_work(most, rows, cols, 5, ctypes.byref(n)) == B.BC_OK and n.value > 0
        assert B.raw().bc_orthogonalize_work(most + 1, rows, cols, 5, ctypes.byref(n)) == B.BC_ERR_SHAPE
    params = (B.bc_matrix * 64)()
    for p in params:
        p.rows, p.cols = 2 ** 22, 200                      # 2^18 tiles each
    assert B.raw().bc_muon_step_many_work(params, 63, 5, ctypes.byref(n)) == B.BC_OK and n.value > 0
    assert B.raw().bc_muon_step_many_work(params, 64, 5, ctypes.byref(n)) == B.BC_ERR_SHAPE


def test_coefficients_of_late_spans(B):
    """Steps 5 and 6 (from 0) are one span. With these coefficients a singular value of 1 stays
    near 1 until step 5 and grows by 2.73 and 6.31 there: their product, 17.2, is beyond the 16
    bits that the span's factor is held in. Fewer steps stay within, in any span."""
    def call(steps, c):
        return B.raw().bc_orthogonalize(A, 0, 1, 500, 1000, ctypes.byref(B.bc_newton_schulz(steps, *c, 0.0)), B_, 0, W,
                                        0, None)

    for c in ((0.45704228, -0.49950711, 1.04263144), (0.45456629, -0.77823198, -0.67638974)):
        assert call(7, c) == B.BC_ERR_UNSUPPORTED, c
        for steps in range(1, 7):                          # the check behind theirs: no workspace
            assert call(steps, c) == B.BC_ERR_CAPACITY, (steps, c)
    for steps in range(1, 65):
        assert call(steps, (3.4445, -4.7750, 2.0315)) == call(steps, (1.5, -0.5, 0.0)) == B.BC_ERR_CAPACITY


def test_muon_refusals(B):
    lib = B.raw()
    ns = (5, 3.4445, -4.7750, 2.0315, 1e-7)
    n = ctypes.c_int64()
    good = [(A, B_, C, D, 64, 288), (A + (1 << 20), B_ + (1 << 20), C + (1 << 20), None, 128, 64)]

    def params(rows):
        arr = (B.bc_matrix * len(rows))()
        for a, r in zip(arr, rows):
            a.w, a.momentum, a.grad, a.w16, a.rows, a.cols = r
        return arr

    assert lib.bc_muon_step_many_work(params(good), 2, 5, ctypes.byref(n)) == B.BC_OK
    need = n.value
    assert lib.bc_muon_step_many_work(None, 2, 5, ctypes.byref(n)) == B.BC_ERR_NULL
    assert lib.bc_muon_step_many_work(params(good), 2, 5, None) == B.BC_ERR_NULL
    assert lib.bc_muon_step_many_work(params(good), 0, 5, ctypes.byref(n)) == B.BC_ERR_SHAPE
    assert lib.bc_muon_step_many_work(params(good * 33), 65, 5, ctypes.byref(n)) == B.BC_ERR_SHAPE

    def call(rows=good, lr=0.02, mu=0.95, wd=0.0, nesterov=1, ns=ns, dt=1, work=W, nb=need):
        h = B.bc_muon(lr, mu, wd, nesterov, B.bc_newton_schulz(*ns))
        return lib.bc_muon_step_many(params(rows), len(rows), ctypes.byref(h), dt, work, nb, None)

    assert lib.bc_muon_step_many(params(good), 2, None, 1, W, need, None) == B.BC_ERR_NULL
    for k in range(3):
        r = list(good[0])
        r[k] = None
        assert call(rows=[tuple(r), good[1]]) == B.BC_ERR_NULL
    assert call(work=None) == B.BC_ERR_NULL
    assert call(rows=[good[0][:4] + (0, 288)]) == call(lr=NAN) == call(mu=INF) == call(wd=NAN) == B.BC_ERR_SHAPE
    assert call(nesterov=2) == call(ns=(65,) + ns[1:]) == B.BC_ERR_SHAPE
    assert call(dt=0) == B.BC_ERR_DTYPE
    assert call(ns=(5, 3.0, 0.0, 0.0, 1e-7)) == B.BC_ERR_UNSUPPORTED
    assert call(nb=need - 1) == B.BC_ERR_CAPACITY
    for k, v in ((0, B_ + 4), (2, A + 64), (3, A), (3, W), (1, good[1][0])):
        r = list(good[0])
        r[k] = v
        assert call(rows=[tuple(r), good[1]]) == B.BC_ERR_ALIAS, (k, v)


def test_binding_refuses_mismatched_tensors(B):
    x = torch.zeros((1, 4, 4, 16), dtype=torch.bfloat16)
    v, bad = torch.zeros(16), torch.zeros(15)
    out = torch.empty_like(x)
    for args in ((x, B.BC_NHWC, bad, v, None, 1e-5, 0, out), (x, B.BC_NHWC, v, v.bfloat16(), None, 1e-5, 0, out),
                 (x, B.BC_NHWC, v, v, x[:, :2], 1e-5, 0, out), (x, B.BC_NHWC, v, v, None, 1e-5, 0, out.float()),
                 (x.transpose(1, 2), B.BC_NHWC, v, v, None, 1e-5, 0, out)):
        with pytest.raises(ValueError):
            B.bc_sparse_layer_norm(*args, (1, 1), None, None)
    with pytest.raises(ValueError):
        B.bc_layer_norm_grad(x, B.BC_NHWC, v, None, x.float(), 1e-5, out, None, v, v)
    with pytest.raises(ValueError):
        B.bc_layer_norm_grad(x, B.BC_NHWC, v, None, x, 1e-5, out, None, bad, v)
    g = torch.zeros(8, 16)
    with pytest.raises(ValueError):
        B.bc_orthogonalize(g, torch.zeros(16, 8))
    with pytest.raises(ValueError):
        B.bc_orthogonalize(g.T, torch.zeros(16, 8))
    with pytest.raises(ValueError):
        B.bc_muon_step_many([(g, g.clone(), g[:4].clone(), None)], 0.1, 0.9, 0.0)
    with pytest.raises(ValueError):
        B.bc_muon_step_many([(g, g.clone(), g.double(), None)], 0.1, 0.9, 0.0)


def test_workspace_of_fewer_bytes_than_elements(B):
    """A view's elements are not its memory: one element expanded to as many as are needed."""
    x, v, g = torch.zeros((1, 4, 4, 16)), torch.zeros(16), torch.zeros(8, 16)
    params = [(g, g.clone(), g.clone(), None)]
    for work in (torch.zeros(1, dtype=torch.uint8).expand(1 << 20), torch.zeros(2 << 20, dtype=torch.uint8)[::2]):
        with pytest.raises(ValueError):
            B.bc_layer_norm_grad(x, B.BC_NHWC, v, None, x, 1e-5, torch.empty_like(x), None, v, v, work=work)
        with pytest.raises(ValueError):
            B.bc_orthogonalize(g, torch.empty_like(g), work=work)
        with pytest.raises(ValueError):
            B.bc_muon_step_many(params, 0.1, 0.9, 0.0, work=work)


@pytest.mark.parametrize("shape", [(), (0, 16), (4, 0), (0,)])
def test_weights_without_elements(B, shape):
    w = torch.zeros(shape)
    with pytest.raises(ValueError):
        B.bc_muon_step_many([(w, w.clone(), w.clone(), None)], 0.1, 0.9, 0.0)
    with pytest.raises(ValueError):
        B.bc_muon_step_many_work([(w, w.clone(), w.clone(), None)])


def test_copies_of_two_dtypes(B):
    """All 16-bit copies of a step are written in one format: two are refused, in any order."""
    def param(dt):
        w = torch.zeros(8, 16)
        return w, torch.zeros_like(w), torch.zeros_like(w), None if dt is None else torch.zeros(8, 16, dtype=dt)

    bf16, f16, f32 = torch.bfloat16, torch.float16, torch.float32
    for dts in ((bf16, f16), (f16, None, bf16), (f32, bf16), (bf16, bf16, f16, bf16)):
        params = [param(d) for d in dts]
        with pytest.raises(ValueError):
            B.bc_muon_step_many(params, 0.1, 0.9, 0.0)
        with pytest.raises(ValueError):
            B.bc_muon_step_many_work(params)
        with pytest.raises(ValueError):
            B.bc_rmsprop_step_many(params, 0.1, 0.9, 1e-8, 0.0)
    assert B.bc_muon_step_many_work([param(f16), param(None), param(f16)]) > 0


NO_MEMORY = """
#include <cstdlib>
#include <new>
static thread_local bool none;
extern "C" void no_memory(int on) { none = on; }
void *operator new(std::size_t n)
{
    void *p = none ? nullptr : std::malloc(n ? n : 1);
    if (!p) throw std::bad_alloc();
    return p;
}
void operator delete(void *p) noexcept { std::free(p); }
void operator delete(void *p, std::size_t) noexcept { std::free(p); }
"""

CALLS = """
import ctypes
from paper_2108_09376_amd import bc as B
none = ctypes.CDLL(None).no_memory
lib, n = B.raw(), ctypes.c_int64()
ns = B.bc_newton_schulz(64, 1.5, -0.5, 0.0, 1e-7)
h = B.bc_muon(0.1, 0.9, 0.0, 1, ns)
params = (B.bc_matrix * 64)()
for i, p in enumerate(params):
    p.w, p.momentum, p.grad, p.w16 = (0x10000000 * (4 * i + k + 1) for k in range(4))
    p.rows, p.cols = 500 + i, 1000
params[63].grad = params[0].w
for on in (0, 1):                              # without first: the error text has its room then
    none(on)
    got = (lib.bc_orthogonalize_work(3, 1000, 2000, 64, ctypes.byref(n)),
           lib.bc_muon_step_many_work(params, 64, 64, ctypes.byref(n)),
           lib.bc_muon_step_many(params, 64, ctypes.byref(h), 1, 0x7000000000, n.value, None),
           lib.bc_orthogonalize(params[0].w, 0, 3, 1000, 2000, ctypes.byref(ns), params[1].w, 0, None, 0, None))
    none(0)
    assert got == (B.BC_OK, B.BC_OK, B.BC_ERR_ALIAS, B.BC_ERR_NULL), got
"""


def test_no_exception_without_memory(B, tmp_path):
    """The orthogonalising calls allocate nothing on the host: with an operator new that throws
    they check, plan and answer as ever."""
    cxx = shutil.which("g++")
    if not cxx:
        pytest.skip("g++ not found")
    src, lib = tmp_path / "no_memory.cpp", tmp_path / "no_memory.so"
    src.write_text(NO_MEMORY)
    subprocess.check_call([cxx, "-O1", "-shared", "-fPIC", "-o", str(lib), str(src)])
    env = dict(os.environ, LD_PRELOAD=" ".join(filter(None, [str(lib), os.environ.get("LD_PRELOAD")])))
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", CALLS], env=env, cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, (r.returncode, r.stderr[-2000:])


def test_policy_norm_refusal(B):
    from paper_2108_09376_amd import resnet
    with pytest.raises(ValueError):
        resnet.PolicyNet(256, 512, norm="batch", device="cpu")
