"""Orthogonalised updates and the optimiser step through the C ABI, against the definition in 64 bits.

Tolerances, relative in the 2-norm.  The steps amplify what is off in the directions of small singular values by up to
3.4445^steps; what is rounded is known (rg_update.hip):
  fp32           operands of 22 bits, products accumulated in fp32 over n terms: u = 2^-22 on every operand, sqrt(n) 2^-24 on sums.  An
                 error in X of relative size u (of the largest singular value) is amplified 485 times in five steps at worst: 485 * 2^-22
                 = 1.2e-4 for matrices without rank; 1e-5 for those whose singular values lie within a factor of a hundred (a hundredth
                 grows 3.4^4 = 140 times to order one, where the sizes meet)
  16-bit types   the state is fp32, A and P and the copy of X in P X are rounded to 11 bits: every step P X is off by 3 u |P||X| in norm, u = 2^-12 and
                 random in sign, so that the last steps, where |P| <= 2.9, leave 2.9 * 1.7 * 2^-12 = 1.2e-3 a step, 4e-3 over all; and the result's own
                 rounding, 2^-9 / sqrt(3) (bf16) or 2^-12 / sqrt(3) (fp16)
"""
import ctypes as C
import math

import pytest
import torch

from update_cases import CUT_OTHERWISE, EVERY_TILE

pytestmark = pytest.mark.gpu
A, B, CC = 3.4445, -4.7750, 2.0315
BOUND = {torch.float32: 1e-5, torch.bfloat16: 5e-3, torch.float16: 4e-3}


@pytest.fixture(scope="module")
def rg():
    from paper_2509_05207_amd import binding
    binding.lib()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return binding


def definition(g, steps=5, eps=1e-7):
    x = g.double().cpu()
    tall = x.shape[0] > x.shape[1]
    x = x.t() if tall else x
    x = x / (x.norm() + eps)
    for _ in range(steps):
        s = x @ x.t()
        x = A * x + (B * s + CC * s @ s) @ x
    return (x.t() if tall else x).cuda()


def made(rows, cols, dtype, seed, kind="noise"):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def rand(*size):
        return torch.randn(size, generator=g, device="cuda", dtype=torch.float64)
    if kind == "noise":
        t = rand(rows, cols)
    elif kind == "sizes":               # rows of different sizes, as weights of different activations have
        t = rand(rows, cols) * torch.exp(rand(1, cols) * 0.7)
    elif kind == "low":                 # of rank 3 and little noise
        t = rand(rows, 3) @ rand(3, cols) + 0.02 * rand(rows, cols)
    return (0.01 * t).to(dtype)


def off(got, want):
    return float((got.double() - want).norm() / want.norm())


SHAPES = [(1, 1), (1, 7), (9, 1), (2, 3), (16, 16), (47, 256), (41, 512), (63, 65), (64, 64), (65, 63), (100, 47), (128, 129), (256, 602), (602, 256), (333, 1000), (1111, 130), (517, 515),
          (1, 5000), (5000, 2), (60, 9001)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype", list(BOUND))
@pytest.mark.parametrize("kind", ["noise", "sizes"])
def test_orthogonalize(rg, rows, cols, dtype, kind):
    g = made(rows, cols, dtype, rows * 7 + cols, kind)
    out, = rg.rg_orthogonalize([g])
    assert out.shape == g.shape and out.dtype == dtype
    assert off(out, definition(g)) <= BOUND[dtype]


@pytest.mark.parametrize("rows,cols", [(2048, 1030), (1500, 1500), (1025, 4000), (2047, 2177)])
@pytest.mark.parametrize("dtype", list(BOUND))
def test_large(rg, rows, cols, dtype):
    """Matrices that fill the chip with the larger tiles."""
    g = made(rows, cols, dtype, rows + cols, "sizes")
    assert off(rg.rg_orthogonalize([g])[0], definition(g)) <= BOUND[dtype]


@pytest.mark.parametrize("dtype", list(BOUND))
@pytest.mark.parametrize("rows,cols", [(64, 200), (300, 250), (1300, 1400)])
def test_little_rank(rg, dtype, rows, cols):
    """Singular values a thousand times apart."""
    g = made(rows, cols, dtype, 3, "low")
    assert off(rg.rg_orthogonalize([g])[0], definition(g)) <= (1.2e-4 if dtype == torch.float32 else BOUND[dtype])


@pytest.mark.parametrize("steps", [1, 2, 3, 7, 32])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_steps(rg, steps, dtype):
    """Singular values of one or less stay below 1.21 however many steps there are; beyond five they move about one another, and what is off with them."""
    g = made(90, 200, dtype, 4)
    s = 3.5 if steps > 5 else 1.0
    assert off(rg.rg_orthogonalize([g], steps=steps)[0], definition(g, steps)) <= BOUND[dtype] * s


def test_singular_values_come_to_about_one(rg):
    out, = rg.rg_orthogonalize([made(200, 300, torch.float32, 5)])
    s = torch.linalg.svdvals(out.double().cpu())
    assert float(s.min()) > 0.6 and float(s.max()) < 1.25


@pytest.mark.parametrize("dtype", list(BOUND))
def test_many_matrices_in_one_call(rg, dtype):
    """More than a launch takes, of both size classes, some without elements: each as it comes out alone, to the bit."""
    shapes = [(40 + 9 * k, 30 + 17 * k) for k in range(15)] + [(0, 5), (1400, 1500), (7, 0), (1600, 1300), (3, 3)]
    gs = [made(r, c, dtype, k) for k, (r, c) in enumerate(shapes)]
    outs = rg.rg_orthogonalize(gs)
    for g, o in zip(gs, outs):
        assert o.shape == g.shape
        if g.numel():
            assert torch.equal(o, rg.rg_orthogonalize([g])[0])
    assert rg.rg_orthogonalize([]) == []


@pytest.mark.parametrize("dtype", list(BOUND))
@pytest.mark.parametrize("rows,cols", [(300, 400), (900, 200), (30, 2500)])
def test_the_other_matrices_of_a_call_change_no_bit(rg, dtype, rows, cols):
    """A dozen of one size are cut into larger tiles than one alone."""
    gs = [made(rows, cols, dtype, k) for k in range(12)]
    for g, o in zip(gs, rg.rg_orthogonalize(gs)):
        assert torch.equal(o, rg.rg_orthogonalize([g])[0])
    assert off(o, definition(g)) <= BOUND[dtype]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("size", [1e-30, 1e-20, 1e-4, 1e10, 1e25, 3e36])
def test_sizes(rg, dtype, size):
    """The norm is summed in 64 bits: neither small nor large gradients leave the range (eps then decides how small is nothing)."""
    g = (made(70, 90, torch.float64, 6) * size).to(dtype)
    got, = rg.rg_orthogonalize([g], eps=0.0)
    assert off(got, definition(g, eps=0.0)) <= BOUND[dtype]
    got, = rg.rg_orthogonalize([g], eps=1e-7)
    want = definition(g, eps=1e-7)
    assert off(got, want) <= BOUND[dtype] + (0 if float(want.norm()) > 1e-20 else 1.0)


def test_zeros_and_what_is_no_number(rg):
    z = torch.zeros((50, 60), device="cuda")
    assert bool((rg.rg_orthogonalize([z])[0] == 0).all())
    assert bool(rg.rg_orthogonalize([z], eps=0.0)[0].isnan().all())             # 0 / 0
    for bad in (float("nan"), float("inf"), float("-inf")):
        for dtype in BOUND:
            a, b = made(50, 60, dtype, 7), made(70, 40, dtype, 8)
            want = rg.rg_orthogonalize([b])[0]
            a[17, 5] = bad
            x, y = rg.rg_orthogonalize([a, b])
            assert bool(x.isnan().all()) and torch.equal(y, want)              # and no other matrix


@pytest.mark.parametrize("dtype", list(BOUND))
def test_sparse_rows_and_columns(rg, dtype):
    """Matrices of one element, of empty rows and columns: entries of X up to one, where the products' scale has to hold."""
    g = torch.zeros((80, 100), dtype=dtype, device="cuda")
    g[3, 4] = 2.5
    assert off(rg.rg_orthogonalize([g])[0], definition(g)) <= BOUND[dtype]
    g = made(80, 100, dtype, 9)
    g[10:40] = 0
    g[:, 50:60] = 0
    got = rg.rg_orthogonalize([g])[0]
    assert off(got, definition(g)) <= BOUND[dtype]
    assert bool((got[10:40] == 0).all()) and bool((got[:, 50:60] == 0).all())


def step_definition(w, g, m, lr, wd, mu, nesterov, steps=5, eps=1e-7):
    m2 = mu * m.double() + g.double()
    o = definition(g.double() + mu * m2 if nesterov else m2, steps, eps)
    return w.double() * (1 - lr * wd) - lr * math.sqrt(max(1.0, w.shape[0] / w.shape[1])) * o, m2


@pytest.mark.parametrize("dtype", list(BOUND))
@pytest.mark.parametrize("nesterov", [False, True])
@pytest.mark.parametrize("rows,cols", [(47, 256), (300, 100), (1400, 1300)])
def test_muon_step(rg, dtype, nesterov, rows, cols):
    w, g = made(rows, cols, dtype, 10), made(rows, cols, dtype, 11, "sizes")
    m = made(rows, cols, torch.float32, 12) * 4
    want_w, want_m = step_definition(w, g, m, 0.03, 0.1, 0.9, nesterov)
    w2, m2 = torch.empty_like(w), torch.empty_like(m)
    before = [t.clone() for t in (w, g, m)]
    rg.rg_muon_step([w], [g], [m], lr=0.03, weight_decay=0.1, momentum=0.9, nesterov=nesterov, out_weights=[w2], out_momenta=[m2])
    assert all(torch.equal(a, b) for a, b in zip(before, (w, g, m)))
    assert off(m2, want_m) <= 2.0 ** -23
    change = want_w - w.double()
    rounding = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -9, torch.float16: 2.0 ** -12}[dtype] * float(want_w.norm())
    assert float((w2.double() - want_w).norm()) <= BOUND[dtype] * float(change.norm()) + rounding
    rg.rg_muon_step([w], [g], [m], lr=0.03, weight_decay=0.1, momentum=0.9, nesterov=nesterov)          # in place
    assert torch.equal(w, w2) and torch.equal(m, m2)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strides(rg, dtype):
    """Matrices inside larger ones, rows at any phase; what lies between rows stays."""
    for rows, cols in ((33, 70), (150, 61), (1300, 1301)):
        g = made(rows, cols, dtype, 13)
        buf = torch.full((rows, cols + 3), 2.0, dtype=dtype, device="cuda")
        buf[:, 1:cols + 1] = g
        whole = torch.full((rows, cols + 5), 3.0, dtype=dtype, device="cuda")
        rg.rg_orthogonalize([buf[:, 1:cols + 1]], out=[whole[:, 2:cols + 2]])
        assert torch.equal(whole[:, 2:cols + 2], rg.rg_orthogonalize([g])[0])
        assert bool((whole[:, :2] == 3).all()) and bool((whole[:, cols + 2:] == 3).all())
    g = made(1, 80, dtype, 14).expand(50, 80)                                   # one row fifty times
    assert off(rg.rg_orthogonalize([g])[0], definition(g)) <= (1.2e-4 if dtype == torch.float32 else BOUND[dtype])


def test_in_place_on_another_stream_and_again(rg):
    gs = [made(100, 130, torch.float32, 15), made(1400, 1400, torch.float32, 16)]
    want = rg.rg_orthogonalize(gs)
    for a, b in zip(want, rg.rg_orthogonalize(gs)):
        assert torch.equal(a, b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = rg.rg_orthogonalize(gs, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    rg.rg_orthogonalize(gs, out=gs)
    assert all(torch.equal(a, b) for a, b in zip(want, gs))


def test_recorded_into_a_graph(rg):
    w, g, m = [made(60, 90, torch.float32, 17)], [made(60, 90, torch.float32, 18)], [made(60, 90, torch.float32, 19)]
    w2, m2 = [torch.empty_like(w[0])], [torch.empty_like(m[0])]
    ws = torch.empty(rg.rg_update_workspace(g), dtype=torch.uint8, device="cuda")

    def step():
        rg.rg_muon_step(w, g, m, lr=0.1, out_weights=w2, out_momenta=m2, workspace=ws)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        g[0].copy_(made(60, 90, torch.float32, 30 + k))
        graph.replay()
        torch.cuda.synchronize()
        got = w2[0].clone(), m2[0].clone()
        step()
        assert torch.equal(got[0], w2[0]) and torch.equal(got[1], m2[0])


def test_refusals(rg):
    L = rg.lib()
    g = torch.zeros((8, 16), device="cuda")
    out = torch.full((8, 16), 5.0, device="cuda")
    ws = torch.empty(rg.rg_update_workspace([g]), dtype=torch.uint8, device="cuda")

    def update(**kw):
        u = (rg.rg_update * 1)()
        e = u[0]
        e.rows, e.cols = 8, 16
        e.grad = e.weight = e.momentum = g.data_ptr()
        e.momentum_out = e.out = out.data_ptr()
        for k in ("grad", "weight", "momentum", "momentum_out", "out"):
            setattr(e, k + "_stride", 64)
        for k, v in kw.items():
            setattr(e, k, v)
        return u

    def orth(u=None, n=1, t=0, steps=5, eps=1e-7, p=ws.data_ptr(), b=ws.numel(), **kw):
        return L.rg_orthogonalize(update(**kw) if u is None else u, n, t, steps, eps, p, b, None)

    def muon(lr=0.1, wd=0.0, mu=0.9, steps=5, eps=1e-7, p=ws.data_ptr(), b=ws.numel(), **kw):
        return L.rg_muon_step(update(**kw), 1, 0, lr, wd, mu, 1, steps, eps, p, b, None)
    size = C.c_uint64()
    nan, inf = float("nan"), float("inf")
    for status, calls in ((rg.RG_EINVAL, [
            lambda: orth(t=3), lambda: L.rg_orthogonalize(None, 1, 0, 5, 1e-7, ws.data_ptr(), ws.numel(), None), lambda: orth(steps=0), lambda: orth(steps=33), lambda: orth(eps=-1.0),
            lambda: orth(eps=nan), lambda: orth(eps=inf), lambda: orth(grad=None), lambda: orth(out=None), lambda: orth(grad=g.data_ptr() + 2), lambda: orth(grad_stride=66),
            lambda: orth(out_stride=60), lambda: orth(p=None), lambda: orth(p=ws.data_ptr() + 16), lambda: muon(weight=None), lambda: muon(momentum=None), lambda: muon(momentum_out=None),
            lambda: muon(momentum_stride=2), lambda: muon(momentum_out_stride=32), lambda: muon(lr=nan), lambda: muon(wd=inf), lambda: muon(mu=nan),
            lambda: L.rg_update_workspace(update(), 1, 0, None), lambda: L.rg_update_workspace(update(), 1, 5, C.byref(size))]),
        (rg.RG_ERANGE, [lambda: orth(b=ws.numel() - 1), lambda: orth(rows=32769), lambda: orth(cols=2 ** 31), lambda: orth(grad_stride=2 ** 41), lambda: muon(rows=40000),
                        lambda: L.rg_update_workspace(update(cols=40000), 1, 0, C.byref(size))])):
        for k, call in enumerate(calls):
            assert call() == status and L.rg_last_error(), (status, k)
    torch.cuda.synchronize()
    assert bool((out == 5).all())
    assert orth(rows=0, grad=None, p=None, b=0) == rg.RG_OK                     # nothing to do
    for bad in (lambda: rg.rg_orthogonalize([g.t()]), lambda: rg.rg_orthogonalize([g, g.bfloat16()]), lambda: rg.rg_orthogonalize([g], out=[out[:4]]), lambda: rg.rg_orthogonalize([g.double()]),
                lambda: rg.rg_orthogonalize([g.cpu()]), lambda: rg.rg_muon_step([g], [g], [g.half()], lr=0.1), lambda: rg.rg_muon_step([g], [g], [], lr=0.1)):
        with pytest.raises((AssertionError, KeyError)):
            bad()


def test_in_place_with_another_stride_is_refused(rg):
    """Rows that are written where other rows are still to be read."""
    buf = torch.zeros(64 * 80, device="cuda")
    wide, tight = torch.as_strided(buf, (64, 64), (80, 1)), torch.as_strided(buf, (64, 64), (64, 1))
    other = torch.zeros((64, 64), device="cuda")
    for call in (lambda: rg.rg_orthogonalize([wide], out=[tight]),
                 lambda: rg.rg_muon_step([wide], [other], [other.clone()], lr=0.1, out_weights=[tight]),
                 lambda: rg.rg_muon_step([other], [other.clone()], [wide], lr=0.1, out_momenta=[tight])):
        with pytest.raises(rg.RgError) as e:
            call()
        assert e.value.status == rg.RG_EINVAL


def structured(kind, rows, cols, dtype):
    """Matrices whose singular values are all alike, so that their roundings are too and do not average out; and noise."""
    if kind == "unit":
        t = torch.zeros((rows, cols), dtype=torch.float64, device="cuda")
        t.fill_diagonal_(1.0)
    elif kind == "orthonormal":
        g = torch.Generator().manual_seed(rows)
        t = torch.linalg.qr(torch.randn((max(rows, cols), min(rows, cols)), generator=g, dtype=torch.float64))[0]
        t = (t.t() if rows < cols else t).contiguous().cuda()
    else:
        return made(rows, cols, dtype, rows + 3 * cols, kind)
    return t.to(dtype)


@pytest.mark.parametrize("dtype", list(BOUND))
@pytest.mark.parametrize("kind,rows,cols", [("unit", 43, 300), ("unit", 400, 74), ("unit", 79, 260), ("unit", 300, 310), ("orthonormal", 48, 4096), ("orthonormal", 900, 500), ("orthonormal", 1400, 1500),
                                            ("noise", 33, 300), ("noise", 4000, 33), ("noise", 100, 4096), ("noise", 1300, 1400), ("low", 300, 250)])
def test_a_result_is_rounded_once(rg, kind, rows, cols, dtype):
    """Whatever the type, operands have 22 bits (the bounds of fp32 above), and a result is their type's number nearest to what they give.  Of an error e before it a rounding to a grid makes at most
    2 |e| + the distance of the exact result from the grid."""
    g = structured(kind, rows, cols, dtype)
    want = definition(g)
    assert off(rg.rg_orthogonalize([g])[0], want) <= 2 * (1.2e-4 if kind == "low" else 1e-5) + off(want.to(dtype), want)


@pytest.mark.parametrize("dtype", list(BOUND))
@pytest.mark.parametrize("rows,cols", [(43, 300), (1400, 1300)])
def test_muon_step_is_rounded_once(rg, dtype, rows, cols):
    """The same of the new weights: the update's error, lr times as large, and one rounding."""
    w, g, m = made(rows, cols, dtype, 20), structured("unit", rows, cols, dtype), torch.zeros((rows, cols), device="cuda")
    want, _ = step_definition(w, g, m, 0.5, 0.1, 0.9, True)
    before = float((want - w.double() * (1 - 0.5 * 0.1)).norm())
    rg.rg_muon_step([w], [g], [m], lr=0.5, weight_decay=0.1, momentum=0.9)
    # the sum's own rounding to fp32, two of them
    assert float((w.double() - want).norm()) <= 2 * (1e-5 * before + 2.0 ** -23 * float(want.norm())) + float((want.to(dtype).double() - want).norm())


def test_what_a_call_writes_is_known_to_autograd(rg):
    """Results in tensors of the caller's raise their version, and those of what they are detached from."""
    w, g, m, o = (made(8, 20, torch.float32, k) for k in range(4))
    w.requires_grad_()
    versions = lambda: [t._version for t in (w, g, m, o)]                                  # noqa: E731
    assert versions() == [0] * 4
    rg.rg_muon_step([w.detach()], [g], [m], lr=0.1)
    assert versions() == [1, 0, 1, 0]
    rg.rg_muon_step([w.detach()], [g], [m], lr=0.1, out_weights=[o], out_momenta=[m])
    assert versions() == [1, 0, 2, 1]
    rg.rg_orthogonalize([g], out=[g])
    rg.rg_orthogonalize([g])
    assert versions() == [1, 1, 2, 1]


def definition_there(g, steps=5, eps=1e-7):
    """The definition in 64 bits, where the CPU would take minutes."""
    x = g.double()
    tall = x.shape[0] > x.shape[1]
    x = x.t().contiguous() if tall else x
    x = x / (torch.linalg.vector_norm(x) + eps)
    for _ in range(steps):
        s = x @ x.t().contiguous()
        x = A * x + (B * s + CC * (s @ s)) @ x
    return x.t() if tall else x


# Of a square matrix' singular values one in a hundred lies below a hundredth of the largest: sqrt(1 / 100) of 1.2e-4 beside 1e-5 of the others.
SQUARE = 2.2e-5


@pytest.mark.parametrize("rows,cols", EVERY_TILE + [(16_384, 70), (30, 16_384), (16_384, 300)])
@pytest.mark.parametrize("dtype", list(BOUND))
def test_every_tile(rg, dtype, rows, cols):
    """The update and the optimiser step by every tile of either kind of product, none of which divides the sides; and the longest sides."""
    g = made(rows, cols, dtype, rows + 5, "sizes")
    want = definition_there(g)
    assert off(rg.rg_orthogonalize([g])[0], want) <= 2 * SQUARE + off(want.to(dtype), want)
    w, m = made(rows, cols, dtype, rows + 6), made(rows, cols, torch.float32, rows + 7) * 4
    want_m = 0.9 * m.double() + g.double()
    change = 0.5 * math.sqrt(max(1.0, rows / cols)) * definition_there(g.double() + 0.9 * want_m)
    want = w.double() * (1 - 0.5 * 0.1) - change
    rg.rg_muon_step([w], [g], [m], lr=0.5, weight_decay=0.1, momentum=0.9)
    # the sum's own rounding to fp32, two of them
    assert float((w.double() - want).norm()) <= 2 * (SQUARE * float(change.norm()) + 2.0 ** -23 * float(want.norm())) + float((want.to(dtype).double() - want).norm())
    assert off(m, want_m) <= 2.0 ** -23


@pytest.mark.parametrize("dtype", list(BOUND))
@pytest.mark.parametrize("rows,cols,copies", CUT_OTHERWISE)
def test_tiles_that_other_matrices_change_change_no_bit(rg, dtype, rows, cols, copies):
    """Tiles that no waves share, one size for a matrix alone and another for several."""
    gs = [made(rows, cols, dtype, k) for k in range(copies)]
    outs = rg.rg_orthogonalize(gs)
    for k in (0, copies - 1):
        assert torch.equal(outs[k], rg.rg_orthogonalize([gs[k]])[0])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_many_launches_recorded_into_a_graph(rg, dtype):
    """Matrices of several launches a step, of shared tiles and of others, in two groups."""
    shapes = [(300, 400), (1400, 1300), (60, 90), (1300, 40)]
    w, g = [made(r, c, dtype, 40 + r) for r, c in shapes], [made(r, c, dtype, 50 + r) for r, c in shapes]
    m = [made(r, c, torch.float32, 60 + r) for r, c in shapes]
    w2, m2 = [torch.empty_like(t) for t in w], [torch.empty_like(t) for t in m]
    ws = torch.empty(rg.rg_update_workspace(g), dtype=torch.uint8, device="cuda")

    def step():
        rg.rg_muon_step(w, g, m, lr=0.1, out_weights=w2, out_momenta=m2, workspace=ws)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        for t, (r, c) in zip(g, shapes):
            t.copy_(made(r, c, dtype, 70 + r + k))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in w2 + m2]
        for t in w2 + m2:
            t.fill_(7.0)
        step()
        assert all(torch.equal(a, b) for a, b in zip(got, w2 + m2))


def test_the_largest_matrix(rg):
    """RG_MAX_SIDE both ways: operands of 1 GiB, whose offsets are 32 bits."""
    g = torch.randn((16_384, 16_384), generator=torch.Generator(device="cuda").manual_seed(23), device="cuda").bfloat16()
    got, = rg.rg_orthogonalize([g], steps=2)
    want = definition_there(g, steps=2)
    assert off(got, want) <= 2 * SQUARE + off(want.to(g.dtype), want)


# fp32 matrices of few rows.  The polynomial in 64 bits: 1e-9 (singular values that come of nothing, 1e-16, grow 12 times a step); its product with U rounded to fp32, 2^-24.
NARROW = 2.0 ** -24 + 1e-9


@pytest.mark.parametrize("n", [1, 2, 3, 5, 15, 16, 17, 31, 32, 33, 36, 37, 47, 48])
@pytest.mark.parametrize("tall", [False, True])
def test_narrow_matrices_are_exact(rg, n, tall):
    """Every number of blocks, passes of columns, parts and shares, just full and one more or less; a result is its rounding alone off."""
    for m in (n, n + 1, 3 * n + 2, 64, 65, 100, 255, 256, 257, 1023, 1025, 2049, 9001, 16_384):
        if m < n or (n > 36 and m <= 1024):
            continue
        for kind in ("noise", "sizes", "low", "unit"):
            g = structured(kind, m if tall else n, n if tall else m, torch.float32)
            want = definition_there(g)
            assert off(rg.rg_orthogonalize([g])[0], want) <= 2 * NARROW + off(want.float(), want), (m, kind)


@pytest.mark.parametrize("n", [1, 2, 17, 36, 37, 48, 49, 64])
@pytest.mark.parametrize("dtype", list(BOUND))
@pytest.mark.parametrize("tall", [False, True])
def test_few_rows_of_every_type(rg, dtype, n, tall):
    """Either side of what is made in 64 bits, and of what is made in one launch."""
    for m in (n, 100, 255, 256, 257, 1024, 1025, 9001):
        if m < n:
            continue
        g = structured("sizes", m if tall else n, n if tall else m, dtype)
        want = definition_there(g)
        assert off(rg.rg_orthogonalize([g])[0], want) <= 2e-5 + off(want.to(dtype), want), m


@pytest.mark.parametrize("steps", [1, 2, 6, 7, 12, 13, 32])
@pytest.mark.parametrize("rows,cols", [(1, 9), (5, 400), (700, 30), (32, 256), (48, 1100), (20, 30)])
def test_steps_of_narrow_matrices(rg, rows, cols, steps):
    """Beyond six steps the state is rounded to fp32 between them: the bounds of fp32, as for other matrices."""
    g = made(rows, cols, torch.float32, 24)
    want = definition(g, steps)
    assert off(rg.rg_orthogonalize([g], steps=steps)[0], want) <= (2 * NARROW + 2.0 ** -24 if steps <= 6 else BOUND[torch.float32] * 3.5)


@pytest.mark.parametrize("steps", [5, 13, 32])
@pytest.mark.parametrize("rows,cols", [(30, 80), (48, 1300), (300, 7), (2, 300)])
def test_narrow_matrices_without_rank(rg, rows, cols, steps):
    """Rows that are multiples of one row, or empty: directions that the matrix lacks stay out of the result, whose singular values stay below 1.21 however many steps there are."""
    g = torch.zeros((rows, cols), device="cuda")
    g[: (rows + 1) // 2] = made(1, cols, torch.float32, 25) * torch.arange(1, (rows + 1) // 2 + 1, device="cuda")[:, None]
    got = rg.rg_orthogonalize([g], steps=steps)[0]
    assert bool(got.isfinite().all()) and float(torch.linalg.svdvals(got.double().cpu()).max()) <= 1.25
    assert not got[(rows + 1) // 2:].any()
    if steps == 5:
        assert off(got, definition(g)) <= 2 * NARROW + 2.0 ** -24


@pytest.mark.parametrize("dtype", list(BOUND))
@pytest.mark.parametrize("rows,cols", [(3, 5), (41, 512), (1000, 24), (32, 200), (1100, 48), (16, 16_384)])
@pytest.mark.parametrize("steps", [5, 8])
def test_optimiser_step_on_few_rows(rg, dtype, rows, cols, steps):
    """In other tensors, in place, in the gradient's place, and beside others: the same bits; what they are, by the definition of the update that fp32 gives."""
    w, g, m = made(rows, cols, dtype, 26), made(rows, cols, dtype, 27, "sizes"), made(rows, cols, torch.float32, 28) * 4
    options = dict(lr=0.5, weight_decay=0.1, momentum=0.9, steps=steps)
    w2, m2 = torch.empty_like(w), torch.empty_like(m)
    rg.rg_muon_step([w], [g], [m], out_weights=[w2], out_momenta=[m2], **options)
    want_m = 0.9 * m.double() + g.double()
    assert off(m2, want_m) <= 2.0 ** -23
    change = 0.5 * math.sqrt(max(1.0, rows / cols)) * definition_there(g.double() + 0.9 * want_m, steps)
    want = w.double() * (1 - 0.5 * 0.1) - change
    # the update (of which, in 64 bits or not, three roundings make what is orthogonalised); then the sum's roundings, two of them
    e = (3.5e-5 if steps > 6 else 1e-5) * float(change.norm()) + 2.0 ** -23 * float(want.norm())
    assert float((w2.double() - want).norm()) <= 2 * e + float((want.to(dtype).double() - want).norm())
    others = [made(r, c, dtype, 29) for r, c in ((500, 300), (7, 700), (20, 20))]
    w3, m3 = [w.clone()] + [t.clone() for t in others], [m.clone()] + [t.float() for t in others]
    rg.rg_muon_step(w3, [g] + others, m3, **options)
    assert torch.equal(w3[0], w2) and torch.equal(m3[0], m2)
    rg.rg_muon_step([w], [g], [m], out_weights=[g], **options)                  # the result where the gradient was
    assert torch.equal(g, w2) and torch.equal(m, m2)


@pytest.mark.parametrize("rows,cols", [(1, 1), (16, 70), (48, 3000), (9000, 32)])
def test_narrow_matrices_of_nothing_and_of_no_numbers(rg, rows, cols):
    z = torch.zeros((rows, cols), device="cuda")
    assert not rg.rg_orthogonalize([z])[0].any() and bool(rg.rg_orthogonalize([z], eps=0.0)[0].isnan().all())
    for steps in (1, 5, 9):
        for bad in (float("nan"), float("inf"), float("-inf")):
            g = made(rows, cols, torch.float32, 30)
            g[rows // 2, cols // 2] = bad
            assert bool(rg.rg_orthogonalize([g], steps=steps)[0].isnan().all())
    for size in (1e-38, 1e-44, 1e36):
        g = (made(rows, cols, torch.float64, 31) / 0.01 * size).float()
        if g.any():
            want = definition_there(g, eps=0.0)
            assert off(rg.rg_orthogonalize([g], eps=0.0)[0], want) <= 2 * NARROW + 2.0 ** -24
