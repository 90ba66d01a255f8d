"""Layer norm and its gradients through the C ABI, against the formulas in 64 bits.

Tolerances are bounds of rounding, element by element.  u = 2^-24.  A sum of n terms as the kernels take it (a few dozen in a register, then
a tree; long rows and columns one after the other in a thread) is off by at most depth * u of the sum of magnitudes, with depth
= 64 + n / 2048.  From there:
  xhat      (depth mean|x| + 2 |x|) rstd u of the difference, and (depth + 6) u |xhat| of rstd
  y         that times |weight|, and 2 u of the result
  dx        rstd times what q, its two means and xhat are off by
  dweight   depth u sum|dy xhat| and sum|dy| times what xhat is off by; dbias: depth u sum|dy|
and half a unit in the last place of the type that a result is rounded to (its smallest normal number's at least)."""
import ctypes as C

import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
EPS = 1e-5
HALF_ULP = {torch.float32: (2.0 ** -24, 2.0 ** -149), torch.bfloat16: (2.0 ** -8, 2.0 ** -133), torch.float16: (2.0 ** -11, 2.0 ** -24)}


@pytest.fixture(scope="module")
def rg():
    from paper_2509_05207_amd import binding
    binding.lib()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return binding


def rounding(ref, dtype):
    rel, least = HALF_ULP[dtype]
    return ref.abs() * rel + least


def made(rows, cols, dtype, weight, seed, pad=0, lead=0, shift=0.5, scale=1.0):
    """x, dy as views of rows of cols + pad elements that start `lead` elements into their buffer; weight, bias."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def rand(*size):
        return torch.randn(size, generator=g, device="cuda", dtype=torch.float64)

    def view(t):
        buf = torch.full((rows * (cols + pad) + lead + 8,), 7.0, dtype=dtype, device="cuda")
        v = buf[lead: lead + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
        v.copy_(t.to(dtype))
        return v
    x = view((rand(rows, cols) * torch.exp(0.5 * rand(rows, 1)) + shift) * scale)
    dy = view(rand(rows, cols) * torch.exp(0.5 * rand(rows, 1)))
    return x, dy, (1 + 0.3 * rand(cols)).to(weight), (0.2 * rand(cols)).to(weight)


def reference(x, dy, weight, bias, eps=EPS):
    """The formulas in 64 bits, and what rounding may change (see above)."""
    x, dy = x.double(), dy.double()
    rows, d = x.shape
    w = weight.double() if weight is not None else torch.ones(d, dtype=torch.float64, device=x.device)
    b = bias.double() if bias is not None else torch.zeros(d, dtype=torch.float64, device=x.device)
    row, col = 64 + d / 2048, 64 + rows / 2048
    mean = x.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + eps)
    h = (x - mean) * rstd
    dm = row * U * x.abs().mean(1, keepdim=True)
    dr = (row + 6) * U + 2 * dm * rstd                          # relative, of rstd
    dh = (dm + 2 * U * x.abs()) * rstd + dr * h.abs()
    y = h * w + b
    dyy = dh * w.abs() + 2 * U * (y.abs() + (h * w).abs())
    q = dy * w
    m0, m1 = q.mean(1, keepdim=True), (q * h).mean(1, keepdim=True)
    dx = rstd * (q - m0 - h * m1)
    aq = q.abs()
    off = 4 * U * aq + (row + 2) * U * aq.mean(1, keepdim=True) + dh * m1.abs()
    off = off + h.abs() * ((row + 4) * U * (aq * h.abs()).mean(1, keepdim=True) + (aq * dh).mean(1, keepdim=True)) + 4 * U * (m0.abs() + (h * m1).abs())
    ddx = rstd * off + (dr + 4 * U) * dx.abs()
    dw, db = (dy * h).sum(0), dy.sum(0)
    ddw = (col + 2) * U * (dy * h).abs().sum(0) + (dy.abs() * dh).sum(0)
    ddb = col * U * dy.abs().sum(0)
    return dict(y=(y, dyy), mean=(mean[:, 0], dm[:, 0]), rstd=(rstd[:, 0], (dr * rstd)[:, 0]), dx=(dx, ddx), dweight=(dw, ddw), dbias=(db, ddb))


def check(what, got, want):
    ref, tol = want
    tol = tol + rounding(ref.abs() + tol, got.dtype)
    off = (got.double() - ref).abs()
    bad = ~(off <= tol)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} beyond the bound, worst {float((off / tol).max()):.3g} times it"


def run_both(rg, x, dy, weight, bias, eps=EPS, **kw):
    y, mean, rstd = rg.rg_layer_norm(x, weight, bias, eps=eps)
    dx, dw, db = rg.rg_layer_norm_backward(dy, x, weight, mean, rstd, **kw)
    return dict(y=y, mean=mean, rstd=rstd, dx=dx, dweight=dw, dbias=db)


def compare(rg, x, dy, weight, bias, eps=EPS):
    want = reference(x, dy, weight, bias, eps)
    got = run_both(rg, x, dy, weight, bias, eps)
    for k in got:
        check(k, got[k], want[k])
    return got


WIDTHS = [1, 2, 3, 4, 5, 7, 8, 9, 31, 33, 64, 65, 100, 127, 128, 255, 256, 257, 511, 513, 602, 768, 1023, 1024, 1025, 2047, 2049, 4096, 4097, 8191, 8200, 12_289, 16_384, 16_385,
          32_768, 32_771, 70_001]


@pytest.mark.parametrize("cols", WIDTHS)
@pytest.mark.parametrize("dtype,weight", [(torch.float32, torch.float32), (torch.bfloat16, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.float16, torch.float16)])
def test_widths(rg, cols, dtype, weight):
    """Every kernel's rows: just full, one element more, one less."""
    compare(rg, *made(37, cols, dtype, weight, cols))


@pytest.mark.parametrize("rows", [1, 2, 5, 63, 64, 257, 1000, 40_003])
@pytest.mark.parametrize("cols", [24, 77, 602])
def test_heights(rg, rows, cols):
    compare(rg, *made(rows, cols, torch.float32, torch.float32, rows))


@pytest.mark.parametrize("cols", [3, 50, 77, 602, 1001, 5000, 40_001])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("pad,lead", [(0, 1), (3, 0), (6, 5), (1, 3)])
def test_padded_rows_at_every_phase(rg, cols, dtype, pad, lead):
    """Rows as a gather leaves them, and rows that begin at no multiple of an access; what lies between rows stays."""
    x, dy, w, b = made(19, cols, dtype, torch.float32, cols + pad, pad, lead)
    want = reference(x, dy, w, b)
    whole = torch.full((19, cols + pad), 3.0, dtype=dtype, device="cuda")
    y, mean, rstd = rg.rg_layer_norm(x, w, b, eps=EPS, out=whole[:, :cols])
    check("y", y, want["y"])
    assert bool((whole[:, cols:] == 3).all())
    whole2 = torch.full((19 * (cols + pad) + lead,), 3.0, dtype=dtype, device="cuda")
    rows2 = whole2[lead:].view(19, cols + pad)
    dx, dw, db = rg.rg_layer_norm_backward(dy, x, w, mean, rstd, out=rows2[:, :cols])
    for k, t in (("dx", dx), ("dweight", dw), ("dbias", db)):
        check(k, t, want[k])
    assert bool((rows2[:, cols:] == 3).all()) and bool((whole2[:lead] == 3).all())


@pytest.mark.parametrize("cols", [5, 64, 602, 3000, 20_000, 40_000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_in_place(rg, cols, dtype):
    x, dy, w, b = made(300, cols, dtype, torch.float32, 5)
    want = run_both(rg, x, dy, w, b)
    y = x.clone()
    _, mean, rstd = rg.rg_layer_norm(y, w, b, eps=EPS, out=y)
    g = dy.clone()
    dx, dw, db = rg.rg_layer_norm_backward(g, x, w, mean, rstd, out=g)
    for k, t in dict(y=y, mean=mean, rstd=rstd, dx=dx, dweight=dw, dbias=db).items():
        assert torch.equal(t, want[k]), k


@pytest.mark.parametrize("cols", [3, 77, 602, 5000, 40_000])
def test_parts_that_are_not_wanted(rg, cols):
    x, dy, w, b = made(100, cols, torch.float32, torch.float32, 6)
    both = run_both(rg, x, dy, w, b)
    data = run_both(rg, x, dy, w, b, want_dx=False)
    assert data["dx"] is None and torch.equal(data["dweight"], both["dweight"]) and torch.equal(data["dbias"], both["dbias"])
    only = run_both(rg, x, dy, w, b, want_dweight=False, want_dbias=False)
    assert only["dweight"] is None and only["dbias"] is None and torch.equal(only["dx"], both["dx"])
    one = run_both(rg, x, dy, w, b, want_dweight=False)
    assert one["dweight"] is None and torch.equal(one["dbias"], both["dbias"])


@pytest.mark.parametrize("cols", [3, 77, 5000, 40_000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_without_weight_or_bias(rg, cols, dtype):
    x, dy, w, b = made(50, cols, dtype, torch.float32, 8)
    for weight, bias in ((None, None), (w, None), (None, b)):
        want = reference(x, dy, weight, bias)
        for k, t in run_both(rg, x, dy, weight, bias).items():
            check(k, t, want[k])


@pytest.mark.parametrize("cols", [77, 1000, 5000, 40_000])
def test_large_means_and_sizes(rg, cols):
    """The squares are taken around the mean; rows of 1e18 and of 1e-15 do not leave fp32's range (beyond that the squares do, as in any fp32 program)."""
    compare(rg, *made(20, cols, torch.float32, torch.float32, 9, shift=1000.0))
    compare(rg, *made(20, cols, torch.float32, torch.float32, 9, scale=1e15))
    compare(rg, *made(20, cols, torch.float32, torch.float32, 9, scale=1e-10), eps=0.0)


def plain(x, dy, weight, eps=EPS):
    """dx by the formula's operations in 32 bits, each rounded."""
    x, dy, w, d = x.float(), dy.float(), weight.float(), x.shape[1]
    c = x - (x.sum(1, keepdim=True) / d)
    rstd = torch.rsqrt((c * c).sum(1, keepdim=True) / d + eps)
    q, h = dy * w, c * rstd
    return (rstd * (q - q.sum(1, keepdim=True) / d - h * ((q * h).sum(1, keepdim=True) / d)))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("cols", [1, 2])
def test_rows_of_which_nothing_is_left(rg, cols, dtype):
    """What dx is made of cancels: wholly in a row of one column, and to eps / variance in one of two, where nothing but the roundings is left.
    One is exactly zero, and the other as the rounded operations leave it, to the bit."""
    x, dy, weight, bias = made(3001, cols, dtype, torch.float32, 5)
    got = run_both(rg, x, dy, weight, bias)["dx"]
    assert torch.equal(got, plain(x, dy, weight).to(dtype))
    if cols == 1:
        assert not got.any()


def test_constant_rows(rg):
    x = torch.full((9, 300), 0.75, device="cuda")
    y, mean, rstd = rg.rg_layer_norm(x, None, None, eps=EPS)
    assert bool((y == 0).all()) and bool((mean == 0.75).all()) and torch.allclose(rstd, torch.full_like(rstd, EPS ** -0.5), rtol=4 * U)


@pytest.mark.parametrize("cols", [5, 77, 602, 5000, 40_000])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_infinities_and_nan_stay_in_their_row(rg, cols, bad):
    x, dy, w, b = made(23, cols, torch.float32, torch.float32, 10)
    want = run_both(rg, x, dy, w, b)
    x[11, cols // 2] = bad
    got = run_both(rg, x, dy, w, b)
    others = torch.arange(23, device="cuda") != 11
    for k in ("y", "dx"):
        assert torch.equal(got[k][others], want[k][others]) and bool(got[k][11].isnan().all()), k
    assert bool(got["dweight"].isnan().all()) and torch.equal(got["dbias"], want["dbias"])


@pytest.mark.parametrize("cols", [1, 6, 40, 300])
def test_gradients_against_differences(rg, cols):
    """Central differences of the formula in 64 bits, along random directions: <gradient, direction> is the slope of sum(y dy)."""
    x, dy, w, b = made(12, cols, torch.float32, torch.float32, 11)
    got = run_both(rg, x, dy, w, b, eps=0.1)
    g = torch.Generator(device="cuda").manual_seed(12)

    def loss(x, w, b):
        m = x.mean(1, keepdim=True)
        v = ((x - m) ** 2).mean(1, keepdim=True)
        return float((((x - m) / torch.sqrt(v + 0.1) * w + b) * dy.double()).sum())
    at = [t.double() for t in (x, w, b)]
    for i, k in enumerate(("dx", "dweight", "dbias")):
        for _ in range(4):
            way = torch.randn(at[i].shape, generator=g, device="cuda", dtype=torch.float64)
            step = 1e-5
            plus, minus = list(at), list(at)
            plus[i], minus[i] = at[i] + step * way, at[i] - step * way
            slope = (loss(*plus) - loss(*minus)) / (2 * step)
            got_slope = float((got[k].double() * way).sum())
            # differences: third derivatives times step^2 and 64-bit rounding over the step, below 1e-7 of the terms; the gradient itself: 1e-5 of them
            assert abs(slope - got_slope) <= 2e-5 * float((got[k].double() * way).abs().sum() + dy.double().abs().sum())


def test_no_rows(rg):
    for cols in (7, 602, 40_000):
        x, dy, w, b = made(0, cols, torch.float32, torch.float32, 13)
        got = run_both(rg, x, dy, w, b)
        assert got["y"].shape == (0, cols) and got["dx"].shape == (0, cols)
        assert bool((got["dweight"] == 0).all()) and bool((got["dbias"] == 0).all())


def test_broadcast_inputs(rg):
    """Rows that are one row (a stride of zero): what an expanded gradient is."""
    x, dy, w, b = made(40, 130, torch.float32, torch.float32, 14)
    compare(rg, x[:1].expand(40, 130), dy[:1].expand(40, 130), w, b)


def test_rows_beyond_four_gigabytes(rg):
    """Offsets that pass 32 bits: three rows of a buffer of 2^33 bytes and more."""
    stride = 2 ** 32 // 2 + 8                                              # elements of two bytes: 4 GiB and 16 bytes
    buf = torch.empty(2 * stride + 700, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(buf, (3, 602), (stride, 1))
    src, dy, w, b = made(3, 602, torch.bfloat16, torch.float32, 15)
    x.copy_(src)
    want = run_both(rg, src, dy, w, b)
    got = run_both(rg, x, dy, w, b)
    for k in got:
        assert torch.equal(got[k], want[k]), k
    y, mean, rstd = rg.rg_layer_norm(src, w, b, eps=EPS, out=x)
    assert torch.equal(y, want["y"])


@pytest.mark.parametrize("cols", [77, 602, 5000, 40_000])
def test_same_bits_every_time_and_on_another_stream(rg, cols):
    x, dy, w, b = made(3000 if cols < 5000 else 200, cols, torch.bfloat16, torch.float32, 16)
    want = run_both(rg, x, dy, w, b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for stream in (None, side, side.cuda_stream):
        y, mean, rstd = rg.rg_layer_norm(x, w, b, eps=EPS, stream=stream)
        dx, dw, db = rg.rg_layer_norm_backward(dy, x, w, mean, rstd, stream=stream)
        side.synchronize()
        for k, t in dict(y=y, mean=mean, rstd=rstd, dx=dx, dweight=dw, dbias=db).items():
            assert torch.equal(t, want[k]), k


def test_recorded_into_a_graph(rg):
    x, dy, w, b = made(500, 602, torch.float32, torch.float32, 17)
    ws = torch.empty(rg.rg_layer_norm_workspace(500, 602, torch.float32), dtype=torch.uint8, device="cuda")

    def step():
        y, mean, rstd = rg.rg_layer_norm(x, w, b, eps=EPS)
        return (y,) + tuple(rg.rg_layer_norm_backward(dy, x, w, mean, rstd, workspace=ws))
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for k in range(4):
        x.copy_(made(500, 602, torch.float32, torch.float32, 20 + k)[0])
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        for a, c in zip(got, step()):
            assert torch.equal(a, c)


def test_refusals(rg):
    L = rg.lib()
    x = torch.zeros((4, 64), device="cuda")
    y, w = torch.full_like(x, 5.0), torch.ones(64, device="cuda")
    st = torch.zeros((2, 4), device="cuda")
    f32, bf16 = rg.RG_F32, rg.RG_BF16

    def fwd(x=x.data_ptr(), xs=256, n=4, d=64, t=f32, w=w.data_ptr(), b=None, wt=f32, eps=1e-5, y=y.data_ptr(), ys=256, mean=st.data_ptr(), rstd=None):
        return L.rg_layer_norm(x, xs, n, d, t, w, b, wt, eps, y, ys, mean, rstd, None)
    big = torch.zeros(rg.rg_layer_norm_workspace(4, 64, torch.float32), dtype=torch.uint8, device="cuda")

    def bwd(dy=x.data_ptr(), gs=256, x=x.data_ptr(), xs=256, n=4, d=64, t=f32, w=w.data_ptr(), wt=f32, mean=st.data_ptr(), rstd=st.data_ptr(), dx=y.data_ptr(), dxs=256,
            dw=w.data_ptr(), db=None, ws=big.data_ptr(), wb=big.numel()):
        return L.rg_layer_norm_backward(dy, gs, x, xs, n, d, t, w, wt, mean, rstd, dx, dxs, dw, db, ws, wb, None)
    assert fwd() == rg.RG_OK and bwd() == rg.RG_OK
    torch.cuda.synchronize()
    y.fill_(5.0)
    for status, calls in ((rg.RG_EINVAL, [
            lambda: fwd(x=None), lambda: fwd(y=None), lambda: fwd(t=3), lambda: fwd(d=0), lambda: fwd(xs=255), lambda: fwd(ys=252), lambda: fwd(x=x.data_ptr() + 2),
            lambda: fwd(wt=bf16), lambda: fwd(wt=9), lambda: fwd(w=w.data_ptr() + 1), lambda: fwd(eps=-1.0), lambda: fwd(eps=float("nan")), lambda: fwd(eps=float("inf")),
            lambda: fwd(mean=st.data_ptr() + 2), lambda: bwd(dy=None), lambda: bwd(x=None), lambda: bwd(t=7), lambda: bwd(d=0), lambda: bwd(gs=6), lambda: bwd(mean=None),
            lambda: bwd(rstd=None), lambda: bwd(dxs=128), lambda: bwd(wt=bf16), lambda: bwd(ws=None), lambda: bwd(ws=big.data_ptr() + 4),
            lambda: L.rg_layer_norm_workspace(4, 64, 0, None), lambda: L.rg_layer_norm_workspace(4, 0, 0, C.byref(C.c_uint64()))]),
        (rg.RG_ERANGE, [lambda: fwd(d=2 ** 31), lambda: fwd(n=2 ** 40), lambda: fwd(xs=2 ** 41), lambda: bwd(d=2 ** 31), lambda: bwd(n=2 ** 40), lambda: bwd(wb=big.numel() - 1),
                        lambda: L.rg_layer_norm_workspace(2 ** 40, 64, 0, C.byref(C.c_uint64()))])):
        for k, call in enumerate(calls):
            assert call() == status and L.rg_last_error(), (status, k)
    torch.cuda.synchronize()
    assert bool((y == 5).all())
    for bad in (lambda: rg.rg_layer_norm(x.t()), lambda: rg.rg_layer_norm(x.cpu()), lambda: rg.rg_layer_norm(x, w[:32]), lambda: rg.rg_layer_norm(x.double()),
                lambda: rg.rg_layer_norm(x, out=torch.empty((4, 32), device="cuda")), lambda: rg.rg_layer_norm_backward(x[:2], x, w, st[0], st[1])):
        with pytest.raises((AssertionError, KeyError)):
            bad()


def test_in_place_with_another_stride_is_refused(rg):
    """Rows that are written where other rows are still to be read."""
    L = rg.lib()
    buf = torch.zeros(4 * 80, device="cuda")
    v = torch.ones((2, 4), device="cuda")
    p = buf.data_ptr()
    assert L.rg_layer_norm(p, 320, 4, 64, 0, None, None, 0, 1e-5, p, 256, v.data_ptr(), v.data_ptr(), None) == rg.RG_EINVAL
    assert L.rg_layer_norm_backward(p, 320, buf.data_ptr(), 320, 4, 64, 0, None, 0, v.data_ptr(), v.data_ptr(), p, 256, None, None, None, 0, None) == rg.RG_EINVAL
    assert L.rg_layer_norm(p, 320, 1, 64, 0, None, None, 0, 1e-5, p, 256, v.data_ptr(), v.data_ptr(), None) == rg.RG_OK       # a single row has no stride


@pytest.mark.parametrize("rows", [5, 100, 300])
@pytest.mark.parametrize("cols", [5, 64, 602, 3000, 20_000, 40_000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_dx_in_the_place_of_x(rg, rows, cols, dtype):
    """Few long rows are shared by workgroups, of which none may write what another still reads: neither of dy nor of x."""
    x, dy, w, b = made(rows, cols, dtype, torch.float32, 18)
    want = run_both(rg, x, dy, w, b)
    for which in (0, 1):
        at = [x.clone(), dy.clone()]
        dx, dw, db = rg.rg_layer_norm_backward(at[1], at[0], w, want["mean"], want["rstd"], out=at[which])
        assert dx is at[which]
        for k, t in dict(dx=dx, dweight=dw, dbias=db).items():
            assert torch.equal(t, want[k]), (k, which)


def test_dx_in_the_place_of_x_with_another_stride_is_refused(rg):
    buf, dy = torch.zeros(4 * 80, device="cuda"), torch.zeros((4, 64), device="cuda")
    st = torch.ones(4, device="cuda")
    wide, tight = torch.as_strided(buf, (4, 64), (80, 1)), torch.as_strided(buf, (4, 64), (64, 1))
    with pytest.raises(rg.RgError) as e:
        rg.rg_layer_norm_backward(dy, wide, None, st, st, out=tight)
    assert e.value.status == rg.RG_EINVAL


def test_more_columns_than_a_launch_has_work_items(rg):
    """Sums of 2^27 + 33 columns, 32 threads to a column: by a launch whose workgroups take several groups of them."""
    cols = 2 ** 27 + 33
    g = torch.Generator(device="cuda").manual_seed(19)
    x, dy = (torch.randn((1, cols), generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    mean, rstd = x.float().mean(1), torch.ones(1, device="cuda")
    _, dw, db = rg.rg_layer_norm_backward(dy, x, None, mean, rstd, want_dx=False)
    # one term to a sum: the difference rounded, and the product
    assert torch.equal(db, dy[0].float())
    want = dy[0].double() * (x[0].double() - mean.double())
    assert bool(((dw.double() - want).abs() <= 3 * U * (dy[0].double().abs() * (x[0].double().abs() + mean.double().abs()))).all())


@pytest.mark.parametrize("cols", [3, 602, 5000, 20_000, 40_000])
def test_means_whose_squares_are_beyond_the_range(rg, cols):
    """Only differences from the mean are squared: rows around 2^70 are in range as long as these are (eight units in the last place, 2^47 each; of bf16, whose units there are
    2^63, they are not)."""
    g = torch.Generator(device="cuda").manual_seed(20)
    x = (2.0 ** 70 + 2.0 ** 47 * torch.randint(0, 9, (7, cols), generator=g, device="cuda").double()).float()
    y, mean, rstd = rg.rg_layer_norm(x, eps=EPS)
    want = reference(x, x, None, None)
    check("y", y, want["y"])
    check("mean", mean, want["mean"])


@pytest.mark.parametrize("cols", [3, 602, 5000, 20_000, 40_000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_constant_rows_whose_squares_are_beyond_the_range(rg, cols, dtype):
    constant = torch.full((3, cols), 1e30, dtype=dtype, device="cuda")
    y, mean, rstd = rg.rg_layer_norm(constant, eps=EPS)
    assert bool(y.isfinite().all()) and bool(rstd.isfinite().all()) and bool((mean.double() / constant[:, 0].double() - 1).abs().max() <= (64 + cols / 2048) * U)


@pytest.mark.parametrize("cols", WIDTHS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_constant_rows_come_to_nothing(rg, cols, dtype):
    """A mean out of rounded sums is a few units of the last place off; their sum over the row is a whole number of them, and what it leaves is none."""
    x = torch.tensor([0.1, -12.7, 100.1, 1000.1, 30000.3, 1e-3], device="cuda").to(dtype)[:, None].expand(6, cols).contiguous()
    y, mean, rstd = rg.rg_layer_norm(x, eps=EPS)
    assert torch.equal(mean, x[:, 0].float())
    assert not y.any() and torch.allclose(rstd, torch.full_like(rstd, EPS ** -0.5), rtol=4 * U)


@pytest.mark.parametrize("cols", [40, 77, 602, 1000, 5000, 8192, 16_384, 20_000, 40_000, 70_001])
@pytest.mark.parametrize("shift", [100.0, 1e4, -1e4])
def test_rows_far_from_zero_keep_the_digits_of_their_deviations(rg, cols, shift):
    """x - mean is exact there, and the mean is corrected by what is left over: the bound of y (see above) with the deviation r = |x - mean| in the place of |x|.  The mean itself is rounded to fp32 at last."""
    x, _, w, b = made(20, cols, torch.float32, torch.float32, 21, shift=shift)
    y, mean, rstd = rg.rg_layer_norm(x, w, b, eps=EPS)
    xd, row = x.double(), 64 + cols / 2048
    m = xd.mean(1, keepdim=True)
    r = (xd - m).abs()
    s = 1 / torch.sqrt((r ** 2).mean(1, keepdim=True) + EPS)
    dm, dr = (row + 4) * U * r.mean(1, keepdim=True), (row + 6) * U
    dm = dm + (row * U) ** 2 * xd.abs().mean(1, keepdim=True)
    dr = dr + 2 * dm * s
    h = (xd - m) * s
    want = h * w.double() + b.double()
    tol = ((dm + 2 * U * r) * s + dr * h.abs()) * w.double().abs() + 2 * U * (want.abs() + (h * w.double()).abs())
    check("y", y, (want, tol))
    check("mean", mean, (m[:, 0], dm[:, 0]))
    check("rstd", rstd, (s[:, 0], (dr * s)[:, 0]))


def test_what_a_call_writes_is_known_to_autograd(rg):
    """Results in tensors of the caller's raise their version, so that a backward pass that had kept the old values refuses them."""
    x, dy, w, b = made(6, 20, torch.float32, torch.float32, 22)
    _, mean, rstd = rg.rg_layer_norm(x, w, b)
    for write in (lambda t: rg.rg_layer_norm(x, w, b, out=t), lambda t: rg.rg_layer_norm_backward(dy, x, w, mean, rstd, out=t)):
        t, v = torch.zeros((6, 20), device="cuda"), torch.ones((6, 20), device="cuda", requires_grad=True)
        before, product = t._version, t * v
        write(t)
        assert t._version == before + 1
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            product.sum().backward()
    versions = [t._version for t in (x, dy, w, b, mean, rstd)]
    run_both(rg, x, dy, w, b)
    assert versions == [t._version for t in (x, dy, w, b, mean, rstd)]
