"""Layer norm and its gradients against an evaluation in 64 bits.

Tolerances are first-order bounds, computed beside the reference (u = 2^-24 a rounding).  A sum over a row has a depth of 18 additions at most: 8 in a lane (two
sums of 8 values, then both; 12 where a row is a warp's and has 24 values a lane), 5 steps in a warp, 5 over warps.  The mean is then off by 20 u mean|x| (two more roundings for the division), the variance by 24 u of itself and what
the mean's error makes of it, rstd by half of that, 1 u for adding eps and 4 u for the reciprocal root.  Columns of dw and db are summed
over at most 300 roundings here: rows of a thread, groups of a block, then 64 bits.  Being bounds, they are wide for most values, so fp32
results also have to be within 8 u in the root mean square: an output carries about six roundings of half a step.  (From 8 columns on.  Errors of xhat and dx grow with rstd and
its square, and the variance of f normal values is below 1 / k^2 of the expected one with a probability of about k^-(f - 1): of 1000 rows of 3 columns one has
rstd 30 times as large, and its error, 900 times as large, alone makes the root mean square sqrt(900^2 / 1000) = 28 times that of the others; with 8
columns it would take 30^7 rows.)"""
import pytest

torch = pytest.importorskip("torch")

import paper_2104_03058_b200 as g  # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24
EPS = 1e-5


def rand(rows, cols, dtype=F32, ld=None, offset=0, seed=0, scale=1.0, mean=0.0):
    """[rows, cols] normal values with row pitch ld, `offset` elements behind an aligned address; what is around them is NaN."""
    ld = ld or cols
    gen = torch.Generator(device="cuda").manual_seed(seed + 5)
    buf = torch.full((rows * ld + offset + 8,), float("nan"), device="cuda", dtype=dtype)
    view = buf[offset:offset + rows * ld].view(rows, ld)[:, :cols]
    view.copy_(torch.randn((rows, cols), generator=gen, device="cuda") * scale + mean)
    return view


def reference(x, weight, bias, dout=None, eps=EPS):
    """{name: (value, bound)}"""
    n, f = x.shape
    x = x.double()
    w = torch.ones(f, device="cuda", dtype=torch.float64) if weight is None else weight.double()
    b = torch.zeros(f, device="cuda", dtype=torch.float64) if bias is None else bias.double()
    mean = x.mean(1, keepdim=True)
    off = x - mean
    var = (off ** 2).mean(1, keepdim=True)
    rstd = (var + eps) ** -0.5
    e_mean = 20 * U * x.abs().mean(1, keepdim=True)
    e_var = 24 * U * var + 2 * off.abs().mean(1, keepdim=True) * e_mean + e_mean ** 2
    e_r = 0.5 * e_var / (var + eps) + 5 * U
    xhat = off * rstd
    e_xhat = rstd * (e_mean + U * off.abs()) + xhat.abs() * (e_r + U)
    y = xhat * w + b
    res = {"out": (y, e_xhat * w.abs() + U * ((xhat * w).abs() + b.abs())), "mean": (mean[:, 0], e_mean[:, 0]),
           "rstd": (rstd[:, 0], (rstd * e_r)[:, 0])}
    if dout is None:
        return res
    do = dout.double()
    gw = do * w
    m1, m2 = gw.mean(1, keepdim=True), (gw * xhat).mean(1, keepdim=True)
    q1 = 22 * U * gw.abs().mean(1, keepdim=True)
    q2 = 23 * U * (gw * xhat).abs().mean(1, keepdim=True) + (gw.abs() * e_xhat).mean(1, keepdim=True)
    dx = rstd * (gw - m1 - xhat * m2)
    e_dx = rstd * (q1 + xhat.abs() * q2 + e_xhat * m2.abs() + 3 * U * (gw.abs() + m1.abs() + (xhat * m2).abs())) + dx.abs() * (e_r + U)
    chain = (min(n, 300) + 2) * U
    res["dx"] = (dx, e_dx)
    res["dw"] = ((do * xhat).sum(0), (do.abs() * e_xhat).sum(0) + chain * (do * xhat).abs().sum(0))
    res["db"] = (do.sum(0), chain * do.abs().sum(0))
    return res


def check(got, ref, what, rms=True):
    want, bound = ref
    half = torch.finfo(got.dtype).eps / 2
    tol = 1.25 * bound + half * want.abs() + 1e-37
    err = (got.double() - want).abs()
    assert got.shape == want.shape and (err <= tol).all(), "%s: %d of %d off, worst %.3g of its bound" % (
        what, int((~(err <= tol)).sum()), err.numel(), float((err / tol).nan_to_num(1e9).max()))
    if rms and got.dtype == F32 and got.numel() > 1000:
        assert float(err.pow(2).mean().sqrt()) <= 8 * U * float(want.pow(2).mean().sqrt()), what


def both_ways(x, weight, bias, dout, odt=F32, offset=0, rms=True):
    n, f = x.shape
    rms = rms and f >= 8
    guard = torch.full((n * (f + 3) + offset,), 7.0, device="cuda", dtype=odt)
    buf = guard[offset:].view(n, f + 3)
    out, mean, rstd = g.layer_norm(x, weight, bias, EPS, out=buf[:, :f], with_stats=True)
    ref = reference(x, weight, bias, dout)
    assert (buf[:, f:] == 7.0).all() and (guard[:offset] == 7.0).all()
    check(out, ref["out"], "out", rms)
    check(mean, ref["mean"], "mean", False)
    check(rstd, ref["rstd"], "rstd", False)
    check(g.layer_norm(x, weight, bias, EPS, out_dtype=odt), ref["out"], "out, aligned", rms)
    buf.fill_(7.0)
    dx, dw, db = g.layer_norm_backward(dout, x, mean, rstd, weight, out=buf[:, :f])
    assert (buf[:, f:] == 7.0).all() and (guard[:offset] == 7.0).all()
    check(dx, ref["dx"], "dx", rms)
    check(dw, ref["dw"], "dw", False)
    check(db, ref["db"], "db", False)
    again = g.layer_norm_backward(dout, x, mean, rstd, weight, out_dtype=odt, with_params=False)
    assert again[1] is None and again[2] is None
    check(again[0], ref["dx"], "dx, aligned", rms)
    return out, dx, dw, db


@pytest.mark.parametrize("odt", [F32, BF16])
@pytest.mark.parametrize("xdt", [F32, BF16])
@pytest.mark.parametrize("n,f,ld,offset", [
    (1, 1, 1, 0), (3, 2, 2, 0), (1000, 3, 3, 1), (777, 8, 8, 0), (513, 16, 24, 0), (130, 41, 41, 0), (1001, 64, 64, 0), (257, 100, 104, 4), (99, 128, 128, 2),
    (700, 250, 252, 0), (65, 256, 256, 1), (300, 256, 256, 0), (37, 602, 608, 0), (40, 602, 602, 0), (33, 1000, 1000, 0), (21, 1023, 1023, 0), (9, 2048, 2056, 0),
    (7, 2049, 2052, 0), (5, 4100, 4104, 0), (3, 8191, 8191, 0), (2, 8192, 8192, 0), (1, 8190, 8192, 0)])
def test_sizes_and_layouts(xdt, odt, n, f, ld, offset):
    x, dout = rand(n, f, xdt, ld, offset, 1, 2.0, 0.5), rand(n, f, xdt, ld, offset, 2)
    weight, bias = rand(1, f, seed=3, scale=0.3, mean=1.0)[0].clone(), rand(1, f, seed=4)[0].clone()
    both_ways(x, weight, bias, dout, odt, offset)


@pytest.mark.parametrize("weight,bias", [(False, False), (True, False), (False, True)])
def test_without_weight_or_bias(weight, bias):
    x, dout = rand(200, 96, seed=1), rand(200, 96, seed=2)
    both_ways(x, rand(1, 96, seed=3)[0].clone() if weight else None, rand(1, 96, seed=4)[0].clone() if bias else None, dout)


@pytest.mark.parametrize("n,f", [(20_011, 128), (6_007, 602), (100_003, 16), (1_500, 4096)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_more_rows_than_the_blocks_take_at_once(dtype, n, f):
    x, dout = rand(n, f, dtype, seed=1, scale=3.0), rand(n, f, dtype, seed=2)
    both_ways(x, rand(1, f, seed=3, mean=1.0)[0].clone(), rand(1, f, seed=4)[0].clone(), dout, dtype)


def test_values_far_from_zero():
    """The mean is a thousand times the spread: what the bound allows for that is far less than a sum of squares around zero would lose."""
    both_ways(rand(300, 256, seed=1, mean=1000.0), None, None, rand(300, 256, seed=2), rms=False)


def test_constant_rows_and_single_columns_give_the_bias():
    bias = rand(1, 64, seed=1)[0].clone()
    for value in (0.0, 1.0, -1024.0, 3e18):
        assert torch.equal(g.layer_norm(torch.full((5, 64), value, device="cuda"), None, bias), bias.expand(5, 64))
    assert torch.equal(g.layer_norm(rand(9, 1, seed=2).contiguous(), None, bias[:1].clone()), bias[:1].expand(9, 1))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("f", [8, 41, 256, 2048])
def test_bad_values_stay_in_their_row(f, bad, dtype):
    x, dout = rand(70, f, dtype, seed=1), rand(70, f, dtype, seed=2)
    clean, mean, rstd = g.layer_norm(x, with_stats=True)
    dclean = g.layer_norm_backward(dout, x, mean, rstd)[0]
    x[33, f // 2] = bad
    got, mean, rstd = g.layer_norm(x, with_stats=True)
    dgot = g.layer_norm_backward(dout, x, mean, rstd)[0]
    others = torch.arange(70, device="cuda") != 33
    assert torch.equal(got[others], clean[others]) and torch.equal(dgot[others], dclean[others])
    assert torch.isnan(got[33]).all() and torch.isnan(dgot[33]).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_in_place(dtype):
    for f in (40, 602, 3000):
        x, dout = rand(90, f, dtype, seed=1), rand(90, f, dtype, seed=2)
        want, mean, rstd = g.layer_norm(x, out_dtype=dtype, with_stats=True)
        dwant = g.layer_norm_backward(dout, x, mean, rstd, out_dtype=dtype)
        y = x.clone()
        assert g.layer_norm(y, out=y) is y and torch.equal(y, want)
        dgot = g.layer_norm_backward(dout, x, mean, rstd, out=dout)
        assert dgot[0] is dout and all(torch.equal(a, b) for a, b in zip(dgot, dwant))


def test_no_rows():
    x = torch.zeros((0, 24), device="cuda")
    out, mean, rstd = g.layer_norm(x, with_stats=True)
    assert out.shape == (0, 24) and mean.shape == rstd.shape == (0,)
    dx, dw, db = g.layer_norm_backward(x, x, mean, rstd)
    assert dx.shape == (0, 24) and (dw == 0).all() and (db == 0).all()


def test_a_row_does_not_depend_on_its_batch():
    for f in (24, 256, 1500):
        x = rand(1000, f, seed=1)
        whole = g.layer_norm(x)
        for rows in (slice(0, 1), slice(999, 1000), slice(100, 350)):
            assert torch.equal(g.layer_norm(x[rows]), whole[rows])


def test_gradients_agree_with_differences():
    """Central differences in 64 bits of the definition, at the points and along the directions that the call's gradients are then multiplied with: for a step of
    2^-12 of values of size 1 the cut-off error is below 2^-20 of the third derivative; 1e-4 of the sum of magnitudes covers it and the call's roundings."""
    x, dout, v = (rand(40, 48, seed=i).contiguous() for i in (1, 2, 3))
    w, b, vw, vb = (rand(1, 48, seed=i)[0].clone() for i in (4, 5, 6, 7))
    _, mean, rstd = g.layer_norm(x, w, b, with_stats=True)
    dx, dw, db = g.layer_norm_backward(dout, x, mean, rstd, w)

    def value(step):
        xs, ws, bs = x.double() + step * v.double(), w.double() + step * vw.double(), b.double() + step * vb.double()
        off = xs - xs.mean(1, keepdim=True)
        return ((off / ((off ** 2).mean(1, keepdim=True) + EPS).sqrt() * ws + bs) * dout.double()).sum()

    h = 2.0 ** -12
    terms = torch.cat([(t.double() * d.double()).flatten() for t, d in ((dx, v), (dw, vw), (db, vb))])
    assert abs(float((value(h) - value(-h)) / (2 * h) - terms.sum())) <= 1e-4 * float(terms.abs().sum())


def test_captured_and_replayed_and_on_another_stream():
    x, dout = rand(3000, 96, seed=1), rand(3000, 96, seed=2)
    w = rand(1, 96, seed=3)[0].clone()

    def both():
        y, mean, rstd = g.layer_norm(x, w, with_stats=True)
        return (y, *g.layer_norm_backward(dout, x, mean, rstd, w))

    want = [t.clone() for t in both()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y, mean, rstd = g.layer_norm(x, w, with_stats=True, stream=side)
    got = (y, *g.layer_norm_backward(dout, x, mean, rstd, w, stream=side))
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for seed in (11, 12):
        x.copy_(rand(3000, 96, seed=seed))
        want = [t.clone() for t in both()]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_refusals():
    x, m = rand(6, 8, seed=1), torch.zeros(6, device="cuda")
    for call, match in ((lambda: g.layer_norm(x, torch.ones(7, device="cuda")), "weight"), (lambda: g.layer_norm(x, bias=torch.ones(8)), "bias"),
                        (lambda: g.layer_norm(x, out=x[1:]), "rows"), (lambda: g.layer_norm(x.t()), "x must be"),
                        (lambda: g.layer_norm(x[:, :4], out=x[:, 2:6]), "overlap"), (lambda: g.layer_norm(x, f=9), "x must be"),
                        (lambda: g.layer_norm_backward(x[:5].clone(), x, m, m), "dout"), (lambda: g.layer_norm_backward(x.clone(), x, m[:5], m), "mean"),
                        (lambda: g.layer_norm_backward(x.clone(), x, m, m.double()), "rstd"), (lambda: g.layer_norm_backward(x.clone(), x, m, m, out=x), "overlap")):
        with pytest.raises(ValueError, match=match):
            call()
    with pytest.raises(TypeError):
        g.layer_norm_backward(x.to(BF16), x, m, m)
    with pytest.raises(TypeError):
        g.layer_norm(x.double())
    with pytest.raises(g.GnnfdError):
        g.layer_norm(torch.zeros((2, 8200), device="cuda"))
    with pytest.raises(g.GnnfdError):
        g.layer_norm(x, eps=-1.0)
    with pytest.raises(g.GnnfdError):
        g.layer_norm_backward(x.clone(), x, m, m, scratch=torch.zeros(16, device="cuda"))
