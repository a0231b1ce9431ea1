"""Group norm with an activation and its gradients against an evaluation in 64 bits.

Tolerances are first-order bounds, computed beside the reference (u = 2^-24 a rounding, R the largest distance of a value from its mean).  Distances are
counted from the mean of some of the values, so none is above 2 R, and a thread adds up at most 128 rows of them here (pieces of graphs this size are
shorter): the mean is off by at most u |mean| + 128 u 2 R and what per_group / 16 + 42 more additions add; a sum of k <= 128 squares by
(k + 3) u of itself, that is the variance by 135 u 4 R^2, twice that with the square of the sum, and as much again in merging.  Being
bounds, they are wide for most values, so fp32 results also have to be within 16 u in the root mean square: an output carries
about ten roundings, half a step each at most, and the statistics' errors average out over thousands of terms."""
import math

import pytest

torch = pytest.importorskip("torch")

import paper_2104_03058_b200 as g  # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24
EPS = 1e-5


def rand(rows, cols, dtype=F32, ld=None, offset=0, seed=0, scale=1.0, mean=0.0):
    ld = ld or cols
    gen = torch.Generator(device="cuda").manual_seed(seed + 41)
    buf = torch.full((rows * ld + offset + 8,), float("nan"), device="cuda", dtype=dtype)
    view = buf[offset:offset + rows * ld].view(rows, ld)[:, :cols]
    view.copy_(torch.randn((rows, cols), generator=gen, device="cuda") * scale + mean)
    return view


def act_and_slope(z, act):
    """value, slope, bounds of the errors of both beside that of z, whose share is the slope's (at most 1.13) and its slope's (at most 1)"""
    u = U * torch.ones_like(z)
    if act == "relu":
        return z.clamp_min(0), (z > 0).double(), 0 * u, 0 * u
    if act == "elu":
        return torch.where(z > 0, z, torch.expm1(z)), torch.where(z > 0, 1.0, torch.exp(z)), 4 * u, 8 * u
    sig = torch.sigmoid(z)
    if act == "silu":
        return z * sig, sig * (1 + z * (1 - sig)), (8 + 3 * z.abs()) * U * (z * sig).abs(), (16 + 6 * z.abs()) * u
    if act == "gelu":
        cdf = 0.5 * (1 + torch.erf(z / math.sqrt(2)))
        return z * cdf, cdf + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi), 6 * U * z.abs() + U, (16 + 6 * z.abs()) * u
    return z, torch.ones_like(z), 0 * u, 0 * u


def reference(x, groups, weight, bias, ptr, act, eps, dout=None):
    """{name: (value, bound)} of the rows that belong to a graph"""
    n, f = x.shape
    per = f // groups
    ptr = torch.tensor([0, n], device="cuda") if ptr is None else ptr.long()
    graphs = ptr.numel() - 1
    size = ptr[1:] - ptr[:-1]
    used = int(ptr[-1])
    row = torch.repeat_interleave(torch.arange(graphs, device="cuda"), size)
    xs = x[:used].double().reshape(used, groups, per)
    w = (torch.ones(f, device="cuda") if weight is None else weight).double().reshape(groups, per)
    b = (torch.zeros(f, device="cuda") if bias is None else bias).double().reshape(groups, per)
    total = lambda t: torch.zeros((graphs, groups), dtype=torch.float64, device="cuda").index_add_(0, row, t.sum(2))      # noqa: E731
    count = (size.double() * per).clamp_min(1)[:, None]
    mean = total(xs) / count
    off = xs - mean[row][:, :, None]
    var = total(off ** 2) / count
    top = torch.zeros((graphs, groups), dtype=torch.float64, device="cuda").scatter_reduce_(
        0, row[:, None].expand(used, groups), off.abs().amax(2), "amax")
    rstd = (var + eps) ** -0.5
    e_mean = U * mean.abs() + (160 + per / 16 + 10) * U * 2 * top
    e_var = 2 * 135 * U * 4 * top ** 2 * 2 + 4 * U * var
    e_r = 0.5 * e_var / (var + eps) + 2 * U
    rr, er = rstd[row][:, :, None], e_r[row][:, :, None]
    xhat = off * rr
    e_xhat = rr * (e_mean[row][:, :, None] + U * off.abs()) + xhat.abs() * (er + 2 * U)
    z = xhat * w + b
    e_z = e_xhat * w.abs() + 2 * U * ((xhat * w).abs() + b.abs())
    y, sl, e_act, e_sl = act_and_slope(z, act)
    res = {"out": (y.reshape(used, f), (1.13 * e_z + e_act).reshape(used, f)),
           "mean": (mean, e_mean), "rstd": (rstd, rstd * e_r)}
    if dout is None:
        return res
    do = dout[:used].double().reshape(used, groups, per)
    gg = do * sl
    e_sl = e_sl + e_z
    if act == "relu":
        e_sl = torch.where(z.abs() <= e_z, 1.0, 0.0)                      # the side of 0 is not known
    e_g = do.abs() * e_sl + 2 * U * gg.abs()
    gw, e_gw = gg * w, e_g * w.abs() + U * (gg * w).abs()
    e_gwx = e_gw * xhat.abs() + gw.abs() * e_xhat
    chain = 140 * U
    m1, m2 = total(gw) / count, total(gw * xhat) / count
    e_m1 = (total(e_gw) + (chain + per / 16 * U) * total(gw.abs())) / count + U * m1.abs()
    e_m2 = (total(e_gwx) + (chain + per / 16 * U) * total((gw * xhat).abs())) / count + U * m2.abs()
    p1, p2, q1, q2 = (t[row][:, :, None] for t in (m1, m2, e_m1, e_m2))
    dx = rr * (gw - p1 - xhat * p2)
    e_dx = rr * (e_gw + q1 + e_xhat * p2.abs() + xhat.abs() * q2 + 4 * U * (gw.abs() + p1.abs() + (xhat * p2).abs())) + dx.abs() * er
    res["dx"] = (dx.reshape(used, f), e_dx.reshape(used, f))
    res["dw"] = ((gg * xhat).sum(0).reshape(f), ((e_g * xhat.abs() + gg.abs() * e_xhat).sum(0) + chain * (gg * xhat).abs().sum(0)).reshape(f))
    res["db"] = (gg.sum(0).reshape(f), (e_g.sum(0) + chain * gg.abs().sum(0)).reshape(f))
    return res


def check(got, ref, what, rms=False):
    want, bound = ref
    half = torch.finfo(got.dtype).eps / 2
    tol = 1.25 * bound + half * want.abs() + 1e-37
    err = (got.double() - want).abs()
    assert (err <= tol).all(), "%s: %d of %d off, worst %.3g of its bound" % (what, int((~(err <= tol)).sum()), err.numel(),
                                                                             float((err / tol).nan_to_num(1e9).max()))
    if rms and got.dtype == F32 and got.numel() > 1000:
        assert float(err.pow(2).mean().sqrt()) <= 16 * U * float(want.pow(2).mean().sqrt()), what


def both_ways(x, groups, weight, bias, ptr, act, dout, eps=EPS, out_dtype=F32, rms=True):
    n, f = x.shape
    buf = torch.full((n, f + 3), 7.0, device="cuda", dtype=out_dtype)
    out, mean, rstd = g.group_norm(x, groups, weight, bias, ptr, eps, act, out=buf[:, :f], with_stats=True)
    ref = reference(x, groups, weight, bias, ptr, act, eps, dout)
    used = ref["out"][0].shape[0]
    assert (buf[:, f:] == 7.0).all() and (buf[used:] == 7.0).all()
    check(out[:used], ref["out"], "out", rms)
    check(mean, ref["mean"], "mean")
    check(rstd, ref["rstd"], "rstd")
    plain = g.group_norm(x, groups, weight, bias, ptr, eps, act, out_dtype=out_dtype)
    check(plain[:used], ref["out"], "out, aligned", rms)
    buf = torch.full((n, f + 3), 7.0, device="cuda", dtype=out_dtype)
    dx, dw, db = g.group_norm_backward(dout, x, groups, mean, rstd, weight, bias, ptr, act, out=buf[:, :f])
    assert (buf[:, f:] == 7.0).all() and (buf[used:] == 7.0).all()
    check(dx[:used], ref["dx"], "dx", rms and act != "relu")
    check(dw, ref["dw"], "dw")
    check(db, ref["db"], "db")
    again = g.group_norm_backward(dout, x, groups, mean, rstd, weight, bias, ptr, act, out_dtype=out_dtype, with_params=False)
    assert again[1] is None and again[2] is None
    check(again[0][:used], ref["dx"], "dx, aligned", rms and act != "relu")
    return out, dx, dw, db


def offsets(n, graphs, seed=0, itype=torch.int32, last=None):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    last = n if last is None else last
    cuts = torch.randint(last + 1, (graphs - 1,), generator=gen, device="cuda").sort().values
    return torch.cat([cuts.new_zeros(1), cuts, cuts.new_full((1,), last)]).to(itype)


@pytest.mark.parametrize("act", ["none", "relu", "elu", "silu", "gelu"])
@pytest.mark.parametrize("xdt,odt", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
def test_activations_and_types(act, xdt, odt):
    x, dout = rand(1500, 48, xdt, scale=2.0, mean=1.0), rand(1500, 48, xdt, seed=1)
    both_ways(x, 6, rand(1, 48, seed=2)[0].contiguous(), rand(1, 48, seed=3)[0].contiguous(), offsets(1500, 20), act, dout, out_dtype=odt)


@pytest.mark.parametrize("xdt", [F32, BF16])
@pytest.mark.parametrize("n,f,groups,ld,offset", [(1, 1, 1, 1, 0), (1, 8, 2, 8, 0), (63, 5, 5, 5, 0), (64, 41, 41, 44, 0), (65, 602, 7, 608, 0),
                                                  (4097, 602, 1, 602, 0), (3000, 602, 602, 608, 8), (777, 12, 4, 13, 1), (5000, 3, 1, 3, 0),
                                                  (300, 1500, 25, 1504, 0), (40, 8192, 2, 8192, 0), (200, 1100, 10, 1101, 3), (20_000, 16, 4, 16, 0)])
def test_one_graph(xdt, n, f, groups, ld, offset):
    x, dout = rand(n, f, xdt, ld, offset, scale=2.0, mean=-1.0), rand(n, f, xdt, ld, offset, seed=1)
    both_ways(x, groups, rand(1, f, seed=2)[0].contiguous(), rand(1, f, seed=3)[0].contiguous(), None, "silu", dout, rms=n * f // groups > 500)


@pytest.mark.parametrize("itype", [torch.int32, torch.int64])
@pytest.mark.parametrize("n,graphs,f,groups,last", [(100, 7, 16, 4, None), (5000, 4000, 24, 2, None), (5000, 40, 24, 24, 4500), (10_000, 3, 64, 8, None),
                                                    (64, 200, 8, 1, 30), (30_000, 1000, 128, 8, 29_999), (900, 1, 20, 5, 0), (2000, 500, 602, 14, None),
                                                    (3000, 150, 1100, 1, None)])
def test_batches_of_graphs(itype, n, graphs, f, groups, last):
    x, dout = rand(n, f, scale=3.0), rand(n, f, seed=1)
    ptr = offsets(n, graphs, itype=itype, last=last)
    both_ways(x, groups, None, rand(1, f, seed=3)[0].contiguous(), ptr, "gelu", dout, rms=False)
    both_ways(x.bfloat16(), groups, rand(1, f, seed=2)[0].contiguous(), None, ptr, "none", dout.bfloat16(), out_dtype=BF16, rms=False)


@pytest.mark.parametrize("n,empties", [(900, 40), (900, 5000), (70_000, 3000), (400_000, 5000)])
def test_long_graphs_between_many_empty_ones(n, empties):
    third = n // 3
    ptr = torch.cat([torch.full((empties,), at, device="cuda") for at in (0, third, third + 1, 2 * third)] + [torch.full((3,), n, device="cuda")]).int()
    x, dout = rand(n, 12, scale=2.0), rand(n, 12, seed=1)
    both_ways(x, 3, None, None, ptr, "elu", dout, rms=False)


def test_values_far_from_zero_and_an_outlier_in_the_first_row():
    x = rand(3000, 32, scale=1.0, mean=1000.0)
    both_ways(x, 4, None, None, offsets(3000, 3), "none", rand(3000, 32, seed=1), rms=False)
    out = g.group_norm(x, 4, eps=0.0)
    want = reference(x, 4, None, None, None, "none", 0.0)["out"][0]
    assert float((out.double() - want).pow(2).mean().sqrt()) <= 2 * 1000 * U            # the mean itself is rounded: 1000 u of a deviation
    x = rand(5000, 16)
    x[0] = 1e4                                                                          # where distances are counted from
    out = g.group_norm(x, 2)
    want = reference(x, 2, None, None, None, "none", EPS)["out"][0]
    assert float((out.double() - want).abs().max()) <= 70 * 8 * U * float(want.abs().max())


def test_constant_and_single_values_give_the_bias():
    bias = rand(1, 12, seed=3)[0].contiguous()
    for x in (torch.full((500, 12), 3.7, device="cuda"), rand(1, 12)):
        assert torch.equal(g.group_norm(x, 12, None, bias), bias.expand_as(x))
    assert torch.equal(g.group_norm(torch.full((500, 12), -2.3, device="cuda"), 3, None, bias), bias.expand(500, 12))


def test_not_a_number_stays_in_its_graph_and_group():
    x, ptr = rand(300, 8), torch.tensor([0, 100, 180, 300], device="cuda")
    clean = g.group_norm(x, 2, graph_ptr=ptr)
    x[120, 1] = float("nan")
    x[250, 6] = float("inf")
    got = g.group_norm(x, 2, graph_ptr=ptr)
    assert torch.isnan(got[100:180, :4]).all() and torch.isnan(got[180:, 4:]).all()
    assert torch.equal(got[:100], clean[:100]) and torch.equal(got[100:180, 4:], clean[100:180, 4:]) and torch.equal(got[180:, :4], clean[180:, :4])


def test_no_rows_and_only_empty_graphs():
    out, mean, rstd = g.group_norm(torch.empty((0, 6), device="cuda"), 3, graph_ptr=torch.zeros(4, dtype=torch.int32, device="cuda"), with_stats=True)
    assert out.shape == (0, 6) and (mean == 0).all() and torch.allclose(rstd, torch.full_like(rstd, EPS ** -0.5), rtol=4 * U)
    dx, dw, db = g.group_norm_backward(out, out, 3, mean, rstd, graph_ptr=torch.zeros(4, dtype=torch.int32, device="cuda"))
    assert dx.shape == (0, 6) and (dw == 0).all() and (db == 0).all()
    x = rand(70, 6)
    kept = torch.full_like(x, 5.0)
    out, mean, rstd = g.group_norm(x, 3, graph_ptr=torch.zeros(4, dtype=torch.int32, device="cuda"), out=kept, with_stats=True)
    assert (kept == 5.0).all() and (mean == 0).all()


def test_offsets_that_make_no_sense_touch_nothing_outside():
    x = rand(200, 8)
    buf = torch.full((400, 8), 9.0, device="cuda")
    for ptr in ([-5, 90, 400], [0, 150, 60, 200], [300, 100, -1], [2 ** 40, 0, 2 ** 50]):
        out, mean, rstd = g.group_norm(x, 2, graph_ptr=torch.tensor(ptr, device="cuda"), out=buf[100:300], with_stats=True)
        g.group_norm_backward(x.contiguous(), x, 2, mean, rstd, graph_ptr=torch.tensor(ptr, device="cuda"), out=buf[100:300])
        torch.cuda.synchronize()
        assert (buf[:100] == 9.0).all() and (buf[300:] == 9.0).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_in_place(dtype):
    x, dout, ptr = rand(2500, 40, dtype), rand(2500, 40, dtype, seed=1), offsets(2500, 30)
    apart, mean, rstd = g.group_norm(x, 8, graph_ptr=ptr, activation="elu", out_dtype=dtype, with_stats=True)
    dx = g.group_norm_backward(dout, x, 8, mean, rstd, graph_ptr=ptr, activation="elu", out_dtype=dtype)[0]
    gone = dout.clone()
    g.group_norm_backward(gone, x, 8, mean, rstd, graph_ptr=ptr, activation="elu", out=gone)
    mine = x.clone()
    assert g.group_norm(mine, 8, graph_ptr=ptr, activation="elu", out=mine) is mine
    assert torch.equal(mine, apart) and torch.equal(gone, dx)


def test_gradients_agree_with_differences():
    x, ptr = rand(40, 12), torch.tensor([0, 13, 13, 40], device="cuda")
    w, b, dout = rand(1, 12, seed=2)[0].contiguous(), rand(1, 12, seed=3)[0].contiguous(), rand(40, 12, seed=4)
    _, mean, rstd = g.group_norm(x, 3, w, b, ptr, EPS, "gelu", with_stats=True)
    grads = g.group_norm_backward(dout, x, 3, mean, rstd, w, b, ptr, "gelu")
    ref = reference(x, 3, w, b, ptr, "gelu", EPS, dout)
    loss = lambda x, w, b: float((reference(x, 3, w, b, ptr, "gelu", EPS)["out"][0] * dout.double()).sum())      # noqa: E731
    args = [x.double(), w.double(), b.double()]
    for i, name in enumerate(("dx", "dw", "db")):
        step = torch.randn(args[i].shape, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda", dtype=torch.float64)
        sides = []
        for sign in (1e-5, -1e-5):
            moved = list(args)
            moved[i] = args[i] + sign * step
            sides.append(loss(*moved))
        bound = 1.25 * float((ref[name][1] * step.abs()).sum())
        assert abs((sides[0] - sides[1]) / 2e-5 - float((grads[i].double() * step).sum())) <= bound + 1e-6


def test_captured_and_replayed_and_on_another_stream():
    x, dout, ptr = rand(3000, 32), rand(3000, 32, seed=1), offsets(3000, 9)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    out, mean, rstd = g.group_norm(x, 4, graph_ptr=ptr, with_stats=True, stream=stream)
    grads = g.group_norm_backward(dout, x, 4, mean, rstd, graph_ptr=ptr, stream=stream)
    stream.synchronize()
    ref = reference(x, 4, None, None, ptr, "none", EPS, dout)
    for name, got in zip(("out", "dx", "dw", "db"), (out, *grads)):
        check(got, ref[name], name)
    graphs, results = [], []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            o, m, r = g.group_norm(x, 4, graph_ptr=ptr, activation="silu", with_stats=True)
            results.append((o, *g.group_norm_backward(dout, x, 4, m, r, graph_ptr=ptr, activation="silu")))
        graphs.append(graph)
    x.copy_(rand(3000, 32, seed=8))
    ptr.copy_(offsets(3000, 9, seed=2))
    graphs[1].replay()
    graphs[0].replay()
    torch.cuda.synchronize()
    ref = reference(x, 4, None, None, ptr, "silu", EPS, dout)
    for res in results:
        for name, got in zip(("out", "dx", "dw", "db"), res):
            check(got, ref[name], name)


def test_a_layer_and_its_norm():
    """GCN layer, then the norm of its output over the graphs of the batch, in place."""
    n, e = 900, 5000
    gen = torch.Generator(device="cuda").manual_seed(0)
    src, dst = (torch.randint(n, (e,), generator=gen, device="cuda", dtype=torch.int32) for _ in range(2))
    csr = g.build_csr(n, src, dst, g.CSR_ADD_SELF_LOOPS)
    y = g.layer(csr, "gcn", rand(n, 40), rand(32, 40, seed=2), mode="fp32")
    kept, ptr = y.clone(), offsets(n, 5)
    g.group_norm(y, 4, graph_ptr=ptr, activation="relu", out=y)
    check(y, reference(kept, 4, None, None, ptr, "relu", EPS)["out"], "out", True)


def test_refusals():
    x = rand(50, 12)
    ptr = torch.tensor([0, 20, 50], device="cuda")
    with pytest.raises(ValueError, match="groups"):
        g.group_norm(x, 5)
    with pytest.raises(ValueError, match="activation"):
        g.group_norm(x, 3, activation="tanh")
    with pytest.raises(ValueError, match="weight"):
        g.group_norm(x, 3, weight=torch.ones(11, device="cuda"))
    with pytest.raises(ValueError, match="bias"):
        g.group_norm(x, 3, bias=torch.ones(12, device="cuda", dtype=BF16))
    with pytest.raises(ValueError, match="graph_ptr"):
        g.group_norm(x, 3, graph_ptr=ptr[:1])
    with pytest.raises(TypeError, match="graph_ptr"):
        g.group_norm(x, 3, graph_ptr=ptr.float())
    with pytest.raises(ValueError, match="overlap"):
        g.group_norm(x[:, :6], 3, out=x[:, 3:9])
    with pytest.raises(ValueError, match="rows"):
        g.group_norm(x, 3, out=torch.empty((49, 12), device="cuda"))
    with pytest.raises(g.GnnfdError):
        g.group_norm(x, 3, eps=-1.0)
    with pytest.raises(g.GnnfdError) as err:
        g.group_norm(torch.empty((4, 8200), device="cuda"), 1)
    assert err.value.status == g.UNSUPPORTED
    with pytest.raises(g.GnnfdError) as err:
        g.group_norm(x, 3, scratch=torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert err.value.status == g.WORKSPACE_TOO_SMALL
    out, mean, rstd = g.group_norm(x, 3, graph_ptr=ptr, with_stats=True)
    with pytest.raises(ValueError, match="mean"):
        g.group_norm_backward(x, x, 3, mean, rstd)
    with pytest.raises(TypeError, match="dout"):
        g.group_norm_backward(x.bfloat16(), x, 3, mean, rstd, graph_ptr=ptr)
    with pytest.raises(ValueError, match="overlap"):
        g.group_norm_backward(out, x, 3, mean, rstd, graph_ptr=ptr, out=x)
