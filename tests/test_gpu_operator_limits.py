"""The lookup, attention and group norm calls where one bad row stands among good ones, at extreme caps and sizes, and from two host
threads at once.  References and bounds are those of the operators' own tests, unless a test derives its own."""
import threading

import pytest

torch = pytest.importorskip("torch")

import paper_2104_03058_b200 as g  # noqa: E402
import test_gpu_attention as att  # noqa: E402
import test_gpu_embedding as emb  # noqa: E402
import test_gpu_group_norm as norm  # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24
INF = float("inf")


# ---------------------------------------------------------------- attention: bad rows

def with_bad_row(p, row, name, bad):
    """gradients and sums as they are, and with `bad` in row `row` of one operand"""
    clean = p.backward(p.forward(with_lse=True)[1])
    getattr(p, name)[row] = bad
    return clean, p.backward(p.forward(with_lse=True)[1])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("name,bad", [("q", float("nan")), ("q", INF), ("dout", float("nan"))])
@pytest.mark.parametrize("row,hub", [(0, 0), (0, 2500), (9, 0)])
def test_a_bad_row_changes_the_gradients_of_what_it_attends_to_alone(row, hub, name, bad, dtype):
    n = 400
    p = att.Problem(n, *att.edges(n, 3000, hub), 2, 8, dtype, cap=6.0)
    attended = torch.zeros(n, dtype=torch.bool, device="cuda")
    attended[p.col[p.row == row]] = True
    assert 0 < int(attended.sum()) < n
    clean, got = with_bad_row(p, row, name, bad)
    others = torch.arange(n, device="cuda") != row
    assert torch.equal(clean[0][others], got[0][others])                                  # dq
    for was, now in zip(clean[1:3], got[1:3]):                                            # dk, dv
        assert torch.equal(was[~attended], now[~attended])
    assert torch.isnan(got[1][attended]).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("name,bad", [("q", float("nan")), ("q", INF), ("dout", float("nan"))])
def test_a_bad_row_does_not_reach_what_the_bias_hides_from_it(name, bad, dtype):
    """Row 7 attends to the vertices of even number; a bias of -infinity hides the others from it, from other rows some."""
    n, row = 300, 7
    src, dst = att.edges(n, 6000)
    p = att.Problem(n, src, dst, 2, 16, dtype, cap=4.0, buckets=4)
    p.bias[1] = -INF
    dist = torch.randint(0, 4, src.shape, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda").int()
    dist[dst == row] = torch.where(src[dst == row] % 2 == 1, 1, 2).int()
    p.dist, p.dist_t = g.edge_values(p.csr, dist), g.edge_values(p.csr_t, dist)
    here = p.row == row
    attended, hidden = (torch.zeros(n, dtype=torch.bool, device="cuda") for _ in range(2))
    attended[p.col[here & (p.col % 2 == 0)]] = True
    hidden[p.col[here & (p.col % 2 == 1)]] = True
    assert int(attended.sum()) > 3 and int(hidden.sum()) > 3
    clean, got = with_bad_row(p, row, name, bad)
    for was, now in zip(clean[1:3], got[1:3]):
        assert torch.equal(was[~attended], now[~attended])
    assert (got[3][1] == 0).all() and torch.equal(clean[3][[0, 3]], got[3][[0, 3]]) and torch.isnan(got[3][2]).all()
    assert torch.isnan(got[1][attended]).all()


# ---------------------------------------------------------------- attention: caps

def check_capped(p, odt):
    """Against the bounds for a tanh that is within 8 u of its own value."""
    ref = att.reference(p.row, p.col, p.q.float(), p.k, p.v, p.heads, p.dim, p.scale, p.cap, p.dist, p.bias, p.dout)
    out, lse = p.forward(with_lse=True, out_dtype=odt)
    grads = p.backward(lse, out_dtype=odt)
    assert torch.equal(out, p.forward(with_lse=True, out_dtype=odt)[0])
    att.check(p.forward(out_dtype=odt), ref["out"], "out alone")
    want, bound = ref["lse"]
    some = want > -INF
    assert ((att.lse_of(lse) - want).abs() <= 1.25 * bound)[some].all()
    for name, got in zip(("out", "dq", "dk", "dv", "dbias"), (out, *grads)):
        if got is not None:
            att.check(got, ref[name], name)


@pytest.mark.parametrize("dtype,odt,cap", [(BF16, F32, 0.5), (BF16, F32, 30.0), (BF16, BF16, 1e3), (BF16, F32, 1e4), (BF16, BF16, 1e4), (BF16, F32, 1e7),
                                           (BF16, BF16, 1e7), (BF16, F32, 1e30), (F32, F32, 1e7)])
def test_caps_of_any_size(dtype, odt, cap):
    """A large cap is nearly none: scores as exact as without one, whatever the type of the features."""
    for hub in (0, 2300):
        check_capped(att.Problem(500, *att.edges(500, 6000, hub), 3, 16, dtype, cap=cap, buckets=4), odt)


def test_gradients_of_small_caps_are_exact_to_the_features_type():
    """Sums over the graph (the bias's gradient) stay fp32, so the capped scores behind them are as exact as for fp32 features."""
    check_capped(att.Problem(800, *att.edges(800, 20_000), 4, 8, BF16, cap=20.0, buckets=5), F32)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_caps_whose_reciprocal_is_beyond_fp32(dtype):
    """softcap = 1e-39: every score is within 1e-39 of 0, those of exactly 0 among them, so all entries weigh the same."""
    n = 200
    p = att.Problem(n, *att.edges(n, 2000), 2, 8, dtype, cap=1e-39)
    p.q[::2] = 0
    ref = att.reference(p.row, p.col, torch.zeros(n, 16, device="cuda"), p.k, p.v, 2, 8, 1.0, 0.0, dout=p.dout)
    out, lse = p.forward(with_lse=True)
    att.check(out, ref["out"], "out")
    dq, dk, dv, _ = p.backward(lse)
    att.check(dv, ref["dv"], "dv")
    assert torch.isfinite(dq).all() and torch.isfinite(dk).all()


# ---------------------------------------------------------------- gradient of the lookup

@pytest.mark.parametrize("f,itype", [(1, torch.int32), (5, torch.int64), (40, torch.int32)])
def test_the_largest_gradient_of_one_launch(f, itype):
    """As many ids and rows as the one-launch path takes, all of its shared memory in use; beside it one of each more."""
    for n, vocab in ((g.EMBEDDING_FEW_IDS, g.EMBEDDING_FEW_ROWS), (g.EMBEDDING_FEW_IDS + 1, g.EMBEDDING_FEW_ROWS), (g.EMBEDDING_FEW_IDS, g.EMBEDDING_FEW_ROWS + 1)):
        ids = emb.draw_ids(n, vocab, "skew", itype)
        ids[:3] = torch.tensor([vocab - 1, 0, vocab - 1], device="cuda")
        dout = emb.rand(n, f)
        emb.check_grad(g.embedding_backward(ids, dout, vocab, scale=0.7), ids, dout, vocab, 0.7)


def from_threads(calls, turns):
    """what went wrong in `turns` calls of each function, made by host threads at once"""
    wrong, start = [], threading.Barrier(len(calls))

    def work(call):
        start.wait()
        try:
            for _ in range(turns):
                call()
        except Exception as err:                                                          # noqa: BLE001
            wrong.append(err)
    threads = [threading.Thread(target=work, args=(call,)) for call in calls]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    return wrong


def test_gradients_of_different_sizes_from_threads():
    """Through the C call, so that the threads spend their time in it; each waits for its stream now and then, lest a full queue holds it up."""
    vocab, f, calls, jobs = 443, 8, [], []
    for n in (16_384, 9_000):
        ids, dout, out = emb.draw_ids(n, vocab, "even", torch.int32, n), emb.rand(n, f, seed=n), torch.empty((vocab, f), device="cuda")
        stream = torch.cuda.Stream()
        args = (n, ids.data_ptr(), g.I32, dout.data_ptr(), f, g.F32, vocab, f, 1.0, -1, 0, out.data_ptr(), f, g.F32, None, 0, None, stream.cuda_stream)
        jobs.append((ids, dout, out))

        def call(args=args, stream=stream, gradient=g.lib().gnnfd_embedding_backward):
            for _ in range(100):
                if gradient(*args) != g.OK:
                    raise RuntimeError("the call of %d ids failed" % args[0])
            stream.synchronize()
        calls.append(call)
    torch.cuda.synchronize()
    assert not from_threads(calls, 100)
    for ids, dout, out in jobs:
        emb.check_grad(out, ids, dout, vocab, 1.0)


def test_a_transform_as_the_first_call_of_a_thread():
    """A thread that has made no other call yet, the result's memory given."""
    x, w, out = emb.rand(300, 64), emb.rand(16, 64, seed=1), torch.empty((300, 16), device="cuda")
    want = g.combine(x, w)
    assert not from_threads([lambda: g.combine(x, w, out=out)], 1)
    assert torch.equal(out, want)


def test_transforms_of_different_sizes_from_threads():
    """One stream, so that the transforms run one after the other; only the calls meet."""
    calls, jobs = [], []
    for f_in, f_out in ((8, 240), (8, 16), (16, 8)):
        x, w = emb.rand(300, f_in, seed=f_in), emb.rand(f_out, f_in, seed=f_out)
        out = torch.empty((300, f_out), device="cuda")
        args = (300, x.data_ptr(), f_in, g.F32, f_in, w.data_ptr(), f_in, f_out, out.data_ptr(), f_out, g.F32, None, 0)
        jobs.append((out, g.combine(x, w, mode="tf32"), x, w))

        def call(args=args, transform=g.lib().gnnfd_combine):
            for _ in range(100):
                if transform(*args) != g.OK:
                    raise RuntimeError("the transform of %d columns failed" % args[4])
            torch.cuda.synchronize()
        calls.append(call)
    assert not from_threads(calls, 200)
    for out, want, _, _ in jobs:
        assert torch.equal(out, want)


@pytest.mark.parametrize("odt", [F32, BF16])
@pytest.mark.parametrize("vocab", [1000, g.EMBEDDING_FEW_ROWS, g.EMBEDDING_FEW_ROWS + 1, 5_000_000])
def test_the_gradient_of_no_ids(vocab, odt):
    ids, dout = torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty((0, 3), device="cuda")
    buf = torch.full((vocab, 5), 7.0, device="cuda", dtype=odt)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    g.embedding_backward(ids, dout, vocab, accumulate=True, out=buf[:, :3], status=status)
    assert (buf == 7.0).all()
    g.embedding_backward(ids, dout, vocab, out=buf[:, :3], status=status)
    assert (buf[:, :3] == 0).all() and (buf[:, 3:] == 7.0).all() and int(status) == 0
    fresh = g.embedding_backward(ids, torch.empty((0, 8), device="cuda"), vocab, out_dtype=odt)
    assert fresh.shape == (vocab, 8) and (fresh == 0).all()


# ---------------------------------------------------------------- group norm

@pytest.mark.parametrize("n,f,groups", [(3000, 16, 2), (200_000, 64, 32)])
def test_statistics_of_graphs_whose_offsets_go_back(n, f, groups):
    """They count as empty: mean 0 and rstd eps^-1/2, in calls of few pieces and of many."""
    x, eps = norm.rand(n, f), 1e-5
    ptr = torch.tensor([0, n // 2, n // 4, n], dtype=torch.int32, device="cuda")
    out, mean, rstd = torch.zeros_like(x), *(torch.full((3, groups), float("nan"), device="cuda") for _ in range(2))
    scratch = torch.empty(g.group_norm_workspace_bytes(n, f, groups, 3), dtype=torch.uint8, device="cuda")
    status = g.lib().gnnfd_group_norm(n, x.data_ptr(), f, g.F32, f, groups, 3, ptr.data_ptr(), g.I32, None, None, eps, 0, out.data_ptr(), f, g.F32,
                                      mean.data_ptr(), rstd.data_ptr(), scratch.data_ptr(), scratch.numel(), torch.cuda.current_stream().cuda_stream)
    assert status == g.OK
    assert (mean[1] == 0).all() and torch.allclose(rstd[1], torch.full_like(rstd[1], eps ** -0.5), rtol=4 * U)
    assert torch.isfinite(mean[0]).all() and torch.isfinite(rstd[0]).all()


def test_gelu_is_exact_relative_to_itself():
    """With a weight of 0 the norm's output is act(bias) and, of one row, the gradient of the bias act'(bias).  With Phi the normal distribution's
    integral: Phi(-|z|) is a polynomial, off by 13 u (2 u its fit, 5 its evaluation, 6 the reciprocal in it), times e^(-z^2/2): its argument carries
    three roundings, an error of 3 u z^2/2, and the exponential 2 ulp; two products more: 19 + 1.5 z^2, taken as (20 + 2 z^2) u of Phi.  For z > 0 it is
    1 - Phi(-z), one rounding more of results between a half and 1.  Below 2^-126 the exponential is 0.  The slope Phi + z phi adds (8 + 2 z^2) u of its
    second term and 2 u of the sum of both."""
    z = torch.cat([torch.linspace(-13, 13, 8000), torch.tensor([0.0, -0.0, -1e-20, 1e-20, 40.0, -40.0])]).cuda()
    z = torch.cat([z, torch.zeros(8192 - z.numel(), device="cuda")])
    x, w = norm.rand(1, z.numel(), seed=4), torch.zeros_like(z)
    out, mean, rstd = g.group_norm(x, 1, w, z, activation="gelu", with_stats=True)
    db = g.group_norm_backward(torch.ones_like(x), x, 1, mean, rstd, w, z, activation="gelu")[2]
    z = z.double()
    cdf, far = 0.5 * torch.special.erfc(-z / 2 ** 0.5), 0.5 * torch.special.erfc(z.abs() / 2 ** 0.5)
    e_cdf = (20 + 2 * z * z) * U * far + 2 ** -126 + torch.where(z > 0, 2 * U, 0.0)
    assert ((out[0].double() - z * cdf).abs() <= z.abs() * e_cdf + U * (z * cdf).abs() + 1e-37).all()
    part = z * torch.exp(-z * z / 2) / (2 * torch.pi) ** 0.5
    tol = e_cdf + (8 + 2 * z * z) * U * part.abs() + 2 * U * (cdf + part.abs()) + 2 ** -126 * z.abs() + 1e-37
    assert ((db.double() - (cdf + part)).abs() <= tol).all()


@pytest.mark.parametrize("act", ["none", "silu"])
def test_batches_of_small_graphs_in_the_root_mean_square(act):
    """Graphs of a warp each.  An output carries about ten roundings, half a step each at most; the statistics' errors average out over
    the 400 values or more of a group."""
    sizes = torch.randint(25, 60, (1500,), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    ptr = torch.cat([sizes.new_zeros(1), sizes.cumsum(0)])
    n = int(ptr[-1])
    for f, groups in ((128, 8), (64, 1), (48, 3)):
        x, dout = norm.rand(n, f, scale=2.0, mean=0.5), norm.rand(n, f, seed=1)
        w, b = norm.rand(1, f, seed=2)[0].contiguous(), norm.rand(1, f, seed=3)[0].contiguous()
        norm.both_ways(x, groups, w, b, ptr, act, dout, rms=True)
