"""Dot-product attention over a CSR and its gradients against an evaluation in 64 bits.

The tolerances are first-order bounds, computed entry by entry beside the reference from what the kernels do in fp32 (u = 2^-24 a rounding): a
dot product of d terms is off by at most (d + 2) u times the sum of its terms' magnitudes; the scaled score takes one rounding more, the capped one
tanh's (8 u of its value, for 16-bit features of 1) and two; the weight e^(s - m) carries the score's error, two roundings of its argument and 2 ulp of the exponential; a sum of k
terms (k + 4) u times the sum of their magnitudes; weights below 2^-126 are 0 (with scores of thousands, weights of e^-89 = 2e-39 times gradients and
a scale of 300 are results of 1e-36 that the kernels leave out).  These are propagated through the formulas; one rounding to the output type comes
last.  Factor 1.25 for second-order terms and for the few roundings of merging partial results."""
import pytest

torch = pytest.importorskip("torch")

import paper_2104_03058_b200 as g  # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24
TINY = 2.0 ** -126                                   # weights below it become 0: an absolute error of each weight, beside the relative one
INF = float("inf")


def rand(rows, cols, dtype=F32, ld=None, offset=0, seed=0, scale=1.0):
    ld = ld or cols
    gen = torch.Generator(device="cuda").manual_seed(seed + 29)
    buf = torch.full((rows * ld + offset + 8,), float("nan"), device="cuda", dtype=dtype)
    view = buf[offset:offset + rows * ld].view(rows, ld)[:, :cols]
    view.copy_(torch.randn((rows, cols), generator=gen, device="cuda") * scale)
    return view


def edges(n, e, hub=0, seed=0):
    """e random edges, `hub` more that end in vertex n // 2 and as many that start there; the last third of the vertices ends none."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    src = torch.randint(n, (e,), generator=gen, device="cuda")
    dst = torch.randint(max(1, n - n // 3), (e,), generator=gen, device="cuda")
    if hub:
        other = torch.randint(n, (hub,), generator=gen, device="cuda")
        mid = torch.full((hub,), n // 2, device="cuda")
        src, dst = torch.cat([src, other, mid]), torch.cat([dst, mid, other % max(1, n - n // 3)])
    order = torch.randperm(src.numel(), generator=gen, device="cuda")
    return src[order].int(), dst[order].int()


def rowsum(n, index, x):
    return torch.zeros((n,) + x.shape[1:], dtype=torch.float64, device="cuda").index_add_(0, index, x)


def reference(row, col, q, k, v, heads, dim, scale, cap, dist=None, bias=None, dout=None):
    """{name: (value, bound)} with values [n, heads, dim]; entries with a bias of -inf are left out."""
    n = q.shape[0]
    keep = torch.ones_like(row, dtype=torch.bool)
    res = {}
    outs = {name: [] for name in ("out", "lse", "dq", "dk", "dv", "dbias")}
    rough = q.dtype != F32
    q, k, v = (t.double().reshape(n, heads, dim) for t in (q, k, v))
    if dout is not None:
        dout = dout.double().reshape(n, heads, dim)
    buckets = bias.shape[0] if bias is not None else 0
    for h in range(heads):
        r, c = row, col
        d = None
        if bias is not None:
            d = dist.long().clamp(0, buckets - 1)
            b_all = bias[:, h].double()
            keep = b_all[d] != -INF
            r, c, d = row[keep], col[keep], d[keep]
        qr, kc, vc = q[r, h], k[c, h], v[c, h]
        raw = (qr * kc).sum(1) * scale
        e_s = (dim + 3) * U * abs(scale) * (qr * kc).abs().sum(1)
        s, slope, e_slope = raw, torch.ones_like(raw), torch.zeros_like(raw)
        if cap:
            t = torch.tanh(raw / cap)
            s, slope = cap * t, 1 - t * t
            e_t = (e_s / cap + 2 * U * (raw / cap).abs()) * slope + 8 * U * (1 if rough else t.abs())
            e_s = cap * e_t + U * s.abs()
            e_slope = 2 * t.abs() * e_t + 2 * U
        if bias is not None:
            s = s + b_all[d]
            e_s = e_s + U * (s.abs())
        top = torch.full((n,), -INF, dtype=torch.float64, device="cuda").scatter_reduce_(0, r, s, "amax")
        w = torch.exp(s - top[r])
        total = rowsum(n, r, w)
        p = w / total[r]
        cnt = rowsum(n, r, torch.ones_like(s))
        e_w = e_s + 3 * U * (s - top[r]).abs() + 4 * U                       # relative error of a weight under the true maximum
        e_top = torch.zeros(n, dtype=torch.float64, device="cuda").scatter_reduce_(0, r, e_s, "amax")
        e_p = e_w + rowsum(n, r, p * e_w)[r] + ((cnt + 6) * U)[r]
        out = rowsum(n, r, p[:, None] * vc)
        e_abs = p * e_p + TINY                                               # of a weight, absolute
        out_b = rowsum(n, r, e_abs[:, None] * vc.abs()) + (cnt[:, None] + 6) * U * rowsum(n, r, p[:, None] * vc.abs())
        outs["out"].append((out, out_b))
        lse = torch.where(total > 0, top + torch.log(total.clamp_min(1e-300)), -INF)
        outs["lse"].append((lse, e_top + rowsum(n, r, p * e_w) + (cnt + 8) * U + 2 * U * lse.abs().nan_to_num(0, 0, 0)))
        if dout is None:
            continue
        do = dout[r, h]
        dp = (do * vc).sum(1)
        e_dp = (dim + 2) * U * (do * vc).abs().sum(1)
        dd = rowsum(n, r, p * dp)
        e_dd = rowsum(n, r, e_abs * dp.abs() + p * e_dp) + (cnt + 4) * U * rowsum(n, r, p * dp.abs())
        ds = p * (dp - dd[r])
        e_ds = e_abs * (dp - dd[r]).abs() + p * (e_dp + e_dd[r] + 4 * U * (dp.abs() + dd[r].abs()))
        dt, e_dt = ds * slope, e_ds * slope + ds.abs() * e_slope + 2 * U * ds.abs()
        pc = p * slope
        e_pc = e_abs * slope + p * e_slope + 2 * U * pc
        ka = kc.abs()
        a_size, b_size = rowsum(n, r, (pc * dp.abs())[:, None] * ka), rowsum(n, r, pc[:, None] * ka)
        e_dq = (rowsum(n, r, (e_pc * dp.abs() + pc * e_dp)[:, None] * ka) + e_dd[:, None] * b_size + dd.abs()[:, None] * rowsum(n, r, e_pc[:, None] * ka)
                + (cnt[:, None] + 6) * U * (a_size + dd.abs()[:, None] * b_size))
        outs["dq"].append((scale * rowsum(n, r, dt[:, None] * kc), abs(scale) * e_dq))
        ccnt = rowsum(n, c, torch.ones_like(s))[:, None]
        outs["dk"].append((scale * rowsum(n, c, dt[:, None] * qr), abs(scale) * (rowsum(n, c, e_dt[:, None] * qr.abs())
                                                                             + (ccnt + 6) * U * rowsum(n, c, dt.abs()[:, None] * qr.abs()))))
        outs["dv"].append((rowsum(n, c, p[:, None] * do), rowsum(n, c, e_abs[:, None] * do.abs())
                           + (ccnt + 6) * U * rowsum(n, c, p[:, None] * do.abs())))
        if bias is not None:
            bcnt = rowsum(buckets, d, torch.ones_like(s))
            outs["dbias"].append((rowsum(buckets, d, ds), rowsum(buckets, d, e_ds) + (bcnt + 6) * U * rowsum(buckets, d, ds.abs())))
    for name, parts in outs.items():
        if parts:
            res[name] = tuple(torch.stack([p[i] for p in parts], dim=1) for i in (0, 1))
    return res


def check(got, ref, what):
    want, bound = ref
    if want.dim() == 3 and got.dim() == 2:
        got = got.reshape(want.shape)
    half = torch.finfo(got.dtype).eps / 2
    tol = 1.25 * bound + half * want.abs() + 1e-37
    bad = ~((got.double() - want).abs() <= tol)
    assert not bad.any(), "%s: %d of %d off, worst %.3g of its bound" % (what, int(bad.sum()), bad.numel(),
                                                                          float(((got.double() - want).abs() / tol).nan_to_num(1e9).max()))


def lse_of(pair):
    return pair[..., 0].double() + torch.log(pair[..., 1].double())


def rows_of(csr):
    deg = csr.row_ptr[1:] - csr.row_ptr[:-1]
    return torch.repeat_interleave(torch.arange(csr.n, device="cuda"), deg.long()), csr.col_idx.long()


class Problem:
    def __init__(self, n, src, dst, heads, dim, dtype=F32, cap=0.0, buckets=0, flags=0, ld=None, offset=0, scale=None, seed=0):
        f = heads * dim
        self.heads, self.dim, self.cap, self.scale = heads, dim, cap, dim ** -0.5 if scale is None else scale
        self.csr, self.csr_t = g.build_csr(n, src, dst, flags), g.build_csr(n, dst, src, flags)
        self.q, self.k, self.v, self.dout = (rand(n, f, dtype, ld, offset, seed + i) for i in range(4))
        self.bias = rand(buckets, heads, seed=seed + 7) if buckets else None
        self.dist = self.dist_t = None
        if buckets:
            gen = torch.Generator(device="cuda").manual_seed(seed + 3)
            edge_dist = torch.randint(-1, buckets + 2, (src.numel(),), generator=gen, device="cuda").int()
            self.dist, self.dist_t = g.edge_values(self.csr, edge_dist), g.edge_values(self.csr_t, edge_dist)
        self.row, self.col = rows_of(self.csr)

    def forward(self, **kw):
        return g.aggregate_attention(self.csr, self.q, self.k, self.v, self.heads, self.dim, scale=self.scale, softcap=self.cap, dist=self.dist,
                                     bias=self.bias, **kw)

    def backward(self, lse, **kw):
        return g.aggregate_attention_backward(self.csr, self.csr_t, self.q, self.k, self.v, self.dout, lse, self.heads, self.dim,
                                              scale=self.scale, softcap=self.cap, dist=self.dist, dist_t=self.dist_t, bias=self.bias, **kw)

    def reference(self, grads=True):
        return reference(self.row, self.col, self.q, self.k, self.v, self.heads, self.dim, self.scale, self.cap, self.dist, self.bias,
                         self.dout if grads else None)

    def check(self, **kw):
        out, lse = self.forward(with_lse=True, **kw)
        ref = self.reference()
        check(out, ref["out"], "out")
        want, bound = ref["lse"]
        empty = want == -INF
        assert (lse[..., 0][empty] == -INF).all() and (lse[..., 1][empty] == 0).all()
        assert ((lse_of(lse) - want).abs() <= 1.25 * bound)[~empty].all()
        grads = self.backward(lse, **{k: w for k, w in kw.items() if k in ("chunk_width", "out_dtype")})
        for name, got in zip(("dq", "dk", "dv", "dbias"), grads):
            if got is None:
                assert name == "dbias" and self.bias is None
            else:
                check(got, ref[name], name)
        return out, lse, grads


HEADS = [(1, 1), (1, 4), (2, 7), (8, 8), (3, 16), (6, 20), (1, 64), (4, 32), (1, 256), (2, 100), (20, 8), (40, 1)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("heads,dim", HEADS)
def test_head_layouts(heads, dim, dtype):
    src, dst = edges(700, 9000)
    Problem(700, src, dst, heads, dim, dtype, cap=4.0, buckets=5).check(out_dtype=dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("cap,buckets", [(0.0, 0), (2.0, 0), (0.0, 1), (30.0, 90)])
@pytest.mark.parametrize("n,e,hub", [(1, 0, 0), (1, 1, 0), (2, 3, 0), (300, 100, 0), (5000, 20_000, 0), (3000, 30_000, 2500), (400, 3000, 7000)])
def test_graphs(n, e, hub, cap, buckets, dtype):
    src, dst = edges(n, e, hub)
    Problem(n, src, dst, 4, 8, dtype, cap=cap, buckets=buckets).check()


@pytest.mark.parametrize("flags", [0, g.CSR_ADD_SELF_LOOPS, g.CSR_SYMMETRIZE, g.CSR_SYMMETRIZE | g.CSR_ADD_SELF_LOOPS | g.CSR_DEDUP, g.CSR_INPUT_ORDER])
def test_build_flags(flags):
    src, dst = edges(600, 4000, 2300)
    Problem(600, src, dst, 2, 16, cap=0.0, buckets=4, flags=flags).check()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("heads,dim,ld,offset", [(8, 8, 64, 1), (2, 24, 50, 0), (4, 16, 64, 4), (4, 16, 72, 8), (1, 48, 56, 2), (3, 12, 36, 0)])
def test_pitches_and_alignments(heads, dim, ld, offset, dtype):
    src, dst = edges(500, 6000, 2200)
    Problem(500, src, dst, heads, dim, dtype, buckets=3, ld=ld, offset=offset).check()


@pytest.mark.parametrize("heads,dim,width", [(8, 8, 8), (8, 8, 24), (6, 20, 40), (5, 64, 64)])
def test_chunks_of_heads(heads, dim, width):
    src, dst = edges(90, 900, 2100)
    Problem(90, src, dst, heads, dim, buckets=2).check(chunk_width=width)


def test_more_chunks_than_a_grid_has_rows():
    src, dst = edges(4, 7)
    p = Problem(4, src, dst, 70_000, 1)
    out, lse = p.forward(with_lse=True, chunk_width=1)
    grads = p.backward(lse, chunk_width=1)
    some = torch.tensor([0, 65_534, 65_535, 65_536, 69_999], device="cuda")
    ref = reference(p.row, p.col, *(t[:, some] for t in (p.q, p.k, p.v)), 5, 1, p.scale, 0.0, dout=p.dout[:, some])
    for name, got in zip(("out", "dq", "dk", "dv"), (out, *grads)):
        check(got[:, some], ref[name], name)


@pytest.mark.parametrize("n,deg", [(4000, 10), (20_000, 50)])
def test_long_rows_of_small_graphs_shared_by_warps(n, deg):
    src, dst = edges(n, n * deg, 1900)
    out, lse, grads = (p := Problem(n, src, dst, 1, 128, cap=9.0, buckets=3)).check()
    assert torch.equal(out, p.forward())                                                  # equal bits
    assert all(torch.equal(x, y) for x, y in zip(grads, p.backward(lse)))


def test_masked_entries_count_for_nothing_whatever_stands_there():
    n, heads, dim = 60, 2, 8
    src, dst = edges(n, 700)
    p = Problem(n, src, dst, heads, dim, buckets=3, cap=5.0)
    p.bias[1] = -INF                                                                      # bucket 1 is a mask
    p.bias[2, 0] = -INF                                                                   # bucket 2 for one head
    masked = p.dist.clamp(0, 2) == 1
    p.dist[p.row == 3], p.dist_t[p.csr_t.col_idx.long() == 3] = 1, 1                      # row 3 has nothing left
    sources = torch.zeros(n, dtype=torch.bool, device="cuda")
    sources[p.col[(p.dist.clamp(0, 2) != 1)]] = True
    hidden = torch.nonzero(~sources).flatten()
    p.check()
    out, lse = p.forward(with_lse=True)
    assert (out[3] == 0).all() and (lse[3, :, 0] == -INF).all() and (lse[3, :, 1] == 0).all()
    # a vertex that every edge masks may hold anything
    u = int(hidden[0]) if hidden.numel() else 59
    p.dist[p.col == u], p.dist_t[torch.repeat_interleave(torch.arange(n, device="cuda"), (p.csr_t.row_ptr[1:] - p.csr_t.row_ptr[:-1]).long()) == u] = 1, 1
    before = p.forward(with_lse=True)
    grads = p.backward(before[1])
    for bad in (float("nan"), INF, -INF):
        p.k[u], p.v[u] = bad, bad
        after = p.forward(with_lse=True)
        assert torch.equal(before[0], after[0]) and torch.equal(before[1], after[1])
        for x, y in zip(grads, p.backward(after[1])):
            assert torch.equal(x, y)
    assert (grads[1][u] == 0).all() and (grads[2][u] == 0).all()
    assert int(masked.sum()) > 0


def test_biases_of_the_lowest_value():
    n, heads, dim = 40, 2, 16
    src, dst = edges(n, 500)
    p = Problem(n, src, dst, heads, dim, buckets=2)
    lowest = torch.finfo(F32).min
    p.bias[1] = lowest
    p.dist[p.row == 5], p.dist_t[p.csr_t.col_idx.long() == 5] = 1, 1                      # every entry of row 5 has the lowest bias
    out, lse = p.forward(with_lse=True)
    ref = p.reference(grads=False)["out"]
    others = torch.arange(n, device="cuda") != 5
    check(out.reshape(n, heads, dim)[others], tuple(t[others] for t in ref), "out")
    # scores of ordinary size vanish beside the lowest value: all entries weigh the same
    same = p.v[p.col[p.row == 5]].double().mean(0)
    assert ((out[5].double() - same).abs() <= 40 * U * p.v[p.col[p.row == 5]].double().abs().mean(0) + 1e-30).all()
    dq, dk, dv, db = p.backward(lse)
    assert all(torch.isfinite(t).all() for t in (out, dq, dk, dv, db))
    share = 1.0 / int((p.row == 5).sum())
    only5 = torch.zeros(n, device="cuda", dtype=torch.float64).index_add_(0, p.col[p.row == 5], torch.full_like(p.col[p.row == 5], share, dtype=torch.float64))
    p.dout[others] = 0
    dv = p.backward(lse)[2].double()
    assert ((dv - only5[:, None] * p.dout[5].double()).abs() <= 40 * U * only5[:, None] * p.dout[5].double().abs() + 1e-30).all()


def test_large_scores_and_not_a_number():
    n = 50
    src, dst = edges(n, 600)
    p = Problem(n, src, dst, 2, 8, scale=300.0)
    p.check()                                                                            # scores of thousands, weights 0 and 1
    p.q[7] = float("nan")
    out = p.forward()
    rows = (p.row == 7).any()
    assert bool(rows) and torch.isnan(out[7]).all() and torch.isfinite(out[torch.arange(n, device="cuda") != 7]).all()


def test_gradients_agree_with_differences():
    """Differences of the 64-bit formula (step 1e-5: off by about 1e-10 of its curvature) against the kernels' gradients."""
    src, dst = edges(30, 200)
    p = Problem(30, src, dst, 2, 4, cap=3.0, buckets=3)
    _, lse = p.forward(with_lse=True)
    grads, ref = p.backward(lse), p.reference()
    loss = lambda: float((p.reference(False)["out"][0].reshape(30, 8) * p.dout.double()).sum())        # noqa: E731
    for name, grad in zip(("q", "k", "v", "bias"), grads):
        kept = getattr(p, name)
        step = torch.randn(kept.shape, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda", dtype=torch.float64)
        sides = []
        for sign in (1e-5, -1e-5):
            setattr(p, name, kept.double() + sign * step)
            sides.append(loss())
        setattr(p, name, kept)
        bound = float((ref["d" + name][1].reshape(kept.shape) * step.abs()).sum()) * 1.25
        assert abs((sides[0] - sides[1]) / 2e-5 - float((grad.double() * step).sum())) <= bound + 1e-6


def test_captured_replayed_on_other_streams_and_two_graphs_with_their_own_workspaces():
    src, dst = edges(800, 9000, 2600)
    p = Problem(800, src, dst, 4, 16, buckets=4, cap=6.0)
    out, lse = p.forward(with_lse=True)
    grads = p.backward(lse)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    out_s, lse_s = p.forward(with_lse=True, stream=stream)
    grads_s = p.backward(lse_s, stream=stream)
    stream.synchronize()
    assert torch.equal(out, out_s) and all(torch.equal(x, y) for x, y in zip(grads, grads_s))
    graphs, results = [], []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            o, ls = p.forward(with_lse=True)
            results.append((o, *p.backward(ls)))
        graphs.append(graph)
    for t in (p.q, p.k, p.v, p.dout):
        t.copy_(rand(*t.shape, seed=77))
    graphs[1].replay()
    graphs[0].replay()
    torch.cuda.synchronize()
    ref = p.reference()
    for res in results:
        for name, got in zip(("out", "dq", "dk", "dv", "dbias"), res):
            check(got, ref[name], name)


def test_a_run_of_lookup_attention_and_their_gradients():
    """Learned vertex rows looked up, projected slices attended, the gradients carried back into the table."""
    n, heads, dim, vocab = 500, 2, 8, 90
    f = heads * dim
    src, dst = edges(n, 6000)
    ids = torch.randint(vocab, (n,), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    table = rand(vocab, 3 * f)
    x = g.embedding(table, ids, scale=0.5)
    p = Problem(n, src, dst, heads, dim, buckets=3)
    p.q, p.k, p.v = x[:, :f], x[:, f:2 * f], x[:, 2 * f:]                                  # slices of one matrix
    out, lse, grads = p.check()
    dx = torch.cat(grads[:3], dim=1)
    dtable = g.embedding_backward(ids, dx, vocab, scale=0.5)
    leaf = table.double().requires_grad_()
    xx = leaf[ids] * 0.5
    q, k, v = (t.reshape(n, heads, dim) for t in (xx[:, :f], xx[:, f:2 * f], xx[:, 2 * f:]))
    s = (q[p.row] * k[p.col]).sum(2) * dim ** -0.5 + p.bias.double()[p.dist.long().clamp(0, 2)]
    w = torch.exp(s)
    y = rowsum(n, p.row, w[:, :, None] * v[p.col]) if False else torch.zeros((n, heads, dim), dtype=torch.float64, device="cuda").index_add(
        0, p.row, w[:, :, None] * v[p.col])
    y = y / torch.zeros((n, heads), dtype=torch.float64, device="cuda").index_add(0, p.row, w).clamp_min(1e-300)[:, :, None]
    want, = torch.autograd.grad(y, leaf, p.dout.double().reshape(n, heads, dim))
    ref = p.reference()
    bound = torch.cat([ref[name][1].reshape(n, f) for name in ("dq", "dk", "dv")], dim=1)
    size = torch.cat([ref[name][0].reshape(n, f) for name in ("dq", "dk", "dv")], dim=1).abs()
    count = torch.bincount(ids, minlength=vocab)[:, None]
    tol = 0.5 * (1.25 * rowsum(vocab, ids, bound + U * size) + (count + 3) * U * rowsum(vocab, ids, size))
    assert ((dtable.double() - want).abs() <= tol + 1e-30).all()


def test_edge_values():
    src, dst = torch.tensor([0, 1, 2, 2], device="cuda"), torch.tensor([1, 2, 2, 0], device="cuda")
    csr = g.build_csr(3, src, dst, g.CSR_SYMMETRIZE | g.CSR_ADD_SELF_LOOPS)
    got = g.edge_values(csr, torch.tensor([10, 20, 30, 40], device="cuda"), loop=-7)
    row, col = rows_of(csr)
    table = {(1, 0): 10, (0, 1): 10, (2, 1): 20, (1, 2): 20, (0, 2): 40, (2, 0): 40, (0, 0): -7, (1, 1): -7, (2, 2): -7}
    assert [table[int(r), int(c)] for r, c in zip(row, col)] == got.tolist()
    empty = g.build_csr(2, src[:0], dst[:0], g.CSR_ADD_SELF_LOOPS)
    assert g.edge_values(empty, torch.empty(0, device="cuda"), loop=1.5).tolist() == [1.5, 1.5]


def test_refusals():
    src, dst = edges(20, 100)
    p = Problem(20, src, dst, 2, 4, buckets=3)
    f = 8
    call = lambda **kw: g.aggregate_attention(p.csr, kw.pop("q", p.q), kw.pop("k", p.k), p.v, kw.pop("heads", 2), kw.pop("dim", 4), **kw)   # noqa: E731
    with pytest.raises(ValueError, match="come together"):
        call(bias=p.bias)
    with pytest.raises(ValueError, match="nnz"):
        call(bias=p.bias, dist=p.dist[:50])
    with pytest.raises(ValueError, match="nnz"):
        call(bias=p.bias, dist=p.dist.long())
    with pytest.raises(ValueError, match="buckets"):
        call(bias=p.bias[:, :1], dist=p.dist)
    with pytest.raises(ValueError, match="rows"):
        call(k=p.k[:19])
    with pytest.raises(TypeError):
        call(q=p.q.bfloat16())
    with pytest.raises(ValueError, match="overlap"):
        call(out=p.v)
    with pytest.raises(ValueError, match="columns"):
        call(heads=3)
    for kw in (dict(softcap=-1.0), dict(softcap=float("nan")), dict(softcap=INF), dict(scale=float("nan")), dict(chunk_width=3), dict(chunk_width=0)):
        with pytest.raises(g.GnnfdError) as err:
            call(**kw)
        assert err.value.status == g.INVALID_ARG
    with pytest.raises(g.GnnfdError) as err:
        wide = rand(20, 257)
        g.aggregate_attention(p.csr, wide, wide, wide, 1, 257)
    assert err.value.status == g.UNSUPPORTED
    _, lse = p.forward(with_lse=True)
    with pytest.raises(ValueError, match="reverse"):
        g.aggregate_attention_backward(p.csr, g.build_csr(20, src[:5], dst[:5]), p.q, p.k, p.v, p.dout, lse, 2, 4)
    with pytest.raises(ValueError, match="lse"):
        g.aggregate_attention_backward(p.csr, p.csr_t, p.q, p.k, p.v, p.dout, lse[..., 0], 2, 4)
    with pytest.raises(ValueError, match="dist_t"):
        g.aggregate_attention_backward(p.csr, p.csr_t, p.q, p.k, p.v, p.dout, lse, 2, 4, dist=p.dist, bias=p.bias)
    assert p.q.shape[1] == f
