"""The gated linear recurrence and its gradients against a walk from row to row in 64 bits.

Bounds come out of the same walk (u = 2^-24).  M is the walk over magnitudes.  Whatever way the call joins stretches of rows, a term on its way from its
row to another is multiplied and added once a row and once more per joint, of which there are no more than rows, two roundings each: 4 u of M a row, and 8 u where it
starts.  A sigmoid's a and 1 - a are off by (2 |gate| + 8) u of themselves: the exponent's rounding, 4 u for the exponential, 3 u for the reciprocal and
1 u for the product.  The gradients' walk goes the other way with the same errors, and its products with h[t - 1] or h[t - 1] - x
carry the errors of both.  Bounds add up errors that mostly cancel, so fp32 results also have to be within 32 u in the root mean square: states average
over some hundred rows here, whose roundings (a few half steps each) add up like the root of their number."""
import pytest

torch = pytest.importorskip("torch")

import paper_2104_03058_b200 as g  # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24


def rand(rows, cols, dtype=F32, ld=None, offset=0, seed=0, scale=1.0, mean=0.0):
    ld = ld or cols
    gen = torch.Generator(device="cuda").manual_seed(seed + 3)
    buf = torch.full((rows * ld + offset + 8,), float("nan"), device="cuda", dtype=dtype)
    view = buf[offset:offset + rows * ld].view(rows, ld)[:, :cols]
    view.copy_(torch.randn((rows, cols), generator=gen, device="cuda") * scale + mean)
    return view


def gates(form, rows, cols, dtype=F32, ld=None, offset=0, seed=0):
    t = rand(rows, cols, F32, None, 0, seed, 2.0, 1.5)
    out = rand(rows, cols, dtype, ld, offset, seed)
    out.copy_(torch.sigmoid(t) * torch.where(rand(rows, cols, seed=seed + 1) < -1, -1.0, 1.0) if form == "factor" else t)
    return out


def bounds_of(n, graphs, ptr):
    """[(first row, one past the last row)] of each graph, on the host"""
    if ptr is None:
        return [(b * (n // graphs), (b + 1) * (n // graphs)) for b in range(graphs)]
    p = ptr.tolist()
    return list(zip(p[:-1], p[1:]))


def reference(x, gate, form, spans, initial, dout=None, dfinal=None):
    """{name: (value, bound)}.  All graphs side by side, padded to the longest, a row at a time."""
    graphs, f, n = len(spans), x.shape[1], x.shape[0]
    longest = max([e - s for s, e in spans] + [1])
    size = torch.tensor([e - s for s, e in spans], device="cuda")
    at = (torch.tensor([s for s, _ in spans], device="cuda")[:, None] + torch.arange(longest, device="cuda"))
    live = torch.arange(longest, device="cuda") < size[:, None]
    at = at.clamp(0, max(0, n - 1))
    take = lambda t: torch.where(live[:, :, None], t.double()[at] if n else torch.zeros((graphs, longest, f), device="cuda", dtype=torch.float64), 0.0)      # noqa: E731
    xs, gs = take(x), take(gate)
    if form == "factor":
        a, rest, rho = gs, torch.ones_like(gs), torch.zeros_like(gs)
    else:
        a, rest, rho = torch.sigmoid(gs), torch.sigmoid(-gs), (2 * gs.abs() + 8) * U
    b = rest * xs
    h = torch.zeros((graphs, f), dtype=torch.float64, device="cuda") if initial is None else initial.double()
    m, e = h.abs(), torch.zeros_like(h)
    hs, ms, es = [h], [m], [e]
    for t in range(longest):
        on = live[:, t, None]
        e = torch.where(on, a[:, t].abs() * e + (rho[:, t] + 4 * U) * a[:, t].abs() * m + (rho[:, t] + 8 * U) * b[:, t].abs(), e)
        m = torch.where(on, a[:, t].abs() * m + b[:, t].abs(), m)
        h = torch.where(on, a[:, t] * h + b[:, t], h)
        hs.append(h), ms.append(m), es.append(e)

    def put(rows):
        out = torch.zeros((n, f), dtype=torch.float64, device="cuda")
        out[at[live]] = torch.stack(rows, 1)[live]
        return out

    res = {"out": (put(hs[1:]), put(es[1:])), "final": (h, e)}
    if dout is None:
        return res
    ds = take(dout)
    c = torch.zeros((graphs, f), dtype=torch.float64, device="cuda") if dfinal is None else dfinal.double()
    mc, ec = c.abs(), torch.zeros_like(c)
    dx, dg = [None] * longest, [None] * longest
    for t in range(longest - 1, -1, -1):
        on, w, k, p = live[:, t, None], a[:, t], rest[:, t], rho[:, t]
        total, mt = ds[:, t] + c, ds[:, t].abs() + mc
        et = ec + 8 * U * mt
        dx[t] = (k * total, k * et + (p + U) * k * mt)
        if form == "factor":
            other, eo = hs[t], es[t]
        else:
            other = (hs[t] - xs[:, t]) * w * k
            eo = (es[t] + U * (hs[t].abs() + xs[:, t].abs())) * w * k + (2 * p + 3 * U) * other.abs()
        dg[t] = (total * other, et * other.abs() + mt * eo + U * (total * other).abs())
        ec = torch.where(on, w.abs() * et + (p + 4 * U) * w.abs() * mt, ec)
        mc = torch.where(on, w.abs() * mt, mc)
        c = torch.where(on, w * total, c)
    res["dx"], res["dgate"] = ((put([v for v, _ in t]), put([e for _, e in t])) for t in (dx, dg))
    res["dinitial"] = (c, ec)
    return res


def check(got, ref, what, rms=True):
    want, bound = ref
    half = torch.finfo(got.dtype).eps / 2
    tol = 1.25 * bound + half * want.abs() + 1e-36
    err = (got.double() - want).abs()
    assert got.shape == want.shape and (err <= tol).all(), "%s: %d of %d off, worst %.3g of its bound" % (
        what, int((~(err <= tol)).sum()), err.numel(), float((err / tol).nan_to_num(1e9).max()))
    if rms and got.dtype == F32 and got.numel() > 1000:
        assert float(err.pow(2).mean().sqrt()) <= 32 * U * float(want.pow(2).mean().sqrt()), what


def both_ways(n, f, form, graphs=1, ptr=None, xdt=F32, odt=F32, ld=None, offset=0, with_initial=True, seed=0, used=None):
    x, gate, dout = rand(n, f, xdt, ld, offset, seed + 1), gates(form, n, f, xdt, ld, offset, seed + 2), rand(n, f, xdt, ld, offset, seed + 4)
    graphs = graphs if ptr is None else ptr.numel() - 1
    initial, dfinal = (rand(graphs, f, seed=seed + i).contiguous() if with_initial else None for i in (5, 6))
    used = n if used is None else used
    ref = reference(x, gate, form, bounds_of(n, graphs, ptr), initial, dout, dfinal)
    batch = dict(graph_ptr=ptr, graphs=graphs, initial=initial)
    guard = torch.full((n * (f + 3) + offset,), 7.0, device="cuda", dtype=odt)
    buf = guard[offset:].view(n, f + 3)
    out, final, states = g.linear_recurrence(x, gate, form, out=buf[:, :f], with_final=True, with_states=True, **batch)
    assert (buf[:, f:] == 7.0).all() and (guard[:offset] == 7.0).all() and (buf[used:] == 7.0).all()
    check(out[:used], [t[:used] for t in ref["out"]], "out")
    check(final, ref["final"], "final")
    plain = g.linear_recurrence(x, gate, form, out_dtype=odt, **batch)
    check(plain[:used], [t[:used] for t in ref["out"]], "out, aligned")
    dx, dgate, dinitial = g.linear_recurrence_backward(dout, x, gate, states, form, dfinal=dfinal, out_dtype=odt, **batch)
    check(dx[:used], [t[:used] for t in ref["dx"]], "dx")
    check(dgate[:used], [t[:used] for t in ref["dgate"]], "dgate")
    if with_initial:
        check(dinitial, ref["dinitial"], "dinitial")
    else:
        assert dinitial is None


def offsets(n, graphs, seed=0, itype=torch.int32, last=None):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    last = n if last is None else last
    cuts = torch.randint(last + 1, (graphs - 1,), generator=gen, device="cuda").sort().values
    return torch.cat([cuts.new_zeros(1), cuts, cuts.new_full((1,), last)]).to(itype)


@pytest.mark.parametrize("form", ["factor", "sigmoid"])
@pytest.mark.parametrize("xdt,odt", [(F32, F32), (BF16, BF16), (F32, BF16), (BF16, F32)])
@pytest.mark.parametrize("n,f,ld,offset", [(1, 1, 1, 0), (5, 3, 3, 1), (15, 8, 8, 0), (16, 8, 8, 0), (17, 41, 41, 0), (300, 64, 64, 0), (333, 20, 22, 0), (511, 9, 9, 0), (512, 24, 24, 0), (513, 12, 12, 0), (1030, 16, 16, 0), (600, 900, 900, 0),
                                           (2047, 12, 12, 2), (2048, 4, 4, 0), (2049, 4, 4, 0), (2500, 33, 40, 0), (3001, 70, 72, 4), (4100, 301, 301, 0),
                                           (2600, 128, 128, 0), (3000, 260, 260, 2)])
def test_one_graph(n, f, ld, offset, xdt, odt, form):
    both_ways(n, f, form, xdt=xdt, odt=odt, ld=ld, offset=offset)


@pytest.mark.parametrize("form", ["factor", "sigmoid"])
@pytest.mark.parametrize("itype", [torch.int32, torch.int64])
@pytest.mark.parametrize("n,graphs,f,last", [(1, 3, 4, 1), (40, 40, 8, 40), (500, 7, 16, 500), (1000, 900, 12, 1000), (2000, 5, 31, 1800), (3000, 1, 8, 2999),
                                             (3000, 10, 48, 3000), (6000, 300, 20, 6000), (6000, 5000, 9, 5990), (20_000, 40, 16, 20_000)])
def test_batches_of_graphs(n, graphs, f, last, itype, form):
    both_ways(n, f, form, ptr=offsets(n, graphs, n, itype, last), used=last)


@pytest.mark.parametrize("form", ["factor", "sigmoid"])
@pytest.mark.parametrize("n,graphs,f", [(7, 7, 5), (256, 256, 64), (3000, 3000, 24), (4000, 2000, 16), (4800, 300, 36), (4096, 64, 8), (64 * 1200, 1200, 256), (6000, 3, 20), (3300, 100, 16)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_graphs_of_one_length(dtype, n, graphs, f, form):
    both_ways(n, f, form, graphs=graphs, xdt=dtype, odt=dtype)


@pytest.mark.parametrize("n", [1500, 5000])
def test_without_initial_states_and_gradients_of_the_last(n):
    both_ways(n, 24, "sigmoid", with_initial=False)
    both_ways(n, 24, "factor", ptr=offsets(n, 9), with_initial=False)


@pytest.mark.parametrize("n", [600, 4500])
def test_long_graphs_between_many_empty_ones(n):
    """Empty graphs first, last and between: their states go through."""
    cuts = [0] * 2000 + [n // 3] * 3000 + [n // 3 + 1] * 50 + [n] * 2500
    both_ways(n, 16, "sigmoid", ptr=torch.tensor([0] + cuts, device="cuda", dtype=torch.int32))


def test_no_rows_and_only_empty_graphs():
    x = torch.zeros((0, 8), device="cuda")
    initial = rand(5, 8).contiguous()
    for batch in (dict(graph_ptr=torch.zeros(6, device="cuda", dtype=torch.int64)), dict(graphs=5)):
        out, final, states = g.linear_recurrence(x, x, initial=initial, with_final=True, with_states=True, **batch)
        assert out.shape == (0, 8) and states.shape == (0, 8) and torch.equal(final, initial)
        dx, dgate, dinitial = g.linear_recurrence_backward(x, x, x, states, initial=initial, dfinal=initial * 2, **batch)
        assert dx.shape == dgate.shape == (0, 8) and torch.equal(dinitial, initial * 2)
    assert (g.linear_recurrence(x, x, with_final=True)[1] == 0).all()


@pytest.mark.parametrize("n", [1000, 5000])
def test_bad_values_stay_in_their_graph_and_column(n):
    """NaN and infinities in x, gates and states of one graph: other graphs and columns have the bits they had."""
    f, ptr = 24, offsets(n, 12, 3)
    x, gate, dout, initial, dfinal = rand(n, f, seed=1), gates("sigmoid", n, f, seed=2), rand(n, f, seed=3), rand(12, f, seed=4).contiguous(), rand(12, f, seed=5).contiguous()
    def both():
        out, final, states = g.linear_recurrence(x, gate, graph_ptr=ptr, initial=initial, with_final=True, with_states=True)
        return (out, final, *g.linear_recurrence_backward(dout, x, gate, states, graph_ptr=ptr, initial=initial, dfinal=dfinal))
    clean = both()
    size = (ptr[1:] - ptr[:-1]).tolist()
    b = max(range(1, 11), key=lambda i: size[i])
    r0, r1 = int(ptr[b]), int(ptr[b + 1])
    x[r0 + 1, 3], gate[r0 + 2, 5], x[r0, 7], initial[b, 9], dout[r1 - 1, 11], dfinal[b, 13] = (
        float("nan"), float("nan"), float("inf"), float("nan"), float("nan"), float("inf"))
    got = both()
    rows, cols = torch.ones(n, dtype=torch.bool, device="cuda"), torch.ones(f, dtype=torch.bool, device="cuda")
    rows[r0:r1] = False
    cols[[3, 5, 7, 9, 11, 13]] = False
    graphs = torch.arange(12, device="cuda") != b
    for was, now in zip(clean, got):
        keep = rows if was.shape[0] == n else graphs
        assert torch.equal(was[keep], now[keep]) and torch.equal(was[:, cols], now[:, cols])
    assert torch.isnan(got[0][r0 + 1:r1, 3]).all() and torch.isnan(got[0][r0 + 2:r1, 5]).all() and torch.isnan(got[0][r0:r1, 9]).all()
    assert not torch.isfinite(got[0][r0, 7]) and torch.isnan(got[2][r0:r1, 11]).all()


@pytest.mark.parametrize("n", [900, 9000])
def test_gates_at_their_ends(n):
    """Factors of 0 forget, of 1 sum up, of -1 alternate: with small whole numbers as x all sums are exact.  Sigmoid gates of +-infinity keep and replace."""
    x = torch.randint(-3, 4, (n, 4), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).float()
    gate = torch.tensor([0.0, 1.0, -1.0, 1.0], device="cuda").expand(n, 4).contiguous()
    gate[n // 2, 3] = 0.0
    sign = torch.where(torch.arange(n, device="cuda") % 2 == 0, 1.0, -1.0).double()
    xd = x.double()
    tail = xd[:, 3].clone()
    tail[:n // 2] = 0
    want = torch.stack([xd[:, 0], xd[:, 1].cumsum(0), (xd[:, 2] * sign).cumsum(0) * sign,
                        torch.where(torch.arange(n, device="cuda") < n // 2, xd[:, 3].cumsum(0), tail.cumsum(0))], 1)
    assert torch.equal(g.linear_recurrence(x, gate, "factor").double(), want)
    gate = torch.full((n, 4), float("inf"), device="cuda")
    gate[::3] = -float("inf")
    want = x[torch.arange(n, device="cuda") // 3 * 3]
    assert torch.equal(g.linear_recurrence(x, gate, "sigmoid"), want)


@pytest.mark.parametrize("n", [800, 12_000])
def test_growing_products_of_gates_on_a_state_of_zero(n):
    """Factors of 1.5 overflow as products; while the state is 0 and x is too, there is nothing to grow.  Then factors of 0.5."""
    x, gate = torch.zeros((n, 4), device="cuda"), torch.full((n, 4), 1.5, device="cuda")
    x[n - 20:] = 1.0
    gate[n - 20:] = 0.5
    got = g.linear_recurrence(x, gate, "factor")
    want = torch.zeros(n, device="cuda")
    want[n - 20:] = 2 - 0.5 ** torch.arange(20, device="cuda").float()
    assert torch.equal(got, want[:, None].expand(n, 4))


def test_long_memories():
    """A million rows whose gates keep all but 2^-20: the first state is still there at the end, and x builds up.  Relative to the closed form, 2 n u
    of the products' roundings (whose common gate, 1 - 2^-20, is exact)."""
    n, a = 1_000_000, 1 - 2.0 ** -20
    x = torch.full((n, 4), 2.0 ** -20, device="cuda")
    gate = torch.full((n, 4), a, device="cuda")
    out, final = g.linear_recurrence(x, gate, "factor", initial=torch.full((1, 4), 3.0, device="cuda"), with_final=True)
    want = 1 + 2 * a ** torch.arange(1, n + 1, dtype=torch.float64, device="cuda")
    assert float(((out.double() - want[:, None]) / want[:, None]).abs().max()) <= 2 * n * U
    assert torch.equal(final[0], out[-1])


def test_offsets_that_make_no_sense_touch_nothing_outside():
    for n in (700, 5000):
        x, gate = rand(n, 8, seed=1).contiguous(), rand(n, 8, seed=2).contiguous()
        for values in ([0, n + 100], [-5, n], [0, n // 2, n // 4, n], [0, 2 * n, -n, 3], [n, 0], [10, 20, 30]):
            ptr = torch.tensor(values, device="cuda", dtype=torch.int64)
            graphs = len(values) - 1
            guard = torch.full((n + 64, 8), 7.0, device="cuda")
            fin = torch.full((graphs + 64, 8), 7.0, device="cuda")
            out, _, states = g.linear_recurrence(x, gate, graph_ptr=ptr, out=guard[32:32 + n], final=fin[32:32 + graphs], with_states=True)
            g.linear_recurrence_backward(x, x.clone(), gate, states, graph_ptr=ptr)
            torch.cuda.synchronize()
            assert (guard[:32] == 7.0).all() and (guard[32 + n:] == 7.0).all() and (fin[:32] == 7.0).all() and (fin[32 + graphs:] == 7.0).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_single_tokens_go_on_from_a_prompt(dtype):
    """Prompts of different lengths in one call, then 20 tokens each with the states updated in place: what one call over all of them gives."""
    f, lengths, more = 40, [5, 300, 1, 64], 20
    total = [p + more for p in lengths]
    xs, gs = [rand(t, f, dtype, seed=i).contiguous() for i, t in enumerate(total)], [gates("sigmoid", t, f, dtype, seed=50 + i) for i, t in enumerate(total)]
    ptr = torch.tensor([0, *torch.tensor(lengths).cumsum(0).tolist()], device="cuda")
    cat = lambda ts, sl: torch.cat([t[sl(p)] for t, p in zip(ts, lengths)])      # noqa: E731
    _, state = g.linear_recurrence(cat(xs, lambda p: slice(0, p)), cat(gs, lambda p: slice(0, p)), graph_ptr=ptr, with_final=True)
    steps = []
    for k in range(more):
        out, same = g.linear_recurrence(cat(xs, lambda p: slice(p + k, p + k + 1)), cat(gs, lambda p: slice(p + k, p + k + 1)), graphs=4, initial=state, final=state)
        assert same is state
        steps.append(out)
    for i, p in enumerate(lengths):
        ref = reference(xs[i], gs[i], "sigmoid", [(0, total[i])], None)
        check(torch.stack([s[i] for s in steps]), [t[p:] for t in ref["out"]], "tokens", False)
        check(state[i:i + 1], ref["final"], "state", False)


def test_equal_calls_give_equal_bits_and_captured_ones_too():
    for n in (1200, 30_000):
        x, gate, dout, ptr = rand(n, 48, seed=1), gates("sigmoid", n, 48, seed=2), rand(n, 48, seed=3), offsets(n, 20)
        initial = rand(20, 48, seed=4).contiguous()

        def both(stream=None):
            out, final, states = g.linear_recurrence(x, gate, graph_ptr=ptr, initial=initial, with_final=True, with_states=True, stream=stream)
            return (out, final, *g.linear_recurrence_backward(dout, x, gate, states, graph_ptr=ptr, initial=initial, dfinal=final, stream=stream))

        want = [t.clone() for t in both()]
        assert all(torch.equal(a, b) for a, b in zip(both(), want))
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = both(side)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = both()
        for seed in (11, 12):
            x.copy_(rand(n, 48, seed=seed))
            want = [t.clone() for t in both()]
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("form", ["factor", "sigmoid"])
def test_gradients_agree_with_differences(form):
    """Central differences in 64 bits of the definition along a direction: a step of 2^-12 leaves 2^-24 times third derivatives, which grow with the cube of the
    rows that a state remembers (some ten here); 1e-3 of the sum of magnitudes covers them and the call's roundings."""
    n, f = 60, 6
    x, dout, v, vg = (rand(n, f, seed=i).contiguous() for i in (1, 2, 3, 4))
    gate, initial, dfinal, vi = gates(form, n, f, seed=5), *(rand(2, f, seed=i).contiguous() for i in (6, 7, 8))
    ptr = torch.tensor([0, 23, 60], device="cuda")
    _, _, states = g.linear_recurrence(x, gate, form, graph_ptr=ptr, initial=initial, with_final=True, with_states=True)
    grads = g.linear_recurrence_backward(dout, x, gate, states, form, graph_ptr=ptr, initial=initial, dfinal=dfinal)

    def value(step):
        ref = reference(x.double() + step * v.double(), gate.double() + step * vg.double(), form, [(0, 23), (23, 60)], initial.double() + step * vi.double())
        return (ref["out"][0] * dout.double()).sum() + (ref["final"][0] * dfinal.double()).sum()

    h = 2.0 ** -12
    terms = torch.cat([(a.double() * b.double()).flatten() for a, b in zip(grads, (v, vg, vi))])
    assert abs(float((value(h) - value(-h)) / (2 * h) - terms.sum())) <= 1e-3 * float(terms.abs().sum())


def test_refusals():
    x, ptr, state = rand(6, 8).contiguous(), torch.tensor([0, 2, 6], device="cuda"), torch.zeros((2, 8), device="cuda")
    one = torch.zeros((1, 8), device="cuda")
    for call, match in ((lambda: g.linear_recurrence(x, x.clone(), "tanh"), "form"), (lambda: g.linear_recurrence(x, x[:5].clone()), "gate"),
                        (lambda: g.linear_recurrence(x, x.clone(), graphs=4), "graphs of one length"), (lambda: g.linear_recurrence(x, x.clone(), graph_ptr=ptr, graphs=3), "graph_ptr"),
                        (lambda: g.linear_recurrence(x, x.clone(), graph_ptr=ptr.cpu()), "graph_ptr"), (lambda: g.linear_recurrence(x, x.clone(), graph_ptr=ptr[:1]), "graph_ptr"),
                        (lambda: g.linear_recurrence(x, x.clone(), initial=state), "initial"), (lambda: g.linear_recurrence(x, x.clone(), initial=one.double()), "initial"),
                        (lambda: g.linear_recurrence(x, x.clone(), out=x), "overlap"), (lambda: g.linear_recurrence(x.clone(), x, out=x), "overlap"),
                        (lambda: g.linear_recurrence(x, x.clone(), initial=one, final=one), "overlap"),
                        (lambda: g.linear_recurrence(x, x.clone(), final=x[:1]), "overlap"),
                        (lambda: g.linear_recurrence_backward(x.clone(), x, x.clone(), state), "states"),
                        (lambda: g.linear_recurrence_backward(x[:5].clone(), x, x.clone(), one), "dout"),
                        (lambda: g.linear_recurrence_backward(x.clone(), x, x.clone(), one, dfinal=state), "dfinal")):
        with pytest.raises(ValueError, match=match):
            call()
    with pytest.raises(TypeError):
        g.linear_recurrence(x, x.to(BF16))
    with pytest.raises(TypeError):
        g.linear_recurrence(x, x.clone(), graph_ptr=ptr.float())
    with pytest.raises(g.GnnfdError):
        g.linear_recurrence(rand(5000, 8), rand(5000, 8), scratch=torch.zeros(64, device="cuda"))
