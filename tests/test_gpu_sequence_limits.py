"""Layer norm, rotary positions and the linear recurrence at the limits of what they take: operands in one another's memory, values and lengths where
roundings add up.  References and bounds are those of the operators' own tests, or derived where they are used."""
import pytest

torch = pytest.importorskip("torch")

import paper_2104_03058_b200 as g  # noqa: E402
import test_gpu_recurrence as scan  # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24


# ---------------------------------------------------------------- recurrence

@pytest.mark.parametrize("n", [300, 6000])
def test_a_sequence_in_stretches_through_one_buffer(n):
    """The last row of a stretch is the next one's first state: a copy of it gives what one call over all rows gives, the row itself is refused."""
    x, gate = scan.rand(3 * n, 24, seed=1).contiguous(), scan.gates("sigmoid", 3 * n, 24, seed=2)
    ref = scan.reference(x, gate, "sigmoid", [(0, 3 * n)], None)
    buf, state, rows = torch.zeros((n, 24), device="cuda"), None, []
    for k in range(3):
        part = slice(k * n, (k + 1) * n)
        if state is not None:
            with pytest.raises(ValueError, match="initial and out overlap"):
                g.linear_recurrence(x[part], gate[part], initial=buf[-1:], out=buf)
        g.linear_recurrence(x[part], gate[part], initial=state, out=buf)
        state = buf[-1:].clone()
        rows.append(buf.clone())
    scan.check(torch.cat(rows), ref["out"], "out")


def test_single_tokens_in_place_of_their_states():
    for n, f in ((1, 7), (300, 24), (5000, 41)):
        x, gate, state = scan.rand(n, f, seed=1).contiguous(), scan.gates("sigmoid", n, f, seed=2), scan.rand(n, f, seed=3).contiguous()
        want = g.linear_recurrence(x, gate, graphs=n, initial=state)
        assert g.linear_recurrence(x, gate, graphs=n, initial=state, out=state) is state and torch.equal(state, want)


@pytest.mark.parametrize("last", [0, 3, 100, 9_000])
def test_many_rows_behind_the_last_offset(last):
    """Most blocks have no rows, but have sent for some before they know: nothing of that shows in their rows, nor in what comes after on the stream."""
    n, f = 20_000, 64
    x, dout = scan.rand(n, f, seed=1).contiguous(), scan.rand(n, f, seed=2).contiguous()
    want = g.layer_norm(x)
    for form in ("factor", "sigmoid"):
        gate = scan.gates(form, n, f, seed=3)
        ptr = torch.tensor([0, last // 3, last], device="cuda")
        ref = scan.reference(x, gate, form, scan.bounds_of(n, 2, ptr), None, dout)
        for dtype in (F32, BF16):
            ins = [t.to(dtype) for t in (x, gate, dout)]
            if dtype == BF16:
                ref = scan.reference(ins[0], ins[1], form, scan.bounds_of(n, 2, ptr), None, ins[2])
            out = torch.full((n, f), 7.0, device="cuda")
            results = []
            for _ in range(3):
                _, final, states = g.linear_recurrence(ins[0], ins[1], form, graph_ptr=ptr, out=out, with_final=True, with_states=True)
                results.append(g.layer_norm(x))
            dx, dgate, _ = g.linear_recurrence_backward(ins[2], ins[0], ins[1], states, form, graph_ptr=ptr)
            assert all(torch.equal(r, want) for r in results) and (out[last:] == 7.0).all()
            scan.check(out[:last], [t[:last] for t in ref["out"]], "out")
            scan.check(final, ref["final"], "final")
            scan.check(dx[:last], [t[:last] for t in ref["dx"]], "dx")
            scan.check(dgate[:last], [t[:last] for t in ref["dgate"]], "dgate")


@pytest.mark.parametrize("how", ["length", "offsets"])
@pytest.mark.parametrize("n,f", [(3, 5), (900, 64), (900, 33), (9_000, 64), (9_000, 31), (40_000, 512)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_sigmoid_gates_weights_at_any_size(dtype, n, f, how):
    """Graphs of one row: a is what is left of a state of 1 where x is 0, 1 - a what comes of x = 1 where there is no state, a of a gradient of 1 behind the state, 1 - a
    in front of x and a (1 - a) in front of the gate.  Relative to themselves: 4 u for the exponential, 1 u for the product that mends its argument, 0.05 u |gate| for log 2
    in 32 bits, 1 u for adding 1, 3 u for the reciprocal, 1 u for a product; gates up to 69, so that a is above 2^-100.  dgate has two such weights and three products."""
    gen = torch.Generator(device="cuda").manual_seed(n + f)
    gate = ((torch.rand((n, f), generator=gen, device="cuda") - 0.5) * 138).to(dtype)
    batch = dict(graphs=n) if how == "length" else dict(graph_ptr=torch.arange(n + 1, device="cuda"))
    zero, one, state = torch.zeros_like(gate), torch.ones_like(gate), torch.ones((n, f), device="cuda")
    a, rest = torch.sigmoid(gate.double()), torch.sigmoid(-gate.double())
    bound = (0.05 * gate.double().abs() + 10) * U

    def near(got, want, times=1.0, more=0.0):
        assert (((got.double() / want) - 1).abs() <= times * bound + more * U).all(), float(((got.double() / want - 1).abs() / U).max())

    out, _, states = g.linear_recurrence(zero, gate, initial=state, with_final=True, with_states=True, **batch)
    near(out, a)
    near(g.linear_recurrence(one, gate, **batch), rest)
    dx, dgate, dinitial = g.linear_recurrence_backward(one, zero, gate, states, initial=state, **batch)
    near(dx, rest)
    near(dinitial, a)
    near(dgate, a * rest, 2.0, 3.0)


@pytest.mark.parametrize("n,f", [(2_000_003, 4), (1_500_000, 5), (1_000_001, 128)])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_exact_sums_over_millions_of_rows(sign, n, f):
    """Factors of 1 (or -1) add up (or alternate): of small whole numbers, one in ten not 0, every sum and every product of two is below 2^24 and thus exact, whatever
    the joints, of which there are some thousand tiles of chunks."""
    gen = torch.Generator(device="cuda").manual_seed(n)
    some = lambda: torch.randint(-10, 11, (n, f), generator=gen, device="cuda", dtype=torch.int8)      # noqa: E731
    x, dout = ((t == 9).float() - (t == -9).float() for t in (some(), some()))
    ptr = torch.tensor([0, n // 3, n // 3, n - 7, n], device="cuda")
    initial, dfinal = torch.full((4, f), 5.0, device="cuda"), torch.full((4, f), -3.0, device="cuda")
    turn = torch.where(torch.arange(n, device="cuda") % 2 == 0, 1, int(sign))[:, None].double()
    h, before, total = (torch.empty((n, f), device="cuda") for _ in range(3))
    final, dinitial = [], []
    for b, (r0, r1) in enumerate(scan.bounds_of(n, 4, ptr)):
        w, first = turn[r0:r1], initial[b].double()
        if r0 == r1:
            final.append(initial[b]), dinitial.append(dfinal[b])
            continue
        # h[t] w[t] = first w[r0] sign + the sum of x w so far; the gradients the same from the end
        start = first * w[0] * sign
        sums = start + (x[r0:r1].double() * w).cumsum(0)
        h[r0:r1] = (sums * w).float()
        before[r0], before[r0 + 1:r1] = initial[b], h[r0:r1 - 1]
        back = dfinal[b].double() * w[-1] + (dout[r0:r1].double() * w).flip(0).cumsum(0).flip(0)
        total[r0:r1] = (back * w).float()
        final.append(h[r1 - 1]), dinitial.append(sign * total[r0])
    out, last, states = g.linear_recurrence(x, torch.full_like(x, sign), "factor", graph_ptr=ptr, initial=initial, with_final=True, with_states=True)
    assert torch.equal(out, h) and torch.equal(last, torch.stack(final))
    dx, dgate, dfirst = g.linear_recurrence_backward(dout, x, torch.full_like(x, sign), states, "factor", graph_ptr=ptr, initial=initial, dfinal=dfinal)
    assert torch.equal(dx, total) and torch.equal(dgate, total * before) and torch.equal(dfirst, torch.stack(dinitial))
    assert float(total.abs().max()) * float(before.abs().max()) < 2.0 ** 24


@pytest.mark.parametrize("form", ["factor", "sigmoid"])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,graphs,f", [(1_200_000, 1000, 16), (60_000, 60, 256), (150_000, 150, 41)])
def test_longer_batches(n, graphs, f, dtype, form):
    """Tiles by the thousand going back, and threads of eight bf16 columns."""
    length = n // graphs
    jitter = torch.randint(-length // 2, length // 2, (graphs - 1,), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    ptr = torch.cat([jitter.new_zeros(1), torch.arange(1, graphs, device="cuda") * length + jitter, jitter.new_full((1,), n)])
    scan.both_ways(n, f, form, ptr=ptr, xdt=dtype, odt=dtype)


# ---------------------------------------------------------------- layer norm

@pytest.mark.parametrize("xdt", [F32, BF16])
@pytest.mark.parametrize("f", [1, 3, 41, 96, 100, 600, 602, 1000, 4100, 8191])
def test_rows_of_equal_values(f, xdt):
    """A row's mean is a sum of f values (off by 20 u of itself as in the norm's own tests); the distances from it are exact, and their mean, another such sum, is taken off:
    440 u^2 |value| are left (the product with rstd adds one rounding of 20 u), times rstd = eps^-1/2 = 317.  The mean is then the value itself, so that the gradient's
    xhat, dw and the part of dx with xhat are exactly zero: dx = rstd (dout - mean(dout)), rstd within 8 u: (20 u)^2 of the value in
    the variance, less than u of eps for values below 1e4 and 10 u for 12345.678 (half of that in rstd), and 4 u for adding and the root."""
    eps, n = 1e-5, 70
    bias = torch.linspace(-1.0, 1.0, f, device="cuda")
    dout = torch.randn((n, f), generator=torch.Generator(device="cuda").manual_seed(f), device="cuda").to(xdt)
    for value in (0.1, -10.1, 1000.1, 12345.678):
        x = torch.full((n, f), value, device="cuda", dtype=xdt)
        value = abs(float(x[0, 0]))
        out, mean, rstd = g.layer_norm(x, None, bias, eps, with_stats=True)
        assert ((out - bias).abs() <= 317 * 440 * U * U * value + 2 * U * bias.abs()).all(), (value, float((out - bias).abs().max()))
        assert (mean == x[:, 0].float()).all()
        assert ((rstd.double() * eps ** 0.5 - 1).abs() <= 10 * U).all()
        dx, dw, db = g.layer_norm_backward(dout, x, mean, rstd)
        do = dout.double()
        assert (dw == 0).all()
        size = do.abs() + do.abs().mean(1, keepdim=True)
        assert ((dx.double() - eps ** -0.5 * (do - do.mean(1, keepdim=True))).abs() <= 317 * (10 + 24) * U * size).all()
    # squares of the rounded distances beyond the type's range
    assert torch.equal(g.layer_norm(torch.full((n, f), 3e30, device="cuda", dtype=xdt), None, bias), bias.expand(n, f))


@pytest.mark.parametrize("f", [96, 602, 4100])
def test_rows_whose_spread_is_below_the_means_roundings(f):
    """Values 4096 + k 2^-11, k of -8 to 8, all exact in fp32: the mean as a sum is off by more than the spread.  Distances from it are exact or off by a rounding
    of themselves, sums of them and of their squares by 20 and 24 roundings of a distance's size, which is up to 20 u 4096 = 2^-7.7 beside a spread of 2^-8.6: three roundings in place
    of one, (60 + 40) u of xhat's size and as much for the part of rstd."""
    k = torch.randint(-8, 9, (300, f), generator=torch.Generator(device="cuda").manual_seed(f), device="cuda")
    x = 4096 + k.double() * 2.0 ** -11
    out = g.layer_norm(x.float(), eps=1e-9).double()
    off = x - x.mean(1, keepdim=True)
    want = off / ((off ** 2).mean(1, keepdim=True) + 1e-9).sqrt()
    assert float((out - want).abs().max()) <= 200 * U * float(want.abs().max())


def test_sums_over_many_rows():
    """dw and db over 240,000 rows of 1024 columns, 203 for each lane.  Sixteen rows are added up in fp32: a rounding of a sum of k terms of size s is at most evenly spread
    over u sqrt(k) s, 0.58 of that in the root mean square, and those of 2 to 16 terms together 0.58 sqrt(135) u s = 1.7 u of the sixteen terms' own size, 4 s; terms of
    either sign keep that proportion to the last sum.  A block's sum and the result are rounded once more (0.58 u each): 1.9 u in all for db.  The
    terms of dw have errors of their own, 1.3 u: a rounding of the distance, of rstd, of xhat.  (All rows of a lane in fp32: 0.58 sqrt(203 / 2) = 5.8 u at
    most and 4 u as roundings are usually spread.)"""
    n, f = 240_000, 1024
    x, dout = (torch.empty((n, f), device="cuda") for _ in range(2))
    gen = torch.Generator(device="cuda").manual_seed(4)
    x.normal_(generator=gen), dout.normal_(generator=gen)
    _, mean, rstd = g.layer_norm(x, out_dtype=BF16, with_stats=True)
    _, dw, db = g.layer_norm_backward(dout, x, mean, rstd, out_dtype=BF16)
    want = torch.zeros((2, f), dtype=torch.float64, device="cuda")
    for k in range(0, n, 20_000):
        xs, ds = x[k:k + 20_000].double(), dout[k:k + 20_000].double()
        off = xs - xs.mean(1, keepdim=True)
        want[0] += (ds * off / ((off ** 2).mean(1, keepdim=True) + 1e-5).sqrt()).sum(0)
        want[1] += ds.sum(0)
    for got, ref, most in ((dw, want[0], 2.5), (db, want[1], 2.0)):
        assert float((got.double() - ref).pow(2).mean().sqrt()) <= most * U * float(ref.pow(2).mean().sqrt())


@pytest.mark.parametrize("f", [8, 24, 40, 1032])
def test_equal_values_as_large_as_they_come(f):
    """Rows of 2^120 in lanes that have places for more columns than there are: mean * rstd is beyond the type's range, xhat is 0 all the same.  f x 2^120 has few bits, so the sums are exact and their
    product with 1 / f, half a unit off at most, is rounded to 2^120.  1032 x 2^120 is above 2^128, no fp32 number any more: NaN."""
    x = torch.full((50, f), 2.0 ** 120, device="cuda")
    dout = torch.randn((50, f), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    _, mean, rstd = g.layer_norm(x, with_stats=True)
    dx, dw, db = g.layer_norm_backward(dout, x, mean, rstd)
    if f * 2.0 ** 120 >= 2.0 ** 128:
        assert torch.isnan(g.layer_norm(x)).all() and torch.isnan(dx).all()
        return
    do = dout.double()
    want = rstd.double()[:, None] * (do - do.mean(1, keepdim=True))
    assert ((dx.double() - want).abs() <= 24 * U * rstd.double()[:, None] * (do.abs() + do.abs().mean(1, keepdim=True))).all()
    assert (dw == 0).all() and torch.isfinite(db).all() and (rstd > 300).all()
