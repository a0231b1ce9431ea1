"""Rotary positions against complex products in 64 bits.

Bounds (u = 2^-24): a cosine or sine is off by at most 3 u: the angle left after whole quarter turns (at most pi / 4) carries three roundings (to 32
bits, the constant pi / 2, the product), that is pi / 4 * 3 u * sqrt(1 / 2) = 1.7 u in the result, and the polynomial's last two steps add 1.2 u.  The angle itself has 2^-51 of
its size (two products in 64 bits).  Scaling, the products and their sum add 3 u; the result's type half a step."""
import math

import pytest

torch = pytest.importorskip("torch")

import paper_2104_03058_b200 as g  # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24


def rand(rows, cols, dtype=F32, ld=None, offset=0, seed=0):
    ld = ld or cols
    gen = torch.Generator(device="cuda").manual_seed(seed + 9)
    buf = torch.full((rows * ld + offset + 8,), float("nan"), device="cuda", dtype=dtype)
    view = buf[offset:offset + rows * ld].view(rows, ld)[:, :cols]
    view.copy_(torch.randn((rows, cols), generator=gen, device="cuda"))
    return view


def reference(x, freq, heads, dim, positions, interleaved, scale, inverse):
    """(value, bound)"""
    n, half = x.shape[0], freq.numel()
    x = x[:, :heads * dim].double().reshape(n, heads, dim)
    p = torch.arange(n, device="cuda").double() if positions is None else positions.double()
    angle = (p[:, None] * freq)[:, None, :]
    cos, sin = scale * torch.cos(angle), scale * torch.sin(angle) * (-1 if inverse else 1)
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
    y, bound = x.clone(), torch.zeros_like(x)
    y[:, :, a], y[:, :, b] = x[:, :, a] * cos - x[:, :, b] * sin, x[:, :, a] * sin + x[:, :, b] * cos
    size = (x[:, :, a].abs() + x[:, :, b].abs()) * abs(scale) * (6 * U + 2.0 ** -51 * angle.abs())
    bound[:, :, a] = bound[:, :, b] = size
    return y.reshape(n, -1), bound.reshape(n, -1)


def check(got, want, bound):
    half = torch.finfo(got.dtype).eps / 2
    err = (got.double() - want).abs()
    tol = bound + half * want.abs()
    assert got.shape == want.shape and (err <= tol).all(), "%d of %d off, worst %.3g of its bound" % (
        int((~(err <= tol)).sum()), err.numel(), float((err / tol.clamp_min(1e-300)).nan_to_num(1e9).max()))


def run(n, heads, dim, part, xdt=F32, odt=F32, ld=None, offset=0, interleaved=False, scale=1.0, positions=None, freq=None, seed=0):
    f = heads * dim
    x = rand(n, f, xdt, ld, offset, seed)
    freq = g.rotary_frequencies(part) if freq is None else freq
    for inverse in (False, True):
        want, bound = reference(x, freq, heads, dim, positions, interleaved, scale, inverse)
        args = dict(positions=positions, interleaved=interleaved, scale=scale, inverse=inverse)
        check(g.rotary(x, freq, heads, dim, out_dtype=odt, **args), want, bound)
        guard = torch.full((n * (f + 3) + offset,), 7.0, device="cuda", dtype=odt)
        buf = guard[offset:].view(n, f + 3)
        got = g.rotary(x, freq, heads, dim, out=buf[:, :f], **args)
        check(got, want, bound)
        assert (buf[:, f:] == 7.0).all() and (guard[:offset] == 7.0).all()
        y = _copy(x)                                            # in place, the padding being NaN
        assert g.rotary(y, freq, heads, dim, out=y, **args) is y
        assert torch.equal(y, g.rotary(x, freq, heads, dim, out_dtype=xdt, **args))


def _copy(x):
    ld = x.stride(0) if x.shape[0] > 1 else x.shape[1]
    buf = torch.full((x.shape[0], ld), float("nan"), device="cuda", dtype=x.dtype)
    buf[:, :x.shape[1]] = x
    return buf[:, :x.shape[1]]


@pytest.mark.parametrize("odt", [F32, BF16])
@pytest.mark.parametrize("xdt", [F32, BF16])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("n,heads,dim,part,ld,offset", [
    (1, 1, 2, 2, None, 0), (5, 1, 2, 2, 3, 1), (300, 2, 8, 8, None, 0), (77, 3, 10, 6, None, 0), (64, 4, 16, 8, 70, 0), (33, 5, 7, 4, None, 0), (129, 2, 7, 2, 15, 3),
    (1000, 8, 64, 64, None, 0), (11, 12, 80, 40, None, 2), (3, 40, 128, 128, None, 0), (2, 1, 4096, 4096, None, 0), (2, 3, 5000, 4090, None, 0), (4001, 1, 6, 4, None, 0)])
def test_sizes_and_layouts(n, heads, dim, part, ld, offset, interleaved, xdt, odt):
    run(n, heads, dim, part, xdt, odt, ld, offset, interleaved, scale=1.25)


@pytest.mark.parametrize("itype", [torch.int32, torch.int64])
def test_far_and_negative_positions(itype):
    """Up to 2^31 - 1 (and 2^40): a rounding of the angle to 32 bits would be off by many turns."""
    p = torch.tensor([0, 1, -1, 4095, 65_537, 999_999, -1_000_000, 123_456_789, 2**31 - 1, -2**31] + ([2**40 + 1, -2**40] if itype == torch.int64 else []),
                     device="cuda", dtype=itype)
    run(p.numel(), 2, 64, 64, positions=p)
    run(p.numel(), 2, 64, 64, positions=p, freq=g.rotary_frequencies(64, scaling="ramp", factor=32.0, length=4096))


def test_angles_without_meaning_stay_finite():
    """Positions up to the type's ends: x comes back no longer than it was (cosine and sine within 3 u of a point of the circle)."""
    p = torch.tensor([2**63 - 1, -2**63, 2**55 + 1, -2**52 - 1, 2**51], device="cuda")
    x = rand(5, 64)
    for interleaved in (False, True):
        y = g.rotary(x, g.rotary_frequencies(64), 1, 64, p, interleaved)
        assert torch.isfinite(y).all() and (y.norm(dim=1) <= 1.01 * x.norm(dim=1)).all()


@pytest.mark.parametrize("heads,dim,part", [(1, 100_000, 2), (3, 300_000, 4), (1, 1 << 20, 4096), (1 << 18, 4, 2)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rows_of_many_columns(heads, dim, part, interleaved):
    run(3, heads, dim, part, interleaved=interleaved)
    run(700 if heads == 1 and dim == 100_000 else 2, heads, dim, part, BF16, BF16, interleaved=interleaved)


def test_quarter_turns_land_on_the_axes():
    """A frequency of pi / 2: positions are quarter turns (64 bits of pi are off by 1e-16 a turn)."""
    freq = torch.full((1,), math.pi / 2, dtype=torch.float64, device="cuda")
    p = torch.arange(-9, 10, device="cuda")
    x = torch.tensor([[1.0, 0.0]], device="cuda").expand(19, 2).contiguous()
    got = g.rotary(x, freq, 1, 2, p)
    want = torch.tensor([[(1, 0), (0, 1), (-1, 0), (0, -1)][int(k) % 4] for k in p], device="cuda", dtype=F32)
    assert float((got - want).abs().max()) < 1e-14


def test_there_and_back():
    x = rand(500, 256)
    freq = g.rotary_frequencies(32)
    p = torch.randint(1 << 20, (500,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    back = g.rotary(g.rotary(x, freq, 8, 32, p), freq, 8, 32, p, inverse=True)
    assert float((back - x).abs().max()) <= 24 * U * float(x.abs().max())          # twice 6 u (|u| + |v|)


def test_scores_depend_on_distances_alone():
    q, k = rand(1, 64, seed=1), rand(1, 64, seed=2)
    freq = g.rotary_frequencies(64)
    at = lambda t, p: g.rotary(t, freq, 1, 64, torch.tensor([p], device="cuda")).double()      # noqa: E731
    scores = [float((at(q, p + 17) * at(k, p)).sum()) for p in (0, 5, 1000, 1_000_000)]
    size = float((q.abs() * k.abs()).sum()) + float(q.abs().sum() * k.abs().max())
    assert max(scores) - min(scores) <= 4 * 12 * U * size


def test_queries_and_keys_of_a_joint_projection():
    """16 of 24 heads of a matrix of queries, keys and values, in place: the values stay as they are, bit for bit."""
    qkv = rand(700, 384, BF16).contiguous()
    before = qkv.clone()
    freq = g.rotary_frequencies(16)
    want, bound = reference(qkv, freq, 16, 16, None, False, 1.0, False)
    g.rotary(qkv, freq, 16, 16, out=qkv)
    check(qkv[:, :256], want, bound)
    assert torch.equal(qkv[:, 256:], before[:, 256:])


@pytest.mark.parametrize("interleaved", [False, True])
def test_bad_values_stay_in_their_pair(interleaved):
    x = rand(20, 64).contiguous()
    freq = g.rotary_frequencies(16)
    clean = g.rotary(x, freq, 2, 32, interleaved=interleaved)
    x[7, 3] = float("nan")
    x[9, 20] = float("inf")                                      # (a column that does not turn)
    got = g.rotary(x, freq, 2, 32, interleaved=interleaved)
    changed = (got != clean).nonzero().tolist()
    assert changed == [[7, 2], [7, 3], [9, 20]] if interleaved else changed == [[7, 3], [7, 11], [9, 20]]


def test_no_rows_and_captured_calls():
    freq = g.rotary_frequencies(8)
    assert g.rotary(torch.zeros((0, 16), device="cuda"), freq, 2, 8).shape == (0, 16)
    x, p = rand(900, 64), torch.arange(900, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = g.rotary(x, freq, 8, 8, p)
    for shift in (3, 100_000):
        p += shift
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, g.rotary(x, freq, 8, 8, p))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    z = g.rotary(x, freq, 8, 8, p, stream=side)
    side.synchronize()
    assert torch.equal(y, z)


def test_refusals():
    x, freq = rand(6, 32), g.rotary_frequencies(8)
    for call, match in ((lambda: g.rotary(x, freq.float(), 2, 16), "freq"), (lambda: g.rotary(x, freq.cpu(), 2, 16), "freq"),
                        (lambda: g.rotary(x, g.rotary_frequencies(18), 2, 16), "frequencies"), (lambda: g.rotary(x, freq[:0], 2, 16), "frequencies"),
                        (lambda: g.rotary(x, freq, 3, 16), "x must be"), (lambda: g.rotary(x, freq, 2, 16, torch.zeros(5, device="cuda", dtype=torch.int32)), "positions"),
                        (lambda: g.rotary(x, freq, 2, 16, torch.zeros(6, dtype=torch.int32)), "positions"),
                        (lambda: g.rotary(x, freq, 1, 16, out=x[:, 8:24]), "overlap")):
        with pytest.raises(ValueError, match=match):
            call()
    with pytest.raises(TypeError):
        g.rotary(x, freq, 2, 16, torch.zeros(6, device="cuda"))
    with pytest.raises(g.GnnfdError):
        g.rotary(x, freq, 0, 16)
