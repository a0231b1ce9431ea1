"""Layer norm, rotary positions and the linear recurrence beside the attention and the transform: a layer and its gradient, rows far apart, narrower
widths than the operands', two streams, two threads and two captured graphs at once.  References and bounds are those of the operators' own tests."""
import threading

import pytest

torch = pytest.importorskip("torch")

import paper_2104_03058_b200 as g  # noqa: E402
import test_gpu_attention as att  # noqa: E402
import test_gpu_layer_norm as norm  # noqa: E402
import test_gpu_recurrence as scan  # noqa: E402
import test_gpu_rotary as rot  # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24


def product(x, w_t, mode):
    """(x w_t^T in 64 bits, bound): the transform's own bar, 1e-5 of the sum of magnitudes and 1e-6"""
    x, w = x.double(), w_t.double()
    return x @ w.t(), 1e-5 * (x.abs() @ w.abs().t()) + 1e-6


def near(got, ref):
    want, bound = ref
    tol = bound + torch.finfo(got.dtype).eps / 2 * want.abs()
    assert ((got.double() - want).abs() <= tol).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_layer_and_its_gradient(dtype):
    """Documents of different lengths (one of them empty, one of a single token): norm, queries, keys and values from one transform, their positions, attention
    of each token over those up to itself; then norm, transform and the recurrence; and all the way back.  Every stage is checked on what the stage before it gave."""
    heads, dim = 4, 16
    f, sizes = heads * dim, torch.tensor([1, 0, 40, 133, 7, 65], device="cuda")
    ptr = torch.cat([sizes.new_zeros(1), sizes.cumsum(0)])
    n, docs = int(ptr[-1]), sizes.numel()
    doc = torch.repeat_interleave(torch.arange(docs, device="cuda"), sizes)
    positions = torch.arange(n, device="cuda") - ptr[doc]
    pairs = torch.nonzero((doc[:, None] == doc[None, :]) & (positions[None, :] <= positions[:, None]))
    src, dst = pairs[:, 1].int().contiguous(), pairs[:, 0].int().contiguous()
    gen = torch.Generator(device="cuda").manual_seed(5)
    randn = lambda *shape: torch.randn(shape, generator=gen, device="cuda")      # noqa: E731
    x0 = randn(n, f).to(dtype)
    w_in, w_scan = (randn(3 * f, f) * f ** -0.5).to(dtype), (randn(2 * f, f) * f ** -0.5).to(dtype)
    weight, shift = 1 + 0.1 * randn(f), 0.1 * randn(f)
    freq = g.rotary_frequencies(dim, scaling="ramp", factor=4.0, length=64)

    y0, mean0, rstd0 = g.layer_norm(x0, weight, shift, out_dtype=dtype, with_stats=True)
    qkv = g.combine(y0, w_in, out_dtype=dtype, mode="fp32")
    near(qkv, product(y0, w_in, "fp32"))
    turned = qkv.clone()
    g.rotary(turned, freq, 2 * heads, dim, positions, out=turned)
    want, bound = rot.reference(qkv, freq, 2 * heads, dim, positions, False, 1.0, False)
    rot.check(turned[:, :2 * f], want, bound)
    assert torch.equal(turned[:, 2 * f:], qkv[:, 2 * f:])
    p = att.Problem(n, src, dst, heads, dim, dtype)
    p.q, p.k, p.v = turned[:, :f], turned[:, f:2 * f], turned[:, 2 * f:]
    a0, lse = p.forward(with_lse=True, out_dtype=dtype)
    y1, mean1, rstd1 = g.layer_norm(a0, weight, shift, out_dtype=dtype, with_stats=True)
    xg = g.combine(y1, w_scan, out_dtype=dtype, mode="fp32")
    near(xg, product(y1, w_scan, "fp32"))
    initial = randn(docs, f)
    x, gate = xg[:, :f], xg[:, f:]
    out, final, states = g.linear_recurrence(x, gate, graph_ptr=ptr, initial=initial, out_dtype=dtype, with_final=True, with_states=True)

    dout, dfinal = randn(n, f).to(dtype), randn(docs, f)
    dx, dgate, dinitial = g.linear_recurrence_backward(dout, x, gate, states, graph_ptr=ptr, initial=initial, dfinal=dfinal, out_dtype=dtype)
    ref = scan.reference(x, gate, "sigmoid", scan.bounds_of(n, docs, ptr), initial, dout, dfinal)
    for name, got in (("out", out), ("final", final), ("dx", dx), ("dgate", dgate), ("dinitial", dinitial)):
        scan.check(got, ref[name], name)
    dxg = torch.cat([dx, dgate], dim=1)
    back = w_scan.t().contiguous()
    dy1 = g.combine(dxg, back, out_dtype=dtype, mode="fp32")
    near(dy1, product(dxg, back, "fp32"))
    da0, dw1, db1 = g.layer_norm_backward(dy1, a0, mean1, rstd1, weight, out_dtype=dtype)
    ref = norm.reference(a0, weight, shift, dy1)
    for name, got in (("out", y1), ("dx", da0), ("dw", dw1), ("db", db1)):
        norm.check(got, ref[name], name, False)
    p.dout = da0
    ref = p.reference()
    grads = p.backward(lse, out_dtype=dtype)
    for name, got in zip(("out", "dq", "dk", "dv"), (a0, *grads)):
        att.check(got, ref[name], name)
    dqkv = torch.cat(grads[:3], dim=1)
    before = dqkv.clone()
    g.rotary(dqkv, freq, 2 * heads, dim, positions, inverse=True, out=dqkv)
    want, bound = rot.reference(before, freq, 2 * heads, dim, positions, False, 1.0, True)
    rot.check(dqkv[:, :2 * f], want, bound)
    back = w_in.t().contiguous()
    dy0 = g.combine(dqkv, back, out_dtype=dtype, mode="fp32")
    near(dy0, product(dqkv, back, "fp32"))
    dx0, dw0, db0 = g.layer_norm_backward(dy0, x0, mean0, rstd0, weight, out_dtype=dtype)
    ref = norm.reference(x0, weight, shift, dy0)
    for name, got in (("out", y0), ("dx", dx0), ("dw", dw0), ("db", db0)):
        norm.check(got, ref[name], name, False)


def far_rows(rows, cols, pitch, dtype, seed, mean=0.0):
    view = torch.zeros(rows * pitch, device="cuda", dtype=dtype).view(rows, pitch)[:, :cols]
    view.copy_(torch.randn((rows, cols), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda") + mean)
    return view


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_more_than_four_gigabytes_apart(dtype):
    pitch, n, f = 1 << 20, 2500, 24                                    # 2500 rows of 1 Mi elements: 5 to 10 GB a matrix
    x, dout = far_rows(n, f, pitch, dtype, 0), far_rows(n, f, pitch, dtype, 1)
    out = torch.zeros(n * pitch, device="cuda", dtype=dtype).view(n, pitch)[:, :f]
    ref = norm.reference(x, None, None, dout)
    _, mean, rstd = g.layer_norm(x, out=out, with_stats=True)
    norm.check(out, ref["out"], "out")
    g.layer_norm_backward(dout, x, mean, rstd, out=out)
    norm.check(out, ref["dx"], "dx")
    freq = g.rotary_frequencies(8)
    g.rotary(x, freq, 3, 8, out=out)
    rot.check(out, *rot.reference(x, freq, 3, 8, None, False, 1.0, False))
    gate = far_rows(n, f, pitch, dtype, 2, 1.0)
    ref = scan.reference(x, gate, "sigmoid", [(0, n)], None, dout)
    _, states = g.linear_recurrence(x, gate, out=out, with_states=True)
    scan.check(out, ref["out"], "out")
    dx, dgate, _ = g.linear_recurrence_backward(dout, x, gate, states)
    scan.check(dx, ref["dx"], "dx")
    scan.check(dgate, ref["dgate"], "dgate")


def test_widths_narrower_than_the_operands():
    x, dout, gate = scan.rand(300, 20), scan.rand(300, 20, seed=1), scan.rand(300, 20, seed=2)
    for call, want in ((lambda out: g.layer_norm(x, f=9, out=out), norm.reference(x[:, :9], None, None)["out"]),
                       (lambda out: g.linear_recurrence(x, gate, f=9, out=out), scan.reference(x[:, :9], gate[:, :9], "sigmoid", [(0, 300)], None)["out"]),
                       (lambda out: g.rotary(x, g.rotary_frequencies(4), 2, 4, out=out), None)):
        out = torch.full((300, 20), 4.0, device="cuda")
        call(out)
        if want is None:
            rot.check(out[:, :8], *rot.reference(x, g.rotary_frequencies(4), 2, 4, None, False, 1.0, False))
            assert (out[:, 8:] == 4.0).all()
        else:
            scan.check(out[:, :9], want, "out", False)
            assert (out[:, 9:] == 4.0).all()


class Work:
    """One training pass through all three, of its own sizes and inputs."""

    def __init__(self, n, f, seed):
        self.x, self.dout, self.gate = (scan.rand(n, f, seed=seed + i).contiguous() for i in (1, 2, 3))
        self.freq, self.ptr, self.f = g.rotary_frequencies(f // 2), scan.offsets(n, 17, seed), f

    def run(self, stream=None):
        y, mean, rstd = g.layer_norm(self.x, with_stats=True, stream=stream)
        z = g.rotary(y, self.freq, 2, self.f // 2, stream=stream)
        out, final, states = g.linear_recurrence(z, self.gate, graph_ptr=self.ptr, with_final=True, with_states=True, stream=stream)
        dz, dgate, _ = g.linear_recurrence_backward(self.dout, z, self.gate, states, graph_ptr=self.ptr, stream=stream)
        dy = g.rotary(dz, self.freq, 2, self.f // 2, inverse=True, stream=stream)
        return (out, final, dgate, *g.layer_norm_backward(dy, self.x, mean, rstd, stream=stream))


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def test_two_streams_at_once():
    works = [Work(20_000, 64, 1), Work(33_000, 36, 50)]
    want = [w.run() for w in works]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in works], [[], []]
    for _ in range(4):
        for i, w in enumerate(works):
            got[i].append(w.run(streams[i]))
    torch.cuda.synchronize()
    assert all(same(res, want[i]) for i in range(2) for res in got[i])


def test_two_threads_at_once():
    works = [Work(9_000, 1024, 1), Work(1_500, 36, 50), Work(30_000, 40, 90)]
    want = [w.run() for w in works]
    torch.cuda.synchronize()
    failed = []

    def loop(i):
        stream = torch.cuda.Stream()
        try:
            for _ in range(8):
                res = works[i].run(stream)
                stream.synchronize()
                if not same(res, want[i]):
                    failed.append(i)
        except Exception as err:                          # a thread's exception would be lost
            failed.append(err)

    threads = [threading.Thread(target=loop, args=(i,)) for i in range(3)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed


def test_two_captured_graphs_in_turn():
    works = [Work(12_000, 64, 1), Work(7_001, 41 * 4, 50)]
    graphs, got = [], []
    for w in works:
        w.run()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            got.append(w.run())
    for seed in (7, 8):
        for w in works:
            w.x.copy_(scan.rand(*w.x.shape, seed=seed))
        want = [w.run() for w in works]
        for i in (1, 0, 1):
            graphs[i].replay()
        torch.cuda.synchronize()
        assert all(same(got[i], want[i]) for i in range(2))


def test_the_largest_numbers_of_graphs_and_columns():
    """A graph for each of 300,000 single tokens given by offsets, and 20,000 columns: more tiles of columns than blocks of rows."""
    n = 300_000
    x, gate, initial = scan.rand(n, 4, seed=1), scan.rand(n, 4, seed=2), scan.rand(n, 4, seed=3).contiguous()
    ptr = torch.arange(n + 1, device="cuda")
    a = torch.sigmoid(gate.double())
    want = a * initial.double() + torch.sigmoid(-gate.double()) * x.double()
    bound = (2 * gate.double().abs() + 16) * U * (a * initial.double().abs() + (1 - a) * x.double().abs())
    out, final = g.linear_recurrence(x, gate, graph_ptr=ptr, initial=initial, with_final=True)
    scan.check(out, (want, bound), "out")
    assert torch.equal(out, final) and torch.equal(out, g.linear_recurrence(x, gate, graphs=n, initial=initial))
    scan.both_ways(2100, 20_000, "factor", ptr=torch.tensor([0, 5, 2100], device="cuda"))
    scan.both_ways(40, 20_001, "sigmoid")
