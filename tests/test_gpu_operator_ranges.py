"""The lookup, attention and group norm calls where offsets pass 32 bits, with narrower widths than their operands', on two streams at
once, and one after the other as a layer and its gradient.  References and bounds are those of the operators' own tests."""
import pytest

torch = pytest.importorskip("torch")

import paper_2104_03058_b200 as g  # noqa: E402
import test_gpu_attention as att  # noqa: E402
import test_gpu_embedding as emb  # noqa: E402
import test_gpu_group_norm as norm  # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def far_rows(rows, cols, pitch, dtype, seed):
    """[rows, cols] values whose rows are `pitch` elements apart."""
    buf = torch.zeros(rows * pitch, device="cuda", dtype=dtype)
    view = buf.view(rows, pitch)[:, :cols]
    view.copy_(torch.randn((rows, cols), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda"))
    return view


def test_rows_more_than_four_gigabytes_apart():
    pitch = 3 << 19                                                    # 1100 rows of 1.5 Mi bf16 elements: 3.5 GB; of fp32: 6.9 GB
    x = far_rows(1100, 24, pitch, F32, 0)
    ids = emb.draw_ids(5000, 1100, "even", torch.int64)
    assert torch.equal(g.embedding(x, ids), x.contiguous()[ids])
    picked = torch.arange(1099, -1, -1, device="cuda", dtype=torch.int32)
    emb.check_grad(g.embedding_backward(picked % 7, x, 7), picked % 7, x, 7, 1.0)                      # few ids
    out = far_rows(1100, 24, pitch, F32, 1)
    many = emb.draw_ids(20_000, 1100, "even", torch.int32)
    dout = emb.rand(20_000, 24)
    emb.check_grad(g.embedding_backward(many, dout, 1100, out=out), many, dout, 1100, 1.0)             # sorted, into rows far apart
    y = g.group_norm(x, 4, activation="silu", out=out)
    norm.check(y, norm.reference(x, 4, None, None, None, "silu", norm.EPS)["out"], "out")
    src, dst = att.edges(1100, 9000)
    p = att.Problem(1100, src, dst, 3, 8, buckets=2)
    p.q, p.k, p.v, p.dout = (far_rows(1100, 24, pitch, BF16, s) for s in range(4))
    p.check()


def test_widths_narrower_than_the_operands():
    table, ids = emb.rand(50, 20), emb.draw_ids(300, 50, "even", torch.int32)
    assert torch.equal(g.embedding(table, ids, f=9), table[ids.long(), :9])
    dout = emb.rand(300, 20)
    out = torch.full((50, 20), 4.0, device="cuda")
    g.embedding_backward(ids, dout, 50, f=9, out=out)
    emb.check_grad(out[:, :9], ids, dout[:, :9], 50, 1.0)
    assert (out[:, 9:] == 4.0).all()
    x = norm.rand(300, 20)
    out = torch.full((300, 20), 4.0, device="cuda")
    g.group_norm(x, 3, f=9, out=out)
    norm.check(out[:, :9], norm.reference(x[:, :9], 3, None, None, None, "none", norm.EPS)["out"], "out")
    assert (out[:, 9:] == 4.0).all()


def test_two_streams_at_once_and_another_stream_than_the_operands():
    problems = [att.Problem(2000, *att.edges(2000, 40_000, 2500, seed=s), 4, 16, buckets=3, seed=s) for s in (0, 1)]
    ids = [emb.draw_ids(30_000, 2000, "skew", torch.int32, s) for s in (0, 1)]
    dout = emb.rand(30_000, 16)
    x, ptr = norm.rand(20_000, 48), norm.offsets(20_000, 900)
    torch.cuda.synchronize()
    want = []
    for s in (0, 1):
        out, lse = problems[s].forward(with_lse=True)
        want.append((out, *problems[s].backward(lse), g.embedding_backward(ids[s], dout, 2000), g.group_norm(x, 6, graph_ptr=ptr, activation="gelu")))
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [[], []]
    for _ in range(3):
        for s in (0, 1):
            out, lse = problems[s].forward(with_lse=True, stream=streams[s])
            got[s].append((out, *problems[s].backward(lse, stream=streams[s]), g.embedding_backward(ids[s], dout, 2000, stream=streams[s]),
                           g.group_norm(x, 6, graph_ptr=ptr, activation="gelu", stream=streams[s])))
    torch.cuda.synchronize()
    for s in (0, 1):
        for res in got[s]:
            assert all(torch.equal(a, b) for a, b in zip(res, want[s]))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_layer_and_its_gradient(dtype):
    """Vertex rows looked up, attended over a batch of graphs, normalised per graph; then backwards into the table.  Every stage is
    checked on what the stage before it gave."""
    heads, dim, vocab = 4, 8, 70
    f = heads * dim
    sizes = torch.tensor([1, 0, 30, 200, 7, 90, 128, 129], device="cuda")
    ptr = torch.cat([sizes.new_zeros(1), sizes.cumsum(0)])
    n = int(ptr[-1])
    graph = torch.repeat_interleave(torch.arange(8, device="cuda"), sizes)
    pairs = torch.nonzero(graph[:, None] == graph[None, :])            # the graphs attend to themselves alone
    src, dst = pairs[:, 1].int().contiguous(), pairs[:, 0].int().contiguous()
    ids = emb.draw_ids(n, vocab, "skew", torch.int64)
    table = emb.rand(vocab, 3 * f, dtype)
    x = g.embedding(table, ids, scale=1.5, out_dtype=dtype)
    assert torch.equal(x, (table[ids].float() * 1.5).to(dtype))
    p = att.Problem(n, src, dst, heads, dim, dtype, cap=8.0)
    p.bias = att.rand(6, heads)
    hops = (src - dst).abs().clamp(max=5).int()
    p.dist, p.dist_t = g.edge_values(p.csr, hops), g.edge_values(p.csr_t, hops)
    p.q, p.k, p.v = x[:, :f], x[:, f:2 * f], x[:, 2 * f:]
    y, lse = p.forward(with_lse=True, out_dtype=dtype)
    weight, shift = norm.rand(1, f, seed=2)[0].contiguous(), norm.rand(1, f, seed=3)[0].contiguous()
    z, mean, rstd = g.group_norm(y, heads, weight, shift, ptr, activation="silu", out_dtype=dtype, with_stats=True)
    dz = norm.rand(n, f, dtype, seed=9)
    dy, dw, db = g.group_norm_backward(dz, y, heads, mean, rstd, weight, shift, ptr, "silu", out_dtype=dtype)
    ref = norm.reference(y, heads, weight, shift, ptr, "silu", norm.EPS, dz)
    for name, got in (("out", z), ("dx", dy), ("dw", dw), ("db", db)):
        norm.check(got, ref[name], name)
    p.dout = dy
    ref = p.reference()
    grads = p.backward(lse, out_dtype=dtype)
    for name, got in zip(("out", "dq", "dk", "dv", "dbias"), (y, *grads)):
        att.check(got, ref[name], name)
    dx = torch.cat(grads[:3], dim=1)
    emb.check_grad(g.embedding_backward(ids, dx, vocab, scale=1.5), ids, dx, vocab, 1.5)


def test_every_edge_the_same_and_the_same_id_everywhere():
    n = 3000
    src, dst = torch.full((5000,), 7, dtype=torch.int32, device="cuda"), torch.full((5000,), 9, dtype=torch.int32, device="cuda")
    p = att.Problem(n, src, dst, 2, 16, buckets=1)
    out, _, _ = p.check()                                              # one hub row, one hub column
    assert torch.allclose(out[9], p.v[7], rtol=1e-5, atol=1e-6) and int((out != 0).any(1).sum()) == 1
    ids = torch.full((100_000,), 3, device="cuda")
    dout = emb.rand(100_000, 5)
    emb.check_grad(g.embedding_backward(ids, dout, 4), ids, dout, 4, 1.0)
