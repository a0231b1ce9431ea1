"""Embedding lookup and the table's gradient against plain evaluations in 64 bits.

Lookups are one product and one rounding: they are compared bit for bit.  A gradient's sum of k terms in fp32, in any order, is off by at
most (k - 1) * 2^-24 * sum |terms| to first order, the product with the scale adds one rounding, one more rounding comes with the output
type (2^-24 or 2^-8 of the value); the tolerance counts k + 2 and the output's."""
import pytest

torch = pytest.importorskip("torch")

import paper_2104_03058_b200 as g  # noqa: E402

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def rand(rows, cols, dtype=F32, ld=None, offset=0, seed=0):
    """[rows, cols] normal values with row pitch ld, `offset` elements behind an aligned address; what is around them is NaN."""
    ld = ld or cols
    gen = torch.Generator(device="cuda").manual_seed(seed + 17)
    buf = torch.full((rows * ld + offset + 8,), float("nan"), device="cuda", dtype=dtype)
    view = buf[offset:offset + rows * ld].view(rows, ld)[:, :cols]
    view.copy_(torch.randn((rows, cols), generator=gen, device="cuda"))
    return view


def draw_ids(n, vocab, kind, itype, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    u = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)
    if kind == "one":
        u = torch.full_like(u, 0.5)
    if kind == "skew":
        u = u ** 6
    ids = (u * vocab).long().clamp_(max=vocab - 1)
    if kind == "ascending":
        ids = ids.sort().values
    return ids.to(itype)


def reference(ids, dout, vocab, scale):
    """(gradient in 64 bits, sum of the terms' magnitudes, number of terms) per row, by a sort and one product with a 0/1 matrix."""
    ids = ids.long()
    keep = (ids >= 0) & (ids < vocab)
    order = torch.nonzero(keep).flatten()
    order = order[ids[order].argsort(stable=True)]
    ptr = torch.searchsorted(ids[order], torch.arange(vocab + 1, device="cuda"))
    take = torch.sparse_csr_tensor(ptr, order, torch.ones(order.numel(), dtype=torch.float64, device="cuda"), size=(vocab, max(1, dout.shape[0])))
    d = dout.double() if dout.shape[0] else torch.zeros((1, dout.shape[1]), dtype=torch.float64, device="cuda")
    return (take @ d.contiguous()) * scale, (take @ d.abs().contiguous()) * abs(scale), (ptr[1:] - ptr[:-1])


def check_grad(got, ids, dout, vocab, scale, base=None):
    want, size, count = reference(ids, dout, vocab, scale)
    if base is not None:
        want = want + base.double()
    half = torch.finfo(got.dtype).eps / 2
    tol = (count[:, None] + 2) * 2.0 ** -24 * size + half * want.abs() + (2.0 ** -24 * want.abs() if base is not None else 0)
    tol = tol * (1 + 2.0 ** -7)                                          # second-order terms
    assert torch.isfinite(got).all()
    worst = ((got.double() - want).abs() - tol).max()
    assert worst <= 0, float(worst)
    if base is None:
        assert (got[count == 0] == 0).all()


@pytest.mark.parametrize("itype", [torch.int32, torch.int64])
@pytest.mark.parametrize("tdt,odt", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("n,vocab,f,ld,offset", [(1, 1, 1, 1, 0), (1, 5, 602, 608, 0), (513, 100, 3, 3, 0), (77, 19, 8, 8, 1), (4001, 333, 41, 44, 0),
                                                 (20_003, 5000, 64, 64, 0), (50_000, 777, 24, 24, 2), (40_000, 99, 130, 136, 0)])
def test_lookup(itype, tdt, odt, n, vocab, f, ld, offset):
    table = rand(vocab, f, tdt, ld, offset)
    ids = draw_ids(n, vocab, "even", itype)
    out = torch.full((n, ld + 3), 7.0, device="cuda", dtype=odt)
    got = g.embedding(table, ids, scale=1.7, out=out[:, :f])
    want = (table[ids.long()].float() * 1.7).to(odt)
    assert torch.equal(got, want)
    assert (out[:, f:] == 7.0).all()                                    # padding columns stay
    assert torch.equal(g.embedding(table, ids, scale=1.7, out_dtype=odt), want)


def test_lookup_of_nothing_and_of_rows_beyond_two_to_the_31_bytes():
    assert g.embedding(rand(4, 8), torch.empty(0, dtype=torch.int64, device="cuda")).shape == (0, 8)
    table = torch.zeros((5_000_000, 256), device="cuda", dtype=BF16)     # 2.56 GB
    table[-1] = 3.0
    ids = torch.tensor([4_999_999, 0, 4_999_999], device="cuda")
    assert torch.equal(g.embedding(table, ids)[:, 0], torch.tensor([3.0, 0.0, 3.0], device="cuda"))


def test_ids_outside_the_table_give_zeros_and_set_the_status():
    table = rand(10, 5)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ids = torch.tensor([3, -1, 10, 9, 2 ** 40], device="cuda")
    got = g.embedding(table, ids, status=status)
    assert int(status) == 1 and (got[[1, 2, 4]] == 0).all() and torch.equal(got[[0, 3]], table[[3, 9]])
    status.zero_()
    g.embedding(table, torch.tensor([0, 9], device="cuda"), status=status)
    assert int(status) == 0


@pytest.mark.parametrize("ddt,odt", [(F32, F32), (F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("n,vocab,f,ld,offset,kind", [
    (0, 9, 5, 5, 0, "even"), (1, 1, 1, 1, 0, "even"), (2, 3, 602, 608, 0, "one"), (31, 40, 8, 8, 1, "even"), (4096, 19_717, 41, 41, 0, "skew"),
    (8192, 100, 64, 64, 0, "one"), (8193, 100, 64, 64, 0, "one"), (8193, 1, 3, 4, 0, "even"), (9000, 30_000, 130, 136, 0, "even"),
    (20_011, 7, 16, 16, 0, "skew"), (60_000, 250, 602, 608, 0, "skew"), (300_000, 232_965, 32, 32, 0, "skew"), (100_001, 3_000, 200, 200, 2, "ascending"),
    (250_000, 5_000, 1, 1, 0, "skew"), (65_536, 16_384, 24, 24, 0, "skew"), (65_536, 16_383, 24, 24, 0, "skew"),
    (40_000, 60_000, 41, 41, 0, "even"), (12_000, 3_000, 602, 604, 0, "one"), (50_000, 300_000, 9, 12, 1, "skew"), (400_000, 2_100_000, 8, 8, 0, "skew")])
def test_gradient(ddt, odt, n, vocab, f, ld, offset, kind):
    ids = draw_ids(n, vocab, kind, torch.int64 if n % 2 else torch.int32)
    dout = rand(n, f, ddt, ld, offset) if n else torch.empty((0, f), dtype=ddt, device="cuda")
    out = torch.full((vocab, ld + 5), 7.0, device="cuda", dtype=odt)
    got = g.embedding_backward(ids, dout, vocab, scale=0.7, out=out[:, :f])
    check_grad(got, ids, dout, vocab, 0.7)
    assert (out[:, f:] == 7.0).all()
    aligned = g.embedding_backward(ids, dout, vocab, scale=0.7, out_dtype=odt)
    check_grad(aligned, ids, dout, vocab, 0.7)
    assert torch.equal(aligned, g.embedding_backward(ids, dout, vocab, scale=0.7, out_dtype=odt))      # equal bits


@pytest.mark.parametrize("n", [1000, 50_000])
@pytest.mark.parametrize("odt", [F32, BF16])
def test_gradient_added_to_one_that_is_there_with_padding_and_bad_ids(n, odt):
    vocab, f, pad = 700, 20, 5
    ids = draw_ids(n, vocab, "skew", torch.int64)
    ids[::50] = pad
    dout = rand(n, f)
    kept = torch.where(ids == pad, -1, ids)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    base = rand(vocab, f, odt, seed=3).clone()
    got = g.embedding_backward(ids, dout, vocab, padding_idx=pad, accumulate=True, out=base.clone(), status=status)
    check_grad(got, kept, dout, vocab, 1.0, base)
    untouched = reference(kept, dout, vocab, 1.0)[2] == 0
    assert untouched[pad] and torch.equal(got[untouched], base[untouched]) and int(status) == 0
    got = g.embedding_backward(ids, dout, vocab, padding_idx=pad, status=status)
    check_grad(got, kept, dout, vocab, 1.0)
    assert (got[pad] == 0).all() and int(status) == 0
    ids[7], ids[11], ids[n - 1] = -3, vocab, 2 ** 33
    got = g.embedding_backward(ids, dout, vocab, status=status)
    check_grad(got, ids, dout, vocab, 1.0)
    assert int(status) == 1


@pytest.mark.parametrize("n", [300, 8193, 30_000])
def test_only_bad_or_padding_ids(n):
    dout = rand(n, 6)
    for ids in (torch.full((n,), -1, device="cuda"), torch.full((n,), 4, device="cuda")):
        assert (g.embedding_backward(ids, dout, 9, padding_idx=4) == 0).all()


def test_gradient_agrees_with_differences_of_the_lookup():
    table, ids = rand(6, 4).double().float(), torch.tensor([1, 1, 5, 0], device="cuda", dtype=torch.int32)
    dout = rand(4, 4, seed=5)
    grad = g.embedding_backward(ids, dout, 6, scale=3.0)
    loss = lambda t: (g.embedding(t, ids, scale=3.0).double() * dout.double()).sum()      # noqa: E731
    for r, c in ((1, 2), (5, 0), (2, 1)):
        moved = [table.clone(), table.clone()]
        moved[0][r, c] += 0.5
        moved[1][r, c] -= 0.5
        # linear: the difference is the gradient but for the roundings of about 12 products of size 10
        assert abs(float(loss(moved[0]) - loss(moved[1])) - float(grad[r, c])) <= 12 * 2 * 10 * 2.0 ** -24


@pytest.mark.parametrize("n", [2000, 40_000])
def test_captured_and_replayed_and_on_another_stream(n):
    vocab, f = 500, 16
    ids, dout, table = draw_ids(n, vocab, "skew", torch.int32), rand(n, f), rand(vocab, f, seed=9)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    plain = g.embedding_backward(ids, dout, vocab, stream=stream)
    looked = g.embedding(table, ids, stream=stream)
    stream.synchronize()
    check_grad(plain, ids, dout, vocab, 1.0)
    assert torch.equal(looked, table[ids.long()])
    out = torch.empty((vocab, f), device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        again = g.embedding(table, ids)
        g.embedding_backward(ids, again, vocab, out=out)
    for seed in (1, 2):
        ids.copy_(draw_ids(n, vocab, "skew", torch.int32, seed))
        graph.replay()
        torch.cuda.synchronize()
        check_grad(out, ids, table[ids.long()], vocab, 1.0)


@pytest.mark.parametrize("sweep", [0, 1])
def test_a_sort_that_gives_up_is_reported(sweep):
    n, vocab = 70_000, 100_000
    ids, dout = draw_ids(n, vocab, "even", torch.int32), rand(n, 4)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    g.debug_build_fault(256, sweep)
    g.embedding_backward(ids, dout, vocab, status=status)
    assert int(status) == 2
    status.zero_()
    check_grad(g.embedding_backward(ids, dout, vocab, status=status), ids, dout, vocab, 1.0)
    assert int(status) == 0
    g.debug_build_fault(256, 5)                                          # no such digit
    with pytest.raises(g.GnnfdError):
        g.embedding_backward(ids, dout, vocab)


def test_refusals():
    table, ids = rand(10, 8), torch.zeros(4, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="overlap"):
        g.embedding(table, ids, out=table[:4])
    with pytest.raises(ValueError, match="3 rows for 4 ids"):
        g.embedding(table, ids, out=torch.empty((3, 8), device="cuda"))
    with pytest.raises(ValueError, match="contiguous"):
        g.embedding(table, torch.zeros(8, dtype=torch.int32, device="cuda")[::2])
    with pytest.raises(TypeError):
        g.embedding(table, ids.float())
    with pytest.raises(TypeError):
        g.embedding(table.half(), ids)
    with pytest.raises(g.GnnfdError):
        g.embedding(table[:1].expand(10, 8), ids)                        # row pitch 0
    with pytest.raises(ValueError, match="accumulate"):
        g.embedding_backward(ids, rand(4, 8), 10, accumulate=True)
    with pytest.raises(ValueError, match="rows"):
        g.embedding_backward(ids, rand(3, 8), 10)
    with pytest.raises(g.GnnfdError) as err:
        many = torch.zeros(17_000, dtype=torch.int32, device="cuda")
        g.embedding_backward(many, rand(17_000, 8), 10, scratch=torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert err.value.status == g.WORKSPACE_TOO_SMALL
