"""Refusals and workspace sizes of the lookup, attention and group norm calls: host logic, before any launch."""
import os
import re
from types import SimpleNamespace

import pytest

torch = pytest.importorskip("torch")

import paper_2104_03058_b200 as g  # noqa: E402
from paper_2104_03058_b200 import binding as b  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_tensors_on_the_cpu_are_refused():
    x, ids = torch.zeros(4, 8), torch.zeros(3, dtype=torch.int64)
    with pytest.raises(ValueError, match="ids must be a 1-D CUDA tensor"):
        g.embedding(x, ids)
    with pytest.raises(ValueError, match="ids must be a 1-D CUDA tensor"):
        g.embedding_backward(ids, torch.zeros(3, 8), 4)
    with pytest.raises(ValueError, match="x must be a 2-D CUDA tensor"):
        g.group_norm(x, 2)
    with pytest.raises(ValueError, match="x must be a 2-D CUDA tensor"):
        g.group_norm_backward(x, x, 2, torch.zeros(1, 2), torch.ones(1, 2))


def test_attention_operands():
    csr = SimpleNamespace(n=4, nnz=9, device=torch.device("cpu"))
    with pytest.raises(ValueError, match="nnz = 9"):
        b._check_dist(csr, torch.zeros(8, dtype=torch.int32), "dist")
    with pytest.raises(ValueError, match="int32"):
        b._check_dist(csr, torch.zeros(9), "dist")
    with pytest.raises(ValueError, match="contiguous"):
        b._check_dist(csr, torch.zeros(18, dtype=torch.int32)[::2], "dist")
    with pytest.raises(ValueError, match="is on cpu"):
        b._check_dist(SimpleNamespace(nnz=3, device=torch.device("cuda", 0)), torch.zeros(3, dtype=torch.int32), "dist")
    b._check_dist(csr, torch.zeros(9, dtype=torch.int32), "dist")


def test_norm_operands():
    x = torch.zeros(5, 6)
    for kwargs, match in ((dict(groups=4), "groups"), (dict(groups=0), "groups"), (dict(weight=torch.zeros(5)), "weight"),
                          (dict(weight=torch.zeros(6).double()), "weight"), (dict(bias=torch.zeros(12)[::2]), "bias"),
                          (dict(activation="swish"), "activation")):
        args = dict(dict(groups=2, weight=None, bias=None, graph_ptr=None, activation="none"), **kwargs)
        with pytest.raises(ValueError, match=match):
            b._norm_operands(x, args["groups"], args["weight"], args["bias"], args["graph_ptr"], args["activation"], 6)


def test_the_c_calls_refuse_bad_arguments_without_a_device():
    L, p = g.lib(), 4096                                       # p: an aligned address that nothing reads
    emb = lambda n=1, itype=0, vocab=5, ldt=8, tdt=0, f=8, ldo=8, odt=0, ids=p, table=p, out=p: L.gnnfd_embedding(      # noqa: E731
        n, ids, itype, vocab, table, ldt, tdt, f, 1.0, out, ldo, odt, None, None)
    assert emb(n=0) == g.OK
    assert emb(n=-1) == emb(vocab=0) == emb(f=0) == emb(ldt=7) == emb(ldo=7) == emb(ids=None) == emb(table=None) == emb(out=None) == g.INVALID_ARG
    assert emb(itype=2) == emb(tdt=2) == emb(odt=5) == g.UNSUPPORTED
    assert emb(n=1 << 31) == emb(vocab=1 << 31) == g.TOO_LARGE
    grad = lambda n=19_000, itype=0, vocab=5, ldd=8, ddt=0, f=8, ldg=8, gdt=0, ids=p, dout=p, out=p, scr=p, size=1 << 40: (      # noqa: E731
        L.gnnfd_embedding_backward(n, ids, itype, dout, ldd, ddt, vocab, f, 1.0, -1, 0, out, ldg, gdt, scr, size, None, None))
    assert grad(n=-1) == grad(vocab=0) == grad(f=0) == grad(ldd=7) == grad(ldg=7) == grad(ids=None) == grad(dout=None) == grad(out=None) == g.INVALID_ARG
    assert grad(ldd=1 << 31) == grad(scr=None) == grad(scr=p + 8) == g.INVALID_ARG
    assert grad(itype=2) == grad(ddt=2) == grad(gdt=2) == g.UNSUPPORTED
    assert grad(n=1 << 31) == grad(vocab=1 << 31) == g.TOO_LARGE
    assert grad(size=1000) == g.WORKSPACE_TOO_SMALL
    norm = lambda n=9, ldx=8, xdt=0, f=8, groups=2, graphs=1, ptr=None, itype=0, eps=1e-5, act=0, ldo=8, odt=0, mean=None, rstd=None, x=p, out=p, scr=p, size=1 << 40: (      # noqa: E731
        L.gnnfd_group_norm(n, x, ldx, xdt, f, groups, graphs, ptr, itype, None, None, eps, act, out, ldo, odt, mean, rstd, scr, size, None))
    assert norm(n=-1) == norm(f=0) == norm(groups=0) == norm(groups=3) == norm(graphs=0) == norm(graphs=2) == norm(ldx=7) == norm(ldo=7) == g.INVALID_ARG
    assert norm(eps=-1.0) == norm(eps=float("nan")) == norm(mean=p) == norm(rstd=p) == norm(x=None) == norm(out=None) == norm(scr=None) == g.INVALID_ARG
    assert norm(xdt=2) == norm(odt=2) == norm(act=5) == norm(act=-1) == norm(ptr=p, itype=2) == norm(f=8200, ldx=8200, ldo=8200) == g.UNSUPPORTED
    assert norm(n=1 << 31) == norm(ldx=1 << 23) == norm(ldo=1 << 23) == g.TOO_LARGE
    assert norm(size=100) == g.WORKSPACE_TOO_SMALL
    back = lambda n=9, ldd=8, ldx=8, f=8, lddx=8, mean=p, rstd=p, dw=None, db=None, dout=p, scr=p, size=1 << 40: (      # noqa: E731
        L.gnnfd_group_norm_backward(n, dout, ldd, p, ldx, 0, f, 2, 1, None, 0, None, None, mean, rstd, 0, p, lddx, 0, dw, db, scr, size, None))
    assert back(ldd=7) == back(ldx=7) == back(lddx=7) == back(mean=None) == back(rstd=None) == back(dw=p) == back(db=p) == back(dout=None) == g.INVALID_ARG
    assert back(size=100) == g.WORKSPACE_TOO_SMALL and back(ldd=1 << 23) == g.TOO_LARGE
    assert L.gnnfd_aggregate_attention(None, p, 8, p, 8, p, 8, 0, 1, 8, 1.0, 0.0, None, None, 0, p, 8, 0, None, 8, None, 0, None) == g.INVALID_ARG
    assert L.gnnfd_aggregate_attention_backward(None, None, p, 8, p, 8, p, 8, p, 8, 0, p, 1, 8, 1.0, 0.0, None, None, None, 0, p, 8, p, 8, p, 8, 0,
                                                None, 8, p, 0, None) == g.INVALID_ARG


def test_workspaces_grow_with_what_they_are_for():
    sizes = [g.embedding_backward_workspace_bytes(n, 1000, 64) for n in (0, 16_384, 16_385, 20_000, 100_000, 1_000_000, 30_000_000)]
    assert sizes[:2] == [0, 0] and sizes == sorted(sizes)
    assert g.embedding_backward_workspace_bytes(10_000, 3_629_056, 64) == 0 < g.embedding_backward_workspace_bytes(10_000, 3_629_057, 64)
    assert g.group_norm_workspace_bytes(0, 8, 2) > 0
    for backward in (False, True):
        sizes = [g.group_norm_workspace_bytes(n, 64, 8, 1, backward) for n in (1, 100, 10_000, 1_000_000)]
        assert sizes == sorted(sizes)
    for call in (lambda: g.embedding_backward_workspace_bytes(-1, 5, 8), lambda: g.embedding_backward_workspace_bytes(5, 0, 8),
                 lambda: g.group_norm_workspace_bytes(5, 8, 3), lambda: g.group_norm_workspace_bytes(5, 8, 2, 0)):
        with pytest.raises(g.GnnfdError) as err:
            call()
        assert err.value.status == g.INVALID_ARG


def test_constants_of_the_header():
    text = open(os.path.join(ROOT, "include", "gnnfd.h")).read()
    assert int(re.search(r"#define GNNFD_EMBEDDING_FEW_IDS (\d+)", text).group(1)) == g.EMBEDDING_FEW_IDS
    assert int(re.search(r"#define GNNFD_EMBEDDING_FEW_ROWS (\d+)", text).group(1)) == g.EMBEDDING_FEW_ROWS
    for name, code in g.ACTIVATIONS.items():
        assert int(re.search(r"GNNFD_ACT_%s = (\d+)" % name.upper(), text).group(1)) == code


def test_attention_refuses_what_its_grids_do_not_hold():
    """Columns beyond 65535 blocks of 64 and buckets beyond 65535 blocks of 40 are refused before the graph is looked at."""
    L, p = g.lib(), 4096
    fwd = lambda heads, dim: L.gnnfd_aggregate_attention(p, p, 8, p, 8, p, 8, 0, heads, dim, 1.0, 0.0, None, None, 0, p, 8, 0, None, 8, None, 0, None)      # noqa: E731
    back = lambda heads, buckets: L.gnnfd_aggregate_attention_backward(      # noqa: E731
        p, p, p, 8, p, 8, p, 8, p, 8, 0, p, heads, 8, 1.0, 0.0, p, p, p, buckets, p, 8, p, 8, p, 8, 0, p, 8, p, 0, None)
    assert fwd(65_536, 64) == fwd((1 << 31) - 1, 256) == g.TOO_LARGE
    assert back(1, 65_535 * 40 + 1) == back((1 << 31) - 1, 9) == g.TOO_LARGE
