"""Refusals and workspace sizes of the layer norm, rotary and recurrence calls: host logic, before any launch."""
import math
import os
import re

import pytest

torch = pytest.importorskip("torch")

import paper_2104_03058_b200 as g  # noqa: E402
from paper_2104_03058_b200 import binding as b  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 4096                                             # an aligned address that nothing reads


def test_tensors_on_the_cpu_are_refused():
    x, row = torch.zeros(4, 8), torch.zeros(4)
    for call in (lambda: g.layer_norm(x), lambda: g.layer_norm_backward(x, x, row, row), lambda: g.linear_recurrence(x, x),
                 lambda: g.linear_recurrence_backward(x, x, x, torch.zeros(1, 8)), lambda: g.rotary(x, torch.ones(2, dtype=torch.float64), 2, 4)):
        with pytest.raises(ValueError, match="x must be a 2-D CUDA tensor"):
            call()


def test_the_c_calls_refuse_bad_arguments_without_a_device():
    L = g.lib()
    norm = lambda n=9, x=P, ldx=8, xdt=0, f=8, eps=1e-5, out=P, ldo=8, odt=0, mean=None, rstd=None: (      # noqa: E731
        L.gnnfd_layer_norm(n, x, ldx, xdt, f, None, None, eps, out, ldo, odt, mean, rstd, None))
    assert norm(n=0) == g.OK
    assert norm(n=-1) == norm(f=0) == norm(ldx=7) == norm(ldo=7) == norm(eps=-1.0) == norm(eps=float("nan")) == g.INVALID_ARG
    assert norm(mean=P) == norm(rstd=P) == norm(x=None) == norm(out=None) == g.INVALID_ARG
    assert norm(xdt=2) == norm(odt=-1) == norm(f=8193, ldx=8200, ldo=8200) == g.UNSUPPORTED
    assert norm(n=1 << 31) == g.TOO_LARGE
    back = lambda n=9, dout=P, ldd=8, x=P, f=8, mean=P, rstd=P, dx=P, lddx=8, dw=P, db=P, scr=P, size=1 << 30: (      # noqa: E731
        L.gnnfd_layer_norm_backward(n, dout, ldd, x, 8, 0, f, None, mean, rstd, dx, lddx, 0, dw, db, scr, size, None))
    assert back(n=-1) == back(ldd=7) == back(lddx=7) == back(dout=None) == back(x=None) == back(dx=None) == back(mean=None) == back(rstd=None) == g.INVALID_ARG
    assert back(dw=None) == back(db=None) == back(scr=None) == back(scr=P + 8) == g.INVALID_ARG
    assert back(size=100) == g.WORKSPACE_TOO_SMALL and back(n=1 << 31) == g.TOO_LARGE
    turn = lambda n=9, x=P, ldx=16, xdt=0, heads=2, dim=8, part=8, pos=None, itype=0, freq=P, out=P + 64, ldo=16, odt=0: (      # noqa: E731
        L.gnnfd_rotary(n, x, ldx, xdt, heads, dim, part, 0, pos, itype, freq, 1.0, 0, out, ldo, odt, None))
    assert turn(n=0) == g.OK
    assert turn(n=-1) == turn(heads=0) == turn(dim=0) == turn(part=0) == turn(part=7) == turn(part=10) == turn(ldx=15) == turn(ldo=15) == g.INVALID_ARG
    assert turn(freq=None) == turn(x=None) == turn(out=None) == turn(out=P, odt=1) == turn(out=P, ldo=17) == g.INVALID_ARG
    assert turn(xdt=2) == turn(odt=2) == turn(pos=P, itype=2) == turn(heads=1, dim=5000, part=4098, ldx=5000, ldo=5000) == g.UNSUPPORTED
    assert turn(n=1 << 31) == turn(heads=1 << 18, ldx=1 << 21, ldo=1 << 21) == turn(heads=(1 << 31) - 1, dim=(1 << 31) - 2, ldx=1 << 62, ldo=1 << 62) == g.TOO_LARGE
    scan = lambda n=9000, x=P, ldx=8, gate=P, ldg=8, dt=0, f=8, form=1, graphs=1, ptr=None, itype=0, first=None, out=P, ldo=8, odt=0, last=None, scr=P, size=1 << 40: (      # noqa: E731
        L.gnnfd_linear_recurrence(n, x, ldx, gate, ldg, dt, f, form, graphs, ptr, itype, first, out, ldo, odt, last, None, scr, size, None))
    assert scan(n=-1) == scan(f=0) == scan(graphs=0) == scan(graphs=7) == scan(ldx=7) == scan(ldg=7) == scan(ldo=7) == g.INVALID_ARG
    assert scan(x=None) == scan(gate=None) == scan(out=None) == scan(scr=None) == scan(scr=P + 8) == scan(first=P, last=P) == g.INVALID_ARG
    assert scan(dt=2) == scan(odt=2) == scan(form=2) == scan(form=-1) == scan(ptr=P, itype=2) == g.UNSUPPORTED
    assert scan(n=(1 << 31) - 1) == scan(ptr=P, graphs=(1 << 31) - 1) == scan(f=(1 << 20) + 1, ldx=1 << 21, ldg=1 << 21, ldo=1 << 21) == g.TOO_LARGE
    assert scan(size=1000) == g.WORKSPACE_TOO_SMALL
    rev = lambda n=9000, dout=P, ldd=8, x=P, gate=P, f=8, states=P, dx=P, lddx=8, dgate=P, lddg=8, gdt=0, scr=P, size=1 << 40: (      # noqa: E731
        L.gnnfd_linear_recurrence_backward(n, dout, ldd, x, 8, gate, 8, 0, f, 0, 1, None, 0, None, states, None, dx, lddx, dgate, lddg, gdt, None, scr, size, None))
    assert rev(n=-1) == rev(ldd=7) == rev(lddx=7) == rev(lddg=7) == rev(dout=None) == rev(x=None) == rev(gate=None) == rev(states=None) == g.INVALID_ARG
    assert rev(dx=None) == rev(dgate=None) == rev(scr=None) == g.INVALID_ARG and rev(gdt=2) == g.UNSUPPORTED and rev(size=1000) == g.WORKSPACE_TOO_SMALL


def test_workspaces():
    for call in (lambda: g.layer_norm_backward_workspace_bytes(-1, 8), lambda: g.layer_norm_backward_workspace_bytes(8, 0),
                 lambda: g.linear_recurrence_workspace_bytes(-1, 8), lambda: g.linear_recurrence_workspace_bytes(8, 0),
                 lambda: g.linear_recurrence_workspace_bytes(9, 8, 2, True), lambda: g.linear_recurrence_workspace_bytes(9, 8, 0)):
        with pytest.raises(g.GnnfdError) as err:
            call()
        assert err.value.status == g.INVALID_ARG
    sizes = [g.layer_norm_backward_workspace_bytes(n, 64) for n in (0, 1, 100, 10_000, 1_000_000)]
    assert sizes == sorted(sizes) and sizes[-1] == sizes[-2]
    assert g.linear_recurrence_workspace_bytes(g.RECURRENCE_FEW_ROWS, 5000) == 0 < g.linear_recurrence_workspace_bytes(g.RECURRENCE_FEW_ROWS + 1, 8)
    for backward in (False, True):
        assert g.linear_recurrence_workspace_bytes(g.RECURRENCE_FEW_ROWS // 2, g.RECURRENCE_FEW_VALUES // (g.RECURRENCE_FEW_ROWS // 2), 1, False, backward) == 0
        assert g.linear_recurrence_workspace_bytes(1_000_000, 512, 1_000_000, True) == 0                # single tokens
        # for a chunk of 8 rows or more: 8 bytes a column and 16, for every 8 chunks 12 bytes a column more; four arrays, rounded up to 256 bytes each
        for f in (1, 8, 64, 301, 4096):
            for n in (g.RECURRENCE_FEW_ROWS + 1, 10_000, 100_000, 1_000_000, 30_000_000):
                chunks = -(-n // 8)
                assert 0 < g.linear_recurrence_workspace_bytes(n, f, 1, False, backward) <= chunks * (8 * f + 16) + -(-chunks // 8) * 12 * f + 4 * 256


def test_frequencies():
    def want(r, base, scaling, factor, length, low, high):
        if scaling == "base":
            base *= factor ** (r / (r - 2))
        freq = [base ** (-2 * i / r) for i in range(r // 2)]
        if scaling == "position":
            freq = [w / factor for w in freq]
        if scaling == "ramp":
            kept = [min(1, max(0, (w * length / (2 * math.pi) - low) / (high - low))) for w in freq]
            freq = [w * (k + (1 - k) / factor) for w, k in zip(freq, kept)]
        return torch.tensor(freq, dtype=torch.float64)

    for r in (2, 4, 16, 64, 96, 4096):
        for scaling in g.ROTARY_SCALINGS:
            if scaling == "base" and r < 4:
                continue
            for base, factor in ((10_000.0, 8.0), (500_000.0, 1.0), (2.0, 0.5)):
                got = g.rotary_frequencies(r, base, scaling, factor, 8192, (2.0, 16.0), device="cpu")
                ref = want(r, base, scaling, factor, 8192, 2.0, 16.0)
                assert got.shape == (r // 2,) and float((got / ref - 1).abs().max()) <= 2.0 ** -48        # some roundings of 64 bits, the exponent's tenfold
    last = g.rotary_frequencies(64, 10_000.0, "base", 8.0, device="cpu")
    plain = g.rotary_frequencies(64, device="cpu")
    assert last[0] == plain[0] and abs(float(last[-1] / plain[-1]) * 8 - 1) < 1e-12
    with pytest.raises(ValueError, match="scaling"):
        g.rotary_frequencies(64, scaling="linear")
    for args in (dict(rotary_dim=0), dict(rotary_dim=7), dict(rotary_dim=-2), dict(rotary_dim=8, base=0.0), dict(rotary_dim=8, base=float("nan")),
                 dict(rotary_dim=8, factor=0.0), dict(rotary_dim=2, scaling="base"), dict(rotary_dim=8, scaling="ramp"),
                 dict(rotary_dim=8, scaling="ramp", length=100, turns=(5.0, 5.0)), dict(rotary_dim=8, factor=float("inf"))):
        with pytest.raises(g.GnnfdError) as err:
            g.rotary_frequencies(**dict(dict(device="cpu"), **args))
        assert err.value.status == g.INVALID_ARG
    with pytest.raises(g.GnnfdError) as err:
        g.rotary_frequencies(5000, device="cpu")
    assert err.value.status == g.UNSUPPORTED


def test_constants_of_the_header():
    text = open(os.path.join(ROOT, "include", "gnnfd.h")).read()
    for prefix, table in (("ROTARY", g.ROTARY_SCALINGS), ("GATE", g.GATES)):
        for name, code in table.items():
            assert int(re.search(r"GNNFD_%s_%s = (\d+)" % (prefix, name.upper()), text).group(1)) == code
    assert int(re.search(r"#define GNNFD_RECURRENCE_FEW_ROWS (\d+)", text).group(1)) == g.RECURRENCE_FEW_ROWS
    assert int(re.search(r"#define GNNFD_RECURRENCE_FEW_VALUES (\d+)", text).group(1)) == g.RECURRENCE_FEW_VALUES
    assert "fp32 [(n + %d) / %d, f]" % (b.STATE_ROWS - 1, b.STATE_ROWS) in text
