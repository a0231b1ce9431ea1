"""What the layer norm, rotary and recurrence calls refuse or accept at their limits: host logic, before any launch."""
from types import SimpleNamespace

import pytest

torch = pytest.importorskip("torch")

import paper_2104_03058_b200 as g  # noqa: E402
from paper_2104_03058_b200 import binding as b  # noqa: E402

P = 1 << 20                                          # an aligned address that nothing reads


@pytest.fixture
def calls(monkeypatch):
    """The binding's checks on CPU tensors: a library that records its calls, operands taken without the test for their device."""
    made = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: made.append((name, args)) or g.OK

    def matrix(t, cols, name):
        assert t.dim() == 2 and t.shape[1] >= cols
        return t.data_ptr(), t.stride(0)

    monkeypatch.setattr(b, "lib", Library)
    monkeypatch.setattr(b, "_matrix", matrix)
    monkeypatch.setattr(b, "_index_list", lambda t, name: (t.data_ptr(), t.numel(), b.I64))
    monkeypatch.setattr(b, "_stream_handle", lambda index, stream: 0)
    return made


def test_states_do_not_lie_in_the_results(calls):
    """A sequence in stretches that share one buffer: the row that the next stretch starts from is written before other threads read it."""
    n, f = 64, 8
    x, buf, wide = torch.zeros(n, f), torch.zeros(n, f), torch.zeros(n, 2 * f)
    ptr, final = torch.tensor([0, 10, n]), torch.zeros(1, f)
    for more in (dict(), dict(with_final=True), dict(final=final), dict(with_states=True)):
        for initial, out in ((buf[-1:], buf), (buf[:1], buf), (wide[5:6, :f], wide[:, :f]), (wide.view(-1)[12:12 + f][None], wide[:, :f]), (buf[3:4], buf)):
            with pytest.raises(ValueError, match="initial and out overlap"):
                b.linear_recurrence(x, x, initial=initial, out=out, **more)
    with pytest.raises(ValueError, match="initial and out overlap"):
        b.linear_recurrence(x, x, graph_ptr=ptr, initial=buf[:2], out=buf)
    with pytest.raises(ValueError, match="initial and out overlap"):
        b.linear_recurrence(x, x, graphs=n // 4, initial=buf[:n // 4], out=buf)
    assert not calls


def test_states_beside_the_results_and_single_tokens_in_place(calls):
    n, f = 64, 8
    x, buf, wide = torch.zeros(n, f), torch.zeros(n, f), torch.zeros(n, 2 * f)
    b.linear_recurrence(x, x, initial=torch.zeros(1, f), out=buf)
    b.linear_recurrence(x, x, initial=wide[7:8, f:], out=wide[:, :f])             # between two rows of the results
    b.linear_recurrence(x, x, graphs=n, initial=buf, out=buf)
    b.linear_recurrence(x[:1], x[:1], initial=wide[7:8, :f], out=wide[7:8, :f])
    assert len(calls) == 4
    for initial, out in ((buf, wide[:, :f]), (wide.view(-1)[:n * f].view(n, f), wide[:, :f]), (buf.view(-1)[:n * f].view(n, f), buf.view(torch.bfloat16)[:, :f])):
        if initial.data_ptr() == out.data_ptr():
            with pytest.raises(ValueError, match="initial and out overlap"):       # another pitch or type than its own
                b.linear_recurrence(x, x, graphs=n, initial=initial, out=out)


def test_the_c_call_refuses_states_in_the_results():
    L = g.lib()
    scan = lambda first, out=P, ldo=8, odt=0, n=9000, graphs=1, ptr=None: (      # noqa: E731
        L.gnnfd_linear_recurrence(n, 2 * P, 8, 3 * P, 8, 0, 8, 1, graphs, ptr, 0, first, out, ldo, odt, None, None, 4 * P, 1 << 40, None))
    for first in (P, P + 4, P + 8999 * 32, P + 8999 * 32 + 28, P - 28):
        assert scan(first) == g.INVALID_ARG
    assert scan(P + 64 * 77, ldo=16) == scan(P + 64 * 77 + 60, ldo=16) == scan(P + 16 * 33, odt=1) == scan(P, n=9, graphs=3) == g.INVALID_ARG
    assert scan(P, n=9, graphs=9, odt=1) == scan(P, n=9, graphs=9, ldo=9) == scan(P + 32, n=9, graphs=9) == scan(P, n=9, graphs=9, ptr=5 * P) == g.INVALID_ARG


def test_the_c_calls_refuse_results_in_place_of_what_is_still_read():
    L = g.lib()
    norm = lambda n=9, ldx=8, xdt=0, out=P, ldo=8, odt=0: L.gnnfd_layer_norm(n, P, ldx, xdt, 8, None, None, 1e-5, out, ldo, odt, None, None, None)      # noqa: E731
    assert norm(ldo=9) == norm(ldx=9) == norm(odt=1) == norm(xdt=1) == norm(n=1, odt=1) == g.INVALID_ARG
    back = lambda dx, ldd=8, lddx=8, xdt=0, gdt=0, n=9: (      # noqa: E731
        L.gnnfd_layer_norm_backward(n, P, ldd, 2 * P, 8, xdt, 8, None, 3 * P, 3 * P, dx, lddx, gdt, None, None, None, 0, None))
    assert back(P, lddx=9) == back(P, ldd=9) == back(P, gdt=1) == back(P, xdt=1) == back(2 * P) == back(P, n=1, gdt=1) == g.INVALID_ARG
    scan = lambda out: L.gnnfd_linear_recurrence(9000, P, 8, 2 * P, 8, 0, 8, 1, 1, None, 0, None, out, 8, 0, None, None, 5 * P, 1 << 40, None)      # noqa: E731
    assert scan(P) == scan(2 * P) == g.INVALID_ARG
    rev = lambda dx=6 * P, dgate=7 * P, dfinal=None, dinitial=None: (      # noqa: E731
        L.gnnfd_linear_recurrence_backward(9000, P, 8, 2 * P, 8, 3 * P, 8, 0, 8, 0, 1, None, 0, None, 4 * P, dfinal, dx, 8, dgate, 8, 0, dinitial, 5 * P, 1 << 40, None))
    for t in (P, 2 * P, 3 * P):
        assert rev(dx=t) == rev(dgate=t) == g.INVALID_ARG
    assert rev(dgate=6 * P) == rev(dfinal=8 * P, dinitial=8 * P) == g.INVALID_ARG


def test_the_package_has_what_its_binding_has_now(monkeypatch):
    """A function that is replaced in the binding after its first use through the package (a tracer's wrapper) is what the package gives from then on."""
    was = g.rotary_frequencies
    assert was(8, device="cpu").shape == (4,) and was is b.rotary_frequencies
    with monkeypatch.context() as m:
        m.setattr(b, "rotary_frequencies", lambda *args, **kwargs: "wrapped")
        assert g.rotary_frequencies(8, device="cpu") == "wrapped"
    assert g.rotary_frequencies is was
    with pytest.raises(AttributeError, match="no attribute 'rotary_frequency'"):
        g.rotary_frequency


def test_frequencies_of_factors_of_any_size():
    """The last frequency is divided by factor also where factor^(r / (r - 2)) has no number in 64 bits; frequencies that have none are refused."""
    for r in (4, 8, 64):
        plain = g.rotary_frequencies(r, 1e4, device="cpu")
        for factor in (1e-200, 1e-150, 0.25, 8.0, 1e160, 1e200):
            got = g.rotary_frequencies(r, 1e4, "base", factor, device="cpu")
            assert got[0] == 1.0 and abs(float(got[-1]) / (float(plain[-1]) / factor) - 1) <= 2.0 ** -48
            steps = got[1:] / got[:-1]
            assert float((steps / steps[0] - 1).abs().max()) <= 2.0 ** -40          # a geometric series
    for scaling in ("position", "base"):
        with pytest.raises(g.GnnfdError) as err:
            g.rotary_frequencies(8, 1e4, scaling, 1e-320, device="cpu")
        assert err.value.status == g.INVALID_ARG


def test_columns_beyond_32_bits_are_refused():
    """A single row of 2^32 + 8 columns is no row of 8."""
    def row(width):
        return SimpleNamespace(is_cuda=True, dim=lambda: 2, shape=(1, width), stride=lambda: (width, 1), data_ptr=lambda: P)

    for width in (1 << 31, (1 << 32) + 8):
        with pytest.raises(ValueError, match="columns"):
            b._matrix(row(width), width, "x")
    assert b._matrix(row(1 << 32), 8, "x") == (P, 1 << 32)
    assert b._matrix(row((1 << 31) - 1), (1 << 31) - 1, "x") == (P, (1 << 31) - 1)
