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
