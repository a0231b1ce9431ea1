"""What the lookup, attention and group norm calls refuse or accept at their limits: host logic, before any launch."""
import pytest

torch = pytest.importorskip("torch")

import paper_2104_03058_b200 as g  # noqa: E402


def test_no_ids_need_no_workspace():
    for vocab in (1, g.EMBEDDING_FEW_ROWS, g.EMBEDDING_FEW_ROWS + 1, 100_000_000):
        assert g.embedding_backward_workspace_bytes(0, vocab, 64) == 0
