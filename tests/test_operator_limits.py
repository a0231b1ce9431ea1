"""What the lookup, attention and group norm calls refuse or accept at their limits: host logic, before any launch."""
import os
import subprocess
import sys
from types import SimpleNamespace

import pytest

torch = pytest.importorskip("torch")

import paper_2104_03058_b200 as g  # noqa: E402
from paper_2104_03058_b200 import binding as b  # noqa: E402

P = 4096                                             # an aligned address that nothing reads


def lookup(f, n=1, vocab=5):
    return g.lib().gnnfd_embedding(n, P, 0, vocab, P, f, 0, f, 1.0, P, f, 0, None, None)


def gradient(f, n=19_000, vocab=5, out=P):
    return g.lib().gnnfd_embedding_backward(n, P, 0, P, f, 0, vocab, f, 1.0, -1, 0, out, f, 0, P, 1 << 60, None, None)


def test_no_ids_need_no_workspace():
    for vocab in (1, g.EMBEDDING_FEW_ROWS, g.EMBEDDING_FEW_ROWS + 1, 100_000_000):
        assert g.embedding_backward_workspace_bytes(0, vocab, 64) == 0


def test_rows_wider_than_the_grids():
    """65535 column tiles: of 256 columns, of 128 where rows can only be read element by element."""
    for n in (100, 19_000):
        assert gradient(65_535 * 256 + 8, n) == g.TOO_LARGE                       # rows start on 16 bytes
        assert gradient(65_535 * 256 + 2, n) == g.TOO_LARGE                       # on 8
        assert gradient(65_535 * 128 + 1, n) == gradient(65_535 * 128 + 8, n, out=P + 4) == g.TOO_LARGE
        assert gradient((1 << 31) - 1, n) == g.TOO_LARGE
    assert lookup((1 << 31) - 1) == lookup((1 << 31) - 1024) == g.TOO_LARGE       # column counters are 32 bits


def test_edge_values_want_one_value_for_each_edge():
    csr = SimpleNamespace(device=torch.device("cpu"), nnz=6, e=3, perm=torch.tensor([0, 4, 2, 3, -1, 1], dtype=torch.int32))
    assert b.edge_values(csr, torch.tensor([10, 20, 30]), loop=7).tolist() == [10, 20, 30, 10, 7, 20]
    for count in (0, 1, 2, 4, 6):
        with pytest.raises(ValueError, match="3 edges"):
            b.edge_values(csr, torch.zeros(count))


def test_the_package_imports_where_torch_has_no_cuda():
    code = ("import torch\n"
            "for name in [n for n in dir(torch._C) if n.startswith('_cuda')]: delattr(torch._C, name)\n"
            "import paper_2104_03058_b200 as g\n"
            "try: g.group_norm(torch.zeros(4, 8), 2)\n"
            "except ValueError as err: assert 'CUDA tensor' in str(err)\n"
            "else: raise AssertionError\n")
    done = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert done.returncode == 0, done.stderr
