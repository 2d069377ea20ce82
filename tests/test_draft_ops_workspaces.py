"""What the drafted tokens' operators ask for in workspaces (no GPU needed)."""
import pytest

from paper_2607_16074_gb300 import build as B
from paper_2607_16074_gb300 import jnx as J


@pytest.fixture(scope="module", autouse=True)
def built():
    B.build()


@pytest.mark.parametrize("hd", [64, 128, 256])
@pytest.mark.parametrize("tokens", [1, 256, 700, 2048, 4096, 8192, 16_384, 60_000, 70_000, 1 << 20])
@pytest.mark.parametrize("rows,heads", [(1, 8), (768, 32), (16_384, 32)])
def test_tree_workspace_is_what_runs_can_fill(hd, tokens, rows, heads):
    """Sums for a run of every 1,024 tokens, or for the eight (33 at head dim 256) that a
    shorter sequence is cut into: 4 bytes for each of a head's columns and two more, and records."""
    runs = max(1, min(64, -(-tokens // 1024)), min(33 if hd == 256 else 8, -(-tokens // 256)))
    need = J.lib().jnx_op_tree_attention_workspace_bytes(256, rows, heads, hd, tokens)
    sums = rows * heads * runs * (hd + 2) * 4
    assert sums <= need <= sums + 16 * rows + 4096


def test_tree_workspace_of_more_serves_less():
    f = J.lib().jnx_op_tree_attention_workspace_bytes
    for hd in (64, 128, 256):
        sizes = [f(4, 9, 8, hd, t) for t in range(0, 80_000, 63)]
        assert sizes == sorted(sizes)
        sizes = [f(4, n, 8, hd, 5000) for n in range(300)]
        assert sizes == sorted(sizes)
