"""What the torch wrappers accept, without a GPU."""
import pytest

torch = pytest.importorskip("torch")

from paper_2609_01956_amd import binding as kb


def test_workspaces_that_hold_their_bytes():
    """A workspace is used only where its bytes lie side by side: an expanded or strided tensor
    has fewer than it counts, or others' between them."""
    cpu = torch.device("cpu")
    w = torch.empty(4096, dtype=torch.uint8)
    assert kb._fits(w, 4096, cpu) and kb._fits(w, 0, cpu) and kb._fits(w.view(64, 64), 4096, cpu)
    assert not kb._fits(None, 0, cpu) and not kb._fits(w, 4097, cpu)
    assert not kb._fits(w, 1, torch.device("meta"))
    assert not kb._fits(w[:1].expand(4096), 4096, cpu)
    assert not kb._fits(w[::2], 2048, cpu) and not kb._fits(w.view(64, 64).t(), 4096, cpu)
