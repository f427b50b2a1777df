"""A workspace that a caller gives: its bytes are the elements', side by side."""
import pytest

from paper_2606_27216_amd import train_ops as ops


def test_workspaces_with_gaps_or_repeated_elements_are_refused():
    torch = pytest.importorskip("torch")
    like = torch.empty(1)
    for bad in (torch.empty(1, dtype=torch.uint8).expand(1 << 20), torch.empty(64, dtype=torch.uint8)[::2],
                torch.empty(8, 9, dtype=torch.uint8)[:, :8], torch.empty(8, 9, dtype=torch.uint8).t()):
        with pytest.raises(ValueError):
            ops._workspace(16, bad, like)
    for good in (torch.empty(64, dtype=torch.uint8)[16:], torch.empty(4, 5), torch.empty(0, dtype=torch.uint8)):
        held, at, size = ops._workspace(16, good, like)
        assert held is good and at == good.data_ptr() and size == good.numel() * good.element_size()
