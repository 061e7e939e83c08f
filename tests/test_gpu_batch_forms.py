"""Forms of tensors that the handles of a batch take or refuse: without rows, of one row, given twice after a refusal."""
import pytest
import torch

from batch_helpers import BF16, ints
from paper_2406_06237_b200.runtime import Adapters, BlockCache

pytestmark = pytest.mark.gpu


def test_a_batch_without_rows_out_of_wider_buffers():
    cache = BlockCache(4, 16, 2, 64)
    packed = torch.zeros(5, 3, 4, 64, dtype=BF16, device="cuda")
    assert cache.attend(packed[:0, 0], ints([[0]]), ints([5]), ints([0, 0])).shape == (0, 4, 64)
    f = Adapters(torch.zeros(1, 4, 32, dtype=BF16, device="cuda"), torch.zeros(1, 24, 4, dtype=BF16, device="cuda"))
    wide = torch.zeros(5, 100, dtype=BF16, device="cuda")
    assert f(wide[:0, :32], wide[:0, 40:64], ints([0]), ints([0, 0])).shape == (0, 24)
    assert cache.read_status() == 0 and f.read_status() == 0
