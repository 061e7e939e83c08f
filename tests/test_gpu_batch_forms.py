"""Forms of tensors that the handles of a batch take or refuse: without rows, of one row, given twice after a refusal."""
import pytest
import torch

from batch_helpers import BF16, INT, attention, fill_cache, ints
from operator_helpers import rounds_from
from paper_2406_06237_b200 import binding as B
from paper_2406_06237_b200.runtime import Adapters, BlockCache, PageTables

pytestmark = pytest.mark.gpu


def test_a_batch_without_rows_out_of_wider_buffers():
    cache = BlockCache(4, 16, 2, 64)
    packed = torch.zeros(5, 3, 4, 64, dtype=BF16, device="cuda")
    assert cache.attend(packed[:0, 0], ints([[0]]), ints([5]), ints([0, 0])).shape == (0, 4, 64)
    f = Adapters(torch.zeros(1, 4, 32, dtype=BF16, device="cuda"), torch.zeros(1, 24, 4, dtype=BF16, device="cuda"))
    wide = torch.zeros(5, 100, dtype=BF16, device="cuda")
    assert f(wide[:0, :32], wide[:0, 40:64], ints([0]), ints([0, 0])).shape == (0, 24)
    assert cache.read_status() == 0 and f.read_status() == 0


@pytest.mark.parametrize("heads", [1, 2])
@pytest.mark.parametrize("off", [0, 1])
def test_one_token_out_of_a_row_of_any_length(heads, off):
    """With one token (and one head) the distance to the next one is no one's concern."""
    arrays = fill_cache(4, heads, 16, 64)
    cache, tables = BlockCache.wrap(*arrays), ints([[0, 1, 2, 3]])
    flat = torch.randn(128 * heads + 200, device="cuda").to(BF16)
    q = flat.as_strided((1, 2 * heads, 64), (128 * heads + 3, 64, 1), off)
    out = torch.zeros(300 * heads, dtype=BF16, device="cuda").as_strided((1, 2 * heads, 64), (128 * heads + 5, 64, 1), 2 * off)
    want, slack = attention(q, arrays, tables, [50], [0, 1])
    assert rounds_from(cache.attend(q, tables, ints([50]), ints([0, 1])), want, slack).all()
    assert rounds_from(cache.attend(q, tables, ints([50]), ints([0, 1]), out=out), want, slack).all()
    alone = flat.as_strided((3, 1, 64), (64, 67, 1), 0)
    one = BlockCache.wrap(*(t[:, :1].contiguous() for t in arrays))
    want, slack = attention(alone, (one.k_codes, one.k_scales, one.v_codes, one.v_scales), tables, [50], [0, 3])
    assert rounds_from(one.attend(alone, tables, ints([50]), ints([0, 3])), want, slack).all()
    own = flat.as_strided((1, 2 * heads, 64), (128 * heads + 3, 64, 1), 0)
    want, slack = attention(own.clone(), arrays, tables, [50], [0, 1])
    assert cache.attend(own, tables, ints([50]), ints([0, 1]), out=flat[:128 * heads].view(1, 2 * heads, 64)) is not own       # over q
    assert rounds_from(own, want, slack).all() and cache.read_status() == 0


@pytest.mark.parametrize("change", [dict(scale=float("inf")), dict(share=129)])
def test_what_is_refused_is_refused_again(change):
    cache = BlockCache(4, 16, 1, 16)
    q = torch.zeros(2, change.pop("share", 4), 16, dtype=BF16, device="cuda")
    for _ in range(2):
        with pytest.raises(B.AnsError):
            cache.attend(q, ints([[0]]), ints([5]), ints([0, 2]), **change)


def test_sizes_that_32_bits_do_not_hold():
    for page_size in (0, -1, (1 << 20) + 1, (1 << 32) + 16):
        with pytest.raises(ValueError):
            PageTables(page_size)
    many = (1 << 32) + 1
    one, none = ints([0]), ints([])
    with pytest.raises(ValueError):
        PageTables(16)(ints([[0]]), one, one, torch.empty(many, dtype=INT, device="cuda"), one, rows=4)
    f = Adapters(torch.zeros(1, 1, 1, dtype=BF16, device="cuda"), torch.zeros(1, 1, 1, dtype=BF16, device="cuda"))
    x = torch.empty(many, 1, dtype=BF16, device="cuda")
    with pytest.raises(ValueError):
        f(x, x, one, ints([0, 0]), out=x)
    with pytest.raises(ValueError):
        Adapters(torch.empty(1, 1, many, dtype=BF16, device="cuda"), torch.zeros(1, 1, 1, dtype=BF16, device="cuda"))
    assert none.numel() == 0


def test_an_output_whose_rows_lie_over_each_other():
    cache = BlockCache(4, 16, 2, 64)
    q = torch.zeros(3, 4, 64, dtype=BF16, device="cuda")
    flat = torch.zeros(4096, dtype=BF16, device="cuda")
    for strides in ((0, 64, 1), (256, 0, 1), (256, 32, 1), (128, 64, 1), (64, 128, 1)):
        with pytest.raises(ValueError):
            cache.attend(q, ints([[0]]), ints([5]), ints([0, 3]), out=flat.as_strided((3, 4, 64), strides))
    for strides in ((256, 64, 1), (64, 192, 1), (64, 200, 1), (300, 66, 1)):
        cache.attend(q, ints([[0]]), ints([5]), ints([0, 3]), out=flat.as_strided((3, 4, 64), strides))
    assert cache.read_status() == 0
