"""vsr_pages_update at the ends of its sizes."""
import pytest

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


def test_the_last_of_all_pages():
    """2^31 - 1 pages of one position, the last two free: the number after the last one is no
    page, whatever lies behind the counts."""
    torch = _torch()
    from paper_2601_01513_amd import binding as B
    n = 2 ** 31 - 1
    room = torch.ones(n + 65, dtype=torch.int32, device="cuda")
    room[n - 2:] = 0                    # (behind the counts as well)
    refs = room[:n]
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    table, length, held = i32([[7, 7], [7, 7], [7, 7]]), i32([0, 0, 0]), i32([0, 0, 0])
    pages = B.pages(table, length, held, refs, 1)
    ok = B.pages_update(pages, room=i32([1, 1, 1]))
    torch.cuda.synchronize()
    assert ok.tolist() == [1, 1, 0] and held.tolist() == [1, 1, 0]
    assert table.tolist() == [[n - 2, 7], [n - 1, 7], [7, 7]]
    assert refs[-3:].tolist() == [1, 1, 1] and room[n:].tolist() == [0] * 65


def test_very_wide_tables():
    """2^27 columns, more than one launch of a block for each few of them has room for; pages
    held in the first and the last columns."""
    torch = _torch()
    from paper_2601_01513_amd import binding as B
    most, n = 1 << 27, 1 << 18
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    table = torch.empty((2, most), dtype=torch.int32, device="cuda")
    # Sequence 1 holds every column; the pages in turn (a page is then held many times over).
    table[0] = -5
    table[1] = torch.arange(most, device="cuda", dtype=torch.int32) % n
    refs = torch.full((n,), most // n, dtype=torch.int32, device="cuda")
    length, held = i32([0, most]), i32([0, most])
    k = torch.zeros((1, n, 1, 1), dtype=torch.float16, device="cuda")
    pages = B.pages(table, length, held, refs, 1)
    ok = B.pages_update(pages, i32([1, 1]), None, k, k.clone())
    torch.cuda.synchronize()
    assert ok.tolist() == [1, 1] and held.tolist() == [most, most] and length.tolist() == [most, most]
    assert torch.equal(table[0], table[1]) and bool((refs == 2 * (most // n)).all())
    B.pages_update(pages, i32([-1, 1]), None, k, k.clone())
    torch.cuda.synchronize()
    assert held.tolist() == [0, most] and bool((refs == most // n).all())
