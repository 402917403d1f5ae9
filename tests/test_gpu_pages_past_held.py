"""Table entries past the pages that a sequence holds, after vsr_pages_update: as they were,
but for the one behind a copy that got no page."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("seqs", [6, 1000])   # tables forked by one block, and by several
def test_entries_past_held(seqs):
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2601_01513_amd import binding as B
    page, most, n_pages = 4, 5, 7
    i32 = lambda x: torch.tensor(np.asarray(x, np.int32), device="cuda")  # noqa: E731
    table = np.arange(seqs * most, dtype=np.int32).reshape(seqs, most) + 100
    table[0, :3], table[1, :2] = [4, 2, 5], [0, 6]
    length, held, refs = np.zeros(seqs, np.int32), np.zeros(seqs, np.int32), np.zeros(n_pages, np.int32)
    length[:2], held[:2] = [10, 5], [3, 2]
    refs[[4, 2, 5, 0, 6]] = 1
    pages = B.pages(i32(table), i32(length), i32(held), i32(refs), page)
    k, v = (torch.randn((2, n_pages * page, 1, 8), device="cuda") for _ in "kv")
    # Pages 1 and 3 are free, and 0 and 6 when 1 has dropped them. 2 to 5 become 0, whose last
    # page has two rows: each gets one of the four for its copy.
    source = np.arange(seqs)
    source[1:6] = [-1, 0, 0, 0, 0]
    ok = B.pages_update(pages, i32(source), i32([0] * seqs), k, v)
    assert ok.tolist()[:6] == [1, 1, 1, 1, 1, 1]
    room = np.zeros(seqs, np.int32)
    room[2] = 3                     # none is left
    assert B.pages_update(pages, i32(np.arange(seqs)), i32(room), k, v).tolist()[:6] == [1, 1, 0, 1, 1, 1]
    want = table.copy()
    for s, p in zip((2, 3, 4, 5), (0, 1, 3, 6)):
        want[s, :3] = [4, 2, p]
    assert np.array_equal(pages.table.cpu().numpy(), want)
    # 1 becomes 0 as well, and there is no page for the copy.
    source = np.arange(seqs)
    source[1] = 0
    assert B.pages_update(pages, i32(source), None, k, v).tolist()[:6] == [1, 0, 1, 1, 1, 1]
    assert pages.len.tolist()[:6] == [10, 8, 10, 10, 10, 10] and pages.held.tolist()[:2] == [3, 2]
    want[1, :3] = [4, 2, 5]         # 5: past held
    assert np.array_equal(pages.table.cpu().numpy(), want)
    assert pages.refs.tolist() == [1, 1, 6, 1, 6, 1, 1]
