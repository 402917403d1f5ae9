"""Tables, lists and log-sums of the paged operators in the gaps between rows of keys and
values: they meet nothing, and the calls give what they give apart."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def test_arrays_between_rows_are_taken():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2601_01513_amd import binding as B
    g = torch.Generator(device="cuda").manual_seed(1)
    T, heads, hd, page, n_pages = 6, 4, 64, 8, 6
    i32 = lambda x: torch.tensor(np.asarray(x, np.int32), device="cuda")  # noqa: E731
    q = torch.randn((T, heads, hd), generator=g, device="cuda")
    k, v = (torch.randn((n_pages * page, 2, hd), generator=g, device="cuda") for _ in "kv")
    table, length, held, start = i32([[3, 1, 0], [5, 2, 4]]), i32([13, 9]), i32([3, 3]), i32([0, 4, 6])
    pages = B.pages(table, length, held, i32([1] * n_pages), page)
    lse = torch.empty((T, heads), device="cuda")
    want = B.tree_attention(pages, q, k, v, 0.125, start=start, lse=lse)
    # One allocation: keys' slots 1024 elements apart, everything small in the gap of one.
    wide = torch.full((n_pages * page, 1024), float("nan"), device="cuda")
    far = wide.as_strided((n_pages * page, 2, hd), (1024, hd, 1))
    far.copy_(k)
    gap_lse = wide[7, 128:128 + T * heads].view(T, heads)
    ints = wide[11].view(torch.int32)
    small = [ints[200:206].view(2, 3), ints[300:302], ints[400:402], ints[500:506], ints[600:603]]
    for to, x in zip(small, (table, length, held, i32([1] * n_pages), start)):
        to.copy_(x)
    near = B.pages(*small[:4], page)
    got = B.tree_attention(near, q, far, v, 0.125, start=small[4], lse=gap_lse)
    assert torch.equal(got, want) and torch.equal(gap_lse, lse)
    # A cache whose layers leave room for the tables, and what an update and a keep say.
    def cache():
        x = torch.zeros((2, 2, n_pages * page + 3, 2 * hd), device="cuda")
        kk, vv = (x[i, :, :n_pages * page].view(2, n_pages * page, 2, hd) for i in range(2))
        kk.copy_(torch.stack([k, 2 * k]))
        vv.copy_(torch.stack([v, 3 * v]))
        return x, kk, vv
    results = []
    for inside in (False, True):
        x, kk, vv = cache()
        room = x[0, 0, n_pages * page:].view(torch.int32).flatten()
        put = [i32([[3, 1, 0], [5, 2, 4]]), i32([13, 9]), i32([2, 2]), i32([0, 1, 1, 1, 0, 1]),
               i32([1, 1]), i32([[0, 2], [1, 3]]), i32([0, 0])]
        if inside:
            at = 0
            for i, y in enumerate(put):
                view = room[at:at + y.numel()].view(y.shape)
                view.copy_(y)
                put[i], at = view, at + 8
        p = B.pages(*put[:4], page)
        B.pages_update(p, put[4], None, kk, vv, ok=put[6])
        B.pages_update(p, room=i32([5, 5]))
        B.pages_keep(p, put[5], None, kk, vv)
        torch.cuda.synchronize()
        results.append([y.clone() for y in (*put[:4], kk, vv)])
    assert all(map(torch.equal, *results))
