"""Rows of one call for the same place of a page."""
import pytest

from test_gpu_operators import ctx, ints, normal, offsets  # noqa: F401
from test_gpu_window import new_pages

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("heads,dim", [(1, 64), (12, 128)])
@pytest.mark.parametrize("n", [1, 300])
def test_rows_for_one_place(ctx, heads, dim, n):  # noqa: F811
    """Two sequences whose tables share their pages, one that names a page twice, and one with pages of its own: a shared
    place holds values of its rows, value by value, and everything else is as if nothing were shared."""
    page, per = 64, 5
    table = torch.arange(4 * per, dtype=torch.int32).view(4, per)
    table[1] = table[0]
    table[2] = table[2, 0]
    k, v = normal(960, 4 * n, heads, dim), normal(961, 4 * n, heads, dim)
    pages = new_pages(ctx, 4 * per, page, heads, dim, fill=7.0)
    ctx.paged_append(pages, table.cuda(), k.cuda(), v.cuda(), ints([0] * 4), offsets([n] * 4))
    for rows, stored in ((k, pages.k.cpu()), (v, pages.v.cpu())):
        places = {}
        for s in range(4):
            for i in range(n):
                places.setdefault((int(table[s, i // page]), i % page), []).append(s * n + i)
        left = torch.ones(4 * per, page, dtype=torch.bool)
        for (p, t), those in places.items():
            left[p, t] = False
            assert bool((rows[those] == stored[p, t]).any(0).all()), (p, t)
        assert bool((stored[left] == 7).all())
    assert torch.equal(pages.k.cpu()[table[3].long()].reshape(-1, heads, dim)[:n], k[3 * n:])
