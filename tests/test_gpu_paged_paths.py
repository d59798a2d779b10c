"""The paged operators where one call's leftovers could reach the next: workspaces, captured calls, pages given back."""
import pytest

from test_gpu_paged import make_plan, paged  # noqa: F401  (paged: a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bad", [-1, 2 ** 31 - 1, -2 ** 31, "n_pages"])
@pytest.mark.parametrize("requests", [3, 300])
def test_plan_reports_a_bad_page_that_comes_back(paged, bad, requests):
    """An ended request whose row holds no page id inside its length: the call that takes it back says so, and so does the one that
    hands it out; no slot is made of it."""
    cached, new = [40, 20, 33] + [5] * (requests - 3), [-1, 0, 0] + [0] * (requests - 3)
    p, table, free, n_free, n_pages = make_plan(paged, cached, new, 16, 600, slack=0)
    bad = n_pages if bad == "n_pages" else bad
    p.table[0, 1] = bad
    p.d3_page_plan()
    assert int(p.status) == -1
    assert int(p.n_free) == 3 and p.free[:3].tolist() == [int(table[0, 0]), bad, int(table[0, 2])]
    assert p.cached.tolist() == [0] + cached[1:]
    p.status.zero_()
    p.new_tokens.zero_()
    p.new_tokens[1] = 13                       # 20 -> 33: one page, the last that came back
    p.d3_page_plan()
    assert int(p.status) == 0 and int(p.table[1, 2]) == int(table[0, 2])
    p.new_tokens[1] = 16                       # 33 -> 49: the bad one
    p.d3_page_plan()
    assert int(p.status) == -1
    assert p.slots[:16].tolist() == [int(table[0, 2]) * 16 + i for i in range(1, 16)] + [-1]
