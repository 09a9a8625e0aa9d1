"""counts[3] of tl_paged_slots: every token that a request asked for and did not get, however many, up to the largest int."""
import pytest

from tests.test_gpu_paged_slots import run

pytestmark = pytest.mark.gpu
INT_MAX = 2 ** 31 - 1


def left(new, want, **kw):
    """`want`: in exact whole numbers."""
    got = run([0] * len(new), new, width=kw.pop("width", 8), **kw)
    assert int(got["counts"][3]) == min(want, INT_MAX)


@pytest.mark.parametrize("B", [1, 60, 65, 1500], ids=str)
@pytest.mark.parametrize("n", [300000, (1 << 18) + 1, 1 << 28, INT_MAX], ids=str)
def test_requests_that_ask_for_more_than_a_step_holds(n, B):
    """One wave, one workgroup, several requests to a thread; the sum of what is left passes 32 bits in most."""
    rows = min(B * 128, 5000)
    left([n] * B, n * B - rows, T=rows)


def test_largest_step():
    """2^18 rows for one request with room for all of them in its table."""
    left([300000], 300000 - (1 << 18), T=1 << 18, width=300000 // 16, n_pages=20000)
    left([300000], 300000 - 4096, T=1 << 13, max_new=4096, width=300000 // 16, n_pages=20000)


@pytest.mark.parametrize("new", [[300000] * 3, [INT_MAX, 7, 1 << 30], [1 << 18, INT_MAX - (1 << 18)]], ids=str)
def test_in_place_over_several_workgroups(new):
    """Lengths and counts come from a launch of their own there."""
    rows = min(sum(min(n, 8 * 1024) for n in new), 3000)
    left(new, sum(new) - rows, T=rows, width=512, in_place=True, n_pages=2000)
