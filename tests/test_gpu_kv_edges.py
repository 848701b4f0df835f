"""The paged cache's bookkeeping where a step's rows, the pool or the table do not suffice."""
import numpy as np
import pytest

from paper_2512_23367_amd import binding as ql
from paper_2512_23367_amd.layer import PagedRequests

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def U():
    import kv_util
    return kv_util


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("room", [0, 1, 7, 40, 1000])
@pytest.mark.parametrize("pages", [200, 9])
def test_every_token_without_a_slot_is_counted(U, pages, room, in_place):
    """Whatever it lacks: a page of the pool, a column of the table, a row of the step."""
    rng = np.random.default_rng(room)
    n, page, columns = 21, 32, 3
    want = rng.integers(0, 130, n)
    pool = U.ints([0, pages, 0, 0])
    out = pool if in_place else U.ints([7, 7, 7, 0])
    kv_len, cu, slots, positions = U.ints([0] * n), U.ints([0] * (n + 1)), U.ints([-5] * room), U.ints([-5] * room)
    ql.ql_kv_resize(page, U.ints([0] * n), U.ints(want), U.ints(np.arange(pages)), pool, out, U.ints(np.full((n, columns), -1)), kv_len, cu, slots, positions)
    has = kv_len.cpu().numpy()
    assert out.cpu().tolist()[2] == (want - has).sum() and (slots >= 0).sum().item() == has.sum()


def test_a_step_of_more_tokens_than_rows_says_so(U):
    requests = PagedRequests(ql.QlKvFormat(heads=2, head_dim=64, page_size=32, pages=8, bits=8), 3, 4, 16)
    requests.step(U.ints([10, 12, 1]))
    assert requests.kv_len.tolist() == [10, 6, 0] and requests.pool.tolist()[1:3] == [6, 7]
    requests.step(U.ints([10, 12, 1]))
    assert requests.kv_len.tolist() == [10, 12, 1] and requests.pool.tolist()[2] == 0
