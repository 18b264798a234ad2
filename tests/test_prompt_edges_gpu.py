"""Calls of the prompt-side operators that are allowed but unusual: very many sequences, lengths out of range, queries that
are not finite, requests with pages in common, calls side by side."""
import pytest
import torch

from paper_2608_15473_b200 import binding as qf
from paper_2608_15473_b200 import build as qf_build
from prompt_testlib import D, PAGE, Paged, prompt64
from test_prefix_gpu import Shared, check_partial
from test_prompt_attend_gpu import KERNELS, attend, check, compare, queries

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    qf_build.build()


# the schedule is found by a warp per sequence up to 12, a thread each up to 384, in rounds of 384 beyond
@pytest.mark.parametrize("n", [12, 13, 383, 384, 385, 769, 1100])
def test_many_sequences(n):
    check(Paged([(5 * i) % 4 for i in range(n - 1)] + [3], [(37 * i) % 90 for i in range(n)], 2), 4)


@pytest.mark.parametrize("n", [12, 13, 384, 385, 800])
def test_many_groups(n):
    groups = [i % 3 for i in range(n - 1)] + [2]
    check_partial(Shared(groups, [(13 * i) % 60 for i in range(n)], [1] * sum(groups), 1), 2)


@pytest.mark.parametrize("flags", KERNELS)
def test_lengths_out_of_range(flags):
    pg = Paged([20, 3, 200], [0, 61, 0], 2, max_pages=4)      # the last one's table row ends after 64 positions
    q = queries(pg, 4)
    pg.lens = torch.tensor([-5, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32)      # below 0: nothing cached; the table's end
    out, lse, status = attend(pg, q, flags)
    pg.cached = [0, 64, 0]
    compare(out, lse, prompt64(pg, q, max_tokens=64))
    assert status == 0


def test_offsets_out_of_range_leave_the_rest_alone():
    """Offsets beyond the packed rows and below 0 are the caller's error: nothing outside is touched."""
    pg = Paged([40, 30], [5, 0], 2)
    q = queries(pg, 4)
    good, good_lse, _ = attend(pg, q)
    pg.cu = torch.tensor([0, 40, 10 ** 9], dtype=torch.int32)      # the last request claims rows that are not there
    out, lse, _ = attend(pg, q)
    assert torch.equal(out[:70], good) and torch.equal(lse[:70], good_lse)


@pytest.mark.parametrize("flags", KERNELS)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_query_that_is_not_finite_stays_its_own_affair(flags, bad):
    pg = Paged([40, 3, 90], [10, 200, 0], 2)
    q = queries(pg, 4)
    fine, fine_lse, _ = attend(pg, q, flags)
    q2 = q.clone()
    q2[41, 2] = bad           # one row, one head
    out, lse, _ = attend(pg, q2, flags)
    others = torch.ones((pg.total, 4), dtype=torch.bool, device="cuda")
    others[41, 2] = False
    assert torch.equal(out[others], fine[others]) and torch.equal(lse[others], fine_lse[others])
    assert torch.isnan(out[41, 2]).all() and torch.isnan(lse[41, 2])      # scores of both signs of infinity, or NaN


def test_requests_with_pages_in_common():
    """Reading is free: the same pages twice in a batch, and twice in one table row."""
    pg = Paged([30, 30, 17], [100, 100, 300], 2)
    pg.table[1] = pg.table[0]
    pg.table[2, 3], pg.table[2, 4] = pg.table[2, 0], pg.table[0, 0]
    check(pg, 8)


def test_calls_side_by_side_on_two_streams():
    """Two prompts and two prefixes at once, each with a workspace of its own: the same bits as one after the other."""
    pgs = [Paged([900], [700], 2, seed=1), Paged([1] * 50, [40 * i for i in range(50)], 2, seed=2)]
    qs = [queries(pg, 8, seed=i) for i, pg in enumerate(pgs)]
    alone = [attend(pg, q)[:2] for pg, q in zip(pgs, qs)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    state = []
    for pg, q in zip(pgs, qs):
        p = qf.params(pg.B, 8, 2, pg.width, 1, pg.num_pages)
        n = qf.prompt_workspace_bytes(p, pg.total)
        state.append((pg.pools(), pg.table.cuda(), pg.cu.cuda(), pg.lens.cuda(), torch.empty_like(q),
                      torch.empty(q.shape[:2], device="cuda"), p, torch.empty(n, dtype=torch.uint8, device="cuda"), n))
    torch.cuda.synchronize()
    for _ in range(20):
        for (pools, table, cu, lens, out, lse, p, ws, n), q, st in zip(state, qs, streams):
            qf.prompt_attend(q, *pools, table, cu, lens, out, lse, p, q.shape[0], ws, n, 0, st)
    torch.cuda.synchronize()
    for (out, lse), s in zip(alone, state):
        assert torch.equal(out, s[4]) and torch.equal(lse, s[5])
        assert qf.prompt_status(s[7]) == 0


def test_a_batch_of_one_row_of_one_head_at_the_end_of_a_long_row():
    pg = Paged([1], [PAGE * 2000 - 1], 1)
    check(pg, 1)


def test_rows_in_front_of_the_first_request():
    """Padding before the first request is left as it was, like padding behind the last."""
    pg = Paged([40, 30], [5, 0], 2)
    q = queries(pg, 4)
    good, good_lse, _ = attend(pg, q)
    front = 9
    q2 = torch.cat([torch.full((front, 4, D), float("nan"), dtype=torch.bfloat16, device="cuda"), q])
    p = qf.params(2, 4, 2, pg.width, 1, pg.num_pages)
    out = torch.full((front + pg.total, 4, D), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((front + pg.total, 4), 7.0, device="cuda")
    n = qf.prompt_workspace_bytes(p, front + pg.total)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    qf.prompt_attend(q2, *pg.pools(), pg.table.cuda(), pg.cu.cuda() + front, pg.lens.cuda(), out, lse, p, front + pg.total, ws, n)
    torch.cuda.synchronize()
    assert (out[:front] == 7).all() and (lse[:front] == 7).all()
    assert torch.equal(out[front:], good) and torch.equal(lse[front:], good_lse)
