"""Offsets and table entries that are far out of range: nothing outside the arrays is read or written, and what is in range
stays right."""
import pytest
import torch

from paper_2608_15473_b200 import binding as qf
from paper_2608_15473_b200 import build as qf_build
from prompt_testlib import D, PAGE, Paged, attend64
from test_prefix_gpu import Shared, partial
from test_prompt_attend_gpu import KERNELS, attend, compare, queries

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    qf_build.build()


@pytest.mark.parametrize("first", [-1, -2 ** 30, -2 ** 31])
def test_rows_of_a_request_that_begins_far_below_zero(first):
    """The caller's error, but one whose rows lie 2^31 positions into the context: beyond every table row, so that nothing
    is stored.  (At -1 the rows' places are one further on.)"""
    hq, n = 4, 40
    pg = Paged([n], [3], 2, extra_pages=2, max_pages=4)
    pg.table[0, :4] = torch.arange(4, dtype=torch.int32)
    g = torch.Generator().manual_seed(2)
    q, k, v = (torch.randn((n, h * D), generator=g).to(torch.bfloat16).cuda() for h in (hq, 2, 2))
    kc, vc = pg.pools()
    k0, v0, qo = kc.clone(), vc.clone(), torch.empty_like(q)
    p, r = qf.params(1, hq, 2, 4, 1, pg.num_pages), qf.rope_params(n, 0)
    cu = torch.tensor([first, n], dtype=torch.int32).cuda()
    qf.rope_append(q, k, v, qo, None, kc, vc, pg.table.cuda(), cu, pg.lens.cuda(), None, None, None, None, p, r)
    torch.cuda.synchronize()
    assert torch.equal(qo, q)
    if first != -1:
        assert torch.equal(kc, k0) and torch.equal(vc, v0)
    else:
        for pool, x in ((kc, k), (vc, v)):
            rows = pool[:4].permute(0, 2, 1, 3).reshape(64, 2, D)
            assert torch.equal(rows[4:4 + n], x.reshape(n, 2, D))


@pytest.mark.parametrize("rows", [[1], [200], [3, 90, 1, 40]])
def test_bad_entries_that_differ_from_tile_to_tile(rows):
    """Random entries are bad, other ones in every tile of 8 pages, over many turns of the ring of tiles: each tile's
    positions are hidden by its own entries, time after time."""
    cached = [6_000 + 130 * i for i in range(len(rows))]
    pg = Paged(rows, cached, 2, seed=len(rows))
    good = pg.table.clone()
    g = torch.Generator().manual_seed(3)
    gone = torch.rand(pg.table.shape, generator=g) < 0.3
    pg.table[gone] = torch.tensor([-1, pg.num_pages, 2 ** 31 - 1, -2 ** 31])[torch.randint(4, (int(gone.sum()),), generator=g)].to(torch.int32)
    q = queries(pg, 8)
    parts = []
    for b, n in enumerate(rows):
        keep = torch.tensor([i for i in range(cached[b] + n) if not gone[b, i // PAGE]])
        k, v = ((pg.k if w == "k" else pg.v)[good[b][keep // PAGE].long(), :, keep % PAGE].permute(1, 0, 2).double() for w in "kv")
        seen = (keep[None, :] <= cached[b] + torch.arange(n)[:, None]).sum(1)
        parts.append(attend64(q[int(pg.cu[b]):int(pg.cu[b]) + n].double(), k.cuda(), v.cuda(), seen.cuda()))
    ref = {n: torch.cat([d[n] for d in parts]).cpu() for n in parts[0]}
    first = None
    for _ in range(20):
        out, lse, status = attend(pg, q, qf.QF_FLAG_CHECK_BOUNDS)
        assert status == qf.QF_STATUS_BAD_PAGE
        first = first or (out, lse)
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1])
    compare(out, lse, ref)


@pytest.mark.parametrize("flags", KERNELS)
def test_lengths_beyond_the_table_row_are_reported(flags):
    """As the sweep reports them: under QF_FLAG_CHECK_BOUNDS, and only where rows would see positions beyond it."""
    check = flags | qf.QF_FLAG_CHECK_BOUNDS
    for new, cached, want in ((20, 44, 0), (20, 45, 1), (1, 64, 1), (0, 1000, 0), (70, 0, 1), (64, 0, 0)):
        pg = Paged([new, 3], [cached, 2], 2, max_pages=4, extra_pages=80)
        q = queries(pg, 4)
        assert attend(pg, q, flags)[2] == 0
        assert attend(pg, q, check)[2] == (qf.QF_STATUS_BAD_PAGE if want else 0), (new, cached)
    pg = Paged([20, 20], [0, 18], 2, max_pages=4)
    assert attend(pg, queries(pg, 4), check, max_seq_len=38)[2] == 0
    assert attend(pg, queries(pg, 4), check, max_seq_len=37)[2] == qf.QF_STATUS_BAD_PAGE
    for more, want in ((0, 0), (1, 1), (2 ** 31 - 1 - 64, 1)):
        sh = Shared([4, 2], [64, 30], [1] * 6, 2)
        sh.plen[0] += more
        q = torch.randn((6, 4, D), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
        assert partial(sh, q, flags)[3] == 0
        assert partial(sh, q, check)[3] == (qf.QF_STATUS_BAD_PAGE if want else 0), more
