"""The prompt-side operators on pools of which every page lies beyond 2^32 bytes from the start."""
import pytest
import torch

from paper_2608_15473_b200 import binding as qf
from paper_2608_15473_b200 import build as qf_build
from prompt_testlib import D, PAGE, Paged, prompt64
from qf_testlib import ENG_LSE, ENG_OUT
from test_prefix_gpu import Shared, err, partial64
from test_prompt_attend_gpu import KERNELS, attend, compare, queries

pytestmark = pytest.mark.gpu
HKV, FAR = 4, (5 << 30) // (4 * PAGE * D * 2)      # pages before the first that is used: 5 GB


@pytest.fixture(scope="module", autouse=True)
def built():
    qf_build.build()


def far(pg):
    """Pools whose last pages are pg's, behind FAR pages of NaN (token- or head-major), and pg's table moved there."""
    pools = []
    for x in pg.pools():
        big = torch.full((FAR + pg.num_pages, *x.shape[1:]), float("nan"), dtype=torch.bfloat16, device="cuda")
        big[FAR:] = x
        pools.append(big)
    assert pools[0][:FAR].numel() * 2 > 1 << 32
    return pools


@pytest.mark.parametrize("nhd", [False, True])
def test_placing_and_attending_far_pages(nhd):
    pg = Paged([70, 1, 130], [40, 300, 0], HKV, nhd)
    kc, vc = far(pg)
    hq, T = 8, pg.total
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn((T, h, D), generator=g).to(torch.bfloat16).cuda() for h in (hq, HKV, HKV))
    near_k, near_v, qo = kc[FAR:].clone(), vc[FAR:].clone(), torch.empty_like(q)
    p, r = qf.params(pg.B, hq, HKV, pg.width, 1, FAR + pg.num_pages, flags=qf.QF_FLAG_KV_NHD if nhd else 0), qf.rope_params(T, 0)
    table = torch.where(pg.table >= 0, pg.table + FAR, pg.table).cuda()
    qf.rope_append(q, k, v, qo, None, kc, vc, table, pg.cu.cuda(), pg.lens.cuda(), None, None, None, None, p, r)
    p0 = qf.params(pg.B, hq, HKV, pg.width, 1, pg.num_pages, flags=p.flags)
    qf.rope_append(q, k, v, qo, None, near_k, near_v, pg.table.cuda(), pg.cu.cuda(), pg.lens.cuda(), None, None, None, None, p0, r)
    torch.cuda.synchronize()
    assert torch.equal(kc[FAR:], near_k) and torch.equal(vc[FAR:], near_v) and torch.isnan(kc[:FAR:997]).all() and torch.isnan(vc[FAR - 1]).all()
    pg.k, pg.v = pg.head_major(near_k), pg.head_major(near_v)
    ref = prompt64(pg, q)
    pg.table, pg.num_pages = table.cpu(), FAR + pg.num_pages
    for flags in (0, qf.QF_FLAG_SIMPLE_KERNEL):
        out, lse, status = attend(pg, q, flags | qf.QF_FLAG_CHECK_BOUNDS, pools=(kc, vc))
        assert status == 0
        compare(out, lse, ref)


@pytest.mark.parametrize("flags", KERNELS)
@pytest.mark.parametrize("nhd", [False, True])
def test_a_prefix_on_far_pages(flags, nhd):
    sh = Shared([20, 2], [500, 129], [1] * 22, HKV, nhd)
    kc, vc = far(sh.pg)
    g = torch.Generator().manual_seed(2)
    q = (torch.randn((22, 8, D), generator=g) * 2).to(torch.bfloat16).cuda()
    p = qf.params(22, 8, HKV, 1, 1, FAR + sh.pg.num_pages, flags=flags | qf.QF_FLAG_CHECK_BOUNDS | (qf.QF_FLAG_KV_NHD if nhd else 0))
    o, m, l = (torch.full(s, 7.0, device="cuda") for s in ((22, 1, 8, D), (22, 1, 8), (22, 1, 8)))
    n = qf.prefix_workspace_bytes(p)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda").zero_()
    table = torch.where(sh.ptab >= 0, sh.ptab + FAR, sh.ptab).cuda()
    qf.prefix_partial(q, kc, vc, table, sh.plen.cuda(), sh.off.cuda(), o, m, l, p, sh.NG, sh.ptab.shape[1], ws, n)
    torch.cuda.synchronize()
    assert qf.prompt_status(ws) == 0
    ro, rm, rl = partial64(sh, q)
    assert err(o[:, 0], ro, False) <= ENG_OUT and err(m[:, 0], rm, True) <= ENG_LSE and err(l[:, 0], rl, True) <= ENG_LSE
