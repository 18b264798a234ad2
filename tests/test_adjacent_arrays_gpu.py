"""A decode step whose shard arrays lie directly behind one another in memory, as an allocator may place them."""
import pytest
import torch

from paper_2608_15473_b200 import binding as qf
from paper_2608_15473_b200 import build as qf_build
from prompt_testlib import D, Paged, attend64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    qf_build.build()


@pytest.mark.parametrize("group", range(1, 9))
@pytest.mark.parametrize("first", ["lse", "m"])
def test_log_sums_behind_the_vectors(group, first):
    """One request, one shard, one KV head: the unit is not cut, and its log-sum-exps follow its vectors as a segment's
    (maximum, sum) pairs follow theirs in the workspace.  The merged result is the shard's own state, bit for bit."""
    pg = Paged([0], [64], 1, seed=group)
    q = torch.randn((1, group, D), generator=torch.Generator().manual_seed(group)).to(torch.bfloat16)
    p = qf.params(1, group, 1, pg.width, 1, pg.num_pages)
    buf = torch.zeros(group * (D + 2), device="cuda")
    o, a, b = buf[:group * D], buf[group * D:group * (D + 1)], buf[group * (D + 1):]
    lse_part, m_part = (a, b) if first == "lse" else (b, a)
    out, lse = torch.zeros((1, group, D), device="cuda"), torch.zeros((1, group), device="cuda")
    ws = torch.full((qf.workspace_bytes(p),), 0xA5, dtype=torch.uint8, device="cuda")
    kc, vc = pg.pools()
    ranges = torch.tensor([[[0, 64]]], dtype=torch.int32).cuda()
    qf.decode_step(q.cuda(), kc, vc, pg.table.cuda(), pg.lens.cuda(), ranges, None, o, m_part, lse_part, out, lse, p, ws, ws.numel())
    torch.cuda.synchronize()
    assert torch.equal(out.flatten(), o) and ((lse[0] - lse_part).abs() <= 1e-6 * lse_part.abs()).all()
    ref = attend64(q.double(), pg.rows(0, 64, "k"), pg.rows(0, 64, "v"), [64])
    assert float((out.cpu().double() - ref["out"]).abs().max()) < 5e-5
    assert float((lse.cpu().double() - ref["lse"]).abs().max()) < 1e-5
