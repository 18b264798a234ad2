"""Blocks of a scaled cache filled token by token with rows of rising magnitude: what is left of the first rows."""
import numpy as np
import pytest
import torch

from paper_2608_15473_b200 import binding as qf
from paper_2608_15473_b200 import build as qf_build
from prompt_testlib import D, PAGE
from scaled_testlib import KINDS, Scaled, numbers

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    qf_build.build()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("factor", [1.0, 1.3, 2.0, 8.0])
@pytest.mark.parametrize("chunk", [1, 3])
def test_the_first_rows_stay_within_their_bound(kind, factor, chunk):
    """A row, neither normed nor turned, is its own fp32 result.  At any time it is off by at most 2^-4 of itself or 2^-9 of its
    block's present scale (e4m3), or by one scale (int8)."""
    B, hkv = 8, 2
    pg = Scaled([0] * B, [PAGE] * B, hkv, kind)
    pools, table = pg.device(), pg.table.cuda()
    p = qf.params(B, 2 * hkv, hkv, pg.width, 1, pg.num_pages)
    g = torch.Generator().manual_seed(5)
    rows = (torch.randn((B, PAGE, hkv, D), generator=g) * factor ** torch.arange(PAGE)[None, :, None, None]).to(torch.bfloat16)
    for start in range(0, PAGE, chunk):
        n = min(chunk, PAGE - start)
        x = rows[:, start:start + n].reshape(B * n, hkv * D).cuda()
        qf.rope_append_scaled(None, x, x, None, None, *pools, table, torch.arange(0, B * n + 1, n, dtype=torch.int32).cuda(),
                              torch.full((B,), start, dtype=torch.int32).cuda(), None, None, None, None, None, None, p, qf.rope_params(B * n, 0),
                              kv_type=pg.type)
        torch.cuda.synchronize()
        y = rows[:, :start + n].double()
        for w in (0, 1):
            s = pools[2 + w].cpu().double()[pg.table[:, 0].long()][:, None, :, None]
            got = numbers(pools[w].cpu()[pg.table[:, 0].long()], kind)[:, :, :start + n].transpose(1, 2) * s
            bound = torch.maximum(2.0 ** -4 * y.abs(), 2.0 ** -9 * s) if kind == "e4m3" else s.expand_as(y)
            assert ((got - y).abs() <= bound).all(), (start, w, float(((got - y).abs() / bound).max()))
    assert np.log2(float(pools[2].max())) > -9
