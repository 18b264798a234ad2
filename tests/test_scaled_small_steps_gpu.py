"""Which decode steps over a scaled cache are small (sweep and one merging kernel, two launches): those whose units, ends of ranges
included, stay within 16 per SM by the parameters alone.  Both kinds of step against 64 bits."""
import pytest
import torch

from paper_2608_15473_b200 import binding as qf
from paper_2608_15473_b200 import build as qf_build
from scaled_testlib import KINDS, Scaled, even_ranges
from test_scaled_decode_gpu import check, queries, step

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    qf_build.build()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("hkv,shards,tokens", [(8, 1, 200), (4, 1, 500), (2, 3, 100), (1, 1, 2300)])
@pytest.mark.parametrize("side", [-1, 0, 1])
def test_at_the_border(kind, hkv, shards, tokens, side):
    """A shard takes a unit for each 256 positions that its request could have, and one for its end, in every KV head."""
    limit = 16 * min(torch.cuda.get_device_properties(0).multi_processor_count, 160)
    batch = limit // (shards * hkv * (-(-tokens // 256) + 1)) + side
    pg = Scaled([0] * batch, [tokens] * batch, hkv, kind, seed=batch)
    if hkv > 4 or tokens > 1000:
        step(pg, queries(batch, 2 * hkv), even_ranges(pg.cached, shards))
    else:
        check(pg, 2 * hkv, shards)
    # the plan kernel of many (request, shard) pairs is a launch of its own, and such steps are never small
    assert qf.last_launch_count() == (3 if side > 0 or batch * shards > 2048 else 2) + (batch * shards > 2048)
