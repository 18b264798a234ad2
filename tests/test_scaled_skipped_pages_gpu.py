"""The scaled decode sweep over pages that count for nothing, behind pages whose every score is far below zero: pages without a
valid table entry, and pages whose scores are -infinity."""
import pytest
import torch

from paper_2608_15473_b200 import binding as qf
from paper_2608_15473_b200 import build as qf_build
from prompt_testlib import D, PAGE
from scaled_testlib import KINDS, Scaled, codes_of, even_ranges, numbers, scale_for
from test_scaled_decode_gpu import KERNELS, close, lse_close, step

pytestmark = pytest.mark.gpu

# pages of a request and those that count for nothing; a stage of the sweep is 16 pages, two of them for each warp
GONE = {"the last, odd page": (17, [16]), "a pair": (20, [16, 17]), "another warp's pair": (32, [22, 23]),
        "a whole stage": (32, list(range(16, 32))), "half a pair": (32, [19, 24])}


@pytest.fixture(scope="module", autouse=True)
def built():
    qf_build.build()


def far_below(pages, hkv, kind, B=None):
    """So many requests that many of them are swept whole by one CTA; every key near -1 and queries near 13: scores near -147."""
    B = B or 160 // hkv
    pg = Scaled([0] * B, [pages * PAGE] * B, hkv, kind, seed=pages)
    g = torch.Generator().manual_seed(21)
    x = -1 + 0.03 * torch.randn(pg.codes[0].shape, generator=g, dtype=torch.float64)
    s = scale_for(x.abs().amax(dim=(2, 3)), kind)
    pg.codes[0], pg.scale[0] = codes_of(x / s[:, :, None, None], kind), s.float()
    pg.k = numbers(pg.codes[0], kind) * s[:, :, None, None]
    return pg


def check(pg, group, got, keep):
    """Against softmax attention over the kept positions in 64 bits.  A score is off by 2^-20 of sum |q_i k_i| at most, its weight
    relatively as much, the normalised sum by twice that of sum w |v|; the weights' rounding as in the decode tests."""
    assert torch.isfinite(got["o"]).all() and torch.isfinite(got["out"]).all() and torch.isfinite(got["lse"]).all()
    for b in range(0, pg.B, 9):
        n = pg.cached[b]
        k, v = (pg.rows(b, n, w)[:, keep] for w in "kv")
        x = got["q"][b].cpu().double().reshape(pg.Hkv, group, D)
        sc = torch.einsum("cgd,cnd->cgn", x, k) * D ** -0.5
        assert float(sc.max()) < -100
        err = 2.0 ** -20 * torch.einsum("cgd,cnd->cgn", x.abs(), k.abs()).amax(-1) * D ** -0.5
        w = torch.softmax(sc, -1)
        slack = (2 * err[..., None] + 2.0 ** -19) * torch.einsum("cgn,cnd->cgd", w, v.abs()) + 2.0 ** -35 * v.abs().amax(1)[:, None]
        out, lse = torch.einsum("cgn,cnd->cgd", w, v).reshape(-1, D), torch.logsumexp(sc, -1).reshape(-1)
        for name, of in (("o", got["o"][b, 0]), ("out", got["out"][b])):
            close(of, out, slack.reshape(-1, D) + 2.0 ** -20 * out.abs())
        lse_close(got["l"][b, 0], lse, err.reshape(-1))
        lse_close(got["lse"][b], lse, err.reshape(-1))


def run(pg, group, flags, **kw):
    g = torch.Generator().manual_seed(22)
    q = (13 + 0.2 * torch.randn((pg.B, pg.Hkv * group, D), generator=g)).to(torch.bfloat16).cuda()
    return dict(step(pg, q, even_ranges(pg.cached, 1), flags, **kw), q=q)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("flags", KERNELS)
@pytest.mark.parametrize("group,hkv", [(4, 2), (7, 2), (1, 1)])
@pytest.mark.parametrize("gone", GONE)
def test_pages_without_a_table_entry(kind, flags, group, hkv, gone):
    pages, bad = GONE[gone]
    pg = far_below(pages, hkv, kind)
    table = pg.table.clone()
    pg.table[:, bad] = -1
    got = run(pg, group, flags)
    pg.table = table
    check(pg, group, got, torch.tensor([i for i in range(pages * PAGE) if i // PAGE not in bad]))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("flags", KERNELS)
@pytest.mark.parametrize("group,hkv", [(4, 2), (7, 2)])
@pytest.mark.parametrize("gone", GONE)
def test_pages_whose_scores_are_minus_infinity(kind, flags, group, hkv, gone):
    """An infinite scale of keys against products that are all negative."""
    pages, bad = GONE[gone]
    pg = far_below(pages, hkv, kind)
    kc, vc, ks, vs = pg.device()
    ks[pg.table[:, bad].long().flatten().cuda()] = float("inf")
    got = run(pg, group, flags, pools=(kc, vc, ks, vs))
    check(pg, group, got, torch.tensor([i for i in range(pages * PAGE) if i // PAGE not in bad]))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("flags", KERNELS)
@pytest.mark.parametrize("group,hkv", [(4, 2), (7, 2)])
@pytest.mark.parametrize("gone", [[0], [0, 1, 2, 3], list(range(16))])
def test_a_sweep_that_begins_with_scores_of_minus_infinity(kind, flags, group, hkv, gone):
    pg = far_below(20, hkv, kind, B=40)
    kc, vc, ks, vs = pg.device()
    ks[pg.table[:, gone].long().flatten().cuda()] = float("inf")
    got = run(pg, group, flags, pools=(kc, vc, ks, vs))
    check(pg, group, got, torch.tensor([i for i in range(20 * PAGE) if i // PAGE not in gone]))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("flags", KERNELS)
@pytest.mark.parametrize("group,hkv", [(4, 2), (7, 2)])
def test_a_shard_whose_every_score_is_minus_infinity_is_empty(kind, flags, group, hkv):
    pg = far_below(20, hkv, kind, B=3)
    kc, vc, ks, vs = pg.device()
    ks[:] = float("inf")
    got = run(pg, group, flags, pools=(kc, vc, ks, vs))
    assert (got["o"] == 0).all() and (got["out"] == 0).all()
    assert all(torch.isneginf(got[n]).all() for n in ("m", "l", "lse"))
