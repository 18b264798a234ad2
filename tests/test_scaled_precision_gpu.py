"""Where the 16-bit floats of the scaled decode sweep end: queries with one channel far above the others, and weights far below
those of the neighbouring page, on both sides of each limit.  The limits are those of include/qf.h."""
import pytest
import torch

from paper_2608_15473_b200 import build as qf_build
from prompt_testlib import D, PAGE
from scaled_testlib import KINDS, Scaled, even_ranges, numbers
from test_scaled_decode_gpu import KERNELS, close, lse_close, step

pytestmark = pytest.mark.gpu
ONE = {"e4m3": 0x38, "int8": 1}
MINUS_ONE = {"e4m3": 0xb8, "int8": 0xff}


@pytest.fixture(scope="module", autouse=True)
def built():
    qf_build.build()


def expect(pg, q, f, score_error, v_error):
    """softmax attention in 64 bits over every position, and what is allowed beside it: score_error [B, Hkv, G, n] for each score, and
    v_error [B, Hkv, G, D] for the weighted sums.  Both sides of the quotient move with a score, so weights by e^(2 err)."""
    outs, lses, slacks, lse_slacks = [], [], [], []
    for b in range(pg.B):
        k, v = (pg.rows(b, pg.cached[b], w) for w in "kv")
        x = q[b].double().reshape(pg.Hkv, -1, D)
        sc = torch.einsum("cgd,cnd->cgn", x, k) * f
        err = 2.0 ** -20 * torch.einsum("cgd,cnd->cgn", x.abs(), k.abs()) * f + score_error(x, k)
        w = torch.softmax(sc, -1)
        outs.append(torch.einsum("cgn,cnd->cgd", w, v).reshape(-1, D))
        lses.append(torch.logsumexp(sc, -1).reshape(-1))
        e = err.amax(-1)
        spread = torch.einsum("cgn,cnd->cgd", w, v.abs())
        slacks.append(((torch.expm1(2 * e)[..., None] + 2.0 ** -19) * spread + v_error(sc, w, v)).reshape(-1, D))
        lse_slacks.append(e.reshape(-1))
    return [torch.stack(t) for t in (outs, lses, slacks, lse_slacks)]


def compare(got, want):
    out, lse, slack, lse_slack = want
    close(got["out"], out, slack + 2.0 ** -20 * out.abs())
    close(got["o"][:, 0], out, slack + 2.0 ** -20 * out.abs())
    lse_close(got["lse"], lse, lse_slack)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("flags", KERNELS)
@pytest.mark.parametrize("group", [4, 7])
@pytest.mark.parametrize("below", [20, 31, 33, 36, 38])
def test_channels_far_below_the_largest(kind, flags, group, below):
    """The largest channel meets keys that are 0 there, so the small ones alone make the scores.  A channel is exact down to 2^-31
    of the largest (f16 steps end at 2^-24, the largest channel is brought to [2^14, 2^15), eight bits need an exponent of -17);
    below it is off by half a last step: 2^-39 of the largest."""
    pg = Scaled([0, 0], [300, 77], 2, kind)
    pg.codes[0][..., 5] = 0
    pg.k = numbers(pg.codes[0], kind) * pg.scale[0].double()[:, :, None, None]
    g = torch.Generator().manual_seed(below)
    q = (1 + torch.rand((2, 2 * group, D), generator=g)) * (1 - 2 * torch.randint(0, 2, (2, 2 * group, D), generator=g)) * 2.0 ** -below
    q[..., 5] = 1.0
    q = q.to(torch.bfloat16)      # (a rounding up to 2 * 2^-below keeps a single bit)
    f = 0.03 * 2.0 ** below       # scores of about 0.5
    got = step(pg, q.cuda(), even_ranges(pg.cached, 1), flags, sm_scale=f)
    lost = 2.0 ** -39 if below > 31 else 0.0
    compare(got, expect(pg, q, f, lambda x, k: lost * k.abs().sum(-1)[:, None] * f, lambda sc, w, v: 0.0))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("flags", KERNELS)
@pytest.mark.parametrize("group", [4, 7])
@pytest.mark.parametrize("below", [3.3, 10.7, 16.6, 22.3, 30.3, 36.4])
def test_weights_far_below_the_neighbouring_pages(kind, flags, group, below):
    """Two pages of one warp step; the second's weights are 2^-below of the first's and its values 2^(2 below) larger, so that
    the result is the second's.  A weight is off by 2^-22 of itself, or by 2^-39 of the largest of the two pages: 22 bits down to
    2^-17 of it, and 39 - below further down."""
    pg = Scaled([0, 0], [2 * PAGE, 2 * PAGE], 2, kind)
    for b in range(2):
        one, two = (int(x) for x in pg.table[b, :2])
        pg.codes[0][[one, two]] = 0
        pg.codes[0][one, ..., 9], pg.codes[0][two, ..., 9] = ONE[kind], MINUS_ONE[kind]
        pg.scale[0][[one, two]] = 1.0
        pg.scale[1][two] = pg.scale[1][one] * 2.0 ** round(2 * below)
    pg.k, pg.v = (numbers(c, kind) * s.double()[:, :, None, None] for c, s in zip(pg.codes, pg.scale))
    q = torch.zeros((2, 2 * group, D), dtype=torch.bfloat16)
    q[..., 9] = 1.0
    f = below / 2 * float(torch.log(torch.tensor(2.0)))      # scores f and -f
    got = step(pg, q.cuda(), even_ranges(pg.cached, 1), flags, sm_scale=f)
    lost = 2.0 ** -39 if below > 17 else 0.0
    compare(got, expect(pg, q, f, lambda x, k: 0.0,
                        lambda sc, w, v: lost * w.amax(-1)[..., None] * v.abs().sum(1)[:, None]))
