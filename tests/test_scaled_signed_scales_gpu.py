"""Scales below zero, which only other software leaves in a scaled cache: the calls that read take them like any, and placing
behind them keeps what they stand for."""
import pytest
import torch

from paper_2608_15473_b200 import binding as qf
from paper_2608_15473_b200 import build as qf_build
from prompt_testlib import D, PAGE, prompt64
from scaled_testlib import KINDS, Scaled, codes_of, numbers, scale_for, step_of
from test_prompt_attend_gpu import compare
from test_scaled_decode_gpu import KERNELS
from test_scaled_decode_gpu import check as check_decode
from test_scaled_prompt_gpu import attend
from test_scaled_prompt_gpu import queries as prompt_queries

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    qf_build.build()


def signed(pg, seed=3):
    """Half of the blocks get the negative of their scale, and so stand for the negative numbers."""
    g = torch.Generator().manual_seed(seed)
    for w in (0, 1):
        pg.scale[w] = pg.scale[w] * (1 - 2 * torch.randint(0, 2, pg.scale[w].shape, generator=g))
    pg.k, pg.v = (numbers(c, pg.kind) * s.double()[:, :, None, None] for c, s in zip(pg.codes, pg.scale))
    return pg


def place(pg, rows, scales=None):
    """The same rows as keys and as values behind what pg holds, neither normed nor turned: a row is its own fp32 result."""
    x = rows.to(torch.bfloat16).cuda()
    pools = pg.device()
    if scales is not None:
        pools[2], pools[3] = (s.float().cuda() for s in scales)
    p = qf.params(pg.B, 2 * pg.Hkv, pg.Hkv, pg.width, 1, pg.num_pages, flags=qf.QF_FLAG_KV_NHD if pg.nhd else 0)
    qf.rope_append_scaled(None, x, x, None, None, *pools, pg.table.cuda(), pg.cu.cuda(), pg.lens.cuda(), None, None, None, None, None, None, p,
                          qf.rope_params(pg.total, 0), kv_type=pg.type)
    torch.cuda.synchronize()
    order = (0, 2, 1, 3) if pg.nhd else (0, 1, 2, 3)
    return [c.cpu().permute(order).contiguous() for c in pools[:2]], [s.cpu().double() for s in pools[2:]], x.cpu().double().reshape(pg.total, pg.Hkv, D)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("scales", ["power", "any"])
@pytest.mark.parametrize("size", [0.01, 3.0, 50.0])
@pytest.mark.parametrize("nhd", [False, True])
def test_placing_behind_rows_of_a_negative_scale(kind, scales, size, nhd):
    """Rows that fit, rows that make some scales grow, and rows that make all grow."""
    pg = signed(Scaled([3, 2, 1, 4, 1], [5, 8, 1, 12, 31], 2, kind, nhd, scales=scales, seed=6))
    g = torch.Generator().manual_seed(4)
    codes, scale, rows = place(pg, torch.randn((pg.total, pg.Hkv * D), generator=g) * size)
    grown = kept = 0
    for w in (0, 1):
        for b in range(pg.B):      # each request's new rows lie in one page
            held, n = pg.cached[b] % PAGE, pg.new[b]
            page, at = int(pg.table[b, pg.cached[b] // PAGE]), slice(int(pg.cu[b]), int(pg.cu[b]) + n)
            y, old, new = rows[at].transpose(0, 1), pg.scale[w][page].double(), scale[w][page]
            need = scale_for(y.abs().amax(dim=(1, 2)), kind)
            want = torch.where(old.abs() >= need, old, need)
            assert torch.equal(new, want)
            grown, kept = grown + int((want != old).sum()), kept + int(((want == old) & (old < 0)).sum())
            # half a step; a caller's scale that is no power of two takes one or two fp32 roundings more
            for got, z in ((numbers(codes[w][page][:, held:held + n], kind), y / new[:, None, None]),
                           (numbers(codes[w][page][:, :held], kind), numbers(pg.codes[w][page][:, :held], kind) * (old / new)[:, None, None])):
                assert ((got - z).abs() <= 0.5 * step_of(z * (1 + 1e-9), kind) + 2.0 ** -22 * z.abs()).all()
                if scales == "power":
                    assert torch.equal(got, numbers(codes_of(z, kind), kind))
            still = want == old
            assert torch.equal(codes[w][page][still][:, :held], pg.codes[w][page][still][:, :held])
    assert (kept > 0 or size == 50.0) and (grown > 0 or size == 0.01)


def test_the_most_negative_integer_under_a_negative_scale():
    """-128 * -0.999 / 1 is nearer to 128 than to 127, and no code is 128: the largest one stands for it."""
    pg = Scaled([1], [4], 1, "int8")
    page = int(pg.table[0, 0])
    for w in (0, 1):
        pg.codes[w][page], pg.scale[w][page] = 0x80, -0.999
    codes, scale, _ = place(pg, torch.full((1, D), 127.0))
    for w in (0, 1):
        assert scale[w][page, 0] == 1 and (numbers(codes[w][page, 0, :5], "int8") == 127).all()


@pytest.mark.parametrize("kind", KINDS)
def test_scales_that_hold_nothing_readable(kind):
    """Zeros of both signs hold zeros, infinities of both signs and NaN make their block NaN."""
    odd = [0.0, -0.0, float("inf"), -float("inf"), float("nan")]
    pg = Scaled([1] * 5, [4] * 5, 1, kind)
    scales = [s.clone() for s in pg.scale]
    for b, x in enumerate(odd):
        scales[0][int(pg.table[b, 0])] = scales[1][int(pg.table[b, 0])] = x
    codes, scale, rows = place(pg, torch.ones((5, D)), scales)
    for w in (0, 1):
        for b in range(5):
            page = int(pg.table[b, 0])
            if b < 2:
                assert scale[w][page, 0] == scale_for(torch.ones(1), kind) and (numbers(codes[w][page, 0, :4], kind) == 0).all()
                assert (numbers(codes[w][page, 0, 4], kind) * scale[w][page, 0] == 1).all()
            else:
                assert torch.isnan(scale[w][page, 0])


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("flags", KERNELS)
@pytest.mark.parametrize("scales", ["power", "any"])
def test_decode_and_prompts_read_them(kind, flags, scales):
    check_decode(signed(Scaled([0] * 3, [300, 33, 1000], 2, kind, seed=8, scales=scales)), 8, 2, flags)
    if scales == "power":      # (with others the expansion to bf16 rounds, which the tests of prompts cover)
        pg = signed(Scaled([40, 130], [0, 77], 2, kind, seed=9))
        q = prompt_queries(pg, 8)
        out, lse, _ = attend(pg, q, flags)
        compare(out, lse, prompt64(pg, q))
