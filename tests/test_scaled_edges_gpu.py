"""The scaled cache's operators on calls that are allowed and unusual: pools beyond 2^32 bytes, integer codes of every value, two
streams at once, rows that no request owns, scales that other software left, blocks filled by several calls."""
import numpy as np
import pytest
import torch

from paper_2608_15473_b200 import binding as qf
from paper_2608_15473_b200 import build as qf_build
from prompt_testlib import D, PAGE, prompt64
from scaled_testlib import KINDS, Scaled, even_ranges, merge64, numbers, states64
from test_prompt_attend_gpu import compare
from test_scaled_decode_gpu import check, close, lse_close, queries, step
from test_scaled_place_gpu import run
from test_scaled_prompt_gpu import attend
from test_scaled_prompt_gpu import queries as prompt_queries

pytestmark = pytest.mark.gpu
HKV, FAR = 4, (5 << 30) // (4 * PAGE * D)      # pages before the first that is used: 5 GB


@pytest.fixture(scope="module", autouse=True)
def built():
    qf_build.build()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("nhd", [False, True])
def test_far_pages(kind, nhd):
    """Placing, the decode step and prompts on pages that all lie beyond 2^32 bytes, against the same on near ones."""
    pg = Scaled([70, 1, 130], [40, 300, 0], HKV, kind, nhd, seed=3)
    near = pg.device()
    far = []
    for x in near:
        big = torch.full((FAR + pg.num_pages, *x.shape[1:]), 0x7f if x.dtype == torch.uint8 else float("nan"), dtype=x.dtype, device="cuda")
        big[FAR:] = x
        far.append(big)
    assert far[0][:FAR].numel() > 1 << 32
    T, hq = pg.total, 8
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn((T, h, D), generator=g).to(torch.bfloat16).cuda() for h in (hq, HKV, HKV))
    table = torch.where(pg.table >= 0, pg.table + FAR, pg.table)
    qo, flags = torch.empty_like(q), qf.QF_FLAG_KV_NHD if nhd else 0
    for pools, tab, pages in ((near, pg.table, pg.num_pages), (far, table, FAR + pg.num_pages)):
        qf.rope_append_scaled(q, k, v, qo, None, *pools, tab.cuda(), pg.cu.cuda(), pg.lens.cuda(), None, None, None, None, None, None,
                              qf.params(pg.B, hq, HKV, pg.width, 1, pages, flags=flags), qf.rope_params(T, 0), kv_type=pg.type)
    torch.cuda.synchronize()
    for x, y in zip(near, far):
        assert torch.equal(x, y[FAR:])
    assert (far[0][FAR - 1] == 0x7f).all() and torch.isnan(far[2][:FAR:997]).all()
    order = (0, 2, 1, 3) if nhd else (0, 1, 2, 3)
    pg.k, pg.v = (numbers(near[w].cpu().permute(order), kind) * near[2 + w].cpu().double()[:, :, None, None] for w in (0, 1))
    ref = prompt64(pg, q)
    qd, ranges = queries(3, hq), even_ranges(pg.cached, 2)
    want = states64(pg, qd.cpu(), ranges)
    pg.table, pg.num_pages = table, FAR + pg.num_pages
    for extra in (0, qf.QF_FLAG_SIMPLE_KERNEL):
        out, lse, status = attend(pg, q, extra | qf.QF_FLAG_CHECK_BOUNDS, pools=far)
        assert status == 0
        compare(out, lse, ref)
        got = step(pg, qd, ranges, extra | qf.QF_FLAG_CHECK_BOUNDS, pools=far)
        assert got["status"] == 0
        close(got["o"], want["out"], want["slack"])
        lse_close(got["l"], want["lse"], want["lse_slack"])


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("flags", [0, qf.QF_FLAG_SIMPLE_KERNEL])
def test_every_code(kind, flags):
    """All 256 codes but the two that are not numbers, -128 among the integers, at places of every alignment."""
    pg = Scaled([0, 0], [290, 33], 2, kind, seed=4)
    g = torch.Generator().manual_seed(4)
    for w in (0, 1):
        c = torch.randint(0, 256, pg.codes[w].shape, generator=g, dtype=torch.int32).to(torch.uint8)
        if kind == "e4m3":
            c[(c & 0x7f) == 0x7f] = 0x80      # (a negative zero)
        pg.codes[w] = c
        pg.scale[w] = torch.full_like(pg.scale[w], 2.0 ** -9 if kind == "e4m3" else 2.0 ** -6)
    pg.k, pg.v = (numbers(c, kind) * s.double()[:, :, None, None] for c, s in zip(pg.codes, pg.scale))
    check(pg, 8, 2, flags)
    pg.new, pg.cached, pg.total = [140, 20], [150, 13], 160
    pg.cu, pg.lens = torch.tensor([0, 140, 160], dtype=torch.int32), torch.tensor([150, 13], dtype=torch.int32)
    q = prompt_queries(pg, 8)
    out, lse, _ = attend(pg, q, flags)
    compare(out, lse, prompt64(pg, q))


@pytest.mark.parametrize("kind", KINDS)
def test_two_steps_at_once_on_two_streams(kind):
    """Workspaces and outputs of their own: neither sees the other."""
    pgs = [Scaled([0] * 6, [1500, 3, 700, 64, 2000, 31], 4, kind, seed=s) for s in (5, 6)]
    q, ranges = queries(6, 16), even_ranges(pgs[0].cached, 2)
    want = [step(pg, q, ranges) for pg in pgs]
    pools = [pg.device() for pg in pgs]
    tables, lens, rng, p = [pg.table.cuda() for pg in pgs], pgs[0].lens.cuda(), ranges.cuda(), want[0]["p"]
    outs = [[torch.zeros_like(w[n]) for n in ("o", "m", "l", "out", "lse")] for w in want]
    wss = [torch.empty(qf.workspace_bytes(p), dtype=torch.uint8, device="cuda") for _ in pgs]
    streams = [torch.cuda.Stream() for _ in pgs]
    torch.cuda.synchronize()
    for _ in range(5):
        for i, s in enumerate(streams):
            qf.decode_step_scaled(q, *pools[i], tables[i], lens, rng, None, *outs[i], p, wss[i], wss[i].numel(), kv_type=pgs[i].type, stream=s)
    torch.cuda.synchronize()
    for w, o in zip(want, outs):
        assert torch.equal(w["out"], o[3]) and torch.equal(w["lse"], o[4]) and torch.equal(w["o"], o[0])


@pytest.mark.parametrize("kind", KINDS)
def test_rows_before_the_first_and_behind_the_last_request(kind):
    """cu_tokens that starts behind row 0: rows of no request are not touched, whatever they hold."""
    pg = Scaled([20, 7], [3, 0], 2, kind, seed=7)
    lead, T, hq = 5, 40, 4
    g = torch.Generator().manual_seed(7)
    q, k, v = (torch.randn((T, h, D), generator=g).to(torch.bfloat16) for h in (hq, 2, 2))
    p, r = qf.params(2, hq, 2, pg.width, 1, pg.num_pages), qf.rope_params(T, 0)
    a, b = pg.device(), pg.device()
    qa, qb = torch.full((T, hq, D), 9.0, dtype=torch.bfloat16, device="cuda"), torch.full((27, hq, D), 9.0, dtype=torch.bfloat16, device="cuda")
    kk = k.clone()
    kk[:lead], kk[lead + 27:] = float("nan"), float("inf")
    tail = (pg.table.cuda(),)
    qf.rope_append_scaled(q.cuda(), kk.cuda(), v.cuda(), qa, None, *a, *tail, (pg.cu + lead).cuda(), pg.lens.cuda(), None, None, None, None, None,
                          None, p, r, kv_type=pg.type)
    mid = slice(lead, lead + 27)
    qf.rope_append_scaled(q[mid].contiguous().cuda(), k[mid].contiguous().cuda(), v[mid].contiguous().cuda(), qb, None, *b, *tail, pg.cu.cuda(),
                          pg.lens.cuda(), None, None, None, None, None, None, p, qf.rope_params(27, 0), kv_type=pg.type)
    torch.cuda.synchronize()
    assert torch.equal(qa[mid], qb) and (qa[:lead] == 9).all() and (qa[lead + 27:] == 9).all()
    for x, y in zip(a, b):
        assert torch.equal(x, y)


@pytest.mark.parametrize("kind", KINDS)
def test_many_requests_of_odd_lengths(kind):
    """Runs of every length side by side in a tile of 16 rows, empty requests among them."""
    r = np.random.default_rng(5)
    new = r.integers(0, 24, 90)
    run(Scaled(new, r.integers(0, 40, 90), 3, kind, True, seed=8), 6, seed=8)
    run(Scaled([15, 1] * 30, [1, 14] * 30, 2, kind, seed=9), 4, seed=9)
    run(Scaled([16] * 40, [8] * 40, 1, kind, seed=10), 1, seed=10)


@pytest.mark.parametrize("kind", KINDS)
def test_shared_pages_are_read_by_many(kind):
    """Several requests whose tables name the same pages."""
    pg = Scaled([0] * 4, [200, 200, 200, 200], 2, kind, seed=11)
    pg.table[1:] = pg.table[0]
    check(pg, 8, 2)


@pytest.mark.parametrize("kind", KINDS)
def test_overlapping_shards_and_a_second_call_on_the_same_workspace(kind):
    pg = Scaled([0, 0], [500, 90], 2, kind, seed=12)
    q, ranges = queries(2, 8), torch.tensor([[[0, 500], [100, 400], [499, 500]], [[0, 90], [0, 90], [89, 90]]], dtype=torch.int32)
    a = check(pg, 8, 3, ranges=ranges)
    other = Scaled([0, 0], [77, 300], 2, kind, seed=13)
    step(other, q, even_ranges(other.cached, 3), ws=a["ws"])
    b = step(pg, q, ranges, ws=a["ws"])
    assert torch.equal(a["out"], b["out"]) and torch.equal(a["o"], b["o"])
    ref = states64(pg, q.cpu(), ranges)
    out, lse, slack, lse_slack = merge64(ref)
    close(b["out"], out, slack + 2.0 ** -20 * out.abs())
