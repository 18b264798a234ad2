"""qf_prompt_attend on the GPU against softmax attention in 64 bits: every element, both kernels."""
import numpy as np
import pytest
import torch

from paper_2608_15473_b200 import binding as qf
from paper_2608_15473_b200 import build as qf_build
from prompt_testlib import D, PAGE, Paged, prompt64

pytestmark = pytest.mark.gpu
KERNELS = [pytest.param(0, id="staged"), pytest.param(qf.QF_FLAG_SIMPLE_KERNEL, id="simple")]


@pytest.fixture(scope="module", autouse=True)
def built():
    qf_build.build()


def compare(out, lse, ref):
    """out is rounded once to bf16 (2^-8 of the value at most) and each weight once (2^-8 of it at most, so
    2^-8 sum w|v| in all); fp32 scores, sums and exponentials add a few 2^-20 of sum w|v|.  Rounding errors are spread
    evenly over half a step, so their root mean square is 1/sqrt(3) of the bound, weights' errors being independent:
    1.5 times that for the whole output.  lse carries the boundary's contract of 1e-5."""
    got = out.cpu().double()
    r, spread = ref["out"], ref["spread"]
    tol = 2.0 ** -8 * (r.abs() + spread) + 16 * 2.0 ** -20 * spread
    fine = torch.isfinite(r)
    assert torch.equal(torch.isnan(got), torch.isnan(r)) and torch.equal(got[~fine & ~torch.isnan(r)], r[~fine & ~torch.isnan(r)])
    err = (got - r).abs()
    bad = fine & (err > tol)
    assert not bad.any(), (int(bad.sum()), float(err[fine].max()))
    rms = float((err[fine] ** 2).mean().sqrt())
    want = 2.0 ** -8 / 3 ** 0.5 * float((r[fine] ** 2 + ref["noise"][fine]).mean().sqrt()) + 2.0 ** -20 * float(spread[fine].mean())
    assert rms <= 1.5 * want, (rms, want)
    l, rl = lse.cpu().double(), ref["lse"]
    ok = torch.isfinite(rl)
    assert ((l - rl).abs()[ok] <= 1e-5 * rl.abs().clamp(min=1.0)[ok]).all(), float((l - rl).abs()[ok].max())


def attend(pg, q, flags=0, sm_scale=0.0, pad=0, q_stride=0, identity=False, max_seq_len=0, ws=None, pools=None, stream=None):
    hq = q.shape[1]
    T = pg.total + pad
    p = qf.params(pg.B, hq, pg.Hkv, pg.width, 1, pg.num_pages, flags=flags | (qf.QF_FLAG_KV_NHD if pg.nhd else 0),
                  sm_scale=sm_scale, max_seq_len=max_seq_len)
    kc, vc = pools or pg.pools()
    out = torch.full((T, hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((T, hq), 7.0, device="cuda")
    n = qf.prompt_workspace_bytes(p, T)
    ws = torch.full((n,), 0xA5, dtype=torch.uint8, device="cuda") if ws is None else ws
    qf.prompt_attend(q, kc, vc, None if identity else pg.table.cuda(), pg.cu.cuda(), pg.lens.cuda(), out, lse, p, T, ws, n,
                     q_stride, stream)
    torch.cuda.synchronize()
    status = qf.prompt_status(ws)
    assert (out[pg.total:] == 7).all() and (lse[pg.total:] == 7).all()       # rows of no request stay as they were
    return out[:pg.total], lse[:pg.total], status


def queries(pg, hq, seed=5, scale=2.0, pad=0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((pg.total + pad, hq, D), generator=g) * scale).to(torch.bfloat16).cuda()


def check(pg, hq, flags=0, **kw):
    q = queries(pg, hq, pad=kw.get("pad", 0))
    out, lse, status = attend(pg, q, flags, **kw)
    assert status == 0
    compare(out, lse, prompt64(pg, q[:pg.total]))


@pytest.mark.parametrize("flags", KERNELS)
@pytest.mark.parametrize("hq,hkv", [(1, 1), (2, 1), (3, 1), (8, 2), (5, 1), (6, 1), (28, 4), (8, 1), (16, 8)])
@pytest.mark.parametrize("nhd", [False, True])
def test_every_group_size(flags, hq, hkv, nhd):
    check(Paged([70, 1, 0, 33, 150], [0, 40, 5, 129, 3], hkv, nhd, poison=True), hq, flags)


@pytest.mark.parametrize("flags", KERNELS)
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 130, 191, 255, 256, 257, 300, 513])
def test_short_prompts(flags, n):
    check(Paged([n], [0], 2, seed=n, poison=True), 8, flags)


@pytest.mark.parametrize("flags", KERNELS)
@pytest.mark.parametrize("cached", [0, 1, 15, 16, 100, 127, 128, 129, 255, 1000])
@pytest.mark.parametrize("n", [1, 16, 70])
def test_chunks_behind_a_cached_context(flags, cached, n):
    check(Paged([n, 1, n + 3], [cached, cached + 7, max(cached - 1, 0)], 2, nhd=cached % 2 == 1, seed=cached, poison=True), 8, flags)


@pytest.mark.parametrize("new,cached,hq,hkv", [
    ([1] * 40, [(37 * i) % 900 for i in range(40)], 8, 2),                 # decode steps only
    ([1] * 5 + [200, 1, 90], [2000, 3, 700, 64, 0, 50, 900, 0], 14, 2),    # decode steps riding with chunks
    ([2000], [0], 8, 2), ([700, 1300], [5000, 0], 4, 1),
    ([0, 0, 0, 5, 0], [3, 0, 9, 0, 1], 4, 2), ([3] * 300, [i % 70 for i in range(300)], 4, 2),
    ([1], [20000], 8, 1), ([7], [9000], 5, 1), ([130], [6000], 8, 1),
])
def test_batches(new, cached, hq, hkv):
    check(Paged(new, cached, hkv, poison=len(new) < 10), hq)


def test_strided_queries_and_padding_rows():
    pg = Paged([50, 90], [20, 0], 2)
    g = torch.Generator().manual_seed(9)
    rows = torch.randn((pg.total + 9, (8 + 4) * D), generator=g).to(torch.bfloat16).cuda()
    q = rows[:, :8 * D].unflatten(1, (8, D))
    out, lse, _ = attend(pg, q, pad=9, q_stride=rows.stride(0))
    compare(out, lse, prompt64(pg, q[:pg.total]))


@pytest.mark.parametrize("flags", KERNELS)
def test_scale_identity_table_and_length_bound(flags):
    pg = Paged([40, 20], [3, 30], 2, max_pages=4, extra_pages=8)
    pg.table = torch.arange(8, dtype=torch.int32).reshape(2, 4)
    pg.num_pages = pg.k.shape[0]
    q = queries(pg, 4)
    out, lse, _ = attend(pg, q, flags, identity=True)
    compare(out, lse, prompt64(pg, q))
    out, lse, _ = attend(pg, q, flags, identity=True, max_seq_len=37)       # nothing beyond the bound is attended
    compare(out, lse, prompt64(pg, q, max_tokens=37))


def test_explicit_scale():
    pg = Paged([90, 20], [3, 30], 2)
    q = queries(pg, 4)
    out, lse, _ = attend(pg, q, sm_scale=0.03)
    import prompt_testlib as lib
    keep, lib.attend64.__defaults__ = lib.attend64.__defaults__, (0.03,)
    try:
        compare(out, lse, prompt64(pg, q))
    finally:
        lib.attend64.__defaults__ = keep


@pytest.mark.parametrize("flags", KERNELS)
@pytest.mark.parametrize("scale", [8.0, 60.0])
def test_peaked_rows_and_growing_maxima(flags, scale):
    """Large scores, and keys that grow along the context so that every tile raises every row's maximum."""
    pg = Paged([300, 40], [500, 0], 2, seed=3)
    for b in range(2):
        for i in range(pg.new[b] + pg.cached[b]):
            pg.k[int(pg.table[b, i // PAGE]), :, i % PAGE] *= 0.02 + i / 400
    q = queries(pg, 4, scale=scale / 8)
    out, lse, _ = attend(pg, q, flags)
    compare(out, lse, prompt64(pg, q))


@pytest.mark.parametrize("flags", KERNELS)
def test_planted_token_is_seen_exactly_where_the_mask_allows(flags):
    """One position holds a key that takes all the weight: rows from it on return its value, rows before it do not."""
    for spot in [0, 1, 15, 16, 63, 64, 127, 128, 129, 200, 255, 256, 299]:
        pg = Paged([200], [100], 1, seed=spot)
        q = torch.full((200, 4, D), 1.0, dtype=torch.bfloat16, device="cuda")
        pg.k.mul_(0.01)
        page = int(pg.table[0, spot // PAGE])
        pg.k[page, 0, spot % PAGE] = 4.0
        out, lse, _ = attend(pg, q, flags)
        ref = prompt64(pg, q)
        compare(out, lse, ref)
        hit = max(spot - 100, 0)
        assert torch.equal(out.cpu()[hit:], pg.v[page, 0, spot % PAGE].expand_as(out[hit:]))


@pytest.mark.parametrize("flags", KERNELS)
def test_values_behind_the_mask_never_reach_a_row(flags):
    """NaN and infinities at positions of the request that come after a row: rows before them stay clean, rows that see
    them get them."""
    pg = Paged([150, 70], [60, 0], 2, seed=11)
    def put(b, i, ch, val):
        pg.v[int(pg.table[b, i // PAGE]), :, i % PAGE, ch] = val
    put(0, 130, 3, float("nan"))
    put(0, 190, 77, float("inf"))
    put(0, 195, 77, float("-inf"))
    put(1, 69, 5, float("inf"))
    put(1, 10, 6, float("-inf"))
    pg.k[int(pg.table[0, 201 // PAGE]), :, 201 % PAGE] = float("nan")        # a key: the rows that see it are NaN whole
    q = queries(pg, 4)
    out, lse, _ = attend(pg, q, flags)
    got, ref = out.cpu().double(), prompt64(pg, q)
    r = ref["out"]
    for a, b in ((torch.isnan(got), torch.isnan(r)), (torch.isposinf(got), torch.isposinf(r)), (torch.isneginf(got), torch.isneginf(r))):
        assert torch.equal(a, b)
    fine = torch.isfinite(r)
    tol = 2.0 ** -8 * (r.abs() + ref["spread"]) + 1e-4
    assert ((got - r).abs()[fine] <= tol[fine]).all()


@pytest.mark.parametrize("flags", KERNELS)
def test_bad_pages_contribute_nothing_and_are_reported(flags):
    pg = Paged([60], [200], 2, seed=2)
    q = queries(pg, 4)
    good = pg.table.clone()
    for entry, where in ((pg.num_pages, 2), (-1, 9), (2 ** 30, 15)):
        pg.table = good.clone()
        pg.table[0, where] = entry
        out, lse, status = attend(pg, q, flags | qf.QF_FLAG_CHECK_BOUNDS)
        assert status == qf.QF_STATUS_BAD_PAGE
        # the same request without that page's positions
        keep = [i for i in range(260) if i // PAGE != where]
        k, v = (torch.stack([(pg.k if w == "k" else pg.v)[int(good[0, i // PAGE]), :, i % PAGE] for i in keep], 1).double() for w in "kv")
        from prompt_testlib import attend64
        seen = [sum(1 for j in keep if j <= 200 + i) for i in range(60)]
        compare(out, lse, {n: t.cpu() for n, t in attend64(q.double(), k.cuda(), v.cuda(), seen).items()})
    pg.table = good
    assert attend(pg, q, flags | qf.QF_FLAG_CHECK_BOUNDS)[2] == 0


def test_repeatable_and_independent_of_the_workspace():
    pg = Paged([300, 1, 700], [900, 3000, 10], 2)
    q = queries(pg, 8)
    first = attend(pg, q)
    p = qf.params(pg.B, 8, pg.Hkv, pg.width, 1, pg.num_pages)
    ws = torch.zeros(qf.prompt_workspace_bytes(p, pg.total), dtype=torch.uint8, device="cuda")
    for _ in range(3):
        again = attend(pg, q, ws=ws)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_two_streams_and_a_replayed_graph():
    a, b = Paged([400, 30], [100, 2000], 2, seed=1), Paged([1, 1, 250], [700, 20, 0], 2, seed=2)
    work = []
    for pg in (a, b):
        q, (kc, vc) = queries(pg, 8), pg.pools()
        p = qf.params(pg.B, 8, 2, pg.width, 1, pg.num_pages)
        n = qf.prompt_workspace_bytes(p, pg.total)
        dev = (pg.table.cuda(), pg.cu.cuda(), pg.lens.cuda())
        out, lse = torch.empty_like(q), torch.empty((pg.total, 8), device="cuda")
        ws = torch.empty(n, dtype=torch.uint8, device="cuda")
        ref = attend(pg, q)
        work.append((q, kc, vc, *dev, out, lse, p, pg.total, ws, n, ref))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in work]
    for _ in range(5):
        for st, w in zip(streams, work):
            qf.prompt_attend(*w[:12], stream=st)
    torch.cuda.synchronize()
    for w in work:
        assert torch.equal(w[6], w[12][0]) and torch.equal(w[7], w[12][1])
        w[6].zero_()
    graph, st = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=st):
        for w in work:
            qf.prompt_attend(*w[:12], stream=st)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for w in work:
        assert torch.equal(w[6], w[12][0]) and torch.equal(w[7], w[12][1])
    # new queries and a shorter context in the same buffers: the replay follows them
    w = work[0]
    w[0].copy_(queries(a, 8, seed=77))
    w[5].copy_(torch.tensor([50, 1500], dtype=torch.int32))
    graph.replay()
    torch.cuda.synchronize()
    a.cached = [50, 1500]
    compare(w[6], w[7], prompt64(a, w[0]))


@pytest.mark.parametrize("rows", [2, 40])
def test_very_long_chains_of_tiles(rows):
    """Enough requests over the same 77,000 positions that every slice runs through hundreds of tiles of one block."""
    n_req = 160 if rows == 2 else 80
    pg = Paged([rows], [76_800], 1, seed=21)
    pg.table, pg.new, pg.cached = pg.table.repeat(n_req, 1), [rows] * n_req, [76_800] * n_req
    pg.B, pg.total = n_req, rows * n_req
    pg.cu, pg.lens = torch.arange(n_req + 1, dtype=torch.int32) * rows, torch.full((n_req,), 76_800, dtype=torch.int32)
    q = queries(pg, 4)
    out, lse, _ = attend(pg, q)
    from prompt_testlib import attend64
    pick = torch.arange(0, pg.total, 37)
    k, v = (pg.rows(0, 76_800 + rows, w).cuda() for w in "kv")
    ref = attend64(q[pick.cuda()].double(), k, v, (76_801 + pick % rows).cuda())
    compare(out[pick.cuda()], lse[pick.cuda()], {n: t.cpu() for n, t in ref.items()})
