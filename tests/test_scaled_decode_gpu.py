"""qf_decode_partial_scaled and qf_decode_step_scaled on the GPU against their formulas in 64 bits: every element of every
state, both kernels, both code types."""
import numpy as np
import pytest
import torch

from paper_2608_15473_b200 import binding as qf
from paper_2608_15473_b200 import build as qf_build
from prompt_testlib import D, PAGE
from scaled_testlib import KINDS, Scaled, even_ranges, merge64, states64

pytestmark = pytest.mark.gpu
KERNELS = [pytest.param(0, id="staged"), pytest.param(qf.QF_FLAG_SIMPLE_KERNEL, id="simple")]


@pytest.fixture(scope="module", autouse=True)
def built():
    qf_build.build()


def queries(B, hq, seed=5, scale=1.5):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((B, hq, D), generator=g) * scale).to(torch.bfloat16).cuda()


def close(got, ref, slack):
    """fp32 results: a score is off by at most 2^-20 of sum |q_i k_i| (128 products, exact in fp32, added in fp32: seven
    levels of 2^-24 in a tree, sixteen when a tensor core adds them in turn and cuts off), which moves its weight by as
    much, relatively, and the normalised sum by twice that of sum w |v|; the weights' two 16-bit terms (2^-22), exponentials
    (2^-22) and the sums of up to a million weights, rescaled page by page, stay below 2^-19.  The slack says all that."""
    got, finite = got.cpu().double(), torch.isfinite(ref)
    assert torch.equal(torch.isnan(got), torch.isnan(ref)) and torch.equal(got[~finite & ~torch.isnan(ref)], ref[~finite & ~torch.isnan(ref)])
    err = (got - ref).abs()
    bad = finite & (err > slack + 1e-30)
    assert not bad.any(), (int(bad.sum()), float((err / (slack + 1e-30))[finite].max()), float(err[finite].max()))


def lse_close(got, ref, slack):
    close(got, ref, slack + 1e-6 * ref.abs().nan_to_num(0, 0, 0) + 1e-6)


def params_of(pg, hq, S, flags=0, **kw):
    return qf.params(pg.B, hq, pg.Hkv, pg.width, S, pg.num_pages, flags=flags | (qf.QF_FLAG_KV_NHD if pg.nhd else 0), **kw)


def step(pg, q, ranges, flags=0, counts=None, sm_scale=0.0, identity=False, max_seq_len=0, stream=None, pools=None, lens=None, ws=None):
    B, hq, _ = q.shape
    S = ranges.shape[1]
    p = params_of(pg, hq, S, flags, sm_scale=sm_scale, max_seq_len=max_seq_len)
    kc, vc, ks, vs = pools or pg.device()
    f = lambda *s: torch.full(s, 7.0, device="cuda")      # noqa: E731
    o, m, l, out, lse = f(B, S, hq, D), f(B, S, hq), f(B, S, hq), f(B, hq, D), f(B, hq)
    ws = torch.full((qf.workspace_bytes(p),), 0xA5, dtype=torch.uint8, device="cuda") if ws is None else ws
    qf.decode_step_scaled(q, kc, vc, ks, vs, None if identity else pg.table.cuda(), pg.lens.cuda() if lens is None else lens, ranges.cuda(),
                          None if counts is None else torch.as_tensor(counts, dtype=torch.int32).cuda(), o, m, l, out, lse, p,
                          ws, ws.numel(), kv_type=pg.type, stream=stream)
    torch.cuda.synchronize()
    status = qf.read_status(ws)
    return dict(o=o, m=m, l=l, out=out, lse=lse, status=status, p=p, ws=ws)


def check(pg, hq, S=1, flags=0, ranges=None, counts=None, q=None, sm_scale=0.0, **kw):
    q = queries(pg.B, hq) if q is None else q
    ranges = even_ranges(pg.cached, S) if ranges is None else ranges
    got = step(pg, q, ranges, flags, counts, sm_scale, **kw)
    ref = states64(pg, q.cpu(), ranges, sm_scale or None)
    assert got["status"] == 0
    close(got["o"], ref["out"], ref["slack"])
    lse_close(got["m"], ref["m"], ref["lse_slack"])
    lse_close(got["l"], ref["lse"], ref["lse_slack"])
    out, lse, slack, lse_slack = merge64(ref, counts)
    close(got["out"], out, slack + 2.0 ** -20 * out.abs())
    lse_close(got["lse"], lse, lse_slack)
    return got


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("flags", KERNELS)
@pytest.mark.parametrize("hq,hkv", [(1, 1), (2, 1), (3, 1), (8, 2), (5, 1), (6, 1), (28, 4), (8, 1), (16, 8), (32, 8), (40, 8)])
@pytest.mark.parametrize("nhd", [False, True])
def test_every_group_size(kind, flags, hq, hkv, nhd):
    check(Scaled([0] * 4, [70, 1, 333, 16], hkv, kind, nhd, poison=True), hq, 2, flags)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("flags", KERNELS)
@pytest.mark.parametrize("n", [0, 1, 2, 15, 16, 17, 31, 32, 33, 127, 128, 129, 255, 256, 257, 1000, 4096])
def test_lengths(kind, flags, n):
    check(Scaled([0], [n], 2, kind, n % 2 == 1, seed=n, poison=True), 8, 1, flags)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("flags", KERNELS)
@pytest.mark.parametrize("scales", ["power", "any"])
def test_ragged_batches_and_shards(kind, flags, scales):
    pg = Scaled([0] * 9, [700, 1, 0, 2500, 33, 16, 129, 5, 1024], 2, kind, seed=3, poison=True, scales=scales)
    ranges = torch.tensor([[[0, 300], [300, 700], [700, 700]], [[0, 1], [5, 9], [1, 0]], [[0, 0], [0, 5], [-3, 2]],
                           [[17, 1111], [1111, 2500], [0, 17]], [[0, 33], [0, 33], [32, 40]], [[-5, 3], [3, 99], [16, 16]],
                           [[128, 129], [0, 128], [50, 20]], [[0, 5], [0, 0], [4, 5]], [[1, 2], [2, 1023], [1023, 5000]]], dtype=torch.int32)
    check(pg, 8, 3, flags, ranges, counts=[3, 1, 2, 3, 2, 3, 2, 0, 3])


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("hq,hkv,batch,n,S", [(16, 8, 1, 60000, 16), (32, 8, 24, 9000, 5), (28, 4, 60, 3000, 1), (8, 1, 3, 40000, 2)])
def test_long_and_many(kind, hq, hkv, batch, n, S):
    r = np.random.default_rng(batch)
    check(Scaled([0] * batch, r.integers(n // 2, n + 1, batch), hkv, kind, batch % 2 == 1, seed=batch), hq, S)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("batch,S", [(32, 9), (255, 1), (257, 1), (300, 5), (64, 32), (300, 8)])
def test_many_pairs_of_requests_and_shards(kind, batch, S):
    """Fewer than the sweep's threads scan at once, several rounds of them, and (2,400) more than it plans by itself."""
    pg = Scaled([0] * batch, 1 + np.arange(batch) * 7 % 167, 1, kind, seed=8)
    check(pg, 4, S)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("flags", [0, qf.QF_FLAG_DRAW_ALWAYS, qf.QF_FLAG_NO_SMALL_MERGE])
def test_schedules(kind, flags):
    check(Scaled([0] * 5, [8000, 100, 12000, 1, 3333], 4, kind, seed=4), 16, 2, flags)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("flags", KERNELS)
@pytest.mark.parametrize("scale", [2.0 ** -60, 1e-3, 30.0, 2.0 ** 60])
def test_sizes_of_queries(kind, flags, scale):
    """Queries far outside the range of 16-bit floats; the softmax scale brings the scores back."""
    pg = Scaled([0, 0], [300, 77], 2, kind)
    check(pg, 8, 1, flags, q=queries(2, 8, scale=scale), sm_scale=min(0.1, 0.1 / scale) if scale > 1 else min(0.1 / scale, 1e18))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("flags", KERNELS)
def test_one_channel_of_a_query_dwarfs_the_others(kind, flags):
    q = queries(2, 8)
    q[:, :, 5] *= 3e4
    pg = Scaled([0, 0], [300, 77], 2, kind)
    check(pg, 8, 1, flags, q=q, sm_scale=1e-5)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("flags", KERNELS)
def test_scales_of_neighbouring_blocks_far_apart(kind, flags):
    """Value blocks whose scales differ by 2^80 and key blocks by 2^12: a page's weights must keep their precision."""
    pg = Scaled([0, 0], [600, 333], 2, kind)
    g = torch.Generator().manual_seed(1)
    pg.scale[1] *= torch.ldexp(torch.ones(pg.scale[1].shape), torch.randint(-40, 41, pg.scale[1].shape, generator=g))
    pg.scale[0] *= torch.ldexp(torch.ones(pg.scale[0].shape), torch.randint(-9, 3, pg.scale[0].shape, generator=g))
    from scaled_testlib import numbers
    pg.k, pg.v = ((numbers(c, kind) * s.double()[:, :, None, None]) for c, s in zip(pg.codes, pg.scale))
    check(pg, 8, 2, flags)


@pytest.mark.parametrize("kind", KINDS)
def test_many_positions_of_tiny_weight(kind):
    """One position with a weight 2^26 times every other's, 60,000 others: together they count, and none may be rounded away."""
    n = 60000
    pg = Scaled([0], [n], 1, kind)
    q = torch.zeros((1, 4, D), dtype=torch.bfloat16)
    q[..., 0] = 1.0
    for w in (0, 1):
        pg.scale[w][:] = 1.0
    one = {"e4m3": 0x38, "int8": 1}[kind]
    pg.codes[0][:], pg.codes[1][:] = 0, one
    page = int(pg.table[0, 1234 // PAGE])
    pg.codes[0][page, 0, 1234 % PAGE, 0] = one
    pg.codes[1][page, 0, 1234 % PAGE] = 0            # the value of the heavy position is 0
    from scaled_testlib import numbers
    pg.k, pg.v = numbers(pg.codes[0], kind), numbers(pg.codes[1], kind)
    check(pg, 4, 1, q=q.cuda(), sm_scale=26 * float(np.log(2.0)))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("flags", KERNELS)
def test_nan_scales_and_codes(kind, flags):
    """A NaN scale of keys makes the states of its shard NaN, of values their vectors; other shards and requests stay."""
    pg = Scaled([0] * 3, [200, 200, 200], 2, kind)
    kc, vc, ks, vs = pg.device()
    ks[int(pg.table[0, 2]), 1] = float("nan")
    vs[int(pg.table[1, 12]), 0] = float("nan")
    q, ranges = queries(3, 8), even_ranges([200] * 3, 2)
    got = step(pg, q, ranges, flags, pools=(kc, vc, ks, vs))
    ref = states64(pg, q.cpu(), ranges)
    ref["out"][0, 0, 4:], ref["lse"][0, 0, 4:] = float("nan"), float("nan")
    ref["out"][1, 1, :4] = float("nan")
    close(got["o"], ref["out"], ref["slack"])
    lse_close(got["l"], ref["lse"], ref["lse_slack"])
    assert torch.isnan(got["out"][0, 4:]).all() and torch.isfinite(got["out"][2]).all() and torch.isfinite(got["lse"][1]).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("flags", KERNELS)
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_queries_that_are_not_finite(kind, flags, value):
    pg = Scaled([0, 0], [100, 100], 1, kind)
    q = queries(2, 4)
    q[0, 1, 7] = value
    got = step(pg, q, even_ranges([100] * 2, 1), flags)
    assert torch.isnan(got["out"][0, 1]).all() and torch.isnan(got["lse"][0, 1])
    assert torch.isfinite(got["out"][0, 0]).all() and torch.isfinite(got["out"][0, 2:]).all() and torch.isfinite(got["out"][1]).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("flags", KERNELS)
def test_bad_table_entries_are_skipped_and_reported(kind, flags):
    pg = Scaled([0, 0], [170, 40], 2, kind, seed=6)
    good = pg.table.clone()
    pg.table[0, 3], pg.table[0, 7], pg.table[1, 2] = -1, pg.num_pages, 2 ** 31 - 1
    q, ranges = queries(2, 8), even_ranges(pg.cached, 1)
    keep = [torch.tensor([i for i in range(n) if i // PAGE not in gone]) for n, gone in ((170, (3, 7)), (40, (2,)))]
    for extra, want in ((0, 0), (qf.QF_FLAG_CHECK_BOUNDS, qf.QF_STATUS_BAD_PAGE)):
        got = step(pg, q, ranges, flags | extra)
        assert got["status"] == want
        for b in range(2):
            pg.table, table = good, pg.table
            k, v = (pg.rows(b, pg.cached[b], w)[:, keep[b]] for w in "kv")
            pg.table = table
            x = torch.einsum("cgd,cnd->cgn", q[b].cpu().double().reshape(2, 4, D), k) * D ** -0.5
            want_out = torch.einsum("cgn,cnd->cgd", torch.softmax(x, -1), v).reshape(8, D)
            close(got["out"][b], want_out, 2.0 ** -14 * v.abs().amax() * torch.ones_like(want_out))


@pytest.mark.parametrize("kind", KINDS)
def test_a_request_of_bad_pages_only_is_empty(kind):
    """Page 0, whose scale would be read in their place, is NaN throughout."""
    pg = Scaled([0, 0], [100, 60], 2, kind, poison=True)
    pg.table[0, :] = -1
    kc, vc, ks, vs = pg.device()
    if not (pg.table[1, :4] == 0).any():
        ks[0], vs[0] = float("nan"), float("nan")
    got = step(pg, queries(2, 8), even_ranges(pg.cached, 1), pools=(kc, vc, ks, vs))
    assert (got["out"][0] == 0).all() and torch.isneginf(got["lse"][0]).all() and torch.isfinite(got["out"][1]).all()


@pytest.mark.parametrize("kind", KINDS)
def test_lengths_beyond_the_table_row(kind):
    pg = Scaled([0], [64], 1, kind, seed=2)
    ranges = torch.tensor([[[0, 1000]]], dtype=torch.int32)
    q = queries(1, 4)
    a = step(pg, q, ranges, lens=torch.tensor([9999], dtype=torch.int32).cuda())
    b = step(pg, q, ranges)
    assert torch.equal(a["out"], b["out"]) and torch.equal(a["lse"], b["lse"])
    assert step(pg, q, ranges, qf.QF_FLAG_CHECK_BOUNDS, lens=torch.tensor([65], dtype=torch.int32).cuda())["status"] == qf.QF_STATUS_BAD_PAGE


@pytest.mark.parametrize("kind", KINDS)
def test_identity_table(kind):
    pg = Scaled([0] * 3, [64, 64, 64], 2, kind, extra_pages=0)
    pg.table = torch.arange(12, dtype=torch.int32).reshape(3, 4)
    check(pg, 8, 2, identity=True)


@pytest.mark.parametrize("kind", KINDS)
def test_both_layouts_give_the_same_bits(kind):
    a, b = (Scaled([0] * 3, [500, 3, 1200], 4, kind, nhd, seed=9) for nhd in (False, True))
    q, ranges = queries(3, 16), even_ranges(a.cached, 2)
    x, y = step(a, q, ranges), step(b, q, ranges)
    for n in ("o", "m", "l", "out", "lse"):
        assert torch.equal(x[n], y[n]), n


@pytest.mark.parametrize("kind", KINDS)
def test_partial_is_the_step_without_its_merge(kind):
    pg = Scaled([0] * 3, [500, 3, 1200], 4, kind, seed=10)
    q, ranges = queries(3, 16), even_ranges(pg.cached, 2)
    got = step(pg, q, ranges, qf.QF_FLAG_NO_SMALL_MERGE)
    # into slots 1 and 2 of four
    p = params_of(pg, 16, 2, out_shards=4, out_shard_offset=1)
    o, m, l = (torch.full(s, 7.0, device="cuda") for s in ((3, 4, 16, D), (3, 4, 16), (3, 4, 16)))
    kc, vc, ks, vs = pg.device()
    ws = torch.empty(qf.workspace_bytes(p), dtype=torch.uint8, device="cuda")
    qf.decode_partial_scaled(q, kc, vc, ks, vs, pg.table.cuda(), pg.lens.cuda(), ranges.cuda(), o, m, l, p, ws, ws.numel(), kv_type=pg.type)
    torch.cuda.synchronize()
    assert torch.equal(o[:, 1:3], got["o"]) and torch.equal(m[:, 1:3], got["m"]) and torch.equal(l[:, 1:3], got["l"])
    assert (o[:, 0] == 7).all() and (o[:, 3] == 7).all()


@pytest.mark.parametrize("kind", KINDS)
def test_another_stream_and_a_replayed_graph(kind):
    pg = Scaled([0] * 4, [3000, 17, 900, 2222], 2, kind, seed=11)
    q, ranges = queries(4, 8), even_ranges(pg.cached, 3)
    want = step(pg, q, ranges)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step(pg, q, ranges)
    assert torch.equal(want["out"], got["out"]) and torch.equal(want["o"], got["o"])
    p, pools = want["p"], pg.device()
    f = lambda *s: torch.zeros(s, device="cuda")      # noqa: E731
    o, m, l, out, lse = f(4, 3, 8, D), f(4, 3, 8), f(4, 3, 8), f(4, 8, D), f(4, 8)
    table, lens, rng, ws = pg.table.cuda(), pg.lens.cuda(), ranges.cuda(), want["ws"]
    graph, cap = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(cap):
        with torch.cuda.graph(graph, stream=cap):
            qf.decode_step_scaled(q, *pools, table, lens, rng, None, o, m, l, out, lse, p, ws, ws.numel(), kv_type=pg.type)
    for _ in range(3):
        for x in (o, m, l, out, lse):
            x.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want["out"]) and torch.equal(lse, want["lse"]) and torch.equal(o, want["o"])


@pytest.mark.parametrize("kind", KINDS)
def test_results_do_not_change_from_call_to_call(kind):
    pg = Scaled([0] * 8, [3000, 17, 900, 2222, 8000, 1, 555, 64], 8, kind, seed=12)
    q, ranges = queries(8, 32), even_ranges(pg.cached, 2)
    a = step(pg, q, ranges, qf.QF_FLAG_DRAW_ALWAYS)
    for _ in range(3):
        b = step(pg, q, ranges, qf.QF_FLAG_DRAW_ALWAYS)
        assert torch.equal(a["o"], b["o"]) and torch.equal(a["lse"], b["lse"])


@pytest.mark.parametrize("kind", KINDS)
def test_the_current_token_folds_into_the_states(kind):
    """qf_combine_self on scaled states: the cache's positions and one more."""
    pg = Scaled([0] * 2, [333, 50], 2, kind, seed=13)
    q, ranges = queries(2, 8), even_ranges(pg.cached, 2)
    got = step(pg, q, ranges)
    g = torch.Generator().manual_seed(2)
    kn, vn = ((torch.randn((2, 2, D), generator=g)).to(torch.bfloat16) for _ in range(2))
    out, lse = torch.empty((2, 8, D), device="cuda"), torch.empty((2, 8), device="cuda")
    qf.combine_self(got["o"], got["l"], None, q, kn.cuda(), vn.cuda(), out, lse, got["p"])
    torch.cuda.synchronize()
    for b in range(2):
        k = torch.cat([pg.rows(b, pg.cached[b], "k"), kn[b].double()[:, None]], 1)
        v = torch.cat([pg.rows(b, pg.cached[b], "v"), vn[b].double()[:, None]], 1)
        x = torch.einsum("cgd,cnd->cgn", q[b].cpu().double().reshape(2, 4, D), k) * D ** -0.5
        ref = torch.einsum("cgn,cnd->cgd", torch.softmax(x, -1), v).reshape(8, D)
        close(out[b], ref, 2.0 ** -14 * v.abs().amax() * torch.ones_like(ref))
        lse_close(lse[b], torch.logsumexp(x, -1).reshape(8), 1e-5 * torch.ones(8, dtype=torch.float64))
