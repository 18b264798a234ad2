"""qf_prompt_attend_scaled on the GPU against softmax attention in 64 bits: every element, both kernels, both code types."""
import numpy as np
import pytest
import torch

from paper_2608_15473_b200 import binding as qf
from paper_2608_15473_b200 import build as qf_build
from prompt_testlib import D, PAGE, prompt64
from scaled_testlib import KINDS, Scaled
from test_prompt_attend_gpu import compare

pytestmark = pytest.mark.gpu
KERNELS = [pytest.param(0, id="staged"), pytest.param(qf.QF_FLAG_SIMPLE_KERNEL, id="simple")]


@pytest.fixture(scope="module", autouse=True)
def built():
    qf_build.build()


def queries(pg, hq, seed=5, scale=1.5, pad=0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((pg.total + pad, hq, D), generator=g) * scale).to(torch.bfloat16).cuda()


def attend(pg, q, flags=0, sm_scale=0.0, pad=0, q_stride=0, identity=False, max_seq_len=0, ws=None, pools=None, stream=None):
    hq, T = q.shape[1], pg.total + pad
    p = qf.params(pg.B, hq, pg.Hkv, pg.width, 1, pg.num_pages, flags=flags | (qf.QF_FLAG_KV_NHD if pg.nhd else 0),
                  sm_scale=sm_scale, max_seq_len=max_seq_len)
    kc, vc, ks, vs = pools or pg.device()
    out, lse = torch.full((T, hq, D), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((T, hq), 7.0, device="cuda")
    n = qf.prompt_workspace_bytes(p, T)
    ws = torch.full((n,), 0xA5, dtype=torch.uint8, device="cuda") if ws is None else ws
    qf.prompt_attend_scaled(q, kc, vc, ks, vs, None if identity else pg.table.cuda(), pg.cu.cuda(), pg.lens.cuda(), out, lse, p, T, ws, n,
                            q_stride, kv_type=pg.type, stream=stream)
    torch.cuda.synchronize()
    status = qf.prompt_status(ws)
    assert (out[pg.total:] == 7).all() and (lse[pg.total:] == 7).all()       # rows of no request stay as they were
    return out[:pg.total], lse[:pg.total], status


def check(pg, hq, flags=0, **kw):
    q = queries(pg, hq, pad=kw.get("pad", 0))
    out, lse, status = attend(pg, q, flags, **kw)
    assert status == 0
    compare(out, lse, prompt64(pg, q[:pg.total]))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("flags", KERNELS)
@pytest.mark.parametrize("hq,hkv", [(1, 1), (2, 1), (3, 1), (8, 2), (5, 1), (6, 1), (28, 4), (8, 1), (16, 8)])
@pytest.mark.parametrize("nhd", [False, True])
def test_every_group_size(kind, flags, hq, hkv, nhd):
    check(Scaled([70, 1, 0, 33, 150], [0, 40, 5, 129, 3], hkv, kind, nhd, poison=True), hq, flags)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("flags", KERNELS)
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 33, 63, 64, 65, 127, 128, 129, 191, 255, 256, 257, 513])
def test_short_prompts(kind, flags, n):
    check(Scaled([n], [0], 2, kind, seed=n, poison=True), 8, flags)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("flags", KERNELS)
@pytest.mark.parametrize("cached", [0, 1, 15, 100, 127, 128, 129, 255, 1000])
@pytest.mark.parametrize("n", [1, 16, 70])
def test_chunks_behind_a_cached_context(kind, flags, cached, n):
    check(Scaled([n, 1, n + 3], [cached, cached + 7, max(cached - 1, 0)], 2, kind, nhd=cached % 2 == 1, seed=cached, poison=True), 8, flags)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("new,cached,hq,hkv", [
    ([3000], [0], 16, 8), ([700, 1, 1500, 260], [0, 5000, 300, 0], 28, 4), ([1] * 40 + [300, 333], [900] * 42, 8, 2),
    ([512], [12000], 32, 8), ([1], [30000], 8, 1), ([9] * 50, list(range(0, 1000, 20)), 40, 8)])
def test_ragged_and_long(kind, new, cached, hq, hkv):
    check(Scaled(new, cached, hkv, kind, hq == 28, seed=hq, poison=True), hq)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("flags", KERNELS)
def test_scales_that_are_no_powers_of_two(kind, flags):
    """code * scale is rounded to bf16: 2^-8 of every key's and value's number at most, so a score by 2^-8 sum |q_i k_i|,
    its weight relatively as much, and the output by that twice and once more for the values."""
    pg = Scaled([40, 130], [0, 77], 2, kind, seed=4, scales="any", poison=True)
    q = queries(pg, 8)
    out, lse, _ = attend(pg, q, flags)
    ref = prompt64(pg, q)
    mass = max(float(torch.einsum("rcgd,cnd->rcgn", q[int(pg.cu[b]):int(pg.cu[b + 1])].cpu().double().abs().reshape(-1, 2, 4, D),
                                  pg.rows(b, pg.new[b] + pg.cached[b], "k").abs()).max()) * D ** -0.5 for b in range(2))
    tol = 2.0 ** -8 * (ref["out"].abs() + (2 + 2 * mass) * ref["spread"])
    assert ((out.cpu().double() - ref["out"]).abs() <= tol).all()
    assert ((lse.cpu().double() - ref["lse"]).abs() <= 2.0 ** -8 * mass + 1e-5).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("flags", KERNELS)
def test_nan_scales_stay_with_the_rows_that_see_them(kind, flags):
    """Blocks of a NaN scale, also in the part of a tile that later rows alone see."""
    pg = Scaled([150, 60], [10, 0], 2, kind, seed=7)
    kc, vc, ks, vs = pg.device()
    ks[int(pg.table[0, 8]), 0] = float("nan")       # positions 128 to 143 of request 0: rows 118 on
    vs[int(pg.table[1, 2]), 1] = float("nan")       # positions 32 to 47 of request 1
    q = queries(pg, 8)
    out, lse, _ = attend(pg, q, flags, pools=(kc, vc, ks, vs))
    ref = prompt64(pg, q)
    ref["out"][118:150, :4], ref["lse"][118:150, :4] = float("nan"), float("nan")
    ref["out"][150 + 32:, 4:] = float("nan")
    compare(out, lse, ref)


@pytest.mark.parametrize("flags", KERNELS)
def test_nan_codes_stay_with_the_rows_that_see_them(flags):
    pg = Scaled([150, 60], [10, 0], 2, "e4m3", seed=7)
    q = queries(pg, 8)
    ref = prompt64(pg, q)
    pg.codes[0][int(pg.table[0, 8]), 0, 3, 77] = 0x7f       # position 131 of request 0: rows 121 on
    pg.codes[1][int(pg.table[1, 2]), 1, 5, 9] = 0xff        # position 37 of request 1, channel 9
    out, lse, _ = attend(pg, q, flags)
    ref["out"][121:150, :4], ref["lse"][121:150, :4] = float("nan"), float("nan")
    ref["out"][150 + 37:, 4:, 9] = float("nan")
    compare(out, lse, ref)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("flags", KERNELS)
def test_bad_table_entries(kind, flags):
    pg = Scaled([60], [100], 2, kind, seed=8)
    good = pg.table.clone()
    pg.table[0, 2], pg.table[0, 5] = -3, pg.num_pages + 9
    q = queries(pg, 8)
    for extra, want in ((0, 0), (qf.QF_FLAG_CHECK_BOUNDS, qf.QF_STATUS_BAD_PAGE)):
        out, lse, status = attend(pg, q, flags | extra)
        assert status == want
    pg.table = good
    keep = torch.tensor([i for i in range(160) if i // PAGE not in (2, 5)])
    k, v = (pg.rows(0, 160, w)[:, keep] for w in "kv")
    x = torch.einsum("rcgd,cnd->rcgn", q.cpu().double().reshape(60, 2, 4, D), k) * D ** -0.5
    x = x.masked_fill((keep[None, :] > torch.arange(60)[:, None] + 100)[:, None, None], -np.inf)
    ref = torch.einsum("rcgn,cnd->rcgd", torch.softmax(x, -1), v).reshape(60, 8, D)
    assert ((out.cpu().double() - ref).abs() <= 2.0 ** -8 * (ref.abs() + 2 * v.abs().amax())).all()
    assert ((lse.cpu().double() - torch.logsumexp(x, -1).reshape(60, 8)).abs() < 1e-4).all()


@pytest.mark.parametrize("kind", KINDS)
def test_strides_padding_identity_and_bounds(kind):
    pg = Scaled([33, 90], [7, 0], 2, kind, extra_pages=20)
    wide = torch.randn((pg.total, 8 * D + 64), device="cuda").to(torch.bfloat16)
    q = wide[:, :8 * D].reshape(pg.total, 8, D)
    out, lse, _ = attend(pg, wide[:, :8 * D].unflatten(1, (8, D)), q_stride=wide.stride(0))
    compare(out, lse, prompt64(pg, q.contiguous()))
    check(pg, 8, pad=5)
    pg.table = torch.arange(2 * pg.width, dtype=torch.int32).reshape(2, -1)
    check(pg, 8, identity=True)


@pytest.mark.parametrize("kind", KINDS)
def test_same_bits_in_both_layouts_streams_and_replays(kind):
    a, b = (Scaled([700, 1, 90], [300, 2000, 0], 4, kind, nhd, seed=9) for nhd in (False, True))
    q = queries(a, 16)
    x, y = attend(a, q), attend(b, q)
    assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = attend(a, q)
    assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1])
    p = qf.params(a.B, 16, 4, a.width, 1, a.num_pages)
    out, lse = torch.zeros((a.total, 16, D), dtype=torch.bfloat16, device="cuda"), torch.zeros((a.total, 16), device="cuda")
    ws = torch.empty(qf.prompt_workspace_bytes(p, a.total), dtype=torch.uint8, device="cuda")
    pools, table, cu, lens = a.device(), a.table.cuda(), a.cu.cuda(), a.lens.cuda()
    graph, cap = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(cap):
        with torch.cuda.graph(graph, stream=cap):
            qf.prompt_attend_scaled(q, *pools, table, cu, lens, out, lse, p, a.total, ws, ws.numel(), kv_type=a.type)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(x[0], out) and torch.equal(x[1], lse)


@pytest.mark.parametrize("kind", KINDS)
def test_a_chain_as_a_server_runs_it(kind):
    """Two prompts in chunks, then decode steps: placing, attention over the prompts and the decode step on one cache, which is
    followed token by token in 64 bits from the codes that the placing left."""
    hq, hkv, B = 8, 2, 2
    pg = Scaled([200, 90], [0, 0], hkv, kind, extra_pages=2)
    kc, vc, ks, vs = pg.device()
    g = torch.Generator().manual_seed(6)
    p = qf.params(B, hq, hkv, pg.width, 1, pg.num_pages)
    inv = torch.from_numpy(qf.rope_frequencies(128)[0]).cuda()
    lens = torch.zeros(B, dtype=torch.int32)
    table = pg.table.cuda()
    for new in ([130, 40], [60, 44], [1, 1], [1, 1], [1, 1]):
        T = sum(new)
        rows = torch.randn((T, (hq + 2 * hkv) * D), generator=g).to(torch.bfloat16).cuda()
        q, k, v = (t for t in (rows[:, :hq * D], rows[:, hq * D:(hq + hkv) * D], rows[:, (hq + hkv) * D:]))
        cu = torch.tensor([0, new[0], T], dtype=torch.int32)
        qo = torch.empty((T, hq, D), dtype=torch.bfloat16, device="cuda")
        s = rows.stride(0)
        qf.rope_append_scaled(q, k, v, qo, None, kc, vc, ks, vs, table, cu.cuda(), lens.cuda(), None, None, None, None, None, inv, p,
                              qf.rope_params(T, q_stride=s, k_stride=s, v_stride=s), kv_type=pg.type)
        order = (0, 1, 2, 3)
        from scaled_testlib import numbers
        pg.k, pg.v = (numbers(c.cpu().permute(order), kind) * t.cpu().double()[:, :, None, None] for c, t in ((kc, ks), (vc, vs)))
        pg.new, pg.cached, pg.total, pg.cu, pg.lens = new, lens.tolist(), T, cu, lens.clone()
        out, lse, status = attend(pg, qo, pools=(kc, vc, ks, vs))
        assert status == 0
        ref = prompt64(pg, qo)
        compare(out, lse, ref)
        lens = lens + torch.tensor(new, dtype=torch.int32)
        if T == B:      # the same step by the decode sweep: all positions, the new token's among them
            f = lambda *s: torch.empty(s, device="cuda")      # noqa: E731
            o, m, l, out2, lse2 = f(B, 1, hq, D), f(B, 1, hq), f(B, 1, hq), f(B, hq, D), f(B, hq)
            ws = torch.empty(qf.workspace_bytes(p), dtype=torch.uint8, device="cuda")
            ranges = torch.tensor([[[0, int(x)]] for x in lens], dtype=torch.int32).cuda()
            qf.decode_step_scaled(qo, kc, vc, ks, vs, table, lens.cuda(), ranges, None, o, m, l, out2, lse2, p, ws, ws.numel(), kv_type=pg.type)
            torch.cuda.synchronize()
            assert ((out2.cpu().double() - ref["out"]).abs() <= 2.0 ** -14 * ref["spread"]).all()
            assert ((lse2.cpu().double() - ref["lse"]).abs() <= 1e-5 * ref["lse"].abs().clamp(min=1)).all()
