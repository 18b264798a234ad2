"""qf_rope_append on the GPU against its formula in 64 bits: every element of every output."""
import numpy as np
import pytest
import torch

from paper_2608_15473_b200 import binding as qf
from paper_2608_15473_b200 import build as qf_build
from prompt_testlib import D, PAGE, Paged, bf16, rope64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    qf_build.build()


def check_rows(got, ref, coarse):
    """One rounding to bf16: half a step of the value, 2^-8 relative (a step is 2^-7 of the binade's lower end, so half
    of it is at most 2^-8 of the value), plus the fp32 arithmetic before it.  That is bounded per pair by a few fp32
    roundings of its larger member: norm (128-term sum: 2^-24 * 8 levels, square root, reciprocal, two products) and
    rotation (sine and cosine to 2^-23 of one, two products and a sum): 32 * 2^-24 of the row's largest value."""
    got, ref = got.double(), ref.double()
    tol = 2.0 ** -8 * ref.abs() + 32 * 2.0 ** -24 * coarse
    bad = (got - ref).abs() > tol
    assert not bad.any(), (float((got - ref).abs().max()), int(bad.sum()))


def run(pg, hq, rotary=128, interleaved=False, norm=True, fused=False, base=None, rot_scale=1.0, with_q=True, with_kv=True,
        cache=True, k_out=False, pad=0, seed=1, stream=None, inplace=False, theta=1e6, eps=1e-6, identity=False):
    g = torch.Generator().manual_seed(seed)
    T, hkv = pg.total + pad, pg.Hkv
    if fused:
        rows = (torch.randn((T, (hq + 2 * hkv) * D), generator=g) * 1.5).to(torch.bfloat16)
        dev = rows.cuda()
        q, k, v = dev[:, :hq * D], dev[:, hq * D:(hq + hkv) * D], dev[:, (hq + hkv) * D:]
        strides = (rows.shape[1],) * 3
    else:
        rows = (torch.randn((T, (hq + 2 * hkv) * D), generator=g) * 1.5).to(torch.bfloat16)
        q, k, v = (x.contiguous().cuda() for x in (rows[:, :hq * D], rows[:, hq * D:(hq + hkv) * D], rows[:, (hq + hkv) * D:]))
        strides = (0, 0, 0)
    inv = torch.from_numpy(qf.rope_frequencies(rotary, theta)[0]) if rotary else torch.zeros(1)
    qg = bf16(1 + 0.3 * np.random.default_rng(seed).standard_normal(D)) if norm else None
    kg = bf16(1 + 0.3 * np.random.default_rng(seed + 1).standard_normal(D)) if norm else None
    kc, vc = pg.pools()
    p = qf.params(pg.B, hq, hkv, pg.width, 1, pg.num_pages, flags=qf.QF_FLAG_KV_NHD if pg.nhd else 0)
    r = qf.rope_params(T, rotary, interleaved, eps, rot_scale, *strides)
    qo = (q if inplace else torch.full((T, hq, D), float("nan"), dtype=torch.bfloat16, device="cuda")) if with_q else None
    ko = torch.full((T, hkv, D), float("nan"), dtype=torch.bfloat16, device="cuda") if k_out else None
    dev = lambda t: None if t is None else t.cuda()
    qf.rope_append(q if with_q else None, k if with_kv else None, v if with_kv and cache else None, qo, ko,
                   kc if cache else None, vc if cache else None, None if identity else pg.table.cuda(), pg.cu.cuda(),
                   pg.lens.cuda(), dev(base), dev(qg), dev(kg), dev(inv) if rotary else None, p, r, stream)
    assert qf.last_launch_count() == 1
    torch.cuda.synchronize()

    # reference
    req = np.repeat(np.arange(pg.B), pg.new)
    slot = np.concatenate([np.arange(n) + c for n, c in zip(pg.new, pg.cached)]) if pg.total else np.zeros(0, int)
    pos = slot + (base.numpy()[req] if base is not None else 0)
    live = rows[:pg.total]
    turn = lambda x, h, gain: rope64(x.reshape(-1, h, D), pos, inv, rotary, interleaved, gain, eps, rot_scale)
    if with_q:
        ref = turn(live[:, :hq * D], hq, qg)
        got = qo.reshape(T, hq, D).cpu()
        check_rows(got[:pg.total], ref, ref.abs().amax(-1, keepdim=True) + 1)
        if not inplace:
            assert torch.isnan(got[pg.total:]).all()          # rows of no request are left as they were
        else:
            assert torch.equal(got[pg.total:].reshape(-1, hq * D), rows[pg.total:, :hq * D])
    if with_kv:
        kref = turn(live[:, hq * D:(hq + hkv) * D], hkv, kg)
        if k_out:
            check_rows(ko.cpu()[:pg.total], kref, kref.abs().amax(-1, keepdim=True) + 1)
            assert torch.isnan(ko.cpu()[pg.total:]).all()
        vref = live[:, (hq + hkv) * D:].reshape(-1, hkv, D)
        gk, gv = pg.head_major(kc), pg.head_major(vc)
        written = torch.zeros((pg.num_pages, PAGE), dtype=torch.bool)
        for i in range(pg.total if cache else 0):
            b, s = int(req[i]), int(slot[i])
            if s // PAGE >= pg.width:
                continue
            page = b * pg.width + s // PAGE if identity else int(pg.table[b, s // PAGE])
            if not 0 <= page < pg.num_pages:
                continue
            written[page, s % PAGE] = True
            check_rows(gk[page, :, s % PAGE], kref[i], kref[i].abs().amax(-1, keepdim=True) + 1)
            assert torch.equal(gv[page, :, s % PAGE], vref[i])
        keep = ~written[:, None, :, None].expand_as(pg.k)
        bits = lambda t: t.view(torch.int16)
        assert torch.equal(bits(gk)[keep], bits(pg.k)[keep]) and torch.equal(bits(gv)[keep], bits(pg.v)[keep])
    return qo, kc, vc


@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 8), (16, 8), (28, 4), (40, 8), (6, 2)])
@pytest.mark.parametrize("nhd", [False, True])
def test_head_counts_and_layouts(hq, hkv, nhd):
    run(Paged([5, 1, 0, 17, 33], [0, 15, 3, 16, 100], hkv, nhd), hq)


@pytest.mark.parametrize("rotary", [0, 16, 32, 64, 96, 112, 128])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_rotary_part_and_pair_layout(rotary, interleaved, norm):
    run(Paged([3, 40, 1], [7, 0, 31], 2), 6, rotary=rotary, interleaved=interleaved, norm=norm)


@pytest.mark.parametrize("new", [[1], [1] * 8, [1] * 300, [0, 0, 1, 0], [2000], [700, 1, 0, 900, 3]])
@pytest.mark.parametrize("fused", [False, True])
def test_lengths(new, fused):
    run(Paged(new, [(13 * i) % 50 for i in range(len(new))], 4), 8, fused=fused)


def test_positions_near_and_beyond_a_million_are_exact():
    base = torch.tensor([1_000_000, 123_456_789, 2_000_000_000, 0], dtype=torch.int32)
    run(Paged([4, 4, 4, 4], [100, 3, 0, 60000], 2), 4, base=base)
    run(Paged([4, 4, 4, 4], [100, 3, 0, 5], 2), 4, base=base, interleaved=True, rotary=64, theta=10000.0)


def test_rotation_scale_and_padding_rows():
    run(Paged([9, 30], [2, 5], 8), 16, rot_scale=1.3465735, pad=7)
    run(Paged([9, 30], [2, 5], 8), 16, pad=100, fused=True)


def test_optional_parts():
    pg = lambda: Paged([9, 1, 30], [2, 0, 5], 4)
    run(pg(), 8, with_kv=False, cache=False)           # the query alone
    run(pg(), 8, with_q=False)                         # keys and values only
    run(pg(), 8, with_q=False, cache=False, k_out=True)
    run(pg(), 8, k_out=True, pad=3)
    run(pg(), 8, inplace=True, pad=3)
    run(pg(), 8, norm=False, rotary=0)                 # a plain cache write of whole prompts


def test_identity_table():
    pg = Paged([20, 33], [5, 0], 2, max_pages=4, extra_pages=5)
    run(pg, 4, identity=True)


def test_positions_without_a_page_store_nothing():
    pg = Paged([40, 3], [0, 16], 2, max_pages=2, extra_pages=2)      # row of two pages, a request that needs three
    run(pg, 4)
    pg = Paged([40, 3], [0, 16], 2)
    pg.table[0, 1] = pg.num_pages          # outside the pool
    pg.table[1, 1] = -1
    run(pg, 4)


def test_rows_pass_bit_for_bit_without_norm_and_rotation():
    pg = Paged([33], [0], 2)
    qo, kc, vc = run(pg, 4, norm=False, rotary=0)
    g = torch.Generator().manual_seed(1)
    rows = (torch.randn((33, 8 * D), generator=g) * 1.5).to(torch.bfloat16)
    assert torch.equal(qo.cpu().reshape(33, -1), rows[:, :4 * D])


def test_other_stream_and_graph_replay_follow_the_lengths():
    hq, hkv, B = 8, 4, 5
    pg = Paged([1] * B, [14, 15, 16, 31, 0], hkv, max_pages=4, extra_pages=20)
    pg.table[:] = torch.randperm(pg.num_pages)[:B * 4].reshape(B, 4).to(torch.int32)
    g = torch.Generator().manual_seed(3)
    x = torch.randn((B, (hq + 2 * hkv) * D), generator=g).to(torch.bfloat16).cuda()
    inv = torch.from_numpy(qf.rope_frequencies(128, 1e4)[0]).cuda()
    p, r = qf.params(B, hq, hkv, 4, 1, pg.num_pages), qf.rope_params(B, 128, False, 1e-6, 1.0, *[x.shape[1]] * 3)
    q, k, v = x[:, :hq * D], x[:, hq * D:(hq + hkv) * D], x[:, (hq + hkv) * D:]
    table, cu, lens = pg.table.cuda(), pg.cu.cuda(), pg.lens.cuda()

    def go(qo, kc, vc, lens, stream=None):
        qf.rope_append(q, k, v, qo, None, kc, vc, table, cu, lens, None, None, None, inv, p, r, stream)

    qo, (kc, vc) = torch.empty((B, hq, D), dtype=torch.bfloat16, device="cuda"), pg.pools()
    st, live = torch.cuda.Stream(), lens.clone()
    go(qo, kc, vc, live)
    torch.cuda.synchronize()
    kc2, vc2 = pg.pools()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        go(qo, kc2, vc2, live, st)
        live += 1
    for _ in range(4):
        graph.replay()
    torch.cuda.synchronize()
    want_k, want_v = pg.pools()
    want_q = torch.empty_like(qo)
    step = lens.clone()
    for _ in range(4):
        go(want_q, want_k, want_v, step)
        step += 1
    torch.cuda.synchronize()
    assert torch.equal(kc2.view(torch.int16), want_k.view(torch.int16)) and torch.equal(vc2.view(torch.int16), want_v.view(torch.int16))
    assert torch.equal(qo, want_q)
