"""qf_rope_append_scaled and qf_rope_append_axes on the GPU against their rules in 64 bits: every output, code and scale."""
import numpy as np
import pytest
import torch

from paper_2608_15473_b200 import binding as qf
from paper_2608_15473_b200 import build as qf_build
from prompt_testlib import D, PAGE, Paged, bf16
from scaled_testlib import KINDS, Scaled, codes_of, numbers, scale_for, step_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    qf_build.build()


def turn64(x, pos, inv, rotary, interleaved, gain, eps, rot_scale):
    """Norm and rotation of x [rows, heads, D] by positions pos [pairs, rows], in 64 bits."""
    x = x.double()
    if gain is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * gain.double()
    if not rotary:
        return x
    t = torch.as_tensor(pos, dtype=torch.float64).T * inv.double()[None, :]
    c, s = torch.cos(t)[:, None] * rot_scale, torch.sin(t)[:, None] * rot_scale
    y, h = x.clone(), rotary // 2
    one, two = (slice(0, rotary, 2), slice(1, rotary, 2)) if interleaved else (slice(0, h), slice(h, rotary))
    y[..., one], y[..., two] = x[..., one] * c - x[..., two] * s, x[..., two] * c + x[..., one] * s
    return y


def fp32_slack(ref):
    """fp32 arithmetic before the last rounding: norm (sum of 128 squares, root, reciprocal, two products) and rotation (sine
    and cosine to 2^-23 of one, two products and a sum): 32 * 2^-24 of the row's largest value."""
    return 32 * 2.0 ** -24 * ref.abs().amax(-1, keepdim=True)


def check_rows(got, ref):
    got = got.double()
    bad = (got - ref).abs() > 2.0 ** -8 * ref.abs() + fp32_slack(ref)
    assert not bad.any(), (float((got - ref).abs().max()), int(bad.sum()))


def check_pool(pg, name, codes, scale, before, before_scale, want, placed, held):
    """One pool.  want: {(page, slot): row [Hkv, D] in 64 bits}; placed[page] the slots written, held[page] those before them."""
    kind, touched = pg.kind, torch.zeros(codes.shape[:1] + (PAGE,), dtype=torch.bool)
    for page, slots in placed.items():
        rows = torch.stack([want[page, s] for s in slots], 1)                    # [Hkv, n, D]
        slack = fp32_slack(rows)
        old = before_scale[page].double() if held[page] else torch.zeros(pg.Hkv, dtype=torch.float64)
        top = rows.abs().amax(dim=(1, 2))
        # the largest value may lie at a border between scales, within fp32 arithmetic
        reach = slack.amax(dim=(1, 2))
        lo = torch.maximum(old, scale_for((top - reach).clamp(min=0), kind))
        hi = torch.maximum(old, scale_for(top + reach, kind))
        s = scale[page].double()
        assert ((s == lo) | (s == hi)).all(), (name, page, s, lo, hi)
        z = rows / s[:, None, None]
        got = numbers(codes[page][:, slots], kind)
        # half a step, and what fp32 arithmetic can move a number across a border
        bad = (got - z).abs() > step_of(z, kind) * 0.5 + slack / s[:, None, None]
        bad &= (got - z).abs() > step_of(z * (1 + 1e-9), kind) * 0.5 + slack / s[:, None, None]
        assert not bad.any(), (name, page, int(bad.sum()), float((got - z).abs().max()))
        touched[page, slots] = True
        if held[page]:
            again = codes_of(numbers(before[page][:, :held[page]], kind) * (old / s)[:, None, None], kind)
            moved = (old != s)[:, None, None].expand_as(again)
            assert torch.equal(codes[page][:, :held[page]][moved], again[moved]), (name, page)
            touched[page, :held[page]] |= bool((old != s).any())
            still = ~moved
            assert torch.equal(codes[page][:, :held[page]][still], before[page][:, :held[page]][still])
    keep = ~touched[:, None, :, None].expand_as(codes)
    assert torch.equal(codes[keep], before[keep]), name
    others = torch.tensor([p not in placed for p in range(codes.shape[0])])
    assert torch.equal(scale[others].view(torch.int32), before_scale[others].view(torch.int32)), name


def run(pg, hq, rotary=128, interleaved=False, norm=True, fused=False, base=None, axes=None, rot_scale=1.0, with_q=True, with_kv=True,
        cache=True, k_out=False, pad=0, seed=1, stream=None, inplace=False, identity=False, size=1.5, check=True, num_axes=3):
    """axes: None, "stretches" or "woven" (three position axes)."""
    g = torch.Generator().manual_seed(seed)
    T, hkv = pg.total + pad, pg.Hkv
    scaled = isinstance(pg, Scaled)
    rows = torch.randn((T, (hq + 2 * hkv) * D), generator=g) * size * torch.exp(0.7 * torch.randn((T, 1), generator=g))
    rows = rows.to(torch.bfloat16)
    if fused:
        dev = rows.cuda()
        q, k, v, strides = dev[:, :hq * D], dev[:, hq * D:(hq + hkv) * D], dev[:, (hq + hkv) * D:], (rows.shape[1],) * 3
    else:
        q, k, v = (x.contiguous().cuda() for x in (rows[:, :hq * D], rows[:, hq * D:(hq + hkv) * D], rows[:, (hq + hkv) * D:]))
        strides = (0, 0, 0)
    inv = torch.from_numpy(qf.rope_frequencies(rotary, 1e6)[0]) if rotary else torch.zeros(1)
    qg = bf16(1 + 0.3 * np.random.default_rng(seed).standard_normal(D)) if norm else None
    kg = bf16(1 + 0.3 * np.random.default_rng(seed + 1).standard_normal(D)) if norm else None
    positions = pair_axis = None
    if axes:
        positions = torch.randint(-50, 100000, (num_axes, T), generator=g, dtype=torch.int32)
        cut = [rotary // 2 - 2 * (rotary // 6)] + [rotary // 6] * 2 if num_axes == 3 else [rotary // 2] + [0] * (num_axes - 1)
        pair_axis = torch.from_numpy(qf.rope_pair_axes(rotary, cut, axes == "woven"))
    p = qf.params(pg.B, hq, hkv, pg.width, 1, pg.num_pages, flags=qf.QF_FLAG_KV_NHD if pg.nhd else 0)
    r = qf.rope_params(T, rotary, interleaved, 1e-6, rot_scale, *strides)
    qo = (q if inplace else torch.full((T, hq, D), float("nan"), dtype=torch.bfloat16, device="cuda")) if with_q else None
    ko = torch.full((T, hkv, D), float("nan"), dtype=torch.bfloat16, device="cuda") if k_out else None
    up = lambda t: None if t is None else t.cuda()      # noqa: E731
    pools = pg.device() if scaled else list(pg.pools())
    common = (None if identity else pg.table.cuda(), pg.cu.cuda(), pg.lens.cuda())
    heads = (q if with_q else None, k if with_kv else None, v if with_kv and cache else None, qo, ko)
    tail = (up(qg), up(kg), up(inv) if rotary else None, p, r)
    if scaled:
        qf.rope_append_scaled(*heads, *(pools if cache else [None] * 4), *common, up(base), up(positions), up(pair_axis), *tail,
                              kv_type=pg.type, stream=stream)
    else:
        qf.rope_append_axes(*heads, *(pools if cache else [None] * 2), *common, up(positions), up(pair_axis), *tail, stream=stream)
    assert qf.last_launch_count() == 1
    torch.cuda.synchronize()
    if not check:
        return qo, pools

    req = np.repeat(np.arange(pg.B), pg.new)
    slot = np.concatenate([np.arange(n) + c for n, c in zip(pg.new, pg.cached)]) if pg.total else np.zeros(0, int)
    pos = slot + (base.numpy()[req] if base is not None else 0)
    pos = np.broadcast_to(pos, (max(rotary // 2, 1), pg.total)) if positions is None else positions.numpy()[pair_axis.numpy()][:, :pg.total]
    live = rows[:pg.total]
    turn = lambda x, h, gain: turn64(x.reshape(-1, h, D), np.array(pos), inv, rotary, interleaved, gain, 1e-6, rot_scale)  # noqa: E731
    if with_q:
        got = qo.reshape(T, hq, D).cpu()
        check_rows(got[:pg.total], turn(live[:, :hq * D], hq, qg))
        if inplace:
            assert torch.equal(got[pg.total:].reshape(-1, hq * D), rows[pg.total:, :hq * D])
        else:
            assert torch.isnan(got[pg.total:]).all()          # rows of no request are left as they were
    if not with_kv:
        return qo, pools
    kref, vref = turn(live[:, hq * D:(hq + hkv) * D], hkv, kg), live[:, (hq + hkv) * D:].reshape(-1, hkv, D).double()
    if k_out:
        check_rows(ko.cpu()[:pg.total], kref)
        assert torch.isnan(ko.cpu()[pg.total:]).all()
    placed, held, kw, vw = {}, {}, {}, {}
    for i in range(pg.total if cache else 0):
        b, s = int(req[i]), int(slot[i])
        if s // PAGE >= pg.width:
            continue
        page = b * pg.width + s // PAGE if identity else int(pg.table[b, s // PAGE])
        if not 0 <= page < pg.num_pages:
            continue
        held.setdefault(page, s % PAGE)
        placed.setdefault(page, []).append(s % PAGE)
        kw[page, s % PAGE], vw[page, s % PAGE] = kref[i], vref[i]
    if scaled:
        order = (0, 2, 1, 3) if pg.nhd else (0, 1, 2, 3)
        for n, w, want in (("k", 0, kw), ("v", 1, vw)):
            check_pool(pg, n, pools[w].cpu().permute(order).contiguous(), pools[2 + w].cpu(), pg.codes[w], pg.scale[w], want, placed, held)
    else:
        gk, gv = (pg.head_major(x) for x in pools)
        written = torch.zeros((pg.num_pages, PAGE), dtype=torch.bool)
        for (page, s), row in kw.items():
            check_rows(gk[page, :, s], row)
            assert torch.equal(gv[page, :, s].double(), vw[page, s])
            written[page, s] = True
        keep = ~written[:, None, :, None].expand_as(pg.k)
        bits = lambda t: t.view(torch.int16)      # noqa: E731
        assert torch.equal(bits(gk)[keep], bits(pg.k)[keep]) and torch.equal(bits(gv)[keep], bits(pg.v)[keep])
    return qo, pools


# ---------------------------------------------------------------------------------------------- scaled cache
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 8), (16, 8), (28, 4), (40, 8), (6, 2), (3, 3)])
@pytest.mark.parametrize("nhd", [False, True])
def test_head_counts_and_layouts(kind, hq, hkv, nhd):
    run(Scaled([5, 1, 0, 17, 33], [0, 15, 3, 16, 100], hkv, kind, nhd), hq)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rotary", [0, 16, 64, 112, 128])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_rotary_part_and_pair_layout(kind, rotary, interleaved, norm):
    run(Scaled([3, 40, 1], [7, 0, 31], 2, kind), 6, rotary=rotary, interleaved=interleaved, norm=norm)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("new", [[1], [1] * 8, [1] * 300, [0, 0, 1, 0], [2000], [700, 1, 0, 900, 3], [2, 3] * 40, [1] * 20 + [600, 500]])
@pytest.mark.parametrize("fused", [False, True])
def test_lengths(kind, new, fused):
    cached = [(7 * i) % 50 for i in range(len(new))]
    run(Scaled(new, cached, 2, kind, fused), 4, fused=fused, pad=3)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("start", range(16))
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 33])
def test_every_place_within_a_page(kind, start, n):
    run(Scaled([n, 1, n], [start, 15 - start, start + 16], 1, kind, seed=start), 2, seed=n)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("axes", ["stretches", "woven"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rotary", [48, 96, 128])
def test_axes_into_a_scaled_cache(kind, axes, interleaved, rotary):
    run(Scaled([30, 1, 200], [0, 9, 40], 2, kind), 6, rotary=rotary, interleaved=interleaved, axes=axes, pad=2)


@pytest.mark.parametrize("kind", KINDS)
def test_position_base_and_rotation_scale(kind):
    run(Scaled([30, 1], [0, 9], 2, kind), 6, base=torch.tensor([1000000, 77], dtype=torch.int32), rot_scale=1.3)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("what", ["queries", "keys", "keys only out", "in place", "with keys out", "identity"])
def test_what_may_be_left_out(kind, what):
    kw = {"queries": dict(with_kv=False, cache=False), "keys": dict(with_q=False), "keys only out": dict(cache=False, k_out=True),
          "in place": dict(inplace=True, pad=2), "with keys out": dict(k_out=True, pad=5), "identity": dict(identity=True)}[what]
    pg = Scaled([20, 1, 70], [5, 3, 0], 2, kind)
    if what == "identity":
        pg = Scaled([20, 1, 70], [5, 3, 0], 2, kind, extra_pages=20)
    run(pg, 6, **kw)


@pytest.mark.parametrize("kind", KINDS)
def test_positions_without_a_page_store_nothing(kind):
    pg = Scaled([40, 30, 20], [0, 10, 90], 2, kind, max_pages=3)
    pg.table[0, 1], pg.table[1, 0] = -1, pg.num_pages
    run(pg, 4)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("power", [-130, -118, -105, -60, 60, 118])
def test_sizes_at_the_ends_of_the_range(kind, power):
    """Values near the largest bf16, and so small that the smallest scale holds them."""
    run(Scaled([20, 3], [0, 4], 2, kind), 4, norm=False, rotary=0, size=2.0 ** power)


@pytest.mark.parametrize("kind", KINDS)
def test_zeros(kind):
    pg = Scaled([20, 3], [0, 16], 2, kind)
    qo, pools = run(pg, 4, size=0.0)
    assert (pools[2][int(pg.table[0, 0])] == 2.0 ** -100).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_values_that_are_not_finite_make_their_blocks_nan(kind, value):
    hq, hkv, T = 4, 2, 40
    pg = Scaled([T], [0], hkv, kind)
    p, r = qf.params(1, hq, hkv, pg.width, 1, pg.num_pages), qf.rope_params(T, 0)
    g = torch.Generator().manual_seed(4)
    k, v = (torch.randn((T, hkv * D), generator=g).to(torch.bfloat16) for _ in range(2))
    k[17, 5], v[3, D + 9] = value, value
    kc, vc, ks, vs = pg.device()
    qf.rope_append_scaled(None, k.cuda(), v.cuda(), None, None, kc, vc, ks, vs, pg.table.cuda(), pg.cu.cuda(), pg.lens.cuda(), None, None,
                          None, None, None, None, p, r, kv_type=pg.type)
    torch.cuda.synchronize()
    bad_k, bad_v = torch.zeros((pg.num_pages, hkv), dtype=torch.bool), torch.zeros((pg.num_pages, hkv), dtype=torch.bool)
    bad_k[int(pg.table[0, 1]), 0] = bad_v[int(pg.table[0, 0]), 1] = True
    mine = [int(x) for x in pg.table[0, :3]]
    assert torch.equal(torch.isnan(ks.cpu())[mine], bad_k[mine]) and torch.equal(torch.isnan(vs.cpu())[mine], bad_v[mine])
    # the block stays NaN while it fills, and starts afresh with its first slot
    pg.lens[0] = T
    one = torch.ones((1, hkv * D), dtype=torch.bfloat16, device="cuda")
    ks[int(pg.table[0, 2]), 0] = float("nan")
    cu = torch.tensor([0, 1], dtype=torch.int32).cuda()
    for lens, want in ((T, True), (32, False)):
        qf.rope_append_scaled(None, one, one, None, None, kc, vc, ks, vs, pg.table.cuda(), cu, torch.tensor([lens], dtype=torch.int32).cuda(),
                              None, None, None, None, None, None, p, qf.rope_params(1, 0), kv_type=pg.type)
        torch.cuda.synchronize()
        assert bool(torch.isnan(ks[int(pg.table[0, 2]), 0])) == want


@pytest.mark.parametrize("kind", KINDS)
def test_a_scale_that_is_no_power_of_two_stays_while_it_suffices(kind):
    run(Scaled([3, 2, 1], [5, 8, 1], 2, kind, scales="any", k_scale=40.0), 4, size=0.5, norm=False)
    run(Scaled([3, 2, 1], [5, 8, 1], 2, kind, scales="any", k_scale=0.01), 4, size=5.0, norm=False)


@pytest.mark.parametrize("kind", KINDS)
def test_token_by_token_and_at_once(kind):
    """A block filled token by token ends with the scale that it gets at once; e4m3 codes differ only where a rounding under
    an earlier scale fell below the smallest normal number, integers by what the roundings under smaller scales can add."""
    n, hkv = 48, 2
    g = torch.Generator().manual_seed(3)
    rows = (torch.randn((n, hkv * D), generator=g) * torch.exp(1.5 * torch.randn((n, 1), generator=g))).to(torch.bfloat16).cuda()
    pg = Scaled([n], [0], hkv, kind)
    p = qf.params(1, 4, hkv, pg.width, 1, pg.num_pages)
    a, b = pg.device(), pg.device()
    cu = lambda m: torch.tensor([0, m], dtype=torch.int32).cuda()      # noqa: E731
    at = lambda m: torch.tensor([m], dtype=torch.int32).cuda()      # noqa: E731
    go = lambda pools, x, m, start: qf.rope_append_scaled(None, x, x, None, None, *pools, pg.table.cuda(), cu(m), at(start), None, None, None,  # noqa: E731
                                                          None, None, None, p, qf.rope_params(m, 0), kv_type=pg.type)
    go(a, rows, n, 0)
    for i in range(n):
        go(b, rows[i:i + 1], 1, i)
    torch.cuda.synchronize()
    pages = pg.table[0, :3].long()
    for w in (0, 1):
        s = a[2 + w].cpu()[pages]
        assert torch.equal(s, b[2 + w].cpu()[pages])
        x, y = (numbers(t[w].cpu()[pages], kind) for t in (a, b))
        if kind == "e4m3":
            big = x.abs() > 2.0 ** -6
            assert torch.equal(x[big], y[big]) and float((x - y).abs().max()) <= 2.0 ** -9
        else:
            assert float((x - y).abs().max()) <= 1.0      # halves of ever smaller steps before the last one's


@pytest.mark.parametrize("kind", KINDS)
def test_results_do_not_depend_on_the_batch(kind):
    """The same request alone, and behind others that shift its rows against the tiles of 16."""
    alone = Scaled([50], [7], 2, kind, extra_pages=40)
    g = torch.Generator().manual_seed(9)
    rows = torch.randn((50, 8 * D), generator=g).to(torch.bfloat16)
    inv = torch.from_numpy(qf.rope_frequencies(128)[0]).cuda()
    seen = []
    for lead in (0, 1, 13):
        x = torch.cat([torch.randn((lead, 8 * D), generator=g).to(torch.bfloat16), rows]).cuda()
        q, k, v = (t.contiguous() for t in (x[:, :4 * D], x[:, 4 * D:6 * D], x[:, 6 * D:]))
        B = lead + 1
        table = torch.full((B, alone.width), -1, dtype=torch.int32)
        table[-1] = alone.table[0]
        cu = torch.arange(B + 1, dtype=torch.int32)
        cu[-1] = lead + 50
        lens = torch.zeros(B, dtype=torch.int32)
        lens[-1] = 7
        pools = alone.device()
        qo = torch.empty((lead + 50, 4, D), dtype=torch.bfloat16, device="cuda")
        p = qf.params(B, 4, 2, alone.width, 1, alone.num_pages)
        qf.rope_append_scaled(q, k, v, qo, None, *pools, table.cuda(), cu.cuda(), lens.cuda(), None, None, None, None, None, inv, p,
                              qf.rope_params(lead + 50), kv_type=alone.type)
        torch.cuda.synchronize()
        seen.append([qo[lead:].cpu()] + [t.cpu() for t in pools])
    for other in seen[1:]:
        for x, y in zip(seen[0], other):
            assert torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8))


@pytest.mark.parametrize("kind", KINDS)
def test_another_stream_and_a_replayed_graph(kind):
    pg = Scaled([1] * 12, list(range(12)), 2, kind, seed=2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(pg, 4)
    hq, hkv, T = 4, 2, 12
    rows = torch.randn((T, 8 * D), device="cuda").to(torch.bfloat16)
    q, k, v = (t.contiguous() for t in (rows[:, :4 * D], rows[:, 4 * D:6 * D], rows[:, 6 * D:]))
    p, r, inv = qf.params(pg.B, hq, hkv, pg.width, 1, pg.num_pages), qf.rope_params(T), torch.from_numpy(qf.rope_frequencies(128)[0]).cuda()
    table, cu, lens = pg.table.cuda(), pg.cu.cuda(), pg.lens.cuda()
    a, b = pg.device(), pg.device()
    qa, qb = (torch.empty((T, hq, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    go = lambda pools, qo: qf.rope_append_scaled(q, k, v, qo, None, *pools, table, cu, lens, None, None, None, None, None, inv, p, r, kv_type=pg.type)  # noqa: E731
    go(a, qa)
    graph, cap = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(cap):
        with torch.cuda.graph(graph, stream=cap):
            go(b, qb)
    for _ in range(3):      # placing the same rows again changes nothing
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(qa, qb)
    for x, y in zip(a, b):
        assert torch.equal(x, y)


# ---------------------------------------------------------------------------------------------- axes, bf16 cache
@pytest.mark.parametrize("axes", ["stretches", "woven"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rotary", [16, 48, 96, 128])
@pytest.mark.parametrize("norm", [False, True])
def test_axes(axes, interleaved, rotary, norm):
    run(Paged([30, 1, 0, 200], [0, 9, 3, 40], 2), 6, rotary=rotary, interleaved=interleaved, axes=axes, norm=norm, pad=2)


@pytest.mark.parametrize("hq,hkv", [(1, 1), (16, 8), (28, 4), (40, 8)])
@pytest.mark.parametrize("new", [[1], [1] * 70, [3000], [5, 700, 1]])
def test_axes_over_head_counts_and_lengths(hq, hkv, new):
    run(Paged(new, [(11 * i) % 40 for i in range(len(new))], hkv, hq == 28), hq, axes="woven", fused=True, pad=1)


@pytest.mark.parametrize("num_axes", [1, 2, 8])
def test_other_numbers_of_axes(num_axes):
    run(Paged([30, 1], [0, 9], 2), 4, axes="stretches", num_axes=num_axes)


def test_equal_axes_are_plain_positions():
    """With every axis equal to the place in the sequence, the bits are qf_rope_append's."""
    pg = Paged([30, 1, 200], [0, 9, 40], 2)
    T, hq = pg.total, 4
    rows = torch.randn((T, 8 * D), device="cuda").to(torch.bfloat16)
    q, k, v = (t.contiguous() for t in (rows[:, :4 * D], rows[:, 4 * D:6 * D], rows[:, 6 * D:]))
    p, r, inv = qf.params(pg.B, hq, 2, pg.width, 1, pg.num_pages), qf.rope_params(T), torch.from_numpy(qf.rope_frequencies(128)[0]).cuda()
    pos = torch.cat([torch.arange(n) + c for n, c in zip(pg.new, pg.cached)]).to(torch.int32).repeat(3, 1).cuda()
    a, b = pg.pools(), pg.pools()
    qa, qb = (torch.empty((T, hq, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    args = (pg.table.cuda(), pg.cu.cuda(), pg.lens.cuda())
    qf.rope_append(q, k, v, qa, None, *a, *args, None, None, None, inv, p, r)
    qf.rope_append_axes(q, k, v, qb, None, *b, *args, pos, torch.from_numpy(qf.rope_pair_axes(128, [16, 24, 24])).cuda(), None, None, inv, p, r)
    torch.cuda.synchronize()
    assert torch.equal(qa, qb) and torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_axes_out_of_range_count_as_the_nearest():
    pg = Paged([40], [0], 2)
    rows = torch.randn((40, 8 * D), device="cuda").to(torch.bfloat16)
    q, inv = rows[:, :4 * D].contiguous(), torch.from_numpy(qf.rope_frequencies(128)[0]).cuda()
    p, r = qf.params(1, 4, 2, pg.width, 1, pg.num_pages), qf.rope_params(40)
    pos = torch.randint(0, 1000, (2, 40), dtype=torch.int32).cuda()
    outs = []
    for lo, hi in ((0, 1), (-5, 9)):
        axis = torch.tensor([lo] * 32 + [hi] * 32, dtype=torch.int32).cuda()
        out = torch.empty((40, 4, D), dtype=torch.bfloat16, device="cuda")
        qf.rope_append_axes(q, None, None, out, None, None, None, None, pg.cu.cuda(), pg.lens.cuda(), pos, axis, None, None, inv, p, r)
        outs.append(out)
    torch.cuda.synchronize()
    assert torch.equal(*outs)


def test_far_positions_of_an_axis():
    """Positions near 2^31: the angle is formed in 64 bits.  2^31 * 2^-53 of a turn is far below the fp32 that follows."""
    pg = Paged([8], [0], 1)
    x = torch.randn((8, D), device="cuda").to(torch.bfloat16)
    inv = torch.from_numpy(qf.rope_frequencies(128)[0])
    pos = torch.tensor([2 ** 31 - 1 - 7 * i for i in range(8)], dtype=torch.int32)
    axis = torch.zeros(64, dtype=torch.int32)
    out = torch.empty((8, 1, D), dtype=torch.bfloat16, device="cuda")
    qf.rope_append_axes(x, None, None, out, None, None, None, None, pg.cu.cuda(), pg.lens.cuda(), pos[None].cuda(), axis.cuda(), None, None,
                        inv.cuda(), qf.params(1, 1, 1, pg.width, 1, pg.num_pages), qf.rope_params(8))
    torch.cuda.synchronize()
    ref = turn64(x.cpu().reshape(8, 1, D), np.broadcast_to(pos.numpy(), (64, 8)).copy(), inv, 128, False, None, 0, 1.0)
    check_rows(out.cpu(), ref)
