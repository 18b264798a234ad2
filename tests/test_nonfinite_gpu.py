"""Scores and values that are not finite, where a row sees them: few visible positions, the last tile of a cut block, positions
behind pages that are not there.  A NaN (or +infinity) score makes its row NaN, in the result and in its log-sum-exp; the
running maximum carries it too.  Rows that do not see it are what they were."""
import pytest
import torch

from paper_2608_15473_b200 import binding as qf
from paper_2608_15473_b200 import build as qf_build
from prompt_testlib import PAGE, Paged, attend64, prompt64
from qf_testlib import ENG_LSE, ENG_OUT
from test_prefix_gpu import Shared, partial, partial64, step, step64
from test_prompt_attend_gpu import KERNELS, attend, queries

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module", autouse=True)
def built():
    qf_build.build()


def same_kind(got, ref):
    """NaN, +infinity and -infinity stand in the same places."""
    got, ref = got.double().cpu(), ref.cpu()
    for f in (torch.isnan, torch.isposinf, torch.isneginf):
        assert torch.equal(f(got), f(ref)), (f.__name__, int(f(got).sum()), int(f(ref).sum()))
    return got, ref


def check_prompt(out, lse, ref):
    """compare()'s bounds for every finite element, and the same kind of number everywhere else."""
    got, r = same_kind(out, ref["out"])
    fine = torch.isfinite(r)
    tol = 2.0 ** -8 * (r.abs() + ref["spread"]) + 16 * 2.0 ** -20 * ref["spread"]
    assert ((got - r).abs()[fine] <= tol[fine]).all()
    l, rl = same_kind(lse, ref["lse"])
    fine = torch.isfinite(rl)
    assert ((l - rl).abs()[fine] <= 1e-5 * rl.abs().clamp(min=1.0)[fine]).all()


def check_state(o, m, lse, ref):
    for got, want, tol in ((o, ref[0], ENG_OUT), (m, ref[1], None), (lse, ref[2], None)):
        if got is None:
            continue
        got, want = same_kind(got, want)
        fine = torch.isfinite(want)
        bound = ENG_OUT if tol else ENG_LSE * want.abs().clamp(min=1.0)[fine]
        assert ((got - want).abs()[fine] <= bound).all()


def put_key(pg, table_row, i, value):
    """The whole key for a NaN; one channel for an infinity (the queries' first channel is positive)."""
    row = pg.k[int(table_row[i // PAGE]), :, i % PAGE]
    if value != value:
        row[:] = value
    else:
        row[:, 0] = value


def positive_first(q):
    q[..., 0] = q[..., 0].abs() + 0.5
    return q


# ---- prompts
@pytest.mark.parametrize("flags", KERNELS)
@pytest.mark.parametrize("bad", [NAN, INF])
@pytest.mark.parametrize("n", [1, 10, 63, 64, 65, 100, 128, 129, 200])
def test_one_row_and_one_bad_key(flags, bad, n):
    """One request per place of the bad key, each with one row behind n - 1 positions, and a clean one."""
    spots = sorted({0, 5 % n, n // 2, max(n - 65, 0), n - 1})
    pg = Paged([1] * (len(spots) + 1), [n - 1] * (len(spots) + 1), 2, seed=n)
    for b, i in enumerate(spots):
        put_key(pg, pg.table[b], i, bad)
    q = positive_first(queries(pg, 8))
    out, lse, status = attend(pg, q, flags)
    ref = prompt64(pg, q)
    assert torch.isnan(ref["lse"][:-1]).all() and torch.isfinite(ref["lse"][-1]).all() and status == 0
    check_prompt(out, lse, ref)


@pytest.mark.parametrize("flags", KERNELS)
@pytest.mark.parametrize("n,cached", [(40, 0), (64, 0), (16, 40), (200, 30), (300, 0)])
def test_a_bad_key_and_a_bad_query_in_short_prompts(flags, n, cached):
    """Rows before the key are clean, rows from it on are NaN; a bad query is NaN in its own row and head alone."""
    pg = Paged([n, n], [cached, cached], 2, seed=n)
    for i in (cached + n // 2,):
        put_key(pg, pg.table[0], i, NAN)
    q = queries(pg, 8)
    q[n, 3], q[n + n // 2, 5] = NAN, NAN
    out, lse, _ = attend(pg, q, flags)
    check_prompt(out, lse, prompt64(pg, q))


def last_piece_of_one_short_tile(rows, group, heads):
    """A context length whose schedule ends in a piece of one tile with at most 64 positions."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    for cached in range(8_000, 40_000, 3):
        for c, s, h, row0, r, lo, hi, slot, narrow, before, length, _ in qf.rows_schedule(True, [0, rows], [cached], group, heads, 1 << 30, min(sms, 160)).tolist():
            if slot >= 0 and narrow and lo > 0 and hi - lo == 1 and length - lo * 128 <= 64:
                return cached
    raise AssertionError("no such schedule")


@pytest.mark.parametrize("flags", KERNELS)
@pytest.mark.parametrize("rows", [1, 9])
def test_a_bad_key_in_the_last_tile_of_a_cut_block(flags, rows):
    cached = last_piece_of_one_short_tile(rows, 4, 8)
    pg = Paged([rows], [cached], 8, seed=rows)
    clean = pg.k.clone()
    q = queries(pg, 32)
    for i in (cached, cached // 128 * 128, cached // 2, 70, 3):      # the last tile's, and one in pieces before it
        pg.k = clean.clone()
        put_key(pg, pg.table[0], i, NAN)
        out, lse, _ = attend(pg, q, flags)
        check_prompt(out, lse, prompt64(pg, q))


@pytest.mark.parametrize("flags", KERNELS)
@pytest.mark.parametrize("rows", [1, 3, 200])
@pytest.mark.parametrize("gone", [4, 8, 12, 17])
def test_a_bad_key_behind_pages_that_are_not_there(flags, rows, gone):
    """The first `gone` table entries are bad, so the first positions that count come with the NaN, or before it."""
    cached = gone * PAGE + 40
    for late in (0, 1, 39):
        pg = Paged([rows], [cached], 2, seed=gone)
        keep = list(range(gone * PAGE, cached + rows))
        put_key(pg, pg.table[0], gone * PAGE + late, NAN)
        k, v = (torch.stack([(pg.k if w == "k" else pg.v)[int(pg.table[0, i // PAGE]), :, i % PAGE] for i in keep], 1).double() for w in "kv")
        pg.table[0, :gone] = pg.num_pages + 1
        q = queries(pg, 8)
        out, lse, _ = attend(pg, q, flags)
        seen = torch.arange(rows) + 1 + cached - gone * PAGE
        check_prompt(out, lse, attend64(q.cpu().double(), k, v, seen))


@pytest.mark.parametrize("flags", KERNELS)
def test_scores_of_minus_infinity_before_a_nan(flags):
    """Weights of exactly 0 for the first positions, then a NaN: not a row that saw nothing."""
    for n in (70, 200):
        pg = Paged([1, 1], [n, n], 1, seed=n)
        for b in range(2):
            for i in range(66):
                put_key(pg, pg.table[b], i, -INF)
        put_key(pg, pg.table[0], 68, NAN)
        q = positive_first(queries(pg, 4))
        out, lse, _ = attend(pg, q, flags)
        ref = prompt64(pg, q)
        assert torch.isnan(ref["lse"][0]).all() and torch.isfinite(ref["lse"][1]).all()
        check_prompt(out, lse, ref)


# ---- shared prefixes
@pytest.mark.parametrize("flags", KERNELS)
@pytest.mark.parametrize("bad", [NAN, INF])
@pytest.mark.parametrize("n", [1, 16, 63, 64, 65, 100, 128, 200, 1000])
def test_one_bad_key_in_a_prefix(flags, bad, n):
    spots = sorted({0, n // 2, max(n - 65, 0), n - 1})
    sizes = [1, 3, 40, 2][:len(spots)] + [2]
    sh = Shared(sizes, [n] * len(sizes), [1] * sum(sizes), 2, seed=n)
    for g, i in enumerate(spots):
        put_key(sh.pg, sh.ptab[g], i, bad)
    q = positive_first(queries_of(sh, 8))
    ref = partial64(sh, q)
    assert torch.isnan(ref[2][:-2]).all() and torch.isfinite(ref[2][-2:]).all()
    o, m, l, _ = partial(sh, q, flags)
    check_state(o, m, l, ref)


def queries_of(sh, hq, seed=4):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((sh.B, hq, 128), generator=g) * 2.0).to(torch.bfloat16).cuda()


@pytest.mark.parametrize("flags", KERNELS)
def test_one_bad_key_in_a_long_cut_prefix(flags):
    """The pieces' maxima carry it too, whichever piece it is in."""
    sh = Shared([3], [20_000], [1] * 3, 2)
    clean = sh.pg.k.clone()
    q = queries_of(sh, 8)
    for i in (0, 64, 9_999, 19_967, 19_999):
        sh.pg.k = clean.clone()
        put_key(sh.pg, sh.ptab[0], i, NAN)
        o, m, l, _ = partial(sh, q, flags)
        check_state(o, m, l, partial64(sh, q))


@pytest.mark.parametrize("flags", KERNELS)
@pytest.mark.parametrize("n", [1, 40, 64, 300])
def test_a_step_behind_a_prefix_with_a_bad_key(flags, n):
    """Requests of the group are NaN, those of the other group are not."""
    sh = Shared([3, 4], [n, n], [5, 20, 33, 7, 1, 64, 100], 2, seed=n)
    put_key(sh.pg, sh.ptab[0], n // 2, NAN)
    q = queries_of(sh, 8)
    out, lse, _ = step(sh, q, 2, flags)
    ro, rl = step64(sh, q)
    assert torch.isnan(rl[:3]).all() and torch.isfinite(rl[3:]).all()
    check_state(out, None, lse, (ro, None, rl))


@pytest.mark.parametrize("flags", KERNELS)
@pytest.mark.parametrize("n", [1, 40, 300])
def test_a_step_with_nothing_but_a_prefix_with_a_bad_key(flags, n):
    """Requests without own positions: the merge sees one state, and it is NaN."""
    sh = Shared([3, 2], [n, n], [0, 7, 0, 0, 5], 2, seed=n)
    put_key(sh.pg, sh.ptab[0], n // 2, NAN)
    q = queries_of(sh, 8)
    out, lse, _ = step(sh, q, 2, flags)
    ro, rl = step64(sh, q)
    assert torch.isnan(rl[:3]).all() and torch.isfinite(rl[3:]).all()
    check_state(out, None, lse, (ro, None, rl))


@pytest.mark.parametrize("shards", [1, 3, 40])
def test_merge_of_states_of_which_only_a_nan_is_not_empty(shards):
    """qf_combine over log-sum-exps that are -inf but for a NaN, a finite one, or nothing at all."""
    hq = 4
    p = qf.params(3, hq, 2, 1, shards, 1)
    o = torch.zeros((3, shards, hq, 128), device="cuda")
    l = torch.full((3, shards, hq), -INF, device="cuda")
    o[0, shards - 1], l[0, shards - 1] = NAN, NAN
    o[1, 0], l[1, 0] = 2.0, 1.5
    out, lse = torch.full((3, hq, 128), 7.0, device="cuda"), torch.full((3, hq), 7.0, device="cuda")
    qf.combine(o, l, None, out, lse, p)
    torch.cuda.synchronize()
    assert torch.isnan(out[0]).all() and torch.isnan(lse[0]).all()
    assert (out[1] == 2).all() and (lse[1] == 1.5).all() and (out[2] == 0).all() and torch.isneginf(lse[2]).all()


def own_pages(sh, q, bad, flags, S):
    for b, spots in bad.items():
        for i in spots:
            put_key(sh.pg, sh.stab[b], i, NAN)
    out, lse, _ = step(sh, q, S, flags)
    ro, rl = step64(sh, q)
    assert torch.isnan(rl[list(bad)]).all() and int(torch.isnan(rl).sum()) == len(bad) * q.shape[1]
    check_state(out, None, lse, (ro, None, rl))


@pytest.mark.parametrize("flags", KERNELS)
@pytest.mark.parametrize("S", [1, 3])
def test_a_step_whose_own_positions_are_all_bad(flags, S):
    """A request whose own keys are all NaN is NaN, not what its prefix alone gives."""
    sh = Shared([4, 2], [100, 30], [1, 20, 300, 9, 0, 3], 2)
    own_pages(sh, queries_of(sh, 8), {0: [0], 2: range(300), 3: range(9), 5: [0, 1, 2]}, flags, S)


@pytest.mark.parametrize("flags", KERNELS)
def test_a_step_with_one_bad_key_among_own_positions(flags):
    sh = Shared([5], [100], [1, 20, 300, 9, 2000], 2)
    own_pages(sh, queries_of(sh, 8), {1: [19], 2: [0], 4: [1999]}, flags, 1)


@pytest.mark.parametrize("flags", KERNELS + [pytest.param(qf.QF_FLAG_DRAW_ALWAYS, id="drawn")])
def test_sweep_states_whose_scores_are_all_nan(flags):
    """Shards of one to many tokens, one of them cut into pieces: (NaN, ., NaN), and the step's merge of them."""
    lens = [1, 16, 100, 30_000, 40]
    pg = Paged([0] * 5, lens, 2)
    for b in (0, 2, 3):
        for i in range(lens[b]):
            put_key(pg, pg.table[b], i, NAN)
    q = torch.randn((5, 8, 128), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    p = qf.params(5, 8, 2, pg.width, 1, pg.num_pages, flags=flags)
    kc, vc = pg.pools()
    ranges = torch.stack([torch.zeros_like(pg.lens), pg.lens], -1).reshape(5, 1, 2).cuda()
    o, m, l = (torch.full(s, 7.0, device="cuda") for s in ((5, 1, 8, 128), (5, 1, 8), (5, 1, 8)))
    out, lse = torch.full((5, 8, 128), 7.0, device="cuda"), torch.full((5, 8), 7.0, device="cuda")
    n = qf.workspace_bytes(p)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    head = (q, kc, vc, pg.table.cuda(), pg.lens.cuda(), ranges)
    qf.decode_partial(*head, o, m, l, p, ws, n)
    qf.decode_step(*head, None, o.clone(), m.clone(), l.clone(), out, lse, p, ws, n)
    torch.cuda.synchronize()
    bad = torch.tensor([True, False, True, True, False])
    for x in (o[:, 0], l[:, 0], out, lse):
        assert torch.isnan(x[bad.cuda()]).all() and torch.isfinite(x[~bad.cuda()]).all()


def test_small_step_whose_scores_are_all_nan():
    """The same through the merge of small sweeps."""
    lens = [1, 40, 500]
    pg = Paged([0] * 3, lens, 1)
    for b in (0, 2):
        for i in range(lens[b]):
            put_key(pg, pg.table[b], i, NAN)
    q = torch.randn((3, 4, 128), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    for S in (1, 4):
        p = qf.params(3, 4, 1, pg.width, S, pg.num_pages)
        kc, vc = pg.pools()
        cut = -(-pg.lens // S)
        lo = torch.minimum(torch.arange(S)[None] * cut[:, None], pg.lens[:, None])
        ranges = torch.stack([lo, torch.minimum(lo + cut[:, None], pg.lens[:, None])], -1).to(torch.int32).cuda()
        o, m, l = (torch.empty(s, device="cuda") for s in ((3, S, 4, 128), (3, S, 4), (3, S, 4)))
        out, lse = torch.empty((3, 4, 128), device="cuda"), torch.empty((3, 4), device="cuda")
        n = qf.workspace_bytes(p)
        ws = torch.empty(n, dtype=torch.uint8, device="cuda")
        qf.decode_step(q, kc, vc, pg.table.cuda(), pg.lens.cuda(), ranges, None, o, m, l, out, lse, p, ws, n)
        assert qf.last_launch_count() == 2
        torch.cuda.synchronize()
        for x in (out, lse):
            assert torch.isnan(x[0]).all() and torch.isnan(x[2]).all() and torch.isfinite(x[1]).all()


# ---- values
def plant_values(sh, g, n):
    """Channel 3: +infinity; 40: -infinity; 77: both; 90: NaN; 127: +infinity twice; 64: the last position's."""
    def put(i, ch, x):
        sh.pg.v[int(sh.ptab[g, i // PAGE]), :, i % PAGE, ch] = x
    put(n // 2, 3, INF), put(n // 3, 40, -INF), put(n - 1, 64, INF), put(n // 2, 90, NAN), put(0, 127, INF), put(n // 2, 127, INF)
    if n > 1:
        put(0, 77, INF), put(n - 1, 77, -INF)


@pytest.mark.parametrize("flags", KERNELS)
@pytest.mark.parametrize("sizes,n", [([1, 2], 1), ([3, 2], 50), ([3, 1], 100), ([40, 3], 128), ([90, 2], 700), ([2, 1], 20_000), ([40, 5], 9_000)])
def test_infinite_values_of_a_prefix(flags, sizes, n):
    """Every request of the group sees them with a positive weight: infinities of one sign are the result, not NaN."""
    sh = Shared(sizes, [n, 70], [1] * sum(sizes), 2, seed=n)
    plant_values(sh, 0, n)
    q = queries_of(sh, 8)
    ref = partial64(sh, q)
    assert torch.isposinf(ref[0][:sizes[0], :, 3]).all() and torch.isfinite(ref[0][sizes[0]:]).all()
    o, m, l, _ = partial(sh, q, flags)
    check_state(o, m, l, ref)


@pytest.mark.parametrize("flags", KERNELS)
def test_infinite_values_in_a_step(flags):
    sh = Shared([5, 3], [1000, 30], [1 + 9 * i for i in range(8)], 2)
    plant_values(sh, 0, 1000)
    q = queries_of(sh, 8)
    out, lse, _ = step(sh, q, 2, flags)
    ro, rl = step64(sh, q)
    check_state(out, None, lse, (ro, None, rl))


@pytest.mark.parametrize("flags", KERNELS)
def test_infinite_values_and_a_bad_key(flags):
    """A row whose scores are NaN stays NaN; positions behind bad entries hold nothing, whatever the pool holds."""
    sh = Shared([3, 3], [200, 200], [1] * 6, 2)
    plant_values(sh, 0, 200), plant_values(sh, 1, 200)
    put_key(sh.pg, sh.ptab[0], 150, NAN)
    whole = Shared([3, 3], [200, 192], [1] * 6, 2)
    whole.pg, whole.ptab = sh.pg, sh.ptab.clone()
    q = queries_of(sh, 8)
    ref = partial64(whole, q)
    sh.ptab[1, 12] = -5
    o, m, l, _ = partial(sh, q, flags)
    check_state(o, m, l, ref)


@pytest.mark.parametrize("flags", KERNELS)
@pytest.mark.parametrize("n", [1, 30, 64, 100, 150, 300])
def test_rows_whose_every_weight_is_zero(flags, n):
    """All visible scores are -infinity: such a row is an empty set (0, -infinity), whatever the values hold."""
    pg = Paged([n, 1, n], [0, 20, 0], 2, seed=n)
    for b, last in ((0, n), (1, 21), (2, 1 + n // 2)):      # the third request: rows from 1 + n / 2 on see a finite key
        for i in range(last):
            put_key(pg, pg.table[b], i, -INF)
    for b in range(2):
        for ch, x in ((3, INF), (40, NAN), (90, -INF), (127, INF)):
            pg.v[int(pg.table[b, 0]), :, 0, ch] = x
    q = positive_first(queries(pg, 8))
    out, lse, _ = attend(pg, q, flags)
    empty = torch.tensor([True] * n + [True] + [i < 1 + n // 2 for i in range(n)]).cuda()
    assert (out[empty] == 0).all() and torch.isneginf(lse[empty]).all()
    assert torch.isfinite(out[~empty]).all() and torch.isfinite(lse[~empty]).all()


@pytest.mark.parametrize("flags", KERNELS)
@pytest.mark.parametrize("sizes,n", [([2, 1], 1), ([2, 1], 50), ([3, 2], 130), ([90, 2], 700), ([1, 1], 9_000)])
def test_prefixes_whose_every_weight_is_zero(flags, sizes, n):
    sh = Shared(sizes, [n, 70], [1] * sum(sizes), 2, seed=n)
    for i in range(n):
        put_key(sh.pg, sh.ptab[0], i, -INF)
    plant_values(sh, 0, n)
    q = positive_first(queries_of(sh, 8))
    o, m, l, _ = partial(sh, q, flags)
    a = sizes[0]
    assert (o[:a] == 0).all() and torch.isneginf(m[:a]).all() and torch.isneginf(l[:a]).all()
    assert torch.isfinite(o[a:]).all() and torch.isfinite(l[a:]).all()
