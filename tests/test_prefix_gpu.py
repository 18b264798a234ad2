"""qf_prefix_partial and qf_prefix_step on the GPU against softmax attention in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2608_15473_b200 import binding as qf
from paper_2608_15473_b200 import build as qf_build
from prompt_testlib import D, PAGE, Paged, attend64
from qf_testlib import ENG_LSE, ENG_OUT

pytestmark = pytest.mark.gpu
KERNELS = [pytest.param(0, id="staged"), pytest.param(qf.QF_FLAG_SIMPLE_KERNEL, id="simple")]


@pytest.fixture(scope="module", autouse=True)
def built():
    qf_build.build()


class Shared:
    """Groups of requests behind shared prefixes, each request with a suffix of its own, in one pool."""

    def __init__(self, groups, prefix, suffix, hkv, nhd=False, seed=0, poison=True):
        self.groups, self.prefix, self.suffix = list(groups), list(prefix), list(suffix)
        self.B, self.NG = len(suffix), len(groups)
        assert sum(groups) <= self.B
        self.pg = Paged([0] * (self.NG + self.B), self.prefix + self.suffix, hkv, nhd, seed, poison=poison)
        self.off = torch.tensor(np.concatenate([[0], np.cumsum(groups)]), dtype=torch.int32)
        pages = lambda ls: max(1, max(-(-x // PAGE) for x in ls))
        self.ptab = self.pg.table[:self.NG, :pages(prefix)].contiguous()
        self.stab = self.pg.table[self.NG:, :pages(suffix)].contiguous()
        self.plen, self.slen = (torch.tensor(x, dtype=torch.int32) for x in (self.prefix, self.suffix))

    def group_of(self, b):
        for g in range(self.NG):
            if self.off[g] <= b < self.off[g + 1]:
                return g
        return None

    def kv(self, seq, n, which):
        return self.pg.rows(seq, n, which).cuda()


def err(got, ref, rel):
    got, ref = got.double().cpu(), ref.cpu()
    assert torch.equal(torch.isneginf(got), torch.isneginf(ref))
    fine = torch.isfinite(ref)
    assert torch.isfinite(got[fine]).all()
    d = (got - ref).abs()[fine]
    return float((d / ref.abs().clamp(min=1.0)[fine] if rel else d).max()) if d.numel() else 0.0


def queries(B, hq, seed=4, scale=2.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((B, hq, D), generator=g) * scale).to(torch.bfloat16).cuda()


def partial(sh, q, flags=0, slot=0, slots=1):
    hq, pg = q.shape[1], sh.pg
    p = qf.params(sh.B, hq, pg.Hkv, 1, 1, pg.num_pages, flags=flags | (qf.QF_FLAG_KV_NHD if pg.nhd else 0), out_shards=slots, out_shard_offset=slot)
    kc, vc = pg.pools()
    o = torch.full((sh.B, slots, hq, D), 7.0, device="cuda")
    m, l = (torch.full((sh.B, slots, hq), 7.0, device="cuda") for _ in range(2))
    n = qf.prefix_workspace_bytes(p)
    ws = torch.full((n,), 0x5A, dtype=torch.uint8, device="cuda")
    qf.prefix_partial(q, kc, vc, sh.ptab.cuda(), sh.plen.cuda(), sh.off.cuda(), o, m, l, p, sh.NG, sh.ptab.shape[1], ws, n)
    torch.cuda.synchronize()
    status = qf.prompt_status(ws)
    others = [s for s in range(slots) if s != slot]
    assert (o[:, others] == 7).all() and (m[:, others] == 7).all() and (l[:, others] == 7).all()
    return o[:, slot], m[:, slot], l[:, slot], status


def partial64(sh, q):
    B, hq = q.shape[:2]
    o = torch.zeros((B, hq, D), dtype=torch.float64)
    m, l = (torch.full((B, hq), -np.inf, dtype=torch.float64) for _ in range(2))
    for b in range(B):
        g = sh.group_of(b)
        if g is None or sh.prefix[g] == 0:
            continue
        r = attend64(q[b:b + 1].double(), sh.kv(g, sh.prefix[g], "k"), sh.kv(g, sh.prefix[g], "v"), [sh.prefix[g]])
        o[b], m[b], l[b] = r["out"][0], r["m"][0], r["lse"][0]
    return o, m, l


def check_partial(sh, hq, flags=0, **kw):
    q = queries(sh.B, hq)
    o, m, l, status = partial(sh, q, flags, **kw)
    ro, rm, rl = partial64(sh, q)
    assert status == 0
    assert err(o, ro, False) <= ENG_OUT and err(m, rm, True) <= ENG_LSE and err(l, rl, True) <= ENG_LSE, \
        (err(o, ro, False), err(m, rm, True), err(l, rl, True))


@pytest.mark.parametrize("flags", KERNELS)
@pytest.mark.parametrize("hq,hkv", [(1, 1), (2, 1), (3, 1), (8, 2), (5, 1), (6, 1), (28, 4), (8, 1), (16, 8)])
@pytest.mark.parametrize("nhd", [False, True])
def test_every_group_size(flags, hq, hkv, nhd):
    check_partial(Shared([70, 3], [300, 129], [1] * 73, hkv, nhd), hq, flags)


@pytest.mark.parametrize("flags", KERNELS)
@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 100, 127, 128, 129, 255, 256, 257, 500, 1023])
@pytest.mark.parametrize("B", [1, 2, 33])
def test_prefix_lengths(flags, n, B):
    check_partial(Shared([B], [n], [1] * B, 2, seed=n), 8, flags)


@pytest.mark.parametrize("groups,prefix,hq,hkv", [
    ([1, 0, 5, 2], [50, 60, 0, 333], 8, 2),                # an empty group, a group with an empty prefix
    ([2] * 60, [17 * i % 400 for i in range(60)], 4, 2),   # many small groups
    ([200], [3000], 8, 1), ([33, 65], [20000, 40], 4, 1), ([1], [9000], 8, 1), ([3], [4097], 5, 1), ([300], [640], 8, 2),
])
def test_groups(groups, prefix, hq, hkv):
    check_partial(Shared(groups, prefix, [1] * sum(groups), hkv), hq)


@pytest.mark.parametrize("flags", KERNELS)
def test_requests_of_no_group_get_the_empty_state(flags):
    check_partial(Shared([3, 2], [40, 50], [1] * 9, 2), 4, flags)
    sh = Shared([3, 2], [40, 50], [1] * 9, 2)
    sh.off = sh.off + 2                                     # and before the first group
    check_partial(sh, 4, flags)


def test_writes_only_its_slot():
    check_partial(Shared([5], [100], [1] * 5, 2), 8, slot=2, slots=4)


@pytest.mark.parametrize("flags", KERNELS)
def test_growing_maxima(flags):
    sh = Shared([40], [900], [1] * 40, 2, poison=False)
    for i in range(900):
        sh.pg.k[int(sh.ptab[0, i // PAGE]), :, i % PAGE] *= 0.02 + i / 400
    check_partial(sh, 8, flags)


@pytest.mark.parametrize("flags", KERNELS)
def test_lengths_beyond_the_table_are_clamped_and_bad_pages_reported(flags):
    sh = Shared([4], [64], [1] * 4, 2)
    sh.plen += 1000
    check_partial(sh, 4, flags)
    sh = Shared([4], [160], [1] * 4, 2)
    whole = Shared([4], [144], [1] * 4, 2)
    whole.pg, whole.ptab = sh.pg, sh.ptab.clone()
    sh.ptab[0, 9] = sh.pg.num_pages + 5
    q = queries(4, 4)
    o, m, l, status = partial(sh, q, flags | qf.QF_FLAG_CHECK_BOUNDS)
    ro, rm, rl = partial64(whole, q)
    assert status == qf.QF_STATUS_BAD_PAGE and err(o, ro, False) <= ENG_OUT and err(l, rl, True) <= ENG_LSE


def step(sh, q, S=1, flags=0):
    hq, pg, B = q.shape[1], sh.pg, sh.B
    p = qf.params(B, hq, pg.Hkv, sh.stab.shape[1], S, pg.num_pages, flags=flags | (qf.QF_FLAG_KV_NHD if pg.nhd else 0))
    kc, vc = pg.pools()
    cut = -(-sh.slen // S)
    lo = torch.minimum(torch.arange(S)[None] * cut[:, None], sh.slen[:, None])
    ranges = torch.stack([lo, torch.minimum(lo + cut[:, None], sh.slen[:, None])], -1).to(torch.int32).cuda()
    nan = lambda *s: torch.full(s, float("nan"), device="cuda")
    o, m, l, out, lse = nan(B, S + 1, hq, D), nan(B, S + 1, hq), nan(B, S + 1, hq), nan(B, hq, D), nan(B, hq)
    n = qf.prefix_workspace_bytes(p)
    ws = torch.full((n,), 0x5A, dtype=torch.uint8, device="cuda")
    qf.prefix_step(q, kc, vc, sh.stab.cuda(), sh.slen.cuda(), ranges, sh.ptab.cuda(), sh.plen.cuda(), sh.off.cuda(), o, m, l,
                   out, lse, p, sh.NG, sh.ptab.shape[1], ws, n)
    launches = qf.last_launch_count()
    torch.cuda.synchronize()
    assert qf.prefix_status(ws, p) == 0
    return out, lse, launches


def step64(sh, q):
    B, hq = q.shape[:2]
    out, lse = torch.zeros((B, hq, D), dtype=torch.float64), torch.full((B, hq), -np.inf, dtype=torch.float64)
    for b in range(B):
        g = sh.group_of(b)
        parts = [] if g is None else [(g, sh.prefix[g])]
        parts.append((sh.NG + b, sh.suffix[b]))
        k, v = (torch.cat([sh.kv(s, n, w) for s, n in parts], 1) for w in "kv")
        if k.shape[1]:
            r = attend64(q[b:b + 1].double(), k, v, [k.shape[1]])
            out[b], lse[b] = r["out"][0], r["lse"][0]
    return out, lse


@pytest.mark.parametrize("S", [1, 3])
@pytest.mark.parametrize("nhd", [False, True])
@pytest.mark.parametrize("groups,prefix,suffix,hq,hkv", [
    ([8], [1000], [1 + 7 * i for i in range(8)], 16, 8),
    ([3, 1, 0, 9], [100, 0, 50, 2000], [0, 1, 300, 0, 17, 16, 5, 900, 2, 33, 0, 64, 8, 1], 10, 2),   # empty prefixes, suffixes, both
    ([40], [700], [(29 * i) % 400 for i in range(40)], 14, 2),
])
def test_step(S, nhd, groups, prefix, suffix, hq, hkv):
    sh = Shared(groups, prefix, suffix, hkv, nhd)
    q = queries(sh.B, hq)
    out, lse, launches = step(sh, q, S)
    ro, rl = step64(sh, q)
    assert launches >= 3
    assert err(out, ro, False) <= ENG_OUT and err(lse, rl, True) <= ENG_LSE, (err(out, ro, False), err(lse, rl, True))


def test_step_is_repeatable_and_survives_graph_replay():
    sh = Shared([30, 4], [1500, 77], [5 + 11 * i for i in range(34)], 2)
    q = queries(sh.B, 8)
    out, lse, _ = step(sh, q)
    again = step(sh, q)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    pg, B, hq = sh.pg, sh.B, 8
    p = qf.params(B, hq, pg.Hkv, sh.stab.shape[1], 1, pg.num_pages)
    kc, vc = pg.pools()
    ranges = torch.stack([torch.zeros_like(sh.slen), sh.slen], -1).reshape(B, 1, 2).cuda()
    new = lambda *s: torch.empty(s, device="cuda")
    o, m, l, out2, lse2 = new(B, 2, hq, D), new(B, 2, hq), new(B, 2, hq), new(B, hq, D), new(B, hq)
    n = qf.prefix_workspace_bytes(p)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    args = (q, kc, vc, sh.stab.cuda(), sh.slen.cuda(), ranges, sh.ptab.cuda(), sh.plen.cuda(), sh.off.cuda(), o, m, l, out2,
            lse2, p, sh.NG, sh.ptab.shape[1], ws, n)
    graph, st = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=st):
        qf.prefix_step(*args, stream=st)
    for _ in range(3):
        out2.zero_()
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out2, out) and torch.equal(lse2, lse)
    q.copy_(queries(B, hq, seed=99))
    graph.replay()
    torch.cuda.synchronize()
    ro, rl = step64(sh, q)
    assert err(out2, ro, False) <= ENG_OUT and err(lse2, rl, True) <= ENG_LSE


@pytest.mark.parametrize("n_groups,each,length", [(200, 1, 9000), (160, 40, 9100)])
def test_long_chains_keep_their_precision(n_groups, each, length):
    """Groups that share the same pages, so many that every slice runs through whole prefixes: the accumulators are set
    aside several times, and the result is no less exact than a short prefix's."""
    sh = Shared([each], [length], [1] * each, 1)
    sh.ptab, sh.NG, sh.B = sh.ptab.repeat(n_groups, 1), n_groups, n_groups * each
    sh.plen = torch.full((n_groups,), length, dtype=torch.int32)
    sh.off = torch.arange(n_groups + 1, dtype=torch.int32) * each
    q = queries(sh.B, 4)
    o, m, l, status = partial(sh, q)
    pick = torch.arange(0, sh.B, 61).cuda()
    k, v = sh.kv(0, length, "k"), sh.kv(0, length, "v")
    ref = attend64(q[pick].double(), k, v, torch.full((len(pick),), length).cuda())
    assert status == 0
    assert err(o[pick], ref["out"], False) <= ENG_OUT and err(m[pick], ref["m"], True) <= ENG_LSE and err(l[pick], ref["lse"], True) <= ENG_LSE
    rel = float((o[pick].double() - ref["out"]).norm() / ref["out"].norm())
    assert rel <= 8e-6, rel        # 2^-17 of rounding in the weights (4.4e-6 in the mean square) and 4e-6 of drift, together
