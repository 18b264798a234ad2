"""The prompt-side operators together with the decode path, as a serving loop uses them."""
import numpy as np
import pytest
import torch

from paper_2608_15473_b200 import binding as qf
from paper_2608_15473_b200 import build as qf_build
from prompt_testlib import D, PAGE, attend64

pytestmark = pytest.mark.gpu
HQ, HKV, WIDTH = 16, 4, 40


@pytest.fixture(scope="module", autouse=True)
def built():
    qf_build.build()


class Server:
    """A pool, one table row per request, and the calls of one attention layer."""

    def __init__(self, batch, nhd=False, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.B, self.g, self.nhd = batch, g, nhd
        self.num_pages = batch * WIDTH + 8
        shape = (self.num_pages, PAGE, HKV, D) if nhd else (self.num_pages, HKV, PAGE, D)
        nan = lambda: torch.full(shape, float("nan"), dtype=torch.bfloat16, device="cuda")     # nothing unwritten may be read
        self.k, self.v = nan(), nan()
        self.table = torch.randperm(self.num_pages, generator=g)[:batch * WIDTH].reshape(batch, WIDTH).to(torch.int32).cuda()
        self.lens = torch.zeros(batch, dtype=torch.int32, device="cuda")
        inv, self.rot_scale = qf.rope_frequencies(D, 1e6, "yarn", factor=2.0, original_len=4096)
        self.inv = torch.from_numpy(inv).cuda()
        self.qg, self.kg = ((1 + 0.2 * torch.randn(D, generator=g)).to(torch.bfloat16).cuda() for _ in range(2))
        self.p = qf.params(batch, HQ, HKV, WIDTH, 1, self.num_pages, flags=qf.QF_FLAG_KV_NHD if nhd else 0)

    def tokens(self, n):
        return torch.randn((n, (HQ + 2 * HKV) * D), generator=self.g).to(torch.bfloat16).cuda()

    def place(self, rows, new, base=None, table=None, lens=None, p=None):
        """rope_append of `new[b]` rows per request; returns the rotated queries and the offsets."""
        cu = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32).cuda()
        q = torch.empty((rows.shape[0], HQ, D), dtype=torch.bfloat16, device="cuda")
        r = qf.rope_params(rows.shape[0], D, False, 1e-6, self.rot_scale, *[rows.stride(0)] * 3)
        qf.rope_append(rows[:, :HQ * D], rows[:, HQ * D:(HQ + HKV) * D], rows[:, (HQ + HKV) * D:], q, None, self.k, self.v,
                       self.table if table is None else table, cu, self.lens if lens is None else lens, base, self.qg, self.kg,
                       self.inv, p or self.p, r)
        return q, cu

    def attend(self, q, cu):
        T = q.shape[0]
        out, lse = torch.empty_like(q), torch.empty((T, HQ), device="cuda")
        n = qf.prompt_workspace_bytes(self.p, T)
        ws = torch.empty(n, dtype=torch.uint8, device="cuda")
        qf.prompt_attend(q, self.k, self.v, self.table, cu, self.lens, out, lse, self.p, T, ws, n)
        return out, lse

    def cached(self, b, n):
        pages = self.table[b].long()
        x = [(p[pages].permute(2, 0, 1, 3) if self.nhd else p[pages].permute(1, 0, 2, 3)).reshape(HKV, -1, D)[:, :n].double() for p in (self.k, self.v)]
        return x


def decode(s, q, lens):
    """decode_step over `lens` cached positions."""
    B = q.shape[0]
    ranges = torch.stack([torch.zeros_like(lens), lens], -1).reshape(B, 1, 2).contiguous()
    new = lambda *sh: torch.empty(sh, device="cuda")
    o, m, l, out, lse = new(B, 1, HQ, D), new(B, 1, HQ), new(B, 1, HQ), new(B, HQ, D), new(B, HQ)
    n = qf.workspace_bytes(s.p)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    qf.decode_step(q, s.k, s.v, s.table, lens, ranges, None, o, m, l, out, lse, s.p, ws, n)
    return out, lse


@pytest.mark.parametrize("nhd", [False, True])
def test_prompts_then_chunks_then_decode_steps(nhd):
    s = Server(5, nhd)
    for new in ([70, 1, 200, 0, 33], [5, 128, 1, 300, 1], [1, 0, 17, 16, 240]):
        q, cu = s.place(s.tokens(sum(new)), new)
        out, lse = s.attend(q, cu)
        for b, n in enumerate(new):
            if not n:
                continue
            rows = slice(int(cu[b]), int(cu[b]) + n)
            first = int(s.lens[b])
            k, v = s.cached(b, first + n)
            ref = attend64(q[rows].double(), k, v, torch.arange(n).cuda() + first + 1)
            tol = 2.0 ** -8 * (ref["out"].abs() + ref["spread"]) + 16 * 2.0 ** -20 * ref["spread"]
            assert ((out[rows].double() - ref["out"]).abs() <= tol).all()
            assert ((lse[rows].double() - ref["lse"]).abs() <= 1e-5 * ref["lse"].abs().clamp(min=1)).all()
        s.lens += torch.tensor(new, dtype=torch.int32, device="cuda")
    # decode steps: the sweep over everything cached, the token itself included, agrees with one-row prompts
    for _ in range(4):
        q, cu = s.place(s.tokens(5), [1] * 5)
        out, lse = s.attend(q, cu)
        s.lens += 1
        dout, dlse = decode(s, q, s.lens)
        # half a bf16 step of the output, half a step of each weight (at most max |v| altogether), fp32 sums on both sides
        vmax = torch.stack([s.cached(b, int(s.lens[b]))[1].abs().max() for b in range(5)]).float().reshape(5, 1, 1)
        assert ((out.float() - dout).abs() <= 2.0 ** -8 * (dout.abs() + vmax) + 2e-5 * vmax).all()
        assert ((out.float() - dout).norm() <= 5e-3 * dout.norm()) and ((lse - dlse).abs() <= 1e-5 * dlse.abs().clamp(min=1)).all()


@pytest.mark.parametrize("nhd", [False, True])
def test_a_shared_prefix_is_the_same_as_everyones_own_copy(nhd):
    """One prefix placed once for six requests against tables in which every row begins with the prefix's pages."""
    s = Server(6, nhd, seed=3)
    pages = 13
    s.table[:, :pages] = s.table[0, :pages]                 # everyone's row begins with the same pages
    prefix = pages * PAGE
    one = qf.params(1, HQ, HKV, WIDTH, 1, s.num_pages, flags=s.p.flags)
    s.place(s.tokens(prefix), [prefix], table=s.table[:1].contiguous(), lens=s.lens[:1].contiguous(), p=one)
    own = s.table[:, pages:].contiguous()                   # a request's own pages, counted from the prefix's end
    suffix = torch.zeros(6, dtype=torch.int32, device="cuda")
    base = torch.full((6,), prefix, dtype=torch.int32, device="cuda")
    mine = qf.params(6, HQ, HKV, WIDTH - pages, 1, s.num_pages, flags=s.p.flags)
    q = None
    for new in ([30, 1, 17, 100, 2, 64], [1] * 6, [1] * 6):
        q, _ = s.place(s.tokens(sum(new)), new, base=base, table=own, lens=suffix, p=mine)
        suffix += torch.tensor(new, dtype=torch.int32, device="cuda")
    ranges = torch.stack([torch.zeros_like(suffix), suffix], -1).reshape(6, 1, 2).contiguous()
    new = lambda *sh: torch.empty(sh, device="cuda")
    o, m, l, out, lse = new(6, 2, HQ, D), new(6, 2, HQ), new(6, 2, HQ), new(6, HQ, D), new(6, HQ)
    n = qf.prefix_workspace_bytes(mine)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    qf.prefix_step(q, s.k, s.v, own, suffix, ranges, s.table[:1, :pages].contiguous(), torch.tensor([prefix], dtype=torch.int32).cuda(),
                   torch.tensor([0, 6], dtype=torch.int32).cuda(), o, m, l, out, lse, mine, 1, pages, ws, n)
    assert qf.prefix_status(ws, mine) == 0
    dout, dlse = decode(s, q, suffix + prefix)
    # both sides keep 16 bits of each weight (2^-17) and sum in fp32; the values stay below 5
    assert float((out - dout).abs().max()) <= 5e-5 and float((lse - dlse).abs().max()) <= 1e-6 * float(dlse.abs().max().clamp(min=1))
