"""Scaled caches (one byte per number, a scale per page and KV head) for the tests, and their rules in 64 bits."""
import numpy as np
import torch

from paper_2608_15473_b200 import binding as qf
from prompt_testlib import D, PAGE, Paged

KINDS = ["e4m3", "int8"]
TYPES = {"e4m3": qf.QF_KV_E4M3, "int8": qf.QF_KV_INT8}
LIMIT = {"e4m3": 448.0, "int8": 127.0}


def numbers(codes, kind):
    """Bytes -> the numbers they are, in 64 bits, not scaled."""
    return codes.contiguous().view(torch.float8_e4m3fn if kind == "e4m3" else torch.int8).double()


def codes_of(z, kind):
    """Numbers within range, in 64 bits -> the nearest codes, ties to even."""
    if kind == "int8":
        return torch.round(z).clamp(-127, 127).to(torch.int8).view(torch.uint8)
    unit = step_of(z, kind)
    z = torch.round(z / unit) * unit
    return z.to(torch.float32).to(torch.float8_e4m3fn).view(torch.uint8)


def step_of(z, kind):
    """The distance between codes around z: e4m3 has four significant bits, down to steps of 2^-9."""
    if kind == "int8":
        return torch.ones_like(z)
    return torch.ldexp(torch.ones_like(z), torch.frexp(z.abs().clamp(min=2.0 ** -6))[1] - 4)


def scale_for(top, kind):
    """The smallest power of two, 2^-100 at least, with top <= limit * scale; NaN for a top that is not finite."""
    part, power = torch.frexp(top.double() / LIMIT[kind])
    power = torch.where(top > 0, power - (part == 0.5).int(), torch.full_like(power, -100)).clamp(min=-100)
    s = torch.ldexp(torch.ones_like(top, dtype=torch.float64), power)
    return torch.where(torch.isfinite(top), s, torch.full_like(s, float("nan")))


class Scaled(Paged):
    """Paged with a scaled cache.  k, v: the numbers that the codes stand for, in 64 bits.  scales: "power" as the library
    writes them, or "any".  poison: what no request holds is NaN, or a large integer, and so are the scales of pages that
    no request holds."""

    def __init__(self, new, cached, hkv, kind, nhd=False, seed=0, extra_pages=3, max_pages=None, poison=False, scales="power",
                 k_scale=1.0):
        super().__init__(new, cached, hkv, nhd, seed, extra_pages, max_pages, False, k_scale)
        g = torch.Generator().manual_seed(seed + 77)
        self.kind, self.type = kind, TYPES[kind]
        used = torch.zeros((self.num_pages, PAGE), dtype=torch.bool)
        for b in range(self.B):
            for i in range(self.new[b] + self.cached[b]):
                if i // PAGE < self.width:
                    used[int(self.table[b, i // PAGE]), i % PAGE] = True
        self.codes, self.scale = [], []
        for pool in (self.k, self.v):
            x = pool.double() * torch.exp(0.5 * torch.randn((self.num_pages, hkv, 1, 1), generator=g, dtype=torch.float64))
            s = scale_for(x.abs().amax(dim=(2, 3)), kind)
            if scales == "any":
                s = (s * (1 + torch.rand(s.shape, generator=g, dtype=torch.float64))).float().double()
            c = codes_of(x / s[:, :, None, None], kind)
            if poison:
                c[~used[:, None, :, None].expand_as(c)] = 0x7f
                s[~used.any(1)] = float("nan")
            self.codes.append(c)
            self.scale.append(s.float())
        self.k, self.v = ((numbers(c, kind) * s.double()[:, :, None, None]) for c, s in zip(self.codes, self.scale))
        self.g = g

    def device(self):
        """k_cache, v_cache, k_scale, v_scale in the layout asked for."""
        order = (0, 2, 1, 3) if self.nhd else (0, 1, 2, 3)
        return [c.permute(order).contiguous().cuda() for c in self.codes] + [s.cuda() for s in self.scale]


def states64(pg, q, ranges, scale=None):
    """Shard states of single queries q [B, Hq, D] over [beg, end) ranges [B, S, 2] of each request's cached positions: a
    dict of [B, S, Hq(, D)] arrays out, lse, m and slack, what a relative error of 2^-20 of every |q_i k_i| and the weights'
    rounding could do."""
    B, Hq, _ = q.shape
    S, grp = ranges.shape[1], Hq // pg.Hkv
    r = dict(out=torch.zeros((B, S, Hq, D), dtype=torch.float64), lse=torch.full((B, S, Hq), -np.inf, dtype=torch.float64),
             m=torch.full((B, S, Hq), -np.inf, dtype=torch.float64), slack=torch.zeros((B, S, Hq, D), dtype=torch.float64),
             lse_slack=torch.zeros((B, S, Hq), dtype=torch.float64))
    f = D ** -0.5 if scale is None else scale
    for b in range(B):
        n = min(pg.cached[b], pg.width * PAGE)
        k, v = pg.rows(b, n, "k").to(q.device), pg.rows(b, n, "v").to(q.device)
        x = q[b].double().reshape(pg.Hkv, grp, D)
        sc = torch.einsum("cgd,cnd->cgn", x, k) * f
        mass = torch.einsum("cgd,cnd->cgn", x.abs(), k.abs()) * f
        for s in range(S):
            lo, hi = max(int(ranges[b, s, 0]), 0), min(int(ranges[b, s, 1]), n)
            if hi <= lo:
                continue
            y = sc[..., lo:hi]
            m = y.amax(-1)
            z = torch.logsumexp(y, -1)
            w = torch.exp(y - z[..., None])
            err = 2.0 ** -20 * mass[..., lo:hi].amax(-1)      # of any score
            r["out"][b, s] = torch.einsum("cgn,cnd->cgd", w, v[:, lo:hi]).reshape(Hq, D).cpu()
            spread = torch.einsum("cgn,cnd->cgd", w, v[:, lo:hi].abs())
            # a weight's second 16-bit term ends at 2^-25 where its page's largest weight is 2^14, so at 2^-39 of that: sixteen
            # such errors per page, and the pages' largest weights add up to 1 at most, are 2^-35 of the largest value
            floor = 2.0 ** -35 * v[:, lo:hi].abs().amax(1)
            r["slack"][b, s] = ((2 * err[..., None] + 2.0 ** -19) * spread + floor[:, None]).reshape(Hq, D).cpu()
            r["lse_slack"][b, s] = err.reshape(Hq).cpu()
            r["m"][b, s], r["lse"][b, s] = m.reshape(Hq).cpu(), z.reshape(Hq).cpu()
    return r


def merge64(r, counts=None):
    """Shard states -> (out, lse, slack, lse_slack)."""
    lse = r["lse"].clone()
    if counts is not None:
        for b, c in enumerate(counts):
            lse[b, int(c):] = -np.inf
    m = lse.amax(1, keepdim=True)
    safe = torch.where(torch.isneginf(m), torch.zeros_like(m), m)
    w = torch.exp(lse - safe)
    z = w.sum(1)
    w = w / torch.where(z == 0, torch.ones_like(z), z)[:, None]
    return ((w[..., None] * r["out"]).sum(1), safe[:, 0] + torch.log(z),
            (w[..., None] * (r["slack"] + 2 * r["lse_slack"][..., None] * r["out"].abs())).sum(1), r["lse_slack"].amax(1))


def even_ranges(lens, S):
    lens = np.asarray(lens)
    step = -(-lens // S)
    lo = np.minimum(np.arange(S)[None] * step[:, None], lens[:, None])
    return torch.as_tensor(np.stack([lo, np.minimum(lo + step[:, None], lens[:, None])], -1), dtype=torch.int32)
