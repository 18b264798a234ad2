"""Plain 64-bit forms of the prompt-side operators, and the inputs of their tests."""
import numpy as np
import torch

D, PAGE = 128, 16


def bf16(x):
    """float64 array -> nearest bf16 values, as a torch tensor."""
    return torch.from_numpy(np.asarray(x, dtype=np.float32)).to(torch.bfloat16)


class Paged:
    """Ragged requests over a shuffled pool: lens[b] positions cached before n[b] new rows, pages for both."""

    def __init__(self, new, cached, hkv, nhd=False, seed=0, extra_pages=3, max_pages=None, poison=False, k_scale=1.0):
        g = torch.Generator().manual_seed(seed)
        self.new, self.cached = [int(x) for x in new], [int(x) for x in cached]
        self.B, self.Hkv, self.nhd = len(self.new), hkv, nhd
        self.total = sum(self.new)
        counts = [max(0, -(-(n + c) // PAGE)) for n, c in zip(self.new, self.cached)]
        self.width = max_pages or max(1, max(counts))
        self.num_pages = sum(counts) + extra_pages
        perm = torch.randperm(self.num_pages, generator=g)
        self.table = torch.full((self.B, self.width), -7, dtype=torch.int32)   # unread entries are not valid pages
        at = 0
        for b, c in enumerate(counts):
            self.table[b, :min(c, self.width)] = perm[at:at + c][:self.width].to(torch.int32)
            at += c
        self.cu = torch.tensor(np.concatenate([[0], np.cumsum(self.new)]), dtype=torch.int32)
        self.lens = torch.tensor(self.cached, dtype=torch.int32)
        # head-major masters [pages, Hkv, 16, D]
        self.k = (torch.randn((self.num_pages, hkv, PAGE, D), generator=g) * k_scale).to(torch.bfloat16)
        self.v = torch.randn((self.num_pages, hkv, PAGE, D), generator=g).to(torch.bfloat16)
        if poison:      # everything that no request holds is NaN
            used = torch.zeros((self.num_pages, PAGE), dtype=torch.bool)
            for b in range(self.B):
                for i in range(self.new[b] + self.cached[b]):
                    if i // PAGE < self.width:
                        used[int(self.table[b, i // PAGE]), i % PAGE] = True
            dead = ~used[:, None, :, None].expand_as(self.k)
            self.k[dead], self.v[dead] = float("nan"), float("nan")

    def pools(self):
        """Device pools in the layout asked for."""
        order = (0, 2, 1, 3) if self.nhd else (0, 1, 2, 3)
        return self.k.permute(order).contiguous().cuda(), self.v.permute(order).contiguous().cuda()

    def rows(self, b, n, which):
        """The first n positions of request b as float64 [Hkv, n, D]."""
        pool = self.k if which == "k" else self.v
        pages = self.table[b, :-(-n // PAGE)].long()
        return pool[pages].permute(1, 0, 2, 3).reshape(self.Hkv, -1, D)[:, :n].double()

    def head_major(self, dev_pool):
        x = dev_pool.cpu()
        return x.permute(0, 2, 1, 3).contiguous() if self.nhd else x


def attend64(q, k, v, seen, scale=None):
    """q [rows, Hq, D], k, v [Hkv, n, D] in float64; row r sees positions < seen[r].  A dict: out, m, lse, and what the
    rounding of the weights can do: spread = sum w |v|, noise = sum w^2 v^2 (w the normalised weights)."""
    rows, hq, _ = q.shape
    grp = hq // k.shape[0]
    x = torch.einsum("rcgd,cnd->rcgn", q.reshape(rows, k.shape[0], grp, D), k) * (D ** -0.5 if scale is None else scale)
    seen = torch.as_tensor(seen, device=q.device)
    hidden = torch.arange(k.shape[1], device=q.device)[None, :] >= seen[:, None]
    x = x.masked_fill(hidden[:, None, None, :], -np.inf)
    m = x.amax(-1)
    safe = torch.where(torch.isneginf(m), torch.zeros_like(m), m)
    p = torch.exp(x - safe[..., None])
    z = p.sum(-1)
    w = p / torch.where(z == 0, torch.ones_like(z), z)[..., None]
    if torch.isfinite(v).all():
        out = torch.einsum("rcgn,cnd->rcgd", w, v)
    else:      # hidden positions are left out of the sum, whatever their values hold
        out = torch.zeros((rows, k.shape[0], grp, D), dtype=torch.float64, device=q.device)
        for r in range(rows):
            n = int(max(0, min(int(seen[r]), k.shape[1])))
            out[r] = torch.einsum("cgn,cnd->cgd", w[r, ..., :n], v[:, :n])
    fine = torch.nan_to_num(v, nan=0.0, posinf=0.0, neginf=0.0)
    d = dict(out=out, m=m, lse=safe + torch.log(z), spread=torch.einsum("rcgn,cnd->rcgd", w, fine.abs()),
             noise=torch.einsum("rcgn,cnd->rcgd", w * w, fine * fine))
    return {n: t.reshape(rows, hq, D) if t.dim() == 4 else t.reshape(rows, hq) for n, t in d.items()}


def prompt64(pg, q, max_tokens=None):
    """attend64's dict for packed q [total, Hq, D], on whatever device q is on."""
    parts = []
    cap = pg.width * PAGE if max_tokens is None else max_tokens
    for b in range(pg.B):
        n = pg.new[b]
        if n == 0:
            continue
        seen = [min(pg.cached[b] + i + 1, cap) for i in range(n)]
        rows = q[int(pg.cu[b]):int(pg.cu[b]) + n].double()
        L = max(seen)
        parts.append(attend64(rows, pg.rows(b, L, "k").to(q.device), pg.rows(b, L, "v").to(q.device), seen))
    return {n: torch.cat([d[n] for d in parts]).cpu() for n in parts[0]}


def rope64(x, pos, inv_freq, rotary, interleaved, gain=None, eps=1e-6, rot_scale=1.0):
    """Norm and rotation of x [rows, heads, D] at positions pos [rows], in float64."""
    x = x.double()
    if gain is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * gain.double()
    t = torch.as_tensor(pos, dtype=torch.float64)[:, None] * inv_freq.double()[None, :]
    c, s = torch.cos(t)[:, None] * rot_scale, torch.sin(t)[:, None] * rot_scale
    y = x.clone()
    h = rotary // 2
    a, b = (x[..., 0:rotary:2], x[..., 1:rotary:2]) if interleaved else (x[..., :h], x[..., h:rotary])
    ra, rb = a * c - b * s, b * c + a * s
    if interleaved:
        y[..., 0:rotary:2], y[..., 1:rotary:2] = ra, rb
    else:
        y[..., :h], y[..., h:rotary] = ra, rb
    return y
