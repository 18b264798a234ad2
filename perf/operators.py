"""Measured cases of the operators that fill a paged KV cache from prompts and share a prefix between requests.

Three operators, each in its plain form (elementary torch operations) and as the calls a user makes:

  place   binding.rope_append     packed tokens of several requests: per-head norm of queries and keys, rotary
                                  positions, rotated queries out, keys and values into the paged cache
  prompt  binding.prompt_attend   causal attention of packed prompt tokens over the paged cache they were placed in
  prefix  binding.prefix_step     one decode step of requests that share long prefixes: every group's prefix is swept
                                  once for all its requests, each request's own pages after that, and both are merged

``own`` chooses between the two forms.  Head counts are the framework's own (16/8 and 32/8, the group sizes 5 and 7 of
40/8 and 28/4), pages hold 16 tokens of 128 channels in bf16.
"""
import math

import numpy as np
import torch

own = False

D, PAGE = 128, 16
HEADS = {"16/8": (16, 8), "32/8": (32, 8), "40/8": (40, 8), "28/4": (28, 4)}


# ---------------------------------------------------------------------------------------------- cases
def _place(name, heads, batch, new_lo, new_hi, cached_hi, base_hi, rotary, interleaved, norm, fused, nhd):
    return dict(name=name, op="place", heads=heads, batch=batch, new_lo=new_lo, new_hi=new_hi, cached_hi=cached_hi,
                base_hi=base_hi, rotary=rotary, interleaved=interleaved, norm=norm, fused=fused, nhd=nhd)


def _prompt(name, heads, batch, new_lo, new_hi, cached_lo, cached_hi, singles, nhd):
    return dict(name=name, op="prompt", heads=heads, batch=batch, new_lo=new_lo, new_hi=new_hi, cached_lo=cached_lo,
                cached_hi=cached_hi, singles=singles, nhd=nhd)


def _prefix(name, heads, batch, groups, prefix_lo, prefix_hi, suffix_lo, suffix_hi, shards, nhd):
    return dict(name=name, op="prefix", heads=heads, batch=batch, groups=groups, prefix_lo=prefix_lo,
                prefix_hi=prefix_hi, suffix_lo=suffix_lo, suffix_hi=suffix_hi, shards=shards, nhd=nhd)


def listed():
    return [
        # one decode token for each of eight requests: only the launch and a few dependent loads
        _place("place-decode-8", "16/8", 8, 1, 1, 4096, 0, 128, False, True, True, False),
        # a decode batch far into long contexts behind shared prefixes: positions near a million
        _place("place-decode-far-256", "32/8", 256, 1, 1, 2000, 1000000, 128, False, True, True, False),
        # ordinary ragged prompts; interleaved pairs over half of each head, no norms, token-major pages
        _place("place-ragged-partial", "40/8", 9, 1, 1500, 300, 0, 64, True, False, False, True),
        # a whole batch of long prompts at once
        _place("place-long-16k", "32/8", 5, 1000, 5600, 0, 0, 128, False, True, True, False),
        # one short prompt into an empty cache: time to first token
        _prompt("prompt-short-200", "16/8", 1, 200, 200, 0, 0, 0, False),
        # ordinary packed prompts of different lengths
        _prompt("prompt-packed-8", "32/8", 8, 130, 2050, 0, 0, 0, False),
        # the next 512 tokens of a prompt behind 30,000 that are cached already
        _prompt("prompt-chunk-30k", "32/8", 1, 512, 512, 30011, 30011, 0, False),
        # a serving batch: requests that decode one token ride with two prompt chunks, group of seven, token-major
        _prompt("prompt-mixed", "28/4", 24, 500, 700, 100, 3000, 22, True),
        # a long document
        _prompt("prompt-long-16k", "32/8", 1, 16384, 16384, 0, 0, 0, False),
        # eight requests behind one system prompt
        _prefix("prefix-8x1k", "16/8", 8, 1, 1000, 1000, 1, 64, 1, False),
        # three system prompts of different lengths and popularity
        _prefix("prefix-groups", "40/8", 50, 3, 700, 9000, 1, 700, 2, True),
        # many samples of one long document
        _prefix("prefix-256x32k", "32/8", 256, 1, 32768, 32768, 16, 512, 1, False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["place", "prompt", "prefix"])
    heads = rng.choice(sorted(HEADS))
    nhd = rng.random() < 0.3
    if op == "place":
        total = _log(rng, 1, 16000)
        batch = min(total, _log(rng, 1, 256))
        per = max(1, total // batch)
        return _place("", heads, batch, max(1, per // 2), max(1, per + per // 2), rng.randint(0, 600),
                      rng.choice([0, 0, 40000, 1000000]), rng.choice([32, 64, 96, 128, 128, 128]),
                      rng.random() < 0.4, rng.random() < 0.7, rng.random() < 0.6, nhd)
    if op == "prompt":
        if rng.random() < 0.5:      # whole prompts, packed
            longest = _log(rng, 1, 8000)
            batch = rng.randint(1, max(1, min(12, 16000 // longest)))
            return _prompt("", heads, batch, max(1, longest // 8), longest, 0, 0, 0, nhd)
        cached = _log(rng, 1, 30000)      # chunks behind a cached context, singles riding along
        new = _log(rng, 1, 700)
        singles = rng.choice([0, 0, rng.randint(1, 14)])
        batch = singles + rng.randint(1, 2)
        return _prompt("", heads, batch, max(1, new // 2), new, cached // 3, cached, singles, nhd)
    batch = _log(rng, 2, 200)
    groups = min(batch, rng.choice([1, 1, 2, 5]))
    prefix = _log(rng, 40, 28000 // groups)
    return _prefix("", heads, batch, groups, max(1, prefix // 3), prefix, 1, _log(rng, 2, 500), rng.choice([1, 1, 3]), nhd)


def _rng(case):
    """Lengths belong to the case, not to the seed."""
    text = "|".join("%s=%s" % (k, case[k]) for k in sorted(case) if k != "name")
    return np.random.default_rng(list(text.encode()))


def _lengths(case):
    """(new tokens, cached tokens, rotary base) of every request of a place or prompt case."""
    r, B = _rng(case), case["batch"]
    new = r.integers(case["new_lo"], case["new_hi"] + 1, B)
    if case["op"] == "place":
        cached = r.integers(0, case["cached_hi"] + 1, B)
        base = r.integers(0, case["base_hi"] + 1, B)
    else:
        new[:case["singles"]] = 1
        cached = r.integers(case["cached_lo"], case["cached_hi"] + 1, B)
        base = np.zeros(B, dtype=np.int64)
    return new, cached, base


def _groups(case):
    """(group offsets, prefix lengths, suffix lengths) of a prefix case."""
    r, B, NG = _rng(case), case["batch"], case["groups"]
    cuts = np.sort(r.choice(np.arange(1, B), NG - 1, replace=False)) if NG > 1 else np.zeros(0, dtype=np.int64)
    off = np.concatenate([[0], cuts, [B]])
    return off, r.integers(case["prefix_lo"], case["prefix_hi"] + 1, NG), r.integers(case["suffix_lo"], case["suffix_hi"] + 1, B)


def work(case):
    Hq, Hkv = HEADS[case["heads"]]
    if case["op"] == "prefix":
        off, plen, slen = _groups(case)
        tokens = int(plen.sum() + slen.sum())
        pairs = int((np.diff(off) * plen).sum() + slen.sum())
        rows = case["batch"]
        return {"bytes": tokens * Hkv * D * 4 + rows * Hq * (D * 2 + D * 4 + 4) + (tokens // PAGE) * 4,
                "flops": 4 * D * Hq * pairs}
    new, cached, _ = _lengths(case)
    T = int(new.sum())
    if case["op"] == "place":
        return {"bytes": T * (Hq + 2 * Hkv) * D * 2 * 2, "flops": T * (Hq + Hkv) * D * (6 if case["norm"] else 3)}
    pairs = int((new * cached + new * (new + 1) // 2).sum())
    return {"bytes": int((new + cached).sum()) * Hkv * D * 4 + T * Hq * (D * 4 + 4), "flops": 4 * D * Hq * pairs}


# ---------------------------------------------------------------------------------------------- inputs
def _normal(g, shape, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * scale).to(torch.bfloat16)


def _i32(a):
    return torch.as_tensor(np.asarray(a), dtype=torch.int32).cuda()


def _tables(counts, width, seed):
    """A shuffled block table: each request's pages anywhere in the pool, unused entries 0."""
    pages = int(sum(counts))
    perm = np.random.default_rng([seed, 7]).permutation(pages + 3)
    table, at = np.zeros((len(counts), width), dtype=np.int64), 0
    for b, n in enumerate(counts):
        table[b, :n] = perm[at:at + n]
        at += n
    return table, pages + 3


def _pool(g, pages, Hkv, nhd):
    shape = (pages, PAGE, Hkv, D) if nhd else (pages, Hkv, PAGE, D)
    return _normal(g, shape), _normal(g, shape)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    Hq, Hkv = HEADS[case["heads"]]
    B = case["batch"]
    s = dict(case=case, Hq=Hq, Hkv=Hkv, B=B, nhd=case["nhd"])
    if case["op"] == "prefix":
        off, plen, slen = _groups(case)
        ppages, spages = -(-plen // PAGE), -(-slen // PAGE)
        counts = np.concatenate([ppages, spages])
        table, pages = _tables(counts, int(counts.max()), seed)
        NG, S = case["groups"], case["shards"]
        s["k_cache"], s["v_cache"] = _pool(g, pages, Hkv, case["nhd"])
        s["pages"], s["max_prefix"], s["max_suffix"] = pages, int(plen.max()), int(slen.max())
        s["prefix_table"], s["prefix_lens"] = _i32(table[:NG, :int(ppages.max())]).contiguous(), _i32(plen)
        s["block_table"], s["seq_lens"] = _i32(table[NG:, :int(spages.max())]).contiguous(), _i32(slen)
        s["group_offsets"], s["max_group"] = _i32(off), int(np.diff(off).max())
        step = -(-slen // S)
        lo = np.minimum(np.arange(S)[None, :] * step[:, None], slen[:, None])
        hi = np.minimum(lo + step[:, None], slen[:, None])
        s["shard_ranges"] = _i32(np.stack([lo, hi], axis=-1))
        s["q"] = _normal(g, (B, Hq, D), 2.0)
        return s
    new, cached, base = _lengths(case)
    T = int(new.sum())
    counts = -(-(new + cached) // PAGE)
    table, pages = _tables(counts, int(counts.max()), seed)
    s["k_cache"], s["v_cache"] = _pool(g, pages, Hkv, case["nhd"])
    s["pages"], s["T"], s["max_new"], s["max_len"] = pages, T, int(new.max()), int((new + cached).max())
    s["block_table"], s["seq_lens"] = _i32(table), _i32(cached)
    s["cu_tokens"], s["pos_base"] = _i32(np.concatenate([[0], np.cumsum(new)])), _i32(base)
    if case["op"] == "prompt":
        s["q"] = _normal(g, (T, Hq, D), 2.0)
        return s
    if case["fused"]:      # the rows of one fused projection: queries, keys and values side by side
        rows = _normal(g, (T, (Hq + 2 * Hkv) * D), 1.7)
        s["q"], s["k"], s["v"] = rows[:, :Hq * D], rows[:, Hq * D:(Hq + Hkv) * D], rows[:, (Hq + Hkv) * D:]
    else:
        s["q"], s["k"], s["v"] = _normal(g, (T, Hq * D), 1.7), _normal(g, (T, Hkv * D), 1.7), _normal(g, (T, Hkv * D), 1.7)
    s["q_gain"], s["k_gain"] = None, None
    if case["norm"]:
        s["q_gain"] = (1.0 + 0.3 * torch.randn(D, generator=g, device="cuda")).to(torch.bfloat16)
        s["k_gain"] = (1.0 + 0.3 * torch.randn(D, generator=g, device="cuda")).to(torch.bfloat16)
    half = torch.arange(case["rotary"] // 2, dtype=torch.float64) * 2.0 / case["rotary"]
    s["inv_freq"] = (1.0e6 ** -half).to(torch.float32).cuda()
    s["eps"] = 1e-6
    return s


# ---------------------------------------------------------------------------------------------- one pass
def run(state):
    op = state["case"]["op"]
    if own:
        return _own(state, op)
    if op == "place":
        return _plain_place(state)
    return _plain_prompt(state) if op == "prompt" else _plain_prefix(state)


def _own(s, op):
    from paper_2608_15473_b200 import binding as qf

    flags = qf.QF_FLAG_KV_NHD if s["nhd"] else 0
    if "params" not in s:      # what a program keeps between calls: the parameters, the outputs and the scratch
        S = s["case"].get("shards", 1)
        s["params"] = qf.params(s["B"], s["Hq"], s["Hkv"], s["block_table"].shape[1], S, s["pages"], flags=flags)
        new = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
        if op == "place":
            c = s["case"]
            s["rope"] = qf.rope_params(s["T"], c["rotary"], c["interleaved"], s["eps"], 1.0, s["q"].stride(0),
                                       s["k"].stride(0), s["v"].stride(0))
            s["q_out"] = new(s["T"], s["Hq"], D, dtype=torch.bfloat16)
        elif op == "prompt":
            s["out"], s["lse"] = new(s["T"], s["Hq"], D, dtype=torch.bfloat16), new(s["T"], s["Hq"])
            s["ws"] = new(qf.prompt_workspace_bytes(s["params"], s["T"]), dtype=torch.uint8)
        else:
            B, Hq = s["B"], s["Hq"]
            s["o_part"], s["m_part"], s["lse_part"] = new(B, S + 1, Hq, D), new(B, S + 1, Hq), new(B, S + 1, Hq)
            s["out"], s["lse"] = new(B, Hq, D), new(B, Hq)
            s["ws"] = new(qf.prefix_workspace_bytes(s["params"]), dtype=torch.uint8)
    p = s["params"]
    if op == "place":
        qf.rope_append(s["q"], s["k"], s["v"], s["q_out"], None, s["k_cache"], s["v_cache"], s["block_table"],
                       s["cu_tokens"], s["seq_lens"], s["pos_base"], s["q_gain"], s["k_gain"], s["inv_freq"], p, s["rope"])
        return {"q": s["q_out"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    if op == "prompt":
        qf.prompt_attend(s["q"], s["k_cache"], s["v_cache"], s["block_table"], s["cu_tokens"], s["seq_lens"], s["out"],
                         s["lse"], p, s["T"], s["ws"], s["ws"].numel())
    else:
        qf.prefix_step(s["q"], s["k_cache"], s["v_cache"], s["block_table"], s["seq_lens"], s["shard_ranges"],
                       s["prefix_table"], s["prefix_lens"], s["group_offsets"], s["o_part"], s["m_part"], s["lse_part"],
                       s["out"], s["lse"], p, s["case"]["groups"], s["prefix_table"].shape[1], s["ws"], s["ws"].numel())
    return {"out": s["out"], "lse": s["lse"]}


def _owner(s):
    """Request and place within it of every packed token."""
    t = torch.arange(s["T"], device="cuda")
    b = torch.searchsorted(s["cu_tokens"].long(), t, right=True) - 1
    return b, t - s["cu_tokens"].long()[b]


def _plain_place(s):
    c, T = s["case"], s["T"]
    b, i = _owner(s)
    slot = s["seq_lens"].long()[b] + i
    angle = (slot + s["pos_base"].long()[b]).double()[:, None] * s["inv_freq"].double()[None, :]
    cos, sin = angle.cos().float()[:, None, :], angle.sin().float()[:, None, :]
    rot = c["rotary"]

    def turn(x, heads, gain):
        x = x.float().reshape(T, heads, D)
        if gain is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + s["eps"]) * gain.float()
        if c["interleaved"]:
            u, w = x[..., 0:rot:2], x[..., 1:rot:2]
            pairs = torch.stack([u * cos - w * sin, w * cos + u * sin], dim=-1).reshape(T, heads, rot)
        else:
            u, w = x[..., :rot // 2], x[..., rot // 2:rot]
            pairs = torch.cat([u * cos - w * sin, w * cos + u * sin], dim=-1)
        return torch.cat([pairs, x[..., rot:]], dim=-1).to(torch.bfloat16)

    page = s["block_table"].long()[b, slot // PAGE]
    k, v = turn(s["k"], s["Hkv"], s["k_gain"]), s["v"].reshape(T, s["Hkv"], D)
    at = (page, slot % PAGE) if s["nhd"] else (page, slice(None), slot % PAGE)
    s["k_cache"][at], s["v_cache"][at] = k, v
    return {"q": turn(s["q"], s["Hq"], s["q_gain"]), "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _rows(pool, table, nhd):
    """Pages behind a table as [rows of the table, Hkv, tokens, D] in 32 bits."""
    x = pool[table.long()].float()
    x = x.permute(0, 3, 1, 2, 4) if nhd else x.permute(0, 2, 1, 3, 4)
    return x.reshape(x.shape[0], x.shape[1], -1, D)


def _plain_prompt(s):
    B, Hq, Hkv, Q = s["B"], s["Hq"], s["Hkv"], s["max_new"]
    G = Hq // Hkv
    b, i = _owner(s)
    k, v = _rows(s["k_cache"], s["block_table"], s["nhd"]), _rows(s["v_cache"], s["block_table"], s["nhd"])
    q = torch.zeros((B, Q, Hq, D), device="cuda")
    q[b, i] = s["q"].float()
    q = q.reshape(B, Q, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * Q, D)
    w = (q @ k.transpose(2, 3)).mul_(D ** -0.5).reshape(B, Hkv * G, Q, -1)
    last = s["seq_lens"].long()[:, None] + torch.arange(Q, device="cuda")      # the position of each row
    hidden = torch.arange(w.shape[-1], device="cuda")[None, None, :] > last[:, :, None]
    w.masked_fill_(hidden[:, None], -math.inf)
    top = w.amax(-1, keepdim=True)
    w.sub_(top).exp_()
    z = w.sum(-1, keepdim=True)
    out = (w.reshape(B, Hkv, G * Q, -1) @ v).reshape(B, Hq, Q, D) / z
    lse = (top + z.log())[..., 0]
    return {"out": out.transpose(1, 2)[b, i].to(torch.bfloat16), "lse": lse.transpose(1, 2)[b, i]}


def _plain_prefix(s):
    B, Hq, Hkv, R, NG = s["B"], s["Hq"], s["Hkv"], s["max_group"], s["case"]["groups"]
    G = Hq // Hkv
    q = s["q"].float()
    req = torch.arange(B, device="cuda")
    grp = torch.searchsorted(s["group_offsets"].long(), req, right=True) - 1
    at = req - s["group_offsets"].long()[grp]
    kp, vp = _rows(s["k_cache"], s["prefix_table"], s["nhd"]), _rows(s["v_cache"], s["prefix_table"], s["nhd"])
    ks, vs = _rows(s["k_cache"], s["block_table"], s["nhd"]), _rows(s["v_cache"], s["block_table"], s["nhd"])
    qg = torch.zeros((NG, R, Hq, D), device="cuda")
    qg[grp, at] = q
    qg = qg.reshape(NG, R, Hkv, G, D).transpose(1, 2).reshape(NG, Hkv, R * G, D)
    wp = (qg @ kp.transpose(2, 3)).mul_(D ** -0.5).reshape(NG, Hkv, R, G, -1)
    ws = (q.reshape(B, Hkv, G, D) @ ks.transpose(2, 3)).mul_(D ** -0.5)
    tp, ts = torch.arange(wp.shape[-1], device="cuda"), torch.arange(ws.shape[-1], device="cuda")
    wp.masked_fill_((tp[None] >= s["prefix_lens"][:, None])[:, None, None, None], -math.inf)
    ws.masked_fill_((ts[None] >= s["seq_lens"][:, None])[:, None, None], -math.inf)
    mp = wp.amax(-1).transpose(1, 2)[grp, at]                                 # [B, Hkv, G]
    top = torch.maximum(mp, ws.amax(-1))
    topg = torch.zeros((NG, R, Hkv, G), device="cuda")
    topg[grp, at] = top
    wp.sub_(topg.transpose(1, 2)[..., None]).exp_()
    ws.sub_(top[..., None]).exp_()
    op = (wp.reshape(NG, Hkv, R * G, -1) @ vp).reshape(NG, Hkv, R, G, D).transpose(1, 2)[grp, at]
    z = wp.sum(-1).transpose(1, 2)[grp, at] + ws.sum(-1)
    out = (op + ws @ vs) / z[..., None]
    return {"out": out.reshape(B, Hq, D), "lse": (top + z.log()).reshape(B, Hq)}


# ---------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "place":
        return _exact_place(s)
    return _exact_prompt(s) if case["op"] == "prompt" else _exact_prefix(s)


def _dense(pool, pages, length, nhd):
    """The first `length` tokens of a list of pages as [Hkv, length, D] in 64 bits."""
    x = pool[pages[: -(-length // PAGE)].long()].double()
    x = x if nhd else x.transpose(1, 2)
    return x.reshape(-1, x.shape[2], D)[:length].transpose(0, 1)


def _attend64(q, k, v, seen):
    """Softmax attention of q [H, rows, D] over k, v [H, n, D]; row r sees the first seen[r] positions."""
    x = torch.einsum("hrd,hnd->hrn", q, k) / math.sqrt(D)
    x = torch.where(torch.arange(k.shape[1], device="cuda") < seen[:, None], x, torch.tensor(-math.inf, device="cuda", dtype=torch.float64))
    lse = torch.logsumexp(x, dim=-1)
    return torch.einsum("hrn,hnd->hrd", x.sub_(lse[..., None]).exp_(), v), lse


def _exact_place(s):
    c, Hq, Hkv, rot = s["case"], s["Hq"], s["Hkv"], s["case"]["rotary"]
    cu, lens, base = s["cu_tokens"].tolist(), s["seq_lens"].tolist(), s["pos_base"].tolist()
    kc, vc, qo = s["k_cache"].double(), s["v_cache"].double(), []

    def turn(x, gain, pos):
        x = x.double()
        if gain is not None:
            x = x / torch.sqrt(torch.sum(x ** 2, -1, keepdim=True) / D + s["eps"]) * gain.double()
        phase = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), torch.outer(pos.double(), s["inv_freq"].double()))
        even, odd = (slice(0, rot, 2), slice(1, rot, 2)) if c["interleaved"] else (slice(0, rot // 2), slice(rot // 2, rot))
        z = torch.complex(x[..., even], x[..., odd]) * phase[:, None, :]
        y = x.clone()
        y[..., even], y[..., odd] = z.real, z.imag
        return y

    for b in range(s["B"]):
        n = cu[b + 1] - cu[b]
        rows = slice(cu[b], cu[b + 1])
        slot = torch.arange(n, device="cuda") + lens[b]
        pos = slot + base[b]
        qo.append(turn(s["q"][rows].reshape(n, Hq, D), s["q_gain"], pos))
        k = turn(s["k"][rows].reshape(n, Hkv, D), s["k_gain"], pos)
        page = s["block_table"][b].long()[slot // PAGE]
        for pool, x in ((kc, k), (vc, s["v"][rows].reshape(n, Hkv, D).double())):
            (pool if s["nhd"] else pool.transpose(1, 2))[page, slot % PAGE] = x
    return {"q": torch.cat(qo), "k_cache": kc, "v_cache": vc}


def _exact_prompt(s):
    Hq, Hkv = s["Hq"], s["Hkv"]
    cu, lens = s["cu_tokens"].tolist(), s["seq_lens"].tolist()
    out = torch.empty((s["T"], Hq, D), dtype=torch.float64, device="cuda")
    lse = torch.empty((s["T"], Hq), dtype=torch.float64, device="cuda")
    for b in range(s["B"]):
        n = cu[b + 1] - cu[b]
        k = _dense(s["k_cache"], s["block_table"][b], lens[b] + n, s["nhd"]).repeat_interleave(Hq // Hkv, 0)
        v = _dense(s["v_cache"], s["block_table"][b], lens[b] + n, s["nhd"]).repeat_interleave(Hq // Hkv, 0)
        for at in range(0, n, 2048):
            m = min(2048, n - at)
            rows = slice(cu[b] + at, cu[b] + at + m)
            seen = torch.arange(1, m + 1, device="cuda") + lens[b] + at
            o, l = _attend64(s["q"][rows].double().transpose(0, 1), k, v, seen)
            out[rows], lse[rows] = o.transpose(0, 1), l.transpose(0, 1)
    return {"out": out, "lse": lse}


def _exact_prefix(s):
    B, Hq, Hkv = s["B"], s["Hq"], s["Hkv"]
    off, plen, slen = s["group_offsets"].tolist(), s["prefix_lens"].tolist(), s["seq_lens"].tolist()
    out = torch.empty((B, Hq, D), dtype=torch.float64, device="cuda")
    lse = torch.empty((B, Hq), dtype=torch.float64, device="cuda")
    G = Hq // Hkv
    for g in range(s["case"]["groups"]):
        kp = _dense(s["k_cache"], s["prefix_table"][g], plen[g], s["nhd"])
        vp = _dense(s["v_cache"], s["prefix_table"][g], plen[g], s["nhd"])
        for b in range(off[g], off[g + 1]):
            k = torch.cat([kp, _dense(s["k_cache"], s["block_table"][b], slen[b], s["nhd"])], dim=1)
            v = torch.cat([vp, _dense(s["v_cache"], s["block_table"][b], slen[b], s["nhd"])], dim=1)
            seen = torch.full((G,), k.shape[1], device="cuda")
            o, l = _attend64(s["q"][b].double().reshape(Hkv, G, D), k, v, seen)
            out[b], lse[b] = o.reshape(Hq, D), l.reshape(Hq)
    return {"out": out, "lse": lse}
