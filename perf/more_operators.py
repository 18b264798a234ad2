"""Measured cases of the operators around a KV cache that is held in 8 bits, and of rotary positions with several axes.

Four operators, each in its plain form (elementary torch operations) and as the calls a user makes:

  place   binding.rope_append_scaled     packed tokens of several requests: per-head norm of queries and keys, rotary
                                         positions (one axis, or time, height and width), rotated queries out, keys and
                                         values into an 8-bit paged cache with one scale per page and KV head
  axes    binding.rope_append_axes       the same placement into a bf16 cache, with several position axes
  decode  binding.decode_step_scaled     one decode step over the 8-bit cache: shard states and their merge
  prompt  binding.prompt_attend_scaled   causal attention of packed prompt tokens over the 8-bit cache

``own`` chooses between the two forms.  Head counts are the framework's own (16/8 and 32/8, the group sizes 5 and 7 of
40/8 and 28/4), pages hold 16 tokens of 128 channels.  An 8-bit cache holds e4m3 numbers or integers; its scales are
powers of two: the smallest that keeps a block of one page and one KV head in range.
"""
import math

import numpy as np
import torch

own = False

D, PAGE = 128, 16
HEADS = {"16/8": (16, 8), "32/8": (32, 8), "40/8": (40, 8), "28/4": (28, 4)}
# the largest magnitude of a code, as mantissa (in [1, 2)) and exponent: 448 and 127
TOP = {"e4m3": (1.75, 8), "int8": (127 / 64, 6)}
MIN_EXPONENT = -100


# ---------------------------------------------------------------------------------------------- cases
def _rows(name, op, kind, heads, batch, new_lo, new_hi, cached_lo, cached_hi, singles=0, rotary=0, interleaved=False,
          norm=False, fused=False, image=0, woven=False, nhd=False):
    """place, axes and prompt.  image: tokens per side of the images in the prompts (0 = text), woven: how the axes
    share the pairs."""
    return dict(name=name, op=op, kind=kind, heads=heads, batch=batch, new_lo=new_lo, new_hi=new_hi, cached_lo=cached_lo,
                cached_hi=cached_hi, singles=singles, rotary=rotary, interleaved=interleaved, norm=norm, fused=fused,
                image=image, woven=woven, nhd=nhd)


def _decode(name, kind, heads, batch, lo, hi, shards, nhd=False):
    return dict(name=name, op="decode", kind=kind, heads=heads, batch=batch, lo=lo, hi=hi, shards=shards, nhd=nhd)


def listed():
    return [
        # one decode token for each of eight requests, into pages that hold earlier tokens: launch and dependent loads
        _rows("place-decode-8", "place", "e4m3", "16/8", 8, 1, 1, 5, 300, 0, 128, False, True, True),
        # ordinary ragged prompts behind cached tokens, integers, interleaved pairs over half of each head, no norms
        _rows("place-ragged-int8", "place", "int8", "40/8", 9, 1, 1500, 0, 300, 0, 64, True, False, False, nhd=True),
        # a whole batch of long prompts with images in them
        _rows("place-images-16k", "place", "e4m3", "32/8", 5, 1000, 5600, 0, 0, 0, 128, False, True, True, 40, True),
        # a decode batch of a vision-language model on a bf16 cache
        _rows("axes-decode-64", "axes", "bf16", "32/8", 64, 1, 1, 0, 1500, 0, 128, False, True, True, 24, False),
        # prompts of a vision-language model: one large image and text around it
        _rows("axes-images-12k", "axes", "bf16", "28/4", 3, 3000, 5000, 0, 700, 0, 128, False, True, True, 60, False, True),
        # one short request
        _decode("decode-1x4k", "e4m3", "16/8", 1, 4096, 4096, 1),
        # the framework's ragged batch, in integers
        _decode("decode-32-ragged", "int8", "32/8", 32, 1024, 36480, 9),
        # a mixed serving batch, group of seven, token-major pages
        _decode("decode-160-mixed", "e4m3", "28/4", 160, 512, 12000, 3, True),
        # one request of a million tokens, split into shards
        _decode("decode-1x1m", "e4m3", "16/8", 1, 1048576, 1048576, 16),
        # one short prompt into an empty cache: time to first token
        _rows("prompt-short-200", "prompt", "int8", "16/8", 1, 200, 200, 0, 0),
        # the next 512 tokens of a prompt behind 30,000 that are cached already, two decode tokens riding along
        _rows("prompt-chunk-30k", "prompt", "e4m3", "32/8", 3, 512, 512, 30011, 30011, 2, nhd=True),
        # a long document
        _rows("prompt-long-16k", "prompt", "e4m3", "32/8", 1, 16384, 16384, 0, 0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["place", "axes", "decode", "prompt"])
    heads = rng.choice(sorted(HEADS))
    kind = "bf16" if op == "axes" else rng.choice(["e4m3", "int8"])
    nhd = rng.random() < 0.3
    if op in ("place", "axes"):
        total = _log(rng, 1, 14000)
        batch = min(total, _log(rng, 1, 256))
        per = max(1, total // batch)
        image = rng.randint(2, 64) if op == "axes" else rng.choice([0, 0, rng.randint(2, 64)])
        return _rows("", op, kind, heads, batch, max(1, per // 2), max(1, per + per // 2), 0, rng.randint(0, 600), 0,
                     rng.choice([32, 64, 96, 128, 128, 128]), rng.random() < 0.4, rng.random() < 0.7, rng.random() < 0.6,
                     image, rng.random() < 0.5, nhd)
    if op == "decode":
        tokens = _log(rng, 1, 400000)      # of the whole batch
        batch = min(tokens, _log(rng, 1, 160))
        per = max(1, tokens // batch)
        return _decode("", kind, heads, batch, max(1, per // 3), per + per // 3, rng.choice([1, 2, 5, 16]), nhd)
    if rng.random() < 0.5:      # whole prompts, packed
        longest = _log(rng, 1, 8000)
        batch = rng.randint(1, max(1, min(12, 16000 // longest)))
        return _rows("", op, kind, heads, batch, max(1, longest // 8), longest, 0, 0, nhd=nhd)
    cached = _log(rng, 1, 30000)      # chunks behind a cached context, singles riding along
    new = _log(rng, 1, 500)
    singles = rng.choice([0, 0, rng.randint(1, 6)])
    return _rows("", op, kind, heads, singles + rng.randint(1, 2), max(1, new // 2), new, cached // 3, cached, singles, nhd=nhd)


def _rng(case):
    """Lengths belong to the case, not to the seed."""
    text = "|".join("%s=%s" % (k, case[k]) for k in sorted(case) if k != "name")
    return np.random.default_rng(list(text.encode()))


def _lengths(case):
    """(new tokens, cached tokens) of every request; for decode, none and its context."""
    r, B = _rng(case), case["batch"]
    if case["op"] == "decode":
        return np.zeros(B, dtype=np.int64), r.integers(case["lo"], case["hi"] + 1, B)
    new = r.integers(case["new_lo"], case["new_hi"] + 1, B)
    new[:case["singles"]] = 1
    return new, r.integers(case["cached_lo"], case["cached_hi"] + 1, B)


def work(case):
    Hq, Hkv = HEADS[case["heads"]]
    new, cached = _lengths(case)
    T, B = int(new.sum()), case["batch"]
    width = 2 if case["kind"] == "bf16" else 1      # bytes of a cached number
    if case["op"] == "decode":
        tokens = int(cached.sum())
        pages = int((-(-cached // PAGE)).sum())
        return {"bytes": tokens * Hkv * D * 2 + pages * (Hkv * 8 + 4) + B * Hq * (D * 6 + 4), "flops": 4 * D * Hq * tokens}
    if case["op"] == "prompt":
        pairs = int((new * cached + new * (new + 1) // 2).sum())
        return {"bytes": int((new + cached).sum()) * Hkv * D * 2 + T * Hq * (D * 4 + 4), "flops": 4 * D * Hq * pairs}
    return {"bytes": T * D * (Hq * 4 + 2 * Hkv * (2 + width)), "flops": T * (Hq + Hkv) * D * (6 if case["norm"] else 3)}


# ---------------------------------------------------------------------------------------------- inputs
def _normal(g, shape, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * scale).to(torch.bfloat16)


def _i32(a):
    return torch.as_tensor(np.asarray(a), dtype=torch.int32).cuda()


def _exponent(top, kind):
    """The exponent of the smallest power of two that keeps magnitudes up to `top` in range."""
    mantissa, e = torch.frexp(top)
    limit, most = TOP[kind]
    k = (e - 1 - most) + (mantissa * 2 > limit).to(e.dtype)
    return torch.where(top > 0, k, torch.full_like(k, MIN_EXPONENT)).clamp(min=MIN_EXPONENT)


def _power(k):
    """2^k in 32 bits, exactly."""
    return ((k.to(torch.int32) + 127) << 23).view(torch.float32)


def _codes(x, kind):
    """Numbers within range -> the nearest codes, ties to even, as bytes."""
    if kind == "e4m3":
        return x.to(torch.float32).to(torch.float8_e4m3fn).view(torch.uint8)
    return x.round().clamp(-127, 127).to(torch.int8).view(torch.uint8)


def _numbers(codes, kind):
    return codes.view(torch.float8_e4m3fn if kind == "e4m3" else torch.int8)


def _tables(counts, width, seed):
    """A shuffled block table: each request's pages anywhere in the pool, unused entries 0."""
    pages = int(sum(counts))
    perm = np.random.default_rng([seed, 7]).permutation(pages + 3)
    table, at = np.zeros((len(counts), width), dtype=np.int64), 0
    for b, n in enumerate(counts):
        table[b, :n] = perm[at:at + n]
        at += n
    return table, pages + 3


def _pools(g, pages, Hkv, nhd, kind):
    """Keys and values that the cache holds already, [2, pages, ...], and their scales [2, pages, Hkv]."""
    shape = (pages, PAGE, Hkv, D) if nhd else (pages, Hkv, PAGE, D)
    if kind == "bf16":
        return torch.stack([_normal(g, shape), _normal(g, shape)]), None
    pool = torch.empty((2, *shape), dtype=torch.uint8, device="cuda")
    scale = torch.empty((2, pages, Hkv), device="cuda")
    over = (1, 3) if nhd else (2, 3)
    step = max(1, (1 << 27) // (Hkv * PAGE * D))
    for w in range(2):
        for at in range(0, pages, step):
            x = torch.randn((min(step, pages - at), *shape[1:]), generator=g, device="cuda")
            # blocks differ in size, and so in scale
            size = torch.exp(0.4 * torch.randn((x.shape[0], Hkv), generator=g, device="cuda"))
            x *= size[:, None, :, None] if nhd else size[:, :, None, None]
            s = _power(_exponent(x.abs().amax(dim=over), kind))
            scale[w, at:at + x.shape[0]] = s
            x /= s[:, None, :, None] if nhd else s[:, :, None, None]
            pool[w, at:at + x.shape[0]] = _codes(x, kind)
    return pool, scale


def _axes(case, new, cached):
    """Position axes of packed tokens, int32 [3, T]: text counts on, an image's tokens share one time and take a row and a
    column each; the position after an image follows its side."""
    out, side = [], max(1, case["image"])
    for n, c in zip(new, cached):
        i = np.arange(n) + c
        span = side * side + side      # an image, then as many text tokens as its side is long
        where, at = i // span, i % span
        base = where * (2 * side)
        inside = at < side * side
        text = base + side + (at - side * side)
        out.append(np.stack([np.where(inside, base, text), np.where(inside, base + at // side, text), np.where(inside, base + at % side, text)]))
    return np.concatenate(out, axis=1)


def _pair_axis(pairs, woven):
    """Which axis turns each pair: three stretches (half the pairs by time's share first), or in turn."""
    j = np.arange(pairs)
    if woven:
        return j % 3
    return np.where(j < pairs // 4, 0, np.where(j < pairs // 4 + (pairs - pairs // 4) // 2, 1, 2))


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    Hq, Hkv = HEADS[case["heads"]]
    B, op = case["batch"], case["op"]
    s = dict(case=case, op=op, kind=case["kind"], Hq=Hq, Hkv=Hkv, B=B, nhd=case["nhd"])
    new, cached = _lengths(case)
    T = int(new.sum())
    counts = -(-(new + cached) // PAGE)
    table, pages = _tables(counts, int(counts.max()), seed)
    s["pool"], s["scale"] = _pools(g, pages, Hkv, case["nhd"], case["kind"])
    s["pages"], s["T"], s["max_new"], s["max_len"] = pages, T, int(new.max()), int((new + cached).max())
    s["block_table"], s["seq_lens"] = _i32(table), _i32(cached)
    if op == "decode":
        S = case["shards"]
        step = -(-cached // S)
        lo = np.minimum(np.arange(S)[None, :] * step[:, None], cached[:, None])
        s["shard_ranges"] = _i32(np.stack([lo, np.minimum(lo + step[:, None], cached[:, None])], axis=-1))
        s["q"] = _normal(g, (B, Hq, D), 1.5)
        return s
    s["cu_tokens"] = _i32(np.concatenate([[0], np.cumsum(new)]))
    if op == "prompt":
        s["q"] = _normal(g, (T, Hq, D), 1.5)
        return s
    # the packed row with which each page that this step touches begins
    first = [np.concatenate([[0], np.arange(PAGE - c % PAGE, n, PAGE)]) + t for n, c, t in zip(new, cached, np.concatenate([[0], np.cumsum(new)]))]
    s["page_rows"] = torch.as_tensor(np.concatenate(first), dtype=torch.int64).cuda()
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
    s["positions"], s["pair_axis"] = None, None
    if case["image"]:
        s["positions"], s["pair_axis"] = _i32(_axes(case, new, cached)), _i32(_pair_axis(case["rotary"] // 2, case["woven"]))
    s["eps"] = 1e-6
    return s


# ---------------------------------------------------------------------------------------------- one pass
def run(state):
    if own:
        return _own(state)
    if state["op"] == "decode":
        return _plain_decode(state)
    return _plain_prompt(state) if state["op"] == "prompt" else _plain_place(state)


def _held(s):
    """What the pools hold, as values."""
    if s["kind"] == "bf16":
        return s["pool"]
    scale = s["scale"].to(torch.bfloat16)      # powers of two
    return _numbers(s["pool"], s["kind"]).to(torch.bfloat16).mul_(scale[:, :, None, :, None] if s["nhd"] else scale[:, :, :, None, None])


def _own(s):
    from paper_2608_15473_b200 import binding as qf

    op, c = s["op"], s["case"]
    if "params" not in s:      # what a program keeps between calls: the parameters, the outputs and the scratch
        S = c.get("shards", 1)
        s["params"] = qf.params(s["B"], s["Hq"], s["Hkv"], s["block_table"].shape[1], S, s["pages"],
                                flags=qf.QF_FLAG_KV_NHD if s["nhd"] else 0)
        s["k_cache"], s["v_cache"] = s["pool"][0], s["pool"][1]
        if s["scale"] is not None:
            s["k_scale"], s["v_scale"] = s["scale"][0], s["scale"][1]
            s["kv_type"] = qf.QF_KV_E4M3 if s["kind"] == "e4m3" else qf.QF_KV_INT8
        new = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
        if op in ("place", "axes"):
            s["rope"] = qf.rope_params(s["T"], c["rotary"], c["interleaved"], s["eps"], 1.0, s["q"].stride(0),
                                       s["k"].stride(0), s["v"].stride(0))
            s["q_out"] = new(s["T"], s["Hq"], D, dtype=torch.bfloat16)
        elif op == "prompt":
            s["out"], s["lse"] = new(s["T"], s["Hq"], D, dtype=torch.bfloat16), new(s["T"], s["Hq"])
            s["ws"] = new(qf.prompt_workspace_bytes(s["params"], s["T"]), dtype=torch.uint8)
        else:
            B, Hq = s["B"], s["Hq"]
            s["o_part"], s["m_part"], s["lse_part"] = new(B, S, Hq, D), new(B, S, Hq), new(B, S, Hq)
            s["out"], s["lse"] = new(B, Hq, D), new(B, Hq)
            s["ws"] = new(qf.workspace_bytes(s["params"]), dtype=torch.uint8)
    p = s["params"]
    if op == "place":
        qf.rope_append_scaled(s["q"], s["k"], s["v"], s["q_out"], None, s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"],
                              s["block_table"], s["cu_tokens"], s["seq_lens"], None, s["positions"], s["pair_axis"],
                              s["q_gain"], s["k_gain"], s["inv_freq"], p, s["rope"], kv_type=s["kv_type"])
        return {"q": s["q_out"], "kv": _held(s)}
    if op == "axes":
        qf.rope_append_axes(s["q"], s["k"], s["v"], s["q_out"], None, s["k_cache"], s["v_cache"], s["block_table"],
                            s["cu_tokens"], s["seq_lens"], s["positions"], s["pair_axis"], s["q_gain"], s["k_gain"],
                            s["inv_freq"], p, s["rope"])
        return {"q": s["q_out"], "kv": s["pool"]}
    if op == "prompt":
        qf.prompt_attend_scaled(s["q"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["block_table"],
                                s["cu_tokens"], s["seq_lens"], s["out"], s["lse"], p, s["T"], s["ws"], s["ws"].numel(),
                                kv_type=s["kv_type"])
    else:
        qf.decode_step_scaled(s["q"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["block_table"],
                              s["seq_lens"], s["shard_ranges"], None, s["o_part"], s["m_part"], s["lse_part"], s["out"],
                              s["lse"], p, s["ws"], s["ws"].numel(), kv_type=s["kv_type"])
    return {"out": s["out"], "lse": s["lse"]}


def _owner(s):
    """Request and place within it of every packed token."""
    t = torch.arange(s["T"], device="cuda")
    b = torch.searchsorted(s["cu_tokens"].long(), t, right=True) - 1
    return b, t - s["cu_tokens"].long()[b]


def _plain_place(s):
    c, T, rot = s["case"], s["T"], s["case"]["rotary"]
    b, i = _owner(s)
    slot = s["seq_lens"].long()[b] + i
    at = slot[None, :].expand(rot // 2, T) if s["positions"] is None else s["positions"].long()[s["pair_axis"].long()]
    angle = at.double().T * s["inv_freq"].double()[None, :]
    cos, sin = angle.cos().float()[:, None, :], angle.sin().float()[:, None, :]

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
        return torch.cat([pairs, x[..., rot:]], dim=-1)

    page = s["block_table"].long()[b, slot // PAGE]
    k, v = turn(s["k"], s["Hkv"], s["k_gain"]), s["v"].float().reshape(T, s["Hkv"], D)
    place = (page, slot % PAGE) if s["nhd"] else (page, slice(None), slot % PAGE)
    if s["kind"] == "bf16":
        s["pool"][0][place], s["pool"][1][place] = k.to(torch.bfloat16), v.to(torch.bfloat16)
    else:
        first = s["page_rows"]
        group = torch.searchsorted(first, torch.arange(T, device="cuda"), right=True) - 1
        at, held = page[first], slot[first] % PAGE      # the touched pages, and how many earlier tokens each holds
        old_rows = torch.arange(PAGE, device="cuda")[None, :] < held[:, None]
        for x, pool, scale in ((k, s["pool"][0], s["scale"][0]), (v, s["pool"][1], s["scale"][1])):
            top = torch.zeros((first.numel(), s["Hkv"]), device="cuda")
            top.scatter_reduce_(0, group[:, None].expand(T, s["Hkv"]), x.abs().amax(-1), "amax")
            old = torch.where(held[:, None] > 0, scale[at], torch.zeros_like(top))
            to = torch.maximum(old, _power(_exponent(top, s["kind"])))
            codes = pool[at] if s["nhd"] else pool[at].transpose(1, 2)      # [pages, 16, Hkv, D]
            again = _codes(_numbers(codes.contiguous(), s["kind"]).float() * (old / to)[:, None, :, None], s["kind"])
            codes = torch.where(old_rows[:, :, None, None], again, codes)
            pool[at] = codes if s["nhd"] else codes.transpose(1, 2)
            scale[at] = to
            pool[place] = _codes(x / to[group][:, :, None], s["kind"])
    return {"q": turn(s["q"], s["Hq"], s["q_gain"]).to(torch.bfloat16), "kv": _held(s)}


def _dense(s, w):
    """Keys (0) or values (1) behind the table as [B, Hkv, tokens, D] in 32 bits."""
    table = s["block_table"].long()
    x = _numbers(s["pool"][w][table], s["kind"]).float()
    x = x.permute(0, 3, 1, 2, 4) if s["nhd"] else x.permute(0, 2, 1, 3, 4)      # [B, Hkv, pages, 16, D]
    x = x * s["scale"][w][table].transpose(1, 2)[..., None, None]
    return x.reshape(x.shape[0], x.shape[1], -1, D)


def _plain_decode(s):
    B, Hq, Hkv = s["B"], s["Hq"], s["Hkv"]
    k = _dense(s, 0)
    w = (s["q"].float().reshape(B, Hkv, Hq // Hkv, D) @ k.transpose(2, 3)).mul_(D ** -0.5)
    del k
    w.masked_fill_((torch.arange(w.shape[-1], device="cuda")[None] >= s["seq_lens"][:, None])[:, None, None], -math.inf)
    top = w.amax(-1, keepdim=True)
    w.sub_(top).exp_()
    z = w.sum(-1, keepdim=True)
    return {"out": ((w @ _dense(s, 1)) / z).reshape(B, Hq, D), "lse": (top + z.log()).reshape(B, Hq)}


def _plain_prompt(s):
    B, Hq, Hkv, Q = s["B"], s["Hq"], s["Hkv"], s["max_new"]
    G = Hq // Hkv
    b, i = _owner(s)
    q = torch.zeros((B, Q, Hq, D), device="cuda")
    q[b, i] = s["q"].float()
    q = q.reshape(B, Q, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * Q, D)
    w = (q @ _dense(s, 0).transpose(2, 3)).mul_(D ** -0.5).reshape(B, Hkv * G, Q, -1)
    last = s["seq_lens"].long()[:, None] + torch.arange(Q, device="cuda")      # the position of each row
    hidden = torch.arange(w.shape[-1], device="cuda")[None, None, :] > last[:, :, None]
    w.masked_fill_(hidden[:, None], -math.inf)
    top = w.amax(-1, keepdim=True)
    w.sub_(top).exp_()
    z = w.sum(-1, keepdim=True)
    out = (w.reshape(B, Hkv, G * Q, -1) @ _dense(s, 1)).reshape(B, Hq, Q, D) / z
    lse = (top + z.log())[..., 0]
    return {"out": out.transpose(1, 2)[b, i].to(torch.bfloat16), "lse": lse.transpose(1, 2)[b, i]}


# ---------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return _exact_place(s) if case["op"] in ("place", "axes") else _exact_attend(s)


def _values64(s, w, b, length):
    """The first `length` positions of request b, dequantised, as [Hkv, length, D] in 64 bits."""
    pages = s["block_table"][b, : -(-length // PAGE)].long()
    x = _numbers(s["pool"][w][pages], s["kind"]).double()
    x = x if s["nhd"] else x.transpose(1, 2)
    x = x * s["scale"][w][pages].double()[:, None, :, None]
    return x.reshape(-1, s["Hkv"], D)[:length].transpose(0, 1)


def _exact_attend(s):
    Hq, Hkv, decode = s["Hq"], s["Hkv"], s["op"] == "decode"
    lens = s["seq_lens"].tolist()
    cu = list(range(s["B"] + 1)) if decode else s["cu_tokens"].tolist()
    rows_all = cu[-1]
    out = torch.empty((rows_all, Hq, D), dtype=torch.float64, device="cuda")
    lse = torch.empty((rows_all, Hq), dtype=torch.float64, device="cuda")
    for b in range(s["B"]):
        n = cu[b + 1] - cu[b]
        length = lens[b] if decode else lens[b] + n
        k, v = _values64(s, 0, b, length), _values64(s, 1, b, length)
        for at in range(0, n, 1024):
            m = min(1024, n - at)
            rows = slice(cu[b] + at, cu[b] + at + m)
            q = s["q"][rows].double().reshape(m, Hkv, Hq // Hkv, D)
            seen = torch.arange(1, m + 1, device="cuda") + (length - 1 if decode else lens[b] + at)
            for h in range(Hkv):
                x = torch.einsum("rgd,nd->grn", q[:, h], k[h]) / math.sqrt(D)
                x.masked_fill_(torch.arange(length, device="cuda")[None, :] >= seen[:, None], -math.inf)
                z = torch.logsumexp(x, dim=-1)
                part = torch.einsum("grn,nd->rgd", x.sub_(z[..., None]).exp_(), v[h])
                heads = slice(h * (Hq // Hkv), (h + 1) * (Hq // Hkv))
                out[rows, heads], lse[rows, heads] = part, z.T
    return {"out": out, "lse": lse}


def _exact_place(s):
    c, Hq, Hkv, rot = s["case"], s["Hq"], s["Hkv"], s["case"]["rotary"]
    cu, lens, bits8 = s["cu_tokens"].tolist(), s["seq_lens"].tolist(), s["kind"] != "bf16"
    kv, qo = _held(s).double(), []
    even, odd = (slice(0, rot, 2), slice(1, rot, 2)) if c["interleaved"] else (slice(0, rot // 2), slice(rot // 2, rot))

    def turn(x, gain, phase):
        x = x.double()
        if gain is not None:
            x = x / torch.sqrt(torch.sum(x ** 2, -1, keepdim=True) / D + s["eps"]) * gain.double()
        z = torch.complex(x[..., even], x[..., odd]) * phase[:, None, :]
        y = x.clone()
        y[..., even], y[..., odd] = z.real, z.imag
        return y

    for b in range(s["B"]):
        n, rows = cu[b + 1] - cu[b], slice(cu[b], cu[b + 1])
        slot = torch.arange(n, device="cuda") + lens[b]
        pos = slot[None, :].expand(rot // 2, n) if s["positions"] is None else s["positions"][:, rows].long()[s["pair_axis"].long()]
        angle = pos.double().T * s["inv_freq"].double()
        phase = torch.polar(torch.ones_like(angle), angle)
        qo.append(turn(s["q"][rows].reshape(n, Hq, D), s["q_gain"], phase))
        k = turn(s["k"][rows].reshape(n, Hkv, D), s["k_gain"], phase)
        for w, x in ((0, k), (1, s["v"][rows].reshape(n, Hkv, D).double())):
            pool = kv[w] if s["nhd"] else kv[w].transpose(1, 2)      # [pages, 16, Hkv, D]
            table = s["block_table"][b].long()
            pool[table[slot // PAGE], slot % PAGE] = x
            if not bits8:
                continue
            first = lens[b] // PAGE
            pages = table[first: (lens[b] + n - 1) // PAGE + 1]
            y = pool[pages].clone()
            token = torch.arange(pages.numel() * PAGE, device="cuda").reshape(-1, PAGE) + first * PAGE
            fresh = (token >= lens[b]) & (token < lens[b] + n)
            limit = 448.0 if s["kind"] == "e4m3" else 127.0
            top = torch.where(fresh[:, :, None, None], y.abs(), torch.zeros_like(y)).amax(dim=(1, 3))
            part, power = torch.frexp(top / limit)
            step = torch.ldexp(torch.ones_like(top), power - (part == 0.5).int())
            held = lens[b] % PAGE
            if held:
                step[0] = torch.maximum(step[0], s["scale"][w][pages[0]].double())
            z = y / step[:, None, :, None]
            if s["kind"] == "e4m3":      # four significant bits, down to the steps of 2^-9
                unit = torch.ldexp(torch.ones_like(z), torch.frexp(z.abs().clamp(min=2.0 ** -6))[1] - 4)
                z = torch.round(z / unit) * unit
            else:
                z = torch.round(z)
            # rows behind the last one keep their codes, and so mean something else under a new scale
            behind = token >= lens[b] + n
            old = (s["scale"][w][pages].double() / step)[:, None, :, None]
            pool[pages] = torch.where(behind[:, :, None, None], y / old, z * step[:, None, :, None])
    return {"q": torch.cat(qo), "kv": kv}
