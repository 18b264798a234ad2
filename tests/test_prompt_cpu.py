"""The prompt-side operators' boundary without a GPU: refusals, rotary frequencies, workspace sizes."""
import math

import numpy as np
import pytest

from paper_2608_15473_b200 import binding as qf
from paper_2608_15473_b200 import build as qf_build

FAKE = 0x10000      # never dereferenced: validation fails first


@pytest.fixture(scope="module", autouse=True)
def built():
    qf_build.build()


def good(**kw):
    d = dict(batch=4, num_q_heads=16, num_kv_heads=8, max_pages_per_req=8, max_shards=2, num_pages=64)
    d.update(kw)
    return qf.params(**d)


# ---- rotary frequencies
def test_plain_and_linear_frequencies():
    inv, scale = qf.rope_frequencies(128, 1e6)
    want = np.array([1e6 ** (-2 * i / 128) for i in range(64)])
    assert inv.dtype == np.float32 and inv.shape == (64,) and scale == 1.0
    assert np.abs(inv / want - 1).max() <= 2.0 ** -24 + 1e-12          # one rounding to float
    lin, scale = qf.rope_frequencies(64, 1e4, "linear", factor=4.0)
    want = np.array([1e4 ** (-2 * i / 64) / 4 for i in range(32)])
    assert np.abs(lin / want - 1).max() <= 2.0 ** -24 + 1e-12 and scale == 1.0


def test_ntk_frequencies_stretch_the_base():
    inv, _ = qf.rope_frequencies(128, 1e4, "ntk", factor=8.0)
    plain, _ = qf.rope_frequencies(128, 1e4)
    assert inv[0] == 1.0 and abs(inv[-1] * 8.0 / plain[-1] - 1) < 1e-6      # the slowest pair is stretched by the factor


def test_yarn_leaves_fast_pairs_and_interpolates_slow_ones():
    factor, orig, theta, d = 4.0, 32768.0, 1e6, 128
    inv, scale = qf.rope_frequencies(d, theta, "yarn", factor=factor, original_len=orig)
    plain = np.array([theta ** (-2 * i / d) for i in range(d // 2)])
    turns = orig * plain / (2 * math.pi)
    assert np.allclose(inv[turns > 40], plain[turns > 40], rtol=1e-6)
    assert np.allclose(inv[turns < 0.8], plain[turns < 0.8] / factor, rtol=1e-6)
    assert np.all(np.diff(inv) < 0) and np.all(inv <= plain * (1 + 1e-6)) and np.all(inv >= plain / factor * (1 - 1e-6))
    assert abs(scale - (0.1 * math.log(factor) + 1)) < 1e-6
    same, one = qf.rope_frequencies(d, theta, "yarn", factor=1.0, original_len=orig)
    assert np.allclose(same, plain, rtol=1e-6) and one == 1.0


@pytest.mark.parametrize("kw,code", [
    (dict(rotary_dim=0), qf.QF_ERR_BAD_SHAPE), (dict(rotary_dim=-16), qf.QF_ERR_BAD_SHAPE),
    (dict(rotary_dim=24), qf.QF_ERR_UNSUPPORTED), (dict(rotary_dim=144), qf.QF_ERR_UNSUPPORTED),
    (dict(theta=1.0), qf.QF_ERR_BAD_SHAPE), (dict(theta=float("nan")), qf.QF_ERR_BAD_SHAPE),
    (dict(theta=float("inf")), qf.QF_ERR_BAD_SHAPE),
    (dict(scaling="linear", factor=0.5), qf.QF_ERR_BAD_SHAPE), (dict(scaling="ntk", factor=float("nan")), qf.QF_ERR_BAD_SHAPE),
    (dict(scaling="yarn", factor=2.0), qf.QF_ERR_BAD_SHAPE),
    (dict(scaling="yarn", factor=2.0, original_len=100, beta_fast=1, beta_slow=1), qf.QF_ERR_BAD_SHAPE),
])
def test_bad_frequency_arguments(kw, code):
    with pytest.raises(qf.QFError) as e:
        qf.rope_frequencies(**kw)
    assert e.value.status == code


def test_unknown_scaling_is_refused():
    with pytest.raises(ValueError):
        qf.rope_frequencies(scaling="cubic")


# ---- qf_rope_append
def rope(p=None, r=None, **kw):
    a = dict(q=FAKE, k=FAKE, v=FAKE, q_out=FAKE, k_out=None, k_cache=FAKE, v_cache=FAKE, block_table=FAKE, cu_tokens=FAKE,
             seq_lens=FAKE, pos_base=None, q_gain=None, k_gain=None, inv_freq=FAKE)
    a.update(kw)
    return qf.rope_append(*a.values(), p if p is not None else good(), r if r is not None else qf.rope_params(10),
                          stream=0, check=False)


@pytest.mark.parametrize("kw,code", [
    (dict(total_tokens=0), qf.QF_ERR_BAD_SHAPE), (dict(total_tokens=-1), qf.QF_ERR_BAD_SHAPE),
    (dict(total_tokens=4, rotary_dim=-16), qf.QF_ERR_BAD_SHAPE), (dict(total_tokens=4, rotary_dim=20), qf.QF_ERR_UNSUPPORTED),
    (dict(total_tokens=4, rotary_dim=144), qf.QF_ERR_UNSUPPORTED), (dict(total_tokens=4, eps=-1.0), qf.QF_ERR_BAD_SHAPE),
    (dict(total_tokens=4, eps=float("nan")), qf.QF_ERR_BAD_SHAPE), (dict(total_tokens=4, rot_scale=float("inf")), qf.QF_ERR_BAD_SHAPE),
    (dict(total_tokens=4, q_stride=2047), qf.QF_ERR_BAD_SHAPE), (dict(total_tokens=4, q_stride=2052), qf.QF_ERR_BAD_SHAPE),
    (dict(total_tokens=4, k_stride=1016), qf.QF_ERR_BAD_SHAPE), (dict(total_tokens=4, v_stride=-1024), qf.QF_ERR_BAD_SHAPE),
])
def test_rope_append_refuses_bad_parameters(kw, code):
    assert rope(r=qf.rope_params(**kw)) == code


@pytest.mark.parametrize("kw,code", [
    (dict(cu_tokens=None), qf.QF_ERR_NULL), (dict(seq_lens=None), qf.QF_ERR_NULL), (dict(q_out=None), qf.QF_ERR_NULL),
    (dict(q=None, q_out=None, k=None, v=None, k_cache=None, v_cache=None), qf.QF_ERR_NULL),
    (dict(k_cache=None), qf.QF_ERR_NULL), (dict(v_cache=None), qf.QF_ERR_NULL), (dict(v=None), qf.QF_ERR_NULL),
    (dict(k=None), qf.QF_ERR_NULL), (dict(k_cache=None, v_cache=None), qf.QF_ERR_NULL), (dict(inv_freq=None), qf.QF_ERR_NULL),
    (dict(k=None, v=None, k_cache=None, v_cache=None, k_out=FAKE), qf.QF_ERR_NULL),
    (dict(q=FAKE + 8), qf.QF_ERR_BAD_SHAPE), (dict(k_cache=FAKE + 8), qf.QF_ERR_BAD_SHAPE), (dict(q_gain=FAKE + 2), qf.QF_ERR_BAD_SHAPE),
])
def test_rope_append_refuses_bad_pointers(kw, code):
    assert rope(**kw) == code


def test_shared_parameters_are_checked_by_every_call():
    p = good(head_dim=64)
    assert rope(p=p) == qf.QF_ERR_UNSUPPORTED
    assert qf.prompt_workspace_bytes(p, 10) == 0 and qf.prefix_workspace_bytes(p) == 0
    assert prompt(p=p) == qf.QF_ERR_UNSUPPORTED and prefix(p=p) == qf.QF_ERR_UNSUPPORTED and step(p=p) == qf.QF_ERR_UNSUPPORTED
    p = good(num_q_heads=72)
    assert rope(p=p) == qf.QF_ERR_UNSUPPORTED and prompt(p=p) == qf.QF_ERR_UNSUPPORTED


# ---- qf_prompt_attend
def prompt(p=None, tokens=10, stride=0, ws=FAKE, ws_bytes=1 << 30, **kw):
    a = dict(q=FAKE, k_cache=FAKE, v_cache=FAKE, block_table=FAKE, cu_tokens=FAKE, seq_lens=FAKE, out=FAKE, lse=FAKE)
    a.update(kw)
    return qf.prompt_attend(*a.values(), p if p is not None else good(), tokens, ws, ws_bytes, stride, stream=0, check=False)


@pytest.mark.parametrize("kw,code", [
    (dict(tokens=0), qf.QF_ERR_BAD_SHAPE), (dict(stride=100), qf.QF_ERR_BAD_SHAPE), (dict(stride=2050), qf.QF_ERR_BAD_SHAPE),
    (dict(q=None), qf.QF_ERR_NULL), (dict(k_cache=None), qf.QF_ERR_NULL), (dict(v_cache=None), qf.QF_ERR_NULL),
    (dict(cu_tokens=None), qf.QF_ERR_NULL), (dict(seq_lens=None), qf.QF_ERR_NULL), (dict(out=None), qf.QF_ERR_NULL),
    (dict(lse=None), qf.QF_ERR_NULL), (dict(ws=None), qf.QF_ERR_WORKSPACE), (dict(ws=FAKE + 128), qf.QF_ERR_WORKSPACE),
    (dict(ws_bytes=16), qf.QF_ERR_WORKSPACE), (dict(k_cache=FAKE + 64), qf.QF_ERR_BAD_SHAPE), (dict(q=FAKE + 8), qf.QF_ERR_BAD_SHAPE),
])
def test_prompt_attend_refusals(kw, code):
    assert prompt(**kw) == code


# ---- qf_prefix_partial, qf_prefix_step
def prefix(p=None, groups=2, pages=8, ws=FAKE, ws_bytes=1 << 30, **kw):
    a = dict(q=FAKE, k_cache=FAKE, v_cache=FAKE, prefix_table=FAKE, prefix_lens=FAKE, group_offsets=FAKE, o_part=FAKE, m_part=FAKE, lse_part=FAKE)
    a.update(kw)
    return qf.prefix_partial(*a.values(), p if p is not None else good(), groups, pages, ws, ws_bytes, stream=0, check=False)


def step(p=None, groups=2, pages=8, ws=FAKE, ws_bytes=1 << 30, **kw):
    a = dict(q=FAKE, k_cache=FAKE, v_cache=FAKE, block_table=FAKE, seq_lens=FAKE, shard_ranges=FAKE, prefix_table=FAKE, prefix_lens=FAKE,
             group_offsets=FAKE, o_part=FAKE, m_part=FAKE, lse_part=FAKE, out=FAKE, lse=FAKE)
    a.update(kw)
    return qf.prefix_step(*a.values(), p if p is not None else good(), groups, pages, ws, ws_bytes, stream=0, check=False)


@pytest.mark.parametrize("call", [prefix, step])
@pytest.mark.parametrize("kw,code", [
    (dict(groups=0), qf.QF_ERR_BAD_SHAPE), (dict(groups=5), qf.QF_ERR_UNSUPPORTED), (dict(pages=0), qf.QF_ERR_BAD_SHAPE),
    (dict(pages=1 << 28), qf.QF_ERR_UNSUPPORTED), (dict(q=None), qf.QF_ERR_NULL), (dict(prefix_lens=None), qf.QF_ERR_NULL),
    (dict(group_offsets=None), qf.QF_ERR_NULL), (dict(o_part=None), qf.QF_ERR_NULL), (dict(lse_part=None), qf.QF_ERR_NULL),
    (dict(ws=None), qf.QF_ERR_WORKSPACE), (dict(ws=FAKE + 64), qf.QF_ERR_WORKSPACE), (dict(ws_bytes=16), qf.QF_ERR_WORKSPACE),
    (dict(v_cache=FAKE + 64), qf.QF_ERR_BAD_SHAPE), (dict(o_part=FAKE + 8), qf.QF_ERR_BAD_SHAPE),
])
def test_prefix_refusals(call, kw, code):
    assert call(**kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(seq_lens=None), qf.QF_ERR_NULL), (dict(shard_ranges=None), qf.QF_ERR_NULL), (dict(out=None), qf.QF_ERR_NULL),
    (dict(lse=None), qf.QF_ERR_NULL), (dict(out=FAKE + 8), qf.QF_ERR_BAD_SHAPE),
])
def test_prefix_step_refusals(kw, code):
    assert step(**kw) == code
    assert step(p=good(out_shards=8)) == qf.QF_ERR_BAD_SHAPE


def test_host_tensors_are_refused():
    import torch
    x = torch.zeros(4)
    with pytest.raises(ValueError):
        qf.rope_append(x, FAKE, FAKE, FAKE, None, FAKE, FAKE, None, FAKE, FAKE, None, None, None, FAKE, good(), qf.rope_params(4), stream=0)
    with pytest.raises(ValueError):
        qf.prompt_attend(FAKE, FAKE, FAKE, None, FAKE, FAKE, x, FAKE, good(), 4, FAKE, 1 << 30, stream=0)


def test_workspace_sizes():
    p = good()
    n = qf.prompt_workspace_bytes(p, 1000)
    assert n > 0 and n % 256 == 0
    assert qf.prompt_workspace_bytes(p, 0) == 0
    m = qf.prefix_workspace_bytes(p)
    assert m % 256 == 0 and m > qf.workspace_bytes(p)


# ---- the schedule of the row kernels (host arithmetic)
def brute_tiles(causal, n, off, length, rows, j):
    last = min((j + 1) * rows, n)
    lim = min(off + last, length) if causal else length
    return -(-lim // 128)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("seed", range(40))
def test_schedule_covers_every_tile_of_every_block_once(causal, seed):
    rng = np.random.default_rng(seed)
    group, heads = int(rng.integers(1, 9)), int(rng.choice([1, 2, 4, 8]))
    n_seq = int(rng.integers(1, 40))
    n = rng.integers(0, int(rng.choice([2, 70, 900])), n_seq)
    lens = rng.integers(0, int(rng.choice([1, 130, 5000, 60000])), n_seq)
    if seed % 4 == 0:
        n, lens, n_seq = np.array([int(rng.integers(1, 20000))]), np.array([int(rng.integers(0, 100000))]), 1
    max_tokens = int(rng.choice([1 << 30, 2000])) if seed % 3 == 0 else 1 << 30
    off = np.concatenate([[0], np.cumsum(n)])
    n_ctas = int(rng.choice([148, 132, 7, 1, 160]))
    rec = qf.rows_schedule(causal, off, lens, group, heads, max_tokens, n_ctas)
    tile_rows = 128 // group
    seen, slots, per_cta = {}, set(), {}
    for c, s, h, row0, rows, lo, hi, slot, narrow, before, length, first_no in rec.tolist():
        assert 0 <= c < n_ctas and lo < hi and 1 <= rows <= 2 * tile_rows and narrow == (rows <= tile_rows)
        j = (row0 - off[s]) // (2 * tile_rows)
        want_len = min(lens[s], max_tokens) + (n[s] if causal else 0)
        assert length == min(want_len, max_tokens) and rows == min(n[s] - j * 2 * tile_rows, 2 * tile_rows)
        nt = brute_tiles(causal, n[s], min(lens[s], max_tokens), length, 2 * tile_rows, j)
        assert hi <= nt and (slot == -1) == (lo == 0 and hi == nt)
        if slot >= 0:
            assert slot // 2 == c and slot % 2 == (0 if lo > 0 else 1) and slot not in slots
            slots.add(slot)
        got = seen.setdefault((s, h, j), [0, nt])
        assert got[0] == lo            # stretches of a block come in order, without gap or overlap
        got[0] = hi
        per_cta.setdefault(c, []).append((hi - lo) * (1 if narrow else 2) + 2)
    for (s, h, j), (end, nt) in seen.items():
        assert end == nt
    cap = lambda s: min(min(lens[s], max_tokens) + (n[s] if causal else 0), max_tokens)
    want = sum(heads * -(-int(n[s]) // (2 * tile_rows)) for s in range(n_seq) if n[s] > 0 and cap(s) > 0)
    assert len(seen) == want
    assert [r[0] for r in rec.tolist()] == sorted(r[0] for r in rec.tolist())


def test_schedule_balances_long_work():
    for causal, n, lens, group in ((True, [16384], [0], 4), (True, [512], [30011], 4), (False, [256], [32768], 4), (True, [1], [100000], 1)):
        rec = qf.rows_schedule(causal, [0, n[0]], lens, group, 8, 1 << 30, 148)
        load = np.zeros(148)
        for r in rec:
            load[r[0]] += (r[6] - r[5]) * (1 if r[8] else 2) + 2
        assert load.max() <= 1.15 * load.mean() + 12, (load.max(), load.mean())
