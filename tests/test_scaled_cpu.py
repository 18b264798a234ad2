"""The scaled cache's boundary and the axes of rotary positions without a GPU: refusals, and which axis turns which pair."""
import numpy as np
import pytest
import torch

from paper_2608_15473_b200 import binding as qf
from paper_2608_15473_b200 import build as qf_build
from test_prompt_cpu import FAKE, good

T8, I8 = qf.QF_KV_E4M3, qf.QF_KV_INT8


@pytest.fixture(scope="module", autouse=True)
def built():
    qf_build.build()


def rope(p=None, r=None, kv_type=T8, num_axes=None, **kw):
    a = dict(q=FAKE, k=FAKE, v=FAKE, q_out=FAKE, k_out=None, k_cache=FAKE, v_cache=FAKE, k_scale=FAKE, v_scale=FAKE, block_table=FAKE,
             cu_tokens=FAKE, seq_lens=FAKE, pos_base=None, positions=None, pair_axis=None, q_gain=None, k_gain=None, inv_freq=FAKE)
    assert set(kw) <= set(a)
    a.update(kw)
    return qf.rope_append_scaled(*a.values(), p if p is not None else good(), r if r is not None else qf.rope_params(10), kv_type=kv_type,
                                 num_axes=num_axes, stream=0, check=False)


def axes(p=None, r=None, num_axes=3, **kw):
    a = dict(q=FAKE, k=FAKE, v=FAKE, q_out=FAKE, k_out=None, k_cache=FAKE, v_cache=FAKE, block_table=FAKE, cu_tokens=FAKE,
             seq_lens=FAKE, positions=FAKE, pair_axis=FAKE, q_gain=None, k_gain=None, inv_freq=FAKE)
    assert set(kw) <= set(a)
    a.update(kw)
    return qf.rope_append_axes(*a.values(), p if p is not None else good(), r if r is not None else qf.rope_params(10), num_axes=num_axes,
                               stream=0, check=False)


def sweep(call, p=None, kv_type=T8, ws=FAKE, ws_bytes=1 << 30, **kw):
    a = dict(q=FAKE, k_cache=FAKE, v_cache=FAKE, k_scale=FAKE, v_scale=FAKE, block_table=FAKE, seq_lens=FAKE, shard_ranges=FAKE)
    if call == "step":
        a.update(shard_counts=FAKE)
    a.update(o_part=FAKE, m_part=FAKE, lse_part=FAKE)
    if call == "step":
        a.update(out=FAKE, lse=FAKE)
    assert set(kw) <= set(a)
    a.update(kw)
    f = qf.decode_step_scaled if call == "step" else qf.decode_partial_scaled
    return f(*a.values(), p if p is not None else good(), ws, ws_bytes, kv_type=kv_type, stream=0, check=False)


def prompt(p=None, tokens=10, stride=0, kv_type=T8, ws=FAKE, ws_bytes=1 << 30, **kw):
    a = dict(q=FAKE, k_cache=FAKE, v_cache=FAKE, k_scale=FAKE, v_scale=FAKE, block_table=FAKE, cu_tokens=FAKE, seq_lens=FAKE, out=FAKE, lse=FAKE)
    assert set(kw) <= set(a)
    a.update(kw)
    return qf.prompt_attend_scaled(*a.values(), p if p is not None else good(), tokens, ws, ws_bytes, stride, kv_type=kv_type, stream=0, check=False)


CALLS = {"rope": rope, "partial": lambda **kw: sweep("partial", **kw), "step": lambda **kw: sweep("step", **kw), "prompt": prompt}


@pytest.mark.parametrize("call", CALLS)
def test_parameters_and_types_are_checked_first(call):
    f = CALLS[call]
    assert f(p=good(head_dim=64)) == qf.QF_ERR_UNSUPPORTED and f(p=good(num_q_heads=72)) == qf.QF_ERR_UNSUPPORTED
    assert f(p=good(page_size=32)) == qf.QF_ERR_UNSUPPORTED and f(p=good(num_q_heads=12)) == qf.QF_ERR_BAD_SHAPE
    for kv_type in (0, 3, -1, 77):
        assert f(kv_type=kv_type) == qf.QF_ERR_UNSUPPORTED
        assert f(p=good(batch=0), kv_type=kv_type) == qf.QF_ERR_BAD_SHAPE
    for kv_type in (T8, I8):
        assert f(kv_type=kv_type, k_scale=None) == qf.QF_ERR_NULL and f(kv_type=kv_type, v_scale=None) == qf.QF_ERR_NULL
        assert f(kv_type=kv_type, k_scale=FAKE + 2) == qf.QF_ERR_BAD_SHAPE and f(kv_type=kv_type, v_scale=FAKE + 1) == qf.QF_ERR_BAD_SHAPE


@pytest.mark.parametrize("call", ["partial", "step", "prompt"])
def test_pointers_and_workspaces(call):
    f = CALLS[call]
    for name in ("q", "k_cache", "v_cache", "seq_lens"):
        assert f(**{name: None}) == qf.QF_ERR_NULL, name
    assert f(k_cache=FAKE + 64) == qf.QF_ERR_BAD_SHAPE and f(v_cache=FAKE + 16) == qf.QF_ERR_BAD_SHAPE and f(q=FAKE + 8) == qf.QF_ERR_BAD_SHAPE
    assert f(ws=None) == qf.QF_ERR_WORKSPACE and f(ws=FAKE + 128) == qf.QF_ERR_WORKSPACE and f(ws_bytes=16) == qf.QF_ERR_WORKSPACE


@pytest.mark.parametrize("call,names", [("partial", "shard_ranges o_part m_part lse_part"), ("step", "shard_ranges o_part m_part lse_part out lse"),
                                        ("prompt", "cu_tokens out lse")])
def test_arrays_that_must_be_there(call, names):
    for name in names.split():
        assert CALLS[call](**{name: None}) == qf.QF_ERR_NULL, name


def test_a_step_owns_its_shard_table_and_a_partial_fits_its_own():
    assert sweep("step", p=good(out_shards=4)) == qf.QF_ERR_BAD_SHAPE
    assert sweep("partial", p=good(out_shards=1)) == qf.QF_ERR_BAD_SHAPE


def test_prompt_sizes():
    assert prompt(tokens=0) == qf.QF_ERR_BAD_SHAPE and prompt(stride=100) == qf.QF_ERR_BAD_SHAPE
    assert prompt(tokens=(1 << 30) + 1) == qf.QF_ERR_UNSUPPORTED and prompt(out=FAKE + 16) == qf.QF_ERR_BAD_SHAPE


@pytest.mark.parametrize("f", [rope, axes])
@pytest.mark.parametrize("kw,code", [
    (dict(total_tokens=0), qf.QF_ERR_BAD_SHAPE), (dict(total_tokens=4, rotary_dim=20), qf.QF_ERR_UNSUPPORTED),
    (dict(total_tokens=4, eps=-1.0), qf.QF_ERR_BAD_SHAPE), (dict(total_tokens=4, rot_scale=float("inf")), qf.QF_ERR_BAD_SHAPE),
    (dict(total_tokens=4, q_stride=2047), qf.QF_ERR_BAD_SHAPE), (dict(total_tokens=4, v_stride=-1024), qf.QF_ERR_BAD_SHAPE),
    (dict(total_tokens=(1 << 30) + 1), qf.QF_ERR_UNSUPPORTED),
])
def test_placing_refuses_bad_sizes(f, kw, code):
    assert f(r=qf.rope_params(**kw)) == code


@pytest.mark.parametrize("f", [rope, axes])
@pytest.mark.parametrize("kw,code", [
    (dict(cu_tokens=None), qf.QF_ERR_NULL), (dict(seq_lens=None), qf.QF_ERR_NULL), (dict(q_out=None), qf.QF_ERR_NULL),
    (dict(k_cache=None), qf.QF_ERR_NULL), (dict(v_cache=None), qf.QF_ERR_NULL), (dict(v=None), qf.QF_ERR_NULL), (dict(k=None), qf.QF_ERR_NULL),
    (dict(k_cache=None, v_cache=None), qf.QF_ERR_NULL), (dict(inv_freq=None), qf.QF_ERR_NULL), (dict(q=FAKE + 8), qf.QF_ERR_BAD_SHAPE),
    (dict(k_cache=FAKE + 8), qf.QF_ERR_BAD_SHAPE), (dict(q_gain=FAKE + 2), qf.QF_ERR_BAD_SHAPE),
])
def test_placing_refuses_bad_pointers(f, kw, code):
    assert f(**kw) == code


def test_axes_and_their_number():
    assert axes(positions=None) == qf.QF_ERR_NULL and axes(pair_axis=None) == qf.QF_ERR_NULL
    assert axes(num_axes=0) == qf.QF_ERR_BAD_SHAPE and axes(num_axes=-1) == qf.QF_ERR_BAD_SHAPE and axes(num_axes=9) == qf.QF_ERR_UNSUPPORTED
    assert rope(positions=FAKE, num_axes=3) == qf.QF_ERR_NULL
    assert rope(positions=FAKE, pair_axis=FAKE, num_axes=0) == qf.QF_ERR_BAD_SHAPE
    assert rope(positions=FAKE, pair_axis=FAKE, num_axes=9) == qf.QF_ERR_UNSUPPORTED
    assert axes(positions=None, p=good(head_dim=64)) == qf.QF_ERR_UNSUPPORTED
    with pytest.raises(ValueError, match="num_axes"):
        axes(num_axes=None)
    with pytest.raises(ValueError, match="num_axes"):
        rope(positions=FAKE, pair_axis=FAKE)


def test_the_type_must_be_told_or_tell_itself():
    with pytest.raises(ValueError, match="kv_type"):
        rope(kv_type=None)
    with pytest.raises(ValueError, match="kv_type"):
        sweep("step", kv_type=None)
    # no cache, no codes: only what else is wrong
    assert rope(kv_type=None, k_cache=None, v_cache=None, k_out=FAKE, cu_tokens=None) == qf.QF_ERR_NULL

    class Pool:      # what the binding looks at
        def __init__(self, dtype):
            self.dtype = dtype
    assert qf._kv_type(None, Pool(torch.float8_e4m3fn), FAKE) == T8 and qf._kv_type(None, FAKE, Pool(torch.int8)) == I8
    assert qf._kv_type(I8, Pool(torch.uint8), Pool(torch.uint8)) == I8
    for said, dtype in ((T8, torch.int8), (I8, torch.float8_e4m3fn)):
        with pytest.raises(ValueError, match="does not hold"):
            qf._kv_type(said, Pool(dtype), FAKE)
    with pytest.raises(ValueError, match="does not hold"):
        qf._kv_type(None, Pool(torch.int8), Pool(torch.float8_e4m3fn))


@pytest.mark.parametrize("call", [*CALLS, "axes"])
@pytest.mark.parametrize("x", [torch.zeros(64), np.zeros(64, np.float32), [0] * 64], ids=["host tensor", "array", "list"])
def test_host_memory_is_refused(call, x):
    f = {**CALLS, "axes": axes}[call]
    names = ["q", "k_cache", "v_cache", "block_table", "seq_lens"] + ([] if call == "axes" else ["k_scale", "v_scale"])
    names += ["positions", "pair_axis", "k_gain", "inv_freq", "k_out"] if call in ("rope", "axes") else []
    for name in names:
        with pytest.raises(ValueError):
            f(**{name: x})


# ---- which axis turns which pair
def test_axes_in_stretches():
    a = qf.rope_pair_axes(128, [16, 24, 24])
    assert a.dtype == np.int32 and a.tolist() == [0] * 16 + [1] * 24 + [2] * 24
    assert qf.rope_pair_axes(32, [0, 16, 0]).tolist() == [1] * 16 and qf.rope_pair_axes(16, [8]).tolist() == [0] * 8


def test_axes_in_turn():
    a = qf.rope_pair_axes(128, [24, 20, 20], interleaved=True).tolist()
    assert a[:60] == [0, 1, 2] * 20 and a[60:] == [0, 0, 0, 0]
    b = qf.rope_pair_axes(16, [6, 1, 1], interleaved=True).tolist()
    assert b == [0, 1, 2, 0, 0, 0, 0, 0]
    for sections in ([24, 20, 20], [22, 21, 21], [64, 0, 0], [44, 0, 20]):
        c = np.bincount(qf.rope_pair_axes(128, sections, True), minlength=3)
        assert c.tolist() == sections


@pytest.mark.parametrize("args,code", [
    ((0, [0]), qf.QF_ERR_BAD_SHAPE), ((24, [12]), qf.QF_ERR_UNSUPPORTED), ((144, [72]), qf.QF_ERR_UNSUPPORTED), ((128, [16, 24, 23]), qf.QF_ERR_BAD_SHAPE),
    ((128, [70, -6]), qf.QF_ERR_BAD_SHAPE), ((128, [8] * 9), qf.QF_ERR_UNSUPPORTED), ((128, []), qf.QF_ERR_BAD_SHAPE),
    ((128, [20, 22, 22], True), qf.QF_ERR_BAD_SHAPE),      # 22 pairs of axis 2 in turn would need 68
])
def test_bad_axes(args, code):
    with pytest.raises(qf.QFError) as e:
        qf.rope_pair_axes(*args)
    assert e.value.status == code
