"""What the binding refuses before a prompt-side call reaches the library: every argument, without a GPU."""
import numpy as np
import pytest
import torch

from paper_2608_15473_b200 import binding as qf
from paper_2608_15473_b200 import build as qf_build
from test_prompt_cpu import FAKE, good

CALLS = {
    "rope_append": ("q k v q_out k_out k_cache v_cache block_table cu_tokens seq_lens pos_base q_gain k_gain inv_freq",
                    lambda a: (*a.values(), good(), qf.rope_params(4))),
    "prompt_attend": ("q k_cache v_cache block_table cu_tokens seq_lens out lse", lambda a: (*a.values(), good(), 4, FAKE, 1 << 30)),
    "prefix_partial": ("q k_cache v_cache prefix_table prefix_lens group_offsets o_part m_part lse_part",
                       lambda a: (*a.values(), good(), 2, 8, FAKE, 1 << 30)),
    "prefix_step": ("q k_cache v_cache block_table seq_lens shard_ranges prefix_table prefix_lens group_offsets o_part m_part lse_part out lse",
                    lambda a: (*a.values(), good(), 2, 8, FAKE, 1 << 30)),
}
ARGS = [(call, name) for call, (names, _) in CALLS.items() for name in names.split()]


@pytest.fixture(scope="module", autouse=True)
def built():
    qf_build.build()


def go(call, **kw):
    """The call with an address for everything but `kw`, and a batch that the library refuses: nothing is ever launched."""
    names, args = CALLS[call]
    a = dict.fromkeys(names.split(), FAKE)
    assert set(kw) <= set(a)
    a.update(kw)
    args = list(args(a))
    p = next(x for x in args if isinstance(x, qf.QFParams))
    p.head_dim = 64
    return getattr(qf, call)(*args, stream=0, check=False)


@pytest.mark.parametrize("call", CALLS)
def test_addresses_reach_the_library(call):
    assert go(call) == qf.QF_ERR_UNSUPPORTED


@pytest.mark.parametrize("call,name", ARGS)
def test_host_memory_is_refused_whatever_the_argument(call, name):
    for x in (torch.zeros(64, dtype=torch.int32), torch.zeros(64), np.zeros(64, np.float32), np.zeros(64, np.int32), [0] * 64):
        with pytest.raises(ValueError):
            go(call, **{name: x})


def test_the_array_of_rope_frequencies_is_refused():
    inv, _ = qf.rope_frequencies(128, 1e6)
    with pytest.raises(ValueError, match="numpy"):
        go("rope_append", inv_freq=inv)


@pytest.mark.parametrize("call", ["prompt_attend", "prefix_partial", "prefix_step"])
def test_a_workspace_in_host_memory_is_refused(call):
    names, args = CALLS[call]
    args = list(args(dict.fromkeys(names.split(), FAKE)))
    args[args.index(FAKE, len(names.split()))] = torch.zeros(1024, dtype=torch.uint8)
    with pytest.raises(ValueError):
        getattr(qf, call)(*args, stream=0, check=False)


class OnDevice:
    """Stands in for a CUDA tensor of a machine with several GPUs."""

    def __init__(self, index, dtype=torch.bfloat16):
        self.index, self.dtype, self.device, self.is_cuda = index, dtype, f"cuda:{index}", True

    def get_device(self):
        return self.index

    def data_ptr(self):
        return FAKE


@pytest.mark.parametrize("call,name", ARGS)
def test_a_tensor_of_another_gpu_is_refused_whatever_the_argument(call, name, monkeypatch):
    assert go(call) == qf.QF_ERR_UNSUPPORTED           # the number of GPUs has been looked up
    monkeypatch.setattr(qf, "_many_gpus", True)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError, match="current device"):
        go(call, **{name: OnDevice(1, types(call, name)[0][0])})


def types(call, name):
    """Element types that an argument may have, and some that it may not."""
    if name in INTS:
        return [torch.int32], [torch.int64, torch.int16, torch.float32]
    if name in FLOATS or (call == "prefix_step" and name == "out"):
        return [torch.float32], [torch.float64, torch.bfloat16, torch.int32]
    return [torch.bfloat16, torch.int16, torch.uint16], [torch.float16, torch.float32, torch.float8_e4m3fn, torch.int32]


INTS = {"block_table", "cu_tokens", "seq_lens", "pos_base", "shard_ranges", "prefix_table", "prefix_lens", "group_offsets"}
FLOATS = {"inv_freq", "lse", "o_part", "m_part", "lse_part"}


@pytest.mark.parametrize("call,name", ARGS)
def test_other_element_types_are_refused_whatever_the_argument(call, name):
    """Offsets from torch.cumsum are 64 bits wide, gains of a model may be fp32, fp16 is not bf16: all would be misread."""
    fine, wrong = types(call, name)
    for t in wrong:
        with pytest.raises(ValueError, match="expected elements"):
            go(call, **{name: OnDevice(0, t)})
    for t in fine:
        assert go(call, **{name: OnDevice(0, t)}) == qf.QF_ERR_UNSUPPORTED
