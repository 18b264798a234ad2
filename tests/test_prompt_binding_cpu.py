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
        self.index, self.dtype, self.device = index, dtype, f"cuda:{index}"

    def get_device(self):
        return self.index

    def data_ptr(self):
        return FAKE


@pytest.mark.parametrize("call,name", ARGS)
def test_a_tensor_of_another_gpu_is_refused_whatever_the_argument(call, name, monkeypatch):
    monkeypatch.setattr(qf, "_many_gpus", True)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError, match="current device"):
        go(call, **{name: OnDevice(1)})
