"""What the serving calls of the binding refuse before they reach the library: no call here touches a GPU."""
import pytest
import torch

import __graft_entry__ as entry

I8, I32, F32, BF16 = torch.int8, torch.int32, torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def tlq():
    entry.build()
    from paper_2602_07899_b200 import tlq as mod
    return mod


@pytest.fixture
def host(tlq):
    """Arguments that are right in everything but that they lie in host memory."""
    cache = tlq.KvCache.empty(3, 2, 64, "cpu")
    batch = tlq.KvBatch(torch.tensor([0, 1, 2], dtype=I32), torch.tensor([1, 1], dtype=I32), torch.zeros(2, 2, dtype=I32), 1)
    return dict(linear=dict(Xq=torch.zeros(2, 32, dtype=I8), t=torch.zeros(2), Wq=torch.zeros(8, 32, dtype=I8), u=torch.zeros(8)),
                store=dict(qkv=torch.zeros(2, 8 * 64, dtype=BF16), n_heads=4, cache=cache, batch=batch),
                attention=dict(q=torch.zeros(2, 4, 64, dtype=BF16), cache=cache, batch=batch, scale=0.125))


def calls(tlq):
    return dict(linear=tlq.tlq_linear_i8, store=tlq.tlq_kv_store, attention=tlq.tlq_kv_attention)


@pytest.mark.parametrize("name", ["linear", "store", "attention"])
def test_tensors_in_host_memory_are_refused(tlq, host, name):
    """A kernel that is given a host pointer faults the GPU."""
    with pytest.raises(ValueError, match="device"):
        calls(tlq)[name](**host[name])
    with pytest.raises(ValueError, match="device"):
        calls(tlq)[name](**host[name], workspace=torch.zeros(1 << 16, dtype=torch.uint8))


class At:
    """Stands for a tensor on device number `at` (-1: host memory)."""

    def __init__(self, at):
        self.at = at

    def get_device(self):
        return self.at


def test_all_tensors_of_a_call_have_to_lie_on_the_current_device(tlq, monkeypatch):
    monkeypatch.setattr(tlq, "_raw_device", lambda: 1)
    tlq._on_device("call", At(1), At(1), None, At(1))
    for wrong in ((At(-1),), (At(1), At(-1)), (At(1), None, At(0)), (At(0), At(0)), (At(0), At(1))):
        with pytest.raises(ValueError, match="device"):
            tlq._on_device("call", *wrong)


def test_caches_and_batches_know_where_they_lie(tlq, monkeypatch, host):
    cache, batch = host["attention"]["cache"], host["attention"]["batch"]
    assert cache.get_device() == -1 and batch.get_device() == -1
    # one tensor of them elsewhere
    seen = iter([0, 0, -1, 0])
    monkeypatch.setattr(torch.Tensor, "get_device", lambda self: next(seen))
    with pytest.raises(ValueError, match="device"):
        tlq.KvCache(cache.k_codes, cache.v_codes, cache.k_steps, cache.v_steps)
    seen = iter([0, 0, 1])
    with pytest.raises(ValueError, match="device"):
        tlq.KvBatch(batch.cu_q, batch.kv_len, batch.block_table, 1)


@pytest.mark.parametrize("name", ["linear", "store", "attention"])
def test_workspaces_that_are_not_plain_memory_are_refused(tlq, host, name):
    """The library is told the number of elements as the number of bytes: a view that repeats or skips memory has fewer."""
    for bad in (torch.zeros(1, dtype=torch.uint8).expand(1 << 20), torch.zeros(1 << 20, dtype=torch.uint8)[::2],
                torch.zeros(1, 1 << 10, dtype=torch.uint8).expand(1 << 10, -1)):
        with pytest.raises(ValueError, match="workspace"):
            calls(tlq)[name](**host[name], workspace=bad)
