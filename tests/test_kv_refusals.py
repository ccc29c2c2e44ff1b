"""What the paged KV$ binding passes on to the library and what it refuses, without a
GPU: tensors that are not on the handle's device, whose addresses the kernels must
not get, and windows of any size."""

import pytest
import torch

import paper_2607_08565_gb300 as pkg

BF = torch.bfloat16


class Library:
    """Notes the calls that come through."""

    def __init__(self):
        self.calls, self.args = [], None

    def __getattr__(self, name):
        def call(*args):
            self.calls.append(name)
            self.args = args
            return 0
        return call


class Elsewhere(torch.Tensor):
    """A tensor that says it is on a GPU of the given number."""

    at = 0

    def get_device(self):
        return self.at


def on(x, device):
    y = x.as_subclass(Elsewhere)
    y.at = device
    return y


@pytest.fixture
def kv(monkeypatch):
    lib = Library()
    monkeypatch.setattr(pkg, "lib", lambda: lib)
    monkeypatch.setattr(pkg, "smetric_kv_create", lambda cfg: 1)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 0, raising=False)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    kv = pkg.SMetricKV(head_dim=64, num_q_heads=4, num_kv_heads=2, page_size=16, num_pages=3, max_batch_requests=2, max_batch_tokens=8)
    kv.library = lib
    kv.plan(*(on(x, 0) for x in plan()), 4)
    lib.calls.clear()
    yield kv
    kv.handle = None


def plan():
    return torch.tensor([0, 4]), torch.tensor([20], dtype=torch.int32), torch.zeros(1, 2, dtype=torch.int32)


CACHE = (3, 16, 2, 64)
ARGS = {
    "append": dict(k_cache=CACHE, v_cache=CACHE, k=(4, 2, 64), v=(4, 2, 64), q=(4, 4, 64), q_out=(4, 4, 64), cos_sin=(30, 64), q_norm=(64,),
                   k_norm=(64,)),
    "qk_norm_rope": dict(q=(4, 4, 64), k=(4, 2, 64), positions=(4,), cos_sin=(30, 64), q_norm=(64,), k_norm=(64,), q_out=(4, 4, 64),
                         k_out=(4, 2, 64)),
    "paged_attention": dict(q=(4, 4, 64), k_cache=CACHE, v_cache=CACHE, out=(4, 4, 64)),
}
TYPES = {"cos_sin": torch.float32, "positions": torch.int32}


@pytest.mark.parametrize("device", [-1, 1])  # the host, another GPU
@pytest.mark.parametrize("call,name", [(c, n) for c, names in ARGS.items() for n in names])
def test_tensors_elsewhere_are_refused(kv, call, name, device):
    args = {n: on(torch.zeros(s, dtype=TYPES.get(n, BF)), 0) for n, s in ARGS[call].items()}
    getattr(kv, call)(**args)
    assert kv.library.calls == ["smetric_" + ("kv_append" if call == "append" else call)]
    args[name].at = device
    with pytest.raises(ValueError, match="device|cuda"):
        getattr(kv, call)(**args)
    assert len(kv.library.calls) == 1


@pytest.mark.parametrize("device", [-1, 1])
@pytest.mark.parametrize("which", [0, 1, 2])
def test_a_plans_tensors_elsewhere_are_refused(kv, which, device):
    args = [on(x, 0) for x in plan()]
    args[which].at = device
    with pytest.raises(ValueError, match="device|cuda"):
        kv.plan(*args, 4)
    assert not kv.library.calls


@pytest.mark.parametrize("window,passed", [(0, 0), (5, 5), (2 ** 31 - 1, 2 ** 31 - 1), (2 ** 31, 2 ** 31 - 1), (2 ** 32 + 5, 2 ** 31 - 1),
                                           (2 ** 63 - 1, 2 ** 31 - 1), (-1, -1), (-2 ** 32, -2 ** 31)])
def test_windows_past_32_bits_are_as_wide_as_any_sequence(kv, window, passed):
    """And negative ones stay negative, which the library refuses."""
    kv.plan(*(on(x, 0) for x in plan()), 4, window=window)
    assert kv.library.args[8] == passed
