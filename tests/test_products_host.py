"""What the binding of the operators around matrix products checks before it reaches the device; no GPU needed."""
import types

import pytest
import torch

from paper_2506_00486_b200 import Context
from paper_2506_00486_b200.binding import ACTIVATIONS


def stub(index):
    return types.SimpleNamespace(device=torch.device("cuda", index))


def tensor_on(index):
    return types.SimpleNamespace(is_cuda=True, device=torch.device("cuda", index))


def test_tensors_of_another_device_are_refused():
    Context._here(stub(1), h=tensor_on(1), residual=None)
    with pytest.raises(ValueError, match="h is on cuda:0, the context on cuda:1"):
        Context._here(stub(1), target=tensor_on(1), h=tensor_on(0))


def test_activations_by_name():
    assert [Context._act(a) for a in ("silu", "gelu", "gelu_tanh", "relu")] == list(ACTIVATIONS.values()) == [0, 1, 2, 3]
    for bad in ("swish", 0, None):
        with pytest.raises(ValueError, match="silu, gelu, gelu_tanh, relu"):
            Context._act(bad)


def test_calls_fail_cleanly_without_a_context():
    import __graft_entry__ as entry
    entry.build()
    from paper_2506_00486_b200 import binding
    lib = binding.lib()
    for name in ("gg_cross_entropy", "gg_cross_entropy_grad", "gg_gated_linear", "gg_gated_linear_grad", "gg_dropout"):
        assert getattr(lib, name)(None, None, None) == 1
