"""Tensors that require a gradient: the operators have none to give, and say so before they look at anything else."""
import pytest
import torch

import paper_2512_21835_amd as P


def _adapter():
    t = {"x": torch.zeros(2, 8), "base": torch.zeros(2, 8), "out": torch.zeros(2, 8), "a": torch.zeros(1, 4, 8).bfloat16(),
         "b": torch.zeros(1, 8, 4).bfloat16(), "ids": torch.zeros(2, dtype=torch.int32), "scales": torch.ones(1)}
    return P.stage_adapter_add, t


def _window():
    q = torch.zeros(2, 4, 64)
    return P.stage_window_attention, {"q": q, "out": q.clone(), "pool": torch.zeros(1, 2, 2, 16, 64), "batch": None}


def _append():
    return P.stage_norm_rope_append, {"qkv": torch.zeros(2, 8, 64), "q_out": torch.zeros(2, 4, 64), "pool": torch.zeros(1, 2, 2, 16, 64),
                                      "batch": None, "cos": torch.zeros(8, 32), "sin": torch.zeros(8, 32),
                                      "q_gain": torch.ones(64).bfloat16(), "k_gain": torch.ones(64).bfloat16()}


@pytest.mark.parametrize("make,name", [(_adapter, n) for n in ("x", "base", "out", "a", "b", "scales")] +
                         [(_window, n) for n in ("q", "out", "pool")] +
                         [(_append, n) for n in ("qkv", "q_out", "pool", "cos", "sin", "q_gain", "k_gain")])
def test_a_tensor_that_requires_a_gradient_is_refused(make, name):
    call, tensors = make()
    tensors[name].requires_grad_()
    with pytest.raises(ValueError, match="no backward pass"):
        call(**tensors)
    with torch.no_grad(), pytest.raises(ValueError, match="on a GPU"):      # (there it goes on to the next check)
        call(**tensors)


def test_workspace_sizes_too():
    call, tensors = _adapter()
    tensors["a"].requires_grad_()
    with pytest.raises(ValueError, match="no backward pass"):
        P.stage_adapter_workspace(*(tensors[n] for n in ("x", "base", "out", "a", "b", "ids")))
