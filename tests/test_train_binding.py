"""What the Python entry points of the training and adapter operators say of an argument that is missing.  No GPU is involved: the stand-ins below have
a GPU tensor's answers, and each call has to be refused before it looks at an address."""
import pytest
import torch

import paper_2605_23911_amd as moe


class Tensor:
    """A tensor on cuda:0 as far as the binding asks."""

    def __init__(self, *shape, dtype=torch.bfloat16):
        self.shape, self.dtype = torch.Size(shape), dtype

    def get_device(self):
        return 0

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 4096

    def dim(self):
        return len(self.shape)


T, D, F, E = 4, 64, 128, 2
I32, F32 = torch.int32, torch.float32


def _train(missing):
    a = dict(x_perm=Tensor(T, D), offsets=Tensor(E + 1, dtype=I32), W_gate=Tensor(E, F, D), W_up=Tensor(E, F, D), W_down=Tensor(E, D, F), g=Tensor(T, F), u=Tensor(T, F),
             h=Tensor(T, F), y_perm=Tensor(T, D), workspace=Tensor(1 << 20, dtype=torch.uint8))
    moe.moe_grouped_ffn_train(moe.MoEConfig.of(T, D, F, E, 1), **{**a, missing: None})


def _backward(missing):
    a = dict(x_perm=Tensor(T, D), offsets=Tensor(E + 1, dtype=I32), W_gate=Tensor(E, F, D), W_up=Tensor(E, F, D), W_down=Tensor(E, D, F), g=Tensor(T, F), u=Tensor(T, F),
             dy_perm=Tensor(T, D), dx_perm=Tensor(T, D), dW_gate=Tensor(E, F, D), dW_up=Tensor(E, F, D), dW_down=Tensor(E, D, F), workspace=Tensor(1 << 20, dtype=torch.uint8))
    moe.moe_grouped_ffn_backward(moe.MoEConfig.of(T, D, F, E, 1), **{**a, missing: None})


def _combine(missing):
    a = dict(dy=Tensor(T, D), y_perm=Tensor(T, D), row_of=Tensor(T, 1, dtype=I32), topk_w=Tensor(T, 1, dtype=F32), dy_perm=Tensor(T, D), d_topk_w=Tensor(T, 1, dtype=F32))
    moe.moe_combine_backward(moe.MoEConfig.of(T, D, F, E, 1), **{**a, missing: None})


def _linear(missing):
    a = dict(x=Tensor(T, D), W=Tensor(F, D), A=Tensor(E, 8, D), B=Tensor(E, F, 8), scale=None, adapter_of=Tensor(T, dtype=I32), y=Tensor(T, F),
             workspace=Tensor(1 << 20, dtype=torch.uint8))
    moe.moe_adapter_linear(moe.AdapterConfig.of(T, F, D, E, 8), **{**a, missing: None})


def _gated(missing):
    a = dict(x=Tensor(T, D), W_gate=Tensor(F, D), W_up=Tensor(F, D), A_gate=Tensor(E, 8, D), A_up=Tensor(E, 8, D), B_gate=Tensor(E, F, 8), B_up=Tensor(E, F, 8), scale=None,
             adapter_of=Tensor(T, dtype=I32), h=Tensor(T, F), workspace=Tensor(1 << 20, dtype=torch.uint8))
    moe.moe_adapter_gated_up(moe.AdapterConfig.of(T, F, D, E, 8), **{**a, missing: None})


@pytest.mark.parametrize("call,names", [
    (_train, "x_perm offsets W_gate W_up W_down g u h y_perm workspace"), (_backward, "x_perm offsets W_gate W_up W_down g u dy_perm workspace"),
    (_combine, "dy y_perm row_of topk_w dy_perm d_topk_w"), (_linear, "x A B adapter_of y workspace"),
    (_gated, "x W_gate W_up A_gate A_up B_gate B_up adapter_of h workspace")], ids=lambda v: v.__name__ if callable(v) else "")
def test_a_missing_argument_is_named(call, names):
    for name in names.split():
        with pytest.raises(ValueError, match=rf"^{name} is required"):
            call(name)
