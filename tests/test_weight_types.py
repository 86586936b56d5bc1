"""Weights of a type that no kernel reads are refused, in the calls that take a tensor of them; on the host, before anything
would be launched."""
import pytest
import torch

import paper_2609_15039_amd as sp

OTHER = [torch.float16, torch.float64, torch.int16, torch.int8, torch.uint8]
if hasattr(torch, "float8_e4m3fn"):
    OTHER.append(torch.float8_e4m3fn)
PF, PB = sp.SPLITEE_PREC_F32, sp.SPLITEE_PREC_BF16


def weights(shape, dtype):
    return torch.zeros(shape, dtype=torch.uint8).to(dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_types_that_are_read(dtype):
    assert sp._wtype(weights((16, 32), dtype)) == (sp.SPLITEE_F32 if dtype == torch.float32 else sp.SPLITEE_BF16)


@pytest.mark.parametrize("dtype", OTHER)
@pytest.mark.parametrize("prec", [PF, PB])
def test_products_refuse(dtype, prec):
    A = torch.zeros(4, 32, dtype=torch.float32 if prec == PF else torch.bfloat16)
    W, E = weights((16, 32), dtype), weights((2, 16, 32), dtype)
    with pytest.raises(ValueError, match="W: expected float32 or bfloat16"):
        sp.linear_epilogue(A, prec, W)
    with pytest.raises(ValueError, match="W: expected float32 or bfloat16"):
        sp.grouped_linear(A, prec, E, torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError, match="W: expected float32 or bfloat16"):
        sp.masked_linear(A[None], prec, W)


@pytest.mark.parametrize("dtype", OTHER)
@pytest.mark.parametrize("which", ["W_gate_up", "W_down"])
def test_expert_ffn_refuses(dtype, which):
    """Before the router and the first noise are launched."""
    W = dict(W_gate_up=torch.zeros(4, 48, 32), W_down=torch.zeros(4, 16, 24))
    W[which] = weights(W[which].shape, dtype)
    with pytest.raises(ValueError, match="%s: expected float32 or bfloat16" % which):
        sp.expert_ffn(torch.zeros(6, 32), torch.zeros(6, 4), 2, W["W_gate_up"], W["W_down"], prec=PF)


@pytest.mark.parametrize("dtype", OTHER + [torch.float32])
def test_tiled_weights_are_bfloat16(dtype):
    """The tiled order is read from the data's address: its size in bytes counts, and by expert its strides."""
    A = torch.zeros(4, 64, dtype=torch.bfloat16)
    if dtype.is_floating_point or dtype.itemsize < 2:  # or as many elements as the tiled order has, in half the bytes
        with pytest.raises(ValueError, match="tiled weights are bfloat16|tiled order"):
            sp.linear_epilogue(A, PB, sp.TiledWeights(weights((2048,), dtype), 16, 64))
    if dtype != torch.int16:  # (whose bits may be bfloat16's)
        with pytest.raises(ValueError, match="bfloat16"):
            sp.grouped_linear(A, PB, sp.TiledWeights(weights((2, 4096), dtype), 16, 64), torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError, match="W: expected bfloat16"):
        sp.tile_weights(weights((16, 64), dtype))


def test_tiled_weights_in_one_piece():
    with pytest.raises(ValueError, match="tiled order"):
        sp.linear_epilogue(torch.zeros(4, 64, dtype=torch.bfloat16), PB,
                           sp.TiledWeights(torch.zeros(4096, dtype=torch.bfloat16)[::2], 16, 64))
