"""Weights held in 4 bits at the edges of what the calls allow, against the definition in 64 bits.  Tolerances: those of
tests/test_gpu_w4.py."""
import pytest
import torch

from tests.test_gpu_w4 import call_ffn, check_ffn, check_linear, ffn_case, ffn_reference, gen, make_w4, tokens

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pb():
    import __graft_entry__ as entry
    entry.build()
    from paper_2607_27591_b200 import binding
    return binding


@pytest.mark.parametrize("K", [12288, 12320, 12416, 12544, 12576])
@pytest.mark.parametrize("B", [6, 7, 8, 16, 19])
def test_linear_rows_between_four_blocks_and_eight(pb, K, B):
    """Groups of 32: for 7 and 8 tokens K = 12320 .. 12544 fits in neither a cluster of four nor one of eight."""
    N, group = 130, 32
    w = make_w4(K + B, N, K, group, B == 8)
    x = tokens(B, B, K, torch.bfloat16)
    y = torch.full((B, N), float("nan"), device="cuda")
    pb.prox_w4_linear(w, N, K, group, x, K, 0, B, y, N, 1)
    check_linear(y, w, group, x, K, 1)


def lists(seed, B, F, k2):
    return torch.rand(B, F, device="cuda", generator=gen(seed)).argsort(1)[:, :k2].sort(1).values.to(torch.int32).contiguous()


@pytest.mark.parametrize("powers", [[-55], [-60], [58], [-58, 0, 55], [-52, -60, 58, 3, -45]])
@pytest.mark.parametrize("zeros", [False, True])
def test_ffn_small_and_large_inputs(pb, powers, zeros):
    """h goes with the square of the inputs: from near the least to near the largest number of fp32.  (Inputs of one size a token; y stays
    a normal number, so the bound is as tight as for inputs near 1.)"""
    D, F, k2, B = 512, 1408, 500, len(powers)
    gate, up, down, x = ffn_case(300 + B, D, F, 128, B, zeros)
    x = (x.float() * torch.exp2(torch.tensor(powers, device="cuda", dtype=torch.float32))[:, None]).bfloat16()
    sel = lists(301, B, F, k2)
    y = call_ffn(pb, (gate, up, down, x), D, F, 128, B, sel, None, k2, 1)
    ref = ffn_reference(gate, up, down, 128, x, [sel[b].long() for b in range(B)])
    assert (ref[0].abs().amax(1) > 2.0 ** -126).all()
    check_ffn(y, ref, 1)
