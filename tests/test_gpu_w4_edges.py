"""Weights held in 4 bits at the edges of what the calls allow, against the definition in 64 bits.  Tolerances: those of
tests/test_gpu_w4.py."""
import pytest
import torch

from tests.test_gpu_w4 import DT, check_linear, make_w4, tokens

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
