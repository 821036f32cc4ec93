"""Reordering of states at the limits of its layout: numbers of pieces next to 2^31, lengths beyond what a state holds."""
import pytest
import torch

import paper_2511_15898_b200 as G
from paper_2511_15898_b200.build import build_library

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    build_library()


@pytest.mark.parametrize("pieces", [(1 << 31) - 1, (1 << 31) - 70000])
def test_as_many_pieces_as_there_can_be(pieces):
    # two states of `pieces` pieces of a byte; the last CTA's next piece lies beyond 2^31
    x = torch.zeros(1, 2, pieces, 1, dtype=torch.uint8, device="cuda")
    ends = torch.arange(1, 201, device="cuda", dtype=torch.uint8)
    x[0, 1, -200:, 0] = ends
    x[0, 1, :200, 0] = ends
    x[0, 0, 1 << 30] = 7
    one = torch.ones(1, 2, dtype=torch.int32, device="cuda")
    G.reorder_states([x], torch.tensor([[1, 0]], dtype=torch.int32, device="cuda"), lengths=one, token_dim=3)
    torch.cuda.synchronize()
    assert torch.equal(x[0, 0, -200:, 0], ends) and torch.equal(x[0, 0, :200, 0], ends) and int(x[0, 1, 1 << 30]) == 7
    assert int(x[0, 0, 200:-200].max()) == 0 and int(x[0, 1, -200:].max()) == 0 and int(x[0, 1, :200].max()) == 0


def test_pieces_longer_than_a_cta_takes():
    # the same for pieces that are not short
    x = torch.zeros(1, 2, 70000, 9000, dtype=torch.uint8, device="cuda")
    x[0, 1] = torch.arange(70000, device="cuda").remainder(251).to(torch.uint8).unsqueeze(1)
    n = torch.tensor([[1 << 30, (1 << 31) - 1]], dtype=torch.int32, device="cuda")
    G.reorder_states([x], torch.tensor([[1, -1]], dtype=torch.int32, device="cuda"), lengths=n, token_dim=3)
    torch.cuda.synchronize()
    assert torch.equal(x[0, 0], x[0, 1])


@pytest.mark.parametrize("length", [2, 3, 100, (1 << 31) - 1])
def test_lengths_beyond_the_state_of_large_tokens(length):
    # a token of 4 GB and 32 bytes: a length times that passes 64 bits
    token = (1 << 32) + 32
    x = torch.zeros(1, 2, 2, token, dtype=torch.uint8, device="cuda")
    x[0, 1, :, -50:] = 3
    n = torch.full((1, 2), length, dtype=torch.int32, device="cuda")
    G.reorder_states([x], torch.tensor([[1, 1]], dtype=torch.int32, device="cuda"), lengths=n, token_dim=2)
    torch.cuda.synchronize()
    assert torch.equal(x[0, 0, :, -50:], x[0, 1, :, -50:]) and int(x[0, 0, :, :-50].max()) == 0
