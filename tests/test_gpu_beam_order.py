"""The order between hypotheses whose keys are equal or nearly so."""

import pytest
import torch

import paper_2511_15898_b200 as G
from paper_2511_15898_b200.build import build_library
from tests.test_gpu_beam import check, reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    build_library()


@pytest.mark.parametrize("penalty", [1.0, 2.0, 0.5, 1.5, -1.0])
def test_equal_quotients_are_equal_keys(penalty):
    """Finished hypotheses of totals -c L^a: all keys are -c, the lower hypothesis comes first."""
    g = torch.Generator().manual_seed(3)
    B, W, V = 24, 32, 300
    n = torch.randint(1, 200, (B, W), generator=g, dtype=torch.int32)
    n[0, :2] = torch.tensor([49, 1])
    n[1:12] = torch.randint(1, 13, (11, W), generator=g, dtype=torch.int32) ** 2
    c = 2.0 ** torch.randint(-3, 4, (B, 1), generator=g)
    if penalty != int(penalty):
        n[0], n[12:] = 4, n[12:].clamp(max=14) ** 2        # (squares: the power is a whole number)
    if penalty < 0:
        n = 2 ** (n % 12)                                  # (and a fraction that fp32 holds)
    s = (-c * n.double() ** penalty).float()
    assert torch.equal(s.double() / n.double() ** penalty, -c.double().expand(B, W))
    x = torch.zeros(B, W, V, device="cuda")
    done = torch.ones(B, W, dtype=torch.bool, device="cuda")
    n, s = n.int().cuda(), s.cuda()
    r = G.beam_select(x, s, W, lengths=n, done=done, eos=2, length_penalty=penalty)
    torch.cuda.synchronize()
    assert torch.equal(r.parent.cpu(), torch.arange(W, dtype=torch.int32).expand(B, W))
    check(r, reference(x, s, W, 1.0, n, done, 2, penalty), W, V, n)
