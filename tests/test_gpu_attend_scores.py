"""Attention over scores of any size: scales and queries to the ends of their ranges, scores beyond what 32 bits resolve."""
import math

import pytest
import torch

import paper_2511_15898_b200 as G
from tests import paged_cache as P

pytestmark = pytest.mark.gpu
I32 = dict(dtype=torch.int32, device="cuda")


def _one_dim(n, D, seed=5):
    """A cache whose keys have one number, at dim 0: a whole multiple of 1 / 8 from -1 to 7 / 8, exact in 4 bits."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    bs = 8
    N = -(-n // bs)
    kv = G.KVCache.empty(N, bs, 1, D, torch.uint8)
    k = torch.zeros(N * bs, 1, D, device="cuda")
    k[:, 0, 0] = torch.randint(-8, 7, (N * bs,), generator=g, device="cuda") / 8.0
    k[n // 3, 0, 0] = 7 / 8.0
    k[:, 0, 1] = -1.0                                                          # (the element of largest magnitude)
    v = torch.randn(N * bs, 1, D, generator=g, device="cuda")
    G.cache_append(kv, k, v, torch.arange(N * bs, device="cuda"))
    return kv, torch.arange(N, **I32).view(1, -1)


@pytest.mark.parametrize("group,news,D", [(2, 1, 64), (4, 3, 64), (8, 4, 64), (1, 1, 256)])
@pytest.mark.parametrize("scale,size", [(1.0, 1.0), (1e3, 1.0), (1e5, 1.0), (1e7, 3.0), (1e9, 1.0), (1e12, 7.0), (1e20, 1.0), (1e31, 1.0), (1e33, 1.0), (1.6e38, 1.0),
                                        (1e33, 2.0 ** -115), (1.6e38, 2.0 ** -126), (0.1, 1e37), (1.0, 3e38), (1e38, 3e38), (1e-37, 3e38), (-1e10, 1.0), (-1e35, 1.0)])
def test_scores_of_any_size(scale, size, group, news, D):
    """One number to a query and to a key: scores are exact, and however large they are the largest take the weight."""
    for n in (40, 700, 9000):
        kv, table = _one_dim(n, D)
        q = torch.zeros(news, group, D, dtype=torch.bfloat16, device="cuda")
        q[:, :, 0] = size
        got = G.cache_attend(q, kv, table, torch.tensor([0, news], **I32), torch.arange(n - news, n, **I32), scale=scale)
        k, v, _, vs = (torch.from_numpy(x).cuda() for x in P.all4(kv.keys.cpu().numpy()))
        for i in range(news):
            m = n - news + i + 1
            x = float(torch.tensor(scale, dtype=torch.float32)) * k[:m, 0, 0] * float(q[i, 0, 0])
            # (scores themselves, before they are told apart, are right to 2^-20 of them: codes times 16-bit queries, one fp32 sum with the largest, one
            # product with the scale; what that is of the weight's exponent is added to the bound)
            w = (x - x.max()).exp()
            assert torch.isfinite(w).all()
            s = vs[:m, 0].abs()
            dx = 2.0 ** -20 * (x.max() - x)
            want = w @ v[:m, 0] / w.sum()
            bound = ((16 * 2.0 ** -12 + 16 * (m / 16 + 8) * 2.0 ** -22) * (w @ s) + 8 * (m * 2.0 ** -29 + 2.0 ** -24 * w.sum()) * s.max()
                     + (2 * dx * w + 2.0 ** -20 * w) @ v[:m, 0].abs()) / w.sum()
            off = (got.out[i].double() - want).abs()
            assert (off <= bound + 2.0 ** -8 * (want.abs() + bound)).all(), (n, float(off.max()))
        assert (got.status == 0).all()


def test_scores_near_and_beyond_the_largest_in_pieces():
    """Random scores, by factors up to where 32 bits do not resolve them any more: numbers, and never beyond the values'."""
    g = torch.Generator(device="cuda").manual_seed(6)
    n, D, bs = 9000, 64, 8
    kv = G.KVCache.empty(n // bs, bs, 1, D, torch.uint8)
    k, v = (torch.randn(n, 1, D, generator=g, device="cuda") for _ in range(2))
    G.cache_append(kv, k, v, torch.arange(n, device="cuda"))
    table = torch.arange(n // bs, **I32).view(1, -1)
    held = torch.from_numpy(P.all4(kv.keys.cpu().numpy())[1]).cuda()
    for group, news in ((2, 1), (8, 2), (8, 5)):
        q = torch.randn(news, group, D, generator=g, device="cuda").bfloat16()
        for e in range(0, 40, 3):
            got = G.cache_attend(q, kv, table, torch.tensor([0, news], **I32), torch.arange(n - news, n, **I32), scale=math.ldexp(1.0, e))
            top = held.abs().amax(0)[0]
            assert torch.isfinite(got.out).all() and (got.out.double().abs() <= top * (1 + 2.0 ** -7)).all(), e
            assert (got.out.double().abs().amax(-1) > 0.05).all(), e
