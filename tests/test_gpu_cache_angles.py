"""Rotations by angles of any size: positions to the last, frequencies far beyond those of a model; from 2^50 on there are none."""
import numpy as np
import pytest
import torch

import paper_2511_15898_b200 as G
from tests import paged_cache as P

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("T", [7, 2400])
def test_far_angles(T, inter):
    """Within three roundings of 2^-24 of |a| + |b| for the cosine and the sine, the products and the sum (four with room for their
    squares); angles are 64-bit numbers, and their cosines are those of numpy.  Pairs turned by 2^50 and more are NaN."""
    g = torch.Generator(device="cuda").manual_seed(T)
    freq = np.array([1.0, 3.7, 2.0 ** 19, 1.3e6, 2.0 ** 20, 1e9, 2.0 ** 50, 1e15, 2.3e15, 1e18, 7e22, 1e30, 1e100, 1e290, 1e-300, 0.0])
    positions = torch.tensor([1, 2, 2 ** 31 - 1, -5, 1 << 30, 12345, 0], dtype=torch.int32).repeat(-(-T // 7))[:T].cuda()
    H, D = 2, 40
    k, q = (torch.randn(T, H, D, generator=g, device="cuda") for _ in range(2))
    kv = G.KVCache.empty(-(-T // 8), 8, H, D, torch.float32)
    slots = torch.arange(T, device="cuda")
    f = torch.from_numpy(freq).cuda()
    q_out = G.cache_append(kv, k, k, slots, positions, f, interleaved=inter, q=q)
    served = (positions >= 0).cpu().numpy()
    for got, x, some in ((kv.keys.view(-1, H, D)[:T], k, np.ones(T, bool)), (q_out, q, served)):
        pos = positions.cpu().numpy()
        want = P.rotated(P.to_numpy(x).astype(np.float64), pos, freq, inter)
        far = np.zeros(want.shape, bool)
        for c, turns in enumerate(np.abs(pos[:, None].astype(np.float64) * freq[None]).T >= 2.0 ** 50):
            far[:, :, [2 * c, 2 * c + 1] if inter else [c, c + len(freq)]] = turns[:, None, None]
        got = P.to_numpy(got).astype(np.float64)
        assert np.array_equal(np.isnan(got)[some], far[some]) and far[some].any()
        off = np.where(far, 0, np.abs(got - want))[some]
        assert (off <= 4 * 2.0 ** -24 * 2 * np.abs(P.to_numpy(x)).max()).all(), off.max()
    assert (q_out[positions < 0] == 0).all()
    wrong = torch.tensor([float("inf"), float("nan")], dtype=torch.float64, device="cuda")
    plain = G.KVCache.empty(1, 8, H, D, torch.float32)
    G.cache_append(plain, k[:1], k[:1], slots[:1], positions[:1], wrong)
    assert torch.isnan(plain.keys[0, 0][:, :4]).all() and torch.equal(plain.keys[0, 0][:, 4:], k[0, :, 4:])
