"""Numbers at and beyond the range of a 4-bit group's scale, in every place of a word of codes: byte by byte against the model."""
import numpy as np
import pytest
import torch

import paper_2511_15898_b200 as G
from tests import paged_cache as P

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _group(g, place, peak, dtype):
    """32 numbers: a peak among ordinary ones, some of its own size beside it, of either sign."""
    x = torch.randn(32, generator=g, device="cuda") * 1e4
    x[place] = peak
    x[(place + 9) % 32] = -peak * 0.75
    x[(place + 13) % 32] = -0.5 * peak
    x[(place + 22) % 32] = peak * 0.9375
    return x.to(dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("peak", [5.2e5, 5.3e5, 5.5e5, 5.6e5, 6e5, 1e6, 3e6, 1e8, 1e9, 1e11, 1e13, 1e15, 1e20, 1e30, 3e38])
def test_codes_of_a_clamped_scale(peak, dtype):
    g = torch.Generator(device="cuda").manual_seed(1)
    H, D, bs = 2, 64, 16
    k, v = (torch.stack([torch.cat([_group(g, (i + h) % 32, peak * (1 if (i // 8 + h) % 2 else -1), DT[dtype]),
                                    torch.randn(32, generator=g, device="cuda").to(DT[dtype])]).roll(32 * (i % 2)) for i in range(24) for h in range(H)])
            .view(24, H, D) for _ in range(2))
    slots = torch.randperm(3 * bs, generator=g, device="cuda")[:24]
    kv = G.KVCache.empty(3, bs, H, D, torch.uint8)
    want = kv.keys.cpu().numpy().copy()
    G.cache_append(kv, k, v, slots)
    for z, a, b in zip(slots.tolist(), P.to_numpy(k).astype(np.float32), P.to_numpy(v).astype(np.float32)):
        P.write4(want, bs, z, a, b)
    assert np.array_equal(kv.keys.cpu().numpy(), want)
    # and in the windows of many tokens
    many = G.KVCache.empty(300, bs, H, D, torch.uint8)
    at = torch.arange(2400, device="cuda")
    G.cache_append(many, k.repeat(100, 1, 1), v.repeat(100, 1, 1), at)
    one = G.KVCache.empty(300, bs, H, D, torch.uint8)
    for lo in range(0, 2400, 24):
        G.cache_append(one, k, v, at[lo:lo + 24])
    assert torch.equal(many.keys, one.keys)
    for a, b in zip(G.cache_read(kv, slots, torch.float32), P.read4(want, bs, slots.tolist())):
        assert np.array_equal(P.to_numpy(a).astype(np.float64), b)
