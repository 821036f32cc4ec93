"""Attention whose weights and values are of any size: a token that takes most of the weight before thousands that share the rest, small
and large values.  Bounds are relative to the weighted scales."""
import pytest
import torch

import paper_2511_15898_b200 as G
from tests import paged_cache as P

pytestmark = pytest.mark.gpu
I32 = dict(dtype=torch.int32, device="cuda")


def _model(q, kv, table, offsets, positions, scale, window=0):
    """out in 64 bits, and a bound of the error before the last rounding.

    A weight w (of 1 for the largest) is rounded to 11 bits, its product with the scale s once more: 2^-12 of each, taken u - 8 times, up to 8:
    16 2^-12 w |s|.  Numbers below 2^-14 are off by 2^-25 instead.  The largest weight is held as 2^10 at least (where the largest scale S is above 2, as that over
    S / 2 rounded up to a power of two), so that is 2^-35 max(1, S) for a weight, times s, and for a product, 8 times.  Scores are off by dx: eight
    roundings of 2^-23 of sum |q| 16 |s| (codes up to 15 and the sum of the queries times 8).  Sums of n / 16 products and eight joins in 32 bits: 2^-22
    of 16 w |s| each."""
    held = [torch.from_numpy(x).cuda() for x in P.all4(kv.keys.cpu().numpy())]
    k, v, ks, vs = held
    T, Hq, D = q.shape
    H = k.shape[1]
    out, bound = (torch.zeros(T, Hq, D, dtype=torch.float64, device="cuda") for _ in range(2))
    for r in range(len(offsets) - 1):
        for i in range(int(offsets[r]), int(offsets[r + 1])):
            p = int(positions[offsets[r]]) + i - int(offsets[r])
            t = torch.arange(max(0, p - window + 1) if window else 0, p + 1, device="cuda")
            z = table[r, t // kv.block_size].long() * kv.block_size + t % kv.block_size
            for h in range(Hq):
                g = h // (Hq // H)
                x = scale * (k[z, g] @ q[i, h].double())
                dx = 8 * 2.0 ** -23 * float((abs(scale) * 16 * ks[z, g].abs() @ q[i, h].double().abs()).max())
                w = (x - x.max()).exp()
                s = vs[z, g].abs()
                n, ws = len(z), w @ s
                out[i, h] = w @ v[z, g] / w.sum()
                bound[i, h] = ((16 * 2.0 ** -12 + 16 * (n / 16 + 8) * 2.0 ** -22) * ws + 8 * n * 2.0 ** -35 * s.max().clamp(min=1) * (1 + s.max())
                               + (2 * dx + 2.0 ** -20) * (w @ v[z, g].abs())) / w.sum()
    return out, bound


def _check(q, kv, table, offsets, positions, scale, window=0):
    got = G.cache_attend(q, kv, table, torch.tensor(offsets, **I32), torch.tensor(positions, **I32), scale=scale, window=window)
    assert (got.status == 0).all()
    want, bound = _model(q, kv, table, offsets, positions, scale, window)
    off = (got.out.double() - want).abs()
    limit = bound + torch.finfo(q.dtype).eps / 2 * (want.abs() + bound) + torch.finfo(q.dtype).smallest_normal * torch.finfo(q.dtype).eps / 2
    assert torch.isfinite(off).all() and (off <= limit).all(), float((off / limit).max())
    return got, want, bound


def _sink(gap, n, v_size, D, H=1, seed=0):
    """A cache of n tokens whose first has a score `gap` nats above the others' for a query of ones (scale 1), values of v_size around their mean."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    bs = 16
    N = -(-n // bs)
    kv = G.KVCache.empty(N, bs, H, D, torch.uint8)
    k = torch.zeros(N * bs, H, D, device="cuda")
    k[0] = gap / D
    v = (1 + 0.3 * torch.randn(N * bs, H, D, generator=g, device="cuda")) * v_size
    v[0] = -v[0]
    G.cache_append(kv, k, v, torch.arange(N * bs, device="cuda"))
    return kv, torch.arange(N, **I32).view(1, -1)


@pytest.mark.parametrize("group,news,D", [(2, 1, 64), (4, 3, 64), (8, 4, 64), (4, 1, 128), (4, 1, 256)])
@pytest.mark.parametrize("v_size", [1e-5, 1e-3, 0.01, 0.05, 1.0, 300.0, 4e5])
def test_much_weight_in_small_parts(v_size, group, news, D):
    dtype = torch.bfloat16 if v_size > 1000 else torch.float16
    for n, gaps in ((600, (3.0, 9.0)), (8000, (10.0, 11.0, 13.0)), (40000, (12.0, 16.0))):
        if n == 40000 and (group, news, D) != (2, 1, 64):
            continue
        for gap in gaps:
            kv, table = _sink(gap, n, v_size, D)
            q = torch.ones(news, group, D, dtype=dtype, device="cuda")
            _check(q, kv, table, [0, news], list(range(n - news, n)), 1.0)


def test_groups_of_different_sizes():
    """Values of 100, 1 and 0.01 in one head; larger ones that come late."""
    n, D = 4000, 96
    kv, table = _sink(8.0, n, 1.0, D)
    g = torch.Generator(device="cuda").manual_seed(2)
    v = torch.randn(n, 1, D, generator=g, device="cuda") * torch.tensor([100.0, 1.0, 0.01], device="cuda").repeat_interleave(32)
    k = torch.randn(n, 1, D, generator=g, device="cuda") * 0.2
    v[n - 700:] *= 50
    v[:64] *= 1e-3
    G.cache_append(kv, k, v, torch.arange(n, device="cuda"))
    for group, news in ((1, 1), (8, 2), (8, 5)):
        q = torch.randn(news, group, D, generator=g, device="cuda").bfloat16()
        for window in (0, 900):
            _check(q, kv, table, [0, news], list(range(n - news, n)), 0.4, window)


@pytest.mark.parametrize("news,group", [(1, 2), (4, 4), (9, 4)])
def test_large_values_that_are_not_seen_do_not_tell(news, group):
    g = torch.Generator(device="cuda").manual_seed(3)
    bs, H, D, N = 16, 1, 64, 40
    lengths = [100, 37, 300]
    kv = G.KVCache.empty(N, bs, H, D, torch.uint8)
    k, v = (torch.randn(N * bs, H, D, generator=g, device="cuda") for _ in range(2))
    G.cache_append(kv, k, v * 0.02, torch.arange(N * bs, device="cuda"))
    table = torch.full((3, 20), -1, **I32)
    order = torch.randperm(N, generator=g, device="cuda").int()
    at = 0
    for r, n in enumerate(lengths):
        table[r, :-(-n // bs)] = order[at:at + -(-n // bs)]
        at += -(-n // bs)
    offsets = torch.arange(0, 3 * news + 1, news, **I32)
    positions = torch.cat([torch.arange(n - news, n, **I32) for n in lengths])
    q = torch.randn(3 * news, H * group, D, generator=g, device="cuda").half()
    want = [G.cache_attend(q, kv, table, offsets, positions, window=w).out.clone() for w in (0, 30)]
    bad = torch.ones(N * bs, dtype=torch.bool, device="cuda")
    for r, n in enumerate(lengths):
        t = torch.arange(n, device="cuda")
        bad[table[r, t // bs].long() * bs + t % bs] = False
    slots = bad.nonzero().view(-1)
    big = torch.full((len(slots), H, D), 4e5, device="cuda")
    G.cache_append(kv, big, big, slots)
    for w, x in zip((0, 30), want):
        assert torch.equal(G.cache_attend(q, kv, table, offsets, positions, window=w).out, x)
    # the last token of each row tells only its own query, the first ones none with a window
    last = torch.tensor([int(table[r, (n - 1) // bs]) * bs + (n - 1) % bs for r, n in enumerate(lengths)], device="cuda")
    first = table[:, 0].long() * bs
    kept = kv.keys.clone()
    G.cache_append(kv, k[:3], big[:3], last)
    got = G.cache_attend(q, kv, table, offsets, positions).out.view(3, news, -1)
    assert torch.equal(got[:, :-1], want[0].view(3, news, -1)[:, :-1]) and not torch.equal(got[:, -1], want[0].view(3, news, -1)[:, -1])
    kv.keys.copy_(kept)
    G.cache_append(kv, big[:3], big[:3], first)
    got = G.cache_attend(q, kv, table, offsets, positions, window=20).out
    kv.keys.copy_(kept)
    assert torch.equal(got, G.cache_attend(q, kv, table, offsets, positions, window=20).out)


def test_a_group_that_is_no_number():
    """One group of one token's values: all that see the token are no numbers, all that do not are as before."""
    n, D = 200, 96
    kv, table = _sink(3.0, n, 1.0, D)
    for group, news in ((2, 1), (2, 8), (8, 8)):
        q = torch.ones(news, group, D, dtype=torch.float16, device="cuda")
        call = (q, kv, table, torch.tensor([0, news], **I32), torch.arange(n - news, n, **I32))
        words = kv.keys.view(torch.float16)
        for token, windows in ((n - 1, (0,)), (50, (0, 100))):
            want = [G.cache_attend(*call, window=w).out.clone() for w in windows]
            words[token // 16, 0, token % 16 // 8][(8 * D + D // 2) // 2 + (token % 8 // 2 * (D // 32) + 1) * 2 + token % 2] = float("nan")
            for w, before in zip(windows, want):
                got = G.cache_attend(*call, window=w).out
                sees = torch.tensor([(p >= token and (not w or p - w < token)) for p in range(n - news, n)], device="cuda")
                assert torch.isnan(got[sees]).all() and torch.equal(got[~sees], before[~sees])
            kv, table = _sink(3.0, n, 1.0, D)
            call = (q, kv, *call[2:])
            words = kv.keys.view(torch.float16)


@pytest.mark.parametrize("D", [32, 96, 160, 192, 224])
@pytest.mark.parametrize("group,news", [(3, 1), (4, 3), (8, 4)])
def test_heads_of_other_sizes(D, group, news):
    for v_size, n, gap in ((0.02, 3000, 9.5), (50.0, 1500, 6.0), (2e4, 700, 2.0)):
        kv, table = _sink(gap, n, v_size, D, seed=D)
        q = torch.ones(news, group, D, dtype=torch.bfloat16, device="cuda")
        for window in (0, 333):
            _check(q, kv, table, [0, news], list(range(n - news, n)), 1.0, window)
