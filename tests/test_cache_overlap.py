"""Arrays that a call writes and that share bytes with one another, or with what it reads, are refused by the C entry points before anything is
launched, arrays that lie between one another's places are not: against a plain look at every byte.  No GPU needed: without the last
pointer that they look at the calls answer -2 after everything else."""
import random

import pytest

import paper_2511_15898_b200 as G
from paper_2511_15898_b200.build import build_library

A = 1 << 20
CACHE = 1 << 40


@pytest.fixture(scope="module", autouse=True)
def lib():
    build_library()


def places(at, size, steps, sizes):
    out = {at}
    for n, s in zip(sizes, steps):
        out = {a + i * s for a in out for i in range(n)}
    return {a + i for a in out for i in range(size)}


def strides(rng, dim, tokens, heads):
    """Strides of [tokens, heads, dim] in either order, with or without gaps."""
    span, step = dim, [0, 0]
    for i in rng.sample(range(2), 2):
        n = (tokens, heads)[i]
        step[i] = span + rng.choice([0, 0, 1, rng.randint(0, 2 * span)])
        span += step[i] * (n - 1)
    return step, span


def layout(dim, heads, **kw):
    a = dict(format=G.GR_F16, heads=heads, dim=dim, block_size=2, num_blocks=2, block_stride=2 * heads * dim, token_stride=heads * dim, head_stride=dim)
    a.update(kw)
    return G.CacheLayout(*[a[n] for n, _ in G.CacheLayout._fields_])


def test_read():
    rng = random.Random(1)
    met = {True: 0, False: 0}
    for _ in range(4000):
        dim, heads, tokens = 2 * rng.randint(1, 3), rng.randint(1, 4), rng.randint(1, 5)
        ks, span = strides(rng, dim, tokens, heads)
        vs = ks if rng.random() < 0.6 else strides(rng, dim, tokens, heads)[0]
        v = A + 2 * rng.randint(-span, span)
        want = bool(places(A, 2 * dim, [2 * s for s in ks], (tokens, heads)) & places(v, 2 * dim, [2 * s for s in vs], (tokens, heads)))
        rc = G.gr_cache_read(CACHE, CACHE + (1 << 30), layout(dim, heads), 0, tokens, G.GR_F16, A, *ks, v, *vs, 0)
        assert rc in (-1, -2) and (rc == -1) == want, (dim, heads, tokens, ks, vs, v - A)
        met[want] += 1
    assert min(met.values()) > 300
    # keys and values by turns, of many tokens; one token's in the other's
    big = layout(64, 8)
    assert G.gr_cache_read(CACHE, CACHE + (1 << 30), big, 0, 1 << 20, G.GR_F16, A, 1024, 64, A + 2 * 512, 1024, 64, 0) == -2
    assert G.gr_cache_read(CACHE, CACHE + (1 << 30), big, 0, 1 << 20, G.GR_F16, A, 1024, 64, A + 2 * 511, 1024, 64, 0) == -1
    assert G.gr_cache_read(CACHE, CACHE + (1 << 30), big, 0, 1 << 20, G.GR_F16, A, 1024, 128, A + 2 * 64, 1024, 128, 0) == -2
    # slots among the outputs
    assert G.gr_cache_read(CACHE, CACHE + (1 << 30), big, A + 4096, 100, G.GR_F16, A, 1024, 64, A + (1 << 30), 1024, 64, 0) == -1
