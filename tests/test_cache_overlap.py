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


def append(k, v, q, q_out, dim, heads, q_heads, tokens, ks, vs, qs, os, keys=CACHE, values=CACHE + (1 << 30), lay=None, slots=0, positions=0, freq=0, rot=0):
    x = G.CacheTokens(k, v, q, q_out, G.GR_F16, q_heads, *ks, *vs, *qs, *os)
    return G.gr_cache_append(keys, values, lay or layout(dim, heads), x, tokens, slots, positions, freq, rot, 0, 0)


def test_append():
    rng = random.Random(2)
    met = {True: 0, False: 0}
    for _ in range(4000):
        dim, heads, q_heads, tokens = 2 * rng.randint(1, 3), rng.randint(1, 3), rng.randint(1, 4), rng.randint(1, 5)
        os, span = strides(rng, dim, tokens, q_heads)
        sizes = {"k": heads, "v": heads, "q": q_heads}
        step = {n: os if rng.random() < 0.5 else strides(rng, dim, tokens, h)[0] for n, h in sizes.items()}
        at = {n: A + 2 * rng.randint(-2 * span, 2 * span) for n in sizes}
        if rng.random() < 0.3:
            at["q"], step["q"] = A, os                      # in place
        mine = places(A, 2 * dim, [2 * s for s in os], (tokens, q_heads))
        want = any(places(at[n], 2 * dim, [2 * s for s in step[n]], (tokens, h)) & mine for n, h in sizes.items() if at[n] != A or n != "q")
        if at["q"] == A and any(n > 1 and a != b for n, a, b in zip((tokens, q_heads), step["q"], os)):
            want = True                                     # in place at other strides
        rc = append(at["k"], at["v"], at["q"], A, dim, heads, q_heads, tokens, step["k"], step["v"], step["q"], os)
        assert rc in (-1, -2) and (rc == -1) == want, (dim, heads, q_heads, tokens, os, step, at)
        met[want] += 1
    assert min(met.values()) > 300


def test_append_within_a_projection():
    # [tokens, q heads + 2 heads, dim], of many tokens, queries in place; one element further on
    T, H, Hq, D = 1 << 19, 8, 32, 128
    row = (Hq + 2 * H) * D
    s = (row, D)
    at = [A + 2 * Hq * D, A + 2 * (Hq + H) * D]
    assert append(*at, A, A, D, H, Hq, T, s, s, s, s) == -2
    assert append(at[0] - 2, at[1], A, A, D, H, Hq, T, s, s, s, s) == -1
    assert append(at[0], at[1], A + (1 << 38), A + 2, D, H, Hq, T, s, s, s, s) == -1
    assert append(at[0], at[1], A + 2, A, D, H, Hq, T, s, s, s, s) == -1


def test_caches():
    rng = random.Random(3)
    met = {True: 0, False: 0}
    for _ in range(2000):
        dim, heads, block, blocks = 2 * rng.randint(1, 2), rng.randint(1, 3), rng.randint(1, 3), rng.randint(1, 3)
        span, step = dim, [0, 0, 0]
        for i in rng.sample(range(3), 3):
            n = (blocks, block, heads)[i]
            step[i] = span + rng.choice([0, 0, 1, rng.randint(0, 2 * span)])
            span += step[i] * (n - 1)
        lay = layout(dim, heads, block_size=block, num_blocks=blocks, block_stride=step[0], token_stride=step[1], head_stride=step[2])
        values = CACHE + 2 * rng.randint(-span, span)
        of = [places(p, 2 * dim, [2 * s for s in step], (blocks, block, heads)) for p in (CACHE, values)]
        want = bool(of[0] & of[1])
        rc = append(A, A, 0, 0, dim, heads, 0, 3, (dim, dim), (dim, dim), (0, 0), (0, 0), values=values, lay=lay)
        assert rc in (-1, -2) and (rc == -1) == want, (dim, step, values - CACHE)
        met[want] += 1
    assert min(met.values()) > 200
    # lists among what is written
    s, far = (256, 64), A + (1 << 36)
    for kw in (dict(slots=A + 8), dict(slots=far, positions=A + 512), dict(slots=far, positions=far + 4096, freq=A, rot=2), dict(slots=CACHE + 64), dict(slots=far, positions=CACHE + (1 << 30))):
        assert append(far - (1 << 32), far - (1 << 32), far - (1 << 33), A, 64, 2, 4, 3, s, s, s, s, **kw) == -1, kw


def test_token_logprobs():
    rng = random.Random(4)
    met = {True: 0, False: 0}
    far = 1 << 36

    def call(at, V, ld, rows, given, top, dtype=G.GR_BF16, status=0):
        return G.gr_token_logprobs(at["logits"], dtype, V, ld, rows, 1.0, at["tokens"], given, top, at["logprob"], at["entropy"], at["top_token"], at["top_logprob"], status, 0)

    for _ in range(4000):
        V, rows, given, top = rng.randint(1, 12), rng.randint(1, 4), rng.randint(0, 3), rng.randint(0, 3)
        ld = V + rng.choice([0, 0, 1, 14])
        size = {"tokens": 4 * rows * given, "logprob": 4 * rows * given, "entropy": 4 * rows, "top_token": 4 * rows * top, "top_logprob": 4 * rows * top}
        at = {n: A + (i + 1) * far for i, n in enumerate(size)}
        at["logits"] = A
        a, b = rng.sample(list(at), 2)
        at[b] = at[a] + 4 * rng.randint(-20, 20)
        bytes_of = {n: places(at[n], size[n], (), ()) for n in size}
        bytes_of["logits"] = places(at["logits"], 2 * V, (2 * ld,), (rows,))
        want = {a, b} != {"tokens", "logits"} and bool(bytes_of[a] & bytes_of[b])
        rc = call(at, V, ld, rows, given, top)
        assert rc in (-1, -2) and (rc == -1) == want, (V, ld, rows, given, top, a, b, at[b] - at[a])
        met[want] += 1
    assert min(met.values()) > 300
    at = {n: A + (i + 1) * far for i, n in enumerate(("logits", "tokens", "logprob", "entropy", "top_token", "top_logprob"))}
    for n in ("logits", "tokens", "logprob", "entropy", "top_token", "top_logprob"):
        assert call(at, 1000, 1000, 4, 2, 5, status=at[n] + 4) == -1, n
    assert call({**at, "entropy": 0}, 1000, 1000, 4, 2, 5) == -2
    # an output in the gap between two rows of logits
    assert call({**at, "logits": A, "entropy": A + 2 * 1000}, 1000, 1024, 4, 0, 0) == -2
    assert call({**at, "logits": A, "entropy": A + 2 * 1024 - 12}, 1000, 1024, 4, 0, 0) == -1


def test_attend():
    T, R, width, H, Hq, D = 6, 3, 4, 2, 4, 32
    lay = G.CacheLayout(G.GR_Q4, H, D, 16, 5, 2 * 2 * 9 * D, 0, 0)
    far = 1 << 36
    size = {"q": 2 * T * Hq * D, "out": 2 * T * Hq * D, "table": 4 * R * width, "offsets": 4 * R + 4, "positions": 4 * T, "ws": G.gr_attend_workspace_bytes(H, Hq, D, R, T),
            "status": 4 * R, "cache": 5 * 2 * 2 * 9 * D}
    at = {n: A + (i + 1) * far for i, n in enumerate(size)}

    def call(at):
        return G.gr_cache_attend(at["q"], G.GR_F16, Hq, Hq * D, D, at["cache"], lay, at["table"], width, R, at["offsets"], at["positions"], T, 0.1, 0, at["ws"], at["out"], Hq * D, D,
                                 at["status"], 0)

    written = ("out", "ws", "status")
    for a in written:
        for b in size:
            if a == b:
                continue
            for where, meets in ((0, True), (size[a] - 32 if size[a] >= 32 else 0, True), (size[a] + 31 & ~31, False), (-(size[b] + 31 & ~31), False)):
                # (without a status the call answers -2 where it has found nothing)
                moved = {**at, b: at[a] + where}
                if "status" not in (a, b):
                    moved["status"] = 0
                elif not meets:
                    continue
                assert call(moved) == (-1 if meets else -2), (a, b, where)
