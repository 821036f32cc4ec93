"""gr_cache_append and gr_cache_read against a model in 64 bits (tests/paged_cache.py)."""
import numpy as np
import pytest
import torch

import paper_2511_15898_b200 as G
from tests import paged_cache as P

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "q4": torch.uint8}


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _freq(rot):
    return None if not rot else 10000.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)


def _eps(t):
    return torch.finfo(t).eps / 2


def _close(got, want, size, dtype):
    """|got - want| within one rounding to the type and the 32-bit arithmetic before it: cosine and sine 2^-24 of at most 1, two products
    and a sum 2^-24 each, of numbers up to `size` = |a| + |b| (three roundings of each part, 4 * 2^-24 with room for their squares).  The
    type's smallest number covers what is subnormal."""
    bound = _eps(dtype) * (np.abs(want) + 4 * 2.0 ** -24 * size) + 4 * 2.0 ** -24 * size + torch.finfo(dtype).smallest_normal * _eps(dtype)
    worst = np.max(np.abs(got - want) - bound, initial=-1.0)
    assert worst <= 0, worst


def _case(seed, T, H, D, bs, dtype, far=5000):
    """Tokens in rows of several, at random blocks; some without a slot."""
    g = _gen(seed)
    N = -(-T // bs) + 4
    order = torch.randperm(N, generator=g, device="cuda")
    start = int(torch.randint(0, bs, (1,), generator=g, device="cuda"))
    at = torch.arange(T, device="cuda") + start
    slots = order[(at // bs) % N] * bs + at % bs
    some = torch.rand(T, generator=g, device="cuda") < 0.9
    slots = torch.where(some, slots, torch.randint(-3, 0, (T,), generator=g, device="cuda"))
    if T > 4:
        slots[T // 2] = N * bs + 5                       # outside, on the other side
    positions = torch.randint(0, far, (T,), generator=g, device="cuda", dtype=torch.int32)
    k, v = (torch.randn(T, H, D, generator=g, device="cuda").to(dtype) for _ in range(2))
    return g, N, slots, positions, k, v


@pytest.mark.parametrize("T,H,Hq,D,rot,bs,dtype,cache,inter", [
    (1, 1, 1, 64, 64, 16, "bf16", "bf16", False),
    (33, 3, 6, 128, 128, 16, "bf16", "bf16", True),
    (40, 2, 0, 128, 64, 5, "f16", "f16", False),
    (19, 2, 5, 80, 80, 1, "f32", "f32", False),
    (19, 2, 5, 80, 24, 7, "f32", "bf16", True),
    (9, 1, 2, 2, 2, 3, "bf16", "f32", False),
    (9, 1, 2, 6, 2, 3, "bf16", "f16", True),
    (17, 2, 2, 66, 30, 16, "f16", "bf16", False),
    (17, 2, 2, 66, 34, 16, "bf16", "bf16", True),
    (12, 1, 3, 512, 512, 8, "bf16", "bf16", False),
    (12, 1, 3, 510, 510, 8, "f32", "f16", False),
    (50, 2, 2, 96, 0, 32, "bf16", "bf16", False),
    (2500, 2, 4, 64, 64, 16, "bf16", "bf16", False),
    (2501, 1, 1, 128, 96, 64, "f16", "f32", True),
])
def test_append(T, H, Hq, D, rot, bs, dtype, cache, inter):
    g, N, slots, positions, k, v = _case(T * 7 + D, T, H, D, bs, DT[dtype], far=1_000_000)
    kv = G.KVCache.empty(N, bs, H, D, DT[cache])
    for t in kv.tensors():
        t.normal_(generator=g)
    before = [P.to_numpy(t).astype(np.float64) for t in kv.tensors()]
    freq = _freq(rot)
    q = torch.randn(T, Hq, D, generator=g, device="cuda").to(DT[dtype]) if Hq else None
    positions[T // 3] = -1 if T > 2 else positions[T // 3]
    if T > 2:
        slots[T // 3] = -1
    q_out = None if q is None else torch.full_like(q, 7.0)
    got = G.cache_append(kv, k, v, slots, positions, freq, interleaved=inter, q=q, q_out=q_out)
    assert got is q_out
    f = None if freq is None else freq.cpu().numpy()
    pos, z = positions.cpu().numpy(), slots.cpu().numpy()
    held = (z >= 0) & (z < N * bs)
    x = P.to_numpy(k).astype(np.float64)
    want_k = before[0].copy().reshape(N * bs, H, D)
    size = np.zeros_like(want_k)
    want_k[z[held]] = P.rotated(x, pos, f, inter)[held]
    size[z[held]] = np.abs(x[held]).max() * 2
    want_v = before[1].copy().reshape(N * bs, H, D)
    want_v[z[held]] = P.cast(P.to_numpy(v)[held], DT[cache])
    _close(P.to_numpy(kv.keys).astype(np.float64).reshape(N * bs, H, D), want_k, size if rot else 0 * size, DT[cache])
    assert np.array_equal(P.to_numpy(kv.values).astype(np.float64).reshape(N * bs, H, D), want_v)
    untouched = np.ones(N * bs, bool)
    untouched[z[held]] = False
    assert np.array_equal(P.to_numpy(kv.keys).astype(np.float64).reshape(N * bs, H, D)[untouched], want_k[untouched])
    if q is not None:
        x = P.to_numpy(q).astype(np.float64)
        want = P.rotated(x, pos, f, inter)
        want[pos < 0] = 7.0
        _close(P.to_numpy(q_out).astype(np.float64), want, np.full_like(want, np.abs(x).max() * 2 if rot else 0), DT[dtype])
        # in place
        G.cache_append(kv, k, v, slots, positions, freq, interleaved=inter, q=q, q_out=q)
        assert torch.equal(q[positions >= 0], q_out[positions >= 0])


@pytest.mark.parametrize("T,H,D,rot,bs,dtype,inter", [
    (1, 1, 32, 32, 8, "bf16", False), (7, 2, 64, 64, 16, "f16", False), (50, 1, 96, 48, 24, "bf16", True),
    (64, 2, 128, 128, 64, "bf16", False), (30, 2, 128, 64, 16, "f32", False), (21, 1, 256, 256, 8, "bf16", True),
    (20, 1, 160, 0, 40, "f32", False), (23, 1, 224, 222, 16, "f32", False), (2400, 1, 64, 64, 16, "bf16", False),
    (9601, 1, 64, 64, 24, "f16", False), (37890, 1, 32, 32, 40, "bf16", False),
])
def test_append_in_four_bits(T, H, D, rot, bs, dtype, inter):
    g, N, slots, positions, k, v = _case(T * 3 + D, T, H, D, bs, DT[dtype])
    kv = G.KVCache.empty(N, bs, H, D, torch.uint8)
    kv.keys.random_(0, 256, generator=g)
    want = kv.keys.cpu().numpy().copy()
    freq = _freq(rot)
    q = torch.randn(T, 3, D, generator=g, device="cuda").to(DT[dtype])
    k[0, 0, :32] = 0                                       # a group of zeros
    v[T // 2, 0, :32] = 0
    v[T // 2, 0, 3], v[T // 2, 0, 7] = 2.0, -2.0           # two of the largest magnitude
    v[T - 1, 0, :32] = torch.arange(-16, 16, device="cuda") / 4      # quotients on borders between codes
    q_out = G.cache_append(kv, k, v, slots, positions, freq, interleaved=inter, q=q)
    pos, z = positions.cpu().numpy(), slots.cpu().numpy()
    f = None if freq is None else freq.cpu().numpy()
    kr, vr = P.rotated32(P.to_numpy(k), pos, f, inter), P.to_numpy(v).astype(np.float32)
    few = T <= 64
    if few:
        for i in range(T):
            if 0 <= z[i] < N * bs:
                P.write4(want, bs, z[i], kr[i], vr[i])
        assert np.array_equal(kv.keys.cpu().numpy(), want)
    else:
        gk, gv = P.read4(kv.keys.cpu().numpy(), bs, z)
        held = (z >= 0) & (z < N * bs)
        for x, y in ((gk, kr), (gv, vr)):
            code, scale, _ = P.groups(y[held])
            assert np.array_equal(x[held].reshape(code.shape), (code.astype(np.float64) - 8) * scale.astype(np.float64)[..., None])
    # the queries are those of a 16- or 32-bit cache
    other = G.KVCache.empty(N, bs, H, D, DT[dtype])
    assert torch.equal(G.cache_append(other, k, v, slots, positions, freq, interleaved=inter, q=q), q_out)
    # and what is read back is what the codes stand for
    gk, gv = P.read4(kv.keys.cpu().numpy(), bs, z)
    for t in (torch.float32, torch.bfloat16, torch.float16):
        rk, rv = G.cache_read(kv, slots, t)
        assert np.array_equal(P.to_numpy(rk).astype(np.float64), P.cast(gk, t)) and np.array_equal(P.to_numpy(rv).astype(np.float64), P.cast(gv, t))


def test_numbers_at_the_ends_of_the_range():
    kv = G.KVCache.empty(2, 8, 1, 64, torch.uint8)
    k = torch.zeros(4, 1, 64, device="cuda")
    k[0, 0, :32] = 3e38
    k[0, 0, 5] = -3.4e38
    k[1, 0, 3], k[1, 0, 40] = float("nan"), 1.0
    k[2, 0, 33], k[2, 0, 1] = float("-inf"), -2.0
    k[3, 0, :32] = 1e-38
    slots = torch.arange(4, device="cuda") + 2
    G.cache_append(kv, k, k, slots)
    rk, rv = (x.cpu() for x in G.cache_read(kv, slots, torch.float32))
    assert torch.equal(rk, rv) or (torch.isnan(rk) == torch.isnan(rv)).all()
    assert rk[0, 0, 5] == -8 * 65504.0 and (rk[0, 0, :5] == 7 * 65504.0).all() and (rk[0, 0, 32:] == 0).all()
    assert torch.isnan(rk[1, 0, :32]).all() and rk[1, 0, 40] == 1.0 and (rk[1, 0, 41:] == 0).all()
    assert torch.isnan(rk[2, 0, 32:]).all() and rk[2, 0, 1] == -2.0
    assert (rk[3] == 0).all()


@pytest.mark.parametrize("cache,D,bs", [("bf16", 128, 16), ("f32", 66, 5), ("f16", 40, 1), ("q4", 96, 24)])
@pytest.mark.parametrize("out", ["f32", "bf16", "f16"])
def test_read_any_slots(cache, D, bs, out):
    g = _gen(5)
    kv = G.KVCache.empty(9, bs, 3, D, DT[cache])
    if cache == "q4":
        G.cache_append(kv, *(torch.randn(9 * bs, 3, D, generator=g, device="cuda") for _ in range(2)), torch.arange(9 * bs, device="cuda"))
        k, v = P.read4(kv.keys.cpu().numpy(), bs, range(9 * bs))
    else:
        for t in kv.tensors():
            t.normal_(generator=g)
        k, v = (P.to_numpy(t).astype(np.float64).reshape(9 * bs, 3, D) for t in kv.tensors())
    slots = torch.randint(-2, 9 * bs + 2, (77,), generator=g, device="cuda")
    slots[3] = slots[2]                                    # the same slot twice
    z = slots.cpu().numpy()
    held = (z >= 0) & (z < 9 * bs)
    buf = torch.full((77, 2, 3, D + 3), 5.0, dtype=DT[out], device="cuda")
    got = G.cache_read(kv, slots, out=(buf[:, 0, :, :D], buf[:, 1, :, :D]))
    for x, y in zip(got, (k, v)):
        want = np.zeros((77, 3, D))
        want[held] = y[z[held]]
        assert np.array_equal(P.to_numpy(x).astype(np.float64), P.cast(want, DT[out]))
    assert (buf[..., D:] == 5).all()


def test_strides_and_alignment():
    """Keys, values and queries out of one projection's rows, queries in place; a cache whose keys and values share a buffer, by heads."""
    g = _gen(6)
    T, H, Hq, D, bs, N = 21, 2, 4, 64, 16, 5
    freq, slots = _freq(64), torch.randperm(N * bs, generator=g, device="cuda")[:T]
    positions = torch.arange(T, device="cuda", dtype=torch.int32) * 1000
    for shift in (0, 1, 4):
        row = torch.randn(T, (Hq + 2 * H) * D + 8, generator=g, device="cuda").to(torch.bfloat16)
        qkv = row[:, shift:shift + (Hq + 2 * H) * D].unflatten(1, (Hq + 2 * H, D))
        q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
        plain = G.KVCache.empty(N, bs, H, D)
        want_q = G.cache_append(plain, k.contiguous(), v.contiguous(), slots, positions, freq, q=q.contiguous())
        both = torch.zeros(N, H, 2, bs, D, dtype=torch.bfloat16, device="cuda")
        cache = G.KVCache(both[:, :, 0].transpose(1, 2), both[:, :, 1].transpose(1, 2), bs, H, D)
        kept = row.clone()
        G.cache_append(cache, k, v, slots, positions, freq, q=q, q_out=q)
        assert torch.equal(q, want_q) and torch.equal(cache.keys, plain.keys) and torch.equal(cache.values, plain.values)
        kept[:, shift:shift + Hq * D] = q.flatten(1)
        assert torch.equal(kept, row)
        # one token's keys for all
        one = k[:1].expand(T, H, D)
        G.cache_append(cache, one, one, slots)
        assert torch.equal(cache.keys.reshape(N * bs, H, D)[slots], one) and torch.equal(cache.values.reshape(N * bs, H, D)[slots], one)
        four, same = (G.KVCache.empty(N, bs, H, D, torch.uint8) for _ in range(2))
        G.cache_append(four, k, v, slots, positions, freq)
        G.cache_append(same, k.contiguous(), v.contiguous(), slots, positions, freq)
        assert torch.equal(four.keys, same.keys)


def test_far_places():
    """Slots beyond 2^31 elements and bytes of the cache."""
    H, D, bs = 8, 128, 16
    N = (1 << 32) // (bs * H * D * 2) + 3                  # 4 GB each of keys and values
    kv = G.KVCache(torch.empty(N, bs, H, D, dtype=torch.bfloat16, device="cuda"), torch.empty(N, bs, H, D, dtype=torch.bfloat16, device="cuda"), bs, H, D)
    g = _gen(7)
    slots = torch.tensor([N * bs - 1, 3, N * bs // 2 + 1], device="cuda")
    k, v = (torch.randn(3, H, D, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    G.cache_append(kv, k, v, slots)
    assert torch.equal(kv.keys.view(-1, H, D)[slots], k) and torch.equal(kv.values.view(-1, H, D)[slots], v)
    rk, rv = G.cache_read(kv, slots)
    assert torch.equal(rk, k) and torch.equal(rv, v)
    del kv
    N = (1 << 32) // (bs * H * 9 * D // 8) + 3
    kv = G.KVCache(torch.empty(N, H, bs // 8, 9 * D, dtype=torch.uint8, device="cuda"), None, bs, H, D)
    slots = torch.tensor([N * bs - 1, 3, N * bs // 2 + 1], device="cuda")
    G.cache_append(kv, k, v, slots)
    near = G.KVCache.empty(1, 8, H, D, torch.uint8)
    at = torch.arange(3, device="cuda")
    G.cache_append(near, k, v, at)
    for x, y in zip(G.cache_read(kv, slots), G.cache_read(near, at)):
        assert torch.equal(x, y)


def test_streams_and_graphs():
    g = _gen(8)
    T, H, D = 40, 2, 128
    kv = G.KVCache.empty(6, 16, H, D, torch.uint8)
    k, v, q = (torch.randn(T, H, D, generator=g, device="cuda").to(torch.bfloat16) for _ in range(3))
    slots = torch.randperm(96, generator=g, device="cuda")[:T]
    positions, freq = torch.arange(T, device="cuda", dtype=torch.int32), _freq(D)
    q_out, out = torch.empty_like(q), tuple(torch.empty_like(k) for _ in range(2))

    def step():
        G.cache_append(kv, k, v, slots, positions, freq, q=q, q_out=q_out)
        G.cache_read(kv, slots, out=out)

    step()
    want = [x.clone() for x in (kv.keys, q_out, *out)]
    side = torch.cuda.Stream()
    for x in (kv.keys, q_out, *out):
        x.zero_()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (kv.keys, q_out, *out)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for x in (kv.keys, q_out, *out):
        x.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (kv.keys, q_out, *out)))


def test_nothing_to_do():
    kv = G.KVCache.empty(2, 8, 1, 32, torch.uint8)
    none = torch.zeros(0, 1, 32, device="cuda")
    G.cache_append(kv, none, none, torch.zeros(0, dtype=torch.int64, device="cuda"))
    k, v = G.cache_read(kv, torch.zeros(0, dtype=torch.int64, device="cuda"))
    assert k.shape == (0, 1, 32) and v.shape == (0, 1, 32)
    empty = G.KVCache.empty(0, 8, 1, 32)
    x = torch.ones(2, 1, 32, device="cuda")
    G.cache_append(empty, x, x, torch.zeros(2, dtype=torch.int64, device="cuda"))
    k, v = G.cache_read(empty, torch.zeros(2, dtype=torch.int64, device="cuda"))
    assert (k == 0).all() and (v == 0).all()
