"""gr_cache_attend against a model in 64 bits (tests/paged_cache.py, which also bounds the error)."""
import numpy as np
import pytest
import torch

import paper_2511_15898_b200 as G
from tests import paged_cache as P

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f16": torch.float16}


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _fill(g, N, bs, H, D, k_size=1.0, v_size=1.0):
    kv = G.KVCache.empty(N, bs, H, D, torch.uint8)
    k, v = (torch.randn(N * bs, H, D, generator=g, device="cuda") * s for s in (k_size, v_size))
    G.cache_append(kv, k, v, torch.arange(N * bs, device="cuda"))
    return kv


def _rows(g, lengths, news, bs, width, N):
    """Tables of random blocks, offsets and positions of rows of these lengths, the last `news` of them the queries."""
    R = len(lengths)
    order = torch.randperm(N, generator=g, device="cuda").tolist()
    table = np.full((R, width), -1, np.int32)
    for r, n in enumerate(lengths):
        for b in range(-(-n // bs)):
            table[r, b] = order.pop()
    offsets = np.concatenate([[0], np.cumsum(news)]).astype(np.int32)
    positions = np.concatenate([np.arange(n - m, n) for n, m in zip(lengths, news)] + [[]]).astype(np.int32)
    return table, offsets, positions


def _check(kv, q, table, offsets, positions, scale=None, window=0, out=None, held=None):
    cuda = [torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in (table, offsets, positions)]
    got = G.cache_attend(q, kv, *cuda, scale=scale, window=window, out=out)
    held = P.all4(kv.keys.cpu().numpy()) if held is None else held
    want, bound = P.attention(P.to_numpy(q).astype(np.float64), held, kv.block_size, table, offsets, positions,
                              kv.dim ** -0.5 if scale is None else scale, window)
    used = int(offsets[-1])
    off = np.abs(P.to_numpy(got.out).astype(np.float64)[:used] - want[:used])
    bound = bound[:used] + torch.finfo(q.dtype).eps / 2 * (np.abs(want[:used]) + bound[:used]) + 2.0 ** -25
    assert np.isfinite(off).all() and (off <= bound).all(), (np.nanmax(off - bound), np.isfinite(off).all())
    return got


@pytest.mark.parametrize("D", [32, 64, 96, 128, 160, 192, 224, 256])
@pytest.mark.parametrize("H,group,news,dtype", [(2, 1, 1, "bf16"), (1, 4, 1, "f16"), (2, 8, 1, "bf16"), (1, 5, 3, "f16"), (1, 4, 9, "bf16"), (1, 16, 5, "f16")])
def test_attend(D, H, group, news, dtype):
    g = _gen(D + 10 * group + news)
    bs = [8, 16, 24, 64][(D // 32 + group) % 4]
    lengths = [news, 17 + news, 64, 200, 333]
    N = sum(-(-n // bs) for n in lengths) + 3
    kv = _fill(g, N, bs, H, D)
    rows = _rows(g, lengths, [news] * 5, bs, -(-333 // bs) + 1, N)
    q = (2 * torch.randn(5 * news, H * group, D, generator=g, device="cuda")).to(DT[dtype])
    got = _check(kv, q, *rows)
    assert (got.status == 0).all()
    for window in (1, 40, 64, 300):
        _check(kv, q, *rows, window=window)


@pytest.mark.parametrize("D,group", [(64, 4), (128, 8), (128, 1), (256, 4)])
def test_ragged_rows(D, group):
    """Rows of no, one, a few and many queries, of one to many tokens, and one that was not served; what lies behind stays."""
    g = _gen(D + group)
    bs, H = 16, 2
    lengths, news = [1, 700, 5, 40, 129, 64, 2000, 30, 1], [1, 1, 0, 40, 7, 64, 33, 5, 1]
    N = sum(-(-n // bs) for n in lengths) + 3
    kv = _fill(g, N, bs, H, D)
    table, offsets, positions = _rows(g, lengths, news, bs, 130, N)
    positions[offsets[7]:offsets[8]] = -1
    T = offsets[-1] + 6
    positions = np.concatenate([positions, np.full(6, -1, np.int32)])
    q = torch.randn(T, H * group, D, generator=g, device="cuda").to(torch.bfloat16)
    kept = None
    for window in (0, 50):
        kept = _check(kv, q, table, offsets, positions, window=window, out=kept)
        assert (kept.status == 0).all() and (kept.out[offsets[7]:offsets[8]] == 0).all() and (kept.out[offsets[-1]:] == 0).all()
    kept.out.fill_(3.0)
    kept = _check(kv, q, table, offsets, positions, out=kept)
    assert (kept.out[offsets[-1]:] == 3).all() and (kept.out[offsets[7]:offsets[8]] == 0).all()


def test_long_row_in_pieces():
    """One row in hundreds of pieces, one large score in the middle, and one that comes last."""
    g = _gen(3)
    bs, H, D, n = 64, 1, 128, 40000
    kv = _fill(g, 640, bs, H, D)
    rows = _rows(g, [n], [1], bs, 640, 640)
    q = torch.randn(1, 4, D, generator=g, device="cuda").to(torch.bfloat16)
    held = P.all4(kv.keys.cpu().numpy())
    _check(kv, q, *rows, held=held)
    for at in (20001, n - 1):
        slot = int(rows[0][0, at // bs]) * bs + at % bs
        q[0, 0] = torch.from_numpy(held[0][slot, 0]).cuda().to(torch.bfloat16)
        _check(kv, q, *rows, held=held, scale=0.5)


@pytest.mark.parametrize("news,group", [(1, 2), (4, 4), (9, 4)])
def test_what_is_not_seen_does_not_tell(news, group):
    """NaN and infinities in places behind a query, before its window, in blocks of nobody and in the rest of the last block."""
    g = _gen(4)
    bs, H, D = 16, 2, 64
    lengths = [100, 37, 300]
    N = 60
    kv = _fill(g, N, bs, H, D)
    rows = _rows(g, lengths, [news] * 3, bs, 20, N)
    q = torch.randn(3 * news, H * group, D, generator=g, device="cuda").to(torch.bfloat16)
    clean = [_check(kv, q, *rows, window=w).out.clone() for w in (0, 70)]
    table = torch.from_numpy(rows[0]).cuda()
    data = kv.keys.view(torch.float16)
    bad = torch.ones(N * bs, dtype=torch.bool, device="cuda")
    for r, n in enumerate(lengths):
        t = torch.arange(n, device="cuda")
        bad[table[r, t // bs].long() * bs + t % bs] = False
    nan = torch.full((int(bad.sum()), H, D), float("nan"), device="cuda")
    G.cache_append(kv, nan, nan, bad.nonzero().view(-1))
    assert torch.isnan(data).any()
    for w, want in zip((0, 70), clean):
        assert torch.equal(G.cache_attend(q, kv, table, *(torch.from_numpy(x).cuda() for x in rows[1:]), window=w).out, want)
    # the last token of each row: the queries before it do not see it
    last = torch.tensor([int(rows[0][r, (n - 1) // bs]) * bs + (n - 1) % bs for r, n in enumerate(lengths)], device="cuda")
    G.cache_append(kv, nan[:3], nan[:3], last)
    got = G.cache_attend(q, kv, table, *(torch.from_numpy(x).cuda() for x in rows[1:])).out.view(3, news, -1)
    assert torch.isnan(got[:, -1]).all() and torch.equal(got[:, :-1], clean[0].view(3, news, -1)[:, :-1])
    # the first ones: outside the window
    first = table[:, 0].long() * bs
    G.cache_append(kv, nan[:3], nan[:3], first)
    got = G.cache_attend(q, kv, table, *(torch.from_numpy(x).cuda() for x in rows[1:]), window=20).out.view(3, news, -1)
    short = G.cache_attend(q, kv, table, *(torch.from_numpy(x).cuda() for x in rows[1:]), window=70).out.view(3, news, -1)
    assert not torch.isnan(got[:, :-1]).any() and torch.isnan(short[1, :-1]).all() and not torch.isnan(short[2, :-1]).any()


def test_bad_rows():
    """Ids outside the pool, positions beyond the table: left out, and said so; the other rows as ever."""
    g = _gen(5)
    bs, H, D = 16, 1, 64
    N = 40
    kv = _fill(g, N, bs, H, D)
    table, offsets, positions = _rows(g, [100, 100, 60, 90, 50], [2] * 5, bs, 8, N)
    q = torch.randn(10, 4, D, generator=g, device="cuda").to(torch.float16)
    good = _check(kv, q, table, offsets, positions).out.clone()
    table[1, 2], table[3, 0], table[2, 5] = N, -7, 1 << 30      # (the last is behind its row's tokens)
    positions[offsets[4]:] = [127, 128]                    # 128 places
    got = _check(kv, q, table, offsets, positions)
    assert got.status.tolist() == [0, 10, 0, 10, 10]
    assert torch.equal(got.out[:2], good[:2]) and torch.equal(got.out[4:6], good[4:6])
    table[0, :] = -1
    got = _check(kv, q, table, offsets, positions)
    assert got.status[0] == 10 and (got.out[:2] == 0).all()
    positions[2:4] = [(1 << 31) - 2, (1 << 31) - 1]
    got = _check(kv, q, table, offsets, positions)
    assert got.status[1] == 10
    got = G.cache_attend(q, kv, *(torch.from_numpy(x).cuda() for x in (table, np.array([0, 2, 1, 6, 99, -3], np.int32), positions)))
    assert got.status.tolist()[1] == 10 and got.status.tolist()[3:] == [10, 10]


def test_ends_of_the_range():
    g = _gen(6)
    bs, H, D = 8, 1, 64
    kv = _fill(g, 20, bs, H, D)
    rows = _rows(g, [150], [1], bs, 20, 20)
    q = torch.randn(1, 3, D, generator=g, device="cuda").to(torch.bfloat16)
    q[0, 1] = 0
    q[0, 2] *= 1e30
    _check(kv, q, *rows, scale=0.0)
    _check(kv, q, *rows, scale=1e-30)
    q[0, 2] = q[0, 0] * 2.0 ** -120
    _check(kv, q, *rows)
    _check(kv, q, *rows, scale=-0.3)
    _check(kv, q, *rows, scale=50.0)
    large = _fill(g, 20, bs, H, D, v_size=60000.0)
    _check(large, q, *rows)
    small = _fill(g, 20, bs, H, D, v_size=1e-3)
    _check(small, q, *rows)
    q[0, 0, 3] = float("nan")
    got = G.cache_attend(q, kv, *(torch.from_numpy(x).cuda() for x in rows)).out
    assert torch.isnan(got[0, 0]).all() and not torch.isnan(got[0, 1:]).any()


def test_strides():
    g = _gen(7)
    bs, H, D = 16, 2, 64
    kv = _fill(g, 30, bs, H, D)
    rows = _rows(g, [90, 33], [3, 2], bs, 8, 30)
    cuda = [torch.from_numpy(x).cuda() for x in rows]
    for shift in (0, 1, 4):
        row = torch.randn(5, 8 * D + 3 * D + 8, generator=g, device="cuda").to(torch.bfloat16)
        q = row[:, shift:shift + 8 * D].unflatten(1, (8, D))
        want = G.cache_attend(q.contiguous(), kv, *cuda)
        got = G.cache_attend(q, kv, *cuda)
        assert torch.equal(got.out, want.out)
        buf = torch.full((8, 5, D + shift), 2.0, dtype=torch.bfloat16, device="cuda")
        out = G.Attended(buf.transpose(0, 1)[:, :, shift:], got.status, got.workspace, got.shape)
        assert torch.equal(G.cache_attend(q, kv, *cuda, out=out).out, want.out) and (buf[:, :, :shift] == 2).all()
    # heads of a block's octets apart from the next block's
    wide = torch.zeros(30, kv.keys[0].numel() + 32, dtype=torch.uint8, device="cuda")
    wide[:, :kv.keys[0].numel()] = kv.keys.view(30, -1)
    apart = G.KVCache(wide[:, :kv.keys[0].numel()].view(30, *kv.keys.shape[1:]), None, bs, H, D)
    assert torch.equal(G.cache_attend(q, apart, *cuda).out, want.out)


def test_streams_and_graphs():
    """Two captured calls with workspaces of their own, replayed at the same time; the same results every time."""
    g = _gen(8)
    bs, H, D = 16, 4, 128
    kv = _fill(g, 400, bs, H, D)
    calls, kept = [], []                                   # (a graph reads its inputs where they were)
    for lengths, news in (([900, 20, 300], [1, 1, 1]), ([500, 1500], [5, 9])):
        rows = [torch.from_numpy(x).cuda() for x in _rows(g, lengths, news, bs, 100, 400)]
        q = torch.randn(sum(news), 4 * H, D, generator=g, device="cuda").to(torch.bfloat16)
        out = G.cache_attend(q, kv, *rows)
        want = out.out.clone()
        for _ in range(5):
            assert torch.equal(G.cache_attend(q, kv, *rows, out=out).out, want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            G.cache_attend(q, kv, *rows, out=out)
        calls.append((graph, out, want, torch.cuda.Stream()))
        kept.append((rows, q))
    for _ in range(20):
        for _, out, _, _ in calls:
            out.out.zero_()
        torch.cuda.synchronize()
        for graph, _, _, stream in calls:
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out.out, want) for _, out, want, _ in calls)


def test_nothing_to_do():
    kv = G.KVCache.empty(3, 8, 1, 64, torch.uint8)
    i32 = dict(dtype=torch.int32, device="cuda")
    q = torch.ones(2, 2, 64, dtype=torch.bfloat16, device="cuda")
    got = G.cache_attend(q, kv, torch.zeros(0, 4, **i32), torch.zeros(1, **i32), torch.zeros(2, **i32))
    assert (got.out == 0).all()
    got = G.cache_attend(q[:0], kv, torch.zeros(3, 4, **i32), torch.zeros(4, **i32), torch.zeros(0, **i32))
    assert got.status.tolist() == [0, 0, 0]
    got = G.cache_attend(q, kv, torch.zeros(2, 0, **i32), torch.arange(3, **i32), torch.zeros(2, **i32))
    assert (got.out == 0).all() and got.status.tolist() == [10, 10]
    empty = G.KVCache.empty(0, 8, 1, 64, torch.uint8)
    got = G.cache_attend(q, empty, torch.zeros(2, 1, **i32), torch.arange(3, **i32), torch.zeros(2, **i32))
    assert (got.out == 0).all() and got.status.tolist() == [10, 10]
    # a cache of zeros
    got = G.cache_attend(q, kv, torch.zeros(2, 1, **i32), torch.arange(3, **i32), torch.full((2,), 5, **i32))
    assert (got.out == 0).all() and got.status.tolist() == [0, 0]


def test_far_blocks():
    """A cache beyond 2^31 bytes, blocks at its end."""
    H, D, bs = 8, 128, 16
    N = (1 << 32) // (bs * H * 9 * D // 8) + 9
    kv = G.KVCache(torch.zeros(N, H, bs // 8, 9 * D, dtype=torch.uint8, device="cuda"), None, bs, H, D)
    near = _fill(_gen(9), 6, bs, H, D)
    kv.keys[-6:] = near.keys
    table = torch.tensor([[N - 6, N - 1, N - 3]], dtype=torch.int32, device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    q = torch.randn(1, 16, D, generator=_gen(10), device="cuda").to(torch.bfloat16)
    got = G.cache_attend(q, kv, table, torch.arange(2, **i32), torch.full((1,), 45, **i32))
    want = G.cache_attend(q, near, table - (N - 6), torch.arange(2, **i32), torch.full((1,), 45, **i32))
    assert torch.equal(got.out, want.out)


def test_a_step_of_decoding():
    """Rows of beams: planned, shared blocks copied, new tokens appended and attended over, twice, against the rows' own histories."""
    g = _gen(11)
    B, W, H, group, D, bs = 2, 3, 2, 4, 64, 8
    R = B * W
    tables = G.BlockTables.empty(R, 16, 120, bs, beams=W)
    kv = G.KVCache.empty(120, bs, H, D, torch.uint8)
    freq = 10000.0 ** (-torch.arange(0, D, 2, device="cuda", dtype=torch.float64) / D)
    history = [([], []) for _ in range(R)]                 # what each row's cache stands for, token by token
    counts = [[13, 13, 13, 29, 29, 29], [1] * R, [4] * R]
    parents = [None, [[0, 0, 2], [1, 1, 1]], [[2, 1, 0], [0, 2, 0]]]
    for count, parent in zip(counts, parents):
        append = torch.tensor(count, dtype=torch.int32, device="cuda")
        T = sum(count)
        to = None if parent is None else torch.tensor(parent, dtype=torch.int32, device="cuda")
        plan = G.block_plan(tables, append, T, parents=to)
        assert (plan.status == 0).all()
        G.copy_blocks(kv.tensors(), plan.copy_src, plan.copy_dst)
        if parent is not None:
            history = [tuple(list(x) for x in history[r // W * W + parent[r // W][r % W]]) for r in range(R)]
        k, v, q = (torch.randn(T, h, D, generator=g, device="cuda").to(torch.bfloat16) for h in (H, H, H * group))
        G.cache_append(kv, k, v, plan.slots, plan.positions, freq, q=q, q_out=q)
        rk, rv = G.cache_read(kv, plan.slots, torch.float32)
        out = G.cache_attend(q, kv, tables.table, plan.offsets, plan.positions)
        assert (out.status == 0).all()
        i = 0
        for r in range(R):
            for _ in range(count[r]):
                history[r][0].append(rk[i].double())
                history[r][1].append(rv[i].double())
                keys, values = (torch.stack(x).repeat_interleave(group, 1) for x in history[r])
                w = torch.softmax(torch.einsum("hd,thd->ht", q[i].double(), keys) * D ** -0.5, 1)
                want = torch.einsum("ht,thd->hd", w, values)
                # one rounding to bf16 (at 2^e and more numbers are 2^(e - 7) apart, so half of that, 2^-8 of the value, not 2^-9) and two of the
                # weights, 2^-12 each, taken up to 8 times a scale of at most |v| / 7
                assert (out.out[i].double() - want).abs().max() <= 2.0 ** -8 * want.abs().max() + 16 * 2.0 ** -12 * values.abs().max() / 7
                i += 1
