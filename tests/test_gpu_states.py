"""Reordering of per-hypothesis states and copies of cache blocks on the GPU: every byte against plain indexing."""
import pytest
import torch

import paper_2511_15898_b200 as G
from paper_2511_15898_b200.build import build_library

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    build_library()


def expected(x, parents, lengths=None, token_dim=None, out=None):
    """What becomes of x (in place) or of out."""
    y = (x if out is None else out).clone()
    for b in range(parents.shape[0]):
        for j in range(parents.shape[1]):
            p = int(parents[b, j])
            if not 0 <= p < x.shape[1]:
                continue
            if lengths is None:
                y[b, j] = x[b, p]
            else:
                d = token_dim - 2
                n = min(max(int(lengths[b, p]), 0), x.shape[token_dim])
                y[b, j].narrow(d, 0, n).copy_(x[b, p].narrow(d, 0, n))
    return y


def same(a, b):
    kind = {1: torch.uint8, 2: torch.int16, 4: torch.int32, 8: torch.int64}[a.element_size()]
    return torch.equal(a.contiguous().view(kind), b.contiguous().view(kind))


def rand(shape, dtype, seed):
    g = torch.Generator(device="cuda"); g.manual_seed(seed)
    if dtype.is_floating_point:
        return torch.randn(shape, generator=g, device="cuda").to(dtype)
    return torch.randint(0, 100, shape, generator=g, device="cuda").to(dtype)


DTYPES = [torch.float32, torch.bfloat16, torch.float16, torch.uint8, torch.float64]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", [(1, 1, 1), (2, 3, 5), (1, 4, 1024), (3, 8, 7, 33), (2, 32, 129), (5, 17, 3, 16), (64, 2, 8),
                                   (2, 5, 40001), (1, 9, 4096)])
def test_whole_states_in_place(dtype, shape):
    x = [rand(shape, dtype, 10 + i) for i in range(3)]
    g = torch.Generator(device="cuda"); g.manual_seed(1)
    parents = torch.randint(-2, shape[1] + 1, shape[:2], generator=g, device="cuda", dtype=torch.int32)
    want = [expected(t, parents) for t in x]
    got = G.reorder_states(x, parents)
    torch.cuda.synchronize()
    assert all(a is b for a, b in zip(got, x)) and all(same(a, b) for a, b in zip(got, want))


def test_cycles_and_repeated_parents():
    for W in (2, 4, 7, 16, 31):
        x = rand((3, W, 1000), torch.float32, W)
        parents = torch.stack([(torch.arange(W) + 1) % W, torch.zeros(W, dtype=torch.long), torch.arange(W).flip(0)]).int().cuda()
        want = expected(x, parents)
        G.reorder_states([x], parents)
        assert same(x, want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.uint8])
@pytest.mark.parametrize("heads,tokens,width", [(1, 1, 1), (2, 7, 33), (8, 64, 128), (3, 100, 5), (1, 333, 250), (4, 16, 80)])
def test_used_tokens_only(dtype, heads, tokens, width):
    B, W = 4, 5
    g = torch.Generator(device="cuda"); g.manual_seed(heads + tokens)
    x = [rand((B, W, heads, tokens, width), dtype, i) for i in range(2)]
    parents = torch.randint(-1, W, (B, W), generator=g, device="cuda", dtype=torch.int32)
    lengths = torch.randint(-1, tokens + 3, (B, W), generator=g, device="cuda", dtype=torch.int32)
    want = [expected(t, parents, lengths, 3) for t in x]
    G.reorder_states(x, parents, lengths=lengths, token_dim=3)
    torch.cuda.synchronize()
    assert all(same(a, b) for a, b in zip(x, want))
    # tokens before the heads, and a number of chosen states of its own in other tensors
    y = [t.transpose(2, 3).contiguous() for t in x]
    chosen = torch.randint(-1, W, (B, 7), generator=g, device="cuda", dtype=torch.int32)
    out = [rand((B, 7, tokens, heads, width), dtype, 50 + i) for i in range(2)]
    want = [expected(t, chosen, lengths, 2, o) for t, o in zip(y, out)]
    before = [t.clone() for t in y]
    got = G.reorder_states(y, chosen, lengths=lengths, token_dim=2, out=out)
    torch.cuda.synchronize()
    assert all(a is b for a, b in zip(got, out)) and all(same(a, b) for a, b in zip(out, want))
    assert all(same(a, b) for a, b in zip(y, before))


def test_layouts():
    B, W = 3, 4
    parents = torch.tensor([[1, 0, 3, 2], [0, 0, 0, 0], [3, -1, 1, 1]], dtype=torch.int32, device="cuda")
    # slices of one buffer by layer and by kind, tensors of several types and shapes in one call, padded rows
    buf = rand((2, 2, B, W, 6, 10, 16), torch.bfloat16, 3)
    odd = rand((B, W, 11), torch.float32, 4)
    padded = rand((B, W, 3, 24), torch.float32, 5)[:, :, :, 1:20]
    inner = rand((B, 2, W, 12), torch.float32, 6)[:, 1]
    states = [buf[0, 0], buf[0, 1], buf[1, 0], buf[1, 1], odd, inner]
    want = [expected(t, parents) for t in states]
    everything = buf.clone()
    G.reorder_states(states, parents)
    torch.cuda.synchronize()
    assert all(same(a, b) for a, b in zip(states, want)) and not same(everything, buf)
    all19 = torch.full((B, W), 19, dtype=torch.int32, device="cuda")
    want = expected(padded, parents, all19, 3)
    G.reorder_states([padded], parents, lengths=all19, token_dim=3)
    assert same(padded, want)
    # a prompt's state given to all hypotheses
    prompt = rand((B, 1, 50), torch.float32, 7)
    out = [torch.zeros(B, W, 50, device="cuda")]
    G.reorder_states([prompt], torch.zeros(B, W, dtype=torch.int32, device="cuda"), out=out)
    assert same(out[0], prompt.expand(B, W, 50))
    out = [torch.zeros(B, W, 50, device="cuda")]
    G.reorder_states([prompt.expand(B, 9, 50)], torch.full((B, W), 8, dtype=torch.int32, device="cuda"), out=out)
    assert same(out[0], prompt.expand(B, W, 50))
    # no bytes beside the states' own: every second beam of a larger buffer
    big = rand((B, 2 * W, 33), torch.float32, 8)
    keep = big.clone()
    half = big[:, ::2]
    want = expected(half, parents)
    G.reorder_states([half], parents)
    assert same(half, want) and same(big[:, 1::2], keep[:, 1::2])


def test_more_states_than_one_launch_takes():
    x = [rand((2, 3, 5), torch.float32, i) for i in range(300)]
    parents = torch.tensor([[2, 0, 1], [1, 1, 1]], dtype=torch.int32, device="cuda")
    want = [expected(t, parents) for t in x]
    G.reorder_states(x, parents)
    assert all(same(a, b) for a, b in zip(x, want))


def test_offsets_beyond_32_bits():
    # states of 2.2 GB: the second hypothesis begins beyond 2^31 bytes
    n = 2_200_000_016
    x = torch.zeros(1, 2, n, dtype=torch.uint8, device="cuda")
    x[0, 1, -100:] = torch.arange(100, device="cuda", dtype=torch.uint8)
    x[0, 0, :50] = 7
    G.reorder_states([x], torch.tensor([[1, 0]], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert x[0, 0, -100:].tolist() == list(range(100)) and x[0, 1, :50].tolist() == [7] * 50
    assert int(x[0, 0, :-100].max()) == 0 and int(x[0, 1, 50:].max()) == 0
    # and a pool of 4.4 GB
    pool = x.view(4, -1)
    G.copy_blocks([pool], torch.tensor([1, -1, 4], dtype=torch.int32, device="cuda"),
                  torch.tensor([3, 0, 2], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert pool[3, -100:].tolist() == list(range(100)) and int(pool[3, :-100].max()) == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.uint8])
@pytest.mark.parametrize("blocks,shape,pairs", [(1, (4,), 1), (9, (1,), 4), (40, (3, 5), 17), (600, (16, 33), 280), (64, (8, 16, 128), 20),
                                               (2000, (40,), 900)])
def test_copied_blocks(dtype, blocks, shape, pairs):
    caches = [rand((blocks,) + shape, dtype, i) for i in range(3)]
    g = torch.Generator(device="cuda"); g.manual_seed(blocks)
    order = torch.randperm(blocks, generator=g, device="cuda").int()
    half = max(1, min(pairs, blocks // 2))
    dst = torch.full((pairs,), -1, dtype=torch.int32, device="cuda")
    src = dst.clone()
    dst[:half] = order[:half]
    if blocks > half:
        src[:half] = order[half:][torch.randint(0, blocks - half, (half,), generator=g, device="cuda")]
    src[3:half:3] = -1
    if pairs > 3:
        src[1], dst[2] = blocks + 5, -7        # outside the pool: skipped
    want = [c.clone() for c in caches]
    for a, b in zip(src.tolist(), dst.tolist()):
        if 0 <= a < blocks and 0 <= b < blocks:
            for c, w in zip(caches, want):
                w[b] = c[a]
    G.copy_blocks(caches, src, dst)
    torch.cuda.synchronize()
    assert all(same(a, b) for a, b in zip(caches, want))


def test_caches_within_a_larger_buffer():
    buf = rand((2, 30, 2, 64), torch.float32, 1)     # [kind, block, half, element]: a cache is one half of the blocks
    keep = buf.clone()
    src = torch.tensor([3, -1, 5], dtype=torch.int32, device="cuda")
    dst = torch.tensor([9, 2, 0], dtype=torch.int32, device="cuda")
    G.copy_blocks([buf[0, :, 1], buf[1, :, 0]], src, dst)
    keep[0, 9, 1] = keep[0, 3, 1]; keep[0, 0, 1] = keep[0, 5, 1]
    keep[1, 9, 0] = keep[1, 3, 0]; keep[1, 0, 0] = keep[1, 5, 0]
    torch.cuda.synchronize()
    assert same(buf, keep)


def test_in_a_graph_and_on_another_stream():
    x = rand((4, 4, 2000), torch.bfloat16, 1)
    parents = torch.randint(0, 4, (4, 4), device="cuda", dtype=torch.int32)
    start = x.clone()
    G.reorder_states([x], parents)
    torch.cuda.synchronize()
    x.copy_(start)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        G.reorder_states([x], parents)
    for k in range(3):
        parents.copy_(torch.randint(-1, 4, (4, 4), device="cuda", dtype=torch.int32))
        want = expected(x, parents)
        graph.replay()
        torch.cuda.synchronize()
        assert same(x, want)
    side = torch.cuda.Stream()
    want = expected(x, parents)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        G.reorder_states([x], parents)
    side.synchronize()
    assert same(x, want)


def test_outs_that_meet_the_states_and_repeats_are_refused():
    x = rand((2, 8, 64), torch.float32, 1)
    parents = torch.zeros(2, 4, dtype=torch.int32, device="cuda")
    keep = x.clone()
    with pytest.raises(G.GrError):
        G.reorder_states([x], parents, out=[x[:, 4:]])
    with pytest.raises(G.GrError):
        G.reorder_states([x, x], torch.zeros(2, 8, dtype=torch.int32, device="cuda"))
    odd = rand((2, 8, 10), torch.float32, 2)
    with pytest.raises(G.GrError):
        G.reorder_states([x, odd, x], torch.zeros(2, 8, dtype=torch.int32, device="cuda"))
    with pytest.raises(G.GrError):
        G.reorder_states([x, odd], parents, out=[torch.empty(2, 4, 64, device="cuda"), odd[:, :4]])
    with pytest.raises(G.GrError):
        G.reorder_states([x], torch.zeros(2, 9, dtype=torch.int32, device="cuda"))
    with pytest.raises(G.GrError):
        G.copy_blocks([x[0], x[0]], parents[0], parents[1])
    torch.cuda.synchronize()
    assert same(x, keep)
    # halves of one buffer do not meet
    buf = rand((2, 2, 4, 33), torch.float32, 3)
    G.reorder_states([buf[0]], parents, out=[buf[1]])
    torch.cuda.synchronize()
    assert same(buf[1], buf[0][:, :1].expand(2, 4, 33))
