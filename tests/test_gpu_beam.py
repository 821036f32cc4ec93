"""Beam search's selection on the GPU against its definition in 64 bits: order, scores, lengths and finished flags over
types, odd sizes, masks, ties, strides, split rows, and the rows whose sums are taken again."""
import math

import pytest
import torch

import paper_2511_15898_b200 as G
from paper_2511_15898_b200.build import build_library

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    build_library()


def reference(logits, scores, K, T=1.0, lengths=None, done=None, eos=-1, penalty=0.0):
    """Of every group: (unusable, number of continuations, and of the K best their totals, parents, tokens, flags, lengths)."""
    B, W, V = logits.shape
    x = logits.double().cpu() / float(torch.tensor(T, dtype=torch.float32))
    pen = float(torch.tensor(penalty, dtype=torch.float32))
    out = []
    for b in range(B):
        key, tot, at, tok, fin, ln = [], [], [], [], [], []
        bad = False
        for w in range(W):
            s = float(scores[b, w])
            if s == -math.inf:
                continue
            if not s < math.inf:
                bad = True
                continue
            n = int(lengths[b, w]) if lengths is not None else 0
            if done is not None and bool(done[b, w]):
                t, v, f, n = torch.tensor([s], dtype=torch.float64), torch.tensor([eos]), True, max(1, n)
            else:
                if bool((~(x[b, w] < math.inf)).any()):
                    bad = True
                    continue
                v = torch.nonzero(x[b, w] > -math.inf).view(-1)
                t = s + (x[b, w][v] - torch.logsumexp(x[b, w][v], 0)) if len(v) else torch.empty(0, dtype=torch.float64)
                f, n = False, max(1, n + 1)
                # (within a row the order is that of the logits: a difference that the sum rounds away still counts)
                o = torch.sort(x[b, w][v], descending=True, stable=True).indices[:K]
                v, t = v[o], t[o]
            key.append(t / float(n) ** pen); tot.append(t); tok.append(v)
            at.append(torch.full_like(v, w)); fin.append((v == eos) | f); ln.append(torch.full_like(v, n))
        if bad or not key:
            out.append((bad, 0))
            continue
        key, tot, at, tok, fin, ln = (torch.cat(z) for z in (key, tot, at, tok, fin, ln))
        o = torch.sort(key, descending=True, stable=True).indices[:K]
        out.append((False, len(o), tot[o], at[o], tok[o], fin[o], ln[o]))
    return out


def check(r, want, K, V, lengths=None):
    torch.cuda.synchronize()
    # scores: one rounding to fp32, and the streamed sum's error: ex2 2^-22, two FMAs of 2^-24 |y| each with a mean |y| of at
    # most log2 V + 1 under the softmax, fp32 sums of up to 16 terms
    lse = 2.0 ** -22 + math.log(2) * 2.0 ** -23 * (math.log2(max(V, 2)) + 1) + 16 * 2.0 ** -24
    for b, ref in enumerate(want):
        bad, n = ref[0], ref[1]
        assert int(r.status[b]) == (G.GR_BAD_LOGITS if bad else G.GR_OK), b
        if n:
            assert r.parent[b, :n].tolist() == ref[3].tolist(), b
            assert r.token[b, :n].tolist() == ref[4].tolist(), b
            assert r.done[b, :n].tolist() == ref[5].tolist(), b
            if lengths is not None:
                assert r.length[b, :n].tolist() == ref[6].tolist(), b
            got = r.score[b, :n].double().cpu()
            assert bool(((got - ref[2]).abs() <= lse + 2.0 ** -24 * ref[2].abs()).all()), (b, got - ref[2])
        assert r.token[b, n:].tolist() == [-1] * (K - n) and r.parent[b, n:].tolist() == [-1] * (K - n)
        assert bool((r.score[b, n:] == -math.inf).all()) and not bool(r.done[b, n:].any())
        assert r.length[b, n:].tolist() == [0] * (K - n)


def make(B, W, V, dtype, seed, spread=3.0):
    g = torch.Generator(device="cuda"); g.manual_seed(seed)
    x = (spread * torch.randn(B, W, V, generator=g, device="cuda")).to(dtype)
    s = -5.0 - 3.0 * torch.rand(B, W, generator=g, device="cuda")
    return x, s, g


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,W,V,K", [(1, 1, 1, 1), (2, 1, 1, 3), (3, 2, 5, 10), (1, 4, 17, 8), (2, 3, 257, 5), (5, 4, 1000, 8),
                                     (2, 32, 1025, 64), (1, 7, 2047, 14), (1, 5, 2049, 128), (3, 4, 4099, 16), (70, 9, 8191, 18),
                                     (1, 4, 32000, 8), (2, 6, 50257, 12), (40, 8, 16385, 16), (1, 32, 32001, 128),
                                     (300, 4, 1031, 4), (1, 1, 151936, 50)])
def test_sizes(dtype, B, W, V, K):
    x, s, _ = make(B, W, V, dtype, 11 * V + K)
    check(G.beam_select(x, s, K), reference(x, s, K), K, V)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,W,V,K", [(90, 7, 4099, 10), (150, 8, 5003, 16), (60, 20, 2053, 48), (60, 20, 2053, 49), (1, 32, 1027, 32),
                                     (600, 5, 1029, 10), (25, 24, 9001, 40), (1200, 1, 3001, 5)])
def test_numbers_of_rows(dtype, B, W, V, K):
    """Few rows, one wave of CTAs and several, by the larger CTAs and the smaller ones."""
    x, s, _ = make(B, W, V, dtype, B + V)
    check(G.beam_select(x, s, K), reference(x, s, K), K, V)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,W", [(700, 1), (160, 8), (40, 3)])
def test_ties_masks_and_order_among_many_rows(dtype, B, W):
    V, K = 6001, 12
    x, s, g = make(B, W, V, dtype, B)
    x[0] = 1.5                                             # nothing but ties
    x[1, :, 9:] = torch.finfo(dtype).min                   # fewer tokens than are asked for beside the masked ones
    x[2] = x[2].sort(dim=1).values
    x[3, :, 5:] = -math.inf
    x[4] = -math.inf
    x[5, 0] = x[5, 0].sort(descending=True).values
    x[6] = torch.round(x[6])                               # many ties at the border
    s[7] = -math.inf
    x[8, W - 1, V - 1] = math.nan
    x[9, :, 1:4] = 40.0                                    # peaks
    check(G.beam_select(x, s, K), reference(x, s, K), K, V)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,W,V,K,ld", [(1, 1, 40000, 8, 40000), (3, 2, 20011, 40, 20013), (700, 1, 9001, 5, 9001), (2, 4, 70001, 128, 70002)])
def test_more_ties_than_are_listed(dtype, B, W, V, K, ld):
    low = torch.finfo(dtype).min
    g = torch.Generator(device="cuda").manual_seed(V)
    x = torch.randn(B * W, ld, device="cuda", generator=g).to(dtype)[:, :V]
    r = 0

    def row():
        nonlocal r
        r += 1
        return x[(r - 1) % (B * W)]

    row()[K - 2:] = low                                    # fewer unmasked tokens than are asked for: the first masked ones follow
    y = row(); y[:V - 3] = low                             # ... at the end of the row
    y = row(); y[:] = -10000.5; y[V // 2] = 1.0            # another value than the type's lowest
    y = row(); y[:] = -math.inf; y[V // 3:] = -1e9; y[V - 1] = 2.0
    y = row(); y[:] = 0.0; y[1::2] = -0.0                  # the two zeros are one value
    y = row(); y[:] = torch.round(y * 0.5)                 # few values in all
    # a few threads meet all that is above the others' values (vectors that lie a warp apart)
    n = 4 if dtype == torch.float32 else 8
    y = row(); y[:] = 0.0
    for i in range(n):
        z = y[i::32 * n]
        z.copy_(torch.randn(z.shape, device="cuda", generator=g).abs() + 1)
    s = torch.zeros(B, W, device="cuda")
    full = torch.as_strided(x, (B, W, V), (W * ld, ld, 1))
    check(G.beam_select(full, s, K), reference(full, s, K), K, V)


@pytest.mark.parametrize("T", [0.3, 0.7, 1.0, 2.5])
def test_temperature_and_penalty(T):
    for penalty in (0.0, 0.6, 1.0, -0.5, 32.0):
        x, s, g = make(4, 5, 5003, torch.float32, 77)
        n = torch.randint(0, 50, (4, 5), generator=g, device="cuda", dtype=torch.int32)
        done = torch.rand(4, 5, generator=g, device="cuda") < 0.3
        r = G.beam_select(x, s, 10, T, lengths=n, done=done, eos=3, length_penalty=penalty)
        check(r, reference(x, s, 10, T, n, done, 3, penalty), 10, 5003, n)


def test_finished_and_absent_hypotheses_are_not_read():
    x, s, _ = make(3, 4, 6007, torch.float32, 5)
    done = torch.zeros(3, 4, dtype=torch.uint8, device="cuda")
    done[0, 1] = 1; done[1] = 1
    s[2, 1:] = -math.inf                       # the first step: one hypothesis
    clean = x.clone()
    x[0, 1] = math.nan; x[1] = math.inf; x[2, 2] = math.nan
    r = G.beam_select(x, s, 8, done=done, eos=6006)
    check(r, reference(clean, s, 8, done=done, eos=6006), 8, 6007)
    s[:] = -math.inf
    check(G.beam_select(x, s, 8), reference(clean, s, 8), 8, 6007)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [300, 5003, 40001])
def test_masks(dtype, V):
    x, s, g = make(6, 3, V, dtype, V)
    keep = torch.zeros(V, dtype=torch.bool, device="cuda")
    keep[torch.randperm(V, generator=g, device="cuda")[:40]] = True
    x[0, :, ~keep] = -math.inf                 # few tokens left
    x[1, 1] = -math.inf                        # a row without any
    x[2] = -math.inf                           # a group without any
    x[3, :, ~keep] = torch.finfo(dtype).min    # masked by the type's lowest value: still continuations, the last ones
    x[4, 0] = torch.finfo(dtype).min           # ... a whole row of it is a uniform one
    x[5, :, 7:] = -math.inf
    check(G.beam_select(x, s, 24), reference(x, s, 24), 24, V)


@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_unusable_rows(value):
    x, s, _ = make(4, 3, 9001, torch.float32, 3)
    for b, w, v in ((0, 0, 0), (1, 2, 9000), (2, 1, 4500)):
        x[b, w, v] = value
    r = G.beam_select(x, s, 6)
    check(r, reference(x, s, 6), 6, 9001)
    assert r.status.tolist() == [3, 3, 3, 0]
    x, s, _ = make(2, 3, 100, torch.bfloat16, 3)
    s[0, 1] = value
    assert G.beam_select(x, s, 6).status.tolist() == [3, 0]


def test_ties_go_to_the_lower_beam_and_token():
    # equal rows that begin at different alignments, equal logits within a row
    for V in (401, 4099, 20001):
        x = torch.full((2, 5, V), -1.0, device="cuda")
        x[1, :, ::2] = 2.5
        s = torch.full((2, 5), -3.0, device="cuda")
        check(G.beam_select(x, s, 12), reference(x, s, 12), 12, V)
        y, _, _ = make(1, 1, V, torch.float32, 9)
        y = y.expand(1, 6, V).contiguous()
        s = torch.full((1, 6), -3.0, device="cuda")
        check(G.beam_select(y, s, 16), reference(y, s, 16), 16, V)


def test_scores_that_nearly_tie_are_ordered_by_their_64_bit_values():
    # rows that differ in one unlikely logit, whose sums differ by 1e-9 to 1e-7
    B, W, V = 40, 4, 3001
    g = torch.Generator(device="cuda"); g.manual_seed(8)
    x = torch.randn(B, 1, V, generator=g, device="cuda").expand(B, W, V).contiguous()
    for w in range(W):
        x[:, w, 17] = -9.0 - 3.0 * torch.rand(B, generator=g, device="cuda")
    s = torch.full((B, W), -2.0, device="cuda")
    check(G.beam_select(x, s, 16), reference(x, s, 16), 16, V)


def test_large_offsets_and_spreads():
    x, s, _ = make(2, 3, 7001, torch.float32, 21)
    for scale, shift in ((1.0, 1000.0), (1e4, 0.0), (1e30, 0.0), (1e38 / 20, 0.0), (1e-30, 0.0), (1.0, -3e4)):
        y = x * scale + shift
        check(G.beam_select(y, s, 9), reference(y, s, 9), 9, 7001)


@pytest.mark.parametrize("T", [1e-30, 1e-3, 1e6, 1e37, 3e38])
def test_extreme_temperatures_and_masks(T):
    # (half of the tokens masked: a product with -infinity, or with a mask clamped to a number, must not count)
    for dtype in (torch.float32, torch.bfloat16):
        x, s, _ = make(3, 4, 3001, dtype, 15)
        x[:, :, ::2] = -math.inf
        x[1, 2] = -math.inf
        x[2, 3, 1] = torch.finfo(dtype).max
        check(G.beam_select(x, s, 9, T), reference(x, s, 9, T), 9, 3001)
        # the same with rows whose sums are taken again
        s[:] = -2.0
        x[:, 1] = x[:, 0]
        check(G.beam_select(x, s, 9, T), reference(x, s, 9, T), 9, 3001)


def test_ascending_rows_and_long_lists():
    for dtype in (torch.float32, torch.bfloat16):
        x, s, _ = make(2, 3, 60001, dtype, 4)
        x = x.sort(dim=2).values.contiguous()
        check(G.beam_select(x, s, 64), reference(x, s, 64), 64, 60001)


def test_rows_at_any_distance():
    # the last position of every sequence's logits, without a copy; rows that do not begin on 16 bytes
    g = torch.Generator(device="cuda"); g.manual_seed(2)
    for dtype, V in ((torch.float32, 1003), (torch.bfloat16, 5001)):
        full = torch.randn(3, 4, 5, V, generator=g, device="cuda").to(dtype)
        x = full.view(12, 5, V)[:, 2].view(3, 4, V)
        s = -torch.rand(3, 4, generator=g, device="cuda")
        assert not x.is_contiguous()
        check(G.beam_select(x, s, 8), reference(x, s, 8), 8, V)
        padded = torch.randn(2, 3, V + 5, generator=g, device="cuda").to(dtype)[:, :, 3:V + 3]
        check(G.beam_select(padded, s[:2, :3].contiguous(), 6), reference(padded, s[:2, :3], 6), 6, V)


def test_results_written_again_another_stream_and_a_graph():
    x, s, _ = make(4, 4, 3001, torch.float32, 31)
    y, t, _ = make(4, 4, 3001, torch.float32, 32)
    out = G.beam_select(x, s, 8)
    first = out.token.clone()
    again = G.beam_select(y, t, 8, out=out)
    assert again is out
    check(out, reference(y, t, 8), 8, 3001)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        r = G.beam_select(x, s, 8)
    side.synchronize()
    assert torch.equal(r.token, first)
    static = x.clone()
    G.beam_select(static, s, 8, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        G.beam_select(static, s, 8, out=out)
    static.copy_(y)
    graph.replay()
    check(out, reference(y, s, 8), 8, 3001)
    static.copy_(x)
    graph.replay()
    check(out, reference(x, s, 8), 8, 3001)


def test_same_inputs_give_the_same_bits():
    x, s, _ = make(3, 8, 50257, torch.float32, 41)
    a, b = G.beam_select(x, s, 16), G.beam_select(x, s, 16)
    torch.cuda.synchronize()
    assert torch.equal(a.score, b.score) and torch.equal(a.token, b.token)
