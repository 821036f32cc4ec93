"""gr_token_logprobs against log_softmax in 64 bits."""
import math

import pytest
import torch

import paper_2511_15898_b200 as G

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _zipf(g, R, V, dtype):
    x = -torch.log1p(torch.rand(R, V, generator=g, device="cuda") * V)
    return (x + 0.5 * torch.randn(R, V, generator=g, device="cuda")).to(dtype)


def _check(logits, tokens, top, T=1.0, rows=64):
    """Equal orders, and values within the roundings: with y the logits' distances from the largest in units of log 2 (at most one more from
    the reference) an exponential is off by 2^-22 and by ln 2 of y's error, 2 2^-24 |y| (its own rounding and that of the scale), sums of up to 13
    additions in 32 bits by 2^-24 each, the results by 2^-24 of themselves."""
    r = G.token_logprobs(logits, tokens, top, T)
    T = float(torch.tensor(T, dtype=torch.float32))
    for lo in range(0, logits.shape[0], rows):
        x = logits[lo:lo + rows].double() / T
        top_x = x.amax(1, keepdim=True)
        live = top_x[:, 0] > -math.inf
        lp = torch.where(live.view(-1, 1), torch.log_softmax(x, 1), -math.inf)
        p = torch.where(live.view(-1, 1), lp.exp(), 0)
        y = torch.where(p > 0, (top_x - x) / math.log(2), 0) + 1
        ey, ey2 = (p * y).sum(1), (p * y * y).sum(1)
        want = -torch.where(p > 0, p * lp, 0).sum(1)
        part = 2.0 ** -22 + 13 * 2.0 ** -24
        sum_off = part + 2 * math.log(2) * 2.0 ** -24 * ey + 1e-9
        off = (r.entropy[lo:lo + rows].double() - want).abs()
        bound = 2 * sum_off + math.log(2) * (part * ey + 2.0 ** -24 * (3 * ey + 2 * math.log(2) * ey2)) + 2.0 ** -24 * want
        assert (off <= bound).all(), (off - bound).max()

        def near(got, want):
            got = got.double()
            inf = torch.isinf(want.float())                # (beyond 32 bits: -infinity)
            assert torch.equal(torch.isinf(got), inf) and not torch.isnan(got).any()
            assert ((got - want).abs()[~inf] <= (sum_off.view(-1, 1) + 2.0 ** -24 * want.abs())[~inf]).all()

        if tokens is not None:
            t = tokens[lo:lo + rows].long()
            t = t.view(len(t), -1)
            some = (t >= 0) & (t < x.shape[1])
            near(r.logprob[lo:lo + rows], torch.where(some, lp.gather(1, t.clamp(0, x.shape[1] - 1)), -math.inf))
        if top:
            k = min(top, x.shape[1])
            order = torch.sort(logits[lo:lo + rows].float(), dim=1, descending=True, stable=True).indices[:, :k]
            best = lp.gather(1, order)
            some = best > -math.inf
            got = r.top_token[lo:lo + rows]
            assert torch.equal(got[:, :k].long(), torch.where(some, order, -1)) and (got[:, k:] == -1).all()
            near(r.top_logprob[lo:lo + rows][:, :k], best)
            assert (r.top_logprob[lo:lo + rows][:, k:] == -math.inf).all()
    assert (r.status == 0).all()
    return r


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R,V,given,top,T", [
    (1, 1, 1, 1, 1.0), (3, 2, 2, 5, 0.5), (5, 7, 1, 7, 1.0), (2, 100, 1, 0, 1.3), (4, 1023, 3, 20, 1.0), (3, 1025, 64, 128, 0.7),
    (1, 32000, 1, 5, 1.0), (2, 50257, 1, 128, 0.8), (9, 128256, 2, 20, 1.0), (20, 33001, 1, 1, 1.0), (40, 65541, 0, 10, 1.0), (300, 9001, 1, 0, 1.0),
    (700, 20011, 1, 48, 1.0), (1300, 5003, 2, 49, 0.7), (2500, 3001, 1, 8, 1.0), (1, 2097152, 1, 16, 1.0), (160, 152064, 1, 128, 1.0),
    (1300, 5003, 1, 8, 1.0),
])
def test_logprobs(R, V, given, top, T, dtype):
    g = _gen(R + V)
    logits = _zipf(g, R, V, DT[dtype])
    tokens = torch.randint(0, V, (R, given), generator=g, device="cuda", dtype=torch.int32) if given else None
    r = _check(logits, tokens, top, T, rows=max(1, (1 << 24) // V))
    again = G.token_logprobs(logits, tokens, top, T)
    assert all(torch.equal(getattr(r, n), getattr(again, n)) for n in ("logprob", "entropy", "top_token", "top_logprob"))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R,V", [(3, 500), (5, 40000), (400, 12000), (1300, 9000)])
def test_masks_and_ties(R, V, dtype):
    g = _gen(V)
    dt = DT[dtype]
    low = torch.finfo(dt).min
    base = _zipf(g, R, V, dt)
    tokens = torch.randint(0, V, (R, 3), generator=g, device="cuda", dtype=torch.int32)
    tokens[:, 2] = torch.where(torch.arange(R, device="cuda") % 2 == 0, -1, V).int()
    for mask in (-math.inf, low, -1e9):
        for share in (0.3, 0.999, 1.0):
            banned = torch.rand(R, V, generator=g, device="cuda") < share
            if share == 1.0:
                banned[1:, V // 2] = False                 # the first row is masked as a whole, the others but for one token
            _check(base.masked_fill(banned, mask), tokens, 16, rows=max(1, (1 << 22) // V))
    few = torch.randint(-3, 4, (R, V), generator=g, device="cuda").to(dt)
    _check(few, tokens, 100)
    _check(torch.full((R, V), -2.5, dtype=dt, device="cuda"), tokens, 128)
    _check(torch.where(torch.rand(R, V, generator=g, device="cuda") < 0.5, 0.0, -0.0).to(dt), tokens, 20)
    _check(base.sort(dim=1).values.contiguous(), tokens, 48)
    one = torch.full((R, V), -30.0, dtype=dt, device="cuda")
    one[:, V // 3] = 25.0
    r = _check(one, tokens, 2)
    assert (r.entropy >= 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sizes_of_logits_and_temperatures(dtype):
    g = _gen(3)
    logits = torch.randn(6, 9000, generator=g, device="cuda")
    tokens = torch.randint(0, 9000, (6, 2), generator=g, device="cuda", dtype=torch.int32)
    for scale, shift, T in ((1.0, 1000.0, 1.0), (1.0, -60000.0, 1.0), (100.0, 0.0, 1.0), (1.0, 0.0, 1e-3), (1.0, 0.0, 1e-20), (1e30, 0.0, 1.0), (1e30, 0.0, 1e30),
                            (1e-30, 0.0, 1e-35), (1.0, 0.0, 1e10), (1.0, 0.0, 3e38), (1.0, 0.0, 1e-38)):
        x = (logits * scale + shift).to(DT[dtype])
        # (where probabilities are those of the largest alone, 64 bits of log_softmax hold them as these calls do)
        _check(x, tokens, 4, T)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("R,V", [(6, 30000), (6, 150), (700, 5000)])
def test_bad_rows(R, V, dtype):
    g = _gen(4)
    logits = _zipf(g, R, V, DT[dtype])
    good = logits.clone()
    logits[1, V - 1], logits[2, 0], logits[4, V // 2] = float("nan"), float("inf"), float("nan")
    logits[5] = -math.inf
    good[5] = -math.inf
    logits[3, :] = -math.inf
    logits[3, 7] = float("nan")
    tokens = torch.randint(0, V, (R, 2), generator=g, device="cuda", dtype=torch.int32)
    r, want = G.token_logprobs(logits, tokens, 6), G.token_logprobs(good, tokens, 6)
    bad = torch.zeros(R, dtype=torch.bool, device="cuda")
    bad[1:5] = True
    assert torch.equal(r.status == G.GR_BAD_LOGITS, bad) and (r.status[~bad] == 0).all()
    assert torch.isnan(r.logprob[bad]).all() and torch.isnan(r.entropy[bad]).all() and (r.top_token[bad] == -1).all() and (r.top_logprob[bad] == -math.inf).all()
    for n in ("logprob", "entropy", "top_token", "top_logprob"):
        assert torch.equal(getattr(r, n)[~bad], getattr(want, n)[~bad])
    assert (r.logprob[5] == -math.inf).all() and r.entropy[5] == 0 and (r.top_token[5] == -1).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides_streams_and_graphs(dtype):
    g = _gen(5)
    wide = _zipf(g, 12, 5300, DT[dtype])
    tokens = torch.randint(0, 5001, (12,), generator=g, device="cuda", dtype=torch.int32)
    for shift in (0, 1, 2, 3, 8):
        x = wide[:, shift:shift + 5001]
        r, want = G.token_logprobs(x, tokens, 9, 0.9), G.token_logprobs(x.contiguous(), tokens, 9, 0.9)
        assert torch.equal(r.top_token, want.top_token) and r.logprob.shape == (12, 1)
        _check(x, tokens, 9, 0.9)
        _check(x[::3], tokens[::3].contiguous(), 9, 0.9)
    out = G.token_logprobs(x, tokens, 9)
    want = [t.clone() for t in (out.logprob, out.entropy, out.top_token, out.top_logprob)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        G.token_logprobs(x, tokens, 9, out=out)
    side = torch.cuda.Stream()
    for replay in (True, False):
        for t in (out.logprob, out.entropy, out.top_token, out.top_logprob):
            t.zero_()
        torch.cuda.synchronize()
        if replay:
            graph.replay()
        else:
            with torch.cuda.stream(side):
                G.token_logprobs(x, tokens, 9, out=out)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (out.logprob, out.entropy, out.top_token, out.top_logprob)))


def test_nothing_to_do():
    x = torch.randn(3, 50, device="cuda")
    r = G.token_logprobs(x[:0], None, 3)
    assert r.top_token.shape == (0, 3)
    r = G.token_logprobs(x)
    assert r.logprob.shape == (3, 0) and r.top_token.shape == (3, 0)
    p = torch.softmax(x.double(), 1)
    assert (r.entropy.double() + (p * p.log()).sum(1)).abs().max() < 1e-5


def test_rows_of_the_beam_selection():
    """A beam's continuations out of its row's likeliest: the same tokens, and totals that differ by the scores."""
    g = _gen(6)
    logits = _zipf(g, 8, 50257, torch.float32)
    scores = -torch.rand(8, 1, generator=g, device="cuda")
    beams = G.beam_select(logits.view(8, 1, -1), scores, 7, 0.8)
    r = G.token_logprobs(logits, beams.token, 7, 0.8)
    assert torch.equal(r.top_token, beams.token) and torch.equal(r.top_logprob, r.logprob)
    assert (beams.score.double() - scores.double() - r.logprob.double()).abs().max() < 1e-5
