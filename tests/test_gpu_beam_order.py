"""The order between hypotheses whose keys are equal or nearly so: on rows whose streamed sums err most and each in its own way
(rows of one value or of two, where every element has the same error), next to one another at a distance of a few units of a score."""
import math

import pytest
import torch

import paper_2511_15898_b200 as G
from paper_2511_15898_b200.build import build_library
from tests.test_gpu_beam import check, reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    build_library()


@pytest.mark.parametrize("penalty", [1.0, 2.0, 0.5, 1.5, -1.0])
def test_equal_quotients_are_equal_keys(penalty):
    """Finished hypotheses of totals -c L^a: all keys are -c, the lower hypothesis comes first."""
    g = torch.Generator().manual_seed(3)
    B, W, V = 24, 32, 300
    n = torch.randint(1, 200, (B, W), generator=g, dtype=torch.int32)
    n[0, :2] = torch.tensor([49, 1])
    n[1:12] = torch.randint(1, 13, (11, W), generator=g, dtype=torch.int32) ** 2
    c = 2.0 ** torch.randint(-3, 4, (B, 1), generator=g)
    if penalty != int(penalty):
        n[0], n[12:] = 4, n[12:].clamp(max=14) ** 2        # (squares: the power is a whole number)
    if penalty < 0:
        n = 2 ** (n % 12)                                  # (and a fraction that fp32 holds)
    s = (-c * n.double() ** penalty).float()
    assert torch.equal(s.double() / n.double() ** penalty, -c.double().expand(B, W))
    x = torch.zeros(B, W, V, device="cuda")
    done = torch.ones(B, W, dtype=torch.bool, device="cuda")
    n, s = n.int().cuda(), s.cuda()
    r = G.beam_select(x, s, W, lengths=n, done=done, eos=2, length_penalty=penalty)
    torch.cuda.synchronize()
    assert torch.equal(r.parent.cpu(), torch.arange(W, dtype=torch.int32).expand(B, W))
    check(r, reference(x, s, W, 1.0, n, done, 2, penalty), W, V, n)


def near_scores(x, T, g):
    """Scores that bring the best continuations of a group's rows within a few units in the last place of one another."""
    B, W, _ = x.shape
    s = torch.empty(B, W, dtype=torch.float32)
    for b in range(B):
        y = x[b].double().cpu() / T
        best = y.amax(1) - torch.logsumexp(y, 1)
        t = float(best.min()) - 0.0625
        for w in range(W):
            near = torch.tensor(t - float(best[w]), dtype=torch.float32)
            unit = float(torch.nextafter(near, torch.tensor(math.inf))) - float(near)
            s[b, w] = float(near) + unit * int(torch.randint(-3, 4, (1,), generator=g))
    return s.cuda()


def check_order(r, x, s, K, T=1.0, lengths=None, done=None, eos=-1, penalty=0.0):
    """The K largest keys in descending order, each row's tokens in the order of the logits.  Two orders of a pair count where its
    keys are one number but for the roundings of 64-bit arithmetic, which rows of one value shifted against one another make happen:
    x / T, score and log-sum are each rounded a few times (of 2^-53 of themselves), the sum of exponentials by its additions in halves
    and by its terms (each off by its exponent's rounding); 32 units of the largest of them together bound both sides."""
    torch.cuda.synchronize()
    B, W, V = x.shape
    y = x.double() / T
    total = s.double().unsqueeze(2) + (y - torch.logsumexp(y, 2, keepdim=True))
    length = (lengths.double() + 1 if lengths is not None else torch.ones(B, W, device="cuda", dtype=torch.float64))
    if done is not None:
        total[done] = -math.inf
        total[done, eos] = s[done].double()
        length = length - done.double()
    key = total / (length.clamp(min=1) ** float(torch.tensor(penalty, dtype=torch.float32))).unsqueeze(2)
    tol = 32 * 2.0 ** -53 * (float(y.abs().max()) + float(s.abs().max()) + math.log2(V))
    assert tol < 1e-11                                    # (the keys differ by units of fp32 scores, 1e-9 and more, or not at all)
    at = r.parent.long() * V + r.token.long()
    assert r.status.tolist() == [G.GR_OK] * B and int(r.parent.min()) >= 0
    flat = key.view(B, -1)
    got = flat.gather(1, at)
    assert bool((got[:, 1:] <= got[:, :-1] + tol).all())
    others = flat.scatter(1, at, -math.inf).amax(1)
    assert bool((others <= got[:, -1] + tol).all())
    # of each row the tokens that the logits' order begins with
    order = x.sort(dim=2, descending=True, stable=True).indices[:, :, :K]
    for b in range(B):
        parents, tokens = r.parent[b].tolist(), r.token[b].tolist()
        for w in set(parents):
            mine = [t for p, t in zip(parents, tokens) if p == w]
            assert mine == ([eos] if done is not None and bool(done[b, w]) else order[b, w, :len(mine)].tolist())


def test_two_plateaus():
    V = 131072
    x = torch.empty(1, 2, V, device="cuda")
    x[0, 0], x[0, 1] = -8.875, -11.625
    x[:, :, ::512] = 0.0
    s = torch.tensor([[-0.0625, -0.12696360051631927]], device="cuda")
    want = reference(x, s, 16)
    assert want[0][3].tolist() == [0] * 16                # (ahead by 8.5e-8)
    check(G.beam_select(x, s, 16), want, 16, V)


# (few CTAs, one wave, several waves of the smaller CTAs)
SHAPES = [(1, 4, 131072), (3, 8, 20011), (40, 4, 30001), (40, 32, 2053), (330, 8, 4099)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,W,V", SHAPES)
def test_rows_of_two_values(dtype, B, W, V):
    g = torch.Generator().manual_seed(V + B)
    x = torch.empty(B, W, V)
    for b in range(B):
        for w in range(W):
            x[b, w] = -16.0 * float(torch.rand(1, generator=g))
            x[b, w, int(torch.randint(0, 7, (1,), generator=g))::int(torch.randint(200, 700, (1,), generator=g))] = float(torch.randn(1, generator=g))
    x = x.to(dtype).cuda()
    s = near_scores(x, 1.0, g)
    check_order(G.beam_select(x, s, 2 * W), x, s, 2 * W)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [0.5, 1.0, 1.75])
@pytest.mark.parametrize("B,W,V", SHAPES)
def test_rows_of_one_value(dtype, T, B, W, V):
    g = torch.Generator().manual_seed(V + W)
    x = (10.0 * torch.randn(B, W, 1, generator=g)).expand(B, W, V).to(dtype).cuda()
    s = near_scores(x, T, g)
    # (every row's best tokens tie; the first token alone stands for the row's place)
    x[:, :, V // 2] += 1.0
    s2 = near_scores(x, T, g)
    check_order(G.beam_select(x, s2, W, T), x, s2, W, T)
    x[:, :, V // 2] = x[:, :, 0]
    check_order(G.beam_select(x, s, W, T), x, s, W, T)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,W,V", SHAPES[1:])
def test_penalties_and_finished_hypotheses(dtype, B, W, V):
    g = torch.Generator().manual_seed(B + W)
    x = (10.0 * torch.randn(B, W, 1, generator=g)).expand(B, W, V).to(dtype).cuda()
    x[:, :, 5] += 3.0
    for penalty in (1.0, 0.6):
        n = torch.randint(0, 40, (B, W), generator=g, dtype=torch.int32)
        done = torch.rand(B, W, generator=g) < 0.4
        y = x.double().cpu()
        best = y.amax(2) - torch.logsumexp(y, 2)
        length = torch.where(done, n, n + 1).clamp(min=1).double()
        # keys next to one another: total = key L^a
        s = (-15.0 * length ** float(torch.tensor(penalty, dtype=torch.float32)) - torch.where(done, 0.0, best)).float()
        s = torch.where(torch.rand(B, W, generator=g) < 0.5, s, torch.nextafter(s, torch.tensor(0.0))).cuda()
        n, done = n.cuda(), done.cuda()
        K = min(W + 3, int((~done).sum(1).min()) * V + 1)
        check_order(G.beam_select(x, s, K, lengths=n, done=done, eos=9, length_penalty=penalty), x, s, K, 1.0, n, done, 9, penalty)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_long_lists_in_many_groups(dtype):
    """As many groups as leave what they cannot tell apart to clusters, with the longest lists there are, beside groups without a doubt
    and groups that are of no use."""
    B, W, V, K = 90, 32, 1500, 128
    g = torch.Generator().manual_seed(6)
    x = (10.0 * torch.randn(B, W, 1, generator=g)).expand(B, W, V).to(dtype)
    x = x + torch.randn(B, W, V, generator=g).to(dtype) * (torch.arange(B) % 3 == 0).view(B, 1, 1)
    x = x.cuda()
    s = near_scores(x, 1.0, g)
    x[7, 3, 11] = math.nan
    s[8] = -math.inf
    x[9] = 1e32 * (1 + torch.rand(W, V, generator=g).to(dtype).cuda())
    r = G.beam_select(x, s, K)
    want = torch.tensor([G.GR_OK] * B)
    want[7] = G.GR_BAD_LOGITS
    assert torch.equal(r.status.cpu().long(), want)
    assert r.token[7:9].unique().tolist() == [-1] and r.parent[7:9].unique().tolist() == [-1]
    good = [b for b in range(B) if b not in (7, 8, 9)]

    def part(rows):
        return type(r)(*[getattr(r, n)[rows] for n in ("token", "parent", "score", "length", "done", "status")], r.workspace, r.shape)

    check_order(part(good), x[good], s[good], K)
    one, t = x[9:10].contiguous(), s[9:10].contiguous()
    for got in (part([9]), G.beam_select(one, t, K)):
        check(got, reference(one, t, K), K, V)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_totals_whose_units_are_larger_than_the_errors_of_sums(dtype):
    """Totals of -1e11, which 64 bits hold to 1.5e-5: rows of equal log-probabilities tie, though an error of 1e-7 may carry one of them
    to the next number."""
    B, W, V = 400, 8, 3001
    g = torch.Generator().manual_seed(9)
    x = (torch.randint(-64, 65, (B, W, 1), generator=g) / 8.0).expand(B, W, V).contiguous()
    x[:, :, V // 3] += torch.randint(4, 40, (B, 1), generator=g) / 8.0
    if dtype == torch.float32:
        x[:, :, V // 3] += torch.randint(0, 1024, (B, 1), generator=g) / 8192.0
    y = x.to(dtype)
    assert torch.equal(y.float(), x)
    y, s = y.cuda(), torch.full((B, W), -1e11, device="cuda")
    r = G.beam_select(y, s, W)
    torch.cuda.synchronize()
    assert torch.equal(r.parent.cpu(), torch.arange(W, dtype=torch.int32).expand(B, W))
    assert r.token.unique().tolist() == [V // 3]
