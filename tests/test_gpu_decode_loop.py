"""The operators around a decoding step in a loop, as a serving loop runs them: a beam search whose caches are reordered
densely and through block tables, against one that keeps whole sequences; and multi-draft verification whose accepted
drafts' states and cache entries stay while the others are dropped."""
import math

import pytest
import torch

import paper_2511_15898_b200 as G
from paper_2511_15898_b200 import workloads as W
from paper_2511_15898_b200.build import build_library

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    build_library()


class Toy:
    """A model whose logits depend on every token that came before, through a cache entry for each."""

    def __init__(self, V, D, seed):
        g = torch.Generator(device="cuda"); g.manual_seed(seed)
        self.V, self.D = V, D
        self.entry = torch.randn(V, D, generator=g, device="cuda")
        self.out = torch.randn(D, V, generator=g, device="cuda")
        self.decay = 0.8

    def logits(self, cache, length):
        """cache [rows, T, D], length [rows]: a weighted sum of the entries, the latest weighing most."""
        t = torch.arange(cache.shape[1], device="cuda")
        age = (length.view(-1, 1) - 1 - t).double()
        weight = torch.where(age >= 0, self.decay ** age, 0.0)
        return ((weight.unsqueeze(2) * cache.double()).sum(1) @ self.out.double() / math.sqrt(self.D)).float()


def plain_beam_search(model, prompt, beams, steps, eos, penalty):
    """One request: (tokens, total, length, finished) of each hypothesis, from whole sequences and 64-bit sums."""
    hyps = [(list(prompt), 0.0, 0, False)]
    for _ in range(steps):
        cand = []
        for w, (toks, total, n, fin) in enumerate(hyps):
            if fin:
                cand.append((total / max(n, 1) ** penalty, -w, 0, toks, total, n, True))
                continue
            x = model.logits(model.entry[torch.tensor(toks, device="cuda")].unsqueeze(0), torch.tensor([len(toks)], device="cuda"))[0].double()
            lp = (x - torch.logsumexp(x, 0)).cpu()
            for v in torch.topk(lp, beams).indices.tolist():
                t = total + float(lp[v])
                cand.append((t / (n + 1) ** penalty, -w, -v, toks + [v], t, n + 1, v == eos))
        cand.sort(key=lambda c: c[:3], reverse=True)
        hyps = [c[3:] for c in cand[:beams]]
    return hyps


@pytest.mark.parametrize("beams,block", [(1, 4), (4, 4), (5, 3)])
def test_beam_search_over_dense_and_paged_caches(beams, block):
    V, D, steps, B, eos, penalty = 301, 24, 9, 3, 7, 0.7
    model = Toy(V, D, 5)
    g = torch.Generator().manual_seed(3)
    prompts = [torch.randint(8, V, (n,), generator=g).tolist() for n in (2, 5, 9)]
    T = max(map(len, prompts)) + steps + 1
    rows = B * beams
    i32 = dict(dtype=torch.int32, device="cuda")
    width, blocks = -(-T // block), 2 * rows * -(-T // block)
    tables = G.BlockTables.empty(rows, width, blocks, block, beams)
    pages = [torch.zeros(blocks, block, D, device="cuda") for _ in range(2)]       # (two layers that hold the same)
    dense = [torch.zeros(B, beams, T, D, device="cuda") for _ in range(2)]
    # prompts are admitted in the first row of each group, the others go on from it
    append = torch.zeros(rows, **i32)
    append[::beams] = torch.tensor([len(p) for p in prompts], **i32)
    plan = G.block_plan(tables, append, sum(map(len, prompts)))
    flat = torch.tensor(sum(prompts, []), device="cuda")
    for pool in pages:
        pool.view(-1, D)[plan.slots] = model.entry[flat]
    for b, p in enumerate(prompts):
        for layer in dense:
            layer[b, 0, :len(p)] = model.entry[torch.tensor(p, device="cuda")]
    used = torch.tensor([len(p) for p in prompts], **i32).view(B, 1).expand(B, beams).contiguous()
    fork = torch.zeros(B, beams, **i32)
    G.block_plan(tables, torch.zeros(rows, **i32), 0, parents=fork)
    G.reorder_states(dense, fork, lengths=used, token_dim=2)
    scores = torch.full((B, beams), -math.inf, device="cuda")
    scores[:, 0] = 0.0
    lengths, done = torch.zeros(B, beams, **i32), torch.zeros(B, beams, dtype=torch.bool, device="cuda")
    text = [[list(p) for _ in range(beams)] for p in prompts]
    outs, plan = [None, None], None
    for step in range(steps):
        # logits from the paged cache, and from the dense one
        slot = tables.table.long().clamp(min=0).repeat_interleave(block, 1) * block + torch.arange(width * block, device="cuda") % block
        paged = model.logits(pages[step % 2].view(-1, D)[slot], tables.lengths)
        direct = model.logits(dense[step % 2].view(rows, T, D), used.view(-1))
        live = (scores > -math.inf).view(-1)
        assert torch.equal(paged[live], direct[live])
        r = outs[step % 2] = G.beam_select(paged.view(B, beams, V), scores, beams, lengths=lengths, done=done, eos=eos,
                                           length_penalty=penalty, out=outs[step % 2])
        assert r.status.tolist() == [0] * B
        text = [[text[b][p] + ([t] if not bool(done[b, p]) else []) for p, t in zip(r.parent[b].tolist(), r.token[b].tolist())]
                for b in range(B)]
        # states and tables follow; hypotheses that were finished before get no further entry
        grow = ~done.gather(1, r.parent.long())
        plan = G.block_plan(tables, grow.view(-1).int(), rows, parents=r.parent, out=plan)
        assert int(plan.status.max()) == 0
        G.copy_blocks(pages, plan.copy_src, plan.copy_dst)
        G.reorder_states(dense, r.parent, lengths=used, token_dim=2)
        used = used.gather(1, r.parent.long())
        entry = model.entry[r.token.long()]
        for pool in pages:
            n = int(plan.offsets[-1])
            pool.view(-1, D)[plan.slots[:n]] = entry.view(rows, D)[grow.view(-1)]
        for layer in dense:
            b, w = grow.nonzero(as_tuple=True)
            layer[b, w, used[b, w].long()] = entry[b, w]
        used += grow.int()
        assert torch.equal(tables.lengths, used.view(-1))
        scores, lengths, done = r.score, r.length, r.done
    for b, p in enumerate(prompts):
        want = plain_beam_search(model, p, beams, steps, eos, penalty)
        assert [h[0] for h in want] == text[b]
        assert [h[2] for h in want] == lengths[b].tolist() and [h[3] for h in want] == done[b].tolist()
        # totals: each of the steps' additions is rounded to fp32 (half a unit of 2^-23 relative), each log-sum is good to
        # 2^-22 + the products' 2^-23 (log2 V + 1) log 2 + 2^-20
        per = 2.0 ** -22 + math.log(2) * 2.0 ** -23 * (math.log2(V) + 1) + 2.0 ** -20
        for h, s in zip(want, scores[b].tolist()):
            assert abs(h[1] - s) <= steps * (per + 2.0 ** -24 * max(1.0, abs(h[1])))
    # nothing is held twice or lost: the counts are those of the tables
    held = tables.table[tables.table >= 0].long()
    assert torch.equal(torch.bincount(held, minlength=blocks).int(), tables.refs)
    G.block_plan(tables, torch.zeros(rows, **i32), 0, parents=torch.full((rows,), -1, **i32))
    assert int(tables.refs.abs().max()) == 0 and int(tables.table.max()) == -1


def test_verification_keeps_the_accepted_draft():
    """Each step drafts n tokens per request as rows of one group, verifies them and goes on from the emitted one: the
    accepted draft's hidden state and cache blocks, or a fresh entry where a token was resampled."""
    B, n, D, block, steps = 6, 4, 16, 4, 7
    i32 = dict(dtype=torch.int32, device="cuda")
    entry = torch.randn(5000, D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    tables = G.BlockTables.empty(B * n, 8, 400, block, n)
    pool = torch.zeros(400, block, D, device="cuda")
    hidden = [torch.zeros(B, 1, D, device="cuda")]
    text = [[] for _ in range(B)]
    for step in range(steps):
        wl = W.config3(batch=B, device="cuda", seed=900 + step, V=5000, n=n, topk=20)
        # drafts: every row of a group goes on from the group's first row and writes its own drafted token
        base = tables.lengths.view(B, n)[:, 0].clone()
        plan = G.block_plan(tables, torch.ones(B * n, **i32), B * n, parents=torch.zeros(B, n, **i32))
        assert int(plan.status.max()) == 0
        G.copy_blocks([pool], plan.copy_src, plan.copy_dst)
        pool.view(-1, D)[plan.slots] = entry[wl.draft_tokens.view(-1).long()]
        drafted = entry[wl.draft_tokens.long()] + 0.5 * hidden[0]
        sv, v = G.solve_verify(wl.q_logits, wl.p_logits, wl.draft_tokens, wl.uniforms, wl.topk, wl.temp_target, wl.temp_draft)
        same = wl.draft_tokens == v.token.view(B, 1)
        chosen = torch.where(v.accepted.view(B, 1).bool(), same.int().argmax(1, keepdim=True).int(), -1)
        # the accepted draft's state into place (a rejected group's is left, and made from the emitted token)
        kept = [entry[v.token.long()].view(B, 1, D) + 0.5 * hidden[0]]
        G.reorder_states([drafted], chosen, out=kept)
        hidden = kept
        # every row goes on from the accepted draft's; after a rejection from the first row cut back, with a new entry
        keep = torch.where(v.accepted.bool(), base + 1, base).int()
        plan = G.block_plan(tables, torch.zeros(B * n, **i32), 0, keep=keep.repeat_interleave(n),
                            parents=chosen.clamp(min=0).expand(B, n).contiguous())
        again = (~v.accepted.bool()).view(B, 1) & (torch.arange(n, device="cuda") == 0)
        plan = G.block_plan(tables, again.view(-1).int(), B)
        G.copy_blocks([pool], plan.copy_src, plan.copy_dst)
        some = plan.slots[:int(plan.offsets[-1])]
        pool.view(-1, D)[some] = entry[v.token[~v.accepted.bool()].long()]
        for b, t in enumerate(v.token.tolist()):
            text[b].append(t)
        for b in range(B):
            r = b * n
            assert int(tables.lengths[r]) == len(text[b])
            slots = [int(tables.table[r, t // block]) * block + t % block for t in range(len(text[b]))]
            assert torch.equal(pool.view(-1, D)[slots], entry[torch.tensor(text[b], device="cuda")])
            state = torch.zeros(D, device="cuda")
            for t in text[b]:
                state = entry[t] + 0.5 * state
            assert torch.equal(hidden[0][b, 0], state)
