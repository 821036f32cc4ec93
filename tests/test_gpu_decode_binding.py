"""The two ways of the tensor front ends around a decoding step (the compiled module's and the one in Python): the same results,
and the same refusals, whichever a call takes."""
import pytest
import torch

import paper_2511_15898_b200 as G
import paper_2511_15898_b200.binding as Bn
from paper_2511_15898_b200.build import build_library

pytestmark = pytest.mark.gpu
I32 = dict(dtype=torch.int32, device="cuda")


@pytest.fixture(scope="module", autouse=True)
def lib():
    build_library()
    assert Bn._tensors is not None


def both(monkeypatch, call):
    """What `call` gives by either way; it is told whether the module takes part."""
    first = call()
    with monkeypatch.context() as m:
        m.setattr(Bn, "_tensors", None)
        second = call()
    torch.cuda.synchronize()
    assert len(first) == len(second)
    for a, b in zip(first, second):
        assert torch.equal(a, b)


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def test_same_results(monkeypatch):
    for dtype in (torch.float32, torch.bfloat16):
        x = torch.randn(3, 4, 1001, generator=gen(1), device="cuda").to(dtype)
        s = -torch.rand(3, 4, generator=gen(2), device="cuda")
        n, d = torch.randint(0, 9, (3, 4), **I32), torch.rand(3, 4, device="cuda") < 0.3
        for view in (x, x[:, :, :999], x[:, 1:2], x[:1, :, 3:]):
            B, W, V = view.shape
            def select():
                out = G.beam_select(view, s[:B, :W].contiguous(), 5)
                out.token.fill_(-9)
                out = G.beam_select(view, s[:B, :W].contiguous(), 5, 0.7, n[:B, :W].contiguous(), d[:B, :W].contiguous(), 3, 0.5, out)
                again = G.beam_select(view, s[:B, :W].contiguous(), 5, 0.7, done=d[:B, :W].byte().contiguous(), eos=3, out=None)
                return [out.token.clone(), out.parent, out.score, out.length, out.done, out.status, again.token, again.done]
            both(monkeypatch, select)
    parents = torch.randint(-1, 5, (3, 5), generator=gen(3), **I32)
    lengths = torch.randint(0, 9, (3, 5), generator=gen(4), **I32)
    base = torch.randn(2, 3, 5, 4, 8, 6, generator=gen(5), device="cuda")

    def reorder():
        a, b, d = base.clone(), base.clone(), base[0].clone()
        G.reorder_states([a[0], a[1]], parents)
        G.reorder_states([b[0], b[1]], parents, lengths=lengths, token_dim=4)
        out = [torch.zeros(3, 2, 4, 8, 6, device="cuda") for _ in range(2)]
        G.reorder_states([base[0], base[1]], parents[:, :2].contiguous(), out=out)
        G.reorder_states([d[:, :, 1:3, :, :]], parents, lengths=lengths, token_dim=3)
        mixed = [base[0].clone(), base[1].bfloat16(), base[0, :, :, 0].clone()]
        G.reorder_states(mixed, parents)
        return [a, b, d, *out, *mixed]
    both(monkeypatch, reorder)

    def plan():
        t = G.BlockTables.empty(12, 6, 80, 4, beams=4)
        out = G.block_plan(t, torch.full((12,), 5, **I32), 60)
        p = torch.randint(-1, 4, (3, 4), generator=gen(7), **I32)
        first = G.block_plan(t, torch.ones(12, **I32), 60, keep=torch.full((12,), 4, **I32), parents=p, out=out)
        a = [first.slots.clone(), first.copy_src.clone(), t.table.clone(), t.refs.clone()]
        second = G.block_plan(t, torch.ones(12, **I32), 60, parents=p.view(-1), out=out)
        return a + [second.slots, second.positions, second.offsets, second.copy_dst, second.status, t.table, t.lengths, t.refs]
    both(monkeypatch, plan)

    def copy():
        pools = torch.randn(3, 20, 7, 4, generator=gen(8), device="cuda")
        src, dst = torch.tensor([3, -1, 5], **I32), torch.tensor([9, 2, 0], **I32)
        G.copy_blocks([pools[0], pools[1]], src, dst)
        G.copy_blocks([pools[2][:, :3]], src, dst)
        G.copy_blocks([pools[0][:10], pools[1]], dst[1:].contiguous(), torch.tensor([17, 8], **I32))
        return [pools]
    both(monkeypatch, copy)


def test_same_refusals(monkeypatch):
    x, s = torch.randn(2, 3, 50, device="cuda"), torch.zeros(2, 3, device="cuda")
    out, wide = G.beam_select(x, s, 4), G.beam_select(x, s, 3)
    parents, ln = torch.zeros(2, 3, **I32), torch.ones(2, 3, **I32)
    state = torch.zeros(2, 3, 4, 8, device="cuda")
    t = G.BlockTables.empty(6, 4, 20, 4, beams=3)
    ones = torch.ones(6, **I32)
    plan = G.block_plan(t, ones, 6)
    pool, idx = torch.zeros(20, 8, device="cuda"), torch.zeros(4, **I32)
    wrong = [
        lambda: G.beam_select(x.half(), s, 4, out=out), lambda: G.beam_select(x, s.double(), 4, out=out), lambda: G.beam_select(x, s[:1], 4, out=out),
        lambda: G.beam_select(x, s, 4, lengths=ln.long(), out=out), lambda: G.beam_select(x, s, 4, done=ln, eos=1, out=out),
        lambda: G.beam_select(x, s, 4, eos=50, out=out), lambda: G.beam_select(x, s, 4, 0.0, out=out), lambda: G.beam_select(x, s, 200, out=out),
        lambda: G.beam_select(x, s, 4, done=ln.bool(), out=out), lambda: G.beam_select(x, s, 4, length_penalty=1.0, out=out),
        lambda: G.beam_select(x.transpose(1, 2), s, 4, out=out), lambda: G.beam_select(x.cpu(), s, 4, out=out),
        lambda: G.beam_select(x, wide.score, 3, out=wide), lambda: G.beam_select(x, s, 3, done=wide.done, eos=1, out=wide),
        lambda: G.reorder_states([state], parents.long()), lambda: G.reorder_states([state], parents[:1]), lambda: G.reorder_states([state.cpu()], parents),
        lambda: G.reorder_states([state, state], parents), lambda: G.reorder_states([state], parents, lengths=ln), lambda: G.reorder_states([state], parents, token_dim=3),
        lambda: G.reorder_states([state], parents, lengths=ln, token_dim=1), lambda: G.reorder_states([state], parents, lengths=ln, token_dim=4),
        lambda: G.reorder_states([state], parents, out=[torch.zeros(2, 3, 4, 7, device="cuda")]), lambda: G.reorder_states([state], parents, out=[state.double()]),
        lambda: G.reorder_states([state], parents, out=[]), lambda: G.reorder_states([state[:, :, :, ::2]], parents), lambda: G.reorder_states([3], parents),
        lambda: G.reorder_states([torch.zeros(2, 40, 4, device="cuda")], parents),
        lambda: G.block_plan(t, ones.long(), 6, out=plan), lambda: G.block_plan(t, ones[:3], 6, out=plan), lambda: G.block_plan(t, ones, -1, out=plan),
        lambda: G.block_plan(t, ones, 6, keep=ones[:2], out=plan), lambda: G.block_plan(t, ones, 6, parents=parents.view(3, 2), out=plan),
        lambda: G.block_plan(G.BlockTables(t.table, t.lengths, t.refs, 0, 3), ones, 6, out=plan),
        lambda: G.block_plan(G.BlockTables(t.table, t.lengths.long(), t.refs, 4, 3), ones, 6, out=plan),
        lambda: G.block_plan(G.BlockTables(t.table, t.lengths, t.refs, 4, 4), ones, 6, out=plan),
        lambda: G.block_plan(G.BlockTables(t.table.t(), t.lengths, t.refs, 4, 3), ones, 6, out=plan),
        lambda: G.copy_blocks([pool], idx.long(), idx), lambda: G.copy_blocks([pool], idx, idx[:2]), lambda: G.copy_blocks([pool.t()], idx, idx),
        lambda: G.copy_blocks([pool, pool], idx, idx), lambda: G.copy_blocks([pool.cpu()], idx, idx), lambda: G.copy_blocks([7], idx, idx),
    ]
    keep = t.table.clone(), t.refs.clone()
    for i, call in enumerate(wrong):
        for module in (Bn._tensors, None):
            with monkeypatch.context() as m:
                m.setattr(Bn, "_tensors", module)
                with pytest.raises(G.GrError):
                    call()
                    pytest.fail(f"call {i} by {module}")
    torch.cuda.synchronize()
    assert torch.equal(t.table, keep[0]) and torch.equal(t.refs, keep[1]) and int(state.abs().max()) == 0
