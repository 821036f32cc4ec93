"""What the tensor front ends around a decoding step refuse or take at the edges of their arguments, by the compiled module's way and
by the one in Python."""
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


@pytest.fixture(params=["module", "python"])
def way(request, monkeypatch):
    if request.param == "python":
        monkeypatch.setattr(Bn, "_tensors", None)


def test_numbers_beyond_32_bits_are_refused(way):
    wide = 1 << 32
    x, s = torch.randn(2, 3, 50, device="cuda"), torch.zeros(2, 3, device="cuda")
    done = torch.zeros(2, 3, dtype=torch.bool, device="cuda")
    out = G.beam_select(x, s, 4)
    t = G.BlockTables.empty(6, 4, 20, 4, beams=3)
    ones = torch.ones(6, **I32)
    plan = G.block_plan(t, ones, 6)
    for call in (lambda: G.beam_select(x, s, wide + 4), lambda: G.beam_select(x, s, 4, done=done, eos=wide + 1),
                 lambda: G.beam_select(x, s, 4, done=done, eos=wide + 1, out=out), lambda: G.block_plan(t, ones, wide + 6),
                 lambda: G.block_plan(G.BlockTables(t.table, t.lengths, t.refs, wide + 4, 3), ones, 6),
                 lambda: G.block_plan(G.BlockTables(t.table, t.lengths, t.refs, wide + 4, 3), ones, 6, out=plan),
                 lambda: G.block_plan(G.BlockTables(t.table, t.lengths, t.refs, 4, wide + 3), ones, 6, out=plan)):
        with pytest.raises(G.GrError):
            call()
    # 2^32 pieces of a byte, 2^32 blocks of a byte
    state = torch.zeros(1, 2, wide, 1, dtype=torch.uint8, device="cuda")
    with pytest.raises(G.GrError):
        G.reorder_states([state], torch.zeros(1, 2, **I32), lengths=torch.ones(1, 2, **I32), token_dim=3)
    with pytest.raises(G.GrError):
        G.copy_blocks([state.view(-1, 1)], torch.zeros(1, **I32), torch.ones(1, **I32))


def test_token_dimensions_that_are_none(way):
    state, parents = torch.arange(48.0, device="cuda").view(2, 3, 8), torch.zeros(2, 3, **I32)
    keep = state.clone()
    for dim in (-1, -2, -9):
        with pytest.raises(G.GrError):
            G.reorder_states([state], parents, token_dim=dim)
        with pytest.raises(G.GrError):
            G.reorder_states([state], parents, lengths=torch.ones(2, 3, **I32), token_dim=dim)
    with pytest.raises(Exception) as e:
        G.reorder_states([state], parents, token_dim="2")
    assert not isinstance(e.value, SystemError)
    torch.cuda.synchronize()
    assert torch.equal(state, keep)


def test_no_lengths_of_an_earlier_call_remain(way):
    x, s = torch.randn(2, 3, 50, device="cuda"), torch.zeros(2, 3, device="cuda")
    n = torch.full((2, 3), 6, **I32)
    out = G.beam_select(x, s, 4, lengths=n)
    assert out.length.tolist() == [[7] * 4] * 2
    assert G.beam_select(x, s, 4, out=out).length.tolist() == [[0] * 4] * 2
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        G.beam_select(x, s, 4, lengths=n, out=out)
    for _ in range(2):
        graph.replay()
        assert out.length.tolist() == [[7] * 4] * 2
        assert G.beam_select(x, s, 4, out=out).length.tolist() == [[0] * 4] * 2
