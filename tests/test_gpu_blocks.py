"""Block plans on the GPU against the plain model: whole runs of steps with admissions, forks, rollbacks, releases and pools
that run out; refused rows; sizes from none to many."""
import random

import pytest
import torch

import paper_2511_15898_b200 as G
from paper_2511_15898_b200.build import build_library
from tests import block_pool

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    build_library()


def dev(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")


class Pair:
    """The tables on the GPU and in the plain model, taken through the same steps."""

    def __init__(self, rows, width, blocks, block, beams=1):
        self.t = G.BlockTables.empty(rows, width, blocks, block, beams)
        self.table = [[-1] * width for _ in range(rows)]
        self.lengths, self.refs, self.block, self.beams = [0] * rows, [0] * blocks, block, beams
        self.out = None

    def step(self, append, max_tokens, keep=None, parents=None, reuse=True):
        want = block_pool.plan(self.table, self.lengths, self.refs, self.block, self.beams, append, max_tokens, keep, parents)
        self.out = G.block_plan(self.t, dev(append), max_tokens, dev(keep), dev(parents), self.out if reuse else None)
        torch.cuda.synchronize()
        o = self.out
        got = (o.slots, o.positions, o.offsets, o.copy_src, o.copy_dst, o.status)
        for name, g, w in zip(("slots", "positions", "offsets", "copy_src", "copy_dst", "status"), got, want):
            assert g.tolist() == w, name
        assert self.t.table.tolist() == self.table
        assert self.t.lengths.tolist() == self.lengths
        assert self.t.refs.tolist() == self.refs
        return want[5]


@pytest.mark.parametrize("rows,beams,width,blocks,block", [(1, 1, 1, 1, 1), (5, 1, 4, 9, 3), (12, 4, 7, 40, 8), (64, 8, 33, 500, 16),
                                                        (96, 32, 20, 900, 5), (1030, 1, 9, 4000, 7), (60, 12, 70, 1500, 4), (6, 2, 1, 3, 16),
                                                        (1200, 4, 6, 5000, 8), (4, 2, 600, 2300, 2)])
def test_runs_of_steps(rows, beams, width, blocks, block):
    rng = random.Random(rows * 31 + block)
    p = Pair(rows, width, blocks, block, beams)
    cap = width * block
    seen = set()
    for step in range(12):
        kind = rng.choice(["decode", "decode", "prefill", "fork", "fork", "rollback", "mixed"])
        parents = keep = None
        if kind == "decode":
            append = [1] * rows
        elif kind == "prefill":
            append = [rng.randint(0, cap) if n == 0 or rng.random() < 0.1 else 0 for n in p.lengths]
        else:
            append = [rng.choice([0, 1, 1, rng.randint(0, 2 * block)]) for _ in range(rows)]
        if kind in ("fork", "mixed"):
            parents = [rng.choice([-1] + list(range(beams)) * 3) for _ in range(rows)]
            append = [1] * rows if rng.random() < 0.5 else append
        if kind in ("rollback", "mixed"):
            keep = [rng.randint(0, cap + 5) for _ in range(rows)]
        total = sum(append)
        seen |= set(p.step(append, rng.choice([total, total + 3, max(0, total - 1)]), keep, parents, rng.random() < 0.7))
    assert G.GR_OK in seen


def test_one_row_keeps_the_block_that_the_others_copy():
    p = Pair(4, 4, 12, 4, 4)
    p.step([6, 0, 0, 0], 6)
    p.step([0, 0, 0, 0], 0, parents=[0, 0, 0, 0])
    assert p.refs[:2] == [4, 4]
    p.step([1, 1, 1, 1], 4)                        # all write: the first keeps the block, three copy
    assert p.out.copy_src.tolist() == [-1, 1, 1, 1] and p.out.copy_dst.tolist() == [-1, 2, 3, 4]
    p = Pair(4, 4, 12, 4, 4)
    p.step([6, 0, 0, 0], 6)
    p.step([0, 0, 0, 0], 0, parents=[0, 0, 0, 0])
    p.step([1, 0, 1, 1], 3)                        # one only reads: all that write copy
    assert p.out.copy_src.tolist() == [1, -1, 1, 1]
    p = Pair(2, 4, 12, 4, 2)
    p.step([7, 0], 7)
    p.step([0, 0], 0, parents=[0, 0], keep=[5, 7])
    p.step([1, 1], 2)                              # the row with more tokens in the block keeps it
    assert p.out.copy_src.tolist() == [1, -1]


def test_rows_that_cannot_be_served():
    p = Pair(5, 3, 6, 4)
    st = p.step([4, 13, 9, 8, 0], 40)              # row 1 is full (12 tokens at most); 1 + 3 + 2 blocks are all there are
    assert st == [0, 9, 0, 0, 0]
    st = p.step([1, 1, 1, -2, 1], 2)               # no block is left; the slot map holds two tokens
    assert st == [8, 8, 9, 10, 9]
    # ids, lengths and parents that make no sense are refused by row; the others go on
    t = G.BlockTables.empty(6, 4, 8, 4, 2)
    t.lengths.copy_(dev([5, 5, -3, 99, 4, 4]))
    t.table[0, 0], t.table[0, 1] = 0, 77
    t.table[1, 0], t.table[1, 1] = 1, -1
    t.table[4, 0], t.table[5, 0] = 2, 3
    t.refs[:4] = 1
    o = G.block_plan(t, dev([1] * 6), 6, parents=dev([0, 1, 0, 1, 0, 7]))
    torch.cuda.synchronize()
    assert o.status.tolist() == [10, 10, 10, 10, 0, 10]
    # (row 5 goes on from nothing: its block 3 is free again, and row 4 takes it)
    assert o.slots.tolist() == [-1, -1, -1, -1, 12, -1] and t.lengths.tolist() == [5, 5, 0, 16, 5, 0]
    assert t.refs.tolist() == [1, 1, 1, 1, 0, 0, 0, 0] and t.table[5].tolist() == [-1] * 4


@pytest.mark.parametrize("others", [[1, 2, 3], [1, 3, 2]])
def test_ids_outside_the_pool_where_rows_go_on_from_themselves(others):
    # row 0 goes on from itself: whether its first block's id makes sense is not looked at, whatever its neighbours do
    t = G.BlockTables.empty(4, 4, 16, 4, 4)
    t.lengths.copy_(dev([8, 8, 8, 8]))
    t.table[:, :2] = dev([[99, 0], [1, 2], [3, 4], [5, 6]])
    t.refs[:7] = 1
    o = G.block_plan(t, dev([1] * 4), 4, parents=dev([0] + others))
    assert o.status.tolist() == [0] * 4
    assert t.table[:, 2].tolist() == [7, 8, 9, 10] and t.table[0, :2].tolist() == [99, 0]
    # a row that goes on from row 0 is refused
    o = G.block_plan(t, dev([1] * 4), 4, parents=dev([0, 0, 2, 3]))
    assert o.status.tolist() == [0, 10, 0, 0]


def test_empty_and_large():
    t = G.BlockTables.empty(0, 4, 8, 4)
    o = G.block_plan(t, dev([]), 5)
    torch.cuda.synchronize()
    assert o.slots.tolist() == [-1] * 5 and o.offsets.tolist() == [0]
    t = G.BlockTables.empty(3, 0, 0, 4)
    o = G.block_plan(t, dev([0, 1, 0]), 1)
    assert o.status.tolist() == [0, 9, 0]
    # a million blocks, long prompts: slots beyond 2^31
    t = G.BlockTables.empty(2, 1 << 19, 1 << 21, 2048)
    t.refs[:1_100_000] = 1
    o = G.block_plan(t, dev([5, 2049]), 2100)
    torch.cuda.synchronize()
    assert o.slots[:3].tolist() == [1_100_000 * 2048 + i for i in range(3)] and int(o.slots[5]) == 1_100_001 * 2048
    assert int(o.slots[2053]) == 1_100_002 * 2048 and int(o.slots[2054]) == -1


def test_in_a_graph_with_padding():
    t = G.BlockTables.empty(4, 8, 40, 4)
    append = dev([3, 5, 0, 1])
    out = G.block_plan(t, append, 16)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        G.block_plan(t, append, 16, out=out)
    p = Pair(4, 8, 40, 4)
    p.step([3, 5, 0, 1], 16)
    for a in ([1, 1, 1, 1], [0, 6, 2, 0], [1, 1, 0, 1]):
        append.copy_(dev(a))
        graph.replay()
        torch.cuda.synchronize()
        want = block_pool.plan(p.table, p.lengths, p.refs, 4, 1, a, 16)
        assert out.slots.tolist() == want[0] and t.table.tolist() == p.table and t.refs.tolist() == p.refs


def test_lengths_as_what_is_kept():
    """A step that only appends to what is there, told so by the lengths themselves; and two tables side by side on two streams."""
    p = Pair(6, 5, 40, 4, 2)
    p.step([3, 9, 0, 1, 5, 2], 20)
    want = block_pool.plan(p.table, p.lengths, p.refs, 4, 2, [1] * 6, 6, list(p.lengths), [1, 1, 0, 0, 1, 0])
    o = G.block_plan(p.t, dev([1] * 6), 6, keep=p.t.lengths, parents=dev([1, 1, 0, 0, 1, 0]))
    torch.cuda.synchronize()
    assert o.slots.tolist() == want[0] and p.t.lengths.tolist() == p.lengths and p.t.refs.tolist() == p.refs
    a, b = Pair(300, 20, 3000, 8), Pair(300, 20, 3000, 8)
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    steps = [dev([(r * 7 + k) % 9 for r in range(300)]) for k in range(6)]
    torch.cuda.synchronize()
    outs = [None, None]
    for k in range(6):
        for i, (pair, stream) in enumerate(((a, one), (b, two))):
            with torch.cuda.stream(stream):
                outs[i] = G.block_plan(pair.t, steps[k], 2400, out=outs[i])
    torch.cuda.synchronize()
    for k in range(6):
        want = block_pool.plan(a.table, a.lengths, a.refs, 8, 1, steps[k].tolist(), 2400)
    for pair, out in ((a, outs[0]), (b, outs[1])):
        assert out.slots.tolist() == want[0] and pair.t.table.tolist() == a.table and pair.t.refs.tolist() == a.refs
