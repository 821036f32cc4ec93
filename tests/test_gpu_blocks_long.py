"""Block plans with slot maps of thousands of tokens against the plain model: maps that the plan writes itself, four tokens a thread, and
maps that are written by a kernel of their own; with parents, with more rows than a CTA holds, and off the vectors' alignment."""
import dataclasses
import random

import pytest
import torch

import paper_2511_15898_b200 as G
from paper_2511_15898_b200.build import build_library
from tests.test_gpu_blocks import Pair

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    build_library()


def shifted(out, slots, positions):
    """The result with maps that begin some elements behind a 16-byte boundary."""
    n = out.shape[2]
    a = torch.full((n + 4,), -7, dtype=torch.int64, device="cuda")
    b = torch.full((n + 4,), -7, dtype=torch.int32, device="cuda")
    return dataclasses.replace(out, slots=a[slots:n + slots], positions=b[positions:n + positions]), a, b


# rows, beams, width, blocks, block; tokens of an admission in all
@pytest.mark.parametrize("rows,beams,width,blocks,block,tokens", [
    (7, 1, 900, 5000, 16, 8193), (48, 4, 300, 9000, 8, 20011), (48, 4, 300, 9000, 8, 32768), (48, 4, 300, 9000, 8, 32769),
    (5, 5, 9000, 30000, 7, 40003), (1, 1, 6000, 6000, 16, 70001), (1026, 2, 40, 30000, 6, 9001), (1100, 4, 60, 40000, 3, 50002),
    (1030, 1, 3, 4000, 64, 33001)])
@pytest.mark.parametrize("shift", [(0, 0), (1, 0), (0, 3)])
def test_long_maps(rows, beams, width, blocks, block, tokens, shift):
    rng = random.Random(rows + tokens)
    p = Pair(rows, width, blocks, block, beams)
    cap = width * block

    def spread(n, free):
        cut = sorted(rng.randint(0, n) for _ in range(rows - 1))
        return [min(b - a, f + 3) for a, b, f in zip([0] + cut, cut + [n], free)]

    guards = []

    def step(append, most, keep=None, parents=None):
        out = G.block_plan(G.BlockTables.empty(rows, width, blocks, block, beams), torch.zeros(rows, dtype=torch.int32, device="cuda"), most)
        p.out, a, b = shifted(out, *shift)
        guards[:] = [a, b]
        p.step(append, most, keep, parents)
        # what lies beside the maps is left as it was
        for t, at in ((a, shift[0]), (b, shift[1])):
            assert t[:at].tolist() == [-7] * at and t[tokens_of(t) + at:].tolist() == [-7] * (4 - at)

    def tokens_of(t):
        return t.numel() - 4

    # an admission, with room left in the map and without
    append = spread(tokens, [cap] * rows)
    step(append, tokens + 5)
    # most of it given back, and another with forks, in a map that ends before the last token
    keep = [rng.randint(0, n) if rng.random() < 0.8 else n for n in p.lengths]
    append = spread(tokens, [cap - min(k, n) for k, n in zip(keep, p.lengths)])
    step(append, max(0, sum(append) - 1), keep, [rng.choice([-1] + list(range(beams)) * 2) for _ in range(rows)])
    # a token each, in a map that is longer than needed by far
    step([1] * rows, tokens, None, [rng.randrange(beams) for _ in range(rows)])
