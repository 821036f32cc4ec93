"""Tensors of one layout that share bytes are refused by the C entry points before anything is launched, tensors that lie between one
another's pieces are not: against a plain look at every byte.  No GPU needed: without parents or lists of pairs the calls look at
everything else and then answer -2."""
import random

import pytest

import paper_2511_15898_b200 as G
from paper_2511_15898_b200.build import build_library

A = 1 << 20


@pytest.fixture(scope="module", autouse=True)
def lib():
    build_library()


def pieces(at, sizes, strides):
    out = [at]
    for n, s in zip(sizes, strides):
        out = [a + k * s for a in out for k in range(n)]
    return out


def share_a_byte(places, sizes, strides, size):
    seen = set()
    for at in places:
        mine = {a + i for a in pieces(at, sizes, strides) for i in range(size)}
        if mine & seen:
            return True
        seen |= mine
    return False




def call(places, groups, beams, parts, strides, size):
    layout = G.StateLayout(groups, beams, beams, parts, *strides, *strides, size, 1)
    rc = G.gr_reorder_states(places, places, layout, 0, 0, 0)
    assert rc in (-1, -2)
    return rc


def test_one_state_within_another():
    # x[:, :, 0:2] and x[:, :, 1:3] of [2, 4, 3 heads, 16 bytes] share the second head
    strides = (192, 48, 16)
    assert call([A, A + 16], 2, 4, 2, strides, 16) == -1
    assert call([A, A + 32], 2, 4, 1, strides, 16) != -1
    # every second group, every second state; one behind the last byte of another
    assert call([A, A + 192], 2, 4, 3, (384, 48, 16), 16) != -1
    assert call([A, A + 48], 2, 4, 3, (384, 96, 16), 16) != -1
    assert call([A, A + 96], 2, 4, 3, (384, 96, 16), 16) == -1
    assert call([A, A + 384], 2, 4, 3, (384, 96, 16), 16) == -1
    assert call([A, A + 384 + 96 * 3 + 32], 2, 4, 3, (384, 96, 16), 16) == -1
    assert call([A, A + 384 + 96 * 3 + 48], 2, 4, 3, (384, 96, 16), 16) != -1


def test_random_layouts_against_every_byte():
    rng = random.Random(4)
    met = {True: 0, False: 0}
    for _ in range(4000):
        size = rng.randint(1, 6)
        sizes = [rng.randint(1, 4) for _ in range(3)]
        span, strides = size, [0, 0, 0]
        for i in rng.sample(range(3), 3):
            strides[i] = span + rng.choice([0, 0, 1, rng.randint(0, 3 * span)])
            span += strides[i] * (sizes[i] - 1)
        places = [A + rng.randint(0, 2 * span) for _ in range(rng.randint(2, 4))]
        want = share_a_byte(places, sizes, strides, size)
        assert (call(places, sizes[0], sizes[1], sizes[2], strides, size) == -1) == want, (places, sizes, strides, size)
        met[want] += 1
    assert min(met.values()) > 500


def test_random_caches_against_every_byte():
    rng = random.Random(5)
    met = {True: 0, False: 0}
    for _ in range(2000):
        size, blocks = rng.randint(1, 9), rng.randint(1, 6)
        stride = size + rng.choice([0, 1, rng.randint(0, 30)])
        places = [A + rng.randint(0, 2 * stride * blocks) for _ in range(rng.randint(2, 4))]
        want = share_a_byte(places, [blocks], [stride], size)
        assert (G.gr_copy_blocks(places, blocks, stride, size, 0, 0, 4, 0) == -1) == want, (places, blocks, stride, size)
        met[want] += 1
    assert min(met.values()) > 200


def test_many_layers_of_one_buffer():
    # [2, layers, 4, 3, 16 bytes], [2, 4, layers, 3, 16], [2, 4, 3, layers, 16] in any order, and with one layer twice
    rng = random.Random(6)
    n = 200
    for strides, step in (((n * 192, 48, 16), 192), ((n * 192, n * 48, 16), 48), ((n * 192, n * 48, n * 16), 16)):
        places = [A + i * step for i in range(n)]
        rng.shuffle(places)
        assert call(places, 2, 4, 3, strides, 16) != -1
        assert call(places + [places[7] + 1], 2, 4, 3, strides, 16) == -1
