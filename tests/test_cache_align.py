"""Lists that are not aligned to their elements are refused by the C entry points of caches and log probabilities, before anything is launched (a load
from there ends the process's use of the GPU).  No GPU needed."""
import pytest

import paper_2511_15898_b200 as G
from paper_2511_15898_b200.build import build_library

A = 1 << 20
B, C, D, E, F, H, K = (A + (i << 36) for i in range(1, 8))


@pytest.fixture(scope="module", autouse=True)
def lib():
    build_library()


def _layout(four):
    return G.CacheLayout(G.GR_Q4 if four else G.GR_BF16, 2, 64, 16, 5, 2304 if four else 2048, 128, 64)


@pytest.mark.parametrize("four", [False, True])
def test_slots_positions_frequencies(four):
    x = G.CacheTokens(B, C, D, D, G.GR_BF16, 4, 128, 64, 128, 64, 256, 64, 256, 64)
    for slots, positions, freq in ((E + 4, F, H), (E + 1, F, H), (E, F + 2, H), (E, F, H + 4)):
        assert G.gr_cache_append(A, A + (1 << 30), _layout(four), x, 3, slots, positions, freq, 64, 0, 0) == -3
    assert G.gr_cache_append(A, A + (1 << 30), _layout(four), x, 3, E, F + 2, 0, 0, 0, 0) == -3
    for off in (1, 2, 4):
        assert G.gr_cache_read(A, A + (1 << 30), _layout(four), E + off, 3, G.GR_F32, B, 128, 64, C, 128, 64, 0) == -3


def test_attend():
    ok = dict(table=E, off=F, pos=H, status=K)
    for name in ok:
        for off in (1, 2):
            a = {**ok, name: ok[name] + off}
            assert G.gr_cache_attend(B, G.GR_BF16, 8, 512, 64, A, _layout(True), a["table"], 4, 3, a["off"], a["pos"], 5, 0.1, 0, C, D, 512, 64, a["status"], 0) == -3


def test_token_logprobs():
    ok = dict(tokens=B, lp=C, ent=D, tok=E, tlp=F, st=H)
    for name in ok:
        for off in (1, 2):
            a = {**ok, name: ok[name] + off}
            assert G.gr_token_logprobs(A, G.GR_F32, 1000, 1000, 4, 1.0, a["tokens"], 2, 5, a["lp"], a["ent"], a["tok"], a["tlp"], a["st"], 0) == -3, name
