"""Refusals of the operators that fill and read a paged cache: what the C entry points and the tensor front end reject on the host,
before anything is launched.  No GPU needed."""
import numpy as np
import pytest
import torch

import paper_2511_15898_b200 as G
from paper_2511_15898_b200.build import build_library
from tests import paged_cache as P

A = 1 << 20                      # any aligned non-null address: nothing is dereferenced on these paths
B, C, D, E, F = (A + (i << 36) for i in range(1, 6))


@pytest.fixture(scope="module", autouse=True)
def lib():
    build_library()
    return G.load_library()


def _layout(four=False, **kw):
    a = dict(format=G.GR_BF16, heads=2, dim=64, block_size=16, num_blocks=5, block_stride=16 * 2 * 64, token_stride=2 * 64, head_stride=64)
    if four:
        a.update(format=G.GR_Q4, block_stride=2 * 2 * 9 * 64)
    a.update(kw)
    return G.CacheLayout(*[a[n] for n, _ in G.CacheLayout._fields_])


_BAD_LAYOUTS = [dict(format=4), dict(format=-1), dict(heads=0), dict(heads=1025), dict(dim=0), dict(dim=63), dict(dim=514, head_stride=1 << 10, token_stride=1 << 12, block_stride=1 << 20),
                dict(block_size=0), dict(num_blocks=-1), dict(head_stride=63), dict(token_stride=127), dict(block_stride=16 * 128 - 1),
                dict(head_stride=0), dict(block_stride=1 << 60), dict(block_stride=-1)]
_BAD_FOUR = [dict(dim=48), dict(dim=288, block_stride=1 << 20), dict(block_size=12), dict(block_stride=2 * 2 * 9 * 64 - 16), dict(block_stride=2 * 2 * 9 * 64 + 8), dict(block_stride=1 << 60)]


def test_append():
    fields = dict(k=B, v=C, q=D, q_out=E, dtype=G.GR_BF16, q_heads=4, k_token=128, k_head=64, v_token=128, v_head=64, q_token=256,
                  q_head=64, out_token=256, out_head=64)

    def call(keys=A, values=A + (1 << 30), layout=None, four=False, tokens=3, slots=F, positions=F, freq=F, rot=64, inter=0, lay=None, **kw):
        a = dict(fields); a.update(kw)
        x = G.CacheTokens(*[a[n] for n, _ in G.CacheTokens._fields_])
        return G.gr_cache_append(keys, values, _layout(four, **(lay or {})), x, tokens, slots, positions, freq, rot, inter, 0)

    for bad in _BAD_LAYOUTS:
        assert call(lay=bad) == -1, bad
    for bad in _BAD_FOUR:
        assert call(four=True, lay=bad) == -1, bad
    assert G.gr_cache_append(A, A, None, G.CacheTokens(), 1, F, F, F, 0, 0, 0) == -2 and G.gr_cache_append(A, A, _layout(), None, 1, F, F, F, 0, 0, 0) == -2
    assert call(tokens=-1) == -1 and call(rot=-2) == -1 and call(rot=3) == -1 and call(rot=66) == -1
    assert call(dtype=G.GR_Q4) == -1 and call(dtype=7) == -1 and call(q_heads=-1) == -1 and call(q_heads=1025) == -1
    for name in ("k_token", "k_head", "v_token", "v_head", "q_token", "q_head"):
        assert call(**{name: -1}) == -1 and call(**{name: 1 << 60}) == -1, name
    assert call(out_head=63) == -1 and call(out_token=255) == -1 and call(out_token=0) == -1
    assert call(q=E, q_token=512) == -1 and call(q=E, q_head=128) == -1             # in place at other strides
    for name in ("k", "v", "q", "q_out"):
        assert call(**{name: 0}) == -2 and call(**{name: B + 1 + (1 << 34)}) == -3, name
    assert call(keys=0) == -2 and call(values=0) == -2 and call(slots=0) == -2 and call(positions=0) == -2 and call(freq=0) == -2
    assert call(keys=A + 1) == -3 and call(values=A + 1) == -3 and call(four=True, keys=A + 8) == -3
    # the cache lies apart from what is read and from the queries; keys and values are two
    assert call(k=A + 64) == -1 and call(v=A + 64) == -1 and call(q=A + 64) == -1 and call(q_out=A + 64) == -1 and call(values=A) == -1
    assert call(k=A + 5 * 4096 - 2) == -1 and call(four=True, k=A + 5 * 2304 - 2) == -1
    assert call(tokens=0) == 0 and call(tokens=0, k=0, slots=0) == 0


def test_read():
    def call(keys=A, values=A + (1 << 30), four=False, slots=F, tokens=3, dtype=G.GR_F32, k=B, kt=128, kh=64, v=C, vt=128, vh=64, lay=None):
        return G.gr_cache_read(keys, values, _layout(four, **(lay or {})), slots, tokens, dtype, k, kt, kh, v, vt, vh, 0)

    for bad in _BAD_LAYOUTS:
        assert call(lay=bad) == -1, bad
    for bad in _BAD_FOUR:
        assert call(four=True, lay=bad) == -1, bad
    assert G.gr_cache_read(A, A, None, F, 3, 0, B, 128, 64, C, 128, 64, 0) == -2
    assert call(tokens=-1) == -1 and call(dtype=G.GR_Q4) == -1 and call(dtype=-1) == -1
    assert call(kt=127) == -1 and call(kh=63) == -1 and call(vt=0) == -1 and call(vh=-64) == -1 and call(v=B) == -1
    assert call(keys=0) == -2 and call(values=0) == -2 and call(slots=0) == -2 and call(k=0) == -2 and call(v=0) == -2
    assert call(k=B + 2) == -3 and call(v=C + 1) == -3 and call(keys=A + 1) == -3 and call(four=True, keys=A + 8) == -3
    assert call(k=A + 64) == -1 and call(v=A + (1 << 30)) == -1
    assert call(tokens=0) == 0


def test_attend():
    ok = dict(q=B, dtype=G.GR_BF16, heads=8, qt=512, qh=64, cache=A, table=F, width=4, rows=3, off=F, pos=F, tokens=5, scale=0.1, window=0,
              ws=C, out=D, ot=512, oh=64, status=E)

    def call(four=True, lay=None, **kw):
        a = dict(ok); a.update(kw)
        return G.gr_cache_attend(a["q"], a["dtype"], a["heads"], a["qt"], a["qh"], a["cache"], _layout(four, **(lay or {})), a["table"], a["width"], a["rows"],
                                 a["off"], a["pos"], a["tokens"], a["scale"], a["window"], a["ws"], a["out"], a["ot"], a["oh"], a["status"], 0)

    for bad in _BAD_FOUR:
        assert call(lay=bad) == -1, bad
    assert call(four=False) == -1                          # 16 bits
    assert G.gr_cache_attend(B, 1, 8, 512, 64, A, None, F, 4, 3, F, F, 5, 0.1, 0, C, D, 512, 64, E, 0) == -2
    assert call(dtype=G.GR_F32) == -1 and call(dtype=G.GR_Q4) == -1 and call(heads=7) == -1 and call(heads=0) == -1 and call(heads=1026) == -1
    assert call(rows=-1) == -1 and call(tokens=-1) == -1 and call(width=-1) == -1 and call(window=-1) == -1 and call(rows=(1 << 20) + 1) == -1
    assert call(width=1 << 27) == -1 and call(rows=1 << 20, width=1 << 11) == -1 and call(tokens=1 << 29) == -1
    assert call(scale=float("nan")) == -1 and call(scale=float("inf")) == -1 and call(scale=2e38) == -1 and call(scale=-2e38) == -1
    assert call(qt=-1) == -1 and call(qh=-1) == -1 and call(qt=1 << 60) == -1 and call(oh=63) == -1 and call(ot=511) == -1
    for name in ("q", "cache", "table", "off", "pos", "ws", "out", "status"):
        assert call(**{name: 0}) == -2, name
    assert call(q=B + 1) == -3 and call(out=D + 1) == -3 and call(ws=C + 16) == -3 and call(cache=A + 8) == -3
    assert call(out=A + 64) == -1 and call(out=B) == -1 and call(out=B + 4 * 1024) == -1
    assert call(rows=0) == 0 and call(rows=0, q=0, ws=0) == 0
    assert G.gr_attend_workspace_bytes(2, 8, 64, 3, 5) > 0
    for bad in ((0, 8, 64, 3, 5), (3, 8, 64, 3, 5), (2, 8, 48, 3, 5), (2, 8, 288, 3, 5), (2, 8, 64, -1, 5), (2, 8, 64, 3, -5)):
        assert G.gr_attend_workspace_bytes(*bad) == 0, bad


def test_tensor_front_ends_want_cuda_tensors():
    x = torch.zeros(2, 1, 32)
    with pytest.raises(G.GrError):
        G.KVCache.empty(1, 12, 1, 32, torch.uint8, device="cpu")
    with pytest.raises(G.GrError):
        G.KVCache.empty(1, 8, 1, 48, torch.uint8, device="cpu")
    with pytest.raises(G.GrError):
        G.KVCache.empty(1, 8, 1, 32, torch.float64, device="cpu")
    for dtype in (torch.uint8, torch.bfloat16):
        cache = G.KVCache.empty(1, 8, 1, 32, dtype, device="cpu")
        assert len(cache.tensors()) == (1 if dtype is torch.uint8 else 2)
        with pytest.raises(G.GrError):
            G.cache_append(cache, x, x, torch.zeros(2, dtype=torch.int64))
        with pytest.raises(G.GrError):
            G.cache_read(cache, torch.zeros(2, dtype=torch.int64))


def test_the_model_of_the_cache():
    """Bytes of an octet are each in one place; what is written is read, within half a step of its group (a step where the largest
    magnitude is of the other sign: the codes end at 7)."""
    for dim in (32, 96, 256):
        byte, shift, word = P.tables(dim)
        codes = {(int(b), int(z)) for b, z in zip(byte.reshape(-1), shift.reshape(-1))}
        scales = {(int(w) * 2 + i, z) for w in word.reshape(-1) for i in range(2) for z in (0, 4)}
        assert len(codes) == 16 * dim and len(scales) == 2 * dim and not codes & scales and len(codes | scales) == 18 * dim
    rng = np.random.default_rng(1)
    data = np.zeros((3, 2, 2, 9 * 64), np.uint8)
    k, v = rng.normal(size=(2, 5, 2, 64)).astype(np.float32)
    slots = [0, 47, 17, 16, 8]
    for z, a, b in zip(slots, k, v):
        P.write4(data, 16, z, a, b)
    for got, x in zip(P.read4(data, 16, slots), (k, v)):
        step = np.abs(x.reshape(5, 2, 2, 32)).max(-1).repeat(32, -1).reshape(5, 2, 64) / 8
        assert (np.abs(got - x) <= step * (1 + 2.0 ** -9)).all()


def test_token_logprobs():
    ok = dict(logits=A, dtype=G.GR_F32, V=1000, ld=1000, rows=4, T=1.0, tokens=B, given=2, top=5, lp=C, ent=D, tok=E, tlp=F, st=F)

    def call(**kw):
        a = dict(ok); a.update(kw)
        return G.gr_token_logprobs(a["logits"], a["dtype"], a["V"], a["ld"], a["rows"], a["T"], a["tokens"], a["given"], a["top"], a["lp"], a["ent"],
                                   a["tok"], a["tlp"], a["st"], 0)

    assert call(V=0) == -1 and call(V=(1 << 21) + 1, ld=1 << 22) == -1 and call(ld=999) == -1 and call(dtype=G.GR_F16) == -1 and call(dtype=G.GR_Q4) == -1
    assert call(rows=-1) == -1 and call(rows=(1 << 26) + 1) == -1 and call(T=0.0) == -1 and call(T=-1.0) == -1 and call(T=float("nan")) == -1 and call(T=float("inf")) == -1
    assert call(given=-1) == -1 and call(given=65) == -1 and call(top=-1) == -1 and call(top=129) == -1
    for name in ("logits", "tokens", "lp", "tok", "tlp", "st"):
        assert call(**{name: 0}) == -2, name
    assert call(logits=A + 2) == -3 and call(logits=A + 1, dtype=G.GR_BF16) == -3
    assert call(rows=0) == 0 and call(rows=0, logits=0) == 0
    with pytest.raises(G.GrError):
        G.token_logprobs(torch.zeros(2, 5))
