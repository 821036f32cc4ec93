"""Refusals of the operators around a decoding step: what the C entry points and the tensor front end reject on the host,
before anything is launched.  No GPU needed."""
import pytest
import torch

import paper_2511_15898_b200 as G
from paper_2511_15898_b200.build import build_library
from tests import block_pool

A = 1 << 20                      # any aligned non-null address: nothing is dereferenced on these paths


@pytest.fixture(scope="module", autouse=True)
def lib():
    build_library()
    return G.load_library()


def test_beam_select():
    ok = dict(logits=A, dtype=G.GR_F32, V=1000, ld=1000, beams=4, batch=2, T=1.0, scores=A, lengths=0, done=0, eos=-1,
              penalty=0.0, select=8, ws=A, tok=A, par=A, sc=A, ln=0, fin=A, st=A)

    def call(**kw):
        a = dict(ok); a.update(kw)
        return G.gr_beam_select(a["logits"], a["dtype"], a["V"], a["ld"], a["beams"], a["batch"], a["T"], a["scores"],
                                a["lengths"], a["done"], a["eos"], a["penalty"], a["select"], a["ws"], a["tok"], a["par"],
                                a["sc"], a["ln"], a["fin"], a["st"], 0)

    assert call(V=0) == -1 and call(V=(1 << 21) + 1, ld=1 << 22) == -1 and call(ld=999) == -1 and call(dtype=2) == -1
    assert call(beams=0) == -1 and call(beams=33) == -1 and call(select=0) == -1 and call(select=129) == -1
    assert call(batch=-1) == -1 and call(T=0.0) == -1 and call(T=float("nan")) == -1 and call(T=float("inf")) == -1
    assert call(penalty=1.0) == -1 and call(penalty=33.0, lengths=A) == -1 and call(penalty=float("nan"), lengths=A) == -1
    assert call(eos=1000) == -1 and call(eos=-2) == -1 and call(done=A) == -1
    for name in ("logits", "scores", "ws", "tok", "par", "sc", "fin", "st"):
        assert call(**{name: 0}) == -2, name
    assert call(logits=A + 2) == -3 and call(ws=A + 8) == -3 and call(logits=A + 1, dtype=G.GR_BF16) == -3
    assert call(batch=0) == 0
    assert G.gr_beam_workspace_bytes(1000, 4, 8, 2) > 0 and G.gr_beam_workspace_bytes(1000, 33, 8, 2) == 0
    assert G.gr_beam_workspace_bytes(0, 4, 8, 2) == 0 and G.gr_beam_workspace_bytes(1000, 4, 129, 2) == 0
    # a larger batch never needs less
    sizes = [G.gr_beam_workspace_bytes(50257, 4, 8, b) // b for b in (1, 3, 40, 400)]
    assert sizes == sorted(sizes, reverse=True)


def _layout(**kw):
    a = dict(batch=2, beams_in=4, beams_out=4, parts=3, src_group=4096, src_beam=1024, src_part=128, dst_group=4096,
             dst_beam=1024, dst_part=128, part_bytes=128, token_bytes=16)
    a.update(kw)
    return G.StateLayout(*[a[n] for n, _ in G.StateLayout._fields_])


def test_reorder_states():
    def call(src=(A,), dst=(A,), parents=A, lengths=0, **kw):
        return G.gr_reorder_states(list(src), list(dst), _layout(**kw), parents, lengths, 0)

    assert G.gr_reorder_states([A], [A], None, A, 0, 0) == -2
    assert call(parents=0) == -2 and call(src=(0,)) == -2 and call(dst=(0,)) == -2
    assert call(beams_in=0) == -1 and call(beams_in=33) == -1 and call(beams_out=33) == -1 and call(beams_out=0) == -1
    assert call(batch=-1) == -1 and call(parts=-1) == -1 and call(part_bytes=-1) == -1 and call(src_beam=-16) == -1
    assert call(lengths=A, token_bytes=0) == -1 and call(lengths=A, token_bytes=48) == -1
    assert call(beams_in=3) == -1                                  # in place, more states than there are
    assert call(dst_beam=512, dst_group=2048) == -1                # in place at other strides
    assert call(src=(A, A), dst=(A, A)) == -1                      # the same tensor twice
    assert call(src=(A, A + 64), dst=(A, A + 64)) == -1            # two that overlap
    assert call(src=(A, A + 99999), dst=(A, A + 8192)) == -1       # some in place, some not
    B = A + (1 << 24)
    assert call(dst=(A + 7551,)) == -1 and call(src=(A, A + 16384), dst=(B, A + 7040)) == -1    # a dst that meets a src (7552 bytes)
    assert call(dst=(B,), dst_beam=0) == -1 and call(dst=(B,), dst_part=64) == -1 and call(dst=(B,), dst_group=1024) == -1
    assert call(dst=(B,), dst_beam=1 << 47) == -1 and call(part_bytes=1 << 47) == -1
    assert call(batch=1 << 20, parts=1 << 12, src_group=1 << 22, dst_group=1 << 22) == -1
    assert call(batch=0) == 0 and call(parts=0) == 0 and call(part_bytes=0) == 0 and call(src=(), dst=()) == 0
    with pytest.raises(G.GrError):
        G.gr_reorder_states([A, A], [A], _layout(), A, 0, 0)


def test_block_plan():
    ok = dict(table=A, rows=8, width=4, beams=2, bs=16, lengths=A, refs=A, blocks=10, parents=A, keep=0, append=A, tokens=4,
              ws=A, slots=A, pos=A, off=A, src=A, dst=A, st=A)

    def call(**kw):
        a = dict(ok); a.update(kw)
        return G.gr_block_plan(a["table"], a["rows"], a["width"], a["beams"], a["bs"], a["lengths"], a["refs"], a["blocks"],
                               a["parents"], a["keep"], a["append"], a["tokens"], a["ws"], a["slots"], a["pos"], a["off"],
                               a["src"], a["dst"], a["st"], 0)

    assert call(rows=-2) == -1 and call(rows=7) == -1 and call(rows=(1 << 20) + 2) == -1 and call(width=-1) == -1
    assert call(beams=0) == -1 and call(beams=33, rows=33) == -1 and call(bs=0) == -1 and call(blocks=-1) == -1
    assert call(blocks=(1 << 26) + 1) == -1 and call(tokens=-1) == -1
    assert call(rows=1 << 16, width=1 << 15) == -1 and call(width=1 << 16, bs=1 << 15) == -1
    for name in ("table", "lengths", "refs", "append", "ws", "slots", "pos", "off", "src", "dst", "st"):
        assert call(**{name: 0}) == -2, name
    assert call(ws=A + 4) == -3
    assert call(rows=0, tokens=0) == 0
    assert G.gr_block_workspace_bytes(-1, 4) == 0 and G.gr_block_workspace_bytes(4, -1) == 0
    assert G.gr_block_workspace_bytes(4, 4) > 0


def test_copy_blocks():
    def call(caches=(A,), blocks=10, stride=256, size=256, src=A, dst=A, pairs=4):
        return G.gr_copy_blocks(list(caches), blocks, stride, size, src, dst, pairs, 0)

    assert call(blocks=-1) == -1 and call(stride=128) == -1 and call(size=-1) == -1 and call(pairs=-1) == -1
    assert call(stride=1 << 45) == -1
    assert call(caches=(A, A)) == -1 and call(caches=(A, A + 128)) == -1
    assert call(caches=(0,)) == -2 and call(src=0) == -2 and call(dst=0) == -2
    assert call(pairs=(1 << 24) + 1) == -5
    assert call(blocks=0) == 0 and call(pairs=0) == 0 and call(size=0) == 0 and call(caches=()) == 0


def test_strerror():
    for code in (8, 9, 10):
        assert G.gr_strerror(code) not in ("", "unknown code")


def test_tensor_front_end_refuses_what_is_not_on_the_device():
    i32 = torch.int32
    with pytest.raises(G.GrError):
        G.beam_select(torch.zeros(1, 2, 8), torch.zeros(1, 2))
    with pytest.raises(G.GrError):
        G.reorder_states([torch.zeros(1, 2, 8)], torch.zeros(1, 2, dtype=i32))
    with pytest.raises(G.GrError):
        G.block_plan(G.BlockTables.empty(2, 2, 4, 4, device="cpu"), torch.zeros(2, dtype=i32), 2)
    with pytest.raises(G.GrError):
        G.copy_blocks([torch.zeros(4, 8)], torch.zeros(1, dtype=i32), torch.zeros(1, dtype=i32))
    assert G.reorder_states([], torch.zeros(1, 2, dtype=i32)) == []
    G.copy_blocks([], torch.zeros(1, dtype=i32), torch.zeros(1, dtype=i32))


def test_plain_model_keeps_its_books():
    """The model that the GPU plans are compared with: counts equal the tables' entries, and rows read what was written for
    them, through forks, copies and releases."""
    import random
    for seed in range(30):
        rng = random.Random(seed)
        beams, groups, block, width = rng.choice([1, 2, 3, 5]), rng.randint(1, 4), rng.choice([1, 3, 4, 8]), rng.randint(1, 8)
        R, N = beams * groups, rng.randint(1, 60)
        table, lengths, refs = [[-1] * width for _ in range(R)], [0] * R, [0] * N
        cache = [[None] * block for _ in range(N)]
        text = [[] for _ in range(R)]
        for step in range(25):
            append = [rng.choice([0, 1, 1, 2, rng.randint(0, 2 * block)]) for _ in range(R)]
            parents = [rng.randint(-1, beams - 1) for _ in range(R)] if rng.random() < 0.6 else None
            keep = [rng.randint(0, width * block) for _ in range(R)] if rng.random() < 0.5 else None
            before = [list(t) for t in text]
            total = sum(append)
            slots, positions, offsets, src, dst, status = block_pool.plan(table, lengths, refs, block, beams, append, total, keep, parents)
            for r in range(R):                                # copies first, then the new tokens
                if src[r] >= 0:
                    cache[dst[r]] = list(cache[src[r]])
            for r in range(R):
                p = r if parents is None else (r // beams * beams + parents[r] if parents[r] >= 0 else None)
                old = [] if p is None else before[p]
                text[r] = old[:min(len(old), keep[r])] if keep is not None else list(old)
                for i in range(offsets[r], offsets[r + 1]):
                    if slots[i] >= 0:
                        token = (step, r, i)
                        assert positions[i] == len(text[r])
                        cache[slots[i] // block][slots[i] % block] = token
                        text[r].append(token)
            counts = [0] * N
            for r in range(R):
                assert lengths[r] == len(text[r])
                held = -(-lengths[r] // block)
                assert all(b >= 0 for b in table[r][:held]) and all(b == -1 for b in table[r][held:])
                for b in table[r][:held]:
                    counts[b] += 1
            assert counts == refs
            for r in range(R):
                assert [cache[table[r][t // block]][t % block] for t in range(lengths[r])] == text[r], (seed, step, r)
