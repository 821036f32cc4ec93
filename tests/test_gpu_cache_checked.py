"""The operators that fill and read a paged cache, and log probabilities, through the bounds-checked build, in a child process: what the kernels read and write in
the tensors they are given, in the workspace and in shared memory.  No access is skipped, and the results are those of the regular build."""
import json
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu

CHILD = r"""
import hashlib, json, sys
sys.path.insert(0, %(root)r)
import torch
import paper_2511_15898_b200.binding as Bn
from paper_2511_15898_b200.build import build_library
checked = bool(%(checked)d)
Bn._LIB_PATH = build_library(check=checked)
import paper_2511_15898_b200 as G
lib = G.load_library()
out = []
DT = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "q4": torch.uint8}
def gen(seed):
    g = torch.Generator(device="cuda"); g.manual_seed(seed); return g
def digest(*t):
    return hashlib.sha256(b"".join(x.contiguous().view(torch.uint8).cpu().numpy().tobytes() for x in t)).hexdigest()
def skipped():
    torch.cuda.synchronize()
    return lib.gr_cache_check() + lib.gr_attend_check() if checked else 0
def rows(g, T, heads, D, dtype, shift):
    # (a head's elements next to one another, off the vectors' alignment)
    x = torch.randn(T, heads * D + shift + 3, generator=g, device="cuda").to(DT[dtype])
    return x[:, shift:shift + heads * D].unflatten(1, (heads, D))
for T, H, Hq, D, rot, bs, dtype, cache, inter, shift in (
        (1, 1, 1, 64, 64, 16, "bf16", "bf16", 0, 5), (33, 3, 6, 128, 128, 16, "bf16", "bf16", 1, 0), (40, 2, 0, 128, 64, 5, "f16", "f16", 0, 5), (19, 2, 5, 80, 80, 1, "f32", "f32", 0, 1),
        (19, 2, 5, 80, 24, 7, "f32", "bf16", 1, 5), (9, 1, 2, 2, 2, 3, "bf16", "f32", 0, 5), (9, 1, 2, 6, 2, 3, "bf16", "f16", 1, 5), (17, 2, 2, 66, 34, 16, "bf16", "bf16", 1, 5),
        (12, 1, 3, 512, 512, 8, "bf16", "bf16", 0, 5), (50, 2, 2, 96, 0, 32, "bf16", "bf16", 0, 5), (2500, 2, 4, 64, 64, 16, "bf16", "bf16", 0, 5), (2501, 1, 1, 128, 96, 64, "f16", "f32", 1, 5),
        (9000, 3, 5, 128, 128, 16, "bf16", "bf16", 0, 5), (1, 1, 0, 32, 32, 8, "bf16", "q4", 0, 5), (7, 2, 3, 64, 64, 16, "f16", "q4", 0, 5), (50, 1, 1, 96, 48, 24, "bf16", "q4", 1, 5),
        (30, 2, 3, 128, 64, 16, "f32", "q4", 0, 1), (21, 1, 2, 256, 256, 8, "bf16", "q4", 1, 5), (20, 1, 1, 160, 0, 40, "f32", "q4", 0, 1), (23, 1, 1, 224, 222, 16, "f32", "q4", 0, 1),
        (2400, 1, 3, 64, 64, 16, "bf16", "q4", 0, 5), (9601, 2, 0, 128, 64, 24, "f16", "q4", 0, 5), (37890, 1, 0, 32, 32, 40, "bf16", "q4", 0, 5), (38000, 8, 0, 64, 64, 16, "bf16", "q4", 0, 5)):
    g = gen(T + D)
    N = -(-T // bs) + 3
    slots = torch.randperm(N, generator=g, device="cuda").repeat_interleave(bs) * bs + torch.arange(N * bs, device="cuda") %% bs
    slots = slots[2:T + 2].clone()
    slots[::7] = torch.randint(-9, 1 << 40, (len(slots[::7]),), generator=g, device="cuda") * 1000003 + N * bs
    positions = torch.randint(-2, 100000, (T,), generator=g, device="cuda", dtype=torch.int32)
    freq = 10000.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot) if rot else None
    for off in (0, shift):
        kv = G.KVCache.empty(N, bs, H, D, DT[cache])
        k, v = rows(g, T, H, D, dtype, off), rows(g, T, H, D, dtype, 0)
        q = rows(g, T, Hq, D, dtype, off) if Hq else None
        G.cache_append(kv, k, v, slots, positions, freq, interleaved=bool(inter), q=q, q_out=q)
        got = [digest(*kv.tensors(), *([q] if Hq else []))]
        for t in ("f32", "bf16", "f16"):
            to = rows(g, T, H, D, t, off), rows(g, T, H, D, t, 0)
            G.cache_read(kv, slots, out=to)
            got.append(digest(*to))
        out.append([[7 if skipped() else 0], got])
for D in (32, 64, 96, 128, 160, 192, 224, 256):
    for H, group, dtype, bs, lengths, news in ((2, 1, "bf16", 8, [1, 17, 64, 200, 333], [1] * 5), (1, 5, "f16", 24, [5, 70, 2000], [3, 2, 1]), (1, 4, "bf16", 16, [9, 500, 64, 1500], [9, 0, 20, 9]),
                                               (1, 16, "f16", 16, [300, 40], [5, 40]), (8, 4, "bf16", 16, [900], [1]), (2, 8, "f16", 64, [40000], [1])):
        if lengths[0] == 40000 and D not in (64, 128):
            continue
        g = gen(D + group)
        N = sum(-(-n // bs) for n in lengths) + 2
        width = -(-max(lengths) // bs)
        kv = G.KVCache.empty(N, bs, H, D, torch.uint8)
        k, v = (torch.randn(N * bs, H, D, generator=g, device="cuda") for _ in range(2))
        v[::13] *= 500
        G.cache_append(kv, k, v, torch.arange(N * bs, device="cuda"))
        order, table, at = torch.randperm(N, generator=g, device="cuda").int(), torch.full((len(lengths), width), -1, dtype=torch.int32, device="cuda"), 0
        for r, n in enumerate(lengths):
            table[r, :-(-n // bs)] = order[at:at + -(-n // bs)]
            at += -(-n // bs)
        offsets = torch.tensor([0, *torch.tensor(news).cumsum(0).tolist()], dtype=torch.int32, device="cuda")
        positions = torch.cat([torch.arange(n - m, n, dtype=torch.int32, device="cuda") for n, m in zip(lengths, news)])
        q = rows(g, sum(news), H * group, D, dtype, 0)
        for window, offs, where in ((0, offsets, positions), (45, offsets, positions), (0, offsets.flip(0).contiguous(), positions + width * bs), (0, offsets, positions - 2000)):
            r = G.cache_attend(q, kv, table, offs, where, window=window)
            clean = offs is offsets
            out.append([r.status.tolist() + [7 if skipped() else 0], digest(r.out) if clean else ""])
for dtype in ("f32", "bf16"):
    for R, V, given, top in ((1, 1, 1, 1), (5, 7, 1, 7), (4, 1023, 3, 20), (3, 1025, 64, 128), (2, 50257, 1, 128), (9, 128256, 2, 20), (20, 33001, 1, 1), (300, 9001, 1, 0), (700, 5011, 1, 48), (2500, 3001, 1, 8)):
        x = (4 * torch.randn(R, V, generator=gen(V), device="cuda")).to(DT[dtype])
        if R > 4:
            x[3, V // 2], x[4] = float("nan"), float("-inf")
        r = G.token_logprobs(x, torch.randint(-1, V + 1, (R, given), generator=gen(R), device="cuda", dtype=torch.int32), top)
        out.append([r.status.tolist(), digest(r.logprob, r.entropy, r.top_token, r.top_logprob)])
print("RESULT " + json.dumps(out))
"""


def _run(checked: int):
    res = subprocess.run([sys.executable, "-c", CHILD % {"root": ROOT, "checked": checked}], capture_output=True, text=True, timeout=900)
    assert res.returncode == 0, res.stdout[-2000:] + res.stderr[-4000:]
    return json.loads([ln for ln in res.stdout.splitlines() if ln.startswith("RESULT ")][-1][len("RESULT "):])


def test_checked_build_reports_nothing_and_agrees():
    chk, ref = _run(1), _run(0)
    GR_CHECK_FAILED = 7
    assert len(chk) == len(ref) > 200
    for i, (a, b) in enumerate(zip(chk, ref)):
        assert GR_CHECK_FAILED not in a[0], i
        assert a == b, i
