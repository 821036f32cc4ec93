"""More of the operators around a decoding step through the bounds-checked build, in a child process: long slot maps, forked tables in
parts, states and copies of blocks in every vector width, and sums of a beam selection that are taken again.  No access is skipped, and
the results are those of the regular build."""
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
def gen(seed):
    g = torch.Generator(device="cuda"); g.manual_seed(seed); return g
def digest(*t):
    return hashlib.sha256(b"".join(x.contiguous().view(torch.uint8).cpu().numpy().tobytes() for x in t)).hexdigest()
def skipped():
    torch.cuda.synchronize()
    return lib.gr_states_check() if checked else 0
for rows, beams, width, blocks, block, tokens in ((7, 1, 900, 5000, 16, 8193), (48, 4, 300, 9000, 8, 32769), (4, 4, 9000, 30000, 7, 40003),
                                                  (1100, 4, 60, 40000, 3, 50002), (1026, 2, 40, 30000, 6, 9001), (6, 2, 40, 400, 1, 200)):
    g = gen(rows)
    t = G.BlockTables.empty(rows, width, blocks, block, beams)
    for step in range(4):
        a = torch.randint(0, 2 * tokens // rows + 1, (rows,), generator=g, device="cuda", dtype=torch.int32)
        p = G.block_plan(t, a, tokens, keep=torch.randint(0, width * block, (rows,), generator=g, device="cuda", dtype=torch.int32) if step else None,
                         parents=torch.randint(-1, beams, (rows,), generator=g, device="cuda", dtype=torch.int32) if step %% 2 else None)
        out.append([p.status.tolist(), digest(p.slots, p.positions, p.offsets, p.copy_src, p.copy_dst, t.table, t.lengths, t.refs)])
for dtype in (torch.float64, torch.float32, torch.bfloat16, torch.uint8):
    for W, shape in ((1, (5,)), (3, (2, 7, 33)), (4, (1, 40001)), (8, (3, 16, 8)), (13, (64, 2, 4)), (32, (129,)), (20, (2, 9, 16))):
        g = gen(W)
        B = 3
        x = [(100 * torch.rand((B, W) + shape, generator=g, device="cuda")).to(dtype) for _ in range(3)]
        parents = torch.randint(-1, W, (B, W), generator=g, device="cuda", dtype=torch.int32)
        G.reorder_states(x, parents)
        made = [torch.zeros((B, 5) + shape, dtype=dtype, device="cuda") for _ in x]
        G.reorder_states(x, parents[:, :1].expand(B, 5).contiguous(), out=made)
        n = torch.randint(-1, 70, (B, W), generator=g, device="cuda", dtype=torch.int32)
        for d in range(2, 2 + len(shape)):
            G.reorder_states(x, parents, lengths=n, token_dim=d)
        out.append([[7 if skipped() else 0], digest(*x, *made)])
    for blocks, shape, pairs in ((9, (1,), 4), (600, (16, 33), 280), (64, (8, 16, 128), 20), (700, (5,), 600)):
        g = gen(blocks)
        caches = [(100 * torch.rand((blocks,) + shape, generator=g, device="cuda")).to(dtype) for _ in range(3)]
        order = torch.randperm(blocks, generator=g, device="cuda").int()
        half = min(pairs, blocks // 2)
        src, dst = torch.full((pairs,), -1, dtype=torch.int32, device="cuda"), torch.full((pairs,), blocks, dtype=torch.int32, device="cuda")
        dst[:half], src[:half] = order[:half], order[half:2 * half]
        G.copy_blocks(caches, src, dst)
        if shape[0] > 4:
            G.copy_blocks([c[:, 1:4] for c in caches], src, dst)
        out.append([[7 if skipped() else 0], digest(*caches)])
for dtype in (torch.float32, torch.bfloat16):
    for B, W, V, K in ((1, 3, 5, 4), (3, 8, 20011, 16), (40, 4, 3001, 8), (200, 5, 1031, 9), (400, 3, 2053, 3)):
        x = (10 * torch.randn(B, W, 1, generator=gen(B), device="cuda")).expand(B, W, V).to(dtype).contiguous()
        x[:, :, ::7] += 1e30 if B == 40 else 2.0                       # (sums of no use, rows that err)
        if B == 200:
            x[5, 1, 3] = float("nan")
        r = G.beam_select(x, torch.full((B, W), -2.0, device="cuda"), K)
        out.append([r.status.tolist(), digest(r.token, r.parent, r.score)])
print("RESULT " + json.dumps(out))
"""


def _run(checked: int):
    res = subprocess.run([sys.executable, "-c", CHILD % {"root": ROOT, "checked": checked}], capture_output=True, text=True, timeout=900)
    assert res.returncode == 0, res.stdout[-2000:] + res.stderr[-4000:]
    return json.loads([ln for ln in res.stdout.splitlines() if ln.startswith("RESULT ")][-1][len("RESULT "):])


def test_checked_build_reports_nothing_and_agrees():
    chk, ref = _run(1), _run(0)
    GR_CHECK_FAILED = 7
    for i, (a, b) in enumerate(zip(chk, ref)):
        assert GR_CHECK_FAILED not in a[0], i
        assert a == b, i
