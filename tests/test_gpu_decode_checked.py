"""The operators around a decoding step through the bounds-checked build of the library, in a child process: no access is
skipped, and the results are those of the regular build."""
import json
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu

CHILD = r"""
import json, sys
sys.path.insert(0, %(root)r)
import torch
import paper_2511_15898_b200.binding as Bn
from paper_2511_15898_b200.build import build_library
Bn._LIB_PATH = build_library(check=bool(%(checked)d))
import paper_2511_15898_b200 as G
out = []
def gen(seed):
    g = torch.Generator(device="cuda"); g.manual_seed(seed); return g
for dtype in (torch.float32, torch.bfloat16):
    for B, W, V, K in ((1, 1, 1, 1), (3, 2, 5, 10), (2, 32, 1025, 64), (1, 5, 2049, 128), (70, 9, 8191, 18), (2, 6, 50257, 12),
                       (300, 4, 1031, 4), (1, 32, 32001, 128), (700, 1, 20001, 8)):
        g = gen(V + K)
        x = (3 * torch.randn(B, W, V, generator=g, device="cuda")).to(dtype)
        s = -5 * torch.rand(B, W, generator=g, device="cuda")
        r = G.beam_select(x, s, K)
        out.append([r.status.tolist(), r.token.tolist(), r.parent.tolist()])
        y = x.sort(dim=2).values.contiguous()                       # lists that overflow
        y[0, 0] = float(y[0, 0, 0])                                     # a row of ties
        r = G.beam_select(y, s, K)
        out.append([r.status.tolist(), r.token.tolist(), r.parent.tolist()])
        r = G.beam_select(x[:1, :1].expand(B, W, V).contiguous(), torch.zeros(B, W, device="cuda"), K)    # sums taken again
        out.append([r.status.tolist(), r.token.tolist(), r.parent.tolist()])
for rows, beams, width, blocks, block in ((1, 1, 1, 1, 1), (12, 4, 7, 40, 8), (96, 32, 20, 900, 5), (1030, 1, 9, 4000, 7), (1536, 3, 9, 6000, 7),
                                          (64, 8, 33, 500, 16)):
    g = gen(rows)
    t = G.BlockTables.empty(rows, width, blocks, block, beams)
    def ints(lo, hi, n=rows): return torch.randint(lo, hi + 1, (n,), generator=g, device="cuda", dtype=torch.int32)
    for step in range(6):
        a = ints(0, 2 * block)
        p = G.block_plan(t, a, int(a.sum()) + (40000 if step == 3 else 0), keep=ints(0, width * block) if step %% 2 else None,
                         parents=ints(-1, beams - 1) if step %% 3 == 2 else None)
        out.append([p.status.tolist(), p.slots[:500].tolist(), p.copy_dst.tolist(), t.refs.tolist()])
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
