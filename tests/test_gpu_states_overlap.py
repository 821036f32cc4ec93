"""Lists of tensors that share bytes are refused by the tensor front ends and left as they are, tensors that lie between one another's
pieces are taken."""
import pytest
import torch

import paper_2511_15898_b200 as G
import paper_2511_15898_b200.binding as Bn
from paper_2511_15898_b200.build import build_library
from tests.test_gpu_states import expected, rand, same

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def lib():
    build_library()


@pytest.fixture(params=["module", "python"], autouse=True)
def way(request, monkeypatch):
    if request.param == "python":
        monkeypatch.setattr(Bn, "_tensors", None)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def test_one_layout():
    x = rand((2, 4, 3, 5, 8), torch.float32, 1)
    keep, parents, n = x.clone(), ints([[1, 0, 3, 3], [2, 2, 0, 1]]), torch.full((2, 4), 5, dtype=torch.int32, device="cuda")
    for states in ([x[:, :, 0:2], x[:, :, 1:3]], [x[:, :, 0:1], x[:, :, 2:3], x[:, :, 2:3]]):
        with pytest.raises(G.GrError):
            G.reorder_states(states, parents, lengths=n, token_dim=3)
    with pytest.raises(G.GrError):
        G.copy_blocks([x.view(8, 120)[:6], x.view(8, 120)[1:7]], ints([0]), ints([3]))
    torch.cuda.synchronize()
    assert same(x, keep)
    states = [x[:, :, 2:3], x[:, :, 0:1], x[:, :, 1:2]]
    G.reorder_states(states, parents, lengths=n, token_dim=3)
    torch.cuda.synchronize()
    assert same(x, expected(keep, parents, n, 3))
    # every second block of a pool
    pool = rand((12, 7), torch.float32, 2)
    keep = pool.clone()
    G.copy_blocks([pool[::2], pool[1::2]], ints([0, -1, 4]), ints([3, 2, 5]))
    torch.cuda.synchronize()
    keep[6:8], keep[10:12] = keep[0:2].clone(), keep[8:10].clone()
    assert same(pool, keep)


def test_several_layouts():
    x = rand((2, 4, 3, 40), torch.float32, 1)
    keep, parents = x.clone(), ints([[1, 0, 3, 3], [2, 2, 0, 1]])
    other = rand((2, 4, 9), torch.float32, 2)
    first = other.clone()
    n = torch.full((2, 4), 3, dtype=torch.int32, device="cuda")
    for call in (lambda: G.reorder_states([x, x[:, :, 1:]], parents),                                   # (one begins within the other)
                 lambda: G.reorder_states([other, x[:, :, 0, :8], x[:, :, 0, 7:]], parents),
                 lambda: G.reorder_states([other, x[:, :, 0].expand(2, 4, 40)[:1].expand(2, 4, 40)], parents),   # (two groups in one place)
                 lambda: G.reorder_states([x[:, :, 0, :8], x[:, :, 0, 9:]], parents, out=[torch.zeros(2, 4, 8, device="cuda"), x[:, :, 1, 9:]]),
                 lambda: G.reorder_states([x[:, :, 0, :8], x[:, :, 0, 9:]], parents, out=[x[:, :, 0, 20:28], torch.zeros(2, 4, 31, device="cuda")]),
                 lambda: G.reorder_states([other, x], parents, out=[torch.zeros_like(other), x]),
                 lambda: G.copy_blocks([other.view(8, 9), x.view(24, 40), x.view(8, 120)], ints([0]), ints([1])),
                 lambda: G.copy_blocks([other.view(8, 9), x.view(8, 120)[:, :50], x.view(8, 120)[:, 49:]], ints([0]), ints([1]))):
        with pytest.raises(G.GrError):
            call()
    torch.cuda.synchronize()
    assert same(x, keep) and same(other, first)
    # parts of one row of different lengths, and a tensor of its own
    states = [x[:, :, 0, :8], x[:, :, 0, 8:], x[:, :, 1:], other]
    want = [expected(t, parents) for t in states]
    G.reorder_states(states[:2] + [other], parents)
    G.reorder_states([states[2]], parents)
    torch.cuda.synchronize()
    assert all(same(a, b) for a, b in zip(states, want))
    # outs beside the states in one buffer
    buf = rand((5000,), torch.float32, 3)
    a, b, c, d = buf[:64].view(2, 4, 8), buf[64:136].view(2, 4, 9), buf[136:200].view(2, 4, 8), buf[200:272].view(2, 4, 9)
    want = [expected(a, parents, out=c), expected(b, parents, out=d)]
    G.reorder_states([a, b], parents, out=[c, d])
    torch.cuda.synchronize()
    assert same(c, want[0]) and same(d, want[1])
    # blocks of two sizes that lie in turn
    pool = rand((10, 30), torch.float32, 4)
    keep = pool.clone()
    G.copy_blocks([pool[:, :11], pool[:, 11:], x.view(24, 40)[:10]], ints([2]), ints([7]))
    torch.cuda.synchronize()
    keep[7] = keep[2]
    assert same(pool, keep)
