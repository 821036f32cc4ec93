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
