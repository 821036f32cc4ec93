"""The two ways of the tensor front ends of caches and log probabilities (the compiled module's and the one in Python): the same results, and the same
refusals, whichever a call takes; what is refused writes nothing."""
import dataclasses

import pytest
import torch

import paper_2511_15898_b200 as G
import paper_2511_15898_b200.binding as Bn
from paper_2511_15898_b200.build import build_library

pytestmark = pytest.mark.gpu
I32 = dict(dtype=torch.int32, device="cuda")


@pytest.fixture(scope="module", autouse=True)
def lib():
    build_library()
    assert Bn._tensors is not None


def both(monkeypatch, call):
    first = call()
    with monkeypatch.context() as m:
        m.setattr(Bn, "_tensors", None)
        second = call()
    torch.cuda.synchronize()
    assert len(first) == len(second)
    for a, b in zip(first, second):
        assert torch.equal(a, b)


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _made(dtype):
    kv = G.KVCache.empty(9, 8, 2, 64, dtype)
    k, v, q = (torch.randn(20, h, 64, generator=gen(h), device="cuda").bfloat16() for h in (2, 2, 6))
    slots = torch.randperm(72, generator=gen(9), device="cuda")[:20]
    positions, freq = torch.arange(20, **I32), 0.5 ** torch.arange(32, dtype=torch.float64, device="cuda")
    return kv, k, v, q, slots, positions, freq


@pytest.mark.parametrize("dtype", [torch.uint8, torch.bfloat16, torch.float32])
def test_same_results_of_caches(monkeypatch, dtype):
    def call():
        kv, k, v, q, slots, positions, freq = _made(dtype)
        got = []
        for inter in (False, True):
            q_out = torch.zeros_like(q)
            G.cache_append(kv, k, v, slots, positions, freq, interleaved=inter, q=q, q_out=q_out)
            got += [q_out, G.cache_append(kv, k, v, slots, positions, freq[:8].contiguous(), inter, q)]
            G.cache_append(kv, v, k.transpose(0, 1).contiguous().transpose(0, 1), slots)
            got += [t.clone() for t in kv.tensors()]
        out = (torch.zeros(20, 2, 64, device="cuda"), torch.zeros(20, 2, 64, device="cuda"))
        got += [*G.cache_read(kv, slots), *G.cache_read(kv, slots, torch.float16), *G.cache_read(kv, slots, out=out)]
        part = G.KVCache(kv.keys[2:5], None if kv.values is None else kv.values[2:5], 8, 2, 64)
        got += [*G.cache_read(part, slots - 16)]
        if dtype is torch.uint8:
            table, offsets = torch.randperm(9, generator=gen(3), device="cuda").int().view(3, 3), torch.tensor([0, 5, 12, 20], **I32)
            at = torch.cat([torch.arange(n, 24, **I32) for n in (19, 17, 16)])
            r = G.cache_attend(q, kv, table, offsets, at)
            r.out.zero_()
            r = G.cache_attend(q, kv, table, offsets, at, out=r)
            got += [r.out.clone(), r.status.clone()]
            r = G.cache_attend(q, kv, table, offsets, at, scale=0.3, window=7, out=r)
            got += [r.out, r.status]
        return got
    both(monkeypatch, call)


def test_same_results_of_log_probabilities(monkeypatch):
    def call():
        got = []
        for dtype in (torch.float32, torch.bfloat16):
            x = torch.randn(7, 1001, generator=gen(1), device="cuda").to(dtype)
            t = torch.randint(0, 1001, (7, 3), generator=gen(2), **I32)
            for view in (x, x[:, :999], x[::2], x[:1, 3:]):
                given = t[:view.shape[0]].contiguous()
                r = G.token_logprobs(view, given, 5)
                r.top_token.fill_(-9)
                r = G.token_logprobs(view, given, 5, 0.7, out=r)
                one = G.token_logprobs(view, given[:, 0].contiguous(), 0, out=G.token_logprobs(view, given[:, 0].contiguous()))
                got += [r.logprob, r.entropy, r.top_token, r.top_logprob, r.status, one.logprob, one.entropy]
        return got
    both(monkeypatch, call)


def test_same_refusals(monkeypatch):
    kv, k, v, q, slots, positions, freq = _made(torch.uint8)
    wide = G.KVCache.empty(9, 8, 2, 64)
    table, offsets = torch.zeros(3, 3, **I32), torch.tensor([0, 5, 12, 20], **I32)
    r = G.cache_attend(q, kv, table, offsets, positions)
    x, t = torch.randn(4, 50, device="cuda"), torch.zeros(4, 2, **I32)
    lp = G.token_logprobs(x, t, 3)
    pair = (torch.zeros(20, 2, 64, device="cuda"), torch.zeros(20, 2, 64, device="cuda"))

    def cache(**kw):
        return G.KVCache(**{**dict(keys=kv.keys, values=None, block_size=8, heads=2, dim=64), **kw})

    wrong = [
        lambda: G.cache_append(cache(block_size=16), k, v, slots), lambda: G.cache_append(cache(heads=3), k, v, slots), lambda: G.cache_append(cache(dim=32), k, v, slots),
        lambda: G.cache_append(cache(values=kv.keys), k, v, slots), lambda: G.cache_append(cache(keys=kv.keys.cpu()), k, v, slots),
        lambda: G.cache_append(cache(keys=kv.keys.transpose(1, 2)), k, v, slots), lambda: G.cache_append(cache(keys=kv.keys.to(torch.int8)), k, v, slots),
        lambda: G.cache_append(G.KVCache(wide.keys, None, 8, 2, 64), k, v, slots), lambda: G.cache_append(G.KVCache(wide.keys, wide.values.float(), 8, 2, 64), k, v, slots),
        lambda: G.cache_append(G.KVCache(wide.keys, wide.keys, 8, 2, 64), k, v, slots), lambda: G.cache_append(G.KVCache(wide.keys[:1].expand(9, 8, 2, 64), wide.values[:1].expand(9, 8, 2, 64), 8, 2, 64), k, v, slots),
        lambda: G.cache_append(kv, k.double(), v, slots), lambda: G.cache_append(kv, k, v.float(), slots), lambda: G.cache_append(kv, k[:3], v, slots),
        lambda: G.cache_append(kv, k[:, :1], v, slots), lambda: G.cache_append(kv, k, v, slots.int()), lambda: G.cache_append(kv, k, v, slots[:3]),
        lambda: G.cache_append(kv, k.transpose(1, 2), v, slots), lambda: G.cache_append(kv, k, v, slots, positions.long(), freq), lambda: G.cache_append(kv, k, v, slots, None, freq),
        lambda: G.cache_append(kv, k, v, slots, positions, freq.float()), lambda: G.cache_append(kv, k, v, slots, positions, torch.ones(33, dtype=torch.float64, device="cuda")),
        lambda: G.cache_append(kv, k, v, slots, positions, freq, q=q.float(), q_out=q.float()), lambda: G.cache_append(kv, k, v, slots, positions, freq, q=q, q_out=q[:, :2]),
        lambda: G.cache_append(kv, k, v, slots, q_out=q), lambda: G.cache_append(kv, k, v, slots, q=q, q_out=q[:1].expand(20, 6, 64)), lambda: G.cache_append(wide, wide.keys.view(-1, 2, 64)[:20], v, slots),
        lambda: G.cache_append(kv, k, v, slots, q=q[:, :5], q_out=q.as_strided((20, 5, 64), (320, 64, 1))),
        lambda: G.cache_read(kv, slots.int()), lambda: G.cache_read(kv, slots, torch.float64), lambda: G.cache_read(kv, slots, out=(pair[0], pair[1].half())),
        lambda: G.cache_read(kv, slots, out=(pair[0], pair[0])), lambda: G.cache_read(kv, slots, out=(pair[0][:3], pair[1])), lambda: G.cache_read(kv, slots.view(4, 5)),
        lambda: G.cache_read(wide, slots, out=(wide.keys.view(-1, 2, 64)[:20], pair[1].bfloat16())), lambda: G.cache_read(cache(dim=96), slots),
        lambda: G.cache_attend(q, wide, table, offsets, positions, out=r), lambda: G.cache_attend(q.float(), kv, table, offsets, positions, out=r),
        lambda: G.cache_attend(q[:, :5], kv, table, offsets, positions, out=r), lambda: G.cache_attend(q[..., :32], kv, table, offsets, positions, out=r),
        lambda: G.cache_attend(q, kv, table.long(), offsets, positions, out=r), lambda: G.cache_attend(q, kv, table, offsets[:3], positions, out=r),
        lambda: G.cache_attend(q, kv, table, offsets, positions[:9], out=r), lambda: G.cache_attend(q, kv, table, offsets, positions, window=-1, out=r),
        lambda: G.cache_attend(q, kv, table, offsets, positions, scale=float("nan"), out=r), lambda: G.cache_attend(r.out, kv, table, offsets, positions, out=r),
        lambda: G.cache_attend(q.cpu(), kv, table, offsets, positions, out=r), lambda: G.cache_attend(q, cache(dim=128), table, offsets, positions, out=r),
        lambda: G.token_logprobs(x.half(), t, 3, out=lp), lambda: G.token_logprobs(x, t.long(), 3, out=lp), lambda: G.token_logprobs(x, t[:2], 3, out=lp),
        lambda: G.token_logprobs(x, t, 3, 0.0, out=lp), lambda: G.token_logprobs(x, t, 3, float("inf"), out=lp), lambda: G.token_logprobs(x, t, 129), lambda: G.token_logprobs(x, t, -1),
        lambda: G.token_logprobs(x.t(), t, 3, out=lp), lambda: G.token_logprobs(x.cpu(), t, 3, out=lp), lambda: G.token_logprobs(x[:1].expand(4, 50), t, 3, out=lp),
        lambda: G.token_logprobs(x, lp.top_token, 3, out=G.Logprobs(torch.zeros(4, 3, device="cuda"), lp.entropy, lp.top_token, lp.top_logprob, lp.status, (4, 3, 3))),
        lambda: G.token_logprobs(x, torch.zeros(4, 65, **I32)),
        # results whose parts were replaced by ones that do not hold what the call writes
        lambda: G.cache_attend(q, kv, table, offsets, positions, out=dataclasses.replace(r, workspace=r.workspace[:-1])),
        lambda: G.cache_attend(q, kv, table, offsets, positions, out=dataclasses.replace(r, workspace=r.workspace[::2])),
        lambda: G.cache_attend(q, kv, table, offsets, positions, out=dataclasses.replace(r, out=r.out[:9])),
        lambda: G.cache_attend(q, kv, table, offsets, positions, out=dataclasses.replace(r, status=r.status[:2])),
        lambda: G.cache_attend(q, kv, table, offsets, positions, out=dataclasses.replace(r, status=r.status.short())),
        lambda: G.token_logprobs(x, t, 3, out=dataclasses.replace(lp, logprob=lp.logprob.half())),
        lambda: G.token_logprobs(x, t, 3, out=dataclasses.replace(lp, entropy=lp.entropy[:3])),
        lambda: G.token_logprobs(x, t, 3, out=dataclasses.replace(lp, top_token=lp.top_token.t())),
        lambda: G.token_logprobs(x, t, 3, out=dataclasses.replace(lp, top_logprob=lp.top_logprob.cpu())),
        lambda: G.token_logprobs(x, t, 3, out=dataclasses.replace(lp, status=lp.status.short())),
    ]
    kept = [z.clone() for z in (kv.keys, wide.keys, wide.values, q, r.out, lp.logprob, lp.top_token, *pair)]
    for i, call in enumerate(wrong):
        for module in (Bn._tensors, None):
            with monkeypatch.context() as m:
                m.setattr(Bn, "_tensors", module)
                with pytest.raises(G.GrError):
                    call()
                    pytest.fail(f"call {i} by {module}")
    torch.cuda.synchronize()
    for a, b in zip(kept, (kv.keys, wide.keys, wide.values, q, r.out, lp.logprob, lp.top_token, *pair)):
        assert torch.equal(a, b)


def test_another_device_is_refused_or_made_current():
    if torch.cuda.device_count() < 2:
        pytest.skip("one device")
    kv, k, v, q, slots, positions, freq = _made(torch.uint8)
    with pytest.raises(G.GrError):
        G.cache_append(kv, k.to("cuda:1"), v, slots)
    other = G.KVCache.empty(9, 8, 2, 64, torch.uint8, device="cuda:1")
    G.cache_append(other, k.to("cuda:1"), v.to("cuda:1"), slots.to("cuda:1"))
    G.cache_append(kv, k, v, slots)
    assert torch.equal(other.keys.cpu(), kv.keys.cpu())
