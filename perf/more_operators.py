"""Performance cases of the operators that fill and read a paged cache, and of the log probabilities of tokens.

A case is a dict of plain values; `op` says which operator it passes through:
  "append"    cache_append: new tokens' keys are rotated by their positions and written to their slots with the values, the
              queries are rotated on the way; a cache held in 4 bits is read back at these slots (cache_read), as the numbers that it holds
  "read"      cache_read: keys and values of listed slots out of a cache held in 4 bits
  "attend"    cache_attend: attention of each row's last `new` tokens over the row's tokens in a cache held in 4 bits
  "logprobs"  token_logprobs: log probabilities of `given` tokens a row, the row's entropy and its `top` likeliest tokens

`own` chooses between the operators' plain form in elementary tensor operations and the package's calls.
"""
from __future__ import annotations

import math

import torch

own = False


# ---------------------------------------------------------------- cases

def _append(name, rows, new, heads, queries, dim, rot, block, cache="bf16", dtype="bf16", interleaved=False, far=4096):
    return {"name": name, "op": "append", "rows": rows, "new": new, "heads": heads, "queries": queries, "dim": dim, "rot": rot,
            "block": block, "cache": cache, "dtype": dtype, "interleaved": interleaved, "far": far}


def _read(name, tokens, heads, dim, block, dtype="bf16"):
    return {"name": name, "op": "read", "tokens": tokens, "heads": heads, "dim": dim, "block": block, "dtype": dtype}


def _attend(name, rows, context, new, heads, group, dim, block, dtype="bf16", window=0):
    return {"name": name, "op": "attend", "rows": rows, "context": context, "new": new, "heads": heads, "group": group,
            "dim": dim, "block": block, "dtype": dtype, "window": window}


def _logprobs(name, rows, V, given, top, dtype="f32", temperature=1.0, masked=0.0):
    return {"name": name, "op": "logprobs", "rows": rows, "V": V, "given": given, "top": top, "dtype": dtype,
            "temperature": temperature, "masked": masked}


def listed():
    return [
        # a decode batch: one token a row into a 16-bit cache, the queries rotated in the same call; latency
        _append("append-decode", 64, 1, 8, 32, 128, 128, 16),
        # prompts admitted together, of ragged lengths, 16-bit cache, heads rotated in part, neighbours paired
        _append("append-prompts", 12, 1000, 8, 32, 128, 64, 64, dtype="f16", cache="f16", interleaved=True),
        # the same into 4 bits
        _append("append-prompts-4bit", 12, 1000, 8, 0, 128, 128, 64, cache="q4"),
        # some drafted tokens looked at again
        _read("read-few", 300, 8, 128, 16, dtype="f32"),
        # a long prefix taken out for a prompt's own attention
        _read("read-prefix", 65536, 8, 128, 16),
        # one request, a short context: the latency of a step's attention
        _attend("attend-one", 1, 900, 1, 8, 4, 128, 16),
        # one request with a long context, large groups of query heads
        _attend("attend-long", 1, 131072, 1, 8, 8, 128, 32),
        # a decode batch of ragged contexts
        _attend("attend-decode", 64, 8000, 1, 8, 4, 128, 16),
        # verification: eight drafted tokens and the one before them, each row its own context
        _attend("attend-drafts", 32, 4000, 9, 8, 4, 128, 16, dtype="f16"),
        # one request's tokens scored
        _logprobs("logprobs-few", 4, 50257, 1, 5),
        # the rows of the headline batch of verification: the emitted tokens' probabilities, alternatives beside them
        _logprobs("logprobs-v128k", 1024, 128256, 1, 20, temperature=0.7, masked=0.1),
        # a prompt scored by a 152k-vocabulary model in bf16: two tokens of interest a row
        _logprobs("logprobs-v152k-bf16", 2048, 152064, 2, 8, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["append", "read", "attend", "attend", "logprobs"])
    if op == "append":
        cache = rng.choice(["q4", "bf16", "f16", "f32"])
        dtype = "f32" if cache == "f32" else rng.choice(["bf16", "f16"])
        dim = rng.choice([64, 96, 128, 192, 256])
        heads, new = rng.randint(1, 12), rng.choice([1, rng.randint(2, 9), _log_int(rng, 10, 2000)])
        rows = _log_int(rng, 1, max(1, min(300, 10_000_000 // (heads * dim * new))))
        case = _append("", rows, new, heads, 0 if cache == "q4" else heads * rng.choice([1, 2, 4]), dim,
                       rng.choice([dim, dim // 2, 0]), rng.choice([8, 16, 24, 32, 64, 128]), cache, dtype, rng.choice([True, False]),
                       _log_int(rng, 100, 1_000_000))
    elif op == "read":
        heads, dim = rng.randint(1, 12), rng.choice([32, 64, 96, 128, 192, 256])
        case = _read("", _log_int(rng, 1, min(100_000, 60_000_000 // (heads * dim))), heads, dim, rng.choice([8, 16, 24, 32, 64, 128]),
                     rng.choice(["bf16", "f16", "f32"]))
    elif op == "attend":
        dim, heads, group = rng.choice([64, 96, 128, 192, 256]), rng.randint(1, 12), rng.choice([1, 2, 4, 5, 8])
        new = rng.choice([1, 1, rng.randint(2, 9)])
        context = _log_int(rng, new, 100_000)
        rows = _log_int(rng, 1, max(1, min(200, 400_000_000 // (heads * dim * context * (1 if new * group <= 16 else new * group // 8)))))
        case = _attend("", rows, context, new, heads, group, dim, rng.choice([8, 16, 24, 32, 64, 128]), rng.choice(["bf16", "f16"]),
                       rng.choice([0, 0, _log_int(rng, 1, 4000)]))
    else:
        V, dtype = _log_int(rng, 200, 152064), rng.choice(["f32", "bf16"])
        case = _logprobs("", _log_int(rng, 1, max(1, min(4096, 120_000_000 // V))), V, rng.randint(1, 4), rng.choice([0, 1, rng.randint(2, 64)]),
                         dtype, rng.choice([0.7, 1.0, 1.3]), rng.choice([0.0, 0.3, 0.9]))
    return {k: v for k, v in case.items() if k != "name"}


# ---------------------------------------------------------------- the 4-bit layout, by reshaping
#
# A cache in 4 bits is [blocks, heads, block / 8, 9 dim] bytes: eight tokens ("an octet") of a head at a time.  Groups of 32
# dims share a 16-bit scale s; a code u of 4 bits stands for s (u - 8).  With J = dim / 32 an octet holds
#   keys' codes    [8 tokens][4][J] words: word (t, j) holds dims 32 j + 8 t .. + 7, the first in its lowest bits
#   keys' scales   [8 tokens][J]
#   values' codes  [8][4 pairs of tokens][J][2 tokens] half words: half word (g, ., j, .) holds dims 32 j + 4 g .. + 3
#   values' scales [4 pairs of tokens][J][2 tokens]

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "q4": torch.uint8}


def _nibbles(b):
    return torch.stack([b & 15, b >> 4], -1).flatten(-2)


def _unpack(octets, dim):
    """[..., 9 dim] bytes -> keys, values [..., 8, dim] in 32 bits."""
    J, lead = dim // 32, octets.shape[:-1]
    n = len(lead)
    kc, ks, vc, vs = octets.split([4 * dim, dim // 2, 4 * dim, dim // 2], -1)
    keep = list(range(n))
    k = _nibbles(kc.reshape(*lead, 8, 4, J, 4)).permute(*keep, n, n + 2, n + 1, n + 3)              # token, j, t, 8
    v = _nibbles(vc.reshape(*lead, 8, 4, J, 2, 2)).permute(*keep, n + 1, n + 3, n + 2, n, n + 4)     # pair, token, j, g, 4
    ks = ks.contiguous().view(torch.float16).reshape(*lead, 8, J, 1)
    vs = vs.contiguous().view(torch.float16).reshape(*lead, 4, J, 2).transpose(-1, -2).reshape(*lead, 8, J, 1)
    k = (k.reshape(*lead, 8, J, 32).float() - 8) * ks.float()
    v = (v.reshape(*lead, 8, J, 32).float() - 8) * vs.float()
    return k.reshape(*lead, 8, dim), v.reshape(*lead, 8, dim)


def _quantise(x):
    """[..., dim] in 32 bits -> codes [..., J, 32] and scales [..., J] in 16 bits."""
    x = x.reshape(*x.shape[:-1], -1, 32)
    hi, lo = x.amax(-1), x.amin(-1)
    s = torch.where(hi >= -lo, hi, lo).div(-8).clamp(-65504, 65504).half()
    # (in 64 bits: whether a quotient lies on a border between two codes is exact there)
    u = (x.double() / torch.where(s == 0, 1, s).double().unsqueeze(-1)).round().clamp(-8, 7) + 8
    return torch.where((s == 0).unsqueeze(-1), 8, u).to(torch.uint8), s


def _bytes(s):
    return s.contiguous().view(torch.uint8)


def _pack(k, v):
    """Whole octets: [..., 8, dim] -> [..., 9 dim] bytes."""
    lead, dim = k.shape[:-2], k.shape[-1]
    J, n = dim // 32, k.dim() - 2
    keep = list(range(n))
    ku, ks = _quantise(k)
    vu, vs = _quantise(v)
    ku = ku.reshape(*lead, 8, J, 4, 8).permute(*keep, n, n + 2, n + 1, n + 3)
    vu = vu.reshape(*lead, 4, 2, J, 8, 4).permute(*keep, n + 3, n, n + 2, n + 1, n + 4)
    ku, vu = (u[..., 0::2] | u[..., 1::2] << 4 for u in (ku, vu))
    vs = vs.reshape(*lead, 4, 2, J).transpose(-1, -2)
    return torch.cat([ku.reshape(*lead, -1), _bytes(ks.reshape(*lead, -1)), vu.reshape(*lead, -1), _bytes(vs.reshape(*lead, -1))], -1)


# ---------------------------------------------------------------- inputs

def _ceil_div(a, b):
    return (a + b - 1) // b


def _rand(g, *shape):
    return torch.rand(*shape, generator=g, device="cuda")


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _randint(g, lo, hi, *shape):
    return torch.randint(lo, hi + 1, shape, generator=g, device="cuda", dtype=torch.int32)


def _tables(g, lengths, block, width):
    """Rows' tokens in blocks of a pool, in random order, with some blocks left: table, number of blocks."""
    held = _ceil_div(lengths, block)
    some = torch.arange(width, device="cuda") < held.view(-1, 1)
    blocks = lengths.numel() * width + 3
    order = torch.randperm(blocks, generator=g, device="cuda", dtype=torch.int64).to(torch.int32)
    number = (some.reshape(-1).cumsum(0) - 1).clamp(min=0)
    return torch.where(some, order[number].view(some.shape), -1).to(torch.int32), blocks


def _prepare_append(c, g):
    R, n, H, D, bs = c["rows"], c["new"], c["heads"], c["dim"], c["block"]
    dt, kind = _TYPES[c["dtype"]], _TYPES[c["cache"]]
    # each row's new tokens, ragged where there are many, come behind a few that its first block holds already
    append = _randint(g, (n + 1) // 2, n, R) if n > 9 else _randint(g, n, n, R)
    before = _randint(g, 0, bs - 1, R)
    table, blocks = _tables(g, before + append, bs, _ceil_div(n + bs, bs))
    # (room for the most; slots and positions are -1 behind the last token, as block_plan leaves them)
    T = R * n
    end = append.cumsum(0)
    i = torch.arange(T, device="cuda")
    row = torch.searchsorted(end, i, right=True).clamp(max=R - 1)
    at = i - (end - append)[row] + before[row]
    some = i < end[-1]
    slots = torch.where(some, table[row, torch.where(some, at // bs, 0)].long() * bs + at % bs, -1)
    # (positions are as far as a prompt's beginning or a long context's end)
    positions = torch.where(some, at + _randint(g, 0, c["far"], R)[row], -1).to(torch.int32)
    # keys of a model: some channels are larger than others
    k = (_normal(g, T, H, D) * (1 + _rand(g, H, D))).to(dt)
    s = {"k": k, "v": _normal(g, T, H, D).to(dt), "slots": slots, "positions": positions, "q": None, "q_out": None, "freq": None}
    if c["queries"]:
        s["q"] = _normal(g, T, c["queries"], D).to(dt)
        s["q_out"] = torch.zeros_like(s["q"])
    if c["rot"]:
        s["freq"] = 10000.0 ** (-torch.arange(0, c["rot"], 2, device="cuda", dtype=torch.float64) / c["rot"])
    if c["cache"] == "q4":
        s["keys"], s["values"] = torch.zeros(blocks, H, bs // 8, 9 * D, dtype=torch.uint8, device="cuda"), None
    else:
        s["keys"] = torch.zeros(blocks, bs, H, D, dtype=kind, device="cuda")
        s["values"] = torch.zeros(blocks, bs, H, D, dtype=kind, device="cuda")
    return s


def _filled(g, blocks, H, bs, D):
    """A cache in 4 bits with quantised keys and values in all places."""
    data = torch.empty(blocks, H, bs // 8, 9 * D, dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 26) // (H * bs * D))
    wide = 1 + _rand(g, H, 1, 1, D)
    for lo in range(0, blocks, step):
        part = data[lo:lo + step]
        shape = (*part.shape[:3], 8, D)
        part.copy_(_pack(_normal(g, *shape) * wide, _normal(g, *shape)))
    return data


def _prepare_read(c, g):
    T, H, D, bs = c["tokens"], c["heads"], c["dim"], c["block"]
    table, blocks = _tables(g, torch.full((1,), T, dtype=torch.int32, device="cuda"), bs, _ceil_div(T, bs))
    at = torch.arange(T, device="cuda")
    return {"keys": _filled(g, blocks, H, bs, D), "values": None, "slots": table[0, at // bs].long() * bs + at % bs}


def _prepare_attend(c, g):
    R, n, H, D, bs = c["rows"], c["new"], c["heads"], c["dim"], c["block"]
    lengths = _randint(g, max(n, (c["context"] + 1) // 2), c["context"], R) if R > 1 else torch.full((1,), c["context"], dtype=torch.int32, device="cuda")
    table, blocks = _tables(g, lengths, bs, _ceil_div(c["context"], bs) + 1)
    offsets = torch.arange(0, R * n + 1, n, device="cuda", dtype=torch.int32)
    positions = (lengths.view(R, 1) - n + torch.arange(n, device="cuda", dtype=torch.int32)).reshape(-1).to(torch.int32)
    q = (_normal(g, R * n, H * c["group"], D) * 1.5).to(_TYPES[c["dtype"]])
    return {"q": q, "keys": _filled(g, blocks, H, bs, D), "values": None, "table": table, "lengths": lengths, "offsets": offsets,
            "positions": positions, "kept": None}


def _prepare_logprobs(c, g):
    R, V = c["rows"], c["V"]
    # the shape of a model's logits: a Zipf law over token ids in no order, and noise
    logits = torch.empty(R, V, dtype=_TYPES[c["dtype"]], device="cuda")
    step = max(1, (1 << 27) // V)
    for lo in range(0, R, step):
        x = torch.log1p(_rand(g, min(step, R - lo), V) * V).neg_()
        logits[lo:lo + step] = x.add_(_normal(g, *x.shape), alpha=0.5)
    if c["masked"] > 0:
        logits.masked_fill_(_rand(g, V) < c["masked"], -math.inf)
    # the given tokens: likely ones for the most part, as those that were emitted
    tokens = torch.stack([logits[:, torch.randint(0, V, (min(V, 1000),), generator=g, device="cuda")].float().argmax(1),
                          *(torch.randint(0, V, (R,), generator=g, device="cuda") for _ in range(c["given"] - 1))], 1)
    return {"logits": logits, "tokens": tokens.to(torch.int32).contiguous(), "kept": None}


_PREPARE = {"append": _prepare_append, "read": _prepare_read, "attend": _prepare_attend, "logprobs": _prepare_logprobs}


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return {"case": case, **_PREPARE[case["op"]](case, g)}


# ---------------------------------------------------------------- the plain forms

def _rotated(x, s):
    """[T, heads, dim] in 32 bits, the first `rot` dims turned; angles in 64 bits."""
    c = s["case"]
    x = x.float()
    if s["freq"] is None:
        return x
    angle = s["positions"].double().view(-1, 1, 1) * s["freq"]
    cos, sin = angle.cos().float(), angle.sin().float()
    turn = x[..., :c["rot"]]
    a, b = (turn[..., 0::2], turn[..., 1::2]) if c["interleaved"] else turn.chunk(2, -1)
    a, b = a * cos - b * sin, b * cos + a * sin
    turn = torch.stack([a, b], -1).flatten(-2) if c["interleaved"] else torch.cat([a, b], -1)
    return torch.cat([turn, x[..., c["rot"]:]], -1)


def _plain_append(s):
    c = s["case"]
    bs, D = c["block"], c["dim"]
    some = s["slots"] >= 0
    if s["q"] is not None:
        s["q_out"].copy_(torch.where(some.view(-1, 1, 1), _rotated(s["q"], s), s["q_out"].float()))
    k, v, slots = _rotated(s["k"], s)[some], s["v"][some].float(), s["slots"][some]
    block, at = slots // bs, slots % bs
    if c["cache"] != "q4":
        s["keys"][block, at] = k.to(s["keys"].dtype)
        s["values"][block, at] = v.to(s["values"].dtype)
        return {"keys": s["keys"], "values": s["values"], "q": s["q_out"]}
    # a token's own bytes of its octet: codes in 4 J words of the keys, in half words of the values
    J, T, H = D // 32, k.shape[0], c["heads"]
    ku, ks = _quantise(k)
    vu, vs = _quantise(v)
    octet, o = at // 8, at % 8
    ku = ku.view(T, H, J, 4, 8).transpose(2, 3)
    ku, vu = (u[..., 0::2] | u[..., 1::2] << 4 for u in (ku, vu.view(T, H, J, 8, 4)))
    kc, kz, vc, vz = s["keys"].split([4 * D, D // 2, 4 * D, D // 2], -1)
    kc.unflatten(-1, (8, 4, J, 4))[block, :, octet, o] = ku
    kz.unflatten(-1, (8, J, 2))[block, :, octet, o] = ks.unsqueeze(-1).view(torch.uint8)
    vc.unflatten(-1, (8, 4, J, 2, 2))[block, :, octet, :, o // 2, :, o % 2] = vu.transpose(2, 3)
    vz.unflatten(-1, (4, J, 2, 2))[block, :, octet, o // 2, :, o % 2] = vs.unsqueeze(-1).view(torch.uint8)
    return _plain_read({**s, "case": {**c, "dtype": "bf16"}})


def _plain_read(s):
    c = s["case"]
    bs, dt = c["block"], _TYPES[c["dtype"]]
    slots = s["slots"].clamp(min=0)
    block, at = slots // bs, slots % bs
    k, v = _unpack(s["keys"][block, :, at // 8], c["dim"])
    at = (at % 8).view(-1, 1, 1, 1).expand(-1, c["heads"], 1, c["dim"])
    some = (s["slots"] >= 0).view(-1, 1, 1)
    return {"k": torch.where(some, k.gather(2, at).squeeze(2), 0).to(dt), "v": torch.where(some, v.gather(2, at).squeeze(2), 0).to(dt)}


def _plain_attend(s):
    c = s["case"]
    R, n, H, G, D = c["rows"], c["new"], c["heads"], c["group"], c["dim"]
    k, v = _unpack(s["keys"][s["table"].clamp(min=0).long()], D)             # rows, blocks, heads, octets, 8, dim
    k, v = (x.transpose(1, 2).reshape(R, H, 1, -1, D) for x in (k, v))
    q = s["q"].float().view(R, n, H, G, D).permute(0, 2, 3, 1, 4).reshape(R, H, 1, G * n, D)
    x = (q @ k.transpose(-1, -2)).view(R, H, G, n, -1) / math.sqrt(D)
    at = torch.arange(x.shape[-1], device="cuda")
    p = s["positions"].view(R, 1, 1, n, 1)
    seen = at <= p if not c["window"] else (at <= p) & (at > p - c["window"])
    x = torch.where(seen, x, -math.inf)
    e = (x - x.amax(-1, keepdim=True)).exp()
    out = (e.view(R, H, 1, G * n, -1) @ v).view(R, H, G, n, D) / e.sum(-1, keepdim=True)
    return out.permute(0, 3, 1, 2, 4).reshape(R * n, H * G, D).to(s["q"].dtype)


def _plain_logprobs(s):
    c = s["case"]
    R, V, K = c["rows"], c["V"], c["top"]
    x = s["logits"].float() / c["temperature"]
    largest = x.amax(1, keepdim=True)
    e = (x - largest).exp_()
    total = e.sum(1, keepdim=True, dtype=torch.float64)
    lse = (total.log() + largest).float()
    # log p is -infinity where p is 0
    entropy = (total.log() - (e * (x - largest).clamp_(min=-1e30)).sum(1, keepdim=True, dtype=torch.float64) / total).float()
    del e
    out = {"logprob": x.gather(1, s["tokens"].long()) - lse, "entropy": entropy.view(R)}
    if K:
        # equal logits in the order of their ids: whole numbers that hold both
        bits = (s["logits"].float() + 0.0).view(torch.int32)
        key = torch.where(bits < 0, bits ^ 0x7fffffff, bits).long() << 32
        key += V - 1 - torch.arange(V, device="cuda")
        best = V - 1 - (key.topk(min(K, V), dim=1).values & 0xffffffff)
        lp = x.gather(1, best) - lse
        some = lp > -math.inf
        pad = (0, K - best.shape[1])
        out["top_token"] = torch.nn.functional.pad(torch.where(some, best, -1), pad, value=-1).int()
        out["top_logprob"] = torch.nn.functional.pad(lp, pad, value=-math.inf)
    return out


_PLAIN = {"append": _plain_append, "read": _plain_read, "attend": _plain_attend, "logprobs": _plain_logprobs}


# ---------------------------------------------------------------- one pass

def _own(s):
    import paper_2511_15898_b200 as G
    c = s["case"]
    if c["op"] == "logprobs":
        r = s["kept"] = G.token_logprobs(s["logits"], s["tokens"], c["top"], c["temperature"], out=s["kept"])
        out = {"logprob": r.logprob, "entropy": r.entropy}
        return {**out, "top_token": r.top_token, "top_logprob": r.top_logprob} if c["top"] else out
    cache = s.get("cache")
    if cache is None:
        cache = s["cache"] = G.KVCache(s["keys"], s["values"], c["block"], c["heads"], c["dim"])
    if c["op"] == "attend":
        r = s["kept"] = G.cache_attend(s["q"], cache, s["table"], s["offsets"], s["positions"], window=c["window"], out=s["kept"])
        return r.out
    if c["op"] == "append":
        G.cache_append(cache, s["k"], s["v"], s["slots"], s["positions"], s["freq"], interleaved=c["interleaved"], q=s["q"], q_out=s["q_out"])
        if c["cache"] != "q4":
            return {"keys": s["keys"], "values": s["values"], "q": s["q_out"]}
    k, v = G.cache_read(cache, s["slots"], torch.bfloat16 if c["op"] == "append" else _TYPES[c["dtype"]])
    return {"k": k, "v": v}


def run(state):
    return _own(state) if own else _PLAIN[state["case"]["op"]](state)


# ---------------------------------------------------------------- what a pass cannot do without

_SIZE = {"f32": 4, "bf16": 2, "f16": 2, "q4": 9 / 16}


def work(case):
    c = case
    if c["op"] == "append":
        # keys, values and queries read, cache and queries written, slots and positions read; 4 bits: read back as bf16
        tokens = c["rows"] * (0.75 * c["new"] if c["new"] > 9 else c["new"])
        e, held = _SIZE[c["dtype"]], _SIZE[c["cache"]]
        kv = 2 * c["heads"] * c["dim"]
        return {"bytes": tokens * (kv * (e + held) + 2 * c["queries"] * c["dim"] * e + 12 + (kv * (held + 2) if c["cache"] == "q4" else 0)),
                "flops": 6.0 * tokens * (c["heads"] + c["queries"]) * c["rot"]}
    if c["op"] == "read":
        return {"bytes": c["tokens"] * (2 * c["heads"] * c["dim"] * (9 / 16 + _SIZE[c["dtype"]]) + 8), "flops": 0}
    if c["op"] == "attend":
        # each row's tokens that a query sees read once, queries read, outputs written
        length = 0.75 * c["context"] if c["rows"] > 1 else c["context"]
        seen = min(length, c["window"] + c["new"] - 1) if c["window"] else length
        rows, heads = c["rows"], c["heads"] * c["group"]
        each = min(length, c["window"]) if c["window"] else length
        return {"bytes": rows * (seen * c["heads"] * c["dim"] * 9 / 8 + 4 * c["new"] * heads * c["dim"] + 4 * length / c["block"]),
                "flops": 4.0 * rows * c["new"] * heads * c["dim"] * each}
    return {"bytes": c["rows"] * (c["V"] * _SIZE[c["dtype"]] + 8 * c["given"] + 8 * c["top"] + 4), "flops": 5.0 * c["rows"] * c["V"]}


# ---------------------------------------------------------------- by the definition, in 64 bits

def _places(dim):
    """Of an octet: byte and shift of the code of (token, dim), and place of its scale among the 16-bit words, of keys and of values."""
    t = torch.arange(8, device="cuda").view(8, 1)
    d = torch.arange(dim, device="cuda").view(1, dim)
    J = dim // 32
    j, r = d // 32, d % 32
    key = t * (dim // 2) + (r // 8 * J + j) * 4 + r % 8 // 2
    value = 9 * dim // 2 + ((r // 4 * 4 + t // 2) * J + j) * 4 + t % 2 * 2 + r % 4 // 2
    return key, value, (d % 2 * 4).expand(8, dim), 2 * dim + t * J + j, 2 * dim + dim // 4 + 2 * dim + (t // 2 * J + j) * 2 + t % 2


def _held(octets, dim):
    """Keys and values [n, 8, dim] in 64 bits of the octets [n, 9 dim], one place after another."""
    key, value, shift, ks, vs = _places(dim)
    words = octets.contiguous().view(torch.float16).double()
    octets = octets.int()
    return ((((octets[:, key] >> shift) & 15) - 8).double() * words[:, ks], (((octets[:, value] >> shift) & 15) - 8).double() * words[:, vs])


def _turned(x, s):
    c, half = s["case"], s["case"]["rot"] // 2
    y = x.double().clone()
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + half)
        angle = (s["positions"].double() * s["freq"][i]).view(-1, 1)
        y[..., a] = x[..., a].double() * angle.cos() - x[..., b].double() * angle.sin()
        y[..., b] = x[..., a].double() * angle.sin() + x[..., b].double() * angle.cos()
    return y


def _four_bits(x):
    """What 4 bits hold of x [T, heads, dim], in 64 bits."""
    y = x.reshape(-1, 32)
    peak = y.gather(1, y.abs().argmax(1, keepdim=True))
    peak = torch.where((y == -peak).any(1, keepdim=True), peak.abs(), peak)
    scale = (-peak / 8).half().double()
    code = torch.where(scale == 0, 0.0, (y / torch.where(scale == 0, 1.0, scale)).round().clamp(-8, 7))
    return (code * scale).view(x.shape)


def exact(case, seed):
    """From the definitions, row by row where there are rows."""
    c, s = case, prepare(case, seed)
    if c["op"] == "append":
        k, v = _turned(s["k"], s) if s["freq"] is not None else s["k"].double(), s["v"].double()
        used = int((s["slots"] >= 0).sum())
        if c["cache"] == "q4":
            k, v = _four_bits(k), _four_bits(v)
            k[used:], v[used:] = 0, 0
            return {"k": k, "v": v}
        keys, values = s["keys"].double(), s["values"].double()
        keys.view(-1, c["heads"], c["dim"])[s["slots"][:used]] = k[:used]
        values.view(-1, c["heads"], c["dim"])[s["slots"][:used]] = v[:used]
        q = None if s["q"] is None else (_turned(s["q"], s) if s["freq"] is not None else s["q"].double())
        if q is not None:
            q[used:] = 0
        return {"keys": keys, "values": values, "q": q}
    if c["op"] == "read":
        out = []
        for lo in range(0, c["tokens"], 4096):
            slots = s["slots"][lo:lo + 4096]
            at = slots % c["block"]
            octets = s["keys"][slots // c["block"], :, at // 8]
            kv = _held(octets.reshape(-1, octets.shape[-1]), c["dim"])
            one = (at % 8).view(-1, 1).expand(-1, c["heads"]).reshape(-1)
            rows = torch.arange(one.numel(), device="cuda")
            out.append([x[rows, one].view(-1, c["heads"], c["dim"]) for x in kv])
        return {"k": torch.cat([x[0] for x in out]), "v": torch.cat([x[1] for x in out])}
    if c["op"] == "attend":
        n, H, G, D, bs = c["new"], c["heads"], c["group"], c["dim"], c["block"]
        out = torch.empty(c["rows"] * n, H * G, D, dtype=torch.float64, device="cuda")
        for r in range(c["rows"]):
            length = int(s["lengths"][r])
            blocks = s["table"][r, :-(-length // bs)].long()
            for h in range(H):
                octets = s["keys"][blocks, h].reshape(-1, 9 * D)
                k, v = (x.reshape(-1, D)[:length] for x in _held(octets, D))
                for i in range(n):
                    end = length - n + i + 1
                    begin = max(0, end - c["window"]) if c["window"] else 0
                    x = s["q"][r * n + i, h * G:(h + 1) * G].double() @ k[begin:end].T / math.sqrt(D)
                    out[r * n + i, h * G:(h + 1) * G] = torch.softmax(x, 1) @ v[begin:end]
        return out
    T, K = c["temperature"], c["top"]
    cols = {"logprob": [], "entropy": [], "top_token": [], "top_logprob": []}
    step = max(1, (1 << 26) // c["V"])
    for lo in range(0, c["rows"], step):
        lp = torch.log_softmax(s["logits"][lo:lo + step].double() / T, 1)
        p = lp.exp()
        cols["logprob"].append(lp.gather(1, s["tokens"][lo:lo + step].long()))
        cols["entropy"].append(-torch.where(p > 0, p * lp, 0.0).sum(1))
        if K:
            order = torch.sort(s["logits"][lo:lo + step].float(), dim=1, descending=True, stable=True).indices[:, :K]
            top = lp.gather(1, order)
            pad = (0, K - order.shape[1])
            cols["top_token"].append(torch.nn.functional.pad(torch.where(top > -math.inf, order, -1), pad, value=-1).int())
            cols["top_logprob"].append(torch.nn.functional.pad(top, pad, value=-math.inf))
    return {name: torch.cat(v) for name, v in cols.items() if v}
