"""Performance cases of the operators around a decoding step: beam search's selection over beams and vocabulary, the
reordering of what the models keep per hypothesis, the block tables and slot maps of a paged cache, and the copies of
blocks that two hypotheses share until one of them writes.

A case is a dict of plain values; `op` says which operator it passes through:
  "beam"     beam_select: the `select` best continuations of `beams` hypotheses over `V` tokens, for `batch` groups
  "reorder"  reorder_states: hypothesis j goes on from the state of its parent, in `tensors` tensors of one layout
  "plan"     block_plan: the rows' tokens are cut back, forked and extended; blocks are found for them, and slots
  "copy"     copy_blocks: listed blocks are copied within `tensors` paged caches

`own` chooses between the operators' plain form in elementary tensor operations and the package's calls.
"""
from __future__ import annotations

import math

import torch

own = False


# ---------------------------------------------------------------- cases

def _beam(name, batch, beams, V, select, dtype="f32", temperature=1.0, done=0.0, penalty=0.0, masked=0.0):
    return {"name": name, "op": "beam", "batch": batch, "beams": beams, "V": V, "select": select, "dtype": dtype,
            "temperature": temperature, "done": done, "penalty": penalty, "masked": masked}


def _reorder(name, batch, beams, chosen, tensors, heads, tokens, width, dtype="bf16", ragged=True):
    return {"name": name, "op": "reorder", "batch": batch, "beams": beams, "chosen": chosen, "tensors": tensors,
            "heads": heads, "tokens": tokens, "width": width, "dtype": dtype, "ragged": ragged}


def _plan(name, batch, beams, block, blocks, width, held, append, fork=False):
    return {"name": name, "op": "plan", "batch": batch, "beams": beams, "block": block, "blocks": blocks,
            "width": width, "held": held, "append": append, "fork": fork}


def _copy(name, pairs, share, tensors, blocks, block_bytes, dtype="bf16"):
    return {"name": name, "op": "copy", "pairs": pairs, "share": share, "tensors": tensors, "blocks": blocks,
            "block_bytes": block_bytes, "dtype": dtype}


def listed():
    return [
        # one request of a 32k-vocabulary model under beam search: the latency of a step
        _beam("beam-one", 1, 4, 32000, 8),
        # a small batch on an odd vocabulary, with finished hypotheses, banned tokens and a length penalty
        _beam("beam-v50k-penalty", 24, 5, 50257, 10, done=0.2, penalty=0.8, masked=0.3),
        # as many rows as the headline batch of verification, in groups of eight
        _beam("beam-v128k", 128, 8, 128256, 16, temperature=0.7),
        # bf16 logits of a 152k-vocabulary model, wide beams, twice as many candidates as beams
        _beam("beam-v152k-bf16", 256, 16, 152064, 32, dtype="bf16", temperature=0.8),
        # small recurrent states of a draft model: many tensors, few bytes
        _reorder("states-small", 2, 4, 4, 24, 1, 4, 512, ragged=False),
        # dense key / value caches of a beam search, ragged prompts, reordered in place
        _reorder("states-cache", 8, 4, 4, 8, 8, 2048, 128),
        # after verification: of each position's eight drafted states the accepted one is kept, fp32
        _reorder("states-drafts", 512, 8, 1, 2, 1, 1, 4096, dtype="f32", ragged=False),
        # one token for each of a full decode batch
        _plan("plan-decode", 256, 1, 16, 32768, 512, 1500, 1),
        # prompts of ragged lengths are admitted together
        _plan("plan-prompts", 48, 1, 64, 16384, 512, 0, 8000),
        # a beam step over a paged cache: rows fork, share blocks, and copy what they write
        _plan("plan-beams", 64, 8, 16, 65536, 256, 2000, 1, fork=True),
        # a handful of shared blocks copied in the caches of a small model
        _copy("copy-few", 16, 0.5, 8, 1024, 16384),
        # a wide beam step's copies, 32 KB blocks
        _copy("copy-many", 1024, 0.5, 16, 2560, 32768),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["beam", "beam", "reorder", "plan", "copy"])
    if op == "beam":
        beams = _log_int(rng, 1, 32)
        V = _log_int(rng, 200, 152064)
        dtype = rng.choice(["f32", "bf16"])
        batch = _log_int(rng, 1, max(1, min(256, 120_000_000 // (V * beams))))
        case = _beam("", batch, beams, V, rng.randint(1, min(64, 2 * beams)), dtype, rng.choice([0.7, 1.0, 1.3]),
                     rng.choice([0.0, 0.2]), rng.choice([0.0, 0.6, 1.0]), rng.choice([0.0, 0.3, 0.9]))
    elif op == "reorder":
        beams, dtype = _log_int(rng, 2, 32), rng.choice(["bf16", "f32"])
        heads, width, tokens = rng.randint(1, 12), rng.choice([33, 64, 80, 96, 128, 250]), _log_int(rng, 1, 2048)
        tensors = max(1, min(rng.randint(1, 32), 160_000_000 // (beams * heads * width * tokens)))
        batch = _log_int(rng, 1, max(1, min(64, 300_000_000 // (tensors * beams * heads * width * tokens * 4))))
        case = _reorder("", batch, beams, rng.choice([beams, beams, rng.randint(1, beams)]), tensors, heads, tokens, width,
                        dtype, rng.choice([True, False]))
    elif op == "plan":
        fork = rng.choice([True, False])
        beams = rng.randint(2, 16) if fork else 1
        batch, block = _log_int(rng, 1, max(1, 640 // beams)), rng.choice([8, 16, 24, 32, 64, 128])
        append = rng.choice([1, 1, rng.randint(2, 9), _log_int(rng, 10, 4000)])
        held = _log_int(rng, 1, 2500)
        width = -(-(held + append) // block) + rng.randint(1, 40)
        most = batch * beams * width
        case = _plan("", batch, beams, block, min(1 << 20, int(most * rng.uniform(0.9, 2.0)) + 64), width, held, append, fork)
    else:
        pairs, tensors, size = _log_int(rng, 1, 1500), rng.randint(1, 24), 16 * _log_int(rng, 4, 4096)
        tensors = max(1, min(tensors, 1_500_000_000 // (size * (2 * pairs + 40))))
        case = _copy("", pairs, rng.choice([0.1, 0.5, 0.9]), tensors, 2 * pairs + rng.randint(1, 40), size,
                     rng.choice(["bf16", "f32"]))
    return {k: v for k, v in case.items() if k != "name"}


# ---------------------------------------------------------------- inputs

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _ceil_div(a, b):
    return (a + b - 1) // b


def _rand(g, *shape):
    return torch.rand(*shape, generator=g, device="cuda")


def _randint(g, lo, hi, *shape):
    return torch.randint(lo, hi + 1, shape, generator=g, device="cuda", dtype=torch.int32)


def _prepare_beam(c, g):
    B, W, V = c["batch"], c["beams"], c["V"]
    # the shape of a model's logits: a Zipf law over token ids in no order, and noise
    logits = torch.empty(B, W, V, dtype=_TYPES[c["dtype"]], device="cuda")
    step = max(1, (1 << 27) // (W * V))
    for lo in range(0, B, step):
        x = torch.log1p(_rand(g, min(step, B - lo), W, V) * V).neg_()
        logits[lo:lo + step] = x.add_(torch.randn(x.shape, generator=g, device="cuda"), alpha=0.5)
    if c["masked"] > 0:
        banned = _rand(g, V) < c["masked"]
        logits.masked_fill_(banned, -math.inf)
    s = {"logits": logits, "scores": -4.0 - 3.0 * _rand(g, B, W), "lengths": None, "done": None, "eos": -1, "kept": None}
    if c["penalty"] > 0:
        s["lengths"] = _randint(g, 1, 60, B, W)
    if c["done"] > 0:
        s["done"], s["eos"] = _rand(g, B, W) < c["done"], 2 % V
    return s


def _prepare_reorder(c, g):
    B, W, H, S, D = c["batch"], c["beams"], c["heads"], c["tokens"], c["width"]
    states = [torch.empty(B, W, H, S, D, dtype=_TYPES[c["dtype"]], device="cuda").normal_(generator=g)
              for _ in range(c["tensors"])]
    parents = _randint(g, 0, W - 1, B, c["chosen"])
    s = {"states": states, "parents": parents, "lengths": None, "out": None}
    if c["ragged"]:
        s["lengths"] = _randint(g, (S + 1) // 2, S, B, 1).expand(B, W).contiguous()
    if c["chosen"] < W:
        # (the states that are chosen from stay as they are: the chosen ones have a place of their own)
        s["out"] = [torch.zeros(B, c["chosen"], H, S, D, dtype=_TYPES[c["dtype"]], device="cuda") for _ in states]
    return s


def _prepare_plan(c, g):
    B, W, bs, N, cap = c["batch"], c["beams"], c["block"], c["blocks"], c["width"]
    R = B * W
    # lengths in use; of a group's rows the front part is shared, as after a prompt and some steps of a beam search
    if c["held"] > 0:
        lengths = _randint(g, (c["held"] + 1) // 2, c["held"], B, 1).expand(B, W).reshape(R).contiguous()
    else:
        lengths = torch.zeros(R, dtype=torch.int32, device="cuda")
    held = _ceil_div(lengths, bs)
    col = torch.arange(cap, device="cuda")
    shared = (held.view(B, W, 1) * 3 // 4 > col) & (torch.arange(W, device="cuda") > 0).view(1, W, 1)
    mine = (col < held.view(B, W, 1)) & ~shared
    # blocks of the pool in random order, a new one for each entry that is a row's own
    order = torch.randperm(N, generator=g, device="cuda", dtype=torch.int64).to(torch.int32)
    number = mine.reshape(-1).cumsum(0) - 1
    have = number < N
    table = torch.where(mine.reshape(-1) & have, order[number.clamp(0, N - 1)], -1).view(B, W, cap)
    table = torch.where(shared, table[:, :1], table).reshape(R, cap).contiguous()
    # (a row whose blocks the pool did not hold ends before the first that is missing)
    lost = ((table < 0) & (col < held.view(R, 1))).int()
    first = torch.where(lost.any(1), lost.argmax(1), held)
    lengths = torch.minimum(lengths, (first * bs).to(torch.int32))
    table = torch.where(col < _ceil_div(lengths, bs).view(R, 1), table, -1).to(torch.int32).contiguous()
    refs = torch.bincount(table[table >= 0].long(), minlength=N).to(torch.int32)
    append = _randint(g, (c["append"] + 1) // 2, c["append"], R)
    s = {"table": table, "lengths": lengths, "refs": refs, "block": bs, "beams": W, "append": append,
         # every pass cuts the rows back to the tokens that were there at first, as after a step whose tokens were rejected
         "keep": lengths.clone(), "parents": None, "max_tokens": R * c["append"], "plan": None, "tables": None}
    if c["fork"]:
        s["parents"] = _randint(g, 0, W - 1, B, W)
    return s


def _prepare_copy(c, g):
    n, N = c["pairs"], c["blocks"]
    dt = _TYPES[c["dtype"]]
    caches = [torch.empty(N, c["block_bytes"] // dt.itemsize, dtype=dt, device="cuda").normal_(generator=g)
              for _ in range(c["tensors"])]
    order = torch.randperm(N, generator=g, device="cuda", dtype=torch.int64).to(torch.int32)
    copied = _rand(g, n) < c["share"]
    # (blocks that are copied from may be copied to several places)
    src = torch.where(copied, order[n + _randint(g, 0, max(0, (N - n) // 2), n).long().clamp(max=N - n - 1)], -1)
    return {"caches": caches, "src": src.to(torch.int32), "dst": torch.where(copied, order[:n], -1).to(torch.int32)}


_PREPARE = {"beam": _prepare_beam, "reorder": _prepare_reorder, "plan": _prepare_plan, "copy": _prepare_copy}


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return {"case": case, **_PREPARE[case["op"]](case, g)}


# ---------------------------------------------------------------- the plain forms

def _plain_beam(s):
    c = s["case"]
    B, W, V, K = c["batch"], c["beams"], c["V"], c["select"]
    # in 64 bits: continuations of different beams are ordered by their scores, and many lie close together
    x = s["logits"].double() / c["temperature"]
    top = x.amax(2, keepdim=True)
    lse = (x - top).exp().sum(2, keepdim=True).log() + top
    score = s["scores"].double().view(B, W, 1)
    total = score + (x - lse)
    length = torch.ones(B, W, dtype=torch.int64, device="cuda") if s["lengths"] is None else s["lengths"].long() + 1
    if s["done"] is not None:
        done = s["done"].view(B, W, 1)
        eos = torch.arange(V, device="cuda").view(1, 1, V) == s["eos"]
        total = torch.where(done, torch.where(eos, score, -math.inf), total)
        length = length - s["done"].long()
    scale = length.clamp(min=1).double() ** c["penalty"]
    key = (total / scale.view(B, W, 1)).view(B, W * V)
    total = total.view(B, W * V)
    # everything from the `select`-th largest key on; equal keys in the order of beams and tokens
    count = min(K, W * V)
    least = key.topk(count, dim=1).values[:, -1:]
    group, at = ((key >= least) & (key > -math.inf)).nonzero(as_tuple=True)
    per = torch.bincount(group, minlength=B)
    place = torch.arange(group.numel(), device="cuda") - (per.cumsum(0) - per)[group]
    room = max(K, int(per.max()))
    keys = torch.full((B, room), -math.inf, dtype=torch.float64, device="cuda")
    ids = torch.full((B, room), -1, dtype=torch.int64, device="cuda")
    keys[group, place], ids[group, place] = key[group, at], at
    order = keys.sort(dim=1, descending=True, stable=True).indices[:, :K]
    ids = ids.gather(1, order)
    some = ids >= 0
    parent = torch.where(some, ids // V, -1)
    token = torch.where(some, ids % V, -1)
    of = parent.clamp(min=0)
    ended = torch.zeros_like(some) if s["done"] is None else s["done"].gather(1, of) | (token == s["eos"])
    return {"token": token.int(), "parent": parent.int(), "done": (ended & some),
            "score": torch.where(some, total.gather(1, ids.clamp(min=0)), -math.inf).float(),
            "length": torch.where(some, length.gather(1, of), 0).int() if s["lengths"] is not None else None}


def _plain_reorder(s):
    states, parents, lengths = s["states"], s["parents"].long(), s["lengths"]
    c = s["case"]
    B, S = c["batch"], c["tokens"]
    row = torch.arange(B, device="cuda").view(B, 1)
    if s["out"] is not None:
        to = s["out"]
    else:
        to = [x[:, :c["chosen"]] for x in states]
    if lengths is None:
        done = [y.copy_(x[row, parents]) for y, x in zip(to, states)]
    else:
        used = (torch.arange(S, device="cuda") < lengths.gather(1, parents).view(B, -1, 1)).view(B, -1, 1, S, 1)
        done = [y.copy_(torch.where(used, x[row, parents], y)) for y, x in zip(to, states)]
    return done if s["out"] is not None else states


def _plain_plan(s):
    table, lengths, refs, bs, W = s["table"], s["lengths"], s["refs"], s["block"], s["beams"]
    R, cap = table.shape
    N, T = refs.numel(), s["max_tokens"]
    row = torch.arange(R, device="cuda")
    col = torch.arange(cap, device="cuda").view(1, cap)
    # each row goes on from its parent, cut back to `keep` tokens
    of = row if s["parents"] is None else row // W * W + s["parents"].reshape(R)
    base = torch.minimum(lengths[of], s["keep"]).long()
    before, kept = _ceil_div(lengths.long(), bs), _ceil_div(base, bs)
    held = table[of].long()
    drop = torch.bincount(table[col < before.view(R, 1)].long(), minlength=N)
    take = torch.bincount(held[col < kept.view(R, 1)], minlength=N)
    count = refs.long() - drop + take
    new = torch.where(col < kept.view(R, 1), held, torch.where(col < before.view(R, 1), -1, table.long()))
    # tokens to append
    ask = s["append"].long()
    end = ask.cumsum(0)
    fits = (base + ask <= cap * bs) & (end <= T)
    app = torch.where(fits, ask, 0)
    # a partly filled last block that other rows hold too is copied, but by the one row that the others copy it from
    writes = (app > 0) & (base % bs > 0)
    last = new.gather(1, (base // bs).clamp(max=cap - 1).view(R, 1)).view(R).clamp(min=0)
    writers = torch.zeros(N, dtype=torch.int64, device="cuda").index_add_(0, last, writes.long())
    rank = base % bs * R + (R - 1 - row)
    best = torch.full((N,), -1, dtype=torch.int64, device="cuda").scatter_reduce_(0, last, torch.where(writes, rank, -1), "amax")
    keeps = (writers[last] == count[last]) & (best[last] == rank)
    copies = writes & (count[last] > 1) & ~keeps
    need = copies.long() + _ceil_div(base + app, bs) - kept
    free = (count == 0).nonzero().view(-1)
    upto = need.cumsum(0)
    served = (need == 0) | (upto <= free.numel())
    app = torch.where(served, app, 0)
    copies = copies & served
    after = _ceil_div(base + app, bs)
    start = (upto - need).view(R, 1)
    pool = torch.cat([free, free.new_full((1,), -1)])

    def number(i):
        return pool[i.clamp(0, pool.numel() - 1)]

    fresh = (col >= kept.view(R, 1)) & (col < after.view(R, 1))
    new = torch.where(fresh, number(start + copies.view(R, 1).long() + col - kept.view(R, 1)), new)
    copy = copies.view(R, 1) & (col == (base // bs).view(R, 1))
    copy_src = torch.where(copies, last, -1)
    copy_dst = torch.where(copies, number(start.view(R)), -1)
    new = torch.where(copy, copy_dst.view(R, 1), new)
    count = count.index_add(0, last, -copies.long())
    count = count + torch.bincount(new[fresh | copy], minlength=N)
    # slots of the tokens, one row after another
    token_row = torch.repeat_interleave(row, ask)[:T]
    used = token_row.numel()
    position = base[token_row] + torch.arange(used, device="cuda") - (end - ask)[token_row]
    block = new[token_row, (position // bs).clamp(max=cap - 1)]
    written = position < (base + app)[token_row]
    slots = torch.full((T,), -1, dtype=torch.int64, device="cuda")
    slots[:used] = torch.where(written, block * bs + position % bs, -1)
    positions = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    positions[:used] = torch.where(written, position, -1).int()
    status = torch.where(~fits, 9, torch.where(served, 0, 8)).int()
    table.copy_(new)
    lengths.copy_(base + app)
    refs.copy_(count)
    offsets = torch.cat([end.new_zeros(1), end]).clamp(max=T).int()
    return {"table": table, "lengths": lengths, "refs": refs, "slots": slots, "positions": positions, "offsets": offsets,
            "copy_src": copy_src.int(), "copy_dst": copy_dst.int(), "status": status}


def _plain_copy(s):
    some = s["src"] >= 0
    src, dst = s["src"][some].long(), s["dst"][some].long()
    return [x.index_copy_(0, dst, x[src]) for x in s["caches"]]


_PLAIN = {"beam": _plain_beam, "reorder": _plain_reorder, "plan": _plain_plan, "copy": _plain_copy}


# ---------------------------------------------------------------- one pass

def _own(s):
    import paper_2511_15898_b200 as G
    c = s["case"]
    if c["op"] == "beam":
        r = s["kept"] = G.beam_select(s["logits"], s["scores"], c["select"], c["temperature"], lengths=s["lengths"],
                                      done=s["done"], eos=s["eos"], length_penalty=c["penalty"], out=s["kept"])
        return {"token": r.token, "parent": r.parent, "done": r.done, "score": r.score,
                "length": r.length if s["lengths"] is not None else None}
    if c["op"] == "reorder":
        return G.reorder_states(s["states"], s["parents"], lengths=s["lengths"],
                                token_dim=None if s["lengths"] is None else 3, out=s["out"])
    if c["op"] == "plan":
        if s["tables"] is None:
            s["tables"] = G.BlockTables(s["table"], s["lengths"], s["refs"], s["block"], s["beams"])
        r = s["plan"] = G.block_plan(s["tables"], s["append"], s["max_tokens"], keep=s["keep"], parents=s["parents"],
                                     out=s["plan"])
        return {"table": s["table"], "lengths": s["lengths"], "refs": s["refs"], "slots": r.slots,
                "positions": r.positions, "offsets": r.offsets, "copy_src": r.copy_src, "copy_dst": r.copy_dst,
                "status": r.status}
    G.copy_blocks(s["caches"], s["src"], s["dst"])
    return s["caches"]


def run(state):
    return _own(state) if own else _PLAIN[state["case"]["op"]](state)


# ---------------------------------------------------------------- what a pass cannot do without

def _distinct(W, chosen):
    """Expected numbers, over parents drawn evenly from W: rows whose parent is another one, and such parents."""
    moved = chosen * (1 - 1 / W)
    parents = sum(1 - (1 - 1 / W) ** (chosen - (1 if w < chosen else 0)) for w in range(W))
    return moved, parents


def work(case):
    c = case
    if c["op"] == "beam":
        # logits read once (finished hypotheses' are not needed), results written; a logit's exponential and its sum
        rows = c["batch"] * c["beams"] * (1 - c["done"])
        esize = 2 if c["dtype"] == "bf16" else 4
        per = 13 + (4 if c["penalty"] > 0 else 0)
        return {"bytes": rows * c["V"] * esize + c["batch"] * (c["beams"] * 9 + c["select"] * per),
                "flops": 4.0 * rows * c["V"]}
    if c["op"] == "reorder":
        esize = 2 if c["dtype"] == "bf16" else 4
        tokens = 0.75 * c["tokens"] if c["ragged"] else c["tokens"]
        row = c["heads"] * tokens * c["width"] * esize
        W = c["beams"]
        if c["chosen"] < W:      # (out of place: every chosen row is written, every distinct parent read)
            rows = c["chosen"] + W * (1 - (1 - 1 / W) ** c["chosen"])
        else:
            rows = sum(_distinct(W, c["chosen"]))
        return {"bytes": c["batch"] * (rows * row * c["tensors"] + 4 * c["chosen"]), "flops": 0}
    if c["op"] == "plan":
        # counts of the pool read, rows' numbers read and written, a forked row's held blocks read and written, tokens' slots
        rows = c["batch"] * c["beams"]
        held = rows * 0.75 * c["held"] / c["block"] if c["fork"] else rows
        tokens = rows * c["append"]
        fresh = rows * 0.75 * c["append"] / c["block"]
        return {"bytes": 4 * c["blocks"] + rows * 40 + 8 * held + 8 * fresh + 12 * tokens, "flops": 0}
    return {"bytes": 2.0 * c["pairs"] * c["share"] * c["tensors"] * c["block_bytes"] + 8 * c["pairs"], "flops": 0}


# ---------------------------------------------------------------- by the definition, in 64 bits

def exact(case, seed):
    """Group by group from the definitions.  The plans of blocks are whole numbers: there is nothing to round."""
    c, s = case, prepare(case, seed)
    if c["op"] == "plan":
        return None
    if c["op"] == "reorder":
        if c["batch"] * c["chosen"] * c["tensors"] > 20000 or c["tensors"] * s["states"][0].numel() > 3e8:
            return None
        out = []
        parents = s["parents"].tolist()
        used = None if s["lengths"] is None else s["lengths"].tolist()
        for i, x in enumerate(s["states"]):
            y = (x if s["out"] is None else s["out"][i]).double()
            for b, chosen in enumerate(parents):
                for j, p in enumerate(chosen):
                    n = c["tokens"] if used is None else used[b][p]
                    y[b, j, :, :n] = x[b, p, :, :n].double()
            out.append(y)
        return out
    if c["op"] == "copy":
        if c["tensors"] * c["blocks"] * c["block_bytes"] > 2e9:
            return None
        pairs = list(zip(s["src"].tolist(), s["dst"].tolist()))
        out = []
        for x in s["caches"]:
            y = x.double()
            for a, b in pairs:
                if a >= 0:
                    y[b] = x[a].double()
            out.append(y)
        return out
    K, T = c["select"], float(c["temperature"])
    cols = {"token": [], "parent": [], "done": [], "score": [], "length": []}
    for b in range(c["batch"]):
        lp = torch.log_softmax(s["logits"][b].double() / T, dim=1)
        at, tok, tot, key, fin, ln = [], [], [], [], [], []
        for w in range(c["beams"]):
            score = float(s["scores"][b, w])
            n = 0 if s["lengths"] is None else int(s["lengths"][b, w])
            if s["done"] is not None and bool(s["done"][b, w]):
                t, v, f = torch.tensor([score], dtype=torch.float64, device="cuda"), torch.tensor([s["eos"]], device="cuda"), True
            else:
                n, f = n + 1, False
                v = torch.sort(lp[w], descending=True, stable=True).indices[:K]
                t = lp[w][v] + score
                v, t = v[t > -math.inf], t[t > -math.inf]
            at.append(torch.full_like(v, w)); tok.append(v); tot.append(t); key.append(t / float(max(n, 1)) ** c["penalty"])
            fin.append(torch.full_like(v, f, dtype=torch.bool)); ln.append(torch.full_like(v, n))
        at, tok, tot, key, fin, ln = (torch.cat(z) for z in (at, tok, tot, key, fin, ln))
        best = torch.sort(key, descending=True, stable=True).indices[:K]
        pad = K - best.numel()

        def column(z, none):
            return torch.cat([z[best], z.new_full((pad,), none)])

        cols["token"].append(column(tok, -1)); cols["parent"].append(column(at, -1)); cols["score"].append(column(tot, -math.inf))
        cols["done"].append(column(fin | ((tok == s["eos"]) & (s["done"] is not None)), False)); cols["length"].append(column(ln, 0))
    out = {k: torch.stack(v) for k, v in cols.items()}
    if s["lengths"] is None:
        out["length"] = None
    return out
