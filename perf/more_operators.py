"""Timed cases of a serving step that verifies drafts over a paged 8-bit cache.

A case is a plain dict.  ``op`` says which operator a pass goes through:

* ``plan``    block tables, slots and positions of a step's tokens from request lengths and a stack of free blocks,
* ``append``  keys and values into the 8-bit cache by slot, and the blocks that were touched read back,
* ``attend``  grouped-query attention of the step's tokens over the cache through the block tables,
* ``verify``  drafted tokens accepted or replaced by the target's and the drafter's logits and given random numbers.

The cache holds bytes u that stand for (u - 128) * scale, one scale for each block of tokens, head, and keys or values.
Keys lie in tiles of 16 tokens x 64 dimensions, values in tiles of 32 tokens x 32 dimensions (``_key_rows``,
``_value_rows`` put them into rows).  With ``own`` false a pass is the plain form (elementary torch operations in 32
bits, 64 for the few numbers that decide a choice); with ``own`` true it is the call that a user makes of the library.
"""
import math
import random
from types import SimpleNamespace

import torch

own = False

_F64 = torch.float64


def _case(op, name, **kw):
    c = dict(op=op, batch=1, length=0, new=1, ragged=False, n_q=32, n_kv=8, d=128, block=64, dtype="bfloat16")
    if op == "verify":
        c = dict(op=op, batch=1, drafts=1, vocab=151936, dtype="bfloat16", temperature=1.0, drafter=True, pad=0)
    if op == "plan":
        c = dict(op=op, batch=1, length=0, new=1, ragged=False, block=64, ends=False)
    c.update(kw, name=name)
    return c


def listed():
    return [
        # one decode step of 32 long requests: a few of them enter a new block
        _case("plan", "plan 32 step", batch=32, length=8192, new=2),
        # 256 prompts of different lengths are admitted, and at the end give their blocks back
        _case("plan", "plan 256 prompts", batch=256, new=1024, ragged=True, ends=True),
        # a step's single tokens into 32 blocks that already hold others
        _case("append", "append 32", batch=32, length=8191),
        # prompts of odd lengths, fp32 keys and values of a small model
        _case("append", "append 7 prompts fp32", batch=7, length=3000, new=2333, ragged=True, n_q=4, n_kv=2, d=64,
              block=32, dtype="float32"),
        # a long prompt's chunk
        _case("append", "append 8192", batch=1, length=12345, new=8192),
        # one request, one token: latency
        _case("attend", "attend 1 x 2048", batch=1, length=2048),
        # a full batch, one token each
        _case("attend", "attend 32 x 8192", batch=32, length=8192),
        # drafts are verified: three tokens a request over long contexts, the fp32 rows of the library's own layers
        _case("attend", "attend 8 x 16384 x 3", batch=8, length=16384, new=3, dtype="float32"),
        # requests of very different lengths, a small model's heads, blocks of 32
        _case("attend", "attend 41 ragged", batch=41, length=12001, new=2, ragged=True, n_q=16, n_kv=2, d=64, block=32),
        # a prompt's chunk on top of what is cached
        _case("attend", "attend 2048 on 8192", batch=1, length=8192, new=2048),
        # one request, one draft: latency
        _case("verify", "verify 1 x 1", batch=1, drafts=1, dtype="float32"),
        # a full batch with four drafts each
        _case("verify", "verify 64 x 4", batch=64, drafts=4, temperature=0.6),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["plan", "append", "attend", "attend", "attend", "verify", "verify"])
    if op == "verify":
        c = _case(op, "", drafts=rng.randint(1, 8), vocab=_log(rng, 1000, 151936), pad=rng.choice([0, 0, rng.randint(1, 40)]),
                  temperature=rng.choice([0.0, 1.0, round(rng.uniform(0.5, 1.5), 2)]), drafter=rng.random() < 0.75,
                  dtype=rng.choice(["float32", "bfloat16"]))
        c["batch"] = _log(rng, 1, min(256, max(1, 64 * 4 * 151936 // (c["vocab"] * c["drafts"]))))
    elif op == "plan":
        c = _case(op, "", batch=_log(rng, 1, 1024), block=rng.choice([32, 64, 128, 256]), ragged=rng.random() < 0.7,
                  ends=rng.random() < 0.5)
        c["new"] = _log(rng, 1, 2 ** 17 // c["batch"])
        c["length"] = 0 if c["ends"] else _log(rng, 1, 16384)
    else:
        c = _case(op, "", batch=_log(rng, 1, 64), d=rng.choice([64, 128]), n_kv=rng.choice([1, 2, 4, 8]),
                  block=rng.choice([32, 64, 128, 256]), dtype=rng.choice(["float32", "bfloat16"]), ragged=rng.random() < 0.6)
        c["n_q"] = c["n_kv"] * rng.choice([1, 2, 4, 4, 7, 8])
        if op == "append":
            c["new"] = rng.choice([1, rng.randint(2, 8), _log(rng, 9, 8192 // c["batch"] + 9)])
            c["new"] = max(1, min(c["new"], 8192 // c["batch"]))
            c["length"] = c["new"] + _log(rng, 1, 8192)
        else:
            c["length"] = _log(rng, 1, max(2, min(32768, 32 * 8192 // c["batch"])))
            most = min(2 ** 29 // (c["batch"] * c["n_q"] * c["length"]), c["length"])
            c["new"] = max(1, min(rng.choice([1, 1, 1, rng.randint(2, 8), _log(rng, 9, 2048)]), most))
    del c["name"]
    return c


def _lengths(case):
    """Tokens of each request before the step and new in it; they go by the case, so that every seed has the same work."""
    R, L, n = case["batch"], case["length"], case["new"]
    rng = random.Random("%d %d %d" % (R, L, n))
    if not case["ragged"]:
        news = [n] * R
        ends = [L - rng.randrange(min(64, L)) if L > n and R > 1 else max(L, n) for _ in range(R)]
    else:
        news = [n] + [rng.randint(1, n) for _ in range(R - 1)]
        ends = [max(L, n)] + [max(m, int(L ** rng.uniform(0.3, 1.0))) for m in news[1:]]
    if case["op"] == "plan":        # the length is what is there already
        return [int(L * rng.random()) if case["ragged"] else max(0, L - rng.randrange(64)) for _ in range(R)], news
    return [max(e - m, 0) for e, m in zip(ends, news)], news


# ---- inputs ------------------------------------------------------------------------------------------------------

def _gpu(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype).cuda()


def _prepare_plan(case, gen):
    before, news = _lengths(case)
    B, R = case["block"], case["batch"]
    held = [-(-x // B) for x in before]
    need = [-(-(x + n) // B) for x, n in zip(before, news)]
    s = SimpleNamespace(case=case, block=B, rows=sum(news))
    order = torch.randperm(sum(need) + 9, generator=gen, device="cuda").int()
    width = max(need) + 3
    at = torch.arange(width, device="cuda")
    s.held = _gpu(held)
    first = torch.cumsum(s.held, 0) - s.held
    s.tables = torch.where(at < s.held[:, None], order[(first[:, None] + at).clamp(max=len(order) - 1)], -1).int()
    s.free = torch.cat([order[sum(held):], order[:sum(held)]]).contiguous()     # a stack: what is behind its top does not matter
    s.n_free = _gpu([len(order) - sum(held)])
    s.lens, s.new, s.ended = _gpu(before), _gpu(news), torch.full((R,), -1, dtype=torch.int32, device="cuda")
    return s


def _prepare_cache(case, gen):
    before, news = _lengths(case)
    B, H, D, R = case["block"], case["n_kv"], case["d"], case["batch"]
    totals = [x + n for x, n in zip(before, news)]
    need = [-(-t // B) for t in totals]
    P, N = sum(need) + 3, sum(news)
    s = SimpleNamespace(case=case, block=B)

    def codes(*shape):      # what quantised activations look like; bytes that no token has reached are anything
        x = torch.empty((P, H) + shape, dtype=torch.float16, device="cuda").normal_(128.0, 40.0, generator=gen)
        return x.round_().clamp_(1, 255).to(torch.uint8)

    s.keys, s.values = codes(B // 16, D // 64, 64, 16), codes(B // 32, D // 32, 64, 16)
    s.scales = 0.02 + 0.02 * torch.rand((P, H, 2), generator=gen, device="cuda")
    order = torch.randperm(P, generator=gen, device="cuda").int()
    held, at = _gpu(need), torch.arange(max(need), device="cuda")
    first = torch.cumsum(held, 0) - held
    s.tables = torch.where(at < held[:, None], order[(first[:, None] + at).clamp(max=P - 1)], -1).int()
    s.total = _gpu(totals)
    s.starts = torch.cat([_gpu([0]), torch.cumsum(_gpu(news), 0).int()])
    row = torch.arange(N, device="cuda")
    seq = torch.searchsorted(s.starts, row, right=True) - 1
    pos = s.total[seq] - (s.starts[seq + 1] - row)
    s.slots = (s.tables[seq, pos // B].long() * B + pos % B).int()
    # a layer's projections in one tensor: rows of queries, keys and values side by side
    wide = torch.randn((N, case["n_q"] + 2 * H, D), generator=gen, device="cuda")
    wide[:, case["n_q"]:] *= torch.exp(0.5 * torch.randn((N, 2 * H, 1), generator=gen, device="cuda"))
    wide = wide.to(getattr(torch, case["dtype"]))
    s.q, s.k, s.v = wide[:, :case["n_q"]], wide[:, case["n_q"]:case["n_q"] + H], wide[:, case["n_q"] + H:]
    if case["op"] == "append":      # every token of the blocks that are touched, up to each request's last one
        from_, cnt = [x // B * B for x in before], [t - x // B * B for x, t in zip(before, totals)]
        start = torch.repeat_interleave(_gpu(from_), _gpu(cnt))
        seq = torch.repeat_interleave(torch.arange(R, device="cuda"), _gpu(cnt))
        pos = start + torch.arange(len(seq), device="cuda") - (torch.cumsum(_gpu(cnt), 0) - _gpu(cnt))[seq]
        s.touched = (s.tables[seq, pos // B].long() * B + pos % B).int()
        # the other tokens of a block that the new ones enter: as small as what they come with
        s.scales.mul_(0.6)
    return s


def _rows(gen, n, V, pad):
    """Logit rows as a language model's: a broad floor and forty tokens of each position raised above it."""
    x = torch.randn((n, V + pad), generator=gen, device="cuda").mul_(2.0)
    at = torch.randint(0, V, (n, 40), generator=gen, device="cuda")
    return x.scatter_add_(1, at, 14.0 * torch.rand((n, 40), generator=gen, device="cuda"))


def _softmax64(z, temperature):
    return torch.softmax(z.double() / temperature, -1)


def _prepare_verify(case, gen):
    R, K, V, dt = case["batch"], case["drafts"], case["vocab"], getattr(torch, case["dtype"])
    s = SimpleNamespace(case=case)
    base = _rows(gen, R * (K + 1), V, case["pad"])
    near = torch.empty_like(base).normal_(0.0, 0.7, generator=gen).add_(base)
    s.logits = base.to(dt)[:, :V]
    s.drafter = near.view(R, K + 1, -1)[:, :K].to(dt)[:, :, :V]
    T = case["temperature"]
    s.u = torch.rand((R, K + 1), generator=gen, device="cuda")
    if T <= 0:      # greedy: the drafter's own choice, mostly the target's too
        s.drafts = s.drafter.float().argmax(2).int()
        s.drafter = None
        return s
    q = _softmax64(s.drafter, T).view(R * K, V)
    d = torch.multinomial(q, 1, generator=gen)
    q = q.gather(1, d).view(R, K) if case["drafter"] else 1.0
    s.drafts = d.view(R, K).int()
    edge = _softmax64(s.logits.view(R, K + 1, V)[:, :K], T).gather(2, d.view(R, K, 1))[:, :, 0] / q
    if not case["drafter"]:
        s.drafter = None
    # a choice must not hang on the last bits: numbers near a border move off it
    x = s.u[:, :K]
    x = torch.where((x - edge).abs() < 1e-4, torch.where(x > 0.5, x - 3e-4, x + 3e-4), x).float()
    j = torch.cumprod((x < edge).int(), 1).sum(1)
    mass = _plain_residual(s, j)
    cum = torch.cumsum(mass, 1)
    pick = torch.searchsorted(cum, (s.u[:, K:].double() * cum[:, -1:]).contiguous(), right=True).clamp(max=V - 1)
    pick = torch.where(mass.gather(1, pick) > 1e-5 * cum[:, -1:], pick, mass.argmax(1, keepdim=True))
    inside = 0.25 + 0.5 * torch.rand((R, 1), generator=gen, device="cuda", dtype=_F64)
    last = (cum.gather(1, pick) - inside * mass.gather(1, pick)) / cum[:, -1:]
    s.u = torch.cat([x, last.float()], 1)
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return {"plan": _prepare_plan, "verify": _prepare_verify}.get(case["op"], _prepare_cache)(case, gen)


# ---- the plain forms ---------------------------------------------------------------------------------------------

def _key_rows(x):
    """Key tiles [.., block/16, d/64, 64, 16] as rows [.., block, d]: lane 16 g + r has token r, dimensions 16 g ..."""
    U, H, T, C = x.shape[:4]
    return x.view(U, H, T, C, 4, 16, 16).permute(0, 1, 2, 5, 3, 4, 6).reshape(U, H, T * 16, C * 64)


def _key_tiles(x):
    U, H, B, D = x.shape
    return x.view(U, H, B // 16, 16, D // 64, 4, 16).permute(0, 1, 2, 4, 5, 3, 6).reshape(U, H, B // 16, D // 64, 64, 16)


def _value_rows(x):
    """Value tiles [.., block/32, d/32, 64, 16] as rows: lane 16 g + r has dimensions r and 16 + r, of each the
    tokens 4 g .. 4 g + 3 and 16 + 4 g .. 16 + 4 g + 3."""
    U, H, T, C = x.shape[:4]
    return x.view(U, H, T, C, 4, 16, 2, 2, 4).permute(0, 1, 2, 7, 4, 8, 3, 6, 5).reshape(U, H, T * 32, C * 32)


def _value_tiles(x):
    U, H, B, D = x.shape
    x = x.view(U, H, B // 32, 2, 4, 4, D // 32, 2, 16).permute(0, 1, 2, 6, 4, 8, 7, 3, 5)
    return x.reshape(U, H, B // 32, D // 32, 64, 16)


def _plain_plan(s, new):
    B, R, W, rows = s.block, s.held.shape[0], s.tables.shape[1], s.rows
    ended, at = new < 0, torch.arange(W, device="cuda")
    n = new.clamp(min=0).long()
    starts = torch.cat([torch.zeros_like(n[:1]), torch.cumsum(n, 0)])
    # the blocks of requests that ended go back, the first of them on top
    back = torch.where(ended, s.held, 0).long()
    rank = (torch.cumsum(back, 0) - back)[:, None] + at
    given, count, top = at < back[:, None], back.sum(), s.n_free.long()
    s.free = torch.cat([s.free, s.free[:1]])        # one more place for what is not given
    s.free[torch.where(given, top + count - 1 - rank, len(s.free) - 1)] = s.tables
    s.free, top = s.free[:-1].contiguous(), top + count
    held = torch.where(ended, 0, s.held).long()
    want = (s.lens + n + B - 1) // B
    need = torch.where(ended, 0, (want - held).clamp(min=0))
    done = torch.cumsum(need, 0)
    fits = ~ended & ((need == 0) | (done <= top)) & (want <= W) & (starts[1:] <= rows)
    take = torch.where(fits, need, 0)
    nth = (done - need)[:, None] + at - held[:, None]
    fresh = (at >= held[:, None]) & (at < (held + take)[:, None])
    s.tables = torch.where(ended[:, None], -1, torch.where(fresh, s.free[(top - 1 - nth).clamp(0, len(s.free) - 1)], s.tables))
    s.held, s.n_free = (held + take).int(), (top - take.sum()).int()
    row = torch.arange(rows, device="cuda")
    seq = (torch.searchsorted(starts, row, right=True) - 1).clamp(max=R - 1)
    pos = s.lens[seq] + row - starts[seq]
    on = (row < starts[-1]) & fits[seq]
    slots = torch.where(on, s.tables[seq, (pos // B).clamp(max=W - 1)].long() * B + pos % B, -1)
    return starts.int(), torch.where(fits, s.lens + n, 0).int(), slots.int(), torch.where(on, pos, -1).int()


def _plain_append(s, x, store, which):
    B, D = s.block, x.shape[2]
    blocks, run_of, sizes = torch.unique_consecutive(s.slots // B, return_inverse=True, return_counts=True)
    to_rows, to_tiles = (_key_rows, _key_tiles) if which == 0 else (_value_rows, _value_tiles)
    off, blocks = (s.slots % B).long(), blocks.long()
    top = torch.zeros((len(blocks), x.shape[1]), device="cuda")
    top = top.scatter_reduce(0, run_of[:, None].expand(-1, x.shape[1]), x.float().abs().amax(2), "amax")
    first = off[torch.cumsum(sizes, 0) - sizes]
    old = torch.where((first == 0)[:, None], 0.0, s.scales[blocks, :, which])
    scale = torch.maximum(old, top / torch.full_like(top, 127.0))
    scale = torch.where(scale < 2.0 ** -126, 0.0, scale)
    # which whole number is the nearest is decided in 64 bits
    unit = torch.where(scale > 0, scale, math.inf).double()
    held = to_rows(store[blocks]).float() - 128.0
    q = torch.round(held.double() * old.double()[:, :, None, None] / unit[:, :, None, None]).float()
    q = torch.where((scale == old)[:, :, None, None], held, q).clamp(-127, 127)
    mine = torch.round(x.double() / unit[run_of][:, :, None]).clamp(-127, 127).float()
    q[run_of, :, off] = mine
    store[blocks] = to_tiles((q + 128.0).to(torch.uint8))
    s.scales[blocks, :, which] = scale


def _plain_read(s, store, which, dtype):
    at, off = (s.touched // s.block).long(), (s.touched % s.block).long()
    # by element: where row `off` of a block lies in its tiles
    U, H, B, D = 1, store.shape[1], s.block, s.case["d"]
    place = torch.arange(B * D, device="cuda").view(store.shape[2:])[None, None]
    place = (_key_rows if which == 0 else _value_rows)(place)[0, 0][off]
    x = store.view(store.shape[0], H, B * D)[at[:, None, None], torch.arange(H, device="cuda")[:, None], place[:, None, :]]
    return ((x.float() - 128.0) * s.scales[at, :, which][:, :, None]).to(dtype)


def _plain_attend(s):
    c = s.case
    R, n, B, D, H, G = c["batch"], c["new"], s.block, c["d"], c["n_kv"], c["n_q"] // c["n_kv"]
    blocks = s.tables.clamp(min=0).long()
    L = blocks.shape[1] * B
    wide = lambda x, which, rows: ((rows(x[blocks.view(-1)]).float() - 128.0) * s.scales[blocks.view(-1), :, which][:, :, None, None]  # noqa: E731
                                   ).view(R, -1, H, B, D).transpose(1, 2).reshape(R, H, L, D)
    k, v = wide(s.keys, 0, _key_rows), wide(s.values, 1, _value_rows)
    mine = s.starts[:-1, None] + torch.arange(n, device="cuda")
    q = s.q[mine.clamp(max=s.q.shape[0] - 1)].float()                       # [R, n, n_q, D]
    q = q.view(R, n, H, G, D).permute(0, 2, 3, 1, 4).reshape(R, H, G * n, D)
    x = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(1.0 / math.sqrt(D)).view(R, H, G, n, L)
    pos = s.total[:, None] - s.starts[1:, None] + mine                      # each query's own position
    hidden = torch.arange(L, device="cuda") > pos[:, :, None]
    x = x.masked_fill_(hidden[:, None, None], -math.inf)
    x = torch.exp(x - x.amax(4, keepdim=True))
    x = x.div_(x.sum(4, keepdim=True)).view(R, H, G * n, L)
    o = torch.matmul(x, v).view(R, H, G, n, D).permute(0, 3, 1, 2, 4).reshape(R, n, H * G, D)
    row = torch.arange(s.q.shape[0], device="cuda")
    seq = torch.searchsorted(s.starts, row, right=True) - 1
    return o[seq, row - s.starts[seq]].to(s.q.dtype)


def _plain_rows(z, temperature):
    """exp(x - max) of x = z / temperature in 32 bits, and their sum in 64."""
    x = z.float() / temperature
    e = torch.exp(x - x.amax(-1, keepdim=True))
    return e, e.sum(-1, keepdim=True, dtype=_F64)


def _plain_residual(s, j):
    """Masses, in 64 bits, from which the token behind j accepted drafts is drawn."""
    c = s.case
    R, K, T = c["batch"], c["drafts"], c["temperature"]
    e, total = _plain_rows(s.logits[torch.arange(R, device="cuda") * (K + 1) + j], T)
    p, r, i = e.double() / total, torch.arange(R, device="cuda"), j.clamp(max=K - 1)
    if s.drafter is None:
        left = p.scatter(1, s.drafts.long().gather(1, i[:, None]), 0.0)
    else:
        e, total = _plain_rows(s.drafter[r, i], T)
        left = (p - e.double() / total).clamp(min=0.0)
    left = torch.where(left.sum(1, keepdim=True) > 0, left, p)
    return torch.where((j < K)[:, None], left, p)


def _plain_verify(s):
    c = s.case
    R, K, V, T = c["batch"], c["drafts"], c["vocab"], c["temperature"]
    d = s.drafts.long()
    if T <= 0:
        best = s.logits.float().argmax(1).view(R, K + 1)
        j = torch.cumprod((best[:, :K] == d).int(), 1).sum(1)
        last = best.gather(1, j[:, None])
    else:
        row = torch.arange(R, device="cuda")[:, None] * (K + 1) + torch.arange(K, device="cuda")
        e, total = _plain_rows(s.logits, T)
        p = e[row, d].double() / total[row, 0]
        if s.drafter is None:
            q = 1.0
        else:
            e, total = _plain_rows(s.drafter, T)
            q = e.gather(2, d[:, :, None])[:, :, 0].double() / total[:, :, 0]
        j = torch.cumprod((s.u[:, :K].double() * q < p).int(), 1).sum(1)
        cum = torch.cumsum(_plain_residual(s, j), 1)
        last = torch.searchsorted(cum, (s.u[:, K:].double() * cum[:, -1:]).contiguous(), right=True).clamp(max=V - 1)
    at = torch.arange(K + 1, device="cuda")
    tokens = torch.where(at < j[:, None], torch.cat([d, d[:, :1]], 1), torch.where(at == j[:, None], last, -1))
    return tokens.int(), j.int()


def run(s):
    c = s.case
    if own:
        from paper_2605_27255_amd import Kv8Cache, kv8_append, kv8_attention, kv8_plan, kv8_read, verify_drafts
    if c["op"] == "plan":
        if own:
            step = lambda new: kv8_plan(s.lens, new, s.tables, s.held, s.free, s.n_free, rows=s.rows, block=s.block)  # noqa: E731
        else:
            step = lambda new: _plain_plan(s, new)  # noqa: E731
        out = dict(zip(("starts", "total", "slots", "positions"), step(s.new)))
        if c["ends"]:
            out["after"] = step(s.ended)[2]
        top = torch.arange(s.free.shape[0], device="cuda") < s.n_free
        return dict(out, tables=s.tables, held=s.held, free=torch.where(top, s.free, -1), n_free=s.n_free)
    if c["op"] == "append":
        if own:
            cache = Kv8Cache(s.keys, s.values, s.scales)
            kv8_append(cache, s.k, s.v, s.slots)
            k, v = kv8_read(cache, s.touched, dtype=s.k.dtype)
        else:
            _plain_append(s, s.k, s.keys, 0)
            _plain_append(s, s.v, s.values, 1)
            k, v = _plain_read(s, s.keys, 0, s.k.dtype), _plain_read(s, s.values, 1, s.v.dtype)
        return {"k": k, "v": v}
    if c["op"] == "attend":
        if own:
            return {"out": kv8_attention(s.q, Kv8Cache(s.keys, s.values, s.scales), s.tables, s.starts, s.total)}
        return {"out": _plain_attend(s)}
    if own:
        tokens, accepted = verify_drafts(s.logits, s.drafts, s.u, draft_logits=s.drafter, temperature=c["temperature"])
    else:
        tokens, accepted = _plain_verify(s)
    return {"tokens": tokens, "accepted": accepted}


def work(case):
    es = 2 if case.get("dtype") == "bfloat16" else 4
    if case["op"] == "verify":
        R, K, V = case["batch"], case["drafts"], case["vocab"]
        rows = R * (2 * K + 1 if case["drafter"] and case["temperature"] > 0 else K + 1)
        return {"bytes": rows * V * es + R * (K + 1) * 12, "flops": rows * V * 4}
    before, news = _lengths(case)
    N, blocks = sum(news), sum(-(-(x + n) // case["block"]) for x, n in zip(before, news))
    if case["op"] == "plan":        # lengths, tables and positions of the step; where requests end, their blocks again
        return {"bytes": 16 * len(news) + 8 * N + 4 * blocks * (3 if case["ends"] else 1), "flops": 8 * N}
    H, D = case["n_kv"], case["d"]
    if case["op"] == "append":      # new rows in and their bytes out; then what is read back, bytes in and rows out
        back = sum(n + x % case["block"] for x, n in zip(before, news))
        return {"bytes": 2 * H * D * (N * (es + 1) + back * (1 + es)) + 16 * H * blocks, "flops": 2 * H * D * (4 * N + 2 * back)}
    seen = sum(n * x + n * (n + 1) // 2 for x, n in zip(before, news))
    tokens = sum(x + n for x, n in zip(before, news))
    return {"bytes": 2 * H * D * tokens + 8 * H * blocks + 2 * N * case["n_q"] * D * es, "flops": 4 * seen * case["n_q"] * D}


# ---- in 64 bits, from the definitions ----------------------------------------------------------------------------

def _one_block(keys, values, scales, block, at, D):
    """A block's keys and values [n_kv, block, D] in 64 bits, element by element of the tiles' definition."""
    t, e = torch.arange(block, device="cuda")[:, None], torch.arange(D, device="cuda")[None, :]
    k = keys[at][:, :, t // 16, e // 64, 16 * (e % 64 // 16) + t % 16, e % 16]
    v = values[at][:, :, t // 32, e // 32, 16 * (t % 16 // 4) + e % 16, 8 * (e % 32 // 16) + 4 * (t % 32 // 16) + t % 4]
    sc = scales[at].double()
    return (k.double() - 128) * sc[:, :, 0, None, None], (v.double() - 128) * sc[:, :, 1, None, None]


def _exact_attend(s):
    c = s.case
    B, D, G, out = s.block, c["d"], c["n_q"] // c["n_kv"], []
    for r, (x, n) in enumerate(zip(*_lengths(c))):
        used = s.tables[r, :-(-(x + n) // B)].long()
        k, v = (y.transpose(0, 1).flatten(1, 2)[:, :x + n] for y in _one_block(s.keys, s.values, s.scales, B, used, D))
        q = s.q[len(out):len(out) + n].double().transpose(0, 1)         # [n_q, n, D]
        own_pos = x + torch.arange(n, device="cuda")
        got = torch.empty((n, c["n_q"], D), dtype=_F64, device="cuda")
        for h in range(c["n_q"]):
            y = (q[h] @ k[h // G].T.contiguous()) / math.sqrt(D)
            y = y.masked_fill(torch.arange(x + n, device="cuda") > own_pos[:, None], -math.inf)
            got[:, h] = torch.softmax(y, 1) @ v[h // G]
        out.extend(got.unbind(0))
    return torch.stack(out)


def _exact_append(s):
    """Block by block: the scale from the largest magnitude, what was there rounded again where it grew."""
    B, D, H = s.block, s.case["d"], s.case["n_kv"]
    slots, place = s.slots.tolist(), {}
    for i, slot in enumerate(slots):
        place.setdefault(slot // B, []).append((slot % B, i))
    kept = {}
    for b, rows in place.items():
        off, idx = [torch.tensor(x, device="cuda") for x in zip(*rows)]
        got = []
        for which, (x, old) in enumerate(zip((s.k, s.v), _one_block(s.keys, s.values, s.scales, B, torch.tensor([b], device="cuda"), D))):
            x, old = x[idx].double().transpose(0, 1), old[0]
            was = s.scales[b, :, which].double() * float(rows[0][0] != 0)
            now = torch.maximum(was, (x.abs().amax((1, 2)) / 127).float().double())[:, None, None]     # held in 32 bits
            y = torch.where(now == was[:, None, None], old, torch.round(old / now) * now)
            y[:, off] = torch.round(x / now) * now
            got.append(y)
        kept[b] = torch.stack(got)
    touched = s.touched.tolist()
    names = {b: i for i, b in enumerate(kept)}
    every = torch.stack([kept[b] for b in names])           # [blocks, 2, H, B, D]
    at = torch.tensor([names[t // B] for t in touched], device="cuda")
    off = torch.tensor([t % B for t in touched], device="cuda")
    return every[at, 0, :, off], every[at, 1, :, off]


def exact(case, seed):
    if case["op"] == "attend":
        return {"out": _exact_attend(prepare(case, seed))}
    if case["op"] == "append":
        return dict(zip("kv", _exact_append(prepare(case, seed))))
    return None         # whole numbers
