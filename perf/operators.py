"""The paged-cache operators beside the routing step, at the sizes their users run them at.

A decode worker keeps its requests' K/V in blocks of a fixed number of tokens.  From the request lengths that the
routing step leaves on the GPU come, for every worker of every fleet,

* ``tables``  the block tables: blocks of ended and shrunken requests are taken back, grown and new ones served;
* ``slots``   the slot map: where the K/V of each request's newest tokens go;
* ``pages``   the page lists: the running requests packed, with their blocks, as an attention call reads them.

Fleet shapes and length distributions are those of the configurations in ``workload.py`` (c0, c1, c3, c4, h80) and ragged
ones.  Blocks are dealt from a shuffled pool, as after hours of service.  All outputs are whole numbers.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
EMPTY = -(2 ** 31)                     # a free slot, as in the router's act_base
MOST = 2 ** 31 - 1

# N fleets of G workers with B slots; blocks of `block` tokens, `columns` of them a table row, `pool` a worker.
# mu, sigma, lo, hi: lognormal request lengths.  stepped: lengths come as the router keeps them, relative to the step.
_BASE = dict(N=1, G=16, B=64, block=16, columns=2048, pool=10000, mu=7.0, sigma=1.0, lo=16, hi=32000, running=1.0, stepped=True)


def _case(op, name=None, **kw):
    c = dict(_BASE, op=op)
    if op == "tables":
        c.update(ended=0.0, refill=0.0, grow=1)
    if op == "slots":
        c.update(new="one", room=64)
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one small fleet (c0) between two decode steps: call latency
        _case("tables", "tables_c0_step", G=4, pool=9001, running=0.5, ended=0.002, refill=0.01),
        # 1,024 fleets at the deployed setting (h80), a decode step: few blocks move, counts and lengths are read
        _case("tables", "tables_h80_step", N=1024, G=8, block=32, columns=512, pool=10240, mu=8.0, sigma=0.8, hi=16000,
              running=0.98, ended=0.001, refill=0.05),
        # 16 of the largest fleets (c4) fill their empty caches with prompts of up to 131,072 tokens
        _case("tables", "tables_c4_fill", N=16, G=64, columns=8192, pool=65536, mu=8.0, sigma=1.5, hi=131072, running=0.0,
              refill=1.0, stepped=False),
        # a burst replaces a third of the requests of ragged fleets whose pools run short
        _case("tables", "tables_ragged_burst", N=61, G=33, B=40, block=24, columns=700, pool=4001, mu=7.5, sigma=1.2,
              hi=16000, running=0.7, ended=0.33, refill=0.8, grow=7),
        # one fleet (c1), one new token a request
        _case("slots", "slots_c1_decode"),
        # 1,024 fleets (c3), one new token a request
        _case("slots", "slots_c3_decode", N=1024, G=32, block=128, columns=64, pool=2500, mu=7.5, sigma=1.2, hi=8192,
              running=0.9),
        # whole prompts of up to 131,072 tokens, four of the largest fleets (c4)
        _case("slots", "slots_c4_prompts", N=4, G=64, columns=8192, pool=65536, mu=8.0, sigma=1.5, hi=131072, new="prompt",
              room=800000, stepped=False),
        # prompts in chunks, blocks of 24 tokens, odd sizes
        _case("slots", "slots_ragged_chunks", N=8, G=33, B=40, block=24, columns=700, pool=5001, mu=7.5, sigma=1.2,
              hi=16000, running=0.8, new="chunk", room=12345),
        # the page lists of one fleet at the deployed setting (h80)
        _case("pages", "pages_h80_one", G=8, columns=1024, pool=20000, mu=8.0, sigma=0.8, hi=16000, running=0.97),
        # 16 of the largest fleets (c4), full caches
        _case("pages", "pages_c4_fleets", N=16, G=64, columns=8192, pool=65536, mu=8.0, sigma=1.5, hi=131072),
        # many small pools of many short requests, half the slots free
        _case("pages", "pages_ragged", N=301, G=7, B=248, block=24, columns=171, pool=9999, mu=6.0, sigma=1.3, lo=1,
              hi=4100, running=0.5),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["tables", "slots", "pages"])
    block = rng.choice([8, 16, 16, 24, 32, 48, 64, 128, 256])
    G, B = _spread(rng, 1, 64), _spread(rng, 4, 256)
    hi = _spread(rng, 500, 131072)
    columns = (hi + 64) // block + 1
    rows = 2 ** 29 // columns                                     # 2 GB of tables at most
    N = _spread(rng, 1, max(1, min(4096, 2 ** 22 // (G * B), rows // (G * B))))
    mu, sigma = rng.uniform(5.0, math.log(hi)), rng.uniform(0.3, 1.6)
    c = dict(op=op, N=N, G=G, B=B, block=block, columns=columns, mu=round(mu, 3), sigma=round(sigma, 3), lo=rng.choice([1, 16]),
             hi=hi, running=round(rng.uniform(0.3, 1.0), 3), stepped=rng.random() < 0.7)
    each = _mean_length(c)                                        # tokens a request
    while c["N"] > 1 and c["N"] * G * B * each > 1.2e8:
        c["N"] //= 2
    c["pool"] = max(8, int(B * (each / block + 0.5) * rng.uniform(0.6, 1.6)))
    if op == "tables":
        c.update(ended=round(rng.choice([0.002, 0.05, 0.5]) * rng.uniform(0.5, 1.5), 4), refill=round(rng.uniform(0.0, 1.0), 3),
                 grow=rng.choice([1, 1, 1, 5, 64]))
    if op == "slots":
        new = rng.choice(["one", "prompt", "chunk"])
        per = {"one": 1.0, "prompt": each, "chunk": 300.0}[new]
        c.update(new=new, room=max(B, int(B * per * rng.uniform(0.5, 1.3))))
    return c


def _draws(case, shape, gen, device, count):
    return [torch.rand(shape, generator=gen, device=device, dtype=torch.float64) for _ in range(count)]


def _lognormal(case, u):
    z = torch.special.ndtri(u.clamp(1e-9, 1 - 1e-9))
    return torch.exp(case["mu"] + case["sigma"] * z).round().clamp(case["lo"], case["hi"]).to(torch.int64)


def _mean_length(case):
    return float(_lognormal(case, (torch.arange(4096, dtype=torch.float64) + 0.5) / 4096).double().mean())


def _before_and_after(case, shape, gen, device):
    """Tokens a slot's request had when the tables were last brought up to date, and has now (0: free)."""
    u = _draws(case, shape, gen, device, 2)
    before = torch.where(u[0] < case["running"], _lognormal(case, u[1]), 0)
    if case["op"] != "tables":
        return before, before
    u = _draws(case, shape, gen, device, 3)
    after = torch.where((before > 0) & (u[0] >= case["ended"]), before + case["grow"], 0)
    return before, torch.where((after == 0) & (u[1] < case["refill"]), _lognormal(case, u[2]), after)


def _newest(case, tokens, gen, device):
    """How many of each request's tokens are new: all of a prompt, or a chunk of a third of the prompts."""
    u = _draws(case, tokens.shape, gen, device, 2)
    if case["new"] == "prompt":
        return tokens
    chunk = torch.where(u[0] < 1 / 3, 1 + (u[1] ** 2 * 2048).to(torch.int64), 0)
    return torch.minimum(chunk, tokens)


def _held(case, need):
    """Blocks each request holds: all it needs, in slot order, while the pool lasts."""
    return torch.where(need.cumsum(-1) <= case["pool"], need, 0)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(int(seed))
    N, G, B, block, T, P = (case[k] for k in ("N", "G", "B", "block", "columns", "pool"))
    before, after = _before_and_after(case, (N, G, B), gen, DEVICE)
    held = _held(case, (before + block - 1) // block)
    deal = torch.rand((N, G, P), generator=gen, device=DEVICE).argsort(-1).to(torch.int32)       # each worker's blocks, shuffled
    start = held.cumsum(-1) - held
    columns = torch.arange(T, device=DEVICE)
    table = torch.empty((N, G, B, T), dtype=torch.int32, device=DEVICE)
    for i in range(N):                                                                             # (a fleet at a time: the indices are large)
        at = (start[i, :, :, None] + columns).clamp_(max=P - 1)
        rows = deal[i, :, None, :].expand(G, B, P).gather(-1, at)
        table[i] = torch.where(columns < held[i, :, :, None], rows, -1)
    total = held.sum(-1, keepdim=True)
    at = total + torch.arange(P, device=DEVICE)
    free = torch.where(at < P, deal.gather(-1, at.clamp(max=P - 1)), -1)
    step = torch.randint(0, 2000, (N,), generator=gen, device=DEVICE, dtype=torch.int32)
    if case["stepped"]:
        length = torch.where(after > 0, after - step[:, None, None], EMPTY).to(torch.int32)
    else:
        length, step = after.to(torch.int32), None
    s = dict(case=case, length=length, step=step, block=block, table=table, n_blocks=held.to(torch.int32), free_list=free,
             n_free=(P - total[..., 0]).to(torch.int32))
    if case["op"] == "tables":
        s.update(n_blocks_out=torch.zeros_like(s["n_blocks"]), n_free_out=torch.zeros_like(s["n_free"]),
                 short_blocks=torch.zeros_like(s["n_free"]))
    elif case["op"] == "slots":
        s.update(cu=torch.zeros((N, G, B + 1), dtype=torch.int32, device=DEVICE),
                 slots=torch.full((N, G, case["room"]), -7, dtype=torch.int64, device=DEVICE),
                 n_new=None if case["new"] == "one" else _newest(case, after, gen, DEVICE).to(torch.int32))
    else:
        s.update(n_seq=torch.zeros((N, G), dtype=torch.int32, device=DEVICE),
                 seq_slot=torch.zeros((N, G, B), dtype=torch.int32, device=DEVICE),
                 indptr=torch.zeros((N, G, B + 1), dtype=torch.int32, device=DEVICE),
                 indices=torch.full((N, G, P), -7, dtype=torch.int32, device=DEVICE),
                 last_tokens=torch.zeros((N, G, B), dtype=torch.int32, device=DEVICE))
    return s


def _outputs(s):
    names = {"tables": ("table", "free_list", "n_blocks_out", "n_free_out", "short_blocks"), "slots": ("cu", "slots"),
             "pages": ("n_seq", "seq_slot", "indptr", "indices", "last_tokens")}[s["case"]["op"]]
    return {n: s[n] for n in names}


def run(state):
    s, op = state, state["case"]["op"]
    if own:
        cache = s.get("cache")
        if cache is None:                                          # the handle that a user's program makes once for its buffers
            from paper_2605_06113_b200.binding import BlockCache
            cache = s["cache"] = BlockCache(s["table"], s["n_blocks"], s["free_list"], s["n_free"], s["block"])
        if op == "tables":
            cache.block_tables(s["length"], s["n_blocks_out"], s["n_free_out"], s["short_blocks"], step=s["step"])
        elif op == "slots":
            cache.slot_map(s["length"], s["cu"], s["slots"], n_new=s["n_new"], step=s["step"])
        else:
            cache.page_lists(s["length"], s["n_seq"], s["seq_slot"], s["indptr"], s["indices"], s["last_tokens"], step=s["step"])
    elif op == "tables":
        _plain_tables(s)
    elif op == "slots":
        _plain_slots(s)
    else:
        _plain_pages(s)
    return _outputs(s)


def _tokens(s):
    """[N G, B] tokens of each slot's request, 0 for a free slot."""
    n = s["length"].to(torch.int64)
    if s["step"] is not None:
        n = torch.where(n == EMPTY, 0, n + s["step"][:, None, None])
    return n.clamp(0, MOST).flatten(0, 1)


def _ragged(count):
    """Rows of `count` [W, B] items one after another: each item's row (flat), its place in the row and in its worker."""
    each = count.flatten()
    row = torch.repeat_interleave(each)
    j = torch.arange(row.numel(), device=row.device) - (each.cumsum(0) - each)[row]
    within = (count.cumsum(1) - count).flatten()
    return row, j, within[row] + j


def _plain_tables(s):
    B, T, P = s["table"].shape[2], s["table"].shape[3], s["free_list"].shape[2]
    table, free = s["table"].view(-1), s["free_list"].view(-1)
    n, have, n_free = _tokens(s), s["n_blocks"].flatten(0, 1).to(torch.int64), s["n_free"].flatten().to(torch.int64)
    need = (n + s["block"] - 1) // s["block"]
    want, back = (need - have).clamp_min(0), (have - need).clamp_min(0)
    ask = torch.where(need <= T, want, 0)
    R = back.sum(1)
    give = torch.where(ask.cumsum(1) <= (n_free + R)[:, None], ask, 0)
    A = give.sum(1)
    # the blocks taken back, by slot and place
    row, j, rank = _ragged(back)
    w = row // B
    blocks = table[row * T + need.flatten()[row] + j]
    first = R.cumsum(0) - R
    # those blocks serve the growth first, then the free list from its end
    row_g, j_g, rank_g = _ragged(give)
    w_g = row_g // B
    old = rank_g < R[w_g]
    top = free[(w_g * P + (n_free + R)[w_g] - 1 - rank_g).clamp(min=0, max=free.numel() - 1)]
    if blocks.numel():
        top = torch.where(old, blocks[(first[w_g] + rank_g).clamp(max=blocks.numel() - 1)], top)
    table[row_g * T + have.flatten()[row_g] + j_g] = top
    # what is left of them joins the free list, the first on top
    left = rank >= A[w]
    free[(w * P + n_free[w] + R[w] - 1 - rank)[left]] = blocks[left]
    s["n_blocks_out"].copy_((have + give - back).view_as(s["n_blocks"]))
    s["n_free_out"].copy_((n_free + R - A).view_as(s["n_free"]))
    s["short_blocks"].copy_((want - give).sum(1).clamp(max=MOST).view_as(s["n_free"]))


def _plain_slots(s):
    B, T, block, room = s["table"].shape[2], s["table"].shape[3], s["block"], s["slots"].shape[2]
    n, have = _tokens(s), s["n_blocks"].flatten(0, 1).to(torch.int64)
    q = (n > 0).to(torch.int64) if s["n_new"] is None else torch.minimum(s["n_new"].flatten(0, 1).to(torch.int64).clamp_min(0), n)
    row, j, at = _ragged(q)
    p = (n - q).flatten()[row] + j
    column = p // block
    slot = s["table"].view(-1)[row * T + column.clamp(max=T - 1)].to(torch.int64) * block + p % block
    slot = torch.where(column < have.flatten()[row], slot, -1)
    inside = at < room
    s["slots"].view(-1)[((row // B) * room + at)[inside]] = slot[inside]
    s["cu"].view(-1, B + 1)[:, 1:] = q.cumsum(1).clamp(max=MOST)
    s["cu"].view(-1, B + 1)[:, 0] = 0


def _plain_pages(s):
    B, T, block, P = s["table"].shape[2], s["table"].shape[3], s["block"], s["free_list"].shape[2]
    n, have = _tokens(s), s["n_blocks"].flatten(0, 1).to(torch.int64)
    need = (n + block - 1) // block
    pages = torch.minimum(need, have)
    last = torch.where(need <= have, n - (need - 1) * block, block)
    last = torch.where(pages > 0, last, 0)
    running = n > 0
    count = running.sum(1, keepdim=True)
    order = torch.sort(running.to(torch.int8), dim=1, descending=True, stable=True).indices         # running slots first
    packed = torch.arange(B, device=n.device) < count
    s["n_seq"].copy_(count.view_as(s["n_seq"]))
    s["seq_slot"].copy_(torch.where(packed, order, -1).view_as(s["seq_slot"]))
    s["last_tokens"].copy_(torch.where(packed, last.gather(1, order), 0).view_as(s["last_tokens"]))
    indptr = s["indptr"].view(-1, B + 1)
    indptr[:, 1:] = torch.where(packed, pages.gather(1, order), 0).cumsum(1)
    indptr[:, 0] = 0
    row, j, at = _ragged(pages)
    s["indices"].view(-1)[(row // B) * P + at] = s["table"].view(-1)[row * T + j]


def work(case):
    """What a pass reads and writes once, from a sample of the case's own distributions."""
    W, B, block = case["N"] * case["G"], case["B"], case["block"]
    rows = min(W, max(1, 65536 // B))
    gen = torch.Generator().manual_seed(1)
    before, after = _before_and_after(case, (rows, B), gen, "cpu")
    held, need = _held(case, (before + block - 1) // block), (after + block - 1) // block
    slots, scale = W * B, W / rows
    once = 4 * case["N"] if case["stepped"] else 0
    if case["op"] == "tables":
        back, ask = (held - need).clamp_min(0), (need - held).clamp_min(0)
        R = back.sum(1)
        room = case["pool"] - held.sum(1) + R
        A = torch.where(ask.cumsum(1) <= room[:, None], ask, 0).sum(1)
        moved = float(torch.maximum(A, R).sum()) * scale          # blocks that change place, each read and written
        return {"bytes": 12 * slots + 12 * W + once + 8 * moved, "flops": 0}
    if case["op"] == "slots":
        q = (after > 0).to(torch.int64) if case["new"] == "one" else _newest(case, after, gen, "cpu")
        tokens = float(q.sum(1).clamp(max=case["room"]).sum()) * scale
        reads = float(torch.where(q > 0, (after - 1) // block - (after - q) // block + 1, 0).sum()) * scale
        return {"bytes": (12 if case["new"] == "one" else 16) * slots + 4 * W + once + 4 * reads + 8 * tokens, "flops": 0}
    pages = float(torch.minimum(need, held).sum()) * scale
    return {"bytes": 20 * slots + 8 * W + once + 8 * pages, "flops": 0}


def exact(case, seed):
    """The same by the definition, one request at a time; None for cases with too many requests or blocks for that."""
    if case["N"] * case["G"] * case["B"] > 150000 or case["N"] * case["G"] * case["B"] * case["columns"] > 2 ** 27:
        return None

    def tables(h, at, tokens):
        block, T = case["block"], case["columns"]
        table, free, held, n_free = h["table"][at], h["free_list"][at], h["n_blocks"][at].tolist(), int(h["n_free"][at])
        stack = free[:n_free].tolist()
        need = [-(-n // block) for n in tokens]
        back = []
        for b, k in enumerate(held):
            if need[b] < k:
                back += table[b, need[b]:k].tolist()
                held[b] = need[b]
        stack += back[::-1]                                            # the first block taken back is the first one given out
        missing = []
        full = False
        for b, k in enumerate(need):
            if k > held[b]:
                full = full or (k <= T and k - held[b] > len(stack))
                if k > T or full:
                    missing.append(k - held[b])
                    continue
                for c in range(held[b], k):
                    table[b, c] = stack.pop()
                held[b] = k
        if len(stack) > n_free:
            free[n_free:len(stack)] = stack[n_free:]
        h["n_blocks_out"][at], h["n_free_out"][at], h["short_blocks"][at] = held, len(stack), min(MOST, sum(missing))

    def slots(h, at, tokens):
        block, room = case["block"], case["room"]
        out, place = h["slots"][at], 0
        for b, n in enumerate(tokens):
            q = (1 if n else 0) if case["new"] == "one" else min(n, max(0, int(h["n_new"][at][b])))
            h["cu"][at][b] = min(place, MOST)
            p = np.arange(n - q, n, dtype=np.int64)[: max(0, room - place)]
            column = p // block
            ids = h["table"][at][b].astype(np.int64)[np.minimum(column, case["columns"] - 1)]
            out[place: place + p.size] = np.where(column < h["n_blocks"][at][b], ids * block + p % block, -1)
            place += q
        h["cu"][at][len(tokens)] = min(place, MOST)

    def pages(h, at, tokens):
        block = case["block"]
        h["seq_slot"][at], h["last_tokens"][at] = -1, 0
        r = place = 0
        for b, n in enumerate(tokens):
            if n:
                k = min(-(-n // block), int(h["n_blocks"][at][b]))
                h["seq_slot"][at][r], h["indptr"][at][r] = b, place
                h["last_tokens"][at][r] = min(block, n - (k - 1) * block) if k else 0
                h["indices"][at][place: place + k] = h["table"][at][b, :k]
                place += k
                r += 1
        h["n_seq"][at], h["indptr"][at][r:] = r, place

    s = prepare(case, seed)
    host = {k: v.cpu().numpy() for k, v in s.items() if isinstance(v, torch.Tensor)}
    one = {"tables": tables, "slots": slots, "pages": pages}[case["op"]]
    for i in range(case["N"]):
        step = 0 if s["step"] is None else int(host["step"][i])
        for g in range(case["G"]):
            tokens = [0 if v == EMPTY else max(0, int(v) + step) for v in host["length"][i, g]]
            one(host, (i, g), tokens)
    return {n: host[n] for n in _outputs(s)}
