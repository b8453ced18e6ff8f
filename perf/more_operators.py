"""Operators of serving with shared prefixes and a bounded cache: what they compute, plainly, and their workloads.

Each case is a dict of plain values.  ``listed()`` gives fixed ones, ``draw(rng)`` one more of the same
ranges; ``prepare`` makes the inputs on the GPU, ``run`` makes one pass (with ``own`` through the
framework's entry points, else in elementary torch operations), ``work`` counts the bytes and operations
that pass cannot do without, ``exact`` computes the result in 64 bits from the definitions.

Operations:
  shared   one token per session; the sessions of a group have the first blocks of their tables in common
  weights  the same, and each key's attention probability, summed over the query heads of its KV head,
           is added to the key's accumulated weight (a new token's is set)
  prompt   the same sums over the last rows of a turn of n new tokens, causally
  evict    of each session that is longer than a limit, every layer and KV head keeps `budget` tokens: the
           first ones, the latest ones and those of the largest accumulated weight (ties: the lower slot);
           the i-th evicted slot below the budget takes the i-th kept token from behind it, and the blocks
           behind the budget go back to the ring of free blocks
"""
import math
import random

import numpy as np
import torch

own = False

BLOCK = 16


def _decode(name, op, sessions, lo, hi, hq, hkv, d, groups=0, grouped=0, p_lo=0, p_hi=0, first=0, dist="uniform", shape=1):
    c = {"op": op, "sessions": sessions, "lo": lo, "hi": hi, "dist": dist, "groups": groups, "grouped": grouped,
         "p_lo": p_lo, "p_hi": p_hi, "first": first, "hq": hq, "hkv": hkv, "d": d, "shape": shape}
    return dict(c, name=name) if name else c


def _prompt(name, sessions, n_lo, n_hi, c_lo, c_hi, rows, hq, hkv, d, first=0, shape=1):
    c = {"op": "prompt", "sessions": sessions, "n_lo": n_lo, "n_hi": n_hi, "c_lo": c_lo, "c_hi": c_hi, "rows": rows,
         "first": first, "hq": hq, "hkv": hkv, "d": d, "shape": shape}
    return dict(c, name=name) if name else c


def _evict(name, sessions, lo, hi, budget, limit, recent, first, layers, hkv, d, fresh=False, shape=1):
    c = {"op": "evict", "sessions": sessions, "lo": lo, "hi": hi, "budget": budget, "limit": limit, "recent": recent,
         "first": first, "layers": layers, "hkv": hkv, "d": d, "fresh": fresh, "shape": shape}
    return dict(c, name=name) if name else c


def listed():
    return [
        # Three callers of one service, early in their conversations: the instructions are shared, latency counts.
        _decode("shared three callers", "shared", 3, 1, 200, 32, 4, 128, groups=1, grouped=3, p_lo=40, p_hi=40),
        # A thinker batch of 64 sessions that all begin with the same 4096 tokens of instructions and tools.
        _decode("shared thinker 64", "shared", 64, 64, 4096, 32, 4, 128, groups=1, grouped=64, p_lo=256, p_hi=256,
                dist="lognormal"),
        # A talker step: 256 sessions in eight voices, each with its own prompt; some sessions use none.
        _decode("shared talker 256", "shared", 256, 50, 1500, 16, 2, 128, groups=8, grouped=240, p_lo=32, p_hi=96),
        # A small model of as many KV heads as query heads, ragged groups, half of the sessions in none.
        _decode("shared ragged d64", "shared", 41, 1, 700, 8, 8, 64, groups=5, grouped=23, p_lo=1, p_hi=150),
        # One user's decode step while the cache fills up: latency.
        _decode("weights one session", "weights", 1, 1789, 1789, 32, 4, 128),
        # The thinker's batch before anything is evicted: lognormal contexts of up to 16k.
        _decode("weights thinker 64", "weights", 64, 512, 16384, 32, 4, 128, first=4, dist="lognormal"),
        # A talker step over bounded caches behind two shared voice prompts.
        _decode("weights talker 256", "weights", 256, 900, 1100, 16, 2, 128, groups=2, grouped=200, p_lo=20, p_hi=60),
        # One user's turn of a few hundred tokens: its last 32 rows say what of the history matters.
        _prompt("prompt one turn", 1, 301, 301, 1789, 1789, 32, 32, 4, 128),
        # A batch of next turns over long histories, observed by their last 64 rows.
        _prompt("prompt next turn 32", 32, 256, 2048, 2048, 8192, 64, 32, 4, 128, first=4),
        # First turns of a small model, every row observed.
        _prompt("prompt first d64", 8, 50, 700, 0, 0, 700, 8, 8, 64),
        # Steps of 64 sessions around their limit: half of them fall back to the budget, in eight layers.
        _evict("evict step 64", 64, 2047, 2079, 2048, 2063, 256, 4, 8, 4, 128),
        # Prompts just read are cut to their budget.
        _evict("evict prompts 8", 8, 900, 16384, 1024, 1039, 128, 16, 4, 4, 128, fresh=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    shape = rng.randrange(1, 1 << 30)
    op = rng.choice(["shared", "shared", "weights", "prompt", "evict"])
    d = rng.choice([64, 128, 128])
    hkv = rng.choice([1, 2, 4, 4, 8])
    hq = hkv * rng.choice([1, 2, 4, 8, 8])
    if op in ("shared", "weights"):
        sessions = _log_int(rng, 1, 256)
        hi = _log_int(rng, 1, 4096 if op == "shared" else 16384)
        lo = max(1, int(hi * rng.uniform(0.02, 1.0)))
        groups = 0 if op == "weights" and rng.random() < 0.5 else min(sessions, rng.choice([1, 1, 2, 3, 8]))
        grouped = rng.randrange(groups, sessions + 1) if groups else 0
        p_hi = _log_int(rng, 1, 256)
        p_lo = max(1, int(p_hi * rng.uniform(0.2, 1.0)))
        # (the plain form goes over the shared blocks once per session)
        while sessions > max(1, groups) and sessions * (hi + p_hi * BLOCK) * hkv * d > 64 * 8192 * 4 * 128:
            sessions -= 1
        return _decode(None, op, sessions, lo, hi, hq, hkv, d, groups=groups, grouped=min(grouped, sessions), p_lo=p_lo,
                       p_hi=p_hi, first=rng.choice([0, 0, 4, 16, 37]) if op == "weights" else 0,
                       dist=rng.choice(["uniform", "lognormal"]), shape=shape)
    if op == "prompt":
        sessions = _log_int(rng, 1, 32)
        n_hi = _log_int(rng, 1, 2048)
        n_lo = max(1, int(n_hi * rng.uniform(0.1, 1.0)))
        c_hi = 0 if rng.random() < 0.15 else _log_int(rng, 16, 8192)
        c_lo = int(c_hi * rng.uniform(0.1, 1.0))
        rows = rng.choice([1, 16, 32, 64, 64, n_hi])
        while sessions > 1 and sessions * min(rows, n_hi) * hq * (n_hi + c_hi) > 32 * 64 * 32 * 8192:
            sessions -= 1
        while rows > 64 and min(rows, n_hi) * hq * (n_hi + c_hi) > 32 * 64 * 32 * 8192:
            rows -= 64
        return _prompt(None, sessions, n_lo, n_hi, c_lo, c_hi, rows, hq, hkv, d, first=rng.choice([0, 0, 4, 37]), shape=shape)
    sessions = _log_int(rng, 1, 64)
    budget = _log_int(rng, 40, 2048)
    recent = rng.randrange(0, budget // 2)
    first = rng.choice([0, 4, 16, rng.randrange(0, budget // 4)])
    limit = budget + rng.choice([0, 15, 15, 31, 100])
    fresh = rng.random() < 0.4
    hi = _log_int(rng, limit + 1, 16384) if fresh else limit + 16
    lo = max(1, int(limit * rng.uniform(0.5, 1.0)))
    layers = _log_int(rng, 1, 8)
    while sessions > 1 and sessions * layers * hkv * hi * d > 64 * 2079 * 8 * 4 * 128:
        sessions -= 1
    return _evict(None, sessions, lo, hi, budget, limit, recent, first, layers, hkv, d, fresh=fresh, shape=shape)


# ---------------------------------------------------------------------------------------------------
# Lengths and inputs


def _lens(c):
    """New tokens, tokens in the cache before them, and blocks shared with others, per session; the members
    of each group: part of the case, the same for every seed."""
    r = random.Random(c["shape"])
    s = c["sessions"]
    if c["op"] == "prompt":
        n = [r.randint(c["n_lo"], c["n_hi"]) for _ in range(s)]
        x = [r.randint(c["c_lo"], c["c_hi"]) for _ in range(s)]
        return np.asarray(n), np.asarray(x), np.zeros(s, dtype=np.int64), []
    lo, hi = c["lo"], c["hi"]
    if c.get("dist") == "lognormal":
        mid = math.sqrt(lo * hi) * 1.4
        x = [min(hi, max(lo, round(math.exp(math.log(mid) + r.gauss(0.0, 1.0))))) for _ in range(s)]
    else:
        x = [r.randint(lo, hi) for _ in range(s)]
    x, shared = np.asarray(x), np.zeros(s, dtype=np.int64)
    if c["op"] == "evict":
        return np.zeros(s, dtype=np.int64), x, shared, []
    order = list(range(s))
    r.shuffle(order)
    cuts = sorted(r.sample(range(1, c["grouped"]), c["groups"] - 1)) if c["groups"] > 1 else []
    members = [order[a:b] for a, b in zip([0] + cuts, cuts + [c["grouped"]])] if c["groups"] else []
    for m in members:
        shared[m] = r.randint(c["p_lo"], c["p_hi"])
    return np.ones(s, dtype=np.int64), x - 1 + shared * BLOCK, shared, members


def _kept(c, x):
    """Tokens that a session keeps."""
    m = np.minimum(x, max(c["budget"], c["first"] + c["recent"]))
    return np.where(x > c["limit"], m, x)


def prepare(case, seed):
    torch.cuda.set_device(0)
    g = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16)

    def int32(a):
        return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()

    n, ctx, shared, members = _lens(case)
    s, op, hkv, d = len(n), case["op"], case["hkv"], case["d"]
    total = n + ctx
    need = -(-total // BLOCK)
    width = int(need.max())
    # The ids of a shuffled pool a quarter larger than the blocks in use; a group's first blocks are those of its first member.
    j = np.arange(width)[None]
    leader = np.arange(s)
    for m in members:
        leader[m] = m[0]
    mine = (j < need[:, None]) & ((j >= shared[:, None]) | (leader == np.arange(s))[:, None])
    at = np.cumsum(mine.reshape(-1)).reshape(s, width) - 1
    at = np.where(j < shared[:, None], at[leader], at)
    used = int(mine.sum())
    nb = used + (used + 3) // 4
    perm = torch.randperm(nb, generator=g, device="cuda").to(torch.int32)
    live = torch.from_numpy(j < need[:, None]).cuda()
    tables = torch.where(live, perm[torch.from_numpy(at).cuda().clamp(min=0)], -1).to(torch.int32).contiguous()
    layers = case.get("layers", 1)
    t = {"op": op, "tables": tables, "lens": int32(total), "pool": normal(layers, nb, 2, hkv, BLOCK * d),
         "longest": int(total.max()), "scale": d ** -0.5}
    first = case["first"]
    t["first"] = torch.full((s,), first, dtype=torch.int32, device="cuda") if first else None
    if op in ("shared", "weights"):
        t["q"] = normal(s, case["hq"], d)
        t["out"] = torch.empty_like(t["q"])
        t["starts"] = int32(np.cumsum([0] + [len(m) for m in members])) if members else None
        t["members"] = int32(np.concatenate(members)) if members else None
        t["prefix"] = int32([shared[m[0]] for m in members]) if members else None
        t["shared"] = int32(shared)
    if op in ("weights", "prompt"):
        t["reused"] = int32(ctx)
        # A conversation whose cache was cut before: the new tokens are further on than their place in the cache says.
        t["begin"] = int32(ctx * 2 + 5)
    if op == "prompt":
        cu = np.concatenate([[0], np.cumsum(n)])
        t["q"], t["cu"] = normal(int(cu[-1]), case["hq"], d), int32(cu)
        t["max_new"], t["rows"] = int(n.max()), case["rows"]
    if op != "shared":
        shape = (layers, nb, hkv, BLOCK)
        # what tokens gather over many steps: a few of them much, most of them little
        t["weights"] = torch.randn(shape, generator=g, device="cuda").mul_(1.5).exp_()
        t["positions"] = torch.full(shape, -1, dtype=torch.int32, device="cuda")
    if op == "evict":
        t.update({k: case[k] for k in ("budget", "limit", "recent")})
        # Tokens stand in their order after a prompt, anywhere after earlier evictions.
        lens = t["lens"].long()
        t["next_pos"] = t["lens"] if case["fresh"] else t["lens"] * 3
        slot = torch.arange(width * BLOCK, device="cuda")
        live = slot < lens[:, None]
        key = slot.expand(layers, hkv, s, -1).float() if case["fresh"] else torch.rand(
            (layers, hkv, s, width * BLOCK), generator=g, device="cuda")
        age = key.masked_fill(~live, -1.0).argsort(-1, descending=True).argsort(-1)      # 0: the latest token
        if not case["fresh"]:
            age = torch.where(age < case["recent"], age, 2 * age - case["recent"])
        pos = (t["next_pos"].long()[:, None] - 1 - age).to(torch.int32)
        where = tables.long().clamp(min=0).repeat_interleave(BLOCK, 1)
        rows = live.nonzero(as_tuple=True)
        t["positions"][:, where[rows], :, rows[1] % BLOCK] = pos[:, :, rows[0], rows[1]].permute(2, 0, 1)
        t["weights_next"], t["positions_next"] = torch.zeros_like(t["weights"]), torch.zeros_like(t["positions"])
        t["next"] = torch.empty_like(t["lens"])
        start = (1 << 33) + int(seed) % 1000              # a ring in use for long
        t["ring"] = torch.full((nb,), -1, dtype=torch.int32, device="cuda")
        t["ring"][(torch.arange(nb - used, device="cuda") + start) % nb] = perm[used:]
        t["counts"] = torch.tensor([start, start + nb - used], dtype=torch.int64, device="cuda")
        t["next_counts"] = torch.empty_like(t["counts"])
    if own:
        # The pool's handle and the workspace that a serving program keeps.
        from paper_2606_22983_amd import kv
        t["handle"] = h = kv.kv_pool_create(t["pool"], layers, nb, hkv, d)
        size = 0
        if op == "shared":
            size = kv.decode_shared_workspace_bytes(h, s, case["hq"], len(members), case["grouped"])
        elif op == "weights":
            size = kv.decode_weights_workspace_bytes(h, s, case["hq"], len(members), case["grouped"])
        elif op == "prompt":
            size = kv.weights_prefill_workspace_bytes(h, s, case["hq"], int(n.sum()), t["max_new"], case["rows"], width)
        t["ws"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    return t


# ---------------------------------------------------------------------------------------------------
# The plain forms


def _views(pool, d):
    """The K tiles as [block][head][d / 8][16 tokens][8] and the V tiles as [block][head][d][16 tokens]."""
    nb, hkv = pool.shape[0], pool.shape[2]
    return pool[:, 0].view(nb, hkv, d // 8, BLOCK, 8), pool[:, 1].view(nb, hkv, d, BLOCK)


def _probabilities(t, q, pos):
    """q [S][R][hq][d], whose rows stand at positions pos [S][R] (-1: no row): their probabilities over the
    session's slots, [S][hkv][R][G][slots], and the slots' blocks."""
    s, r, hq, d = q.shape
    kt, _ = _views(t["pool"][0], d)
    hkv = kt.shape[1]
    key = torch.arange(t["longest"], device=q.device)
    block = t["tables"][:, key // BLOCK].long().clamp(min=0)
    k = kt[block, :, :, key % BLOCK].reshape(s, -1, hkv, d).transpose(1, 2).float().reshape(s * hkv, -1, d)
    qg = q.float().view(s, r, hkv, hq // hkv, d).transpose(1, 2).reshape(s * hkv, -1, d)
    x = torch.bmm(qg, k.transpose(1, 2).contiguous()).mul_(t["scale"]).view(s, hkv, r, hq // hkv, -1)
    unseen = (key > pos[:, :, None])[:, None, :, None]
    x.masked_fill_(unseen, -math.inf)
    x.sub_(x.amax(-1, keepdim=True).clamp(min=-1e30)).exp_()
    return x.div_(x.sum(-1, keepdim=True).clamp(min=1e-30)), block, key


def _gather(t, p, block, key, begin, upto):
    """Sums p [S][hkv][slots] into the weights of the slots begin .. upto - 1; tokens that are new are set."""
    s = p.shape[0]
    use = ((key >= begin[:, None]) & (key < upto[:, None])).nonzero(as_tuple=True)
    b, o = block[use], key[use[1]] % BLOCK
    new = (use[1] >= t["reused"][use[0]])[:, None]
    add = p[use[0], :, use[1]]
    w, pos = t["weights"][0], t["positions"][0]
    w[b, :, o] = torch.where(new, add, w[b, :, o] + add)
    at = (t["begin"][use[0]] + use[1] - t["reused"][use[0]]).to(torch.int32)[:, None]
    pos[b, :, o] = torch.where(new, at, pos[b, :, o])


def _plain_decode(t):
    s, hq, d = t["q"].shape
    hkv = t["pool"].shape[3]
    lens = t["lens"].long()
    p, block, key = _probabilities(t, t["q"][:, None], (lens - 1)[:, None])
    _, vt = _views(t["pool"][0], d)
    v = vt[block, :, :, key % BLOCK].transpose(1, 2).float().reshape(s * hkv, -1, d)
    t["out"].copy_(torch.bmm(p.view(s * hkv, hq // hkv, -1), v).view(s, hq, d))
    if t["op"] == "weights":
        begin = t["shared"].long() * BLOCK
        begin = begin if t["first"] is None else torch.maximum(begin, t["first"].long())
        _gather(t, p.sum((2, 3)), block, key, begin, lens)


def _plain_prompt(t):
    cu, ctx = t["cu"].long(), t["reused"].long()
    n = cu[1:] - cu[:-1]
    # the last rows of each turn, counted from its end
    back = torch.arange(min(t["rows"], t["max_new"]), device=cu.device)
    there = back < n[:, None]
    row = (cu[1:, None] - 1 - back).clamp(min=0)
    pos = torch.where(there, (ctx + n)[:, None] - 1 - back, -1)
    p, block, key = _probabilities(t, t["q"][row], pos)
    begin = torch.zeros_like(ctx) if t["first"] is None else t["first"].long()
    _gather(t, p.sum((2, 3)), block, key, begin, ctx + n)


def _plain_evict(t):
    lens, tables, ring, counts = t["lens"].long(), t["tables"].long(), t["ring"], t["counts"]
    s, width = tables.shape
    layers, nb, _, hkv = t["pool"].shape[:4]
    d = t["pool"].shape[4] // BLOCK
    first = torch.zeros_like(lens) if t["first"] is None else t["first"].long()
    keep = torch.minimum(lens, (first + t["recent"]).clamp(min=t["budget"]))
    keep = torch.where(lens > t["limit"], keep, lens)
    slot = torch.arange(t["longest"], device=lens.device)
    block, off = tables[:, slot // BLOCK].clamp(min=0), slot % BLOCK
    w = t["weights"][:, block, :, off].permute(2, 3, 0, 1)           # [layer][head][session][slot]
    pos = t["positions"][:, block, :, off].permute(2, 3, 0, 1)
    top = (slot < first[:, None]) | (pos >= t["next_pos"][:, None] - t["recent"])
    w = w.masked_fill(top, math.inf).masked_fill(slot >= lens[:, None], -math.inf)
    order = w.sort(dim=-1, descending=True, stable=True).indices
    rank = torch.empty_like(order).scatter_(-1, order, slot.expand_as(order))
    stays = rank < keep[:, None]
    below = slot < keep[:, None]
    # both in rows of (layer, head, session) and, within one, in the order of the slots: the i-th belong together
    hole, mover = (below & ~stays).nonzero(as_tuple=True), (stays & ~below).nonzero(as_tuple=True)
    la, h = hole[0], hole[1]
    db, do = block[hole[2], hole[3]], hole[3] % BLOCK
    sb, so = block[mover[2], mover[3]], mover[3] % BLOCK
    kt, vt = t["pool"][:, :, 0].view(layers, nb, hkv, d // 8, BLOCK, 8), t["pool"][:, :, 1].view(layers, nb, hkv, d, BLOCK)
    kt[la, db, h, :, do] = kt[la, sb, h, :, so]
    vt[la, db, h, :, do] = vt[la, sb, h, :, so]
    live = below.nonzero(as_tuple=True)
    lb, lo = block[live], live[1] % BLOCK
    for name in ("weights", "positions"):
        old, new = t[name], t[name + "_next"]
        new[:, lb, :, lo] = old[:, lb, :, lo]
        new[la, db, h, do] = old[la, sb, h, so]
    t["next"].copy_(keep)
    j = torch.arange(width, device=lens.device)
    give = (j >= ((keep + BLOCK - 1) // BLOCK)[:, None]) & (j < ((lens + BLOCK - 1) // BLOCK)[:, None])
    ids = tables[give]
    ring[(counts[1] + torch.arange(ids.numel(), device=ids.device)) % ring.numel()] = ids.to(torch.int32)
    t["next_counts"].copy_(torch.stack([counts[0], counts[1] + ids.numel()]))


def run(state):
    t = state
    op = t["op"]
    if own:
        from paper_2606_22983_amd import kv
        if op == "shared":
            kv.paged_attn_decode_shared(t["handle"], 0, t["q"], t["tables"], t["lens"], t["starts"], t["members"],
                                        t["prefix"], t["scale"], t["out"], t["ws"])
        elif op == "weights":
            kv.paged_attn_decode_weights(t["handle"], 0, t["q"], t["tables"], t["lens"], t["scale"], t["out"],
                                         t["weights"], t["positions"], t["ws"], reused_lens=t["reused"],
                                         first_positions=t["begin"], first_lens=t["first"], group_starts=t["starts"],
                                         group_members=t["members"], prefix_blocks=t["prefix"])
        elif op == "prompt":
            kv.kv_weights_prefill(t["handle"], 0, t["q"], t["cu"], t["reused"], t["max_new"], t["tables"], t["rows"],
                                  t["scale"], t["weights"], t["positions"], t["ws"], first_positions=t["begin"],
                                  first_lens=t["first"])
        else:
            kv.kv_evict(t["handle"], t["lens"], t["tables"], t["budget"], t["limit"], t["recent"], t["next_pos"],
                        t["weights"], t["positions"], t["next"], weights_next=t["weights_next"],
                        positions_next=t["positions_next"], first_lens=t["first"], free_ring=t["ring"],
                        free_counts=t["counts"], next_counts=t["next_counts"])
    elif op == "prompt":
        _plain_prompt(t)
    elif op == "evict":
        _plain_evict(t)
    else:
        _plain_decode(t)
    if op == "shared":
        return {"out": t["out"]}
    if op == "weights":
        return {k: t[k] for k in ("out", "weights", "positions")}
    if op == "prompt":
        return {k: t[k] for k in ("weights", "positions")}
    return {k: t[k] for k in ("pool", "weights_next", "positions_next", "next", "ring", "next_counts")}


def work(case):
    n, ctx, shared, members = _lens(case)
    s, hkv, d, op, first = len(n), case["hkv"], case["d"], case["op"], case["first"]
    total = n + ctx
    if op == "evict":
        m = _kept(case, total)
        cut = total > m
        rows = case["layers"] * hkv
        # Each slot's weight and position read and the kept ones written; tokens that move (all from behind the budget
        # that stay: at least the latest ones) read and written; lengths, table entries and ring.
        late = np.minimum(total - m, case["recent"]) if case["fresh"] else ((total - m) * m / np.maximum(total, 1)).astype(np.int64)
        moved = int(late[cut].sum()) * rows
        gone = int((-(-total // BLOCK) - -(-m // BLOCK)).sum())
        return {"bytes": rows * 8 * int(total.sum() + m.sum()) + moved * 2 * 4 * d + 12 * s + 4 * int((-(-total // BLOCK)).sum())
                + 8 * gone + 32, "flops": 0}
    hq = case["hq"]
    if op == "prompt":
        seen = np.minimum(n, case["rows"])
        keys = int(total.sum())
        pairs = int((seen * total - seen * (seen - 1) // 2).sum())
        q_rows, lead = int(seen.sum()), 0
        summed = int(np.maximum(total - first, 0).sum())
        flops = 2 * hq * d * pairs                            # the scores alone: no values are read
        per_key = 2 * d
    else:
        own_keys = int((total - shared * BLOCK).sum())
        lead = sum(int(shared[m[0]]) * BLOCK for m in members)
        keys, pairs, q_rows = own_keys + lead, int(total.sum()), 2 * s
        summed = int(np.maximum(total - np.maximum(shared * BLOCK, first), 0).sum())
        flops = 4 * hq * d * pairs
        per_key = 4 * d
    # K (and V) of every key read once, a shared one once for its group, rows of q read and of out written, block ids, lengths
    size = keys * hkv * per_key + q_rows * hq * d * 2 + keys // BLOCK * 4 + 8 * s
    if op != "shared":
        # old tokens' weights read, all written, new ones' positions written
        size += hkv * (8 * summed - 4 * int(n.sum()) + 4 * int(n.sum()))
    return {"bytes": size, "flops": flops}


# ---------------------------------------------------------------------------------------------------
# The result in 64 bits


def _exact_evict(case, t):
    """One layer, KV head and session after the other, from sorted lists on the host."""
    w, pos = t["weights"].cpu().numpy(), t["positions"].cpu().numpy()
    wn, pn = np.zeros_like(w), np.zeros_like(pos)
    tables, lens, begin = t["tables"].cpu().numpy(), t["lens"].tolist(), t["next_pos"].tolist()
    ring, (taken, given) = t["ring"].cpu().numpy().copy(), t["counts"].tolist()
    first, recent, keep, moves = case["first"], case["recent"], [], []
    for s, n in enumerate(lens):
        m = n if n <= case["limit"] else min(n, max(case["budget"], first + recent))
        keep.append(m)
        b, o = tables[s, np.arange(n) // BLOCK], np.arange(n) % BLOCK
        for la in range(w.shape[0]):
            for h in range(w.shape[2]):
                ws, ps = w[la, b, h, o], pos[la, b, h, o]
                src = np.arange(m)
                if m < n:
                    sure = (np.arange(n) < first) | (ps >= begin[s] - recent)
                    other = np.nonzero(~sure)[0]
                    # largest weight first, then the lower slot
                    chosen = other[np.lexsort((other, -ws[other].astype(np.float64)))][:m - int(sure.sum())]
                    stay = set(np.nonzero(sure)[0].tolist()) | set(chosen.tolist())
                    late = sorted(i for i in stay if i >= m)
                    for i, to in zip(late, sorted(set(range(m)) - stay)):
                        src[to] = i
                        moves.append((la, h, b[i], o[i], b[to], o[to]))
                wn[la, b[:m], h, o[:m]], pn[la, b[:m], h, o[:m]] = ws[src], ps[src]
        for c in range(-(-m // BLOCK), -(-n // BLOCK)):
            ring[given % len(ring)] = tables[s, c]
            given += 1
    pool = t["pool"]
    if moves:
        layers, nb, _, hkv, tile = pool.shape
        d = tile // BLOCK
        la, h, sb, so, db, do = (torch.from_numpy(np.asarray(x, dtype=np.int64)).cuda()[:, None] for x in zip(*moves))
        e = torch.arange(d, device="cuda")
        flat = pool.view(-1)

        def at(b, kv, o):
            base = (((la * nb + b) * 2 + kv) * hkv + h) * tile
            return base + (e * BLOCK + o if kv else (e // 8) * 128 + o * 8 + e % 8)

        k, v = flat[at(sb, 0, so)], flat[at(sb, 1, so)]
        flat[at(db, 0, do)], flat[at(db, 1, do)] = k, v
    return {"pool": pool, "weights_next": torch.from_numpy(wn).cuda(), "positions_next": torch.from_numpy(pn).cuda(),
            "next": torch.tensor(keep, dtype=torch.int32, device="cuda"), "ring": torch.from_numpy(ring).cuda(),
            "next_counts": torch.tensor([taken, given], device="cuda")}


def exact(case, seed):
    t = prepare(case, seed)
    if case["op"] == "evict":
        return _exact_evict(case, t)
    n, ctx, shared, _ = _lens(case)
    hkv, grp, d, op = case["hkv"], case["hq"] // case["hkv"], case["d"], case["op"]
    pool, tables = t["pool"][0], t["tables"].long()
    out = torch.empty(t["q"].shape, dtype=torch.float64, device="cuda")
    if op != "shared":
        w, pos = t["weights"].double(), t["positions"]
    row = np.concatenate([[0], np.cumsum(n)])
    for s in range(len(n)):
        have, c = int(n[s] + ctx[s]), int(ctx[s])
        key = torch.arange(have, device="cuda")
        b, o = tables[s, key // BLOCK], key % BLOCK
        kk = pool[b, 0].view(have, hkv, d // 8, BLOCK, 8)[key, :, :, o].reshape(have, hkv, d)
        vv = pool[b, 1].view(have, hkv, d, BLOCK)[key, :, :, o]
        r0 = max(0, int(n[s]) - case["rows"]) if op == "prompt" else 0
        begin = max(case["first"], int(shared[s]) * BLOCK)
        for g in range(hkv):
            got = torch.zeros(have, dtype=torch.float64, device="cuda")
            for r in range(r0, int(n[s]), 64):
                e = min(int(n[s]), r + 64)
                q = t["q"][int(row[s]) + r:int(row[s]) + e, g * grp:(g + 1) * grp].double()
                x = q.reshape(-1, d) @ kk[:, g].double().t().contiguous() * d ** -0.5
                future = key[None] > torch.arange(c + r, c + e, device="cuda")[:, None]
                p = torch.softmax(x.view(e - r, grp, have).masked_fill(future[:, None], -math.inf), -1)
                if op != "prompt":
                    out[s, g * grp:(g + 1) * grp] = p[0] @ vv[:, g].double()
                got += p.sum((0, 1))
            if op != "shared":
                # a token of before adds up, one of this call begins
                was = torch.where(key < c, w[0, b, g, o], 0.0)
                w[0, b[begin:], g, o[begin:]] = (was + got)[begin:]
                fresh = max(begin, c)
                pos[0, b[fresh:], g, o[fresh:]] = (key[fresh:] - c + int(t["begin"][s])).to(torch.int32)
    if op == "shared":
        return {"out": out}
    return {"out": out, "weights": w, "positions": pos} if op == "weights" else {"weights": w, "positions": pos}
