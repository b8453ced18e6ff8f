"""Operators of windowed serving over the paged KV cache: what they compute, plainly, and their workloads.

Each case is a dict of plain values.  ``listed()`` gives fixed ones, ``draw(rng)`` one more of the same
ranges; ``prepare`` makes the inputs on the GPU, ``run`` makes one pass (with ``own`` through the
framework's entry points, else in elementary torch operations), ``work`` counts the bytes and operations
that pass cannot do without, ``exact`` computes the result in 64 bits from the definitions.

Operations (positions count from 0; a row at position p sees key t when t <= p and either t < sinks or
t > p - window):
  decode   one token per session over its paged context
  prefill  a turn of n new tokens per session over c tokens in the pool
  tables   block tables, slot map and prefix sums of a step, from the sessions' lengths
  append   K and V rows into the slots that a slot map names
"""
import math
import random

import numpy as np
import torch

own = False

BLOCK = 16
TILE = 64                       # query rows that the plain prefill takes at a time


def _decode(name, sessions, lo, hi, window, sinks, hq, hkv, d, append=False, lens="host", dist="uniform", shape=1):
    c = {"op": "decode", "sessions": sessions, "lo": lo, "hi": hi, "dist": dist, "shape": shape, "window": window,
         "sinks": sinks, "hq": hq, "hkv": hkv, "d": d, "append": append, "lens": lens}
    return dict(c, name=name) if name else c


def _prefill(name, sessions, n_lo, n_hi, c_lo, c_hi, window, sinks, hq, hkv, d, append=True, lens="host", shape=1):
    c = {"op": "prefill", "sessions": sessions, "n_lo": n_lo, "n_hi": n_hi, "c_lo": c_lo, "c_hi": c_hi,
         "shape": shape, "window": window, "sinks": sinks, "hq": hq, "hkv": hkv, "d": d, "append": append, "lens": lens}
    return dict(c, name=name) if name else c


def _tables_case(name, sessions, n_lo, n_hi, c_lo, c_hi, window, sinks, pad=0, shape=1):
    c = {"op": "tables", "sessions": sessions, "n_lo": n_lo, "n_hi": n_hi, "c_lo": c_lo, "c_hi": c_hi,
         "window": window, "sinks": sinks, "pad": pad, "shape": shape}
    return dict(c, name=name) if name else c


def _append_case(name, sessions, n_lo, n_hi, c_lo, c_hi, hkv, d, fused=False, pad=0, shape=1):
    c = {"op": "append", "sessions": sessions, "n_lo": n_lo, "n_hi": n_hi, "c_lo": c_lo, "c_hi": c_hi, "hkv": hkv,
         "d": d, "fused": fused, "pad": pad, "shape": shape}
    return dict(c, name=name) if name else c


def listed():
    return [
        # One user talking to the thinker, far into the conversation: one windowed layer, where latency is everything.
        _decode("decode window one session", 1, 9043, 9043, 1024, 4, 32, 4, 128),
        # The benchmark's thinker batch in a windowed layer: lognormal contexts up to 16k, the last 4096 tokens seen.
        _decode("decode window thinker 64", 64, 512, 16384, 4096, 16, 32, 4, 128, dist="lognormal"),
        # The benchmark's talker step in a windowed layer: 256 sessions, each appending the step's own token.
        _decode("decode window talker 256", 256, 512, 4096, 1024, 4, 16, 2, 128, append=True),
        # A small model (head_dim 64), a short window without sinks, lengths known only on the GPU.
        _decode("decode window d64", 48, 100, 3000, 256, 0, 16, 4, 64, append=True, lens="device"),
        # One user's next turn of a few hundred tokens late in the conversation.
        _prefill("prefill window one turn", 1, 301, 301, 9043, 9043, 2048, 4, 32, 4, 128),
        # The benchmark's next-turn batch in a windowed layer: 32 sessions, turns up to 2048 over up to 32k.
        _prefill("prefill window next turn 32", 32, 256, 2048, 2048, 32768, 4096, 16, 32, 4, 128),
        # First turns of new sessions of a small model with one query head per KV head, lengths only on the GPU.
        _prefill("prefill window first d64", 8, 50, 700, 0, 0, 256, 0, 8, 8, 64, lens="device"),
        # A talker's decode step: one token per session, blocks behind the window given back.
        _tables_case("tables talker step 256", 256, 1, 1, 512, 4096, 1024, 4),
        # The step that begins the next-turn batch: turns of 256 to 2048 tokens, padded to a fixed size.
        _tables_case("tables next turn 32", 32, 256, 2048, 2048, 32768, 4096, 16, pad=1000),
        # The talker step's 256 rows, each into a block of its own.
        _append_case("append talker step 256", 256, 1, 1, 512, 4096, 2, 128),
        # The next-turn batch's rows, K and V as views of a fused projection.
        _append_case("append next turn 32", 32, 256, 2048, 2048, 32768, 4, 128, fused=True),
        # First turns of a small model, behind them rows that belong to no session.
        _append_case("append first turns d64", 8, 50, 700, 0, 37, 8, 64, pad=100),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    shape = rng.randrange(1, 1 << 30)
    kind = rng.choice(["decode", "decode", "prefill", "prefill", "tables", "append"])
    d = rng.choice([64, 128, 128])
    hkv = rng.choice([1, 2, 4, 4, 8])
    hq = hkv * rng.choice([1, 2, 4, 8, 8])
    window = _log_int(rng, 16, 4096)
    sinks = rng.choice([0, 1, 4, 16, rng.randrange(0, 70)])
    if kind == "decode":
        sessions = _log_int(rng, 1, 256)
        hi = _log_int(rng, 64, 16384)
        lo = max(1, int(hi * rng.uniform(0.05, 1.0)))
        while sessions > 1 and sessions * min(hi, window + sinks) * hkv > 64 * 4096 * 4:
            sessions -= 1
        return _decode(None, sessions, lo, hi, window, sinks, hq, hkv, d, append=rng.random() < 0.6,
                       lens=rng.choice(["host", "device"]), dist=rng.choice(["uniform", "lognormal"]), shape=shape)
    if kind == "prefill":
        sessions = _log_int(rng, 1, 32)
        n_hi = _log_int(rng, 8, 2048)
        n_lo = max(1, int(n_hi * rng.uniform(0.1, 1.0)))
        c_hi = 0 if rng.random() < 0.15 else _log_int(rng, 64, 32768)
        c_lo = int(c_hi * rng.uniform(0.1, 1.0))
        while sessions > 1 and sessions * n_hi * hq * d * (window + sinks) > 32 * 1100 * 32 * 128 * 4000:
            sessions -= 1
        return _prefill(None, sessions, n_lo, n_hi, c_lo, c_hi, window, sinks, hq, hkv, d, append=rng.random() < 0.8,
                        lens=rng.choice(["host", "host", "device"]), shape=shape)
    step = rng.random() < 0.5
    sessions = _log_int(rng, 1, 256 if step else 32)
    n_hi = 1 if step else _log_int(rng, 8, 2048)
    n_lo = 1 if step else max(1, int(n_hi * rng.uniform(0.1, 1.0)))
    c_hi = 0 if rng.random() < 0.15 else _log_int(rng, 64, 32768)
    c_lo = int(c_hi * rng.uniform(0.1, 1.0))
    pad = rng.choice([0, 0, rng.randrange(1, 200)])
    if kind == "tables":
        return _tables_case(None, sessions, n_lo, n_hi, c_lo, c_hi, rng.choice([0, window]), sinks, pad=pad, shape=shape)
    while sessions > 1 and sessions * n_hi * hkv * d > 32 * 1100 * 4 * 128:
        sessions -= 1
    return _append_case(None, sessions, n_lo, n_hi, c_lo, c_hi, hkv, d, fused=rng.random() < 0.5, pad=pad, shape=shape)


# ---------------------------------------------------------------------------------------------------
# Lengths and inputs


def _lens(c):
    """(new tokens, tokens in the pool) per session: part of the case, the same for every seed."""
    r = random.Random(c["shape"])
    if c["op"] == "decode":
        lo, hi = c["lo"], c["hi"]
        if c["dist"] == "lognormal":
            mid = math.sqrt(lo * hi) * 1.4
            x = [min(hi, max(lo, round(math.exp(math.log(mid) + r.gauss(0.0, 1.0))))) for _ in range(c["sessions"])]
        else:
            x = [r.randint(lo, hi) for _ in range(c["sessions"])]
        n = [1 if c["append"] else 0] * c["sessions"]
    else:
        n = [r.randint(c["n_lo"], c["n_hi"]) for _ in range(c["sessions"])]
        x = [r.randint(c["c_lo"], c["c_hi"]) for _ in range(c["sessions"])]
    return np.asarray(n, dtype=np.int64), np.asarray(x, dtype=np.int64)


def _dead(x, window, sinks):
    """Blocks that no query at position x or later sees (counted behind the blocks of the sinks)."""
    if not window:
        return np.zeros_like(x)
    return np.maximum((x - window + 1) // BLOCK - -(-sinks // BLOCK), 0)


def _ids(g, need):
    """Block tables over a shuffled pool a quarter larger than the blocks in use: ids where `need` is true, -1 elsewhere."""
    flat = np.cumsum(need.reshape(-1)) - 1
    total = int(flat[-1]) + 1
    num_blocks = total + (total + 3) // 4
    perm = torch.randperm(num_blocks, generator=g, device="cuda").to(torch.int32)
    at = torch.from_numpy(np.maximum(flat, 0).reshape(need.shape)).cuda()
    mask = torch.from_numpy(np.array(need)).cuda()
    return torch.where(mask, perm[at], torch.full_like(at, -1, dtype=torch.int32)).contiguous(), num_blocks, perm[total:]


def prepare(case, seed):
    torch.cuda.set_device(0)
    g = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16)

    def int32(a):
        return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()

    n, ctx = _lens(case)
    s, op = len(n), case["op"]
    t = {"op": op, "window": case.get("window", 0), "sinks": case.get("sinks", 0), "max_new": int(n.max())}
    cu = np.concatenate([[0], np.cumsum(n)])
    total, rows = n + ctx, int(cu[-1])
    width = int((-(-total // BLOCK)).max())
    j = np.arange(width)[None]
    if op == "tables":
        # The session's blocks so far, of which those behind the window are gone; the rest of the pool is free.
        w, k = t["window"], t["sinks"]
        before = np.broadcast_to(j < -(-ctx // BLOCK)[:, None], (s, width))
        first = -(-k // BLOCK)
        gone = (j >= first) & (j < (first + _dead(ctx, w, k))[:, None])
        live, held, spare = _ids(g, np.concatenate([before & ~gone, np.ones((1, width), dtype=bool)]))
        # (the extra row keeps the pool from being empty when no session has a token yet)
        need = int((-(-total // BLOCK) - -(-ctx // BLOCK)).sum())
        more = torch.arange(held, held + max(0, need - spare.numel()), device="cuda", dtype=torch.int32)
        free = torch.cat([spare, live[-1], more])
        t["tables"] = live[:-1].contiguous()
        t["num_blocks"] = held + more.numel()
        # (twice the pool's blocks: room for what a turn longer than the window takes and gives at once)
        t["ring"] = torch.full((2 * t["num_blocks"],), -1, dtype=torch.int32, device="cuda")
        start = (1 << 33) + int(seed) % 1000              # a ring in use for long
        at = (torch.arange(free.numel(), device="cuda") + start) % t["ring"].numel()
        t["ring"][at] = free
        t["counts"] = torch.tensor([start, start + free.numel()], dtype=torch.int64, device="cuda")
        t["lens"], t["new"] = int32(ctx), int32(n)
        t["next_counts"] = torch.empty_like(t["counts"])
        t["next"], t["reused"] = torch.empty_like(t["lens"]), torch.empty_like(t["lens"])
        t["cu"] = torch.empty(s + 1, dtype=torch.int32, device="cuda")
        t["slots"] = torch.empty(rows + case["pad"], dtype=torch.int64, device="cuda")
        if own:
            # A handle with the pool's geometry; the pool itself is not touched.
            from paper_2606_22983_amd import kv
            t["pool"] = torch.empty(kv.ls_kv_pool_bytes(1, t["num_blocks"], 1, 64), dtype=torch.uint8, device="cuda")
            t["handle"] = kv.kv_pool_create(t["pool"], 1, t["num_blocks"], 1, 64)
        return t
    hkv, d = case["hkv"], case["d"]
    blocks = np.broadcast_to(j < -(-total // BLOCK)[:, None], (s, width))
    if op == "append":
        tables, nb, _ = _ids(g, blocks)
        t["pool"] = normal(nb, 2, hkv, BLOCK * d)
        pos = np.concatenate([np.arange(a, a + m) for a, m in zip(ctx, n)])
        who = np.repeat(np.arange(s), n)
        ids = tables[torch.from_numpy(who).cuda(), torch.from_numpy(pos // BLOCK).cuda()].long()
        slots = ids * BLOCK + torch.from_numpy(pos % BLOCK).cuda()
        t["slots"] = torch.cat([slots, torch.full((case["pad"],), -1, device="cuda", dtype=torch.int64)])
        rows += case["pad"]
        if case["fused"]:
            # one projection's output: query heads (as many as KV heads here), K heads, V heads
            qkv = normal(rows, 3 * hkv, d)
            t["k_new"], t["v_new"] = qkv[:, hkv:2 * hkv], qkv[:, 2 * hkv:]
        else:
            t["k_new"], t["v_new"] = normal(rows, hkv, d), normal(rows, hkv, d)
    else:
        # Blocks that no row of the call sees are gone, as they are once the window has passed them.
        first_p = ctx if op == "prefill" or case["append"] else ctx - 1
        lowest = np.maximum(first_p - case["window"] + 1, 0) // BLOCK
        seen = blocks & ((j * BLOCK < case["sinks"]) | (j >= lowest[:, None]))
        t["tables"], nb, _ = _ids(g, seen)
        t["pool"] = normal(nb, 2, hkv, BLOCK * d)
        q_rows = rows if op == "prefill" else s
        t["q"] = normal(q_rows, case["hq"], d)
        t["out"] = torch.empty_like(t["q"])
        t["k_new"] = normal(q_rows, hkv, d) if case["append"] else None
        t["v_new"] = normal(q_rows, hkv, d) if case["append"] else None
        t["lens"], t["cu"] = int32(ctx), int32(cu)
        t["lens_host"] = None
        if case["lens"] == "host":
            t["lens_host"] = np.ascontiguousarray(ctx if op == "decode" else np.stack([n, ctx], 1), dtype=np.int32)
        t["longest"] = int(total.max())
        t["scale"] = d ** -0.5
    if own:
        # The pool's handle and the workspace that a serving program keeps.
        from paper_2606_22983_amd import kv
        t["handle"] = kv.kv_pool_create(t["pool"], 1, nb, hkv, d)
        if op == "decode":
            size = kv.decode_window_workspace_bytes(t["handle"], s, case["hq"], width, case["window"], case["sinks"])
            t["ws"] = torch.empty(size, dtype=torch.uint8, device="cuda")
        elif op == "prefill":
            t["ws"] = (torch.empty(kv.PREFILL_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
                       if case["lens"] == "host" else None)
    return t


# ---------------------------------------------------------------------------------------------------
# The plain forms


def _views(pool, d):
    """The K tiles as [block][head][d / 8][16 tokens][8] and the V tiles as [block][head][d][16 tokens]."""
    nb, hkv = pool.shape[0], pool.shape[2]
    return pool[:, 0].view(nb, hkv, d // 8, BLOCK, 8), pool[:, 1].view(nb, hkv, d, BLOCK)


def _write(pool, slots, k_new, v_new):
    """Rows into their slots; a negative slot leaves its row out."""
    hkv, d = k_new.shape[1], k_new.shape[2]
    kt, vt = _views(pool, d)
    keep = slots >= 0
    b, o = slots[keep] // BLOCK, slots[keep] % BLOCK
    kt[b, :, :, o] = k_new[keep].reshape(-1, hkv, d // 8, 8)
    vt[b, :, :, o] = v_new[keep]


def _attend(t, session, pos, q):
    """q [X][R][hq][d]: R rows of a session at positions pos, pos + 1, ...; their outputs, in 32 bits."""
    x, r, hq, d = q.shape
    w, sinks, pool, tables = t["window"], t["sinks"], t["pool"], t["tables"]
    hkv = pool.shape[2]
    dev = q.device
    lo = (pos - w + 1).clamp(min=sinks)                       # the first key behind the sinks
    count = min(w, t["longest"]) + r - 1
    key = torch.cat([torch.arange(sinks, device=dev).expand(x, sinks), lo[:, None] + torch.arange(count, device=dev)], 1)
    row = pos[:, None] + torch.arange(r, device=dev)
    seen = (key[:, None] <= row[:, :, None]) & ((key[:, None] < sinks) | (key[:, None] > row[:, :, None] - w))
    block = tables[session[:, None], (key // BLOCK).clamp(max=tables.shape[1] - 1)].long().clamp(min=0)
    kt, vt = _views(pool, d)
    k = kt[block, :, :, key % BLOCK].reshape(x, -1, hkv, d).transpose(1, 2).float().contiguous()
    v = vt[block, :, :, key % BLOCK].transpose(1, 2).float().contiguous()
    # [X hkv][R G][d] times [X hkv][d][keys]
    qg = q.float().view(x, r, hkv, hq // hkv, d).transpose(1, 2).reshape(x * hkv, -1, d)
    s = torch.bmm(qg, k.view(x * hkv, -1, d).transpose(1, 2).contiguous()).mul_(t["scale"])
    s = s.view(x, hkv, r, hq // hkv, -1).masked_fill_(~seen[:, None, :, None], -math.inf)
    s.sub_(s.amax(-1, keepdim=True)).exp_()
    s.div_(s.sum(-1, keepdim=True))
    o = torch.bmm(s.view(x * hkv, r * (hq // hkv), -1), v.view(x * hkv, -1, d))
    return o.view(x, hkv, r, hq // hkv, d).transpose(1, 2).reshape(x, r, hq, d)


def _plain_decode(t):
    lens = t["lens"].long()
    session = torch.arange(lens.numel(), device=lens.device)
    if t["k_new"] is not None:
        _write(t["pool"], t["tables"][session, lens // BLOCK].long() * BLOCK + lens % BLOCK, t["k_new"], t["v_new"])
        pos = lens
    else:
        pos = lens - 1
    t["out"].copy_(_attend(t, session, pos, t["q"][:, None])[:, 0])


def _plain_prefill(t):
    cu, ctx, q = t["cu"].long(), t["lens"].long(), t["q"]
    dev, s, rows = q.device, ctx.numel(), q.shape[0]
    if t["k_new"] is not None:
        i = torch.arange(rows, device=dev)
        who = torch.searchsorted(cu[1:], i, right=True)
        at = ctx[who] + i - cu[who]
        _write(t["pool"], t["tables"][who, at // BLOCK].long() * BLOCK + at % BLOCK, t["k_new"], t["v_new"])
    tiles = -(-t["max_new"] // TILE)
    session = torch.arange(s, device=dev).repeat_interleave(tiles)
    j0 = torch.arange(tiles, device=dev).repeat(s) * TILE
    j = j0[:, None] + torch.arange(TILE, device=dev)
    row = cu[session][:, None] + j
    past = j >= (cu[session + 1] - cu[session])[:, None]      # rows behind the turn's last are left out
    o = _attend(t, session, ctx[session] + j0, q[row.clamp(max=rows - 1)])
    whole = torch.empty((rows + 1,) + q.shape[1:], dtype=q.dtype, device=dev)
    whole[row.masked_fill(past, rows)] = o.to(q.dtype)
    t["out"].copy_(whole[:rows])


def _plain_tables(t):
    lens, n, tables, ring, counts = t["lens"].long(), t["new"].long(), t["tables"], t["ring"], t["counts"]
    s, width = tables.shape
    dev, size = tables.device, ring.numel()
    b0, b1 = (lens + BLOCK - 1) // BLOCK, (lens + n + BLOCK - 1) // BLOCK
    need = b1 - b0
    first = -(-t["sinks"] // BLOCK)
    w = t["window"]
    d0 = ((lens - w + 1) // BLOCK - first).clamp(min=0) if w else torch.zeros_like(lens)
    d1 = ((lens + n - w + 1) // BLOCK - first).clamp(min=0) if w else torch.zeros_like(lens)
    rel = d1 - d0
    base, rbase = need.cumsum(0) - need, rel.cumsum(0) - rel
    cu = torch.cat([torch.zeros(1, dtype=torch.int64, device=dev), n.cumsum(0)])
    j = torch.arange(width, device=dev)[None]
    # new blocks, then the ones behind the window (a block may be both, in a turn longer than the window)
    i = (j - b0[:, None])
    take = (i >= 0) & (j < b1[:, None])
    tables.copy_(torch.where(take, ring[(counts[0] + base[:, None] + i) % size], tables))
    i = j - first - d0[:, None]
    give = (i >= 0) & (i < rel[:, None])
    to = ((counts[1] + rbase[:, None] + i) % size).masked_fill(~give, size)
    wide = torch.cat([ring, ring[:1]])
    wide[to] = tables
    ring.copy_(wide[:size])
    p = torch.arange(t["slots"].numel(), device=dev)
    who = torch.searchsorted(cu[1:], p, right=True).clamp(max=s - 1)
    at = (lens[who] + p - cu[who]).clamp(max=width * BLOCK - 1)
    slot = tables[who, at // BLOCK].long() * BLOCK + at % BLOCK
    t["slots"].copy_(slot.masked_fill(p >= cu[-1], -1))
    t["cu"].copy_(cu)
    t["reused"].copy_(lens)
    t["next"].copy_(lens + n)
    t["next_counts"].copy_(counts + torch.stack([need.sum(), rel.sum()]))


def run(state):
    t = state
    op = t["op"]
    if own:
        from paper_2606_22983_amd import kv
        if op == "decode":
            kv.paged_attn_decode_window(t["handle"], 0, t["q"], t["tables"], t["lens"], t["window"], t["sinks"],
                                        t["scale"], t["out"], t["ws"], t["k_new"], t["v_new"],
                                        context_lens_host=t["lens_host"])
        elif op == "prefill":
            kv.paged_attn_prefill_window(t["handle"], 0, t["q"], t["cu"], t["lens"], t["max_new"], t["tables"],
                                         t["window"], t["sinks"], t["scale"], t["out"], t["k_new"], t["v_new"],
                                         lens_host=t["lens_host"], workspace=t["ws"])
        elif op == "tables":
            kv.kv_tables_update(t["handle"], t["lens"], t["new"], t["max_new"], t["tables"], t["next"], t["cu"],
                                t["reused"], t["slots"], free_ring=t["ring"], free_counts=t["counts"],
                                next_counts=t["next_counts"], window=t["window"], sinks=t["sinks"])
        else:
            kv.kv_append(t["handle"], 0, t["k_new"], t["v_new"], t["slots"])
    elif op == "decode":
        _plain_decode(t)
    elif op == "prefill":
        _plain_prefill(t)
    elif op == "tables":
        _plain_tables(t)
    else:
        _write(t["pool"], t["slots"], t["k_new"], t["v_new"])
    if op == "tables":
        return {k: t[k] for k in ("tables", "ring", "next_counts", "cu", "reused", "next", "slots")}
    if op == "append":
        return {"pool": t["pool"]}
    # an appending call also writes the new tokens' K and V into the pool
    return {"out": t["out"], "pool": t["pool"]} if t["k_new"] is not None else {"out": t["out"]}


def _visible(p, window, sinks):
    """Keys that a row at position p sees."""
    return np.minimum(p + 1, window) + np.minimum(sinks, np.maximum(p + 1 - window, 0))


def work(case):
    n, ctx = _lens(case)
    s, rows = len(n), int(n.sum())
    op = case["op"]
    if op == "tables":
        need = int((-(-(ctx + n) // BLOCK) - -(-ctx // BLOCK)).sum())
        w, k = case["window"], case["sinks"]
        rel = int((_dead(ctx + n, w, k) - _dead(ctx, w, k)).sum())
        # lengths read, the three length arrays written, open blocks' ids read, ids moved, slots written, counts
        return {"bytes": 8 * s + 12 * s + 4 + 4 * int((ctx % BLOCK > 0).sum()) + 8 * need + 8 * rel
                + 8 * (rows + case["pad"]) + 32, "flops": 0}
    hkv, d = case["hkv"], case["d"]
    if op == "append":
        return {"bytes": 2 * rows * 2 * hkv * d * 2 + 8 * (rows + case["pad"]), "flops": 0}
    w, k = case["window"], case["sinks"]
    if op == "decode":
        p = ctx + n - 1
        pairs = keys = int(_visible(p, w, k).sum())
        rows = s
        app = s if case["append"] else 0
    else:
        pos = np.concatenate([np.arange(a, a + m) for a, m in zip(ctx, n)])
        pairs = int(_visible(pos, w, k).sum())
        low = np.maximum(ctx - w + 1, 0)                      # keys that some row of the turn sees
        keys = int((ctx + n - low + np.minimum(k, low)).sum())
        app = rows if case["append"] else 0
    # K and V of every seen key read once, q read, out written, new rows written to the pool, block ids and lengths
    return {"bytes": keys * 2 * hkv * d * 2 + 2 * rows * case["hq"] * d * 2 + app * 2 * hkv * d * 2
            + keys // BLOCK * 4 + 8 * s, "flops": 4 * case["hq"] * d * pairs}


# ---------------------------------------------------------------------------------------------------
# The result in 64 bits


def _exact_append(pool, slots, k_new, v_new):
    """Element by element: dimension e of the token in slot b * 16 + o lies at [e / 8][o][e % 8] of K's tile, [e][o] of V's."""
    rows, hkv, d = k_new.shape
    flat, tile = pool.view(-1), BLOCK * d
    for i0 in range(0, rows, 4096):
        sl = slots[i0:i0 + 4096]
        at = (sl >= 0).nonzero()[:, 0]
        b, o = (sl[at] // BLOCK).view(-1, 1, 1), (sl[at] % BLOCK).view(-1, 1, 1)
        h = torch.arange(hkv, device="cuda").view(1, -1, 1)
        e = torch.arange(d, device="cuda").view(1, 1, -1)
        kt, vt = (b * 2 * hkv + h) * tile, (b * 2 * hkv + hkv + h) * tile
        flat[kt + (e // 8) * 128 + o * 8 + e % 8] = k_new[i0:i0 + 4096][at]
        flat[vt + e * BLOCK + o] = v_new[i0:i0 + 4096][at]


def _exact_tables(t):
    """Session by session and token by token, on the host."""
    lens, n = t["lens"].tolist(), t["new"].tolist()
    tables, ring = t["tables"].cpu().numpy().copy(), t["ring"].cpu().numpy().copy()
    taken, given = t["counts"].tolist()
    slots = np.full(t["slots"].numel(), -1, dtype=np.int64)
    cu, w, size = [0], t["window"], len(ring)
    first = 0
    while first * BLOCK < t["sinks"]:
        first += 1
    gone = []
    for s, (have, new) in enumerate(zip(lens, n)):
        for p in range(have, have + new):
            if p % BLOCK == 0:                               # the token opens a block
                tables[s, p // BLOCK] = ring[taken % size]
                taken += 1
            slots[cu[-1] + p - have] = int(tables[s, p // BLOCK]) * BLOCK + p % BLOCK
        cu.append(cu[-1] + new)
        if w:
            # Query p sees no key before p - w + 1: what the next query misses and this turn's first could not.
            for b in range(first, tables.shape[1]):
                last = b * BLOCK + BLOCK - 1
                if last < have + new - w + 1 and not last < have - w + 1:
                    gone.append(tables[s, b])
    for b in gone:
        ring[given % size] = b
        given += 1
    i32 = dict(dtype=torch.int32, device="cuda")
    return {"tables": torch.tensor(tables, **i32), "ring": torch.tensor(ring, **i32),
            "next_counts": torch.tensor([taken, given], device="cuda"), "cu": torch.tensor(cu, **i32),
            "reused": torch.tensor(lens, **i32), "next": torch.tensor([a + b for a, b in zip(lens, n)], **i32),
            "slots": torch.from_numpy(slots).cuda()}


def exact(case, seed):
    t = prepare(case, seed)
    if t["op"] == "tables":
        return _exact_tables(t)
    pool = t["pool"]
    if t["op"] == "append":
        _exact_append(pool, t["slots"], t["k_new"], t["v_new"])
        return {"pool": pool}
    n, ctx = _lens(case)
    hkv, grp, d, w, sinks = case["hkv"], case["hq"] // case["hkv"], case["d"], case["window"], case["sinks"]
    if t["op"] == "decode" and not case["append"]:
        ctx, n = ctx - 1, n + 1
    row = np.concatenate([[0], np.cumsum(n)])
    tables = t["tables"].long()
    out = torch.empty(t["q"].shape, dtype=torch.float64, device="cuda")
    for s in range(len(n)):
        lo, hi, c = int(row[s]), int(row[s + 1]), int(ctx[s])
        if case["append"]:
            p = torch.arange(c, c + hi - lo, device="cuda")
            _exact_append(pool, tables[s, p // BLOCK] * BLOCK + p % BLOCK, t["k_new"][lo:hi], t["v_new"][lo:hi])
        step = 256
        for r in range(lo, hi, step):
            e = min(hi, r + step)
            p = torch.arange(c + r - lo, c + e - lo, device="cuda")
            old = torch.arange(min(sinks, c + e - lo), device="cuda")
            end = c + e - lo
            near = torch.arange(min(end, max(sinks, c + r - lo - w + 1)), end, device="cuda")
            key = torch.cat([old, near[near >= sinks]])
            mask = (key[None] > p[:, None]) | ((key[None] >= sinks) & (key[None] <= p[:, None] - w))
            b, o = tables[s, key // BLOCK], key % BLOCK
            kk = pool[b, 0].view(-1, hkv, d // 8, BLOCK, 8)[torch.arange(len(key), device="cuda"), :, :, o].reshape(-1, hkv, d)
            vv = pool[b, 1].view(-1, hkv, d, BLOCK)[torch.arange(len(key), device="cuda"), :, :, o]
            for g in range(hkv):
                x = t["q"][r:e, g * grp:(g + 1) * grp].double().reshape(-1, d) @ kk[:, g].double().t().contiguous()
                x = (x * d ** -0.5).view(e - r, grp, -1).masked_fill(mask[:, None], -math.inf)
                out[r:e, g * grp:(g + 1) * grp] = torch.softmax(x, -1) @ vv[:, g].double()
    return {"out": out, "pool": pool} if case["append"] else {"out": out}
