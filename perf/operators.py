"""Serving operators over a paged key/value pool, measured over their real ranges.

A serving step places its new tokens in the pool (``ckv_build_slots``), then
every layer attends: over a sliding window with a few first tokens that stay
visible (``ckv_attend_window``), or, where the sequences of a batch begin with
the same long prompt, over that prompt once for all and over each sequence's
own tokens (``ckv_attend_shared``).

A case is one pass through one of the three calls on seeded inputs held in GPU
memory.  Keys, values and queries are N(0, 1), one key in a hundred scaled by 4
(the heavy hitters of the repository's synthetic workloads).  Pools are larger
than what the sequences hold, and the sequences' rows lie scattered in them, as
after some time of serving.

Kinds: ``window``, ``shared`` and ``slots``.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
_CTX = []          # one context per process, as a serving worker holds it
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def _context():
    import paper_2608_07855_amd as P
    if not _CTX:
        _CTX.append(P.Context(0))
    return _CTX[0]


# ------------------------------------------------------------------- cases
#
# n: sequences; hq, hkv, d: heads and width; rows: query rows of a sequence
# (the most of them, where ragged); tokens: resident tokens of a sequence (the
# most of them); low: the fewest as a share of the most (1: all alike);
# gaps: absolute positions with gaps, as a compressed cache has them.

def _window(n, hq, hkv, d, rows, tokens, window, sinks, paged=True, gaps=False, low=1.0, type="bf16"):
    return dict(kind="window", n=n, hq=hq, hkv=hkv, d=d, rows=rows, tokens=tokens, window=window,
                sinks=sinks, paged=paged, gaps=gaps, low=low, type=type)


def _shared(n, hq, hkv, d, rows, prefix, tokens, low=0.25, type="bf16"):
    return dict(kind="shared", n=n, hq=hq, hkv=hkv, d=d, rows=rows, prefix=prefix, tokens=tokens, low=low, type=type)


def _slots(n, block, tokens, new, ends):
    return dict(kind="slots", n=n, block=block, tokens=tokens, new=new, ends=ends)


def listed():
    return [
        # one token of one sequence of a small model: nothing but latency
        dict(_window(1, 4, 1, 64, 1, 2048, 256, 4, paged=False), name="window_token_tiny"),
        # one token each of 16 compressed caches at the paper's operating point (gapped positions)
        dict(_window(16, 40, 8, 128, 1, 4224, 1024, 4, gaps=True, low=0.5), name="window_token_paper"),
        # one token each of 64 long ragged sequences
        dict(_window(64, 32, 8, 128, 1, 32768, 4096, 16, low=0.05), name="window_tokens_batch"),
        # one token of two 128K sequences, every token visible: the longest axis, the fewest rows
        dict(_window(2, 64, 8, 128, 1, 131072, 0, 0), name="window_token_128k"),
        # a whole prompt from the first token on
        dict(_window(1, 32, 8, 128, 8192, 8192, 1024, 4, paged=False), name="window_prompt"),
        # chunks of eight prompts behind their caches, ragged, in the other type
        dict(_window(8, 32, 8, 128, 509, 16512, 4096, 4, low=0.2, type="fp16"), name="window_chunks"),
        # eight short answers to one 2K prompt
        dict(_shared(8, 40, 8, 128, 1, 2048, 128), name="shared_token_small"),
        # 64 agents on one 32K system prompt, one token each
        dict(_shared(64, 32, 8, 128, 1, 32768, 2048), name="shared_tokens"),
        # the largest batch: 256 samples of one 64K prompt, 64 query heads
        dict(_shared(256, 64, 8, 128, 1, 65536, 512), name="shared_tokens_large"),
        # 16 sequences that each add a chunk (a tool's answer) behind one prompt
        dict(_shared(16, 32, 8, 128, 250, 16384, 1000, type="fp16"), name="shared_chunks"),
        # a decoding step: 64 sequences take one more token
        dict(_slots(64, 16, 4224, 1, 0.0), name="slots_step"),
        # a step that admits prompts, lets others go on and ends some
        dict(_slots(1024, 16, 4096, 2048, 0.1), name="slots_prompts"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["window", "window", "window", "shared", "shared", "slots"])
    if kind == "slots":
        n = _log_int(rng, 1, 1024)
        most = max(1, min(2048, (1 << 20) // n))
        return _slots(n, rng.choice([1, 16, 32, 64]), _log_int(rng, 64, 4096),
                      1 if rng.random() < 0.4 else _log_int(rng, 1, most), rng.choice([0.0, 0.1, 0.5]))
    hq, hkv, d = rng.choice([(4, 1, 64), (8, 8, 64), (32, 8, 128), (40, 8, 128), (64, 8, 128), (16, 1, 128)])
    type = rng.choice(["bf16", "bf16", "fp16"])
    low = rng.choice([0.05, 0.3, 1.0])
    if kind == "window":
        window = rng.choice([0, _log_int(rng, 1, 8192), _log_int(rng, 128, 8192)])
        sinks = rng.choice([0, 4, rng.randint(1, 64)])
        if rng.random() < 0.6:        # single tokens
            n = _log_int(rng, 1, 64)
            tokens = _log_int(rng, 1, min(131072, (1 << 20) // n))
            return _window(n, hq, hkv, d, rng.choice([1, 1, 1, 4]), tokens, window, sinks,
                           paged=rng.random() < 0.7, gaps=rng.random() < 0.3, low=low, type=type)
        n = _log_int(rng, 1, 8)
        rows = _log_int(rng, 2, 4096 // n)
        tokens = _log_int(rng, rows, max(rows, (1 << 27) // (n * hq * rows) // 8))
        return _window(n, hq, hkv, d, rows, tokens, window, sinks, paged=rng.random() < 0.7,
                       gaps=rng.random() < 0.3, low=low, type=type)
    if rng.random() < 0.7:
        n = _log_int(rng, 1, 256)
        prefix = _log_int(rng, 64, 65536)
        tokens = _log_int(rng, 1, min(2048, (1 << 17) // n))
        return _shared(n, hq, hkv, d, 1, prefix, tokens, low, type)
    n = _log_int(rng, 2, 16)
    rows = _log_int(rng, 2, 256)
    return _shared(n, hq, hkv, d, rows, _log_int(rng, 64, 16384), rows + _log_int(rng, 1, 1024), low, type)


# ------------------------------------------------------------------ inputs

def _counts(rng, n, low, most):
    """n counts from low * most to most, one of them the most."""
    c = rng.integers(max(1, round(low * most)), most + 1, n)
    c[rng.integers(n)] = most
    return c


def _shape(c):
    """Counts of a case, the same whatever the seed: resident tokens and query rows of every sequence (for the
    slots: resident and new tokens, -1 where the sequence ends)."""
    rng = np.random.default_rng([260807855, c["n"], c["tokens"]])
    if c["kind"] == "slots":
        n = c["n"]
        old = rng.integers(0, c["tokens"] + 1, n)
        new = rng.integers(0, c["new"] + 1, n) if c["new"] > 1 else np.ones(n, np.int64)
        ends = rng.random(n) < c["ends"]
        return old, np.where(ends, -1, new)
    rows = _counts(rng, c["n"], c["low"], c["rows"]) if c["rows"] > 1 else np.ones(c["n"], np.int64)
    tokens = np.maximum(_counts(rng, c["n"], c["low"], c["tokens"]), rows)
    return tokens, rows


def _i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(DEV)


def _normal(gen, shape, type):
    return torch.randn(shape, generator=gen, device=DEV, dtype=TYPES[type])


def prepare(case, seed):
    c = case
    tokens, rows = _shape(c)
    rng = np.random.default_rng([260807855, seed])
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    if c["kind"] == "slots":
        return _prepare_slots(c, rng, tokens, rows)
    n, hq, hkv, d, type = c["n"], c["hq"], c["hkv"], c["d"], c["type"]
    prefix = c.get("prefix", 0)
    s = dict(c=c, most=int(tokens.max()), n_rows=int(rows.sum()), most_rows=int(rows.max()))
    total = int(tokens.sum()) + prefix
    paged = c.get("paged", True)
    if paged:
        pool = total + total // 8 + 1
        s["k"], s["v"] = _normal(gen, (hkv, pool, d), type), _normal(gen, (hkv, pool, d), type)
        s["k"][:, torch.rand(pool, generator=gen, device=DEV) < 0.01] *= 4
        place = torch.randperm(pool, generator=gen, device=DEV).to(torch.int32)
        if prefix:
            s["prefix_slot"] = place[None, :prefix].contiguous()
            s["prefix_tokens"] = _i32([prefix])
        at = np.zeros((n, s["most"]), np.int64)
        first = prefix + np.cumsum(tokens) - tokens
        at[:] = first[:, None] + np.minimum(np.arange(s["most"])[None], tokens[:, None] - 1)
        s["slot"] = place[torch.from_numpy(at).to(DEV)].contiguous()
    else:
        s["k"], s["v"] = _normal(gen, (n, hkv, s["most"], d), type), _normal(gen, (n, hkv, s["most"], d), type)
        s["k"][:, :, torch.rand(s["most"], generator=gen, device=DEV) < 0.01] *= 4
        s["slot"] = None
    s["q"] = _normal(gen, (s["n_rows"], hq, d), type)
    s["n_tokens"], s["cu_rows"] = _i32(tokens), _i32(np.concatenate([[0], np.cumsum(rows)]))
    if c.get("gaps"):
        step = rng.integers(1, 4, (n, s["most"]))
        s["pos"] = _i32(np.cumsum(step, 1) - 1)
    else:
        s["pos"] = None
    s["o"] = torch.empty_like(s["q"])
    s["lse"] = torch.empty((s["n_rows"], hq), dtype=torch.float32, device=DEV)
    if own:
        import paper_2608_07855_amd as P
        s["ctx"] = _context()
        s["kv"] = P.batch_view(s["k"], s["v"], s["n_tokens"], slot=s["slot"], pos=s["pos"], max_tokens=s["most"])
        s["rows"] = P.query_view(s["q"], s["cu_rows"], max_rows=s["most_rows"])
        if prefix:
            s["prefix"] = P.batch_view(s["k"], s["v"], s["prefix_tokens"], slot=s["prefix_slot"], max_tokens=prefix)
    return s


def _prepare_slots(c, rng, old, new):
    n, B = c["n"], c["block"]
    width = int((old + np.maximum(new, 0)).max()) + 1
    blocks_old = -(-old // B)
    blocks_new = -(-(old + np.maximum(new, 0)) // B)
    n_blocks = int(blocks_new.sum() * 1.25) + 64
    perm = rng.permutation(n_blocks).astype(np.int32)
    cols = -(-width // B)
    table = np.full((n, cols), -1, np.int32)
    has = np.arange(cols)[None] < blocks_old[:, None]
    table[has] = perm[:has.sum()]
    free = np.full(n_blocks, -1, np.int32)
    n_free = n_blocks - int(has.sum())
    free[:n_free] = perm[has.sum():]
    t = np.arange(width)
    row = np.repeat(table, B, 1)[:, :width].astype(np.int64) * B + t[None] % B
    live = t[None] < old[:, None]
    shift = rng.integers(0, 1000, n)          # positions behind what earlier checkpoints dropped
    slot = np.where(live, row, -1)
    pos = np.where(live, t[None] + shift[:, None], -1)
    most = int(np.maximum(new, 0).sum())
    s = dict(c=c, n_blocks=n_blocks, n_tokens=_i32(old), n_new=_i32(new), next_pos=_i32(old + shift),
             free=_i32(free), n_free=_i32([n_free]), block_table=_i32(table), slot=_i32(slot), pos=_i32(pos),
             n_tokens_out=_i32(np.zeros(n)), n_free_out=_i32([0]), cu_new=_i32(np.zeros(n + 1)),
             new_row=_i32(np.full(max(1, most), -1)), new_pos=_i32(np.full(max(1, most), -1)), status=_i32([-1]))
    if own:
        import paper_2608_07855_amd as P
        s["ctx"] = _context()
        s["step"] = P.slot_step(s["n_tokens"], s["n_new"], s["free"], s["n_free"], s["slot"], block_size=B,
                                block_table=s["block_table"], pos=s["pos"], next_pos=s["next_pos"],
                                n_tokens_out=s["n_tokens_out"], n_free_out=s["n_free_out"], cu_new=s["cu_new"],
                                new_row=s["new_row"], new_pos=s["new_pos"], status=s["status"])
    return s


# --------------------------------------------------------------------- run

def run(s):
    c = s["c"]
    if own:
        import paper_2608_07855_amd as P
        if c["kind"] == "window":
            P.ckv_attend_window(s["ctx"], s["kv"], s["rows"], window=c["window"], n_sink=c["sinks"], o=s["o"], lse=s["lse"])
            return dict(o=s["o"], lse=s["lse"])
        if c["kind"] == "shared":
            P.ckv_attend_shared(s["ctx"], s["prefix"], s["kv"], s["rows"], o=s["o"], lse=s["lse"])
            return dict(o=s["o"], lse=s["lse"])
        P.ckv_build_slots(s["ctx"], s["step"])
        return _slot_outputs(s)
    if c["kind"] == "slots":
        return _plain_slots(s)
    return _plain_attend(s)


def _slot_outputs(s):
    names = ("n_tokens_out", "n_free_out", "cu_new", "new_row", "new_pos", "status", "free", "block_table", "slot", "pos")
    return {k: s[k] for k in names}


def _softmax_parts(q, k, v, seen):
    """q [b, rows, d], k, v [b, t, d], seen [b or 1, rows or 1, t]: largest score, sum and weighted values of each
    row over the tokens it sees, in 32 bits."""
    x = torch.matmul(q, k.transpose(1, 2).contiguous()) * (1.0 / math.sqrt(q.shape[2]))
    x.masked_fill_(~seen, -math.inf)
    m = x.amax(2, keepdim=True).clamp(min=-3e38)
    x.sub_(m).exp_()
    return m, x.sum(2, keepdim=True), torch.matmul(x, v)


def _plain_attend(s):
    """The rows of a batch padded to the longest sequence, all sequences and heads in batched products."""
    c, q = s["c"], s["q"]
    n, hq, hkv, d = c["n"], c["hq"], c["hkv"], c["d"]
    grp, T, R = hq // hkv, s["most"], s["most_rows"]
    cu, lens = s["cu_rows"].long(), s["n_tokens"].long()
    rows = cu[1:] - cu[:-1]
    j = torch.arange(R, device=DEV)
    live = j[None] < rows[:, None]                                    # [n, R]
    at = torch.where(live, cu[:-1, None] + j[None], 0)
    qp = q[at].float().view(n, R, hkv, grp, d).permute(0, 2, 1, 3, 4).reshape(n * hkv, R * grp, d)
    t = torch.arange(T, device=DEV)
    if s["slot"] is not None:
        slot = s["slot"].long()
        k, v = (x[:, slot].transpose(0, 1).float().reshape(n * hkv, T, d) for x in (s["k"], s["v"]))
    else:
        k, v = (x.float().view(n * hkv, T, d) for x in (s["k"], s["v"]))
    base = c.get("prefix", 0)
    pos = (t[None] + base).expand(n, T) if s["pos"] is None else s["pos"].long()
    mine = (lens[:, None] - rows[:, None] + j[None]).clamp(0, T - 1)
    qpos = pos.gather(1, mine)                                        # a row is its own last tokens'
    seen = (t[None, None] < lens[:, None, None]) & (pos[:, None] <= qpos[:, :, None])
    if c.get("window", 0) > 0:
        seen &= (qpos[:, :, None] - pos[:, None] < c["window"]) | (pos[:, None] < c["sinks"])
    seen = seen[:, None, :, None].expand(n, hkv, R, grp, T).reshape(n * hkv, R * grp, T)
    m, l, u = _softmax_parts(qp, k, v, seen)
    del k, v, seen
    if base:
        # every row sees all of the prefix: one product for the rows of all sequences
        ps = s["prefix_slot"][0].long()
        allq = q.float().view(-1, hkv, grp, d).permute(1, 0, 2, 3).reshape(hkv, -1, d)
        everything = torch.ones((1, 1, 1), dtype=torch.bool, device=DEV)
        mp, lp, up = _softmax_parts(allq, s["k"][:, ps].float(), s["v"][:, ps].float(), everything)

        def padded(x):
            x = x.view(hkv, -1, grp, x.shape[2])[:, at]               # [hkv, n, R, grp, .]
            return x.transpose(0, 1).reshape(n * hkv, R * grp, -1)
        mp, lp, up = padded(mp), padded(lp), padded(up)
        top = torch.maximum(m, mp)
        a, b = (m - top).exp(), (mp - top).exp()
        m, l, u = top, l * a + lp * b, u * a + up * b
    out = (u / l).view(n, hkv, R, grp, d).permute(0, 2, 1, 3, 4).reshape(n, R, hq, d)
    lse = (m + l.log()).view(n, hkv, R, grp).permute(0, 2, 1, 3).reshape(n, R, hq)
    return dict(o=out[live].to(q.dtype), lse=lse[live])


def _plain_slots(s):
    """Blocks of the sequences that end go on top of the free stack in the order of sequences; the new blocks of the
    others come off its top in the order of sequences."""
    B = s["c"]["block"]
    old, new, free, n_free = s["n_tokens"].long(), s["n_new"].long(), s["free"], s["n_free"].long()
    table, width = s["block_table"], s["slot"].shape[1]
    ends, grow = new < 0, new.clamp(min=0)
    have = (old + B - 1) // B
    want = torch.where(ends, have, (old + grow + B - 1) // B)
    # released blocks join the stack
    cols = torch.arange(table.shape[1], device=DEV)
    back = table[ends[:, None] & (cols[None] < have[:, None])]
    stack = torch.cat([free[:n_free], back])
    fresh = (cols[None] >= have[:, None]) & (cols[None] < want[:, None])
    seq, col = fresh.nonzero(as_tuple=True)
    take = stack.shape[0] - 1 - torch.arange(seq.shape[0], device=DEV)
    table[seq, col] = stack[take]
    left = stack.shape[0] - seq.shape[0]
    free[:left] = stack[:left]
    # new tokens
    t = torch.arange(width, device=DEV)
    fresh = (t[None] >= old[:, None]) & (t[None] < (old + grow)[:, None])
    seq, tok = fresh.nonzero(as_tuple=True)
    row = table[seq, tok // B] * B + (tok % B).to(torch.int32)
    at = s["next_pos"][seq] + (tok - old[seq]).to(torch.int32)
    s["slot"][seq, tok], s["pos"][seq, tok] = row, at
    s["new_row"][:row.shape[0]], s["new_pos"][:row.shape[0]] = row, at
    s["cu_new"][1:] = grow.cumsum(0)
    s["n_tokens_out"][:] = torch.where(ends, 0, old + grow)
    s["n_free_out"][:] = left
    s["status"][:] = 0
    return _slot_outputs(s)


# -------------------------------------------------------------------- work

def work(case):
    c = case
    tokens, rows = _shape(c)
    if c["kind"] == "slots":
        B, grow = c["block"], np.maximum(rows, 0)
        have = -(-tokens // B)
        back, take = have[rows < 0].sum(), (-(-(tokens + grow) // B) - have)[rows >= 0].sum()
        # counts in and out, a word in and one out for each block, four words for each new token
        return {"bytes": float(4 * (5 * c["n"] + 4) + 8 * int(back + take) + 16 * int(grow.sum())), "flops": 0.0}
    per_token = c["hkv"] * c["d"] * 4 + 4 * bool(c.get("paged", True)) + 4 * bool(c.get("gaps"))
    out = float(rows.sum()) * c["hq"] * (c["d"] * 4 + 4)
    base = c.get("prefix", 0)
    seen, touched = 0.0, 0.0
    for t, r in zip(tokens, rows):
        p = t - r + np.arange(r) + 1.0                 # tokens up to each row's own
        if c.get("window", 0) > 0:
            # positions with gaps of 1 to 3 hold half as many tokens in the same window
            w = c["window"] / (2.0 if c.get("gaps") else 1.0)
            p_seen = np.minimum(p, w + c["sinks"])
            touched += min(t, w + r - 1 + c["sinks"])
        else:
            p_seen = p
            touched += t
        seen += (p_seen + base).sum()
    return {"bytes": float((touched + base) * per_token + out), "flops": float(4.0 * seen * c["hq"] * c["d"])}


# ------------------------------------------------------------------- exact

def exact(case, seed):
    """By the definition, in 64 bits: for each sequence and head the softmax over the tokens that each row sees."""
    c = case
    if c["kind"] == "slots":
        return None                                    # whole numbers: nothing is rounded
    s = prepare(c, seed)
    tokens, rows = _shape(c)
    hq, hkv, d, base = c["hq"], c["hkv"], c["d"], c.get("prefix", 0)
    grp, f8 = hq // hkv, torch.float64
    o = torch.empty((s["n_rows"], hq, d), dtype=f8, device=DEV)
    lse = torch.empty((s["n_rows"], hq), dtype=f8, device=DEV)
    first = 0
    for i, (t, r) in enumerate(zip(tokens.tolist(), rows.tolist())):
        p = torch.arange(base, base + t, device=DEV) if s["pos"] is None else s["pos"][i, :t].long()
        mine = p[t - r:]
        hide = p[None] > mine[:, None]
        if c.get("window", 0) > 0:
            hide |= (p[None] <= mine[:, None] - c["window"]) & (p[None] >= c["sinks"])
        if base:
            hide = torch.cat([torch.zeros((r, base), dtype=torch.bool, device=DEV), hide], 1)
        keep = ~hide.all(0)                            # tokens that some row sees
        hide = hide[:, keep]
        for g in range(hkv):
            if s["slot"] is None:
                k, v = s["k"][i, g, :t], s["v"][i, g, :t]
            else:
                own_rows = s["slot"][i, :t]
                if base:
                    own_rows = torch.cat([s["prefix_slot"][0], own_rows])
                k, v = s["k"][g, own_rows.long()], s["v"][g, own_rows.long()]
            k, v = k[keep].to(f8), v[keep].to(f8)
            for h in range(g * grp, (g + 1) * grp):
                x = (s["q"][first:first + r, h].to(f8) @ k.T) / math.sqrt(d)
                x.masked_fill_(hide, -math.inf)
                e = torch.logsumexp(x, 1)
                lse[first:first + r, h] = e
                o[first:first + r, h] = (x - e[:, None]).exp_() @ v
        first += r
    return dict(o=o, lse=lse)
