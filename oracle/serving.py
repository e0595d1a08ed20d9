"""fp64 oracle of the serving calls (test infrastructure only): attention of a
ragged batch with a sliding window and visible first tokens, attention behind a
shared prefix, and the block and slot tables of a step.

Plain NumPy, written from the definitions; it shares nothing with the HIP path.
"""
from __future__ import annotations

import math

import numpy as np


def sees(pos, qpos, window=0, n_sink=0):
    """vis[p, i]: p_i <= p, and p - p_i < window (0: no window) or p_i < n_sink."""
    pos, qpos = np.asarray(pos, np.int64)[None, :], np.asarray(qpos, np.int64)[:, None]
    vis = pos <= qpos
    if window:
        vis &= (qpos - pos < window) | (pos < n_sink)
    return vis


def attend_rows(q, k, v, vis, scale=None):
    """One sequence.  q [R, Hq, d], k, v [n, Hkv, d] (real arrays), vis [R, n].
    Returns o [R, Hq, d], lse [R, Hq] and w [R, Hq, d] = sum_i a_i |v_i|, the scale that the
    rounding of the weights a_i reaches o with.  Only tokens that a row sees enter its sums; a row that
    sees none has o = 0, lse = -inf."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    R, Hq, d = q.shape
    grp = Hq // k.shape[1]
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    o, w = np.zeros((R, Hq, d)), np.zeros((R, Hq, d))
    lse = np.full((R, Hq), -np.inf)
    for r in range(R):
        t = np.flatnonzero(vis[r])
        if t.size == 0:
            continue
        for h in range(Hq):
            x = scale * (k[t, h // grp] @ q[r, h])
            m = x.max()
            if m == -np.inf:
                continue
            e = np.exp(x - m)
            lse[r, h] = m + math.log(e.sum())
            a = e / e.sum()
            o[r, h] = a @ v[t, h // grp]
            w[r, h] = a @ np.abs(v[t, h // grp])
    return o, lse, w


SLOTS_OK, NO_BLOCKS, TABLE, MAX_NEW, BAD_COUNT = range(5)


def build_slots(n_tokens, n_new, free, n_free, table, slot, pos, next_pos, block_size, max_new, n_blocks):
    """One step, one sequence and one block after the other.  Arrays are copied; returns a dict of all
    tables and outputs after the step (new_row and new_pos as lists)."""
    n_tokens, n_new = [int(x) for x in n_tokens], [int(x) for x in n_new]
    free, table, slot = np.array(free), None if table is None else np.array(table), np.array(slot)
    pos = None if pos is None else np.array(pos)
    n, B = len(n_tokens), block_size
    blocks = slot if table is None else table

    def count(t):
        return -(-t // B)
    status = SLOTS_OK
    bad = [t < 0 or m < -1 for t, m in zip(n_tokens, n_new)]
    good = [(t, m) for t, m, x in zip(n_tokens, n_new, bad) if not x]
    back = sum(count(t) for t, m in good if m < 0)
    need = sum(count(t + m) - count(t) for t, m in good if m >= 0)
    if need > n_free + back:
        status = NO_BLOCKS
    if any(t + max(m, 0) > slot.shape[1] or count(t + max(m, 0)) > blocks.shape[1] for t, m in good):
        status = TABLE
    if sum(max(m, 0) for _, m in good) > max_new:
        status = MAX_NEW
    if any(bad) or not 0 <= n_free <= n_blocks or n_free + back > n_blocks:
        status = BAD_COUNT
    res = dict(free=free, table=table, slot=slot, pos=pos, status=status, new_row=[], new_pos=[])
    if status:
        res.update(n_tokens=n_tokens, n_free=n_free, cu_new=[0] * (n + 1))
        return res
    stack = [int(b) for b in free[:n_free]]
    for s in range(n):
        if n_new[s] < 0:
            stack += [int(blocks[s, i]) for i in range(count(n_tokens[s]))]
    out_tokens, cu = [], [0]
    for s in range(n):
        old, m = n_tokens[s], n_new[s]
        for i in range(count(old), count(old + m) if m >= 0 else count(old)):
            blocks[s, i] = stack.pop()
        for j in range(max(m, 0)):
            t = old + j
            row = min(max(int(blocks[s, t // B]), 0), n_blocks - 1) * B + t % B if blocks[s, t // B] >= 0 else \
                (n_blocks - 1) * B + t % B
            p = (old if next_pos is None else int(next_pos[s])) + j
            slot[s, t] = row
            if pos is not None:
                pos[s, t] = p
            res["new_row"].append(row)
            res["new_pos"].append(p)
        out_tokens.append(0 if m < 0 else old + m)
        cu.append(cu[-1] + max(m, 0))
    free[:len(stack)] = stack
    res.update(n_tokens=out_tokens, n_free=len(stack), cu_new=cu)
    return res
