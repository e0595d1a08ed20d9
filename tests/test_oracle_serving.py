"""Pins of the serving oracle (CPU): hand values, the window oracle of the measurement, invariants of the tables."""
import math

import numpy as np
import pytest

import oracle as O
from oracle import serving as S


def _vis(pos, qpos, window, n_sink):
    return [[int(x) for x in row] for row in S.sees(pos, qpos, window, n_sink)]


def test_visibility_by_hand():
    assert _vis([0, 1, 2, 3], [3], 0, 0) == [[1, 1, 1, 1]]
    assert _vis([0, 1, 2, 3], [3], 2, 0) == [[0, 0, 1, 1]]
    assert _vis([0, 1, 2, 3], [3], 2, 1) == [[1, 0, 1, 1]]
    assert _vis([0, 1, 2, 3], [1, 0], 1, 9) == [[1, 1, 0, 0], [1, 0, 0, 0]]
    assert _vis([0, 5, 9], [9], 5, 0) == [[0, 1, 1]]          # positions with gaps: 9 - 5 < 5
    assert _vis([0, 5, 9], [9], 4, 0) == [[0, 0, 1]]
    assert _vis([7], [6], 3, 99) == [[0]]                     # a sink of the future stays hidden
    big = 2**31 - 1
    assert _vis([0, big], [big], 5, 0) == [[0, 1]]


def test_two_tokens_by_hand():
    k = np.array([[[0.0, 0.0]], [[math.log(3.0), 0.0]]])
    v = np.array([[[1.0, 0.0]], [[0.0, 1.0]]])
    o, lse, _ = S.attend_rows(np.array([[[1.0, 0.0]]]), k, v, S.sees([0, 1], [1]), scale=1.0)
    assert np.allclose(o, [[[0.25, 0.75]]]) and np.allclose(lse, math.log(4.0))
    o, lse, _ = S.attend_rows(np.array([[[1.0, 0.0]]]), k, v, S.sees([0, 1], [1], window=1), scale=1.0)
    assert np.allclose(o, [[[0.0, 1.0]]]) and np.allclose(lse, math.log(3.0))
    o, lse, _ = S.attend_rows(np.array([[[1.0, 0.0]]]), k, v, S.sees([5, 6], [1]), scale=1.0)
    assert np.all(o == 0) and np.all(np.isneginf(lse))


def test_unbounded_window_is_the_measurement_oracle():
    rng = np.random.default_rng(0)
    n, R, Hq, Hkv, d = 50, 6, 4, 2, 8
    q, k, v = rng.standard_normal((R, Hq, d)), rng.standard_normal((n, Hkv, d)), rng.standard_normal((n, Hkv, d))
    pos, qpos = np.arange(n) * 2, np.array([3, 20, 41, 60, 97, 98])
    o, lse, _ = S.attend_rows(q, k, v, S.sees(pos, qpos))
    for h in range(Hq):
        s = O.head_logits(q[:, h], k[:, h // 2], 1 / math.sqrt(d))
        vis = O.visibility(pos, qpos)
        a, oo = O.attend(s, vis, v[:, h // 2])
        assert np.allclose(o[:, h], oo, rtol=1e-12, atol=1e-14)
        assert np.allclose(lse[:, h], np.log(np.where(vis, np.exp(s), 0).sum(1)), rtol=1e-12)


def test_hidden_tokens_do_not_count():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((1, 2, 4)), rng.standard_normal((9, 1, 4)), rng.standard_normal((9, 1, 4))
    vis = S.sees(np.arange(9), [8], window=3, n_sink=2)
    a = S.attend_rows(q, k, v, vis)
    k[2:6], v[2:6] = np.nan, np.inf
    b = S.attend_rows(q, k, v, vis)
    assert all(np.array_equal(x, y) for x, y in zip(a, b))


def test_shift_of_logits_moves_lse_only():
    rng = np.random.default_rng(2)
    q, k, v = rng.standard_normal((2, 2, 4)), rng.standard_normal((7, 1, 4)), rng.standard_normal((7, 1, 4))
    k[..., 0], q[..., 0] = 1.0, 0.0
    vis = S.sees(np.arange(7), [4, 6])
    o, lse, _ = S.attend_rows(q, k, v, vis, scale=1.0)
    q[..., 0] = 2.5
    o2, lse2, _ = S.attend_rows(q, k, v, vis, scale=1.0)
    assert np.allclose(o, o2) and np.allclose(lse + 2.5, lse2)


def _step(n_tokens, n_new, free, table, block, width=16, max_new=99, next_pos=None, n_blocks=10, n_free=None):
    free = np.array(free + [-1] * (n_blocks - len(free)))
    slot, pos = np.full((len(n_tokens), width), -1), np.full((len(n_tokens), width), -1)
    return S.build_slots(n_tokens, n_new, free, len([f for f in free if f >= 0]) if n_free is None else n_free,
                         np.array(table), slot, pos, next_pos, block, max_new, n_blocks)


def test_slots_by_hand():
    r = _step([3, 4], [2, 1], [5, 8, 2], [[1, -1], [0, -1]], 4)
    assert r["status"] == 0 and r["n_tokens"] == [5, 5] and r["cu_new"] == [0, 2, 3]
    assert r["table"].tolist() == [[1, 2], [0, 8]] and r["n_free"] == 1 and r["free"][0] == 5
    assert r["new_row"] == [7, 8, 32] and r["new_pos"] == [3, 4, 4]
    assert r["slot"][0].tolist()[:6] == [-1, -1, -1, 7, 8, -1] and r["pos"][1][4] == 4


def test_slots_of_an_ended_sequence_are_taken_first():
    r = _step([5, 0], [-1, 1], [9], [[3, 4], [-1, -1]], 4, next_pos=[0, 70])
    assert r["n_tokens"] == [0, 1] and r["table"].tolist() == [[3, 4], [4, -1]]
    assert r["n_free"] == 2 and r["free"][:2].tolist() == [9, 3] and r["new_pos"] == [70]


@pytest.mark.parametrize("kw,status", [
    (dict(n_tokens=[4], n_new=[1], free=[], table=[[1, -1]]), S.NO_BLOCKS),
    (dict(n_tokens=[8], n_new=[1], free=[5], table=[[1, 2]]), S.TABLE),
    (dict(n_tokens=[0], n_new=[3], free=[5], table=[[-1, -1]], max_new=2), S.MAX_NEW),
    (dict(n_tokens=[0], n_new=[-2], free=[5], table=[[-1, -1]]), S.BAD_COUNT),
    (dict(n_tokens=[-1], n_new=[1], free=[5], table=[[-1, -1]]), S.BAD_COUNT),
    (dict(n_tokens=[0], n_new=[1], free=[5], table=[[-1, -1]], n_free=11), S.BAD_COUNT),
])
def test_slots_refusals_change_nothing(kw, status):
    r = _step(block=4, **kw)
    assert r["status"] == status and r["n_tokens"] == kw["n_tokens"] and set(r["cu_new"]) == {0}
    assert r["table"].tolist() == kw["table"] and np.all(r["slot"] == -1) and r["new_row"] == []


def test_slots_keep_every_block_once():
    """Over a run of random steps no block is lost or held twice."""
    rng = np.random.default_rng(3)
    n, B, nb, width = 6, 4, 40, 40
    tok, table = [0] * n, np.full((n, 10), -1)
    slot, pos = np.full((n, width), -1), np.full((n, width), -1)
    free, nf = rng.permutation(nb), nb
    for _ in range(200):
        new = [int(rng.integers(-1, min(9, width - t + 1))) for t in tok]
        r = S.build_slots(tok, new, free, nf, table, slot, pos, None, B, 1000, nb)
        if r["status"]:
            assert r["status"] == S.NO_BLOCKS
            continue
        tok, table, slot, pos, free, nf = r["n_tokens"], r["table"], r["slot"], r["pos"], r["free"], r["n_free"]
        held = [int(b) for s in range(n) for b in table[s, :-(-tok[s] // B)]]
        assert sorted(held + free[:nf].tolist()) == list(range(nb))
        for s in range(n):
            assert [int(x) for x in slot[s, :tok[s]]] == [int(table[s, t // B]) * B + t % B for t in range(tok[s])]
