"""Attention over caches in 4 bits (ckv_attend_packed) against the fp64 oracle.

Storage that no token owns holds NaN scales, and rows of no sequence a fill that must stay."""
import numpy as np
import pytest
import torch

from oracle import packed as O
from tests.packed_util import PackedBatch, check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ckv():
    import paper_2608_07855_amd as P
    ctx = P.Context(0)
    yield P, ctx
    ctx.close()


def _run(ckv, b, window=0, n_sink=0, max_rows=None, what=""):
    P, ctx = ckv
    got = b.run(P, ctx, b.device(P, max_rows=max_rows), window, n_sink)
    check(b, got, b.want(window, n_sink), what)
    return got


HEADS = [(4, 1, 64), (8, 8, 64), (8, 2, 128), (40, 8, 128), (16, 1, 128), (34, 2, 64)]


@pytest.mark.parametrize("type", ["bf16", "fp16"])
@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("paged", [False, True])
def test_single_tokens(ckv, hq, hkv, d, paged, type):
    """One row each behind caches of 1 to 400 tokens, tile edges among them."""
    lens = [1, 2, 15, 16, 17, 31, 32, 33, 63, 65, 97, 129, 400]
    b = PackedBatch(1, lens, [1] * len(lens), hq, hkv, d, type, paged)
    _run(ckv, b, what="all")
    _run(ckv, b, 1, what="own token")
    _run(ckv, b, 37, 5, what="window and sinks")


@pytest.mark.parametrize("type", ["bf16", "fp16"])
@pytest.mark.parametrize("hq,hkv,d", HEADS)
def test_prompts(ckv, hq, hkv, d, type):
    """Whole prompts and chunks behind caches, ragged."""
    b = PackedBatch(2, [1, 77, 130, 300, 64], [1, 77, 65, 33, 64], hq, hkv, d, type, lead=3, tail=2)
    _run(ckv, b, what="all")
    _run(ckv, b, 64, what="window 64")
    _run(ckv, b, 50, 7, what="window and sinks")


@pytest.mark.parametrize("rows", [2, 3, 4, 8, 17])
def test_few_rows(ckv, rows):
    """Drafted tokens: a few rows per sequence."""
    b = PackedBatch(3, [rows, 100, 333], [rows] * 3, 8, 2, 128)
    _run(ckv, b, what="all")
    _run(ckv, b, 40, 4, what="window")


@pytest.mark.parametrize("window,n_sink", [(0, 0), (0, 9), (1, 0), (1, 1), (2, 300), (63, 0), (64, 64), (65, 1), (299, 1),
                                           (300, 0), (2**31 - 1, 2**31 - 1)])
def test_window_edges(ckv, window, n_sink):
    b = PackedBatch(4, [300, 64, 5], [70, 1, 5], 4, 2, 64)
    _run(ckv, b, window, n_sink, what=f"window {window}, sinks {n_sink}")


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("rows", [1, 40])
@pytest.mark.parametrize("window,n_sink", [(0, 0), (50, 0), (50, 11), (1, 0)])
def test_gapped_positions(ckv, paged, rows, window, n_sink):
    """Compressed caches: absolute positions with gaps."""
    b = PackedBatch(5, [200, 1, 90, 513], [min(rows, t) for t in (200, 1, 90, 513)], 8, 2, 128, paged=paged, gaps=True)
    _run(ckv, b, window, n_sink, what="gaps")


@pytest.mark.parametrize("seed", range(40))
def test_any_batch(ckv, seed):
    """Batches drawn over everything a view may hold."""
    rng = np.random.default_rng(seed)
    n = int(rng.choice([1, 2, 5, 70]))
    long = int(rng.choice([40, 300, 1500])) if n < 70 else 30
    lens = rng.integers(0, long + 1, n)
    few = rng.random() < 0.5
    rows = rng.integers(0, 3 if few else 90, n) if n < 70 else rng.integers(0, 4, n)
    hq, hkv, d = [(4, 1, 64), (6, 6, 64), (8, 2, 128), (20, 4, 64), (17, 1, 128)][int(rng.integers(5))]
    gaps, given = rng.random() < 0.5, rng.random() < 0.3
    qpos = None
    if given:
        qpos = [rng.integers(-3, 3 * long + 3, r) for r in rows]
    elif not gaps:
        lens = np.maximum(lens, rows) if rng.random() < 0.7 else lens
    b = PackedBatch(1000 + seed, lens, rows, hq, hkv, d, "fp16" if rng.random() < 0.5 else "bf16", rng.random() < 0.6, gaps, qpos,
                    lead=int(rng.integers(3)), tail=int(rng.integers(3)))
    window = int(rng.choice([0, 1, 30, 64, 500, 1 << 30]))
    n_sink = int(rng.choice([0, 1, 40, 1 << 30]))
    _run(ckv, b, window, n_sink, max_rows=int(rng.choice([1, max(1, int(rows.max(initial=1))), 500])), what=f"seed {seed}")


@pytest.mark.parametrize("window", [0, 8])
def test_given_positions(ckv, window):
    """Rows at positions of their own, out of order and far apart, some before every token, one at the far end."""
    far = 2**31 - 1
    qpos = [[-5, 150, 0, 149, 30, far, 75, 75], [-1], [63, 2, far - 1]]
    for gaps in (False, True):
        b = PackedBatch(6, [150, 40, 64], [8, 1, 3], 4, 2, 64, qpos=qpos, gaps=gaps)
        _run(ckv, b, window, 2 if window else 0, what="positions")


def test_empty_sequences(ckv):
    """No tokens, no rows, neither; rows whose tokens are not in the cache."""
    b = PackedBatch(7, [0, 5, 0, 20, 3], [1, 0, 0, 2, 5], 4, 2, 64, lead=1)
    o, lse = _run(ckv, b, what="empty")
    assert np.all(o[0] == 0) and np.all(np.isneginf(lse[0]))
    _run(ckv, b, 4, 1, what="empty, window")
    b = PackedBatch(8, [0], [3], 4, 2, 64, tables=1)
    _run(ckv, b, what="nothing at all")


def test_empty_views(ckv):
    """No sequences; sequences without room for tokens."""
    P, ctx = ckv
    i = torch.zeros(4, dtype=torch.int32, device="cuda")
    pool = torch.zeros((2, 5, 80), dtype=torch.uint8, device="cuda")
    q = torch.ones((2, 4, 64), dtype=torch.bfloat16, device="cuda")
    o = torch.full((2, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    P.ckv_attend_packed(ctx, P.packed_view(pool, i[:0], slot=i[:0].view(0, 1)), P.query_view(q, i[:1]), o=o)
    ctx.sync()
    assert torch.all(o == 7)
    kv = P.packed_view(pool, i[:1] + 3, slot=torch.zeros((1, 0), dtype=torch.int32, device="cuda"))
    P.ckv_attend_packed(ctx, kv, P.query_view(q, torch.tensor([0, 2], dtype=torch.int32, device="cuda")), o=o)
    ctx.sync()
    assert torch.all(o == 0)


def test_many_sequences(ckv):
    """More sequences than a workgroup has threads, most of them tiny."""
    rng = np.random.default_rng(9)
    lens = rng.integers(0, 6, 1300)
    b = PackedBatch(9, lens, (rng.random(1300) < 0.7).astype(int), 2, 1, 64)
    _run(ckv, b, what="many")
    b = PackedBatch(9, lens, rng.integers(0, 4, 1300), 2, 1, 64)
    _run(ckv, b, 5, 2, what="many, few rows")


@pytest.mark.parametrize("rows", [1, 5, 60])
def test_long_axis(ckv, rows):
    """A long cache split over the device, ragged."""
    b = PackedBatch(10, [6001, 70, 2500], [rows, rows, rows], 4, 1, 128)
    _run(ckv, b, what="long")
    _run(ckv, b, 2000, 3, what="long, window")


@pytest.mark.parametrize("guess", [1, 2, 1000])
def test_any_estimate_of_rows(ckv, guess):
    """max_rows is an estimate: results hold whatever it says."""
    b = PackedBatch(11, [150, 64, 33, 7], [130, 1, 33, 2], 4, 2, 64)
    _run(ckv, b, max_rows=guess, what=f"estimate {guess}")
    _run(ckv, b, 20, 3, max_rows=guess, what=f"estimate {guess}, window")


@pytest.mark.parametrize("scale", [1.0, 0.02])
def test_scale(ckv, scale):
    b = PackedBatch(12, [200, 90], [1, 33], 4, 2, 64, scale=scale)
    _run(ckv, b, what=f"scale {scale}")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows", [1, 40])
def test_queries_of_any_size(ckv, d, rows):
    """bf16 queries far above and below what fp16 holds, each row with a scale of its own (the logits as they were)."""
    b = PackedBatch(13, [150, 60], [rows, 1], 4, 2, d, heavy=False)
    want = b.want()
    sizes = 2.0**np.random.default_rng(1).integers(-60, 61, (rows + 1, 4))
    for size in (2.0**60, 2.0**-60, 2.0**100):
        c = PackedBatch(13, [150, 60], [rows, 1], 4, 2, d, heavy=False, scale=1.0 / size / d**0.5)
        c.q = [x * size for x in b.q]
        _check = c.run(*ckv, c.device(ckv[0]))
        check(b, _check, want, f"size {size:.0e}")
    # rows of different sizes: what is tiny weights all tokens alike, what is huge picks one
    at, q = 0, []
    for x in b.q:
        q.append(x * torch.from_numpy(sizes[at:at + x.shape[0]])[..., None].to(x.dtype))
        at += x.shape[0]
    small = [(x.abs().amax(-1) < 2**-20).numpy() for x in q]
    b.q = q
    o, _ = b.run(*ckv, b.device(ckv[0]))
    wo, _, w = b.want()
    pick = np.concatenate(small)
    assert np.all(np.abs(o - wo)[pick] <= 2.0**-8 * np.abs(wo)[pick] + 2.0**-10 * w[pick] + 1e-6)


def test_zero_queries(ckv):
    b = PackedBatch(14, [70, 33], [1, 20], 4, 2, 128)
    b.q = [torch.zeros_like(x) for x in b.q]
    _run(ckv, b, what="zeros")


@pytest.mark.parametrize("value_scale", [1e-4, 1000.0])
def test_values_of_any_size(ckv, value_scale):
    b = PackedBatch(15, [200, 90], [1, 33], 4, 2, 128, value_scale=value_scale)
    _run(ckv, b, what=f"values {value_scale}")


@pytest.mark.parametrize("type", ["bf16", "fp16"])
def test_many_small_weights(ckv, type):
    """A dominant token and thousands of small weights that make up the output together."""
    b = PackedBatch(16, [3000, 3000], [1, 20], 4, 2, 64, type, heavy=False)
    for s in range(2):
        q = b.q[s][0].float().mean(0)
        k, v = np.zeros((1, 2, 64), np.float32), np.zeros((1, 2, 64), np.float32)
        k[0, :] = (q * (90.0 / float(q @ q))).numpy() / 2        # a logit some units above the rest
        b.set_rows(s, slice(5, 6), O.pack(k, v))
    _run(ckv, b, what="dominant")


def test_strides(ckv):
    """Token-major pools, padded rows, tables wider than used, queries inside a wider tensor."""
    P, ctx = ckv
    b = PackedBatch(17, [90, 130, 17], [1, 20, 17], 8, 2, 64)
    want = b.want(33, 4)
    v = b.device(P)
    pool, lens, slot, _ = v["kv"]._keep
    big = torch.full((pool.shape[1], 3, 2, 96), 0xFF, dtype=torch.uint8, device="cuda")
    big[:, 1, :, :80] = pool.transpose(0, 1)
    wide = torch.full((3, slot.shape[1] + 30), 1 << 30, dtype=torch.int32, device="cuda")
    wide[:, :slot.shape[1]] = slot
    qq, cu, _ = v["q"]._keep
    qw = torch.full((qq.shape[0], 5, 8, 80), float("nan"), dtype=qq.dtype, device="cuda")
    qw[:, 2, :, 8:72] = qq
    kv2 = P.packed_view(big[:, 1, :, :80].transpose(0, 1), lens, slot=wide[:, :slot.shape[1]])
    check(b, b.run(P, ctx, dict(kv=kv2, q=P.query_view(qw[:, 2, :, 8:72], cu, max_rows=20)), 33, 4), want, "strides")


def test_clamped_slots_and_counts(ckv):
    """Rows outside the pool read its last row; lengths past max_tokens count as that, negative ones as 0."""
    P, ctx = ckv
    b = PackedBatch(18, [40, 70], [1, 3], 4, 2, 64)
    v = b.device(P, fill=0)
    pool, lens, slot, _ = v["kv"]._keep
    s2, last = slot.clone(), pool.shape[1] - 1
    s2[0, 3], s2[0, 17], s2[1, 60] = -1, 1 << 30, last + 1
    got = b.run(P, ctx, dict(kv=P.packed_view(pool, lens, slot=s2), q=v["q"]))
    s3 = s2.clone()
    s3[(s2 < 0) | (s2 > last)] = last
    same = b.run(P, ctx, dict(kv=P.packed_view(pool, lens, slot=s3), q=v["q"]))
    assert all(np.array_equal(x, y) for x, y in zip(got, same))
    far = b.run(P, ctx, dict(kv=P.packed_view(pool, torch.tensor([40, 1 << 30], dtype=torch.int32, device="cuda"), slot=slot), q=v["q"]))
    assert all(np.array_equal(x, y) for x, y in zip(far, b.run(P, ctx, v)))
    o, lse = b.run(P, ctx, dict(kv=P.packed_view(pool, torch.tensor([-5, 70], dtype=torch.int32, device="cuda"), slot=slot), q=v["q"]))
    assert np.all(o[0] == 0) and np.all(np.isneginf(lse[0]))


@pytest.mark.parametrize("rows", [1, 7, 40])
@pytest.mark.parametrize("d", [64, 128])
def test_hidden_tokens_hold_anything(ckv, rows, d):
    """Any bytes in tokens that a row does not see stay out of that row."""
    P, ctx = ckv
    n = 200
    junk = np.random.default_rng(0).integers(0, 256, (n, 2, O.row_bytes(d)), dtype=np.uint8)
    junk[::2, :, d:] = 0xFF                                      # NaN scales and bases
    junk[1::2, :, d:] = [0xFF, 0x7B] * (d // 8)                  # the largest ones
    for case in ("before the window", "behind every row", "seen by later rows only"):
        b = PackedBatch(19, [n, 60], [rows, 1], 4, 2, d, qpos=[n - 61 + np.arange(rows), [59]])
        want = b.want(32, 3)
        clean = rows
        if case == "before the window":
            bad = slice(10, 100)
        elif case == "behind every row":
            bad = slice(n - 61 + rows, n)
        else:
            bad, clean = slice(n - 61 + rows - 1, n), rows - 1
        b.bytes[0][bad] = junk[:b.bytes[0][bad].shape[0]]
        v = b.device(P)
        if case == "seen by later rows only":
            o = torch.zeros((rows + 1, 4, d), dtype=torch.bfloat16, device="cuda")
            lse = torch.zeros((rows + 1, 4), dtype=torch.float32, device="cuda")
            P.ckv_attend_packed(ctx, v["kv"], v["q"], window=32, n_sink=3, o=o, lse=lse)
            with pytest.raises(P.CKVError, match="NONFINITE"):
                ctx.sync()
            got = o.cpu().double().numpy(), lse.cpu().double().numpy()
            pick = list(range(clean)) + [rows]
            assert not np.isfinite(got[0][clean:rows]).all()
        else:
            got, pick = b.run(P, ctx, v, 32, 3), list(range(rows + 1))
        check(b, tuple(x[pick] for x in got), tuple(x[pick] for x in want), case)


def test_large_logits(ckv):
    """Rows with one dominant token, logits of several hundred, past 2^24, and all alike."""
    b = PackedBatch(20, [300, 300], [1, 64], 4, 2, 64, heavy=False)
    for s in range(2):
        for t, by in ((7, 16), (150, -16)):
            k = b.k[s][t:t + 1].float().numpy() * by
            b.set_rows(s, slice(t, t + 1), O.pack(k, b.v[s][t:t + 1].float().numpy()))
    _run(ckv, b, what="dominant")
    zero = O.pack(np.zeros((300, 2, 64), np.float32), np.random.default_rng(0).standard_normal((300, 2, 64)).astype(np.float32))
    for s in range(2):
        b.set_rows(s, slice(0, 300), zero)
    _run(ckv, b, what="alike")
    # equal keys of 16384 and a scale of 2^10: logits of 2^30 and more, all alike, weights must be alike
    k = np.full((300, 2, 64), 16384.0, np.float32)
    c = PackedBatch(21, [300, 300], [1, 64], 4, 2, 64, heavy=False, scale=1024.0)
    for s in range(2):
        c.q[s] = torch.ones_like(c.q[s])
        c.set_rows(s, slice(0, 300), O.pack(k, c.v[s].float().numpy()))
    o, lse = c.run(*ckv, c.device(ckv[0]))
    wo, wl, w = c.want()
    assert np.all(np.abs(o - wo) <= 2.0**-8 * np.abs(wo) + 2.0**-10 * w + 1e-6) and np.all(np.abs(lse - wl) <= 2.0**-22 * wl)


def test_equals_the_16_bit_call_on_what_the_rows_stand_for(ckv):
    """Read back to fp16 and attended to by ckv_attend_window: the same numbers."""
    P, ctx = ckv
    b = PackedBatch(22, [700, 90, 333], [1, 50, 3], 8, 2, 128, "fp16", gaps=True)
    v = b.device(P)
    _, lens, _, pos = v["kv"]._keep
    wide = P.ckv_unpack_tokens(ctx, v["kv"], dtype=torch.float16)
    got = P.ckv_attend_window(ctx, P.batch_view(wide["k"], wide["v"], lens, pos=pos), v["q"], window=300, n_sink=2, want=("o", "lse"))
    ctx.sync()
    want = b.want(300, 2)
    check(b, (got["o"].cpu().double().numpy(), got["lse"].cpu().double().numpy()), want, "16 bits")
    check(b, b.run(P, ctx, v, 300, 2), want, "4 bits")


# ------------------------------------------------------- streams, capture, memory

def _graph_case(P, b, window):
    v = b.device(P)
    total = int(b.rows.sum())
    o = torch.zeros((total, b.hq, b.d), dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros((total, b.hq), dtype=torch.float32, device="cuda")

    def call(ctx):
        P.ckv_attend_packed(ctx, v["kv"], v["q"], window=window, n_sink=2 if window else 0, o=o, lse=lse)
    return v, o, lse, call


@pytest.mark.parametrize("rows", [1, 70])
def test_captured_step_serves_grown_caches(ckv, rows):
    """A captured call replays with the lengths of the moment; larger eager calls in between do not move its memory."""
    P, _ = ckv
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = P.Context(0, stream)
        b = PackedBatch(40, [4000, 900, rows], [rows] * 3, 8, 2, 128, tables=4100)
        v, o, lse, call = _graph_case(P, b, 3500)
        call(ctx)
        stream.synchronize()
        eager = o.clone(), lse.clone()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            call(ctx)
        big = PackedBatch(41, [400] * 20, [30] * 20, 8, 2, 128)
        vb = big.device(P)
        for n in (4000, rows + 2, 2000):
            lens = v["kv"]._keep[1]
            lens[0] = n
            o.zero_()
            lse.zero_()
            g.replay()
            stream.synchronize()
            got = o.clone(), lse.clone()
            big.run(P, ctx, vb)
            o.zero_()
            call(ctx)
            stream.synchronize()
            assert torch.equal(o, got[0]) and torch.equal(lse, got[1])
            if n == 4000:
                assert torch.equal(got[0], eager[0]) and torch.equal(got[1], eager[1])
        ctx.close()


def test_two_contexts_on_two_streams(ckv):
    """Calls of two contexts that run at the same time do not share memory."""
    P, ctx = ckv
    cases = [_graph_case(P, PackedBatch(42 + i, [4000, 500], [1, 1], 8, 2, 128), 0) for i in range(2)]
    want = []
    for c in cases:
        c[3](ctx)
        ctx.sync()
        want.append((c[1].clone(), c[2].clone()))
        c[1].zero_()
    torch.cuda.synchronize()
    ctxs = [P.Context(0, torch.cuda.Stream()) for _ in range(2)]
    for _ in range(20):
        for c, x in zip(cases, ctxs):
            c[3](x)
    torch.cuda.synchronize()
    for c, w in zip(cases, want):
        assert torch.equal(c[1], w[0]) and torch.equal(c[2], w[1])
    for x in ctxs:
        x.close()


@pytest.mark.parametrize("rows", [1, 70])
def test_workspace_limit(ckv, rows):
    """Without room for partial sums the call still answers, and right."""
    P, _ = ckv
    ctx = P.Context(0)
    ctx.set_workspace_limit(4096)
    b = PackedBatch(44, [5000, 100], [rows, rows], 8, 2, 128)
    check(b, b.run(P, ctx, b.device(P)), b.want(), "limit")
    assert ctx.workspace_bytes() <= 4096
    ctx.close()


def test_same_bits_again(ckv):
    """Two calls give the same bits, whatever ran between them."""
    P, ctx = ckv
    b = PackedBatch(45, [3000, 77, 2001], [1, 20, 1], 8, 2, 128)
    other = PackedBatch(46, [300], [300], 8, 2, 128)
    v = b.device(P)
    first = b.run(P, ctx, v, 1500, 4)
    other.run(P, ctx, other.device(P))
    again = b.run(P, ctx, v, 1500, 4)
    assert all(np.array_equal(x, y) for x, y in zip(first, again))


def test_rows_out_of_order(ckv):
    """cu_rows that do not ascend: any outputs, no row past n_rows, and the next call is right again."""
    P, ctx = ckv
    b = PackedBatch(47, [3000, 2000, 1000, 500], [1, 1, 1, 1], 8, 2, 128, lead=1, tail=1)
    v, want = b.device(P), b.want()
    for cu in ([5, 0, 3, 1, 4], [0, 6, 0, 6, 0], [-9, 100, -9, 100, 2], [6, 6, 0, 0, 6]):
        for most in (1, 200):
            w = P.query_view(v["q"]._keep[0], torch.tensor(cu, dtype=torch.int32, device="cuda"), max_rows=most)
            o = torch.zeros((8, 8, 128), dtype=torch.bfloat16, device="cuda")
            lse = torch.zeros((8, 8), device="cuda")
            P.ckv_attend_packed(ctx, v["kv"], w, o=o[:6], lse=lse[:6])
            torch.cuda.synchronize()
            assert not o[6:].any() and not lse[6:].any()
            check(b, b.run(P, ctx, v), want, f"after {cu}")


# ------------------------------------------------------------------- refusals

def test_refusals(ckv):
    P, ctx = ckv
    b = PackedBatch(50, [20, 30], [1, 2], 4, 2, 64)
    v = b.device(P)
    kv, q = v["kv"], v["q"]
    o = torch.zeros((3, 4, 64), dtype=torch.bfloat16, device="cuda")
    qq, cu, _ = q._keep

    def code(*a, **kw):
        with pytest.raises(P.CKVError) as e:
            P.ckv_attend_packed(ctx, *a, **kw)
        return e.value.code
    assert code(kv, q, window=-1, o=o) == -1
    assert code(kv, q, n_sink=-1, o=o) == -1
    assert code(kv, q, o=qq) == -1                    # output over the queries
    assert code(kv, P.query_view(qq, cu, scale=float("nan")), o=o) == -1
    assert code(kv, P.query_view(qq, cu, max_rows=0), o=o) == -2
    for field, value, want in [("n_kv_heads", 3, -2), ("row_stride", 72, -1), ("row_stride", 64, -2), ("head_stride", 8, -1),
                               ("pool_rows", 0, -2), ("slot_stride", 1, -2), ("n_tokens", None, -1), ("data", None, -1),
                               ("data", kv._keep[0].data_ptr() + 8, -1), ("max_tokens", -1, -2), ("row_stride", 1 << 31, -4)]:
        bad = type(kv).from_buffer_copy(kv)
        bad.__dict__.update(kv.__dict__)
        setattr(bad, field, value)
        assert code(bad, q, o=o) == want, field
    assert ctx._lib.ckv_attend_packed(ctx.handle, kv, q, 5, 0, 0, o.data_ptr(), None) == -1      # unknown type
    for call in (lambda: P.ckv_attend_packed(ctx, kv, P.query_view(qq, cu[:2])), lambda: P.ckv_attend_packed(ctx, kv, q, o=o[:, :2]),
                 lambda: P.ckv_attend_packed(ctx, kv, q, o=o, lse=o), lambda: P.ckv_attend_packed(ctx, kv, q, o=o.half()),
                 lambda: P.ckv_attend_packed(ctx, kv, q, window=2**32 + 5, o=o),
                 lambda: P.ckv_attend_packed(ctx, kv, P.query_view(torch.zeros((3, 4, 128), dtype=torch.bfloat16, device="cuda"), cu))):
        with pytest.raises(ValueError):
            call()
    ctx.sync()
    assert torch.all(o == 0)
    P.ckv_attend_packed(ctx, kv, P.query_view(qq[:0], torch.zeros(3, dtype=torch.int32, device="cuda")))    # no rows
    ctx.sync()
