"""Attention of ragged batches (ckv_attend_window, ckv_attend_shared) against the fp64 oracle.

Storage that no token owns holds NaN, and rows of no sequence a fill that must stay."""
import numpy as np
import pytest
import torch

from tests.serving_util import Batch, check

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
    """One row each behind caches of 1 to 700 tokens, tile edges among them."""
    lens = [1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 129, 257, 700]
    b = Batch(1, lens, [1] * len(lens), hq, hkv, d, type, paged)
    _run(ckv, b, what="all")
    _run(ckv, b, 1, what="own token")
    _run(ckv, b, 37, 5, what="window and sinks")


@pytest.mark.parametrize("type", ["bf16", "fp16"])
@pytest.mark.parametrize("hq,hkv,d", HEADS)
def test_prompts(ckv, hq, hkv, d, type):
    """Whole prompts and chunks behind caches, ragged."""
    b = Batch(2, [1, 77, 130, 300, 64], [1, 77, 65, 33, 64], hq, hkv, d, type, lead=3, tail=2)
    _run(ckv, b, what="all")
    _run(ckv, b, 64, what="window 64")
    _run(ckv, b, 50, 7, what="window and sinks")


@pytest.mark.parametrize("rows", [2, 3, 4, 8, 17])
def test_few_rows(ckv, rows):
    """Drafted tokens: a few rows per sequence."""
    b = Batch(3, [rows, 100, 333], [rows] * 3, 8, 2, 128)
    _run(ckv, b, what="all")
    _run(ckv, b, 40, 4, what="window")


@pytest.mark.parametrize("window,n_sink", [(0, 0), (0, 9), (1, 0), (1, 1), (2, 300), (63, 0), (64, 64), (65, 1), (299, 1),
                                           (300, 0), (2**31 - 1, 2**31 - 1)])
def test_window_edges(ckv, window, n_sink):
    b = Batch(4, [300, 64, 5], [70, 1, 5], 4, 2, 64)
    _run(ckv, b, window, n_sink, what=f"window {window}, sinks {n_sink}")


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("window,n_sink", [(0, 0), (50, 0), (50, 11), (1, 0)])
def test_gapped_positions(ckv, paged, window, n_sink):
    """Compressed caches: absolute positions with gaps."""
    b = Batch(5, [200, 1, 90, 513], [1, 1, 40, 3], 8, 2, 128, paged=paged, gaps=True)
    _run(ckv, b, window, n_sink, what="gaps")


@pytest.mark.parametrize("rows", [1, 3])
@pytest.mark.parametrize("window,n_sink", [(0, 0), (0, 4), (50, 0), (50, 11), (1, 0), (5000, 3)])
def test_gapped_single_tokens(ckv, rows, window, n_sink):
    """The same, few rows each, with caches that are split among others."""
    b = Batch(51, [200, 3, 90, 513, 9000], [rows] * 5, 8, 2, 128, gaps=True)
    _run(ckv, b, window, n_sink, what="gaps")


@pytest.mark.parametrize("seed", range(48))
def test_any_batch(ckv, seed):
    """Batches drawn over everything a view may hold."""
    rng = np.random.default_rng(seed)
    n = int(rng.choice([1, 2, 5, 70]))
    long = int(rng.choice([40, 300, 2500])) if n < 70 else 30
    lens = rng.integers(0, long + 1, n)
    few = rng.random() < 0.5
    rows = rng.integers(0, 3 if few else 90, n) if n < 70 else rng.integers(0, 4, n)
    hq, hkv, d = [(4, 1, 64), (6, 6, 64), (8, 2, 128), (20, 4, 64), (17, 1, 128)][int(rng.integers(5))]
    gaps, given = rng.random() < 0.5, rng.random() < 0.3
    prefix = int(rng.choice([0, 0, 1, 130, 700]))
    qpos = None
    if given:
        qpos = [rng.integers(-3, 3 * (prefix + long) + 3, r) for r in rows]
    elif not gaps or prefix:
        lens = np.maximum(lens, rows) if rng.random() < 0.7 else lens
    b = Batch(1000 + seed, lens, rows, hq, hkv, d, "fp16" if rng.random() < 0.5 else "bf16", rng.random() < 0.6, gaps, qpos,
              prefix, gaps, lead=int(rng.integers(3)), tail=int(rng.integers(3)))
    window = 0 if prefix else int(rng.choice([0, 1, 30, 64, 500, 1 << 30]))
    n_sink = 0 if prefix else int(rng.choice([0, 1, 40, 1 << 30]))
    _run(ckv, b, window, n_sink, max_rows=int(rng.choice([1, max(1, int(rows.max(initial=1))), 500])), what=f"seed {seed}")


@pytest.mark.parametrize("window", [0, 8])
def test_given_positions(ckv, window):
    """Rows at positions of their own, out of order and far apart, some before every token, one at the far end."""
    far = 2**31 - 1
    qpos = [[-5, 150, 0, 149, 30, far, 75, 75], [-1], [63, 2, far - 1]]
    b = Batch(6, [150, 40, 64], [8, 1, 3], 4, 2, 64, qpos=qpos)
    _run(ckv, b, window, 2 if window else 0, what="positions")
    b = Batch(6, [150, 40, 64], [8, 1, 3], 4, 2, 64, qpos=qpos, gaps=True)
    _run(ckv, b, window, 2 if window else 0, what="gapped positions")


def test_empty_sequences(ckv):
    """No tokens, no rows, neither; rows whose tokens are not in the cache."""
    b = Batch(7, [0, 5, 0, 20, 3], [1, 0, 0, 2, 5], 4, 2, 64, lead=1)
    o, lse = _run(ckv, b, what="empty")
    assert np.all(o[0] == 0) and np.all(np.isneginf(lse[0]))
    _run(ckv, b, 4, 1, what="empty, window")
    b = Batch(7, [0, 5, 0, 20, 3], [1, 0, 0, 2, 5], 4, 2, 64, gaps=True)
    _run(ckv, b, 4, 1, what="empty, positions")
    b = Batch(8, [0], [3], 4, 2, 64, tables=1)
    _run(ckv, b, what="nothing at all")


def test_many_sequences(ckv):
    """More sequences than a workgroup has threads, most of them tiny."""
    rng = np.random.default_rng(9)
    lens = rng.integers(0, 12, 1300)
    b = Batch(9, lens, (rng.random(1300) < 0.7).astype(int), 2, 1, 64)
    _run(ckv, b, what="many")
    b = Batch(9, lens, rng.integers(0, 4, 1300), 2, 1, 64)
    _run(ckv, b, 5, 2, what="many, few rows")


@pytest.mark.parametrize("rows", [1, 5])
def test_long_axis(ckv, rows):
    """A long cache split over the device, ragged."""
    b = Batch(10, [9001, 40, 4097], [rows, rows, rows], 4, 2, 128)
    _run(ckv, b, what="long")
    _run(ckv, b, 3000, 3, what="long, window")


@pytest.mark.parametrize("guess", [1, 2, 1000])
def test_any_estimate_of_rows(ckv, guess):
    """max_rows is an estimate: results hold whatever it says."""
    b = Batch(11, [150, 64, 33, 7], [130, 1, 33, 2], 4, 2, 64)
    _run(ckv, b, max_rows=guess, what=f"estimate {guess}")
    _run(ckv, b, 20, 3, max_rows=guess, what=f"estimate {guess}, window")


@pytest.mark.parametrize("scale", [1.0, 0.02])
def test_scale(ckv, scale):
    """A softmax scale of the caller's: sharp and flat rows."""
    b = Batch(12, [200, 90], [1, 33], 4, 2, 64, scale=scale)
    _run(ckv, b, what=f"scale {scale}")


def test_strides(ckv):
    """Heads inside rows (token-major storage), padded rows, queries inside a wider tensor, tables wider than used."""
    P, ctx = ckv
    b = Batch(13, [90, 130, 17], [1, 20, 17], 8, 2, 64)
    want = b.want(33, 4)
    v = b.device(P)
    kv, q = v["kv"], v["q"]
    k, vv, lens, slot, _ = kv._keep
    big = torch.full((2, k.shape[1], 3, 2, 64 + 8), float("nan"), dtype=k.dtype, device="cuda")   # [k/v][row][..][head][d + pad]
    for i, x in enumerate((k, vv)):
        big[i, :, 1, :, :64] = x.transpose(0, 1)
    ks, vs = (big[i, :, 1, :, :64].transpose(0, 1) for i in range(2))
    wide = torch.full((3, slot.shape[1] + 30), 1 << 30, dtype=torch.int32, device="cuda")
    wide[:, :slot.shape[1]] = slot
    qq, cu, _ = q._keep
    qw = torch.full((qq.shape[0], 5, 8, 64 + 16), float("nan"), dtype=qq.dtype, device="cuda")
    qw[:, 2, :, 8:72] = qq
    kv2 = P.batch_view(ks, vs, lens, slot=wide[:, :slot.shape[1]])
    q2 = P.query_view(qw[:, 2, :, 8:72], cu, max_rows=20)
    check(b, b.run(P, ctx, dict(kv=kv2, q=q2), 33, 4), want, "strides")


def test_clamped_slots(ckv):
    """Rows outside the pool read its last row, and never past it."""
    P, ctx = ckv
    b = Batch(14, [40, 70], [1, 3], 4, 2, 64)
    v = b.device(P)
    k, vv, lens, slot, _ = v["kv"]._keep
    k[:, -1], vv[:, -1] = 0.5, 0.25
    s2, last = slot.clone(), k.shape[1] - 1
    s2[0, 3], s2[0, 17], s2[1, 60] = -1, 1 << 30, last + 1
    got = b.run(P, ctx, dict(kv=P.batch_view(k, vv, lens, slot=s2), q=v["q"]))
    s3 = s2.clone()
    s3[(s2 < 0) | (s2 > last)] = last
    s3[slot < 0] = slot[slot < 0]
    same = b.run(P, ctx, dict(kv=P.batch_view(k, vv, lens, slot=s3), q=v["q"]))
    assert all(np.array_equal(x, y) for x, y in zip(got, same))


def test_counts_are_clamped(ckv):
    """Lengths past max_tokens count as max_tokens, negative ones as 0; row bounds stay inside the rows."""
    P, ctx = ckv
    b = Batch(15, [30, 30, 30], [2, 2, 2], 4, 2, 64, tables=30)
    v = b.device(P)
    k, vv, lens, slot, _ = v["kv"]._keep
    want = b.run(P, ctx, v)
    bad = torch.tensor([31, 1 << 30, 30], dtype=torch.int32, device="cuda")
    got = b.run(P, ctx, dict(kv=P.batch_view(k, vv, bad, slot=slot), q=v["q"]))
    assert all(np.array_equal(x, y) for x, y in zip(got, want))
    q, cu, _ = v["q"]._keep
    wild = torch.tensor([-9, 2, 4, 1 << 30], dtype=torch.int32, device="cuda")
    got = b.run(P, ctx, dict(kv=v["kv"], q=P.query_view(q, wild, max_rows=2)))
    assert all(np.array_equal(x, y) for x, y in zip(got, want))
    none = torch.tensor([-5, 30, 30], dtype=torch.int32, device="cuda")
    o, lse = b.run(P, ctx, dict(kv=P.batch_view(k, vv, none, slot=slot), q=v["q"]))
    assert np.all(o[:2] == 0) and np.all(np.isneginf(lse[:2]))


@pytest.mark.parametrize("rows", [1, 40])
def test_hidden_tokens_hold_anything(ckv, rows):
    """NaN and infinities in keys and values of tokens that a row does not see stay out of that row."""
    P, ctx = ckv
    n = 200
    for case in ("before the window", "behind every row", "seen by later rows only"):
        b = Batch(16, [n, 60], [rows, 1], 4, 2, 64, qpos=[n - 61 + np.arange(rows), [59]])
        want = b.want(32, 3)
        clean = rows
        if case == "before the window":
            bad = slice(10, 100)
        elif case == "behind every row":
            bad = slice(n - 61 + rows, n)
        else:
            bad, clean = slice(n - 61 + rows - 1, n), rows - 1
        b.k[0][bad] = torch.tensor([float("nan"), float("inf"), -float("inf"), 1.0]).repeat(16).to(b.k[0].dtype)
        b.v[0][bad] = float("inf")
        b.v[0][bad][::2] = float("nan")
        v = b.device(P)
        if case == "seen by later rows only":
            with pytest.raises(P.CKVError):
                b.run(P, ctx, v, 32, 3)
            keep = v["q"]
            o = torch.zeros((rows + 1, 4, 64), dtype=torch.bfloat16, device="cuda")
            lse = torch.zeros((rows + 1, 4), dtype=torch.float32, device="cuda")
            P.ckv_attend_window(ctx, v["kv"], keep, window=32, n_sink=3, o=o, lse=lse)
            with pytest.raises(P.CKVError, match="NONFINITE"):
                ctx.sync()
            got = o.cpu().double().numpy(), lse.cpu().double().numpy()
            pick = list(range(clean)) + [rows]
            assert not np.isfinite(got[0][clean:rows]).all()
        else:
            got, pick = b.run(P, ctx, v, 32, 3), list(range(rows + 1))
        check(b, tuple(x[pick] for x in got), tuple(x[pick] for x in want), case)


def test_sequences_do_not_touch_each_other(ckv):
    """A sequence's results do not depend on what the others hold."""
    P, ctx = ckv
    b = Batch(17, [100, 100], [1, 1], 4, 2, 64)
    want = b.want()
    b.v[1][50] = float("nan")
    v = b.device(P)
    o = torch.zeros((2, 4, 64), dtype=torch.bfloat16, device="cuda")
    P.ckv_attend_window(ctx, v["kv"], v["q"], o=o)
    with pytest.raises(P.CKVError, match="NONFINITE"):
        ctx.sync()
    o = o.cpu().double().numpy()
    b.v[1][50] = 0
    check(b, (o[:1], want[1][:1]), tuple(x[:1] for x in want), "beside a NaN")
    assert np.isnan(o[1]).any()


def test_extreme_logits(ckv):
    """Rows with one dominant token, logits of several hundred, and all logits alike."""
    b = Batch(18, [300, 300], [1, 64], 4, 2, 64, heavy=False)
    for s in range(2):
        b.k[s][7] *= 16
        b.k[s][150] *= -16
    _run(ckv, b, what="dominant")
    b.k = [torch.zeros_like(x) for x in b.k]
    _run(ckv, b, what="alike")


def test_same_bits_again(ckv):
    """Two calls give the same bits, whatever ran between them."""
    P, ctx = ckv
    b = Batch(19, [5000, 77, 3001], [1, 20, 1], 8, 2, 128)
    other = Batch(20, [900], [900], 8, 2, 128)
    v = b.device(P)
    first = b.run(P, ctx, v, 2500, 4)
    other.run(P, ctx, other.device(P))
    again = b.run(P, ctx, v, 2500, 4)
    assert all(np.array_equal(x, y) for x, y in zip(first, again))


# ------------------------------------------------------------------- shared prefix

@pytest.mark.parametrize("type", ["bf16", "fp16"])
@pytest.mark.parametrize("hq,hkv,d", HEADS)
def test_shared_single_tokens(ckv, hq, hkv, d, type):
    lens = [1, 2, 17, 64, 65, 130]
    for prefix in (1, 63, 300):
        b = Batch(30, lens, [1] * len(lens), hq, hkv, d, type, prefix=prefix)
        _run(ckv, b, what=f"prefix {prefix}")


@pytest.mark.parametrize("paged", [False, True])
def test_shared_chunks(ckv, paged):
    b = Batch(31, [50, 7, 129, 64], [50, 1, 100, 3], 8, 2, 128, prefix=200, lead=1, tail=4, paged=paged)
    _run(ckv, b, what="chunks")
    b = Batch(31, [50, 7, 129, 64], [50, 1, 100, 3], 8, 2, 128, prefix=200, gaps=True, prefix_gaps=True, paged=paged)
    _run(ckv, b, what="gapped chunks")


def test_shared_without_own_tokens(ckv):
    """Rows that read the prefix alone, at positions inside and behind it."""
    b = Batch(32, [0, 4, 0], [2, 1, 0], 4, 2, 64, prefix=90, qpos=[[89, 10], [93], []])
    _run(ckv, b, what="prefix alone")
    b = Batch(32, [0, 4], [1, 1], 4, 2, 64, prefix=90, qpos=[[-1], [93]])
    o, lse = _run(ckv, b, what="nothing")
    assert np.all(np.isneginf(lse[0])) and np.all(o[0] == 0)


def test_shared_many_rows(ckv):
    """A batch of many samples: more rows per KV head than any tile."""
    b = Batch(33, np.random.default_rng(1).integers(1, 40, 90), [1] * 90, 8, 1, 128, prefix=1000)
    _run(ckv, b, what="many")


def test_shared_equals_window_on_copies(ckv):
    """The shared call against the window call on caches that hold the prefix each."""
    P, ctx = ckv
    b = Batch(34, [30, 61], [1, 9], 8, 2, 128, prefix=500)
    got = b.run(P, ctx, b.device(P))
    c = Batch(34, [530, 561], [1, 9], 8, 2, 128)
    c.k, c.v = [torch.cat([b.pk, x]) for x in b.k], [torch.cat([b.pv, x]) for x in b.v]
    c.q = b.q
    check(b, c.run(P, ctx, c.device(P)), b.want(), "copies")
    check(b, got, b.want(), "shared")


# ------------------------------------------------------- streams, capture, memory

def _graph_case(P, b, window):
    v = b.device(P)
    total = int(b.rows.sum())
    o = torch.zeros((total, b.hq, b.d), dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros((total, b.hq), dtype=torch.float32, device="cuda")

    def call(ctx):
        if b.prefix:
            P.ckv_attend_shared(ctx, v["prefix"], v["kv"], v["q"], o=o, lse=lse)
        else:
            P.ckv_attend_window(ctx, v["kv"], v["q"], window=window, n_sink=2 if window else 0, o=o, lse=lse)
    return v, o, lse, call


@pytest.mark.parametrize("prefix", [0, 700])
def test_captured_step_serves_grown_caches(ckv, prefix):
    """A captured call replays with the lengths of the moment; larger eager calls in between do not move its memory."""
    P, _ = ckv
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = P.Context(0, stream)
        b = Batch(40, [4000, 900, 1], [1, 1, 1], 8, 2, 128, tables=4100, prefix=prefix)
        window = 0 if prefix else 3500
        v, o, lse, call = _graph_case(P, b, window)
        call(ctx)
        stream.synchronize()
        eager = o.clone(), lse.clone()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            call(ctx)
        big = Batch(41, [600] * 40, [30] * 40, 8, 2, 128)
        vb = big.device(P)
        for n in (4000, 3, 2000):
            lens = v["kv"]._keep[2]
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
    b = [Batch(42 + i, [6000, 500], [1, 1], 8, 2, 128) for i in range(2)]
    cases = [_graph_case(P, x, 0) for x in b]
    want = []
    for c in cases:
        c[3](ctx)
        ctx.sync()
        want.append((c[1].clone(), c[2].clone()))
        c[1].zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    ctxs = [P.Context(0, s) for s in streams]
    for _ in range(20):
        for c, x in zip(cases, ctxs):
            c[3](x)
    torch.cuda.synchronize()
    for c, w in zip(cases, want):
        assert torch.equal(c[1], w[0]) and torch.equal(c[2], w[1])
    for x in ctxs:
        x.close()


def test_workspace_limit(ckv):
    """Without room for partial sums the call still answers, and right."""
    P, _ = ckv
    ctx = P.Context(0)
    ctx.set_workspace_limit(4096)
    b = Batch(44, [9000, 100], [1, 1], 8, 2, 128)
    check(b, b.run(P, ctx, b.device(P)), b.want(), "limit")
    b = Batch(44, [60, 10], [1, 1], 8, 2, 128, prefix=3001)
    check(b, b.run(P, ctx, b.device(P)), b.want(), "limit, shared")
    assert ctx.workspace_bytes() <= 4096
    ctx.close()


def test_workspace_limit_counts_partial_sums(ckv):
    """What the attention holds counts for the calls that come after it, single ones and batches."""
    from tests.test_gpu_batch import WANT, _problem
    P, _ = ckv
    one = _problem(P, 16, 8, 64, 4096, 8, 16, False, seed=3)
    ctx = P.Context(0)
    b = Batch(46, [9000, 100], [1, 1], 8, 2, 128)
    b.run(P, ctx, b.device(P))
    held = ctx.workspace_bytes()
    assert held > 0
    ctx.set_workspace_limit(held + 4096)
    with pytest.raises(P.CKVError) as e:
        P.ckv_measure_page_effects(ctx, *one[:3], want=WANT)
    assert e.value.code == -5
    ctx.set_workspace_limit(held + (64 << 20))
    got = P.ckv_measure_page_effects_batch(ctx, *[[one[j]] * 3 for j in range(3)], want=WANT)
    assert len(got) == 3 and ctx.workspace_bytes() <= held + (64 << 20)
    ctx.close()


@pytest.mark.parametrize("prefix", [0, 300])
def test_rows_out_of_order(ckv, prefix):
    """cu_rows that do not ascend: any outputs, no row past n_rows, and the next call is right again."""
    P, ctx = ckv
    b = Batch(47, [5000, 4000, 6000, 3000], [1, 1, 1, 1], 8, 2, 128, prefix=prefix, lead=1, tail=1)
    v = b.device(P)
    for cu in ([5, 0, 3, 1, 4], [0, 6, 0, 6, 0], [-9, 100, -9, 100, 2], [6, 6, 0, 0, 6]):
        for most in (1, 200):
            w = P.query_view(v["q"]._keep[0], torch.tensor(cu, dtype=torch.int32, device="cuda"), max_rows=most)
            o = torch.zeros((8, 8, 128), dtype=torch.bfloat16, device="cuda")
            lse = torch.zeros((8, 8), device="cuda")
            if prefix:
                P.ckv_attend_shared(ctx, v["prefix"], v["kv"], w, o=o[:6], lse=lse[:6])
            else:
                P.ckv_attend_window(ctx, v["kv"], w, o=o[:6], lse=lse[:6])
            torch.cuda.synchronize()
            assert not o[6:].any() and not lse[6:].any()
            check(b, b.run(P, ctx, v), b.want(), f"after {cu}")


# ------------------------------------------------------------------- refusals

def test_more_than_a_launch_holds(ckv):
    """2^20 sequences of 32 KV heads, none with a row: more row blocks than a grid has."""
    P, ctx = ckv
    n = 1 << 20
    k = torch.zeros((32, 4, 64), dtype=torch.bfloat16, device="cuda")
    zero = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
    kv = P.batch_view(k, k.clone(), zero[:n], slot=torch.zeros((n, 1), dtype=torch.int32, device="cuda"))
    q = torch.zeros((n, 32, 64), dtype=torch.bfloat16, device="cuda")
    o = torch.zeros_like(q)
    for most in (1, 1000):
        with pytest.raises(P.CKVError) as e:
            P.ckv_attend_window(ctx, kv, P.query_view(q, zero, max_rows=most), o=o)
        assert e.value.code == -4



def test_refusals(ckv):
    P, ctx = ckv
    b = Batch(50, [20, 30], [1, 2], 4, 2, 64, prefix=8)
    v = b.device(P)
    kv, q, pre = v["kv"], v["q"], v["prefix"]
    o = torch.zeros((3, 4, 64), dtype=torch.bfloat16, device="cuda")
    k, vv, lens, slot, _ = kv._keep

    def code(fn, *a, **kw):
        with pytest.raises(P.CKVError) as e:
            fn(ctx, *a, **kw)
        return e.value.code
    assert code(P.ckv_attend_window, kv, q, window=-1, o=o) == -1
    assert code(P.ckv_attend_window, kv, q, n_sink=-1, o=o) == -1
    qq, cu, _ = q._keep
    assert code(P.ckv_attend_window, kv, q, o=qq) == -1                    # output over the queries
    assert code(P.ckv_attend_window, kv, P.query_view(qq, cu, scale=float("nan")), o=o) == -1
    assert code(P.ckv_attend_window, kv, P.query_view(qq, cu, max_rows=0), o=o) == -2
    for field, value, want in [("head_dim", 96, None), ("dtype", 5, -1), ("n_kv_heads", 3, -2), ("tok_stride", 65, -1),
                               ("tok_stride", 56, -2), ("pool_rows", 0, -2), ("slot_stride", 1, -2), ("n_tokens", None, -1),
                               ("k", None, -1), ("k", k.data_ptr() + 2, -1), ("max_tokens", -1, -2)]:
        bad = type(kv).from_buffer_copy(kv)
        bad.__dict__.update(kv.__dict__)
        setattr(bad, field, value)
        if want is None:
            with pytest.raises(ValueError):
                P.ckv_attend_window(ctx, bad, q, o=o)
        else:
            assert code(P.ckv_attend_window, bad, q, o=o) == want, field
            assert code(P.ckv_attend_shared, pre, bad, q, o=o) == want, field
    # the binding's own
    half = P.query_view(qq.half(), cu)
    for call in (lambda: P.ckv_attend_window(ctx, kv, half), lambda: P.ckv_attend_shared(ctx, kv, kv, q),
                 lambda: P.ckv_attend_window(ctx, kv, P.query_view(qq, cu[:2])),
                 lambda: P.ckv_attend_window(ctx, kv, q, o=o[:, :2]),
                 lambda: P.ckv_attend_window(ctx, kv, q, o=o, lse=o),
                 lambda: P.batch_view(k, vv, lens.long(), slot=slot), lambda: P.batch_view(k, vv, lens, slot=slot[:1]),
                 lambda: P.batch_view(k.float(), vv.float(), lens, slot=slot),
                 lambda: P.batch_view(k, vv, lens, slot=slot, max_tokens=slot.shape[1] + 1),
                 lambda: P.query_view(qq.cpu(), cu), lambda: P.query_view(qq, cu.cpu()),
                 lambda: P.batch_view(k, vv, lens, slot=slot.cpu())):
        with pytest.raises(ValueError):
            call()
    # none of it was enqueued
    ctx.sync()
    assert torch.all(o == 0)
    # an empty batch is served
    none = P.query_view(qq[:0], torch.zeros(3, dtype=torch.int32, device="cuda"))
    P.ckv_attend_window(ctx, kv, none)
    ctx.sync()
