"""Attention where a batch or its storage is large: more sequences than a wave or a workgroup has lanes, with their work
cut, and rows that 32-bit offsets do not reach; and the precision that few rows keep."""
import numpy as np
import pytest
import torch

from oracle import serving as S
from tests.serving_util import HALF, TYPES, Batch, check

pytestmark = pytest.mark.gpu


@pytest.fixture()
def ckv():
    """A context of each test's own, whose memory tells whether a call had partial sums."""
    import paper_2608_07855_amd as P
    ctx = P.Context(0)
    yield P, ctx
    ctx.close()


# ------------------------------------------------------------ many sequences

def _ragged(n, seed, long, low=40):
    """Lengths below ``low``, and one of ``long`` at a few places all over the batch, the last among them."""
    lens = np.random.default_rng(seed).integers(1, low, n)
    at = np.linspace(3, n - 1, len(long)).astype(int)
    lens[at] = long
    return lens, at


@pytest.mark.parametrize("n,hq,hkv,d", [(70, 4, 1, 64), (200, 4, 1, 64), (300, 8, 2, 64), (600, 4, 2, 64), (80, 4, 1, 128),
                                        (300, 8, 2, 128), (300, 2, 2, 128)])
@pytest.mark.parametrize("prefix", [0, 150])
def test_single_tokens_in_splits(ckv, n, hq, hkv, d, prefix):
    """One row each of more than 64 sequences, some of them in several splits."""
    P, ctx = ckv
    lens, at = _ragged(n, n + d, [4500, 6100, 5003, 8191])
    # splits have at least 2048 tokens, and as many as leave about 1024 of them
    chunk = max(2048, -(-int(lens.sum()) * hkv // 1024))
    assert np.all(lens[at] > 2 * chunk)
    b = Batch(n, lens, [1] * n, hq, hkv, d, prefix=prefix)
    v = b.device(P)
    got = b.run(P, ctx, v)
    assert ctx.workspace_bytes() > 0
    check(b, got, b.want(), f"{n} sequences")
    check(b, b.run(P, ctx, v), b.want(), "again")


def _cut(lens, rows, group, hkv, prefix):
    """Whether blocks of 256 rows are cut: whole ones would leave some of the 256 / hkv workgroups of a head more than
    six tiles behind the others."""
    work, most, blocks = 0, 0, 0
    step = max(256 // group, 1)
    for n, r in zip(lens, rows):
        k = -(-r * group // 256)
        see = [prefix + min(max(n - r + min(r, step), 1) + i * step, n) for i in range(k)]
        work, most, blocks = work + sum(see), max([most] + [prefix + n] * int(k > 0)), blocks + k
    W = 256 // hkv
    return -(-blocks // W) * most > work / W + 6 * 64


@pytest.mark.parametrize("n", [70, 130, 600])
@pytest.mark.parametrize("prefix", [0, 200])
@pytest.mark.parametrize("d", [64, 128])
def test_many_rows_in_shares(ckv, n, prefix, d):
    """Single tokens, short chunks, sequences without rows and a few long chunks: shares begin and end in sequences past
    the first 64 and past the first 512."""
    P, ctx = ckv
    hq, hkv = 16, 8
    lens, at = _ragged(n, n, [700, 500, 811, 640], 25)
    rows = np.minimum(lens, np.random.default_rng(n + 1).integers(0, 4, n))
    rows[at] = lens[at] - [5, 0, 200, 1]
    assert _cut(lens, rows, hq // hkv, hkv, prefix) and at[-1] == n - 1
    b = Batch(n + d, lens, rows, hq, hkv, d, prefix=prefix)
    got = b.run(P, ctx, b.device(P))
    assert ctx.workspace_bytes() > 0
    check(b, got, b.want(), f"{n} sequences")


# --------------------------------------------------------------- many heads

@pytest.mark.parametrize("hq,hkv,lens,rows", [(300, 1, [400, 3], [20, 1]), (300, 1, [2500, 40], [1, 1]),
                                              (300, 300, [5000, 9], [1, 1]), (520, 260, [150, 30], [70, 2])])
@pytest.mark.parametrize("prefix", [0, 70])
def test_many_heads(ckv, hq, hkv, lens, rows, prefix):
    """Groups of more query heads than a block has rows, and more KV heads than workgroups at a time."""
    P, ctx = ckv
    b = Batch(hq + hkv, lens, rows, hq, hkv, 64, prefix=prefix)
    check(b, b.run(P, ctx, b.device(P)), b.want(), f"{hq} heads on {hkv}")


# ---------------------------------------------------------------- far rows

@pytest.mark.parametrize("rows", [1, 600])
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("pool,tok_stride", [(1100, 1 << 21), (1000, 1 << 21), ((1 << 24) + 500, 64)])
def test_far_rows(ckv, pool, tok_stride, paged, rows):
    """Rows 4 MiB apart, past 4 GiB and just short of it, and more than 2^24 rows: n tokens at the end of a contiguous
    cache, behind a window, or anywhere in a pool, where they are a shared prefix, too."""
    P, ctx = ckv
    d, n = 64, 900 if pool > 1000 else 1000
    b = Batch(rows, [n, 1], [rows, 1], 4, 1, d, heavy=False)
    if tok_stride > d:       # k and v in one buffer: most of it is never touched
        mem = torch.empty(pool * tok_stride, dtype=torch.bfloat16, device="cuda")
        kp, vp = (mem.as_strided((1, pool, d), (d, tok_stride, 1), off) for off in (0, 2 * d))
    else:
        kp, vp = (torch.empty((1, pool, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    at = np.arange(pool - n, pool)
    if paged:
        inner = np.random.default_rng(3).choice(np.arange(1, pool - 1), n - 2, replace=False)
        at = np.concatenate([[pool - 1, 0], inner])
    at = torch.from_numpy(at).cuda()
    kp[0, at], vp[0, at] = b.k[0][:, 0].cuda(), b.v[0][:, 0].cuda()

    def view(k, v, tokens, slot=None):
        return P.batch_view(k, v, torch.tensor([tokens], dtype=torch.int32, device="cuda"), slot=slot)
    far = view(kp, vp, n, at.to(torch.int32)[None].contiguous()) if paged else view(kp[None], vp[None], pool)
    q = P.query_view(b.q[0].cuda(), torch.tensor([0, rows], dtype=torch.int32, device="cuda"))

    def same(got, k, v, window, what):
        ctx.sync()
        vis = S.sees(np.arange(len(k)), np.arange(rows) + len(k) - rows, window)
        want = S.attend_rows(b.q[0].double().numpy(), k.double().numpy(), v.double().numpy(), vis)
        check(b, tuple(got[x].cpu().double().numpy() for x in ("o", "lse")), want, what)
    window = 0 if paged else n - rows + 1      # no row sees what lies before the n tokens
    same(P.ckv_attend_window(ctx, far, q, window=window, want=("o", "lse")), b.k[0], b.v[0], window, "alone")
    if paged:
        own = view(*(x[1].transpose(0, 1)[None].contiguous().cuda() for x in (b.k, b.v)), 1)
        same(P.ckv_attend_shared(ctx, far, own, q, want=("o", "lse")), torch.cat(b.k), torch.cat(b.v), 0, "shared")


# ------------------------------------------------------- hidden shared tokens

@pytest.mark.parametrize("limited", [False, True])
@pytest.mark.parametrize("rows", [1, 60])
@pytest.mark.parametrize("type", ["bf16", "fp16"])
def test_hidden_shared_tokens_hold_anything(ckv, type, rows, limited):
    """Rows at positions inside the prefix, behind which it holds what is not finite, as the sequences' own tokens do;
    then one row that sees the first of it, in the block of rows that do not."""
    P, ctx = ckv
    if limited:
        ctx.set_workspace_limit(4096)
    qpos = [np.arange(rows) + 100 - rows, [40], [99] * rows]
    b = Batch(40, [rows, 5, 70], [rows, 1, rows], 8, 2, 64, type, prefix=300, qpos=qpos)
    want = b.want()
    bad = torch.tensor([float("nan"), float("inf"), -float("inf"), 1.0]).repeat(16).to(TYPES[type])

    def device():
        """The batch's views with the hidden tokens overwritten; the host (of whose values the tolerances are) stays."""
        hidden = [b.pk[100:], b.pv[100:]] + b.k + b.v
        keep = [x.clone() for x in hidden]
        for x in hidden:
            x[:] = bad
        v = b.device(P)
        for x, y in zip(hidden, keep):
            x[:] = y
        return v
    check(b, b.run(P, ctx, device()), want, "none sees it")
    b.given_qpos[1] = [100]
    v = device()
    o, lse = torch.zeros((2 * rows + 1, 8, 64), dtype=TYPES[type], device="cuda"), torch.zeros((2 * rows + 1, 8), device="cuda")
    P.ckv_attend_shared(ctx, v["prefix"], v["kv"], v["q"], o=o, lse=lse)
    with pytest.raises(P.CKVError, match="NONFINITE"):
        ctx.sync()
    got = o.cpu().double().numpy(), lse.cpu().double().numpy()
    assert not np.isfinite(got[0][rows]).any()
    rest = np.arange(2 * rows + 1) != rows
    check(b, tuple(x[rest] for x in got), tuple(x[rest] for x in want), "one sees it")


# ------------------------------------------------------------- what few rows keep

def _rounded(q, k, v, type):
    """The oracle's rows over all tokens, with every weight (against the largest one) rounded once to the type."""
    out = np.zeros(q.shape)
    for h in range(q.shape[1]):
        g = h // (q.shape[1] // k.shape[1])
        x = k[:, g] @ q[0, h] / np.sqrt(q.shape[2])
        e = np.exp(x - x.max())
        r = torch.from_numpy(e).to(TYPES[type]).double().numpy()
        out[0, h] = r @ v[:, g] / e.sum()
    return out


@pytest.mark.parametrize("type", ["bf16", "fp16"])
@pytest.mark.parametrize("paged", [False, True])
def test_few_rows_keep_their_weights(ckv, paged, type):
    """Few rows' weights are two values of the type: what is left of their rounding is h^2 of them, for half a step h.
    Beside it stands o's own rounding, 2^-13 of the weights for float32, and in fp16 2^-40 of the largest weight a
    token (values stay below 8).  Weights rounded once would pass that."""
    P, ctx = ckv
    lens = [2, 3, 4, 5, 17, 33, 400]
    b = Batch(5, lens, [1] * len(lens), 34, 2, 64, type, paged, heavy=False)
    o, lse = b.run(P, ctx, b.device(P))
    wo, wl, w = b.want()
    h = HALF[type]
    tol = h * np.abs(wo) + (h * h + 2.0**-13) * w + max(lens) * 8 * 2.0**-40 * (type == "fp16") + 2.0**-24
    e = np.abs(o - wo) / tol
    print(f"[parity] o {e.max():.3g} of the tolerance", flush=True)
    assert e.max() <= 1
    once = np.concatenate([_rounded(*(x[s].double().numpy() for x in (b.q, b.k, b.v)), type) for s in range(b.n)])
    miss = np.abs(once - wo) / ((h * h + 2.0**-13) * w + 2.0**-24)
    print(f"[parity] weights rounded once: {miss.max():.3g} of what is left beside o's rounding", flush=True)
    assert (miss > 1).any()
