"""bf16 queries of very different size in one call over 4-bit caches: every row keeps its own logits, whatever the rows
beside it hold, in both kernels."""
import numpy as np
import pytest
import torch

from oracle import packed as O
from tests.packed_util import HALF, PackedBatch, check

pytestmark = pytest.mark.gpu

MANY = 1 << 28            # an estimate of rows that the many-rows kernel takes


@pytest.fixture(scope="module")
def ckv():
    import paper_2608_07855_amd as P
    ctx = P.Context(0)
    yield P, ctx
    ctx.close()


def _check_large(b, big, got, want, seen, what):
    """Rows ``big`` [n_rows, Hq], whose largest logit leaves the others behind.  A logit's 64 to 128 products are exact in
    float32; each sum of two is off by 2^-24 of sum |q k|, d of them, and its scaling and the exponential's reference by
    2^-22 of it.  Where the second largest lies 256 behind, one token has all the weight: the output is its value."""
    o, lse = got
    wo, wl, _ = want
    scale = b.d**-0.5 if b.scale is None else b.scale
    q = np.concatenate([x.double().numpy() for x in b.q])
    at, checked, rows = 0, 0, 0
    for s in range(b.n):
        k = b.k[s].double().numpy()
        for r in range(int(b.rows[s])):
            vis = seen[s][r]
            for h in range(b.hq):
                if not big[at, h] or not vis.any():
                    continue
                kk = k[vis, h // (b.hq // b.hkv)]
                x = np.sort(kk @ q[at, h] * scale)
                off = b.d * 2.0**-24 * scale * float((np.abs(kk) @ np.abs(q[at, h])).max()) + 2.0**-22 * abs(wl[at, h]) + 2.0**-13
                assert abs(lse[at, h] - wl[at, h]) <= off, f"{what}: lse of row {at}, head {h}"
                rows += 1
                if x.size == 1 or x[-1] - x[-2] > 256 + 2 * off:
                    checked += 1
                    assert np.all(np.abs(o[at, h] - wo[at, h]) <= HALF["bf16"] * np.abs(wo[at, h]) + 2.0**-24), f"{what}: row {at}, head {h}"
            at += 1
    assert rows and checked >= 0.8 * rows


def _sees(b, window, n_sink):
    from oracle import serving as S
    return [S.sees(b.positions(s), b.qpos(s), window, n_sink) for s in range(b.n)]


@pytest.mark.parametrize("most", [None, MANY])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("log", [13, 15, 20, 24, 28, 40, 60, 100])
def test_rows_beside_larger_ones(ckv, log, d, most):
    """Every other row 2^log as large as the rest."""
    P, ctx = ckv
    b = PackedBatch(log, [150, 60], [40, 3], 4, 2, d, heavy=False)
    big = np.zeros((43, 4), bool)
    big[::2] = True
    b.q[0][::2] *= 2.0**log
    b.q[1][1::2] *= 2.0**log              # (rows 40, 41, 42 of the batch)
    got, want = b.run(P, ctx, b.device(P, max_rows=most)), b.want()
    big[40:] = [[False], [True], [False]]
    small = ~big
    pick = [x[small][:, None] for x in got], [x[small][:, None] for x in want]
    check(b, *pick, f"2^{log}, the small rows")
    _check_large(b, big, got, want, _sees(b, 0, 0), f"2^{log}")


@pytest.mark.parametrize("most", [None, MANY])
def test_heads_beside_larger_ones(ckv, most):
    """Single heads of single rows far above and below the others, with windows, first tokens and gapped positions, in
    caches long enough to fall into several shares."""
    P, ctx = ckv
    for d, gaps, paged in ((64, True, True), (128, False, False)):
        b = PackedBatch(3, [2100, 90, 500], [30, 90, 1], 8, 2, d, gaps=gaps, paged=paged, heavy=False)
        rng = np.random.default_rng(4)
        big, at = np.zeros((121, 8), bool), 0
        for x in b.q:
            up, down = rng.random(x.shape[:2]) < 0.1, rng.random(x.shape[:2]) < 0.1
            x[torch.from_numpy(up)] *= 2.0**30
            x[torch.from_numpy(down & ~up)] *= 2.0**-30
            big[at:at + x.shape[0]] = up
            at += x.shape[0]
        for window, n_sink in ((0, 0), (60, 5)):
            got, want = b.run(P, ctx, b.device(P, max_rows=most), window, n_sink), b.want(window, n_sink)
            check(b, [x[~big][:, None] for x in got], [x[~big][:, None] for x in want], f"window {window}")
            _check_large(b, big, got, want, _sees(b, window, n_sink), f"window {window}")


@pytest.mark.parametrize("most", [None, MANY])
def test_tiny_rows_beside_ordinary_ones(ckv, most):
    """Rows whose logits are next to nothing (and rows of zeros) weight all tokens alike."""
    P, ctx = ckv
    b = PackedBatch(5, [150, 60], [40, 3], 4, 2, 64, heavy=False)
    for size, rows in ((2.0**-30, slice(1, None, 3)), (2.0**-126, slice(2, None, 6)), (0.0, slice(5, None, 6))):
        b.q[0][rows] *= size
    check(b, b.run(P, ctx, b.device(P, max_rows=most)), b.want(), "tiny rows")


@pytest.mark.parametrize("most", [None, MANY])
def test_a_hidden_row_of_bytes_beside_large_queries(ckv, most):
    """Rows taken apart do not see what their window hides either."""
    P, ctx = ckv
    b = PackedBatch(6, [200, 60], [40, 1], 4, 2, 64, heavy=False)
    b.q[0][::2] *= 2.0**40
    want = b.want(32, 3)
    b.bytes[0][10:100] = 0xFF             # NaN scales and bases behind every row's window
    got = b.run(P, ctx, b.device(P, max_rows=most), 32, 3)
    big = np.zeros((41, 4), bool)
    big[:40:2] = True
    check(b, [x[~big][:, None] for x in got], [x[~big][:, None] for x in want], "hidden bytes")
    _check_large(b, big, got, want, _sees(b, 32, 3), "hidden bytes")


@pytest.mark.parametrize("most", [None, MANY])
@pytest.mark.parametrize("top", [1.0, 1.9921875])
def test_small_elements_of_a_row(ckv, most, top):
    """An element far below its row's largest one is off by 2^-39 of that at most: fp16's last place is 2^-24, and the
    largest element lies at 2^14 or above.  One token, whose logit is that element's alone, made visible by the scale."""
    P, ctx = ckv
    x = torch.cat([torch.tensor([0.0]), 2.0 ** torch.linspace(-42, -28, 113)]).to(torch.bfloat16)
    b = PackedBatch(8, [1], [x.numel()], 1, 1, 64, scale=2.0**20, qpos=[[0] * x.numel()])
    b.q[0].zero_()
    b.q[0][:, 0, 0], b.q[0][:, 0, 40] = top, x
    k = np.zeros((1, 1, 64), np.float32)
    k[..., 32:] = 16384.0
    b.set_rows(0, slice(0, 1), O.pack(k, np.ones((1, 1, 64), np.float32)))
    o, lse = b.run(P, ctx, b.device(P, max_rows=most))
    want = x.double().numpy() * 16384 * 2.0**20
    assert np.array_equal(b.want()[1][:, 0], want)
    assert np.all(np.abs(lse[:, 0] - want) <= 2.0**-39 * top * 2.0**34 + 2.0**-22 * want + 2.0**-22) and np.all(o == 1)
