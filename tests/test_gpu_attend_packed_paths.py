"""ckv_attend_packed on large batches and storage: splits that are joined in a tree, many heads and sequences, rows past
4 GiB in both kernels, unequal splits of many-rows blocks, one row's queries beside others'."""
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


@pytest.mark.parametrize("tokens", [8192, 13057, 13089, 40000, 66001])
@pytest.mark.parametrize("type,d", [("bf16", 128), ("fp16", 64)])
def test_one_long_cache(ckv, tokens, type, d):
    """Up to 87 splits of one block: 16 and fewer, a last group of one, several groups."""
    _run(ckv, PackedBatch(1, [tokens], [1], 4, 1, d, type), what=f"{tokens}")


@pytest.mark.parametrize("n", [9, 33, 70, 300])
def test_many_sequences_in_splits(ckv, n):
    """Ragged lengths with a few long ones, below and above 64 sequences and a row block a compute unit."""
    rng = np.random.default_rng(n)
    lens = rng.integers(1, 400, n)
    lens[:: max(1, n // 4)] = 9000 if n < 100 else 5000
    _run(ckv, PackedBatch(2, lens, [1] * n, 4, 2, 64), what=f"{n} sequences")


def test_many_heads(ckv):
    b = PackedBatch(3, [300, 40, 7], [1, 1, 2], 192, 96, 64)
    _run(ckv, b, what="96 heads")
    b = PackedBatch(3, [60, 90], [40, 9], 80, 40, 64)
    _run(ckv, b, 30, 2, what="40 heads, chunks")


@pytest.mark.parametrize("guess", [1, 4, 400])
def test_rows_that_differ_by_much(ckv, guess):
    """One prompt among single tokens, whatever the estimate."""
    b = PackedBatch(4, [700, 40, 3000, 1, 90], [300, 1, 1, 1, 5], 8, 2, 128)
    _run(ckv, b, max_rows=guess, what=f"estimate {guess}")
    _run(ckv, b, 200, 5, max_rows=guess, what=f"estimate {guess}, window")


@pytest.mark.parametrize("type", ["bf16", "fp16"])
def test_blocks_in_several_shares(ckv, type):
    """Many rows behind long caches: blocks fall into shares, partial sums are joined."""
    _run(ckv, PackedBatch(5, [5000, 900, 2600], [130, 257, 64], 2, 1, 64, type), what="shares")
    _run(ckv, PackedBatch(5, [3000, 700], [70, 150], 4, 1, 128, type, paged=False), 900, 7, what="shares, window")


@pytest.mark.parametrize("rows", [1, 300])
@pytest.mark.parametrize("where", ["rows", "heads"])
def test_far_storage(ckv, rows, where):
    """Rows and heads whose byte offsets pass 32 bits."""
    P, ctx = ckv
    b = PackedBatch(6, [310, 50], [rows, 1], 4, 2, 128)
    v = b.device(P)
    pool, lens, slot, _ = v["kv"]._keep
    last = pool.shape[1] - 1
    if where == "rows":
        big = torch.full(((5 << 30) // 160, 1, 160), 0xFF, dtype=torch.uint8, device="cuda")
        # head 1 lies inside head 0's rows, 2^31 bytes and some on
        big = big.view(-1)
        gap = (1 << 31) // 160 * 160 + 160 * 1000
        far = (big.numel() - gap) // 160 - last - 2
        view = big.as_strided((2, far + last + 1, 160), (gap, 160, 1))
        table = torch.where(slot >= 0, slot + far, slot)
        for g in range(2):
            view[g, far:far + last + 1] = pool[g]
        kv = P.packed_view(view, lens, slot=table)
        # (heads on each other are fine to read)
    else:
        big = torch.full((2, (3 << 30) // 160, 160), 0xFF, dtype=torch.uint8, device="cuda")
        big[:, :last + 1] = pool
        kv = P.packed_view(big[:, :last + 1], lens, slot=slot)
    check(b, b.run(P, ctx, dict(kv=kv, q=v["q"])), b.want(), where)


def test_more_row_blocks_than_large_workgroups_in_a_launch(ckv):
    """6 million row blocks under an estimate of one row: 2^32 threads are 5.6 million workgroups of 12 waves."""
    P, ctx = ckv
    b = PackedBatch(9, [3], [3], 64, 64, 64, qpos=[[0, 1, 2]])
    v = b.device(P)
    o3, lse3 = (torch.from_numpy(x).cuda() for x in b.run(P, ctx, v))
    n = 1500000
    q = v["q"]._keep[0][:1].expand(n, 64, 64)
    qpos = (torch.arange(n, device="cuda") % 3).to(torch.int32)
    view = P.query_view(q, torch.tensor([0, n], dtype=torch.int32, device="cuda"), qpos, max_rows=1)
    got = P.ckv_attend_packed(ctx, v["kv"], view, want=("o", "lse"))
    one = P.ckv_attend_packed(ctx, v["kv"], P.query_view(q[:3], torch.tensor([0, 3], dtype=torch.int32, device="cuda"), qpos[:3]), want=("o", "lse"))
    ctx.sync()
    assert torch.equal(one["o"][0].double(), o3[0]) and torch.equal(one["lse"][0].double(), lse3[0])
    for i in range(0, n, 150000):
        assert torch.all(got["o"][i:i + 150000].view(-1, 3, 64, 64) == one["o"]) and torch.all(got["lse"][i:i + 150000].view(-1, 3, 64) == one["lse"])


def test_a_row_beside_larger_ones(ckv):
    """bf16 rows of very different size in one block: each keeps its own logits (to 2^-40 of the largest one's)."""
    for rows in (3, 40):
        b = PackedBatch(7, [200], [rows], 4, 2, 64, heavy=False)
        b.q[0][::2] *= 2.0**12                                   # logits of 4096 times the others'
        P, ctx = ckv
        o, lse = b.run(P, ctx, b.device(P))
        wo, wl, w = b.want()
        small = np.arange(rows) % 2 == 1
        c = PackedBatch(7, [200], [rows], 4, 2, 64, heavy=False)
        check(c, (o[small], lse[small]), (wo[small], wl[small], w[small]), f"{rows} rows, the small ones")
        # the large ones: one token takes all; float32 logits of 2^15 are off by 2^-9 at most
        big = ~small
        assert np.all(np.abs(lse[big] - wl[big]) <= 2.0**-22 * np.abs(wl[big]) + 2.0**-8)


def test_a_row_of_nan_stays_alone(ckv):
    """Queries that are not finite spoil their own row."""
    P, ctx = ckv
    for rows, bad in ((3, float("nan")), (40, float("inf")), (40, float("nan"))):
        b = PackedBatch(8, [90], [rows], 4, 2, 64)
        want = b.want()
        b.q[0][1, 2, 5] = bad
        v = b.device(P)
        o = torch.zeros((rows, 4, 64), dtype=torch.bfloat16, device="cuda")
        lse = torch.zeros((rows, 4), device="cuda")
        P.ckv_attend_packed(ctx, v["kv"], v["q"], o=o, lse=lse)
        with pytest.raises(P.CKVError, match="NONFINITE"):
            ctx.sync()
        o, lse = o.cpu().double().numpy().reshape(-1, 64), lse.cpu().double().numpy().reshape(-1)
        assert not np.isfinite(o[4 + 2]).any()
        pick = np.arange(rows * 4) != 4 + 2
        check(b, (o[pick][:, None], lse[pick][:, None]), tuple(x.reshape(rows * 4, 1, -1)[pick] if x.ndim == 3 else x.reshape(-1, 1)[pick] for x in want),
              "beside a bad row")


def test_struct_layouts_match_the_header():
    import ctypes

    from paper_2608_07855_amd import _abi
    assert ctypes.sizeof(_abi.PackedPool) == 8 * 3 + 4 * 3 + 4
    assert ctypes.sizeof(_abi.KVRows) == 8 * 5 + 4 + 4
    assert ctypes.sizeof(_abi.PackedView) == 8 * 9 + 4 * 5 + 4
