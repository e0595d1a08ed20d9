"""Tokens quantised into packed rows and read back (ckv_pack_tokens, ckv_unpack_tokens): bytes and values are the
oracle's, bit for bit."""
import numpy as np
import pytest
import torch

from oracle import packed as O
from tests.serving_util import TYPES

pytestmark = pytest.mark.gpu
KEEP = 0xA5


@pytest.fixture(scope="module")
def ckv():
    import paper_2608_07855_amd as P
    ctx = P.Context(0)
    yield P, ctx
    ctx.close()


def _tokens(rng, n, hkv, d, type):
    """Keys and values over many scales: groups of 1e-7 to 1e4, constant ones, ones far from zero, borders."""
    x = rng.standard_normal((2, n, hkv, d // 32, 32)).astype(np.float32)
    x *= np.float32(10.0) ** rng.integers(-7, 5, x.shape[:-1] + (1,)).astype(np.float32) ** (rng.random(x.shape[:-1] + (1,)) < 0.5)
    x += (rng.random(x.shape[:-1] + (1,)) < 0.2) * rng.standard_normal(x.shape[:-1] + (1,)).astype(np.float32) * 10
    x[rng.random(x.shape[:-1]) < 0.05] = 3.5
    steps = rng.integers(0, 31, x.shape) / 2.0 * 0.25             # on codes and half way between two
    on = rng.random(x.shape[:-1]) < 0.2
    x[on] = steps[on].astype(np.float32)
    x = np.clip(x, -6e4, 6e4)
    k, v = (torch.from_numpy(y.reshape(n, hkv, d)).to(TYPES[type]) for y in x)
    return k, v


def _dev(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


def _want_pool(pool, k, v, row, live):
    want, row = pool.copy(), np.asarray(row)[:live]
    rows = O.pack(k[:live].float().numpy(), v[:live].float().numpy())
    there = (row >= 0) & (row < want.shape[1])
    want[:, row[there]] = rows[there].transpose(1, 0, 2)
    return want


@pytest.mark.parametrize("type", ["bf16", "fp16"])
@pytest.mark.parametrize("hkv,d", [(1, 64), (8, 64), (3, 128), (8, 128)])
@pytest.mark.parametrize("n", [1, 2, 7, 33, 300])
def test_bytes(ckv, n, hkv, d, type):
    P, ctx = ckv
    rng = np.random.default_rng(n * 1000 + d + hkv)
    k, v = _tokens(rng, n, hkv, d, type)
    pool = np.full((hkv, n + 9, O.row_bytes(d)), KEEP, np.uint8)
    row = rng.permutation(n + 9)[:n]
    dev = torch.from_numpy(pool).cuda()
    P.ckv_pack_tokens(ctx, k.cuda(), v.cuda(), _dev(row), dev)
    ctx.sync()
    assert np.array_equal(dev.cpu().numpy(), _want_pool(pool, k, v, row, n))


@pytest.mark.parametrize("type", ["bf16", "fp16"])
@pytest.mark.parametrize("d", [64, 128])
def test_every_number_of_a_group(ckv, d, type):
    """Groups with every exponent of the type as their scale, and their smallest steps apart."""
    P, ctx = ckv
    rng = np.random.default_rng(3)
    n = 600
    e = rng.uniform(-26, 16, (2, n, 1, d // 32, 1))
    x = (rng.standard_normal((2, n, 1, d // 32, 32)) * 2.0**e + (rng.random(e.shape) < 0.5) * 2.0**rng.uniform(-10, 13, e.shape))
    k, v = (torch.from_numpy(np.clip(y, -6e4, 6e4).astype(np.float32).reshape(n, 1, d)).to(TYPES[type]) for y in x)
    pool = torch.zeros((1, n, O.row_bytes(d)), dtype=torch.uint8, device="cuda")
    P.ckv_pack_tokens(ctx, k.cuda(), v.cuda(), _dev(np.arange(n)), pool)
    ctx.sync()
    want = O.pack(k.float().numpy(), v.float().numpy())[:, 0]
    got = pool[0].cpu().numpy()
    assert np.array_equal(got, want), f"{(got != want).any(1).sum()} rows differ"


def test_rows_outside_and_dead_tokens(ckv):
    """Rows outside the pool and tokens from n_live on write nothing; counts are clamped."""
    P, ctx = ckv
    rng = np.random.default_rng(5)
    n, hkv, d = 40, 2, 64
    k, v = _tokens(rng, n, hkv, d, "bf16")
    row = rng.permutation(n).astype(np.int64)
    row[[3, 8, 20, 30]] = [-1, n, 2**31 - 1, -2**31]
    for live in (-5, 0, 1, 17, n, n + 1, 2**31 - 1):
        pool = np.full((hkv, n, O.row_bytes(d)), KEEP, np.uint8)
        big = torch.from_numpy(np.pad(pool, ((0, 0), (2, 3), (0, 0)), constant_values=KEEP)).cuda()
        P.ckv_pack_tokens(ctx, k.cuda(), v.cuda(), _dev(row), big[:, 2:n + 2], n_live=_dev([live]))
        ctx.sync()
        got = big.cpu().numpy()
        assert np.array_equal(got[:, 2:n + 2], _want_pool(pool, k, v, row, min(max(live, 0), n))), live
        assert np.all(got[:, :2] == KEEP) and np.all(got[:, n + 2:] == KEEP)


@pytest.mark.parametrize("type", ["bf16", "fp16"])
def test_strides(ckv, type):
    """Tokens inside a projection's rows, pools that are token-major or padded."""
    P, ctx = ckv
    rng = np.random.default_rng(6)
    n, hkv, d = 21, 4, 128
    k, v = _tokens(rng, n, hkv, d, type)
    qkv = torch.full((n, 6 + 2 * hkv, d), float("nan"), dtype=TYPES[type], device="cuda")
    qkv[:, 6:6 + hkv], qkv[:, 6 + hkv:] = k.cuda(), v.cuda()
    row = rng.permutation(n)
    want = _want_pool(np.zeros((hkv, n, O.row_bytes(d)), np.uint8), k, v, row, n)
    for shape, view in (((n, hkv, 160), lambda x: x.transpose(0, 1)), ((hkv, n, 256), lambda x: x[..., 32:192]),
                        ((hkv, 2 * n, 160), lambda x: x[:, ::2])):
        store = torch.full(shape, KEEP, dtype=torch.uint8, device="cuda")
        P.ckv_pack_tokens(ctx, qkv[:, 6:6 + hkv], qkv[:, 6 + hkv:], _dev(row), view(store))
        ctx.sync()
        assert np.array_equal(view(store).cpu().numpy(), want)
        assert (store == KEEP).sum() >= store.numel() - want.size
        # and back, into rows that alternate between keys and values
        out = torch.full((1, hkv, n, 2, d), 9.0, dtype=TYPES[type], device="cuda")
        P.ckv_unpack_tokens(ctx, P.packed_view(view(store), _dev([n]), slot=_dev(row[None])), k=out[:, :, :, 0], v=out[:, :, :, 1])
        ctx.sync()
        for i, x in enumerate(O.unpack(want[:, row])):
            assert torch.equal(out[0, :, :, i].cpu(), torch.from_numpy(x).to(TYPES[type]))


@pytest.mark.parametrize("type", ["bf16", "fp16"])
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("hkv,d", [(1, 64), (3, 128)])
def test_read_back(ckv, hkv, d, paged, type):
    """Values that rows stand for, ragged, rows past the last token as they were."""
    P, ctx = ckv
    rng = np.random.default_rng(7)
    lens = np.array([5, 0, 77, 1, 40])
    most = 80
    rows = [O.pack(*(x.float().numpy() for x in _tokens(rng, t, hkv, d, "fp16"))) for t in lens]
    if paged:
        place, at = rng.permutation(lens.sum() + 4), 0
        pool = np.full((hkv, lens.sum() + 4, O.row_bytes(d)), 0xFF, np.uint8)
        slot = np.full((5, most), -3, np.int32)
        for s, t in enumerate(lens):
            pool[:, place[at:at + t]] = rows[s].transpose(1, 0, 2)
            slot[s, :t] = place[at:at + t]
            at += t
        slot = _dev(slot)
    else:
        pool, slot = np.full((5, hkv, most, O.row_bytes(d)), 0xFF, np.uint8), None
        for s, t in enumerate(lens):
            pool[s, :, :t] = rows[s].transpose(1, 0, 2)
    kv = P.packed_view(torch.from_numpy(pool).cuda(), _dev(lens), slot=slot)
    out = P.ckv_unpack_tokens(ctx, kv, k=torch.full((5, hkv, most, d), 9.0, dtype=TYPES[type], device="cuda"),
                              v=torch.full((5, hkv, most, d), 9.0, dtype=TYPES[type], device="cuda"))
    ctx.sync()
    for s, t in enumerate(lens):
        for name, x in zip("kv", O.unpack(rows[s])):
            want = torch.from_numpy(x).to(torch.float16).to(TYPES[type]).transpose(0, 1)
            assert torch.equal(out[name][s, :, :t].cpu(), want) and torch.all(out[name][s, :, t:] == 9)


def test_read_back_clamps(ckv):
    """Lengths past max_tokens and negative ones, slots outside the pool."""
    P, ctx = ckv
    rng = np.random.default_rng(8)
    rows = O.pack(*(x.float().numpy() for x in _tokens(rng, 9, 1, 64, "bf16")))
    pool = torch.from_numpy(rows.transpose(1, 0, 2).copy()).cuda()
    slot = _dev([[0, -1, 9, 2**31 - 1], [1, 2, 3, 4], [5, 6, 7, 8]])
    out = P.ckv_unpack_tokens(ctx, P.packed_view(pool, _dev([4, -2, 2**31 - 1]), slot=slot), dtype=torch.float16)
    ctx.sync()
    k = O.unpack(rows)[0][:, 0].astype(np.float16)
    got = out["k"][:, 0].cpu().numpy()
    assert np.array_equal(got[0], k[[0, 8, 8, 8]]) and not got[1].any() and np.array_equal(got[2], k[[5, 6, 7, 8]])


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_non_finite_groups(ckv, bad):
    """One element spoils its group of 32, nothing else; reading back tells."""
    P, ctx = ckv
    k, v = torch.ones((3, 2, 128), dtype=torch.bfloat16), torch.ones((3, 2, 128), dtype=torch.bfloat16)
    k[1, 0, 70], v[2, 1, 0] = bad, bad
    pool = torch.zeros((2, 3, 160), dtype=torch.uint8, device="cuda")
    P.ckv_pack_tokens(ctx, k.cuda(), v.cuda(), _dev([0, 1, 2]), pool)
    out = P.ckv_unpack_tokens(ctx, P.packed_view(pool, _dev([3]), slot=_dev([[0, 1, 2]])))
    ctx.sync()
    for name, s, g, at in (("k", 1, 0, 64), ("v", 2, 1, 0)):
        x = out[name][0].transpose(0, 1).cpu().float()
        assert torch.all(torch.isnan(x[s, g, at:at + 32]))
        x[s, g, at:at + 32] = 1
        assert torch.all(x == 1)
    assert np.array_equal(pool.cpu().numpy().transpose(1, 0, 2), O.pack(k.float().numpy(), v.float().numpy()))


def test_capture(ckv):
    """A captured step packs whatever count and tokens it finds, into the rows it finds."""
    P, _ = ckv
    stream = torch.cuda.Stream()
    rng = np.random.default_rng(9)
    with torch.cuda.stream(stream):
        ctx = P.Context(0, stream)
        n, hkv, d = 50, 2, 128
        k, v = (torch.zeros((n, hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        row, live = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        pool = torch.zeros((hkv, 64, 160), dtype=torch.uint8, device="cuda")
        out = [torch.zeros((1, hkv, n, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        kv = P.packed_view(pool, live, slot=row[None])

        def step():
            P.ckv_pack_tokens(ctx, k, v, row, pool, n_live=live)
            P.ckv_unpack_tokens(ctx, kv, k=out[0], v=out[1])
        step()
        stream.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            step()
        for count in (50, 3, 0, 31):
            hk, hv = _tokens(rng, n, hkv, d, "bf16")
            place = rng.permutation(64)[:n]
            k.copy_(hk), v.copy_(hv), row.copy_(torch.from_numpy(place.astype(np.int32))), live.fill_(count)
            before = pool.cpu().numpy()
            for x in out:
                x.fill_(5)
            g.replay()
            stream.synchronize()
            want = _want_pool(before, hk, hv, place, count)
            assert np.array_equal(pool.cpu().numpy(), want)
            for x, y in zip(out, O.unpack(want[:, place[:count]])):
                assert torch.equal(x[0, :, :count].cpu(), torch.from_numpy(y).to(torch.bfloat16)) and torch.all(x[0, :, count:] == 5)
        ctx.close()


def test_rows_past_4_gib(ckv):
    """Rows whose byte offset passes 32 bits, written, read back and attended to."""
    P, ctx = ckv
    rows = (1 << 32) // 160 + 1000
    pool = torch.zeros((1, rows, 160), dtype=torch.uint8, device="cuda")
    k, v = _tokens(np.random.default_rng(10), 4, 1, 128, "bf16")
    at = [rows - 1, 5, rows - 700, (1 << 31) // 160 + 7]
    P.ckv_pack_tokens(ctx, k.cuda(), v.cuda(), _dev(at), pool)
    kv = P.packed_view(pool, _dev([4]), slot=_dev([at]))
    out = P.ckv_unpack_tokens(ctx, kv)
    ctx.sync()
    want = O.unpack(O.pack(k.float().numpy(), v.float().numpy()))
    for name, x in zip("kv", want):
        assert torch.equal(out[name][0, 0].cpu(), torch.from_numpy(x[:, 0]).to(torch.bfloat16))
    # zero queries weight all tokens alike
    q = P.query_view(torch.zeros((1, 2, 128), dtype=torch.bfloat16, device="cuda"), _dev([0, 1]))
    o = P.ckv_attend_packed(ctx, kv, q)["o"]
    ctx.sync()
    mean = want[1][:, 0].mean(0)
    assert np.all(np.abs(o[0, 1].cpu().double().numpy() - mean) <= 2.0**-8 * np.abs(mean) + 2.0**-11 * np.abs(want[1][:, 0]).mean(0) + 1e-6)


def test_nothing_to_do(ckv):
    """No tokens, no sequences, no room."""
    P, ctx = ckv
    none = torch.zeros((0, 2, 64), dtype=torch.bfloat16, device="cuda")
    pool = torch.full((2, 5, 80), KEEP, dtype=torch.uint8, device="cuda")
    P.ckv_pack_tokens(ctx, none, none, _dev([]), pool)
    some = torch.zeros((1, 2, 64), dtype=torch.bfloat16, device="cuda")
    P.ckv_pack_tokens(ctx, some, some, _dev([0]), pool[:, :0])
    assert P.ckv_unpack_tokens(ctx, P.packed_view(pool, _dev([]), slot=_dev(np.zeros((0, 4)))))["k"].shape == (0, 2, 4, 64)
    assert P.ckv_unpack_tokens(ctx, P.packed_view(pool, _dev([3]), slot=_dev(np.zeros((1, 0)))))["k"].shape == (1, 2, 0, 64)
    ctx.sync()
    assert torch.all(pool == KEEP)


def test_refusals(ckv):
    P, ctx = ckv
    pool = torch.full((2, 8, 80), KEEP, dtype=torch.uint8, device="cuda")
    k, v = (torch.ones((3, 2, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    row, lens, slot = _dev([0, 1, 2]), _dev([3]), _dev([[0, 1, 2]])
    for call in (lambda: P.ckv_pack_tokens(ctx, k.float(), v.float(), row, pool), lambda: P.ckv_pack_tokens(ctx, k, v[:, :, ::2], row, pool),
                 lambda: P.ckv_pack_tokens(ctx, k, v, row.long(), pool), lambda: P.ckv_pack_tokens(ctx, k, v, row[:2], pool),
                 lambda: P.ckv_pack_tokens(ctx, k, v, row, pool[:1]), lambda: P.ckv_pack_tokens(ctx, k, v, row, pool[..., :64]),
                 lambda: P.ckv_pack_tokens(ctx, k, v, row, pool.view(torch.int8)), lambda: P.ckv_pack_tokens(ctx, k.cpu(), v.cpu(), row, pool),
                 lambda: P.ckv_pack_tokens(ctx, k, v, row, pool, n_live=lens.long()), lambda: P.packed_view(pool, lens),
                 lambda: P.packed_view(pool, lens, slot=slot.long()), lambda: P.packed_view(pool, lens, slot=_dev([[0], [1]])),
                 lambda: P.packed_view(pool, lens, slot=slot, max_tokens=4), lambda: P.packed_view(pool, lens, slot=slot.cpu()),
                 lambda: P.ckv_unpack_tokens(ctx, P.packed_view(pool, lens, slot=slot), k=k),
                 lambda: P.ckv_unpack_tokens(ctx, P.packed_view(pool, lens, slot=slot), dtype=torch.float32),
                 lambda: P.ckv_unpack_tokens(ctx, P.packed_view(pool, lens, slot=slot), k=k[None], v=v[None])):
        with pytest.raises(ValueError):
            call()

    def code(fn, *a, **kw):
        with pytest.raises(P.CKVError) as e:
            fn(ctx, *a, **kw)
        return e.value.code
    # strides and addresses that are no multiples of 16 bytes (8 elements)
    odd = torch.zeros((2, 8, 88), dtype=torch.uint8, device="cuda")
    assert code(P.ckv_pack_tokens, k, v, row, odd[..., :80]) == -1
    assert code(P.ckv_pack_tokens, k, v, row, odd.view(-1)[8:1288].view(2, 8, 80)) == -1
    kk = torch.ones((3, 2, 68), dtype=torch.bfloat16, device="cuda")[..., :64]
    assert code(P.ckv_pack_tokens, kk, kk, row, pool) == -1
    # heads on each other
    assert code(P.ckv_pack_tokens, k, v, row, pool.as_strided((2, 8, 80), (80, 80, 1))) == -2
    # the pool over its tokens
    both = torch.zeros(4096, dtype=torch.uint8, device="cuda")
    inside = both[:768].view(torch.bfloat16).view(3, 2, 64)
    assert code(P.ckv_pack_tokens, inside, v, row, both[640:1920].view(2, 8, 80)) == -1
    assert code(P.ckv_pack_tokens, k, inside, row, both[640:1920].view(2, 8, 80)) == -1
    kv = P.packed_view(both[640:1920].view(2, 8, 80), lens, slot=slot)
    out = [torch.zeros((1, 2, 3, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    assert code(P.ckv_unpack_tokens, kv, k=inside.view(1, 2, 3, 64), v=out[0]) == -1
    assert code(P.ckv_unpack_tokens, kv, k=out[0], v=out[0]) == -1
    assert code(P.ckv_unpack_tokens, kv, k=out[0].expand(1, 2, 3, 64)[:, :1].expand(1, 2, 3, 64), v=out[1][:, :1].expand(1, 2, 3, 64)) == -2
    for field, value, want in [("head_dim", 96, -2), ("n_kv_heads", 0, -2), ("row_stride", 64, -2), ("row_stride", 84, -1),
                               ("pool_rows", 0, -2), ("n_tokens", None, -1), ("data", None, -1), ("data", pool.data_ptr() + 8, -1),
                               ("max_tokens", -1, -2), ("n_seq", -1, -2), ("head_stride", -16, -2)]:
        bad = type(kv).from_buffer_copy(kv)
        bad.__dict__.update(kv.__dict__)
        setattr(bad, field, value)
        if field in ("n_seq", "max_tokens", "n_kv_heads", "head_dim"):
            rc = ctx._lib.ckv_unpack_tokens(ctx.handle, bad, P.binding.KVRows(out[0].data_ptr(), out[1].data_ptr(), 384, 192, 64, 0))
            assert rc == want, field
        else:
            assert code(P.ckv_unpack_tokens, bad, k=out[0], v=out[1]) == want, field
    ctx.sync()
    assert torch.all(pool == KEEP) and not any(x.any() for x in out)


@pytest.mark.parametrize("d", [64, 128])
def test_more_than_a_launch_of_items(ckv, d):
    """More (sequence, head) pairs and tiles of tokens than workgroups; far more room than tokens."""
    P, ctx = ckv
    rng = np.random.default_rng(11)
    n, hkv = 9001, 64                                # 9001 sequences of 64 heads, up to 2 tokens each
    lens = rng.integers(0, 3, n)
    rows = int(lens.sum())
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randn((rows, hkv, d), generator=g).to(torch.bfloat16) for _ in range(2))
    pool = torch.zeros((hkv, rows, O.row_bytes(d)), dtype=torch.uint8, device="cuda")
    P.ckv_pack_tokens(ctx, k.cuda(), v.cuda(), _dev(np.arange(rows)), pool)
    slot = np.zeros((n, 40), np.int64)
    first = np.cumsum(lens) - lens
    slot[:, 0], slot[:, 1] = first, first + 1
    out = P.ckv_unpack_tokens(ctx, P.packed_view(pool, _dev(lens), slot=_dev(slot)),
                              k=torch.full((n, hkv, 40, d), 9.0, dtype=torch.bfloat16, device="cuda"),
                              v=torch.full((n, hkv, 40, d), 9.0, dtype=torch.bfloat16, device="cuda"))
    ctx.sync()
    some = rng.choice(rows, 200, replace=False)
    assert np.array_equal(pool[:, torch.from_numpy(some).cuda()].cpu().numpy().transpose(1, 0, 2),
                          O.pack(k[some].float().numpy(), v[some].float().numpy()))
    seq = np.repeat(np.arange(n), lens)
    want = O.unpack(pool.cpu().numpy())
    for name, x in zip("kv", want):
        got = out[name][torch.from_numpy(seq).cuda(), :, torch.from_numpy(np.arange(rows) - first[seq]).cuda()].cpu()
        assert torch.equal(got, torch.from_numpy(x).to(torch.bfloat16).transpose(0, 1))
        assert torch.all(out[name][:, :, 2:] == 9) and torch.all(out[name][torch.from_numpy(lens == 0).cuda()] == 9)
