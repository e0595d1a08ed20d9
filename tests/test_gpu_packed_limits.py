"""Packing at the edges of its definition: groups at the largest elements, and what rounds to zero."""
import numpy as np
import pytest
import torch

from oracle import packed as O
from tests.serving_util import TYPES

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ckv():
    import paper_2608_07855_amd as P
    ctx = P.Context(0)
    yield P, ctx
    ctx.close()


def _packed(ckv, k, v):
    P, ctx = ckv
    n, hkv, d = k.shape
    pool = torch.zeros((hkv, n, O.row_bytes(d)), dtype=torch.uint8, device="cuda")
    P.ckv_pack_tokens(ctx, k.cuda(), v.cuda(), torch.arange(n, dtype=torch.int32, device="cuda"), pool)
    ctx.sync()
    return pool.cpu().numpy().transpose(1, 0, 2)


@pytest.mark.parametrize("type", ["bf16", "fp16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("spread", [8, 50, 300, 2000, 20000])
def test_groups_at_the_largest_elements(ckv, spread, d, type):
    """Elements on both sides of +-16384: those past it count as it, to the bit.  (There b is rounded by up to 8, more
    than a step of a narrow group, so an element's own place decides its code.)"""
    rng = np.random.default_rng(spread + d)
    n = 2000
    side = rng.choice([-16384.0, 16384.0], (2, n, 1, d // 32, 1))
    x = (side + spread * rng.uniform(-1, 1, (2, n, 1, d // 32, 32))).astype(np.float32)
    k, v = (torch.from_numpy(y.reshape(n, 1, d)).to(TYPES[type]) for y in x)
    if spread > 128:                      # (16384 and its next bf16 neighbours are 64 and 128 apart)
        assert float(k.abs().max()) > 16384
    got, want = _packed(ckv, k, v), O.pack(k.float().numpy(), v.float().numpy())
    assert np.array_equal(got, want), f"{(got != want).any((1, 2)).sum()} of {n} rows differ"
    # one past the limit among ordinary ones, the type's largest, and all of a group past it
    k, v = torch.ones((4, 1, d)).to(TYPES[type]), torch.ones((4, 1, d)).to(TYPES[type])
    k[0, 0, 3], v[0, 0, 40], k[1], v[1] = 16400, -60000, 16400, -16400
    k[2, 0, ::2], v[2, 0, 1::2], v[3] = torch.finfo(TYPES[type]).max, torch.finfo(TYPES[type]).min, 50000
    assert np.array_equal(_packed(ckv, k, v), O.pack(k.float().numpy(), v.float().numpy()))


@pytest.mark.parametrize("d", [64, 128])
def test_a_zero_base_has_no_sign(ckv, d):
    """Groups of -0, and of tiny negative numbers whose base rounds to zero, hold +0 (all bytes 0)."""
    k = torch.tensor([-0.0, -1e-8, -2.0**-25, -1e-30], dtype=torch.bfloat16).view(4, 1, 1).expand(4, 1, d).contiguous()
    v = k.clone()
    v[:, :, ::3] = 0.0                    # both zeros in a group
    got = _packed(ckv, k, v)
    assert np.array_equal(got, O.pack(k.float().numpy(), v.float().numpy())) and not got.any()


def test_a_row_named_twice(ckv):
    """Every 32-bit word of such a row is one of its tokens'; rows named once and rows not named are as ever."""
    P, ctx = ckv
    rng = np.random.default_rng(12)
    n, hkv, d = 3000, 2, 128
    k, v = (torch.from_numpy(rng.standard_normal((n, hkv, d), dtype=np.float32)).to(torch.bfloat16) for _ in range(2))
    row = np.arange(n, dtype=np.int32)
    row[1:1000:2], row[2999] = row[0:999:2], 1500       # neighbours, and tokens of workgroups far apart
    pool = torch.full((hkv, n, O.row_bytes(d)), 0xA5, dtype=torch.uint8, device="cuda")
    P.ckv_pack_tokens(ctx, k.cuda(), v.cuda(), torch.from_numpy(row).cuda(), pool)
    ctx.sync()
    got = pool.cpu().numpy().transpose(1, 0, 2).copy().view("<u4")
    each = O.pack(k.float().numpy(), v.float().numpy()).view("<u4")
    for r in range(n):
        who = np.flatnonzero(row == r)
        if len(who) == 0:
            assert np.all(got[r] == 0xA5A5A5A5)
        else:
            assert np.all((got[r][None] == each[who]).any(0)), r
