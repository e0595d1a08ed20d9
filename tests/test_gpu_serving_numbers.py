"""Numbers that the C structs of the serving calls cannot hold: refused, not cut to 32 bits."""
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


@pytest.mark.parametrize("far", [2**31, 2**32 + 5, 2**33 + 100, -2**32 + 5])
def test_numbers_past_32_bits(ckv, far):
    """2^32 + 5 is no window of 5 positions."""
    P, ctx = ckv
    b = Batch(1, [200, 30], [1, 2], 4, 2, 64)
    v = b.device(P)
    o = torch.full((3, 4, 64), 7, dtype=torch.bfloat16, device="cuda")
    q, cu, _ = v["q"]._keep
    i = torch.zeros(8, dtype=torch.int32, device="cuda")
    for call in (lambda: P.ckv_attend_window(ctx, v["kv"], v["q"], window=far, o=o),
                 lambda: P.ckv_attend_window(ctx, v["kv"], v["q"], window=4, n_sink=far, o=o),
                 lambda: P.query_view(q, cu, max_rows=far),
                 lambda: P.slot_step(i[:1], i[1:2], i[2:4], i[4:5], i[6:8].view(1, 2), block_size=far),
                 lambda: P.slot_step(i[:1], i[1:2], i[2:4], i[4:5], i[6:8].view(1, 2), block_size=1, max_new=far)):
        with pytest.raises(ValueError):
            call()
    ctx.sync()
    assert torch.all(o == 7)


def test_the_largest_window(ckv):
    """2^31 - 1 hides nothing."""
    P, ctx = ckv
    b = Batch(2, [300, 30], [1, 20], 4, 2, 64, gaps=True)
    check(b, b.run(P, ctx, b.device(P), 2**31 - 1, 2**31 - 1), b.want(), "largest")
    check(b, b.run(P, ctx, b.device(P), 2**31 - 1, 0), b.want(), "largest, no first tokens")


def test_tables_past_32_bits(ckv):
    """A table of 2^32 + 8 slots is none of 8; its first ones are there for who asks for them."""
    P, ctx = ckv
    far = 2**32 + 8
    slot = torch.empty((1, far), dtype=torch.int32, device="cuda")
    slot[0, :20] = torch.arange(20, device="cuda")
    lens = torch.tensor([20], dtype=torch.int32, device="cuda")
    pool, k = torch.zeros((2, 20, 80), dtype=torch.uint8, device="cuda"), torch.ones((2, 20, 64), dtype=torch.bfloat16, device="cuda")
    q, cu = torch.ones((1, 4, 64), dtype=torch.bfloat16, device="cuda"), torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    for call in (lambda: P.packed_view(pool, lens, slot=slot), lambda: P.packed_view(pool, lens, slot=slot, max_tokens=far),
                 lambda: P.batch_view(k, k, lens, slot=slot), lambda: P.packed_view(pool[:1].expand(far, 20, 80), lens, slot=slot[:, :20]),
                 lambda: P.batch_view(k[:1].expand(far, 20, 64), k[:1].expand(far, 20, 64), lens, slot=slot[:, :20]),
                 lambda: P.query_view(q[:, :1].expand(1, far, 64), cu), lambda: P.query_view(q.expand(far, 4, 64), cu),
                 lambda: P.kv_view(k, k, slot[0], slot=slot[0])):
        with pytest.raises(ValueError):
            call()
    view = P.query_view(q, cu)
    o = P.ckv_attend_packed(ctx, P.packed_view(pool, lens, slot=slot, max_tokens=20), view)["o"]
    p = P.ckv_attend_window(ctx, P.batch_view(k, k, lens, slot=slot, max_tokens=20), view)["o"]
    ctx.sync()
    assert not o.any() and torch.all(p == 1)
