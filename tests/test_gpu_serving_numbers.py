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
