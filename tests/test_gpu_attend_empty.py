"""Attention calls over views that hold nothing: no sequence, or no room for a token."""
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


def _i32(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _without_room(P, n, hkv=2, d=64, paged=False):
    k = torch.zeros((hkv, 5, d) if paged else (n, hkv, 0, d), dtype=torch.bfloat16, device="cuda")
    table = torch.zeros((n, 0), dtype=torch.int32, device="cuda")
    return P.batch_view(k, k.clone(), torch.zeros(n, dtype=torch.int32, device="cuda"), slot=table if paged else None)


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("rows", [0, 3])
def test_no_sequences(ckv, rows, paged):
    """Nothing to do: rows of no sequence stay as they were."""
    P, ctx = ckv
    pre = Batch(1, [4], [1], 4, 2, 64, prefix=20).device(P)["prefix"]
    kv = _without_room(P, 0, paged=paged)
    q = P.query_view(torch.zeros((rows, 4, 64), dtype=torch.bfloat16, device="cuda"), _i32(0))
    for most in (1, 100):
        q.max_rows = most
        for call in (lambda **kw: P.ckv_attend_window(ctx, kv, q, **kw), lambda **kw: P.ckv_attend_shared(ctx, pre, kv, q, **kw)):
            o = torch.full((rows, 4, 64), 7, dtype=torch.bfloat16, device="cuda")
            lse = torch.full((rows, 4), 7, dtype=torch.float32, device="cuda")
            call(o=o, lse=lse)
            ctx.sync()
            assert torch.all(o == 7) and torch.all(lse == 7)


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("rows", [1, 40])
def test_no_room_for_tokens(ckv, rows, paged):
    """Sequences that can hold no token: a row sees nothing, or the shared tokens alone.  Shared tokens that hold nothing
    leave a sequence its own."""
    P, ctx = ckv
    b = Batch(2, [0, 0], [rows, 1], 4, 2, 64, prefix=90, qpos=[[89] * rows, [30]])
    v = b.device(P)
    v["kv"] = _without_room(P, 2, paged=paged)
    check(b, b.run(P, ctx, v), b.want(), "shared tokens alone")
    o, lse = torch.full((rows + 1, 4, 64), 7, dtype=torch.bfloat16, device="cuda"), torch.zeros((rows + 1, 4), device="cuda")
    P.ckv_attend_window(ctx, v["kv"], v["q"], window=5, n_sink=2, o=o, lse=lse)
    ctx.sync()
    assert torch.all(o == 0) and torch.all(lse == -float("inf"))
    b = Batch(3, [70, 9], [rows, 1], 4, 2, 64, paged=paged)
    v = b.device(P)
    o, lse = torch.zeros_like(o), torch.zeros_like(lse)
    P.ckv_attend_shared(ctx, _without_room(P, 1, paged=paged), v["kv"], v["q"], o=o, lse=lse)
    ctx.sync()
    check(b, (o.cpu().double().numpy(), lse.cpu().double().numpy()), b.want(), "nothing shared")
