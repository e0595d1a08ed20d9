"""What the attention calls hold of a context's memory: growth, limits, captured calls."""
import pytest
import torch

from tests.serving_util import Batch, check

pytestmark = pytest.mark.gpu

LIMIT = 6 << 20


@pytest.mark.parametrize("captured", [False, True])
def test_growth_leaves_room_under_a_limit(captured):
    """Two attention calls, the second a little larger, need 2.2 MB each; a measurement of 1.4 MB finds its room under a
    limit of 6 MiB, also where a captured call keeps the first one's memory."""
    import paper_2608_07855_amd as P
    from tests.test_gpu_batch import WANT, _problem
    one = _problem(P, 16, 8, 64, 4096, 8, 16, False, seed=3)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = P.Context(0, stream)
        ctx.set_workspace_limit(LIMIT)
        a, b = Batch(1, [9000, 100], [1, 1], 8, 2, 128), Batch(2, [9000, 100, 2000], [1, 1, 1], 8, 2, 128)
        va, vb = a.device(P), b.device(P)
        check(a, a.run(P, ctx, va), a.want(), "first")
        first = ctx.workspace_bytes()
        o = torch.zeros((2, 8, 128), dtype=torch.bfloat16, device="cuda")
        P.ckv_attend_window(ctx, va["kv"], va["q"], o=o)
        stream.synchronize()
        eager = o.clone()
        if captured:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                P.ckv_attend_window(ctx, va["kv"], va["q"], o=o)
        check(b, b.run(P, ctx, vb), b.want(), "second")
        held = ctx.workspace_bytes()
        assert first < held < (2.5 if captured else 1.5) * first
        P.ckv_measure_page_effects(ctx, *one[:3], want=WANT)
        ctx.sync()
        assert held < ctx.workspace_bytes() <= LIMIT
        for _ in range(3 if captured else 0):
            o.zero_()
            g.replay()
            stream.synchronize()
            assert torch.equal(o, eager)
            check(b, b.run(P, ctx, vb), b.want(), "between replays")
        ctx.close()


def test_growth_without_captures_holds_one_workspace():
    """What no capture refers to is given back when it is outgrown."""
    import paper_2608_07855_amd as P
    ctx = P.Context(0)
    sizes = []
    for n in (1, 2, 8, 24):
        b = Batch(n, [3000] * n, [1] * n, 8, 2, 128)
        check(b, b.run(P, ctx, b.device(P)), b.want(), f"{n} sequences")
        sizes.append(ctx.workspace_bytes())
    # growth doubles: never more than twice what the largest call needs
    fresh = P.Context(0)
    b.run(P, fresh, b.device(P))
    assert sizes == sorted(sizes) and sizes[-1] <= 2 * fresh.workspace_bytes()
    fresh.close()
    ctx.close()
