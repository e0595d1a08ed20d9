"""Block and slot tables of more sequences than the kernel keeps sums for (2048), in groups of 2 and more, the last of
them not full: equal to the step-by-step oracle in every word."""
import numpy as np
import pytest

from tests.test_gpu_slots import Pool

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ckv():
    import paper_2608_07855_amd as P
    ctx = P.Context(0)
    yield P, ctx
    ctx.close()


@pytest.mark.parametrize("block", [1, 3, 16])
@pytest.mark.parametrize("n,width", [(2048, 40), (2049, 40), (5000, 40), (70001, 7)])
def test_many_sequences(ckv, n, width, block):
    """Prompts, then a step with sequences that end, go on and stay, then single tokens."""
    P, ctx = ckv
    p = Pool(n + block, n, block, n * -(-width // block) + 9, width)
    for new in (p.rng.integers(0, width // 2, n),
                np.where(p.rng.random(n) < 0.4, -1, p.rng.integers(0, 3, n)),
                np.ones(n, np.int64)):
        r = p.step(P, ctx, new, next_pos=p.rng.integers(0, 1 << 30, n))
        assert r["status"] == 0
        p.take(r)


def test_refused_steps_of_many_sequences(ckv):
    """Reasons that single sequences give, the last one among them, and a shortage over all of them."""
    P, ctx = ckv
    n = 5000
    p = Pool(1, n, 3, 4 * n, 10)
    p.take(p.step(P, ctx, p.rng.integers(0, 8, n)))
    one = np.ones(n, np.int64)
    for at, what, status in ((n - 1, -2, 4), (2500, 11, 2), (0, -7, 4)):
        new = one.copy()
        new[at] = what
        assert p.step(P, ctx, new)["status"] == status
    assert p.step(P, ctx, one, max_new=n - 1)["status"] == 3
    p.nf = 5
    assert p.step(P, ctx, np.where(p.tokens < 7, 3, 0))["status"] == 1
