"""Logits far past 2^24, where a float32 one carries no fraction: what the softmax does with equal and with far lower
ones stays as it is."""
import numpy as np
import pytest
import torch

from oracle import serving as S
from tests.serving_util import HALF, TYPES, Batch

pytestmark = pytest.mark.gpu

# keys and queries of all-equal elements: raw products of 64 c^2 (up to 2^38 in fp16, 2^126 in bf16)
SIZES = [("fp16", 2.0**12 * 3), ("fp16", 60000.0), ("bf16", 3.0 * 2**13), ("bf16", 3.0 * 2**18), ("bf16", 3.0 * 2**58)]


@pytest.fixture(scope="module")
def ckv():
    import paper_2608_07855_amd as P
    ctx = P.Context(0)
    yield P, ctx
    ctx.close()


@pytest.mark.parametrize("type,size", SIZES)
@pytest.mark.parametrize("rows,prefix,window", [(1, 0, 0), (1, 0, 300), (40, 0, 0), (40, 0, 200), (1, 900, 0), (40, 900, 0)])
@pytest.mark.parametrize("sign", [1, -1])
def test_large_logits(ckv, rows, prefix, window, sign, type, size):
    """A third of the tokens have half the key of the others, the first 70 none: with queries of the keys' sign the
    latter two count for nothing, with the other sign only the first 70 do, or the third where no row sees these."""
    P, ctx = ckv
    b = Batch(1, [700, 90], [rows, 1], 4, 2, 64, type, prefix=prefix, heavy=False)
    t = TYPES[type]
    size = float(torch.tensor(size).to(t))
    for k in b.k + [b.pk]:
        k[:] = size
        k[::3] = size / 2
    (b.pk if prefix else b.k[0])[:70] = 0
    for q in b.q:
        q[:] = sign * size
    o, lse = b.run(P, ctx, b.device(P), window, 0)
    wo, wl, w = b.want(window, 0)
    # Weights of equal logits are equal, the others are 0: nothing but o's rounding (and the sums') is left.  lse: the
    # products are exact, and the scale, its product with them and the way back from log2 units are rounded once each.
    eo, el = np.abs(o - wo) / (HALF[type] * np.abs(wo) + 2.0**-13 * w + 2.0**-24), np.abs(lse - wl) / (2.0**-13 + 2.0**-21 * np.abs(wl))
    print(f"[parity] o {eo.max():.3g}, lse {el.max():.3g} of the tolerance", flush=True)
    assert np.isfinite(o).all() and eo.max() <= 1 and el.max() <= 1


def test_the_oracle_separates_them():
    """Of these logits the oracle's weights are 0 or equal."""
    k = np.full((4, 1, 64), 3.0 * 2**13)
    k[:2] /= 2
    v = np.arange(4.0)[:, None, None] * np.ones((1, 1, 64))
    o, _, _ = S.attend_rows(np.full((1, 1, 64), 3.0 * 2**13), k, v, np.ones((1, 4), bool))
    assert np.all(o == 2.5)
