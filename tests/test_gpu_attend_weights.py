"""Attention where one token takes nearly all of the weight and holds nothing: the output is what many far smaller
weights add up to."""
import numpy as np
import pytest
import torch

from tests.serving_util import HALF, TYPES

pytestmark = pytest.mark.gpu

D = 64


@pytest.fixture(scope="module")
def ckv():
    import paper_2608_07855_amd as P
    ctx = P.Context(0)
    yield P, ctx
    ctx.close()


@pytest.fixture(scope="module")
def limited():
    """A context without room for partial sums: nothing is split."""
    import paper_2608_07855_amd as P
    ctx = P.Context(0)
    ctx.set_workspace_limit(4096)
    yield P, ctx
    ctx.close()


class Dominated:
    """One sequence of n tokens, the first of them in the shared prefix (if any).  Token 0 has the key (8, 0, ..) and
    no value, the others no key and values in [0.5, 1.5]; a query head of gap g is (g, 0, ..), so that token 0's logit
    is g, and the others' are 0."""

    def __init__(self, n, rows, type, prefix=0, *, gaps):
        t = TYPES[type]
        rng = np.random.default_rng(n + rows)
        self.n, self.rows, self.type, self.prefix = n, rows, type, prefix
        self.v = torch.from_numpy(rng.uniform(0.5, 1.5, (n, D)).astype(np.float32)).to(t)
        self.v[0] = 0
        self.k = torch.zeros((n, D), dtype=t)
        self.k[0, 0] = 8
        self.q = torch.zeros((rows, len(gaps), D), dtype=t)
        self.q[:, :, 0] = torch.tensor(gaps).to(t)

    def run(self, P, ctx):
        def view(k, v):
            k, v = (x[None, None].contiguous().cuda() for x in (k, v))
            return P.batch_view(k, v, torch.tensor([k.shape[2]], dtype=torch.int32, device="cuda"))
        p = self.prefix
        q = P.query_view(self.q.cuda(), torch.tensor([0, self.rows], dtype=torch.int32, device="cuda"))
        if p:
            got = P.ckv_attend_shared(ctx, view(self.k[:p], self.v[:p]), view(self.k[p:], self.v[p:]), q, want=("o", "lse"))
        else:
            got = P.ckv_attend_window(ctx, view(self.k, self.v), q, want=("o", "lse"))
        ctx.sync()
        return got["o"].cpu().double().numpy(), got["lse"].cpu().double().numpy()

    def want(self):
        """Row j sees m = n - rows + j + 1 tokens: o = sum of their values / (e^g + m - 1), lse = log of that."""
        m = self.n - self.rows + np.arange(self.rows) + 1
        sums = np.cumsum(self.v.double().numpy(), 0)[m - 1]
        z = np.exp(self.q[:, :, 0].double().numpy()) + m[:, None] - 1
        return sums[:, None] / z[..., None], np.log(z)


def _check(case, got, want, what):
    """Values are not negative, so that a relative error of every weight is one of the output.  Half a step of the type
    for the output's rounding, as much for the weights', and 2^-13 for the logits, exponentials and sums in float32
    (an absolute error in lse).  An fp16 weight may be off by 2^-38 of the largest one as well, n of them."""
    (o, lse), (wo, wl) = got, want
    h = HALF[case.type]
    far = case.n * 2.0**-38 * 1.5 if case.type == "fp16" else 0.0
    eo, el = np.abs(o - wo) / ((2 * h + 2.0**-13) * wo + far), np.abs(lse - wl) / (2.0**-13 + 2.0**-22 * wl)
    print(f"[parity] {what}: o {eo.max():.3g}, lse {el.max():.3g} of the tolerance", flush=True)
    assert eo.max() <= 1 and el.max() <= 1, what


@pytest.mark.parametrize("n,rows", [(1 << 19, 1), (1 << 17, 64)])
def test_sums_without_splits(limited, n, rows):
    """Each of the weights is lost in a float32 sum that the dominant one has already entered; not split, a row's sum
    has only few places to begin from."""
    P, ctx = limited
    c = Dominated(n + 1, rows, "bf16", gaps=[12.0, 16.6, 17.0, 17.4, 18.0])
    _check(c, c.run(P, ctx), c.want(), f"{n} tokens, {rows} rows")


@pytest.mark.parametrize("type", ["bf16", "fp16"])
@pytest.mark.parametrize("rows", [1, 64])
@pytest.mark.parametrize("prefix", [0, 131008])
@pytest.mark.parametrize("split", [True, False])
def test_many_small_weights(ckv, limited, split, rows, prefix, type):
    """131072 tokens behind a dominant one: few and many rows, over one cache and over a shared prefix, in splits (of
    which one alone holds the dominant token) and whole."""
    P, ctx = ckv if split else limited
    c = Dominated(131073, rows, type, prefix, gaps=[12.0, 16.6, 17.0, 18.0])
    _check(c, c.run(P, ctx), c.want(), f"{rows} rows, prefix {prefix}")
