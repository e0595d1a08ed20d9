"""Block and slot tables of a step (ckv_build_slots) against the step-by-step oracle: equal in every word."""
import numpy as np
import pytest
import torch

from oracle import serving as S

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ckv():
    import paper_2608_07855_amd as P
    ctx = P.Context(0)
    yield P, ctx
    ctx.close()


def _dev(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


class Pool:
    def __init__(self, seed, n, block, n_blocks, width, positions=True, table=True):
        self.rng = np.random.default_rng(seed)
        self.n, self.B, self.nb, self.width = n, block, n_blocks, width
        self.tokens = np.zeros(n, np.int64)
        self.cols = -(-width // block)
        self.table = np.full((n, self.cols), -1) if table else None
        self.slot = np.full((n, width), -1)
        self.pos = np.full((n, width), -1) if positions else None
        self.free, self.nf = self.rng.permutation(n_blocks), n_blocks

    def step(self, P, ctx, new, next_pos=None, max_new=None, pad=0):
        """One step on both sides; every table and output is compared.  Returns the oracle's."""
        most = int(np.maximum(new, 0).sum()) + 5 if max_new is None else max_new

        def table(x):
            if x is None:
                return None
            t = torch.full((x.shape[0], x.shape[1] + pad), -99, dtype=torch.int32, device="cuda")
            t[:, :x.shape[1]] = _dev(x)
            return t[:, :x.shape[1]]
        free, tab, slot, pos = _dev(self.free), table(self.table), table(self.slot), table(self.pos)
        step = P.slot_step(_dev(self.tokens), _dev(new), free, _dev([self.nf]), slot, block_size=self.B, block_table=tab,
                           pos=pos, next_pos=None if next_pos is None else _dev(next_pos),
                           new_row=torch.full((most,), -5, dtype=torch.int32, device="cuda"),
                           new_pos=torch.full((most,), -5, dtype=torch.int32, device="cuda"))
        out = P.ckv_build_slots(ctx, step)
        ctx.sync()
        want = S.build_slots(self.tokens, new, self.free, self.nf, self.table, self.slot, self.pos, next_pos, self.B,
                             most, self.nb)
        got = {k: x.cpu().numpy() for k, x in out.items()}
        assert got["status"][0] == want["status"]
        assert got["n_tokens"].tolist() == [int(x) for x in want["n_tokens"]] and got["n_free"][0] == want["n_free"]
        assert got["cu_new"].tolist() == want["cu_new"]
        m = len(want["new_row"])
        assert got["new_row"][:m].tolist() == want["new_row"] and np.all(got["new_row"][m:] == -5)
        assert got["new_pos"][:m].tolist() == want["new_pos"] and np.all(got["new_pos"][m:] == -5)
        for name, g, w in (("free", free, want["free"]), ("table", tab, want["table"]), ("slot", slot, want["slot"]),
                           ("pos", pos, want["pos"])):
            if w is not None:
                assert np.array_equal(g.cpu().numpy(), w), name
        if pad:
            for t in (tab, slot, pos):
                if t is not None:
                    assert torch.all(t._base[:, t.shape[1]:] == -99)
        return want

    def take(self, r):
        self.tokens, self.free, self.nf = np.array(r["n_tokens"], np.int64), r["free"], r["n_free"]
        self.table, self.slot, self.pos = r["table"], r["slot"], r["pos"]


@pytest.mark.parametrize("block", [1, 3, 16, 64])
@pytest.mark.parametrize("n", [1, 5, 64, 300, 1500])
def test_steps(ckv, n, block):
    """A run of steps: prompts, single tokens, sequences that end, odd block sizes."""
    P, ctx = ckv
    width = 150
    p = Pool(n * 100 + block, n, block, int(n * (-(-width // block)) * 0.8) + 2, width)
    for i in range(6):
        if i % 3 == 0:
            new = p.rng.integers(0, 40, n)
        elif i % 3 == 1:
            new = np.ones(n, np.int64)
        else:
            new = np.where(p.rng.random(n) < 0.4, -1, p.rng.integers(0, 3, n))
        new = np.where(new > 0, np.minimum(new, width - p.tokens), new)
        r = p.step(P, ctx, new, next_pos=p.rng.integers(0, 1 << 30, n) if i % 2 else None, pad=3 if i == 4 else 0)
        if r["status"] == 0:
            p.take(r)


@pytest.mark.parametrize("table", [False, True])
def test_single_row_blocks(ckv, table):
    """block_size 1, where the slot table is the block table."""
    P, ctx = ckv
    p = Pool(7, 20, 1, 900, 60, table=table)
    for new in (p.rng.integers(0, 40, 20), np.ones(20, np.int64), np.where(np.arange(20) % 3 == 0, -1, 2)):
        r = p.step(P, ctx, new)
        assert r["status"] == 0
        p.take(r)


def test_without_positions(ckv):
    P, ctx = ckv
    p = Pool(8, 4, 16, 30, 64, positions=False)
    p.take(p.step(P, ctx, np.array([17, 0, 33, 1])))


def test_long_prompts(ckv):
    """One sequence with very many tokens beside short ones; every block of the pool in use."""
    P, ctx = ckv
    p = Pool(9, 3, 16, 1260, 20000)
    r = p.step(P, ctx, np.array([20000, 1, 100]), next_pos=[5, 6, 7])
    assert r["status"] == 0
    p.take(r)
    p.take(p.step(P, ctx, np.array([-1, 159, 12])))
    r = p.step(P, ctx, np.array([19700, 0, -1]))
    assert r["status"] == 0


def test_shortages_change_nothing(ckv):
    P, ctx = ckv
    p = Pool(10, 4, 4, 12, 20)
    p.take(p.step(P, ctx, np.array([8, 8, 8, 8])))
    assert p.step(P, ctx, np.array([20, 1, 1, 1]))["status"] == S.TABLE
    assert p.step(P, ctx, np.array([5, 5, 5, 5]))["status"] == S.NO_BLOCKS
    assert p.step(P, ctx, np.array([1, 1, 1, 1]), max_new=3)["status"] == S.MAX_NEW
    assert p.step(P, ctx, np.array([1, -2, 1, 1]))["status"] == S.BAD_COUNT
    assert p.step(P, ctx, np.array([5, 5, -1, 4]))["status"] == 0       # the ended one's blocks serve the others
    p.nf = 13
    assert p.step(P, ctx, np.array([0, 0, 0, 0]))["status"] == S.BAD_COUNT
    p.nf, p.tokens = 4, np.array([8, -8, 8, 8])
    assert p.step(P, ctx, np.array([0, 0, 0, 0]))["status"] == S.BAD_COUNT
    p.tokens = np.array([8, 8, 8, 8])
    p.nf = 11                                                            # more free blocks than the sequences leave
    assert p.step(P, ctx, np.array([-1, 0, 0, 0]))["status"] == S.BAD_COUNT
    p.tokens = np.array([8, 8, 8, 2**31 - 1])
    assert p.step(P, ctx, np.array([0, 0, 0, 2**31 - 1]), max_new=100)["status"] == S.MAX_NEW


def test_bad_block_numbers_stay_in_the_pool(ckv):
    """Table entries outside the pool give rows of its last block."""
    P, ctx = ckv
    p = Pool(11, 2, 4, 12, 20)
    p.take(p.step(P, ctx, np.array([5, 6])))
    p.table[0, 1], p.table[1, 1] = -3, 1 << 29
    r = p.step(P, ctx, np.array([2, 1]))
    assert all(11 * 4 <= x < 12 * 4 for x in r["new_row"])


def test_no_sequences(ckv):
    P, ctx = ckv
    p = Pool(12, 0, 4, 12, 20)
    r = p.step(P, ctx, np.zeros(0, np.int64))
    assert r["status"] == 0 and r["cu_new"] == [0]


def test_captured_steps(ckv):
    """Two steps that hand their counts to each other, captured and replayed."""
    P, _ = ckv
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = P.Context(0, stream)
        n, B, nb, width = 10, 4, 200, 64
        a, b, fa, fb = _dev(np.zeros(n)), _dev(np.zeros(n)), _dev([nb]), _dev([0])
        free, tab = _dev(np.arange(nb)), _dev(np.full((n, 16), -1))
        slot, new = _dev(np.full((n, width), -1)), _dev(np.arange(n) % 3)
        kw = dict(block_size=B, block_table=tab, max_new=64)
        one = P.slot_step(a, new, free, fa, slot, n_tokens_out=b, n_free_out=fb, **kw)
        two = P.slot_step(b, new, free, fb, slot, n_tokens_out=a, n_free_out=fa, **kw)
        stream.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            P.ckv_build_slots(ctx, one)
            P.ckv_build_slots(ctx, two)
        tok, f, nf, t, sl = [0] * n, np.arange(nb), nb, np.full((n, 16), -1), np.full((n, width), -1)
        for k in range(3):
            g.replay()
            stream.synchronize()
            for _ in range(2):
                r = S.build_slots(tok, (np.arange(n) + k) % 3, f, nf, t, sl, None, None, B, 64, nb)
                tok, f, nf, t, sl = r["n_tokens"], r["free"], r["n_free"], r["table"], r["slot"]
            assert a.tolist() == tok and int(fa) == nf
            assert np.array_equal(tab.cpu().numpy(), t) and np.array_equal(slot.cpu().numpy(), sl)
            new.copy_(_dev((np.arange(n) + k + 1) % 3))
            stream.synchronize()
        ctx.close()


def test_columns_of_wider_tables(ckv):
    """Tables that are columns of wider ones: a step past their width changes nothing beside them."""
    P, ctx = ckv
    B, nb = 4, 40
    wide_slot, wide_tab = _dev(np.full((2, 20), -1)), _dev(np.full((2, 9), -1))
    slot, tab = wide_slot[:, 12:], wide_tab[:, 6:]
    for new, want in (((8, 8), 0), ((1, 0), 2), ((0, 9), 2)):
        st = P.slot_step(_dev([0, 0]) if want == 0 else _dev([8, 8] if new[0] else [8, 0]), _dev(new),
                         _dev(np.arange(nb)), _dev([nb]), slot, block_size=B, block_table=tab, max_new=32)
        assert int(P.ckv_build_slots(ctx, st)["status"]) == want
    st = P.slot_step(_dev([0, 0]), _dev([0, 0]), _dev(np.arange(nb)), _dev([nb]), slot, block_size=B, block_table=tab, max_new=32)
    st.slot_stride = 7
    with pytest.raises(P.CKVError) as e:
        P.ckv_build_slots(ctx, st)
    assert e.value.code == -1
    assert wide_slot[:, 12:].min() >= 0 and torch.all(wide_slot[:, :12] == -1) and torch.all(wide_tab[:, :6] == -1)
    assert wide_tab[:, 6:8].min() >= 0 and torch.all(wide_tab[:, 8] == -1)


def test_refusals(ckv):
    P, ctx = ckv
    n, B, nb = 3, 4, 20

    def step(**kw):
        a = dict(n_tokens=_dev(np.zeros(n)), n_new=_dev(np.ones(n)), free=_dev(np.arange(nb)), n_free=_dev([nb]),
                 slot=_dev(np.full((n, 16), -1)), block_size=B, block_table=_dev(np.full((n, 4), -1)), max_new=8)
        a.update(kw)
        return P.slot_step(a.pop("n_tokens"), a.pop("n_new"), a.pop("free"), a.pop("n_free"), a.pop("slot"), **a)

    def code(s):
        with pytest.raises(P.CKVError) as e:
            P.ckv_build_slots(ctx, s)
        return e.value.code
    assert code(step(block_size=0)) == -1
    assert code(step(block_size=1 << 30)) == -1
    assert code(step(block_table=None)) == -1
    same = _dev(np.zeros(n))
    assert code(step(n_tokens=same, n_tokens_out=same)) == -1
    both = _dev(np.zeros(8))
    assert code(step(new_row=both, new_pos=both)) == -1
    nf = _dev([nb])
    assert code(step(n_free=nf, n_free_out=nf)) == -1
    for field in ("n_tokens", "n_new", "n_free", "free_blocks", "slot", "n_tokens_out", "n_free_out", "cu_new", "new_row",
                  "status"):
        s = step()
        setattr(s, field, None)
        assert code(s) == -1, field
    for call in (lambda: step(n_new=_dev(np.zeros(n - 1))), lambda: step(slot=_dev(np.zeros((n + 1, 4)))),
                 lambda: step(pos=_dev(np.zeros((n, 5)))), lambda: step(n_tokens=_dev(np.zeros(n)).long()),
                 lambda: step(n_free=_dev(np.zeros(0))), lambda: step(free=_dev(np.zeros(4)).cpu())):
        with pytest.raises(ValueError):
            call()
