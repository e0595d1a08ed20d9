"""The 4-bit calls as a server uses them together: slots placed, tokens packed into them, attention over the packed
caches, caches read back and measured, tokens dropped and attention over what is left; eager and captured."""
import numpy as np
import pytest
import torch

import oracle as Oracle
from oracle import packed as O
from oracle import serving as S
from tests.packed_util import check

pytestmark = pytest.mark.gpu

HQ, HKV, D = 8, 2, 64


@pytest.fixture(scope="module")
def ckv():
    import paper_2608_07855_amd as P
    ctx = P.Context(0)
    yield P, ctx
    ctx.close()


def _dev(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


class _Rows:
    """What check() of tests/packed_util.py asks of a batch."""

    def __init__(self, type, v):
        self.type, self.v, self.lens = type, v, np.array([x.shape[0] for x in v])


class Server:
    def __init__(self, P, ctx, n, block, width, seed, most_new):
        self.P, self.ctx, self.n, self.block, self.most_new = P, ctx, n, block, most_new
        self.rng = np.random.default_rng(seed)
        n_blocks = n * -(-width // block) + 5
        self.pool = torch.full((HKV, n_blocks * block, O.row_bytes(D)), 0xFF, dtype=torch.uint8, device="cuda")
        self.tokens, self.n_new = _dev(np.zeros(n)), _dev(np.zeros(n))
        self.free, self.n_free = _dev(self.rng.permutation(n_blocks)), _dev([n_blocks])
        self.slot, self.pos = _dev(np.full((n, width), -1)), _dev(np.full((n, width), 2**31 - 1))
        table = _dev(np.full((n, -(-width // block)), -1)) if block > 1 else None
        self.next_pos = _dev(np.zeros(n))
        self.step = P.slot_step(self.tokens, self.n_new, self.free, self.n_free, self.slot, block_size=block, block_table=table,
                                pos=self.pos, next_pos=self.next_pos, max_new=most_new)
        out = self.out = self.step._out
        self.k, self.v = (torch.zeros((most_new, HKV, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        self.q = torch.zeros((most_new, HQ, D), dtype=torch.bfloat16, device="cuda")
        self.o = torch.zeros_like(self.q)
        self.lse = torch.zeros((most_new, HQ), dtype=torch.float32, device="cuda")
        self.kv = P.packed_view(self.pool, out["n_tokens"], slot=self.slot, pos=self.pos)
        self.rows = P.query_view(self.q, out["cu_new"], out["new_pos"], max_rows=8)
        self.hk, self.hv, self.hp = ([np.zeros((0, HKV, D))] * n for _ in range(3))
        self.hp = [np.zeros(0, np.int64) for _ in range(n)]

    def device_step(self):
        """Everything a step does on the device: nothing here depends on the counts of the moment."""
        P, out = self.P, self.out
        P.ckv_build_slots(self.ctx, self.step)
        P.ckv_pack_tokens(self.ctx, self.k, self.v, out["new_row"], self.pool, n_live=out["cu_new"][self.n:])
        P.ckv_attend_packed(self.ctx, self.kv, self.rows, window=40, n_sink=3, o=self.o, lse=self.lse)

    def set_inputs(self, new):
        total = int(sum(new))
        self.n_new.copy_(_dev(new))
        q, k, v = (torch.from_numpy(self.rng.standard_normal((total, h, D), dtype=np.float32)).to(torch.bfloat16) for h in (HQ, HKV, HKV))
        self.q[:total], self.k[:total], self.v[:total] = q.cuda(), k.cuda(), v.cuda()
        at = 0
        self.want = []
        for s, m in enumerate(new):
            part = slice(at, at + m)
            at += m
            p0 = int(self.next_pos[s])
            kk, vv = O.unpack(O.pack(k[part].float().numpy(), v[part].float().numpy()))
            self.hk[s], self.hv[s] = np.concatenate([self.hk[s], kk]), np.concatenate([self.hv[s], vv])
            pos = p0 + np.arange(m)
            self.hp[s] = np.concatenate([self.hp[s], pos])
            self.want.append(S.attend_rows(q[part].double().numpy(), self.hk[s], self.hv[s], S.sees(self.hp[s], pos, 40, 3)))
        return total

    def after(self, new, total):
        """The step's outputs become the next step's inputs."""
        self.ctx.sync()
        assert int(self.out["status"]) == 0
        want = tuple(np.concatenate([w[i] for w in self.want]) for i in range(3))
        got = self.o[:total].cpu().double().numpy(), self.lse[:total].cpu().double().numpy()
        check(_Rows("bf16", [torch.from_numpy(x) for x in self.hv]), got, want, f"step {new}")
        self.tokens.copy_(self.out["n_tokens"])
        self.n_free.copy_(self.out["n_free"])
        self.next_pos += _dev(new)


STEPS = [[50, 7, 90], [1, 1, 1], [3, 0, 8], [0, 60, 1], [1, 1, 1]]


@pytest.mark.parametrize("block", [1, 16])
def test_steps(ckv, block):
    P, ctx = ckv
    sv = Server(P, ctx, 3, block, 200, 1, 160)
    for new in STEPS:
        total = sv.set_inputs(new)
        sv.device_step()
        sv.after(new, total)


def test_captured_steps(ckv):
    """One graph of a whole step, replayed with other counts and tokens; the pool keeps what earlier replays stored."""
    P, _ = ckv
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = P.Context(0, stream)
        sv = Server(P, ctx, 3, 16, 200, 2, 160)
        total = sv.set_inputs(STEPS[0])
        sv.device_step()
        sv.after(STEPS[0], total)
        sv.n_new.zero_()
        sv.device_step()                     # as the capture will find it: nothing new
        stream.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            sv.device_step()
        for new in STEPS[1:]:
            total = sv.set_inputs(new)
            g.replay()
            sv.after(new, total)
        ctx.close()


def test_measured_and_compressed(ckv):
    """A packed cache read back for the measurement, its selection applied to the slot table, attention over the rest."""
    P, ctx = ckv
    sv = Server(P, ctx, 2, 1, 200, 3, 200)
    total = sv.set_inputs([120, 60])
    sv.device_step()
    sv.after([120, 60], total)
    wide = P.ckv_unpack_tokens(ctx, sv.kv)
    n, W = 120, 8
    qw = torch.from_numpy(sv.rng.standard_normal((HQ, W, D), dtype=np.float32)).to(torch.bfloat16)
    qpos = _dev(np.arange(n - W, n))
    pages = P.Pages(np.arange(0, 96, 16), [16] * 6)
    got = P.ckv_measure_page_effects(ctx, P.kv_view(wide["k"][0], wide["v"][0], sv.pos[0], n), P.window_view(qw.cuda(), qpos), pages,
                                     want=("R", "token_mass"))
    ctx.sync()
    # (against the oracle on what the rows stand for, rounded to bf16 as the call reads it)
    k16, v16 = (torch.from_numpy(x[0]).to(torch.bfloat16) for x in (sv.hk, sv.hv))
    assert torch.equal(wide["k"][0, :, :n].cpu(), k16.transpose(0, 1)) and torch.equal(wide["v"][0, :, :n].cpu(), v16.transpose(0, 1))

    def bits(t):
        return t.contiguous().view(torch.int16).numpy().view(np.uint16)
    want, _ = Oracle.page_effects(bits(k16.transpose(0, 1)), bits(v16.transpose(0, 1)), np.arange(n), bits(qw), np.arange(n - W, n),
                                  [(s, 16) for s in range(0, 96, 16)])
    r = got["R"].cpu().double().numpy()
    assert np.all(np.abs(r - want) <= 2e-3 * np.maximum(want, 1e-6))
    # the selection drops tokens of sequence 0; its slot and position rows are re-indexed, the packed rows stay
    budget = 50
    none = [P.Pages([], [])]
    sel = P.ckv_select_and_compact(ctx, wide["k"][:1, None], wide["v"][:1, None], sv.pos[:1], [n], got["token_mass"][None].contiguous(),
                                   none, none, [None], budget=budget, keep_recent=W, compact=False)
    ctx.sync()
    kept = sel["kept"][0].long()
    assert int(sel["n_kept"]) == budget
    for t in (sv.slot, sv.pos):
        t[0, :budget] = t[0, kept].clone()
    sv.tokens[0] = budget
    idx = kept.cpu().numpy()
    sv.hk[0], sv.hv[0], sv.hp[0] = sv.hk[0][idx], sv.hv[0][idx], sv.hp[0][idx]
    for new in ([5, 1], [1, 1]):
        total = sv.set_inputs(new)
        sv.device_step()
        sv.after(new, total)
