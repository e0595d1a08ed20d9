"""The serving calls as a step uses them: tables built on the device, new keys and values stored through them,
attention over the pool, sequences that come and go, and a checkpoint that drops single tokens."""
import numpy as np
import pytest
import torch

from oracle import serving as S
from tests.serving_util import HALF

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


class Server:
    """A pool, its tables on the device, and on the host what every sequence has seen."""

    def __init__(self, P, ctx, n, block, n_blocks, width, seed):
        self.P, self.ctx, self.n, self.block, self.width = P, ctx, n, block, width
        self.rng = np.random.default_rng(seed)
        rows = n_blocks * block
        self.k = torch.full((HKV, rows, D), float("nan"), dtype=torch.bfloat16, device="cuda")
        self.v = self.k.clone()
        self.free, self.n_free = _dev(self.rng.permutation(n_blocks)), [_dev([n_blocks]), _dev([0])]
        self.tokens = [_dev(np.zeros(n)), _dev(np.zeros(n))]
        self.table = _dev(np.full((n, -(-width // block)), -1)) if block > 1 else None
        self.slot, self.pos = _dev(np.full((n, width), -1)), _dev(np.full((n, width), 2**31 - 1))
        self.next_pos = np.zeros(n, np.int64)
        self.hk = [np.zeros((0, HKV, D)) for _ in range(n)]
        self.hv = [np.zeros((0, HKV, D)) for _ in range(n)]
        self.hp = [np.zeros(0, np.int64) for _ in range(n)]

    def _draw(self, *shape):
        return torch.from_numpy(self.rng.standard_normal(shape, dtype=np.float32)).to(torch.bfloat16)

    def step(self, new):
        """Places the new tokens; returns their rows' query view and the host queries."""
        P, new = self.P, np.asarray(new)
        total = int(np.maximum(new, 0).sum())
        st = P.slot_step(self.tokens[0], _dev(new), self.free, self.n_free[0], self.slot, block_size=self.block,
                         block_table=self.table, pos=self.pos, next_pos=_dev(self.next_pos), n_tokens_out=self.tokens[1],
                         n_free_out=self.n_free[1], max_new=max(total, 1))
        out = P.ckv_build_slots(self.ctx, st)
        q, k, v = self._draw(total, HQ, D), self._draw(total, HKV, D), self._draw(total, HKV, D)
        rows = out["new_row"][:total].long()
        self.k[:, rows], self.v[:, rows] = k.transpose(0, 1).cuda(), v.transpose(0, 1).cuda()
        assert int(out["status"]) == 0
        self.tokens.reverse()
        self.n_free.reverse()
        at = 0
        for s in range(self.n):
            if new[s] < 0:
                self.hk[s], self.hv[s], self.hp[s], self.next_pos[s] = self.hk[s][:0], self.hv[s][:0], self.hp[s][:0], 0
                continue
            part = slice(at, at + int(new[s]))
            at += int(new[s])
            self.hk[s] = np.concatenate([self.hk[s], k[part].double().numpy()])
            self.hv[s] = np.concatenate([self.hv[s], v[part].double().numpy()])
            self.hp[s] = np.concatenate([self.hp[s], self.next_pos[s] + np.arange(new[s])])
            self.next_pos[s] += new[s]
        view = P.query_view(q.cuda(), out["cu_new"], out["new_pos"][:total] if total else None, max_rows=max(1, int(new.max())))
        return view, q.double().numpy(), np.maximum(new, 0)

    def view(self):
        return self.P.batch_view(self.k, self.v, self.tokens[0], slot=self.slot, pos=self.pos)

    def check(self, o, q, new, window, n_sink, what):
        o = o.cpu().double().numpy()
        at = 0
        for s in range(self.n):
            m = int(new[s])
            if not m:
                continue
            vis = S.sees(self.hp[s], self.hp[s][-m:], window, n_sink)
            wo, _, w = S.attend_rows(q[at:at + m], self.hk[s], self.hv[s], vis)
            tol = HALF["bf16"] * np.abs(wo) + (HALF["bf16"] + 2.0**-13) * w + 2.0**-24
            assert np.all(np.abs(o[at:at + m] - wo) <= tol), f"{what}, sequence {s}"
            at += m


@pytest.mark.parametrize("block", [1, 16])
def test_steps_of_a_server(ckv, block):
    """Prompts, single tokens, sequences that end and others that take their place."""
    P, ctx = ckv
    srv = Server(P, ctx, 5, block, 700 // block, 260, 1)
    steps = [[100, 7, 0, 33, 1], [1, 1, 60, 1, 1], [1, 1, 1, 1, 1], [1, -1, 1, 1, 20], [-1, 130, 1, 1, 1], [90, 1, 1, -1, 1],
             [1, 1, 1, 0, 1]]
    for i, new in enumerate(steps):
        q, hq, rows = srv.step(new)
        for window, n_sink in ((0, 0), (40, 4)):
            o = P.ckv_attend_window(ctx, srv.view(), q, window=window, n_sink=n_sink)["o"]
            ctx.sync()
            srv.check(o, hq, rows, window, n_sink, f"step {i}, window {window}")


def test_checkpoint_between_steps(ckv):
    """Blocks of one row: a checkpoint keeps single tokens by the window's mass, the slot table is gathered through
    the kept indices, the dropped rows go back to the stack, and serving goes on at gapped positions."""
    P, ctx = ckv
    n, W, budget = 2, 8, 96
    srv = Server(P, ctx, n, 1, 400, 200, 2)
    srv.step([150, 131])
    q, hq, rows = srv.step([W, W])
    lens = [len(p) for p in srv.hp]
    keep_idx, none = [], P.Pages([], [])
    slot, pos = srv.slot.clone(), srv.pos.clone()
    for s in range(n):
        kv = P.kv_view(srv.k, srv.v, srv.pos[s], lens[s], slot=srv.slot[s].contiguous())
        win = P.window_view(q._keep[0][s * W:(s + 1) * W].transpose(0, 1), srv.pos[s, lens[s] - W:lens[s]].contiguous())
        mass = P.ckv_measure_page_effects(ctx, kv, win, none, want=("R", "o", "token_mass"))
        # the measurement's window outputs are the attention's
        o = P.ckv_attend_window(ctx, srv.view(), q)["o"][s * W:(s + 1) * W].transpose(0, 1)
        assert torch.allclose(mass["o"], o.float(), rtol=2.0**-7, atol=2.0**-7)
        sel = P.ckv_select_and_compact(ctx, srv.k[None, None][:, :, :, :lens[s]], srv.v[None, None][:, :, :, :lens[s]],
                                       srv.pos[s:s + 1, :lens[s]], [lens[s]], mass["token_mass"][None].contiguous(), [none],
                                       [none], [None], budget=budget, eta=0.0, keep_recent=W, compact=False)
        ctx.sync()
        kept = sel["kept"][0, :int(sel["n_kept"][0])].long()
        keep_idx.append(kept.cpu().numpy())
        slot[s, :len(kept)], pos[s, :len(kept)] = srv.slot[s][kept], srv.pos[s][kept]
    nf = int(srv.n_free[0])
    for s in range(n):
        gone = np.setdiff1d(np.arange(lens[s]), keep_idx[s])
        srv.free[nf:nf + len(gone)] = srv.slot[s][torch.from_numpy(gone).cuda()]
        nf += len(gone)
        srv.hk[s], srv.hv[s], srv.hp[s] = srv.hk[s][keep_idx[s]], srv.hv[s][keep_idx[s]], srv.hp[s][keep_idx[s]]
    srv.slot, srv.pos = slot, pos
    srv.n_free[0], srv.tokens[0] = _dev([nf]), _dev([len(k) for k in keep_idx])
    assert np.any(np.diff(srv.hp[0]) > 1)
    for i, new in enumerate([[1, 1], [1, 40], [3, 1]]):
        q, hq, rows = srv.step(new)
        for window, n_sink in ((0, 0), (60, 2)):
            o = P.ckv_attend_window(ctx, srv.view(), q, window=window, n_sink=n_sink)["o"]
            ctx.sync()
            srv.check(o, hq, rows, window, n_sink, f"step {i} after the checkpoint, window {window}")


def test_samples_of_one_prompt(ckv):
    """A prompt placed once as a sequence of its own; the samples behind it hold their own tokens only."""
    P, ctx = ckv
    n = 6
    srv = Server(P, ctx, 1 + n, 16, 80, 200, 3)
    srv.step([150] + [0] * n)
    prefix = P.batch_view(srv.k, srv.v, srv.tokens[0][:1].clone(), slot=srv.slot[:1].contiguous())
    hk, hv = srv.hk[0], srv.hv[0]
    srv.next_pos[1:] = 150
    for new in ([0] + [1] * n, [0, 1, 1, 30, 1, -1, 1], [0, 1, 1, 1, 1, 2, 1]):
        q, hq, rows = srv.step(new)
        if -1 in new:
            srv.next_pos[1 + new[1:].index(-1)] = 150
        cu = q._keep[1][1:].contiguous()                       # the prompt itself owns no rows
        kv = P.batch_view(srv.k, srv.v, srv.tokens[0][1:].clone(), slot=srv.slot[1:], pos=srv.pos[1:])
        qs = P.query_view(q._keep[0], cu, q._keep[2], max_rows=int(max(new)))
        o = P.ckv_attend_shared(ctx, prefix, kv, qs)["o"]
        ctx.sync()
        o, at = o.cpu().double().numpy(), 0
        for s in range(1, 1 + n):
            m = int(rows[s])
            if not m:
                continue
            p = np.concatenate([np.arange(150), srv.hp[s]])
            wo, _, w = S.attend_rows(hq[at:at + m], np.concatenate([hk, srv.hk[s]]), np.concatenate([hv, srv.hv[s]]),
                                     S.sees(p, srv.hp[s][-m:]))
            tol = HALF["bf16"] * np.abs(wo) + (HALF["bf16"] + 2.0**-13) * w + 2.0**-24
            assert np.all(np.abs(o[at:at + m] - wo) <= tol), f"sample {s}"
            at += m
