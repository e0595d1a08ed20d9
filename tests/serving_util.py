"""Batches for the tests of the serving calls: host arrays, their device views and the comparison with the oracle."""
import numpy as np
import torch

from oracle import serving as S

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
# half a step of a rounding to the type, relative to the value
HALF = {"bf16": torch.finfo(torch.bfloat16).eps / 2, "fp16": torch.finfo(torch.float16).eps / 2}


class Batch:
    """lens: resident tokens, rows: query rows of each sequence.  Everything lives on the host in float32 that the
    type holds exactly; ``device`` lays it out."""

    def __init__(self, seed, lens, rows, hq=4, hkv=2, d=64, type="bf16", paged=True, gaps=False, qpos=None, prefix=0,
                 prefix_gaps=False, tables=None, lead=0, tail=0, scale=None, heavy=True):
        rng = self.rng = np.random.default_rng(seed)
        self.lens, self.rows = np.array(lens, np.int64), np.array(rows, np.int64)
        self.n, self.hq, self.hkv, self.d, self.type = len(lens), hq, hkv, d, type
        self.paged, self.prefix, self.lead, self.tail, self.scale = paged, prefix, lead, tail, scale
        self.most = int(max(self.lens.max(initial=0), 1)) if tables is None else tables
        self.pool = int(self.lens.sum()) + prefix + 13

        def draw(*shape):
            return torch.from_numpy(rng.standard_normal(shape, dtype=np.float32)).to(TYPES[type])
        self.k = [draw(t, hkv, d) for t in self.lens]
        self.v = [draw(t, hkv, d) for t in self.lens]
        self.pk, self.pv = draw(prefix, hkv, d), draw(prefix, hkv, d)
        for x in self.k + [self.pk] if heavy else []:
            x[rng.random(x.shape[0]) < 0.02] *= 4
        self.q = [draw(r, hq, d) for r in self.rows]
        self.base = prefix
        self.ppos = np.cumsum(rng.integers(1, 4, prefix)) - 1 if prefix_gaps else np.arange(prefix)
        if gaps:
            self.pos = [self.base * (3 if prefix_gaps else 1) + np.cumsum(rng.integers(1, 4, t)) - 1 for t in self.lens]
        else:
            self.pos = None
        self.given_qpos = qpos

    def positions(self, s):
        return self.base + np.arange(self.lens[s]) if self.pos is None else self.pos[s]

    def qpos(self, s):
        if self.given_qpos is not None:
            return np.asarray(self.given_qpos[s])
        p, n, R = self.positions(s), int(self.lens[s]), int(self.rows[s])
        if self.pos is None:
            return self.base + n - R + np.arange(R)
        return np.array([p[n - R + j] if n - R + j >= 0 else -2**31 for j in range(R)], np.int64)

    def want(self, window=0, n_sink=0, only=None):
        """o, lse, w of every sequence's rows (packed), from the oracle."""
        out = []
        for s in range(self.n) if only is None else only:
            k = np.concatenate([self.pk.double().numpy(), self.k[s].double().numpy()])
            v = np.concatenate([self.pv.double().numpy(), self.v[s].double().numpy()])
            vis = S.sees(np.concatenate([self.ppos, self.positions(s)]), self.qpos(s), window, n_sink)
            out.append(S.attend_rows(self.q[s].double().numpy(), k, v, vis, self.scale))
        return tuple(np.concatenate(x) for x in zip(*out))

    def device(self, P, fill=float("nan"), max_rows=None):
        """Views of the batch; storage that no token owns holds ``fill``."""
        n, hkv, d, t = self.n, self.hkv, self.d, TYPES[self.type]
        dev = "cuda"
        place = self.rng.permutation(self.pool)
        views = {}
        if self.paged or self.prefix:
            kp = torch.full((hkv, self.pool, d), fill, dtype=t)
            vp = kp.clone()
            slot = np.full((n, self.most), -7, np.int32)
            at = 0
            parts = [(self.pk, self.pv)] + (list(zip(self.k, self.v)) if self.paged else [])
            rows = []
            for k, v in parts:
                r = place[at:at + k.shape[0]]
                at += k.shape[0]
                kp[:, r], vp[:, r] = k.transpose(0, 1), v.transpose(0, 1)
                rows.append(r)
            for s in range(n) if self.paged else []:
                slot[s, :self.lens[s]] = rows[1 + s]
            kp, vp = kp.to(dev), vp.to(dev)
            views["pool"] = (kp, vp)
        if self.paged:
            k, v, slot = kp, vp, torch.from_numpy(slot).to(dev)
        else:
            k = torch.full((n, hkv, self.most, d), fill, dtype=t)
            v = k.clone()
            for s in range(n):
                k[s, :, :self.lens[s]], v[s, :, :self.lens[s]] = self.k[s].transpose(0, 1), self.v[s].transpose(0, 1)
            k, v, slot = k.to(dev), v.to(dev), None
        pos = None
        if self.pos is not None:
            pos = np.full((n, self.most), 2**31 - 1, np.int32)
            for s in range(n):
                pos[s, :self.lens[s]] = self.pos[s]
            pos = torch.from_numpy(pos).to(dev)
        lens = torch.from_numpy(self.lens.astype(np.int32)).to(dev)
        kv = P.batch_view(k, v, lens, slot=slot, pos=pos, max_tokens=self.most)
        q = torch.cat([torch.zeros((self.lead, self.hq, d), dtype=t)] + self.q +
                      [torch.zeros((self.tail, self.hq, d), dtype=t)]).to(dev)
        cu = torch.from_numpy((self.lead + np.concatenate([[0], np.cumsum(self.rows)])).astype(np.int32)).to(dev)
        qpos = None
        if self.given_qpos is not None:
            qpos = np.concatenate([np.zeros(self.lead)] + [np.asarray(x) for x in self.given_qpos] + [np.zeros(self.tail)])
            qpos = torch.from_numpy(qpos.astype(np.int32)).to(dev)
        views.update(kv=kv, q=P.query_view(q, cu, qpos, max_rows=max_rows or max(1, int(self.rows.max(initial=1))),
                                           scale=0.0 if self.scale is None else self.scale))
        if self.prefix:
            ppos = torch.from_numpy(self.ppos.astype(np.int32))[None].contiguous().to(dev)
            views["prefix"] = P.batch_view(kp, vp, torch.tensor([self.prefix], dtype=torch.int32, device=dev),
                                           slot=torch.from_numpy(rows[0].astype(np.int32))[None].contiguous().to(dev),
                                           pos=ppos, max_tokens=self.prefix)
        return views

    def run(self, P, ctx, views, window=0, n_sink=0, fill=7.0):
        """o, lse as float64 arrays of the sequences' rows; rows of no sequence must keep their fill."""
        t, total = TYPES[self.type], int(self.rows.sum()) + self.lead + self.tail
        o = torch.full((total, self.hq, self.d), fill, dtype=t, device="cuda")
        lse = torch.full((total, self.hq), fill, dtype=torch.float32, device="cuda")
        if self.prefix:
            P.ckv_attend_shared(ctx, views["prefix"], views["kv"], views["q"], o=o, lse=lse)
        else:
            P.ckv_attend_window(ctx, views["kv"], views["q"], window=window, n_sink=n_sink, o=o, lse=lse)
        ctx.sync()
        o, lse = o.cpu().double().numpy(), lse.cpu().double().numpy()
        mine = slice(self.lead, total - self.tail)
        rest = np.ones(total, bool)
        rest[mine] = False
        assert np.all(o[rest] == fill) and np.all(lse[rest] == fill), "rows of no sequence were written"
        return o[mine], lse[mine]


def tolerances(b, o, lse, w):
    """|o| is rounded once to the type (half a step), and so is each softmax weight: half a step of sum a |v|, plus,
    in fp16, weights below 2^-14 of the reference (a reference may lag the largest logit by 2^8), which are off by
    2^-25 each, n of them.  float32 logits: d products and a sum each off by 2^-24 of sum |q k| (below 2^6 here),
    and the exponential and the sums: 2^-13 in all, relative to the weights and absolute in lse."""
    h = HALF[b.type]
    vmax = max(float(x.abs().max()) if x.numel() else 0.0 for x in b.v + [b.pv])
    tiny = (int(b.lens.max()) + b.prefix) * 2.0**-25 * 2**8 * vmax * 2.0**-8 if b.type == "fp16" else 0.0
    return h * np.abs(o) + (h + 2.0**-13) * w + tiny + 2.0**-24, 2.0**-13 + 2.0**-22 * np.abs(lse)


def check(b, got, want, what=""):
    o, lse = got
    wo, wl, w = want
    to, tl = tolerances(b, wo, np.where(np.isfinite(wl), wl, 0), w)
    assert np.array_equal(np.isneginf(lse), np.isneginf(wl)), f"{what}: rows that see nothing differ"
    fin = np.isfinite(wl)
    eo, el = np.abs(o - wo) / to, np.abs(lse[fin] - wl[fin]) / tl[fin]
    print(f"[parity] {what}: o {eo.max(initial=0):.3g}, lse {el.max(initial=0):.3g} of the tolerance", flush=True)
    assert np.all(np.isfinite(o)) and eo.max(initial=0) <= 1, f"{what}: o off at {np.unravel_index(np.argmax(eo), eo.shape)}"
    assert el.max(initial=0) <= 1, f"{what}: lse off"
