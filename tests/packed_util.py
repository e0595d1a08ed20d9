"""Batches whose caches are held in 4 bits: the oracle's rows in a pool, and the comparison with the oracle."""
import numpy as np
import torch

from oracle import packed as O
from tests.serving_util import HALF, TYPES, Batch


class PackedBatch(Batch):
    """A Batch whose keys and values are what its packed rows stand for.  ``fill``: the byte that storage of no token
    holds (0xFF: NaN scales and bases)."""

    def __init__(self, *args, value_scale=1.0, **kw):
        super().__init__(*args, **kw)
        assert not self.prefix
        self.bytes = []
        for s in range(self.n):
            rows = O.pack(self.k[s].float().numpy(), self.v[s].float().numpy() * np.float32(value_scale))
            self.bytes.append(rows)
            self.k[s], self.v[s] = (torch.from_numpy(x) for x in O.unpack(rows))

    def set_rows(self, s, at, rows):
        """Rows [t, Hkv, row bytes] for tokens ``at`` of sequence s."""
        self.bytes[s][at] = rows
        k, v = O.unpack(rows)
        self.k[s][at], self.v[s][at] = torch.from_numpy(k), torch.from_numpy(v)

    def device(self, P, fill=0xFF, max_rows=None):
        rb, dev = O.row_bytes(self.d), "cuda"
        slot = None
        if self.paged:
            place, at = self.rng.permutation(self.pool), 0
            pool = np.full((self.hkv, self.pool, rb), fill, np.uint8)
            slot = np.full((self.n, self.most), -7, np.int32)
            for s in range(self.n):
                r = place[at:at + self.lens[s]]
                at += int(self.lens[s])
                pool[:, r] = self.bytes[s].transpose(1, 0, 2)
                slot[s, :self.lens[s]] = r
            slot = torch.from_numpy(slot).to(dev)
        else:
            pool = np.full((self.n, self.hkv, self.most, rb), fill, np.uint8)
            for s in range(self.n):
                pool[s, :, :self.lens[s]] = self.bytes[s].transpose(1, 0, 2)
        pos = None
        if self.pos is not None:
            pos = np.full((self.n, self.most), 2**31 - 1, np.int32)
            for s in range(self.n):
                pos[s, :self.lens[s]] = self.pos[s]
            pos = torch.from_numpy(pos).to(dev)
        lens = torch.from_numpy(self.lens.astype(np.int32)).to(dev)
        kv = P.packed_view(torch.from_numpy(pool).to(dev), lens, slot=slot, pos=pos, max_tokens=self.most)
        t = TYPES[self.type]
        q = torch.cat([torch.zeros((self.lead, self.hq, self.d), dtype=t)] + self.q +
                      [torch.zeros((self.tail, self.hq, self.d), dtype=t)]).to(dev)
        cu = torch.from_numpy((self.lead + np.concatenate([[0], np.cumsum(self.rows)])).astype(np.int32)).to(dev)
        qpos = None
        if self.given_qpos is not None:
            qpos = np.concatenate([np.zeros(self.lead)] + [np.asarray(x) for x in self.given_qpos] + [np.zeros(self.tail)])
            qpos = torch.from_numpy(qpos.astype(np.int32)).to(dev)
        return dict(kv=kv, q=P.query_view(q, cu, qpos, max_rows=max_rows or max(1, int(self.rows.max(initial=1))),
                                          scale=0.0 if self.scale is None else self.scale))

    def run(self, P, ctx, views, window=0, n_sink=0, fill=7.0):
        t, total = TYPES[self.type], int(self.rows.sum()) + self.lead + self.tail
        o = torch.full((total, self.hq, self.d), fill, dtype=t, device="cuda")
        lse = torch.full((total, self.hq), fill, dtype=torch.float32, device="cuda")
        P.ckv_attend_packed(ctx, views["kv"], views["q"], window=window, n_sink=n_sink, o=o, lse=lse)
        ctx.sync()
        o, lse = o.cpu().double().numpy(), lse.cpu().double().numpy()
        mine = slice(self.lead, total - self.tail)
        rest = np.ones(total, bool)
        rest[mine] = False
        assert np.all(o[rest] == fill) and np.all(lse[rest] == fill), "rows of no sequence were written"
        return o[mine], lse[mine]


def tolerances(b, o, lse, w):
    """|o| is rounded once to the output's type (half a step) and each softmax weight once to fp16 (2^-11 of it; formed
    2^13 times as large at least, a weight below fp16's normal numbers is off by 2^-38).  A bf16 query element below
    2^-29 of its row's largest is off by 2^-40 of that: nothing here.  float32 logits: d products and a sum each off
    by 2^-24 of sum |q k| (below 2^6 here), and the exponential and the sums: 2^-13 in all, relative to the weights and
    absolute in lse."""
    vmax = max((float(x.abs().nan_to_num(0).max()) for x in b.v if x.numel()), default=0.0)
    tiny = int(b.lens.max(initial=0)) * 2.0**-38 * vmax
    return HALF[b.type] * np.abs(o) + (2.0**-11 + 2.0**-13) * w + tiny + 2.0**-24, 2.0**-13 + 2.0**-22 * np.abs(lse)


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
