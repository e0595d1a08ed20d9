"""Outputs that a call allocates, where the context's stream is not torch's current one: nothing that the current
stream still does reaches them."""
import numpy as np
import pytest
import torch

from oracle import packed as O
from tests.packed_util import PackedBatch
from tests.serving_util import Batch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ckv():
    """A context on a stream of its own, and the current stream kept busy for half a second on demand."""
    import paper_2608_07855_amd as P
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    torch.cuda._sleep(1000)
    a.record()
    torch.cuda._sleep(100000)
    b.record()
    b.synchronize()
    cycles = int(100000 * 500 / a.elapsed_time(b))

    def busy():
        torch.cuda._sleep(cycles)
        e = torch.cuda.Event()
        e.record()
        return e
    # streams share a few hardware queues: one that does not wait behind the current stream's
    x = torch.zeros(1, device="cuda")
    for stream in [torch.cuda.Stream() for _ in range(6)]:
        torch.cuda.synchronize()
        running = busy()
        with torch.cuda.stream(stream):
            x.add_(1)
        stream.synchronize()
        if not running.query():
            break
    ctx = P.Context(0, stream)
    yield P, ctx, busy
    torch.cuda.synchronize()
    ctx.close()


def _calls(P, ctx):
    """Calls that allocate their outputs, by name; inputs are in place."""
    wide, packed = Batch(1, [200, 30], [1, 20], 4, 2, 64), PackedBatch(1, [200, 30], [1, 20], 4, 2, 64)
    w, p = wide.device(P), packed.device(P)
    score = torch.rand((2, 500), device="cuda")
    R = [torch.rand(40, device="cuda") for _ in range(2)]
    n_pages, hkv, S, d = 12, 2, 200, 64
    g = torch.Generator().manual_seed(0)
    k, v = (torch.randn((hkv, S, d), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    pos = torch.arange(S, dtype=torch.int32, device="cuda")
    q = torch.randn((4, 8, d), generator=g).to(torch.bfloat16).cuda()
    qpos = torch.arange(S - 8, S, dtype=torch.int32, device="cuda")
    kv, win, pages = P.kv_view(k, v, pos, S), P.window_view(q, qpos), P.Pages(np.arange(n_pages) * 16, [16] * n_pages)
    state = torch.rand((1, S), device="cuda")
    none = [P.Pages([], [])]
    return dict(
        unpack=lambda: P.ckv_unpack_tokens(ctx, p["kv"]),
        attend_packed=lambda: P.ckv_attend_packed(ctx, p["kv"], p["q"], want=("o", "lse")),
        attend_window=lambda: P.ckv_attend_window(ctx, w["kv"], w["q"], want=("o", "lse")),
        pool_scores=lambda: dict(out=P.ckv_pool_scores(ctx, score, [500, 77])),
        classify=lambda: P.ckv_classify_pages(ctx, *R),
        measure=lambda: P.ckv_measure_page_effects(ctx, kv, win, pages, want=("R", "R_head", "o", "lse", "token_mass")),
        batch=lambda: P.ckv_measure_page_effects_batch(ctx, [kv] * 2, [win] * 2, [pages] * 2, want=("R", "o"))[1],
        select=lambda: P.ckv_select_and_compact(ctx, k[None, None], v[None, None], pos[None], [S], state, none, none, [None],
                                                budget=50, keep_recent=8))


NAMES = ["unpack", "attend_packed", "attend_window", "pool_scores", "classify", "measure", "batch", "select"]


def _host(out):
    return {name: x.cpu() for name, x in out.items() if x is not None}


@pytest.mark.parametrize("name", NAMES)
def test_outputs_beside_a_busy_stream(ckv, name):
    """Memory that a fill under way on the current stream still writes is not handed out; no fill of the call's own
    waits behind that stream's work and runs over the outputs."""
    P, ctx, busy = ckv
    call = _calls(P, ctx)[name]
    torch.cuda.synchronize()
    out = call()
    ctx.sync()
    torch.cuda.synchronize()
    want, sizes = _host(out), [(x.untyped_storage().nbytes(), x.dtype) for x in out.values() if x is not None]
    # where outputs may lie next: blocks of the current stream's, freed with a fill of them still to come
    old = [torch.empty(n, dtype=torch.uint8, device="cuda") for n, _ in sizes for _ in range(2)]
    del out
    torch.cuda.synchronize()
    running = busy()
    for x in old:
        x.fill_(0x3C)
    del old, x
    out = call()
    ctx.sync()
    print(f"[streams] {name}: the current stream was {'through' if running.query() else 'busy still'}", flush=True)
    torch.cuda.synchronize()
    got = _host(out)
    for key, x in want.items():
        # (bytes: nothing that a fill left, and zeros where zeros belong)
        assert torch.equal(got[key].contiguous().view(torch.uint8), x.contiguous().view(torch.uint8)), key


def test_outputs_of_a_stream_given_by_its_handle(ckv):
    """The same with a stream that torch knows by its handle only, the default stream, and a changed one."""
    P, _, busy = ckv
    side = torch.cuda.Stream()
    rows = O.pack(*np.random.default_rng(0).standard_normal((2, 9, 1, 64)).astype(np.float32))
    want = torch.from_numpy(O.unpack(rows)[0].astype(np.float32)).to(torch.bfloat16).transpose(0, 1)
    pool = torch.from_numpy(rows.transpose(1, 0, 2).copy()).cuda()
    slot, lens = torch.arange(12, dtype=torch.int32, device="cuda")[None] % 9, torch.tensor([9], dtype=torch.int32, device="cuda")
    for ctx, here in ((P.Context(0, side.cuda_stream), torch.cuda.default_stream()), (P.Context(0, 0), side)):
        kv = P.packed_view(pool, lens, slot=slot)
        for _ in range(2):
            torch.cuda.synchronize()
            with torch.cuda.stream(here):
                busy()
                out = P.ckv_unpack_tokens(ctx, kv)
                ctx.sync()
            torch.cuda.synchronize()
            assert torch.equal(out["k"][0, :, :9].cpu(), want) and not out["k"][0, :, 9:].any()
            ctx.set_stream(torch.cuda.Stream())
        ctx.close()
