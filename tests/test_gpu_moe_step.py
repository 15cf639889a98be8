"""The operators together, as a mixture-of-experts layer and its training step
use them: router, dispatch, the MoE plans' products, combination; the
gradients back to logits and tokens; clipping into the AdamW plan's flat
gradient.  And as captured graphs, and on other streams."""
import threading

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2608_13757_amd as bfsp  # noqa: E402
from oracle.mathref import adamw_step  # noqa: E402
from paper_2608_13757_amd import GradSet, Plan, bfs  # noqa: E402
from paper_2608_13757_amd.ops import DISPATCH_ALONE  # noqa: E402
from tests.gpu_util import trip_tensors  # noqa: E402
from workloads import ADAM_HP, adamw_default_wg, adamw_program, adamw_worklist, moe_program, moe_worklist  # noqa: E402

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
RTOL = 2e-2           # the MoE plans' bar: bf16 products, h rounded between them


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    bfs.lib()


def _normal(seed, shape, dtype=torch.float32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dtype).cuda()


def _experts_products(rows_of, off, weights, n_rows, x, hidden, ffn, bm):
    """The two launches of the MoE plans over rows grouped by expert: row i
    gathers x[rows_of[i]], the result stays in grouped order."""
    wg, wu, wd = weights
    counts = np.diff(off.cpu().numpy())
    identity = torch.arange(n_rows, dtype=torch.int32, device="cuda")
    h = torch.zeros((n_rows, ffn), dtype=torch.bfloat16, device="cuda")
    y = torch.zeros((n_rows, hidden), dtype=torch.bfloat16, device="cuda")
    for phase, perm, data in ((1, rows_of, [x, wg, wu, h]), (2, identity, [h, wd, y])):
        wl = moe_worklist(counts, phase, hidden, ffn, bm=bm)
        trips, toff = trip_tensors(wl.trips)
        plan = Plan(moe_program(phase, hidden, ffn, bm=bm))
        plan.run([torch.from_numpy(wl.work.reshape(-1)).cuda(), perm, off, *data], trips, toff, wl.trips.n_wg)
        plan.status()
    return h, y


@pytest.mark.parametrize("t,e,k,bm", [(300, 5, 2, 128), (130, 8, 3, 256), (700, 4, 1, 256)])
def test_layer_forward(t, e, k, bm):
    hidden, ffn = 256, 256
    x, logits = _normal(1, (t, hidden), torch.bfloat16), _normal(2, (t, e), torch.bfloat16)
    logits[5] = logits[t - 1] = float("-inf")                       # padding: no expert
    logits[:, 1] = float("-inf")                                    # an expert without tokens
    weights = [_normal(3 + i, (e, ffn, hidden) if i < 2 else (e, hidden, ffn), torch.bfloat16, 0.05) for i in range(3)]
    experts, w = bfsp.moe_route(logits, k)
    perm, off, pos, rows = bfsp.moe_dispatch(experts, e, x)
    n = int(off[-1])
    assert n == (t - 2) * k and int(off[2]) == int(off[1])
    # rows gathered by the plan through perm, and rows laid out by the dispatch
    h, out = _experts_products(perm, off, weights, n, x, hidden, ffn, bm)
    identity = torch.arange(n, dtype=torch.int32, device="cuda")
    h2, out2 = _experts_products(identity, off, weights, n, rows, hidden, ffn, bm)
    assert torch.equal(h, h2) and torch.equal(out, out2)
    y = bfsp.moe_combine(out, pos, w)
    ref = np.zeros((t, hidden))
    xs, (wg, wu, wd) = x.double().cpu().numpy(), [v.double().cpu().numpy() for v in weights]
    ids, ww = experts.cpu().numpy(), w.double().cpu().numpy()
    for i in range(t):
        for j in range(k):
            if ids[i, j] >= 0:
                a, b = wg[ids[i, j]] @ xs[i], wu[ids[i, j]] @ xs[i]
                ref[i] += ww[i, j] * (wd[ids[i, j]] @ (a / (1 + np.exp(-a)) * b))
    err = np.abs(y.double().cpu().numpy() - ref) / np.maximum(np.abs(ref), np.sqrt((ref ** 2).mean()))
    assert err.max() <= RTOL and (y[5] == 0).all()


@pytest.mark.parametrize("renorm", [True, False])
def test_training_step(renorm):
    """A layer whose experts scale their rows, y = sum_j w_j s[e_j] x, with a
    linear router: all gradients against autograd of the dense form in 64
    bits, then clipped and applied by the AdamW plan."""
    t, e, k, hidden = 200, 12, 3, 64
    x, wr, s = _normal(1, (t, hidden)), _normal(2, (e, hidden), scale=0.3), _normal(3, (e,)) + 2.0
    dy = _normal(4, (t, hidden))
    logits = (x.double() @ wr.double().t()).float()
    experts, w = bfsp.moe_route(logits, k, renormalize=renorm)
    perm, off, pos, rows = bfsp.moe_dispatch(experts, e, x)
    of_row = torch.repeat_interleave(torch.arange(e, device="cuda"), off.diff().long())
    ys = rows * s[of_row, None]
    y = bfsp.moe_combine(ys, pos, w)
    dys, dw = bfsp.moe_combine_grad(dy, ys, pos, w)
    ds = torch.zeros(e, device="cuda").index_add_(0, of_row, (dys * rows).sum(1))
    dx = bfsp.moe_dispatch_grad(dys * s[of_row, None], pos)
    dlogits = bfsp.moe_route_grad(logits, experts, dw, renormalize=renorm)
    dwr = dlogits.t().contiguous() @ x
    # the dense form
    x64, s64, z64 = (v.double().cpu().requires_grad_() for v in (x, s, logits))
    p = torch.softmax(z64, 1)
    sel = torch.gather(p, 1, experts.cpu().long())
    w64 = sel / sel.sum(1, keepdim=True) if renorm else sel
    y64 = (w64 * s64[experts.cpu().long()]).sum(1, keepdim=True) * x64
    y64.backward(dy.double().cpu())
    # sums of up to k * hidden products of numbers of a few units in fp32, each
    # term at most 8 times the result's scale: 8 (k hidden + 64) u of the scale
    tol = 8 * (k * hidden + 64) * U
    for got, ref in ((y, y64), (dx, x64.grad), (dlogits, z64.grad), (ds, s64.grad)):
        ref = ref.detach().numpy()
        # ds sums over about t * k / e tokens
        scale = np.abs(ref).max() * (t if got is ds else 1)
        assert np.abs(got.double().cpu().numpy() - ref).max() <= tol * scale
    # clip into the flat gradient, then one AdamW step on it
    n = e * hidden + e
    flat = torch.zeros(n, device="cuda")
    norm = GradSet([dwr, ds], out=flat).clip(1.0)
    g64 = torch.cat([dwr.reshape(-1), ds]).double().cpu().numpy()
    ref_norm = np.sqrt((g64 ** 2).sum())
    assert abs(float(norm) - ref_norm) <= 2 * U * ref_norm
    clipped = g64 * min(1.0, 1.0 / (ref_norm + 1e-6))
    assert np.abs(flat.double().cpu().numpy() - clipped).max() <= 4 * U * np.abs(clipped).max()
    par = torch.cat([wr.reshape(-1), s])
    m, v = _normal(5, (n,), scale=0.01), _normal(6, (n,), scale=0.01).square()
    hp = ADAM_HP
    ref = adamw_step(*(a.cpu().numpy() for a in (par, flat, m, v)),
                     *(hp[q] for q in ("lr", "b1", "b2", "eps", "wd", "t")))
    n_wg = adamw_default_wg(n, 256)
    base, tt = adamw_worklist(n, 256, n_wg)
    trips, toff = trip_tensors(tt)
    plan = Plan(adamw_program(n, 256, **hp))
    plan.run([torch.from_numpy(base).cuda(), par, flat, m, v], trips, toff, n_wg)
    plan.status()
    for got, want in zip((par, m, v), ref):
        assert np.abs(got.double().cpu().numpy() - want).max() <= 1e-5


class _Step:
    """Every operator once, on buffers that stay."""

    def __init__(self, t, e, k, h, dtype, seed=0):
        self.k, self.e = k, e
        self.logits, self.x, self.dy = _normal(seed, (t, e), dtype), _normal(seed + 1, (t, h), dtype), _normal(seed + 2, (t, h), dtype)
        self.grads = [_normal(seed + 3, (n,), torch.float32) for n in (4000, 17, 30000)]
        self.flat = torch.empty(34017, device="cuda")
        self.set = GradSet(self.grads, out=self.flat)

    def refill(self, seed):
        for i, a in enumerate((self.logits, self.x, self.dy, *self.grads)):
            a.copy_(_normal(seed * 100 + i, a.shape, a.dtype))
        self.logits[0] = float("-inf")

    def run(self):
        experts, w = bfsp.moe_route(self.logits, self.k)
        perm, off, pos, rows = bfsp.moe_dispatch(experts, self.e, self.x)
        rows[self.dy.shape[0] * self.k - self.k:] = 0.0           # the rows that padding leaves unwritten
        perm[self.dy.shape[0] * self.k - self.k:] = 0
        y = bfsp.moe_combine(rows, pos, w)
        drows, dw = bfsp.moe_combine_grad(self.dy, rows, pos, w)
        dx = bfsp.moe_dispatch_grad(drows, pos)
        dz = bfsp.moe_route_grad(self.logits, experts, dw)
        norm = self.set.clip(1.0)
        return [experts, w, perm, off, pos, rows, y, drows, dw, dx, dz, self.flat.clone(), norm]


@pytest.mark.parametrize("t,e,k,h,dtype", [(9, 16, 2, 64, torch.bfloat16), (3000, 64, 4, 136, torch.float16),
                                           (600, 300, 2, 77, torch.float32)])
def test_captured_and_replayed(t, e, k, h, dtype):
    """Two graphs of the same sizes, replayed in turn with eager work between
    and new inputs each time: every replay equals the eager calls."""
    steps = [_Step(t, e, k, h, dtype), _Step(t, e, k, h, dtype, seed=50)]
    graphs, outs = [], []
    for s in steps:
        s.refill(1)
        s.run()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(s.run())
        graphs.append(g)
    for n in range(4):
        for i, s in enumerate(steps):
            s.refill(10 * n + i + 2)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for s, got in zip(steps, outs):
            for q, (a, b) in enumerate(zip(got, s.run())):
                assert torch.equal(a, b), (n, q)


def test_two_streams_at_once():
    """Two streams with their own buffers, and a stream given by argument with
    every output."""
    steps = [_Step(2500, 64, 2, 256, torch.bfloat16, seed=7 * i) for i in range(2)]
    for i, s in enumerate(steps):
        s.refill(i + 1)
    want = [s.run() for s in steps]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [None, None]
    for _ in range(3):
        for i, (s, st) in enumerate(zip(steps, streams)):
            with torch.cuda.stream(st):
                got[i] = s.run()
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert all(torch.equal(p, q) for p, q in zip(a, b))
    s, st = steps[0], streams[1]
    out = [torch.zeros_like(v) for v in want[0]]
    ws = torch.empty(bfsp.moe_dispatch_workspace(2500, 2, 64), dtype=torch.uint8, device="cuda")
    gs = GradSet(s.grads, out=out[11])
    gw = torch.empty(gs.workspace_bytes, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    bfsp.moe_route(s.logits, 2, experts=out[0], weights=out[1], stream=st)
    bfsp.moe_dispatch(out[0], 64, s.x, perm=out[2], expert_off=out[3], pos=out[4], rows=out[5], workspace=ws, stream=st)
    bfsp.moe_combine(out[5], out[4], out[1], out=out[6], stream=st.cuda_stream)
    bfsp.moe_combine_grad(s.dy, out[5], out[4], out[1], grad_rows=out[7], grad_weights=out[8], stream=st)
    bfsp.moe_dispatch_grad(out[7], out[4], out=out[9], stream=st)
    bfsp.moe_route_grad(s.logits, out[0], out[8], grad_logits=out[10], stream=st)
    gs.clip(1.0, norm=out[12], workspace=gw, stream=st)
    st.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(out, want[0]))


def test_two_threads_at_once():
    """Two host threads, each with its own stream and buffers; the set of
    gradients is shared, its calls read it only."""
    steps = [_Step(1200, 32, 4, 192, torch.bfloat16, seed=9 * i) for i in range(2)]
    for i, s in enumerate(steps):
        s.refill(i + 3)
    shared = GradSet(steps[0].grads)
    want = [s.run() + [shared.norm()] for s in steps]
    torch.cuda.synchronize()
    got, errors = [None, None], []

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(20):
                    got[i] = steps[i].run() + [shared.norm()]
                torch.cuda.current_stream().synchronize()
        except Exception as e:          # noqa: BLE001
            errors.append(e)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors
    for a, b in zip(got, want):
        assert all(torch.equal(p, q) for p, q in zip(a, b))


# Dispatches that work in a table of counts; of the second a launch of its own sums it.
WITH_TABLE = [dict(t=6000, e=64, k=2, h=128, dtype=torch.bfloat16), dict(t=9000, e=300, k=3, h=72, dtype=torch.float16)]


def _with_table(t, e, k, **_):
    assert t * k > DISPATCH_ALONE and bfsp.moe_dispatch_workspace(t, k, e) > 0
    return -(-t // (1024 // k)) * e                    # counts of the table


def test_tables_of_counts_on_two_streams():
    """The calls' own workspaces, and one for each stream given by argument."""
    assert _with_table(**WITH_TABLE[0]) <= 4096 < _with_table(**WITH_TABLE[1])
    for sizes in (WITH_TABLE, WITH_TABLE[::-1], WITH_TABLE[1:] * 2):
        steps = [_Step(**z, seed=11 * i) for i, z in enumerate(sizes)]
        for i, s in enumerate(steps):
            s.refill(i + 1)
        want = [s.run() for s in steps]
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        tables = [torch.full((bfsp.moe_dispatch_workspace(z["t"], z["k"], z["e"]),), 0xff, dtype=torch.uint8, device="cuda") for z in sizes]
        outs = [[torch.zeros_like(v) for v in w[2:6]] for w in want]
        torch.cuda.synchronize()
        got = [None, None]
        for _ in range(4):
            for i, (s, st) in enumerate(zip(steps, streams)):
                with torch.cuda.stream(st):
                    got[i] = s.run()
                perm, off, pos, rows = outs[i]
                bfsp.moe_dispatch(want[i][0], s.e, s.x, perm=perm, expert_off=off, pos=pos, rows=rows, workspace=tables[i], stream=st)
        torch.cuda.synchronize()
        for a, b, c in zip(got, want, outs):
            assert all(torch.equal(p, q) for p, q in zip(a, b))
            n = int(b[3][-1])
            assert 0 < n == b[4].numel() - int((b[4] < 0).sum())
            assert torch.equal(c[1], b[3]) and torch.equal(c[2], b[4]) and torch.equal(c[0][:n], b[2][:n]) and torch.equal(c[3][:n], b[5][:n])


def test_tables_of_counts_in_two_threads():
    """Two host threads, each with its own stream and buffers."""
    steps = [_Step(**z, seed=9 * i) for i, z in enumerate(WITH_TABLE)]
    for i, (s, z) in enumerate(zip(steps, WITH_TABLE)):
        _with_table(**z)
        s.refill(i + 3)
    want = [s.run() for s in steps]
    torch.cuda.synchronize()
    got, errors = [None, None], []

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(20):
                    got[i] = steps[i].run()
                torch.cuda.current_stream().synchronize()
        except Exception as e:          # noqa: BLE001
            errors.append(e)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors
    for a, b in zip(got, want):
        assert all(torch.equal(p, q) for p, q in zip(a, b))


@pytest.mark.parametrize("sizes", WITH_TABLE, ids=lambda z: f"{z['t']}x{z['k']}")
def test_tables_of_counts_captured(sizes):
    """Two graphs whose dispatches have a table each, replayed in turn and on
    two streams at once, with new inputs each time."""
    _with_table(**sizes)
    steps = [_Step(**sizes), _Step(**sizes, seed=50)]
    graphs, outs = [], []
    for s in steps:
        s.refill(1)
        s.run()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(s.run())
        graphs.append(g)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for n in range(4):
        for i, s in enumerate(steps):
            s.refill(10 * n + i + 2)
        torch.cuda.synchronize()
        for g, st in zip(graphs, streams):
            if n % 2:
                with torch.cuda.stream(st):
                    g.replay()
            else:
                g.replay()
        torch.cuda.synchronize()
        for s, got in zip(steps, outs):
            for q, (a, b) in enumerate(zip(got, s.run())):
                assert torch.equal(a, b), (n, q)
