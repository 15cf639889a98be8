"""The router, dispatch and combination of a mixture of experts and their
gradients, against their definitions in 64 bits.

Bounds, with u = 2^-24 and h = half a step of the result's type (eps / 2):

* softmax weights (fp32): exp's argument z - m is rounded once (relative
  error |z - m| u of the exponential), expf is within 2 steps (4 u), the sum
  of E positive terms within (E / 16 + 8) u (16 or more lanes add in
  parallel; 6 joining steps, at most 16 in a lane), the division and the
  final value 2 u: (|z - m| + E / 16 + 20) u, with a factor 2 for the second
  order and the terms' own errors in the sum.
* router gradient: p_i (d_i - s), s = sum of k products p g.  With G = the
  largest |g|: |d_i| <= k G and |s| <= G, each with the weights' relative
  error r and k + 2 roundings: |error| <= p_i (k + 1) G (3 r + (k + 4) u),
  then h of the rounded result.
* combination: k products and k - 1 sums in fp32: (k + 1) u sum |w r|, h.
* its gradient: rows one product and one rounding: (u + h) |w g|; weights a
  dot product of H terms, H / 64 in a lane and 6 joining steps:
  (H / 64 + 16) u sum |g r| (lanes hold up to 8 terms more in a last chunk).
* results below the type's smallest normal number: half its smallest step.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2608_13757_amd as bfsp  # noqa: E402
from paper_2608_13757_amd import BfsError, bfs  # noqa: E402

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DTYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    bfs.lib()


def _f64(t):
    return t.detach().double().cpu().numpy()


def _close(got, ref, bound, dtype=torch.float32):
    """|got - ref| <= bound + half a step of the type."""
    fi = torch.finfo(dtype)
    got = _f64(got)
    err = np.abs(got - ref)
    # (a value past the largest finite one by less than half its step would round to it)
    allowed = bound + fi.eps / 2 * (np.abs(ref) + bound) + fi.tiny * fi.eps / 2
    bad = ~(err <= allowed)
    assert not bad.any(), (np.argwhere(bad)[:4].tolist(), got[bad][:4], ref[bad][:4], allowed[bad][:4])


def _normal(seed, shape, dtype=torch.float32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dtype).cuda()


def _padded(t, pad):
    """The same values in longer rows, starting one element in."""
    if not pad:
        return t
    buf = torch.full((t.shape[0], t.shape[1] + pad), float("nan"), dtype=t.dtype, device="cuda")
    buf[:, 1:1 + t.shape[1]] = t
    return buf[:, 1:1 + t.shape[1]]


def _guarded(shape, dtype, pad):
    """An output inside a larger buffer of sentinels, and the buffer."""
    buf = torch.full((shape[0] + 2, shape[1] + pad), 77, dtype=dtype, device="cuda")
    lo = 1 if pad else 0
    return buf[1:-1, lo:lo + shape[1]], buf


def _untouched(buf, view):
    view.fill_(77)
    return bool((buf == 77).all())


# ---------------------------------------------------------------------------
# router
# ---------------------------------------------------------------------------
def _route_reference(z, k, renorm):
    """Experts and weights by the definition; z float64 without NaN."""
    t, e = z.shape
    order = np.argsort(-z, axis=1, kind="stable")[:, :k]
    top = np.take_along_axis(z, order, axis=1)
    m = np.where(np.isneginf(z.max(axis=1)), 0.0, z.max(axis=1))[:, None]
    w = np.exp(top - m)
    total = w.sum(1) if renorm else np.exp(z - m).sum(1)
    experts = np.where(np.isneginf(top), -1, order)
    return experts, np.where(experts < 0, 0.0, w / np.where(total == 0, 1, total)[:, None]), top - m


SHAPES = [(1, 1, 1), (1, 64, 8), (3, 2, 2), (17, 16, 4), (5, 17, 16), (33, 31, 3), (64, 64, 2), (100, 65, 8), (7, 127, 16),
          (50, 128, 1), (9, 200, 5), (31, 256, 8), (6, 257, 8), (4, 500, 16), (13, 512, 6), (3, 777, 9), (2, 1024, 16)]


@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("t,e,k", SHAPES)
def test_route(t, e, k, dtype, renorm):
    z = _padded(_normal(t * e, (t, e), dtype, 3.0), 3 if e % 2 else 0)
    experts, weights = bfsp.moe_route(z, k, renormalize=renorm)
    ref_e, ref_w, arg = _route_reference(_f64(z), k, renorm)
    assert experts.dtype == torch.int32 and np.array_equal(experts.cpu().numpy(), ref_e)
    _close(weights, ref_w, 2 * (np.abs(arg) + e / 16 + 20) * U * ref_w)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("e", [7, 64, 300])
def test_route_ties_and_masks(e, dtype):
    """Equal logits (also -0 and 0) go to the lower index; masked experts are
    never chosen, rows with fewer than k left hold -1, also with logits of the
    type's lowest value, which is not a mask."""
    k, n = 6, 40
    g = torch.Generator().manual_seed(e)
    z = torch.randint(-1, 2, (n, e), generator=g).float() * 0.0                  # 0 and -0
    z[10:20] = torch.randint(0, 3, (10, e), generator=g).float()
    z[20:30] = torch.where(torch.rand((10, e), generator=g) < 0.9, float("-inf"), z[10:20])
    z[30:36] = torch.finfo(dtype).min
    z[33:36, 2:] = float("-inf")
    z[36:] = float("-inf")
    z[37, e - 1] = -5.0
    z = z.to(dtype).cuda()
    for renorm in (True, False):
        experts, weights = bfsp.moe_route(z, k, renormalize=renorm)
        ref_e, ref_w, arg = _route_reference(_f64(z), k, renorm)
        assert np.array_equal(experts.cpu().numpy(), ref_e)
        arg = np.where(ref_e < 0, 0.0, arg)
        _close(weights, ref_w, 2 * (np.abs(arg) + e / 16 + 20) * U * ref_w)
        assert (weights[experts < 0] == 0).all() and (experts[36] == -1).all()


@pytest.mark.parametrize("t,e,k", [(40, 65, 3), (64, 128, 8), (33, 256, 4), (50, 256, 16), (21, 300, 8), (13, 512, 16), (9, 1024, 5),
                                   (16, 100, 16), (40, 64, 8)])
@pytest.mark.parametrize("kind", ["steps", "ties", "few", "bf16", "masked"])
def test_route_close_logits(t, e, k, kind):
    """fp32 logits that differ in their last bits, or not at all, among the
    chosen ones and at their border, in some rows or in all."""
    g = torch.Generator().manual_seed(e * k)
    z = torch.randn((t, e), generator=g) * 3.0
    step = torch.randint(0, 6, (t, e), generator=g, dtype=torch.int32)
    if kind == "steps":                                # all within a few steps of one value, of either sign
        z = (torch.full((t, e), 1.5).view(torch.int32) + step).view(torch.float32) * torch.where(torch.arange(t) % 2 == 0, 1.0, -1.0)[:, None]
    elif kind == "ties":                               # large ones all equal, more or fewer than k
        z = torch.where(torch.rand((t, e), generator=g) < torch.rand((t, 1), generator=g) * 2 * k / e, torch.tensor(9.25), z)
    elif kind == "few":                                # every seventh row has three near-equal largest ones, out of order
        i = torch.arange(0, t, 7)
        for n, (c, d) in enumerate(((e - 1, 2), (e // 2, 1), (0, 3))):
            z[i, c] = (torch.tensor([11.0]).view(torch.int32) + d).view(torch.float32)
    elif kind == "bf16":
        z = z.bfloat16().float()
    else:
        z = torch.where(torch.rand((t, e), generator=g) < 0.97, torch.tensor(float("-inf")), z)
        z[::3] = torch.where(step[::3] > 2, torch.tensor(torch.finfo(torch.float32).min), torch.tensor(-float("inf")))
    z = z.cuda()
    for renorm in (True, False):
        experts, weights = bfsp.moe_route(z, k, renormalize=renorm)
        ref_e, ref_w, arg = _route_reference(_f64(z), k, renorm)
        assert np.array_equal(experts.cpu().numpy(), ref_e)
        arg = np.where(ref_e < 0, 0.0, arg)
        _close(weights, ref_w, 2 * (np.abs(arg) + e / 16 + 20) * U * ref_w)


@pytest.mark.parametrize("e", [64, 256, 600])
def test_route_nan_and_inf(e):
    """NaN ranks above everything and makes its token's weights NaN; +inf
    does so too; other tokens are not touched by it."""
    z = _normal(1, (8, e))
    clean = bfsp.moe_route(z, 4)
    z[2, 7] = float("nan")
    z[3, 9] = -float("nan")
    z[4, 11] = float("inf")
    experts, weights = bfsp.moe_route(z, 4)
    assert experts[2, 0] == 7 and experts[3, 0] == 9 and experts[4, 0] == 11
    assert weights[2:5, 0].isnan().all()
    keep = [0, 1, 5, 6, 7]
    assert torch.equal(experts[keep], clean[0][keep]) and torch.equal(weights[keep], clean[1][keep])


def _route_grad_reference(z, experts, dw, renorm):
    t, e = z.shape
    dz, err = np.zeros_like(z), np.zeros_like(z)
    for i in range(t):
        kept = [(j, x) for j, x in enumerate(experts[i]) if 0 <= x < e]
        big = max([abs(dw[i, j]) for j, _ in kept], default=0.0)
        if renorm:
            zz = np.array([z[i, x] for _, x in kept])
            m = max(zz, default=0.0)
            p = np.exp(zz - (0.0 if np.isneginf(m) else m))
            p = p / (p.sum() or 1.0)
            s = sum(p[n] * dw[i, j] for n, (j, _) in enumerate(kept))
            for n, (j, x) in enumerate(kept):
                dz[i, x] += p[n] * (dw[i, j] - s)
                err[i, x] += p[n] * big
        else:
            m = z[i].max()
            p = np.exp(z[i] - (0.0 if np.isneginf(m) else m))
            p = p / (p.sum() or 1.0)
            d = np.zeros(e)
            for j, x in kept:
                d[x] += dw[i, j]
            dz[i] = p * (d - (p * d).sum())
            err[i] = p * big
    return dz, err


@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("t,e,k", SHAPES)
def test_route_grad(t, e, k, dtype, renorm):
    z = _padded(_normal(t * e, (t, e), dtype, 2.0), 5 if e % 2 else 0)
    experts, _ = bfsp.moe_route(z, k, renormalize=renorm)
    if t > 4:
        experts[1, k - 1] = -1                        # a slot without an expert
        experts[2] = -1                               # a token without any
        experts[3, k - 1] = experts[3, 0]             # the same expert twice
        experts[4, 0] = e                             # out of range: none
    dw = _normal(k, (t, k))
    out, buf = _guarded((t, e), dtype, 2 if e % 2 else 0)
    assert bfsp.moe_route_grad(z, experts, dw, renormalize=renorm, grad_logits=out) is out
    ref, p_big = _route_grad_reference(_f64(z), experts.cpu().numpy(), _f64(dw), renorm)
    span = np.abs(_f64(z)).max() * 2
    r = 2 * (span + e / 16 + 20) * U
    _close(out, ref, p_big * (k + 1) * (3 * r + (k + 4) * U), dtype)
    assert _untouched(buf, out)


def test_route_grad_masked_row():
    """A row whose mask leaves nothing, and masked experts, have zero gradients."""
    z = _normal(5, (4, 32))
    z[1] = float("-inf")
    z[2, :20] = float("-inf")
    experts, _ = bfsp.moe_route(z, 3, renormalize=False)
    dw = _normal(6, (4, 3))
    for renorm in (True, False):
        dz = bfsp.moe_route_grad(z, experts, dw, renormalize=renorm)
        assert torch.isfinite(dz).all() and (dz[1] == 0).all() and (dz[2, :20] == 0).all()
        # experts forced onto masked logits
        forced = torch.zeros_like(experts)
        dz = bfsp.moe_route_grad(z, forced, dw, renormalize=renorm)
        assert torch.isfinite(dz).all() and (dz[2] == 0).all()


@pytest.mark.parametrize("renorm", [True, False])
def test_route_grad_against_differences(renorm):
    """<dz, d> against the central difference of <weights, dw> along d in the
    64-bit definition: second order in the step, so 1e-6 of the sizes."""
    z, k = _normal(11, (6, 40)), 5
    experts, _ = bfsp.moe_route(z, k, renormalize=renorm)
    dw, d = _normal(12, (6, k)), _f64(_normal(13, (6, 40)))
    dz = _f64(bfsp.moe_route_grad(z, experts, dw, renormalize=renorm))
    eps, ix = 1e-4, experts.cpu().numpy()

    def loss(zz):
        p = np.exp(zz - zz.max(1, keepdims=True))
        w = np.take_along_axis(p, ix, 1)
        return (w / (w if renorm else p).sum(1, keepdims=True) * _f64(dw)).sum(1)
    z64 = _f64(z)
    slope = (loss(z64 + eps * d) - loss(z64 - eps * d)) / (2 * eps)
    assert np.abs((dz * d).sum(1) - slope).max() <= 1e-6 * np.abs(_f64(dw)).max() * np.abs(d).max() * 40


# ---------------------------------------------------------------------------
# dispatch
# ---------------------------------------------------------------------------
def _experts(seed, t, k, e, drop=0.0, skew=False):
    g = torch.Generator().manual_seed(seed)
    x = torch.randint(0, e, (t, k), generator=g)
    if skew:
        x = torch.where(torch.rand((t, k), generator=g) < 0.8, torch.tensor(e // 2), x)
    x[torch.rand((t, k), generator=g) < drop] = -1
    return x.int().cuda()


def _dispatch_reference(experts, e):
    flat = experts.cpu().numpy().reshape(-1)
    slots = np.concatenate([np.flatnonzero(flat == i) for i in range(e)])
    off = np.concatenate([[0], np.cumsum([(flat == i).sum() for i in range(e)])])
    pos = np.full(flat.shape, -1)
    pos[slots] = np.arange(len(slots))
    return slots // experts.shape[1], off, pos.reshape(experts.shape)


# around one wave's batch, one group (1024 slots) and one launch's limit (8192)
DISPATCH = [(0, 2, 5, 8), (1, 1, 1, 1), (1, 8, 64, 4096), (3, 1, 5, 7), (8, 2, 64, 130), (63, 1, 3, 16), (65, 1, 1, 33),
            (128, 8, 64, 24), (1024, 1, 17, 8), (1025, 1, 17, 9), (512, 2, 1024, 12), (342, 3, 300, 65), (4096, 1, 64, 4),
            (4097, 1, 64, 3), (1500, 7, 256, 40), (9001, 4, 33, 17), (7000, 2, 16, 40), (6500, 8, 8, 120), (6200, 3, 5, 250), (9001, 5, 7, 131), (6144, 16, 9, 1), (6000, 2, 31, 300), (4100, 3, 17, 1030), (30000, 3, 12, 260), (1365, 3, 90, 11), (1366, 3, 90, 11), (4096, 2, 31, 12), (4097, 2, 31, 12), (2731, 3, 200, 9), (128, 4, 900, 3), (129, 4, 900, 3), (257, 1, 6, 5), (9300, 1, 1024, 20), (511, 5, 1024, 6), (585, 7, 2, 19), (2047, 2, 700, 5), (2, 64, 100, 20), (300, 64, 1000, 8)]


@pytest.mark.parametrize("t,k,e,h", DISPATCH)
@pytest.mark.parametrize("dtype", DTYPES)
def test_dispatch(t, k, e, h, dtype):
    experts = _experts(t + e, t, k, e, drop=0.1 if t % 2 else 0.0, skew=t % 3 == 0)
    x = _padded(_normal(h, (t, h), dtype), 3 if h % 2 else 0)
    rows, buf = _guarded((t * k, h), dtype, 5 if h % 2 else 0)
    perm = torch.full((t * k,), -9, dtype=torch.int32, device="cuda")
    perm, off, pos, got = bfsp.moe_dispatch(experts, e, x, perm=perm, rows=rows)
    ref_perm, ref_off, ref_pos = _dispatch_reference(experts, e)
    n = len(ref_perm)
    assert got is rows and np.array_equal(off.cpu().numpy(), ref_off) and np.array_equal(pos.cpu().numpy(), ref_pos)
    assert np.array_equal(perm[:n].cpu().numpy(), ref_perm) and (perm[n:] == -9).all()
    assert torch.equal(rows[:n], x[torch.from_numpy(ref_perm).cuda().long()])
    assert (rows[n:] == 77).all() and _untouched(buf, rows)
    # without rows, and with buffers of the caller's
    again = bfsp.moe_dispatch(experts, e)
    assert again[3] is None and torch.equal(again[0][:n], perm[:n]) and torch.equal(again[1], off) and torch.equal(again[2], pos)


@pytest.mark.parametrize("t,k", [(40, 2), (5000, 1)])
def test_dispatch_ids_out_of_range_and_all_dropped(t, k):
    """Ids outside the experts count as none, whatever their value."""
    experts = _experts(1, t, k, 8)
    experts[1] = 8
    experts[3] = -(1 << 31)
    experts[5] = (1 << 31) - 1
    x = _normal(2, (t, 12))
    perm, off, pos, rows = bfsp.moe_dispatch(experts, 8, x)
    ref_perm, ref_off, ref_pos = _dispatch_reference(experts, 8)
    n = len(ref_perm)
    assert np.array_equal(off.cpu().numpy(), ref_off) and np.array_equal(pos.cpu().numpy(), ref_pos)
    assert torch.equal(rows[:n], x[torch.from_numpy(ref_perm).cuda().long()])
    experts.fill_(-1)
    perm, off, pos, rows = bfsp.moe_dispatch(experts, 8, x, perm=perm.fill_(-9), rows=rows.fill_(7))
    assert (off == 0).all() and (pos == -1).all() and (perm == -9).all() and (rows == 7).all()
    y = bfsp.moe_combine(rows, pos, torch.ones((t, k), device="cuda"))
    assert (y == 0).all()


def test_dispatch_rows_behind_32_bits():
    """Rows whose element offsets pass 2^31 (4.3 GB of fp32)."""
    t, k, h = 34000, 4, 8192
    experts = _experts(3, t, k, 16)
    x = torch.arange(t, device="cuda", dtype=torch.float32)[:, None].expand(t, h)     # one value a row, unit stride missing
    with pytest.raises(BfsError):
        bfsp.moe_dispatch(experts, 16, x)
    x = x.contiguous().half()
    perm, off, pos, rows = bfsp.moe_dispatch(experts, 16, x)
    assert rows.numel() >= 2 ** 30 and torch.equal(rows[:, 0], x[perm.long(), 0]) and torch.equal(rows[:, -1], x[perm.long(), 0])
    wide = torch.empty((t * k, 2 * h), dtype=torch.float16, device="cuda")[:, :h]      # the last row from element 2.2e9
    bfsp.moe_dispatch(experts, 16, x, rows=wide)
    assert torch.equal(wide[:, 5], rows[:, 5]) and torch.equal(wide[-1], rows[-1])
    w = torch.full((t, k), 0.25, device="cuda")
    y = bfsp.moe_combine(wide, pos, w)
    assert torch.equal(y, x)                                                             # four equal rows of weight 1/4
    grad = torch.empty((t * k, 2 * h), dtype=torch.float16, device="cuda")[:, :h]
    bfsp.moe_combine_grad(x, wide, pos, w, grad_rows=grad)
    assert torch.equal(grad[:, 5], (rows[:, 5].float() * 0.25).half()) and torch.equal(grad[-1], (rows[-1].float() * 0.25).half())


def test_dispatch_workspace():
    """A workspace of the caller's, on another stream; one that is too short is
    refused, and none is needed for few slots."""
    t, k, e, h = 9000, 2, 77, 24
    experts, x = _experts(12, t, k, e, drop=0.1), _normal(13, (t, h), torch.bfloat16)
    want = bfsp.moe_dispatch(experts, e, x)
    size = bfsp.moe_dispatch_workspace(t, k, e)
    assert size > 0 and bfsp.moe_dispatch_workspace(4096, k, e) == 0
    buf = torch.full((size + 64,), 77, dtype=torch.uint8, device="cuda")
    got = [torch.zeros_like(v) for v in want]
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    bfsp.moe_dispatch(experts, e, x, perm=got[0], expert_off=got[1], pos=got[2], rows=got[3], workspace=buf[:size], stream=stream)
    stream.synchronize()
    n = int(want[1][-1])
    assert torch.equal(got[1], want[1]) and torch.equal(got[2], want[2])
    assert torch.equal(got[0][:n], want[0][:n]) and torch.equal(got[3][:n], want[3][:n]) and (buf[size:] == 77).all()
    for bad in (buf[:size - 4], buf[2:2 + size]):
        with pytest.raises(BfsError) as err:
            bfsp.moe_dispatch(experts, e, x, workspace=bad)
        assert err.value.status == bfs.E_INVALID


def test_broadcast_inputs():
    """Inputs with one row for all tokens (row stride 0), as a broadcast gradient has."""
    t, k, e, h = 37, 2, 6, 50
    experts = _experts(4, t, k, e)
    one = _normal(5, (1, h))
    x = one.expand(t, h)
    assert x.stride(0) == 0
    perm, off, pos, rows = bfsp.moe_dispatch(experts, e, x)
    assert torch.equal(rows, one.expand(t * k, h))
    w, r = _normal(6, (t, k)), _normal(7, (t * k, h))
    a, b = bfsp.moe_combine_grad(x, r, pos, w)
    c, d = bfsp.moe_combine_grad(x.contiguous(), r, pos, w)
    assert torch.equal(a, c) and torch.equal(b, d)
    z = _normal(8, (1, 9)).expand(t, 9)
    assert torch.equal(bfsp.moe_route(z, 3)[0], bfsp.moe_route(z.contiguous(), 3)[0])


# ---------------------------------------------------------------------------
# combination
# ---------------------------------------------------------------------------
def _combine_reference(rows, pos, w):
    y, a = np.zeros((pos.shape[0], rows.shape[1])), np.zeros((pos.shape[0], rows.shape[1]))
    for j in range(pos.shape[1]):
        ok = (pos[:, j] >= 0) & (pos[:, j] < rows.shape[0])
        r = rows[np.where(ok, pos[:, j], 0)] * np.where(ok, w[:, j], 0.0)[:, None] if rows.shape[0] else 0.0 * y
        r = np.where(ok[:, None], r, 0.0)
        y += r
        a += np.abs(r)
    return y, a


COMBINE = [(1, 1, 1, 1), (1, 8, 64, 4096), (3, 1, 5, 7), (8, 2, 64, 130), (33, 3, 9, 255), (64, 5, 8, 513), (100, 8, 32, 1001),
           (700, 2, 8, 64), (257, 7, 20, 24), (40, 16, 64, 96), (10, 64, 128, 72), (5000, 2, 16, 40), (2, 4, 8, 8200),
           (512, 3, 6, 700), (513, 3, 6, 700), (20, 5, 6, 519), (700, 2, 6, 2600), (7000, 2, 16, 40), (6500, 8, 8, 120), (7001, 5, 9, 17), (6200, 3, 5, 250), (6144, 1, 3, 8), (9001, 7, 5, 129), (6144, 64, 70, 5)]


@pytest.mark.parametrize("t,k,e,h", COMBINE)
@pytest.mark.parametrize("dtype", DTYPES)
def test_combine_and_dispatch_grad(t, k, e, h, dtype):
    pos = bfsp.moe_dispatch(_experts(t, t, k, e, drop=0.2 if t > 1 else 0.0), e)[2]
    rows, w = _padded(_normal(h, (t * k, h), dtype), 3 if h % 2 else 0), _normal(k, (t, k))
    if t > 2:
        pos[2, 0] = t * k                              # outside the rows: adds nothing
        w[1, k - 1] = 0.0
    dropped = (pos < 0) | (pos >= t * k)
    w[dropped] = float("nan")                          # weights of slots without a row are not used
    p = pos.cpu().numpy()
    for weights in (w, None):
        out, buf = _guarded((t, h), dtype, 4 if h % 2 else 0)
        if weights is None:
            bfsp.moe_dispatch_grad(rows, pos, out=out)
        else:
            bfsp.moe_combine(rows, pos, weights, out=out)
        ref, size = _combine_reference(_f64(rows), p, np.ones(p.shape) if weights is None else np.nan_to_num(_f64(w)))
        _close(out, ref, (k + 1) * U * size, dtype)
        assert _untouched(buf, out)


@pytest.mark.parametrize("t,k,e,h", COMBINE)
@pytest.mark.parametrize("dtype", DTYPES)
def test_combine_grad(t, k, e, h, dtype):
    pos = bfsp.moe_dispatch(_experts(t, t, k, e, drop=0.2 if t > 1 else 0.0), e)[2]
    n = int(pos.max()) + 1
    rows, dy, w = _padded(_normal(h, (t * k, h), dtype), 3 if h % 2 else 0), _padded(_normal(h + 1, (t, h), dtype), 1), _normal(k, (t, k))
    rows[n:] = float("nan")                            # rows behind the last one are not read
    if t > 2:
        w[1, k - 1] = 0.0
    out, buf = _guarded((t * k, h), dtype, 4 if h % 2 else 0)
    dw = torch.full((t, k), 5.0, device="cuda")
    bfsp.moe_combine_grad(dy, rows, pos, w, grad_rows=out, grad_weights=dw)
    p, g, r = pos.cpu().numpy(), _f64(dy), _f64(rows)
    ok = p >= 0
    prod = g[:, None, :] * np.where(ok[..., None], r[np.where(ok, p, 0)], 0.0)
    _close(dw, prod.sum(2), (h / 64 + 16) * U * np.abs(prod).sum(2))
    token = np.repeat(np.arange(t), k).reshape(t, k)
    ref = np.zeros((t * k, h))
    ref[p[ok]] = g[token[ok]] * _f64(w)[ok][:, None]
    _close(out[:n], ref[:n], U * np.abs(ref[:n]), dtype)
    assert (out[n:] == 77).all() and (dw.cpu().numpy()[~ok] == 0).all() and _untouched(buf, out)


def test_combine_gradient_against_differences():
    """The gradients along random directions against central differences of
    the 64-bit combination, which is bilinear: exact up to the differences'
    rounding, so fp32's error on the sums is the bound."""
    t, k, e, h = 20, 3, 5, 48
    pos = bfsp.moe_dispatch(_experts(9, t, k, e, drop=0.1), e)[2]
    rows, w, dy = _normal(1, (t * k, h)), _normal(2, (t, k)), _normal(3, (t, h))
    drows, dw = bfsp.moe_combine_grad(dy, rows, pos, w)
    p, r64, w64, g64 = pos.cpu().numpy(), _f64(rows), _f64(w), _f64(dy)
    dr, dk = _f64(_normal(4, (t * k, h))), _f64(_normal(5, (t, k)))
    eps = 1e-3

    def loss(r, ww):
        return (_combine_reference(r, p, ww)[0] * g64).sum()
    by_rows = (loss(r64 + eps * dr, w64) - loss(r64 - eps * dr, w64)) / (2 * eps)
    by_weights = (loss(r64, w64 + eps * dk) - loss(r64, w64 - eps * dk)) / (2 * eps)
    n = t * k * h
    assert abs((_f64(drows) * dr).sum() - by_rows) <= 4 * U * np.abs(_f64(drows) * dr).sum() + 1e-10 * n
    assert abs((_f64(dw) * dk).sum() - by_weights) <= 40 * U * n + 1e-10 * n


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_combine_extremes(dtype):
    """Infinities and NaN of a row reach its token alone; sums beyond the
    type's range are infinite; zero weights do not hide NaN (0 * NaN)."""
    pos = torch.arange(8, dtype=torch.int32, device="cuda").reshape(4, 2)
    rows = torch.ones((8, 9), dtype=dtype, device="cuda")
    rows[2, 3], rows[5, 4] = float("inf"), float("nan")
    rows[6:, 8] = torch.finfo(dtype).max
    w = torch.ones((4, 2), device="cuda")
    w[2, 1] = 0.0
    y = bfsp.moe_combine(rows, pos, w).float()
    assert y[1, 3] == float("inf") and y[2, 4].isnan() and y[3, 8] == float("inf")
    y[1, 3] = y[2, 4] = y[3, 8] = 0.0
    assert torch.isfinite(y).all() and (y[0] == 2).all()


@pytest.mark.parametrize("t,k,e,h,dtype,shift,drop", [
    (9001, 3, 40, 1409, torch.float16, 0, 0.0), (9001, 3, 40, 1409, torch.float16, 3, 0.1), (300_001, 2, 7, 65, torch.bfloat16, 1, 0.3),
    (4000, 8, 64, 1027, torch.float32, 5, 0.2), (260_000, 2, 9, 33, torch.float32, 0, 0.5), (6001, 2, 3, 4098, torch.bfloat16, 0, 0.0),
    (500_000, 1, 4, 64, torch.bfloat16, 7, 0.1), (400_000, 1, 4, 63, torch.bfloat16, 0, 0.1), (20_000, 2, 4, 1024, torch.bfloat16, 32, 0.9),
    (9001, 3, 40, 1409, torch.bfloat16, 1, 1.0)])
def test_dispatch_past_the_caches(t, k, e, h, dtype, shift, drop):
    """Calls whose rows are not kept in the caches: rows that share lines, from
    an aligned address or not, rows of a line and less, many slots dropped.
    What lies before the rows, and behind the last one, is left as it was."""
    assert (k + 1) * t * h * dtype.itemsize > 96 << 20 or h < 64
    experts = _experts(t, t, k, e, drop=drop)
    x = _normal(h, (1 << 12, h), dtype)[torch.arange(t, device="cuda") * 7919 % (1 << 12)]
    x[:, 0] = torch.arange(t, device="cuda") % 1021
    x[:, -1] = torch.arange(t, device="cuda") // 1021
    buf = torch.full((t * k * h + 64 + shift,), 77, dtype=dtype, device="cuda")
    rows = buf[shift:shift + t * k * h].view(t * k, h)
    perm, off, pos, _ = bfsp.moe_dispatch(experts, e, x, rows=rows)
    n = int(off[-1])
    assert n == int((experts >= 0).sum())
    assert torch.equal(rows[:n], x[perm[:n].long()])
    assert (buf[:shift] == 77).all() and (buf[shift + n * h:] == 77).all()
    ref = bfsp.moe_dispatch(experts, e)
    assert torch.equal(ref[0][:n], perm[:n]) and torch.equal(ref[2], pos)


@pytest.mark.parametrize("t,k,h,dtype,shift", [
    (6001, 3, 1409, torch.float16, 0), (6001, 3, 1409, torch.bfloat16, 3), (3000, 5, 1153, torch.float32, 7), (9000, 1, 2500, torch.float16, 1),
    (2001, 2, 5003, torch.float32, 2), (4001, 2, 4104, torch.bfloat16, 0), (5000, 7, 1152, torch.bfloat16, 5), (1001, 16, 2047, torch.float16, 0)])
def test_combine_grad_past_the_caches(t, k, h, dtype, shift):
    """Rows of the gradient that begin anywhere in a line, some of them
    dropped; what lies before them and behind the last one stays."""
    assert (2 * k + 1) * t * h * dtype.itemsize >= 96 << 20
    pos = bfsp.moe_dispatch(_experts(t, t, k, 9, drop=0.15), 9)[2]
    n = int(pos.max()) + 1
    rows, dy, w = _normal(h, (t * k, h), dtype), _normal(h + 1, (t, h), dtype), _normal(k, (t, k))
    buf = torch.full((t * k * h + 64 + shift,), 77, dtype=dtype, device="cuda")
    out, dw = bfsp.moe_combine_grad(dy, rows, pos, w, grad_rows=buf[shift:shift + t * k * h].view(t * k, h))
    ok = pos >= 0
    at, token = pos[ok].long(), torch.arange(t, device="cuda")[:, None].expand(t, k)[ok]
    # a product rounded to fp32 and then to the type, or (one instruction does both for fp16) to the type at once
    fi, ref = torch.finfo(dtype), w[ok][:, None].double() * dy[token].double()
    assert bool(((out[at].double() - ref).abs() <= ref.abs() * (U + fi.eps / 2 * (1 + U)) + fi.tiny * fi.eps / 2).all())
    assert (buf[:shift] == 77).all() and (buf[shift + n * h:] == 77).all() and (dw[~ok] == 0).all()
    for j in range(k):
        m = ok[:, j]
        prod = dy[m].double() * rows[pos[m, j].long()].double()
        assert bool(((dw[m, j].double() - prod.sum(1)).abs() <= (h / 64 + 16) * U * prod.abs().sum(1)).all())


@pytest.mark.parametrize("t,k,e", [(3_000_001, 2, 5), (2_500_000, 1, 300)])
def test_dispatch_of_many_tokens(t, k, e):
    """Thousands of groups of slots, whose counts a launch of their own sums;
    a narrow row for each."""
    g = torch.Generator(device="cuda").manual_seed(e)
    experts = torch.randint(-1, e, (t, k), generator=g, device="cuda", dtype=torch.int32)
    x = torch.arange(t, device="cuda", dtype=torch.float32)[:, None]
    perm, off, pos, rows = bfsp.moe_dispatch(experts, e, x)
    flat = experts.reshape(-1)
    key, order = torch.sort(torch.where(flat < 0, e, flat), stable=True)
    n = int((key < e).sum())
    assert torch.equal(off.long(), torch.searchsorted(key, torch.arange(e + 1, device="cuda", dtype=torch.int32)))
    assert torch.equal(perm[:n].long(), order[:n] // k) and torch.equal(rows[:n, 0], x[order[:n] // k, 0])
    want = torch.full((t * k,), -1, dtype=torch.int32, device="cuda")
    want[order[:n]] = torch.arange(n, device="cuda", dtype=torch.int32)
    assert torch.equal(pos.reshape(-1), want)
    z = torch.randn((t, 8), generator=g, device="cuda")
    ids, w = bfsp.moe_route(z, 1, renormalize=False)
    assert torch.equal(ids[:, 0].long(), z.argmax(1)) and torch.allclose(w, torch.softmax(z, 1).amax(1, keepdim=True), rtol=1e-5)


@pytest.mark.parametrize("dtype", DTYPES)
def test_no_width_and_no_tokens(dtype):
    for t, h in ((5, 0), (0, 7), (0, 0), (1500, 0)):
        experts = _experts(1, t, 2, 4)
        x = torch.empty((t, h), dtype=dtype, device="cuda")
        perm, off, pos, rows = bfsp.moe_dispatch(experts, 4, x)
        assert rows.shape == (2 * t, h) and int(off[-1]) == 2 * t and pos.shape == (t, 2)
        w = torch.ones((t, 2), device="cuda")
        assert bfsp.moe_combine(rows, pos, w).shape == (t, h) and bfsp.moe_dispatch_grad(rows, pos).shape == (t, h)
        drows, dw = bfsp.moe_combine_grad(x, rows, pos, w)
        assert drows.shape == (2 * t, h) and dw.shape == (t, 2) and (dw == 0).all()
    z = torch.empty((0, 12), dtype=dtype, device="cuda")
    ids, w = bfsp.moe_route(z, 3)
    assert ids.shape == (0, 3) and bfsp.moe_route_grad(z, ids, w).shape == (0, 12)


def test_no_rows_at_all():
    pos = torch.zeros((3, 2), dtype=torch.int32, device="cuda")
    rows, w = torch.empty((0, 16), device="cuda"), torch.ones((3, 2), device="cuda")
    assert (bfsp.moe_combine(rows, pos, w) == 0).all()
    drows, dw = bfsp.moe_combine_grad(torch.ones((3, 16), device="cuda"), rows, pos, w)
    assert drows.shape == (0, 16) and (dw == 0).all()


# ---------------------------------------------------------------------------
# arguments
# ---------------------------------------------------------------------------
def test_refusals():
    z, w = _normal(1, (4, 8)), torch.ones((4, 2), device="cuda")
    ids = torch.zeros((4, 2), dtype=torch.int32, device="cuda")
    rows = _normal(2, (8, 16))
    bad = [
        lambda: bfsp.moe_route(z.cpu(), 2), lambda: bfsp.moe_route(z.double(), 2), lambda: bfsp.moe_route(z[0], 2),
        lambda: bfsp.moe_route(z, 0), lambda: bfsp.moe_route(z, 9), lambda: bfsp.moe_route(z.t(), 2),
        lambda: bfsp.moe_route(z, 2, experts=ids.long()), lambda: bfsp.moe_route(z, 2, weights=w[:3]),
        lambda: bfsp.moe_route_grad(z, ids.long(), w), lambda: bfsp.moe_route_grad(z, ids, w.half()),
        lambda: bfsp.moe_route_grad(z, ids, w, grad_logits=z.half()),
        lambda: bfsp.moe_dispatch(ids.long(), 8), lambda: bfsp.moe_dispatch(ids, 0), lambda: bfsp.moe_dispatch(ids, 8, rows),
        lambda: bfsp.moe_dispatch(ids, 8, rows[:4], rows=rows.half()), lambda: bfsp.moe_dispatch(ids, 8, rows=rows),
        lambda: bfsp.moe_dispatch(ids, 8, perm=ids), lambda: bfsp.moe_dispatch(ids[0], 8),
        lambda: bfsp.moe_dispatch(ids, 8, rows[:4], rows=torch.empty((16, 16), device="cuda")),
        lambda: bfsp.moe_combine(rows, ids, None), lambda: bfsp.moe_combine(rows, ids, w.double()),
        lambda: bfsp.moe_combine(rows, ids, w, out=rows), lambda: bfsp.moe_combine(rows.int(), ids, w),
        lambda: bfsp.moe_combine(rows, ids, w, out=rows[:1].expand(4, 16)),
        lambda: bfsp.moe_combine_grad(rows[:4].half(), rows, ids, w), lambda: bfsp.moe_combine_grad(rows[:3], rows, ids, w),
    ]
    for n, call in enumerate(bad):
        with pytest.raises(BfsError) as e:
            call()
        assert e.value.status == bfs.E_INVALID, n
    with pytest.raises(BfsError) as e:
        bfsp.moe_route(_normal(1, (2, 1025)), 2)
    assert e.value.status == bfs.E_RESOURCE
    other = torch.cuda.Stream()
    for call in (lambda: bfsp.moe_route(z, 2, stream=other), lambda: bfsp.moe_dispatch(ids, 8, stream=other),
                 lambda: bfsp.moe_combine(rows, ids, w, stream=other)):
        with pytest.raises(BfsError):
            call()


def _check_dispatch(t, k, e, h, dtype, shift, drop, skew=False):
    """A dispatch into the middle of a buffer against the definition; what lies
    outside the rows that have a slot stays."""
    experts = _experts(t + e, t, k, e, drop=drop, skew=skew)
    x = _normal(h, (1 << 10, h), dtype)[torch.arange(t, device="cuda") * 7919 % (1 << 10)]
    x[:, 0] = torch.arange(t, device="cuda") % 211
    x[:, -1] = torch.arange(t, device="cuda") // 211 % 211
    buf = torch.full((t * k * h + 64 + shift,), 77, dtype=dtype, device="cuda")
    perm = torch.full((t * k,), -9, dtype=torch.int32, device="cuda")
    perm, off, pos, rows = bfsp.moe_dispatch(experts, e, x, perm=perm, rows=buf[shift:shift + t * k * h].view(t * k, h))
    ref_perm, ref_off, ref_pos = _dispatch_reference(experts, e)
    n = len(ref_perm)
    assert np.array_equal(off.cpu().numpy(), ref_off) and np.array_equal(pos.cpu().numpy(), ref_pos)
    assert np.array_equal(perm[:n].cpu().numpy(), ref_perm) and (perm[n:] == -9).all()
    assert torch.equal(rows[:n], x[torch.from_numpy(ref_perm).cuda().long()])
    assert (buf[:shift] == 77).all() and (buf[shift + n * h:] == 77).all()


@pytest.mark.parametrize("t,k,e,h,dtype,shift,drop", [
    (2048, 8, 64, 4096, torch.bfloat16, 0, 0.0), (2048, 8, 64, 4096, torch.bfloat16, 3, 0.15), (2048, 8, 64, 4095, torch.float16, 1, 0.15),
    (2048, 4, 31, 4096, torch.float32, 0, 0.1), (1200, 6, 300, 8190, torch.bfloat16, 5, 0.3), (1600, 7, 1000, 4097, torch.float16, 0, 0.0)])
def test_dispatch_past_the_caches_by_the_ranking_workgroups(t, k, e, h, dtype, shift, drop):
    """96 MiB and more, of so few long rows that the workgroups that rank a
    group's slots copy them too (a wave for each part of a row, 512 workgroups
    at most), with a table of counts and, up to 8192 slots, without one."""
    steps = -(-h * dtype.itemsize // 1024)
    spans, group = max(2, min(steps, -(-512 // t))), 1024 // k
    assert (k + 1) * t * h * dtype.itemsize >= 96 << 20 and steps >= 4
    assert -(-t // group) * -(-min(t, group) * spans // 8) <= 512
    _check_dispatch(t, k, e, h, dtype, shift, drop)


@pytest.mark.parametrize("t,k,e,h,drop", [(4700, 2, 300, 8, 0.1), (6400, 2, 300, 24, 0.0), (1900, 7, 290, 9, 0.2), (9217, 1, 400, 5, 0.1),
                                          (6000, 3, 200, 8, 0.1), (8700, 1, 455, 3, 0.0), (26_600, 1, 150, 4, 0.3), (22_000, 2, 90, 3, 0.1)])
def test_dispatch_sums_of_many_groups(t, k, e, h, drop):
    """More than 8192 slots whose counts every ranking workgroup sums by
    itself: of more groups than its threads load ahead."""
    groups = -(-t // (1024 // k))
    assert t * k > 8192 and 1024 <= groups * e <= 4096 and groups > 8 * (512 // e)
    for skew in (False, True):
        _check_dispatch(t, k, e, h, torch.bfloat16, 1, drop, skew)


@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("e,k", [(40, 3), (64, 8), (200, 2), (256, 16), (600, 6)])
def test_not_a_number_and_infinity(e, k, dtype, renorm):
    """In every form of the router: NaN of either sign before +inf before the
    rest, equal ones by index; all weights of such a token are NaN, and its
    gradients over all experts; others as without it."""
    z = _normal(e, (9, e), dtype)
    z[1] = float("-inf")                               # a token without experts between them
    clean = bfsp.moe_route(z, k, renormalize=renorm)
    dw = _normal(k, (9, k))
    clean_dz = bfsp.moe_route_grad(z, clean[0], dw, renormalize=renorm)
    z[2, e - 1], z[2, 3], z[2, 5] = float("nan"), float("inf"), -float("nan")
    z[4, 7] = z[4, 6] = float("inf")
    z[6] = float("nan")
    experts, weights = bfsp.moe_route(z, k, renormalize=renorm)
    dz = bfsp.moe_route_grad(z, experts, dw, renormalize=renorm)
    first = experts.cpu().numpy()
    assert np.array_equal(first[2, :3], [5, e - 1, 3][:k]) and np.array_equal(first[4, :2], [6, 7])
    assert np.array_equal(first[6], np.arange(k)) and (first[1] == -1).all() and (weights[1] == 0).all()
    bad, keep = [2, 4, 6], [0, 1, 3, 5, 7, 8]
    assert weights[bad].isnan().all()
    taking_part = dz[bad].gather(1, experts[bad].long()) if renorm else dz[bad]
    assert taking_part.isnan().all()
    assert torch.equal(experts[keep], clean[0][keep]) and torch.equal(weights[keep], clean[1][keep]) and torch.equal(dz[keep], clean_dz[keep])
