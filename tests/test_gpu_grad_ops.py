"""The global gradient norm and clipping against their definition in 64 bits.

Bounds (u = 2^-24, h half a step of the output's type): the squares of fp32
values are exact to 2^-53 and summed in 64 bits, so the norm is off by its one
rounding to fp32, u, and n 2^-52 of the sum; the scale is rounded once (u) and
so is the product (u, then h for a 16-bit output)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2608_13757_amd as bfsp  # noqa: E402
from paper_2608_13757_amd import BfsError, GradSet, bfs  # noqa: E402

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DTYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    bfs.lib()


def _grads(seed, sizes, dtypes, scale=0.01):
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(n, generator=g) * scale).to(dtypes[i % len(dtypes)]).cuda() for i, n in enumerate(sizes)]


def _norm64(grads):
    return float(np.sqrt(sum((g.double().cpu().numpy() ** 2).sum() for g in grads)))


def _check_norm(got, grads):
    ref, n = _norm64(grads), sum(g.numel() for g in grads)
    assert got.shape == () and got.dtype == torch.float32
    assert abs(float(got) - ref) <= ref * (U + n * 2.0 ** -52) * 1.001, (float(got), ref)
    return ref


def _check_out(out, g, scale, dtype):
    fi, ref = torch.finfo(dtype), g.double().cpu().numpy().reshape(-1) * scale
    allowed = np.abs(ref) * (3 * U + fi.eps / 2 * (1 + 3 * U)) + fi.tiny * fi.eps / 2 + 2.0 ** -150
    err = np.abs(out.double().cpu().numpy().reshape(-1) - ref)
    assert (err <= allowed).all(), err.max()


SIZES = [[1], [7], [4096], [8191, 1, 8193], [5, 0, 100000, 3, 0, 16384], [1] * 200, [300 * i + 1 for i in range(140)],
         [3_000_001, 17, 64]]


@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{max(s)}")
@pytest.mark.parametrize("dtypes", [DTYPES[:1], DTYPES[1:2], DTYPES], ids=["fp32", "bf16", "mixed"])
@pytest.mark.parametrize("max_norm", [0.05, 1e9])
def test_norm_and_clip(sizes, dtypes, max_norm):
    grads = _grads(len(sizes), sizes, dtypes)
    ref = _check_norm(GradSet(grads).norm(), grads)
    scale = min(1.0, max_norm / (ref + 1e-6))
    # into a flat fp32 vector, between sentinels and off any alignment
    buf = torch.full((sum(sizes) + 8,), 77.0, device="cuda")
    flat = buf[3:3 + sum(sizes)]
    norm = GradSet(grads, out=flat).clip(max_norm)
    _check_norm(norm, grads)
    assert (buf[:3] == 77).all() and (buf[3 + sum(sizes):] == 77).all()
    for o, g in zip(flat.split(sizes), grads):
        _check_out(o, g, scale, torch.float32)
    # a tensor for each, of the gradients' type, then in place: the same bits
    outs = [torch.full_like(g, 5) for g in grads]
    GradSet(grads, out=outs).clip(max_norm)
    for o, g in zip(outs, grads):
        _check_out(o, g, scale, g.dtype)
    norm2 = GradSet(grads).clip(max_norm)
    assert torch.equal(norm, norm2) and all(torch.equal(o, g) for o, g in zip(outs, grads))


def test_thousands_of_tensors():
    """More chunks than the launches of most sets have workgroups for."""
    g = torch.Generator().manual_seed(10)
    flat_in = (torch.randn(63000, generator=g) * 0.01).bfloat16().cuda()
    sizes = [1 + i % 5 for i in range(21000)]
    grads = list(flat_in.split(sizes))
    ref = _check_norm(GradSet(grads).norm(), [flat_in])
    out = torch.full((63000,), 5.0, device="cuda")
    _check_norm(GradSet(grads, out=out).clip(0.25), [flat_in])
    _check_out(out, flat_in, 0.25 / (ref + 1e-6), torch.float32)
    assert GradSet(grads).clip(0.25) > 0                      # in place
    _check_out(flat_in.float(), out, 1.0, torch.bfloat16)


@pytest.mark.parametrize("dtype,n", [(torch.bfloat16, 2 ** 27 + 12345), (torch.float32, 2 ** 27)])
def test_more_than_the_last_level_cache(dtype, n):
    g = torch.Generator(device="cuda").manual_seed(11)
    flat_in = torch.empty(n, dtype=dtype, device="cuda").normal_(0, 0.01, generator=g)
    grads = list(flat_in.split([n // 2 + 1, 77, n - n // 2 - 78]))
    ref = float(sum(x.double().square().sum() for x in grads)) ** 0.5
    out = torch.empty(n, device="cuda")
    for norm in (GradSet(grads).norm(), GradSet(grads, out=out).clip(1.0)):
        assert abs(float(norm) - ref) <= ref * (U + n * 2.0 ** -52) * 1.001
    want = flat_in.double().mul_(1.0 / (ref + 1e-6))
    assert bool(((out.double() - want).abs() <= want.abs() * 4 * U).all())


def test_same_bits_every_run_and_one_shot_calls():
    grads = _grads(3, [100003, 5000, 77], DTYPES, 1.0)
    s = GradSet(grads)
    first = s.norm()
    for _ in range(5):
        assert torch.equal(s.norm(), first)
    assert torch.equal(bfsp.grad_norm(grads), first)
    want = [(g.float() * float(np.float32(2.0 / (_norm64(grads) + 1e-6)))).to(g.dtype) for g in grads]
    assert torch.equal(bfsp.grad_clip(grads, 2.0), first)
    for g, w in zip(grads, want):
        assert (g.float() - w.float()).abs().max() <= torch.finfo(g.dtype).eps * w.float().abs().max()


@pytest.mark.parametrize("dtype,big", [(torch.float32, 1e30), (torch.bfloat16, 1e30), (torch.float32, 1e-30)])
def test_squares_outside_fp32(dtype, big):
    """Squares beyond fp32's range (or below it) do not spoil the norm."""
    grads = [(torch.randn(1000, generator=torch.Generator().manual_seed(4)) * big).to(dtype).cuda()]
    ref = _check_norm(GradSet(grads).norm(), grads)
    out = torch.empty(1000, device="cuda")
    GradSet(grads, out=out).clip(0.5)
    _check_out(out, grads[0], min(1.0, 0.5 / (ref + 1e-6)), torch.float32)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_norm_not_finite(bad):
    """The norm says so; the gradients stay as they are, in place or copied."""
    grads = _grads(5, [100, 9000], [torch.float32])
    grads[1][8500] = bad
    before = [g.clone() for g in grads]
    out = torch.empty(9100, device="cuda")
    norm = GradSet(grads, out=out).clip(0.01)
    assert norm.isnan() if bad != bad else norm == float("inf")
    assert torch.equal(torch.nan_to_num(out), torch.nan_to_num(torch.cat(before)))
    GradSet(grads).clip(0.01)
    assert all(torch.equal(torch.nan_to_num(a), torch.nan_to_num(b)) for a, b in zip(grads, before))


def test_zeros_empty_and_max_norm_zero():
    assert GradSet([]).norm() == 0 and GradSet([]).clip(1.0) == 0
    empty = [torch.empty(0, device="cuda"), torch.empty((3, 0), device="cuda")]
    assert GradSet(empty).norm() == 0 and GradSet(empty).clip(1.0) == 0
    zeros = [torch.zeros(100, device="cuda")]
    assert GradSet(zeros).clip(1.0) == 0 and (zeros[0] == 0).all()
    g = _grads(6, [50], [torch.float32])
    assert GradSet(g).clip(0.0) > 0 and (g[0] == 0).all()


def test_shared_gradient_counts_twice_in_the_norm():
    """The same tensor named twice adds twice to the norm (out of place)."""
    g = _grads(7, [500], [torch.float32])[0]
    assert abs(float(GradSet([g, g]).norm()) - 2 ** 0.5 * _norm64([g])) <= 4 * U * _norm64([g])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("max_norm", [1e-3, 1e-12])
def test_scale_below_fp32(dtype, max_norm):
    """Norms near fp32's largest value: the scale is below its normal numbers,
    the clipped gradients are not (two roundings of scale and product, as
    ever, and the norm's)."""
    g = torch.Generator().manual_seed(8)
    grads = [(torch.rand(1000, generator=g) * 2e38 / 40).to(dtype).cuda(), torch.tensor([1.0, -2e-30, 0.0], dtype=dtype).cuda()]
    ref = _check_norm(GradSet(grads).norm(), grads)
    out = torch.empty(1003, device="cuda")
    GradSet(grads, out=out).clip(max_norm)
    for o, x in zip(out.split([1000, 3]), grads):
        _check_out(o, x, max_norm / (ref + 1e-6), torch.float32)
    assert abs(_norm64([out]) - max_norm) <= 1e-5 * max_norm


def test_norm_beyond_fp32():
    """A norm that fp32 does not hold is reported as infinite, and nothing is
    scaled, as the documentation says."""
    g = torch.full((5000,), 3e38, device="cuda")
    out = torch.empty_like(g)
    assert GradSet([g], out=out).clip(1.0) == float("inf") and torch.equal(out, g)


def test_overlapping_outputs():
    """Refused by the clipping; their norm is as good as any."""
    buf = _grads(9, [1000], [torch.float32])[0]
    a, b, c = buf[:400], buf[400:], buf[300:500]
    for grads, out in (([a, a], None), ([a, c], None), ([a, b], [buf[100:500], b.clone()])):
        s, before = GradSet(grads, out=out), buf.clone()
        _check_norm(s.norm(), grads)
        with pytest.raises(BfsError) as e:
            s.clip(0.1)
        assert e.value.status == bfs.E_INVALID and torch.equal(buf, before)
    # gradients that share memory, to outputs of their own; neighbours in place
    for grads, out in (([a, c], [torch.empty_like(a), torch.empty_like(c)]), ([a, b], None), ([a, b], buf)):
        want = torch.cat(grads).double() * min(1.0, 0.1 / (_norm64(grads) + 1e-6))
        GradSet(grads, out=out).clip(0.1)
        got = torch.cat(out if isinstance(out, list) else [a, b]).double()
        assert (got - want).abs().max() <= 4 * U * want.abs().max()


def test_refusals():
    g = torch.zeros(8, device="cuda")
    for call in (lambda: GradSet([g.cpu()]), lambda: GradSet([g[::2]]), lambda: GradSet([g.int()]),
                 lambda: GradSet([g], out=torch.empty(7, device="cuda")), lambda: GradSet([g], out=torch.empty(8)),
                 lambda: GradSet([g], out=g.half()), lambda: GradSet([g], out=[]), lambda: GradSet([g], out=[g[:4]]),
                 lambda: GradSet([g.half()], out=[g.bfloat16()]), lambda: GradSet([g]).clip(-1.0),
                 lambda: GradSet([g]).clip(float("nan")), lambda: GradSet([g]).norm(norm=torch.empty(1, device="cuda")),
                 lambda: GradSet([g]).norm(workspace=torch.empty(1, dtype=torch.uint8, device="cuda")),
                 lambda: GradSet([g]).norm(stream=torch.cuda.Stream())):
        with pytest.raises(BfsError) as e:
            call()
        assert e.value.status == bfs.E_INVALID


@pytest.mark.parametrize("call", ["one_shot", "handle", "current"])
def test_set_dropped_while_another_stream_uses_it(call):
    """The set's table is not given to the allocations that follow its release
    while a stream other than the set's is still to run the call."""
    grads = _grads(12, [70_001, 33, 5000], [torch.bfloat16])
    want = [g.double() * min(1.0, 0.5 / (_norm64(grads) + 1e-6)) for g in grads]
    out, norm = torch.zeros(75_034, device="cuda"), torch.zeros((), device="cuda")
    s = GradSet(grads, out=out)
    s.clip(0.5)                                        # (the kernels are loaded)
    workspace = torch.empty(s.workspace_bytes, dtype=torch.uint8, device="cuda")
    out.zero_()
    del s
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        torch.cuda._sleep(20_000_000)                  # milliseconds, before the call's kernels
    if call == "one_shot":
        bfsp.grad_clip(grads, 0.5, out=out, norm=norm, workspace=workspace, stream=stream)
    elif call == "handle":
        GradSet(grads, out=out).clip(0.5, norm=norm, workspace=workspace, stream=stream.cuda_stream)
    else:
        s = GradSet(grads, out=out)
        with torch.cuda.stream(stream):
            s.clip(0.5, norm=norm, workspace=workspace)
        del s
    zeros = [torch.zeros(n, dtype=torch.uint8, device="cuda") for n in [512, 1024, 2048, 4096, 8192] * 40]
    stream.synchronize()
    _check_norm(norm, grads)
    for o, g, w in zip(out.split([g.numel() for g in grads]), grads, want):
        assert bool(((o.double() - w).abs() <= w.abs() * 4 * U).all())
    assert all((z == 0).all() for z in zeros[:5])


def test_set_dropped_while_the_default_stream_uses_it():
    """A set made on a stream of its own, its call on the default stream."""
    grads = _grads(13, [9001, 70_001], [torch.float32])
    want = [g.double() * min(1.0, 0.25 / (_norm64(grads) + 1e-6)) for g in grads]
    out, norm = torch.zeros(79_002, device="cuda"), torch.zeros((), device="cuda")
    workspace = torch.empty(GradSet(grads).workspace_bytes, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    torch.cuda._sleep(20_000_000)
    with torch.cuda.stream(torch.cuda.Stream()):
        bfsp.grad_clip(grads, 0.25, out=out, norm=norm, workspace=workspace, stream=torch.cuda.default_stream().cuda_stream)
        zeros = [torch.zeros(n, dtype=torch.uint8, device="cuda") for n in [512, 1024, 2048, 4096, 8192] * 40]
    torch.cuda.synchronize()
    _check_norm(norm, grads)
    for o, w in zip(out.split([g.numel() for g in grads]), want):
        assert bool(((o.double() - w).abs() <= w.abs() * 4 * U).all())
    assert all((z == 0).all() for z in zeros[:5])
