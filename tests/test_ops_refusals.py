"""Refusals of the operators beside the plans, on the host: every call here
returns an error (or has nothing to do) before anything would be launched, so
the addresses are never used."""
import ctypes as C
import struct
import subprocess
import sys

import pytest

from paper_2608_13757_amd import BfsError, bfs

A = 1 << 20                     # an address that no call uses
F32, BF16, F16 = 0, 1, 2


def _named(name, *args):
    return getattr(bfs.lib(), name)(*args)


_status = _named


def _route(logits=A, dtype=F32, t=4, e=8, stride=8, k=2, flags=1, experts=A, weights=A):
    return _status("bfs_moe_route", logits, dtype, t, e, stride, k, flags, experts, weights, None)


def _route_grad(logits=A, dtype=F32, t=4, e=8, stride=8, experts=A, k=2, dw=A, flags=1, out=A, out_stride=8):
    return _status("bfs_moe_route_grad", logits, dtype, t, e, stride, experts, k, dw, flags, out, out_stride, None)


def _dispatch(experts=A, t=4, k=2, e=8, perm=A, off=A, pos=A, x=A, dtype=BF16, width=16, x_stride=16, rows=A,
              rows_stride=16, ws=None, ws_bytes=0):
    return _status("bfs_moe_dispatch", experts, t, k, e, perm, off, pos, x, dtype, width, x_stride, rows, rows_stride, ws,
                   ws_bytes, None)


def _combine(rows=A, dtype=BF16, n=8, width=16, stride=16, pos=A, w=A, t=4, k=2, y=A, y_stride=16):
    return _status("bfs_moe_combine", rows, dtype, n, width, stride, pos, w, t, k, y, y_stride, None)


def _combine_grad(dy=A, dtype=BF16, t=4, width=16, dy_stride=16, rows=A, n=8, stride=16, pos=A, w=A, k=2, out=A,
                  out_stride=16, dw=A):
    return _status("bfs_moe_combine_grad", dy, dtype, t, width, dy_stride, rows, n, stride, pos, w, k, out, out_stride, dw,
                   None)


def _list(values, kind):
    return (kind * max(1, len(values)))(*values)


def _table(grads=(A,), outs=(A,), numel=(4,), dtypes=(F32,), out_dtypes=(F32,), n=None, image=False, image_bytes=1 << 20,
           made=True):
    made = bfs.GradSetStruct() if made else None
    buf = C.create_string_buffer(1 << 20) if image else None
    st = _status("bfs_grad_table", _list(grads, C.c_void_p), _list(outs, C.c_void_p), _list(numel, C.c_int64),
                 _list(dtypes, C.c_int32), _list(out_dtypes, C.c_int32), len(grads) if n is None else n,
                 C.byref(made) if made is not None else None, buf, image_bytes)
    return st if st != bfs.OK else (made, buf)


def _grad_call(change=None, image=A, ws=A, ws_bytes=1 << 20, set_=True, **kw):
    made, _ = _table()
    if change:
        setattr(made, *change)
    made = C.byref(made) if set_ else None
    if "max_norm" in kw:
        return _status("bfs_grad_clip", made, image, kw["max_norm"], A, ws, ws_bytes, None)
    return _status("bfs_grad_norm", made, image, kw.get("norm", A), ws, ws_bytes, None)


INVALID = [
    (_route, dict(t=-1)), (_route, dict(e=0)), (_route, dict(k=0)), (_route, dict(k=9)), (_route, dict(stride=-1)),
    (_route, dict(flags=2)), (_route, dict(dtype=3)), (_route, dict(dtype=-1)), (_route, dict(logits=None)),
    (_route, dict(experts=None)), (_route, dict(weights=None)),
    (_route_grad, dict(out_stride=7)), (_route_grad, dict(stride=-8)), (_route_grad, dict(k=9)),
    (_route_grad, dict(experts=None)), (_route_grad, dict(dw=None)), (_route_grad, dict(out=None)),
    (_route_grad, dict(flags=8)), (_route_grad, dict(dtype=7)),
    (_dispatch, dict(t=-1)), (_dispatch, dict(k=0)), (_dispatch, dict(e=0)), (_dispatch, dict(experts=None)),
    (_dispatch, dict(perm=None)), (_dispatch, dict(off=None)), (_dispatch, dict(pos=None)), (_dispatch, dict(x=None)),
    (_dispatch, dict(rows=None)), (_dispatch, dict(width=-1)), (_dispatch, dict(rows_stride=15)),
    (_dispatch, dict(x_stride=-16)), (_dispatch, dict(dtype=3)), (_dispatch, dict(t=1 << 14)),
    (_dispatch, dict(t=1 << 14, ws=A, ws_bytes=4)), (_dispatch, dict(t=1 << 14, ws=A + 2, ws_bytes=1 << 20)),
    (_combine, dict(n=-1)), (_combine, dict(width=-1)), (_combine, dict(t=-1)), (_combine, dict(k=0)),
    (_combine, dict(stride=-1)), (_combine, dict(y_stride=15)), (_combine, dict(dtype=3)), (_combine, dict(pos=None)),
    (_combine, dict(y=None)), (_combine, dict(rows=None)),
    (_combine_grad, dict(out_stride=15)), (_combine_grad, dict(dy_stride=-1)), (_combine_grad, dict(stride=-1)),
    (_combine_grad, dict(w=None)), (_combine_grad, dict(dw=None)), (_combine_grad, dict(dy=None)),
    (_combine_grad, dict(rows=None)), (_combine_grad, dict(out=None)), (_combine_grad, dict(dtype=5)),
    (_table, dict(n=-1)), (_table, dict(numel=(-4,))), (_table, dict(grads=(None,))), (_table, dict(outs=(None,))),
    (_table, dict(dtypes=(3,))), (_table, dict(out_dtypes=(BF16,))), (_table, dict(dtypes=(BF16,), out_dtypes=(F16,))),
    (_table, dict(out_dtypes=(9,))), (_table, dict(dtypes=(BF16,))), (_table, dict(grads=(A + 2,))),
    (_table, dict(outs=(A + 1,), dtypes=(BF16,), out_dtypes=(BF16,))), (_table, dict(image=True, image_bytes=8)),
    (_table, dict(made=False)), (_grad_call, dict(set_=False)), (_grad_call, dict(image=None)), (_grad_call, dict(image=A + 8)),
    (_grad_call, dict(norm=None)), (_grad_call, dict(ws=None)), (_grad_call, dict(ws_bytes=4)), (_grad_call, dict(ws=A + 4)),
    (_grad_call, dict(max_norm=-1.0)), (_grad_call, dict(max_norm=float("nan"))), (_grad_call, dict(max_norm=1.0, ws=None)),
    (_grad_call, dict(max_norm=1.0, change=("overlap", 1))),
    (_grad_call, dict(change=("n_blocks", 0))), (_grad_call, dict(change=("n_blocks", 1 << 20))),
    (_grad_call, dict(change=("chunk", 0))), (_grad_call, dict(change=("n_entries", -1))),
]


@pytest.mark.parametrize("call,kw", INVALID, ids=lambda v: getattr(v, "__name__", str(v)))
def test_invalid_arguments(call, kw):
    assert call(**kw) == bfs.E_INVALID
    assert bfs.lib().bfs_last_error()


CALLS = {"bfs_moe_route": (0, "PqqqqqqPPP"), "bfs_moe_route_grad": (1, "PqqqqPqPqPqP"), "bfs_moe_dispatch": (2, "PqqqPPPPqqqPqPqP"),
         "bfs_moe_combine": (3, "PqqqqPPqqPqP"), "bfs_moe_combine_grad": (4, "PqqqqPqqPPqPqPP"), "bfs_grad_norm": (5, "PPPPqP"),
         "bfs_grad_clip": (6, "PPdPPqP")}


def _words(name, *args):
    op, kinds = CALLS[name]
    values = [C.addressof(a._obj) if hasattr(a, "_obj") else 0 if a is None else a for a in args]
    return bfs.lib().bfs_call(struct.pack("qq" + kinds, op, len(kinds), *values))


@pytest.mark.parametrize("call,kw", [c for c in INVALID if c[0] is not _table], ids=lambda v: getattr(v, "__name__", str(v)))
def test_invalid_arguments_as_words(call, kw, monkeypatch):
    monkeypatch.setattr(sys.modules[__name__], "_status", lambda name, *a: (_words if name in CALLS else _named)(name, *a))
    assert call(**kw) == bfs.E_INVALID
    assert bfs.lib().bfs_last_error()


def test_words():
    """The array itself: its operator, its count, integers that do not fit."""
    call = bfs.lib().bfs_call
    assert call(None) == bfs.E_INVALID
    for op, n, extra in ((-1, 0, ""), (7, 0, ""), (0, 9, "10q"), (0, 11, "11q"), (2, 10, "16q")):
        assert call(struct.pack("qq" + extra, op, n, *[0] * (int(extra[:-1]) if extra else 0))) == bfs.E_INVALID
    route = [A, F32, 0, 8, 8, 2, 1, A, A, 0]                     # no tokens: nothing to do
    assert call(struct.pack("12q", 0, 10, *route)) == bfs.OK
    for i, bad in ((1, 1 << 32), (3, (1 << 32) + 8), (5, (1 << 32) + 2), (5, -(1 << 31) - 1), (6, 1 << 32), (6, -1)):
        assert call(struct.pack("12q", 0, 10, *[bad if j == i else v for j, v in enumerate(route)])) == bfs.E_INVALID


RESOURCE = [(_route, dict(e=1025, stride=1025)), (_route, dict(e=64, stride=64, k=17)), (_route, dict(t=1 << 31)),
            (_dispatch, dict(e=1025)), (_dispatch, dict(k=65)), (_dispatch, dict(t=1 << 30)), (_combine, dict(k=65)),
            (_combine, dict(t=1 << 30)), (_combine, dict(n=1 << 31)), (_combine_grad, dict(t=1 << 30)),
            (_dispatch, dict(width=1 << 62, x_stride=1 << 62, rows_stride=1 << 62)), (_combine, dict(width=(1 << 28) + 1, y_stride=1 << 30)),
            (_combine_grad, dict(width=1 << 40, out_stride=1 << 40)),
            (_table, dict(numel=(1 << 44,))),
            (_table, dict(grads=(A, A), outs=(A, A), numel=(1 << 42, 1 << 43), dtypes=(F32, F32), out_dtypes=(F32, F32)))]


@pytest.mark.parametrize("call,kw", RESOURCE, ids=lambda v: getattr(v, "__name__", str(v)))
def test_beyond_the_limits(call, kw):
    assert call(**kw) == bfs.E_RESOURCE


def test_nothing_to_do():
    """No tokens, or no width: done without a buffer."""
    assert _route(t=0, logits=None, experts=None, weights=None) == bfs.OK
    assert _route_grad(t=0, logits=None, experts=None, dw=None, out=None) == bfs.OK
    assert _combine(t=0, rows=None, n=0, pos=None, w=None, y=None) == bfs.OK
    assert _combine(width=0, stride=0, y_stride=0, rows=None, y=None) == bfs.OK
    assert _combine_grad(t=0, dy=None, rows=None, n=0, pos=None, w=None, out=None, dw=None) == bfs.OK


def test_workspaces():
    torch = pytest.importorskip("torch")
    from paper_2608_13757_amd import GradSet, moe_dispatch_workspace
    from paper_2608_13757_amd.ops import DISPATCH_ALONE
    for k in (1, 2, 3, 7, 64):
        most = DISPATCH_ALONE // k
        assert moe_dispatch_workspace(0, k, 64) == 0 and moe_dispatch_workspace(most, k, 64) == 0
        assert moe_dispatch_workspace(most + 1, k, 64) > 0
    assert moe_dispatch_workspace(32768, 2, 64) > 0
    for bad in ((-1, 1, 4), (4, 0, 4), (4, 1, 0)):
        with pytest.raises(BfsError) as e:
            moe_dispatch_workspace(*bad)
        assert e.value.status == bfs.E_INVALID
    for n_experts in (1025, (1 << 32) + 8):           # (no 32 bits of it pass for another number)
        with pytest.raises(BfsError) as e:
            moe_dispatch_workspace(4, 1, n_experts)
        assert e.value.status == bfs.E_RESOURCE
    with pytest.raises(BfsError):
        GradSet([torch.zeros(3)])                     # not on a device


def _entries(made, buf):
    """(in, out, n, first, chunks, type, index) of each tensor, and of the one that each workgroup begins in."""
    raw = buf.raw[:made.image_bytes]
    assert len(raw) == 40 * (made.n_entries + made.n_blocks)
    rows = [struct.unpack_from("<QQqiiii", raw, 40 * i) for i in range(made.n_entries + made.n_blocks)]
    return rows[:made.n_entries], rows[made.n_entries:]


@pytest.mark.parametrize("sizes", [[1], [5, 0, 100000, 3, 0, 16384], [1] * 2000, [7] + [1 << 20] * 30, [1 << 33, 9], []])
def test_grad_table(sizes):
    """Every tensor's chunks cover it, in order; a workgroup's first chunk
    lies in the tensor that the table names."""
    n = len(sizes)
    got = _table([A] * n, [A] * n, sizes, [BF16] * n, [BF16] * n, image=True, image_bytes=1 << 20)
    made, buf = got
    rows, start = _entries(made, buf)
    assert [r[2] for r in rows] == [s for s in sizes if s] and all(r[0] == r[1] == A and r[5] == BF16 * 17 for r in rows)
    at = 0
    assert [r[6] for r in rows] == list(range(len(rows)))
    for _, _, size, first, chunks, _, _ in rows:
        assert first == at and (chunks - 1) * made.chunk < size <= chunks * made.chunk
        at += chunks
    assert at == made.n_chunks and made.n_blocks == (4096 if at >= 16384 else min(at, 1024)) == len(start)
    assert made.grad_bytes == 2 * sum(sizes)
    for b, r in enumerate(start):
        c = made.n_chunks * b // made.n_blocks
        assert r == rows[r[6]] and r[3] <= c < r[3] + r[4]


@pytest.mark.parametrize("grads,outs,numel,dtypes,out_dtypes,overlap", [
    ([A, A], [A, A], [4, 4], [F32, F32], [F32, F32], 1),                     # the same one twice, in place
    ([A, A], [A + 64, A + 128], [4, 4], [F32, F32], [F32, F32], 0),          # ... to outputs of their own
    ([A, A + 16], [A, A + 16], [4, 4], [F32, F32], [F32, F32], 0),           # neighbours in place
    ([A, A + 12], [A, A + 12], [4, 4], [F32, F32], [F32, F32], 1),
    ([A, A + 1024], [A + 4, A + 1024], [4, 4], [F32, F32], [F32, F32], 1),   # an output elsewhere in its gradient
    ([A, A + 1024], [A + 1024, A + 2048], [4, 4], [F32, F32], [F32, F32], 1),  # an output on another gradient
    ([A, A + 8], [A + 4096, A + 4112], [4, 4], [BF16, BF16], [F32, F32], 0),  # one flat output behind the gradients
    ([A, A + 8], [A + 4096, A + 4108], [4, 4], [BF16, BF16], [F32, F32], 1),
    ([A, A, None], [A + 64, A + 64, None], [4, 0, 0], [F32] * 3, [F32] * 3, 0),  # empty tensors overlap nothing
    ([A + 512, A], [A + 512, A], [128, 128], [F32, F32], [F32, F32], 0),
    ([A + 508, A], [A + 508, A], [128, 128], [F32, F32], [F32, F32], 1)])
def test_grad_table_overlap(grads, outs, numel, dtypes, out_dtypes, overlap):
    made, _ = _table(grads, outs, numel, dtypes, out_dtypes)
    assert made.overlap == overlap


def test_package_imports_without_the_operators():
    """The operators are loaded at their first use: the binding alone needs no torch."""
    code = ("import sys; import paper_2608_13757_amd as p; assert 'torch' not in sys.modules; p.lib(); "
            "assert 'torch' not in sys.modules\ntry:\n p.no_such_name\nexcept AttributeError: pass\nelse: raise SystemExit(1)")
    subprocess.run([sys.executable, "-c", code], check=True)


def _on_device(torch, *args, **kw):
    """A tensor of the host that says it is on device 0."""
    class T(torch.Tensor):
        is_cuda = True

        def get_device(self):
            return 0
    return torch.zeros(*args, **kw).as_subclass(T)


@pytest.mark.parametrize("given", ["handle", "current"])
def test_set_of_gradients_belongs_to_the_streams_that_use_it(given, monkeypatch):
    """Calls on another stream than the set was made on: before the first of
    each stream is enqueued the allocator knows that it uses the table and the
    gradients, so that a set dropped at once (the one-shot calls do) is not
    given away under the kernels.  On the host, with the launch left out."""
    torch = pytest.importorskip("torch")
    from types import SimpleNamespace

    from paper_2608_13757_amd import ops
    real, current, events = bfs.lib(), [0], []
    monkeypatch.setattr(ops, "_device", lambda: 0)
    monkeypatch.setattr(ops, "_raw_stream", lambda device: current[0])
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: events.append((t.data_ptr(), s)), raising=False)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle: handle)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda: current[0])
    monkeypatch.setattr(bfs, "_lib", SimpleNamespace(bfs_grad_table=real.bfs_grad_table,
                                                     bfs_call=lambda words: events.append("call") or 0))
    grads = [_on_device(torch, 50), _on_device(torch, 7, dtype=torch.bfloat16)]
    flat = _on_device(torch, 57)
    kw = dict(norm=_on_device(torch, ()), workspace=_on_device(torch, 1024, dtype=torch.float64))

    def run(method, *args, on, **more):
        events.clear()
        if given == "current":
            current[0] = on
        else:
            kw["stream"] = on
        method(*args, **kw, **more)

    s = ops.GradSet(grads, out=flat)
    memory = {s._args[1], flat.data_ptr(), flat[50:].data_ptr(), *(g.data_ptr() for g in grads)}
    run(s.norm, on=0)
    assert events == ["call"]                          # the set's own stream
    for method, args in ((s.norm, ()), (s.clip, (1.0,))):
        run(method, *args, on=7)
        if method == s.norm:
            assert events[-1] == "call" and set(events[:-1]) == {(p, 7) for p in memory}
        else:
            assert events == ["call"]                  # known already
    run(s.clip, 1.0, on=9)
    assert events[-1] == "call" and {e[1] for e in events[:-1]} == {9}
    current[0] = 0
    if given == "handle":                              # a set that nothing but the call holds
        run(ops.grad_clip, grads, 1.0, on=7, out=flat)
        assert events[-1] == "call" and len({e[0] for e in events[:-1]}) == 5 and {e[1] for e in events[:-1]} == {7}


@pytest.mark.parametrize("shape", [(), (4,), (1, 4, 2), (3, 2), (0,)])
def test_ids_that_are_no_matrix(shape, monkeypatch):
    """Ids and positions of any other shape are refused as BfsError, a number
    of no dimension too.  On the host, before anything would be launched."""
    torch = pytest.importorskip("torch")
    from paper_2608_13757_amd import ops
    monkeypatch.setattr(ops, "_device", lambda: 0)
    monkeypatch.setattr(ops, "_raw_stream", lambda device: 0)
    ids, w, x = _on_device(torch, shape, dtype=torch.int32), _on_device(torch, 4, 2), _on_device(torch, 4, 16)
    for call in (lambda: ops.moe_route_grad(x, ids, w), lambda: ops.moe_combine_grad(x, x, ids, w),
                 lambda: ops.moe_combine(x, ids, w), lambda: ops.moe_dispatch(ids, 8, x)):
        with pytest.raises(BfsError) as e:
            call()
        assert e.value.status == bfs.E_INVALID


def test_set_of_gradients_used_on_the_default_stream(monkeypatch):
    """Of a set made on a stream of its own, called by the default stream's
    handle, which is 0: torch's wrapper of handles would make another stream of
    that.  On the host, with the launch left out."""
    torch = pytest.importorskip("torch")
    from types import SimpleNamespace

    from paper_2608_13757_amd import ops
    real, events = bfs.lib(), []
    monkeypatch.setattr(ops, "_device", lambda: 0)
    monkeypatch.setattr(ops, "_raw_stream", lambda device: 5)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: events.append(s), raising=False)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle: "external")
    monkeypatch.setattr(torch.cuda, "default_stream", lambda: "default")
    monkeypatch.setattr(bfs, "_lib", SimpleNamespace(bfs_grad_table=real.bfs_grad_table,
                                                     bfs_call=lambda words: events.append("call") or 0))
    ops.grad_norm([_on_device(torch, 50)], norm=_on_device(torch, ()), workspace=_on_device(torch, 64, dtype=torch.float64), stream=0)
    assert events == ["default"] * 3 + ["call"]         # the gradient twice (it is its own output), the table
