"""The operators around a mixture-of-experts layer's products and its
optimizer step, by which their performance is measured: the router, the
dispatch of tokens to their experts, the weighted combination of the experts'
rows, the gradient of each, and the global gradient norm with clipping.

Where ``own`` is false a pass computes the operator in elementary torch
operations, in 32 bits (the global norm's long sum in 64); where it is true,
by the library's calls, with the output buffers that such a program keeps.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def listed():
    return [
        # The router of one decoding step: eight sequences, a token each.
        # Latency only.
        dict(name="route_8tok", op="route", tokens=8, experts=64, k=2, dtype="fp32", renorm=True),
        # ... of a prefill, eight experts of 64 for each token, logits of a
        # bf16 projection (equal logits are common).
        dict(name="route_32768tok_64e", op="route", tokens=32768, experts=64, k=8, dtype="bf16", renorm=True),
        # Its gradient in training, many small experts, softmax weights as
        # they are (every logit has a gradient).
        dict(name="route_grad_16384tok_256e", op="route_grad", tokens=16384, experts=256, k=8, dtype="fp32",
             renorm=False),
        # Tokens to experts in a decoding step.
        dict(name="dispatch_8tok", op="dispatch", tokens=8, experts=64, k=2, hidden=4096, dtype="bf16", zipf=0.5,
             drop=0.0, pad=0),
        # ... of a prefill with skewed routing (Zipf 1.1 over 64 experts).
        dict(name="dispatch_32768tok_64e", op="dispatch", tokens=32768, experts=64, k=2, hidden=4096, dtype="bf16",
             zipf=1.1, drop=0.0, pad=0),
        # The gradient of a padded batch's dispatch: an odd number of tokens,
        # a tenth of them padding without an expert, rows of odd length.
        dict(name="dispatch_grad_ragged", op="dispatch_grad", tokens=5003, experts=8, k=4, hidden=1409, dtype="fp16",
             zipf=0.5, drop=0.1, pad=0),
        # The experts' rows back to one token, and to a small batch's.
        dict(name="combine_1tok", op="combine", tokens=1, experts=64, k=8, hidden=4096, dtype="bf16", zipf=0.0,
             drop=0.0, pad=0),
        dict(name="combine_2048tok_8e", op="combine", tokens=2048, experts=8, k=2, hidden=1024, dtype="fp32", zipf=0.5,
             drop=0.0, pad=0),
        # ... to a prefill's, and the gradient of that: the weights' dot
        # products and the experts' rows of the output's gradient.
        dict(name="combine_16384tok_64e", op="combine", tokens=16384, experts=64, k=8, hidden=2048, dtype="bf16",
             zipf=1.1, drop=0.0, pad=0),
        dict(name="combine_grad_32768tok_64e", op="combine_grad", tokens=32768, experts=64, k=2, hidden=4096,
             dtype="bf16", zipf=1.1, drop=0.0, pad=0),
        # The gradients of a small model, clipped into the optimizer's flat
        # gradient vector (a million parameters in 24 tensors).
        dict(name="clip_1m_24", op="clip", params=1 << 20, tensors=24, dtype="fp32"),
        # ... of a large one: bf16 gradients in 290 tensors, some of them
        # short, of 2^28 parameters, to fp32.
        dict(name="clip_268m_290", op="clip", params=1 << 28, tensors=290, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: sizes spread over the logarithm of their ranges, two
    thirds of the widths multiples of eight, a few padded batches and strided
    rows, no more bytes than the largest listed case."""
    op = rng.choice(["route", "route_grad", "dispatch", "dispatch_grad", "combine", "combine_grad", "clip"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if op == "clip":
        tensors = _log_int(rng, 1, 300)
        return dict(op=op, params=max(tensors, _log_int(rng, 1 << 10, 1 << 27)), tensors=tensors, dtype=dtype)
    tokens, experts = _log_int(rng, 1, 32768), _log_int(rng, 4, 512)
    k = rng.randint(1, min(8, experts))
    if op in ("route", "route_grad"):
        return dict(op=op, tokens=tokens, experts=experts, k=k, dtype=dtype, renorm=rng.random() < 0.5)
    hidden = 8 * _log_int(rng, 8, 1024) if rng.random() < 0.67 else _log_int(rng, 16, 8192)
    tokens = min(tokens, int(1.2e9 / (hidden * DTYPES[dtype].itemsize * (2 * k + 1))))
    return dict(op=op, tokens=tokens, experts=experts, k=k, hidden=hidden, dtype=dtype, zipf=round(rng.uniform(0, 1.2), 2),
                drop=rng.choice([0.0, 0.0, 0.1]), pad=rng.choice([0, 0, 8, 5]))


# ---------------------------------------------------------------------------
# what a program has in hand before the call
# ---------------------------------------------------------------------------
def _gen(seed, stream):
    return torch.Generator(device="cuda").manual_seed(1000003 * (seed + 1) + stream)


def _normal(seed, stream, shape, scale=1.0, dtype=torch.float32):
    return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, scale, generator=_gen(seed, stream))


def _rows(seed, stream, n, case):
    """[n, hidden] of N(0, 1); with ``pad`` a view of longer rows."""
    return _normal(seed, stream, (n, case["hidden"] + case["pad"]), 1.0, DTYPES[case["dtype"]])[:, : case["hidden"]]


def _sizes(case):
    """The tensors' sizes of a model: weights of equal size, every third a
    short vector; the remainder goes to the last."""
    n, t = case["params"], case["tensors"]
    sizes = [max(1, n // t // 512) if i % 3 == 1 else n // t for i in range(t)]
    sizes[-1] += n - sum(sizes)
    return sizes


def _experts(case, seed):
    """k different experts for each token, popularity by Zipf's law in a
    seeded order; dropped tokens (padding) have none."""
    t, e = case["tokens"], case["experts"]
    pop = torch.arange(1, e + 1, device="cuda").float().pow(-case["zipf"])[torch.randperm(e, device="cuda", generator=_gen(seed, 1))]
    noise = torch.empty((t, e), device="cuda").exponential_(generator=_gen(seed, 2))
    experts = torch.topk(pop / noise, case["k"], dim=1).indices.int()
    if case["drop"]:
        experts[torch.rand(t, device="cuda", generator=_gen(seed, 3)) < case["drop"]] = -1
    return experts.contiguous()


def _positions(experts):
    """Each slot's row among the rows grouped by expert; -1 without one."""
    flat = experts.reshape(-1).long()
    order = torch.argsort(torch.where(flat < 0, 1 << 30, flat), stable=True)
    pos = torch.empty_like(order).scatter_(0, order, torch.arange(flat.numel(), device="cuda"))
    return torch.where(flat < 0, -1, pos).int().reshape(experts.shape).contiguous()


def prepare(case, seed):
    op, dtype = case["op"], DTYPES[case["dtype"]]
    if op == "clip":
        grads = [_normal(seed, 10 + i, (n,), 0.01, dtype) for i, n in enumerate(_sizes(case))]
        state = dict(case=case, grads=grads, flat=torch.zeros(case["params"], device="cuda"),
                     norm=torch.zeros((), device="cuda"))
        if own:      # the handle of a model's gradients, which a training program makes once
            from paper_2608_13757_amd import GradSet
            state["set"] = GradSet(grads, out=state["flat"])
        return state
    t, k = case["tokens"], case["k"]
    i32 = dict(dtype=torch.int32, device="cuda")
    if op in ("route", "route_grad"):
        logits = _normal(seed, 1, (t, case["experts"]), 2.0, dtype)
        if op == "route":
            return dict(case=case, logits=logits, experts=torch.zeros((t, k), **i32), weights=torch.zeros((t, k), device="cuda"))
        experts = torch.topk(logits, k, dim=1).indices.int().contiguous()
        return dict(case=case, logits=logits, experts=experts, dw=_normal(seed, 2, (t, k)), dlogits=torch.zeros_like(logits))
    n, h = t * k, case["hidden"]
    experts = _experts(case, seed)
    if op == "dispatch":
        return dict(case=case, experts=experts, x=_rows(seed, 4, t, case), perm=torch.zeros(n, **i32),
                    off=torch.zeros(case["experts"] + 1, **i32), pos=torch.zeros((t, k), **i32),
                    rows=torch.zeros((n, h), dtype=dtype, device="cuda"))
    state = dict(case=case, pos=_positions(experts), rows=_rows(seed, 4, n, case), y=torch.zeros((t, h), dtype=dtype, device="cuda"))
    if op != "dispatch_grad":
        state["weights"] = torch.softmax(_normal(seed, 5, (t, k)), dim=1)
    if op == "combine_grad":
        state |= dict(dy=_rows(seed, 6, t, case), drows=torch.zeros((n, h), dtype=dtype, device="cuda"),
                      dw=torch.zeros((t, k), device="cuda"))
        del state["y"]
    return state


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------
def _route(logits, k, renorm):
    z = logits.float()
    top, experts = torch.sort(z, dim=1, descending=True, stable=True)
    top, experts = top[:, :k], experts[:, :k]
    e = torch.exp(top - top[:, :1])
    total = e.sum(1, keepdim=True) if renorm else torch.exp(z - top[:, :1]).sum(1, keepdim=True)
    return torch.where(top == -math.inf, -1, experts).int(), e / total


def _route_grad(logits, experts, dw, renorm):
    z, index = logits.float(), experts.long()
    if renorm:
        top = torch.gather(z, 1, index)
        e = torch.exp(top - top.amax(1, keepdim=True))
        w = e / e.sum(1, keepdim=True)
        dz = torch.zeros_like(z).scatter_add_(1, index, w * (dw - (w * dw).sum(1, keepdim=True)))
    else:
        e = torch.exp(z - z.amax(1, keepdim=True))
        p = e / e.sum(1, keepdim=True)
        dp = torch.zeros_like(z).scatter_add_(1, index, dw)
        dz = p * (dp - (p * dp).sum(1, keepdim=True))
    return dz.to(logits.dtype)


def _dispatch(experts, n_experts, x):
    t, k = experts.shape
    flat = experts.reshape(-1).long()
    key, order = torch.sort(torch.where(flat < 0, n_experts, flat), stable=True)
    kept = key < n_experts
    off = torch.searchsorted(key, torch.arange(n_experts + 1, device=key.device)).int()
    place = torch.where(kept, torch.arange(t * k, device=key.device), -1)
    pos = torch.empty_like(place).scatter_(0, order, place).int().reshape(t, k)
    token = order // k
    return torch.where(kept, token, 0).int(), off, pos, torch.where(kept[:, None], x[token], 0)


def _combine(rows, pos, weights):
    kept = pos >= 0
    w = kept.float() if weights is None else torch.where(kept, weights, 0)
    return (rows[pos.clamp(min=0).long()].float() * w[..., None]).sum(1).to(rows.dtype)


def _combine_grad(dy, rows, pos, weights):
    n, kept, g = rows.shape[0], pos >= 0, dy.float()
    dw = torch.where(kept, (rows[pos.clamp(min=0).long()].float() * g[:, None, :]).sum(2), 0)
    to = torch.where(kept, pos, n).reshape(-1).long()
    drows = torch.zeros((n + 1, rows.shape[1]), dtype=rows.dtype, device=rows.device)
    drows.index_copy_(0, to, (weights[..., None] * g[:, None, :]).to(rows.dtype).reshape(-1, rows.shape[1]))
    return drows[:n], dw


def _clip(grads, max_norm):
    norm = torch.stack([g.double().square().sum() for g in grads]).sum().sqrt()
    scale = torch.clamp(max_norm / (norm + 1e-6), max=1.0).float()
    return torch.cat([g.float() * scale for g in grads]), norm.float()


def run(s):
    case = s["case"]
    op = case["op"]
    if own:
        import paper_2608_13757_amd as bfs
        if op == "route":
            return bfs.moe_route(s["logits"], case["k"], renormalize=case["renorm"], experts=s["experts"], weights=s["weights"])
        if op == "route_grad":
            return bfs.moe_route_grad(s["logits"], s["experts"], s["dw"], renormalize=case["renorm"], grad_logits=s["dlogits"])
        if op == "dispatch":
            return bfs.moe_dispatch(s["experts"], case["experts"], s["x"], perm=s["perm"], expert_off=s["off"], pos=s["pos"],
                                    rows=s["rows"])
        if op == "dispatch_grad":
            return bfs.moe_dispatch_grad(s["rows"], s["pos"], out=s["y"])
        if op == "combine":
            return bfs.moe_combine(s["rows"], s["pos"], s["weights"], out=s["y"])
        if op == "combine_grad":
            return bfs.moe_combine_grad(s["dy"], s["rows"], s["pos"], s["weights"], grad_rows=s["drows"], grad_weights=s["dw"])
        norm = s["set"].clip(1.0, norm=s["norm"])
        return s["flat"], norm
    if op == "route":
        return _route(s["logits"], case["k"], case["renorm"])
    if op == "route_grad":
        return _route_grad(s["logits"], s["experts"], s["dw"], case["renorm"])
    if op == "dispatch":
        return _dispatch(s["experts"], case["experts"], s["x"])
    if op == "dispatch_grad":
        return _combine(s["rows"], s["pos"], None)
    if op == "combine":
        return _combine(s["rows"], s["pos"], s["weights"])
    if op == "combine_grad":
        return _combine_grad(s["dy"], s["rows"], s["pos"], s["weights"])
    return _clip(s["grads"], 1.0)


def work(case):
    """Every input read once, every output written once."""
    op, b = case["op"], DTYPES[case["dtype"]].itemsize
    if op == "clip":
        n = case["params"]
        return {"bytes": n * (b + 4) + 4, "flops": 3 * n}
    t, k, e = case["tokens"], case["k"], case["experts"]
    if op == "route":
        return {"bytes": t * e * b + t * k * 8, "flops": t * (4 * e + k * e)}
    if op == "route_grad":
        return {"bytes": 2 * t * e * b + t * k * 8, "flops": t * (6 * e + 4 * k)}
    h, slots = case["hidden"], t * k
    if op == "dispatch":
        return {"bytes": (t + slots) * h * b + 4 * (3 * slots + e + 1), "flops": 0}
    if op == "dispatch_grad":
        return {"bytes": (t + slots) * h * b + 4 * slots, "flops": slots * h}
    if op == "combine":
        return {"bytes": (t + slots) * h * b + 8 * slots, "flops": 2 * slots * h}
    return {"bytes": (t + 2 * slots) * h * b + 12 * slots, "flops": 3 * slots * h}


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "clip":
        total = math.fsum(float(torch.dot(g, g)) for g in (x.double() for x in s["grads"]))
        scale = min(1.0, 1.0 / (math.sqrt(total) + 1e-6))
        out = torch.empty(case["params"], dtype=torch.float64, device="cuda")
        at = 0
        for g in s["grads"]:
            out[at : at + g.numel()] = g.double().mul_(scale)
            at += g.numel()
        return out, torch.tensor(math.sqrt(total), dtype=torch.float64)
    k = case["k"]
    if op == "route":
        z = s["logits"].double().cpu().numpy()
        order = np.argsort(-z, axis=1, kind="stable")[:, :k]
        p = np.exp(z - z.max(axis=1, keepdims=True))
        w = np.take_along_axis(p, order, axis=1)
        return torch.from_numpy(order.astype(np.int32)), torch.from_numpy(w / (w if case["renorm"] else p).sum(axis=1, keepdims=True))
    if op == "route_grad":
        # by the Jacobian of the softmax over the experts that take part
        z, dw = s["logits"].double(), s["dw"].double()
        chosen = torch.zeros_like(z, dtype=torch.bool)
        g = torch.zeros_like(z)
        for j in range(k):
            row = torch.arange(z.shape[0], device="cuda"), s["experts"][:, j].long()
            chosen[row] = True
            g[row] = dw[:, j]
        logp = z - torch.logsumexp(torch.where(chosen, z, -math.inf) if case["renorm"] else z, 1, keepdim=True)
        p = torch.where(chosen, logp.exp(), 0) if case["renorm"] else logp.exp()
        return g * p - p * (g * p).sum(1, keepdim=True)
    if op == "dispatch":
        flat, n = s["experts"].reshape(-1), s["experts"].numel()
        groups = [torch.nonzero(flat == e).reshape(-1) for e in range(case["experts"])]
        off = np.concatenate([[0], np.cumsum([len(g) for g in groups])]).astype(np.int32)
        slots = torch.cat(groups)
        m = slots.numel()
        perm, pos = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.full((n,), -1, dtype=torch.int32, device="cuda")
        rows = torch.zeros((n, case["hidden"]), dtype=torch.float64, device="cuda")
        perm[:m] = torch.div(slots, k, rounding_mode="floor").int()
        pos[slots] = torch.arange(m, dtype=torch.int32, device="cuda")
        rows[:m] = s["x"].double()[perm[:m].long()]
        return perm, torch.from_numpy(off), pos.reshape(-1, k), rows
    y = torch.zeros((case["tokens"], case["hidden"]), dtype=torch.float64, device="cuda")
    if op in ("combine", "dispatch_grad"):
        for j in range(k):
            t = torch.nonzero(s["pos"][:, j] >= 0).reshape(-1)
            r = s["rows"][s["pos"][t, j].long()].double()
            y[t] += r if op == "dispatch_grad" else r * s["weights"][t, j].double()[:, None]
        return y
    drows = torch.zeros(s["rows"].shape, dtype=torch.float64, device="cuda")
    dw = torch.zeros(s["pos"].shape, dtype=torch.float64, device="cuda")
    for j in range(k):
        t = torch.nonzero(s["pos"][:, j] >= 0).reshape(-1)
        at, g = s["pos"][t, j].long(), s["dy"][t].double()
        drows[at] = g * s["weights"][t, j].double()[:, None]
        dw[t, j] = torch.linalg.vecdot(g, s["rows"][at].double())
    return drows, dw
