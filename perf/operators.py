"""Layer norm and its gradients, attention to states of another length and its gradients, and the clipping of gradients by
their global norm, as a list of cases.

Every case is a dict of plain values. `prepare` makes what a program holds before the call, `run` is one pass through one
operator: with `own` through the library's entry points, else in its plain form, elementary torch operations in binary32 that
round once at the end. `exact` says in binary64 what comes out."""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
EPS = 1e-5
DEV = "cuda"


# --------------------------------------------------------------------------- cases


def _norm(name, rows, channels, dtype, gather):
    return {"name": name, "kind": "norm", "rows": rows, "channels": channels, "dtype": dtype, "gather": gather}


def _norm_grad(name, rows, channels, dtype, gather, residual):
    return {"name": name, "kind": "norm_grad", "rows": rows, "channels": channels, "dtype": dtype, "gather": gather, "residual": residual}


def _attend(name, batch, q, kv, ragged, heads, kv_heads, head_dim, dtype, padded=False, lse=False):
    return {"name": name, "kind": "attend", "batch": batch, "q": q, "kv": kv, "ragged": ragged, "heads": heads, "kv_heads": kv_heads,
            "head_dim": head_dim, "dtype": dtype, "padded": padded, "lse": lse}


def _attend_grad(name, batch, q, kv, ragged, heads, kv_heads, head_dim, padded=False):
    return {"name": name, "kind": "attend_grad", "batch": batch, "q": q, "kv": kv, "ragged": ragged, "heads": heads, "kv_heads": kv_heads,
            "head_dim": head_dim, "dtype": "bf16", "padded": padded, "lse": True}


def _clip(name, params, layers, dtype, mixed):
    return {"name": name, "kind": "clip", "params": params, "layers": layers, "dtype": dtype, "mixed": mixed}


def listed():
    return [
        # a decoder's step of a few sequences: latency
        _norm("norm_tokens", 33, 256, "f16", False),
        # one layer of a batch of driving scans, rows gathered into bucket-major order, statistics kept for the backward pass
        _norm("norm_lidar8", 914601, 256, "bf16", True),
        # the backward of that layer: the gradient of the residual path is added, rows go back to the points' order
        _norm_grad("norm_grad_lidar8", 914601, 256, "bf16", True, True),
        # a wide layer of odd width in binary32
        _norm_grad("norm_grad_odd", 9001, 1537, "f32", False, False),
        # one query per request against its own cached states, shared heads, a cache of fixed length filled to different degrees
        _attend("attend_one_token", 32, 1, 4096, 0.7, 32, 8, 128, "bf16", padded=True),
        # the smallest request: one query of one object and a short prompt
        _attend("attend_prompt", 1, 1, 77, 0.0, 4, 4, 16, "f16"),
        # a batch of driving scans whose points look at a few hundred image or map states of their own scan
        _attend("attend_lidar8", 8, 114325, 256, 0.0005, 8, 8, 32, "bf16", lse=True),
        # ragged batches of decoder rows and encoder states in binary16, shared heads
        _attend("attend_f16_ragged", 16, 2047, 1500, 0.6, 12, 4, 64, "f16"),
        # training: the points of a room and a prompt of 77 states
        _attend_grad("attend_grad_indoor", 1, 200000, 77, 0.0, 4, 4, 16),
        # training: ragged batches of decoder rows and encoder states, shared wide heads
        _attend_grad("attend_grad_ragged", 8, 2047, 1500, 0.5, 16, 4, 128),
        # a small network's gradients: hundreds of tensors, weights in bfloat16, vectors in binary32
        _clip("clip_small", 1500000, 24, "bf16", True),
        # a large one's
        _clip("clip_large", 400000000, 48, "bf16", False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _unnamed(case):
    return {k: v for k, v in case.items() if k != "name"}


def draw(rng):
    kind = rng.choice(["norm", "norm_grad", "attend", "attend", "attend_grad", "clip"])
    if kind in ("norm", "norm_grad"):
        channels = rng.choice([_log_int(rng, 16, 4096), 64, 128, 256, 512, 1024, 2048])
        rows = _log_int(rng, 1, 110000000 // max(channels, 256))
        dtype, gather = rng.choice(["bf16", "bf16", "f16", "f32"]), rng.random() < 0.5
        if kind == "norm":
            return _unnamed(_norm("", rows, channels, dtype, gather))
        return _unnamed(_norm_grad("", rows, channels, dtype, gather, rng.random() < 0.5))
    if kind == "clip":
        return _unnamed(_clip("", _log_int(rng, 100000, 200000000), rng.randint(2, 48), rng.choice(["bf16", "f16", "f32"]), rng.random() < 0.5))
    head_dim = rng.choice([16, 32, 64, 128])
    kv_heads = rng.choice([1, 2, 3, 4, 8])
    heads = kv_heads * rng.choice([1, 1, 2, 3, 4] if head_dim < 128 else [1, 2, 4])
    batch, ragged, padded = _log_int(rng, 1, 24), rng.choice([0.0, 0.2, 0.7]), rng.random() < 0.3
    form, dtype, lse = rng.choice(["single", "few", "rows", "points"]), rng.choice(["bf16", "bf16", "f16"]), rng.random() < 0.5
    if form == "single":
        q, kv = 1, _log_int(rng, 1, 8192)
    elif form == "few":
        q, kv = rng.randint(2, 64), _log_int(rng, 8, 4096)
    elif form == "rows":
        q, kv = _log_int(rng, 65, 2048), _log_int(rng, 17, 2048)
    else:
        batch = rng.randint(1, 4)
        q, kv = _log_int(rng, 5000, 100000), _log_int(rng, 1, 400)
    while True:     # no more than the largest listed ones
        if kind == "attend":
            c = _attend("", batch, q, kv, ragged, heads, kv_heads, head_dim, dtype, padded, lse)
        else:
            c = _attend_grad("", batch, q, kv, ragged, heads, kv_heads, head_dim, padded)
        if work(c)["bytes"] <= 1.8e9 and work(c)["flops"] <= (2.2e11 if kind == "attend" else 2.8e11):
            return _unnamed(c)
        q, kv = max(1, q * 2 // 3), max(1, kv * 2 // 3)


def _lengths(case):
    """Query rows and states of every segment: the longest first, the others shorter by up to the case's share."""
    part = [0.0] + [math.fmod(0.6180339887 * i, 1.0) for i in range(1, case["batch"])]
    q = [max(1, round(case["q"] * (1.0 - case["ragged"] * f))) for f in part]
    return q, [max(1, round(case["kv"] * (1.0 - case["ragged"] * math.fmod(7.0 * f, 1.0)))) for f in part]


def _shapes(case):
    """The tensors of a network of that many layers: per layer four maps of c x c, one c x 4c and back, and eight vectors."""
    c = max(3, round(math.sqrt(case["params"] / (12.0 * case["layers"]))))
    vector = DTYPES["f32" if case["mixed"] else case["dtype"]]
    layer = [((c, c), DTYPES[case["dtype"]])] * 4 + [((4 * c, c), DTYPES[case["dtype"]]), ((c, 4 * c), DTYPES[case["dtype"]])] + [((c,), vector)] * 8
    return layer * case["layers"]


def work(case):
    size = {"bf16": 2, "f16": 2, "f32": 4}[case["dtype"]]
    if case["kind"] == "norm":
        elements = case["rows"] * case["channels"]
        return {"bytes": 2 * elements * size + case["rows"] * (12 if case["gather"] else 8), "flops": 8 * elements}
    if case["kind"] == "norm_grad":
        elements = case["rows"] * case["channels"]
        return {"bytes": (4 if case["residual"] else 3) * elements * size + case["rows"] * (12 if case["gather"] else 8), "flops": 14 * elements}
    if case["kind"] == "clip":
        elements = [(math.prod(s), 4 if t == torch.float32 else 2) for s, t in _shapes(case)]
        return {"bytes": 2 * sum(n * b for n, b in elements), "flops": 3 * sum(n for n, _ in elements)}
    q, kv = _lengths(case)
    rows = sum(q) * case["heads"] * case["head_dim"] * 2
    states = sum(kv) * case["kv_heads"] * case["head_dim"] * 2
    pairs = sum(a * b for a, b in zip(q, kv)) * case["heads"] * case["head_dim"]
    lse = 4 * sum(q) * case["heads"] if case["lse"] else 0
    if case["kind"] == "attend":
        return {"bytes": 2 * rows + 2 * states + lse, "flops": 4 * pairs}
    return {"bytes": 4 * rows + 4 * states + lse, "flops": 10 * pairs}


# --------------------------------------------------------------------------- inputs


def _inputs(case, seed):
    """The data of a case, from the seed alone."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    t = DTYPES[case["dtype"]]

    def normal(*shape, dtype=t, scale=1.0, shift=0.0):
        return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32).mul_(scale).add_(shift).to(dtype)

    if case["kind"] in ("norm", "norm_grad"):
        n, c = case["rows"], case["channels"]
        offset = normal(c, dtype=torch.float32, scale=0.5)          # features whose channels have means of their own
        d = {"x": (normal(n, c, dtype=torch.float32) + offset).to(t), "gamma": normal(c, dtype=torch.float32, scale=0.2, shift=1.0),
             "beta": normal(c, dtype=torch.float32, scale=0.2)}
        d["row_in"] = torch.randperm(n, generator=g, device=DEV).to(torch.int32) if case["gather"] else None
        if case["kind"] == "norm_grad":
            d["dy"] = normal(n, c, scale=0.05)
            d["residual"] = normal(n, c, scale=0.05) if case["residual"] else None
            rows = d["x"] if d["row_in"] is None else d["x"].index_select(0, d["row_in"])
            d["mean"] = rows.mean(1, dtype=torch.float32)
            d["rstd"] = (rows.float() - d["mean"][:, None]).square().mean(1).add(EPS).rsqrt()
        return d
    if case["kind"] == "clip":
        return {"grads": [normal(*s, dtype=dt, scale=1e-3) for s, dt in _shapes(case)], "max_norm": 1.0}
    q_len, kv_len = _lengths(case)
    H, K, D = case["heads"], case["kv_heads"], case["head_dim"]

    def ends(lengths):
        return torch.tensor([0, *torch.tensor(lengths).cumsum(0).tolist()], dtype=torch.int32, device=DEV)

    longest = [case["kv"]] * case["batch"] if case["padded"] else kv_len
    d = {"q": normal(sum(q_len), H * D, scale=1.5), "k": normal(sum(longest), K * D), "v": normal(sum(longest), K * D),
         "q_offsets": ends(q_len), "kv_offsets": ends(longest), "max_q": max(q_len), "max_kv": max(longest),
         "kv_lens": torch.tensor(kv_len, dtype=torch.int32, device=DEV) if case["padded"] else None}
    if case["kind"] == "attend_grad":
        d["dout"] = normal(sum(q_len), H * D, scale=0.1)
        d["out"], d["lse"] = _attention(d, H, K, D)                 # what the forward pass has left
    return d


def _buffers(tensors, dtype=None):
    """One flat buffer for all tensors of a type, as a program that exchanges or updates them together keeps them, and its views of
    the tensors' shapes, each beginning at a multiple of 64 elements."""
    ends, at = {}, []
    for x in tensors:
        at.append(ends.get(x.dtype, 0))
        ends[x.dtype] = at[-1] + (x.numel() + 63) // 64 * 64
    flat = {t: torch.zeros(n, dtype=dtype or t, device=DEV) for t, n in ends.items()}
    return list(flat.values()), [flat[x.dtype][i:i + x.numel()].view(x.shape) for i, x in zip(at, tensors)]


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["kind"] == "norm":
        s["y"], s["mean"], s["rstd"] = torch.empty_like(s["x"]), *(torch.empty(case["rows"], device=DEV) for _ in range(2))
    elif case["kind"] == "norm_grad":
        s["dx"] = torch.empty_like(s["x"])
    elif case["kind"] == "clip":
        s["buffers"], s["outs"] = _buffers(s["grads"])
    elif case["kind"] == "attend":
        s["o"] = torch.empty_like(s["q"])
        s["l"] = torch.empty(s["q"].shape[0], case["heads"], device=DEV) if case["lse"] else None
    return s


# --------------------------------------------------------------------------- plain forms


def _padded(x, offsets, longest, heads):
    """[rows, heads * d] -> binary32 [batch, heads, longest, d]; rows behind a segment's end repeat some row."""
    at = (offsets[:-1, None].long() + torch.arange(longest, device=DEV)).clamp(max=x.shape[0] - 1)
    return x.float()[at].unflatten(2, (heads, -1)).transpose(1, 2).contiguous()


def _rows(x, offsets, n):
    """[batch, heads, longest, d] -> [n, heads * d]: row i of the segment that begins at offsets[b] is row offsets[b] + i."""
    i = torch.arange(n, device=DEV)
    b = torch.searchsorted(offsets[1:].long().contiguous(), i, right=True).clamp(max=x.shape[0] - 1)
    return x[b, :, i - offsets.long()[b]].flatten(1)


def _valid(lengths, longest):
    return torch.arange(longest, device=DEV)[None] < lengths[:, None]


def _scores(s, H, K, D):
    """Queries and states per segment with the shared heads' queries below each other, and their scaled scores."""
    q = _padded(s["q"], s["q_offsets"], s["max_q"], H).unflatten(1, (K, H // K)).flatten(2, 3)
    k, v = (_padded(s[x], s["kv_offsets"], s["max_kv"], K) for x in "kv")
    lengths = s["kv_lens"] if s["kv_lens"] is not None else s["kv_offsets"].diff()
    sees = _valid(lengths, s["max_kv"])[:, None, None]
    return q, k, v, torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(1.0 / math.sqrt(D)).masked_fill_(~sees, -math.inf)


def _back(x, s, H, K):
    """Results of the shared heads, below each other, as rows of all heads."""
    return _rows(x.unflatten(2, (H // K, s["max_q"])).flatten(1, 2), s["q_offsets"], s["q"].shape[0])


def _attention(s, H, K, D):
    _, _, v, scores = _scores(s, H, K, D)
    top = scores.amax(3, keepdim=True)
    p = scores.sub_(top).exp_()
    total = p.sum(3, keepdim=True)
    out = torch.matmul(p, v).div_(total)
    return _back(out, s, H, K).to(s["q"].dtype), _back(top + total.log(), s, H, K)


def _attention_grad(s, H, K, D):
    q, k, v, scores = _scores(s, H, K, D)
    group, scale, n = H // K, 1.0 / math.sqrt(D), s["k"].shape[0]
    rows = _valid(s["q_offsets"].diff(), s["max_q"]).repeat(1, group)[:, None, :, None]
    o, do = (_padded(s[x], s["q_offsets"], s["max_q"], H).unflatten(1, (K, group)).flatten(2, 3) for x in ("out", "dout"))
    lse = _padded(s["lse"], s["q_offsets"], s["max_q"], H).unflatten(1, (K, group)).flatten(2, 3)
    p = scores.sub_(lse).exp_().masked_fill_(~rows, 0.0)
    dv = torch.matmul(p.transpose(2, 3).contiguous(), do)
    ds = torch.matmul(do, v.transpose(2, 3).contiguous()).sub_((o * do).sum(3, keepdim=True)).mul_(p).mul_(scale)
    dk = torch.matmul(ds.transpose(2, 3).contiguous(), q)
    t = s["q"].dtype
    return _back(torch.matmul(ds, k), s, H, K).to(t), _rows(dk, s["kv_offsets"], n).to(t), _rows(dv, s["kv_offsets"], n).to(t)


def _layer_norm(s):
    x = (s["x"] if s["row_in"] is None else s["x"].index_select(0, s["row_in"])).float()
    mean = x.mean(1, keepdim=True)
    x = x.sub(mean)
    rstd = x.square().mean(1, keepdim=True).add_(EPS).rsqrt_()
    return x.mul_(rstd).mul_(s["gamma"]).add_(s["beta"]).to(s["x"].dtype), mean[:, 0], rstd[:, 0]


def _layer_norm_grad(s):
    x = (s["x"] if s["row_in"] is None else s["x"].index_select(0, s["row_in"])).float()
    rstd, dy = s["rstd"][:, None], s["dy"].float()
    xhat = x.sub(s["mean"][:, None]).mul_(rstd)
    g = dy * s["gamma"]
    dx = g.sub(g.mean(1, keepdim=True)).sub_(xhat * (g * xhat).mean(1, keepdim=True)).mul_(rstd)
    if s["row_in"] is not None:
        dx = torch.empty_like(dx).index_copy_(0, s["row_in"].long(), dx)
    if s["residual"] is not None:
        dx = dx.add_(s["residual"])
    return dx.to(s["x"].dtype), dy.mul(xhat).sum(0), dy.sum(0)


def _clipped(s):
    norm = torch.stack([x.float().square().sum() for x in s["grads"]]).sum().sqrt()
    c = (s["max_norm"] / (norm + 1e-6)).clamp(max=1.0)
    _ = [out.copy_(x.float() * c) for x, out in zip(s["grads"], s["outs"])]
    return norm[None], s["buffers"]


# --------------------------------------------------------------------------- one pass


def run(s):
    case = s["case"]
    kind = case["kind"]
    if not own:
        if kind == "norm":
            return _layer_norm(s)
        if kind == "norm_grad":
            return _layer_norm_grad(s)
        if kind == "clip":
            return _clipped(s)
        heads = (case["heads"], case["kv_heads"], case["head_dim"])
        if kind == "attend":
            out, lse = _attention(s, *heads)
            return (out, lse) if case["lse"] else out
        return _attention_grad(s, *heads)
    import paper_2412_16481_amd as f3d
    if kind == "norm":
        f3d.layer_norm(s["x"], s["gamma"], s["beta"], EPS, s["row_in"], out=s["y"], mean=s["mean"], rstd=s["rstd"])
        return s["y"], s["mean"], s["rstd"]
    if kind == "norm_grad":
        return f3d.layer_norm_bwd(s["dy"], s["x"], s["mean"], s["rstd"], s["gamma"], s["row_in"], residual=s["residual"], dx=s["dx"])
    if kind == "clip":
        return f3d.clip_grads(s["grads"], s["max_norm"], outs=s["outs"]), s["buffers"]
    shape = {"kv_heads": case["kv_heads"], "max_q": s["max_q"], "max_kv": s["max_kv"], "kv_lens": s["kv_lens"]}
    if kind == "attend":
        out = f3d.cross_attn(s["q"], s["k"], s["v"], s["q_offsets"], s["kv_offsets"], case["heads"], case["head_dim"], out=s["o"], lse=s["l"], **shape)
        return (out, s["l"]) if case["lse"] else out
    return f3d.cross_attn_bwd(s["q"], s["k"], s["v"], s["out"], s["dout"], s["lse"], s["q_offsets"], s["kv_offsets"], case["heads"],
                              case["head_dim"], **shape)


# --------------------------------------------------------------------------- binary64


def exact(case, seed):
    s = _inputs(case, seed)
    if case["kind"] in ("norm", "norm_grad"):
        x = s["x"].double()
        if s["row_in"] is not None:
            x = x[s["row_in"].long()]
        if case["kind"] == "norm":
            var, mean = torch.var_mean(x, 1, correction=0)
            rstd = 1.0 / torch.sqrt(var + EPS)
            return (x - mean[:, None]) * rstd[:, None] * s["gamma"].double() + s["beta"].double(), mean, rstd
        mean, rstd, dy = s["mean"].double()[:, None], s["rstd"].double()[:, None], s["dy"].double()
        xhat = (x - mean) * rstd
        g = dy * s["gamma"].double()
        dx = torch.zeros_like(x) if s["residual"] is None else s["residual"].double()
        term = rstd * (g - g.sum(1, keepdim=True) / case["channels"] - xhat * ((g * xhat).sum(1, keepdim=True) / case["channels"]))
        if s["row_in"] is None:
            dx = dx + term
        else:
            dx.index_add_(0, s["row_in"].long(), term)
        return dx, (dy * xhat).sum(0), dy.sum(0)
    if case["kind"] == "clip":
        norm = math.sqrt(sum(float(x.double().pow(2).sum()) for x in s["grads"]))
        flat, views = _buffers(s["grads"], torch.float64)
        for x, out in zip(s["grads"], views):
            out.copy_(x).mul_(min(1.0, s["max_norm"] / (norm + 1e-6)))
        return torch.tensor([norm], dtype=torch.float64), flat
    q_len, kv_len = _lengths(case)
    H, K, D = case["heads"], case["kv_heads"], case["head_dim"]
    q0, k0 = s["q_offsets"].tolist(), s["kv_offsets"].tolist()
    n = s["q"].shape[0]
    if case["kind"] == "attend":
        out, lse = torch.empty(n, H, D, dtype=torch.float64, device=DEV), torch.empty(n, H, dtype=torch.float64, device=DEV)
        for b, (m, l) in enumerate(zip(q_len, kv_len)):
            for h in range(H):
                q = s["q"][q0[b]:q0[b] + m, h * D:(h + 1) * D].double()
                k, v = (s[x][k0[b]:k0[b] + l, h * K // H * D:(h * K // H + 1) * D].double() for x in "kv")
                score = q @ k.T / math.sqrt(D)
                lse[q0[b]:q0[b] + m, h] = torch.logsumexp(score, 1)
                out[q0[b]:q0[b] + m, h] = torch.softmax(score, 1) @ v
        return (out.flatten(1), lse) if case["lse"] else out.flatten(1)
    dq = torch.empty(n, H, D, dtype=torch.float64, device=DEV)
    dk, dv = (torch.zeros(s["k"].shape[0], K, D, dtype=torch.float64, device=DEV) for _ in range(2))
    for b, (m, l) in enumerate(zip(q_len, kv_len)):
        for h in range(H):
            rows, at, j = slice(q0[b], q0[b] + m), slice(k0[b], k0[b] + l), h * K // H
            col, kcol = slice(h * D, (h + 1) * D), slice(j * D, (j + 1) * D)
            q, do, o = (s[x][rows, col].double() for x in ("q", "dout", "out"))
            k, v = (s[x][at, kcol].double() for x in "kv")
            p = torch.exp(q @ k.T / math.sqrt(D) - s["lse"][rows, h].double()[:, None])
            ds = p * (do @ v.T - (do * o).sum(1, keepdim=True)) / math.sqrt(D)
            dq[rows, h] = ds @ k
            dk[at, j] += ds.T @ q
            dv[at, j] += p.T @ do
    return dq.flatten(1), dk.flatten(1), dv.flatten(1)
