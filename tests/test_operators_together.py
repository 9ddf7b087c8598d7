"""Layer norm, cross attention, their backward passes and the clipping of all gradients in one training step, as a block of a network runs
them: the points of a batch of scans are bucketized and attend inside their scopes, are pooled, and then attend to the pooled points of
their own scan (`pooled_offsets` are the states' offsets). Every operator's result is checked against the definition in binary64 on
what the step handed to it, and the step gives the same bits eagerly, on another stream and replayed from a graph.
"""
import math

import pytest
import torch

import paper_2412_16481_amd as f3d
from test_cross_attention import check_forward as check_attention
from test_norm_and_clip import forward64, half, least, U

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
C, H, K, D = 64, 4, 2, 16


def block(scans):
    """What a network has in hand: coordinates, features, weights, buckets, and everything the step writes."""
    g = torch.Generator(device=DEV).manual_seed(sum(scans))
    n = sum(scans)
    r = lambda *s: torch.randn(*s, generator=g, device=DEV)   # noqa: E731
    bo = torch.tensor([sum(scans[:i]) for i in range(len(scans) + 1)], dtype=torch.int32, device=DEV)
    coords = torch.rand(n, 3, generator=g, device=DEV) * 4
    p = f3d.make_params(0.05, 256, 4, max_scan_points=max(scans))
    bk = f3d.psh_bucketize(coords, bo, p)
    bf = torch.bfloat16
    return {"n": n, "bo": bo, "coords": coords, "bk": bk, "max_q": max(scans), "x": r(n, C).to(bf), "feat": r(n, C).to(bf),
            "gamma": 1 + 0.2 * r(C), "beta": 0.2 * r(C), "wkv": (r(2 * K * D, C) / 8).to(bf), "dout": (0.1 * r(n, H * D)).to(bf),
            "dw": 0.01 * r(513, 7)}


def step(d):
    """One step. The points' own rows are normalised into bucket-major order and are the queries."""
    n, o = d["n"], {}
    pooled = f3d.inbucket_pool(d["coords"], d["bk"].perm, d["feat"], d["bo"], 256, 4, 0.05)
    o["kv_off"] = pooled.pooled_offsets
    o["k"], o["v"] = f3d.ln_linear(pooled.feat, d["wkv"], n_outs=2)
    o["mean"], o["rstd"] = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    o["y"] = f3d.layer_norm(d["x"], d["gamma"], d["beta"], 1e-5, d["bk"].perm, mean=o["mean"], rstd=o["rstd"])
    o["lse"] = torch.empty(n, H, device=DEV)
    o["out"] = f3d.cross_attn(o["y"], o["k"], o["v"], d["bo"], o["kv_off"], H, D, K, d["max_q"], lse=o["lse"])
    o["dq"], o["dk"], o["dv"] = f3d.cross_attn_bwd(o["y"], o["k"], o["v"], o["out"], d["dout"], o["lse"], d["bo"], o["kv_off"], H, D, K, d["max_q"])
    o["dx"], o["dgamma"], o["dbeta"] = f3d.layer_norm_bwd(o["dq"], d["x"], o["mean"], o["rstd"], d["gamma"], d["bk"].perm)
    grads = [o["dx"], o["dk"], o["dv"], o["dgamma"], o["dbeta"], d["dw"]]
    o["clipped"] = [torch.empty_like(x) for x in grads]
    o["norm"] = f3d.clip_grads(grads, 0.5, o["clipped"])
    return o


def tensors(o):
    """The results, without the rows of pooled points that there are not."""
    rows = int(o["kv_off"][-1])
    for name, x in o.items():
        if name == "clipped":
            yield from x
        else:
            yield x[:rows] if name in ("k", "v") else x


def close(got, want, bound, what):
    bad = (got.double() - want).abs() - bound
    assert bool((bad <= 0).all()), f"{what}: off by up to {float(bad.max()):.3g} more than the bound"


@pytest.mark.parametrize("scans", [[700], [1000, 0, 37, 2000], [1] * 5])
def test_a_block_of_points_and_pooled_points(scans):
    d = block(scans)
    o = step(d)
    perm, n = d["bk"].perm, d["n"]
    bf = torch.bfloat16
    # layer norm
    want, mean, rstd = forward64(d["x"], d["gamma"], d["beta"], 1e-5, perm)
    close(o["y"], want, half(bf) * want.abs() + 512 * U * (1 + want.abs()) * 8, "y")
    # attention to the pooled points; what lies behind them is nobody's
    off = o["kv_off"].tolist()
    assert off[-1] > 0 and off[-1] <= o["k"].shape[0]
    c = {"q": o["y"], "k": o["k"], "v": o["v"], "q_off": d["bo"], "kv_off": o["kv_off"], "q_len": scans, "kv_len": [b - a for a, b in zip(off, off[1:])],
         "H": H, "K": K, "D": D, "t": bf}
    check_attention(c, o["out"], o["lse"], untouched=False)
    # its gradients: relative to the size of what was added up, a rounding of P or dS (2^-8), one of the result, and what lse and the
    # sums in binary32 leave, below 2^-12 for these lengths
    for b, m in enumerate(scans):
        rows, keys = slice(int(d["bo"][b]), int(d["bo"][b + 1])), slice(off[b], off[b + 1])
        dk, dv = torch.zeros(keys.stop - keys.start, K * D, dtype=torch.float64, device=DEV), None
        dv, size_k, size_v = dk.clone(), dk.clone(), dk.clone()
        for h in range(H):
            j = h * K // H
            col, kc = slice(h * D, (h + 1) * D), slice(j * D, (j + 1) * D)
            q, k, v = (x.double() for x in (o["y"][rows, col], o["k"][keys, kc], o["v"][keys, kc]))
            do, out = d["dout"][rows, col].double(), o["out"][rows, col].double()
            p = torch.exp(q @ k.T / 4 - o["lse"][rows, h].double()[:, None])
            ds = p * (do @ v.T - (do * out).sum(1, keepdim=True))
            magnitude = p * (do.abs() @ v.abs().T + (do * out).abs().sum(1, keepdim=True))
            room = half(bf) * ds.abs() + 2.0 ** -12 * magnitude
            want = ds @ k / 4
            close(o["dq"][rows, col], want, room @ k.abs() / 2 + half(bf) * want.abs() + least(bf), f"dq of scan {b}")
            dk[:, kc] += ds.T @ q / 4
            size_k[:, kc] += room.T @ q.abs() / 2
            dv[:, kc] += p.T @ do
            size_v[:, kc] += ((half(bf) + 2.0 ** -12) * p).T @ do.abs() * 2
        close(o["dk"][keys], dk, size_k + half(bf) * dk.abs() + least(bf), f"dk of scan {b}")
        close(o["dv"][keys], dv, size_v + half(bf) * dv.abs() + least(bf), f"dv of scan {b}")
    assert bool((o["dk"][off[-1]:] == 0).all()) and bool((o["dv"][off[-1]:] == 0).all())
    # layer norm's gradients, to the rows' own places
    rows = perm.long()
    xh = (d["x"].double()[rows] - mean[:, None]) * rstd[:, None]
    dy = o["dq"].double()
    g = dy * d["gamma"].double()
    want = torch.empty_like(xh)
    want[rows] = rstd[:, None] * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    room = torch.empty_like(xh)
    room[rows] = 2048 * U * rstd[:, None] * (g.abs() + g.abs().mean(1, keepdim=True) + (1 + xh.abs()) * (g.abs() * (1 + xh.abs())).mean(1, keepdim=True))
    close(o["dx"], want, half(bf) * want.abs() + room + least(bf), "dx")
    close(o["dgamma"], (dy * xh).sum(0), 2048 * U * (dy.abs() * (1 + xh.abs())).sum(0), "dgamma")
    close(o["dbeta"], dy.sum(0), 512 * U * dy.abs().sum(0), "dbeta")
    # all of them together
    grads = [o["dx"], o["dk"], o["dv"], o["dgamma"], o["dbeta"], d["dw"]]
    total = math.sqrt(sum(float(x.double().square().sum()) for x in grads))
    assert abs(float(o["norm"]) - total) <= 4 * U * total
    factor = min(1.0, 0.5 / (total + 1e-6))
    for x, y in zip(grads, o["clipped"]):
        want = x.double() * factor
        close(y, want, (half(x.dtype) + 4 * U) * want.abs() + least(x.dtype), "clipped")


def test_a_block_gives_the_same_bits_on_another_stream_and_from_a_graph():
    d = block([900, 0, 1400])
    want = [x.clone() for x in tensors(step(d))]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        o = step(d)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(tensors(o), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o = step(d)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(tensors(o), want))
        assert all(torch.equal(a, b) for a, b in zip(tensors(step(d)), want))
        torch.cuda.synchronize()
