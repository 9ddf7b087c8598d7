"""Attention to states of another length, forward and backward, on the GPU through the C ABI against the definition in binary64.

Tolerances, with u = 2^-24 and h half a step of the 16-bit type relative to the value (bf16 2^-8, binary16 2^-11). A score is a sum of
head_dim products, off by at most e = scale (head_dim + 8) u sum |q||k| plus 8 u of its size (scaling, fma, the exponential); that changes
its probability by the factor 1 + 2 e at most. Probabilities are rounded to 16 bits (h), in binary16 below 2^-14 by up to 2^-25 of
the reference, which no row's sum is below. Sums in binary32 over n terms are off by (n + 8) u of the sum of the magnitudes.
"""
import math

import pytest
import torch

import paper_2412_16481_amd as f3d

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U = 2.0 ** -24
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def half(t):
    return torch.finfo(t).eps / 2


def least(t):
    return torch.finfo(t).smallest_normal * torch.finfo(t).eps / 2


def close(got, want, bound, what):
    assert got.shape == want.shape
    bad = (got.double() - want).abs() - bound
    assert bool((bad <= 0).all()), f"{what}: {int((~(bad <= 0)).sum())} of {bad.numel()} outside, by up to {float(bad.max()):.3g}"


def ends(lengths, first=0):
    at = [first]
    for n in lengths:
        at.append(at[-1] + n)
    return torch.tensor(at, dtype=torch.int32, device=DEV)


def make(q_len, kv_len, H, K, D, t, seed=0, q_scale=1.0, first=(0, 0), behind=(0, 0)):
    """Tensors of the segments, with `first` rows in front of them and `behind` rows past them that belong to nobody."""
    g = torch.Generator(device=DEV).manual_seed(seed + sum(q_len) * 131 + sum(kv_len) * 17 + H * 7 + D)
    n, m = first[0] + sum(q_len) + behind[0], first[1] + sum(kv_len) + behind[1]
    r = lambda rows, c, s=1.0: (torch.randn(rows, c, generator=g, device=DEV) * s).to(TYPES[t])   # noqa: E731
    return {"q": r(n, H * D, q_scale), "k": r(m, K * D), "v": r(m, K * D), "dout": r(n, H * D, 0.1), "q_off": ends(q_len, first[0]),
            "kv_off": ends(kv_len, first[1]), "q_len": q_len, "kv_len": kv_len, "H": H, "K": K, "D": D, "t": TYPES[t],
            "max_q": max(q_len + [1]), "max_kv": max(kv_len + [1])}


def forward(d, lse=True, scale=0.0, q_lens=None, kv_lens=None, bounds=True, **kw):
    out = torch.full_like(d["q"], 7.0)
    l = torch.full((d["q"].shape[0], d["H"]), 7.0, device=DEV) if lse else None
    m = {"max_q": d["max_q"], "max_kv": d["max_kv"]} if bounds else {}
    f3d.cross_attn(d["q"], d["k"], d["v"], d["q_off"], d["kv_off"], d["H"], d["D"], d["K"], q_lens=q_lens, kv_lens=kv_lens, softmax_scale=scale,
                   out=out, lse=l, **m, **kw)
    return out, l


def pieces(d, q_lens, kv_lens):
    """(query rows, key rows, head, key/value head, rows behind the length) of every segment and head."""
    q0, k0 = d["q_off"].tolist(), d["kv_off"].tolist()
    for b in range(len(d["q_len"])):
        m = d["q_len"][b] if q_lens is None else q_lens[b]
        l = d["kv_len"][b] if kv_lens is None else kv_lens[b]
        for h in range(d["H"]):
            yield slice(q0[b], q0[b] + m), slice(k0[b], k0[b] + l), h, h * d["K"] // d["H"], slice(q0[b] + m, q0[b + 1])


def scores(d, rows, keys, h, j, scale):
    D = d["D"]
    q, k = d["q"][rows, h * D:(h + 1) * D].double(), d["k"][keys, j * D:(j + 1) * D].double()
    s = q @ k.T * scale
    e = (scale * (q.abs() @ k.abs().T) * (D + 8) * U + 8 * U * (1 + s.abs()))
    return q, k, s, e


def check_forward(d, out, lse, scale=0.0, q_lens=None, kv_lens=None, untouched=True):
    D, t = d["D"], d["t"]
    sc = scale or 1 / math.sqrt(D)
    mine = torch.zeros(out.shape[0], dtype=torch.bool, device=DEV)
    mine[int(d["q_off"][0]):int(d["q_off"][-1])] = True
    if untouched:
        assert bool((out[~mine] == 7).all()) and (lse is None or bool((lse[~mine] == 7).all())), "rows of no segment"
    for rows, keys, h, j, rest in pieces(d, q_lens, kv_lens):
        col = slice(h * D, (h + 1) * D)
        if keys.stop == keys.start:
            rest = slice(rows.start, rest.stop)
        assert bool((out[rest, col] == 0).all()) and (lse is None or bool((lse[rest, h] == -math.inf).all())), "rows without keys"
        if keys.stop == keys.start or rows.stop == rows.start:
            continue
        _, _, s, e = scores(d, rows, keys, h, j, sc)
        v = d["v"][keys, j * D:(j + 1) * D].double()
        n = keys.stop - keys.start
        p = torch.softmax(s, 1)
        worst = e.amax(1, keepdim=True)
        want, size = p @ v, p @ v.abs()
        room = size * (half(t) + 2 * worst + (n + 8) * U) + (n * 2.0 ** -25 * v.abs().amax() if t == torch.float16 else 0)
        close(out[rows, col], want, room * (1 + half(t)) + (half(t) + U) * want.abs() + least(t), f"out, head {h}, rows {rows}")
        if lse is not None:
            wl = torch.logsumexp(s, 1)
            close(lse[rows, h], wl, 2 * worst[:, 0] + (n + 8) * U + 8 * U * (1 + wl.abs()), f"lse, head {h}, rows {rows}")


def check_backward(d, scale=0.0, q_lens=None, kv_lens=None, bounds=True, **kw):
    lens = {k: None if v is None else torch.tensor(v, dtype=torch.int32, device=DEV) for k, v in (("q_lens", q_lens), ("kv_lens", kv_lens))}
    out, lse = forward(d, scale=scale, bounds=bounds, **lens)
    check_forward(d, out, lse, scale, q_lens, kv_lens)
    m = {"max_q": d["max_q"], "max_kv": d["max_kv"]} if bounds else {}
    run = lambda: f3d.cross_attn_bwd(d["q"], d["k"], d["v"], out, d["dout"], lse, d["q_off"], d["kv_off"], d["H"], d["D"], d["K"],   # noqa: E731
                                     softmax_scale=scale, **lens, **m, **kw)
    dq, dk, dv = run()
    assert all(torch.equal(a, b) for a, b in zip((dq, dk, dv), run())), "another call, other bits"
    D, t, sc = d["D"], d["t"], scale or 1 / math.sqrt(d["D"])
    want = [torch.zeros(x.shape, dtype=torch.float64, device=DEV) for x in (dq, dk, dv)]
    room = [torch.zeros_like(x) for x in want]
    for rows, keys, h, j, _ in pieces(d, q_lens, kv_lens):
        if keys.stop == keys.start or rows.stop == rows.start:
            continue
        col, kcol = slice(h * D, (h + 1) * D), slice(j * D, (j + 1) * D)
        q, k, s, e = scores(d, rows, keys, h, j, sc)
        v, do, o = d["v"][keys, kcol].double(), d["dout"][rows, col].double(), out[rows, col].double()
        p = torch.exp(s - lse[rows, h].double()[:, None])
        inner = do @ v.T - (do * o).sum(1, keepdim=True)
        off = (D + 8) * U * (do.abs() @ v.abs().T + (do * o).abs().sum(1, keepdim=True))     # of dP - D
        ds = p * inner
        e2 = 2 * e + 4 * U * (1 + lse[rows, h].double().abs()[:, None])
        room_p, room_s = p * (half(t) + e2), ds.abs() * (half(t) + e2) * (1 + half(t)) + p * off
        want[0][rows, col] = sc * ds @ k
        room[0][rows, col] = sc * (room_s + (len(k) + 8) * U * ds.abs()) @ k.abs()
        want[1][keys, kcol] += sc * ds.T @ q
        room[1][keys, kcol] += sc * (room_s + (d["H"] // d["K"] * len(q) + 8) * U * ds.abs()).T @ q.abs()
        want[2][keys, kcol] += p.T @ do
        room[2][keys, kcol] += (room_p + (d["H"] // d["K"] * len(q) + 8) * U * p).T @ do.abs()
    for name, got, w, r in zip(("dq", "dk", "dv"), (dq, dk, dv), want, room):
        close(got, w, r * (1 + half(t)) + (half(t) + U) * w.abs() + least(t), name)
    return out, lse, dq, dk, dv


SHAPES = [  # query rows and states of the segments
    ([1], [1]), ([1], [77]), ([5], [31]), ([33], [32]), ([128], [64]), ([130], [129]), ([257], [300]),
    ([1, 1, 1], [5, 200, 1]), ([3, 0, 40, 7], [60, 33, 0, 1]), ([0, 0], [4, 0]), ([300, 1, 129], [1, 513, 40]),
]


@pytest.mark.parametrize("D", [16, 32, 64, 128])
@pytest.mark.parametrize("t", ["bf16", "f16"])
@pytest.mark.parametrize("heads", [(1, 1), (4, 4), (6, 2), (5, 1)])
def test_cross_attention_shapes(D, t, heads):
    for q_len, kv_len in SHAPES:
        d = make(q_len, kv_len, *heads, D, t, q_scale=1.5)
        out, lse = forward(d)
        check_forward(d, out, lse)
        again, none = forward(d, lse=False)
        assert none is None and torch.equal(again, out)


@pytest.mark.parametrize("D", [16, 32, 64, 128])
@pytest.mark.parametrize("heads", [(1, 1), (4, 4), (6, 2), (5, 1)])
def test_cross_attention_gradients(D, heads):
    for q_len, kv_len in SHAPES:
        check_backward(make(q_len, kv_len, *heads, D, "bf16", q_scale=1.5))


@pytest.mark.parametrize("D", [16, 32, 64, 128])
@pytest.mark.parametrize("t", ["bf16", "f16"])
def test_cross_attention_single_queries_over_long_caches(D, t):
    # one query per segment, caches of a fixed length filled to different degrees: the keys are split over workgroups
    kv_lens = [4096, 1, 0, 2000, 4095, 129, 128]
    d = make([1] * 7, [4096] * 7, 8, 2, D, t)
    lens = torch.tensor(kv_lens, dtype=torch.int32, device=DEV)
    assert f3d.cross_attn_workspace_bytes(7, 7 * 4096, 7, 1, 4096, 8, 2, D) > 0
    out, lse = forward(d, kv_lens=lens)
    check_forward(d, out, lse, kv_lens=kv_lens)


@pytest.mark.parametrize("D", [16, 32, 64, 128])
@pytest.mark.parametrize("q,kv,H,K", [(20000, 77, 4, 4), (20000, 77, 4, 2), (3, 9000, 2, 1), (70000, 40, 2, 2), (200, 3000, 8, 8)])
def test_cross_attention_long_and_short_beside_each_other(D, q, kv, H, K):
    # many rows and few keys: two row tiles a wave, row sums in parts; few rows and many keys: the keys in parts
    check_backward(make([q, 1, q // 7], [kv, 3, kv], H, K, D, "bf16"))


def test_cross_attention_every_form_is_taken():
    few = f3d.cross_attn_workspace_bytes(4, 400, 4, 1, 100, 4, 4, 32)
    split = f3d.cross_attn_workspace_bytes(4, 40000, 4, 1, 10000, 4, 4, 32)
    rows_split = f3d.cross_attn_workspace_bytes(200, 40000, 1, 200, 40000, 4, 4, 32)
    whole = f3d.cross_attn_workspace_bytes(200000, 77, 1, 200000, 77, 4, 4, 32)
    assert few == 0 and whole == 0 and split > 0 and rows_split > 0


@pytest.mark.parametrize("D", [32, 128])
def test_cross_attention_padded_batches(D):
    # lengths inside a padded layout; what lies behind them holds NaN and infinities, which reach nothing
    q_lens, kv_lens = [40, 0, 17, 64], [1, 50, 0, 300]
    for H, K in ((4, 4), (4, 1)):
        d = make([64] * 4, [300] * 4, H, K, D, "bf16")
        clean = {k: d[k].clone() for k in ("q", "k", "v", "dout")}
        for b in range(4):
            d["q"][64 * b + q_lens[b]:64 * (b + 1)] = math.nan
            d["dout"][64 * b + q_lens[b]:64 * (b + 1)] = math.inf
            d["k"][300 * b + kv_lens[b]:300 * (b + 1)] = math.nan
            d["v"][300 * b + kv_lens[b]:300 * (b + 1)] = math.inf
        lens = {"q_lens": torch.tensor(q_lens, dtype=torch.int32, device=DEV), "kv_lens": torch.tensor(kv_lens, dtype=torch.int32, device=DEV)}
        out, lse = forward(d, **lens)
        dirty = f3d.cross_attn_bwd(d["q"], d["k"], d["v"], out, d["dout"], lse, d["q_off"], d["kv_off"], H, D, K, 64, 300, **lens)
        d.update(clean)
        want = check_backward(d, q_lens=q_lens, kv_lens=kv_lens)
        for a, b in zip((out, lse, *dirty), want):
            assert torch.equal(a, b)


def test_cross_attention_rows_of_no_segment():
    # rows in front of the first segment and behind the last: results keep what they held, gradients are zero
    # (more rows in front than a block has: slots that no segment owns)
    for shape, first in ((([50, 3], [40, 70]), (5, 9)), (([1, 1], [900, 2000]), (5, 9)), (([4000, 1], [33, 2]), (5, 9)),
                         (([50, 3], [40, 70]), (1000, 1300)), (([1, 1], [900, 2000]), (700, 3000))):
        d = make(*shape, 4, 2, 32, "bf16", first=first, behind=(11, 300))
        d["k"][:first[1]] = math.nan
        d["v"][-300:] = math.nan
        d["q"][:first[0]] = math.nan
        _, _, dq, dk, dv = check_backward(d)
        assert bool((dq[:first[0]] == 0).all()) and bool((dk[:first[1]] == 0).all()) and bool((dv[-300:] == 0).all())


def test_cross_attention_without_offsets_and_without_bounds():
    d = make([100], [60], 4, 2, 64, "bf16")
    want = check_backward(d)
    d["q_off"] = d["kv_off"] = None
    out = f3d.cross_attn(d["q"], d["k"], d["v"], None, None, 4, 64, 2)
    got = f3d.cross_attn_bwd(d["q"], d["k"], d["v"], want[0], d["dout"], want[1], None, None, 4, 64, 2)
    assert torch.equal(out, want[0]) and all(torch.equal(a, b) for a, b in zip(got, want[2:]))
    # bounds left out: another form of the launch, results within the same bounds
    check_backward(make([1, 1, 1], [40, 1000, 3], 4, 2, 64, "bf16"), bounds=False)
    check_backward(make([10, 200, 1], [40, 1000, 3], 4, 2, 128, "bf16"), bounds=False)


def test_cross_attention_many_segments():
    # more segments than a wave has lanes, empty ones among them
    g = torch.Generator().manual_seed(3)
    for n in (63, 64, 65, 200, 5000):
        q_len, kv_len = (torch.randint(0, 4, (n,), generator=g).tolist() for _ in range(2))
        d = make(q_len, kv_len, 2, 1, 16, "bf16")
        out, lse = forward(d)
        dq, dk, dv = f3d.cross_attn_bwd(d["q"], d["k"], d["v"], out, d["dout"], lse, d["q_off"], d["kv_off"], 2, 16, 1, 3, 3)
        if n <= 200:
            check_backward(d)
            continue
        # block-diagonal mask over everything at once
        seg = lambda off, rows: torch.searchsorted(off[1:].long(), torch.arange(rows, device=DEV), right=True)   # noqa: E731
        sees = seg(d["q_off"], len(d["q"]))[:, None] == seg(d["kv_off"], len(d["k"]))[None]
        for h in range(2):
            s = (d["q"][:, 16 * h:16 * h + 16].float() @ d["k"].float().T / 4).masked_fill(~sees, -math.inf)
            p = torch.softmax(s, 1).nan_to_num(0.0)
            assert float((out[:, 16 * h:16 * h + 16].float() - p @ d["v"].float()).abs().max()) <= 0.05


@pytest.mark.parametrize("t", ["bf16", "f16"])
@pytest.mark.parametrize("D", [16, 32, 64, 128])
def test_cross_attention_scales_and_sharp_scores(D, t):
    # scores of a few hundred: one key takes nearly everything, and the reference moves many times
    for q_len, kv_len in (([70], [600]), ([2, 1], [500, 40])):
        for scale in (0.01, 1.0, 8.0):
            d = make(q_len, kv_len, 4, 2, D, t, q_scale=2.0)
            d["k"] = (d["k"].float() * torch.linspace(0.1, 3.0, len(d["k"]), device=DEV)[:, None]).to(d["t"])
            out, lse = forward(d, scale=scale)
            check_forward(d, out, lse, scale)


@pytest.mark.parametrize("D", [16, 32, 64, 128])
def test_cross_attention_gradients_at_the_smallest_scale(D):
    # every probability is 1 / n; rows that only fill a tile up must not count, however small their scaled scores are
    check_backward(make([70, 3], [200, 33], 4, 2, D, "bf16"), scale=2.0 ** -100)
    check_backward(make([70, 3], [90, 33], 4, 2, D, "bf16"), scale=2.0 ** -100)


@pytest.mark.parametrize("D", [16, 64, 128])
@pytest.mark.parametrize("kv", [100, 700])
def test_cross_attention_values_as_large_as_they_may_be(D, kv):
    # scores about 45 above the others: exponentials of 2^65, times values of 2^79
    d = make([200], [kv], 2, 1, D, "bf16", q_scale=0.05)
    d["q"] += 4.0
    d["k"] *= 0.05
    d["k"][kv // 2] = 45.0 / math.sqrt(D) / 4
    for power in (79, -70):
        e = {**d, "v": (d["v"].float() * 2.0 ** power).to(torch.bfloat16)}
        out, lse = forward(e)
        check_forward(e, out, lse)


# a workgroup takes a run of two to eight row blocks here; keys that stay in LDS and keys that stream
@pytest.mark.parametrize("t", ["bf16", "f16"])
@pytest.mark.parametrize("kv", [90, 700])
@pytest.mark.parametrize("D,H,n", [(16, 16, 200000), (32, 8, 200003), (128, 2, 400000)])
def test_cross_attention_runs_of_blocks_some_of_which_are_sharp(D, H, n, kv, t):
    g = torch.Generator(device=DEV).manual_seed(n + D + kv)
    r = lambda rows: torch.randn(rows, H * D, generator=g, device=DEV)   # noqa: E731
    q, k, v = r(n), r(kv).to(TYPES[t]), r(kv).to(TYPES[t])
    sharp = [0, 130, 511, 1023, 1024, 128 * 31 + 5, n // 2, n - 300, n - 1]
    q[sharp] *= 60
    rows = sorted(set(sharp + [x + i for x in sharp for i in (-128, -1, 1, 64, 128) if 0 <= x + i < n] + list(range(7, n, n // 200))))
    q = q.to(TYPES[t])
    lse = torch.empty(n, H, device=DEV)
    out = f3d.cross_attn(q, k, v, None, None, H, D, lse=lse)
    part = {"q": q[rows].contiguous(), "k": k, "v": v, "q_off": ends([len(rows)]), "kv_off": ends([kv]), "q_len": [len(rows)], "kv_len": [kv], "H": H, "K": H,
            "D": D, "t": TYPES[t]}
    check_forward(part, out[rows], lse[rows])
    plain = f3d.cross_attn(q, k, v, None, None, H, D)                   # without lse: another form of the kernel
    assert torch.equal(plain, out)
    if t == "f16":
        return
    dout = (0.1 * r(n)).to(TYPES[t])
    dq, _, _ = f3d.cross_attn_bwd(q, k, v, out, dout, lse, None, None, H, D)
    for h in range(H):
        col = slice(h * D, (h + 1) * D)
        _, kk, s, e = scores(part, slice(0, len(rows)), slice(0, kv), h, h, 1 / math.sqrt(D))
        vv, do, o = v[:, col].double(), dout[rows, col].double(), out[rows, col].double()
        p = torch.exp(s - lse[rows, h].double()[:, None])
        ds = p * (do @ vv.T - (do * o).sum(1, keepdim=True))
        off = (D + 8) * U * (do.abs() @ vv.abs().T + (do * o).abs().sum(1, keepdim=True))
        e2 = 2 * e + 4 * U * (1 + lse[rows, h].double().abs()[:, None])
        b = half(TYPES[t])
        room = (ds.abs() * (b + e2) * (1 + b) + p * off + (kv + 8) * U * ds.abs()) @ kk.abs() / math.sqrt(D)
        want = ds @ kk / math.sqrt(D)
        close(dq[rows, col], want, room * (1 + b) + (b + U) * want.abs() + least(TYPES[t]), f"dq, head {h}")


@pytest.mark.parametrize("D,kv", [(16, n) for n in (1, 31, 32, 33, 64, 65, 95, 96, 97, 128, 129)] + [(32, n) for n in (1, 31, 32, 33, 64, 65, 95, 96, 97)])
def test_cross_attention_gradients_of_few_keys(D, kv):
    # segments of many rows, whose sums are split, beside short ones, and a padded batch in which rows and keys are missing
    d = make([1500, 1, 0, 129], [kv, max(kv - 1, 0), 1, kv], 4, 2, D, "bf16")
    check_backward(d)
    for name, rows in (("q", slice(400, 1500)), ("k", slice(kv // 2, kv))):
        d[name][rows] = math.nan                                        # behind the lengths
    d["v"][kv // 2:kv] = math.nan
    check_backward(d, q_lens=[400, 1, 0, 100], kv_lens=[kv // 2, max(kv - 1, 0), 0, kv])


def test_cross_attention_one_key_returns_its_value():
    # the probability is exactly one
    d = make([10, 200, 1], [1, 1, 1], 4, 2, 64, "bf16", q_scale=3.0)
    out, _ = forward(d)
    for b in range(3):
        rows = slice(int(d["q_off"][b]), int(d["q_off"][b + 1]))
        for h in range(4):
            assert bool((out[rows, 64 * h:64 * h + 64] == d["v"][b, 64 * (h // 2):64 * (h // 2) + 64]).all())


def test_cross_attention_gradients_against_differences():
    # central differences of a scalar function of the output in binary64, of the definition that the forward pass is checked
    # against: step 2^-8 of inputs that are exact in bf16, third derivatives leave 1e-5, the gradients' own rounding 2^-8 of their sums
    d = make([3, 2], [4, 6], 2, 1, 16, "bf16")
    out, lse = forward(d)
    dq, dk, dv = f3d.cross_attn_bwd(d["q"], d["k"], d["v"], out, d["dout"], lse, d["q_off"], d["kv_off"], 2, 16, 1, 3, 6)

    def value(x):
        total = 0.0
        for rows, keys, h, j, _ in pieces(d, None, None):
            s = x["q"][rows, 16 * h:16 * h + 16] @ x["k"][keys, :16].T / 4
            total += float((torch.softmax(s, 1) @ x["v"][keys, :16] * d["dout"][rows, 16 * h:16 * h + 16].double()).sum())
        return total

    x = {k: d[k].double() for k in "qkv"}
    step = 2.0 ** -8
    for name, grad in (("q", dq), ("k", dk), ("v", dv)):
        size = float(grad.abs().max())
        for i, c in ((0, 0), (1, 5), (3, 15), (4, 9)):
            up, down = ({**x, name: x[name].clone()} for _ in range(2))
            up[name][i, c] += step
            down[name][i, c] -= step
            assert abs((value(up) - value(down)) / (2 * step) - float(grad[i, c])) <= 1e-4 + 4 * 2.0 ** -8 * size, name


def test_cross_attention_rows_behind_offsets_that_pass_32_bits():
    # a cache of 5 GB, of which the last segment begins past 2^32 bytes and past 2^31 elements
    H, D, n = 8, 128, 2_500_000
    k = torch.empty(n, H * D, dtype=torch.bfloat16, device=DEV)
    v = torch.empty_like(k)
    g = torch.Generator(device=DEV).manual_seed(5)
    tail = 300
    for x in (k, v):
        x[-tail:] = torch.randn(tail, H * D, generator=g, device=DEV).to(torch.bfloat16)
    q = torch.randn(2, H * D, generator=g, device=DEV).to(torch.bfloat16)
    off = torch.tensor([n - tail, n - tail + 1, n], dtype=torch.int32, device=DEV)
    got = f3d.cross_attn(q, k, v, ends([1, 1]), off, H, D, max_q=1, max_kv=tail)
    want = f3d.cross_attn(q, k[-tail:].clone(), v[-tail:].clone(), ends([1, 1]), ends([1, tail - 1]), H, D, max_q=1, max_kv=tail)
    assert float((got.float() - want.float()).abs().max()) <= 2 * half(torch.bfloat16) * float(want.float().abs().max())
    del k, v


def test_cross_attention_inconsistent_offsets_stay_inside_the_tensors():
    # decreasing, negative and too large: unspecified results, but the rows around the tensors keep what they held
    room = torch.full((3, 4000, 64), 3.0, dtype=torch.bfloat16, device=DEV)
    q, out, dq = (room[i, 1000:1300] for i in range(3))
    q.normal_()
    k, v = torch.randn(500, 64, device=DEV).to(torch.bfloat16), torch.randn(500, 64, device=DEV).to(torch.bfloat16)
    lse = torch.zeros(300, 4, device=DEV)
    for a, b in (([0, 200, 100, 300], [0, 600, 20, 500]), ([-5, 100, 2 ** 31 - 1, 10], [400, 300, 200, 100]), ([7, 7, 7, 7], [0, 0, 0, 9])):
        for lens in (None, torch.tensor([2 ** 31 - 1, -7, 5], dtype=torch.int32, device=DEV)):
            qo, ko = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in (a, b))
            f3d.cross_attn(q, k, v, qo, ko, 4, 16, q_lens=lens, kv_lens=lens, out=out, lse=lse)
            f3d.cross_attn_bwd(q, k, v, out, q, lse, qo, ko, 4, 16, q_lens=lens, kv_lens=lens)
            torch.cuda.synchronize()
            for i in range(3):
                assert bool((room[i, :1000] == 3).all()) and bool((room[i, 1300:] == 3).all())


def test_cross_attention_empty_tensors():
    k = torch.randn(20, 32, device=DEV).to(torch.bfloat16)
    none = torch.empty(0, 32, dtype=torch.bfloat16, device=DEV)
    assert f3d.cross_attn(none, k, k, None, None, 1, 32).shape == (0, 32)
    lse = torch.full((20, 1), 7.0, device=DEV)
    out = f3d.cross_attn(k, none, none, None, None, 1, 32, lse=lse)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())
    dq, dk, dv = f3d.cross_attn_bwd(k, none, none, out, k, lse, None, None, 1, 32)
    assert bool((dq == 0).all()) and dk.shape == (0, 32)
    dq, dk, dv = f3d.cross_attn_bwd(none, k, k, none, none, torch.empty(0, 1, device=DEV), None, None, 1, 32)
    assert dq.shape == (0, 32) and bool((dk == 0).all()) and bool((dv == 0).all())


def test_cross_attention_on_another_stream_and_replayed_from_graphs():
    # two graphs that share one workspace, replayed in turn with eager calls in between; the second splits its keys
    cases = [make([300, 20], [77, 200], 4, 2, 32, "bf16"), make([1, 1, 1], [2000, 900, 3], 4, 2, 64, "bf16")]
    need = max(f3d.cross_attn_workspace_bytes(len(d["q"]), len(d["k"]), len(d["q_len"]), d["max_q"], d["max_kv"], 4, 2, d["D"], backward)
               for d in cases for backward in (False, True))
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)

    def step(d, to):
        args = (d["q_off"], d["kv_off"], 4, d["D"], 2, d["max_q"], d["max_kv"])
        f3d.cross_attn(d["q"], d["k"], d["v"], *args, out=to["out"], lse=to["lse"], workspace=ws)
        to["dq"], to["dk"], to["dv"] = f3d.cross_attn_bwd(d["q"], d["k"], d["v"], to["out"], d["dout"], to["lse"], *args, workspace=ws)

    def room(d):
        return {"out": torch.empty_like(d["q"]), "lse": torch.empty(len(d["q"]), 4, device=DEV)}

    want = []
    for d in cases:
        to = room(d)
        step(d, to)
        want.append({k: v.clone() for k, v in to.items()})
    torch.cuda.synchronize()
    side, to = torch.cuda.Stream(), room(cases[1])
    with torch.cuda.stream(side):
        step(cases[1], to)
    side.synchronize()
    assert all(torch.equal(to[k], v) for k, v in want[1].items())
    graphs, rooms = [], [room(d) for d in cases]
    for d, to in zip(cases, rooms):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(d, to)
        graphs.append(graph)
    for _ in range(3):
        for graph, to, w in zip(graphs, rooms, want):
            for x in to.values():
                x.fill_(1.0)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(to[k], v) for k, v in w.items())
            step(cases[0], room(cases[0]))
            torch.cuda.synchronize()


def test_cross_attention_refusals_by_the_binding():
    q, k = torch.zeros(8, 64, dtype=torch.bfloat16, device=DEV), torch.zeros(5, 32, dtype=torch.bfloat16, device=DEV)
    off = torch.tensor([0, 8], dtype=torch.int32, device=DEV)
    with pytest.raises(TypeError):
        f3d.cross_attn(q.float(), k.float(), k.float(), None, None, 2, 32, 1)
    with pytest.raises(TypeError):
        f3d.cross_attn(q, k.half(), k, None, None, 2, 32, 1)
    with pytest.raises(ValueError):
        f3d.cross_attn(q, k, k[:4], None, None, 2, 32, 1)
    with pytest.raises(ValueError):
        f3d.cross_attn(q, k, k, None, None, 2, 32, 2)
    with pytest.raises(ValueError):
        f3d.cross_attn(q, k, k, off, torch.tensor([0, 2, 5], dtype=torch.int32, device=DEV), 2, 32, 1)
    with pytest.raises(ValueError):
        f3d.cross_attn(q, k, k, None, torch.tensor([0, 2, 5], dtype=torch.int32, device=DEV), 2, 32, 1)
    with pytest.raises(TypeError):
        f3d.cross_attn(q, k, k, off.long(), off, 2, 32, 1)
    with pytest.raises(ValueError):
        f3d.cross_attn(q.t().contiguous().t(), k, k, None, None, 2, 32, 1)
    with pytest.raises(f3d.Flash3DError) as err:
        f3d.cross_attn(torch.zeros(8, 48, dtype=torch.bfloat16, device=DEV), torch.zeros(5, 24, dtype=torch.bfloat16, device=DEV),
                       torch.zeros(5, 24, dtype=torch.bfloat16, device=DEV), None, None, 2, 24, 1)
    assert err.value.code == f3d.ERR_UNSUPPORTED
    long = torch.zeros(9000, 32, dtype=torch.bfloat16, device=DEV)
    with pytest.raises(f3d.Flash3DError) as err:
        f3d.cross_attn(q[:1].contiguous(), long, long, None, None, 2, 32, 1, workspace=torch.empty(256, dtype=torch.uint8, device=DEV))
    assert err.value.code == f3d.ERR_WORKSPACE_TOO_SMALL
    with pytest.raises(TypeError):
        f3d.cross_attn_bwd(q.half(), k.half(), k.half(), q.half(), q.half(), torch.zeros(8, 2, device=DEV), None, None, 2, 32, 1)
