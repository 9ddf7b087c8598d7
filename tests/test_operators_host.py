"""Host-side refusals of the layer norm, clipping and cross attention entry points: no GPU, nothing is launched, no pointer followed."""
import ctypes

import pytest

import paper_2412_16481_amd as f3d

AT = 0x10000                 # a well-aligned address that no call may follow
OK, INVALID, ALIGN, SMALL, UNSUPPORTED = 0, f3d.ERR_INVALID_ARG, f3d.ERR_BAD_ALIGNMENT, f3d.ERR_WORKSPACE_TOO_SMALL, f3d.ERR_UNSUPPORTED


def norm(**kw):
    a = dict(x=AT, row_in=None, gamma=AT, beta=AT, eps=1e-5, n=10, channels=64, dtype=0, y=AT, mean=AT, rstd=AT, stream=None)
    a.update(kw)
    return f3d.lib().f3d_layer_norm(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(n=-1), INVALID), (dict(channels=0), INVALID), (dict(dtype=3), INVALID), (dict(dtype=-1), INVALID), (dict(eps=-1.0), INVALID),
    (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID), (dict(x=None), INVALID), (dict(y=None), INVALID),
    (dict(channels=8193), UNSUPPORTED), (dict(n=1 << 31), UNSUPPORTED), (dict(x=AT + 1), ALIGN), (dict(dtype=2, y=AT + 2), ALIGN),
    (dict(gamma=AT + 2), ALIGN), (dict(row_in=AT + 1), ALIGN), (dict(mean=AT + 2), ALIGN), (dict(n=0, x=None, y=None), OK)])
def test_layer_norm_refuses(kw, code):
    assert norm(**kw) == code


def norm_bwd(**kw):
    a = dict(dy=AT, x=AT, row_in=None, mean=AT, rstd=AT, gamma=AT, residual=None, n=10, channels=64, dtype=0, dx=AT, dgamma=AT, dbeta=AT,
             workspace=AT, workspace_bytes=1 << 30, stream=None)
    a.update(kw)
    return f3d.lib().f3d_layer_norm_bwd(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(n=-1), INVALID), (dict(channels=-3), INVALID), (dict(dtype=7), INVALID), (dict(dy=None), INVALID), (dict(x=None), INVALID),
    (dict(mean=None), INVALID), (dict(rstd=None), INVALID), (dict(dx=None), INVALID), (dict(workspace=None), INVALID),
    (dict(workspace=AT + 64), ALIGN), (dict(workspace_bytes=5 * 2 * 64 * 4 - 1), SMALL), (dict(channels=9000), UNSUPPORTED),
    (dict(residual=AT + 1), ALIGN), (dict(dgamma=AT + 1), ALIGN), (dict(rstd=AT + 3), ALIGN), (dict(n=0, dgamma=None, dbeta=None, dx=None), OK)])
def test_layer_norm_bwd_refuses(kw, code):
    assert norm_bwd(**kw) == code


def test_layer_norm_refuses_results_over_what_is_still_read():
    far = AT + (1 << 20)
    assert norm(row_in=far) == INVALID                                  # y is x, and rows are gathered
    for moved in (AT + 128, AT - 128, AT + 10 * 128 - 16):
        assert norm(y=moved) == INVALID
    assert norm_bwd(dy=AT, x=far, row_in=far) == INVALID
    for name in ("dy", "x", "residual"):
        assert norm_bwd(**{"dy": far, "x": far, "residual": far, name: AT + 128}) == INVALID


def clip(tensors, outs=None, max_norm=1.0, norm=AT, workspace=AT, workspace_bytes=1 << 30):
    """tensors: (address, elements, type); outs: addresses or None for in place."""
    n = len(tensors)
    grads = (ctypes.c_void_p * n)(*[t[0] for t in tensors])
    sizes = (ctypes.c_int64 * n)(*[t[1] for t in tensors])
    types = (ctypes.c_int32 * n)(*[t[2] for t in tensors])
    to = None if outs is None else (ctypes.c_void_p * n)(*outs)
    return f3d.lib().f3d_clip_grads(grads, to, sizes, types, n, max_norm, norm, workspace, workspace_bytes, None)


def test_clip_grads_refuses():
    one = [(AT, 100, 2)]
    assert clip(one, norm=None) == INVALID
    assert clip(one, workspace=None) == INVALID
    assert clip(one, max_norm=-1.0) == INVALID
    assert clip(one, max_norm=float("nan")) == INVALID
    assert clip(one, norm=AT + 2) == ALIGN
    assert clip(one, workspace=AT + 16) == ALIGN
    assert clip(one, workspace_bytes=1000) == SMALL
    assert clip([(AT, -1, 2)]) == INVALID
    assert clip([(AT, 1, 3)]) == INVALID
    assert clip([(None, 1, 2)]) == INVALID
    assert clip([(AT + 2, 1, 2)]) == ALIGN
    assert clip([(AT + 1, 1, 0)]) == ALIGN
    assert clip([(AT, 1 << 45, 0)]) == UNSUPPORTED
    assert f3d.lib().f3d_clip_grads(None, None, None, None, 1, 1.0, AT, AT, 1 << 30, None) == INVALID
    assert f3d.lib().f3d_clip_grads(None, None, None, None, -1, 1.0, AT, AT, 1 << 30, None) == INVALID
    size = ctypes.c_size_t(0)
    assert f3d.lib().f3d_clip_grads_workspace_bytes(65537, ctypes.byref(size)) == UNSUPPORTED
    assert f3d.lib().f3d_clip_grads_workspace_bytes(1, None) == INVALID


def test_clip_grads_refuses_outputs_that_share_memory():
    a, b = AT, AT + 4096
    assert clip([(a, 100, 2), (a, 100, 2)]) == INVALID                         # the same tensor twice, in place
    assert clip([(a, 100, 2), (a + 396, 100, 2)]) == INVALID                   # one element shared
    assert clip([(a, 100, 2), (b, 100, 2)], [b + 4096, b + 4096]) == INVALID   # two outputs
    assert clip([(a, 100, 2), (b, 100, 2)], [b, a]) == INVALID                 # another's gradient
    assert clip([(a, 100, 2)], [a + 4]) == INVALID                             # its own gradient, moved
    assert clip([(a, 2000, 2), (a + 400, 10, 2)], [b + 8192, a + 4000]) == INVALID   # inside a long one that began earlier


def cross(entry="f3d_cross_attn", **kw):
    a = dict(q=AT, k=AT, v=AT, q_offsets=AT, kv_offsets=AT, q_lens=None, kv_lens=None, n_q=100, n_kv=50, n_segments=3, max_q=60, max_kv=40,
             heads=8, kv_heads=2, head_dim=32, scale=0.0, out=AT, lse=AT, workspace=AT, workspace_bytes=1 << 40, stream=None)
    a.update(kw)
    return getattr(f3d.lib(), entry)(*a.values())


def cross_bwd(**kw):
    a = dict(q=AT, k=AT, v=AT, out=AT, dout=AT, lse=AT, q_offsets=AT, kv_offsets=AT, q_lens=None, kv_lens=None, n_q=100, n_kv=50, n_segments=3,
             max_q=60, max_kv=40, heads=8, kv_heads=2, head_dim=32, scale=0.0, dq=AT, dk=AT, dv=AT, workspace=AT, workspace_bytes=1 << 40,
             stream=None)
    a.update(kw)
    return f3d.lib().f3d_cross_attn_bwd(*a.values())


SHARED = [
    (dict(n_q=-1), INVALID), (dict(n_kv=-1), INVALID), (dict(n_segments=0), INVALID), (dict(max_q=-1), INVALID), (dict(max_kv=-2), INVALID),
    (dict(heads=0), INVALID), (dict(kv_heads=0), INVALID), (dict(heads=8, kv_heads=3), INVALID), (dict(head_dim=24), UNSUPPORTED),
    (dict(head_dim=256), UNSUPPORTED), (dict(n_segments=65536), UNSUPPORTED), (dict(n_q=1 << 29), UNSUPPORTED), (dict(n_kv=1 << 31), UNSUPPORTED),
    (dict(heads=4096, kv_heads=4096), UNSUPPORTED), (dict(scale=-1.0), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(scale=float("inf")), INVALID), (dict(q=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID),
    (dict(q_offsets=None), INVALID), (dict(kv_offsets=None), INVALID), (dict(q=AT + 8), ALIGN), (dict(v=AT + 2), ALIGN),
    (dict(kv_lens=AT + 1), ALIGN), (dict(q_offsets=AT + 2), ALIGN), (dict(out=None), INVALID), (dict(out=AT + 8), ALIGN), (dict(lse=AT + 2), ALIGN)]
LONG = dict(n_q=3, n_kv=30000, max_q=1, max_kv=10000)       # the keys are split: a workspace is needed


@pytest.mark.parametrize("kw,code", SHARED + [
    ({**LONG, "workspace": None}, INVALID), ({**LONG, "workspace": AT + 16}, ALIGN), ({**LONG, "workspace_bytes": 100}, SMALL),
    (dict(n_q=0, q=None, out=None), OK)])
def test_cross_attn_refuses(kw, code):
    assert cross(**kw) == code
    assert cross("f3d_cross_attn_f16", **kw) == code


@pytest.mark.parametrize("kw,code", SHARED + [
    (dict(workspace=None), INVALID), (dict(workspace=AT + 128), ALIGN), (dict(workspace_bytes=100 * 8 * 4 - 1), SMALL), (dict(dout=None), INVALID),
    (dict(lse=None), INVALID), (dict(dq=None), INVALID), (dict(dk=None), INVALID), (dict(dv=None), INVALID), (dict(dk=AT + 4), ALIGN),
    (dict(scale=2.0 ** -101), UNSUPPORTED),
    (dict(n_q=0, n_kv=0, q=None, k=None, v=None, out=None, workspace=None), OK)])
def test_cross_attn_bwd_refuses(kw, code):
    assert cross_bwd(**kw) == code


def test_cross_attn_refuses_results_over_what_is_still_read():
    far = lambda i: AT + (i << 24)   # noqa: E731
    assert [cross(q=far(1), k=far(2), v=far(3), out=far(x) + d) for x, d in ((1, 0), (2, 16), (3, 50 * 64 * 2 - 16), (1, -16))] == [INVALID] * 4
    names = ("q", "k", "v", "out", "dout", "dq", "dk", "dv")
    apart = {x: far(i + 1) for i, x in enumerate(names)}
    for result in ("dq", "dk", "dv"):
        for other in names:
            if other != result:
                assert cross_bwd(**{**apart, result: apart[other] + 16}) == INVALID, (result, other)


def test_cross_attn_workspace_refuses():
    size = ctypes.c_size_t(0)
    for name in ("f3d_cross_attn_workspace_bytes", "f3d_cross_attn_bwd_workspace_bytes"):
        call = getattr(f3d.lib(), name)
        assert call(10, 10, 1, 0, 0, 4, 2, 32, None) == INVALID
        assert call(10, 10, 1, 0, 0, 4, 3, 32, ctypes.byref(size)) == INVALID
        assert call(10, 10, 1, 0, 0, 4, 2, 40, ctypes.byref(size)) == UNSUPPORTED
        assert call(10, 10, 1, 0, 0, 4, 2, 32, ctypes.byref(size)) == OK
