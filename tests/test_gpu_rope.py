"""Rotary positions on the GPU against their definition in 64 bits, and a whole layer with the attention behind them."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

import window_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def _nr():
    from paper_2608_00029_b200 import nova_rope
    return nova_rope


def _randn(g, *shape):
    return torch.randn(shape, generator=g).to(torch.bfloat16).to(DEV)


def _check(got, x, positions, inv_freq, interleaved, amplitude, backward):
    """One rounding, and errors of 32-bit sines, products and sums: 2^-20 of both ends of a pair."""
    want = ref.rope(x, positions, inv_freq, interleaved, amplitude, backward)
    R = 2 * inv_freq.numel()
    ends = torch.zeros_like(want)
    a = x.double().abs()
    if interleaved:
        ends[..., 0:R:2] = ends[..., 1:R:2] = a[..., 0:R:2] + a[..., 1:R:2]
    else:
        ends[..., :R // 2] = ends[..., R // 2:R] = a[..., :R // 2] + a[..., R // 2:R]
    bound = ref.HALF * want.abs() + 2.0**-20 * abs(amplitude) * ends
    err = (got.double() - want).abs()
    assert (err <= bound).all(), float((err - bound).max())
    assert torch.equal(got[..., R:], x[..., R:]), "what is not turned is copied"


SHAPES = [
    # B, H, KV, T, D, rotary
    (1, 1, 1, 1, 8, 2), (2, 3, 1, 5, 64, 64), (1, 12, 12, 130, 64, 64), (2, 4, 2, 77, 128, 128), (2, 4, 1, 33, 128, 32),
    (1, 5, 5, 19, 64, 16), (3, 2, 2, 9, 64, 24), (1, 2, 1, 40, 128, 6), (1, 2, 1, 40, 128, 126), (2, 2, 2, 7, 80, 20),
    (1, 3, 1, 11, 256, 254), (32, 16, 4, 1, 128, 128), (4, 8, 8, 1000, 64, 32), (1, 2, 2, 3, 1024, 1024),
]


@pytest.mark.parametrize("fused", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("B,H,KV,T,D,rotary", SHAPES)
def test_rope(B, H, KV, T, D, rotary, interleaved, fused):
    nr = _nr()
    g = torch.Generator().manual_seed(T + rotary)
    inv_freq = nr.nova_rope_frequencies(rotary)[0].to(DEV)
    if fused:
        x, y = _randn(g, B, T, H + KV + 1, D), torch.full((B, T, H + KV + 1, D), 7.0, dtype=torch.bfloat16, device=DEV)
        cut = lambda z: (z.transpose(1, 2)[:, :H], z.transpose(1, 2)[:, H:H + KV], z.transpose(1, 2)[:, H + KV:])
        (q, k, _), (qo, ko, spare) = cut(x), cut(y)
    else:
        q, k = _randn(g, B, H, T, D), _randn(g, B, KV, T, D)
        qo, ko = torch.empty_like(q), torch.empty_like(k)
        spare = torch.full((1,), 7.0)
    start = torch.arange(T, dtype=torch.int32, device=DEV)
    each = (torch.randint(-1000, 10**6, (B, 1), generator=g).to(torch.int32).to(DEV) + start).contiguous()
    for backward, positions, amplitude in ((False, None, 1.0), (True, start, 1.0), (False, each, 1.25), (True, each, 0.5)):
        call = nr.nova_rope_bwd if backward else nr.nova_rope_fwd
        call(q, k, qo, ko, inv_freq, positions, interleaved=interleaved, amplitude=amplitude)
        pos = (start if positions is None else positions).expand(B, T)
        _check(qo, q, pos, inv_freq, interleaved, amplitude, backward)
        _check(ko, k, pos, inv_freq, interleaved, amplitude, backward)
    assert (spare == 7.0).all(), "written outside the outputs"
    # where it lies, and Q alone
    q2, k2 = q.clone(memory_format=torch.preserve_format), k.clone(memory_format=torch.preserve_format)
    nr.nova_rope_bwd(q2, k2, q2, k2, inv_freq, each, interleaved=interleaved, amplitude=0.5)
    assert torch.equal(q2, qo) and torch.equal(k2, ko)
    q3 = torch.empty_like(q)
    nr.nova_rope_bwd(q, None, q3, None, inv_freq, each, interleaved=interleaved, amplitude=0.5)
    assert torch.equal(q3, qo)


def test_far_positions():
    """Positions at the end of 31 bits, in both directions: angles of 2 10^9 are as exact as those of 2."""
    nr = _nr()
    g = torch.Generator().manual_seed(1)
    q = _randn(g, 1, 2, 64, 128)
    out = torch.empty_like(q)
    inv_freq = nr.nova_rope_frequencies(128)[0].to(DEV)
    for first in (2**31 - 64, -2**31, 16777216):
        pos = (torch.arange(64) + first).to(torch.int32).to(DEV)
        nr.nova_rope_fwd(q, None, out, None, inv_freq, pos)
        _check(out, q, pos.expand(1, 64), inv_freq, False, 1.0, False)


def test_positions_with_strides_and_graph():
    nr = _nr()
    g = torch.Generator().manual_seed(2)
    B, T = 3, 10
    q = _randn(g, B, 4, T, 64)
    out = torch.empty_like(q)
    table = torch.randint(0, 5000, (B, T + 7), generator=g).to(torch.int32).to(DEV)
    pos = table[:, :T]
    inv_freq = nr.nova_rope_frequencies(64)[0].to(DEV)
    nr.nova_rope_fwd(q, None, out, None, inv_freq, pos)
    _check(out, q, pos, inv_freq, False, 1.0, False)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out2 = torch.empty_like(q)
    nr.nova_rope_fwd(q, None, out2, None, inv_freq, pos, stream=s)
    s.synchronize()
    assert torch.equal(out, out2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        nr.nova_rope_fwd(q, None, out2, None, inv_freq, pos)
    table.add_(17)
    graph.replay()
    torch.cuda.synchronize()
    _check(out2, q, pos, inv_freq, False, 1.0, False)


def test_nan_stays_in_its_pair():
    nr = _nr()
    q = torch.ones((1, 1, 4, 64), dtype=torch.bfloat16, device=DEV)
    q[0, 0, 2, 5] = math.nan
    out = torch.empty_like(q)
    nr.nova_rope_fwd(q, None, out, None, nr.nova_rope_frequencies(32)[0].to(DEV))
    bad = torch.isnan(out).nonzero().tolist()
    assert bad == [[0, 0, 2, 5], [0, 0, 2, 21]]


def test_a_layer_forward_backward_and_its_next_token():
    """Projection output -> rotary positions where it lies -> window attention -> its gradients -> turned back, against the
    definition's gradients by automatic differentiation in 64 bits; then the next token over the same keys and values."""
    from paper_2608_00029_b200 import nova_attn as na, nova_window as nw
    nr = _nr()
    B, H, KV, T, D, window, sinks = 2, 6, 2, 300, 64, 64, 4
    g = torch.Generator().manual_seed(3)
    qkv, do = _randn(g, B, T, H + 2 * KV, D), _randn(g, B, T, H, D).transpose(1, 2)
    inv_freq, amplitude = nr.nova_rope_frequencies(D, kind="yarn", factor=4.0, original=128)
    inv_freq = inv_freq.to(DEV)
    scale = 1.0 / math.sqrt(D)
    cut = lambda z: (z.transpose(1, 2)[:, :H], z.transpose(1, 2)[:, H:H + KV], z.transpose(1, 2)[:, H + KV:])
    turned = qkv.clone()
    q, k, v = cut(turned)
    nr.nova_rope_fwd(q, k, q, k, inv_freq, amplitude=amplitude)
    o, rest = (torch.empty((B, T, H, D), dtype=torch.bfloat16, device=DEV).transpose(1, 2) for _ in range(2))
    lse, delta = (torch.empty((B, H, T), device=DEV) for _ in range(2))
    grad = torch.empty_like(qkv)
    dq, dk, dv = cut(grad)
    nw.nova_window_fwd(q, k, v, o, lse, scale, window, sinks, O_rest=rest)
    nw.nova_window_bwd_preprocess(o, rest, do, delta)
    nw.nova_window_bwd(q, k, v, do, lse, delta, dq, dk, dv, scale, window, sinks)
    nr.nova_rope_bwd(dq, dk, dq, dk, inv_freq, amplitude=amplitude)
    na.nova_attn_poll_device_status()
    # in 64 bits from the same projection output
    x = qkv.double().requires_grad_(True)
    xq, xk, xv = cut(x)
    pos = torch.arange(T, device=DEV).expand(B, T)
    a = pos.double()[:, None, :, None] * inv_freq.double()
    def turn(z):
        z0, z1 = z[..., :D // 2], z[..., D // 2:]
        return torch.cat((z0 * a.cos() - z1 * a.sin(), z1 * a.cos() + z0 * a.sin()), -1) * amplitude
    want, _, _ = ref.forward(turn(xq), turn(xk), xv, scale, window, sinks)
    (want * do.double()).sum().backward()
    # one rounding more than in the attention's own tests, that of Q and K: scores off by 2^-8 of their products
    assert ref.rel_rms(o, want.detach()) < 8e-3
    assert ref.rel_rms(grad, x.grad) < 1.2e-2
    # the token after the last: its key and value are put behind the others, it looks at them through the window
    new = _randn(g, B, 1, H + 2 * KV, D)
    nq, nk, nv = cut(new)
    at = torch.full((B, 1), T, dtype=torch.int32, device=DEV)
    nr.nova_rope_fwd(nq, nk, nq, nk, inv_freq, at, amplitude=amplitude)
    ck, cv = (torch.full((B, KV, 512, D), math.nan, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    ck[:, :, :T], cv[:, :, :T] = k, v
    ck[:, :, T:T + 1], cv[:, :, T:T + 1] = nk, nv
    no, nl = torch.empty((B, H, 1, D), dtype=torch.bfloat16, device=DEV), torch.empty((B, H, 1), device=DEV)
    nw.nova_window_decode(nq, ck, cv, at.squeeze(1) + 1, no, nl, scale, window, sinks)
    w, wl, mass = ref.decode(nq.double(), ck.double(), cv.double(), [T + 1] * B, scale, window, sinks)
    assert ((no.double() - w).abs() <= ref.HALF * w.abs() + 2.0**-14 * mass).all()
    # a training step's eager graph of the same leaves lives on while the backward is captured
    graph = torch.cuda.CUDAGraph()
    before = grad.clone()
    with torch.cuda.graph(graph):
        nw.nova_window_bwd(q, k, v, do, lse, delta, dq, dk, dv, scale, window, sinks)
        nr.nova_rope_bwd(dq, dk, dq, dk, inv_freq, amplitude=amplitude)
    grad.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(grad, before)
