"""The forms of the windowed forward on the GPU against 64 bits: without O_rest (evaluation, prompts), and with weights of two bf16
numbers, which it takes where O_rest is asked for and a row keeps few keys."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

import window_reference as ref  # noqa: E402
from test_gpu_window import SHAPES, Problem  # noqa: E402

pytestmark = pytest.mark.gpu


def _libs():
    from paper_2608_00029_b200 import nova_attn, nova_window
    return nova_attn, nova_window


@pytest.mark.parametrize("fused", [False, True])
@pytest.mark.parametrize("B,H,KV,T,D,window,sinks", SHAPES)
def test_without_rest(B, H, KV, T, D, window, sinks, fused):
    """O and LSE, and the gradients from a Delta that carries the rounding of O: by dP - Delta it reaches dS with the weight P."""
    na, _ = _libs()
    p = Problem(B, H, KV, T, D, fused, seed=T + D + sinks % 1000)
    p.run(window, sinks, rest=False)
    na.nova_attn_poll_device_status()
    q, k, v, do = (x.double() for x in (p.q, p.k, p.v, p.do))
    o, lse, w = ref.forward(q, k, v, p.scale, window, sinks)
    assert torch.isfinite(p.o.float()).all()
    assert ((p.o.double() - o).abs() <= ref.forward_bound(w, v, o)).all()
    assert ((p.lse.double() - lse).abs() <= 3e-4 + 1e-6 * lse.abs()).all()
    grads, bounds, _ = ref.backward(q, k, v, do, p.scale, window, sinks)
    more = w * (ref.SLACK * ref.HALF * (do * o).abs()).sum(-1, keepdim=True)
    G = H // KV
    more_dq = more @ k.repeat_interleave(G, 1).abs() * p.scale
    more_dk = (more.mT @ q.abs()).unflatten(1, (KV, G)).sum(2) * p.scale
    for name, got, want, bound in zip(("dQ", "dK", "dV"), (p.dq, p.dk, p.dv), grads, (bounds[0] + more_dq, bounds[1] + more_dk, bounds[2])):
        assert torch.isfinite(got.float()).all(), name
        assert ((got.double() - want).abs() <= bound).all(), f"{name}: {float(((got.double() - want).abs() / bound).max()):.2f} of the bound"
    if T >= 64 and window >= 16:
        assert ref.rel_rms(p.o, o) <= 4e-3 and ref.rel_rms(p.dv, grads[2]) <= 5e-3
    assert (p.rest == 7.0).all()
    for x in (p.o, p.dq, p.dk, p.dv):
        x.fill_(7.0)
    assert all(bool((b == 7.0).all()) for b in p.buffers), "written outside an output"


@pytest.mark.parametrize("fused", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("window,sinks", [(16, 1), (60, 4), (64, 0)])
def test_weights_of_two_numbers(window, sinks, D, fused):
    """O + O_rest where a row keeps at most 64 keys.  What is off, relative to P |V|: the weights' second rounding, 2^-8 of what the
    first one left, which is 2^-8; twice a score's error (in its weight and in the sum of weights), which is D / 16 sums of 2^-22 of
    sum |q k|; the sums of at most 32 products with V, 2^-22 each; 2^-20 for exponentials and sums of weights.  And O_rest is
    rounded in its turn, 2^-16 of O.  Weights of one number are off by 2^-8 each, which has to be told from this."""
    na, nw = _libs()
    p = Problem(2, 6, 2, 333, D, fused, seed=window + D)
    nw.nova_window_fwd(p.q, p.k, p.v, p.o, p.lse, p.scale, window, sinks, O_rest=p.rest)
    na.nova_attn_poll_device_status()
    q, k, v = (x.double() for x in (p.q, p.k, p.v))
    want, _, w = ref.forward(q, k, v, p.scale, window, sinks)
    kx, vx = (x.repeat_interleave(3, 1) for x in (k, v))
    hidden = ~ref.kept(333, window, sinks, q.device)
    most = (q.abs() @ kx.abs().mT).masked_fill(hidden, 0.0).amax(-1, keepdim=True)
    off = 2.0**-16 + 2 * (D / 16) * 2.0**-22 * most * p.scale + 32 * 2.0**-22 + 2.0**-20
    bound = off * (w @ vx.abs()) + ref.HALF**2 * want.abs() + 1e-30
    err = (p.o.double() + p.rest.double() - want).abs()
    assert (err <= bound).all(), f"{float((err / bound).max()):.2f} of the bound"
    s = (q @ kx.mT * p.scale).masked_fill(hidden, -math.inf)
    e = (s - s.amax(-1, keepdim=True)).exp()
    one = (e.to(torch.bfloat16).double() @ vx) / e.sum(-1, keepdim=True)
    assert ((one - want).abs() > bound).double().mean() > 0.5, "the bound would not tell weights of one number"


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("window,sinks", [(32, 150), (64, 1), (40, 2**31 - 1), (1, 64)])
def test_rows_that_keep_many_keys_have_weights_of_one_number(window, sinks, D):
    """Sinks count as the window does: with more than 64 keys to a row O has the same bits whether O_rest is asked for or not."""
    _, nw = _libs()
    p = Problem(2, 4, 2, 300, D, False, seed=D + window)
    nw.nova_window_fwd(p.q, p.k, p.v, p.o, p.lse, p.scale, window, sinks)
    o, lse = p.o.clone(), p.lse.clone()
    nw.nova_window_fwd(p.q, p.k, p.v, p.o, p.lse, p.scale, window, sinks, O_rest=p.rest)
    assert torch.equal(p.o, o) and torch.equal(p.lse, lse)


def test_rest_in_another_layout_of_the_same_places():
    """One head: [B,1,T,D] and a view of [B,T,1,D] have the same elements at the same places, whatever the stride of the one head."""
    _, nw = _libs()
    for D in (64, 128):
        p = Problem(2, 1, 1, 200, D, False, seed=D, pad=0)
        rest = torch.empty((2, 200, 1, D), dtype=torch.bfloat16, device=p.o.device).transpose(1, 2)
        assert rest.stride() != p.o.stride()
        nw.nova_window_fwd(p.q, p.k, p.v, p.o, p.lse, p.scale, 50, 2, O_rest=rest)
        nw.nova_window_bwd_preprocess(p.o, rest, p.do, p.delta)
        delta = p.delta.clone()
        nw.nova_window_fwd(p.q, p.k, p.v, p.o, p.lse, p.scale, 50, 2, O_rest=p.rest)
        nw.nova_window_bwd_preprocess(p.o, p.rest, p.do, p.delta)
        assert torch.equal(rest, p.rest) and torch.equal(delta, p.delta)
        one = torch.empty((1, 4, 1, D), dtype=torch.bfloat16, device=p.o.device)  # one token: neither its stride nor the sequence's
        wide = torch.empty((3, 4, 9, D), dtype=torch.bfloat16, device=p.o.device)[:1, :, :1]
        with pytest.raises(ValueError):  # other heads' places
            nw.nova_window_fwd(one, one, one, one.clone(), torch.empty((1, 4, 1), device=p.o.device), 0.1, 4, O_rest=wide)


def test_rotation_in_place_through_another_view():
    """In place is the same elements at the same places: the stride of a single head or sequence does not count."""
    from paper_2608_00029_b200 import nova_rope as nr
    g = torch.Generator().manual_seed(3)
    x = torch.randn((1, 1, 50, 64), generator=g).to(torch.bfloat16).to("cuda:0")
    freq, _ = nr.nova_rope_frequencies(64)
    freq = freq.to("cuda:0")
    want = torch.empty_like(x)
    nr.nova_rope_fwd(x, None, want, None, freq)
    other = x.as_strided((1, 1, 50, 64), (64, 64, 64, 1))
    nr.nova_rope_fwd(x, None, other, None, freq)
    assert torch.equal(x, want)
    with pytest.raises(_libs()[0].NovaAttnError):  # other places
        nr.nova_rope_fwd(x[:, :, :25], None, x.as_strided((1, 1, 25, 64), (3200, 3200, 128, 1)), None, freq)
