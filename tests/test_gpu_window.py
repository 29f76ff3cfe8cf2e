"""The attention with a sliding window and sinks on the GPU against its definition in 64 bits: forward, backward, single tokens."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

import window_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def _libs():
    from paper_2608_00029_b200 import nova_attn, nova_window
    return nova_attn, nova_window


def _randn(g, *shape):
    return torch.randn(shape, generator=g).to(torch.bfloat16).to(DEV)


class Problem:
    """Inputs, and outputs among sentinels: views of larger buffers, in which nothing else may be written."""

    def __init__(self, B, H, KV, T, D, fused, seed=0, qk=1.0, pad=3):
        g = torch.Generator().manual_seed(seed)
        self.buffers = []
        self.scale = 1.0 / math.sqrt(D)

        def views(heads, make):
            """One view [B,h,T,D] per entry of `heads`."""
            if fused:  # [B, T + pad, sum of heads + 1, D], the last head and the last tokens unused
                buf = make(B, T + pad, sum(heads) + 1, D).transpose(1, 2)[:, :, :T]
                at = [sum(heads[:i]) for i in range(len(heads))]
                return [buf[:, a:a + h] for a, h in zip(at, heads)]
            return [make(B, h, T + pad, D)[:, :, :T] if pad else make(B, h, T, D) for h in heads]

        def random(*shape):
            return _randn(g, *shape)

        def sentinel(*shape):
            x = torch.full(shape, 7.0, dtype=torch.bfloat16, device=DEV)
            self.buffers.append(x)
            return x

        self.q, self.k, self.v = views((H, KV, KV), random)
        if qk != 1.0:
            self.q, self.k = self.q * qk, self.k * qk
        self.do, = views((H,), random)
        self.o, = views((H,), sentinel)
        self.rest, = views((H,), sentinel)
        self.dq, self.dk, self.dv = views((H, KV, KV), sentinel)
        self.lse = torch.full((B, H, T), 7.0, dtype=torch.float32, device=DEV)
        self.delta = torch.full((B, H, T), 7.0, dtype=torch.float32, device=DEV)

    def run(self, window, sinks, rest=True, workspace=None, stream=None):
        _, nw = _libs()
        r = self.rest if rest else None
        nw.nova_window_fwd(self.q, self.k, self.v, self.o, self.lse, self.scale, window, sinks, O_rest=r, stream=stream)
        nw.nova_window_bwd_preprocess(self.o, r, self.do, self.delta, stream=stream)
        nw.nova_window_bwd(self.q, self.k, self.v, self.do, self.lse, self.delta, self.dq, self.dk, self.dv, self.scale, window,
                           sinks, workspace=workspace, stream=stream)

    def outputs(self):
        return self.o, self.lse, self.dq, self.dk, self.dv

    def check(self, window, sinks, rms=True):
        na, _ = _libs()
        na.nova_attn_poll_device_status()
        q, k, v, do = (x.double() for x in (self.q, self.k, self.v, self.do))
        o, lse, p = ref.forward(q, k, v, self.scale, window, sinks)
        grads, bounds, delta = ref.backward(q, k, v, do, self.scale, window, sinks)

        def close(name, got, want, bound):
            err = (got.double() - want).abs()
            assert torch.isfinite(got.float()).all(), f"{name}: not finite"
            assert (err <= bound).all(), f"{name}: off by up to {float((err / bound).max()):.2f} of the bound"

        close("O", self.o, o, ref.forward_bound(p, v, o))
        close("LSE", self.lse, lse, 3e-4 + 1e-6 * lse.abs())
        for name, got, want, bound in zip(("dQ", "dK", "dV"), (self.dq, self.dk, self.dv), grads, bounds):
            close(name, got, want, bound)
        if rms:  # roundings add up in squares: two of 2^-8 / sqrt(3) at most, Delta's share besides
            for name, got, want, most in (("O", self.o, o, 4e-3), ("dQ", self.dq, grads[0], 6e-3), ("dK", self.dk, grads[1], 6e-3),
                                          ("dV", self.dv, grads[2], 5e-3)):
                r = ref.rel_rms(got, want)
                assert r <= most, f"{name}: relative RMS error {r:.2e}"
        for x in (self.o, self.rest, self.dq, self.dk, self.dv):  # what is left of the buffers is the sentinel
            x.fill_(7.0)
        assert all(bool((b == 7.0).all()) for b in self.buffers), "written outside an output"


SHAPES = [
    # B, H, KV, T, D, window, sinks
    (1, 1, 1, 1, 64, 1, 0),
    (2, 2, 1, 1, 128, 5, 3),
    (1, 2, 2, 2, 64, 2, 0),
    (1, 2, 2, 17, 64, 1, 0),          # every query keeps itself alone
    (1, 2, 1, 70, 128, 1, 1),
    (2, 4, 2, 64, 64, 16, 1),
    (1, 3, 1, 65, 128, 64, 0),
    (1, 2, 2, 127, 64, 128, 0),
    (1, 2, 1, 128, 128, 3, 130),      # more sinks than tokens
    (1, 4, 2, 129, 64, 63, 1),
    (1, 2, 2, 200, 64, 65, 4),
    (2, 6, 2, 333, 128, 100, 64),
    (1, 2, 1, 384, 64, 128, 128),     # a window and sinks of whole tiles
    (1, 2, 1, 385, 128, 129, 129),
    (1, 8, 1, 500, 128, 200, 5),      # one key/value head for all
    (1, 1, 1, 777, 64, 128, 4),
    (1, 3, 3, 1025, 128, 256, 150),
    (1, 2, 2, 1537, 64, 1000, 0),
    (1, 2, 2, 300, 64, 100000, 0),    # the whole triangle
    (1, 4, 4, 700, 128, 2**31 - 1, 2**31 - 1),
    (40, 4, 4, 130, 64, 33, 2),       # more items than SMs
    (20, 6, 3, 260, 128, 40, 1),
    (3, 12, 4, 640, 64, 64, 4),
    (1, 64, 2, 300, 64, 90, 7),
    (1, 8, 1, 3000, 64, 100, 4),      # the sinks' tile, and the others, in parts
    (1, 6, 2, 2600, 128, 300, 200),   # two tiles with sinks
    (2, 12, 1, 1100, 128, 1100, 0),   # long lists on few heads
    (1, 16, 1, 200, 64, 200, 0),
    (6, 12, 4, 700, 128, 200, 70),    # pairs of query tiles in dQ
    (12, 16, 16, 300, 128, 30, 1),    # the last pair has one tile
    (5, 16, 2, 900, 128, 64, 130),
    (4, 12, 4, 1500, 128, 300, 0),
]


@pytest.mark.parametrize("fused", [False, True])
@pytest.mark.parametrize("B,H,KV,T,D,window,sinks", SHAPES)
def test_forward_and_backward(B, H, KV, T, D, window, sinks, fused):
    p = Problem(B, H, KV, T, D, fused, seed=T + D + window % 1000)
    p.run(window, sinks)
    p.check(window, sinks, rms=T >= 64 and window >= 16)
    if T == 1:
        p.run(window, sinks)
        assert torch.equal(p.o, p.v.repeat_interleave(H // KV, 1)), "a single token attends to itself only"


def test_contiguous_tensors():
    p = Problem(2, 6, 2, 515, 64, False, seed=3, pad=0)
    assert p.q.is_contiguous() and p.dk.is_contiguous()
    p.run(130, 4)
    p.check(130, 4)
    p = Problem(1, 4, 4, 515, 128, False, seed=4, pad=0)
    p.run(130, 4)
    p.check(130, 4)


def test_random_shapes():
    g = torch.Generator().manual_seed(11)
    pick = lambda *xs: xs[int(torch.randint(len(xs), (1,), generator=g))]
    for n in range(24):
        T = int(torch.randint(1, 900, (1,), generator=g))
        KV, G, D = pick(1, 2, 3, 8), pick(1, 2, 4), pick(64, 128)
        window, sinks = int(torch.randint(1, T + 1, (1,), generator=g)), pick(0, 0, 1, 4, 64, 65, 200)
        p = Problem(pick(1, 2, 3), KV * G, KV, T, D, pick(False, True), seed=n)
        p.run(window, sinks)
        p.check(window, sinks, rms=False)


def test_peaked_rows():
    """Scores of tens: the running maximum moves, most weights vanish."""
    for D in (64, 128):
        p = Problem(1, 4, 2, 600, D, False, seed=5, qk=3.0)
        p.run(200, 3)
        p.check(200, 3)


def test_sinks_of_great_weight():
    """A first key that outweighs the window by more than the rescaling threshold, and one that vanishes beside it."""
    for D in (64, 128):
        for factor in (6.0, -6.0):
            p = Problem(1, 2, 2, 450, D, False, seed=6)
            p.q[..., 0] = 3.0
            p.k[:, :, :, 0] = 0.0
            p.k[:, :, 0, 0] = factor
            p.run(100, 1)
            p.check(100, 1)


def test_whole_triangle_is_the_causal_attention():
    na, nw = _libs()
    p = Problem(1, 3, 3, 1000, 64, False, seed=7, pad=0)
    p.run(1000, 0)
    o, lse = torch.empty_like(p.o), torch.empty_like(p.lse)
    na.nova_attn_fwd(p.q, p.k, p.v, o, lse, p.scale, True)
    assert (lse - p.lse).abs().max() < 1e-4
    assert ref.rel_rms(p.o, o.double()) < 4e-3


def test_rest_and_delta():
    """O + O_rest is the sum before it was rounded, and Delta takes it in; without it Delta is rowsum(dO * O)."""
    na, nw = _libs()
    for fused in (False, True):
        p = Problem(2, 4, 2, 300, 64, fused, seed=8)
        p.run(50, 2)
        o, rest, delta = p.o.double(), p.rest.double(), p.delta.clone()
        assert (rest.abs() <= ref.HALF * o.abs() + 1e-30).all() and rest.abs().max() > 0
        q, k, v, do = (x.double() for x in (p.q, p.k, p.v, p.do))
        want, _, w = ref.forward(q, k, v, p.scale, 50, 2)
        bound = ref.SLACK * ref.HALF * (w @ v.repeat_interleave(2, 1).abs()) + ref.HALF**2 * want.abs() + 1e-6
        assert ((o + rest - want).abs() <= bound).all()
        exact = (do * (o + rest)).sum(-1)
        assert ((delta.double() - exact).abs() <= 2.0**-18 * (do * (o + rest)).abs().sum(-1) + 1e-30).all()
        nw.nova_window_bwd_preprocess(p.o, None, p.do, p.delta)
        plain = (do * o).sum(-1)
        assert ((p.delta.double() - plain).abs() <= 2.0**-18 * (do * o).abs().sum(-1) + 1e-30).all()


def test_same_bits_every_time():
    for D in (64, 128):
        p = Problem(2, 8, 2, 700, D, True, seed=9)
        p.run(130, 4)
        first = [x.clone() for x in p.outputs()]
        ws = torch.full((_libs()[1].nova_window_bwd_workspace_bytes(2, 8, 2, 700, D, 130, 4),), 255, dtype=torch.uint8, device=DEV)
        for _ in range(3):
            p.run(130, 4, workspace=ws)
            assert all(torch.equal(a, b) for a, b in zip(first, p.outputs()))


@pytest.mark.parametrize("B,H,KV,T,D", [(1, 4, 2, 900, 64), (1, 4, 2, 900, 128), (4, 12, 4, 1100, 64), (4, 12, 4, 1100, 128)])
def test_passes_one_behind_the_other(B, H, KV, T, D):
    """Kernels begin before the one ahead of them has ended: nothing may be read that is still to be written, or written that is still to
    be read.  Passes through the same buffers, by turns with other row terms and other parts."""
    na, nw = _libs()
    p = Problem(B, H, KV, T, D, False, seed=T + D)
    masks = [(130, 4), (40, 0), (700, 130)]
    ws = torch.empty(max(nw.nova_window_bwd_workspace_bytes(B, H, KV, T, D, w, s) for w, s in masks), dtype=torch.uint8, device=DEV)
    alone = []
    for w, s in masks:
        p.run(w, s, workspace=ws)
        torch.cuda.synchronize()
        alone.append([x.clone() for x in p.outputs()])
    got = []
    for i in range(12):
        p.run(*masks[i % 3], workspace=ws)
        if i >= 9:
            got.append([x.clone() for x in p.outputs()])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for i in range(9):
            p.run(*masks[i % 3], workspace=ws)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    na.nova_attn_poll_device_status()
    for want, x in zip(alone, got):
        assert all(torch.equal(a, b) for a, b in zip(want, x))
    assert all(torch.equal(a, b) for a, b in zip(alone[2], p.outputs()))


def test_streams_and_graphs():
    """Two problems on two streams at once, each captured into a graph and replayed on new inputs."""
    na, _ = _libs()
    ps = [Problem(2, 4, 2, 500, D, False, seed=10 + D) for D in (64, 128)]
    for p in ps:
        p.run(100, 4)  # the one call before capturing
    streams = [torch.cuda.Stream() for _ in ps]
    torch.cuda.synchronize()
    for p, s in zip(ps, streams):
        p.run(100, 4, stream=s)
    torch.cuda.synchronize()
    eager = [[x.clone() for x in p.outputs()] for p in ps]
    graphs = []
    for p in ps:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            p.run(100, 4)
    for p in ps:
        for x in p.outputs():
            x.fill_(5.0)
    for g, s in zip(graphs, streams):
        with torch.cuda.stream(s):
            g.replay()
    torch.cuda.synchronize()
    for p, want in zip(ps, eager):
        assert all(torch.equal(a, b) for a, b in zip(want, p.outputs()))
    for p in ps:
        for x in (p.q, p.k, p.v, p.do):
            x.copy_(x.flip(2).clone())
    for g, s in zip(graphs, streams):
        g.replay()
    torch.cuda.synchronize()
    for p in ps:
        p.check(100, 4)


def test_strides_of_dimensions_of_size_one():
    """A view may have any stride where there is one element: it is not used."""
    na, nw = _libs()
    g = torch.Generator().manual_seed(12)
    T, D = 150, 64
    q, k, v, do = (_randn(g, T, D).as_strided((1, 1, T, D), (3, 1, D, 1)) for _ in range(4))
    o, rest, dq, dk, dv = (torch.empty((T, D), dtype=torch.bfloat16, device=DEV).as_strided((1, 1, T, D), (0, 5, D, 1)) for _ in range(5))
    lse, delta = torch.empty((1, 1, T), device=DEV), torch.empty((1, 1, T), device=DEV)
    nw.nova_window_fwd(q, k, v, o, lse, 0.125, 40, 3, O_rest=rest)
    nw.nova_window_bwd_preprocess(o, rest, do, delta)
    nw.nova_window_bwd(q, k, v, do, lse, delta, dq, dk, dv, 0.125, 40, 3)
    na.nova_attn_poll_device_status()
    ref_o, _, p = ref.forward(q.double(), k.double(), v.double(), 0.125, 40, 3)
    assert ((o.double() - ref_o).abs() <= ref.forward_bound(p, v.double(), ref_o)).all()
    grads, bounds, _ = ref.backward(q.double(), k.double(), v.double(), do.double(), 0.125, 40, 3)
    for got, want, bound in zip((dq, dk, dv), grads, bounds):
        assert ((got.double() - want).abs() <= bound).all()
    one = q[:, :, -1:].as_strided((1, 1, 1, D), (1, 1, 1, 1), q.storage_offset() + (T - 1) * D)
    o1, lse1 = torch.empty((1, 1, 1, D), dtype=torch.bfloat16, device=DEV), torch.empty((1, 1, 1), device=DEV)
    nw.nova_window_decode(one, k, v, torch.tensor([T], dtype=torch.int32, device=DEV), o1, lse1, 0.125, 40, 3)
    assert ((o1.double() - ref_o[:, :, -1:]).abs() <= ref.HALF * ref_o[:, :, -1:].abs() + 2.0**-14 * (p @ v.double().abs())[:, :, -1:]).all()


def test_refusals():
    na, nw = _libs()
    p = Problem(1, 4, 2, 64, 64, False, seed=1, pad=0)
    run = lambda **kw: nw.nova_window_fwd(*[kw.get(n, getattr(p, n)) for n in ("q", "k", "v", "o", "lse")], 0.125, kw.get("window", 8),
                                          kw.get("sinks", 0), O_rest=kw.get("rest"))
    for kw, error in (({"window": 2.5}, TypeError), ({"window": 2**31}, ValueError), ({"k": p.k[:, :, :32]}, ValueError),
                      ({"v": p.q}, ValueError), ({"q": p.q.float()}, TypeError), ({"lse": p.lse[:, :2]}, TypeError),
                      ({"q": p.q.transpose(2, 3)}, TypeError), ({"rest": p.rest.transpose(1, 2).contiguous().transpose(1, 2)}, ValueError),
                      ({"o": p.o.cpu()}, TypeError)):
        with pytest.raises(error):
            run(**kw)
    for kw, status in (({"window": 0}, na.ERR_SHAPE), ({"sinks": -1}, na.ERR_SHAPE), ({"k": p.k[:, :1].expand(1, 3, 64, 64), "v": p.v[:, :1].expand(1, 3, 64, 64)}, na.ERR_SHAPE),
                       ({"k": p.k[:, :1].expand(1, 2, 64, 64)}, na.ERR_SHAPE)):
        with pytest.raises(na.NovaAttnError) as e:
            run(**kw)
        assert e.value.status == status
    small = torch.empty(8, dtype=torch.uint8, device=DEV)
    with pytest.raises(na.NovaAttnError) as e:
        nw.nova_window_bwd(p.q, p.k, p.v, p.do, p.lse, p.delta, p.dq, p.dk, p.dv, 0.125, 8, 0, workspace=small)
    assert e.value.status == na.ERR_WORKSPACE
    with pytest.raises(ValueError):  # one token per sequence
        nw.nova_window_decode(p.q, p.k, p.v, torch.zeros(1, dtype=torch.int32, device=DEV), p.o, p.lse, 0.125, 8)
    torch.cuda.synchronize()
    assert (p.o == 7.0).all() and (p.dq == 7.0).all(), "a refused call must not launch anything"


# ---------------------------------------------------------------- single tokens

DECODE = [
    # B, H, KV, T_max, D, window, sinks, lengths
    (1, 1, 1, 1, 64, 1, 0, [1]),
    (3, 2, 1, 20, 64, 7, 2, [0, 5, 20]),
    (2, 12, 12, 300, 64, 256, 4, [300, 17]),
    (4, 8, 1, 130, 128, 16, 0, [130, 1, 16, 64]),       # one tile
    (3, 32, 4, 1000, 128, 500, 4, [1000, 504, 505]),
    (2, 32, 2, 700, 64, 700, 0, [700, 333]),             # sixteen query heads to a key/value head
    (2, 40, 2, 300, 128, 100, 9, [299, 41]),             # twenty: two groups
    (2, 9, 1, 200, 128, 64, 200, [200, 150]),            # sinks reach into the window
    (1, 3, 1, 5000, 128, 4000, 100, [5000]),
    (2, 2, 2, 3000, 64, 10**6, 0, [3000, 2999]),
    (3, 4, 2, 50, 64, 10, 3, [-5, 51, 10**9]),           # outside: the nearer end
    (8, 12, 12, 1000, 64, 1000, 0, [1000, 999, 1, 0, 170, 500, 192, 193]),  # a cluster for each of many rows
    (16, 16, 8, 500, 128, 450, 20, list(range(10, 490, 30))),
    (3, 24, 2, 1700, 64, 1700, 0, [1700, 256, 900]),     # eight runs
    (100, 4, 4, 1500, 64, 1400, 30, list(range(1, 1500, 15))),  # more rows than the GPU holds at once
]


@pytest.mark.parametrize("by_token", [False, True])
@pytest.mark.parametrize("B,H,KV,T,D,window,sinks,lengths", DECODE)
def test_single_tokens(B, H, KV, T, D, window, sinks, lengths, by_token):
    na, nw = _libs()
    g = torch.Generator().manual_seed(T + H)
    q = _randn(g, B, H, 1, D)
    k, v = ((_randn(g, B, T, KV, D).transpose(1, 2) if by_token else _randn(g, B, KV, T, D)) for _ in range(2))
    # what is not kept is not read: neither what lies behind a sequence nor what its window has left behind
    for b, n in enumerate(lengths):
        n = min(max(n, 0), T)
        gone = torch.ones(T, dtype=torch.bool, device=DEV)
        gone[[j for j in range(n) if n - 1 - j < window or j < sinks]] = False
        k[b, :, gone], v[b, :, gone] = math.nan, math.inf
    buf = torch.full((B, H + 2, 1, D), 7.0, dtype=torch.bfloat16, device=DEV)
    o, lse = buf[:, 1:-1], torch.full((B, H, 1), 7.0, device=DEV)
    scale = 1.0 / math.sqrt(D)
    length = torch.tensor([max(-2**31, min(n, 2**31 - 1)) for n in lengths], dtype=torch.int32, device=DEV)
    nw.nova_window_decode(q, k, v, length, o, lse, scale, window, sinks)
    na.nova_attn_poll_device_status()
    want, want_lse, mass = ref.decode(q.double(), k.double(), v.double(), lengths, scale, window, sinks)
    # weights keep 16 bits, scores are off by less than 3e-5
    bound = ref.HALF * want.abs() + 2.0**-14 * mass + 1e-30
    assert ((o.double() - want).abs() <= bound).all(), float(((o.double() - want).abs() / bound).max())
    empty = torch.isinf(want_lse)
    assert torch.equal(torch.isinf(lse), empty) and (lse[empty] < 0).all() and (o[empty.squeeze(-1)] == 0).all()
    assert ((lse.double() - want_lse)[~empty].abs() <= 3e-5 + 1e-6 * want_lse[~empty].abs()).all()
    assert (buf[:, 0] == 7.0).all() and (buf[:, -1] == 7.0).all()
    o2, lse2 = torch.empty_like(o), torch.empty_like(lse)
    ws = torch.full((nw.nova_window_decode_workspace_bytes(B, H, KV, T, D, window, sinks),), 255, dtype=torch.uint8, device=DEV)
    nw.nova_window_decode(q, k, v, length, o2, lse2, scale, window, sinks, workspace=ws if ws.numel() else None)
    assert torch.equal(o, o2) and torch.equal(lse, lse2), "the same bits in every run"


def test_infinities_reach_what_keeps_them_only():
    na, nw = _libs()
    g = torch.Generator().manual_seed(2)
    B, H, KV, T, D = 2, 4, 2, 400, 64
    q, k, v = _randn(g, B, H, 1, D), _randn(g, B, KV, T, D), _randn(g, B, KV, T, D)
    v[1, 0, 390] = math.inf
    length = torch.tensor([400, 400], dtype=torch.int32, device=DEV)
    o, lse = torch.empty((B, H, 1, D), dtype=torch.bfloat16, device=DEV), torch.empty((B, H, 1), device=DEV)
    nw.nova_window_decode(q, k, v, length, o, lse, 0.125, 64, 4)
    assert torch.isfinite(o[0]).all() and torch.isfinite(o[1, 2:]).all() and not torch.isfinite(o[1, :2]).any()
    assert torch.isfinite(lse).all()


def test_rolling_cache_and_last_row():
    """The last row of the forward, the same from a whole cache, and from one that holds sinks + window tokens in any order."""
    na, nw = _libs()
    for D in (64, 128):
        H, KV, T, window, sinks = 6, 2, 555, 96, 4
        p = Problem(1, H, KV, T, D, False, seed=D, pad=0)
        p.run(window, sinks)
        q = p.q[:, :, -1:]
        o, lse = torch.empty((1, H, 1, D), dtype=torch.bfloat16, device=DEV), torch.empty((1, H, 1), device=DEV)
        nw.nova_window_decode(q, p.k, p.v, torch.tensor([T], dtype=torch.int32, device=DEV), o, lse, p.scale, window, sinks)
        want, want_lse, mass = ref.decode(q.double(), p.k.double(), p.v.double(), [T], p.scale, window, sinks)
        assert ((o.double() - p.o[:, :, -1:].double()).abs() <= 2 * ref.HALF * want.abs() + 2 * ref.HALF * mass).all()
        assert (lse - p.lse[:, :, -1:]).abs().max() < 3e-4
        slots = list(range(sinks)) + [T - window + (i - (T - sinks)) % window for i in range(window)]
        rk, rv = p.k[:, :, slots].contiguous(), p.v[:, :, slots].contiguous()
        o2, lse2 = torch.empty_like(o), torch.empty_like(lse)
        nw.nova_window_decode(q, rk, rv, torch.tensor([sinks + window], dtype=torch.int32, device=DEV), o2, lse2, p.scale, window, sinks)
        assert ((o2.double() - want).abs() <= ref.HALF * want.abs() + 2.0**-14 * mass).all()
        assert (lse2.double() - want_lse).abs().max() < 3e-5


def test_offsets_past_32_bits():
    """A cache of more than 2^32 elements, of which one sequence's window lies at the far end."""
    na, nw = _libs()
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 20 GB")
    B, KV, D = 1, 1, 64
    token = 1 << 17  # elements from token to token
    T = (1 << 32) // token + 600
    buf = torch.zeros(T * token, dtype=torch.bfloat16, device=DEV)
    g = torch.Generator().manual_seed(1)
    k = buf.as_strided((B, KV, T, D), (T * token, D, token, 1))
    v = buf.as_strided((B, KV, T, D), (T * token, D, token, 1), 64)
    k[:, :, -100:], v[:, :, -100:] = _randn(g, B, KV, 100, D), _randn(g, B, KV, 100, D)
    q = _randn(g, B, 2, 1, D)
    o, lse = torch.empty_like(q), torch.empty((B, 2, 1), device=DEV)
    nw.nova_window_decode(q, k, v, torch.tensor([T], dtype=torch.int32, device=DEV), o, lse, 0.125, 100, 0)
    want, want_lse, mass = ref.decode(q.double(), k[:, :, -100:].double(), v[:, :, -100:].double(), [100], 0.125, 100, 0)
    assert ((o.double() - want).abs() <= ref.HALF * want.abs() + 2.0**-14 * mass).all()


def test_decode_in_a_graph_and_on_a_stream():
    na, nw = _libs()
    g = torch.Generator().manual_seed(4)
    B, H, KV, T, D = 3, 8, 2, 900, 128
    q, k, v = _randn(g, B, H, 1, D), _randn(g, B, KV, T, D), _randn(g, B, KV, T, D)
    length = torch.tensor([5, 900, 321], dtype=torch.int32, device=DEV)
    o, lse = torch.empty_like(q), torch.empty((B, H, 1), device=DEV)
    nw.nova_window_decode(q, k, v, length, o, lse, 0.1, 300, 4)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    o2, lse2 = torch.empty_like(o), torch.empty_like(lse)
    nw.nova_window_decode(q, k, v, length, o2, lse2, 0.1, 300, 4, stream=s)
    s.synchronize()
    assert torch.equal(o, o2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        nw.nova_window_decode(q, k, v, length, o2, lse2, 0.1, 300, 4)
    length.copy_(torch.tensor([900, 0, 77], dtype=torch.int32))  # the next tokens, other lengths
    graph.replay()
    torch.cuda.synchronize()
    want, want_lse, mass = ref.decode(q.double(), k.double(), v.double(), [900, 0, 77], 0.1, 300, 4)
    assert ((o2.double() - want).abs() <= ref.HALF * want.abs() + 2.0**-14 * mass + 1e-30).all()
