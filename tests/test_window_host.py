"""Host side of the rotary positions and of the attention with a sliding window: exported symbols, argument checks before anything
is launched, which tiles a tile of queries or keys visits, frequencies, and the reference itself.  No GPU."""
import ctypes
import math
import os
import re
import subprocess
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

import window_reference as ref  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_00029_b200", "csrc")


@pytest.fixture(scope="module")
def lib():
    from paper_2608_00029_b200 import build, nova_attn
    build.build()
    return nova_attn.load()


def _ptrs(na):
    return ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1008), na.Strides


def test_headers_are_exported(lib):
    for header, prefix, want in (("nova_rope.h", "nova_rope", {"nova_rope_fwd", "nova_rope_bwd", "nova_rope_frequencies"}),
                                 ("nova_window.h", "nova_window", {"nova_window_fwd", "nova_window_bwd_preprocess", "nova_window_bwd",
                                                                   "nova_window_bwd_workspace_bytes", "nova_window_decode",
                                                                   "nova_window_decode_workspace_bytes"})):
        text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", header)).read(), flags=re.S)
        names = set(re.findall(r"\b(%s_[a-z_0-9]+)\s*\(" % prefix, text))
        assert names == want
        for n in names:
            assert hasattr(lib, n)


def _c(lib, name, types):
    f = getattr(lib, name)
    f.restype = ctypes.c_int
    return lambda *a: f(*[t(x) if t in (ctypes.c_float, ctypes.c_int, ctypes.c_longlong, ctypes.c_size_t) else x for t, x in zip(types, a)])


def test_window_calls_refuse_bad_arguments(lib):
    from paper_2608_00029_b200 import nova_attn as na
    p, odd, S = _ptrs(na)
    vp, i, sp, f, sz = ctypes.c_void_p, ctypes.c_int, ctypes.POINTER(na.Strides), ctypes.c_float, ctypes.c_size_t
    fwd = lib.nova_window_fwd
    fwd.argtypes, fwd.restype = [vp] * 6 + [i] * 7 + [sp] * 4 + [f, vp], i
    s = S(4 * 16 * 64, 16 * 64, 64)

    def call(ptrs=(p, p, p, p, None, p), dims=(1, 4, 2, 16, 64), window=4, sinks=0, strides=(s, s, s, s), scale=1.0):
        return fwd(*ptrs, *dims, window, sinks, *strides, scale, None)

    assert call(ptrs=(p, None, p, p, None, p)) == na.ERR_NULL
    assert call(ptrs=(p, p, p, p, None, None)) == na.ERR_NULL
    assert call(dims=(0, 4, 2, 16, 64)) == na.ERR_SHAPE
    assert call(dims=(1, 4, 3, 16, 64)) == na.ERR_SHAPE       # 3 does not divide 4
    assert call(dims=(1, 4, 0, 16, 64)) == na.ERR_SHAPE
    assert call(dims=(1, 4, 8, 16, 64)) == na.ERR_SHAPE
    assert call(dims=(1, 4, 2, 0, 64)) == na.ERR_SHAPE
    assert call(dims=(1, 4, 2, 16, 96)) == na.ERR_UNSUPPORTED
    assert call(window=0) == na.ERR_SHAPE and call(window=-3) == na.ERR_SHAPE and call(sinks=-1) == na.ERR_SHAPE
    assert call(ptrs=(p, odd, p, p, None, p)) == na.ERR_ALIGNMENT
    assert call(ptrs=(p, p, p, p, odd, p)) == na.ERR_ALIGNMENT
    assert call(scale=0.0) == na.ERR_SCALE and call(scale=math.nan) == na.ERR_SCALE
    assert call(strides=(s, None, s, s)) == na.ERR_NULL
    assert call(strides=(s, s, S(4096, 1020, 64), s)) == na.ERR_ALIGNMENT
    assert call(strides=(s, s, s, S(4096, 1024, 32))) == na.ERR_SHAPE

    pre = lib.nova_window_bwd_preprocess
    pre.argtypes, pre.restype = [vp] * 4 + [i] * 4 + [sp, sp, vp], i
    assert pre(p, None, None, p, 1, 4, 16, 64, s, s, None) == na.ERR_NULL
    assert pre(p, odd, p, p, 1, 4, 16, 64, s, s, None) == na.ERR_ALIGNMENT
    assert pre(p, None, p, p, 1, 4, 16, 32, s, s, None) == na.ERR_UNSUPPORTED

    bwd = lib.nova_window_bwd
    bwd.argtypes, bwd.restype = [vp] * 9 + [i] * 7 + [sp] * 7 + [f, vp, sz, vp], i

    def back(ptrs=(p,) * 9, dims=(1, 4, 2, 16, 64), window=4, sinks=0, strides=(s,) * 7, scale=1.0, ws=p, n=1 << 30):
        return bwd(*ptrs, *dims, window, sinks, *strides, scale, ws, n, None)

    assert back(ptrs=(p,) * 8 + (None,)) == na.ERR_NULL
    assert back(dims=(1, 4, 3, 16, 64)) == na.ERR_SHAPE
    assert back(window=0) == na.ERR_SHAPE
    assert back(ws=None) == na.ERR_WORKSPACE and back(n=16) == na.ERR_WORKSPACE
    assert back(ws=odd) == na.ERR_ALIGNMENT
    assert back(scale=-1.0) == na.ERR_SCALE
    assert back(strides=(s,) * 6 + (S(4096, 1024, 56),)) == na.ERR_SHAPE

    dec = lib.nova_window_decode
    dec.argtypes, dec.restype = [vp] * 6 + [i] * 7 + [sp] * 4 + [f, vp, sz, vp], i

    def one(ptrs=(p,) * 6, dims=(1, 4, 2, 4000, 64), window=4000, sinks=0, strides=(s,) * 4, scale=1.0, ws=p, n=1 << 30):
        return dec(*ptrs, *dims, window, sinks, *strides, scale, ws, n, None)

    assert one(ptrs=(p, p, p, None, p, p)) == na.ERR_NULL
    assert one(dims=(1, 4, 3, 4000, 64)) == na.ERR_SHAPE
    assert one(window=0) == na.ERR_SHAPE and one(sinks=-1) == na.ERR_SHAPE
    assert one(dims=(1, 4, 2, 4000, 80)) == na.ERR_UNSUPPORTED
    assert one(ws=None, n=0) == na.ERR_WORKSPACE and one(n=64) == na.ERR_WORKSPACE
    assert one(ptrs=(p, p, p, ctypes.c_void_p(0x1002), p, p)) == na.ERR_ALIGNMENT
    assert one(scale=math.inf) == na.ERR_SCALE


def test_workspace_queries(lib):
    from paper_2608_00029_b200 import nova_window as nw
    for D in (64, 128):  # nothing in parts, and the tile of the sinks in parts
        assert nw.nova_window_bwd_workspace_bytes(2, 4, 2, 100, D, 10, 1) == 256
        assert nw.nova_window_bwd_workspace_bytes(1, 4, 1, 8000, D, 64, 4) % (2 * 128 * D * 4) == 0
        assert nw.nova_window_bwd_workspace_bytes(1, 4, 1, 8000, D, 64, 4) > 2 * 128 * D * 4
    for bad in ((0, 4, 2, 100, 64, 10, 1), (2, 4, 3, 100, 64, 10, 1), (2, 4, 2, 100, 96, 10, 1), (2, 4, 2, 100, 64, 0, 1),
                (2, 4, 2, 100, 64, 10, -1)):
        assert nw.nova_window_bwd_workspace_bytes(*bad) == 0 and nw.nova_window_decode_workspace_bytes(*bad) == 0
    assert nw.nova_window_decode_workspace_bytes(1, 2, 1, 16, 64, 16, 0) == 0  # one run of keys: nothing to join
    assert nw.nova_window_decode_workspace_bytes(1, 2, 1, 10**6, 64, 10**6, 0) > 0
    with pytest.raises(ValueError):
        nw.nova_window_bwd_workspace_bytes(1, 2, 1, 64, 64, 2**31, 0)
    with pytest.raises(TypeError):
        nw.nova_window_decode_workspace_bytes(1, 2, 1, 64, 64, 8.5, 0)


def test_rope_calls_refuse_bad_arguments(lib):
    from paper_2608_00029_b200 import nova_attn as na
    p, odd, S = _ptrs(na)
    vp, i, sp, f = ctypes.c_void_p, ctypes.c_int, ctypes.POINTER(na.Strides), ctypes.c_float
    s = S(4 * 16 * 64, 16 * 64, 64)
    for name in ("nova_rope_fwd", "nova_rope_bwd"):
        fn = getattr(lib, name)
        fn.argtypes, fn.restype = [vp] * 6 + [i] * 7 + [f, ctypes.c_longlong] + [sp] * 4 + [vp], i

        def call(ptrs=(p,) * 6, dims=(1, 4, 2, 16, 64), rotary=64, amplitude=1.0, stride=16, strides=(s,) * 4):
            return fn(*ptrs, *dims, rotary, 0, amplitude, stride, *strides, None)

        q = ctypes.c_void_p(0x9000)
        assert call(ptrs=(None, p, p, p, p, p)) == na.ERR_NULL
        assert call(ptrs=(p, p, p, None, p, p)) == na.ERR_NULL      # K without its output
        assert call(ptrs=(p, p, p, p, None, p)) == na.ERR_NULL
        assert call(dims=(1, 4, 2, 0, 64)) == na.ERR_SHAPE
        assert call(dims=(1, 4, 0, 16, 64)) == na.ERR_SHAPE
        assert call(dims=(1, 4, 2, 16, 60)) == na.ERR_SHAPE
        assert call(dims=(1, 4, 2, 16, 1032)) == na.ERR_SHAPE
        for r in (0, 7, 66, -2):
            assert call(rotary=r) == na.ERR_SHAPE
        assert call(stride=-1) == na.ERR_SHAPE
        assert call(ptrs=(p, p, odd, p, p, p)) == na.ERR_ALIGNMENT
        assert call(ptrs=(p, p, p, p, p, ctypes.c_void_p(0x1002))) == na.ERR_ALIGNMENT
        assert call(amplitude=math.nan) == na.ERR_SCALE
        assert call(ptrs=(p, q, p, q, p, p), strides=(s, s, S(8192, 1024, 64), s)) == na.ERR_SHAPE  # in place, other strides
        assert call(ptrs=(p, q, q, q, p, p), strides=(s, S(4096, 1024, 36), s, s)) == na.ERR_ALIGNMENT


@pytest.mark.parametrize("bad", ["device", "dtype", "not a tensor"])
def test_binding_rejects_wrong_tensors(lib, bad):
    from paper_2608_00029_b200 import nova_rope as nr, nova_window as nw
    x = {"device": torch.zeros(1, 1, 4, 64, dtype=torch.bfloat16), "dtype": torch.zeros(1, 1, 4, 64), "not a tensor": None}[bad]
    for call in (lambda: nr.nova_rope_fwd(x, x, x, x, x), lambda: nr.nova_rope_bwd(x, None, x, None, x),
                 lambda: nw.nova_window_fwd(x, x, x, x, x, 0.1, 4), lambda: nw.nova_window_bwd_preprocess(x, None, x, x),
                 lambda: nw.nova_window_bwd(x, x, x, x, x, x, x, x, x, 0.1, 4), lambda: nw.nova_window_decode(x, x, x, x, x, x, 0.1, 4)):
        with pytest.raises(TypeError):
            call()


# ---------------------------------------------------------------- which tiles are visited

SPANS = r"""
#include "%s/kernels.h"
extern "C" {
void span(int window, int sinks, int q0, int rows, int T, int unit, int* out) {
    const nova::Window w{window, sinks, 1};
    const nova::KeySpan s = nova::key_span(w, q0, rows, T, unit);
    out[0] = s.n;
    for (int j = 0; j < s.n && j < 63; ++j) out[1 + j] = s.at(j);
}
int steps(int window, int sinks, int k0, int keys, int T, int unit) {
    return nova::query_steps(nova::Window{window, sinks, 1}, k0, keys, T, unit);
}
// kt, bh, part, parts, slot, first step, steps
void item(int n_tiles, int sink_tiles, int sink_parts, int parts, int BH, int idx, int all, int* out) {
    const nova::KvItem it = nova::kv_item(nova::KvParts{n_tiles, sink_tiles, sink_parts, parts}, BH, idx);
    out[0] = it.kt, out[1] = it.bh, out[2] = it.part, out[3] = it.parts, out[4] = it.slot;
    nova::kv_part(all, it.part, it.parts, out + 5, out + 6);
}
long long slots(int n_tiles, int sink_tiles, int sink_parts, int parts, int BH) {
    return nova::KvParts{n_tiles, sink_tiles, sink_parts, parts}.slots(BH);
}
long long items(int n_tiles, int sink_tiles, int sink_parts, int parts, int BH) {
    return nova::KvParts{n_tiles, sink_tiles, sink_parts, parts}.items(BH);
}
}
"""


@pytest.fixture(scope="module")
def spans(tmp_path_factory):
    d = tmp_path_factory.mktemp("spans")
    (d / "s.cpp").write_text(SPANS % CSRC)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I/usr/local/cuda/include", "-o", str(d / "s.so"), str(d / "s.cpp")])
    return ctypes.CDLL(str(d / "s.so"))


def test_tiles_visited_are_those_with_something_kept(spans):
    """Against the mask itself, at a sixteenth of the kernels' tile sizes: every tile with a kept pair is visited once, in order, and
    no tile is visited that has none."""
    out = (ctypes.c_int * 64)()
    rows, unit = 8, 4
    for T in (1, 3, 4, 7, 8, 9, 16, 21, 40, 47):
        for window in (1, 2, 3, 4, 5, 8, 9, 13, 40, 47):
            for sinks in (0, 1, 3, 4, 5, 8, 9, 20, 47):
                window_, sinks_ = min(window, T), min(sinks, T)
                m = ref.kept(T, window_, sinks_)
                for q0 in range(0, T, rows):
                    spans.span(window_, sinks_, q0, rows, T, unit, out)
                    want = [k // unit for k in range(0, T, unit) if m[q0:q0 + rows, k:k + unit].any()]
                    assert list(out[1:1 + out[0]]) == want, (T, window, sinks, q0)
                for k0 in range(0, T, rows):  # key tiles: queries from the tile's own on, without a gap
                    n = spans.steps(window_, sinks_, k0, rows, T, unit)
                    kept = [q // unit for q in range(0, T, unit) if m[q:q + unit, k0:k0 + rows].any()]
                    assert k0 // unit == kept[0] and k0 // unit + n - 1 == kept[-1], (T, window, sinks, k0)


def test_every_part_of_every_tile_is_dealt_out_once(spans):
    out = (ctypes.c_int * 7)()
    spans.slots.restype = spans.items.restype = ctypes.c_longlong
    for n_tiles, sink_tiles, sink_parts, parts, BH in ((1, 0, 1, 1, 1), (7, 1, 5, 1, 6), (9, 2, 3, 4, 2), (5, 0, 1, 8, 3), (6, 6, 4, 1, 2), (8, 3, 1, 2, 5)):
        seen, slots = {}, []
        for idx in range(spans.items(n_tiles, sink_tiles, sink_parts, parts, BH)):
            spans.item(n_tiles, sink_tiles, sink_parts, parts, BH, idx, 37, out)
            kt, bh, part, of, slot, first, n = out
            assert 0 <= kt < n_tiles and 0 <= bh < BH and of == (sink_parts if kt < sink_tiles else parts)
            assert n >= 37 // of and (slot >= 0) == (of > 1)
            seen.setdefault((kt, bh), []).append((first, n))
            slots += [slot] if slot >= 0 else []
            if slot >= 0:  # where window_sum_kernel looks for it: a tile's parts BH apart
                before = kt * of * BH if kt < sink_tiles else (sink_tiles * sink_parts * BH if sink_parts > 1 else 0) + (kt - sink_tiles) * of * BH
                assert slot == before + bh + part * BH
        assert len(seen) == n_tiles * BH
        for parts_of in seen.values():
            at = 0
            for first, n in sorted(parts_of):
                assert first == at
                at += n
            assert at == 37
        assert sorted(slots) == list(range(spans.slots(n_tiles, sink_tiles, sink_parts, parts, BH)))


def test_kernels_of_the_subfolder_wait_for_their_predecessor():
    """As in the files above it: a kernel that lets its successor start early waits for its own predecessor, all threads of it, before it
    touches global memory."""
    kernels = 0
    for name in sorted(os.listdir(os.path.join(CSRC, "ops"))):
        if not name.endswith(".cu"):
            continue
        text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "ops", name)).read())
        for m in re.finditer(r"^(?:template[^\n]*\n)?__global__[^{;]*\{\n(.*?)^\}", text, re.M | re.S):
            body = m.group(1)
            kernels += 1
            if "window_dq_kernel" in m.group(0):  # begins before dK/dV has ended, and ends after it
                before, after = body.split("    dq_roles<")
                assert "    if (threadIdx.x == 0 || warp >= 4) griddep_taken_over();" in before and "\n    griddep_wait();" in after
                assert before.index("griddep_taken_over();") < before.index("dq_set_up<") < before.index("griddep_launch_dependents();")
                continue
            if "window_dkdv_kernel" in m.group(0):  # lets it, having waited itself (and waits before it gives up)
                assert re.search(r"\n    griddep_wait\(\);\s+griddep_launch_dependents\(\);\s+kv_roles<", body)
                assert re.search(r"griddep_wait\(\);\s+if \(threadIdx.x == 0\) atomicExch\([^;]*;\s+return;", body) and body.count("return") == 1
                continue
            assert body.count("griddep_launch_dependents();") == 1 and body.count("\n    griddep_wait();") == 1, name
            ahead = body.split("\n    griddep_wait();")[0]
            ahead = re.sub(r"auto \w+ = \[&\].*?\n    \};", "", ahead, flags=re.S)  # defined there, called later
            assert not re.search(r"\breturn\b|__ld|\[[^\]]*\] =|atomic|lengths|decode_keys", ahead), name
    assert kernels >= 3
    # past L1, because dQ did not wait; and the roles that both kernels share wait for nothing but barriers
    roles = {n: re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, n)).read()) for n in ("attn_dq.cuh", "attn_dkdv.cuh")}
    assert "return kWindow ? __ldcg(p) : *p;" in roles["attn_dq.cuh"] and not re.search(r"(LSE|Delta)\[", roles["attn_dq.cuh"])
    assert not any("griddep" in r for r in roles.values())
    for n, call in (("attn_dq.cu", "    dq_roles<"), ("attn_dkdv.cu", "    kv_roles<")):
        text = open(os.path.join(CSRC, n)).read()
        assert text.index("\n    griddep_wait();") < text.index(call) and text.count(call) == 1, n
    api = open(os.path.join(CSRC, "ops", "window_api.cu")).read()
    assert re.search(r"launch_window_dkdv\([^;]*;\s+if \(e == cudaSuccess\)\s+e = launch_window_dq\(", api)


# ---------------------------------------------------------------- frequencies and the reference

def test_frequencies(lib):
    from paper_2608_00029_b200 import nova_attn as na, nova_rope as nr
    f, a = nr.nova_rope_frequencies(64)
    i = torch.arange(0, 64, 2, dtype=torch.float64)
    want = 10000.0 ** (-i / 64)
    assert a == 1.0 and torch.equal(f, want.float())
    assert torch.equal(nr.nova_rope_frequencies(64, kind="linear", factor=4.0)[0], (want / 4).float())
    stretched = nr.nova_rope_frequencies(64, kind="base", factor=8.0)[0].double()
    assert abs(stretched[0] - 1) < 1e-7 and abs(stretched[-1] * 8 / want[-1] - 1) < 1e-6
    for kind in ("bands", "yarn"):
        f, a = nr.nova_rope_frequencies(128, 500000.0, kind, 8.0, 8192, 1.0, 32.0)
        j = torch.arange(0, 128, 2, dtype=torch.float64)
        plain = 500000.0 ** (-j / 128)
        turns = 8192 * plain / (2 * math.pi)
        ratio = f.double() / plain
        assert (abs(ratio[turns >= 40] - 1) < 1e-6).all() and (abs(ratio[turns <= 0.8] * 8 - 1) < 1e-6).all()
        assert (ratio[1:] <= ratio[:-1] + 1e-6).all()
        assert a == (1.0 if kind == "bands" else pytest.approx(0.1 * math.log(8) + 1, abs=1e-6))
    r = ((8192 * plain / (2 * math.pi)) - 1) / 31
    r = r.clamp(0, 1)
    f = nr.nova_rope_frequencies(128, 500000.0, "bands", 8.0, 8192, 1.0, 32.0)[0].double()
    assert ((f - plain * (r + (1 - r) / 8)).abs() <= 2.0**-23 * f).all()
    for bad in (dict(rotary=7), dict(rotary=0), dict(rotary=64, base=1.0), dict(rotary=64, base=math.nan),
                dict(rotary=64, kind="linear", factor=0.5), dict(rotary=2, kind="base", factor=2.0),
                dict(rotary=64, kind="yarn", factor=2.0, original=0), dict(rotary=64, kind="bands", factor=2.0, original=8, low=4.0, high=4.0)):
        with pytest.raises(na.NovaAttnError) as e:
            nr.nova_rope_frequencies(**bad)
        assert e.value.status == na.ERR_SHAPE
    with pytest.raises(ValueError):
        nr.nova_rope_frequencies(64, kind="other")
    for bad in ({"rotary": 2**32 + 2}, {"rotary": 64, "original": 2**63}):  # would wrap to numbers that it takes
        with pytest.raises(ValueError):
            nr.nova_rope_frequencies(**bad)
    with pytest.raises(TypeError):
        nr.nova_rope_frequencies(64.5)


def test_reference_gradients_against_differences():
    g = torch.Generator().manual_seed(0)
    B, H, KV, T, D, window, sinks, scale = 1, 4, 2, 11, 8, 4, 2, 0.35
    q, do = (torch.randn(B, H, T, D, generator=g, dtype=torch.float64) for _ in range(2))
    k, v = (torch.randn(B, KV, T, D, generator=g, dtype=torch.float64) for _ in range(2))
    grads, _, _ = ref.backward(q, k, v, do, scale, window, sinks)
    loss = lambda: float((ref.forward(q, k, v, scale, window, sinks)[0] * do).sum())
    h = 1e-6
    for x, dx in zip((q, k, v), grads):
        for _ in range(40):
            at = tuple(int(torch.randint(n, (1,), generator=g)) for n in x.shape)
            keep = float(x[at])
            x[at] = keep + h
            up = loss()
            x[at] = keep - h
            down = loss()
            x[at] = keep
            assert abs((up - down) / (2 * h) - float(dx[at])) < 1e-7


def test_reference_mask_and_single_token():
    m = ref.kept(7, 3, 2)
    assert [[j for j in range(7) if m[i, j]] for i in (0, 2, 4, 6)] == [[0], [0, 1, 2], [0, 1, 2, 3, 4], [0, 1, 4, 5, 6]]
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn(2, h, 9, 8, generator=g, dtype=torch.float64) for h in (4, 2, 2))
    o, lse, _ = ref.forward(q, k, v, 0.3, 4, 1)
    o1, lse1, _ = ref.decode(q[:, :, -1:], k, v, [9, 9], 0.3, 4, 1)
    assert torch.allclose(o1, o[:, :, -1:], atol=1e-12) and torch.allclose(lse1, lse[:, :, -1:], atol=1e-12)
