"""Work of the rotary positions and of the attention with a sliding window and sinks, as a list of measurable cases.

  rope     one pass over Q and K: rotated by their tokens' positions (forward), or their gradients rotated back (backward)
  window   one layer's attention in which a query sees the last `window` keys, itself among them, and the first `sinks`:
           the forward alone (prefill, evaluation) or a training pass (forward, Delta, backward)
  decode   the same attention of one new token per sequence over a cache of keys and values of ragged lengths

Query heads may share key/value heads (`KV` of them for `H` query heads).  Layout "heads" is [B,H,T,D]; "fused" are views of one
projection output [B,T,H+2*KV,D], and of one gradient buffer of that shape.
"""
import math

import torch

own = False


def rope(name, B, H, KV, T, D, rotary, interleaved=False, layout="heads", positions="start", scaled=False, backward=False):
    c = {"op": "rope", "B": B, "H": H, "KV": KV, "T": T, "D": D, "rotary": rotary, "interleaved": interleaved,
         "layout": layout, "positions": positions, "scaled": scaled, "backward": backward}
    return dict(c, name=name) if name else c


def window(name, B, H, KV, T, D, window, sinks, layout="heads", train=False):
    c = {"op": "window", "B": B, "H": H, "KV": KV, "T": T, "D": D, "window": window, "sinks": sinks, "layout": layout,
         "train": train}
    return dict(c, name=name) if name else c


def decode(name, B, H, KV, T, D, window, sinks, ragged=True, layout="heads"):
    c = {"op": "decode", "B": B, "H": H, "KV": KV, "T": T, "D": D, "window": window, "sinks": sinks, "ragged": ragged,
         "layout": layout}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one layer of GPT-2 small at its training batch, in the projection's own layout
        rope("rope_train_fused", 8, 12, 12, 1024, 64, 64, layout="fused"),
        # gradients of a long context whose positions start far out, neighbouring pairs, half of the head rotated
        rope("rope_long_backward", 2, 12, 4, 8192, 128, 64, interleaved=True, positions="far", scaled=True, backward=True),
        # one new token of each of 32 sequences: latency
        rope("rope_tokens", 32, 16, 4, 1, 128, 128, positions="each"),
        # the smallest training pass: two query heads on one key/value head, all launch latency
        window("window_tiny_train", 1, 2, 1, 64, 64, 16, 1, train=True),
        # prefill of one prompt of odd length
        window("window_prompt", 1, 12, 12, 777, 64, 128, 4),
        # one layer of GPT-2 medium reading the fused projection output in place, no sinks
        window("window_medium_fused", 8, 16, 16, 1024, 64, 256, 0, layout="fused"),
        # long prompt, head dimension 128, three query heads to a key/value head
        window("window_long_forward", 2, 12, 4, 8192, 128, 1024, 4),
        # one layer of GPT-2 small at its training batch
        window("window_small_train", 8, 12, 12, 1024, 64, 256, 4, train=True),
        # training on a long context, the largest call
        window("window_long_train", 2, 12, 4, 8192, 128, 1024, 4, train=True),
        # one new token of one sequence: latency
        decode("decode_one", 1, 12, 12, 1024, 64, 256, 4, ragged=False),
        # a batch of chats of all lengths
        decode("decode_batch", 64, 32, 8, 8192, 128, 4096, 4),
        # two very long contexts without a window to speak of
        decode("decode_long", 2, 12, 4, 131072, 128, 131072, 0, layout="fused"),
    ]


def _log_int(rng, low, high):
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    """One more case of the same ranges, none dearer than the dearest listed one of its kind."""
    op = rng.choice(["rope", "window", "window", "decode"])
    KV = rng.choice([1, 2, 3, 4, 8, 12, 16])
    H = KV * rng.choice([1, 1, 2, 3, 4, 8])
    D = rng.choice([64, 128])
    layout = rng.choice(["heads", "fused"])
    if op == "rope":
        c = rope(None, _log_int(rng, 1, 64), H, KV, _log_int(rng, 1, 8192), D, rng.choice([D, D, D // 2, D // 4, 2 * rng.randint(1, D // 2)]),
                 rng.random() < 0.4, layout, rng.choice(["start", "far", "each"]), rng.random() < 0.3, rng.random() < 0.5)
        while c["B"] * c["T"] * (H + KV) * D > 30_000_000:
            c["B" if c["B"] > 1 else "T"] //= 2
        return c
    if op == "window":
        train = rng.random() < 0.6
        # a lone token has no gradient to speak of: a training sequence has 16 at least, and its window 8
        T = _log_int(rng, 16 if train else 1, 8192)
        if rng.random() < 0.3 and T >= 128:
            T = T // 128 * 128
        c = window(None, _log_int(rng, 1, 16), H, KV, T, D, _log_int(rng, 8 if train else 1, max(8, min(T, 2048))),
                   rng.choice([0, 1, 4, 16, 150]), layout, train)
        most = work(listed()[8 if train else 6])["flops"]
        while work(c)["flops"] > most or c["B"] * H * c["T"] ** 2 > 1.6e9 or c["B"] * c["T"] * H * D > 25_000_000:
            c["B" if c["B"] > 1 else "T"] //= 2
        return c
    T = _log_int(rng, 1, 65536)
    c = decode(None, _log_int(rng, 1, 64), H, KV, T, D, _log_int(rng, 1, max(1, T)), rng.choice([0, 1, 4, 16, 150]), rng.random() < 0.8,
               layout)
    while c["B"] * KV * c["T"] * D > 120_000_000 or c["B"] * H * c["T"] > 16_000_000:
        c["B" if c["B"] > 1 else "T"] //= 2
    return c


def _randn(g, *shape):
    return torch.randn(shape, dtype=torch.float32, generator=g, device="cuda").to(torch.bfloat16)


def _split(x, H, KV):
    """Views [B,H,T,D], [B,KV,T,D], [B,KV,T,D] of a fused buffer [B,T,H+2*KV,D]."""
    x = x.transpose(1, 2)
    return x[:, :H], x[:, H:H + KV], x[:, H + KV:]


def _lengths(case, g):
    """Tokens in each sequence's cache, the new one among them."""
    if not case["ragged"]:
        return torch.full((case["B"],), case["T"], dtype=torch.int32, device="cuda")
    return torch.randint(1, case["T"] + 1, (case["B"],), generator=g, device="cuda").to(torch.int32)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    B, H, KV, T, D = (case[k] for k in ("B", "H", "KV", "T", "D"))
    s = {"case": case}
    bf16 = {"dtype": torch.bfloat16, "device": "cuda"}
    if case["op"] == "rope":
        if case["layout"] == "fused":
            s["q"], s["k"], _ = _split(_randn(g, B, T, H + 2 * KV, D), H, KV)
            s["q_out"], s["k_out"], _ = _split(torch.empty((B, T, H + 2 * KV, D), **bf16), H, KV)
        else:
            s["q"], s["k"] = _randn(g, B, H, T, D), _randn(g, B, KV, T, D)
            s["q_out"], s["k_out"] = torch.empty_like(s["q"]), torch.empty_like(s["k"])
        i = torch.arange(0, case["rotary"], 2, dtype=torch.float64)
        # a context stretched eightfold: the slower half of the frequencies is divided, and the scores' scale goes by an amplitude
        f = 500000.0 ** (-i / case["rotary"]) if case["scaled"] else 10000.0 ** (-i / case["rotary"])
        s["inv_freq"] = (torch.where(i >= case["rotary"] // 2, f / 8, f) if case["scaled"] else f).to(torch.float32).cuda()
        s["amplitude"] = 1.2079441541679836 if case["scaled"] else 1.0
        t = torch.arange(T, dtype=torch.int32, device="cuda")
        if case["positions"] == "start":
            s["positions"] = t.expand(B, T).contiguous()
        else:
            first = torch.randint(0, 120000, (B, 1), generator=g, device="cuda").to(torch.int32)
            s["positions"] = (t + (first if case["positions"] == "each" else 120000)).expand(B, T).contiguous()
        return s
    s["scale"] = 1.0 / math.sqrt(D)
    if case["op"] == "decode":
        s["q"] = _randn(g, B, H, 1, D)
        if case["layout"] == "fused":  # a cache that holds a token's heads side by side
            s["k"], s["v"] = (_randn(g, B, T, KV, D).transpose(1, 2) for _ in range(2))
        else:
            s["k"], s["v"] = (_randn(g, B, KV, T, D) for _ in range(2))
        s["lengths"] = _lengths(case, g)
        s["out"] = torch.empty((B, H, 1, D), **bf16)
        s["lse"] = torch.empty((B, H, 1), dtype=torch.float32, device="cuda")
        return s
    if case["layout"] == "fused":
        s["q"], s["k"], s["v"] = _split(_randn(g, B, T, H + 2 * KV, D), H, KV)
        s["dq"], s["dk"], s["dv"] = _split(torch.empty((B, T, H + 2 * KV, D), **bf16), H, KV)
        s["dout"] = _randn(g, B, T, H, D).transpose(1, 2)
        s["out"], s["rest"] = (torch.empty((B, T, H, D), **bf16).transpose(1, 2) for _ in range(2))
    else:
        s["q"], s["k"], s["v"], s["dout"] = (_randn(g, B, n, T, D) for n in (H, KV, KV, H))
        s["out"], s["rest"], s["dq"], s["dk"], s["dv"] = (torch.empty((B, n, T, D), **bf16) for n in (H, H, H, KV, KV))
    s["lse"], s["delta"] = (torch.empty((B, H, T), dtype=torch.float32, device="cuda") for _ in range(2))
    return s


def _plain_rope(s):
    c = s["case"]
    half = c["rotary"] // 2
    # a far position times a frequency needs more than 32 bits; its sine and cosine do not
    angle = s["positions"].double()[:, None, :, None] * s["inv_freq"].double()
    cos, sin = angle.cos().float() * s["amplitude"], angle.sin().float() * s["amplitude"]
    sin = -sin if c["backward"] else sin

    def turn(x):
        x = x.float()
        r, rest = x[..., :2 * half], x[..., 2 * half:]
        if c["interleaved"]:
            a, b = r[..., 0::2], r[..., 1::2]
            y = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
        else:
            a, b = r[..., :half], r[..., half:]
            y = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
        return torch.cat((y, rest), -1).to(torch.bfloat16)

    return turn(s["q"]), turn(s["k"])


def _plain_window(s):
    c = s["case"]
    B, H, KV, T, D = (c[k] for k in ("B", "H", "KV", "T", "D"))
    q, do = (s[n].float().reshape(B, KV, H // KV, T, D) for n in ("q", "dout"))
    k, v = (s[n].float().unsqueeze(2) for n in ("k", "v"))
    i = torch.arange(T, device="cuda")
    back = i[:, None] - i
    keep = (back >= 0) & ((back < c["window"]) | (i < c["sinks"]))
    p = (q @ k.mT * s["scale"]).masked_fill_(~keep, -math.inf)
    top = p.amax(-1, keepdim=True)
    p = p.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    lse = (top + total.log()).reshape(B, H, T)
    p = p.div_(total)
    o = p @ v
    out = o.reshape(B, H, T, D).to(torch.bfloat16)
    if not c["train"]:
        return out, lse
    ds = do @ v.mT
    ds = ds.sub_((do * o).sum(-1, keepdim=True)).mul_(p)
    dq = (ds @ k * s["scale"]).reshape(B, H, T, D).to(torch.bfloat16)
    dk = ((ds.mT @ q).sum(2) * s["scale"]).to(torch.bfloat16)
    dv = (p.mT @ do).sum(2).to(torch.bfloat16)
    return out, lse, dq, dk, dv


def _plain_decode(s):
    c = s["case"]
    B, H, KV, T, D = (c[k] for k in ("B", "H", "KV", "T", "D"))
    q = s["q"].float().reshape(B, KV, H // KV, D)
    j = torch.arange(T, device="cuda")
    back = s["lengths"].long()[:, None] - 1 - j
    keep = (back >= 0) & ((back < c["window"]) | (j < c["sinks"]))
    p = (q @ s["k"].float().mT * s["scale"]).masked_fill_(~keep[:, None, None], -math.inf)
    top = p.amax(-1, keepdim=True)
    p = p.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = (p @ s["v"].float() / total).reshape(B, H, 1, D).to(torch.bfloat16)
    return out, (top + total.log()).reshape(B, H, 1)


def _own(s):
    from paper_2608_00029_b200 import nova_rope, nova_window

    c = s["case"]
    if c["op"] == "rope":
        call = nova_rope.nova_rope_bwd if c["backward"] else nova_rope.nova_rope_fwd
        call(s["q"], s["k"], s["q_out"], s["k_out"], s["inv_freq"], s["positions"], interleaved=c["interleaved"],
             amplitude=s["amplitude"])
        return s["q_out"], s["k_out"]
    if c["op"] == "decode":
        nova_window.nova_window_decode(s["q"], s["k"], s["v"], s["lengths"], s["out"], s["lse"], s["scale"], c["window"], c["sinks"])
        return s["out"], s["lse"]
    if not c["train"]:
        nova_window.nova_window_fwd(s["q"], s["k"], s["v"], s["out"], s["lse"], s["scale"], c["window"], c["sinks"])
        return s["out"], s["lse"]
    # what rounding took from the output is kept too, for Delta
    nova_window.nova_window_fwd(s["q"], s["k"], s["v"], s["out"], s["lse"], s["scale"], c["window"], c["sinks"], O_rest=s["rest"])
    nova_window.nova_window_bwd_preprocess(s["out"], s["rest"], s["dout"], s["delta"])
    nova_window.nova_window_bwd(s["q"], s["k"], s["v"], s["dout"], s["lse"], s["delta"], s["dq"], s["dk"], s["dv"], s["scale"],
                                c["window"], c["sinks"])
    return s["out"], s["lse"], s["dq"], s["dk"], s["dv"]


def run(state):
    if own:
        return _own(state)
    return {"rope": _plain_rope, "window": _plain_window, "decode": _plain_decode}[state["case"]["op"]](state)


def _pairs(T, window, sinks):
    """Kept (query, key) pairs of T queries: the window's, and the sinks before it."""
    w, s = min(window, T), min(sinks, T)
    inside = w * (w + 1) // 2 + (T - w) * w
    m = T - w  # queries with keys before their window: 1, 2, ..., m of them
    return inside + (s * (s + 1) // 2 + (m - s) * s if m > s else m * (m + 1) // 2)


def work(case):
    B, H, KV, T, D = (case[k] for k in ("B", "H", "KV", "T", "D"))
    if case["op"] == "rope":
        rows = B * T * (H + KV)
        return {"bytes": 4 * rows * D + 4 * B * T + 2 * case["rotary"], "flops": 3 * rows * case["rotary"]}
    if case["op"] == "decode":
        # ragged lengths are uniform over the cache: the keys that the mean sequence reads
        n = case["window"] + case["sinks"]
        mean = min(T, n) if not case["ragged"] else (T + 1) / 2 if n >= T else (n * (n + 1) / 2 + (T - n) * n) / T
        return {"bytes": int(4 * B * KV * mean * D + 4 * B * H * D + 4 * B * H + 4 * B), "flops": int(4 * B * H * mean * D)}
    rows, kv_rows = B * H * T, B * KV * T
    pairs = B * H * _pairs(T, case["window"], case["sinks"])
    bytes_ = 4 * rows * D + 4 * kv_rows * D + 4 * rows  # Q, O; K, V; LSE
    if case["train"]:
        bytes_ += 4 * rows * D + 4 * kv_rows * D  # dO, dQ; dK, dV
    return {"bytes": bytes_, "flops": pairs * D * (14 if case["train"] else 4)}


def exact(case, seed):
    """The same from the definition, in 64 bits, one key/value head of one sequence at a time."""
    s = prepare(case, seed)
    B, H, KV, T, D = (case[k] for k in ("B", "H", "KV", "T", "D"))
    G = H // KV
    if case["op"] == "rope":
        # each pair is a complex number, turned by exp(+-i * position * frequency)
        sign = -1.0 if case["backward"] else 1.0
        a = torch.einsum("bt,f->btf", s["positions"].double(), s["inv_freq"].double()) * sign
        unit = torch.polar(torch.full_like(a, s["amplitude"]), a)
        R = case["rotary"]
        res = []
        for x in (s["q"], s["k"]):
            y = x.double().clone()
            first, second = (slice(0, R, 2), slice(1, R, 2)) if case["interleaved"] else (slice(0, R // 2), slice(R // 2, R))
            for h in range(x.shape[1]):
                z = torch.complex(x[:, h, :, first].double(), x[:, h, :, second].double()) * unit
                y[:, h, :, first], y[:, h, :, second] = z.real, z.imag
            res.append(y)
        return tuple(res)
    f64 = {"dtype": torch.float64, "device": "cuda"}
    if case["op"] == "decode":
        out, lse = torch.zeros((B, H, 1, D), **f64), torch.full((B, H, 1), -math.inf, **f64)
        for b, n in enumerate(s["lengths"].tolist()):
            seen = [j for j in range(min(n, case["sinks"])) if n - 1 - j >= case["window"]]
            at = torch.tensor(seen + list(range(max(0, n - case["window"]), n)), device="cuda", dtype=torch.long)
            for kv in range(KV):
                k, v = s["k"][b, kv, at].double(), s["v"][b, kv, at].double()
                z = s["q"][b, kv * G:(kv + 1) * G, 0].double() @ k.T / math.sqrt(D)
                lse[b, kv * G:(kv + 1) * G, 0] = torch.logsumexp(z, 1)
                out[b, kv * G:(kv + 1) * G, 0] = torch.softmax(z, 1) @ v
        return out, lse
    out, lse = torch.zeros((B, H, T, D), **f64), torch.zeros((B, H, T), **f64)
    dq, dk, dv = torch.zeros((B, H, T, D), **f64), torch.zeros((B, KV, T, D), **f64), torch.zeros((B, KV, T, D), **f64)
    row, col = torch.arange(T, device="cuda").unsqueeze(1), torch.arange(T, device="cuda").unsqueeze(0)
    hidden = (col > row) | ((col <= row - case["window"]) & (col >= case["sinks"]))
    for b in range(B):
        for h in range(H):
            kv = h // G
            q, k, v, do = (x.double() for x in (s["q"][b, h], s["k"][b, kv], s["v"][b, kv], s["dout"][b, h]))
            z = torch.where(hidden, -math.inf, torch.mm(q, k.T) / math.sqrt(D))
            lse[b, h] = torch.logsumexp(z, 1)
            p = torch.softmax(z, 1)
            out[b, h] = torch.mm(p, v)
            if case["train"]:
                # the Jacobian of the softmax applied to dP, row by row
                dp = torch.mm(do, v.T)
                dz = p * dp - p * (p * dp).sum(1, keepdim=True)
                dq[b, h] = torch.mm(dz, k) / math.sqrt(D)
                dk[b, kv] += torch.mm(dz.T, q) / math.sqrt(D)
                dv[b, kv] += torch.mm(p.T, do)
    return (out, lse, dq, dk, dv) if case["train"] else (out, lse)
