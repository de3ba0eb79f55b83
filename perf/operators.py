"""What is measured of the operators around a streaming DiT block's attention.

Four operators, each in its plain form (elementary torch operations in 32
bits) and through the library's public calls:

  rotary   rotary positions on the queries and keys of a block, and the
           gradient (the transposed rotation);
  norm     the residual update x + gate * norm(y) fused with the next block's
           modulated norm, and its gradients;
  append   a chunk's keys and values quantised into a cache of 4-bit codes
           with one scale for each 32 values, and read back as bfloat16;
  attn     attention of a chunk's queries (from one token to a whole video
           chunk) over such a cache.
"""
import math

import torch

own = False

BF16 = torch.bfloat16


# --------------------------------------------------------------------- cases
def listed():
    return [
        # one new token of 16 streams, positions deep into an extended context
        dict(name="rotary-decode", op="rotary", batch=16, tokens=1, heads=32,
             kv_heads=8, dim=128, rot=128, layout="half", axes=1,
             scaling="yarn", factor=8.0, context=16384, span=131072,
             grad=False, dtype="bf16"),
        # a 1080p chunk (2 frames of 68 x 120 tokens) straight from the fused
        # QKV projection, three-axis video positions
        dict(name="rotary-1080p-chunk", op="rotary", batch=1, tokens=16320,
             heads=12, kv_heads=12, dim=128, rot=128, layout="interleaved",
             axes=3, scaling="none", factor=1.0, context=0, span=120,
             grad=False, dtype="bf16"),
        # gradients of a training clip (12 frames of 32 x 32 tokens), half of
        # each head rotated
        dict(name="rotary-clip-grad", op="rotary", batch=1, tokens=12288,
             heads=24, kv_heads=24, dim=128, rot=64, layout="half", axes=1,
             scaling="linear", factor=4.0, context=0, span=12288,
             grad=True, dtype="bf16"),
        # one new token of 16 streams
        dict(name="norm-decode", op="norm", batch=16, tokens=1, groups=1,
             dim=1536, pre="rms", post="rms", res="bf16", grad=False),
        # between two blocks of a 1080p chunk, one modulation per frame
        dict(name="norm-1080p-chunk", op="norm", batch=1, tokens=16320,
             groups=2, dim=1536, pre="layer", post="none", res="bf16",
             grad=False),
        # the same place in training: a clip of 12 frames, float32 residual
        dict(name="norm-clip-grad", op="norm", batch=1, tokens=12288,
             groups=12, dim=1536, pre="layer", post="rms", res="f32",
             grad=True),
        # a 480p chunk into the cache
        dict(name="append-480p-chunk", op="append", batch=1, frame=1590,
             frames=2, kv_heads=12, dim=128, window=4),
        # a chunk of the windowed 1080p stream
        dict(name="append-1080p-chunk", op="append", batch=1, frame=8160,
             frames=3, kv_heads=24, dim=128, window=4),
        # one new token against a window of 4096 earlier ones: latency
        dict(name="attn-decode-4k", op="attn", batch=1, heads=12, kv_heads=12,
             dim=128, frame=1, frames=1, visible=4097, window=4096, first=7,
             ragged=False),
        # one new token of 8 streams that joined at different times, shared
        # key heads, long context
        dict(name="attn-decode-batch-64k", op="attn", batch=8, heads=32,
             kv_heads=8, dim=128, frame=1, frames=1, visible=65533,
             window=65532, first=1001, ragged=True),
        # the last chunk of the 480p stream
        dict(name="attn-480p-chunk", op="attn", batch=1, heads=12,
             kv_heads=12, dim=128, frame=1590, frames=2, visible=8, window=7,
             first=3, ragged=False),
        # the last chunk of the 720p stream
        dict(name="attn-720p-chunk", op="attn", batch=1, heads=12,
             kv_heads=12, dim=128, frame=3600, frames=2, visible=8, window=7,
             first=0, ragged=False),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo),
                                                          math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rotary", "norm", "append", "attn", "attn"])
    if op == "rotary":
        dim = rng.choice([64, 128])
        heads = rng.choice([4, 8, 12, 16, 24])
        kv = rng.choice([h for h in (1, 2, 4, 8, 12, 16, 24)
                         if heads % h == 0])
        axes = rng.choice([1, 3])
        rot = dim if axes == 3 else rng.choice([dim // 2, dim, dim - 24])
        batch = rng.choice([1, 1, 2, 5])
        tokens = _log(rng, 1, 16320 * 12 * 2 * 128 //
                      (batch * (heads + kv) * dim))
        scaling = rng.choice(["none", "linear", "ntk", "yarn"])
        return dict(op=op, batch=batch, tokens=min(tokens, 24480), heads=heads,
                    kv_heads=kv, dim=dim, rot=rot,
                    layout=rng.choice(["interleaved", "half"]), axes=axes,
                    scaling=scaling,
                    factor=1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.0]),
                    context=4096 if scaling == "yarn" else 0,
                    span=rng.choice([512, 4096, 65536]) if axes == 1 else 120,
                    grad=rng.choice([False, True]),
                    dtype=rng.choice(["bf16", "bf16", "f32"]))
    if op == "norm":
        dim = rng.choice([64, 520, 1024, 1536, 2048, 5120])
        batch = rng.choice([1, 2, 3])
        groups = rng.choice([1, 2, 3, 12])
        per = _log(rng, 1, max(1, 12288 * 1536 // (batch * groups * dim)))
        return dict(op=op, batch=batch, tokens=groups * per, groups=groups,
                    dim=dim, pre=rng.choice(["rms", "layer"]),
                    post=rng.choice(["none", "rms", "layer"]),
                    res=rng.choice(["bf16", "f32"]),
                    grad=rng.choice([False, True]))
    if op == "append":
        dim = rng.choice([64, 128])
        kv = rng.choice([1, 2, 8, 12, 24])
        batch = rng.choice([1, 2, 6])
        frames = rng.choice([1, 2, 3])
        frame = _log(rng, 1, max(1, 3 * 8160 * 24 * 128 //
                                 (batch * kv * dim * frames)))
        return dict(op=op, batch=batch, frame=min(frame, 8160), frames=frames,
                    kv_heads=kv, dim=dim, window=rng.choice([0, 1, 4]))
    dim = rng.choice([64, 128])
    kv = rng.choice([1, 2, 8, 12])
    heads = kv * rng.choice([1, 1, 2, 4])
    if rng.random() < 0.6:  # few queries
        batch = rng.choice([1, 2, 4, 8])
        frames = rng.choice([1, 1, 2])
        frame = rng.choice([1, 1, 2, 5, 17, 64, 150])
        cap = 8 * 8 * 65533 // (batch * kv * frames * frame)
        visible = _log(rng, 1, max(1, min(65533, cap)))
    else:                   # chunks of video
        batch = rng.choice([1, 2])
        frames = rng.choice([1, 2, 3])
        frame = _log(rng, 200, 3600)
        visible = rng.choice([1, 2, 5, 8])
        while batch * heads * (frames * frame) ** 2 * visible * dim > \
                12 * 7200 ** 2 * 8 * 128:
            frame = frame * 2 // 3
    # a stream at its start (first = 0) may not have filled its window yet
    first = rng.choice([0, 0, 1, 2, 5])
    return dict(op=op, batch=batch, heads=heads, kv_heads=kv, dim=dim,
                frame=frame, frames=frames, visible=visible,
                window=visible - 1 + (0 if first else rng.choice([0, 1, 3])),
                first=first, ragged=rng.choice([False, True]))


# -------------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _dt(name):
    return torch.float32 if name == "f32" else BF16


def _sections(case):
    pairs = case["rot"] // 2
    if case["axes"] == 1:
        return [pairs]
    side = pairs // 3
    return [pairs - 2 * side, side, side]


def _rotary_inputs(case, seed):
    g = _gen(seed)
    B, L = case["batch"], case["tokens"]
    H, K, d = case["heads"], case["kv_heads"], case["dim"]
    # the fused projection's output, heads of q, k and v side by side (for
    # the gradient: the attention's dq and dk in the same order)
    qkv = _randn(g, B, L, H + 2 * K, d).to(_dt(case["dtype"]))
    if case["axes"] == 1:
        start = torch.randint(0, max(1, case["span"] - L), (B, 1), generator=g,
                              device="cuda")
        pos = (start + torch.arange(L, device="cuda"))[:, :, None]
    else:  # frames of a grid as wide as the span allows
        wide = min(case["span"], L)
        t = torch.arange(L, device="cuda")
        high = 68
        t0 = int(torch.randint(0, 64, (1,), generator=g, device="cuda"))
        pos = torch.stack([t0 + t // (wide * high), t // wide % high,
                           t % wide], -1)[None]
    return qkv, pos.to(torch.int32).contiguous()


def _norm_inputs(case, seed):
    g = _gen(seed)
    B, L, G, D = case["batch"], case["tokens"], case["groups"], case["dim"]
    # a residual stream has a few channels far larger than the others, and
    # drifts away from zero mean
    chan = torch.where(torch.rand(D, generator=g, device="cuda") < 0.01,
                       12.0, 1.0)
    s = dict(x=(_randn(g, B, L, D) * chan + 0.3).to(_dt(case["res"])),
             y=(_randn(g, B, L, D) * 0.7).to(BF16),
             gate=_randn(g, B, G, D) * 0.5, scale=_randn(g, B, G, D) * 0.3,
             shift=_randn(g, B, G, D) * 0.3, pre_weight=None, post_weight=None)
    if case["pre"] == "rms":
        s["pre_weight"] = 1 + 0.2 * _randn(g, D)
    if case["post"] == "rms":
        s["post_weight"] = 1 + 0.2 * _randn(g, D)
    if case["grad"]:
        s["dr"] = (_randn(g, B, L, D) * 0.1).to(_dt(case["res"]))
        s["dh"] = (_randn(g, B, L, D) * 0.1).to(BF16)
    return s


def _kv(g, B, T, K, d):
    # keys have a few strong channels, values do not
    chan = torch.where(torch.rand((K, d), generator=g, device="cuda") < 0.03,
                       4.0, 1.0)
    k = torch.empty((B, T, K, d), dtype=BF16, device="cuda")
    v = torch.empty_like(k)
    step = max(1, (1 << 26) // max(1, B * K * d))
    for t in range(0, T, step):
        n = min(step, T - t)
        k[:, t:t + n] = (_randn(g, B, n, K, d) * chan).to(BF16)
        v[:, t:t + n] = _randn(g, B, n, K, d).to(BF16)
    return k, v


def _append_inputs(case, seed):
    g = _gen(seed)
    return _kv(g, case["batch"], case["frame"] * case["frames"],
               case["kv_heads"], case["dim"])


def _attn_inputs(case, seed):
    g = _gen(seed)
    B, n = case["batch"], case["frame"] * case["frames"]
    k, v = _kv(g, B, n * case["visible"], case["kv_heads"], case["dim"])
    q = _randn(g, B, n, case["heads"], case["dim"]).to(BF16)
    first = None
    if case["ragged"]:
        # the chunk at which each stream of the batch joined
        first = case["first"] + torch.randint(0, case["visible"], (B,),
                                              generator=g, device="cuda")
        first = first.to(torch.int32)
    return q, k, v, first


# ------------------------------------------------------ the plain forms' plans
def _rotary_tables(case):
    """cos and sin for every position up to the span, as a program keeps
    them: per axis [span, pairs of the axis] in float32."""
    s, tables = case["factor"], []
    mag = 1.0
    if case["scaling"] == "yarn":
        mag = 0.1 * math.log(s) + 1.0
    for n in _sections(case):
        i = torch.arange(n, dtype=torch.float64, device="cuda")
        base = 10000.0
        if case["scaling"] == "ntk" and n > 1:
            base *= s ** (n / (n - 1))
        f = base ** (-i / n)
        if case["scaling"] == "linear":
            f = f / s
        if case["scaling"] == "yarn":
            turns = case["context"] * f / (2 * math.pi)
            keep = ((turns - 1.0) / (32.0 - 1.0)).clamp(0, 1)
            f = f / s * (1 - keep) + f * keep
        span = max(case["span"], case["tokens"], 68,
                   64 + case["tokens"] // 68 + 1) + 1
        a = torch.arange(span, dtype=torch.float64, device="cuda")[:, None] * f
        tables.append(((a.cos() * mag).float(), (a.sin() * mag).float()))
    return tables


def _rotary_plain(case, x, cos, sin):
    r, sign = case["rot"], -1.0 if case["grad"] else 1.0
    f = x.float()
    c, s = cos[:, :, None], sign * sin[:, :, None]
    if case["layout"] == "half":
        a, b = f[..., :r // 2], f[..., r // 2:r]
        y = torch.cat([a * c - b * s, b * c + a * s, f[..., r:]], -1)
    else:
        a, b = f[..., 0:r:2], f[..., 1:r:2]
        y = torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)
        y = torch.cat([y, f[..., r:]], -1)
    return y.to(x.dtype)


def _spread(m, L):
    """[B, G, D] to [B, L, D]."""
    return m.repeat_interleave(L // m.shape[1], 1)


def _unit(v, kind):
    """v normalised over its last axis, and 1 / its deviation."""
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
    rho = 1 / torch.sqrt((v * v).mean(-1, keepdim=True) + 1e-6)
    return v * rho, rho


def _unit_grad(du, u, rho, kind):
    g = du - u * (du * u).mean(-1, keepdim=True)
    if kind == "layer":
        g = g - du.mean(-1, keepdim=True)
    return g * rho


def _norm_plain(case, s):
    L = case["tokens"]
    f = {n: (None if t is None else t.float()) for n, t in s.items()
         if torch.is_tensor(t) or t is None}
    gate, scale, shift = (_spread(f[n], L) for n in ("gate", "scale", "shift"))
    u, rho_y = f["y"], None
    if case["post"] != "none":
        u, rho_y = _unit(u, case["post"])
    w = 1.0 if f["pre_weight"] is None else f["pre_weight"]
    pw = 1.0 if f["post_weight"] is None else f["post_weight"]
    if not case["grad"]:
        r = f["x"] + gate * (u * pw)
        n, _ = _unit(r, case["pre"])
        h = n * w * (1 + scale) + shift
        return r.to(s["x"].dtype), h.to(BF16)
    # the state's x is the residual after the update
    n, rho = _unit(f["x"], case["pre"])
    dh = f["dh"]
    B, G, D = f["gate"].shape
    fold = lambda t: t.view(B, G, L // G, D).sum(2)
    dx = f["dr"] + _unit_grad(dh * (1 + scale) * w, n, rho, case["pre"])
    out = [dx.to(s["x"].dtype)]
    du = dx * gate * pw
    if rho_y is not None:
        out.append(_unit_grad(du, u, rho_y, case["post"]).to(BF16))
    else:
        out.append(du.to(BF16))
    out += [fold(dx * u * pw), fold(dh * n * w), fold(dh)]
    if f["pre_weight"] is not None:
        out.append((dh * (1 + scale) * n).sum((0, 1)))
    if f["post_weight"] is not None:
        out.append((dx * gate * u).sum((0, 1)))
    return tuple(out)


def _quantise(x):
    """Codes 1..15 [..., d] (uint8) and scales [..., d / 32] (float32) of a
    bfloat16 tensor: scale = max / 7 kept to five significant bits, code =
    8 + the nearest whole multiple of the scale, ties toward zero."""
    f = x.float().unflatten(-1, (-1, 32))
    s = f.abs().amax(-1) / 7
    m, e = torch.frexp(s)
    s = torch.ldexp(torch.round(m * 32) / 32, e)
    t = f / torch.where(s > 0, s, 1.0)[..., None]
    n = torch.sign(t) * torch.ceil(t.abs() - 0.5).clamp(max=7)
    return (n + 8).to(torch.uint8).flatten(-2), s


def _pack(c):
    return c[..., 0::2] | (c[..., 1::2] << 4)


def _values(codes, scales):
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    f = (c.float() - 8).unflatten(-1, (-1, 32)) * scales[..., None]
    return f.flatten(-2)


# ------------------------------------------------------------ states and runs
def prepare(case, seed):
    if own:
        from paper_2609_36757_gb300 import fastvr as FV
    op = case["op"]
    if op == "rotary":
        qkv, pos = _rotary_inputs(case, seed)
        s = dict(case=case, qkv=qkv, pos=pos)
        if own:
            s["plan"] = FV.make_rotary_config(
                case["dim"], rotary_dim=case["rot"], layout=case["layout"],
                sections=_sections(case), scaling=case["scaling"],
                factors=[case["factor"]] * case["axes"],
                original_contexts=[case["context"]] * case["axes"])
        else:
            s["plan"] = _rotary_tables(case)
        return s
    if op == "norm":
        s = _norm_inputs(case, seed)
        s["case"] = case
        if own:
            s["plan"] = FV.make_norm_config(pre=case["pre"],
                                            post=case["post"])
        return s
    if op == "append":
        k, v = _append_inputs(case, seed)
        s = dict(case=case, k=k, v=v)
        B, K, d = case["batch"], case["kv_heads"], case["dim"]
        T = k.shape[1] * (case["window"] + 1)
        if own:
            s["stream"] = FV.StreamingAttention4(
                FV.make_config(B, K, d, case["frame"], case["frames"],
                               case["window"]))
        else:
            s["codes"] = torch.zeros((2, B, K, T, d // 2), dtype=torch.uint8,
                                     device="cuda")
            s["scales"] = torch.zeros((2, B, K, T, d // 32), dtype=BF16,
                                      device="cuda")
            s["slot"] = 0
        return s
    q, k, v, first = _attn_inputs(case, seed)
    s = dict(case=case, q=q, first=first)
    if own:
        att = FV.StreamingAttention4(
            FV.make_config(case["batch"], case["heads"], case["dim"],
                           case["frame"], case["frames"], case["window"]),
            kv_heads=case["kv_heads"])
        if case["first"]:
            att.set_state(case["first"], case["frames"])
        att.append(k, v)
        s["stream"] = att
    else:
        for n, x in (("k", k), ("v", v)):
            codes, scales = zip(*(_quantise(x[:, :, h])
                                  for h in range(case["kv_heads"])))
            s[n] = _pack(torch.stack(codes, 1))
            s[n + "_scale"] = torch.stack(scales, 1).to(BF16)
    return s


def _append_plain(s):
    n, T = s["k"].shape[1], s["codes"].shape[3]
    t = s["slot"] * n
    out = []
    for i, x in enumerate((s["k"], s["v"])):
        codes, scales = _quantise(x.transpose(1, 2))
        s["codes"][i, :, :, t:t + n] = _pack(codes)
        s["scales"][i, :, :, t:t + n] = scales.to(BF16)
        back = _values(s["codes"][i, :, :, t:t + n],
                       s["scales"][i, :, :, t:t + n].float())
        out.append(back.to(BF16).transpose(1, 2).contiguous())
    s["slot"] = (t + n) % T // n
    return tuple(out)


def _attn_plain(s):
    case = s["case"]
    B, H, K, d = (case[n] for n in ("batch", "heads", "kv_heads", "dim"))
    n, G = case["frame"] * case["frames"], H // K
    T = n * case["visible"]
    out = torch.empty((B, n, H, d), dtype=BF16, device="cuda")
    lse = torch.empty((B, H, n), dtype=torch.float32, device="cuda")
    chunk = case["first"] + torch.arange(T, device="cuda") // n
    hs = max(1, min(K, (1 << 28) // (T * max(d, G * n))))  # key heads at once
    step = max(1, (1 << 29) // (G * T * hs))                # and tokens
    for b in range(B):
        for h in range(0, K, hs):
            j = min(K, h + hs) - h
            kf = _values(s["k"][b, h:h + j], s["k_scale"][b, h:h + j].float())
            vf = _values(s["v"][b, h:h + j], s["v_scale"][b, h:h + j].float())
            for t in range(0, n, step):
                q = s["q"][b, t:t + step, h * G:(h + j) * G].float()
                m = q.shape[0]
                q = q.transpose(0, 1).reshape(j, G * m, d)
                x = (q @ kf.transpose(1, 2)) * d ** -0.5
                if s["first"] is not None:
                    x = x.masked_fill(chunk < s["first"][b], -math.inf)
                top = x.amax(-1, keepdim=True)
                x = torch.exp(x - top)
                z = x.sum(-1, keepdim=True)
                o = (x @ vf) / z
                out[b, t:t + m, h * G:(h + j) * G] = \
                    o.view(j * G, m, d).transpose(0, 1).to(BF16)
                lse[b, h * G:(h + j) * G, t:t + m] = \
                    (top + torch.log(z)).view(j * G, m)
    return out, lse


def run(state):
    case, op = state["case"], state["case"]["op"]
    if own:
        from paper_2609_36757_gb300 import fastvr as FV
    if op == "rotary":
        H, K = case["heads"], case["kv_heads"]
        q, k = state["qkv"][:, :, :H], state["qkv"][:, :, H:H + K]
        if own:
            f = FV.rotary_bwd if case["grad"] else FV.rotary
            return f(state["plan"], q, k, state["pos"])
        at = [(c[state["pos"][..., a].long()], s[state["pos"][..., a].long()])
              for a, (c, s) in enumerate(state["plan"])]
        cos, sin = (torch.cat(t, -1) for t in zip(*at))
        return (_rotary_plain(case, q, cos, sin),
                _rotary_plain(case, k, cos, sin))
    if op == "norm":
        if not own:
            return _norm_plain(case, state)
        weights = dict(pre_weight=state["pre_weight"],
                       post_weight=state["post_weight"])
        if not case["grad"]:
            return FV.gated_norm(state["plan"], state["x"], state["y"],
                                 state["gate"], state["scale"],
                                 state["shift"], **weights)
        g = FV.gated_norm_bwd(state["plan"], state["dr"], state["dh"],
                              state["x"], state["y"], state["gate"],
                              state["scale"], **weights)
        return tuple(t for t in g if t is not None)
    if op == "append":
        if not own:
            return _append_plain(state)
        state["stream"].append(state["k"], state["v"])
        return state["stream"].read()
    if not own:
        return _attn_plain(state)
    return state["stream"].forward(state["q"], first_chunk=state["first"],
                                   want_lse=True)


# ------------------------------------------------------------------------ work
def work(case):
    op, e = case["op"], 4 if case.get("dtype") == "f32" else 2
    if op == "rotary":
        n = case["batch"] * case["tokens"] * (case["heads"] + case["kv_heads"])
        shared = case["tokens"] * case["axes"] * 4
        return dict(bytes=2 * e * n * case["dim"] + shared,
                    flops=3 * n * case["rot"])
    if op == "norm":
        n = case["batch"] * case["tokens"] * case["dim"]
        m = case["batch"] * case["groups"] * case["dim"] * 4
        r = 4 if case["res"] == "f32" else 2
        if case["grad"]:  # dr, x, dx; dh, y, dy; gate, scale and gradients
            return dict(bytes=n * (3 * r + 3 * 2) + 5 * m, flops=40 * n)
        return dict(bytes=n * (2 * r + 2 * 2) + 3 * m, flops=16 * n)
    if op == "append":
        n = 2 * case["batch"] * case["frame"] * case["frames"] * \
            case["kv_heads"] * case["dim"]
        return dict(bytes=n * 4 + n // 2 + n // 16, flops=4 * n)
    q = case["batch"] * case["frame"] * case["frames"] * case["heads"]
    T = case["frame"] * case["frames"] * case["visible"]
    kv = 2 * case["batch"] * T * case["kv_heads"] * case["dim"]
    part = 0.5 if case["ragged"] else 1.0  # streams see half on average
    return dict(bytes=int(part * (kv // 2 + kv // 16)) +
                q * (4 * case["dim"] + 4),
                flops=int(part * 4 * q * T * case["dim"]))


# ------------------------------------------------- the definition in 64 bits
def _rotate_exact(x, angle, mag, layout, rot, transpose):
    y = x.double().clone()
    pairs = rot // 2
    first = torch.arange(pairs, device="cuda")
    if layout == "interleaved":
        first, second = 2 * first, 2 * first + 1
    else:
        second = first + pairs
    z = torch.complex(y[..., first], y[..., second])
    turn = torch.polar(torch.full_like(angle, mag),
                       -angle if transpose else angle)
    z = z * turn[:, :, None, :]
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _rotary_exact(case, seed):
    qkv, pos = _rotary_inputs(case, seed)
    H, K, s = case["heads"], case["kv_heads"], case["factor"]
    cols = []
    for axis, n in enumerate(_sections(case)):
        for i in range(n):
            theta = math.pow(10000.0, -i / n)
            if case["scaling"] == "linear":
                theta = theta / s
            elif case["scaling"] == "ntk" and n > 1:
                theta = math.pow(10000.0 * math.pow(s, 2 * n / (2 * n - 2)),
                                 -i / n)
            elif case["scaling"] == "yarn":
                ramp = (case["context"] * theta / (2 * math.pi) - 1) / 31
                ramp = min(1.0, max(0.0, ramp))
                theta = (1 - ramp) * theta / s + ramp * theta
            cols.append(pos[..., axis].double() * theta)
    angle = torch.stack(cols, -1)
    mag = 1 + 0.1 * math.log(s) if case["scaling"] == "yarn" else 1.0
    return tuple(_rotate_exact(x, angle, mag, case["layout"], case["rot"],
                               case["grad"])
                 for x in (qkv[:, :, :H], qkv[:, :, H:H + K]))


def _moments(v, kind):
    mu = v.mean(-1, keepdim=True) if kind == "layer" else torch.zeros_like(
        v[..., :1])
    var = ((v - mu) ** 2).mean(-1, keepdim=True)
    return mu, torch.rsqrt(var + 1e-6)


def _norm_exact(case, seed):
    s = {n: (t.double() if torch.is_tensor(t) else t)
         for n, t in _norm_inputs(case, seed).items()}
    B, L, G, D = case["batch"], case["tokens"], case["groups"], case["dim"]
    one = torch.ones(D, dtype=torch.float64, device="cuda")
    w = one if s["pre_weight"] is None else s["pre_weight"]
    pw = one if s["post_weight"] is None else s["post_weight"]
    cut = lambda t: t.reshape(B, G, L // G, D)
    x, y = cut(s["x"]), cut(s["y"])
    gate, scale, shift = (s[n][:, :, None] for n in ("gate", "scale", "shift"))
    yn, ry = y, None
    if case["post"] != "none":
        mu, ry = _moments(y, case["post"])
        yn = (y - mu) * ry
    u = yn * pw
    if not case["grad"]:
        r = x + gate * u
        mu, rho = _moments(r, case["pre"])
        h = (r - mu) * rho * w * (1 + scale) + shift
        return r.reshape(B, L, D), h.reshape(B, L, D)
    dr, dh = cut(s["dr"]), cut(s["dh"])
    mu, rho = _moments(x, case["pre"])
    xn = (x - mu) * rho

    def through(d, n, rho, kind):  # gradient of (v - mu) * rho at v
        d0 = d.mean(-1, keepdim=True) if kind == "layer" else 0.0
        return rho * (d - d0 - n * (d * n).mean(-1, keepdim=True))

    dx = dr + through(dh * w * (1 + scale), xn, rho, case["pre"])
    du = dx * gate
    dy = du * pw
    if ry is not None:
        dy = through(dy, yn, ry, case["post"])
    out = [dx.reshape(B, L, D), dy.reshape(B, L, D), (dx * u).sum(2),
           (dh * xn * w).sum(2), dh.sum(2)]
    if s["pre_weight"] is not None:
        out.append((dh * (1 + scale) * xn).sum((0, 1, 2)))
    if s["post_weight"] is not None:
        out.append((du * yn).sum((0, 1, 2)))
    return tuple(out)


def _stored_exact(x):
    """The values that the 4-bit cache holds for a bfloat16 tensor."""
    g = x.double().reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    top = g.abs().max(-1, keepdim=True).values
    s = top / 7
    unit = torch.exp2(torch.floor(torch.log2(s.clamp(min=1e-300))) - 4)
    s = torch.round(s / unit) * unit
    t = torch.where(s > 0, g / s.clamp(min=1e-300), 0.0)
    low = torch.floor(t.abs())
    n = low + (t.abs() - low > 0.5).double()
    return (torch.sign(t) * n.clamp(max=7) * s).reshape(x.shape)


def _attn_exact(case, seed):
    B, H, K, d = (case[n] for n in ("batch", "heads", "kv_heads", "dim"))
    n, G = case["frame"] * case["frames"], H // K
    T = n * case["visible"]
    # about 1 TFLOP/s in 64 bits
    if 4.0 * B * H * n * T * d > 1.2e13:
        return None
    q, k, v, first = _attn_inputs(case, seed)
    out = torch.zeros((B, n, H, d), dtype=torch.float64, device="cuda")
    lse = torch.empty((B, H, n), dtype=torch.float64, device="cuda")
    for b in range(B):
        lo = 0
        if first is not None:
            lo = min(T, max(0, int(first[b]) - case["first"]) * n)
        for h in range(H):
            kd = _stored_exact(k[b, lo:, h // G])
            vd = _stored_exact(v[b, lo:, h // G])
            rows = max(1, (1 << 28) // max(1, T - lo))
            for t in range(0, n, rows):
                score = q[b, t:t + rows, h].double() @ kd.T / math.sqrt(d)
                z = torch.logsumexp(score, -1)
                lse[b, h, t:t + rows] = z
                out[b, t:t + rows, h] = torch.exp(score - z[:, None]) @ vd
    return out, lse


def exact(case, seed):
    op = case["op"]
    if op == "rotary":
        return _rotary_exact(case, seed)
    if op == "norm":
        return _norm_exact(case, seed)
    if op == "append":
        return tuple(_stored_exact(x) for x in _append_inputs(case, seed))
    return _attn_exact(case, seed)
