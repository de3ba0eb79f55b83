"""What is measured of a conditioned DiT block's other two operators.

Each in its plain form (elementary torch operations in 32 bits) and through
the library's public calls:

  cross  attention of a chunk's queries (from one token to a 1080p chunk) to
         an encoder's states of another length, a length for each batch entry
         where the prompts differ, key heads shared where there are fewer;
         with grad, the forward and the gradients of q, k and v;
  ffn    the gated feed-forward's first half, act(x Wg^T) * (x Wu^T); with
         grad, the forward and the gradients of x and both weights.
"""
import math

import torch

own = False

BF16 = torch.bfloat16


# --------------------------------------------------------------------- cases
def listed():
    return [
        # one new token against a short text prompt: latency
        dict(name="cross-decode", op="cross", batch=1, tokens=1, heads=12,
             kv_heads=12, dim=128, keys=77, ragged=False, grad=False),
        # one new token of 16 streams, each with a prompt of its own length,
        # shared key heads
        dict(name="cross-decode-batch", op="cross", batch=16, tokens=1,
             heads=32, kv_heads=8, dim=128, keys=512, ragged=True,
             grad=False),
        # a 480p chunk (2 frames of 30 x 53 tokens) against 226 text tokens
        dict(name="cross-480p-chunk", op="cross", batch=1, tokens=3180,
             heads=12, kv_heads=12, dim=128, keys=226, ragged=False,
             grad=False),
        # a 1080p chunk (2 frames of 68 x 120 tokens) against a long prompt
        dict(name="cross-1080p-chunk", op="cross", batch=1, tokens=16320,
             heads=12, kv_heads=12, dim=128, keys=512, ragged=False,
             grad=False),
        # training: a clip of 12 frames of 32 x 32 tokens, one prompt
        dict(name="cross-clip-grad", op="cross", batch=1, tokens=12288,
             heads=24, kv_heads=24, dim=128, keys=512, ragged=False,
             grad=True),
        # training: four short clips with prompts of different lengths, some
        # of them dropped, shared key heads, smaller heads
        dict(name="cross-batch-grad", op="cross", batch=4, tokens=1590,
             heads=16, kv_heads=4, dim=64, keys=333, ragged=True, grad=True),
        # one token: latency
        dict(name="ffn-decode", op="ffn", tokens=1, dim=1536, hidden=4096,
             act="silu", grad=False),
        # one token of 16 streams
        dict(name="ffn-decode-batch", op="ffn", tokens=16, dim=1536,
             hidden=4096, act="silu", grad=False),
        # a 480p chunk
        dict(name="ffn-480p-chunk", op="ffn", tokens=3180, dim=1536,
             hidden=4096, act="silu", grad=False),
        # a 1080p chunk
        dict(name="ffn-1080p-chunk", op="ffn", tokens=16320, dim=1536,
             hidden=4096, act="gelu_tanh", grad=False),
        # training: a clip of 12 frames of 32 x 32 tokens
        dict(name="ffn-clip-grad", op="ffn", tokens=12288, dim=1536,
             hidden=4096, act="silu", grad=True),
        # training: a few frames left of a clip, sizes that no tile divides
        dict(name="ffn-odd-grad", op="ffn", tokens=1061, dim=1000,
             hidden=2728, act="gelu", grad=True),
    ]


def _log(rng, lo, hi):
    hi = max(lo, hi)
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo),
                                                          math.log(hi)))))))


def draw(rng):
    op = rng.choice(["cross", "cross", "ffn", "ffn"])
    grad = rng.random() < 0.4
    if op == "cross":
        dim = rng.choice([64, 128])
        kv = rng.choice([1, 2, 4, 8, 12, 24])
        heads = kv * rng.choice([1, 1, 2, 4])
        batch = rng.choice([1, 1, 2, 3, 6, 16])
        keys = _log(rng, 1, 2048)
        # no more tokens than the largest listed cases have
        most = 12288 * 24 if grad else 16320 * 12
        most = min(most * 128 // (batch * heads * dim),
                   most * 128 * 512 // (batch * heads * dim * keys))
        tokens = _log(rng, 1, max(1, min(16320, most)))
        if not grad and rng.random() < 0.3:
            tokens = rng.choice([1, 1, 2, 5])
        return dict(op=op, batch=batch, tokens=tokens, heads=heads,
                    kv_heads=kv, dim=dim, keys=keys,
                    ragged=rng.choice([False, True]), grad=grad)
    dim = 8 * _log(rng, 8, 256)
    hidden = 8 * _log(rng, 8, 704)
    most = (12288 if grad else 16320) * 1536 * 4096 // (dim * hidden)
    tokens = _log(rng, 1, max(1, min(16320, most)))
    if rng.random() < 0.3:
        tokens = rng.choice([1, 2, 7, 16, 33])
    return dict(op=op, tokens=tokens, dim=dim, hidden=hidden,
                act=rng.choice(["silu", "gelu", "gelu_tanh"]), grad=grad)


# -------------------------------------------------------------------- inputs
def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _cross_inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    B, L, T = case["batch"], case["tokens"], case["keys"]
    H, K, d = case["heads"], case["kv_heads"], case["dim"]
    q = _randn(g, B, L, H, d).to(BF16)
    # the fused projection of the encoder's states: the heads of k and of v
    # side by side; keys have a few strong channels
    chan = torch.ones((2 * K, d), device="cuda")
    chan[:K] = torch.where(torch.rand((K, d), generator=g, device="cuda")
                           < 0.03, 3.0, 1.0)
    kv = (_randn(g, B, T, 2 * K, d) * chan).to(BF16)
    lens = None
    if case["ragged"]:
        # prompts of all lengths; a stream without a prompt has none
        lens = torch.randint(0, T + 1, (B,), generator=g, device="cuda")
        lens = lens.to(torch.int32)
    do = (_randn(g, B, L, H, d) * 0.1).to(BF16) if case["grad"] else None
    return q, kv, lens, do


def _ffn_inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    M, D, F = case["tokens"], case["dim"], case["hidden"]
    x = _randn(g, M, D).to(BF16)
    # the gate's weights are the larger ones: its unit saturates at times
    wg = (_randn(g, F, D) * (1.5 / math.sqrt(D))).to(BF16)
    wu = (_randn(g, F, D) / math.sqrt(D)).to(BF16)
    dh = (_randn(g, M, F) * 0.1).to(BF16) if case["grad"] else None
    return x, wg, wu, dh


def prepare(case, seed):
    if own:
        from paper_2609_36757_gb300 import fastvr as FV
    s = dict(case=case)
    if case["op"] == "cross":
        s["q"], s["kv"], s["lens"], s["do"] = _cross_inputs(case, seed)
        if own:
            s["plan"] = FV.make_cross_config()
    else:
        s["x"], s["wg"], s["wu"], s["dh"] = _ffn_inputs(case, seed)
        if own:
            s["plan"] = FV.make_ffn_config(case["act"])
    return s


# --------------------------------------------------------------- plain forms
def _cross_plain(case, q, kv, lens, do):
    B, L, H, d = q.shape
    K, T = case["kv_heads"], case["keys"]
    G, scale = H // K, d ** -0.5
    out = torch.zeros_like(q)
    lse = torch.full((B, H, L), -math.inf, device="cuda")
    if case["grad"]:
        dq = torch.zeros_like(q)
        dk, dv = (torch.zeros((B, T, K, d), dtype=BF16, device="cuda")
                  for _ in range(2))
    step = max(1, (1 << 28) // (G * L * max(T, d)))  # key heads at once
    col = torch.arange(T, device="cuda")
    for b in range(B):
        for h in range(0, K, step):
            j = min(K, h + step) - h
            rows = lambda t: t[b, :, h * G:(h + j) * G].float().transpose(
                0, 1).reshape(j, G * L, d)
            back = lambda t: t.view(j * G, L, d).transpose(0, 1).to(BF16)
            k = kv[b, :, h:h + j].float().transpose(0, 1)
            v = kv[b, :, K + h:K + h + j].float().transpose(0, 1)
            x = rows(q) @ k.transpose(1, 2) * scale
            if lens is not None:
                x = x.masked_fill(col >= lens[b], -math.inf)
            top = x.amax(-1, keepdim=True)
            top = torch.where(top == -math.inf, 0.0, top)
            p = torch.exp(x - top)
            z = p.sum(-1, keepdim=True)
            p = p / torch.where(z == 0, 1.0, z)
            o = p @ v
            hs = slice(h * G, (h + j) * G)
            out[b, :, hs] = back(o)
            lse[b, hs] = (top + torch.log(z)).view(j * G, L)
            if case["grad"]:
                g = rows(do)
                dp = g @ v.transpose(1, 2)
                ds = p * (dp - (g * o).sum(-1, keepdim=True)) * scale
                dq[b, :, hs] = back(ds @ k)
                dk[b, :, h:h + j] = (ds.transpose(1, 2) @ rows(q)).transpose(
                    0, 1).to(BF16)
                dv[b, :, h:h + j] = (p.transpose(1, 2) @ g).transpose(
                    0, 1).to(BF16)
    return (out, lse, dq, dk, dv) if case["grad"] else (out, lse)


_TANH_A, _TANH_B = math.sqrt(2 / math.pi), 0.044715


def _act_plain(g, kind):
    """act(g) and its derivative."""
    if kind == "silu":
        s = 1 / (1 + torch.exp(-g))
        return g * s, s * (1 + g * (1 - s))
    if kind == "gelu":
        c = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
        return g * c, c + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
    t = torch.tanh(_TANH_A * (g + _TANH_B * g ** 3))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * _TANH_A \
        * (1 + 3 * _TANH_B * g * g)


def _ffn_plain(case, x, wg, wu, dh):
    x, wg, wu = x.float(), wg.float(), wu.float()
    g, u = x @ wg.T, x @ wu.T
    a, slope = _act_plain(g, case["act"])
    h = (a * u).to(BF16)
    if not case["grad"]:
        return h
    dh = dh.float()
    dg, du = dh * u * slope, dh * a
    dx = dg @ wg + du @ wu
    return h, dx.to(BF16), (dg.T @ x).to(BF16), (du.T @ x).to(BF16)


# ---------------------------------------------------------------------- runs
def run(state):
    case = state["case"]
    if case["op"] == "cross":
        q, kv, lens, do = (state[n] for n in ("q", "kv", "lens", "do"))
        if not own:
            return _cross_plain(case, q, kv, lens, do)
        from paper_2609_36757_gb300 import fastvr as FV
        K, plan = case["kv_heads"], state["plan"]
        k, v = kv[:, :, :K], kv[:, :, K:]
        out, lse = FV.cross_attention(plan, q, k, v, lens, want_lse=True)
        if not case["grad"]:
            return out, lse
        return (out, lse) + tuple(FV.cross_attention_bwd(
            plan, q, k, v, out, do, lse, lens))
    x, wg, wu, dh = (state[n] for n in ("x", "wg", "wu", "dh"))
    if not own:
        return _ffn_plain(case, x, wg, wu, dh)
    from paper_2609_36757_gb300 import fastvr as FV
    if not case["grad"]:
        return FV.gated_ffn(state["plan"], x, wg, wu)
    h, saved = FV.gated_ffn(state["plan"], x, wg, wu, want_saved=True)
    return (h,) + tuple(FV.gated_ffn_bwd(state["plan"], dh, x, wg, wu, saved))


# ---------------------------------------------------------------------- work
def work(case):
    if case["op"] == "cross":
        part = 0.5 if case["ragged"] else 1.0  # prompts are half as long
        n = case["batch"] * case["tokens"] * case["heads"] * case["dim"]
        kv = 2 * case["batch"] * case["keys"] * case["kv_heads"] * case["dim"]
        lse = case["batch"] * case["tokens"] * case["heads"] * 4
        if case["grad"]:  # q, do, out, dq; k, v, dk, dv
            return dict(bytes=8 * n + int(2 * (1 + part) * kv) + lse,
                        flops=int(14 * part * n * case["keys"]))
        return dict(bytes=4 * n + int(2 * part * kv) + lse,
                    flops=int(4 * part * n * case["keys"]))
    M, D, F = case["tokens"], case["dim"], case["hidden"]
    if case["grad"]:  # x, dx; dh, h; both weights and their gradients
        return dict(bytes=2 * (2 * M * D + 2 * M * F + 4 * D * F),
                    flops=12 * M * D * F)
    return dict(bytes=2 * (M * D + M * F + 2 * D * F), flops=4 * M * D * F)


# ------------------------------------------------- the definition in 64 bits
def _cross_exact(case, seed):
    q, kv, lens, do = _cross_inputs(case, seed)
    B, L, H, d = q.shape
    K, T = case["kv_heads"], case["keys"]
    # about 1 TFLOP/s in 64 bits
    if (14.0 if case["grad"] else 4.0) * B * H * L * T * d > 1.2e13:
        return None
    f64 = dict(dtype=torch.float64, device="cuda")
    out, lse = torch.zeros((B, L, H, d), **f64), torch.empty((B, H, L), **f64)
    dq = torch.zeros((B, L, H, d), **f64)
    dk, dv = (torch.zeros((B, T, K, d), **f64) for _ in range(2))
    for b in range(B):
        n = T if lens is None else int(lens[b])
        for h in range(H):
            if n == 0:
                lse[b, h] = -math.inf
                continue
            i = h // (H // K)
            leaf = [t.double().requires_grad_(case["grad"]) for t in
                    (q[b, :, h], kv[b, :n, i], kv[b, :n, K + i])]
            score = torch.einsum("ld,td->lt", leaf[0], leaf[1]) / math.sqrt(d)
            o = torch.softmax(score, -1) @ leaf[2]
            out[b, :, h] = o.detach()
            lse[b, h] = torch.logsumexp(score.detach(), -1)
            if case["grad"]:
                grads = torch.autograd.grad(o, leaf, do[b, :, h].double())
                dq[b, :, h] = grads[0]
                dk[b, :n, i] += grads[1]
                dv[b, :n, i] += grads[2]
    return (out, lse, dq, dk, dv) if case["grad"] else (out, lse)


def _ffn_exact(case, seed):
    x, wg, wu, dh = _ffn_inputs(case, seed)
    leaf = [t.double().requires_grad_(case["grad"]) for t in (x, wg, wu)]
    gate = torch.einsum("md,fd->mf", leaf[0], leaf[1])
    up = torch.einsum("md,fd->mf", leaf[0], leaf[2])
    f = torch.nn.functional
    act = f.silu(gate) if case["act"] == "silu" else f.gelu(
        gate, approximate="tanh" if case["act"] == "gelu_tanh" else "none")
    h = act * up
    if not case["grad"]:
        return h
    return (h.detach(),) + torch.autograd.grad(h, leaf, dh.double())


def exact(case, seed):
    return _cross_exact(case, seed) if case["op"] == "cross" else \
        _ffn_exact(case, seed)
