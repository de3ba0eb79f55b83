"""Cross attention and the gated feed-forward on the CPU: every refusal happens
on the host before any device work, and the bindings' checks of tensors."""
import ctypes

import pytest
import torch

FAKE = 1 << 40  # a 256-aligned address that no call reaches


@pytest.fixture(scope="module")
def fv():
    from paper_2609_36757_gb300 import build
    build.build()
    from paper_2609_36757_gb300 import fastvr
    return fastvr


def _refused(fv, code, f, *a, **kw):
    with pytest.raises(fv.FastVRError) as e:
        f(*a, **kw)
    assert e.value.status == code, (e.value, a, kw)


def _at(i):
    return FAKE + (i << 32)


def _cross(fv, **kw):
    c = fv.make_cross_config()
    for n, x in {**dict(batch=2, q_tokens=5, kv_tokens=7, heads=4, kv_heads=2,
                        head_dim=64), **kw}.items():
        setattr(c, n, x)
    return c


FWD = dict(q=_at(0), q_str=None, k=_at(1), k_str=None, v=_at(2), v_str=None,
           kv_len=_at(3), out=_at(4), out_str=None, lse=_at(5), stream=0)
BWD = dict(q=_at(0), q_str=None, k=_at(1), k_str=None, v=_at(2), v_str=None,
           kv_len=_at(3), out=_at(4), out_str=None, dout=_at(6),
           dout_str=None, lse=_at(5), dq=_at(7), dq_str=None, dk=_at(8),
           dk_str=None, dv=_at(9), dv_str=None, scratch=_at(10),
           scratch_bytes=1 << 30, stream=0)


@pytest.mark.parametrize("kw", [
    dict(batch=0), dict(q_tokens=0), dict(kv_tokens=0), dict(heads=0),
    dict(kv_heads=0), dict(kv_heads=3), dict(head_dim=0),
    dict(softmax_scale=-1.0), dict(softmax_scale=float("nan")),
    dict(softmax_scale=float("inf")), dict(q_tokens=1 << 30),
    dict(kv_tokens=1 << 30), dict(batch=1 << 20, heads=1 << 12),
    dict(batch=1 << 20, heads=1 << 8, q_tokens=257),
])
def test_cross_config_refused(fv, kw):
    c = _cross(fv, **kw)
    bad = fv.FASTVR_ERR_INVALID_ARG
    _refused(fv, bad, fv.fastvr_cross_attn_fwd, c, **FWD)
    _refused(fv, bad, fv.fastvr_cross_attn_bwd, c, **BWD)
    _refused(fv, bad, fv.fastvr_cross_attn_bwd_scratch_bytes, c)


@pytest.mark.parametrize("d", [8, 32, 96, 256])
def test_cross_head_dim_unsupported(fv, d):
    c = _cross(fv, head_dim=d)
    _refused(fv, fv.FASTVR_ERR_UNSUPPORTED, fv.fastvr_cross_attn_fwd, c, **FWD)
    _refused(fv, fv.FASTVR_ERR_UNSUPPORTED, fv.fastvr_cross_attn_bwd, c, **BWD)


@pytest.mark.parametrize("kw", [
    dict(q=0), dict(k=0), dict(v=0), dict(out=0), dict(q=FAKE + 8),
    dict(k=FAKE + 2), dict(v=FAKE + 4), dict(out=FAKE + 8),
    dict(kv_len=FAKE + 2), dict(lse=FAKE + 1), dict(out=FWD["q"]),
    dict(out=FWD["k"]), dict(out=FWD["v"]),
])
def test_cross_fwd_refuses(fv, kw):
    _refused(fv, fv.FASTVR_ERR_INVALID_ARG, fv.fastvr_cross_attn_fwd,
             _cross(fv), **{**FWD, **kw})


@pytest.mark.parametrize("kw", [
    *(dict([(n, 0)]) for n in ("q", "k", "v", "out", "dout", "lse", "dq",
                               "dk", "dv", "scratch")),
    *(dict([(n, FAKE + 8)]) for n in ("q", "k", "v", "out", "dout", "dq",
                                      "dk", "dv", "scratch")),
    dict(kv_len=FAKE + 2), dict(lse=FAKE + 2), dict(dq=BWD["q"]),
    dict(dk=BWD["k"]), dict(dv=BWD["dout"]), dict(dk=BWD["dv"]),
    dict(dq=BWD["dk"]), dict(scratch=BWD["q"]),
])
def test_cross_bwd_refuses(fv, kw):
    _refused(fv, fv.FASTVR_ERR_INVALID_ARG, fv.fastvr_cross_attn_bwd,
             _cross(fv), **{**BWD, **kw})


def test_cross_strides(fv):
    S, c, bad = fv.fastvr_strides_t, _cross(fv), fv.FASTVR_ERR_INVALID_ARG
    for s in (S(4096, 260, 64), S(4096, 256, 68), S(4100, 256, 64),
              S(4096, 0, 64), S(4096, 256, 0), S(-4096, 256, 64),
              S(4096, 1 << 39, 64)):
        for n in ("q_str", "k_str", "v_str", "out_str"):
            _refused(fv, bad, fv.fastvr_cross_attn_fwd, c, **{**FWD, n: s})
        for n in ("q_str", "k_str", "v_str", "out_str", "dout_str", "dq_str",
                  "dk_str", "dv_str"):
            _refused(fv, bad, fv.fastvr_cross_attn_bwd, c, **{**BWD, n: s})
    # one place for several batch entries: inputs only
    s = S(0, 256, 64)
    _refused(fv, bad, fv.fastvr_cross_attn_fwd, c, **{**FWD, "out_str": s})
    for n in ("dq_str", "dk_str", "dv_str"):
        _refused(fv, bad, fv.fastvr_cross_attn_bwd, c, **{**BWD, n: s})


def test_cross_scratch(fv):
    c = _cross(fv)
    n = fv.fastvr_cross_attn_bwd_scratch_bytes(c)
    assert n >= 2 * 4 * 5 * 4
    _refused(fv, fv.FASTVR_ERR_CAPACITY, fv.fastvr_cross_attn_bwd, c,
             **{**BWD, "scratch_bytes": n - 1})


def test_cross_scratch_on_16_bytes_has_room_for_parts_on_32(fv):
    """Scratch lies on 16 bytes; partial sums are written 32 bytes at a time."""
    c = fv.fastvr_cross_config_t(1, 700, 640, 3, 3, 128, 0.0)
    rows = 2 * 3 * 768 * 4
    n = fv.fastvr_cross_attn_bwd_scratch_bytes(c)
    assert n > rows and (n - rows) % 32 == 16


def _ffn(fv, **kw):
    c = fv.make_ffn_config("gelu")
    for n, x in {**dict(tokens=5, dim=16, hidden=24), **kw}.items():
        setattr(c, n, x)
    return c


FFN = dict(x=_at(0), x_row=0, w_gate=_at(1), w_up=_at(2), h=_at(3), g=_at(4),
           u=_at(5), stream=0)
FFB = dict(dh=_at(6), x=_at(0), x_row=0, w_gate=_at(1), w_up=_at(2), g=_at(4),
           u=_at(5), dx=_at(7), dw_gate=_at(8), dw_up=_at(9), scratch=_at(10),
           scratch_bytes=1 << 20, stream=0)


@pytest.mark.parametrize("kw", [
    dict(tokens=0), dict(tokens=(1 << 28) + 1), dict(tokens=1 << 30),
    dict(tokens=1 << 28, dim=65536, hidden=131072), dict(dim=0), dict(dim=12),
    dict(dim=65544), dict(hidden=0), dict(hidden=20), dict(hidden=262152),
    dict(activation=-1), dict(activation=3),
])
def test_ffn_config_refused(fv, kw):
    c, bad = _ffn(fv, **kw), fv.FASTVR_ERR_INVALID_ARG
    _refused(fv, bad, fv.fastvr_gated_ffn_fwd, c, **FFN)
    _refused(fv, bad, fv.fastvr_gated_ffn_bwd, c, **FFB)
    _refused(fv, bad, fv.fastvr_gated_ffn_bwd_scratch_bytes, c)


@pytest.mark.parametrize("kw", [
    *(dict([(n, 0)]) for n in ("x", "w_gate", "w_up", "h", "g", "u")),
    *(dict([(n, FAKE + 8)]) for n in ("x", "w_gate", "w_up", "h", "g", "u")),
    dict(x_row=8), dict(x_row=20), dict(x_row=-16), dict(x_row=1 << 39),
    dict(h=FFN["x"]), dict(h=FFN["g"]), dict(g=FFN["u"]), dict(u=FFN["x"]),
    dict(h=FFN["w_up"]),
])
def test_ffn_fwd_refuses(fv, kw):
    _refused(fv, fv.FASTVR_ERR_INVALID_ARG, fv.fastvr_gated_ffn_fwd, _ffn(fv),
             **{**FFN, **kw})


@pytest.mark.parametrize("kw", [
    *(dict([(n, 0)]) for n in ("dh", "x", "w_gate", "w_up", "g", "u", "dx",
                               "dw_gate", "dw_up", "scratch")),
    *(dict([(n, FAKE + 8)]) for n in ("dh", "x", "w_gate", "w_up", "g", "u",
                                      "dx", "dw_gate", "dw_up", "scratch")),
    dict(x_row=8), dict(dx=FFB["x"]), dict(dx=FFB["dh"]), dict(dw_up=FFB["g"]),
    dict(dw_gate=FFB["dw_up"]), dict(scratch=FFB["g"]),
    dict(dx=FFB["scratch"]),
])
def test_ffn_bwd_refuses(fv, kw):
    _refused(fv, fv.FASTVR_ERR_INVALID_ARG, fv.fastvr_gated_ffn_bwd, _ffn(fv),
             **{**FFB, **kw})


def test_ffn_scratch(fv):
    c = _ffn(fv)
    n = fv.fastvr_gated_ffn_bwd_scratch_bytes(c)
    assert n >= 2 * 2 * 5 * 24
    _refused(fv, fv.FASTVR_ERR_CAPACITY, fv.fastvr_gated_ffn_bwd, c,
             **{**FFB, "scratch_bytes": n - 1})


def test_struct_sizes_match_the_header(fv):
    assert ctypes.sizeof(fv.fastvr_cross_config_t) == 28
    assert ctypes.sizeof(fv.fastvr_ffn_config_t) == 16


# The bindings refuse tensors by type and shape before anything else, and host
# tensors before the library is called.
BF = torch.bfloat16


def _qkv(q=(2, 5, 4, 64), kv=(2, 7, 2, 64), dtype=BF):
    return (torch.zeros(q, dtype=dtype), torch.zeros(kv, dtype=dtype),
            torch.zeros(kv, dtype=dtype))


@pytest.mark.parametrize("change", [
    lambda q, k, v: (q.float(), k, v),
    lambda q, k, v: (q, k, v.float()),
    lambda q, k, v: (q[0], k, v),
    lambda q, k, v: (q, k, v[:, :6]),
    lambda q, k, v: (q, k[:1], v[:1]),
    lambda q, k, v: (q[..., :32], k, v),
    lambda q, k, v: (q.transpose(2, 3), k, v),
    lambda q, k, v: (q, k.transpose(1, 3), v),
])
def test_cross_tensors_refused(fv, change):
    q, k, v = change(*_qkv())
    with pytest.raises(ValueError):
        fv.cross_attention(fv.make_cross_config(), q, k, v)


@pytest.mark.parametrize("kv_len", [
    torch.zeros(2, dtype=torch.int64), torch.zeros(3, dtype=torch.int32),
    torch.zeros(4, dtype=torch.int32)[::2],
    torch.zeros((2, 1), dtype=torch.int32),
])
def test_cross_kv_len_refused(fv, kv_len):
    with pytest.raises(ValueError):
        fv.cross_attention(fv.make_cross_config(), *_qkv(), kv_len)


def test_cross_bwd_tensors_refused(fv):
    q, k, v = _qkv()
    lse = torch.zeros((2, 4, 5))
    for out, dout, row in ((q.float(), q, lse), (q, q[:, :4], lse),
                           (q, q, lse.double()), (q, q, lse[:, :3]),
                           (q, q.transpose(2, 3), lse)):
        with pytest.raises(ValueError):
            fv.cross_attention_bwd(fv.make_cross_config(), q, k, v, out, dout,
                                   row)


def test_host_tensors_refused(fv, monkeypatch):
    fv._setup()
    monkeypatch.setattr(fv, "_current_device", lambda: 0)
    q, k, v = _qkv()
    with pytest.raises(ValueError):
        fv.cross_attention(fv.make_cross_config(), q, k, v)
    x, w = torch.zeros((5, 16), dtype=BF), torch.zeros((24, 16), dtype=BF)
    with pytest.raises(ValueError):
        fv.gated_ffn(fv.make_ffn_config(), x, w, w.clone())


@pytest.mark.parametrize("change", [
    lambda x, g, u: (x.float(), g, u),
    lambda x, g, u: (x, g.float(), u),
    lambda x, g, u: (x[..., :8], g, u),
    lambda x, g, u: (x, g, u[:16]),
    lambda x, g, u: (x, g.T.contiguous().T, u),
    lambda x, g, u: (x[:, :, ::2], g[:, ::2], u[:, ::2]),
    lambda x, g, u: (x[:, :3].transpose(0, 1), g, u),
    lambda x, g, u: (x[0, :1].expand(5, 16), g, u),
    lambda x, g, u: (x, g[None], u[None]),
])
def test_ffn_tensors_refused(fv, change):
    x, g, u = change(torch.zeros((2, 5, 16), dtype=BF),
                     *torch.zeros((2, 24, 16), dtype=BF))
    with pytest.raises(ValueError):
        fv.gated_ffn(fv.make_ffn_config(), x, g, u)


def test_ffn_activation_names(fv):
    with pytest.raises(KeyError):
        fv.make_ffn_config("relu")
    assert [fv.make_ffn_config(n).activation
            for n in ("silu", "gelu", "gelu_tanh")] == [0, 1, 2]


@pytest.mark.parametrize("at", ["B", "T", "L"])
def test_cross_sizes_past_32_bits_are_refused(fv, at):
    """ctypes would cut a size to its low 32 bits: 2^32 + 2 must not pass for 2."""
    n = {"B": 1, "L": 2, "T": 3, at: 2 ** 32 + 2}
    q = torch.empty(n["B"], n["L"], 1, 64, dtype=torch.bfloat16, device="meta")
    k = torch.empty(n["B"], n["T"], 1, 64, dtype=torch.bfloat16, device="meta")
    with pytest.raises(ValueError, match="2\\^31"):
        fv._cross_call(fv.make_cross_config(), q, k, k, None)


@pytest.mark.parametrize("tokens,hidden,dim", [
    (2 ** 32 + 5, 8, 8), (5, 2 ** 32 + 8, 8), (5, 8, 2 ** 32 + 8),
    (2 ** 31, 8, 8)])
def test_ffn_sizes_past_32_bits_are_refused(fv, tokens, hidden, dim):
    x = torch.empty(tokens, dim, dtype=torch.bfloat16, device="meta")
    w = torch.empty(hidden, dim, dtype=torch.bfloat16, device="meta")
    with pytest.raises(ValueError, match="2\\^31"):
        fv._ffn_call(fv.make_ffn_config(), x, w, w, ())


@pytest.mark.parametrize("kw", [
    dict(scratch=BWD["dq"]), dict(scratch=BWD["dk"]), dict(scratch=BWD["dv"]),
    dict(scratch=BWD["lse"]), dict(scratch=BWD["dout"]), dict(lse=BWD["dk"])])
def test_cross_bwd_refuses_shared_scratch_and_lse(fv, kw):
    _refused(fv, fv.FASTVR_ERR_INVALID_ARG, fv.fastvr_cross_attn_bwd,
             _cross(fv), **{**BWD, **kw})


def test_cross_fwd_refuses_lse_in_out(fv):
    _refused(fv, fv.FASTVR_ERR_INVALID_ARG, fv.fastvr_cross_attn_fwd,
             _cross(fv), **{**FWD, "lse": FWD["out"]})
