"""CPU tests of the block operators' C ABI: every refusal happens on the host
before any device work, and the 4-bit plan's sizes and sequencing."""
import ctypes

import pytest

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


ROT_ARGS = dict(batch=1, tokens=4, heads=2, kv_heads=2, dtype=0, q=FAKE,
                q_str=None, k=FAKE, k_str=None, positions=FAKE, pos_batch=0,
                q_out=FAKE, q_out_str=None, k_out=FAKE, k_out_str=None,
                transpose=0, stream=0)


@pytest.mark.parametrize("kw", [
    dict(batch=0), dict(tokens=0), dict(heads=0), dict(kv_heads=-1),
    dict(dtype=2), dict(q=0), dict(q=FAKE + 8), dict(k=FAKE + 2),
    dict(q_out=0), dict(q_out=FAKE + 4), dict(k_out=0), dict(k=0),
    dict(kv_heads=0), dict(positions=0), dict(positions=FAKE + 2),
    dict(batch=1 << 20, tokens=1 << 20), dict(heads=1 << 24),
])
def test_rotary_refuses(fv, kw):
    cfg = fv.make_rotary_config(64)
    _refused(fv, fv.FASTVR_ERR_INVALID_ARG, fv.fastvr_rotary, cfg,
             **{**ROT_ARGS, **kw})


def test_rotary_refuses_unaligned_strides(fv):
    cfg = fv.make_rotary_config(64)
    bad = fv.fastvr_strides_t(4 * 128, 132, 64)
    for name in ("q_str", "k_str", "q_out_str", "k_out_str"):
        _refused(fv, fv.FASTVR_ERR_INVALID_ARG, fv.fastvr_rotary, cfg,
                 **{**ROT_ARGS, name: bad})
    # outputs with several tokens (or heads) in one place
    for bad in (fv.fastvr_strides_t(512, 0, 64),
                fv.fastvr_strides_t(512, 128, 0)):
        for name in ("q_out_str", "k_out_str"):
            _refused(fv, fv.FASTVR_ERR_INVALID_ARG, fv.fastvr_rotary, cfg,
                     **{**ROT_ARGS, name: bad})


@pytest.mark.parametrize("kw", [
    dict(head_dim=60), dict(head_dim=520), dict(rotary_dim=66),
    dict(rotary_dim=0), dict(rotary_dim=31), dict(sections=[16, 8]),
    dict(sections=[32, 0]), dict(base=1.0), dict(base=float("nan")),
    dict(magnitude=-1.0), dict(scaling="linear", factors=[0.5]),
    dict(scaling="ntk", factors=[float("inf")]),
    dict(scaling="yarn", factors=[2.0]),
    dict(scaling="yarn", factors=[2.0], original_contexts=[10],
         beta_fast=1.0),
])
def test_rotary_config_refused(fv, kw):
    cfg = fv.make_rotary_config(**{**dict(head_dim=64), **kw})
    _refused(fv, fv.FASTVR_ERR_INVALID_ARG, fv.fastvr_rotary_frequencies, cfg)
    _refused(fv, fv.FASTVR_ERR_INVALID_ARG, fv.fastvr_rotary, cfg, **ROT_ARGS)


def _norm_cfg(fv, **kw):
    cfg = fv.make_norm_config(pre="layer", post="rms")
    for k, v in {**dict(batch=2, tokens=6, dim=64, groups=3), **kw}.items():
        setattr(cfg, k, v)
    return cfg


@pytest.mark.parametrize("kw", [
    dict(batch=0), dict(tokens=0), dict(dim=60), dict(dim=0), dict(dim=8200),
    dict(groups=0), dict(groups=4), dict(groups=7), dict(pre=0), dict(pre=3),
    dict(post=-1), dict(residual_dtype=2), dict(block_dtype=-1),
    dict(eps=0.0), dict(eps=float("nan")), dict(residual_scale=float("inf")),
    dict(batch=1 << 15, tokens=3 << 14),
])
def test_norm_config_refused(fv, kw):
    cfg = _norm_cfg(fv, **kw)
    _refused(fv, 1, fv.fastvr_gated_norm_fwd, cfg, *[FAKE] * 9, 0)
    _refused(fv, 1, fv.fastvr_gated_norm_bwd_scratch_bytes, cfg)
    _refused(fv, 1, fv.fastvr_gated_norm_bwd, cfg, *[FAKE] * 16, 1 << 40, 0)


def test_norm_arguments_refused(fv):
    cfg = _norm_cfg(fv)
    fwd = [FAKE] * 9
    for i, v in [(0, 0), (0, FAKE + 8), (1, FAKE + 2), (2, FAKE + 4),
                 (8, FAKE + 8)]:
        a = list(fwd)
        a[i] = v
        _refused(fv, 1, fv.fastvr_gated_norm_fwd, cfg, *a, 0)
    _refused(fv, 1, fv.fastvr_gated_norm_fwd, cfg, *fwd[:7], 0, 0, 0)
    need = fv.fastvr_gated_norm_bwd_scratch_bytes(cfg)
    bwd = [FAKE] * 16   # dr dh r y gate scale pw qw dx dy dg ds dt dw dv scratch
    for i, v in [(2, 0), (8, 0), (9, 0), (3, 0), (15, 0), (10, FAKE + 4),
                 (15, FAKE + 8)]:
        a = list(bwd)
        a[i] = v
        _refused(fv, 1, fv.fastvr_gated_norm_bwd, cfg, *a, need, 0)
    a = [0, 0] + bwd[2:]
    _refused(fv, 1, fv.fastvr_gated_norm_bwd, cfg, *a, need, 0)
    _refused(fv, fv.FASTVR_ERR_CAPACITY, fv.fastvr_gated_norm_bwd, cfg, *bwd,
             need - 1, 0)


def _q4_cfg(fv, **kw):
    base = dict(batch=1, heads=4, head_dim=64, tokens_per_frame=4,
                frames_per_chunk=2, window_chunks=2, max_chunks=0)
    return fv.make_config(**{**base, **kw})


def _q4_plan(fv, kv_heads=2, **kw):
    cfg = _q4_cfg(fv, **kw)
    return cfg, fv.fastvr_q4_plan(
        cfg, kv_heads, FAKE, fv.fastvr_q4_cache_bytes(cfg, kv_heads), FAKE,
        fv.fastvr_q4_workspace_bytes(cfg, kv_heads))


@pytest.mark.parametrize("kv,kw,code", [
    (2, dict(batch=0), 1), (3, {}, 1), (0, {}, 1), (-2, {}, 1), (8, {}, 1),
    (2, dict(head_dim=96), 2), (2, dict(window_chunks=-1), 1),
    (2, dict(softmax_scale=-1.0), 1),
    # more tokens than 32-bit indices hold
    (2, dict(tokens_per_frame=1 << 29), 1),
    (2, dict(window_chunks=2147483646, tokens_per_frame=2147483647,
             frames_per_chunk=2147483647), 1),
])
def test_q4_config_refused(fv, kv, kw, code):
    cfg = _q4_cfg(fv, **kw)
    _refused(fv, code, fv.fastvr_q4_cache_bytes, cfg, kv)
    _refused(fv, code, fv.fastvr_q4_workspace_bytes, cfg, kv)
    _refused(fv, code, fv.fastvr_q4_plan, cfg, kv, FAKE, 1 << 60, FAKE,
             1 << 60)


def test_q4_cache_is_a_quarter(fv):
    # 8160-token frames: the control block is a vanishing part
    cfg = _q4_cfg(fv, head_dim=128, tokens_per_frame=8160)
    values = 2 * 4 * 128 * 3 * 2 * 8160
    n = fv.fastvr_q4_cache_bytes(cfg, 4)
    assert values * 9 // 16 <= n <= values * 9 // 16 + 8192


def test_q4_plan_refuses_buffers(fv):
    cfg = _q4_cfg(fv)
    c, w = (f(cfg, 2) for f in (fv.fastvr_q4_cache_bytes,
                                fv.fastvr_q4_workspace_bytes))
    for a in [(0, c, FAKE, w), (FAKE + 16, c, FAKE, w), (FAKE, c, 0, w),
              (FAKE, c, FAKE + 128, w)]:
        _refused(fv, 1, fv.fastvr_q4_plan, cfg, 2, *a)
    for a in [(FAKE, c - 1, FAKE, w), (FAKE, c, FAKE, w - 1)]:
        _refused(fv, fv.FASTVR_ERR_CAPACITY, fv.fastvr_q4_plan, cfg, 2, *a)


def test_q4_sequencing(fv):
    CAP, SEQ, ARG = (fv.FASTVR_ERR_CAPACITY, fv.FASTVR_ERR_SEQUENCE,
                     fv.FASTVR_ERR_INVALID_ARG)
    cfg, plan = _q4_plan(fv)
    app = lambda frames, k=FAKE, v=FAKE, s=None: fv.fastvr_q4_append(
        plan, k, s, v, None, frames, 0)
    try:
        _refused(fv, SEQ, fv.fastvr_q4_attn_fwd, plan, FAKE, 0, FAKE + 4096, 0,
                 0)
        _refused(fv, SEQ, fv.fastvr_q4_read, plan, 0, FAKE, FAKE, 0)
        _refused(fv, ARG, app, 0)
        _refused(fv, CAP, app, 3)        # neither <= k nor a multiple
        _refused(fv, CAP, app, 8)        # four chunks, three slots
        _refused(fv, ARG, app, 2, k=FAKE + 8)
        _refused(fv, ARG, app, 2, v=0)
        _refused(fv, ARG, app, 2, s=fv.fastvr_strides_t(0, 68, 64))
        fv.fastvr_plan_set_state(plan, 5, 1)
        _refused(fv, SEQ, app, 2)        # after a ragged chunk
        _refused(fv, SEQ, fv.fastvr_q4_read, plan, 1, FAKE, FAKE, 0)
        _refused(fv, SEQ, fv.fastvr_q4_read, plan, 5, FAKE, FAKE, 0)
        OUT = FAKE + 4096
        for a in [(0, 0, OUT, 0), (FAKE + 8, 0, OUT, 0), (FAKE, 2, OUT, 0),
                  (FAKE, 0, 0, 0), (FAKE, 0, OUT, 2), (FAKE, 0, FAKE, 0)]:
            _refused(fv, ARG, fv.fastvr_q4_attn_fwd, plan, *a, 0)
        # the bfloat16 calls and the 4-bit ones do not take each other's plans
        _refused(fv, ARG, fv.fastvr_kv_append, plan, FAKE, FAKE, 1, 0)
        _refused(fv, ARG, fv.fastvr_chunk_attn_fwd, plan, FAKE, FAKE, 0, 0)
        bf = fv.fastvr_attn_plan(cfg, FAKE, fv.fastvr_kv_cache_bytes(cfg))
        _refused(fv, ARG, fv.fastvr_q4_append, bf, FAKE, None, FAKE, None, 1, 0)
        _refused(fv, ARG, fv.fastvr_q4_attn_fwd, bf, FAKE, 0, FAKE + 4096, 0, 0)
        _refused(fv, ARG, fv.fastvr_q4_read, bf, 0, FAKE, FAKE, 0)
        fv.fastvr_plan_destroy(bf)
        # the shared calls do take it
        fv.fastvr_plan_set_state(plan, 4, 2)
        assert fv.fastvr_plan_visible(plan)[1] == 3 * 2 * 4
        fv.fastvr_plan_reset(plan)
        assert fv.fastvr_plan_get_state(plan) == (0, 0)
    finally:
        fv.fastvr_plan_destroy(plan)
    _, plan = _q4_plan(fv, window_chunks=-1, max_chunks=3)
    try:
        fv.fastvr_plan_set_state(plan, 2, 2)
        _refused(fv, CAP, fv.fastvr_q4_append, plan, FAKE, None, FAKE, None,
                 4, 0)                   # two more chunks, room for one
    finally:
        fv.fastvr_plan_destroy(plan)


def test_device_calls_fail_without_a_gpu(fv):
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    no_gpu = (fv.FASTVR_ERR_CUDA, fv.FASTVR_ERR_UNSUPPORTED)
    _, plan = _q4_plan(fv)
    ncfg = _norm_cfg(fv)
    calls = [
        lambda: fv.fastvr_rotary(fv.make_rotary_config(64), **ROT_ARGS),
        lambda: fv.fastvr_gated_norm_fwd(ncfg, *[FAKE] * 9, 0),
        lambda: fv.fastvr_gated_norm_bwd(ncfg, *[FAKE] * 16, 1 << 30, 0),
        lambda: fv.fastvr_q4_append(plan, FAKE, None, FAKE, None, 2, 0),
    ]
    try:
        for call in calls:
            with pytest.raises(fv.FastVRError) as e:
                call()
            assert e.value.status in no_gpu
        assert fv.fastvr_plan_get_state(plan) == (0, 0)
    finally:
        fv.fastvr_plan_destroy(plan)


def test_struct_sizes_match_the_header(fv):
    assert ctypes.sizeof(fv.fastvr_strides_t) == 24
    assert ctypes.sizeof(fv.fastvr_rotary_config_t) == 112
    assert ctypes.sizeof(fv.fastvr_norm_config_t) == 40
