"""The 4-bit cache and stream capture.  A plan's first call clears its control
block, whose counters the joins of split key ranges rely on, so it cannot be a
captured one: it is refused and changes nothing.  Afterwards a call may be
captured, and its replay equals the call."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _make(N, chunks, seed):
    from paper_2609_36757_gb300 import fastvr as FV
    g = torch.Generator("cuda").manual_seed(seed)
    rnd = lambda n: torch.randn(2, n, 4, 64, generator=g,
                                device="cuda").to(torch.bfloat16)
    att = FV.StreamingAttention4(FV.make_config(2, 4, 64, N, 1, chunks - 1))
    att.cache.fill_(0x5a)  # what the control block holds before it is cleared
    return FV, att, rnd(N), rnd(N * chunks), rnd(N * chunks)


def _capture(f):
    graph = torch.cuda.CUDAGraph()
    mark = torch.zeros(1, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        mark.add_(1)
        out = f()
    return graph, out


@pytest.mark.parametrize("N,chunks", [(1, 3000), (200, 12)])
def test_first_call_is_not_captured(N, chunks):
    FV, att, q, k, v = _make(N, chunks, 1)

    def refused():
        with pytest.raises(FV.FastVRError) as e:
            att.append(k, v)
        assert e.value.status == FV.FASTVR_ERR_SEQUENCE

    _capture(refused)
    assert att.state() == (0, 0) and att.launch_count() == 0
    # a resumed plan, whose first call is the attention or the read-back
    att.set_state(chunks, 1)

    def refused():
        for f in (lambda: att.forward(q), att.read):
            with pytest.raises(FV.FastVRError) as e:
                f()
            assert e.value.status == FV.FASTVR_ERR_SEQUENCE

    _capture(refused)
    assert att.launch_count() == 0
    # called outside, it works, as on a plan that saw no capture
    _, ref, *_ = _make(N, chunks, 1)
    outs = []
    for a in (att, ref):
        a.reset()
        a.append(k, v)
        outs.append((*a.forward(q, want_lse=True), *a.read()))
        assert a.status() == FV.FASTVR_OK
    assert torch.isfinite(outs[0][0]).all()
    assert all(torch.equal(a, b) for a, b in zip(*outs))


@pytest.mark.parametrize("N,chunks", [(1, 3000), (200, 12)])
def test_replay_equals_the_call(N, chunks):
    FV, att, q, k, v = _make(N, chunks, 2)
    att.append(k, v)
    ref = att.forward(q, want_lse=True)
    graph, got = _capture(lambda: att.forward(q, want_lse=True))
    for _ in range(3):
        for t in got:
            t.fill_(7)
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(got, ref))
    assert att.status() == FV.FASTVR_OK
