"""The workspace that a call without one allocates belongs to the stream that the call runs on."""
import contextlib

import numpy as np
import pytest


@pytest.mark.parametrize("named", [None, 7, 0, 1, 99])
def test_the_workspace_is_allocated_on_the_calls_stream(monkeypatch, named):
    """With the allocator and the streams replaced: which stream is current when the workspace is allocated."""
    import torch

    import paper_1808_07217_gb300 as L

    current, at, made, calls = [7], [], [], []

    @contextlib.contextmanager
    def stream(s):
        current.append(s)
        yield
        current.pop()

    class Block:
        def data_ptr(self):
            return 4096

        def record_stream(self, s):
            made.append(s)

    def empty(*args, **kw):
        at.append(current[-1])
        return Block()

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda ptr, device=None: ptr)
    monkeypatch.setattr(torch, "empty", empty)
    monkeypatch.setattr(L, "_stream_of", lambda dev: current[-1])

    def fn(*args):
        calls.append(args)
        return L.OK

    L._launch(0, named, None, 1 << 20, fn, (5,))
    st = 7 if named is None else named
    assert calls == [(5, 4096, 1 << 20, st)]
    assert at == [0 if st == 1 else st] and current == [7]


@pytest.fixture(scope="module")
def P():
    import torch

    from _gpu_common import built_package

    assert torch.cuda.is_available()
    return built_package()


def _calls(P):
    """(bytes of workspace, a call on `stream`, its outputs) for every operator that uses one."""
    import torch

    gen = torch.Generator(device="cuda").manual_seed(3)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    G, B, Pn, C, groups = shape = (1, 2, 13001, 168, 42)
    x, dy, gamma, beta = rand(G, B, Pn, C), rand(G, B, Pn, C), rand(G, C), rand(G, C)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    mean, rstd = torch.empty(G * B * groups, device="cuda"), torch.empty(G * B * groups, device="cuda")
    dgamma, dbeta = torch.empty_like(gamma), torch.empty_like(beta)
    u, g = torch.zeros(2, 300, 257, device="cuda"), rand(2, 300, 257)
    o = torch.empty(2, 300, 257, dtype=torch.bfloat16, device="cuda")
    forward = lambda **kw: P.lsgd_groupnorm_forward(x, gamma, beta, y, mean, rstd, *shape, **kw)  # noqa: E731
    forward()  # the statistics that the backward reads
    return [(P.lsgd_groupnorm_workspace(*shape), forward, [y, mean, rstd]),
            (P.lsgd_groupnorm_workspace(*shape, True),
             lambda **kw: P.lsgd_groupnorm_backward(x, None, dy, gamma, beta, mean, rstd, dx, dgamma, dbeta, *shape, **kw),
             [dx, dgamma, dbeta]),
            (P.lsgd_orthogonal_workspace(2, 300, 257),
             lambda **kw: P.lsgd_orthogonal_direction(u, g, o, 2, 300, 257, momentum=0.0, **kw), [o])]


@pytest.mark.gpu
@pytest.mark.parametrize("which", [0, 1, 2])
def test_work_queued_on_the_current_stream_keeps_a_deleted_tensor(P, which):
    """A tensor of the workspace's size is deleted while kernels that read and write it wait on the current stream: the call
    on another stream neither changes what they read nor finds its sums changed by them."""
    import torch

    nbytes, call, outs = _calls(P)[which]
    call()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    side = torch.cuda.Stream()
    for t in outs:
        t.zero_()
    for _ in range(3):
        tmp = torch.full((nbytes,), 3, dtype=torch.uint8, device="cuda")
        copy = torch.empty_like(tmp)
        torch.cuda.synchronize()
        torch.cuda._sleep(40_000_000)  # about 20 ms
        copy.copy_(tmp)
        for _ in range(20):
            tmp.add_(1)
        del tmp
        call(stream=side.cuda_stream)
        torch.cuda.synchronize()
        assert (copy == 3).all()
        for t, w in zip(outs, want):
            assert torch.equal(t, w)


@pytest.mark.gpu
def test_a_call_on_a_named_stream_joins_a_capture(P):
    """Its workspace comes from the graph's own memory then: replays do not meet what is allocated later."""
    import torch

    for nbytes, call, outs in _calls(P):
        call()
        torch.cuda.synchronize()
        want = [t.clone() for t in outs]
        side = torch.cuda.Stream()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            side.wait_stream(torch.cuda.current_stream())
            call(stream=side.cuda_stream)
            torch.cuda.current_stream().wait_stream(side)
        later = [torch.full((nbytes,), 9, dtype=torch.uint8, device="cuda") for _ in range(8)]
        for _ in range(2):
            for t in outs:
                t.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert all((t == 9).all() for t in later)
            for t, w in zip(outs, want):
                assert torch.equal(t, w)
    assert np.isfinite(want[0].float().cpu().numpy()).all()
