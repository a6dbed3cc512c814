"""The norm of workers' gradients over many tensors, clipping by it and the clipped update, against 64 bits."""
import numpy as np
import pytest

from _gpu_common import built_package

U32 = 2.0 ** -24
# A lane's chain of squares: 64 and two values beside the vectors; halved by the root, whose own rounding and that to fp32 follow.
NORM = 36 * U32


@pytest.fixture(scope="module")
def P():
    import torch

    assert torch.cuda.is_available()
    return built_package()


def _lists():
    rng = np.random.default_rng(7)
    odd = [int(v) for v in rng.integers(1, 5000, 90)]
    return {"one value": [1], "one": [1000], "small": [3, 1, 7, 16, 0, 64, 129], "odd": odd, "large": [300001, 5, 1 << 20],
            "many": [int(v) for v in rng.integers(0, 60, 1500)], "hundreds": [int(v) for v in rng.integers(1, 300, 400)], "huge and tiny": [4_000_003, 1, 2, 3]}


def _make(torch, sizes, G, form, dtype, rng, scale=1.0):
    """Tensors of [G][n] in one of the forms that callers have, over buffers whose other values are a marker."""
    gen = torch.Generator(device="cuda").manual_seed(int(rng.integers(1 << 30)))
    kinds = [dtype if dtype else (torch.float32, torch.bfloat16)[i % 2] for i in range(len(sizes))]
    out, bufs = [], []
    if form == "arena":  # replica-major, one behind another without any alignment
        total = sum(sizes) + 5
        buf = torch.full((G, total), 77.0, dtype=kinds[0], device="cuda")
        at = 3
        for n in sizes:
            out.append(buf[:, at:at + n])
            at += n
        bufs.append(buf)
    else:
        for n, k in zip(sizes, kinds):
            pad = {"packed": 0, "strided": 11}[form]
            buf = torch.full((G, n + pad), 77.0, dtype=k, device="cuda")
            out.append(buf[:, pad // 2:pad // 2 + n])
            bufs.append(buf)
    for t in out:
        t.copy_(torch.randn(t.shape, generator=gen, device="cuda") * scale)
    return out, bufs


def _rest_is_marked(torch, tensors, bufs):
    marked = sum(int((b == 77).sum()) for b in bufs)
    return marked >= sum(b.numel() for b in bufs) - sum(t.numel() for t in tensors)


def _norm64(tensors):
    return np.sqrt(sum((t.double() ** 2).sum(1) for t in tensors).cpu().numpy())


@pytest.mark.gpu
@pytest.mark.parametrize("form,dtype", [("packed", None), ("strided", None), ("arena", "fp32"), ("arena", "bf16")])
@pytest.mark.parametrize("G", [1, 3])
@pytest.mark.parametrize("name", list(_lists()))
def test_norm_and_clip(P, name, G, form, dtype):
    import torch

    kind = {"fp32": torch.float32, "bf16": torch.bfloat16, None: None}[dtype]
    rng = np.random.default_rng(len(name) + G)
    grads, bufs = _make(torch, _lists()[name], G, form, kind, rng)
    for k in range(G):  # workers on either side of the border
        for t in grads:
            t[k] *= (0.5, 2.0, 1.0)[k]
    held = torch.full((G + 4,), 77.0, device="cuda")
    norm = held[2:2 + G]
    T = P.lsgd_tensors_create(grads)
    P.lsgd_gradient_norm(T, norm)
    torch.cuda.synchronize()
    want = _norm64(grads)
    assert (np.abs(norm.cpu().numpy() - want) <= NORM * want).all()
    assert (held[:2] == 77).all() and (held[2 + G:] == 77).all()
    first = norm.clone()
    limit = float(np.float32(want.mean() * (0.7 if G == 1 else 1.0)))
    f = np.float32(limit) / np.maximum(norm.cpu().numpy(), np.float32(limit))
    factor = torch.tensor(f, device="cuda")[:, None]
    # to other places, of either type: one product and one rounding
    for place in (torch.float32, torch.bfloat16):
        outs, obufs = _make(torch, _lists()[name], G, "strided" if form != "strided" else "packed", place, rng)
        P.lsgd_gradient_clip(P.lsgd_tensors_create(grads, outs), norm, limit)
        torch.cuda.synchronize()
        assert torch.equal(norm, first)
        for t, o in zip(grads, outs):
            assert torch.equal(o, (t.float() * factor).to(place))
        assert _rest_is_marked(torch, outs, obufs)
    # in place
    kept = [t.clone() for t in grads]
    P.lsgd_gradient_clip(T, norm, limit)
    torch.cuda.synchronize()
    assert torch.equal(norm, first)
    for t, o in zip(kept, grads):
        assert torch.equal(o, (t.float() * factor).to(t.dtype))
    assert _rest_is_marked(torch, grads, bufs)


@pytest.mark.gpu
@pytest.mark.parametrize("lead_in,lead_out", [(0, 1), (1, 0), (1, 1), (3, 7), (5, 4), (2, 6)])
@pytest.mark.parametrize("types", [("fp32", "fp32"), ("fp32", "bf16"), ("bf16", "bf16"), ("bf16", "fp32")])
def test_clip_between_any_alignments(P, lead_in, lead_out, types):
    import torch

    a, b = ({"fp32": torch.float32, "bf16": torch.bfloat16}[t] for t in types)
    n = 9001
    src = torch.randn(n + 16, device="cuda").to(a)
    dst = torch.full((n + 16,), 77.0, device="cuda", dtype=b)
    g, o = src[lead_in:lead_in + n], dst[lead_out:lead_out + n]
    norm = torch.empty(1, device="cuda")
    P.lsgd_gradient_clip(P.lsgd_tensors_create([g], [o], workers=False), norm, 1.0)
    torch.cuda.synchronize()
    assert torch.equal(o, (g.float() * (np.float32(1.0) / norm)).to(b))
    assert (dst[:lead_out] == 77).all() and (dst[lead_out + n:] == 77).all()


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [1e30, 3e18, 1e-19, 1e-30, 1e-40])
def test_no_overflow_and_no_underflow(P, scale):
    import torch

    x = torch.randn(2, 70001, device="cuda", dtype=torch.float64)
    grads = [(x * scale).float(), torch.zeros(2, 5000, device="cuda")]
    norm = torch.empty(2, device="cuda")
    P.lsgd_gradient_norm(P.lsgd_tensors_create(grads), norm)
    want = _norm64(grads)
    # (values at the bottom of fp32's range: the norm's own rounding is 2^-150 there)
    assert (np.abs(norm.cpu().numpy() - want) <= NORM * want + 2.0 ** -149).all()


@pytest.mark.gpu
def test_large_values_beside_small_ones(P):
    import torch

    g = torch.zeros(1, 40000, device="cuda")
    g[0, 17], g[0, 30000], g[0, 123] = 1e20, 3e19, 1e-25
    norm = torch.empty(1, device="cuda")
    P.lsgd_gradient_norm(P.lsgd_tensors_create([g]), norm)
    want = _norm64([g])
    assert abs(float(norm) - want[0]) <= NORM * want[0]
    g.zero_()
    P.lsgd_gradient_clip(P.lsgd_tensors_create([g]), norm, 1.0)
    assert float(norm) == 0 and (g == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_a_value_that_is_not_finite_stays_with_its_worker(P, bad, dtype):
    import torch

    t = {"fp32": torch.float32, "bf16": torch.bfloat16}[dtype]
    rng = np.random.default_rng(1)
    grads, _ = _make(torch, [100, 3000, 17], 3, "packed", t, rng)
    grads[1][1, 2999] = bad
    outs = [torch.empty_like(g) for g in grads]
    norm = torch.empty(3, device="cuda")
    P.lsgd_gradient_clip(P.lsgd_tensors_create(grads, outs), norm, 5.0)
    n = norm.cpu().numpy()
    want = _norm64([g[[0, 2]] for g in grads])
    assert (np.abs(n[[0, 2]] - want) <= NORM * want).all()
    if np.isnan(bad):
        assert np.isnan(n[1]) and all(torch.isnan(o[1]).all() for o in outs)
    else:
        assert np.isposinf(n[1]) and torch.isnan(outs[1][1, 2999]) and (outs[1][1, :2999] == 0).all() and (outs[0][1] == 0).all()
    f = np.float32(5.0) / n  # (a number over a tensor is its reciprocal's multiple in torch, rounded twice)
    for g, o in zip(grads, outs):
        for k in (0, 2):
            assert torch.equal(o[k], (g[k].float() * float(f[k])).to(t))


@pytest.mark.gpu
def test_equal_values_add_up_without_drift(P):
    import torch

    n = 50_000_001
    g = torch.full((1, n), 0.1, device="cuda")
    norm = torch.empty(1, device="cuda")
    P.lsgd_gradient_norm(P.lsgd_tensors_create([g]), norm)
    want = float(np.float32(0.1)) * np.sqrt(float(n))
    assert abs(float(norm) - want) <= NORM * want


@pytest.mark.gpu
def test_a_tensor_twice_is_summed_twice_and_not_clipped(P):
    import torch

    g = torch.randn(2, 500, device="cuda")
    norm = torch.empty(2, device="cuda")
    T = P.lsgd_tensors_create([g, g[:, 100:200]])
    P.lsgd_gradient_norm(T, norm)
    want = _norm64([g, g[:, 100:200]])
    assert (np.abs(norm.cpu().numpy() - want) <= NORM * want).all()
    with pytest.raises(P.LsgdError) as e:
        P.lsgd_gradient_clip(T, norm, 1.0)
    assert e.value.status == P.EINVAL
    # to places of their own it is clipped twice
    outs = [torch.empty_like(g), torch.empty(2, 100, device="cuda")]
    P.lsgd_gradient_clip(P.lsgd_tensors_create([g, g[:, 100:200]], outs), norm, 1.0)
    assert torch.equal(outs[1], outs[0][:, 100:200])


@pytest.mark.gpu
def test_repeats_streams_and_graphs_give_the_same_bits(P):
    import torch

    rng = np.random.default_rng(3)
    grads, _ = _make(torch, _lists()["odd"] + [200000], 5, "packed", None, rng)
    outs = [torch.empty_like(g) for g in grads]
    T = P.lsgd_tensors_create(grads, outs)
    norm = torch.empty(5, device="cuda")
    P.lsgd_gradient_clip(T, norm, 2.0)
    torch.cuda.synchronize()
    want, kept = norm.clone(), [o.clone() for o in outs]
    side = torch.cuda.Stream()
    for _ in range(3):
        norm.zero_()
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        P.lsgd_gradient_clip(T, norm, 2.0, stream=side.cuda_stream)
        torch.cuda.synchronize()
        assert torch.equal(norm, want) and all(torch.equal(o, k) for o, k in zip(outs, kept))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.lsgd_gradient_clip(T, norm, 2.0)
    del T  # the graph keeps what it needs
    for scale in (1.0, 0.5, 1e-4):
        for g in grads:
            g.copy_(torch.randn(g.shape, device="cuda") * scale)
        graph.replay()
        torch.cuda.synchronize()
        w = _norm64(grads)
        assert (np.abs(norm.cpu().numpy() - w) <= NORM * w).all()
        f = torch.clamp(2.0 / norm, max=1.0)[:, None]
        for g, o in zip(grads, outs):
            assert torch.equal(o, (g.float() * f).to(o.dtype))


@pytest.mark.gpu
@pytest.mark.parametrize("G,sizes", [(3, [4999, 3, 1024, 777] * 20), (1, [300001, 5, 99991, 2]), (1, [260000]), (1, [262148]), (64, [17000, 3]),
                                     (301, [3500]), (305, [3500])])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_calls_one_behind_another_see_what_was_written(P, G, sizes, dtype):
    """Norms and clippings in place, each of what the one before wrote, at sizes on both sides of what takes one launch: the bits of calls
    that are waited for.  Tensors without any alignment share lines of 128 bytes that different SMs read and write."""
    import torch

    kind = {"fp32": torch.float32, "bf16": torch.bfloat16}[dtype]

    def steps(wait):
        grads, bufs = _make(torch, sizes, G, "arena", kind, np.random.default_rng(5))
        T = P.lsgd_tensors_create(grads)
        norms = torch.zeros(40, G, device="cuda")
        for i in range(0, 40, 2):
            P.lsgd_gradient_clip(T, norms[i], limit * 0.98 ** i)
            if wait:
                torch.cuda.synchronize()
            P.lsgd_gradient_norm(T, norms[i + 1])
            if wait:
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        return bufs[0], norms

    limit = float(np.sqrt(sum(sizes)) * 0.9)
    one, other = steps(True), steps(False)
    assert torch.equal(one[0], other[0]) and torch.equal(one[1], other[1])
    # (the clipped gradient's norm: the limit, but for the factor's, the products' and the norm's roundings)
    eps = 2.0 ** -24 if dtype == "fp32" else 2.0 ** -8
    last = one[1][39].cpu().numpy()
    assert (np.abs(last - limit * 0.98 ** 38) <= (2 * NORM + 3 * U32 + eps) * limit).all()


# ---- the update ----
@pytest.mark.gpu
@pytest.mark.parametrize("momentum,nesterov", [(0.0, False), (0.9, False), (0.9, True)])
@pytest.mark.parametrize("shadow", [False, True])
@pytest.mark.parametrize("g_type", ["fp32", "bf16"])
@pytest.mark.parametrize("G,n,decay_end", [(3, 4096, 1000), (1, 8, 8), (16, 250_000, 249_996)])
def test_update_has_the_plain_updates_bits(P, G, n, decay_end, g_type, shadow, momentum, nesterov):
    import torch

    gen = torch.Generator(device="cuda").manual_seed(n)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    w, u, g = rand(G, n), rand(G, n), rand(G, n).to({"fp32": torch.float32, "bf16": torch.bfloat16}[g_type])
    wb = torch.zeros(G, n, device="cuda", dtype=torch.bfloat16) if shadow else None
    norm = torch.empty(G, device="cuda")
    P.lsgd_gradient_norm(P.lsgd_tensors_create([g]), norm)
    limit = float(norm.median())  # clipped and unclipped workers
    w2, u2, wb2 = w.clone(), u.clone(), None if wb is None else wb.clone()
    clipped = g.float() * torch.clamp(torch.tensor(limit, device="cuda") / norm, max=1.0)[:, None]
    P.lsgd_sgd_update(w2, u2, clipped, wb2, G * n, 0.1, momentum, nesterov, 0.01, period=n, decay_end=decay_end)
    P.lsgd_clipped_update(w, u if momentum else None, g, wb, G, n, norm, limit, 0.1, momentum, nesterov, 0.01, decay_end)
    torch.cuda.synchronize()
    assert torch.equal(w, w2) and torch.equal(u, u2) and (wb is None or torch.equal(wb, wb2))


@pytest.mark.gpu
@pytest.mark.parametrize("g_type", ["fp32", "bf16"])
@pytest.mark.parametrize("G,n,w_gs,g_gs,lead", [(1, 1, 1, 1, 0), (3, 1001, 1001, 1003, 0), (2, 1022, 1024, 1028, 0), (2, 70001, 70004, 70008, 1),
                                                (5, 0, 4, 4, 0), (40, 7, 64, 7, 2)])
def test_update_of_any_sizes(P, G, n, w_gs, g_gs, lead, g_type):
    import torch

    gen = torch.Generator(device="cuda").manual_seed(n + lead)
    t = {"fp32": torch.float32, "bf16": torch.bfloat16}[g_type]

    def buffer(gs, dtype=torch.float32):
        b = torch.full((lead + G * gs + 8,), 77.0, device="cuda", dtype=dtype)
        v = b[lead:lead + G * gs].view(G, gs)[:, :n]
        v.copy_(torch.randn(G, n, generator=gen, device="cuda"))
        return b, b[lead:], v

    (wbuf, w, wv), (ubuf, u, uv), (_, g, gv), (sbuf, s, sv) = buffer(w_gs), buffer(w_gs), buffer(g_gs, t), buffer(w_gs, torch.bfloat16)
    norm = (1 + torch.rand(G, generator=gen, device="cuda")).contiguous()
    old, mom, gd = wv.double(), uv.double(), gv.double()
    P.lsgd_clipped_update(w, u, g, s, G, n, norm, 1.5, 0.05, 0.9, True, 0.02, n // 2, w_gs, g_gs)
    torch.cuda.synchronize()
    f = torch.clamp(1.5 / norm.double(), max=1.0)[:, None]
    decay = (torch.arange(n, device="cuda") < n // 2) * float(np.float32(0.02))
    m, lr = float(np.float32(0.9)), float(np.float32(0.05))
    gp = f * gd + decay * old
    wu = m * mom + gp
    ww = old - lr * (gp + m * wu)
    tol = 4 * U32 * (mom.abs() + gd.abs() + old.abs())  # f's, the product's, the sums' roundings
    assert ((uv.double() - wu).abs() <= tol).all() and ((wv.double() - ww).abs() <= tol + U32 * ww.abs()).all()
    assert torch.equal(sv, wv.bfloat16())
    for b, v in ((wbuf, wv), (ubuf, uv), (sbuf, sv)):
        assert int((b == 77).sum()) >= b.numel() - v.numel()


@pytest.mark.gpu
def test_update_with_norms_that_are_not_finite(P):
    import torch

    w, g = torch.ones(3, 100, device="cuda"), torch.ones(3, 100, device="cuda")
    norm = torch.tensor([float("nan"), float("inf"), 2.0], device="cuda")
    P.lsgd_clipped_update(w, None, g, None, 3, 100, norm, 1.0, 0.5)
    assert torch.isnan(w[0]).all() and (w[1] == 1).all() and (w[2] == 0.75).all()


# ---- workspaces ----
def _calls(P):
    """(bytes of workspace, a call on `stream`, its outputs) for the operators that use one."""
    import torch

    gen = torch.Generator(device="cuda").manual_seed(3)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    G, R, C = 2, 900, 1000
    x, dy, gamma, beta = rand(G, R, C), rand(G, R, C), rand(G, C), rand(G, C)
    y, dx, dgamma, dbeta = torch.empty_like(x), torch.empty_like(x), torch.empty_like(gamma), torch.empty_like(gamma)
    mean, rstd = torch.empty(G, R, device="cuda"), torch.empty(G, R, device="cuda")
    P.lsgd_layernorm_forward(x, gamma, beta, y, mean, rstd, G, R, C)
    grads, norm = [rand(2, 1_000_001), rand(2, 333)], torch.empty(2, device="cuda")
    outs = [torch.empty_like(g) for g in grads]
    T, U = P.lsgd_tensors_create(grads), P.lsgd_tensors_create(grads, outs)
    assert T.workspace and U.workspace and P.lsgd_layernorm_workspace(G, R, C)
    return [(P.lsgd_layernorm_workspace(G, R, C),
             lambda **kw: P.lsgd_layernorm_backward(x, None, dy, gamma, beta, mean, rstd, dx, dgamma, dbeta, G, R, C, **kw),
             [dx, dgamma, dbeta]),
            (T.workspace, lambda **kw: P.lsgd_gradient_norm(T, norm, **kw), [norm]),
            (U.workspace, lambda **kw: P.lsgd_gradient_clip(U, norm, 1.0, **kw), [norm, *outs])]


@pytest.mark.gpu
@pytest.mark.parametrize("which", [0, 1, 2])
def test_a_workspace_belongs_to_the_calls_stream(P, which):
    """A tensor of the workspace's size is deleted while kernels that read and write it wait on the current stream: the call
    on another stream neither changes what they read nor finds its sums changed by them; the same with a stream of its own."""
    import torch

    nbytes, call, outs = _calls(P)[which]
    call()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    for t in outs:
        t.zero_()
    call(workspace=torch.empty(nbytes, dtype=torch.uint8, device="cuda"))
    assert all(torch.equal(t, w) for t, w in zip(outs, want))
    side = torch.cuda.Stream()
    for _ in range(3):
        for t in outs:
            t.zero_()
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
        assert all(torch.equal(t, w) for t, w in zip(outs, want))
    with pytest.raises(P.LsgdError) as e:
        call(workspace=torch.empty(nbytes - 16, dtype=torch.uint8, device="cuda"))
    assert e.value.status == P.EINVAL


@pytest.mark.gpu
@pytest.mark.parametrize("which", [0, 1, 2])
def test_a_captured_call_keeps_its_workspace_to_itself(P, which):
    import torch

    nbytes, call, outs = _calls(P)[which]
    call()
    torch.cuda.synchronize()
    want = [t.clone() for t in outs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    later = [torch.full((nbytes,), 9, dtype=torch.uint8, device="cuda") for _ in range(8)]
    for _ in range(2):
        for t in outs:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all((t == 9).all() for t in later)
        assert all(torch.equal(t, w) for t, w in zip(outs, want))


@pytest.mark.gpu
def test_tensors_beyond_32_bits(P):
    import torch

    n = (1 << 31) + 12345
    g = torch.full((1, n), 0.5, dtype=torch.bfloat16, device="cuda")
    g[0, -7:] = 1000.0
    out, norm = torch.empty_like(g), torch.empty(1, device="cuda")
    P.lsgd_gradient_clip(P.lsgd_tensors_create([g], [out]), norm, 100.0)
    want = np.sqrt(0.25 * (n - 7) + 7e6)
    assert abs(float(norm) - want) <= NORM * want
    f = np.float32(100.0) / norm.cpu().numpy()[0]
    assert torch.equal(out[0, -5000:], (g[0, -5000:].float() * float(f)).bfloat16())
    assert int((out[0, :-7] == out[0, 0]).sum()) == n - 7


SCRIPT = """
import torch
import paper_1808_07217_gb300 as P
x = torch.randn(40, 6000, device="cuda").bfloat16()
ga, be = torch.ones(1, 6000, device="cuda"), torch.zeros(1, 6000, device="cuda")
y, dx, m, r = torch.empty_like(x), torch.empty_like(x), torch.empty(40, device="cuda"), torch.empty(40, device="cuda")
dg, db, norm = torch.empty(1, 6000, device="cuda"), torch.empty(1, 6000, device="cuda"), torch.empty(1, device="cuda")
g = torch.randn(1, 3000000, device="cuda")
T = P.lsgd_tensors_create([g, dg, db])
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
def step():
    P.lsgd_layernorm_forward(x, ga, be, y, m, r, 1, 40, 6000)
    P.lsgd_layernorm_backward(x, None, y, ga, be, m, r, dx, dg, db, 1, 40, 6000)
    P.lsgd_gradient_norm(T, norm)
with torch.cuda.graph(graph):
    step()
graph.replay()
torch.cuda.synchronize()
got = [t.clone() for t in (y, dx, dg, db, norm)]
step()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(got, (y, dx, dg, db, norm)))
assert float(norm) > 0 and P.lsgd_device_status() == P.OK
print("ok")
"""


@pytest.mark.gpu
def test_first_calls_may_be_captured():
    import os
    import subprocess
    import sys

    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    run = subprocess.run([sys.executable, "-c", SCRIPT], cwd=root, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and run.stdout.strip() == "ok", run.stderr[-2000:]
