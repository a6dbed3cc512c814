"""What layer norm, the gradients' norm and clipping and the clipped update refuse: checked on the host, with addresses that are
never used."""
import ctypes

import pytest

BIG = 1 << 32


@pytest.fixture(scope="module")
def L():
    from paper_1808_07217_gb300 import _build

    _build.build()
    import paper_1808_07217_gb300 as L

    L.lib()
    return L


vp = ctypes.c_void_p


# ---- layer norm ----
NAMES = ["x", "r", "gamma", "beta", "s", "y", "mean", "rstd", "dy", "ds", "dx", "dgamma", "dbeta", "ws"]


def _rows(L, fn, G=3, R=500, C=40, x_ld=48, y_ld=44, par_gs=64, x_type=1, y_type=0, act=1, eps=1e-5, need=None, **at):
    n = ctypes.c_size_t()
    ok = L.lib().lsgd_layernorm_workspace(G, R, C, ctypes.byref(n)) == L.OK
    need = (n.value if ok else 0) if need is None else need
    N = G * R
    sizes = dict(x=((N - 1) * x_ld + C) * 2, y=((N - 1) * y_ld + C) * 4, mean=4 * N, gamma=4 * ((G - 1) * par_gs + C), ws=need)
    for a, b in (("r", "x"), ("s", "x"), ("ds", "x"), ("dx", "x"), ("dy", "y"), ("rstd", "mean"), ("beta", "gamma"), ("dgamma", "gamma"),
                 ("dbeta", "gamma")):
        sizes[a] = sizes[b]
    p = {k: (i + 1) * BIG for i, k in enumerate(NAMES)}
    p.update({k: v(p, sizes) if callable(v) else v for k, v in at.items()})
    q = {k: vp(v) for k, v in p.items()}
    if fn == "forward":
        s = L.lib().lsgd_layernorm_forward(q["x"], q["r"], x_type, x_ld, q["gamma"], q["beta"], par_gs, q["s"], q["y"], y_type, y_ld,
                                           q["mean"], q["rstd"], G, R, C, eps, act, None)
    else:
        s = L.lib().lsgd_layernorm_backward(q["x"], x_type, x_ld, q["y"], q["dy"], y_type, y_ld, q["ds"], q["gamma"], q["beta"], par_gs,
                                            q["mean"], q["rstd"], q["dx"], q["dgamma"], q["dbeta"], G, R, C, act, q["ws"], need, None)
    return s, L.lsgd_last_error()


@pytest.mark.parametrize("fn", ["forward", "backward"])
@pytest.mark.parametrize("bad", [dict(G=0), dict(G=65536), dict(R=-1), dict(C=0), dict(C=32769, x_ld=32769, y_ld=32769, par_gs=32769),
                                 dict(x_ld=39), dict(y_ld=39), dict(par_gs=39), dict(x_type=2), dict(y_type=-1), dict(act=3),
                                 dict(x=1), dict(x=0), dict(gamma=0), dict(beta=2), dict(mean=0), dict(rstd=6), dict(y=0), dict(y=2),
                                 dict(x_ld=1 << 59), dict(R=1 << 40)])
def test_rows_refused(L, fn, bad):
    s, msg = _rows(L, fn, **bad)
    assert s == L.EINVAL and msg.startswith("lsgd_layernorm_"), (s, msg)


@pytest.mark.parametrize("bad", [dict(r=0), dict(s=0), dict(s=1), dict(eps=0.0), dict(eps=float("nan")), dict(eps=float("inf"))])
def test_forward_refused(L, bad):
    assert _rows(L, "forward", **bad)[0] == L.EINVAL


@pytest.mark.parametrize("bad", [dict(dy=0), dict(dx=0), dict(dx=1), dict(ds=1), dict(dgamma=0), dict(dbeta=1), dict(ws=0), dict(ws=8),
                                 dict(need=64)])
def test_backward_refused(L, bad):
    assert _rows(L, "backward", **bad)[0] == L.EINVAL


WRITTEN = dict(forward=["s", "y", "mean", "rstd"], backward=["dx", "dgamma", "dbeta", "ws"])
READ = dict(forward=["x", "r", "gamma", "beta"], backward=["x", "y", "dy", "ds", "gamma", "beta", "mean", "rstd"])


@pytest.mark.parametrize("fn,out,other", [(f, a, b) for f in WRITTEN for a in WRITTEN[f] for b in WRITTEN[f] + READ[f] if a != b])
def test_what_is_written_meets_nothing(L, fn, out, other):
    step = 16  # within every alignment
    for place in (lambda p, s: p[other], lambda p, s: p[other] - max(s[out] // step * step - step, 0),
                  lambda p, s: p[other] + max(s[other] // step * step - step, 0)):
        s, msg = _rows(L, fn, **{out: place})
        assert s == L.EINVAL and "overlap" in msg, (s, msg)


# ---- lists of tensors ----
def _list(L, entries, G=2):
    table = (L.Tensor * max(1, len(entries)))()
    for t, e in zip(table, entries):
        t.g, t.out, t.n, t.g_gs, t.out_gs, t.g_type, t.out_type = e
    h = vp()
    s = L.lib().lsgd_tensors_create(table, len(entries), G, ctypes.byref(h))
    return s, h


A, B, C = BIG, 2 * BIG, 3 * BIG


@pytest.mark.parametrize("entries,G", [([], 2), ([(A, None, 10, 10, 0, 0, 0)], 0), ([(A, None, 10, 10, 0, 0, 0)], 65536),
                                       ([(A, None, -1, 10, 0, 0, 0)], 2), ([(None, None, 10, 10, 0, 0, 0)], 2),
                                       ([(A, None, 10, 9, 0, 0, 0)], 2), ([(A + 2, None, 10, 10, 0, 0, 0)], 2),
                                       ([(A, None, 10, 10, 0, 2, 0)], 2), ([(A, B, 10, 10, 9, 0, 0)], 2), ([(A, B + 1, 10, 10, 10, 0, 1)], 2),
                                       ([(A, B, 10, 10, 10, 0, 3)], 2), ([(A, B, 10, 10, 10, 0, 0), (C, None, 10, 10, 0, 0, 0)], 2),
                                       ([(A, None, 10, 1 << 51, 0, 0, 0)], 2), ([(A, None, 1 << 41, 1 << 41, 0, 0, 0)], 1)])
def test_lists_refused(L, entries, G):
    s, h = _list(L, entries, G)
    assert s == L.EINVAL and not h.value and L.lsgd_last_error().startswith("lsgd_tensors_create")


def _clip(L, h, norm=C, max_norm=1.0, ws=4 * BIG, need=None):
    n = ctypes.c_size_t()
    assert L.lib().lsgd_gradient_workspace(h, ctypes.byref(n)) == L.OK
    return (L.lib().lsgd_gradient_clip(h, vp(norm), max_norm, vp(ws), n.value if need is None else need, None), L.lsgd_last_error(),
            n.value)


LONG = (A, None, 3_000_000, 3_000_000, 0, 0, 0)


@pytest.mark.parametrize("kw", [dict(norm=0), dict(norm=C + 2), dict(max_norm=0.0), dict(max_norm=-1.0), dict(max_norm=float("nan")),
                                dict(max_norm=float("inf")), dict(ws=0), dict(ws=4 * BIG + 8), dict(need=8),
                                dict(norm=A), dict(norm=A + 8 * 3_000_000 - 4), dict(ws=A + 64), dict(norm=4 * BIG)])
def test_clip_refused(L, kw):
    s, h = _list(L, [LONG])
    assert s == L.OK
    s, msg, need = _clip(L, h, **kw)
    assert need > 0 and s == L.EINVAL and msg.startswith("lsgd_gradient_clip"), (s, msg)
    L.lib().lsgd_tensors_destroy(h)


@pytest.mark.parametrize("entries,overlaps", [
    ([(A, None, 100, 100, 0, 0, 0), (A + 400, None, 100, 200, 0, 0, 0)], True),       # worker 1 of the first at worker 0 of the second
    ([(A, None, 100, 200, 0, 0, 0), (A + 400, None, 100, 200, 0, 0, 0)], False),      # pieces of one buffer
    ([(A, None, 100, 200, 0, 0, 0), (A, None, 100, 200, 0, 0, 0)], True),             # the same tensor twice
    ([(A, None, 100, 200, 0, 0, 0), (A + 396, None, 50, 200, 0, 0, 0)], True),        # one value
    ([(A, A, 100, 200, 200, 0, 0), (B, B, 100, 100, 100, 1, 1)], False),              # in place by name
    ([(A, A, 100, 100, 100, 0, 1)], True),                                            # over itself in another type
    ([(A, B, 100, 100, 100, 0, 0), (A, C, 100, 100, 100, 0, 0)], False),              # read twice, written apart
    ([(A, B, 100, 100, 100, 0, 0), (C, B + 796, 100, 100, 100, 0, 0)], True),         # written twice
    ([(A, B, 100, 100, 100, 0, 0), (B + 796, C, 100, 100, 100, 0, 0)], True),         # written and read
    ([(A, A + 4, 100, 300, 300, 0, 0)], True)])
def test_what_is_clipped_meets_nothing(L, entries, overlaps):
    s, h = _list(L, entries)
    assert s == L.OK
    # (a norm that is refused too, so that no call reaches a GPU: which of the two is reported tells)
    n = ctypes.c_size_t()
    L.lib().lsgd_gradient_workspace(h, ctypes.byref(n))
    s = L.lib().lsgd_gradient_clip(h, vp(5 * BIG), 1.0, vp(6 * BIG), n.value, None) if overlaps else None
    if overlaps:
        assert s == L.EINVAL and "list" in L.lsgd_last_error()
    L.lib().lsgd_tensors_destroy(h)


def test_null_lists(L):
    n = ctypes.c_size_t()
    assert L.lib().lsgd_gradient_workspace(None, ctypes.byref(n)) == L.EINVAL
    assert L.lib().lsgd_gradient_norm(None, vp(A), vp(B), 100, None) == L.EINVAL
    assert L.lib().lsgd_gradient_clip(None, vp(A), 1.0, vp(B), 100, None) == L.EINVAL
    L.lib().lsgd_tensors_destroy(None)


# ---- the update ----
def _update(L, G=2, n=100, w_gs=128, g_gs=112, g_type=1, max_norm=1.0, momentum=0.9, decay_end=100, **at):
    p = dict(w=A, u=B, g=C, Wb=4 * BIG, norm=5 * BIG)
    p.update(at)
    q = {k: vp(v) for k, v in p.items()}
    return L.lib().lsgd_clipped_update(q["w"], q["u"], w_gs, q["g"], g_type, g_gs, q["Wb"], G, n, q["norm"], max_norm, 0.1, momentum, 0,
                                       0.0, decay_end, None)


@pytest.mark.parametrize("bad", [dict(G=0), dict(n=-1), dict(w_gs=99), dict(g_gs=99), dict(g_type=5), dict(max_norm=0.0),
                                 dict(max_norm=float("inf")), dict(max_norm=float("nan")), dict(decay_end=-1), dict(w=0), dict(u=0), dict(g=0),
                                 dict(norm=0), dict(w=A + 2), dict(g=C + 1), dict(Wb=1), dict(norm=5 * BIG + 1),
                                 dict(u=A), dict(u=A + 4 * 227), dict(g=A + 8), dict(g=B), dict(Wb=A + 4 * 227), dict(Wb=B), dict(Wb=C),
                                 dict(norm=A), dict(norm=B + 4 * 226), dict(norm=4 * BIG + 8)])
def test_update_refused(L, bad):
    assert _update(L, **bad) == L.EINVAL
    assert L.lsgd_last_error().startswith("lsgd_clipped_update")


def test_workspace_sizes(L):
    n = ctypes.c_size_t()
    assert L.lib().lsgd_layernorm_workspace(1, 1, 8, ctypes.byref(n)) == L.OK and n.value == 0
    assert L.lib().lsgd_layernorm_workspace(1, 100000, 512, ctypes.byref(n)) == L.OK and 0 < n.value < 1 << 24
    assert L.lib().lsgd_layernorm_workspace(1, 1, 8, None) == L.EINVAL
    assert L.lib().lsgd_layernorm_workspace(0, 1, 8, ctypes.byref(n)) == L.EINVAL
