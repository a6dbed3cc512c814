"""Layer norm of rows with an activation and a residual, forward and backward, against its definition in 64 bits."""
import numpy as np
import pytest

import _operator_refs as R
from _gpu_common import built_package

U32, U16 = 2.0 ** -24, 2.0 ** -8  # largest relative roundings of fp32 and bf16
ACTS = {"none": 0, "relu": 1, "silu": 2}
# Roundings that a value of a row's sums passes through: 8 values of a thread, 5 exchanges in a warp, the same again over the
# warps and CTAs of a row, a division; 40 bounds them.  dgamma and dbeta: 64 rows of a segment, 64 segments, 8 merges of
# teams, then the ranges (at most 64 of a thread) and 5 exchanges; the sizes here stay below 160.
ROW, COLUMN = 40 * U32, 160 * U32

# (G, R, C): single values, parts of warps, one warp and several, odd widths, every vector, the widest rows of one CTA and
# rows of clusters of 2, 5, 8, 10 and 16, one row and many, rows that end inside a CTA's teams
SHAPES = [(1, 1, 1), (2, 3, 5), (1, 70, 8), (3, 33, 24), (2, 130, 77), (1, 40, 256), (1, 9, 258), (2, 21, 300), (1, 50, 777),
          (2, 5, 1024), (1, 7, 2050), (2, 6, 2303), (2, 9, 3333), (3, 2, 4096), (1, 3, 4097), (2, 3, 8200), (1, 2, 20001), (1, 2, 32767), (1, 2, 32768), (5, 1, 513),
          (1, 3000, 16), (2, 700, 100)]


@pytest.fixture(scope="module")
def P():
    import torch

    assert torch.cuda.is_available()
    return built_package()


def _types(torch, name):
    return {"bf16": torch.bfloat16, "fp32": torch.float32}[name]


class Rows:
    """A tensor of N rows of C values at a stride, from `lead` values on, in a buffer of a marker (or of NaN: what must not be
    read is not)."""

    def __init__(self, torch, N, C, ld, dtype, lead, fill):
        self.N, self.C, self.ld, self.lead, self.fill = N, C, ld, lead, fill
        self.span = (N - 1) * ld + C if N else 0
        self.buf = torch.full((lead + self.span + 8,), fill, dtype=dtype, device="cuda")
        self.t = self.buf[lead:lead + self.span]

    def rows(self):
        return self.buf[self.lead:].as_strided((self.N, self.C), (self.ld, 1), self.buf.storage_offset() + self.lead)

    def set(self, v):
        self.rows().copy_(v)
        return self

    def intact(self):
        import torch

        rest = torch.ones_like(self.buf, dtype=torch.bool)
        rest[self.lead:].as_strided((self.N, self.C), (self.ld, 1), self.lead).fill_(False)
        return bool((self.buf[rest] == self.fill).all())


class Case:
    def __init__(self, P, shape, x_type="fp32", y_type="fp32", act="none", residual=False, x_ld=0, y_ld=0, lead=8, par_gs=0,
                 seed=0, offset=0.0):
        import torch

        self.P, self.torch, self.shape, self.act, self.residual = P, torch, shape, act, residual
        G, Rn, C = shape
        self.N, self.x_ld, self.y_ld, self.par_gs, self.lead = G * Rn, x_ld or C, y_ld or C, par_gs or C, lead
        self.xt, self.yt = _types(torch, x_type), _types(torch, y_type)
        rng = np.random.default_rng(seed + sum(shape))
        draw = lambda *s: torch.tensor(rng.standard_normal(s), dtype=torch.float32, device="cuda")  # noqa: E731
        N = self.N
        self.x = self._rows(self.x_ld, self.xt, float("nan")).set(draw(N, C) * 1.5 + draw(C) + offset)
        self.dy = self._rows(self.y_ld, self.yt, float("nan")).set(draw(N, C))
        self.r = self._rows(self.x_ld, self.xt, float("nan")).set(draw(N, C)) if residual else None
        self.ds = self._rows(self.x_ld, self.xt, float("nan")).set(draw(N, C)) if residual else None
        npar = (G - 1) * self.par_gs + C
        pick = (torch.arange(G, device="cuda")[:, None] * self.par_gs + torch.arange(C, device="cuda")).reshape(-1)
        self.pick = pick
        self.gamma, self.beta = torch.full((npar,), float("nan"), device="cuda"), torch.full((npar,), float("nan"), device="cuda")
        self.gamma[pick], self.beta[pick] = 1 + 0.3 * draw(G * C), 0.3 * draw(G * C)

    def _rows(self, ld, dtype, fill):
        return Rows(self.torch, self.N, self.shape[2], ld, dtype, self.lead, fill)

    def kw(self):
        return dict(act=ACTS[self.act], x_ld=self.x_ld, y_ld=self.y_ld, par_gs=self.par_gs)

    def forward(self, **kw):
        t = self.torch
        self.y, self.s = self._rows(self.y_ld, self.yt, 77.0), self._rows(self.x_ld, self.xt, 77.0) if self.residual else None
        stats = [t.full((self.N + 16,), 77.0, device="cuda") for _ in range(2)]
        self.mean, self.rstd = (s[8:8 + self.N] for s in stats)
        self.P.lsgd_layernorm_forward(self.x.t, self.gamma, self.beta, self.y.t, self.mean, self.rstd, *self.shape,
                                      r=self.r.t if self.residual else None, s=self.s.t if self.residual else None,
                                      **self.kw(), **kw)
        t.cuda.synchronize()
        assert self.y.intact() and (not self.residual or self.s.intact())
        assert all((s[:8] == 77).all() and (s[8 + self.N:] == 77).all() for s in stats)
        return self

    def normalised(self):
        return self.s if self.residual else self.x

    def backward(self, **kw):
        t = self.torch
        self.dx = self._rows(self.x_ld, self.xt, 77.0)
        pars = [t.full((self.gamma.numel() + 16,), 77.0, device="cuda") for _ in range(2)]
        dgamma, dbeta = (p[8:8 + self.gamma.numel()] for p in pars)
        self.P.lsgd_layernorm_backward(self.normalised().t, self.y.t if self.act == "relu" else None, self.dy.t, self.gamma,
                                       self.beta, self.mean, self.rstd, self.dx.t, dgamma, dbeta, *self.shape,
                                       ds=self.ds.t if self.residual else None, **self.kw(), **kw)
        t.cuda.synchronize()
        assert self.dx.intact()
        for p in pars:
            rest = t.ones_like(p, dtype=t.bool)
            rest[8 + self.pick] = False
            assert (p[rest] == 77).all()
        self.dgamma, self.dbeta = dgamma[self.pick], dbeta[self.pick]
        return self

    # ---- against 64 bits ----
    def _d(self, rows):
        G, Rn, C = self.shape
        return rows.rows().double().cpu().numpy().reshape(G, Rn, 1, C)

    def _params(self):
        G, _, C = self.shape
        return (t[self.pick].double().cpu().numpy().reshape(G, C) for t in (self.gamma, self.beta))

    def check_forward(self, eps=1e-5):
        G, Rn, C = self.shape
        if self.residual:  # one addition and one rounding
            want = (self.x.rows().float() + self.r.rows().float()).to(self.xt)
            assert self.torch.equal(self.s.rows(), want)
        x = self._d(self.normalised())
        ga, be = self._params()
        wy, wm, wr, z = R.gn_forward(x, ga, be, 1, eps, self.act)
        big = np.abs(x).max((2, 3))[..., None]
        dm = ROW * big  # a mean is off by its roundings times the largest value
        assert (np.abs(self.mean.cpu().numpy().reshape(wm.shape) - wm) <= dm).all()
        dr = wr * (ROW + (dm * wr) ** 2)  # the variance's roundings, the mean's error squared, the root's
        assert (np.abs(self.rstd.cpu().numpy().reshape(wr.shape) - wr) <= dr).all()
        wide = lambda v: v[..., None]  # noqa: E731
        g = np.abs(ga)[:, None, None]
        dz = g * (wide(dm * wr) + np.abs((x - wide(wm)) * wide(wr)) * wide(dr / wr))
        dz = dz + 8 * U32 * (np.abs(z) + g * (np.abs(x) + wide(np.abs(wm))) * wide(wr) + np.abs(be)[:, None, None])
        # |act'| <= 1.1; the activation's own roundings (bf16 results take the fast exponential: 2 + |z| units, below 2^-18)
        yu = U16 if self.yt == self.torch.bfloat16 else U32
        tol = 1.1 * dz + (16 * U32 if yu == U32 else 2.0 ** -18) * np.abs(wy) + yu * np.abs(wy) + 1e-37
        worst = np.abs(self._d(self.y) - wy) / tol
        assert worst.max() <= 1.0, worst.max()

    def check_backward(self):
        G, Rn, C = self.shape
        x, dy = self._d(self.normalised()), self._d(self.dy)
        ga, be = self._params()
        m, r = (t.double().cpu().numpy().reshape(G, Rn, 1) for t in (self.mean, self.rstd))
        wdx, wdg, wdb, dz, xh = R.gn_backward(x, dy, ga, be, m, r, 1, self.act, self._d(self.y) > 0)
        wide = lambda v: v[..., None]  # noqa: E731
        bf16 = self.xt == self.torch.bfloat16
        off = 8 * U32 * ((np.abs(x) + wide(np.abs(m))) * wide(r))  # of xh
        ez = 8 * U32 * np.abs(dz)
        if self.act == "silu":
            z_off = np.abs(ga)[:, None, None] * off + 8 * U32 * (np.abs(xh * ga[:, None, None]) + np.abs(be)[:, None, None])
            ez = np.abs(dy) * (z_off + (2.0 ** -18 if bf16 else 32 * U32) * 1.1)
        tdb = ez.sum((1, 2)) + COLUMN * np.abs(dz).sum((1, 2))
        tdg = (ez * np.abs(xh) + np.abs(dz) * off).sum((1, 2)) + COLUMN * np.abs(dz * xh).sum((1, 2))
        got = lambda t: t.double().cpu().numpy().reshape(G, C)  # noqa: E731
        assert (np.abs(got(self.dbeta) - wdb) <= tdb + 1e-37).all()
        assert (np.abs(got(self.dgamma) - wdg) <= tdg + 1e-37).all()
        g = np.abs(ga)[:, None, None]
        mean_of = lambda t: t.mean(3, keepdims=True)  # noqa: E731
        e1 = mean_of(g * ez + ROW * g * np.abs(dz))
        e2 = mean_of(g * (ez * np.abs(xh) + np.abs(dz) * off) + ROW * g * np.abs(dz * xh))
        m2 = mean_of(ga[:, None, None] * dz * xh)
        tol = wide(r) * (g * ez + e1 + np.abs(xh) * e2 + off * np.abs(m2) +
                         8 * U32 * (g * np.abs(dz) + mean_of(g * np.abs(dz)) + np.abs(xh) * np.abs(m2)))
        if self.residual:
            ds = self._d(self.ds)
            wdx = wdx + ds
            tol = tol + U32 * np.abs(wdx)  # the addition's rounding
        tol = tol + (U16 if bf16 else U32) * np.abs(wdx) + 1e-37
        worst = np.abs(self._d(self.dx) - wdx) / tol
        assert worst.max() <= 1.0, worst.max()


TYPES = [("bf16", "bf16"), ("fp32", "bf16"), ("fp32", "fp32"), ("bf16", "fp32")]


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["none", "relu", "silu"])
@pytest.mark.parametrize("x_type,y_type", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_both_ways(P, shape, x_type, y_type, act):
    residual = (len(act) + len(x_type + y_type) // 2 + shape[2]) % 2 == 0
    c = Case(P, shape, x_type, y_type, act, residual, par_gs=shape[2] + (7 if shape[0] > 1 else 0)).forward()
    c.check_forward()
    c.backward().check_backward()


@pytest.mark.gpu
@pytest.mark.parametrize("x_type,y_type", TYPES)
@pytest.mark.parametrize("shape,x_ld,y_ld", [((2, 9, 61), 64, 64), ((1, 30, 1001), 1008, 1004), ((2, 5, 4099), 4104, 4101),
                                             ((1, 200, 3), 8, 4), ((2, 3, 9001), 9008, 9016), ((1, 4, 70), 1000, 70)])
@pytest.mark.parametrize("residual", [False, True])
def test_rows_at_strides(P, shape, x_ld, y_ld, x_type, y_type, residual):
    c = Case(P, shape, x_type, y_type, "relu", residual, x_ld, y_ld).forward()
    c.check_forward()
    c.backward().check_backward()


@pytest.mark.gpu
@pytest.mark.parametrize("lead", [1, 2, 3, 4, 5])
@pytest.mark.parametrize("x_type,y_type", TYPES)
def test_tensors_that_start_anywhere(P, lead, x_type, y_type):
    c = Case(P, (2, 33, 328), x_type, y_type, "silu", True, lead=lead).forward()
    c.check_forward()
    c.backward().check_backward()


# more rows than the SMs hold at once; segments of rows; ranges that end unevenly; workers by the thousand
@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(1, 40000, 64), (3, 9001, 130), (2, 3001, 1024), (700, 9, 48), (1, 200000, 4), (4, 1200, 2052)])
@pytest.mark.parametrize("x_type", ["bf16", "fp32"])
def test_many_rows(P, shape, x_type):
    c = Case(P, shape, x_type, x_type, "relu", True).forward()
    c.check_forward()
    c.backward().check_backward()


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(2, 49, 90), (1, 5, 5001), (1, 8, 64)])
def test_mean_far_above_the_deviation(P, shape):
    c = Case(P, shape, offset=3000.0).forward()
    c.check_forward()
    # a variance taken as the difference of two second moments would be off by 3000^2 2^-24 ~ 0.5 here
    x = c._d(c.x)
    want = R.gn_forward(x, *c._params(), 1, 1e-5, "none")[2]
    assert np.abs(c.rstd.cpu().numpy().reshape(want.shape) / want - 1).max() < 1e-4


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(2, 9, 40), (1, 6, 1000), (1, 4, 9000)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_a_value_that_is_not_finite_stays_in_its_row(P, shape, bad):
    import torch

    clean, c = (Case(P, shape, "fp32", "bf16", "relu") for _ in range(2))
    clean.forward().backward()
    c.x.rows()[2, shape[2] - 1] = bad
    c.forward().backward()
    others = torch.arange(c.N, device="cuda") != 2
    assert torch.isnan(c.y.rows()[2].float()).all() and torch.isnan(c.dx.rows()[2]).all()
    assert torch.equal(c.y.rows()[others], clean.y.rows()[others]) and torch.equal(c.dx.rows()[others], clean.dx.rows()[others])
    assert torch.equal(c.mean[others], clean.mean[others]) and torch.equal(c.rstd[others], clean.rstd[others])


@pytest.mark.gpu
def test_rows_of_equal_values_and_no_rows(P):
    import torch

    c = Case(P, (1, 5, 64))
    c.x.rows().fill_(1.75)
    c.forward()
    # the mean of equal values is exact here (64 of them), so that every deviation is zero: y = beta
    assert (c.mean == 1.75).all() and torch.equal(c.y.rows(), c.beta.expand(5, 64))
    e = torch.empty(0, device="cuda")
    ga = torch.ones(3, 40, device="cuda")
    P.lsgd_layernorm_forward(e, ga, ga, e, e, e, 3, 0, 40)
    dg, db = torch.full((3, 44), 5.0, device="cuda"), torch.full((3, 44), 5.0, device="cuda")
    P.lsgd_layernorm_backward(e, None, e, torch.ones(3, 44, device="cuda"), torch.ones(3, 44, device="cuda"), e, e, e, dg, db, 3, 0, 40,
                              par_gs=44)
    torch.cuda.synchronize()
    assert (dg[:, :40] == 0).all() and (db[:, :40] == 0).all() and (dg[:2, 40:] == 5).all() and (db[:2, 40:] == 5).all()


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["none", "relu", "silu"])
def test_gradients_against_differences(P, act):
    """The gradient's product with a direction against the central difference of sum(w y + v s) along it."""
    import torch

    shape = G, Rn, C = (2, 7, 131)
    c = Case(P, shape, "fp32", "fp32", act, True).forward().backward()
    gen = torch.Generator(device="cuda").manual_seed(4)
    ux, ug, ub = (torch.randn(n, generator=gen, device="cuda", dtype=torch.float64) for n in (c.N * C, G * C, G * C))

    on = (c.y.rows() > 0).view(G, Rn, C)

    def value(h):
        x = c.x.rows().double() + c.r.rows().double() + h * ux.view(c.N, C)
        ga = (c.gamma[c.pick].double() + h * ug).view(G, 1, C)
        be = (c.beta[c.pick].double() + h * ub).view(G, 1, C)
        x = x.view(G, Rn, C)
        z = (x - x.mean(-1, keepdim=True)) * (x.var(-1, correction=0, keepdim=True) + 1e-5).rsqrt() * ga + be
        if act == "relu":  # the side of the kink that the forward took: a value that crosses it between -h and h has no difference
            assert ((z > 0) == on)[z.abs() > 1e-3].all()
        y = z * on if act == "relu" else z * torch.sigmoid(z) if act == "silu" else z
        return float((y * c.dy.rows().double().view_as(y)).sum() + (x * c.ds.rows().double().view_as(x)).sum())

    h = 1e-5  # the difference's error: h^2 times the third derivative, and 1e-16 / h of the sums
    want = (value(h) - value(-h)) / (2 * h)
    got = float((c.dx.rows().double() * ux.view(c.N, C)).sum() + (c.dgamma.double() * ug).sum() + (c.dbeta.double() * ub).sum())
    # the gradient's own error and that of s (rounded to fp32 here): each of the terms, of either sign, by 1e-5 of its size
    size = float((c.dx.rows().double() * ux.view(c.N, C)).abs().sum() + (c.dgamma.double() * ug).abs().sum())
    assert abs(got - want) <= 1e-5 * size, (got, want)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", [(2, 60, 100), (3, 400, 1031), (1, 6, 9000)])
def test_repeats_streams_and_graphs_give_the_same_bits(P, shape):
    import torch

    c = Case(P, shape, "bf16", "bf16", "silu", True).forward().backward()
    want = [t.clone() for t in (c.y.buf, c.s.buf, c.mean, c.rstd, c.dx.buf, c.dgamma, c.dbeta)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c.forward(stream=side.cuda_stream).backward(stream=side.cuda_stream)
    for t, w in zip((c.y.buf, c.s.buf, c.mean, c.rstd, c.dx.buf, c.dgamma, c.dbeta), want):
        assert torch.equal(t, w)
    # two graphs that run at the same time, with a workspace each, the rows of one of them changed between replays
    other = Case(P, shape, "bf16", "bf16", "silu", True, seed=1).forward().backward()
    other_want = [t.clone() for t in (other.dx.buf, other.dgamma, other.dbeta)]
    graphs, outs = [], []
    for k in (c, other):
        dx, dg, db = k.dx.buf, torch.empty_like(k.gamma), torch.empty_like(k.beta)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            P.lsgd_layernorm_forward(k.x.t, k.gamma, k.beta, k.y.t, k.mean, k.rstd, *shape, r=k.r.t, s=k.s.t, **k.kw())
            P.lsgd_layernorm_backward(k.s.t, None, k.dy.t, k.gamma, k.beta, k.mean, k.rstd, k.dx.t, dg, db, *shape, ds=k.ds.t, **k.kw())
        graphs.append(g)
        outs.append((dx, dg, db))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for (dx, dg, db), w, k in zip(outs, (want[4:], other_want), (c, other)):
        assert torch.equal(dx, w[0]) and torch.equal(dg[k.pick], w[1]) and torch.equal(db[k.pick], w[2])


# dgamma and dbeta over many rows of equal gradients, whose roundings all go one way.  Additions that a value passes through: 64 rows of
# a segment, the segments (or the root of the rows, twice), 8 merges of teams, 64 ranges of a thread and 5 merges.
@pytest.mark.gpu
@pytest.mark.parametrize("shape,additions", [((1, 300000, 640), 64 + 16 + 8 + 69), ((2, 700000, 16), 64 + 64 + 8 + 69), ((1, 40000, 4200), 64 + 16 + 69),
                                             ((1, 9_000_000, 24), 2 * 64 + 8 + 69)])
def test_sums_over_many_rows(P, shape, additions):
    import torch

    G, Rn, C = shape
    gen = torch.Generator(device="cuda").manual_seed(C)
    x = torch.randn(G * Rn, C, generator=gen, device="cuda").bfloat16()
    gamma = torch.ones(G, C, device="cuda")
    dy = torch.full((G * Rn, C), 0.1, device="cuda")
    mean, rstd = torch.zeros(G * Rn, device="cuda"), torch.ones(G * Rn, device="cuda")  # xh = x, without a rounding
    dx, dgamma, dbeta = torch.empty_like(x), torch.empty(G, C, device="cuda"), torch.empty(G, C, device="cuda")
    P.lsgd_layernorm_backward(x, None, dy, gamma, gamma, mean, rstd, dx, dgamma, dbeta, *shape)
    torch.cuda.synchronize()
    v = float(np.float32(0.1))
    assert (dbeta.double() / (v * Rn) - 1).abs().max() <= additions * U32
    for k in range(G):
        rows = x[k * Rn:(k + 1) * Rn]
        want = sum(r.double().sum(0) for r in rows.split(1 << 18)) * v
        size = sum(r.double().abs().sum(0) for r in rows.split(1 << 18)) * v
        assert ((dgamma[k].double() - want).abs() <= (additions + 1) * U32 * size).all()
    assert P.lsgd_device_status() == P.OK


@pytest.mark.gpu
@pytest.mark.parametrize("C", [32768, 4096, 1000])
def test_offsets_beyond_32_bits(P, C):
    import torch

    Rn = (1 << 31) // C + 77
    x = torch.empty(Rn, C, dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(C)
    block = torch.randn(64, C, generator=gen, device="cuda").bfloat16()
    x[:64], x[-64:] = block, block
    x[64:-64] = 1.0
    y, dx = torch.empty_like(x), torch.empty_like(x)
    gamma, beta = torch.rand(1, C, generator=gen, device="cuda") + 0.5, torch.randn(1, C, generator=gen, device="cuda")
    mean, rstd = torch.empty(Rn, device="cuda"), torch.empty(Rn, device="cuda")
    P.lsgd_layernorm_forward(x, gamma, beta, y, mean, rstd, 1, Rn, C)
    dg, db = torch.empty(1, C, device="cuda"), torch.empty(1, C, device="cuda")
    P.lsgd_layernorm_backward(x, None, x, gamma, beta, mean, rstd, dx, dg, db, 1, Rn, C)
    assert torch.equal(y[:64], y[-64:]) and torch.equal(dx[:64], dx[-64:]) and torch.equal(mean[:64], mean[-64:])
    small = Case(P, (1, 64, C), "bf16", "bf16")
    small.x.set(block.float())
    small.gamma, small.beta = gamma.view(-1).clone(), beta.view(-1).clone()
    small.forward()
    assert torch.equal(small.y.rows(), y[:64])
    small.check_forward()
    assert P.lsgd_device_status() == P.OK
