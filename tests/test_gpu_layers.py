"""conef_dropout_*, conef_norm_* and conef_mx_* on the GPU against the plain 64-bit statement of layers_ref.

Dropout and quantisation are compared bit for bit: every value is one or two fp32 operations, which the reference repeats.
The norm's and the product's tolerances follow from the number of roundings on the way to a value (u = 2^-24, a bf16 result
2^-8 of itself more) and are stated where they are used."""
import numpy as np
import pytest

import layers_ref as R

pytestmark = pytest.mark.gpu

SEED, STEP = 0x0123456789ABCDEF, (3 << 32) + 11
U = R.U32


@pytest.fixture(scope="module")
def env():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    from paper_2312_08538_amd import binding as B

    B.lib()
    return torch, B


def rng_of(*key):
    return np.random.default_rng([2024, *key])


class Strided:
    """A rows x cols matrix on the GPU inside a larger buffer: `skip` elements before it, `gap` behind every row, all of them a
    canary that has to survive."""
    CANARY = 77.0

    def __init__(self, torch, rows, cols, bf16, skip=0, gap=0, values=None):
        self.pitch, self.shape, self.skip = cols + gap, (rows, cols), skip
        dt = torch.bfloat16 if bf16 else torch.float32
        self.flat = torch.full((skip + rows * self.pitch + 16,), self.CANARY, dtype=dt, device="cuda:0")
        self.t = self.flat[skip:skip + rows * self.pitch].view(rows, self.pitch)[:, :cols]
        if values is not None:
            self.t.copy_(torch.from_numpy(np.ascontiguousarray(values, np.float32)).cuda())

    def numpy(self):
        return self.t.float().cpu().numpy()

    def check_canary(self):
        f = self.flat.clone()
        f[self.skip:self.skip + self.shape[0] * self.pitch].view(self.shape[0], self.pitch)[:, :self.shape[1]] = self.CANARY
        assert bool((f == self.CANARY).all()), "written outside the matrix"


def same_bits(a, b):
    a, b = np.ascontiguousarray(a, np.float32), np.ascontiguousarray(b, np.float32)
    nan = np.isnan(a)
    assert np.array_equal(nan, np.isnan(b))
    assert np.array_equal(a[~nan], b[~nan])


# ---------------------------------------------------------------------------------------------- dropout
DROP_SHAPES = [(1, 1), (1, 7), (3, 8), (5, 9), (1, 768), (130, 1001), (257, 64), (1000, 3), (64, 4096), (2, 40000)]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("rows,cols", DROP_SHAPES)
@pytest.mark.parametrize("skip,gap", [(0, 0), (3, 5)])
def test_dropout_bits(env, rows, cols, bf16, skip, gap):
    torch, B = env
    g = rng_of(rows, cols)
    x, r = (R.rounded(g.standard_normal((rows, cols)), bf16) for _ in range(2))
    for p, site in ((0.1, 0), (0.5, 3), (0.0, 1), (0.999999, 2)):
        d = B.conef_drop(p=p, site=site, seed=SEED, step=STEP)
        dx, dr, dy = (Strided(torch, rows, cols, bf16, skip, gap, v) for v in (x, r, np.zeros_like(x)))
        B.conef_dropout_forward(d, dx.t, dr.t, dy.t, B.Model.stream_handle())
        same_bits(dy.numpy(), R.dropped_sum(x, r, p, SEED, site, STEP, bf16))
        dy.check_canary()
        B.conef_dropout_forward(d, dx.t, None, dy.t, B.Model.stream_handle())
        alone = R.dropped_sum(x, None, p, SEED, site, STEP, bf16)
        same_bits(dy.numpy(), alone)
        B.conef_dropout_backward(d, dx.t, dx.t, B.Model.stream_handle())          # in place
        same_bits(dx.numpy(), alone)
        dx.check_canary()


def test_dropout_of_what_is_not_finite(env):
    torch, B = env
    x = torch.full((4, 4096), float("nan"), device="cuda:0")
    x[1] = float("inf")
    y = torch.empty_like(x)
    B.conef_dropout_forward(B.conef_drop(p=0.5, site=0, seed=SEED, step=STEP), x, None, y, B.Model.stream_handle())
    keep, _ = R.keep_and_scale((4, 4096), 0.5, SEED, 0, STEP)
    got = y.cpu().numpy()
    assert (got[~keep] == 0).all() and np.isnan(got[[0, 2, 3]][keep[[0, 2, 3]]]).all() and np.isposinf(got[1][keep[1]]).all()


def test_dropout_keeps_its_share_and_changes_with_site_step_and_seed(env):
    torch, B = env
    x = torch.ones(1024, 1024, device="cuda:0")
    n, p, masks = x.numel(), 0.3, []
    for site, seed, step in ((0, 1, 0), (1, 1, 0), (0, 2, 0), (0, 1, 1), (0, 1, 1 << 32)):
        y = torch.empty_like(x)
        B.conef_dropout_forward(B.conef_drop(p=p, site=site, seed=seed, step=step), x, None, y, B.Model.stream_handle())
        m = y != 0
        masks.append(m)
        # a binomial count within six standard deviations
        assert abs(int(m.sum()) - n * (1 - p)) < 6 * (n * p * (1 - p)) ** 0.5
    for i in range(1, len(masks)):
        # independent masks agree in a share (1 - p)^2 + p^2 of their places
        agree = float((masks[0] == masks[i]).float().mean())
        assert abs(agree - ((1 - p) ** 2 + p ** 2)) < 6 * 0.5 / n ** 0.5


# ---------------------------------------------------------------------------------------------- layer norm
NORM_SHAPES = [(1, 1), (3, 2), (5, 7), (4, 8), (7, 9), (2, 63), (300, 64), (9, 65), (5, 511), (6, 512), (1030, 513), (1, 768), (33, 1001),
               (4, 1024), (3, 1025), (1, 2048), (700, 2049), (2, 4096), (3, 5003), (5, 8192), (2, 8193), (3, 16384), (2, 16385), (3, 20001),
               (600, 3071), (2, 3073), (3, 4097), (2, 5120), (5, 5121), (2, 6144), (300, 6145), (3, 7168), (800, 7169), (1100, 1500), (1500, 2500),
               (20000, 5), (17001, 33), (16, 128), (9000, 129), (2049, 255), (40, 257), (300, 12288), (3, 12289)]


def norm_inputs(rows, cols, bf16, key=0):
    g = rng_of(rows, cols, key)
    x = R.rounded(g.standard_normal((rows, cols)) * 2 + 0.7, bf16)
    gamma = np.float32(1 + 0.2 * g.standard_normal(cols))
    beta = np.float32(0.2 * g.standard_normal(cols))
    return g, x, gamma, beta


def depth(cols):
    """Most additions on a value's way into a row's sum: 64 in a lane's registers (wider rows: an eighth of its share of a row), six across a wave, two across
    a workgroup."""
    return max(64, cols // 256 + 8) + 8


def y_tolerance(z, gamma, beta, eps, bf16):
    """The mean of n values is off by at most (depth + 2) u mean|z|; a centred value by that and one rounding; the variance, a mean of squares, by
    twice the relative error of the centred values and depth more roundings; y takes three more."""
    y, mean, rstd, hat = R.norm(z, gamma, beta, eps)
    d = depth(z.shape[1])
    mean_err = (d + 2) * U * np.abs(z).mean(1)
    hat_err = rstd[:, None] * (mean_err[:, None] + U * np.abs(z - mean[:, None]))
    # rstd: half the variance's relative error, and that of the centred values as a whole
    rstd_rel = (d / 2 + 6) * U + rstd * mean_err
    err = np.abs(gamma) * (hat_err + np.abs(hat) * (rstd_rel[:, None] + 3 * U)) + 2 * U * (np.abs(y) + np.abs(hat * gamma))
    return err * 1.01 + (np.abs(y) * R.U16 * 1.01 if bf16 else 0), mean_err + U * np.abs(mean), rstd * (rstd_rel + 2 * U)


def column_vector(torch, v):
    return torch.from_numpy(np.ascontiguousarray(v, np.float32)).cuda()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("rows,cols", NORM_SHAPES)
@pytest.mark.parametrize("skip,gap,p,residual", [(0, 0, None, False), (1, 3, 0.2, True), (0, 0, 0.5, False), (5, 0, None, True)])
def test_norm_forward(env, rows, cols, bf16, skip, gap, p, residual):
    torch, B = env
    g, x, gamma, beta = norm_inputs(rows, cols, bf16)
    r = R.rounded(g.standard_normal((rows, cols)) + 0.3, bf16) if residual else None
    fused = p is not None or residual
    d = B.conef_drop(p=p, site=4, seed=SEED, step=STEP) if p is not None else None
    dx, dy = Strided(torch, rows, cols, bf16, skip, gap, x), Strided(torch, rows, cols, bf16, skip, gap)
    dr = Strided(torch, rows, cols, bf16, gap, skip, r) if residual else None
    dz = Strided(torch, rows, cols, bf16, skip + 2, gap) if fused else None
    mean, rstd = torch.full((rows,), 7.0, device="cuda:0"), torch.full((rows,), 7.0, device="cuda:0")
    eps = 1e-5
    B.conef_norm_forward(d, eps, dx.t, dr.t if residual else None, column_vector(torch, gamma), column_vector(torch, beta),
                         dz.t if fused else None, dy.t, mean, rstd, B.Model.stream_handle())
    z = x
    if fused:
        z = R.dropped_sum(x, r, p or 0.0, SEED, 4, STEP, bf16)
        same_bits(dz.numpy(), z)
        dz.check_canary()
    y, m64, s64, _ = R.norm(z, gamma, beta, eps)
    ty, tm, ts = y_tolerance(z.astype(np.float64), gamma, beta, eps, bf16)
    assert (np.abs(mean.cpu().numpy() - m64) <= tm).all()
    assert (np.abs(rstd.cpu().numpy() - s64) <= ts).all()
    assert (np.abs(dy.numpy() - y) <= ty).all()
    dy.check_canary()
    dx.check_canary()


def test_norm_forward_without_statistics_and_in_place(env):
    torch, B = env
    _, x, gamma, beta = norm_inputs(37, 1000, False)
    a, out = column_vector(torch, x), torch.empty(37, 1000, device="cuda:0")
    G, Bt = column_vector(torch, gamma), column_vector(torch, beta)
    B.conef_norm_forward(None, 1e-5, a, None, G, Bt, None, out, None, None, B.Model.stream_handle())
    B.conef_norm_forward(None, 1e-5, a, None, G, Bt, None, a, None, None, B.Model.stream_handle())
    assert torch.equal(a, out)


def test_norm_of_constant_rows_large_offsets_and_what_is_not_finite(env):
    torch, B = env
    cols = 3000
    x = np.zeros((6, cols), np.float32)
    x[1] = 5.0
    x[2] = 1e4 + rng_of(1).standard_normal(cols)              # a variance that a sum of squares would lose
    x[3] = rng_of(2).standard_normal(cols) * 1e-20
    x[4, 17] = np.nan
    x[5, 0] = np.inf
    gamma, beta = np.float32(rng_of(3).standard_normal(cols)), np.float32(rng_of(4).standard_normal(cols))
    a, y = column_vector(torch, x), torch.empty(6, cols, device="cuda:0")
    B.conef_norm_forward(None, 1e-5, a, None, column_vector(torch, gamma), column_vector(torch, beta), None, y, None, None,
                         B.Model.stream_handle())
    got = y.cpu().numpy()
    ty, _, _ = y_tolerance(x[:4].astype(np.float64), gamma, beta, 1e-5, False)
    want = R.norm(x[:4], gamma, beta, 1e-5)[0]
    assert (np.abs(got[:4] - want) <= ty).all()
    assert np.isnan(got[4]).all() and np.isnan(got[5]).all()


def back_tolerance(dy, hat, a, gamma, rstd, dz, rows, cols, parts, bf16):
    """hat and a are good to 3 u and one rounding; the two means take depth more; dz four roundings on top.  dgamma, dbeta: as many fp32
    additions as a workgroup has rows (and groups), the rest in fp64."""
    d = depth(cols)
    s = rstd.astype(np.float64)[:, None]
    m0, m1 = np.abs(a).mean(1, keepdims=True), np.abs(a * hat).mean(1, keepdims=True)
    err = s * (3 * U * np.abs(a) + (d + 4) * U * m0 + (d + 9) * U * np.abs(hat) * m1) + 4 * U * np.abs(dz)
    n = -(-rows // parts) + 6
    return (err * 1.01 + (np.abs(dz) * R.U16 * 1.01 if bf16 else 0), (n + 5) * U * (np.abs(dy) * np.abs(hat)).sum(0) * 1.01,
            (n + 1) * U * np.abs(dy).sum(0) * 1.01)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("rows,cols", NORM_SHAPES)
@pytest.mark.parametrize("skip,gap,p,residual", [(0, 0, None, False), (1, 3, 0.2, True), (0, 0, 0.5, False), (5, 0, None, True)])
def test_norm_backward(env, rows, cols, bf16, skip, gap, p, residual):
    torch, B = env
    g, z, gamma, beta = norm_inputs(rows, cols, bf16, 1)
    dy = R.rounded(g.standard_normal((rows, cols)), bf16)
    dz_in = R.rounded(g.standard_normal((rows, cols)), bf16) if residual else None
    _, m64, s64, _ = R.norm(z, gamma, beta, 1e-5)
    mean, rstd = np.float32(m64), np.float32(s64)
    d = B.conef_drop(p=p, site=4, seed=SEED, step=STEP) if p is not None else None
    D = {k: Strided(torch, rows, cols, bf16, skip, gap, v) for k, v in (("dy", dy), ("z", z), ("dz", None), ("dx", None))}
    if residual:
        D["dz_in"] = Strided(torch, rows, cols, bf16, gap, skip, dz_in)
    dgamma, dbeta = torch.full((cols,), 7.0, device="cuda:0"), torch.full((cols,), 7.0, device="cuda:0")
    room = B.conef_norm_workspace(rows, cols)
    ws = torch.full((room,), 0xFF, dtype=torch.uint8, device="cuda:0")
    args = (D["dy"].t, D["z"].t, column_vector(torch, gamma), column_vector(torch, mean), column_vector(torch, rstd),
            D["dz_in"].t if residual else None)
    B.conef_norm_backward(d, *args, D["dz"].t, D["dx"].t if d else None, dgamma, dbeta, ws, B.Model.stream_handle())
    want, wg, wb, hat, a = R.norm_back(dy, z, gamma, mean, rstd)
    if residual:
        want = want + dz_in
    parts = room // (8 * cols)
    tz, tg, tb = back_tolerance(dy, hat, a, gamma, rstd, want, rows, cols, parts, bf16)
    assert (np.abs(D["dz"].numpy() - want) <= tz).all()
    assert (np.abs(dgamma.cpu().numpy() - wg) <= tg).all()
    assert (np.abs(dbeta.cpu().numpy() - wb) <= tb).all()
    if d:
        keep, s = R.keep_and_scale((rows, cols), p, SEED, 4, STEP)
        assert (np.abs(D["dx"].numpy() - np.where(keep, want * s, 0.0)) <= np.where(keep, tz * s + 2 * U * np.abs(want * s), 0.0)).all()
    for m in D.values():
        m.check_canary()
    # each output alone, and dz in place of what it is computed from, give the same bits
    for only in ("dz", "columns", "in place"):
        dz2 = Strided(torch, rows, cols, bf16, skip, gap)
        g2, b2 = torch.zeros_like(dgamma), torch.zeros_like(dbeta)
        if only == "dz":
            B.conef_norm_backward(d, *args, dz2.t, None, None, None, None, B.Model.stream_handle())
            assert torch.equal(dz2.t, D["dz"].t)
        elif only == "columns":
            B.conef_norm_backward(d, *args, None, None, g2, b2, ws, B.Model.stream_handle())
            assert torch.equal(g2, dgamma) and torch.equal(b2, dbeta)
        else:
            B.conef_norm_backward(d, *args, D["dy"].t, None, g2, b2, ws, B.Model.stream_handle())
            assert torch.equal(D["dy"].t, D["dz"].t) and torch.equal(g2, dgamma) and torch.equal(b2, dbeta)


def test_norm_backward_of_no_rows_is_zero(env):
    torch, B = env
    none = torch.empty(0, 100, device="cuda:0")
    g, b = torch.ones(100, device="cuda:0"), torch.ones(100, device="cuda:0")
    e = torch.empty(0, device="cuda:0")
    B.conef_norm_backward(None, none, none, torch.ones(100, device="cuda:0"), e, e, None, None, None, g, b, None, B.Model.stream_handle())
    assert not bool(g.any()) and not bool(b.any())


@pytest.mark.parametrize("rows,cols", [(5, 96), (3, 700), (2, 3000)])
def test_norm_gradient_against_differences(env, rows, cols):
    """<gradient, v> against (L(+h v) - L(-h v)) / 2h of L = sum(w y), taken with the library's own forward pass in fp32: the dropout
    and the residual included.  The difference's own error: h^2 times third derivatives (all of order 1: 1e-4 of the terms' sum at h = 1e-2),
    and fp32 roundings of y, u sqrt(n) |w y| / h, 1e-5 of it."""
    torch, B = env
    g, x, gamma, beta = norm_inputs(rows, cols, False, 5)
    r, w = np.float32(g.standard_normal((rows, cols))), np.float32(g.standard_normal((rows, cols)))
    d, eps, st = B.conef_drop(p=0.25, site=1, seed=SEED, step=STEP), 1e-5, B.Model.stream_handle()
    T = lambda v: column_vector(torch, v)                      # noqa: E731

    def forward(x, r, gamma, beta):
        z, y = torch.empty(rows, cols, device="cuda:0"), torch.empty(rows, cols, device="cuda:0")
        mean, rstd = torch.empty(rows, device="cuda:0"), torch.empty(rows, device="cuda:0")
        B.conef_norm_forward(d, eps, T(x), T(r), T(gamma), T(beta), z, y, mean, rstd, st)
        return z, y, mean, rstd

    def loss(*v):
        return float((forward(*v)[1].cpu().numpy().astype(np.float64) * w).sum())

    z, _, mean, rstd = forward(x, r, gamma, beta)
    dz, dx = torch.empty_like(z), torch.empty_like(z)
    dg, db = torch.empty(cols, device="cuda:0"), torch.empty(cols, device="cuda:0")
    ws = torch.empty(B.conef_norm_workspace(rows, cols), dtype=torch.uint8, device="cuda:0")
    B.conef_norm_backward(d, T(w), z, T(gamma), mean, rstd, None, dz, dx, dg, db, ws, st)
    at, h = [x, r, gamma, beta], 1e-2
    for k, grad in enumerate((dx, dz, dg, db)):
        v = np.float32(g.standard_normal(at[k].shape))
        up, down = list(at), list(at)
        up[k], down[k] = np.float32(at[k] + h * v), np.float32(at[k] - h * v)
        numeric = (loss(*up) - loss(*down)) / (2 * h)
        terms = grad.cpu().numpy().astype(np.float64) * v
        assert abs(numeric - terms.sum()) <= 1e-3 * np.sqrt((terms ** 2).sum()) * 3 + 1e-4 * np.abs(terms).sum(), k


# ---------------------------------------------------------------------------------------------- 4-bit floating point
MX_SHAPES = [(1, 1), (1, 31), (3, 32), (2, 33), (15, 64), (16, 127), (17, 128), (63, 129), (64, 256), (65, 100), (130, 515), (1, 2048),
             (300, 7), (128, 128), (129, 384), (1300, 3500)]


def mx_input(rows, cols, bf16):
    """Values over many magnitudes, ties of the grid, zeros (whole blocks of them), the smallest and the largest numbers, infinities, NaN."""
    g = rng_of(rows, cols, 9)
    x = g.standard_normal((rows, cols)) * np.exp2(g.integers(-30, 30, (rows, 1)).astype(float))
    flat = x.reshape(-1)
    n = flat.size
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0, 6.5, -0.25, -5.0, -0.0])
    flat[::5] = np.resize(ties, flat[::5].size)
    if n > 200:
        flat[64:100] = 0.0
        flat[100] = -0.0
        flat[n // 2:n // 2 + 20] = np.resize([1e-45, 3e-39, 1.2e-38, 2e-38, 7e-38, 3.4e38, -3.3e38], 20)
        flat[n // 3] = np.inf
        flat[n // 4] = np.nan
    return R.rounded(x.astype(np.float32), bf16)


def packed_numpy(pair):
    return tuple(t.cpu().numpy() for t in pair)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("rows,cols", MX_SHAPES)
@pytest.mark.parametrize("stochastic", [False, True])
@pytest.mark.parametrize("skip,gap", [(0, 0), (1, 3)])
def test_quantise_bits(env, rows, cols, bf16, stochastic, skip, gap):
    torch, B = env
    x = mx_input(rows, cols, bf16)
    dx = Strided(torch, rows, cols, bf16, skip, gap, x)
    mode, site = (B.MX_STOCHASTIC, 6) if stochastic else (B.MX_NEAREST, 0)
    u = R.draws(rows, cols, R.MX_ROWS + site, SEED, STEP) if stochastic else None
    ut = R.draws(cols, rows, R.MX_COLS + site, SEED, STEP) if stochastic else None
    by_rows, by_cols = R.mx_encode(x, u), R.mx_encode(x.T, ut)
    for which in ("rows", "cols", "both"):
        p = B.mx_alloc(rows, cols) if which != "cols" else None
        pt = B.mx_alloc(cols, rows) if which != "rows" else None
        for pair in (p, pt):
            if pair:
                pair[0].fill_(0xA5)                       # every byte is written, those that fill up the operand too
                pair[1].fill_(0xA5)
        B.conef_mx_quantise(dx.t, mode, SEED, site, STEP, p, pt, B.Model.stream_handle())
        for pair, want in ((p, by_rows), (pt, by_cols)):
            if pair:
                for got, exp in zip(packed_numpy(pair), R.mx_pack(*want)):
                    assert np.array_equal(got, exp), which
        if p:
            for kind in (False, True):
                out = Strided(torch, rows, cols, kind, skip, gap)
                B.conef_mx_dequantise(p, out.t, B.Model.stream_handle())
                same_bits(out.numpy(), R.mx_decode(*by_rows))
                out.check_canary()
    dx.check_canary()


def test_stochastic_rounding_is_unbiased(env):
    """The mean over 4096 steps of a value's rounding against the value: within six standard deviations (of a variable that takes the two
    neighbours) and 2^-16 of their distance."""
    torch, B = env
    g = rng_of(12)
    x = np.float32(g.uniform(-6, 6, (4, 64)))
    x[:, ::32] = 6.0                                     # fixes the scale at 1
    dx, out, p = column_vector(torch, x), torch.empty(4, 64, device="cuda:0"), B.mx_alloc(4, 64)
    total, n = np.zeros((4, 64)), 4096
    acc = torch.zeros(4, 64, dtype=torch.float64, device="cuda:0")
    for step in range(n):
        B.conef_mx_quantise(dx, B.MX_STOCHASTIC, SEED, 0, step, p, None, B.Model.stream_handle())
        B.conef_mx_dequantise(p, out, B.Model.stream_handle())
        acc += out
    total = acc.cpu().numpy() / n
    a = np.abs(x.astype(np.float64))
    low = np.searchsorted(R.GRID, a, side="right") - 1
    up = np.minimum(low + 1, 7)
    gap = R.GRID[up] - R.GRID[low]
    f = np.where(gap > 0, (a - R.GRID[low]) / np.where(gap > 0, gap, 1), 0)
    assert (np.abs(np.abs(total) - a) <= 6 * gap * np.sqrt(f * (1 - f) / n) + gap * 2.0 ** -16 + 1e-12).all()


PRODUCT_SHAPES = [(1, 1, 1), (1, 16, 32), (3, 5, 33), (16, 16, 128), (8, 300, 700), (17, 1, 129), (64, 64, 256), (65, 130, 385), (128, 128, 1024),
                  (130, 257, 2049), (300, 513, 515), (1, 2048, 4096), (7, 1000, 8192), (40, 64, 20000), (256, 256, 512), (513, 768, 1280),
                  (1100, 1300, 900), (2048, 16, 640), (33, 4100, 1500)]


def product_inputs(m, n, k):
    g = rng_of(m, n, k)
    x, w = g.standard_normal((m, k)) * np.exp(g.standard_normal((m, 1))), g.standard_normal((n, k)) / np.sqrt(k)
    return R.mx_encode(x.astype(np.float32)), R.mx_encode(w.astype(np.float32))


def on_gpu(torch, code):
    return tuple(torch.from_numpy(v).cuda() for v in R.mx_pack(*code))


def product_tolerance(A, W, k):
    """Products are exact; a block's and an instruction's sums and the additions to the running sum round once each, to 2^-23 of the sum of
    magnitudes so far at the most, five an instruction of 128 elements; plus those of cutting the axis and of the factors."""
    return (5 * (-(-k // 128)) + 24) * 2.0 ** -23 * (np.abs(A) @ np.abs(W).T)


@pytest.mark.parametrize("m,n,k", PRODUCT_SHAPES)
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("alpha,beta", [(1.0, 0.0), (0.125, 1.0)])
def test_product(env, m, n, k, bf16, alpha, beta):
    torch, B = env
    a, b = product_inputs(m, n, k)
    A, W = R.mx_decode(*a), R.mx_decode(*b)
    old = R.rounded(rng_of(m, n).standard_normal((m, n)), bf16)
    if beta == 0.0:
        old[:] = np.nan                                   # what is not to be read
    c = Strided(torch, m, n, bf16, 1, 2, old)
    room = B.conef_mx_product_workspace(m, n, k)
    ws = torch.full((room,), 0xFF, dtype=torch.uint8, device="cuda:0") if room else None
    B.conef_mx_product(on_gpu(torch, a), on_gpu(torch, b), k, alpha, beta, c.t, ws, B.Model.stream_handle())
    want = alpha * (A @ W.T) + (beta * old.astype(np.float64) if beta else 0)
    tol = alpha * product_tolerance(A, W, k) + 2 * U * (np.abs(want) + (np.abs(old) if beta else 0))
    assert (np.abs(c.numpy() - want) <= tol + (np.abs(want) * R.U16 * 1.01 if bf16 else 0)).all()
    c.check_canary()


@pytest.mark.parametrize("m,n,k", [(2000, 1700, 300), (3500, 3600, 1537), (3500, 3600, 4200), (8200, 8190, 1537), (1000, 65700, 1700),
                                   (60, 16400, 1990)])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("alpha,beta", [(1.0, 0.0), (0.125, 1.0)])
def test_large_product(env, m, n, k, bf16, alpha, beta):
    """As above, with the sums in 64 bits on the device: every tile size, odd and even numbers of pieces, several tiles a workgroup."""
    torch, B = env
    a, b = product_inputs(m, n, k)
    A, W = (torch.from_numpy(R.mx_decode(*v)).cuda().double() for v in (a, b))
    c = torch.full((m, n + 3), float("nan"), dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda:0")
    if beta:
        c.normal_()
    out, old = c[:, :n], c.double()
    room = B.conef_mx_product_workspace(m, n, k)
    ws = torch.full((room,), 0xFF, dtype=torch.uint8, device="cuda:0") if room else None
    B.conef_mx_product(on_gpu(torch, a), on_gpu(torch, b), k, alpha, beta, out, ws, B.Model.stream_handle())
    want = alpha * torch.mm(A, W.t())
    far = alpha * torch.mm(A.abs(), W.abs().t()) * ((5 * (-(-k // 128)) + 24) * 2.0 ** -23)
    if beta:
        want += beta * old[:, :n]
        far += 2 * U * old[:, :n].abs()
    far += want.abs() * (2 * U + (R.U16 * 1.01 if bf16 else 0))
    assert bool(((out.double() - want).abs() <= far).all())
    rest, was = c[:, n:].double(), old[:, n:]
    assert bool(((rest == was) | (rest.isnan() & was.isnan())).all())


def test_product_of_nothing(env):
    torch, B = env
    empty = tuple(torch.empty(0, dtype=torch.uint8, device="cuda:0") for _ in range(2))
    c = torch.full((5, 9), 3.0, device="cuda:0")
    B.conef_mx_product(empty, empty, 0, 1.0, 0.5, c, None, B.Model.stream_handle())
    assert bool((c == 1.5).all())
    c.fill_(float("nan"))
    B.conef_mx_product(empty, empty, 0, 1.0, 0.0, c, None, B.Model.stream_handle())
    assert bool((c == 0).all())


@pytest.mark.parametrize("m,n,k", [(5, 40, 200), (200, 300, 1000), (16, 64, 9000)])
def test_product_with_scales_of_nan_and_zero_operands(env, m, n, k):
    torch, B = env
    (ca, sa), b = product_inputs(m, n, k)
    sa = sa.copy()
    sa[m // 2, -1] = 255
    ca = ca.copy()
    ca[0] = 0
    c = torch.empty(m, n, device="cuda:0")
    room = B.conef_mx_product_workspace(m, n, k)
    ws = torch.empty(room, dtype=torch.uint8, device="cuda:0")
    B.conef_mx_product(on_gpu(torch, (ca, sa)), on_gpu(torch, b), k, 1.0, 0.0, c, ws, B.Model.stream_handle())
    got = c.cpu().numpy()
    assert np.isnan(got[m // 2]).all() and (got[0] == 0).all()
    rest = [i for i in range(m) if i != m // 2]
    assert np.isfinite(got[rest]).all()


def test_product_runs_the_same_twice_and_on_another_stream(env):
    torch, B = env
    m, n, k = 96, 200, 6000
    a, b = (on_gpu(torch, v) for v in product_inputs(m, n, k))
    ws = torch.empty(B.conef_mx_product_workspace(m, n, k), dtype=torch.uint8, device="cuda:0")
    c, c2 = torch.empty(m, n, device="cuda:0"), torch.empty(m, n, device="cuda:0")
    B.conef_mx_product(a, b, k, 1.0, 0.0, c, ws, B.Model.stream_handle())
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        B.conef_mx_product(a, b, k, 1.0, 0.0, c2, ws, B.Model.stream_handle())
    side.synchronize()
    assert torch.equal(c, c2)


@pytest.mark.parametrize("rows,cols", [(40, 900), (700, 1024)])
def test_a_captured_step_replays_to_the_eager_results(env, rows, cols):
    """Norm forward and backward, quantisation and a product in one graph, replayed three times with eager work in between."""
    torch, B = env
    g, x, gamma, beta = norm_inputs(rows, cols, False, 6)
    T = lambda v: column_vector(torch, v)                      # noqa: E731
    X, Rr, G, Bt, W = T(x), T(x * 0.5), T(gamma), T(beta), T(g.standard_normal((192, cols)))
    d = B.conef_drop(p=0.1, site=2, seed=SEED, step=STEP)
    out = {k: torch.zeros(rows, cols, device="cuda:0") for k in ("z", "y", "dz", "dx")}
    out.update(mean=torch.zeros(rows, device="cuda:0"), rstd=torch.zeros(rows, device="cuda:0"), dg=torch.zeros(cols, device="cuda:0"),
               db=torch.zeros(cols, device="cuda:0"), c=torch.zeros(rows, 192, device="cuda:0"))
    ws = torch.zeros(max(B.conef_norm_workspace(rows, cols), B.conef_mx_product_workspace(rows, 192, cols)), dtype=torch.uint8, device="cuda:0")
    yq, wq = B.mx_alloc(rows, cols), B.mx_alloc(192, cols)

    def step():
        st = B.Model.stream_handle()
        B.conef_norm_forward(d, 1e-5, X, Rr, G, Bt, out["z"], out["y"], out["mean"], out["rstd"], st)
        B.conef_mx_quantise(out["y"], B.MX_STOCHASTIC, SEED, 0, 1, yq, None, st)
        B.conef_mx_quantise(W, B.MX_NEAREST, 0, 0, 0, wq, None, st)
        B.conef_mx_product(yq, wq, cols, 1.0, 0.0, out["c"], ws, st)
        B.conef_norm_backward(d, X, out["z"], G, out["mean"], out["rstd"], Rr, out["dz"], out["dx"], out["dg"], out["db"], ws, st)

    step()
    torch.cuda.synchronize()
    want = {k: v.clone() for k, v in out.items()}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        for v in out.values():
            v.zero_()
        ws.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for k in want:
            assert torch.equal(out[k], want[k]), k


# ---------------------------------------------------------------------------------------------- more than 2^31 elements
def test_elements_beyond_31_bits(env):
    """The last rows of matrices of 2.2e9 elements (everything before them zero): dropout, norm, quantisation, product."""
    torch, B = env
    rows, cols, tail = 66001, 33336, 3
    assert rows * cols > 2 ** 31 and (rows - tail) * cols > 2 ** 31
    st = B.Model.stream_handle()
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda:0")
    last = R.bf16(rng_of(31).standard_normal((tail, cols)).astype(np.float32))
    x[-tail:] = torch.from_numpy(last).cuda()
    y = torch.ones_like(x)
    B.conef_dropout_forward(B.conef_drop(p=0.25, site=0, seed=SEED, step=STEP), x, None, y, st)
    per = cols // 8
    # draws of the last rows alone: octets from (rows - tail) per on
    t = int(np.floor(0.25 * 65536 + 0.5))
    u = np.array([[R.philox(((rows - tail + i) * per + o, R.DROP, STEP & 0xFFFFFFFF, STEP >> 32), (SEED & 0xFFFFFFFF, SEED >> 32)) for o in range(0, per, 97)]
                  for i in range(tail)], dtype=np.uint64)
    halves = np.stack([u & np.uint64(0xFFFF), u >> np.uint64(16)], -1).reshape(tail, -1, 8).astype(np.int64)
    octets = last.reshape(tail, per, 8)[:, ::97]
    want = R.bf16(np.where(halves >= t, octets * np.float32(65536.0 / (65536 - t)), np.float32(0)))
    same_bits(y[-tail:].float().cpu().numpy().reshape(tail, per, 8)[:, ::97], want)
    assert not bool(y[:-tail].any())

    gamma, beta = torch.ones(cols, device="cuda:0"), torch.full((cols,), 0.5, device="cuda:0")
    B.conef_norm_forward(None, 1e-5, x, None, gamma, beta, None, y, None, None, st)
    ty, _, _ = y_tolerance(last.astype(np.float64), np.ones(cols), np.full(cols, 0.5), 1e-5, True)
    assert (np.abs(y[-tail:].float().cpu().numpy() - R.norm(last, 1.0, 0.5, 1e-5)[0]) <= ty).all()
    assert bool((y[:-tail] == 0.5).all())
    del y

    p = B.mx_alloc(rows, cols)
    B.conef_mx_quantise(x, B.MX_NEAREST, 0, 0, 0, p, None, st)
    del x
    code = R.mx_encode(last)
    n, k = 48, cols
    b = R.mx_encode(rng_of(32).standard_normal((n, k)).astype(np.float32))
    c = torch.full((rows, n), 7.0, device="cuda:0")
    B.conef_mx_product(p, on_gpu(torch, b), k, 1.0, 0.0, c, torch.empty(B.conef_mx_product_workspace(rows, n, k), dtype=torch.uint8, device="cuda:0"), st)
    A, W = R.mx_decode(*code), R.mx_decode(*b)
    assert (np.abs(c[-tail:].cpu().numpy() - A @ W.T) <= product_tolerance(A, W, k)).all()
    assert not bool(c[:-tail].any())
    del p, c

    m, n, k = 66001, 33336, 96
    a, b = R.mx_encode(rng_of(33).standard_normal((tail, k)).astype(np.float32)), R.mx_encode(rng_of(34).standard_normal((n, k)).astype(np.float32))
    codes, scales = np.zeros((m, k), np.uint8), np.zeros((m, k // 32), np.uint8)
    codes[-tail:], scales[-tail:] = a
    c = torch.full((m, n), 7.0, dtype=torch.bfloat16, device="cuda:0")
    B.conef_mx_product(on_gpu(torch, (codes, scales)), on_gpu(torch, b), k, 1.0, 0.0, c, None, st)
    A, W = R.mx_decode(*a), R.mx_decode(*b)
    want = A @ W.T
    assert (np.abs(c[-tail:].float().cpu().numpy() - want) <= product_tolerance(A, W, k) + np.abs(want) * R.U16 * 1.01).all()
    assert not bool(c[:-tail].any())


def test_every_operator_on_a_stream_of_its_own(env):
    """Inputs made on one stream, the calls on another that waits for it: the same bits as on one stream."""
    torch, B = env
    rows, cols = 300, 1000
    g, x, gamma, beta = norm_inputs(rows, cols, True, 8)
    d = B.conef_drop(p=0.3, site=3, seed=SEED, step=STEP)

    def calls():
        st = B.Model.stream_handle()
        bf = dict(dtype=torch.bfloat16, device="cuda:0")
        X, Rr = torch.from_numpy(x).cuda().bfloat16(), torch.from_numpy(x * 0.25).cuda().bfloat16()
        z, y, dz, dx, o = (torch.zeros(rows, cols, **bf) for _ in range(5))
        mean, rstd = torch.zeros(rows, device="cuda:0"), torch.zeros(rows, device="cuda:0")
        G, Bt = column_vector(torch, gamma), column_vector(torch, beta)
        dg, db = torch.zeros_like(G), torch.zeros_like(G)
        ws = torch.empty(max(B.conef_norm_workspace(rows, cols), B.conef_mx_product_workspace(rows, rows, cols)), dtype=torch.uint8, device="cuda:0")
        B.conef_norm_forward(d, 1e-5, X, Rr, G, Bt, z, y, mean, rstd, st)
        p, pt = B.mx_alloc(rows, cols), B.mx_alloc(cols, rows)
        B.conef_mx_quantise(y, B.MX_STOCHASTIC, SEED, 1, STEP, p, pt, st)
        B.conef_mx_dequantise(p, o, st)
        c, ct = torch.zeros(rows, rows, device="cuda:0"), torch.zeros(cols, cols, device="cuda:0")
        B.conef_mx_product(p, p, cols, 1.0, 0.0, c, ws, st)
        B.conef_mx_product(pt, pt, rows, 1.0, 0.0, ct, None, st)
        B.conef_norm_backward(d, y, z, G, mean, rstd, Rr, dz, dx, dg, db, ws, st)
        B.conef_dropout_backward(d, dz, dz, st)
        return [z, y, mean, rstd, o, c, ct, dz, dx, dg, db, *p, *pt]

    want = calls()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = calls()
    side.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_matrices_of_no_rows(env):
    """An empty batch goes through every call; its tensors have no address."""
    torch, B = env
    st = B.Model.stream_handle()
    d = B.conef_drop(p=0.25, site=0, seed=1, step=0)
    for dtype in (torch.float32, torch.bfloat16):
        e = torch.empty(0, 40, dtype=dtype, device="cuda:0")
        g, none = torch.ones(40, device="cuda:0"), torch.empty(0, device="cuda:0")
        B.conef_dropout_forward(d, e, e, e, st)
        B.conef_dropout_backward(d, e, e, st)
        for drop in (d, None):
            B.conef_norm_forward(drop, 1e-5, e, e, g, g, e, e, none, none, st)
            B.conef_norm_backward(drop, e, e, g, none, none, e, e, e if drop else None, None, None, None, st)
        q, qt = B.mx_alloc(0, 40), B.mx_alloc(40, 0)
        B.conef_mx_quantise(e, B.MX_STOCHASTIC, 1, 0, 0, q, qt, st)
        B.conef_mx_dequantise(q, e, st)
        B.conef_mx_product(q, B.mx_alloc(8, 40), 40, 1.0, 0.0, torch.empty(0, 8, dtype=dtype, device="cuda:0"), None, st)
        c = torch.ones(40, 40, dtype=dtype, device="cuda:0")
        B.conef_mx_product(qt, qt, 0, 1.0, 0.0, c, None, st)                       # a gradient of no tokens
        torch.cuda.synchronize()
        assert (c == 0).all()


def test_binding_refuses_device_tensors_that_do_not_fit(env):
    """None of these reaches a kernel."""
    torch, B = env
    st = B.Model.stream_handle()
    z = lambda *s, **k: torch.zeros(*s, device="cuda:0", **k)                      # noqa: E731
    d, x, v, m = B.conef_drop(p=0.25, site=0, seed=1, step=0), z(4, 8), z(8), z(4)
    q = B.mx_alloc(4, 8)
    bad = [lambda t=t: B.conef_dropout_backward(d, t, x, st) for t in (z(8, 4).t(), z(4, 8).double(), z(32), z(4, 16)[:, ::2], x.cpu())]
    bad += [lambda t=t: B.conef_dropout_forward(d, x, t, x, st) for t in (z(4, 9), x.bfloat16(), z(8, 4).t(), x.cpu())]
    bad += [lambda g=g: B.conef_norm_forward(None, 1e-5, x, None, g, v, None, x, None, None, st)
            for g in (z(7), z(16)[::2], v.bfloat16(), v.cpu(), z(1, 8))]
    bad += [lambda: B.conef_norm_backward(None, x, x, v, m, m, None, x, None, None, v, z(1), st),
            lambda: B.conef_norm_backward(None, x, x, v, m, m, None, x, None, None, v, None, st),
            lambda: B.conef_mx_quantise(z(4, 129), B.MX_NEAREST, 0, 0, 0, q, None, st),
            lambda: B.conef_mx_quantise(x, B.MX_NEAREST, 0, 0, 0, None, None, st),
            lambda: B.conef_mx_quantise(x, B.MX_NEAREST, 0, 0, 0, (q[0], q[1].cpu()), None, st),
            lambda: B.conef_mx_dequantise(q, z(65, 8), st),
            lambda: B.conef_mx_product(q, q, 129, 1.0, 0.0, z(4, 4), None, st),
            lambda: B.conef_mx_product(q, q, 8, 1.0, 0.0, z(4, 65), None, st)]
    for call in bad:
        with pytest.raises(B.ConefError) as e:
            call()
        assert e.value.code == B.EINVAL
