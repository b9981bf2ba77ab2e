"""conef_q8_*, conef_rms_* and conef_loss_* on the GPU against the plain 64-bit statement of step8_ref.

Quantisation is compared bit for bit, the norm's codes, too: it is computed in 64 bits and rounded once.  Other tolerances follow from the
number of roundings on the way to a value (u = 2^-24, a bf16 result 2^-8 of itself more) and are stated where they are used."""
import numpy as np
import pytest

import step8_ref as R
from test_gpu_layers import Strided, column_vector, env, packed_numpy, rng_of, same_bits  # noqa: F401  (env: the fixture)

pytestmark = pytest.mark.gpu

U, U16 = R.U32, R.U16
FORMS = [R.E4M3, R.E5M2]


def on_gpu(torch, code):
    return tuple(torch.from_numpy(v).cuda() for v in R.pack(*code))


def room_of(torch, n):
    return torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda:0") if n else None


# ---------------------------------------------------------------------------------------------- 8-bit floating point
SHAPES = [(1, 1), (1, 127), (3, 128), (2, 129), (15, 64), (16, 255), (17, 256), (63, 130), (64, 300), (65, 100), (130, 515), (1, 2048), (300, 7),
          (128, 128), (129, 384), (700, 1100)]


def q8_input(rows, cols, bf16, form):
    """Values over many magnitudes, ties of the grid, zeros (whole blocks of them), the smallest and the largest numbers, infinities, NaN."""
    g = rng_of(rows, cols, 90 + form)
    x = g.standard_normal((rows, cols)) * np.exp2(g.integers(-30, 30, (rows, 1)).astype(float)) * np.exp2(g.integers(-9, 1, (rows, cols)).astype(float))
    flat = x.reshape(-1)
    n = flat.size
    t = np.unique(np.abs(R.table(form)[R.table(form) <= R.LARGEST[form]]))
    ties = np.concatenate([(t[1:] + t[:-1]) / 2, -(t[1:] + t[:-1]) / 2, t, [R.LARGEST[form] * 1.001, -0.0]])
    if rows > 2:
        flat[:cols] = np.resize(ties, cols)                       # a row on the grid of one scale, and one past a power of it
        flat[cols:2 * cols] = np.resize(ties, cols) * 0.75
    if n > 1000:
        flat[640:896] = 0.0
        flat[700] = -0.0
        flat[n // 2:n // 2 + 20] = np.resize([1e-45, 3e-39, 1.2e-38, 2e-38, 7e-38, 3.4e38, -3.3e38], 20)
        flat[n // 3] = np.inf
        flat[n // 4] = np.nan
        flat[-5:] = [1e-40, 2e-38, 1e-38, -3e-37, 1e-36]
    return R.rounded(x.astype(np.float32), bf16)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("skip,gap", [(0, 0), (1, 3)])
def test_quantise_bits(env, rows, cols, bf16, form, skip, gap):  # noqa: F811
    torch, B = env
    x = q8_input(rows, cols, bf16, form)
    dx = Strided(torch, rows, cols, bf16, skip, gap, x)
    by_rows, by_cols = R.encode(x, form), R.encode(x.T, form)
    for which in ("rows", "cols", "both"):
        p = B.q8_alloc(rows, cols) if which != "cols" else None
        pt = B.q8_alloc(cols, rows) if which != "rows" else None
        for pair in (p, pt):
            if pair:
                pair[0].fill_(0xA5)                       # every byte is written, those that fill up the operand too
                pair[1].fill_(0xA5)
        B.conef_q8_quantise(dx.t, form, p, pt, B.Model.stream_handle())
        for pair, want in ((p, by_rows), (pt, by_cols)):
            if pair:
                for got, exp in zip(packed_numpy(pair), R.pack(*want)):
                    assert np.array_equal(got, exp), which
        for pair, want, shape in ((p, by_rows, (rows, cols)), (pt, by_cols, (cols, rows))):
            if pair:
                for kind in (False, True):
                    out = Strided(torch, *shape, kind, skip, gap)
                    B.conef_q8_dequantise(pair, form, out.t, B.Model.stream_handle())
                    v = R.decode(*want, form)
                    # (a value of fp32's range below its smallest: to a step of 2^-149)
                    with np.errstate(over="ignore"):          # (the largest code over the largest fp32: infinity)
                        exact = R.rounded(v.astype(np.float32), kind)
                    small = np.abs(v) < 2.0 ** -126
                    got = out.numpy()
                    same_bits(np.where(small, 0, got), np.where(small, 0, exact))
                    assert (np.abs(got - v)[small] <= 2.0 ** (-133 if kind else -149)).all()
                    out.check_canary()
    dx.check_canary()


def test_quantise_a_large_matrix(env):  # noqa: F811
    """By rows of 2^31 elements and more: the last rows (everything before them zero)."""
    torch, B = env
    rows, cols, tail = 66001, 33336, 3
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda:0")
    last = R.bf16(rng_of(61).standard_normal((tail, cols)).astype(np.float32))
    x[-tail:] = torch.from_numpy(last).cuda()
    p, pt = B.q8_alloc(rows, cols), B.q8_alloc(cols, rows)
    st = B.Model.stream_handle()
    B.conef_q8_quantise(x, R.E4M3, p, pt, st)
    y = torch.ones_like(x)
    B.conef_q8_dequantise(p, R.E4M3, y, st)
    same_bits(y[-tail:].float().cpu().numpy(), R.decode(*R.encode(last, R.E4M3), R.E4M3))
    assert not bool(y[:-tail].any())
    del x, y
    t = torch.ones(cols, rows, dtype=torch.bfloat16, device="cuda:0")
    B.conef_q8_dequantise(pt, R.E4M3, t, st)
    # the last block of 128 rows holds the three
    block = np.zeros((cols, 128), np.float32)
    first = rows // 128 * 128
    block[:, rows - tail - first:rows - first] = last.T
    same_bits(t[:, first:].float().cpu().numpy(), R.decode(*R.encode(block[:, :rows - first], R.E4M3), R.E4M3))
    assert not bool(t[:, :first].any())
    del pt, t
    n, k = 48, cols
    b = R.encode(rng_of(62).standard_normal((n, k)).astype(np.float32), R.E4M3)
    c = torch.full((rows, n), 7.0, device="cuda:0")
    B.conef_q8_product(p, R.E4M3, on_gpu(torch, b), k, 1.0, 0.0, c, room_of(torch, B.conef_q8_product_workspace(rows, n, k)), st)
    A, W = R.decode(*R.encode(last, R.E4M3), R.E4M3), R.decode(*b, R.E4M3)
    assert (np.abs(c[-tail:].cpu().numpy() - A @ W.T) <= wide_error(np.abs(A) @ np.abs(W).T, k)).all()
    assert not bool(c[:-tail].any())


# ---------------------------------------------------------------------------------------------- products
PRODUCT_SHAPES = [(1, 1, 1), (1, 16, 32), (3, 5, 129), (16, 16, 128), (8, 300, 700), (17, 1, 129), (64, 64, 256), (65, 130, 385), (128, 128, 1024),
                  (130, 257, 2049), (300, 513, 515), (1, 2048, 4096), (7, 1000, 8192), (40, 64, 20000), (256, 256, 512), (513, 768, 1280),
                  (1100, 1300, 900), (2048, 16, 640), (33, 4100, 1500), (129, 64, 9000), (70, 70, 128), (200, 100, 100)]


def product_inputs(m, n, k, form):
    g = rng_of(m, n, k, form)
    x, w = g.standard_normal((m, k)) * np.exp(g.standard_normal((m, 1))), g.standard_normal((n, k)) / np.sqrt(k)
    return R.encode(x.astype(np.float32), form), R.encode(w.astype(np.float32), R.E4M3)


def wide_error(magnitudes, k):
    """C in fp32: products are exact; the sixteen of an instruction and the sum so far meet in five additions at most, each good to 2^-23 of the sum of
    magnitudes so far; plus those of cutting the axis and of the factors."""
    return (5 * (-(-k // 16)) + 24) * 2.0 ** -23 * magnitudes


def cut_error(A, W, k, xp=np):
    """C in bf16, by the instructions of 8 bits: a product loses less than 2^-12 of the largest one of the 128 of its instruction, of which no more is known
    than that it is at most the product of both operands' largest.  Held to the largest of its 64, which is no more than that."""
    total = 0
    for f in range(0, k, 64):
        a, w = abs(A[:, f:f + 64]), abs(W[:, f:f + 64])
        total = total + min(64, k - f) * 2.0 ** -12 * (a.max(1)[:, None] * w.max(1)[None, :] if xp is np else a.amax(1)[:, None] * w.amax(1)[None, :])
    return total


@pytest.mark.parametrize("m,n,k", PRODUCT_SHAPES)
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("alpha,beta", [(1.0, 0.0), (0.125, 1.0)])
def test_product(env, m, n, k, bf16, form, alpha, beta):  # noqa: F811
    torch, B = env
    a, b = product_inputs(m, n, k, form)
    A, W = R.decode(*a, form), R.decode(*b, R.E4M3)
    old = R.rounded(rng_of(m, n).standard_normal((m, n)), bf16)
    if beta == 0.0:
        old[:] = np.nan                                   # what is not to be read
    c = Strided(torch, m, n, bf16, 1, 2, old)
    ws = room_of(torch, B.conef_q8_product_workspace(m, n, k))
    B.conef_q8_product(on_gpu(torch, a), form, on_gpu(torch, b), k, alpha, beta, c.t, ws, B.Model.stream_handle())
    want = alpha * (A @ W.T) + (beta * old.astype(np.float64) if beta else 0)
    tol = alpha * wide_error(np.abs(A) @ np.abs(W).T, k) + 2 * U * (np.abs(want) + (np.abs(old) if beta else 0))
    if bf16:
        tol = tol + alpha * cut_error(A, W, k)
        tol = tol + (np.abs(want) + tol) * U16
    assert (np.abs(c.numpy() - want) <= tol).all()
    if bf16:
        # as a whole: the result's rounding (2^-8 at most, each of its own), and what was cut off, each product's on its own
        far = np.sqrt(((c.numpy() - want) ** 2).sum())
        assert far <= U16 * np.sqrt((want ** 2).sum()) + alpha * np.sqrt((cut_error(A, W, k) ** 2).sum()) / 8 + np.sqrt((tol ** 2).sum()) * 1e-3
    c.check_canary()


def operand(torch, rows, cols, form, key):
    """(packed pair, its values in 64 bits [rows, cols], a scale byte's place (row, block) -> index), made on the device: finite codes of all kinds, scales of 2^-4
    to 2^4."""
    g = torch.Generator(device="cuda:0").manual_seed(key)
    r, c = -(-rows // 64) * 64, -(-cols // 128) * 128
    codes = torch.zeros(r, c, dtype=torch.uint8, device="cuda:0")
    codes[:rows, :cols] = torch.randint(0, 127 if form == R.E4M3 else 124, (rows, cols), dtype=torch.uint8, device="cuda:0", generator=g)
    codes[:rows, :cols] += 128 * torch.randint(0, 2, (rows, cols), dtype=torch.uint8, device="cuda:0", generator=g)
    scales = torch.zeros(c // 128, r, dtype=torch.uint8, device="cuda:0")
    scales[:, :rows] = torch.randint(123, 132, (c // 128, rows), dtype=torch.uint8, device="cuda:0", generator=g)
    t = torch.tensor(R.table(form), device="cuda:0")
    values = t[codes[:rows, :cols].long()] * torch.exp2(scales.t()[:rows].double() - 127).repeat_interleave(128, 1)[:, :cols]
    pc = codes.view(r // 16, 16, c // 128, 8, 16).permute(0, 2, 3, 1, 4).reshape(-1).contiguous()
    return (pc, scales.view(-1)), values, lambda i, b: b * r + i


# every size of tile, odd and even numbers of steps, rows that end on 64 bytes and not, C within the caches and not
@pytest.mark.parametrize("m,n,pitch,k,form", [(2000, 1700, 1703, 300, 0), (3500, 3600, 3600, 1537, 1), (4100, 4221, 4224, 600, 0), (1000, 16700, 16704, 1700, 0),
                                              (8200, 8190, 8192, 1100, 1), (60, 16400, 16401, 1990, 0), (4096, 4096, 4096, 4224, 0), (300, 200, 200, 50257, 1),
                                              (8448, 16381, 16384, 700, 0)])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("beta", [0.0, 1.0])
def test_large_product(env, m, n, pitch, k, form, bf16, beta):  # noqa: F811
    torch, B = env
    (a, A, _), (b, W, _) = operand(torch, m, k, form, 1), operand(torch, n, k, R.E4M3, 2)
    c = torch.full((m, pitch), float("nan"), dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda:0")
    if beta:
        c.normal_(generator=torch.Generator(device="cuda:0").manual_seed(3))
    gap, old = c[:, n:].clone(), c[:, :n].double()
    B.conef_q8_product(a, form, b, k, 0.125, beta, c[:, :n], room_of(torch, B.conef_q8_product_workspace(m, n, k)), B.Model.stream_handle())
    want = 0.125 * torch.mm(A, W.t())
    far = 0.125 * wide_error(torch.mm(A.abs(), W.abs().t()), k) + want.abs() * 2 * U
    if beta:
        want += old
        far += 2 * U * (old.abs() + want.abs())
    if bf16:
        far += 0.125 * cut_error(A, W, k, torch)
        far += (want.abs() + far) * U16
    assert bool(((c[:, :n].double() - want).abs() <= far).all())
    assert torch.equal(c[:, n:].isnan(), gap.isnan()) and torch.equal(c[:, n:].nan_to_num(), gap.nan_to_num())


def test_product_of_nothing(env):  # noqa: F811
    torch, B = env
    empty = tuple(torch.empty(0, dtype=torch.uint8, device="cuda:0") for _ in range(2))
    for shape in ((5, 9), (100, 90)):
        c = torch.full(shape, 3.0, device="cuda:0")
        B.conef_q8_product(empty, R.E4M3, empty, 0, 1.0, 0.5, c, None, B.Model.stream_handle())
        assert bool((c == 1.5).all())
        c.fill_(float("nan"))
        B.conef_q8_product(empty, R.E5M2, empty, 0, 1.0, 0.0, c, None, B.Model.stream_handle())
        assert bool((c == 0).all())


@pytest.mark.parametrize("m,n,k", [(5, 40, 200), (200, 300, 1000), (16, 64, 9000), (2000, 1700, 300), (3500, 3600, 600)])
@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("form", FORMS)
def test_product_with_scales_of_nan_and_zero_operands(env, m, n, k, bf16, form):  # noqa: F811
    torch, B = env
    (a, _, at), (b, _, bt) = operand(torch, m, k, form, 4), operand(torch, n, k, R.E4M3, 5)
    last = -(-k // 128) - 1
    a[1][at(m // 2, last)] = 255
    a[1][[at(0, q) for q in range(last + 1)]] = 0
    first = a[0].view(-(-m // 64) * 4, last + 1, 8, 16, 16)
    first[0, :, :, 0, :] = 0
    b[1][bt(n - 1, 0)] = 255
    c = torch.empty(m, n, dtype=torch.bfloat16 if bf16 else torch.float32, device="cuda:0")
    B.conef_q8_product(a, form, b, k, 1.0, 0.0, c, room_of(torch, B.conef_q8_product_workspace(m, n, k)), B.Model.stream_handle())
    nan = torch.zeros(m, n, dtype=torch.bool, device="cuda:0")
    nan[m // 2] = True
    nan[:, n - 1] = True
    assert torch.equal(c.isnan(), nan) and bool((c[0, :n - 1] == 0).all()) and not bool(c[~nan].isinf().any())


def test_products_of_far_scales(env):  # noqa: F811
    """Operands far from 1, whose product is not: 2^-110 by 2^100."""
    torch, B = env
    for m, n, k in ((3, 40, 300), (100, 90, 300)):
        a, b = product_inputs(m, n, k, R.E4M3)
        A, W = R.decode(*a, R.E4M3), R.decode(*b, R.E4M3)
        a, b = (a[0], (a[1] - 100).astype(np.uint8)), (b[0], (b[1] + 100).astype(np.uint8))
        for bf16 in (False, True):
            c = Strided(torch, m, n, bf16)
            B.conef_q8_product(on_gpu(torch, a), R.E4M3, on_gpu(torch, b), k, 1.0, 0.0, c.t, None, B.Model.stream_handle())
            want, tol = A @ W.T, wide_error(np.abs(A) @ np.abs(W).T, k)
            if bf16:
                tol = tol + cut_error(A, W, k) + np.abs(want) * U16 * 1.01
            assert (np.abs(c.numpy() - want) <= tol).all()


# ---------------------------------------------------------------------------------------------- norm
NORM_SHAPES = [(1, 1), (3, 2), (5, 7), (4, 8), (7, 9), (2, 63), (300, 64), (9, 65), (20, 128), (70, 129), (40, 255), (33, 257), (5, 511), (6, 512),
               (1030, 513), (1, 768), (33, 1001), (4, 1024), (3, 1025), (1, 2048), (700, 2049), (2, 4096), (3, 4097), (3, 5003), (5, 6145), (5, 8192),
               (2, 8193), (3, 16384), (2, 16385), (3, 20001), (9000, 100), (9000, 300), (8500, 600), (8300, 1500), (20000, 5)]


def norm_inputs(rows, cols, bf16, key=0):
    g = rng_of(rows, cols, 70 + key)
    x = R.rounded((g.standard_normal((rows, cols)) * 2 + 0.3) * np.exp(0.5 * g.standard_normal(cols)), bf16)
    return g, x, np.float32(1 + 0.2 * g.standard_normal(cols))


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("rows,cols", NORM_SHAPES)
@pytest.mark.parametrize("skip,gap,residual", [(0, 0, False), (1, 3, True)])
def test_norm_forward(env, rows, cols, bf16, skip, gap, residual):  # noqa: F811
    torch, B = env
    g, x, gamma = norm_inputs(rows, cols, bf16)
    r = R.rounded(g.standard_normal((rows, cols)) + 0.3, bf16) if residual else None
    z = R.rounded(r + x, bf16) if residual else x
    want, rstd64 = R.rms(z, gamma, 1e-5)
    codes = R.pack(*R.encode(want, R.E4M3))
    dx = Strided(torch, rows, cols, bf16, skip, gap, x)
    dr = Strided(torch, rows, cols, bf16, gap, skip, r) if residual else None
    for outputs in ("codes", "y", "both"):
        dz = Strided(torch, rows, cols, bf16, skip + 2, gap) if residual else None
        dy = Strided(torch, rows, cols, bf16, skip, gap) if outputs != "codes" else None
        p = B.q8_alloc(rows, cols) if outputs != "y" else None
        if p:
            p[0].fill_(0xA5)
            p[1].fill_(0xA5)
        rstd = torch.full((rows,), 7.0, device="cuda:0")
        B.conef_rms_forward(1e-5, dx.t, dr.t if residual else None, column_vector(torch, gamma), dz.t if residual else None, dy.t if dy else None, p, rstd,
                            B.Model.stream_handle())
        if residual:
            same_bits(dz.numpy(), z)
            dz.check_canary()
        # rounded once, from 64 bits
        assert (np.abs(rstd.cpu().numpy() - rstd64) <= rstd64 * U * 1.0001).all()
        if dy:
            assert (np.abs(dy.numpy() - want) <= np.abs(want) * (U16 if bf16 else U) * 1.0001 + 1e-44).all()
            dy.check_canary()
        if p:
            for got, exp in zip(packed_numpy(p), codes):
                assert np.array_equal(got, exp), outputs
        dx.check_canary()


def test_norm_forward_in_place_and_without_a_statistic(env):  # noqa: F811
    torch, B = env
    g, x, gamma = norm_inputs(37, 1000, False)
    a, out, G = column_vector(torch, x), torch.empty(37, 1000, device="cuda:0"), column_vector(torch, gamma)
    st = B.Model.stream_handle()
    B.conef_rms_forward(1e-5, a, None, G, None, out, None, None, st)
    b = a.clone()
    B.conef_rms_forward(1e-5, b, None, G, None, b, None, None, st)
    assert torch.equal(b, out)
    # the sum in the place of either of its terms, y in the place of the other
    r = column_vector(torch, g.standard_normal((37, 1000)))
    z, y = torch.empty_like(a), torch.empty_like(a)
    B.conef_rms_forward(1e-5, a, r, G, z, y, None, None, st)
    for first in (True, False):
        a2, r2 = a.clone(), r.clone()
        B.conef_rms_forward(1e-5, a2, r2, G, a2 if first else r2, r2 if first else a2, None, None, st)
        assert torch.equal(a2 if first else r2, z) and torch.equal(r2 if first else a2, y)


@pytest.mark.parametrize("cols", [100, 3000, 20000])
def test_norm_of_zeros_far_magnitudes_and_what_is_not_finite(env, cols):  # noqa: F811
    torch, B = env
    x = np.zeros((7, cols), np.float32)
    x[1] = 5.0
    x[2] = rng_of(1).standard_normal(cols) * 1e30                    # whose squares fp32 does not hold
    x[3] = rng_of(2).standard_normal(cols) * 1e-30
    x[4, 17] = np.nan
    x[5, 0] = np.inf
    x[6] = np.float32(3e38)
    gamma = np.float32(rng_of(3).standard_normal(cols))
    a, y, p = column_vector(torch, x), torch.empty(7, cols, device="cuda:0"), B.q8_alloc(7, cols)
    B.conef_rms_forward(1e-5, a, None, column_vector(torch, gamma), None, y, p, None, B.Model.stream_handle())
    got = y.cpu().numpy()
    rows = [0, 1, 2, 3, 6]
    want, _ = R.rms(x[rows], gamma, 1e-5)
    assert (np.abs(got[rows] - want) <= np.abs(want) * U * 1.0001 + 1e-44).all()
    assert np.isnan(got[4]).all() and np.isnan(got[5, 0]) and (got[5, 1:] == 0).all()
    full = np.zeros((7, cols))
    full[rows] = want
    full[5] = 0.0 * gamma                                 # (zeros times 1 / infinity, each with its sign)
    full[4], full[5, 0] = np.nan, np.nan
    for c, e in zip(packed_numpy(p), R.pack(*R.encode(full, R.E4M3))):
        assert np.array_equal(c, e)


def depth(cols):
    """Most additions on a value's way into a row's sum: 16 in a lane's registers (rows beyond 8192 columns: an eighth of 256th of a row), six across a wave, four across a
    workgroup."""
    return max(16, cols // 256 + 8) + 10


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("fused", [False, True])
@pytest.mark.parametrize("rows,cols", [(600, 1100), (16390, 1100), (513, 2100), (8195, 2100), (700, 4200), (4100, 4200), (600, 6200), (4097, 6200)])
def test_norm_of_many_rows_is_that_of_few(env, rows, cols, bf16, fused):  # noqa: F811
    """How many rows a workgroup takes goes by their number; a row's results do not: bit for bit those of calls on 448 rows each."""
    torch, B = env
    dtype = torch.bfloat16 if bf16 else torch.float32
    g = torch.Generator(device="cuda:0").manual_seed(rows + cols)
    x, r = (torch.randn(rows, cols, device="cuda:0", generator=g).to(dtype) for _ in range(2))
    gamma = torch.rand(cols, device="cuda:0", generator=g) + 0.5

    def norm(x, r):
        n = x.shape[0]
        z, y, rstd, q = torch.empty_like(x), torch.empty_like(x), torch.empty(n, device="cuda:0"), B.q8_alloc(n, cols)
        for t in q:
            t.fill_(0xAA)
        B.conef_rms_forward(1e-5, x, r if fused else None, gamma, z if fused else None, y, q, rstd, B.Model.stream_handle())
        pieces = -(-cols // 128)
        return (z if fused else x), y, rstd, q[0].view(-1, pieces * 2048), q[1].view(pieces, -1).t()

    whole = norm(x, r)
    for at in range(0, rows, 448):
        n = min(448, rows - at)
        z, y, rstd, codes, scales = norm(x[at:at + n], r[at:at + n])
        assert torch.equal(whole[0][at:at + n], z) and torch.equal(whole[1][at:at + n], y) and torch.equal(whole[2][at:at + n], rstd)
        assert torch.equal(whole[3][at // 16:at // 16 + codes.shape[0]], codes) and torch.equal(whole[4][at:at + scales.shape[0]], scales)
    assert not bool(whole[3].view(-1, -(-cols // 128), 8, 16, 16).transpose(1, 3).reshape(-1, 8 * -(-cols // 128) * 16)[rows:].any())
    assert not bool(whole[4][rows:].any())


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("rows,cols", NORM_SHAPES)
@pytest.mark.parametrize("skip,gap,residual", [(0, 0, False), (1, 3, True)])
def test_norm_backward(env, rows, cols, bf16, skip, gap, residual):  # noqa: F811
    torch, B = env
    g, z, gamma = norm_inputs(rows, cols, bf16, 1)
    dy = R.rounded(g.standard_normal((rows, cols)), bf16)
    dz_in = R.rounded(g.standard_normal((rows, cols)), bf16) if residual else None
    rstd = np.float32(R.rms(z, gamma, 1e-5)[1])
    D = {k: Strided(torch, rows, cols, bf16, skip, gap, v) for k, v in (("dy", dy), ("z", z), ("dz", None))}
    if residual:
        D["dz_in"] = Strided(torch, rows, cols, bf16, gap, skip, dz_in)
    dgamma = torch.full((cols,), 7.0, device="cuda:0")
    room = B.conef_rms_workspace(rows, cols)
    ws = room_of(torch, room)
    args = (D["dy"].t, D["z"].t, column_vector(torch, gamma), column_vector(torch, rstd), D["dz_in"].t if residual else None)
    B.conef_rms_backward(*args, D["dz"].t, dgamma, ws, B.Model.stream_handle())
    want, wg, hat, a = R.rms_back(dy, z, gamma, rstd)
    # hat and a take a rounding each, the mean depth and three more, its product with hat two, the difference one, rstd one, dz_in one
    s = rstd.astype(np.float64)[:, None]
    err = s * (2 * U * np.abs(a) + (depth(cols) + 7) * U * np.abs(hat) * np.abs(a * hat).mean(1, keepdims=True)) + 2 * U * np.abs(want)
    if residual:
        want = want + dz_in
        err = err + U * np.abs(want)
    err = err * 1.01 + (np.abs(want) * U16 * 1.01 if bf16 else 0) + 1e-44
    assert (np.abs(D["dz"].numpy() - want) <= err).all()
    n = -(-rows // (room // (4 * cols))) + 6              # rows of a workgroup, one after the other, and across its waves; the rest in fp64
    assert (np.abs(dgamma.cpu().numpy() - wg) <= (n + 4) * U * (np.abs(dy) * np.abs(hat)).sum(0) * 1.01).all()
    for m in D.values():
        m.check_canary()
    # each output alone, and dz in place of what it is computed from, give the same bits
    for only in ("dz", "dgamma", "dy", "z") + (("dz_in",) if residual else ()):
        g2 = torch.zeros_like(dgamma)
        E = {k: Strided(torch, rows, cols, bf16, skip, gap, v) for k, v in (("dy", dy), ("z", z), ("dz", None))}
        E["dz_in"] = Strided(torch, rows, cols, bf16, skip, gap, dz_in) if residual else None
        args = (E["dy"].t, E["z"].t, column_vector(torch, gamma), column_vector(torch, rstd), E["dz_in"].t if residual else None)
        if only == "dz":
            B.conef_rms_backward(*args, E["dz"].t, None, None, B.Model.stream_handle())
        elif only == "dgamma":
            B.conef_rms_backward(*args, None, g2, ws, B.Model.stream_handle())
        else:
            B.conef_rms_backward(*args, E[only].t, g2, ws, B.Model.stream_handle())
        if only != "dgamma":
            assert torch.equal(E[only].t, D["dz"].t), only
        if only != "dz":
            assert torch.equal(g2, dgamma), only


def test_norm_backward_of_no_rows_is_zero(env):  # noqa: F811
    torch, B = env
    none, g, e = torch.empty(0, 100, device="cuda:0"), torch.ones(100, device="cuda:0"), torch.empty(0, device="cuda:0")
    B.conef_rms_backward(none, none, torch.ones(100, device="cuda:0"), e, None, None, g, None, B.Model.stream_handle())
    assert not bool(g.any())


@pytest.mark.parametrize("rows,cols", [(5, 96), (3, 700), (2, 3000)])
def test_norm_gradient_against_differences(env, rows, cols):  # noqa: F811
    """<gradient, v> against (L(+h v) - L(-h v)) / 2h of L = sum(w y), taken with the library's own forward pass in fp32, the residual included.  The
    difference's own error: h^2 times third derivatives (all of order 1: 1e-4 of the terms' sum at h = 1e-2), and fp32 roundings of y, u sqrt(n) |w y| / h, 1e-5 of it."""
    torch, B = env
    g, x, gamma = norm_inputs(rows, cols, False, 5)
    r, w = np.float32(g.standard_normal((rows, cols))), np.float32(g.standard_normal((rows, cols)))
    st = B.Model.stream_handle()
    T = lambda v: column_vector(torch, v)                      # noqa: E731

    def forward(x, r, gamma):
        z, y, rstd = torch.empty(rows, cols, device="cuda:0"), torch.empty(rows, cols, device="cuda:0"), torch.empty(rows, device="cuda:0")
        B.conef_rms_forward(1e-5, T(x), T(r), T(gamma), z, y, None, rstd, st)
        return z, y, rstd

    def total(*v):
        return float((forward(*v)[1].cpu().numpy().astype(np.float64) * w).sum())

    z, _, rstd = forward(x, r, gamma)
    dz, dg = torch.empty_like(z), torch.empty(cols, device="cuda:0")
    B.conef_rms_backward(T(w), z, T(gamma), rstd, None, dz, dg, room_of(torch, B.conef_rms_workspace(rows, cols)), st)
    at, h = [x, r, gamma], 1e-2
    for k, grad in enumerate((dz, dz, dg)):
        v = np.float32(g.standard_normal(at[k].shape))
        up, down = list(at), list(at)
        up[k], down[k] = np.float32(at[k] + h * v), np.float32(at[k] - h * v)
        numeric = (total(*up) - total(*down)) / (2 * h)
        terms = grad.cpu().numpy().astype(np.float64) * v
        assert abs(numeric - terms.sum()) <= 1e-3 * np.sqrt((terms ** 2).sum()) * 3 + 1e-4 * np.abs(terms).sum(), k


# ---------------------------------------------------------------------------------------------- loss
LOSS_SHAPES = [(1, 1, 1), (1, 2, 8), (3, 5, 7), (16, 64, 32), (17, 65, 33), (32, 300, 64), (33, 129, 100), (64, 1000, 48), (70, 40, 200), (130, 700, 264),
               (300, 257, 515), (1, 5000, 72), (200, 3, 16), (520, 1300, 96), (2, 20000, 40)]


def loss_inputs(tokens, vocab, width, bf16, key=0):
    g = rng_of(tokens, vocab, width, key)
    x = R.rounded(g.standard_normal((tokens, width)), bf16)
    w = R.rounded(g.standard_normal((vocab, width)) * 2 / np.sqrt(width), bf16)
    t = g.integers(0, vocab, tokens)
    t[g.random(tokens) < 0.2] = -100
    if tokens > 2:
        t[1] = vocab                                         # none either
        t[2] = 2 ** 62
    t[0] = vocab - 1
    return g, x, w, t.astype(np.int64)


def loss_errors(x, w, p, lse, dloss, there):
    """Errors of lse, of logits and of d in fp32.  A logit: exact products, an addition each (and two of the instruction) to 2^-23 of the magnitudes.  An exponential: that, the
    difference's and its factor's rounding, and two of the function.  A sum of exponentials: 32 in a lane, across a wave and a tile, then of tiles; its
    logarithm adds one, and lse's own.  d: p's error and four roundings of its own."""
    mags = np.abs(x.astype(np.float64)) @ np.abs(w.astype(np.float64)).T
    e_logit = (x.shape[1] + 2) * 2.0 ** -23 * mags
    e_lse = e_logit.max(1) + (60 + 8) * U + 2 * U * (np.abs(lse) + 1)
    span = 2 * mags.max(1)[:, None] + 1
    e_p = p * (e_logit + e_lse[:, None] + 4 * U * span + 4 * U)
    share = np.where(there, np.abs(dloss), 0.0)[:, None]
    return e_lse, e_logit, share * e_p + 4 * U * share * np.minimum(p + 1, 1), share


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("tokens,vocab,width", LOSS_SHAPES)
@pytest.mark.parametrize("skip,gap", [(0, 0), (1, 3), (8, 8)])
@pytest.mark.parametrize("weighted", [False, True])
def test_loss(env, tokens, vocab, width, bf16, skip, gap, weighted):  # noqa: F811
    torch, B = env
    g, x, w, t = loss_inputs(tokens, vocab, width, bf16)
    dloss = np.float32(g.standard_normal(tokens)) if weighted else None
    want_loss, want_lse, logits, p, dx64, dw64 = R.loss(x, w, t, dloss)
    there = (t >= 0) & (t < vocab)
    dx_, dw_ = Strided(torch, tokens, width, bf16, skip, gap, x), Strided(torch, vocab, width, bf16, skip, gap, w)
    targets = torch.from_numpy(t).cuda()
    loss, lse = torch.full((tokens,), 7.0, device="cuda:0"), torch.full((tokens,), 7.0, device="cuda:0")
    ws = room_of(torch, B.conef_loss_workspace(tokens, vocab, width, torch.bfloat16 if bf16 else torch.float32))
    st = B.Model.stream_handle()
    B.conef_loss_forward(dx_.t, dw_.t, targets, loss, lse, ws, st)
    e_lse, e_logit, e_d, share = loss_errors(x, w, p, want_lse, np.ones(tokens) if dloss is None else dloss.astype(np.float64), there)
    assert (np.abs(lse.cpu().numpy() - want_lse) <= e_lse).all()
    at = np.where(there, t, 0)
    e_loss = np.where(there, e_lse + e_logit[np.arange(tokens), at] + 2 * U * np.abs(want_loss), 0.0)
    assert (np.abs(loss.cpu().numpy() - want_loss) <= e_loss).all()
    # alone, they are the same
    for a, b in ((torch.zeros_like(loss), None), (None, torch.zeros_like(lse))):
        B.conef_loss_forward(dx_.t, dw_.t, targets, a, b, ws, st)
        assert torch.equal(a if a is not None else b, loss if a is not None else lse)
    # backward, from the lse that the forward pass left
    alpha, beta = 0.125, 0.5
    old = R.rounded(g.standard_normal((vocab, width)), bf16)
    gx, gw = Strided(torch, tokens, width, bf16, skip, gap), Strided(torch, vocab, width, bf16, gap, skip, old)
    ws.fill_(0xFF)
    B.conef_loss_backward(dx_.t, dw_.t, targets, lse, column_vector(torch, dloss) if weighted else None, alpha, beta, gx.t, gw.t, ws, st)
    onehot = np.zeros_like(p)
    onehot[np.arange(tokens), at] = 1
    if bf16:
        e_d = e_d + U16 * 1.01 * share * np.abs(p - onehot)
    ax, aw = np.abs(x).astype(np.float64), np.abs(w).astype(np.float64)
    ad = share * np.abs(p - onehot)
    e_x = e_d @ aw + (vocab + 40) * 2.0 ** -23 * (ad @ aw) + 4 * U * np.abs(dx64)
    e_w = alpha * (e_d.T @ ax + (tokens + 40) * 2.0 ** -23 * (ad.T @ ax)) + 4 * U * (alpha * np.abs(dw64) + beta * np.abs(old))
    want_w = alpha * dw64 + beta * old
    e_alone = e_w + (alpha * np.abs(dw64) + e_w) * (U16 if bf16 else 0)          # of alpha dw alone, whose rounding goes by its own size, not by what is left beside beta old
    if bf16:
        e_x, e_w = e_x + (np.abs(dx64) + e_x) * U16, e_w + (np.abs(want_w) + e_w) * U16
    assert (np.abs(gx.numpy() - dx64) <= e_x * 1.01).all()
    assert (np.abs(gw.numpy() - want_w) <= e_w * 1.01).all()
    assert (gx.numpy()[~there] == 0).all()
    for m in (dx_, dw_, gx, gw):
        m.check_canary()
    # each gradient alone, and dw into what is not to be read
    gx2, gw2 = Strided(torch, tokens, width, bf16, skip, gap), Strided(torch, vocab, width, bf16, skip, gap, np.full((vocab, width), np.nan, np.float32))
    dl = column_vector(torch, dloss) if weighted else None
    B.conef_loss_backward(dx_.t, dw_.t, targets, lse, dl, alpha, beta, gx2.t, None, ws, st)
    assert torch.equal(gx2.t, gx.t)
    B.conef_loss_backward(dx_.t, dw_.t, targets, lse, dl, alpha, 0.0, None, gw2.t, ws, st)
    assert (np.abs(gw2.numpy() - alpha * dw64) <= e_alone * 1.01).all()


# pieces of the vocabulary, every size of tile
@pytest.mark.parametrize("tokens,vocab,width,bf16", [(8500, 9000, 64, True), (8500, 9001, 36, False), (2100, 20300, 136, True), (3000, 3100, 520, True), (40, 50257, 768, True),
                                                     (1001, 5003, 515, False), (8200, 700, 1030, True), (9000, 4100, 24, True)])
def test_large_loss(env, tokens, vocab, width, bf16):  # noqa: F811
    """As above with 64 bits on the device, and errors as a whole: of a sum of n roundings, each of its own, sqrt(n) of one (times four)."""
    torch, B = env
    g = torch.Generator(device="cuda:0").manual_seed(tokens)
    dt = torch.bfloat16 if bf16 else torch.float32
    x = torch.randn(tokens, width, device="cuda:0", generator=g).to(dt)
    w = (torch.randn(vocab, width, device="cuda:0", generator=g) * (2 / width ** 0.5)).to(dt)
    t = torch.randint(0, vocab, (tokens,), device="cuda:0", generator=g)
    t[::7] = -1
    there = t >= 0
    dloss = torch.rand(tokens, device="cuda:0", generator=g) + 0.5
    loss, lse = torch.empty(tokens, device="cuda:0"), torch.empty(tokens, device="cuda:0")
    ws = room_of(torch, B.conef_loss_workspace(tokens, vocab, width, dt))
    st = B.Model.stream_handle()
    B.conef_loss_forward(x, w, t, loss, lse, ws, st)
    logits = torch.mm(x.double(), w.double().t())
    want = torch.logsumexp(logits, 1)
    rows = torch.nonzero(there)[:, 0]
    # a logit is off by 2^-23 sqrt(width) times the root of its terms' squares, and no more than four times that
    e = 4 * 2.0 ** -23 * width ** 0.5 * 4 + 80 * U + 3 * U * want.abs()
    assert bool(((lse.double() - want).abs() <= e).all())
    assert bool(((loss.double() - torch.where(there, want - logits.gather(1, t.clamp(min=0)[:, None])[:, 0], 0.0)).abs() <= 2 * e).all())
    d = torch.exp(logits - want[:, None])
    d[rows, t[rows]] -= 1
    d *= torch.where(there, dloss.double(), 0.0)[:, None]
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    B.conef_loss_backward(x, w, t, lse, dloss, 0.25, 0.0, dx, dw, ws, st)
    for got, exp in ((dx, d @ w.double()), (dw, 0.25 * (d.t() @ x.double()))):
        far = (got.double() - exp).norm() / exp.norm()
        # bf16: d's rounding and the result's, 2^-8 each at the most; fp32: a logit's error above, and the sums'
        assert float(far) <= (1.5 * U16 if bf16 else 4 * 2.0 ** -23 * (width ** 0.5 + 8)), float(far)
    assert not bool(dx[~there].any())


def test_weights_of_tokens_without_a_target_do_not_count(env):  # noqa: F811
    torch, B = env
    g, x, w, t = loss_inputs(70, 300, 64, True)
    X, W, targets = column_vector(torch, x).bfloat16(), column_vector(torch, w).bfloat16(), torch.from_numpy(t).cuda()
    there = (targets >= 0) & (targets < 300)
    st, ws = B.Model.stream_handle(), room_of(torch, B.conef_loss_workspace(70, 300, 64, torch.bfloat16))
    lse, outs = torch.empty(70, device="cuda:0"), []
    B.conef_loss_forward(X, W, targets, None, lse, ws, st)
    for elsewhere in (0.0, 1e30, float("inf"), float("nan")):
        dloss = torch.where(there, torch.full((70,), 3e-4, device="cuda:0"), elsewhere)
        dx, dw = torch.empty_like(X), torch.empty_like(W)
        B.conef_loss_backward(X, W, targets, lse, dloss, 1.0, 0.0, dx, dw, ws, st)
        outs.append((dx, dw))
    for dx, dw in outs[1:]:
        assert torch.equal(dx, outs[0][0]) and torch.equal(dw, outs[0][1])


@pytest.mark.parametrize("tokens,vocab,width,bf16", [(70001, 40009, 16, True), (66001, 9, 33336, True), (9, 66001, 33337, True), (66001, 5, 17000, False)])
def test_loss_beyond_31_bits(env, tokens, vocab, width, bf16):  # noqa: F811
    """More than 2^31 logits, or elements of x or of w (the last two at least 4 GB): the first and last tokens' losses and gradients, the last words' gradient."""
    torch, B = env
    dt, st = torch.bfloat16 if bf16 else torch.float32, B.Model.stream_handle()
    g = torch.Generator(device="cuda:0").manual_seed(9)
    x, w = torch.zeros(tokens, width, dtype=dt, device="cuda:0"), torch.zeros(vocab, width, dtype=dt, device="cuda:0")
    rows, words = [0, 1, tokens - 2, tokens - 1], [0, 1, vocab - 2, vocab - 1]
    for r in rows:
        x[r] = torch.randn(width, device="cuda:0", generator=g).to(dt)
    for r in words:
        w[r] = (torch.randn(width, device="cuda:0", generator=g) / width ** 0.5).to(dt)
    t = torch.full((tokens,), -1, device="cuda:0")
    t[rows] = torch.tensor([words[3], words[0], words[2], words[3]], device="cuda:0")
    loss, lse = torch.full((tokens,), 7.0, device="cuda:0"), torch.full((tokens,), 7.0, device="cuda:0")
    ws = torch.empty(B.conef_loss_workspace(tokens, vocab, width, dt), dtype=torch.uint8, device="cuda:0")
    B.conef_loss_forward(x, w, t, loss, lse, ws, st)
    X, W = x[rows].double(), w[words].double()
    logits = torch.mm(X, W.t())                                   # of these four words; all others' are 0
    total = torch.logsumexp(torch.cat((logits, torch.zeros(4, vocab - 4, dtype=torch.float64, device="cuda:0")), 1), 1)
    at = torch.tensor([3, 0, 2, 3], device="cuda:0")
    e = 4 * 2.0 ** -23 * width ** 0.5 * 2 + 80 * U + 3 * U * total
    assert bool(((lse[rows].double() - total).abs() <= e).all())
    assert bool(((loss[rows].double() - (total - logits.gather(1, at[:, None])[:, 0])).abs() <= 2 * e).all())
    assert not bool(loss[2:-2].any())
    dx, dw = torch.full_like(x, 7.0), torch.full_like(w, 7.0)
    B.conef_loss_backward(x, w, t, lse, None, 1.0, 0.0, dx, dw, ws, st)
    d = torch.exp(logits - total[:, None])
    d[torch.arange(4), at] -= 1
    for got, want in ((dx[rows], torch.mm(d, W)), (dw[words], torch.mm(d.t(), X))):
        assert float((got.double() - want).norm() / want.norm()) <= (1.5 * U16 if bf16 else 1e-4)
    assert not bool(dx[2:-2].any())


def test_loss_of_no_tokens(env):  # noqa: F811
    torch, B = env
    st = B.Model.stream_handle()
    for dt in (torch.float32, torch.bfloat16):
        x, w, e = torch.empty(0, 40, dtype=dt, device="cuda:0"), torch.ones(70, 40, dtype=dt, device="cuda:0"), torch.empty(0, device="cuda:0")
        t = torch.empty(0, dtype=torch.int64, device="cuda:0")
        B.conef_loss_forward(x, w, t, e, e, None, st)
        dw = torch.full_like(w, 3.0)
        B.conef_loss_backward(x, w, t, e, e, 1.0, 0.5, None, dw, None, st)
        assert bool((dw == 1.5).all())
        dw.fill_(float("nan"))
        B.conef_loss_backward(x, w, t, e, None, 1.0, 0.0, None, dw, None, st)
        assert bool((dw == 0).all())


def test_loss_without_any_target_and_of_what_is_not_finite(env):  # noqa: F811
    torch, B = env
    st = B.Model.stream_handle()
    g, x, w, _ = loss_inputs(40, 300, 64, False)
    X, W = column_vector(torch, x), column_vector(torch, w)
    t = torch.full((40,), -100, device="cuda:0")
    loss, lse, dx, dw = torch.ones(40, device="cuda:0"), torch.ones(40, device="cuda:0"), torch.ones_like(X), torch.ones_like(W)
    ws = room_of(torch, B.conef_loss_workspace(40, 300, 64, torch.float32))
    B.conef_loss_forward(X, W, t, loss, lse, ws, st)
    B.conef_loss_backward(X, W, t, lse, None, 1.0, 0.0, dx, dw, ws, st)
    assert not bool(loss.any()) and not bool(dx.any()) and not bool(dw.any()) and bool(lse.isfinite().all())
    # a row of NaN without a target, whose logits count for nobody; one with an infinity and one of NaN that have targets
    t = torch.arange(40, device="cuda:0")
    t[3] = -1
    X2 = X.clone()
    X2[3] = float("nan")
    X2[5, 0] = float("inf")
    X2[7] = float("nan")
    B.conef_loss_forward(X2, W, t, loss, lse, ws, st)
    assert float(loss[3]) == 0 and bool(loss[7].isnan())
    B.conef_loss_backward(X2, W, t, lse, None, 1.0, 0.0, dx, None, ws, st)
    assert not bool(dx[3].any()) and bool(dx[7].isnan().all())
    others = [i for i in range(40) if i not in (3, 5, 7)]
    assert bool(loss[others].isfinite().all()) and bool(dx[others].isfinite().all())
    # a word that nobody can say: an infinite logit against it
    X3, W3 = X.clone(), W.clone()
    X3[:, 0], W3[9, 0] = 1.0, float("-inf")
    t = torch.full((40,), 5, device="cuda:0")
    B.conef_loss_forward(X3, W3, t, loss, lse, ws, st)
    keep = [i for i in range(300) if i != 9]
    want = torch.logsumexp(torch.mm(X3.double(), W3[keep].double().t()), 1)
    assert bool(((lse.double() - want).abs() <= 1e-5).all())
    # far logits: of hundreds, where exponentials of themselves would not fit
    B.conef_loss_forward(X * 100, W, t, loss, lse, ws, st)
    want = torch.logsumexp(torch.mm((X * 100).double(), W.double().t()), 1)
    assert bool(((lse.double() - want).abs() <= 66 * 2.0 ** -23 * (100 * X.abs()) @ W.abs().t().amax(1) + 80 * U + 2 * U * want.abs()).all())


@pytest.mark.parametrize("tokens,vocab,width", [(7, 90, 40), (70, 300, 65)])
def test_loss_gradient_against_differences(env, tokens, vocab, width):  # noqa: F811
    """<gradient, v> against (L(+h v) - L(-h v)) / 2h of L = sum(dloss loss) with the library's own forward pass.  The difference's own error: h^2 / 6 times third derivatives
    (of order |v|^3: 1e-4 of the terms at h = 1e-2), and roundings of a loss, 2^-22 each, over h."""
    torch, B = env
    g, x, w, t = loss_inputs(tokens, vocab, width, False, 3)
    dl, st = np.float32(g.standard_normal(tokens)), B.Model.stream_handle()
    T = lambda v: column_vector(torch, v)                      # noqa: E731
    targets, ws = torch.from_numpy(t).cuda(), room_of(torch, B.conef_loss_workspace(tokens, vocab, width, torch.float32))
    loss, lse = torch.empty(tokens, device="cuda:0"), torch.empty(tokens, device="cuda:0")

    def total(x, w):
        B.conef_loss_forward(T(x), T(w), targets, loss, None, ws, st)
        return float((loss.cpu().numpy().astype(np.float64) * dl).sum())

    X, W = T(x), T(w)
    B.conef_loss_forward(X, W, targets, loss, lse, ws, st)
    dx, dw = torch.empty_like(X), torch.empty_like(W)
    B.conef_loss_backward(X, W, targets, lse, T(dl), 1.0, 0.0, dx, dw, ws, st)
    for k, grad in enumerate((dx, dw)):
        v = np.float32(g.standard_normal((x, w)[k].shape) / np.sqrt(width))
        h = 1e-2
        ends = [total(x + s * h * v, w) if k == 0 else total(x, w + s * h * v) for s in (1, -1)]
        terms = grad.cpu().numpy().astype(np.float64) * v
        e = 1e-3 * (np.sqrt((terms ** 2).sum()) + 0.1 * np.abs(terms).sum()) + np.abs(dl).sum() * 8 * 2.0 ** -22 / h
        assert abs((ends[0] - ends[1]) / (2 * h) - terms.sum()) <= e, k


# ---------------------------------------------------------------------------------------------- together
def sublayer(torch, B, tokens, width, hidden, vocab, dt, seed):
    """A language model's last sublayer and its loss, forward and backward, in 8 bits: buffers, and a function that runs it"""
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    new = lambda *s, t=dt: torch.zeros(*s, dtype=t, device="cuda:0")               # noqa: E731
    rand = lambda *s: torch.randn(*s, device="cuda:0", generator=g).to(dt)         # noqa: E731
    i = {"x": rand(tokens, width), "res": rand(tokens, width), "w": rand(hidden, width) / width ** 0.5, "out": rand(vocab, hidden) / hidden ** 0.5,
         "gamma": torch.rand(width, device="cuda:0", generator=g) + 0.5, "t": torch.randint(0, vocab, (tokens,), device="cuda:0", generator=g)}
    o = {"z": new(tokens, width), "y": new(tokens, width), "rstd": new(tokens, t=torch.float32), "u": new(tokens, hidden), "loss": new(tokens, t=torch.float32),
         "lse": new(tokens, t=torch.float32), "du": new(tokens, hidden), "dout": new(vocab, hidden), "dy": new(tokens, width), "dw": new(hidden, width),
         "dz": new(tokens, width), "dgamma": new(width, t=torch.float32)}
    q = {"y": B.q8_alloc(tokens, width), "y_t": B.q8_alloc(width, tokens), "w": B.q8_alloc(hidden, width), "w_t": B.q8_alloc(width, hidden),
         "du": B.q8_alloc(tokens, hidden), "du_t": B.q8_alloc(hidden, tokens)}
    ws = new(max(B.conef_loss_workspace(tokens, vocab, hidden, dt), B.conef_rms_workspace(tokens, width),
                 *(B.conef_q8_product_workspace(*s) for s in ((tokens, hidden, width), (tokens, width, hidden), (hidden, width, tokens)))), t=torch.uint8)

    def run():
        st = B.Model.stream_handle()
        B.conef_rms_forward(1e-5, i["x"], i["res"], i["gamma"], o["z"], o["y"], q["y"], o["rstd"], st)
        B.conef_q8_quantise(i["w"], B.E4M3, q["w"], q["w_t"], st)
        B.conef_q8_product(q["y"], B.E4M3, q["w"], width, 1.0, 0.0, o["u"], ws, st)
        B.conef_loss_forward(o["u"], i["out"], i["t"], o["loss"], o["lse"], ws, st)
        B.conef_loss_backward(o["u"], i["out"], i["t"], o["lse"], None, 0.5, 0.0, o["du"], o["dout"], ws, st)
        B.conef_q8_quantise(o["du"], B.E5M2, q["du"], q["du_t"], st)
        B.conef_q8_quantise(o["y"], B.E4M3, None, q["y_t"], st)
        B.conef_q8_product(q["du"], B.E5M2, q["w_t"], hidden, 1.0, 0.0, o["dy"], ws, st)
        B.conef_q8_product(q["du_t"], B.E5M2, q["y_t"], tokens, 0.5, 0.0, o["dw"], ws, st)
        B.conef_rms_backward(o["dy"], o["z"], i["gamma"], o["rstd"], o["z"], o["dz"], o["dgamma"], ws, st)

    return i, o, ws, run


@pytest.mark.parametrize("tokens,width,hidden,vocab", [(40, 72, 100, 300), (700, 300, 512, 5000)])
@pytest.mark.parametrize("bf16", [False, True])
def test_a_sublayer_and_its_loss(env, tokens, width, hidden, vocab, bf16):  # noqa: F811
    """All of them in a row, each one's output checked as a whole against what 64 bits make of its own inputs: one rounding of an 8-bit operand moves a product
    by 2^-4 (E4M3) or 2^-3 (E5M2) of a term at most, here all of them independently, so that a sum moves by that of itself at most."""
    torch, B = env
    i, o, _, run = sublayer(torch, B, tokens, width, hidden, vocab, torch.bfloat16 if bf16 else torch.float32, 5)
    run()
    D = {k: v.double() for k, v in {**i, **o}.items()}
    close = lambda got, want, e: float((got - want).norm()) <= e * float(want.norm())                      # noqa: E731
    u = U16 if bf16 else 1e-5
    assert torch.equal(o["z"], (i["x"].float() + i["res"].float()).to(o["z"].dtype))
    y = D["z"] * D["rstd"][:, None] * D["gamma"]
    assert close(D["y"], y, u) and close(D["u"], y @ D["w"].t(), 2 * 2.0 ** -4 + u)
    logits = D["u"] @ D["out"].t()
    assert close(D["lse"], torch.logsumexp(logits, 1), 1e-5)
    d = torch.softmax(logits, 1)
    d[torch.arange(tokens), i["t"]] -= 1
    assert close(D["du"], d @ D["out"], 2 * u) and close(D["dout"], 0.5 * d.t() @ D["u"], 2 * u)
    assert close(D["dy"], D["du"] @ D["w"], 2.0 ** -3 + 2.0 ** -4 + u) and close(D["dw"], 0.5 * D["du"].t() @ D["y"], 2.0 ** -3 + 2.0 ** -4 + u)
    a, hat = D["dy"] * D["gamma"], D["z"] * D["rstd"][:, None]
    assert close(D["dgamma"], (D["dy"] * hat).sum(0), 1e-5)
    assert close(D["dz"], D["rstd"][:, None] * (a - hat * (a * hat).mean(1, keepdim=True)) + D["z"], u)


@pytest.mark.parametrize("tokens,width,hidden,vocab", [(40, 72, 100, 300), (700, 300, 512, 9000)])
@pytest.mark.parametrize("bf16", [False, True])
def test_a_captured_step_replays_to_the_eager_results_and_runs_on_another_stream(env, tokens, width, hidden, vocab, bf16):  # noqa: F811
    """Replayed three times, with eager runs of the same buffers and clobbered workspaces between; then two graphs that share a workspace, one after the other; then on a
    stream of its own."""
    torch, B = env
    dt = torch.bfloat16 if bf16 else torch.float32
    (_, o, ws, run), (_, o2, _, run2) = (sublayer(torch, B, tokens, width, hidden, vocab, dt, s) for s in (6, 7))
    run()
    run2()
    torch.cuda.synchronize()
    want, want2 = ({k: v.clone() for k, v in out.items()} for out in (o, o2))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
        run2()
    for turn in range(3):
        for v in (*o.values(), *o2.values()):
            v.zero_()
        ws.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for k in want:
            assert torch.equal(o[k], want[k]) and torch.equal(o2[k], want2[k]), (turn, k)
        run()
        torch.cuda.synchronize()
        for k in want:
            assert torch.equal(o[k], want[k]), (turn, k)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for v in o.values():
        v.zero_()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    side.synchronize()
    for k in want:
        assert torch.equal(o[k], want[k]), k


def test_matrices_of_no_rows(env):  # noqa: F811
    """An empty batch goes through every call; its tensors have no address."""
    torch, B = env
    st = B.Model.stream_handle()
    for dt in (torch.float32, torch.bfloat16):
        e, g, none = torch.empty(0, 40, dtype=dt, device="cuda:0"), torch.ones(40, device="cuda:0"), torch.empty(0, device="cuda:0")
        q, qt = B.q8_alloc(0, 40), B.q8_alloc(40, 0)
        B.conef_rms_forward(1e-5, e, e, g, e, e, q, none, st)
        B.conef_rms_backward(e, e, g, none, e, e, None, None, st)
        B.conef_q8_quantise(e, B.E5M2, q, qt, st)
        B.conef_q8_dequantise(q, B.E5M2, e, st)
        B.conef_q8_product(q, B.E5M2, B.q8_alloc(8, 40), 40, 1.0, 0.0, torch.empty(0, 8, dtype=dt, device="cuda:0"), None, st)
        c = torch.ones(40, 40, dtype=dt, device="cuda:0")
        B.conef_q8_product(qt, B.E5M2, qt, 0, 1.0, 0.0, c, None, st)
        torch.cuda.synchronize()
        assert (c == 0).all()


def test_binding_refuses_device_tensors_that_do_not_fit(env):  # noqa: F811
    """None of these reaches a kernel."""
    torch, B = env
    st = B.Model.stream_handle()
    z = lambda *s, **k: torch.zeros(*s, device="cuda:0", **k)                      # noqa: E731
    x, v, m, t, q = z(4, 8), z(8), z(4), z(4, dtype=torch.int64), B.q8_alloc(4, 8)
    w, ws = z(5, 8), z(B.conef_loss_workspace(4, 5, 8, torch.float32), dtype=torch.uint8)
    bad = [lambda a=a: B.conef_q8_quantise(a, B.E4M3, q, None, st) for a in (z(8, 4).t(), z(4, 8).double(), z(32), z(4, 16)[:, ::2], x.cpu(), z(4, 129))]
    bad += [lambda f=f: B.conef_q8_quantise(x, f, q, None, st) for f in (2, -1, 1 << 40)]
    bad += [lambda: B.conef_q8_quantise(x, B.E4M3, None, None, st), lambda: B.conef_q8_quantise(x, B.E4M3, (q[0], q[1].cpu()), None, st),
            lambda: B.conef_q8_quantise(x, B.E4M3, B.mx_alloc(4, 8), None, st), lambda: B.conef_q8_dequantise(q, B.E4M3, z(65, 8), st),
            lambda: B.conef_q8_dequantise(q, 3, x, st), lambda: B.conef_q8_product(q, B.E4M3, q, 129, 1.0, 0.0, z(4, 4), None, st),
            lambda: B.conef_q8_product(q, 2, q, 8, 1.0, 0.0, z(4, 4), None, st), lambda: B.conef_q8_product(q, B.E4M3, q, 8, 1.0, 0.0, z(4, 65), None, st)]
    bad += [lambda g=g: B.conef_rms_forward(1e-5, x, None, g, None, x, None, None, st) for g in (z(7), z(16)[::2], v.bfloat16(), v.cpu(), z(1, 8))]
    bad += [lambda: B.conef_rms_forward(1e-5, x, None, v, None, None, None, None, st), lambda: B.conef_rms_forward(1e-5, x, x, v, None, x, None, None, st),
            lambda: B.conef_rms_forward(-1.0, x, None, v, None, x, None, None, st), lambda: B.conef_rms_forward(1e-5, x, x, v, x, x, None, None, st),
            lambda: B.conef_rms_backward(x, x, v, m, None, x, v, None, st), lambda: B.conef_rms_backward(x, x, v, m, None, x, v, z(1), st),
            lambda: B.conef_rms_backward(x, z(4, 9), v, m, None, x, None, None, st), lambda: B.conef_rms_backward(x, x, v, m, None, None, None, None, st)]
    bad += [lambda a=a: B.conef_loss_forward(x, w, a, m, m.clone(), ws, st) for a in (t.int(), z(5, dtype=torch.int64), t.cpu(), m)]
    bad += [lambda a=a: B.conef_loss_forward(x, a, t, m, m.clone(), ws, st) for a in (z(5, 9), w.bfloat16(), w.cpu(), z(8, 5).t())]
    bad += [lambda: B.conef_loss_forward(x, w, t, None, None, ws, st), lambda: B.conef_loss_forward(x, w, t, m, None, None, st),
            lambda: B.conef_loss_forward(x, w, t, m, None, ws[:16], st), lambda: B.conef_loss_forward(x, w, t, z(5), None, ws, st),
            lambda: B.conef_loss_backward(x, w, t, m, None, 1.0, 0.0, None, None, ws, st), lambda: B.conef_loss_backward(x, w, t, None, None, 1.0, 0.0, z(4, 8), None, ws, st),
            lambda: B.conef_loss_backward(x, w, t, m, None, 1.0, 0.0, x, None, ws, st), lambda: B.conef_loss_backward(x, w, t, m, None, 1.0, 0.0, None, w, ws, st),
            lambda: B.conef_loss_backward(x, w, t, m, z(5), 1.0, 0.0, z(4, 8), None, ws, st), lambda: B.conef_loss_backward(x, w, t, m, None, 1.0, 0.0, z(4, 9), None, ws, st),
            lambda: B.conef_loss_backward(x, w, t, m, None, 1.0, 0.0, None, z(4, 8), ws, st)]
    for k, call in enumerate(bad):
        with pytest.raises(B.ConefError) as e:
            call()
        assert e.value.code == B.EINVAL, k
