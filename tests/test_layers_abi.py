"""Host side of the calls of a training step (conef_dropout_*, conef_norm_*, conef_mx_*): sizes, refusals, and that the reference
the GPU tests use draws what the library's generator is defined to draw.  No kernel is launched."""
import ctypes

import numpy as np
import pytest

import layers_ref as R
from paper_2312_08538_amd import binding as B

P = 4096           # an address that is never read: every call below is refused, or has nothing to do


def drop(p=0.1, site=0):
    return B.conef_drop(p=p, site=site, seed=1, step=2)


def test_reference_draws_are_the_generator_s_words():
    u = R.draws(3, 13, R.DROP + 5, 0x123456789ABCDEF0, (7 << 32) + 9)
    for i, j in [(0, 0), (0, 7), (1, 8), (2, 12)]:
        words = R.philox((i * 2 + j // 8, R.DROP + 5, 9, 7), (0x9ABCDEF0, 0x12345678))
        assert u[i, j] == words[(j & 7) >> 1] >> (16 * (j & 1)) & 0xFFFF
    # the published vector of the generator for a counter and key of zeros
    assert R.philox((0, 0, 0, 0), (0, 0)) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]


@pytest.mark.parametrize("p", [-0.1, 1.0, 1.5, float("nan"), float("inf")])
def test_a_share_dropped_outside_0_to_1_is_refused(p):
    L = B.lib()
    assert L.conef_dropout_forward(drop(p), 4, 8, 0, P, 8, 0, 0, P, 8, 0) == B.EINVAL
    assert L.conef_norm_forward(drop(p), 1e-5, 4, 8, 0, P, 8, 0, 0, P, P, P, 8, P, 8, P, P, 0) == B.EINVAL


def test_dropout_refuses_bad_arguments():
    L = B.lib()
    fwd = L.conef_dropout_forward
    assert fwd(None, 4, 8, 0, P, 8, 0, 0, P, 8, 0) == B.EINVAL
    assert fwd(drop(site=1 << 27), 4, 8, 0, P, 8, 0, 0, P, 8, 0) == B.EINVAL
    assert fwd(drop(), 4, 8, 2, P, 8, 0, 0, P, 8, 0) == B.EINVAL                  # type
    assert fwd(drop(), -1, 8, 0, P, 8, 0, 0, P, 8, 0) == B.EINVAL
    assert fwd(drop(), 4, 0, 0, P, 8, 0, 0, P, 8, 0) == B.EINVAL
    assert fwd(drop(), 1 << 20, 1 << 16, 0, P, 1 << 16, 0, 0, P, 1 << 16, 0) == B.EINVAL      # 2^33 octets
    assert fwd(drop(), 4, 8, 0, 0, 8, 0, 0, P, 8, 0) == B.EINVAL                  # no x
    assert fwd(drop(), 4, 8, 0, P, 8, 0, 0, 0, 8, 0) == B.EINVAL                  # no y
    assert fwd(drop(), 4, 8, 0, P + 2, 8, 0, 0, P, 8, 0) == B.EINVAL              # half an fp32 element off
    assert fwd(drop(), 4, 8, 1, P + 1, 8, 0, 0, P, 8, 0) == B.EINVAL
    assert fwd(drop(), 4, 8, 0, P, 7, 0, 0, P, 8, 0) == B.EINVAL                  # rows overlap
    assert fwd(drop(), 4, 8, 0, P, 8, P, 0, P, 8, 0) == B.EINVAL                  # residual without a pitch
    assert fwd(drop(), 0, 8, 0, 0, 0, 0, 0, 0, 0, 0) == B.OK                      # no rows: nothing to do
    assert L.conef_dropout_backward(drop(), 4, 8, 0, P, 8, 0, 8, 0) == B.EINVAL
    assert L.conef_dropout_backward(None, 0, 8, 0, 0, 8, 0, 8, 0) == B.EINVAL


def test_norm_refuses_bad_arguments():
    L = B.lib()

    def fwd(d=None, eps=1e-5, rows=4, cols=8, dtype=0, x=P, res=0, gamma=P, beta=P, z=0, y=2 * P, mean=P, rstd=P):
        return L.conef_norm_forward(d, eps, rows, cols, dtype, x, 8, res, 8, gamma, beta, z, 8, y, 8, mean, rstd, 0)

    for bad in [dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(cols=0), dict(rows=-1), dict(dtype=3), dict(x=0),
                dict(y=0), dict(gamma=0), dict(beta=0), dict(gamma=P + 2), dict(mean=P + 1), dict(z=P), dict(res=P), dict(d=drop()),
                dict(d=drop(), z=P, y=P), dict(d=drop(site=1 << 30), z=P), dict(x=P + 1, dtype=1), dict(cols=9)]:
        assert fwd(**bad) == B.EINVAL, bad
    assert fwd(rows=0, x=0, y=0, gamma=0, beta=0) == B.OK
    assert fwd(d=drop(), rows=0, x=0, y=0, z=0) == B.OK                           # an empty matrix may have no address

    def bwd(d=None, rows=4, cols=8, dtype=0, dy=P, z=P, gamma=P, mean=P, rstd=P, dz_in=0, dz=2 * P, dx=0, dgamma=P, dbeta=P, ws=P):
        return L.conef_norm_backward(d, rows, cols, dtype, dy, 8, z, 8, gamma, mean, rstd, dz_in, 8, dz, 8, dx, 8, dgamma, dbeta, ws, 0)

    for bad in [dict(dx=P), dict(d=drop(), dx=2 * P), dict(dz=0, dgamma=0, dbeta=0), dict(dy=0), dict(z=0), dict(gamma=0), dict(mean=0),
                dict(rstd=0), dict(ws=0), dict(ws=P + 4), dict(dgamma=P + 2), dict(cols=9), dict(dtype=-1), dict(rows=-2)]:
        assert bwd(**bad) == B.EINVAL, bad
    assert bwd(rows=0, dgamma=0, dbeta=0) == B.OK
    assert bwd(d=drop(), rows=0, dy=0, z=0, mean=0, rstd=0, dz=0, dgamma=0, dbeta=0, ws=0) == B.OK
    v = ctypes.c_size_t()
    assert L.conef_norm_workspace(4, 0, ctypes.byref(v)) == B.EINVAL
    assert L.conef_norm_workspace(4, 8, None) == B.EINVAL
    assert B.conef_norm_workspace(0, 8) == 0
    assert B.conef_norm_workspace(1, 8) >= 64


@pytest.mark.parametrize("rows,cols,codes,scales", [(0, 0, 0, 0), (1, 0, 0, 0), (0, 5, 0, 0), (1, 1, 64 * 64, 64 * 4), (64, 128, 4096, 256),
                                                    (65, 129, 128 * 128, 128 * 8), (50257, 768, 50304 * 384, 50304 * 24)])
def test_packed_sizes(rows, cols, codes, scales):
    assert B.conef_mx_sizes(rows, cols) == {"code_bytes": codes, "scale_bytes": scales}


def test_mx_calls_refuse_bad_arguments():
    L = B.lib()

    def quant(x=P, pitch=8, rows=4, cols=8, dtype=0, rounding=0, site=0, c=P, s=P, ct=0, st=0):
        return L.conef_mx_quantise(x, pitch, rows, cols, dtype, rounding, 1, site, 2, c, s, ct, st, 0)

    for bad in [dict(x=0), dict(x=P + 2), dict(pitch=7), dict(rows=-1), dict(cols=-1), dict(dtype=2), dict(rounding=2), dict(rounding=-1),
                dict(site=1 << 27), dict(c=0, s=0), dict(c=0), dict(s=0), dict(c=P + 8), dict(s=P + 4), dict(ct=P), dict(st=P),
                dict(rows=1 << 31), dict(rows=1 << 18, cols=1 << 18, pitch=1 << 18)]:
        assert quant(**bad) == B.EINVAL, bad
    assert quant(rows=0, x=0, c=0, s=0) == B.OK and quant(cols=0, x=0, c=0, s=0) == B.OK
    deq = L.conef_mx_dequantise
    assert deq(0, P, 4, 8, P, 8, 0, 0) == B.EINVAL and deq(P, P, 4, 8, P, 7, 0, 0) == B.EINVAL
    assert deq(P, P, 4, 8, P, 8, 5, 0) == B.EINVAL and deq(P, P + 1, 4, 8, P, 8, 0, 0) == B.EINVAL
    assert deq(0, 0, 0, 8, 0, 8, 0, 0) == B.OK

    def prod(a=P, sa=P, b=P, sb=P, m=4, n=8, k=32, c=P, pitch=8, dtype=0, ws=P):
        return L.conef_mx_product(a, sa, b, sb, m, n, k, 1.0, 0.0, c, pitch, dtype, ws, 0)

    for bad in [dict(a=0), dict(sa=0), dict(b=0), dict(sb=0), dict(a=P + 4), dict(c=0), dict(c=P + 2), dict(pitch=7), dict(m=-1), dict(n=-1),
                dict(k=-1), dict(dtype=2), dict(m=1 << 31), dict(m=1 << 18, n=1 << 18, pitch=1 << 18), dict(k=1 << 31)]:
        assert prod(**bad) == B.EINVAL, bad
    assert prod(m=0, c=0) == B.OK and prod(n=0, c=0) == B.OK
    v = ctypes.c_size_t()
    assert L.conef_mx_product_workspace(4, 4, -1, ctypes.byref(v)) == B.EINVAL
    assert L.conef_mx_product_workspace(4, 4, 4, None) == B.EINVAL
    # a deep product of few rows and columns is cut along its long axis; what it then needs is asked for, and refused if missing
    room = B.conef_mx_product_workspace(64, 64, 1 << 20)
    if room:
        assert prod(m=64, n=64, k=1 << 20, pitch=64, ws=0) == B.EINVAL
        assert prod(m=64, n=64, k=1 << 20, pitch=64, ws=P + 16) == B.EINVAL


def test_binding_refuses_tensors_that_do_not_fit():
    import torch

    x = torch.zeros(4, 8)
    st = 0
    for bad in [torch.zeros(8, 4).t(), torch.zeros(4, 8).double(), torch.zeros(32), torch.zeros(4, 16)[:, ::2]]:
        with pytest.raises(B.ConefError) as e:
            B.conef_dropout_backward(drop(), bad, x, st)
        assert e.value.code == B.EINVAL
    with pytest.raises(B.ConefError):
        B.conef_dropout_forward(drop(), x, torch.zeros(4, 9), x, st)              # another shape
    with pytest.raises(B.ConefError):
        B.conef_dropout_forward(drop(), x, x.bfloat16(), x, st)                   # another type
    with pytest.raises(B.ConefError):
        B.conef_norm_forward(None, 1e-5, x, None, torch.zeros(7), torch.zeros(8), None, x, None, None, st)
    with pytest.raises(B.ConefError):
        B.conef_norm_backward(None, x, x, torch.zeros(8), torch.zeros(4), torch.zeros(4), None, x, None, None, torch.zeros(8),
                              torch.zeros(1), st)                                  # workspace too small
    packed = tuple(torch.zeros(B.conef_mx_sizes(4, 8)[k], dtype=torch.uint8) for k in ("code_bytes", "scale_bytes"))
    with pytest.raises(B.ConefError):
        B.conef_mx_quantise(torch.zeros(4, 129), B.MX_NEAREST, 0, 0, 0, packed, None, st)       # operand too small
    with pytest.raises(B.ConefError):
        B.conef_mx_product(packed, packed, 129, 1.0, 0.0, torch.zeros(4, 4), None, st)


def test_binding_refuses_host_memory():
    """Everything about these tensors fits but where they are."""
    import torch

    x, v, m = torch.zeros(4, 8), torch.zeros(8), torch.zeros(4)
    packed = tuple(torch.zeros(B.conef_mx_sizes(4, 8)[k], dtype=torch.uint8) for k in ("code_bytes", "scale_bytes"))
    for call in [lambda: B.conef_dropout_forward(drop(), x, None, x, 0), lambda: B.conef_dropout_backward(drop(), x, x, 0),
                 lambda: B.conef_norm_forward(None, 1e-5, x, None, v, v, None, x.clone(), m, m, 0),
                 lambda: B.conef_norm_backward(None, x, x, v, m, m, None, x.clone(), None, None, None, None, 0),
                 lambda: B.conef_mx_quantise(x, B.MX_NEAREST, 0, 0, 0, packed, None, 0), lambda: B.conef_mx_dequantise(packed, x, 0),
                 lambda: B.conef_mx_product(packed, packed, 8, 1.0, 0.0, torch.zeros(4, 4), None, 0)]:
        with pytest.raises(B.ConefError) as e:
            call()
        assert e.value.code == B.EINVAL and "device" in str(e.value)


def test_reference_format_round_trip():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((5, 77)) * np.exp(rng.standard_normal((5, 1)) * 20)
    c, s = R.mx_encode(x)
    v = R.mx_decode(c, s)
    step = np.repeat(2.0 ** (s.astype(float) - 127), 32, 1)[:, :77]
    assert (np.abs(v - x) <= np.where(np.abs(x) >= 6 * step, 2.0, np.where(np.abs(x) >= 4 * step, 1.0, np.where(np.abs(x) >= 2 * step, 0.5, 0.25))) * step).all()
    assert (R.mx_decode(*R.mx_encode(v)) == v).all()                               # values of the format are kept


def test_binding_refuses_tensors_on_another_device_than_the_stream_s():
    """Tensors of two devices that are not there (no memory, no device behind them), and the library's calls as functions that do nothing:
    what is taken is taken, what is refused is refused by its device alone."""
    import torch
    from torch._subclasses.fake_tensor import FakeTensorMode

    calls, on = [], {0: 0, 7: 1}                        # stream 0 belongs to device 0, stream 7 to device 1
    nothing = ctypes.CFUNCTYPE(ctypes.c_int)(lambda: calls.append(1) or B.OK)
    sizes = ctypes.CFUNCTYPE(ctypes.c_int)(lambda: B.OK)

    @ctypes.CFUNCTYPE(ctypes.c_int, ctypes.c_size_t, ctypes.POINTER(ctypes.c_int))
    def device_of(stream, device):
        device[0] = on[stream]
        return 0

    at = lambda f: ctypes.cast(f, ctypes.c_void_p).value                           # noqa: E731
    face = B.face()
    face.connect(B.conef_drop, B.ConefError, (*(at(sizes if i in (3, 7) else nothing) for i in range(9)), at(device_of)))
    try:
        with FakeTensorMode():
            def args(d):
                z = lambda *s, **k: torch.empty(*s, device=f"cuda:{d}", **k)       # noqa: E731
                n = [z(B.conef_mx_sizes(4, 8)[k], dtype=torch.uint8) for k in ("code_bytes", "scale_bytes")]
                return {"x": z(4, 8), "v": z(8), "m": z(4), "q": tuple(n), "c": z(4, 4), "w": z(64, dtype=torch.uint8)}

            t = args(0), args(1)
        d = drop()
        forms = [  # every call, its tensors by name
            (lambda a, s: B.conef_dropout_forward(d, a[0], a[1], a[2], s), "xxx"), (lambda a, s: B.conef_dropout_backward(d, a[0], a[1], s), "xx"),
            (lambda a, s: B.conef_norm_forward(d, 1e-5, *a, s), "xxvvxxmm"), (lambda a, s: B.conef_norm_backward(d, *a, s), "xxvmmxxxvvw"),
            (lambda a, s: B.conef_mx_quantise(a[0], B.MX_NEAREST, 0, 0, 0, a[1], None, s), "xq"), (lambda a, s: B.conef_mx_dequantise(a[0], a[1], s), "qx"),
            (lambda a, s: B.conef_mx_product(a[0], a[1], 8, 1.0, 0.0, a[2], a[3], s), "qqcw")]
        for call, names in forms:
            for stream, device in on.items():
                before = len(calls)
                call([t[device][n] for n in names], stream)
                assert len(calls) == before + 1, names
                for i in range(len(names)):                                        # one of them elsewhere, and all of them
                    for wrong in ({i}, set(range(len(names)))):
                        with pytest.raises(B.ConefError) as e:
                            call([t[1 - device if k in wrong else device][n] for k, n in enumerate(names)], stream)
                        assert e.value.code == B.EINVAL and f"cuda:{device}" in str(e.value), (names, i)
                # codes and scales apart
                if "q" in names:
                    mixed = (t[device]["q"][0], t[1 - device]["q"][1])
                    with pytest.raises(B.ConefError):
                        call([mixed if n == "q" else t[device][n] for n in names], stream)
                assert len(calls) == before + 1
    finally:
        B._face = None
        B.face()
