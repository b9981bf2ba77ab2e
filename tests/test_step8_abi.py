"""Host side of the calls of a step in 8 bits (conef_q8_*, conef_rms_*, conef_loss_*): sizes, refusals, and that the reference the GPU tests use is the format that the header
states.  No kernel is launched."""
import ctypes

import numpy as np
import pytest

import step8_ref as R
from paper_2312_08538_amd import binding as B

P = 4096           # an address that is never read: every call below is refused, or has nothing to do


@pytest.mark.parametrize("rows,cols,codes,scales", [(0, 0, 0, 0), (1, 0, 0, 0), (0, 5, 0, 0), (1, 1, 64 * 128, 64), (64, 128, 8192, 64),
                                                    (65, 129, 128 * 256, 128 * 2), (50257, 768, 50304 * 768, 50304 * 6)])
def test_packed_sizes(rows, cols, codes, scales):
    assert B.conef_q8_sizes(rows, cols) == {"code_bytes": codes, "scale_bytes": scales}


def test_q8_calls_refuse_bad_arguments():
    L = B.lib()

    def quant(x=P, pitch=8, rows=4, cols=8, dtype=0, form=0, c=P, s=P, ct=0, st=0):
        return L.conef_q8_quantise(x, pitch, rows, cols, dtype, form, c, s, ct, st, 0)

    for bad in [dict(x=0), dict(x=P + 2), dict(pitch=7), dict(rows=-1), dict(cols=-1), dict(dtype=2), dict(form=2), dict(form=-1), dict(c=0, s=0), dict(c=0),
                dict(s=0), dict(c=P + 8), dict(s=P + 4), dict(ct=P), dict(st=P), dict(rows=1 << 31), dict(rows=1 << 30, cols=1, pitch=1),
                dict(rows=1 << 18, cols=1 << 18, pitch=1 << 18)]:
        assert quant(**bad) == B.EINVAL, bad
    assert quant(rows=0, x=0, c=0, s=0) == B.OK and quant(cols=0, x=0, c=0, s=0) == B.OK
    deq = L.conef_q8_dequantise
    assert deq(0, P, 4, 8, 0, P, 8, 0, 0) == B.EINVAL and deq(P, P, 4, 8, 0, P, 7, 0, 0) == B.EINVAL
    assert deq(P, P, 4, 8, 2, P, 8, 0, 0) == B.EINVAL and deq(P, P, 4, 8, 0, P, 8, 5, 0) == B.EINVAL and deq(P, P + 1, 4, 8, 0, P, 8, 0, 0) == B.EINVAL
    assert deq(0, 0, 0, 8, 0, 0, 8, 0, 0) == B.OK

    def prod(a=P, sa=P, form=0, b=P, sb=P, m=4, n=8, k=32, c=P, pitch=8, dtype=0, ws=P):
        return L.conef_q8_product(a, sa, form, b, sb, m, n, k, 1.0, 0.0, c, pitch, dtype, ws, 0)

    for bad in [dict(a=0), dict(sa=0), dict(b=0), dict(sb=0), dict(a=P + 4), dict(form=2), dict(c=0), dict(c=P + 2), dict(pitch=7), dict(m=-1), dict(n=-1),
                dict(k=-1), dict(dtype=2), dict(m=1 << 31), dict(m=1 << 18, n=1 << 18, pitch=1 << 18), dict(k=1 << 31)]:
        assert prod(**bad) == B.EINVAL, bad
    assert prod(m=0, c=0) == B.OK and prod(n=0, c=0) == B.OK
    v = ctypes.c_size_t()
    assert L.conef_q8_product_workspace(4, 4, -1, ctypes.byref(v)) == B.EINVAL and L.conef_q8_product_workspace(4, 4, 4, None) == B.EINVAL
    # a deep product of few columns is cut along its long axis; what it then needs is refused if missing
    m, n, k = 128, 64, 1 << 20
    assert B.conef_q8_product_workspace(m, n, k) > 0
    assert prod(m=m, n=n, k=k, pitch=n, ws=0) == B.EINVAL and prod(m=m, n=n, k=k, pitch=n, ws=P + 16) == B.EINVAL


def test_norm_refuses_bad_arguments():
    L = B.lib()

    def fwd(eps=1e-5, rows=4, cols=8, dtype=0, x=P, xp=8, res=0, gamma=P, z=0, y=2 * P, yp=8, c=0, s=0, rstd=P):
        return L.conef_rms_forward(eps, rows, cols, dtype, x, xp, res, 8, gamma, z, 8, y, yp, c, s, rstd, 0)

    for bad in [dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(cols=0), dict(rows=-1), dict(dtype=3), dict(x=0), dict(y=0), dict(gamma=0),
                dict(gamma=P + 2), dict(rstd=P + 1), dict(z=P), dict(res=P), dict(res=P, z=P, y=P), dict(x=P + 1, dtype=1), dict(cols=9), dict(xp=7),
                dict(yp=7), dict(c=P), dict(s=P), dict(c=P + 8, s=P), dict(c=P, s=P + 8), dict(y=0, c=P, s=P, rows=1 << 30, cols=1)]:
        assert fwd(**bad) == B.EINVAL, bad
    assert fwd(rows=0, x=0, y=0, gamma=0) == B.OK and fwd(rows=0, res=P, z=0, c=0, y=0) == B.OK

    def bwd(rows=4, cols=8, dtype=0, dy=P, z=P, gamma=P, rstd=P, dz_in=0, dz=2 * P, dgamma=P, ws=P, pitch=8):
        return L.conef_rms_backward(rows, cols, dtype, dy, pitch, z, 8, gamma, rstd, dz_in, 8, dz, 8, dgamma, ws, 0)

    for bad in [dict(dz=0, dgamma=0), dict(dy=0), dict(z=0), dict(gamma=0), dict(rstd=0), dict(ws=0), dict(ws=P + 4), dict(dgamma=P + 2), dict(cols=9),
                dict(dtype=-1), dict(rows=-2), dict(pitch=7), dict(dz_in=P + 1)]:
        assert bwd(**bad) == B.EINVAL, bad
    assert bwd(rows=0, dgamma=0) == B.OK and bwd(rows=0, dy=0, z=0, rstd=0, dz=0, dgamma=0, ws=0) == B.OK
    v = ctypes.c_size_t()
    assert L.conef_rms_workspace(4, 0, ctypes.byref(v)) == B.EINVAL and L.conef_rms_workspace(4, 8, None) == B.EINVAL
    assert B.conef_rms_workspace(0, 8) == 0 and B.conef_rms_workspace(1, 8) >= 32


def test_loss_refuses_bad_arguments():
    L = B.lib()

    def fwd(t=4, v=9, d=8, dtype=0, x=P, xp=8, w=P, wp=8, targets=P, loss=P, lse=2 * P, ws=P):
        return L.conef_loss_forward(t, v, d, dtype, x, xp, w, wp, targets, loss, lse, ws, 0)

    sizes = [dict(t=-1), dict(v=0), dict(d=0), dict(v=-3), dict(t=1 << 30), dict(v=1 << 30), dict(d=1 << 30, xp=1 << 30, wp=1 << 30), dict(t=1 << 20, v=1 << 15),
             dict(v=1 << 18, d=1 << 17, xp=1 << 17, wp=1 << 17), dict(dtype=2), dict(dtype=-1)]
    for bad in sizes + [dict(x=0), dict(w=0), dict(x=P + 2), dict(w=P + 2), dict(xp=7), dict(wp=7), dict(targets=0), dict(targets=P + 4), dict(loss=0, lse=0), dict(loss=2 * P),
                        dict(loss=P + 2), dict(lse=P + 2), dict(ws=0), dict(ws=P + 128)]:
        assert fwd(**bad) == B.EINVAL, bad
    assert fwd(t=0, x=0, w=0, targets=0, loss=0, lse=0, ws=0) == B.OK

    def bwd(t=4, v=9, d=8, dtype=0, x=P, xp=8, w=2 * P, wp=8, targets=P, lse=P, dloss=0, dx=3 * P, dxp=8, dw=4 * P, dwp=8, ws=P):
        return L.conef_loss_backward(t, v, d, dtype, x, xp, w, wp, targets, lse, dloss, 1.0, 0.0, dx, dxp, dw, dwp, ws, 0)

    for bad in sizes + [dict(x=0), dict(w=0), dict(xp=7), dict(wp=7), dict(targets=0), dict(lse=0), dict(lse=P + 1), dict(dloss=P + 2), dict(dx=0, dw=0), dict(dxp=7),
                        dict(dwp=7), dict(dx=P + 2), dict(dw=P + 2), dict(ws=0), dict(ws=P + 64), dict(dx=P), dict(dx=2 * P), dict(dw=P), dict(dw=2 * P),
                        dict(dx=4 * P)]:
        assert bwd(**bad) == B.EINVAL, bad
    assert bwd(t=0, x=0, w=0, targets=0, lse=0, dx=0, dw=0, ws=0) == B.OK
    v = ctypes.c_size_t()
    assert L.conef_loss_workspace(4, 9, 8, 0, None) == B.EINVAL and L.conef_loss_workspace(4, 0, 8, 0, ctypes.byref(v)) == B.EINVAL
    assert L.conef_loss_workspace(4, 9, 8, 3, ctypes.byref(v)) == B.EINVAL


def test_a_loss_works_on_pieces_of_the_vocabulary():
    """Its workspace does not hold the logits of a large batch, nor the whole of a weight once more."""
    import torch

    tokens, vocab, width = 4096, 50304, 2048
    room = B.conef_loss_workspace(tokens, vocab, width, torch.bfloat16)
    assert room < 2 * tokens * vocab and room == B.conef_loss_workspace(tokens, vocab, width, B.BF16)
    assert B.conef_loss_workspace(65536, 50304, 2048, torch.bfloat16) < 65536 * 50304 * 2 // 2
    with pytest.raises(B.ConefError):
        B.conef_loss_workspace(tokens, vocab, width, torch.float16)


def test_reference_format():
    import torch

    for form, kind in ((R.E4M3, torch.float8_e4m3fn), (R.E5M2, torch.float8_e5m2)):
        codes = torch.arange(256, dtype=torch.uint8)
        want, got = codes.view(kind).double().numpy(), R.table(form)
        fits = np.isfinite(want)
        assert (got[fits] == want[fits]).all() and np.abs(got[fits]).max() == R.LARGEST[form]
        rng = np.random.default_rng(3)
        x = rng.standard_normal((5, 300)) * np.exp(rng.standard_normal((5, 1)) * 20)
        c, s = R.encode(x, form)
        v = R.decode(c, s, form)
        step = np.repeat(2.0 ** (s.astype(float) - 127), 128, 1)[:, :300]
        # half a step of the element's own power, or of the format's smallest
        assert (np.abs(v - x) <= np.maximum(np.abs(x) * 2.0 ** -(R.BITS[form] + 1), step * 2.0 ** (-R.BIAS[form] - R.BITS[form]))).all()
        assert (R.decode(*R.encode(v, form), form) == v).all()
        # no smaller scale would do
        most = np.abs(np.pad(x, ((0, 0), (0, 84)))).reshape(5, 3, 128).max(-1)
        assert (most <= R.LARGEST[form] * 2.0 ** (s.astype(float) - 127)).all() and (most > R.LARGEST[form] * 2.0 ** (s.astype(float) - 128)).all()


def test_binding_refuses_host_memory():
    """Everything about these tensors fits but where they are."""
    import torch

    x, v, m, t, w = torch.zeros(4, 8), torch.zeros(8), torch.zeros(4), torch.zeros(4, dtype=torch.int64), torch.zeros(5, 8)
    packed = tuple(torch.zeros(B.conef_q8_sizes(4, 8)[k], dtype=torch.uint8) for k in ("code_bytes", "scale_bytes"))
    ws = torch.zeros(B.conef_loss_workspace(4, 5, 8, torch.float32), dtype=torch.uint8)
    for call in [lambda: B.conef_q8_quantise(x, B.E4M3, packed, None, 0), lambda: B.conef_q8_dequantise(packed, B.E4M3, x, 0),
                 lambda: B.conef_q8_product(packed, B.E4M3, packed, 8, 1.0, 0.0, torch.zeros(4, 4), None, 0),
                 lambda: B.conef_rms_forward(1e-5, x, None, v, None, x.clone(), packed, m, 0),
                 lambda: B.conef_rms_backward(x, x, v, m, None, x.clone(), None, None, 0), lambda: B.conef_loss_forward(x, w, t, m, m.clone(), ws, 0),
                 lambda: B.conef_loss_backward(x, w, t, m, None, 1.0, 0.0, x.clone(), None, ws, 0)]:
        with pytest.raises(B.ConefError) as e:
            call()
        assert e.value.code == B.EINVAL and "device" in str(e.value)


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
    face.connect(B.conef_drop, B.ConefError, (*(at(nothing) for _ in range(9)), at(device_of)))
    face.connect_8bit(tuple(at(sizes if i in (2, 5, 7) else nothing) for i in range(10)))
    try:
        with FakeTensorMode():
            def args(d):
                z = lambda *s, **k: torch.empty(*s, device=f"cuda:{d}", **k)       # noqa: E731
                n = [z(B.conef_q8_sizes(4, 8)[k], dtype=torch.uint8) for k in ("code_bytes", "scale_bytes")]
                return {"x": z(4, 8), "v": z(8), "m": z(4), "q": tuple(n), "c": z(4, 4), "w": z(64, dtype=torch.uint8), "t": z(4, dtype=torch.int64), "e": z(5, 8)}

            t = args(0), args(1)
        forms = [  # every call, its tensors by name
            (lambda a, s: B.conef_q8_quantise(a[0], B.E4M3, a[1], None, s), "xq"), (lambda a, s: B.conef_q8_dequantise(a[0], B.E5M2, a[1], s), "qx"),
            (lambda a, s: B.conef_q8_product(a[0], B.E5M2, a[1], 8, 1.0, 0.0, a[2], a[3], s), "qqcw"), (lambda a, s: B.conef_rms_forward(1e-5, *a, s), "xxvxxqm"),
            (lambda a, s: B.conef_rms_backward(*a, s), "xxvmxxvw"), (lambda a, s: B.conef_loss_forward(*a, s), "xetmmw"),
            (lambda a, s: B.conef_loss_backward(*a[:5], 1.0, 0.0, *a[5:], s), "xetmmxew")]
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
                if "q" in names:                                                   # codes and scales apart
                    mixed = (t[device]["q"][0], t[1 - device]["q"][1])
                    with pytest.raises(B.ConefError):
                        call([mixed if n == "q" else t[device][n] for n in names], stream)
                assert len(calls) == before + 1
    finally:
        B._face = None
        B.face()
