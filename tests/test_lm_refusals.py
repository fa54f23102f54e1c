"""What the output-end operators refuse, on the host: nothing is launched, no GPU is needed."""
import pytest
import torch


@pytest.fixture(scope="module")
def b():
    from paper_2510_11168_amd import build
    if not build.is_built():
        build.build()
    from paper_2510_11168_amd import binding
    return binding


def refused(b, code, fn, *a, **kw):
    with pytest.raises(b.ElmoError) as e:
        fn(*a, **kw)
    assert e.value.code == code and len(str(e.value)) > 20, str(e.value)
    return str(e.value)


def f(*s):
    return torch.zeros(s)


def i8(*s):
    return torch.zeros(s, dtype=torch.int8)


def i32(*s):
    return torch.zeros(s, dtype=torch.int32)


def test_tensors_that_do_not_fit_together(b):
    bf = torch.bfloat16
    refused(b, -1, b.elmo_rms_norm, None, f(2, 8))
    refused(b, -2, b.elmo_rms_norm, f(2, 8).double(), f(2, 8))
    refused(b, -2, b.elmo_rms_norm, f(2, 8), f(2, 8).half())
    refused(b, -1, b.elmo_rms_norm, f(2, 8), f(2, 9))
    refused(b, -1, b.elmo_rms_norm, f(2, 8), f(8, 2).t())
    refused(b, -1, b.elmo_rms_norm, f(16), f(16))
    refused(b, -2, b.elmo_rms_norm, f(2, 8), f(2, 8), residual=f(2, 8).to(bf))
    refused(b, -1, b.elmo_rms_norm, f(2, 8), f(2, 8), f(16)[::2])
    refused(b, -1, b.elmo_rms_norm, f(2, 8), i8(2, 8), scale_out=f(3))
    refused(b, -2, b.elmo_rms_norm_backward, f(2, 8), f(2, 8).to(bf), f(2, 8))
    refused(b, -2, b.elmo_rms_norm_backward, f(2, 8), f(2, 8), f(2, 8), dweight=f(8).to(bf))
    refused(b, -2, b.elmo_int8_matmul, f(2, 8), f(2), i8(3, 8), f(3), f(2, 3))
    refused(b, -1, b.elmo_int8_matmul, i8(2, 8), f(2), i8(3, 9), f(3), f(2, 3))
    refused(b, -1, b.elmo_int8_matmul, i8(2, 8), f(3), i8(3, 8), f(3), f(2, 3))
    refused(b, -1, b.elmo_int8_matmul, i8(2, 8), f(2), i8(8, 3).t(), f(3), f(2, 3))
    refused(b, -1, b.elmo_int8_matmul, i8(2, 8), f(2), i8(3, 8), f(3), f(2, 3), bias=f(2))
    refused(b, -1, b.elmo_sample, f(2, 8), f(3), i32(2))
    refused(b, -2, b.elmo_sample, f(2, 8), f(2), i32(2).long())
    refused(b, -2, b.elmo_sample, f(2, 8), f(2), i32(2), top_k=f(2))
    refused(b, -1, b.elmo_sample, f(2, 8), f(2), i32(2), top_p=f(4)[::2])
    refused(b, -1, b.elmo_distill, f(2, 8), i32(2, 3), f(2, 4), f(2))
    refused(b, -2, b.elmo_distill, f(2, 8), i32(2, 3).long(), f(2, 3), f(2))
    refused(b, -1, b.elmo_distill, f(2, 8), i32(2, 6)[:, :3], f(2, 3), f(2))
    refused(b, -2, b.elmo_distill, f(2, 8), i32(2, 3), f(2, 3), f(2), f(2, 8).to(bf))
    refused(b, -1, b.elmo_distill, f(2, 8), i32(2, 3), f(2, 3), f(2), f(2, 7))


def test_every_needed_tensor_is_named(b):
    calls = [(b.elmo_rms_norm, [f(2, 8), f(2, 8)]), (b.elmo_rms_norm_backward, [f(2, 8), f(2, 8), f(2, 8)]),
             (b.elmo_int8_matmul, [i8(2, 8), f(2), i8(3, 8), f(3), f(2, 3)]), (b.elmo_sample, [f(2, 8), f(2), i32(2)]),
             (b.elmo_distill, [f(2, 8), i32(2, 3), f(2, 3), f(2)])]
    for fn, tensors in calls:
        for i in range(len(tensors)):
            assert "needed" in refused(b, -1, fn, *tensors[:i], None, *tensors[i + 1:])


def test_host_tensors_are_refused(b):
    assert "GPU" in refused(b, -1, b.elmo_rms_norm, f(2, 8), f(2, 8))
    assert "GPU" in refused(b, -1, b.elmo_rms_norm_backward, f(2, 8), f(2, 8), f(2, 8))
    assert "GPU" in refused(b, -1, b.elmo_int8_matmul, i8(2, 8), f(2), i8(3, 8), f(3), f(2, 3))
    assert "GPU" in refused(b, -1, b.elmo_sample, f(2, 8), f(2), i32(2))
    assert "GPU" in refused(b, -1, b.elmo_distill, f(2, 8), i32(2, 3), f(2, 3), f(2))


P = 4096        # an address that is never read: the calls below end in the host's checks


def _norm(b, **kw):
    a = dict(x=P, xs=64, dt=b.ELMO_BF16, rows=4, d=64, r=None, rs=0, w=None, wt=0, eps=1e-6, s=None, ss=0, y=P, ys=64, yt=b.ELMO_BF16, sc=None)
    a.update(kw)
    b._check(b._lib.elmo_rms_norm(*a.values(), None))


def _back(b, **kw):
    a = dict(dy=P, dys=64, h=P, hs=64, dt=b.ELMO_FP32, rows=4, d=64, w=None, wt=0, eps=1e-6, s=None, ss=0, dh=P, dhs=64, dw=None, ws=None, n=0)
    a.update(kw)
    b._check(b._lib.elmo_rms_norm_backward(*a.values(), None))


def _int8(b, **kw):
    a = dict(a=P, as_=64, sa=P, w=P, bs=64, sb=P, bias=None, M=4, N=4, K=64, out=P, os=4, t=b.ELMO_BF16)
    a.update(kw)
    b._check(b._lib.elmo_int8_matmul(*a.values(), None))


def _sample(b, **kw):
    a = dict(z=P, zs=64, dt=b.ELMO_BF16, rows=4, V=64, u=P, t=None, k=None, p=None, m=None, i=P, q=None, ws=None, n=0)
    a.update(kw)
    b._check(b._lib.elmo_sample(*a.values(), None))


def _distill(b, **kw):
    a = dict(z=P, zs=64, dt=b.ELMO_BF16, rows=4, V=64, i=P, t=P, tt=b.ELMO_FP32, K=8, T=1.0, v=None, loss=P, g=None, gs=0, ws=None, n=0)
    a.update(kw)
    b._check(b._lib.elmo_distill(*a.values(), None))


NAN = float("nan")


@pytest.mark.parametrize("call,code,kw", [
    (_norm, -2, dict(dt=1)), (_norm, -2, dict(dt=7)), (_norm, -2, dict(yt=9)), (_norm, -2, dict(w=P, wt=1)), (_norm, -1, dict(rows=-1)),
    (_norm, -1, dict(rows=1 << 31)), (_norm, -1, dict(d=0)), (_norm, -1, dict(d=16385)), (_norm, -1, dict(eps=-1.0)), (_norm, -1, dict(eps=NAN)),
    (_norm, -1, dict(x=None)), (_norm, -1, dict(y=None)), (_norm, -1, dict(xs=63)), (_norm, -1, dict(ys=-64)), (_norm, -1, dict(r=P, rs=10)),
    (_norm, -1, dict(s=P, ss=64)), (_norm, -1, dict(yt=3)), (_norm, -1, dict(sc=P)), (_norm, -1, dict(x=P + 1)), (_norm, -1, dict(xs=1 << 41)),
    (_back, -2, dict(dt=3)), (_back, -1, dict(d=70000)), (_back, -1, dict(dw=P)), (_back, -1, dict(dw=P, ws=P, n=100)), (_back, -1, dict(dh=None)),
    (_back, -1, dict(h=P + 2)), (_back, -1, dict(s=P, ss=3)), (_back, -1, dict(eps=NAN)),
    (_int8, -2, dict(t=1)), (_int8, -1, dict(K=131072)), (_int8, -1, dict(K=-1)), (_int8, -1, dict(M=-1)), (_int8, -1, dict(N=(1 << 30) + 1)),
    (_int8, -1, dict(a=None)), (_int8, -1, dict(sb=None)), (_int8, -1, dict(as_=63)), (_int8, -1, dict(os=3)), (_int8, -1, dict(out=P + 1)),
    (_int8, -1, dict(bias=P + 2)),
    (_sample, -2, dict(dt=1)), (_sample, -1, dict(V=0)), (_sample, -1, dict(V=1 << 31)), (_sample, -1, dict(rows=-2)), (_sample, -1, dict(u=None)),
    (_sample, -1, dict(i=None)), (_sample, -1, dict(zs=63)), (_sample, -1, dict(k=P + 2)), (_sample, -1, dict(z=P + 1)),
    (_distill, -2, dict(dt=1)), (_distill, -2, dict(tt=3)), (_distill, -1, dict(K=0)), (_distill, -1, dict(K=1025)), (_distill, -1, dict(T=0.0)),
    (_distill, -1, dict(T=NAN)), (_distill, -1, dict(T=-1.0)), (_distill, -1, dict(T=1e9)), (_distill, -1, dict(V=0)), (_distill, -1, dict(loss=None)),
    (_norm, -1, dict(rows=1 << 27)), (_norm, -1, dict(rows=1 << 25, d=2048, xs=2048, ys=2048)), (_sample, -1, dict(rows=1 << 23)),
    (_distill, -1, dict(rows=1 << 24)), (_int8, -1, dict(M=1 << 30, N=1 << 30, os=1 << 30)),
    (_distill, -1, dict(g=P, gs=5)), (_distill, -1, dict(t=P + 2)), (_distill, -1, dict(i=None)),
])
def test_arguments_that_the_library_refuses(b, call, code, kw):
    refused(b, code, call, b, **kw)


def test_calls_without_rows_do_nothing(b):
    _norm(b, rows=0, x=None, y=None)
    _back(b, rows=0, dy=None, h=None, dh=None)
    _int8(b, M=0, a=None)
    _int8(b, N=0, w=None)
    _sample(b, rows=0, z=None)
    _distill(b, rows=0, z=None)


def test_missing_or_small_workspaces_are_refused(b):
    for call, kw in ((_sample, dict(V=1 << 17, zs=1 << 17, rows=2)), (_distill, dict(V=1 << 17, zs=1 << 17, rows=2))):
        need = (b.elmo_sample_bytes if call is _sample else b.elmo_distill_bytes)(2, 1 << 17)
        assert need > 0
        for ws, n in ((None, 0), (P, need - 1), (P + 64, need)):
            assert "workspace" in refused(b, -1, call, b, ws=ws, n=n, **kw)


def test_workspaces(b):
    assert b.elmo_rms_norm_backward_bytes(0, 64) == 0 and 64 * 4 <= b.elmo_rms_norm_backward_bytes(3, 64) <= 3 * 64 * 4
    big = b.elmo_rms_norm_backward_bytes(1 << 20, 4096)
    assert 0 < big <= 4096 * 4096 * 4                        # it does not grow with the rows
    for fn in (b.elmo_sample_bytes, b.elmo_distill_bytes):
        assert fn(0, 5) == 0 and fn(5, 0) == 0
        assert fn(1 << 20, 1 << 17) <= 1 << 28
