"""The operators at the output end of a language model against their 64-bit statements, through the binding.

Tolerances, in units of e = 2^-24 (half a step of FP32, relative) and half = half a step of the output type:
  FP32 sums of n terms in lanes and trees are off by at most (terms one lane adds + levels of the tree) e times the sum of magnitudes;
  v_exp_f32 by 2 e, a product, quotient or square root by e each (2 e where the compiler's division is not correctly rounded).
"""
import numpy as np
import pytest
import torch

from oracle import lm_oracle as o

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
E = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: E, torch.float8_e4m3fn: 2.0 ** -4}
TINY = {torch.bfloat16: 1e-38, torch.float32: 1e-38}


@pytest.fixture(scope="module")
def b():
    from paper_2510_11168_amd import binding
    return binding


def rows_of(t, pad, first=0):
    """The same values as rows of a wider buffer that begins `first` elements behind an aligned address; what is between rows is 72 (a value of every type)."""
    n, d = t.shape
    wide = torch.full((first + n * (d + pad),), 72, dtype=t.dtype, device=t.device)
    v = wide[first:].view(n, d + pad)[:, :d]
    v.copy_(t)
    return v


def between_rows(v):
    """What lies between the rows of `v` in its buffer."""
    n, d = v.shape
    return torch.as_strided(v, (n, v.stride(0)), (v.stride(0), 1))[:, d:] if n > 1 and v.stride(0) > d else None


def f64(t):
    return t.to(torch.float64).cpu().numpy()


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def close(got, want, tol, what):
    err = np.abs(f64(got) - want)
    assert np.all(np.isfinite(f64(got))), what
    worst = float(np.max(err / tol)) if err.size else 0.0
    assert np.all(err <= tol), f"{what}: {worst:.3g} times the tolerance"


# ------------------------------------------------------------------ norm
NORM_SHAPES = [(1, 1), (1, 768), (3, 7), (5, 8), (2, 511), (7, 513), (4, 1000), (3, 2049), (2, 4096), (2, 4104), (1, 8193), (3, 12011), (1, 16384),
               (4100, 65), (4099, 1030), (4097, 4096)]


@pytest.mark.parametrize("rows,d", NORM_SHAPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_norm_and_its_8_bit_rows(b, rows, d, dtype):
    g = gen(rows * 7 + d)
    x, r = torch.randn((rows, d), generator=g).to(dtype), (3 * torch.randn((rows, d), generator=g)).to(dtype)
    w = (1 + 0.3 * torch.randn(d, generator=g)).to(torch.float32 if d % 2 else torch.bfloat16)
    if rows > 1:
        x[rows // 2], r[rows // 2] = 0, 0                    # a row of zeros
    h32 = x.float() + r.float()
    y64, h64, rms = o.rms_norm(f64(x), f64(w), 1e-5, f64(r))
    lane = 8 * 8 + 12                                        # terms of a lane and levels of the tree, with the waves' sums
    rel = (lane / 2 + 8) * E
    pad, first = (0, 0) if d % 8 == 0 and rows % 2 else (3, 1)
    xd, rd, wd = rows_of(x.to(DEV), pad, first), rows_of(r.to(DEV), pad), w.to(DEV)
    for out in (torch.bfloat16, torch.float32, torch.int8, torch.float8_e4m3fn):
        y = rows_of(torch.zeros((rows, d), dtype=out, device=DEV), pad, first)
        s = rows_of(torch.zeros((rows, d), dtype=dtype, device=DEV), pad)
        eight = out in (torch.int8, torch.float8_e4m3fn)
        scale = torch.full((rows,), -1.0, device=DEV) if eight else None
        b.elmo_rms_norm(xd, y, wd, 1e-5, residual=rd, sum_out=s, scale_out=scale)
        assert torch.equal(s.cpu(), h32.to(dtype)), "the stream is the rounded sum"
        if eight:
            most = 127 if out == torch.int8 else 448
            q, m = o.rows_in_8_bits(h32.numpy(), f64(w), most)
            if out == torch.int8:
                assert np.array_equal(y.cpu().numpy(), np.rint(q).astype(np.int8))
            else:
                assert torch.equal(y.cpu().view(torch.uint8), torch.from_numpy(q.astype(np.float32)).to(out).view(torch.uint8))
            close(scale, (m / (most * rms))[:, 0], rel * (m / (most * rms))[:, 0] + 1e-38, "scale")
        else:
            close(y, y64, (HALF[out] + rel) * np.abs(y64) + 3 * E * np.abs(f64(w)) * np.abs(h64) / rms + 1e-38, "y")
        for v in (y, s):
            gap = between_rows(v)
            assert gap is None or bool((gap.float() == 72).all()), "nothing between the rows is written"


def test_norm_without_residual_or_weight_and_in_place(b):
    x = torch.randn((37, 300), generator=gen(1)).to(DEV)
    y = torch.empty_like(x)
    b.elmo_rms_norm(x, y, None, 0.0)
    want = o.rms_norm(f64(x), None, 0.0)[0]
    close(y, want, 60 * E * np.abs(want) + 1e-38, "y")
    r = torch.randn((37, 300), generator=gen(2)).to(DEV)
    ref, stream = torch.empty_like(x), torch.empty_like(x)
    b.elmo_rms_norm(x, ref, None, 1e-6, residual=r, sum_out=stream)
    xi, ri = x.clone(), r.clone()
    b.elmo_rms_norm(xi, xi, None, 1e-6, residual=ri, sum_out=ri)   # y over x, the stream over the residual
    assert torch.equal(xi, ref) and torch.equal(ri, stream)


def test_norm_rows_that_hold_infinities_and_nan(b):
    x = torch.ones((6, 260), device=DEV)
    x[1, 5], x[2, 255], x[3, 0], x[4] = float("nan"), float("inf"), -float("inf"), 3e38
    q, scale = torch.full((6, 260), 9, dtype=torch.int8, device=DEV), torch.empty(6, device=DEV)
    b.elmo_rms_norm(x, q, None, 1e-6, scale_out=scale)
    assert bool(torch.isnan(scale[1:5]).all()) and not q[1:5].any()
    assert bool((q[[0, 5]] == 127).all()) and bool(torch.isfinite(scale[[0, 5]]).all())
    b.elmo_rms_norm(torch.zeros_like(x), q, None, 0.0, scale_out=scale)
    assert not q.any() and not scale.any(), "zeros have scale 0 without eps too"
    w = torch.ones(260, device=DEV)
    w[7] = float("nan")
    b.elmo_rms_norm(x, q, w, 1e-6, scale_out=scale)
    assert bool(torch.isnan(scale).all()), "a weight that is NaN reaches every row's scale"
    y = torch.empty_like(x)
    b.elmo_rms_norm(x, y, None, 1e-6)
    assert bool(torch.isnan(y[1]).all()) and bool(torch.isfinite(y[[0, 5]]).all())


@pytest.mark.parametrize("rows,d", [(0, 64), (1, 1), (1, 768), (3, 9), (2, 1025), (5, 4096), (2, 8200), (1030, 100), (1500, 1001), (2100, 2048), (1, 16384), (700, 9001)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_norm_backward(b, rows, d, dtype):
    g = gen(rows + 31 * d)
    h, dy, ds = (torch.randn((rows, d), generator=g).to(dtype) for _ in range(3))
    w = (1 + 0.3 * torch.randn(d, generator=g)).to(torch.bfloat16 if d % 2 else torch.float32)
    if rows > 1:
        h[0] = 0
    pad = 0 if rows % 2 else 5
    for stream in (True, False):
        dh = rows_of(torch.zeros((rows, d), dtype=dtype, device=DEV), pad)
        dw = torch.full((d,), 3.0, device=DEV)
        sd = ds.to(DEV) if stream else None
        b.elmo_rms_norm_backward(rows_of(dy.to(DEV), pad, 1), rows_of(h.to(DEV), pad), dh, w.to(DEV), 1e-4, dsum=sd, dweight=dw)
        want, wantw = o.rms_norm_backward(f64(dy), f64(h), f64(w), 1e-4, f64(ds) if stream else None)
        if rows == 0:
            assert not dw.any()
            continue
        H, G = f64(h), f64(dy) * f64(w)
        R = 1 / np.sqrt(np.mean(H * H, axis=1, keepdims=True) + 1e-4)
        lane = 64 + 24                                       # terms of a lane, tree, waves
        along = np.sum(np.abs(G * H), axis=1, keepdims=True) / d
        tol = E * ((lane / 2 + 8) * np.abs(G * R) + np.abs(H) * R ** 3 * along * (2.5 * lane + 12)) + (HALF[dtype] + 2 * E) * np.abs(want) + 2 * E * (
            np.abs(f64(ds)) if stream else 0) + 1e-38
        close(dh, want, tol, "dh")
        adds = rows / min(rows, 1024) + 1024 / 16 + 16 + 2   # rows of a team, shares of a wave, waves
        close(dw, wantw, E * (adds + lane / 2 + 8) * np.sum(np.abs(f64(dy) * H * R), axis=0) + 1e-38, "dweight")
        assert between_rows(dh) is None or bool((between_rows(dh).float() == 72).all())
    if rows:
        again, dwa = dy.to(DEV), torch.empty_like(dw)        # the gradient over dy, the same bits
        b.elmo_rms_norm_backward(again, h.to(DEV), again, w.to(DEV), 1e-4, dweight=dwa)
        assert torch.equal(again, dh.contiguous()) and torch.equal(dwa, dw)


# ------------------------------------------------------------------ integer product
INT8_SHAPES = [(1, 1, 1), (1, 1, 0), (1, 5, 3), (3, 64, 16), (1, 256, 4096), (1, 1000, 999), (2, 33, 130), (7, 515, 272), (16, 128, 64), (17, 300, 80), (33, 1027, 512),
               (64, 64, 64), (65, 129, 257), (128, 256, 128), (130, 250, 1040), (256, 256, 256), (300, 700, 640), (257, 513, 1000), (512, 768, 2048),
               (1000, 40, 48), (1, 40000, 32), (1, 16, 40000), (40, 24, 131071), (700, 900, 36)]


@pytest.mark.parametrize("M,N,K", INT8_SHAPES)
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
def test_int8_matmul(b, M, N, K, out):
    g = gen(M + 3 * N + 7 * K)
    a = torch.randint(-128, 128, (M, K), generator=g).to(torch.int8)
    w = torch.randint(-128, 128, (N, K), generator=g).to(torch.int8)
    if K:
        a[0], w[0] = -128, -128                              # the largest sum there is
    sa, sb, bias = torch.rand(M, generator=g) + 0.1, torch.rand(N, generator=g) * 1e-3, torch.randn(N, generator=g)
    sa[M // 2] = 0.0
    for pad, first, with_bias in ((0, 0, False), (5, 3, True), (16, 16, True)):
        y = rows_of(torch.zeros((M, N), dtype=out, device=DEV), pad, first)
        b.elmo_int8_matmul(rows_of(a.to(DEV), pad, first), sa.to(DEV), rows_of(w.to(DEV), pad, first), sb.to(DEV), y, bias=bias.to(DEV) if with_bias else None)
        want = o.int8_matmul(a.numpy(), sa.numpy(), w.numpy(), sb.numpy(), bias.numpy() if with_bias else None)
        plain = np.abs(want - (bias.numpy() if with_bias else 0))
        # sum to FP32, two products, the bias's addition
        close(y, want, 3.01 * E * plain + (HALF[out] + 1.01 * E) * np.abs(want) + 1e-38, f"out, pad {pad}")
        assert between_rows(y) is None or bool((between_rows(y).float() == 72).all())


@pytest.mark.parametrize("M,N", [(3, 40), (40, 70), (200, 300)])
def test_int8_sums_of_nothing(b, M, N):
    bias, y = torch.randn(N, generator=gen(1)).to(DEV), torch.full((M, N), 9.0, device=DEV)
    none = lambda r: torch.empty((r, 0), dtype=torch.int8, device=DEV)  # noqa: E731
    b.elmo_int8_matmul(none(M), torch.ones(M, device=DEV), none(N), torch.ones(N, device=DEV), y, bias=bias)
    assert torch.equal(y, bias.expand(M, N))


def test_int8_offsets_beyond_32_bits(b):
    """Rows of either operand and of the output more than 2^31 elements from the first one."""
    M, N, K = 70, 80, 256
    g = gen(4)
    a, w = (torch.randint(-128, 128, (n, K), generator=g).to(torch.int8) for n in (M, N))
    sa, sb = torch.rand(M, generator=g), torch.rand(N, generator=g)
    big = torch.empty(N * (1 << 26), dtype=torch.int8, device=DEV)              # 5 GiB
    wd = torch.as_strided(big, (N, K), (1 << 26, 1))
    ad = torch.as_strided(big, (M, K), (1 << 26, 1), 4096)
    yd = torch.as_strided(big.view(torch.float32), (M, N), (1 << 24, 1), 4096)
    wd.copy_(w.to(DEV))
    ad.copy_(a.to(DEV))
    want = o.int8_matmul(a.numpy(), sa.numpy(), w.numpy(), sb.numpy())
    b.elmo_int8_matmul(ad, sa.to(DEV), wd, sb.to(DEV), yd)
    close(yd, want, 4.1 * E * np.abs(want) + 1e-38, "out")


# ------------------------------------------------------------------ sampling
def check_tokens(z, u, token, prob, **kw):
    """Every token is the oracle's, or u falls within the weights' rounding of the border between the two: a weight is off by at most half a
    unit of 2^-F of the largest, a filter's border moves by as much."""
    Z, n, V = f64(z), z.shape[0], z.shape[1]
    unit = V * 2.0 ** -min(50, 62 - max(1, (V - 1).bit_length())) + 1e-13
    for r in range(n):
        get = {k: (float(v[r]) if k != "top_k" else int(v[r])) for k, v in kw.items() if v is not None}
        if "t" in get:
            get["t"] = float(np.float64(get["t"]))
        index, c, want, share = o.sample_row(Z[r], float(u[r]), **get)
        got = int(token[r])
        if got != want:
            assert want >= 0 and got in index, (r, got, want, get)
            j = int(np.flatnonzero(index == got)[0])
            at = min(max(float(u[r]), 0.0), 1.0) * c[-1]
            lo = c[j - 1] if j else 0.0
            assert lo - unit <= at <= c[j] + unit, (r, got, want, get)
        else:
            assert abs(float(prob[r]) - share) <= 2 * E * share + unit, (r, float(prob[r]), share)


SAMPLE_SHAPES = [(1, 1), (2, 2), (3, 5), (4, 63), (5, 1000), (3, 1024), (9, 4097), (2, 32000), (3, 50257), (2, 65536), (2, 65537), (3, 131072), (1, 131080),
                 (2, 200003), (300, 700)]
SETTINGS = [dict(), dict(top_k=1), dict(top_k=5), dict(top_k=50, top_p=0.9), dict(top_k=700), dict(top_p=0.5), dict(top_p=0.95), dict(min_p=0.1),
            dict(top_p=0.999, min_p=0.01), dict(top_k=300, min_p=0.02, t=0.5), dict(t=1.7), dict(t=0.0), dict(top_p=0.9, t=3.0)]


@pytest.mark.parametrize("rows,V", SAMPLE_SHAPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_sample(b, rows, V, dtype):
    g = gen(rows + V)
    z = (2.5 * torch.randn((rows, V), generator=g)).to(dtype)
    n = len(SETTINGS)
    for k, kw in enumerate(SETTINGS):
        u = torch.rand(rows, generator=g)
        if k % 4 == 1:
            z[:, ::2] = -float("inf")                        # masked, the last token too where V is odd
        if k % 4 == 3:
            z = (2.5 * torch.randn((rows, V), generator=g)).to(dtype)
        s = {name: torch.full((rows,), v, dtype=torch.int32 if name == "top_k" else torch.float32) for name, v in kw.items()}
        token, prob = torch.full((rows,), -7, dtype=torch.int32, device=DEV), torch.full((rows,), -7.0, device=DEV)
        pad, first = ((0, 0), (3, 1), (8, 8))[k % 3]
        on = {("temperature" if name == "t" else name): v.to(DEV) for name, v in s.items()}
        b.elmo_sample(rows_of(z.to(DEV), pad, first), u.to(DEV), token, prob_out=prob, **on)
        check_tokens(z, u, token.cpu(), prob.cpu(), **s)
    assert n == 13


def test_sample_settings_of_each_row(b):
    rows, V = 64, 20000
    g = gen(11)
    z, u = 3 * torch.randn((rows, V), generator=g), torch.rand(rows, generator=g)
    s = dict(t=torch.rand(rows, generator=g) * 2, top_k=torch.randint(-1, 400, (rows,), generator=g, dtype=torch.int32), top_p=torch.rand(rows, generator=g) * 1.2,
             min_p=torch.rand(rows, generator=g) * 0.2 - 0.05)
    s["t"][:4] = torch.tensor([0.0, -1.0, float("nan"), float("inf")])
    s["top_p"][4:7] = torch.tensor([float("nan"), -0.5, 0.0])
    s["min_p"][7:9] = torch.tensor([float("nan"), 2.0])
    s["top_k"][9:12] = torch.tensor([0, V, 2 ** 31 - 1], dtype=torch.int32)
    token, prob = torch.empty(rows, dtype=torch.int32, device=DEV), torch.empty(rows, device=DEV)
    b.elmo_sample(z.to(DEV), u.to(DEV), token, temperature=s["t"].to(DEV), top_k=s["top_k"].to(DEV), top_p=s["top_p"].to(DEV), min_p=s["min_p"].to(DEV), prob_out=prob)
    want = {k: v.clone() for k, v in s.items()}
    want["t"][3] = 1e30                                      # a temperature of infinity: all alike
    want["top_p"][4] = 1.0
    want["min_p"][7] = 0.0
    check_tokens(z, u, token.cpu(), prob.cpu(), **want)


def test_sample_ties_masks_and_odd_logits(b):
    inf, nan = float("inf"), float("nan")
    z = torch.tensor([[1.0, 1.0, 1.0, 1.0], [-inf, -inf, -inf, -inf], [nan, nan, nan, nan], [nan, 0.0, -inf, 0.0], [inf, 0.0, inf, 5.0],
                      [-3.3e38, -3.3e38, -3.3e38, -3.3e38], [-0.0, 0.0, -0.0, 0.0], [-inf, -1e30, -inf, -inf]])
    n = z.shape[0]
    for dtype in (torch.float32, torch.bfloat16):
        for u, kw, want in ((0.0, {}, [0, -1, -1, 1, 0, 0, 0, 1]), (0.99, {}, [3, -1, -1, 3, 2, 3, 3, 1]), (0.6, {}, [2, -1, -1, 3, 2, 2, 2, 1]),
                            (0.99, dict(top_k=2), [1, -1, -1, 3, 2, 1, 1, 1]), (0.99, dict(top_k=3), [2, -1, -1, 3, 2, 2, 2, 1]),
                            (0.99, dict(top_p=0.5), [1, -1, -1, 1, 0, 1, 1, 1]), (0.99, dict(top_p=0.51), [2, -1, -1, 3, 2, 2, 2, 1]),
                            (0.99, dict(temperature=0.0), [0, -1, -1, 1, 0, 0, 0, 1]), (0.99, dict(min_p=1.0), [3, -1, -1, 3, 2, 3, 3, 1]),
                            (1.5, {}, [3, -1, -1, 3, 2, 3, 3, 1]), (nan, {}, [0, -1, -1, 1, 0, 0, 0, 1]), (-1.0, {}, [0, -1, -1, 1, 0, 0, 0, 1])):
            token, prob = torch.full((n,), -7, dtype=torch.int32, device=DEV), torch.full((n,), -7.0, device=DEV)
            on = {k: torch.full((n,), v, dtype=torch.int32 if k == "top_k" else torch.float32, device=DEV) for k, v in kw.items()}
            b.elmo_sample(z.to(dtype).to(DEV), torch.full((n,), u, device=DEV), token, prob_out=prob, **on)
            assert token.tolist() == want, (dtype, u, kw)
            assert prob[1:3].tolist() == [0.0, 0.0] and bool((prob[3:] > 0).all())


@pytest.mark.parametrize("V", [3000, 131072])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_sample_rows_of_few_values(b, V, dtype):
    """Thousands of equal logits: the border of a filter lies inside a tie, and inside a tile."""
    g = gen(V)
    z = torch.randint(0, 3, (8, V), generator=g).to(dtype)
    z[0] = 1.0
    u = torch.rand(8, generator=g)
    for kw in (dict(), dict(top_k=V // 2 + 1), dict(top_p=0.7), dict(top_k=V // 3, top_p=0.5), dict(min_p=0.2), dict(top_k=1000)):
        token, prob = torch.full((8,), -7, dtype=torch.int32, device=DEV), torch.empty(8, device=DEV)
        s = {k: torch.full((8,), v, dtype=torch.int32 if k == "top_k" else torch.float32) for k, v in kw.items()}
        b.elmo_sample(z.to(DEV), u.to(DEV), token, prob_out=prob, **{k: v.to(DEV) for k, v in s.items()})
        check_tokens(z, u, token.cpu(), prob.cpu(), **s)


@pytest.mark.parametrize("rows,V", [(130, 20011), (3, 16384), (129, 16391), (9, 65543)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_sample_without_top_k_in_one_workgroup_and_in_several(b, rows, V, dtype):
    """Rows on both sides of the number from which a row is no longer split; among them empty ones, ones of infinities, of zeros, of one
    value, of values next to zero, far from zero and spread over the whole type."""
    g = gen(V)
    z = (2.5 * torch.randn((rows, V), generator=g)).to(dtype)
    z[0, V // 2:] = -float("inf")
    z[1, 7], z[1, V - 1] = float("inf"), float("inf")
    z[2] = torch.where(torch.rand(V, generator=g) < 0.3, 0.0, z[2].float()).to(dtype)
    if rows > 8:
        z[3] = -float("inf")
        z[4] = -3.0
        z[5] = (1e-6 * torch.randn(V, generator=g)).to(dtype)
        z[6] = (1000 + 8 * torch.randn(V, generator=g)).to(dtype)
        z[7] = (1e37 * torch.randn(V, generator=g)).to(dtype)
        z[8] = -z[2].abs()
    for kw in (dict(), dict(top_p=0.9), dict(top_p=0.3, t=0.7), dict(min_p=0.05), dict(top_p=0.97, min_p=0.01, t=1.5), dict(t=0.0), dict(top_p=0.5, t=1e30),
               dict(top_p=0.8, t=1e-3)):
        u = torch.rand(rows, generator=g)
        s = {name: torch.full((rows,), v) for name, v in kw.items()}
        token, prob = torch.full((rows,), -7, dtype=torch.int32, device=DEV), torch.full((rows,), -7.0, device=DEV)
        on = {("temperature" if name == "t" else name): v.to(DEV) for name, v in s.items()}
        b.elmo_sample(rows_of(z.to(DEV), 3, 1), u.to(DEV), token, prob_out=prob, **on)
        check_tokens(z, u, token.cpu(), prob.cpu(), **s)
        if "t" not in kw:                                    # the same by one workgroup a row: top-k that keeps everything
            again, prob2 = torch.empty_like(token), torch.empty_like(prob)
            b.elmo_sample(z.to(DEV), u.to(DEV), again, prob_out=prob2, top_k=torch.full((rows,), V, dtype=torch.int32, device=DEV), **on)
            assert torch.equal(again, token) and torch.equal(prob2, prob)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_sample_long_top_k(b, dtype):
    """More tokens than the short list takes, with and without top-p behind them."""
    g = gen(77)
    rows, V = 20, 30001
    z = (2 * torch.randn((rows, V), generator=g)).to(dtype)
    z[1] = z[1].round()
    for k, p in ((513, 1.0), (5000, 0.9), (29999, 0.99), (513, 0.2)):
        u = torch.rand(rows, generator=g)
        s = dict(top_k=torch.full((rows,), k, dtype=torch.int32), top_p=torch.full((rows,), p))
        token, prob = torch.empty(rows, dtype=torch.int32, device=DEV), torch.empty(rows, device=DEV)
        b.elmo_sample(z.to(DEV), u.to(DEV), token, prob_out=prob, **{n: v.to(DEV) for n, v in s.items()})
        check_tokens(z, u, token.cpu(), prob.cpu(), **s)


def test_sample_shares_of_many_draws(b):
    V, n = 40, 20000
    z = torch.randn(V, generator=gen(3))
    u = torch.rand(n, generator=gen(4))
    token = torch.empty(n, dtype=torch.int32, device=DEV)
    b.elmo_sample(z[None, :].repeat(n, 1).to(DEV), u.to(DEV), token, top_k=torch.full((n,), 20, dtype=torch.int32, device=DEV))
    p = np.exp(f64(z))
    p[np.argsort(-p, kind="stable")[20:]] = 0
    p /= p.sum()
    got = np.bincount(token.cpu().numpy(), minlength=V) / n
    assert np.all(np.abs(got - p) <= 5 * np.sqrt(p * (1 - p) / n))


# ------------------------------------------------------------------ distillation
def distill_tolerance(z, idx, tz, T, v, dtype, want):
    """The student's sum: v_exp_f32, its argument's rounding (c = log2(e) / T and the product, each e of |z - m| c), the lanes' sums."""
    Z, V = f64(z) / T, z.shape[1]
    fin = np.where(np.isfinite(Z), Z, -np.inf)
    top = fin.max(axis=1, keepdims=True)
    top = np.where(np.isfinite(top), top, 0.0)
    p = np.exp(fin - top)
    S = p.sum(axis=1, keepdims=True)
    p = np.where(S > 0, p / np.where(S > 0, S, 1.0), 0.0)
    x = np.where(np.isfinite(fin), np.abs(fin - top), 0.0) * 1.4427
    terms = min(V, 8 * (-(-V // (8 * 64)))) + 24             # the longest chain of additions: one wave's lane over the whole row, and the trees
    dS = (E * (terms + 4) + E * 2 * np.sum(p * x, axis=1, keepdims=True))
    vv = np.ones((z.shape[0], 1)) if v is None else f64(v)[:, None]
    loss, grad = want
    ok = (idx.numpy() >= 0) & (idx.numpy() < V)
    at = np.where(ok, idx.numpy(), 0)
    far = np.max(np.where(ok, np.abs(np.take_along_axis(np.where(np.isfinite(Z), Z, 0), at, 1) - top), 0), axis=1) + np.log(np.maximum(S[:, 0], 1e-300))
    tl = np.abs(vv[:, 0]) * T * T * (dS[:, 0] + 4 * E * (far + 1)) + 3 * E * np.abs(loss) + 1e-38
    tg = np.abs(vv) * T * (p * (dS + E * (6 + 2 * x)) + 4 * E * np.abs(grad / np.where(vv == 0, 1, vv) / T - p)) + (HALF[dtype] + E) * np.abs(grad) + 1e-38
    return tl, tg


DISTILL_SHAPES = [(1, 1, 1), (2, 3, 2), (3, 9, 20), (4, 1000, 1), (5, 1003, 16), (2, 8192, 64), (3, 32003, 100), (2, 65536, 7), (2, 65537, 1024), (1, 131072, 64), (2, 131081, 33),
                  (1, 300007, 50), (600, 260, 8), (300, 3001, 8)]


@pytest.mark.parametrize("rows,V,K", DISTILL_SHAPES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_distill(b, rows, V, K, dtype):
    g = gen(rows + V + K)
    z = (2.5 * torch.randn((rows, V), generator=g)).to(dtype)
    idx = torch.randint(0, V, (rows, K), generator=g, dtype=torch.int32)       # with repetitions where K is not far below V
    if K > 3:
        idx[:, 1] = idx[:, 0]                                # the same index twice
        idx[0, 2], idx[rows - 1, 3] = -1, V                  # entries that do not count
        idx[0, K - 1] = V - 1
    if rows > 2:
        idx[1] = -1                                          # a row without a teacher
    tz = 2 * torch.randn((rows, K), generator=g)
    v = torch.rand(rows, generator=g)
    if rows > 2:
        v[2] = 0.0
        z[2, 0] = float("nan")                               # a row of weight 0 is not read
    for T, tt, vv, pad in ((1.0, torch.float32, None if rows <= 2 else v, 0), (2.5, torch.bfloat16, v, 3)):
        t = tz.to(tt)
        zd = rows_of(z.to(DEV), pad, pad)
        loss, grad = torch.full((rows,), -7.0, device=DEV), rows_of(torch.full((rows, V), -7.0, dtype=dtype, device=DEV), pad)
        args = dict(temperature=T, row_weight=None if vv is None else vv.to(DEV))
        b.elmo_distill(zd, idx.to(DEV), t.to(DEV), loss, grad, **args)
        zo = z.clone()
        if rows > 2:
            zo[2, 0] = 0.0
        want = o.distill(f64(zo), idx.numpy(), f64(t), T, None if vv is None else f64(vv))
        tl, tg = distill_tolerance(zo, idx, t, T, vv, dtype, want)
        close(loss, want[0], tl, "loss")
        close(grad, want[1], tg, "gradient")
        assert between_rows(grad) is None or bool((between_rows(grad).float() == 72).all())
        alone = torch.empty(rows, device=DEV)
        b.elmo_distill(zd, idx.to(DEV), t.to(DEV), alone, **args)
        assert torch.equal(alone, loss), "the loss alone is the same number"
        b.elmo_distill(zd, idx.to(DEV), t.to(DEV), alone, zd, **args)
        assert torch.equal(zd, grad) and torch.equal(alone, loss), "the gradient may be written over the logits"


def test_distill_masked_logits_and_odd_teachers(b):
    inf, nan = float("inf"), float("nan")
    V = 2100
    z = torch.randn((8, V), generator=gen(9))
    z[0, 1000:] = -inf                                       # masked vocabulary, the teacher's tokens are not
    z[1, 5] = -inf                                           # a teacher's token is masked: infinite loss, finite gradient
    z[2] = -inf
    z[3, 7], z[4, 7] = nan, inf
    idx = torch.tensor([[0, 5, 10]], dtype=torch.int32).repeat(8, 1)
    tz = torch.zeros((8, 3))
    tz[5] = -inf                                             # no teacher at all
    tz[6, 1] = -inf                                          # an entry without weight
    tz[7, 1] = nan
    loss, grad = torch.empty(8, device=DEV), torch.empty((8, V), device=DEV)
    b.elmo_distill(z.to(DEV), idx.to(DEV), tz.to(DEV), loss, grad)
    keep = [0, 6]
    want = o.distill(f64(z[keep]), idx[keep].numpy(), f64(tz[keep]), 1.0)
    tl, tg = distill_tolerance(z[keep], idx[keep], tz[keep], 1.0, None, torch.float32, want)
    close(loss[keep], want[0], tl, "loss")
    close(grad[keep], want[1], tg, "gradient")
    assert not grad[0, 1000:].any()
    assert loss[1] == inf and bool(torch.isfinite(grad[1]).all()) and abs(float(grad[1, 5]) + 1 / 3) <= 3 * E
    assert loss[2] == inf and abs(float(grad[2].sum()) + 1) <= 8 * E and int((grad[2] != 0).sum()) == 3
    for r in (3, 4, 7):
        assert bool(torch.isnan(loss[r])) and bool(torch.isnan(grad[r]).any())
    assert loss[5] == 0 and not grad[5].any()


@pytest.mark.parametrize("T", [0.5, 1.0, 2.0])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_distill_rows_masked_with_the_types_lowest_value(b, T, dtype):
    """The lowest value as a mask: beside other logits p = 0, in a row of nothing else all tokens alike."""
    low, V = torch.finfo(dtype).min, 1003
    z = torch.randn((3, V), generator=gen(6)).to(dtype)
    z[0, ::2], z[1], z[2] = low, low, -low
    idx, tz = torch.tensor([[1, 3], [0, 7], [0, 7]], dtype=torch.int32), torch.tensor([[0.5, 0.0]] * 3)
    loss, grad = torch.empty(3, device=DEV), torch.empty((3, V), dtype=dtype, device=DEV)
    b.elmo_distill(z.to(DEV), idx.to(DEV), tz.to(DEV), loss, grad, temperature=T)
    want = o.distill(f64(z), idx.numpy(), f64(tz), T)
    tl, tg = distill_tolerance(z, idx, tz, T, None, dtype, want)
    close(loss, want[0], tl, "loss")
    close(grad, want[1], tg, "gradient")
    assert not grad[0, ::2].any()


@pytest.mark.parametrize("rows,V", [(3, 40), (2, 3000)])
def test_distill_gradient_is_that_of_its_loss(b, rows, V):
    """Central differences of the FP32 loss along random directions."""
    g = gen(V)
    z, idx, tz = torch.randn((rows, V), generator=g), torch.randint(0, V, (rows, 12), generator=g, dtype=torch.int32), torch.randn((rows, 12), generator=g)
    grad, loss = torch.empty((rows, V), device=DEV), torch.empty(rows, device=DEV)
    b.elmo_distill(z.to(DEV), idx.to(DEV), tz.to(DEV), loss, grad, temperature=1.5)
    for _ in range(3):
        way = torch.randn((rows, V), generator=g)
        way /= way.norm(dim=1, keepdim=True)
        step, at = 2.0 ** -4, []
        for sign in (1, -1):
            out = torch.empty(rows, device=DEV)
            b.elmo_distill((z + sign * step * way).to(DEV), idx.to(DEV), tz.to(DEV), out, temperature=1.5)
            at.append(f64(out))
        slope = (at[0] - at[1]) / (2 * step)
        # third derivative of log sum exp along a unit way is below 2 / T^3 (times T^2): step^2 / 6 of it; the losses' rounding over the step
        tol = 2 / 1.5 * step ** 2 / 6 + 60 * E * (np.abs(at[0]) + 10) / step
        assert np.all(np.abs(slope - np.sum(f64(grad) * f64(way), axis=1)) <= tol)


# ------------------------------------------------------------------ together, streams, graphs
def _chain(b, st, stream=None):
    b.elmo_rms_norm(st["x"], st["q"], st["w"], 1e-6, residual=st["r"], sum_out=st["h"], scale_out=st["s"], stream=stream)
    b.elmo_int8_matmul(st["q"], st["s"], st["W"], st["ws"], st["z"], stream=stream)
    b.elmo_sample(st["z"], st["u"], st["token"], temperature=st["t"], top_k=st["k"], top_p=st["p"], prob_out=st["prob"], stream=stream)
    b.elmo_distill(st["z"], st["ti"], st["tz"], st["loss"], st["dz"], temperature=2.0, stream=stream)
    b.elmo_rms_norm_backward(st["dy"], st["h"], st["dx"], st["w"], 1e-6, dsum=st["r"], dweight=st["dw"], stream=stream)


def _chain_state(rows, d, V, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    rn = lambda *s: torch.randn(s, device=DEV, generator=g)  # noqa: E731
    z = lambda s, t=torch.float32: torch.zeros(s, dtype=t, device=DEV)  # noqa: E731
    bf = torch.bfloat16
    return dict(x=rn(rows, d).to(bf), r=rn(rows, d).to(bf), w=(1 + 0.1 * rn(d)).to(bf), q=z((rows, d), torch.int8), h=z((rows, d), bf), s=z(rows),
                W=(rn(V, d) * 40).round().clamp(-127, 127).to(torch.int8), ws=0.003 + z(V), z=z((rows, V), bf), u=torch.rand(rows, device=DEV, generator=g),
                token=z(rows, torch.int32), t=0.7 + z(rows), k=40 + z(rows, torch.int32), p=0.9 + z(rows), prob=z(rows),
                ti=torch.randint(0, V, (rows, 8), device=DEV, generator=g, dtype=torch.int32), tz=rn(rows, 8), loss=z(rows), dz=z((rows, V), bf),
                dy=rn(rows, d).to(bf), dx=z((rows, d), bf), dw=z(d))


OUTPUTS = ("q", "h", "s", "z", "token", "prob", "loss", "dz", "dx", "dw")


@pytest.mark.parametrize("rows,d,V", [(1, 256, 4096), (6, 768, 8192), (70, 512, 5003)])
def test_the_operators_one_after_another(b, rows, d, V):
    """Norm -> 8-bit rows -> logits -> token, and the logits' distillation: every stage against the oracle on what the stage before gave."""
    st = _chain_state(rows, d, V, 5)
    _chain(b, st)
    y, h, _ = o.rms_norm(f64(st["x"]), f64(st["w"]), 1e-6, f64(st["r"]))
    back = f64(st["q"]) * f64(st["s"])[:, None]
    most = np.max(np.abs(back), axis=1, keepdims=True)
    assert np.all(np.abs(back - y) <= most / 127 * 0.5 + 100 * E * most), "the 8-bit rows are the norm to half a step"
    want = o.int8_matmul(st["q"].cpu().numpy(), f64(st["s"]), st["W"].cpu().numpy(), f64(st["ws"]))
    close(st["z"], want, (2.0 ** -8 + 5 * E) * np.abs(want) + 1e-38, "logits")
    check_tokens(st["z"].cpu(), st["u"].cpu(), st["token"].cpu(), st["prob"].cpu(), t=st["t"].cpu(), top_k=st["k"].cpu(), top_p=st["p"].cpu())
    ref = o.distill(f64(st["z"]), st["ti"].cpu().numpy(), f64(st["tz"]), 2.0)
    tl, tg = distill_tolerance(st["z"].cpu(), st["ti"].cpu(), st["tz"].cpu(), 2.0, None, torch.bfloat16, ref)
    close(st["loss"], ref[0], tl, "loss")
    close(st["dz"], ref[1], tg, "gradient")


@pytest.mark.parametrize("rows,d,V", [(1, 768, 8192), (40, 512, 70001)])
def test_captured_and_replayed_on_another_stream(b, rows, d, V):
    """A captured run of all operators replays to the eager run's bits, on new inputs and with eager work between the replays."""
    st, side = _chain_state(rows, d, V, 1), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _chain(b, st)                                        # kernels loaded before the capture
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        _chain(b, st)
    for seed in (2, 3, 4):
        new = _chain_state(rows, d, V, seed)
        for k in st:
            st[k].copy_(new[k])
        graph.replay()
        torch.cuda.synchronize()
        _chain(b, new)                                       # eager, between the replays
        torch.cuda.synchronize()
        for k in OUTPUTS:
            assert torch.equal(st[k], new[k]), (seed, k)


def test_two_streams_at_once(b):
    """Two runs that overlap in time do not share anything: each gives what it gives alone."""
    states = [_chain_state(48, 512, 60000, s) for s in (1, 2)]
    alone = []
    for st in states:
        _chain(b, st)
        torch.cuda.synchronize()
        alone.append({k: st[k].clone() for k in OUTPUTS})
        for k in OUTPUTS:
            st[k].zero_()
    streams = [torch.cuda.Stream() for _ in states]
    torch.cuda.synchronize()
    for _ in range(3):
        for st, s in zip(states, streams):
            _chain(b, st, stream=s)
    torch.cuda.synchronize()
    for st, want in zip(states, alone):
        for k in OUTPUTS:
            assert torch.equal(st[k], want[k]), k


def test_norm_feeds_the_head(b):
    """BF16 rows of the norm are a head's inputs: top-k of a head over them finds the label whose weights point along a row."""
    rows, d, L = 12, 256, 3000
    g = gen(8)
    x = torch.randn((rows, d), generator=g).to(torch.bfloat16).to(DEV)
    y = torch.empty_like(x)
    b.elmo_rms_norm(x, y, None, 1e-6)
    head = b.Head(L, d, b.ELMO_BF16, 1024, 0, rows, 64)
    W = 0.01 * torch.randn((L, d), generator=g).to(DEV)
    W[torch.arange(rows) * 17] = y.float() / 16
    head.weights().copy_(W.to(torch.bfloat16).view(torch.int16))
    idx, score = torch.empty((rows, 3), dtype=torch.int32, device=DEV), torch.empty((rows, 3), device=DEV)
    head.topk(y, 3, idx, score)
    assert idx[:, 0].tolist() == [17 * r for r in range(rows)]
    head.close()
