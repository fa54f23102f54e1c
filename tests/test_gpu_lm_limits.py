"""The output-end operators where their numbers, sizes or workspaces are at an end of what the header allows, against the 64-bit statements.

Tolerances in the units of test_gpu_lm.py: E = 2^-24 (half a step of FP32, relative), HALF = half a step of the output type.
"""
import numpy as np
import pytest
import torch

from oracle import lm_oracle as o

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
E = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: E}


@pytest.fixture(scope="module")
def b():
    from paper_2510_11168_amd import binding
    return binding


def f64(t):
    return t.to(torch.float64).cpu().numpy()


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def close(got, want, tol, what):
    assert np.all(np.isfinite(f64(got))), what
    err = np.abs(f64(got) - want)
    assert np.all(err <= tol), f"{what}: {float(np.max(err / tol)):.3g} times the tolerance"


# ------------------------------------------------------------------ norm
@pytest.mark.parametrize("rms,eps", [(1e-36, 0.0), (1e-25, 0.0), (1e-20, 1e-38), (1e-8, 1e-16), (1e16, 1e-6), (1e18, 1e-6), (1e30, 1e-6), (4e37, 0.0)])
@pytest.mark.parametrize("rows,d", [(3, 8), (5, 1001), (3, 2048), (2, 9000)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_norm_of_rows_whose_squares_leave_fp32(b, rows, d, dtype, rms, eps):
    g = gen(d + 1)
    x, r = (rms * torch.randn((rows, d), generator=g)).to(dtype), (rms * torch.randn((rows, d), generator=g)).to(dtype)
    x[0], r[0] = torch.sign(x[0].float()).to(dtype), 0       # an ordinary row beside them
    w = (1 + 0.1 * torch.randn(d, generator=g)).to(dtype)
    h32 = x.float() + r.float()
    assert bool(torch.isfinite(h32).all())
    want, h64, root = o.rms_norm(f64(x), f64(w), float(np.float32(eps)), f64(r))
    # as in back_tolerances: half of a sum of n = 88 additions on the way, a root, a quotient and two products
    rel = (88 / 2 + 11) * E
    args = x.to(DEV), r.to(DEV), w.to(DEV)
    for out in (torch.bfloat16, torch.float32):
        y, s = torch.empty((rows, d), dtype=out, device=DEV), torch.empty((rows, d), dtype=dtype, device=DEV)
        b.elmo_rms_norm(args[0], y, args[2], eps, residual=args[1], sum_out=s)
        # the sum's own rounding to FP32 is E of it
        close(y, want, (HALF[out] + rel) * np.abs(want) + 3 * E * np.abs(f64(w) * h64 / root) + 1e-38, "y")
        assert torch.equal(s.cpu(), h32.to(dtype)), "the stream is the rounded sum"
    q, scale = torch.empty((rows, d), dtype=torch.int8, device=DEV), torch.empty(rows, device=DEV)
    b.elmo_rms_norm(args[0], q, args[2], eps, residual=args[1], scale_out=scale)
    quotients, m = o.rows_in_8_bits(h32.numpy(), f64(w), 127)
    finite = f64(h32 * h32).sum(axis=1) < 3.4e38
    assert np.array_equal(q.cpu().numpy(), np.where(finite[:, None], np.rint(quotients), 0).astype(np.int8))
    assert not np.isfinite(f64(scale)[~finite]).any()
    close(scale[torch.from_numpy(finite)], (m / (127 * root))[finite, 0], (rel + 2 * E) * (m / (127 * root))[finite, 0], "scale")


def back_tolerances(dy, h, w, eps, dtype, want):
    """A lane adds at most 64 terms, the tree and the waves 24 levels: n = 88 additions on the way of a term.  R has half the relative error of the
    sum of squares, all of its terms positive, (n / 2) e, and 8 e of its own; h R^3 mean(g h) has R three times, the sum of g h (n e of the sum of
    magnitudes) and 12 e of products.  A weight gradient adds rows / 512 terms of a team, 3 teams, 8 shares and 6 levels at most."""
    H, G, n = f64(h), f64(dy) * f64(w), 88
    R = 1 / np.sqrt(np.mean(H * H, axis=1, keepdims=True) + eps)
    along = np.mean(np.abs(G * H), axis=1, keepdims=True)
    th = E * ((n / 2 + 8) * np.abs(G * R) + np.abs(H) * R ** 3 * along * (2.5 * n + 12)) + (HALF[dtype] + E) * np.abs(want) + 1e-38
    tw = E * (n / 2 + 8 + len(H) / 512 + 17) * np.sum(np.abs(f64(dy) * H * R), axis=0) + 1e-38
    return th, tw


@pytest.mark.parametrize("rms,eps", [(1e-15, 0.0), (1e-13, 1e-30), (1e14, 1e-6), (1e16, 1e-6), (1e18, 1e-6), (1e30, 1e-6), (1e37, 0.0), (1e-25, 0.0), (1e-36, 0.0)])
@pytest.mark.parametrize("rows,d", [(5, 1001), (3, 2048), (2, 9000)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_norm_backward_of_large_and_small_rows(b, rows, d, dtype, rms, eps):
    """A gradient that goes mostly along h: what the projection takes away is of its size."""
    g = gen(d)
    h = (rms * torch.randn((rows, d), generator=g)).to(dtype)
    dy = (h.float() / rms + 0.1 * torch.randn((rows, d), generator=g)).to(dtype)
    w = (1 + 0.1 * torch.randn(d, generator=g)).to(dtype)
    dh, dw = torch.empty((rows, d), dtype=dtype, device=DEV), torch.empty(d, device=DEV)
    b.elmo_rms_norm_backward(dy.to(DEV), h.to(DEV), dh, w.to(DEV), eps, dweight=dw)
    want, wantw = o.rms_norm_backward(f64(dy), f64(h), f64(w), eps)
    th, tw = back_tolerances(dy, h, w, eps, dtype, want)
    close(dh, want, th, "dh")
    close(dw, wantw, tw, "dweight")


@pytest.mark.parametrize("rows,d", [(2500, 300), (1300, 2048), (1100, 9000)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_norm_backward_of_rows_of_all_sizes_by_one_team(b, rows, d, dtype):
    """A team that takes several rows one after another, ordinary ones and ones that are summed twice."""
    g = gen(rows)
    size = torch.tensor([1e18, 1.0, 1e-25, 3.0, 1.0, 1e30, 1e-25])[torch.randint(0, 7, (rows,), generator=g)][:, None]
    h = (size * torch.randn((rows, d), generator=g)).to(dtype)
    dy = (h.float() / size + 0.1 * torch.randn((rows, d), generator=g)).to(dtype)
    dh, dw, again = torch.empty((rows, d), dtype=dtype, device=DEV), torch.empty(d, device=DEV), torch.empty(d, device=DEV)
    args = dy.to(DEV), h.to(DEV), dh, None, 0.0
    b.elmo_rms_norm_backward(*args, dweight=dw)
    want, wantw = o.rms_norm_backward(f64(dy), f64(h), np.ones(d), 0.0)
    th, tw = back_tolerances(dy, h, torch.ones(d), 0.0, dtype, want)
    close(dh, want, th, "dh")
    close(dw, wantw, tw, "dweight")
    b.elmo_rms_norm_backward(*args, dweight=again)
    assert torch.equal(again, dw)


def test_norm_backward_of_zeros_and_a_very_small_eps(b):
    h, dy = torch.zeros((2, 300), device=DEV), torch.randn((2, 300), generator=gen(1)).to(DEV)
    dh, dw = torch.empty_like(h), torch.empty(300, device=DEV)
    b.elmo_rms_norm_backward(dy, h, dh, None, 1e-28, dweight=dw)
    want = f64(dy) / np.sqrt(np.float64(np.float32(1e-28)))
    close(dh, want, 4 * E * np.abs(want), "dh")
    assert not dw.any()


# ------------------------------------------------------------------ integer product
def rows_of(t, pad, first=0):
    """The same values as rows of a wider buffer that begins `first` elements behind an aligned address; what is between rows is 72."""
    n, d = t.shape
    wide = torch.full((first + n * (d + pad),), 72, dtype=t.dtype, device=t.device)
    v = wide[first:].view(n, d + pad)[:, :d]
    v.copy_(t)
    return v


@pytest.mark.parametrize("tile,M,N,K", [(64, 300, 700, 200), (128, 1500, 1531, 272), (128, 2050, 2060, 130), (128, 1500, 1531, 100), (256, 3001, 3333, 200), (256, 4090, 4090, 130),
                                        (256, 3001, 3333, 100), (256, 3071, 3329, 512)])
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
def test_int8_matmul_in_each_tile(b, tile, M, N, K, out):
    """Ragged rows, columns and K, operands whose rows are 16-byte aligned and not, with and without a bias, in the tile that the rule picks."""
    assert b.elmo_int8_matmul_tile(M, N, K) == tile
    g = gen(M + K)
    a, w = (torch.randint(-128, 128, (n, K), generator=g).to(torch.int8) for n in (M, N))
    a[0], w[0], a[M - 1], w[N - 1] = -128, -128, -128, 127       # the largest sums there are
    sa, sb, bias = torch.rand(M, generator=g) + 0.1, torch.rand(N, generator=g) * 1e-3, torch.randn(N, generator=g)
    plain = (f64(a) @ f64(w).T) * f64(sa)[:, None] * f64(sb)[None, :]     # (whole numbers below 2^53)
    up = -K % 16
    for pad, first, pad_out, with_bias in ((up, 0, 0, False), (up + 16, 16, 1, True), (5 if up != 5 else 7, 3, 3, True)):
        y = rows_of(torch.zeros((M, N), dtype=out, device=DEV), pad_out, first)
        ad, wd = rows_of(a.to(DEV), pad, first), rows_of(w.to(DEV), pad, first)
        assert (first == 3) == bool((ad.data_ptr() | ad.stride(0)) & 15)
        b.elmo_int8_matmul(ad, sa.to(DEV), wd, sb.to(DEV), y, bias=bias.to(DEV) if with_bias else None)
        want = plain + f64(bias) if with_bias else plain
        # sum to FP32, two products, the bias's addition
        close(y, want, 3.01 * E * np.abs(plain) + (HALF[out] + 1.01 * E) * np.abs(want) + 1e-38, f"out, pad {pad}")
        if pad_out:
            assert bool((torch.as_strided(y, (M - 1, pad_out), (N + pad_out, 1), y.storage_offset() + N) == 72).all()), "nothing between the rows is written"


def test_int8_matmul_of_more_outputs_than_the_streaming_kernel_takes(b):
    """2^27 weight rows and some: more than a launch of the kernel of few tokens has workgroups for, and operand offsets beyond 2^31."""
    M, N, K = 2, (1 << 27) + 5, 16
    assert b.elmo_int8_matmul_tile(M, N, 2048) == 64 and b.elmo_int8_matmul_tile(M, (1 << 27) - 16, 2048) == 0
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    a, w = torch.randint(-128, 128, (M, K), device=DEV, generator=g, dtype=torch.int8), torch.randint(-128, 128, (N, K), device=DEV, generator=g, dtype=torch.int8)
    sa, sb = torch.rand(M, device=DEV, generator=g), torch.rand(N, device=DEV, generator=g)
    y = torch.empty((M, N), device=DEV)
    b.elmo_int8_matmul(a, sa, w, sb, y)
    for at in range(0, N, 1 << 24):
        part = w[at:at + (1 << 24)].float()                      # (sums below 2^24: exact)
        for m in range(M):
            assert torch.equal(y[m, at:at + (1 << 24)], (part * a[m].float()).sum(1) * sa[m] * sb[at:at + (1 << 24)])


# ------------------------------------------------------------------ sampling
def draw(b, z, u, **kw):
    token, prob = torch.full((len(u),), -7, dtype=torch.int32, device=DEV), torch.full((len(u),), -7.0, device=DEV)
    b.elmo_sample(z.to(DEV), u.to(DEV), token, prob_out=prob, **{k: v.to(DEV) for k, v in kw.items()})
    return token.cpu(), prob.cpu()


@pytest.mark.parametrize("rows,V", [(3, 700), (3, 20011), (2, 131072), (140, 20000)])
@pytest.mark.parametrize("top_k", [0, 60, 400, 600])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_share_of_a_light_token(b, rows, V, top_k, dtype):
    """u = 0 draws the first kept token, however light: its share has FP32's bits also where a few units of 2^-F are all it weighs."""
    g = gen(V)
    F = min(50, 62 - (V - 1).bit_length())
    z = torch.full((rows, V), -float("inf"))
    live = min(V - 2, 300)                                   # constrained decoding: most tokens are masked
    for r in range(rows):
        z[r, 1 + torch.randperm(V - 1, generator=g)[:live]] = 4 * torch.rand(live, generator=g) - 4
        z[r, V - 1 - r % 3] = 0.0
        z[r, 0] = -[10.0, 24.0, 0.69 * (F - 2)][r % 3]       # the last: a weight of about four units
    z = z.to(dtype)
    if top_k == 60:                                          # a list that ends within the tokens: of few live ones
        z[:, 1:V - 3][torch.rand((rows, V - 4), generator=g) < 0.9] = -float("inf")
    kw = dict(top_k=torch.full((rows,), top_k, dtype=torch.int32)) if top_k else {}
    token, prob = draw(b, z, torch.zeros(rows), **kw)
    assert not token.any()
    w = np.exp(f64(z))                                       # (the largest logit is 0)
    share = w[:, 0] / w.sum(axis=1)
    # one rounding to FP32, the FP64 weight's 2^-51, half a unit of 2^-F for each of the sum's tokens
    close(prob, share, share * (E + 2.0 ** -50 + (live + 3) * 2.0 ** -(F + 1)), "share")


def test_borders_between_two_tokens(b):
    """Temperatures for which the border between two tokens lies 2^-50 to 2^-46 beside a number: the token on the number's side is drawn.  The weight of
    the lighter one is right to 2^-51 and half a unit of 2^-50, the border then to 2^-52, and u times the sum is rounded by 2^-53."""
    ts, us, zs, want = [], [], [], []
    for z in (-1.0, -2.0, -3.0):
        for start in (0x3E800000, 0x3F000000, 0x3F800000, 0x40000000):       # 1/4, 1/2, 1, 2
            t = np.arange(start, start + (1 << 23), dtype=np.uint32).view(np.float32)
            border = 1 / (1 + np.exp(z / t.astype(np.float64)))
            u = border.astype(np.float32)
            off = np.abs(border - u.astype(np.float64))
            at = np.flatnonzero((off > 2.0 ** -50.1) & (off < 2.0 ** -45.9))
            exact = 1 / (1 + np.exp(np.longdouble(z) / t[at].astype(np.longdouble)))
            for i, e in zip(at, exact):
                d = float(u[i].astype(np.longdouble) - e)
                if 2.0 ** -50 <= abs(d) <= 2.0 ** -46:
                    ts.append(float(t[i])), us.append(float(u[i])), zs.append(z), want.append(int(d >= 0))
    assert len(want) >= 20 and 0 < sum(want) < len(want)
    t, u = torch.tensor(ts), torch.tensor(us)
    for dtype in (torch.bfloat16, torch.float32):
        rows = torch.tensor([[0.0, z, -float("inf")] for z in zs]).to(dtype)
        for kw in ({}, dict(top_k=torch.full((len(ts),), 2, dtype=torch.int32))):
            for order in (rows, rows[:, [2, 0, 1]]):
                token, _ = draw(b, order, u, temperature=t, **kw)
                first = 0 if order is rows else 1
                wrong = np.flatnonzero(token.numpy() - first != np.array(want))
                assert not len(wrong), (dtype, list(kw), len(wrong), "of", len(want))


# ------------------------------------------------------------------ workspaces, graphs, streams
def split_state(seed):
    """Sampling without top-k of few long rows, by several workgroups a row, in both types; distillation of few long rows; a norm's backward pass."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    rn = lambda *s: torch.randn(s, device=DEV, generator=g)  # noqa: E731
    bf, rows = torch.bfloat16, 6
    s = dict(z16=(2.5 * rn(rows, 70001)).to(bf), z32=2.5 * rn(rows, 20011), u=torch.rand(rows, device=DEV, generator=g), t=0.5 + torch.rand(rows, device=DEV, generator=g),
             p=torch.rand(rows, device=DEV, generator=g), m=0.02 * torch.rand(rows, device=DEV, generator=g),
             ti=torch.randint(0, 70001, (rows, 30), device=DEV, generator=g, dtype=torch.int32), tz=rn(rows, 30), dy=rn(70, 900), h=rn(70, 900), w=1 + 0.1 * rn(900))
    s["p"][:2] = torch.tensor([1.0, 0.0])                        # off; one token
    s["t"][2] = 0.0                                              # greedy
    s["z32"][3] = 1.0                                            # a bin that overflows the list
    s["z16"][4] *= 1e-6
    for k, n, t in (("k16", (rows,), torch.int32), ("k32", (rows,), torch.int32), ("q16", (rows,), torch.float32), ("q32", (rows,), torch.float32), ("loss", (rows,), torch.float32),
                    ("dz", (rows, 70001), bf), ("dh", (70, 900), torch.float32), ("dw", (900,), torch.float32)):
        s[k] = torch.zeros(n, dtype=t, device=DEV)
    return s


SPLIT_OUTPUTS = ("k16", "q16", "k32", "q32", "loss", "dz", "dh", "dw")


def split_calls(b, s, stream=None, ws=None):
    w = (lambda n: ws[:n]) if ws is not None else (lambda n: None)
    b.elmo_sample(s["z16"], s["u"], s["k16"], temperature=s["t"], top_p=s["p"], min_p=s["m"], prob_out=s["q16"], stream=stream, workspace=w(b.elmo_sample_bytes(*s["z16"].shape)))
    b.elmo_sample(s["z32"], s["u"], s["k32"], temperature=s["t"], top_p=s["p"], prob_out=s["q32"], stream=stream, workspace=w(b.elmo_sample_bytes(*s["z32"].shape)))
    b.elmo_distill(s["z16"], s["ti"], s["tz"], s["loss"], s["dz"], temperature=1.5, stream=stream, workspace=w(b.elmo_distill_bytes(*s["z16"].shape)))
    b.elmo_rms_norm_backward(s["dy"], s["h"], s["dh"], s["w"], 1e-6, dweight=s["dw"], stream=stream, workspace=w(b.elmo_rms_norm_backward_bytes(*s["h"].shape)))


def test_split_rows_give_the_oracles_tokens(b):
    from test_gpu_lm import check_tokens
    s = split_state(3)
    split_calls(b, s)
    get = {k: s[k].cpu() for k in ("t", "p", "m", "u")}
    check_tokens(s["z16"].cpu(), get["u"], s["k16"].cpu(), s["q16"].cpu(), t=get["t"], top_p=get["p"], min_p=get["m"])
    check_tokens(s["z32"].cpu(), get["u"], s["k32"].cpu(), s["q32"].cpu(), t=get["t"], top_p=get["p"])


@pytest.mark.parametrize("own", [False, True])
def test_split_rows_captured_and_replayed(b, own):
    """A captured run replays to the eager run's bits on new inputs, with eager work between the replays; with a workspace of the caller's, all calls of the run one after another
    in the same one."""
    s, side = split_state(1), torch.cuda.Stream()
    ws = torch.full((1 << 21,), 255, dtype=torch.uint8, device=DEV) if own else None
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        split_calls(b, s, ws=ws)                                 # kernels loaded before the capture
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        split_calls(b, s, ws=ws)
    for seed in (2, 3, 4):
        new = split_state(seed)
        for k in s:
            s[k].copy_(new[k])
        graph.replay()
        torch.cuda.synchronize()
        split_calls(b, new)
        torch.cuda.synchronize()
        for k in SPLIT_OUTPUTS:
            assert torch.equal(s[k], new[k]), (seed, k)


def test_split_rows_on_two_streams_at_once(b):
    states = [split_state(s) for s in (5, 6)]
    alone = []
    for s in states:
        split_calls(b, s)
        torch.cuda.synchronize()
        alone.append({k: s[k].clone() for k in SPLIT_OUTPUTS})
        for k in SPLIT_OUTPUTS:
            s[k].zero_()
    streams = [torch.cuda.Stream() for _ in states]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, stream in zip(states, streams):
            split_calls(b, s, stream=stream)
    torch.cuda.synchronize()
    for s, want in zip(states, alone):
        for k in SPLIT_OUTPUTS:
            assert torch.equal(s[k], want[k]), k


def test_one_workspace_for_calls_that_follow_one_another(b):
    """Of exactly the stated size, full of ones at first and of the call before's leavings then, with guards behind it: the bits of calls with fresh workspaces."""
    g = gen(12)
    ws = torch.full((16 << 20,), 255, dtype=torch.uint8, device=DEV)

    def exact(n):
        ws[n:].fill_(255)
        return ws[:n]

    def guarded(n):
        assert bool((ws[n:] == 255).all()), "nothing behind the workspace is written"
    for i, (rows, V, dtype) in enumerate([(6, 70001, torch.bfloat16), (40, 16384, torch.float32), (1, 131072, torch.bfloat16), (3, 30000, torch.float32), (6, 70001, torch.bfloat16),
                                          (128, 16400, torch.float32), (2, 200003, torch.bfloat16), (3, 200003, torch.float32)]):
        z, u = (2.5 * torch.randn((rows, V), generator=g)).to(dtype).to(DEV), torch.rand(rows, generator=g).to(DEV)
        p = None if i % 3 == 2 else torch.rand(rows, generator=g).to(DEV)
        n = b.elmo_sample_bytes(rows, V)
        assert n > 0
        token, prob = (torch.empty(rows, dtype=t, device=DEV) for t in (torch.int32, torch.float32))
        fresh, fresh_prob = torch.empty_like(token), torch.empty_like(prob)
        b.elmo_sample(z, u, token, top_p=p, prob_out=prob, workspace=exact(n))
        guarded(n)
        b.elmo_sample(z, u, fresh, top_p=p, prob_out=fresh_prob)
        assert torch.equal(token, fresh) and torch.equal(prob, fresh_prob), (rows, V)
        ti, tz = torch.randint(0, V, (rows, 9), generator=g, dtype=torch.int32).to(DEV), torch.randn((rows, 9), generator=g).to(DEV)
        n = b.elmo_distill_bytes(rows, V)
        loss, again, grad, grad2 = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV), torch.empty_like(z), torch.empty_like(z)
        b.elmo_distill(z, ti, tz, loss, grad, workspace=exact(n))
        guarded(n)
        b.elmo_distill(z, ti, tz, again, grad2)
        assert torch.equal(loss, again) and torch.equal(grad, grad2), (rows, V)
        d = 100 + 37 * i
        h, dy = torch.randn((rows, d), generator=g).to(DEV), torch.randn((rows, d), generator=g).to(DEV)
        n = b.elmo_rms_norm_backward_bytes(rows, d)
        dh, dw, dw2 = torch.empty_like(h), torch.empty(d, device=DEV), torch.empty(d, device=DEV)
        b.elmo_rms_norm_backward(dy, h, dh, None, 1e-6, dweight=dw, workspace=exact(n))
        guarded(n)
        b.elmo_rms_norm_backward(dy, h, dh, None, 1e-6, dweight=dw2)
        assert torch.equal(dw, dw2)


# ------------------------------------------------------------------ distillation
def records(z):
    """How often a thread's maximum moves at most, wherever the stretch of rounds begins that it takes: octet i of a row is thread i % 512's."""
    rows, V = z.shape
    n = -(-V // 4096)
    top = np.full((rows, n * 512), -np.inf)
    whole = z[:, :V // 8 * 8].reshape(rows, -1, 8)
    top[:, :whole.shape[1]] = whole.max(axis=2)
    top, most = top.reshape(rows, n, 512), 0
    for start in range(n):
        m = np.maximum.accumulate(top[:, start:], axis=1)
        most = max(most, int((np.diff(m, axis=1) > 0).sum(axis=1).max(initial=0)))
    return most


def distill_tolerances(z, idx, T, v, dtype, want):
    """The student's sum: v_exp_f32 (2 e) for a token, for each step of its thread's maximum, and for the steps to the wave's, the workgroup's and the row's; arguments, whose
    difference, constant and product are rounded: 3 e of (max - z) / T over all the steps together; three additions in an octet (3 e); above octets FP64.  The
    loss takes that sum's logarithm and FP64 terms and is rounded once.  The gradient: p with one exponential (2 e and 3 e of the argument), the sum's
    rounding, v T, quotient, product (5 e); q v T with three roundings and an addition; the difference's."""
    Z = f64(z) / T
    fin = np.where(np.isfinite(Z), Z, -np.inf)
    top = fin.max(axis=1, keepdims=True)
    x = np.where(np.isfinite(fin), top - fin, 0.0)
    p = np.exp(fin - top)
    p = p / p.sum(axis=1, keepdims=True)
    vv = np.ones((len(Z), 1)) if v is None else f64(v)[:, None]
    dS = E * (2 * (1 + records(fin) + 3) + 3 + 3 * np.sum(p * x, axis=1, keepdims=True))
    loss, grad = want
    tl = np.abs(vv[:, 0]) * T * T * (dS[:, 0] + 2.0 ** -48 * (np.max(x, axis=1) + 20)) + 1.01 * E * np.abs(loss) + 1e-38
    q = np.abs(grad / np.where(vv == 0, 1, vv) / T - p)
    tg = np.abs(vv) * T * (p * (dS + E * (2 + 3 * x + 5)) + 4 * E * q) + (HALF[dtype] + 2 * E) * np.abs(grad) + 1e-38
    return tl, tg


@pytest.mark.parametrize("rows,V,K,T", [(2, 300, 40, 1.0), (3, 32003, 1000, 1.0), (2, 131072, 1024, 2.0), (200, 20011, 512, 0.75), (1, 300007, 1024, 1.0)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_distill_of_a_student_that_agrees(b, rows, V, K, T, dtype):
    """The teacher's tokens hold practically all of the mass, with the student's logits but for 3e-2: the loss is a small difference of large terms."""
    g = gen(V + K)
    z = 2 * torch.randn((rows, V), generator=g) - 25 * T
    idx = torch.stack([torch.randperm(V, generator=g)[:K] for _ in range(rows)]).to(torch.int32)
    heads = 2 * torch.randn((rows, K), generator=g)
    z = z.scatter(1, idx.long(), heads).to(dtype)
    tz = z.gather(1, idx.long()).float() + 3e-2 * torch.randn((rows, K), generator=g)
    loss, grad = torch.empty(rows, device=DEV), torch.empty((rows, V), dtype=dtype, device=DEV)
    b.elmo_distill(z.to(DEV), idx.to(DEV), tz.to(DEV), loss, grad, temperature=T)
    want = o.distill(f64(z), idx.numpy(), f64(tz), T)
    assert np.all(want[0] < 5e-3)
    tl, tg = distill_tolerances(z, idx, T, None, dtype, want)
    close(loss, want[0], tl, "loss")
    close(grad, want[1], tg, "gradient")


# ------------------------------------------------------------------ long rows
@pytest.mark.parametrize("V", [2_200_003, 3_000_001])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_millions_of_outputs(b, V, dtype):
    """Segments of several rounds (above 2097152 tokens), split and by one workgroup; distillation of such rows."""
    from test_gpu_lm import check_tokens
    g, rows = gen(V), 3
    z = (2.5 * torch.randn((rows, V), generator=g)).to(dtype)
    z[1, ::3] = -float("inf")
    z[2] = z[2].round()                                          # ties of hundreds of thousands
    for kw in (dict(), dict(top_p=0.9), dict(top_p=0.4, min_p=0.001, t=0.8), dict(top_k=50), dict(top_k=5000, top_p=0.9), dict(t=0.0), dict(top_k=2 ** 31 - 1)):
        u = torch.rand(rows, generator=g)
        s = {n: torch.full((rows,), v, dtype=torch.int32 if n == "top_k" else torch.float32) for n, v in kw.items()}
        token, prob = draw(b, z, u, **{"temperature" if n == "t" else n: v for n, v in s.items()})
        check_tokens(z, u, token, prob, **s)
    idx, tz = torch.randint(0, V, (rows, 20), generator=g, dtype=torch.int32), torch.randn((rows, 20), generator=g)
    loss, grad = torch.empty(rows, device=DEV), torch.empty((rows, V), dtype=dtype, device=DEV)
    b.elmo_distill(z.to(DEV), idx.to(DEV), tz.to(DEV), loss, grad)
    want = o.distill(f64(z), idx.numpy(), f64(tz), 1.0)
    tl, tg = distill_tolerances(z, idx, 1.0, None, dtype, want)
    some = np.isfinite(want[0])                                  # (a masked token of the teacher's: infinite, by definition)
    assert np.all(np.isposinf(f64(loss)[~some]))
    close(loss[torch.from_numpy(some)], want[0][some], tl[some], "loss")
    close(grad, want[1], tg, "gradient")


# ------------------------------------------------------------------ beside a head
def test_a_heads_inputs_scores_and_input_gradient(b):
    """The norm's rows are a head's inputs, its top scores the logits to sample from and the teacher of a smaller student, its input gradient what the norm's backward pass takes."""
    from test_gpu_lm import check_tokens
    rows, d, L, k, bf = 24, 256, 5003, 40, torch.bfloat16
    g = gen(21)
    x, r, w = torch.randn((rows, d), generator=g).to(bf).to(DEV), torch.randn((rows, d), generator=g).to(bf).to(DEV), (1 + 0.1 * torch.randn(d, generator=g)).to(DEV)
    y, h = torch.empty_like(x), torch.empty_like(x)
    b.elmo_rms_norm(x, y, w, 1e-6, residual=r, sum_out=h)
    head = b.Head(L, d, b.ELMO_BF16, 1024, b.ELMO_SR, rows, 4 * rows)
    head.weights().copy_((0.2 * torch.randn((L, d), generator=g)).to(bf).to(DEV).view(torch.int16))
    idx, score = torch.empty((rows, k), dtype=torch.int32, device=DEV), torch.empty((rows, k), device=DEV)
    head.topk(y, k, idx, score)

    u, t, p = torch.rand(rows, generator=g), torch.full((rows,), 0.8), torch.full((rows,), 0.9)
    place, prob = draw(b, score, u, temperature=t, top_p=p)
    check_tokens(score.cpu(), u, place, prob, t=t, top_p=p)
    label = idx.gather(1, place.long()[:, None].to(DEV))
    assert bool(((label >= 0) & (label < L)).all())

    z = torch.randn((rows, L), generator=g).to(bf)
    loss, dz = torch.empty(rows, device=DEV), torch.empty((rows, L), dtype=bf, device=DEV)
    b.elmo_distill(z.to(DEV), idx, score, loss, dz, temperature=2.0)
    want = o.distill(f64(z), idx.cpu().numpy(), f64(score), 2.0)
    tl, tg = distill_tolerances(z, idx.cpu(), 2.0, None, bf, want)
    close(loss, want[0], tl, "loss")
    close(dz, want[1], tg, "gradient")

    labels = torch.stack([torch.randperm(L, generator=g)[:3].sort().values for _ in range(rows)]).to(torch.int32)
    indptr = torch.arange(0, 3 * rows + 1, 3, dtype=torch.int32, device=DEV)
    dy, dh, dw = torch.empty_like(x), torch.empty_like(x), torch.empty(d, device=DEV)
    head.step(y, indptr, labels.flatten().to(DEV), 0.01, 1, 1, dX_out=dy)
    b.elmo_rms_norm_backward(dy, h, dh, w, 1e-6, dweight=dw)
    assert bool(dy.float().abs().max() > 0)
    want, wantw = o.rms_norm_backward(f64(dy), f64(h), f64(w), 1e-6)
    th, tw = back_tolerances(dy.cpu(), h.cpu(), w.cpu(), 1e-6, bf, want)
    close(dh, want, th, "dh")
    close(dw, wantw, tw, "dweight")
    head.close()
