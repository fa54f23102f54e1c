"""The operators at the output end of a language model, as cases to be measured.

A case is a dict of plain values.  Kinds:

  norm       root-mean-square norm behind the residual's addition; the result in BF16 / FP32, or in 8 bits with a scale
             for each token (`elmo_rms_norm`);
  norm_back  its backward pass: input gradient and weight gradient (`elmo_rms_norm_backward`);
  int8       8-bit integer product with a scale for each token and each output channel (`elmo_int8_matmul`);
  sample     one token a row by temperature, top-k, top-p and min-p from a given random number (`elmo_sample`);
  distill    distillation from a teacher's top logits, loss and logit gradient in one call (`elmo_distill`).

They follow one another: the norm's 8-bit rows are what the integer product takes, its logits are what is
sampled or distilled.  Sizes are those of `synth.CONFIGS` where those have one (width 768, 8192 and 131072 outputs) and generic
ones.  `pad` is the number of elements between two rows beyond a row's own (rows that are slices of wider buffers).

Definitions (z logits, all sums in exact arithmetic):

  norm      h = x + r,  y = w h / sqrt(mean(h^2) + eps);  stream' = h;
            int8: m = max|w h|, q = round(w h 127 / m), scale = m / (127 sqrt(mean(h^2) + eps));  E4M3: the same with 448
  int8      out = (sum_k a b) sa sb + bias
  sample    tokens ordered by (z falling, index rising), weights exp((z - max z) / t); kept are the first top_k of them, of those
            the shortest prefix with at least top_p of their weight, of those the ones of weight >= min_p;
            the token is the first one in order of INDEX at which the kept weight so far exceeds u times the kept weight
  distill   q = softmax(teacher / T) over the teacher's tokens (index >= 0), p = softmax(z / T) over all:
            loss = v T^2 sum q log(q / p),  gradient = v T (p - q), v a weight for each row
"""
from __future__ import annotations

import math

import numpy as np
import torch

DEV = "cuda:0"
own = False

TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32, "e4m3": torch.float8_e4m3fn, "int8": torch.int8}
EPS = 1e-6


def _norm(name, rows, d, dtype, out, residual=True, weight="bf16", pad=0):
    return dict(name=name, kind="norm", rows=rows, d=d, dtype=dtype, out=out, residual=residual, weight=weight, pad=pad)


def _back(name, rows, d, dtype, stream=True, weight="bf16", pad=0):
    return dict(name=name, kind="norm_back", rows=rows, d=d, dtype=dtype, stream=stream, weight=weight, pad=pad)


def _int8(name, M, N, K, out="bf16", bias=False, pad=0):
    return dict(name=name, kind="int8", M=M, N=N, K=K, out=out, bias=bias, pad=pad)


def _sample(name, rows, V, dtype, top_k, top_p, min_p, masked=0.0, pad=0):
    return dict(name=name, kind="sample", rows=rows, V=V, dtype=dtype, top_k=top_k, top_p=top_p, min_p=min_p, masked=masked, pad=pad)


def _distill(name, rows, V, K, dtype, T=1.0, short=False, pad=0):
    return dict(name=name, kind="distill", rows=rows, V=V, K=K, dtype=dtype, T=T, short=short, pad=pad)


def listed():
    return [
        # One new token of one sequence in front of an 8-bit product: the smallest call, latency counts.
        _norm("norm_token", 1, 768, "bf16", "int8"),
        # A batch of prompts, residual stream in and out, rows in 8 bits for the products behind it.
        _norm("norm_prompts", 16384, 4096, "bf16", "int8"),
        # Training at an odd width in FP32, nothing a multiple of a vector.
        _back("norm_back_odd", 1021, 1001, "fp32", weight="fp32"),
        # A training batch of the same width as the prompts, gradient of the stream joined.
        _back("norm_back_batch", 16384, 4096, "bf16"),
        # One token through one projection: the weights' stream is the work.
        _int8("int8_token", 1, 4096, 4096),
        # A decoding batch through a vocabulary projection, rows and outputs ragged, logits in FP32.
        _int8("int8_decode", 37, 32003, 4096, out="fp32", bias=True),
        # A batch of prompts through a wide projection: the matrix cores are the work.
        _int8("int8_prompts", 8192, 14336, 4096),
        # One sequence decodes a token.
        _sample("sample_one", 1, 131072, "bf16", 50, 0.95, 0.0),
        # A serving batch, top-p alone, so that nothing bounds how many tokens stay.
        _sample("sample_batch", 256, 131072, "bf16", 0, 0.9, 0.0),
        # Constrained decoding: half of the vocabulary masked, an odd one, FP32 rows inside a wider buffer.
        _sample("sample_masked", 33, 100003, "fp32", 0, 0.98, 0.02, masked=0.5, pad=5),
        # A short fine-tuning batch over a small vocabulary.
        _distill("distill_small", 64, 8192, 16, "fp32", T=2.0),
        # A training batch over a large vocabulary: the logits and their gradient are the work.
        _distill("distill_batch", 4096, 131072, 64, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    kind = rng.choice(["norm", "norm_back", "int8", "int8", "sample", "sample", "distill", "distill"])
    pad = rng.choice([0, 0, 0, 8, 5])
    weight = rng.choice(["bf16", "fp32"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    if kind in ("norm", "norm_back"):
        d = rng.choice([_log_int(rng, 64, 8192), 64 * _log_int(rng, 1, 128)])
        rows = _log_int(rng, 1, min(16384, 16384 * 4096 // d // (2 if dtype == "fp32" else 1)))
        if kind == "norm_back":
            return dict(kind=kind, rows=rows, d=d, dtype=dtype, stream=rng.random() < 0.7, weight=weight, pad=pad)
        return dict(kind=kind, rows=rows, d=d, dtype=dtype, out=rng.choice(["int8", "int8", "e4m3", dtype]), residual=rng.random() < 0.8, weight=weight,
                    pad=pad)
    if kind == "int8":
        K = rng.choice([16 * _log_int(rng, 1, 1024), 16 * _log_int(rng, 16, 512), _log_int(rng, 16, 8192)])
        N = min(_log_int(rng, 16, 131072), (1 << 28) // K)
        M = min(_log_int(rng, 1, 8192), max(1, 8192 * 14336 * 4096 // (N * K)), (1 << 28) // N)
        return dict(kind=kind, M=M, N=N, K=K, out=rng.choice(["bf16", "fp32"]), bias=rng.random() < 0.3, pad=pad)
    V = rng.choice([_log_int(rng, 1000, 262144), 8 * _log_int(rng, 125, 32768)])
    if kind == "sample":
        rows = _log_int(rng, 1, min(512, 256 * 131072 // V // (2 if dtype == "fp32" else 1)))
        return dict(kind=kind, rows=rows, V=V, dtype=dtype, top_k=rng.choice([0, 0, 1, 20, 50, 300]), top_p=rng.choice([1.0, 0.5, 0.9, 0.95]),
                    min_p=rng.choice([0.0, 0.0, 0.05]), masked=rng.choice([0.0, 0.0, 0.3]), pad=pad)
    rows = _log_int(rng, 1, min(4096, 4096 * 131072 // V // (2 if dtype == "fp32" else 1)))
    return dict(kind=kind, rows=rows, V=V, K=_log_int(rng, 1, 256), dtype=dtype, T=rng.choice([1.0, 1.0, 2.0, 0.7]), short=rng.random() < 0.4, pad=pad)


# ------------------------------------------------------------------ inputs
def _rows(t, pad):
    """The same values as rows of a wider buffer."""
    if not pad:
        return t
    wide = torch.zeros((t.shape[0], t.shape[1] + pad), dtype=t.dtype, device=t.device)
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


def _logits(gen, rows, V, dtype):
    """Logits as a model gives them: a bulk that is near normal and a few dozen tokens that stand out, more of it in some rows than in others."""
    z = torch.randn((rows, V), device=DEV, generator=gen)
    z *= 1.0 + 1.5 * torch.rand((rows, 1), device=DEV, generator=gen)
    n = min(48, V)
    at = torch.randint(0, V, (rows, n), device=DEV, generator=gen)
    up = 4.0 + 10.0 * torch.rand((rows, 1), device=DEV, generator=gen)
    # the later a token's place among them, the less it stands out
    z.scatter_add_(1, at, up - 1.5 * torch.log1p(torch.arange(n, device=DEV, dtype=torch.float32)) + torch.randn((rows, n), device=DEV, generator=gen))
    return z.to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    randn = lambda *shape: torch.randn(shape, device=DEV, generator=gen)  # noqa: E731
    rand = lambda *shape: torch.rand(shape, device=DEV, generator=gen)  # noqa: E731
    empty = lambda shape, dtype: torch.empty(shape, dtype=dtype, device=DEV)  # noqa: E731
    s = {"case": case}
    kind, pad = case["kind"], case["pad"]
    if kind in ("norm", "norm_back"):
        rows, d, t = case["rows"], case["d"], TYPES[case["dtype"]]
        s["w"] = (1.0 + 0.2 * randn(d)).to(TYPES[case["weight"]])
        # the stream has a few columns that are far larger than the others, as trained models do
        col = torch.where(rand(d) < 0.01, 12.0, 1.0)
        s["x"] = _rows((randn(rows, d) * col).to(t), pad)
        if kind == "norm":
            s["r"] = _rows((2.0 * randn(rows, d) * col).to(t), pad) if case["residual"] else None
            s["sum"] = empty((rows, d), t) if case["residual"] else None
            s["y"] = empty((rows, d), TYPES[case["out"]])
            s["scale"] = empty((rows,), torch.float32) if case["out"] in ("int8", "e4m3") else None
            return s
        s["dy"] = _rows((1e-2 * randn(rows, d)).to(t), pad)
        s["dsum"] = _rows((1e-2 * randn(rows, d)).to(t), pad) if case["stream"] else None
        s["dx"], s["dw"] = empty((rows, d), t), empty((d,), torch.float32)
        return s
    if kind == "int8":
        M, N, K = case["M"], case["N"], case["K"]
        whole = lambda r: _rows((randn(r, K) * 32.0).round_().clamp_(-127, 127).to(torch.int8), pad)  # noqa: E731
        s["a"], s["b"] = whole(M), whole(N)
        s["sa"], s["sb"] = 0.01 + 0.05 * rand(M), 1e-4 + 1e-3 * rand(N)
        s["bias"] = randn(N) if case["bias"] else None
        s["out"] = empty((M, N), TYPES[case["out"]])
        return s
    rows, V, t = case["rows"], case["V"], TYPES[case["dtype"]]
    z = _logits(gen, rows, V, t)
    if kind == "sample":
        if case["masked"]:
            z.masked_fill_(rand(rows, V) < case["masked"], -math.inf)
        s["z"] = _rows(z, pad)
        # requests of one batch have their own settings; 0, 1 and 0 switch a filter off
        s["t"] = 0.6 + 0.6 * rand(rows)
        k = case["top_k"]
        s["top_k"] = torch.randint(1, k + 1, (rows,), device=DEV, generator=gen, dtype=torch.int32).clamp_(min=(k + 1) // 2) if k else None
        s["top_p"] = 1.0 - (1.0 - case["top_p"]) * (0.5 + 0.5 * rand(rows)) if case["top_p"] < 1.0 else None
        s["min_p"] = case["min_p"] * (0.5 + 0.5 * rand(rows)) if case["min_p"] else None
        s["u"] = rand(rows)
        s["token"], s["prob"] = empty((rows,), torch.int32), empty((rows,), torch.float32)
        return s
    K = min(case["K"], V)
    s["z"] = _rows(z, pad)
    # the teacher's top tokens: its logits are the student's, moved
    top, at = (z.float() + 0.7 * randn(rows, V)).topk(K, dim=1) if rows * V <= 1 << 29 else (z + randn(rows, V).to(t)).topk(K, dim=1)
    s["ti"], s["tz"] = at.to(torch.int32), top.float().contiguous()
    if case["short"]:      # rows with fewer tokens than K end in -1
        s["ti"][rand(rows, K).cumsum(1) > 0.75 * K] = -1
    s["v"] = torch.where(rand(rows) < 0.1, 0.0, 1.0 / rows)      # padding counts nothing
    s["loss"], s["grad"] = empty((rows,), torch.float32), empty((rows, V), t)
    return s


# ------------------------------------------------------------------ one pass
def run(s):
    case = s["case"]
    kind = case["kind"]
    if own:
        from paper_2510_11168_amd import binding as b
        if kind == "norm":
            b.elmo_rms_norm(s["x"], s["y"], s["w"], EPS, residual=s["r"], sum_out=s["sum"], scale_out=s["scale"])
            return s["y"], s["sum"], s["scale"]
        if kind == "norm_back":
            b.elmo_rms_norm_backward(s["dy"], s["x"], s["dx"], s["w"], EPS, dsum=s["dsum"], dweight=s["dw"])
            return s["dx"], s["dw"]
        if kind == "int8":
            b.elmo_int8_matmul(s["a"], s["sa"], s["b"], s["sb"], s["out"], bias=s["bias"])
            return s["out"]
        if kind == "sample":
            b.elmo_sample(s["z"], s["u"], s["token"], temperature=s["t"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"], prob_out=s["prob"])
            return s["token"], s["prob"]
        b.elmo_distill(s["z"], s["ti"], s["tz"], s["loss"], s["grad"], temperature=case["T"], row_weight=s["v"])
        return s["loss"], s["grad"]
    return {"norm": _plain_norm, "norm_back": _plain_back, "int8": _plain_int8, "sample": _plain_sample, "distill": _plain_distill}[kind](s, case)


def _plain_norm(s, case):
    h = s["x"].float() if s["r"] is None else s["x"].float() + s["r"].float()
    stream = None if s["r"] is None else h.to(s["x"].dtype)
    inv = torch.rsqrt(h.square().mean(1, keepdim=True) + EPS)
    if case["out"] not in ("int8", "e4m3"):
        return (h * inv * s["w"].float()).to(TYPES[case["out"]]), stream, None
    # quotients next to a rounding border: in 64 bits
    p = h.double() * s["w"].double()
    m = p.abs().amax(1, keepdim=True)
    most = 127.0 if case["out"] == "int8" else 448.0
    q = p * (most / m)
    q = q.round().to(torch.int8) if case["out"] == "int8" else q.float().to(torch.float8_e4m3fn)
    return q, stream, (m.float() * inv / most).squeeze(1)


def _plain_back(s, case):
    h, dy = s["x"].float(), s["dy"].float()
    inv = torch.rsqrt(h.square().mean(1, keepdim=True) + EPS)
    g = dy * s["w"].float()
    dx = inv * (g - h * (inv.square() * (g * h).mean(1, keepdim=True)))
    if s["dsum"] is not None:
        dx = dx + s["dsum"].float()
    return dx.to(s["x"].dtype), (dy * h * inv).sum(0)


def _plain_int8(s, case):
    # 64 bits hold every sum exactly, 32 bits do not
    out = (s["a"].double() @ s["b"].double().t()).float() * s["sa"][:, None] * s["sb"][None, :]
    if s["bias"] is not None:
        out = out + s["bias"]
    return out.to(TYPES[case["out"]])


def _plain_sample(s, case):
    # which token a number falls on is decided next to borders: weights and their sums in 64 bits
    z, order = torch.sort(s["z"].float(), dim=1, descending=True, stable=True)
    w = torch.exp((z.double() - z[:, :1].double()) / s["t"].double()[:, None])
    rank = torch.arange(w.shape[1], device=w.device)[None, :]
    if s["top_k"] is not None:
        w = torch.where(rank < s["top_k"][:, None], w, 0.0)
    if s["top_p"] is not None:
        upto = w.cumsum(1)
        w = torch.where(upto - w < s["top_p"].double()[:, None] * upto[:, -1:], w, 0.0)
    if s["min_p"] is not None:
        w = torch.where(w >= s["min_p"].double()[:, None], w, 0.0)
    w = torch.zeros_like(w).scatter_(1, order, w)
    upto = w.cumsum(1)
    token = (upto > s["u"].double()[:, None] * upto[:, -1:]).to(torch.uint8).argmax(1, keepdim=True)
    return token.squeeze(1).to(torch.int32), (w.gather(1, token) / upto[:, -1:]).squeeze(1).float()


def _plain_distill(s, case):
    T = case["T"]
    z = s["z"].float() / T
    logp = z - z.amax(1, keepdim=True)
    logp = logp - logp.exp().sum(1, keepdim=True).log()
    there = s["ti"] >= 0
    at = s["ti"].clamp(min=0).to(torch.int64)
    t = torch.where(there, s["tz"] / T, -math.inf)
    t = t - t.amax(1, keepdim=True)
    logq = t - t.exp().sum(1, keepdim=True).log()
    q = torch.where(there, logq.exp(), 0.0)
    loss = torch.where(there, q * (logq - logp.gather(1, at)), 0.0).sum(1) * (s["v"] * T * T)
    grad = logp.exp_().scatter_add_(1, at, -q) * (s["v"] * T)[:, None]
    return loss, grad.to(s["z"].dtype)


# ------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    f = lambda v: v.to(torch.float64)  # noqa: E731
    if kind == "norm":
        h = f(s["x"]) + (f(s["r"]) if case["residual"] else 0.0)
        size = torch.linalg.vector_norm(h, dim=1, keepdim=True)
        rms = torch.sqrt(size * size / case["d"] + EPS)
        stream = h if case["residual"] else None
        if case["out"] not in ("int8", "e4m3"):
            return f(s["w"]) * h / rms, stream, None
        most = 127.0 if case["out"] == "int8" else 448.0
        scale = (f(s["w"]) * h).abs().amax(1, keepdim=True) / (most * rms)
        # whole numbers of a rounding border have no nearer value in 64 bits than the plain form's
        return None if case["out"] == "int8" else f(s["w"]) * h / rms / scale, stream, scale[:, 0]
    if kind == "norm_back":
        # through the product rule: y = w h / rms, d rms / d h_j = h_j / (d rms)
        h, dy, w, d = f(s["x"]), f(s["dy"]), f(s["w"]), case["d"]
        rms = torch.sqrt((h * h).sum(1) / d + EPS)[:, None]
        along = torch.matmul((dy * h), w)[:, None]
        dx = dy * w / rms - along * h / (d * rms ** 3)
        return dx + f(s["dsum"]) if case["stream"] else dx, torch.matmul((1.0 / rms).t(), dy * h)[0]
    if kind == "int8":
        out = torch.matmul(f(s["b"]) * f(s["sb"])[:, None], (f(s["a"]) * f(s["sa"])[:, None]).t()).t().contiguous()
        return out + f(s["bias"]) if case["bias"] else out
    if kind == "sample":
        z, rows = f(s["z"]).cpu().numpy(), case["rows"]
        get = lambda n, off: np.full(rows, off) if s[n] is None else f(s[n]).cpu().numpy()  # noqa: E731
        t, k, p, m, u = get("t", 1.0), get("top_k", case["V"]), get("top_p", 1.0), get("min_p", 0.0), get("u", 0.0)
        tokens, probs = np.zeros(rows, np.int64), np.zeros(rows)
        for r in range(rows):
            order = np.argsort(-z[r], kind="stable")[:int(k[r])]
            w = np.exp((z[r][order] - z[r][order[0]]) / t[r])
            keep = int(np.searchsorted(np.cumsum(w), p[r] * w.sum())) + 1 if s["top_p"] is not None else len(w)
            keep = min(keep, int(np.count_nonzero(w >= m[r])))
            by_index = np.sort(order[:keep])
            w = np.exp((z[r][by_index] - z[r][order[0]]) / t[r])
            c = np.cumsum(w)
            j = min(int(np.searchsorted(c, u[r] * c[-1], side="right")), len(w) - 1)
            tokens[r], probs[r] = by_index[j], w[j] / c[-1]
        return tokens, probs
    T = case["T"]
    z = f(s["z"]) / T
    lse = torch.logsumexp(z, 1, keepdim=True)
    t = (f(s["tz"]) / T).masked_fill(s["ti"] < 0, -math.inf)
    logq = t - torch.logsumexp(t, 1, keepdim=True)
    q = torch.exp(logq)
    at = s["ti"].clamp(min=0).long()
    terms = torch.where(s["ti"] < 0, 0.0, q * (logq - (z.gather(1, at) - lse)))
    loss = f(s["v"]) * T * T * terms.sum(1)
    z.sub_(lse).exp_()
    z.scatter_add_(1, at, -q).mul_(T * f(s["v"])[:, None])
    return loss, z


def work(case):
    kind = case["kind"]
    size = lambda t: {"bf16": 2, "fp32": 4, "e4m3": 1, "int8": 1}[case[t]]  # noqa: E731
    if kind == "norm":
        n, e = case["rows"] * case["d"], size("dtype")
        return {"bytes": n * (e * (3 if case["residual"] else 1) + size("out")) + case["d"] * size("weight") + 4 * case["rows"] * (size("out") == 1),
                "flops": 6.0 * n}
    if kind == "norm_back":
        n, e = case["rows"] * case["d"], size("dtype")
        return {"bytes": n * e * (4 if case["stream"] else 3) + case["d"] * (size("weight") + 4), "flops": 12.0 * n}
    if kind == "int8":
        M, N, K = case["M"], case["N"], case["K"]
        return {"bytes": (M + N) * (K + 4) + M * N * size("out") + (4 * N if case["bias"] else 0), "flops": 2.0 * M * N * K}
    n = case["rows"] * case["V"]
    if kind == "sample":
        return {"bytes": n * size("dtype") + 28 * case["rows"], "flops": 4.0 * n}
    return {"bytes": 2 * n * size("dtype") + case["rows"] * (8 * case["K"] + 8), "flops": 8.0 * n}
