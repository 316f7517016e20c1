"""Plain 64-bit attention of packed texts with its backward pass, and how far a result of fewer bits may be from it.

u = 2^-24 bounds the relative error of an fp32 operation, e that of a rounding to the tensors' type (fp32 u, bf16 2^-8).
Products of a kernel are exact or rounded once, sums of n terms are off by n u of the sum of magnitudes, whatever their order:
  s: (hd + 6) u of scale sum |q||k| (terms, scale, base of the logarithm), p = 2^(s - lse): relative
  P = that of every s and lse + (|s| + |lse|) 4 u + 16 u (the subtraction, the exponential, the sum's own n u)
Where probabilities or the scores' gradients are rounded to the tensors' type, e is added.
"""
import math

U = 2.0 ** -24


def half_step(torch, dtype):
    return torch.finfo(dtype).eps / 2


def forward(torch, lens, row0, q, k, v, scale):
    """(out, lse, bound of out, bound of lse) in 64 bits, rows of no text 0 and -infinity (bounds 0)."""
    R, Hq, hd = q.shape
    G = Hq // k.shape[1]
    e = half_step(torch, q.dtype)
    f64 = dict(dtype=torch.float64, device=q.device)
    out, lse = torch.zeros(R, Hq, hd, **f64), torch.full((R, Hq), -math.inf, **f64)
    t_out, t_lse = torch.zeros_like(out), torch.zeros(R, Hq, **f64)
    at = row0
    for n in lens:
        rows = slice(at, at + n)
        at += n
        if n == 0:
            continue
        Q = q[rows].double().transpose(0, 1)
        K, V = (x[rows].double().transpose(0, 1).repeat_interleave(G, 0) for x in (k, v))
        s, hidden, s_err = _scores(torch, Q, K, scale)
        l = torch.logsumexp(s, -1)
        p = torch.exp(s - l[..., None])
        worst = s_err.masked_fill(hidden, 0).amax(-1, keepdim=True)
        P = s_err + worst + (s.masked_fill(hidden, 0).abs() + l.abs()[..., None]) * 4 * U + (16 + n) * U
        o = p @ V
        out[rows], lse[rows] = o.transpose(0, 1), l.T
        rounding = e if q.dtype == torch.bfloat16 else 0.0
        t = (p * (P + rounding + (n + 8) * U)) @ V.abs() + e * o.abs() + 1e-30
        t_out[rows] = t.transpose(0, 1)
        t_lse[rows] = (worst[..., 0] + (16 + n) * U + l.abs() * 8 * U + s.masked_fill(hidden, 0).abs().amax(-1) * 4 * U).T
    return out, lse, t_out, t_lse


def _scores(torch, Q, K, scale):
    n, hd = Q.shape[1:]
    s = Q @ K.transpose(1, 2) * scale
    hidden = torch.ones(n, n, dtype=torch.bool, device=Q.device).triu(1)
    s_err = (Q.abs() @ K.abs().transpose(1, 2)) * (abs(scale) * (hd + 6) * U)
    return s.masked_fill(hidden, -math.inf), hidden, s_err


def backward(torch, lens, row0, q, k, v, d_out, scale, out, lse):
    """[dq, dk, dv] in 64 bits, and their bounds for a call that is given `out` and `lse` (whose own distance from the exact ones
    counts: through delta, and through every probability)."""
    R, Hq, hd = q.shape
    Hkv = k.shape[1]
    G = Hq // Hkv
    e = half_step(torch, q.dtype)
    rounding = e if q.dtype == torch.bfloat16 else 0.0
    f64 = dict(dtype=torch.float64, device=q.device)
    grads = [torch.zeros(R, H, hd, **f64) for H in (Hq, Hkv, Hkv)]
    bounds = [torch.zeros(R, H, hd, **f64) for H in (Hq, Hkv, Hkv)]
    at = row0
    for n in lens:
        rows = slice(at, at + n)
        at += n
        if n == 0:
            continue
        Q, D = (x[rows].double().transpose(0, 1) for x in (q, d_out))
        K, V = (x[rows].double().transpose(0, 1).repeat_interleave(G, 0) for x in (k, v))
        s, hidden, s_err = _scores(torch, Q, K, scale)
        l = torch.logsumexp(s, -1, keepdim=True)
        p = torch.exp(s - l)
        O = p @ V
        delta = (D * O).sum(-1, keepdim=True)
        dp = D @ V.transpose(1, 2)
        ds = p * (dp - delta)
        group = lambda x: x.view(Hkv, G, n, hd).sum(1)
        dv, dk, dq = group(p.transpose(1, 2) @ D), group(ds.transpose(1, 2) @ Q) * scale, ds @ K * scale
        given_l = (lse[rows].double().T[..., None] - l).abs()
        P = s_err + given_l + (s.masked_fill(hidden, 0).abs() + l.abs()) * 4 * U + 16 * U
        given_o = (D.abs() * (out[rows].double().transpose(0, 1) - O).abs()).sum(-1, keepdim=True)
        mag = (D.abs() @ V.abs().transpose(1, 2)) + (D.abs() * (O.abs() + (out[rows].double().transpose(0, 1) - O).abs())).sum(-1, keepdim=True)
        ds_err = ds.abs() * (P + rounding + 4 * U) + p * (1 + P + rounding) * ((hd + 4) * U * mag + given_o)
        m = (n * G + 8) * U
        t_dv = group((p * (P + rounding + m)).transpose(1, 2) @ D.abs())
        t_dk = group((ds_err + ds.abs() * m).transpose(1, 2) @ Q.abs()) * abs(scale)
        t_dq = (ds_err + ds.abs() * m) @ K.abs() * abs(scale)
        for g, b, x, t in zip(grads, bounds, (dq, dk, dv), (t_dq, t_dk, t_dv)):
            g[rows] = x.transpose(0, 1)
            b[rows] = (t + (e + 2 * U) * x.abs() + 1e-30).transpose(0, 1)
    return grads, bounds


def inside(torch, got, want, bound, what):
    got = got.double()
    assert not torch.isnan(got).any(), what
    same = got == want  # (infinities)
    off = torch.where(same, torch.zeros_like(want), (got - want).abs())
    worst = (off - bound).max().item() if off.numel() else 0.0
    assert worst <= 0, f"{what}: beyond its bound by {worst:.3g} (largest difference {off.max().item():.3g})"
