"""Attention over the 8-bit cache in float64, row by row over what the row sees, and how far a
kernel may be off by what it sees alone."""
import torch


def attention(cache, b, q, sees, scale, dtype):
    """q [n, nq, hd] of sequence b, sees bool [n, T].  Per element: half a step of the output's type;
    of the mass sum w |v|: the rounding of P (bf16 rows 2^-11, fp32 rows two parts of f16: 2^-22), the exponent's
    error (fp32 sums of hd products and four roundings, 2^-24 each) in numerator and sum, fp32 sums of at most 2^6
    partial results of a wavefront and page pair (2^-18); and P's smallest step, 2^-30 of the largest a position."""
    bf16 = dtype is torch.bfloat16
    half, p_step = (2.0 ** -8, 2.0 ** -11) if bf16 else (2.0 ** -24, 2.0 ** -22)
    n, nq, hd = q.shape
    T = sees.shape[1]
    k, v = cache.context(b, T)
    q = q.cpu().double()
    out, tol = (torch.zeros((n, nq, hd), dtype=torch.float64) for _ in range(2))
    count = sees.sum(-1, keepdim=True)
    for h in range(nq):
        kh, vh = k[h * cache.nkv // nq], v[h * cache.nkv // nq]
        z = ((q[:, h] @ kh.T) * scale).masked_fill(~sees, -torch.inf)
        m = z.max(-1, keepdim=True).values
        w = torch.where(sees, torch.exp(z - torch.where(m > -torch.inf, m, 0.0)), 0.0)
        w = w / w.sum(-1, keepdim=True).clamp(min=1e-300)
        size = 2.0 ** -24 * (hd + 8) * ((q[:, h].abs() @ kh.abs().T) * scale)
        dz = torch.where(sees, size, 0.0).max(-1, keepdim=True).values
        top = torch.where(sees, vh.abs().max(-1).values, 0.0).max(-1, keepdim=True).values
        out[:, h] = w @ vh
        tol[:, h] = half * out[:, h].abs() + (p_step + 2 * dz + 2.0 ** -18) * (w @ vh.abs()) + count * 2.0 ** -30 * top
    return out, tol


def causal(cached, rows):
    return torch.arange(cached + rows)[None] <= torch.arange(cached, cached + rows)[:, None]
