"""The 8-bit cache in float64 on the CPU, token by token, written from its description in
include/osprey.h: what the GPU tests compare with."""
import math

import torch

PG = 16
MIN_EXP = -100


def e4m3_values():
    """The 127 finite magnitudes, ascending (index = code)."""
    return torch.tensor([(m * 2.0 ** -9) if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)][:127],
                        dtype=torch.float64)


def round8(x):
    """Nearest e4m3 value of |x| <= 448, the even code on ties."""
    tab = e4m3_values()
    a = x.abs().contiguous()
    assert float(a.max() if a.numel() else 0) <= 448.0
    hi = torch.searchsorted(tab, a).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    dl, dh = a - tab[lo], tab[hi] - a
    code = torch.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return torch.copysign(tab[code], x)


def scale_for(amax: float) -> float:
    e = MIN_EXP
    while amax > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def value_places(hd):
    """[16, hd]: where token t, dim e of a value block lies."""
    t, e = torch.meshgrid(torch.arange(PG), torch.arange(hd), indexing="ij")
    return (t // 4) * 4 * hd + (e % 16) * (hd // 4) + (e // 16) * 4 + t % 4


class Cache:
    """Codes' values v [pages, 2, nkv, 16, hd] and scales s [pages, nkv, 2], in float64."""

    def __init__(self, codes, scales, table, hd):
        c = codes.cpu().contiguous().view(torch.float8_e4m3fn).double()
        pages, _, nkv, _ = c.shape
        self.v = torch.empty((pages, 2, nkv, PG, hd), dtype=torch.float64)
        self.v[:, 0] = c[:, 0].view(pages, nkv, PG, hd)
        self.v[:, 1] = c[:, 1][:, :, value_places(hd).flatten()].view(pages, nkv, PG, hd)
        self.s = scales.cpu().double().clone()
        self.table = table.cpu().long()
        self.hd, self.nkv = hd, nkv

    def read(self, b, t):
        """Keys and values [nkv, hd] of position t of sequence b."""
        p = int(self.table[b, t // PG])
        return (self.v[p, 0, :, t % PG] * self.s[p, :, 0, None]).clone(), (self.v[p, 1, :, t % PG] * self.s[p, :, 1, None]).clone()

    def context(self, b, n):
        pages = self.table[b, :(n + PG - 1) // PG]
        x = self.v[pages] * self.s[pages].transpose(1, 2)[..., None, None]
        return tuple(x[:, k].transpose(0, 1).reshape(self.nkv, -1, self.hd)[:, :n] for k in (0, 1))

    def write(self, b, t0, k, v):
        """Positions t0 .. of sequence b take k, v [n, nkv, hd], in one call."""
        n = k.shape[0]
        for p0 in range(t0 // PG, (t0 + n + PG - 1) // PG):
            lo, hi = max(t0, p0 * PG), min(t0 + n, (p0 + 1) * PG)
            page, off = int(self.table[b, p0]), lo - p0 * PG
            for kind, x in ((0, k), (1, v)):
                for h in range(self.nkv):
                    new = x[lo - t0:hi - t0, h]
                    new = torch.where(torch.isfinite(new), new, torch.zeros_like(new))
                    s = scale_for(float(new.abs().max()))
                    if off > 0:
                        old = float(self.s[page, h, kind])
                        s = max(s, old)
                        if s > old:
                            self.v[page, kind, h, :off] = round8(self.v[page, kind, h, :off] * (old / s))
                    self.v[page, kind, h, off:off + hi - lo] = round8(new / s)
                    self.s[page, h, kind] = s

    def keep(self, b, base, path):
        n = len(path)
        kv = [self.read(b, base + p) for p in path]
        if n:
            self.write(b, base, torch.stack([x[0] for x in kv]), torch.stack([x[1] for x in kv]))


def norm_rope(x, gain, eps, cos, sin):
    """x [n, heads, hd] float64; cos, sin [n, hd / 2] or None."""
    if gain is not None:
        x = x * gain.double() / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    if cos is not None:
        a, b = x[..., :x.shape[-1] // 2], x[..., x.shape[-1] // 2:]
        c, s = cos.double()[:, None], sin.double()[:, None]
        x = torch.cat([a * c - b * s, b * c + a * s], -1)
    return x


def attention(cache, b, q, limits, scale, p_step, half_step):
    """q [n, nq, hd] of sequence b; limits [n] sets of visible positions as a bool [n, T].
    The output in float64, and how far a kernel may be off: p_step is the relative error of a
    rounded probability (0 bits less: fp32 sums), half_step that of the output's type."""
    n, nq, hd = q.shape
    T = limits.shape[1]
    k, v = cache.context(b, T)
    q = q.double()
    o, tol = torch.zeros((n, nq, hd), dtype=torch.float64), torch.zeros((n, nq, hd), dtype=torch.float64)
    g = nq // cache.nkv
    for h in range(nq):
        kh, vh = k[h // g], v[h // g]
        z = (q[:, h] @ kh.T) * scale
        z[~limits] = -math.inf
        m = z.max(-1, keepdim=True).values if T else torch.full((n, 1), -math.inf, dtype=torch.float64)
        w = torch.nan_to_num(torch.exp(z - m), nan=0.0)
        total = w.sum(-1, keepdim=True)
        w = w / torch.where(total > 0, total, torch.ones_like(total))
        o[:, h] = w @ vh
        # fp32 sums of hd products (and of the factors of the exponent, up to 4 roundings)
        dz = 2.0 ** -24 * ((hd + 8) * (q[:, h].abs() @ kh.abs().T) * scale)
        dz = torch.where(limits, dz, torch.zeros_like(dz)).max(-1, keepdim=True).values if T else torch.zeros_like(m)
        mass = w @ vh.abs()
        floor = T * 2.0 ** -30 * (vh.abs().max() if T else 0.0)
        tol[:, h] = half_step * o[:, h].abs() + (p_step + 2 * dz + 2.0 ** -18) * mass + floor
    return o, tol
