"""Plain 64-bit forms of the paged cache's calls, for its tests: a cache as tensors of values, the
4-bit format decoded from its bytes one nibble at a time, attention row by row.  Shares no code with
the library."""
import math

import torch

BF16, F32, INT4 = 0, 1, 2


def to_bf16(x):
    return x.to(torch.float32).to(torch.bfloat16)


def rotate(x, pos, inv_freq, interleaved):
    """x [tokens, heads, d] fp64, pos [tokens]: pair i turned by pos * inv_freq[i]."""
    y = x.clone()
    n = len(inv_freq)
    for i in range(n):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
        w = pos.double() * float(inv_freq[i])
        c, s = torch.cos(w)[:, None], torch.sin(w)[:, None]
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., a] * s + x[..., b] * c
    return y


def quantise(x):
    """x [..., d] fp64 -> codes (int64), scale and lowest (fp64, on the bf16 grid) [..., d / 32]."""
    g = x.unflatten(-1, (-1, 32))
    fine = torch.isfinite(g).all(-1)
    lo, hi = torch.where(fine, g.amin(-1), 0.0), torch.where(fine, g.amax(-1), 0.0)
    scale, low = to_bf16((hi - lo) / 15).double(), to_bf16(lo).double()
    t = (torch.nan_to_num(g, nan=0.0, posinf=0.0, neginf=0.0) - low[..., None]) / torch.where(scale == 0, 1.0, scale)[..., None]
    codes = torch.round(t).clamp(0, 15)
    codes = torch.where((scale == 0)[..., None] | ~fine[..., None], 0.0, codes)
    scale = torch.where(fine, scale, math.nan)
    low = torch.where(fine, low, 0.0)
    return codes.long(), scale, low, t


def int4_parts(pages, d, page_size):
    """uint8 [..., page bytes of a head] -> K and V as (codes [..., page, d], scale, lowest [..., page, d/32])."""
    g = d // 32
    raw = pages.reshape(*pages.shape[:-1], page_size // 16, -1).long()
    t, c = torch.arange(16, device=pages.device)[:, None], torch.arange(d, device=pages.device)[None]
    j, r = c // 32, c % 32
    gi = torch.arange(g, device=pages.device)[None]
    nib = lambda at: (raw[..., at] >> (4 * (r % 2))) & 15  # noqa: E731
    num = lambda at: ((raw[..., at] + 256 * raw[..., at + 1]) << 16).to(torch.int32).view(torch.float32).double()  # noqa: E731
    kc = nib(t * (d // 2) + ((r // 8) * g + j) * 4 + r % 8 // 2)
    vc = nib(8 * d + (t // 2) * d + ((r // 4) * g + j) * 4 + t % 2 * 2 + r % 4 // 2)
    pair = 16 * d + ((t // 2) * g + gi) * 4 + t % 2 * 2
    ks, vs, vl = num(pair), num(pair + 64 * g), num(pair + 96 * g)
    kl = num(16 * d + 32 * g + (t * g + gi) * 2)
    flat = lambda x: x.flatten(-3, -2)  # noqa: E731
    return tuple(map(flat, (kc, ks, kl))), tuple(map(flat, (vc, vs, vl)))


def int4_values(codes, scale, low):
    return (low[..., None] + scale[..., None] * codes.unflatten(-1, (-1, 32)).double()).flatten(-2)


def cache_values(pages, kind, layer, d, page_size):
    """One layer's pages as fp64 K, V [pages, kv_heads, page_size, d]."""
    p = pages[layer]
    if kind == INT4:
        k, v = int4_parts(p, d, page_size)
        return int4_values(*k), int4_values(*v)
    return p[:, 0].double(), p[:, 1].double()


def cache_sizes(pages, kind, layer, d, page_size):
    """What the kernels' products are made of, in size: |row|, and for 4 bits scale * code + |lowest|, whose two
    terms are multiplied and summed apart (a small value may be the difference of two large ones)."""
    if kind != INT4:
        return tuple(x.abs() for x in cache_values(pages, kind, layer, d, page_size))
    return tuple(int4_values(c, s, low.abs()) for c, s, low in int4_parts(pages[layer], d, page_size))


def rows_of(values, table_row, length, page_size):
    """[kv_heads, length, d] of one sequence."""
    n = -(-length // page_size)
    at = table_row[:n].long()
    return values[at].transpose(0, 1).flatten(1, 2)[:, :length]


def attend(q, K, V, first_pos, window=0, scale=0.0, sizes=None):
    """q [n, q_heads, d], K, V [kv_heads, length, d], fp64.  The query i stands at first_pos + i.
    Returns out, lse, and per row and channel what a bound on the error needs: the mean of |v| under the
    weights, and the largest sum of |q k| * scale, with `sizes` (cache_sizes) in the place of |k| and |v|."""
    KS, VS = (K.abs(), V.abs()) if sizes is None else sizes
    n, hq, d = q.shape
    hk, L = K.shape[:2]
    scale = scale or 1 / math.sqrt(d)
    out, mean_abs = torch.zeros_like(q), torch.zeros_like(q)
    lse = torch.full((n, hq), -math.inf, dtype=torch.float64, device=q.device)
    s_abs = torch.zeros(n, hq, dtype=torch.float64, device=q.device)
    for i in range(n):
        end = min(first_pos + i + 1, L)
        begin = max(0, first_pos + i + 1 - window) if window else 0
        if end <= begin:
            continue
        k, v = K[:, begin:end], V[:, begin:end]
        qi = q[i].reshape(hk, hq // hk, d)
        s = torch.einsum("hgd,hld->hgl", qi, k) * scale
        lse[i] = torch.logsumexp(s, -1).reshape(hq)
        p = torch.softmax(s, -1)
        out[i] = torch.einsum("hgl,hld->hgd", p, v).reshape(hq, d)
        mean_abs[i] = torch.einsum("hgl,hld->hgd", p, VS[:, begin:end]).reshape(hq, d)
        s_abs[i] = (torch.einsum("hgd,hld->hgl", qi.abs(), KS[:, begin:end]) * scale).amax(-1).reshape(hq)
    return out, lse, mean_abs, s_abs


# Errors of the kernels relative to exact arithmetic, each a bound:
#   out = sum p v / sum p.  A relative error e_p of every p and e_v of every v changes out by at most
#   (2 e_p + e_v) * mean|v|; p = exp(s) turns an absolute error of s into a relative one.  Over 4-bit pages
#   v = scale * code + lowest enters as two products whose weights are rounded apart: |v| is
#   scale * code + |lowest| there, and |k| in the sums of s likewise.
#   s is a sum of d products accumulated in 32 bits (d roundings of at most 2^-23 of sum|q k| each, the
#   matrix units may cut off instead of rounding), times constants (3 roundings), minus a maximum and
#   into ex2.approx (2^-22): d_s = s_abs * (d + 8) * 2^-23, e_p0 = 2 d_s + 2^-21.
#   The sums over tokens are kept in 32 bits: L roundings of 2^-23 at most, of partial sums below the
#   whole's |.|: L * 2^-23 (out and the sum of p both).
#   Roundings below 32 bits per path are added by the caller as e_p (weights), e_k and e_v (rows).
def out_bound(ref, mean_abs, s_abs, d, length, half_out, e_p=0.0, e_k=0.0, e_v=0.0):
    d_s = s_abs[..., None] * ((d + 8) * 2.0 ** -23 + e_k)
    e = 2 * (torch.expm1(d_s) + 2.0 ** -21 + e_p) + e_v + 2 * length * 2.0 ** -23
    return half_out * ref.abs() * (1 + e) + e * mean_abs * (1 + half_out) + 2.0 ** -100


def lse_bound(lse, s_abs, d, length, e_p=0.0, e_k=0.0):
    e = s_abs * ((d + 8) * 2.0 ** -23 + e_k) + 2.0 ** -20 + e_p + length * 2.0 ** -23
    return e + 4 * 2.0 ** -24 * lse.abs()
