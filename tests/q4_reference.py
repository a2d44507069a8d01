"""The 4-bit cache by its definition, in 64 bits: numpy, one step after the other."""
import numpy as np

LIMIT = 65504.0


def _half_toward_zero(v):
    """The largest fp16 that is not above v (v >= 0)"""
    h = v.astype(np.float16)
    above = h.astype(np.float64) > v
    h[above] = np.nextafter(h[above], np.float16(0))
    return h


def quantise(x, group):
    """x [..., n, d] -> codes uint8 [..., n, d / 2], params fp16 [..., d / group, n, 2]"""
    x = np.asarray(x, dtype=np.float64)
    g = x.reshape(x.shape[:-1] + (-1, group))
    bad = ~np.isfinite(g).all(axis=-1)
    g = np.clip(np.where(bad[..., None], 0.0, g), -LIMIT, LIMIT)
    m = g.min(axis=-1).astype(np.float16)
    span = np.maximum(g.max(axis=-1) - m.astype(np.float64), 0.0)
    s = (span / 15).astype(np.float16)
    over = 15 * s.astype(np.float64) > span          # 15 s and the span are exact: toward zero
    s[over] = np.nextafter(s[over], np.float16(0))
    with np.errstate(divide="ignore", invalid="ignore"):
        c = np.rint((g - m.astype(np.float64)[..., None]) / s.astype(np.float64)[..., None])   # halves to even
    c = np.clip(np.where((s > 0)[..., None], c, 0), 0, 15).astype(np.uint8)
    s[bad], m[bad] = np.float16("nan"), np.float16("nan")
    c = c.reshape(x.shape)
    return c[..., 0::2] | (c[..., 1::2] << 4), np.moveaxis(np.stack([s, m], axis=-1), -2, -3).copy()


def values(codes, params):
    """fp16 [..., n, d]"""
    n, d = codes.shape[-2], 2 * codes.shape[-1]
    c = np.empty(codes.shape[:-1] + (d,))
    c[..., 0::2], c[..., 1::2] = codes & 15, codes >> 4
    sm = np.moveaxis(params.astype(np.float64), -3, -2)                       # [..., n, groups, 2]
    s, m = (np.repeat(sm[..., k], d // sm.shape[-2], axis=-1) for k in (0, 1))
    with np.errstate(over="ignore", invalid="ignore"):
        return (s * c + m).astype(np.float16)


def attention(q, k, v, seq_lens, q_lens, scale, causal):
    """q [B, Hq, Tq, d], k and v [B, Hkv, T, d] in 64 bits -> the output, sum_t p_t |v_t| and the largest sum_c |q_c k_c| (what the
    tolerances of a kernel's roundings are multiples of)"""
    q, k, v = (np.asarray(t, dtype=np.float64) for t in (q, k, v))
    B, Hq, Tq, d = q.shape
    out, spread, size = np.zeros_like(q), np.zeros_like(q), np.zeros(q.shape[:3])
    share = Hq // k.shape[1]
    for b in range(B):
        n, qn = int(seq_lens[b]), int(q_lens[b])
        for h in range(Hq):
            kk, vv = k[b, h // share], v[b, h // share]
            for i in range(qn):
                e = min(n, n - qn + i + 1) if causal else n
                if e <= 0:
                    continue
                s = scale * (kk[:e] @ q[b, h, i])
                p = np.exp(s - s.max())
                p /= p.sum()
                out[b, h, i], spread[b, h, i] = p @ vv[:e], p @ np.abs(vv[:e])
                size[b, h, i] = (np.abs(kk[:e]) @ np.abs(q[b, h, i])).max() * scale
    return out, spread, size
