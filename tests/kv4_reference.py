"""The 4-bit cache format and the attention over it, from their definitions in 64 bits (numpy), for the tests."""
import numpy as np

GROUP = 32


def _bf16(x, up):
    """float64 -> the bf16 value next to it, upwards or downwards (finite, or the infinity beyond the range)."""
    x = np.asarray(x, np.float64)
    f = x.astype(np.float32)
    # fp32 first, in the same direction
    wrong = (f.astype(np.float64) < x) if up else (f.astype(np.float64) > x)
    f = np.where(wrong, np.nextafter(f, np.float32(np.inf if up else -np.inf)), f)
    u = f.view(np.uint32)
    t = (u & np.uint32(0xFFFF0000)).view(np.float32)                 # towards zero
    away = (t != f) & ((f > 0) == up)
    t = np.where(away, (t.view(np.uint32) + np.uint32(0x10000)).view(np.float32), t)
    return t.astype(np.float64)


def quantise(x):
    """x [..., dh] -> (codes [..., dh], m and s [..., dh / 32]) as float64; m = s = nan for a group that has no finite form."""
    g = np.asarray(x, np.float64).reshape(x.shape[:-1] + (x.shape[-1] // GROUP, GROUP))
    with np.errstate(all="ignore"):
        finite = np.isfinite(g).all(-1)
        safe = np.where(finite[..., None], g, 0.0)
        m = _bf16(safe.min(-1), False)
        s = _bf16((safe.max(-1) - m) / 15.0, True)
        ok = finite & np.isfinite(m) & np.isfinite(s) & (np.abs((safe.max(-1) - m)) < 3.4028236e38)
        t = (safe - m[..., None]) / np.where(s > 0, s, 1.0)[..., None]
        n = np.where((s > 0)[..., None], np.clip(np.ceil(t - 0.5), 0, 15), 0.0)
    n = np.where(ok[..., None], n, 0.0)
    return n.reshape(x.shape), np.where(ok, m, np.nan), np.where(ok, s, np.nan)


def values(n, m, s):
    return (n.reshape(m.shape + (GROUP,)) * s[..., None] + m[..., None]).reshape(n.shape)


def visible(rows, n_q, mask, mask_rows):
    """[n_q, rows] truth values; mask [n_q, mask_rows] or None."""
    r = np.arange(rows)
    if mask is None:
        return r[None] <= rows - n_q + np.arange(n_q)[:, None]
    see = np.ones((n_q, rows), bool)
    first = rows - mask_rows
    for j in range(mask_rows):
        if first + j >= 0:
            see[:, first + j] = mask[:, j]
    return see


def attention(q, k, v, scale, see):
    """One sequence: q [n_q, Hq, dh]; k, v = (codes, m, s) of [rows, Hkv, .]; see [n_q, rows].  -> (out, bound) [n_q, Hq, dh];
    bound = sum of p (15 s + |m|) per channel (what the products of a softmax are made of), and the largest |score| [n_q, Hq]."""
    n_q, Hq, dh = q.shape
    q = q.astype(np.float64)
    Hkv = k[0].shape[1]
    out, bound, big = np.zeros((n_q, Hq, dh)), np.zeros((n_q, Hq, dh)), np.zeros((n_q, Hq))
    kv = values(*k)
    vv = values(*v)
    reach = np.repeat(15.0 * v[2] + np.abs(v[1]), GROUP, axis=-1)
    for h in range(Hq):
        hk = h // (Hq // Hkv)
        for i in range(n_q):
            w = np.flatnonzero(see[i])
            if not w.size:
                continue
            z = kv[w, hk] @ q[i, h] * scale
            p = np.exp(z - z.max())
            p /= p.sum()
            out[i, h] = p @ vv[w, hk]
            bound[i, h] = p @ reach[w, hk]
            big[i, h] = (np.abs(kv[w, hk]) @ np.abs(q[i, h]) * scale).max()
    return out, bound, big
