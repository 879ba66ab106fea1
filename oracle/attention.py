"""Attention inside groups of rows, its gradient and rotary positions in float64, from their formulas, group by group and head by
head, with a bound on what rounding may cost a correct implementation.  Not used by the GPU path."""
import numpy as np

#: half a step of each storage type relative to the value, and the smallest step that counts
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 2.0 ** -126, "bf16": 2.0 ** -126, "f16": 2.0 ** -24}
U32 = 2.0 ** -24


def groups(perm, offsets, num_groups, n, G):
    """Row numbers of every group: positions offsets[g] .. min(offsets[g+1], offsets[g]+G)-1, cut to 0..n-1, without positions
    whose row there is none of."""
    out = []
    for g in range(max(0, num_groups)):
        a, b = (min(max(int(o), 0), n) for o in offsets[g:g + 2])
        p = np.arange(a, max(a, min(b, a + G)))
        r = p if perm is None else np.asarray(perm)[p]
        out.append(r[(r >= 0) & (r < n)].astype(np.int64))
    return out


def attention(q, k, v, qg, kg, scale, mask=None, dtype="f32"):
    """q [nq, H, D], k and v [nk, K, D] -> out, lse, bound of out, bound of lse; NaN in rows of no group.
    Bounds: a score is a sum of D products and a multiplication, (D + 2) U32 scale sum |q k| off at most; p is off by the
    exponential of twice that and some 2^-22 for the exponential, the sum over L rows and the division; p enters the product rounded
    to the type, once; the result is stored in the type."""
    (nq, H, D), K = q.shape, k.shape[1]
    u, tiny = HALF_STEP[dtype], TINY[dtype]
    out, bound = np.full((nq, H, D), np.nan), np.zeros((nq, H, D))
    lse, lse_bound = np.full((nq, H), np.nan), np.zeros((nq, H))
    for rq, rk in zip(qg, kg):
        rk = rk if mask is None else rk[np.asarray(mask)[rk] != 0]
        for h in range(H):
            kh = h // (H // K)
            if not len(rk):
                out[rq, h], lse[rq, h] = 0.0, -np.inf
                continue
            a, b, c = q[rq, h], k[rk, kh], v[rk, kh]
            s = scale * (a @ b.T)
            off = ((D + 2) * U32 * abs(scale) * (np.abs(a) @ np.abs(b).T)).max(1, keepdims=True)
            off = off + 4 * U32 * np.abs(s).max(1, keepdims=True)      # the scores as multiples of ln 2, and their differences
            top = s.max(1, keepdims=True)
            p = np.exp(s - top)
            total = p.sum(1, keepdims=True)
            p = p / total
            o = p @ c
            out[rq, h], lse[rq, h] = o, (top + np.log(total))[:, 0]
            rel = 2 * off + (len(rk) + 16) * U32
            bound[rq, h] = (u + rel) * (p @ np.abs(c)) + tiny * np.abs(c).sum(0) + u * np.abs(o) + tiny
            lse_bound[rq, h] = (off + (len(rk) + 16) * U32 + 4 * U32 * np.abs(lse[rq, h])[:, None])[:, 0]
    return out, lse, bound, lse_bound


def attention_backward(q, k, v, dout, qg, kg, scale, mask=None, dtype="f32"):
    """(dq, dk, dv) and their bounds, NaN in rows of no group.  Bounds: those of p as above, once more for lse; out as stored enters
    delta; p and e = p (dp - delta) are each rounded to the type before their products."""
    (nq, H, D), (nk, K, _) = q.shape, k.shape
    u, tiny = HALF_STEP[dtype], TINY[dtype]
    dq, bq = np.full((nq, H, D), np.nan), np.zeros((nq, H, D))
    (dk, dv), (bk, bv) = (np.full((nk, K, D), np.nan) for _ in range(2)), (np.zeros((nk, K, D)) for _ in range(2))
    out, lse, out_bound, lse_bound = attention(q, k, v, qg, kg, scale, mask, dtype)
    for rq, rk in zip(qg, kg):
        dk[rk], dv[rk] = 0.0, 0.0
        rk = rk if mask is None else rk[np.asarray(mask)[rk] != 0]
        for h in range(H):
            kh = h // (H // K)
            if not len(rk) or not len(rq):
                dq[rq, h] = 0.0
                continue
            a, b, c, g = q[rq, h], k[rk, kh], v[rk, kh], dout[rq, h]
            s = scale * (a @ b.T)
            p = np.exp(s - lse[rq, h][:, None])
            dp, dp_abs = g @ c.T, np.abs(g) @ np.abs(c).T
            delta = (g * out[rq, h]).sum(1, keepdims=True)
            e = p * (dp - delta)
            off = ((D + 2) * U32 * abs(scale) * (np.abs(a) @ np.abs(b).T)).max(1, keepdims=True) + 4 * U32 * np.abs(s).max(1, keepdims=True)
            rel = 2 * (off + lse_bound[rq, h][:, None] + 8 * U32)
            # float32's exponential ends at its smallest normal number: p is off by 2^-126 beside its relative error, and e = p (dp - delta)
            # by that times |dp - delta| <= sum |g v| + |delta|
            e_off = 2.0 ** -126 * (dp_abs + np.abs(delta)) + p * ((D + 2) * U32 * (dp_abs + (np.abs(g) * np.abs(out[rq, h])).sum(1, keepdims=True)) +
                         (np.abs(g) * out_bound[rq, h]).sum(1, keepdims=True))
            e_bound = (u + rel) * (np.abs(e) + e_off) + e_off + tiny
            p_bound = (u + rel) * p + tiny
            sums = (len(rq) * (H // K) + len(rk) + 16) * U32
            grads = (scale * e @ b, scale * e.T @ a, p.T @ g)
            bounds = (abs(scale) * (e_bound + sums * np.abs(e)) @ np.abs(b), abs(scale) * (e_bound + sums * np.abs(e)).T @ np.abs(a),
                      (p_bound + sums * p).T @ np.abs(g))
            dq[rq, h], bq[rq, h] = grads[0], bounds[0]
            dk[rk, kh] += grads[1]
            dv[rk, kh] += grads[2]
            bk[rk, kh] += bounds[1]
            bv[rk, kh] += bounds[2]
    return (dq, dk, dv), tuple(b + u * np.abs(x) + tiny for b, x in ((bq, dq), (bk, dk), (bv, dv)))


def rotary(x, positions, freqs, half, amplitude=1.0, inverse=False):
    """x [n, H, D] with the pairs of each position column turned by positions[n, axes] x freqs[axes, pairs]."""
    axes, pairs = freqs.shape
    y = np.array(x, dtype=np.float64)
    for c in range(axes):
        for i in range(pairs):
            ia = 2 * pairs * c + (i if half else 2 * i)
            ib = ia + (pairs if half else 1)
            t = positions[:, c].astype(np.float64) * freqs[c, i] * (-1.0 if inverse else 1.0)
            cs, sn = amplitude * np.cos(t)[:, None], amplitude * np.sin(t)[:, None]
            y[..., ia] = x[..., ia] * cs - x[..., ib] * sn
            y[..., ib] = x[..., ia] * sn + x[..., ib] * cs
    return y
