"""Plain forms, in 64 bits on the CPU, of attention over packed prompts, of its
gradient and of the rotation by several axes, with the bounds of the errors that
32-bit sums and one rounding of each weight may make."""
import math

import numpy as np
import torch

from paged_reference import DTYPES, half_step, tolerance  # noqa: F401

E32 = 2.0 ** -24
LOG2E = math.log2(math.e)


def spans(start, B, most, total):
    """(first, number) of each sequence's rows, as the header defines them."""
    if start is None:
        return [(b * most, most) for b in range(B)]
    out = []
    for b in range(B):
        s = min(max(int(start[b]), 0), total)
        e = min(max(int(start[b + 1]), s), total)
        out.append((s, min(e - s, most)))
    return out


class Batch:
    """The sequences' rows and keys, and what each row sees."""

    def __init__(self, rows, keys, row_start=None, key_start=None, T=0, N=0, B=1, causal=True):
        self.rows, self.keys, self.causal = rows, keys, causal
        self.q = spans(row_start, B, T, rows)
        self.k = spans(key_start, B, N, keys)

    def __iter__(self):
        """(rows' slice, keys' slice, seen [t][n])"""
        for (s, t), (ks, n) in zip(self.q, self.k):
            r, l = np.arange(t)[:, None], np.arange(n)[None, :]
            seen = l <= r + n - t if self.causal else np.ones((t, n), bool)
            yield slice(s, s + t), slice(ks, ks + n), seen

    def mine(self, which):
        x = np.zeros(self.rows if which == "q" else self.keys, bool)
        for s, n in (self.q if which == "q" else self.k):
            x[s:s + n] = True
        return x


def scores(q, k, seen, scale):
    """scale q.k and the sum of its terms' magnitudes, -infinity where not seen."""
    with np.errstate(invalid="ignore", over="ignore"):
        s = (q @ k.T) * scale if scale else np.zeros((len(q), len(k)))
        size = abs(scale) * (np.abs(q) @ np.abs(k).T)
    return np.where(seen, s, -np.inf), np.where(seen, size, 0.0)


def attention(q, k, v, scale, batch):
    """(out, lse, mass, spread, seen_n, largest |v|) in float64; mass and spread as
    paged_reference.tolerance takes them."""
    q, k, v = (x.double().cpu().numpy() for x in (q, k, v))
    N, h_q, d = q.shape
    G = h_q // k.shape[1]
    out, mass = np.zeros((N, h_q, d)), np.zeros((N, h_q, d))
    lse, spread = np.full((N, h_q), -np.inf), np.zeros((N, h_q))
    seen_n, top_v = np.zeros(N, np.int64), 0.0
    for rows, keys, seen in batch:
        seen_n[rows] = seen.sum(1)
        if not seen.any():
            continue
        for h in range(h_q):
            kh, vh = k[keys, h // G], v[keys, h // G]
            s, size = scores(q[rows, h], kh, seen, scale)
            with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
                m = s.max(1, keepdims=True)
                m = np.where(m == -np.inf, 0.0, m)
                w = np.exp(s - m)
                z = w.sum(1, keepdims=True)
                for r in range(len(w)):
                    if z[r, 0] == 0:
                        continue
                    on = seen[r]
                    out[rows.start + r, h] = (w[r, on] @ vh[on]) / z[r, 0]
                    mass[rows.start + r, h] = (w[r, on] @ np.abs(vh[on])) / z[r, 0]
                lse[rows, h] = (m + np.log(z))[:, 0]
            spread[rows, h] = size.max(1) if size.shape[1] else 0.0
        vals = np.abs(v[keys])
        top_v = max(top_v, np.nanmax(np.where(np.isinf(vals), np.nan, vals), initial=0.0))
    return out, lse, mass, spread, seen_n, top_v


def lse_tolerance(lse, spread, seen_n, d):
    """A score's error (as in paged_reference.tolerance), the sum's, and the
    logarithm's, product's and result's roundings."""
    scores_ = 2 * (d + 16) * E32 * (spread + 1) * LOG2E
    sums = (seen_n[:, None] / 16 + 64) * 2 * E32
    return 1.01 * (scores_ + sums + 8 * E32 * (np.abs(lse) + spread + 1))


def gradient(q, k, v, out, lse, g, scale, batch, exact=False):
    """(dq, dk, dv, their bounds' parts) in float64, from the out and lse that are
    given, or (exact) from the weights themselves.

    Bounds, before the result's rounding.  A weight P = exp(s - lse): the score's
    error, and lse's and its product's roundings.  dP and delta: sums of d products
    in 32 bits.  dS = P (dP - delta): these, two roundings, and one to the type (u),
    which P has too.  Sums over keys or rows in 32 bits.  With `exact`, out is off by
    half a step of its type and the weights' roundings (3 u in all of |g||out|'s sum
    with |v| weighted in out's place), lse by its own bound."""
    dtype = q.dtype
    u = 0.0 if dtype == torch.float32 else half_step(dtype)
    q, k, v, out, g = (x.double().cpu().numpy() for x in (q, k, v, out, g))
    lse = lse.double().cpu().numpy()
    N, h_q, d = q.shape
    G = h_q // k.shape[1]
    dq, dk, dv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    bq, bk, bv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    tiny = 2.0 ** -25 if dtype == torch.float16 else 0.0
    with np.errstate(invalid="ignore", over="ignore"):
        for rows, keys, seen in batch:
            t, n = seen.shape
            sums = (max(n, t * G) / 16 + 64) * 2 * E32
            for h in range(h_q):
                kh, vh = k[keys, h // G], v[keys, h // G]
                qh, gh = q[rows, h] if scale else 0 * q[rows, h], g[rows, h]
                s, size = scores(qh, kh, seen, scale)
                L = lse[rows, h][:, None]
                p = np.where(seen & (L > -np.inf) | np.isnan(L) & seen,
                             np.exp(s - np.where(L == -np.inf, 0, L)), 0.0)
                oh = out[rows, h]
                dp = np.where(seen, gh @ vh.T, 0.0)
                if np.isnan(dp).any() or not np.isfinite(vh).all():
                    dp = np.zeros((t, n))
                    for r, l in zip(*np.nonzero(seen)):
                        dp[r, l] = gh[r] @ vh[l]
                delta = (gh * oh).sum(1, keepdims=True)
                ds = np.where(seen, p * (dp - delta), 0.0)
                terms = np.abs(gh) @ np.abs(vh).T + (np.abs(gh) * np.abs(oh)).sum(1)[:, None]
                e_p = 2 * (d + 16) * E32 * (size + 1) * LOG2E + 8 * E32 * (np.abs(L) + 1)
                e_d = 2 * (d + 16) * E32 * terms
                if exact:
                    row = size.max(1, keepdims=True) if n else 0.0
                    e_p = e_p + lse_tolerance(L, row, np.full(t, n), d)
                    e_d = e_d + 4 * u * (np.abs(gh) @ (p @ np.abs(vh)).T).diagonal()[:, None] \
                        + 8 * sums * terms
                a_p = p * (u + e_p + sums) + tiny
                a_s = p * (np.abs(dp - delta) * (u + e_p + sums + 4 * E32) + e_d) + tiny
                a_p, a_s = np.where(seen, a_p, 0.0), np.where(seen, a_s, 0.0)

                def add(x, w, y, to, bound, a):
                    """x += w y over pairs that are seen; a's and the sums' bound."""
                    fine = np.isfinite(y).all() and np.isfinite(w).all()
                    if fine:
                        x += w @ y
                    else:
                        for i in range(w.shape[0]):
                            on = to[i]
                            x[i] += w[i, on] @ y[on]
                    bound += a @ np.abs(np.where(np.isfinite(y), y, 0.0))

                add(dv[keys, h // G], p.T, gh, seen.T, bv[keys, h // G], a_p.T)
                add(dk[keys, h // G], scale * ds.T, qh, seen.T, bk[keys, h // G],
                    abs(scale) * (a_s + sums * np.abs(ds)).T)
                add(dq[rows, h], scale * ds, kh, seen, bq[rows, h],
                    abs(scale) * (a_s + sums * np.abs(ds)))
    low = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134, torch.float32: 2.0 ** -126}[dtype]

    def rounded(x, b):
        b = 1.01 * b
        return b + (np.abs(x) + b) * (half_step(dtype) + 2 * E32) + low

    return (dq, dk, dv), (rounded(dq, bq), rounded(dk, bk), rounded(dv, bv))


def rotate(x, positions, table, sections, interleaved, inverse):
    """x [rows][heads][d] turned, in float64; and the bound of the error: two
    products and a sum in 32 bits, and one rounding to the type."""
    dtype = x.dtype
    x = x.double().cpu().numpy()
    table, positions = table.double().cpu().numpy(), positions.cpu().numpy()
    half = table.shape[1] // 2
    y, size = x.copy(), np.abs(x)
    i = 0
    for axis, n in enumerate(sections):
        for i in range(i, i + n):
            pos = positions[axis].astype(np.int64)
            held = (pos >= 0) & (pos < len(table))
            at = np.where(held, pos, 0)
            c = np.where(held, table[at, i], 1.0)[:, None]
            s = np.where(held, table[at, half + i], 0.0)[:, None] * (-1 if inverse else 1)
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
            y[..., a] = x[..., a] * c - x[..., b] * s
            y[..., b] = x[..., b] * c + x[..., a] * s
            both = np.abs(x[..., a] * c) + np.abs(x[..., b] * s)
            cross = np.abs(x[..., b] * c) + np.abs(x[..., a] * s)
            size[..., a], size[..., b] = both, cross
        i = sum(sections[:axis + 1])
    t = 3 * E32 * size
    # A result below the type's normal numbers is rounded to a whole number of its
    # smallest ones: float16, 2^-24 (1 * 2^-14 in steps of 2^-10), so half a step is
    # 2^-25 whatever the result; bfloat16 and float32 may be 0 below 2^-126.
    low = 2.0 ** -25 if dtype == torch.float16 else 2.0 ** -126
    return y, t + (np.abs(y) + t) * half_step(dtype) + low
