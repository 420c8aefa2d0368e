"""Plain 64-bit forms of the paged cache's operators, on the CPU (numpy), and
the makers of their inputs.  Test infrastructure only; shares no code with the
library."""
import math

import numpy as np
import torch

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
LEVELS = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], np.float64)


def half_step(dtype):
    """The largest relative error of one rounding to the type."""
    return torch.finfo(dtype).eps / 2


# --- the 4-bit form ------------------------------------------------------------

def quantise(x):
    """(codes [.., d], scale bytes [.., d/32]) of float64 rows: the nearest level by
    comparing distances, ties to the even code."""
    x = np.asarray(x, np.float64)
    blocks = x.reshape(*x.shape[:-1], -1, 32)
    top = np.abs(blocks).max(-1)
    finite = np.isfinite(blocks).all(-1)
    with np.errstate(divide="ignore", invalid="ignore"):
        X = np.floor(np.log2(np.where((top > 0) & finite, top, 1.0))) - 2
    # log2 of the largest double below a power of two rounds up to it
    X = np.where((top > 0) & (top < 2.0 ** (X + 2)), X - 1, X)
    X = np.maximum(np.where(top > 0, X, -126), -126)
    y = np.abs(np.where(finite[..., None], blocks, 0.0)) / 2.0 ** X[..., None]
    dist = np.abs(y[..., None] - LEVELS)
    best = dist.min(-1, keepdims=True)
    at = dist == best
    first = at.argmax(-1)
    last = 7 - at[..., ::-1].argmax(-1)
    code = np.where(first % 2 == 0, first, last)
    code = code + 8 * np.signbit(blocks)
    code = np.where(finite[..., None], code, 7)
    scale = np.where(finite, X + 127, 255)
    return code.reshape(x.shape).astype(np.uint8), scale.astype(np.uint8)


def values(codes, scales):
    """What codes [.., d] and scale bytes [.., d/32] stand for."""
    m = LEVELS[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return m * np.repeat(s, 32, -1)


def pack_page(codes, scales, value):
    """Bytes of one head's page: codes [P][d], scales [P][d/32]."""
    P, d = codes.shape
    packed = codes[:, 0::2] | codes[:, 1::2] << 4
    if value:
        packed = packed.reshape(P // 8, 8, d // 8, 4).transpose(0, 2, 1, 3)
        scales = scales.reshape(P // 8, 8, d // 32).transpose(0, 2, 1)
    return np.concatenate((packed.reshape(-1), scales.reshape(-1))).astype(np.uint8)


def unpack_page(block, P, d, value):
    """(codes [P][d], scales [P][d/32]) of one head's page."""
    packed, scales = block[:P * d // 2], block[P * d // 2:]
    if value:
        packed = packed.reshape(P // 8, d // 8, 8, 4).transpose(0, 2, 1, 3)
        scales = scales.reshape(P // 8, d // 32, 8).transpose(0, 2, 1)
    packed = packed.reshape(P, d // 2)
    codes = np.stack((packed & 15, packed >> 4), -1).reshape(P, d)
    return codes, scales.reshape(P, d // 32)


def page_rows(pool, page, head, d, value):
    """float64 rows [P][d] of one head's page of a pool (a CPU tensor)."""
    P = pool.shape[2]
    if pool.dtype != torch.uint8:
        return pool[page, head].double().numpy()
    return values(*unpack_page(pool[page, head].reshape(-1).numpy(), P, d, value))


# --- the operators --------------------------------------------------------------

def seq_rows(row_start, B, T, rows):
    """(first row, number of rows) of each sequence."""
    if row_start is None:
        return [(b * T, T) for b in range(B)]
    out = []
    for b in range(B):
        s = min(max(int(row_start[b]), 0), rows)
        e = min(max(int(row_start[b + 1]), s), rows)
        out.append((s, min(e - s, T)))
    return out


def turn(x, pos, table, interleaved):
    """x [heads][d] float64 turned by the angles of position pos."""
    half = table.shape[1] // 2
    y = x.copy()
    c, s = table[pos, :half], table[pos, half:]
    a = slice(0, 2 * half, 2) if interleaved else slice(0, half)
    b = slice(1, 2 * half, 2) if interleaved else slice(half, 2 * half)
    y[:, a] = x[:, a] * c - x[:, b] * s
    y[:, b] = x[:, b] * c + x[:, a] * s
    return y


def place(pages, past, b, r, P, n_pages):
    """(position, page or None, slot) of a row; position None: dropped."""
    cap = pages.shape[1] * P
    p = int(past[b])
    if p < 0 or p + r >= cap:
        return None, None, None
    page = int(pages[b, (p + r) // P])
    return p + r, page if 0 <= page < n_pages else None, (p + r) % P


def attention(q, K, V, pages, past, scale, causal, row_start, T, h_kv):
    """(out, bound) in float64: bound[n,h,:] is the sum of weights times |v| and
    spread[n,h] the sum of |q k| scale that the largest score is made of; rows of
    no sequence are None in `mine`."""
    N, h_q, d = q.shape
    B, P = pages.shape[0], K.shape[2]
    G, cap = h_q // h_kv, pages.shape[1] * K.shape[2]
    qd = q.double().numpy()
    out = np.zeros((N, h_q, d))
    mass = np.zeros((N, h_q, d))
    spread = np.zeros((N, h_q))
    seen_n = np.zeros(N, np.int64)
    mine = np.zeros(N, bool)
    top_v = 0.0
    for b, (start, n) in enumerate(seq_rows(row_start, B, T, N)):
        p = int(past[b])
        last = 0 if p < 0 else min(cap, p + n if causal else p)
        ids = [int(x) for x in pages[b, :-(-last // P)]]
        ok = np.repeat([0 <= x < K.shape[0] for x in ids], P)[:last] if ids else np.zeros(0, bool)
        for h in range(h_kv):
            if ids:
                k = np.concatenate([page_rows(K, x if 0 <= x < K.shape[0] else 0, h, d, False)
                                    for x in ids])[:last]
                v = np.concatenate([page_rows(V, x if 0 <= x < K.shape[0] else 0, h, d, True)
                                    for x in ids])[:last]
            for r in range(n):
                mine[start + r] = True
                seen = 0 if p < 0 else min(cap, p + r + 1) if causal else min(cap, p)
                keep = np.flatnonzero(ok[:seen])
                seen_n[start + r] = len(keep)
                if not len(keep):
                    continue
                ks, vs = k[keep], v[keep]
                x = qd[start + r, h * G:(h + 1) * G]
                with np.errstate(invalid="ignore", over="ignore"):
                    s = scale * (x @ ks.T)
                    m = s.max(1, keepdims=True)
                    m = np.where(m == -np.inf, 0.0, m)
                    w = np.exp(s - m)
                    z = w.sum(1, keepdims=True)
                    o = np.where(z == 0, 0.0, (w @ vs) / np.where(z == 0, 1.0, z))
                    rows = slice(h * G, (h + 1) * G)
                    out[start + r, rows] = o
                    mass[start + r, rows] = (w @ np.abs(vs)) / np.where(z == 0, 1.0, z)
                    spread[start + r, rows] = abs(scale) * (np.abs(x) @ np.abs(ks).T).max(1)
                    top_v = max(top_v, np.abs(vs).max())
    return out, mass, spread, seen_n, mine, top_v


def tolerance(out, mass, spread, seen, top_v, dtype, d):
    """Bound of the error of every output.  Weights: a 16-bit type rounds each to
    half a step u, which the sum that divides them repeats: 2 u of the weights'
    share of |v|.  Scores: sums of d products in 32 bits, each at most spread, then
    the scaling, the subtraction of the reference and the exponential (a few
    roundings of numbers of the scores' size): an error e of a score is one of e
    of its weight, twice with the divisor's.  Sums over keys in 32 bits: chains
    of seen/16 products (the matrix instructions add 4 to 32 at a time, in an
    order of their own) and the merges.  float16 weights below 2^-14 of the
    reference lose up to 2^-25 each (the largest weight is 1 or more).  Then one
    rounding of the result."""
    e32 = 2.0 ** -24
    u = 0.0 if dtype == torch.float32 else half_step(dtype)
    scores = 2 * (d + 16) * e32 * (spread[..., None] + 1) * math.log2(math.e)
    sums = (seen[:, None, None] / 16 + 64) * 2 * e32
    tiny = 2.0 ** -25 * seen[:, None, None] * top_v if dtype == torch.float16 else 0.0
    t = mass * (2 * u + scores + sums) + tiny
    t = t * 1.01
    low = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134, torch.float32: 2.0 ** -150}
    return t + (np.abs(out) + t) * half_step(dtype) + low[dtype]


# --- inputs ---------------------------------------------------------------------

class Cache:
    """Pools and a page table on the CPU, every place that no sequence holds
    poisoned (NaN; scale byte 255), and the page table's unused entries wild."""

    def __init__(self, seed, dtype, fmt, d, h_kv, P, held, wide=None, spare=3):
        rng = np.random.default_rng(seed)
        self.P, self.d, self.h_kv, self.fmt = P, d, h_kv, fmt
        need = [-(-max(n, 0) // P) for n in held]
        total = sum(need) + spare
        order = rng.permutation(total)
        wide = wide or max(max(need), 1)
        self.pages = np.where(rng.random((len(held), wide)) < 0.5, -1, 2 ** 30).astype(np.int32)
        at = 0
        for b, n in enumerate(need):
            self.pages[b, :n] = order[at:at + n]
            at += n
        t = DTYPES[dtype]
        if fmt == "dense":
            self.K = torch.full((total, h_kv, P, d), math.nan, dtype=t)
            self.V = torch.full((total, h_kv, P, d), math.nan, dtype=t)
        else:
            self.K = torch.full((total, h_kv, P, d // 2 + d // 32), 255, dtype=torch.uint8)
            self.V = torch.full((total, h_kv, P, d // 2 + d // 32), 255, dtype=torch.uint8)
        for b, n in enumerate(held):
            for i in range(need[b]):
                rows = min(P, n - i * P)
                for h in range(h_kv):
                    for pool, value in ((self.K, False), (self.V, True)):
                        x = rng.standard_normal((rows, d))
                        page = int(self.pages[b, i])
                        if fmt == "dense":
                            pool[page, h, :rows] = torch.from_numpy(x).to(t)
                        else:
                            c, s = quantise(x)
                            full_c = np.full((P, d), 7, np.uint8)
                            full_s = np.full((P, d // 32), 255, np.uint8)
                            full_c[:rows], full_s[:rows] = c, s
                            pool[page, h] = torch.from_numpy(
                                pack_page(full_c, full_s, value)).reshape(P, -1)
        self.pages = torch.from_numpy(self.pages)

    def to(self, device):
        return self.K.to(device), self.V.to(device), self.pages.to(device)
