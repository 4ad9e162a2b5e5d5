"""The paged 8-bit cache in plain 64-bit loops: what each call of ssba_cache_* is to give, from its
definition, for the tests. Nothing here is shared with the library."""
import math

import numpy as np
import torch

PAGE = 64
E4M3 = torch.float8_e4m3fn


def e4m3_values():
    """The value of each of the 256 bytes."""
    v = np.zeros(256)
    for b in range(256):
        s, e, m = b >> 7, (b >> 3) & 15, b & 7
        x = m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        v[b] = np.nan if (e, m) == (15, 7) else (-x if s else x)
    return v


VALUES = e4m3_values()
_GRID = VALUES[:127]  # 0 ... 448, ascending


def round_e4m3(x):
    """Nearest e4m3 value to each |x| <= 448, ties to the even byte; NaN stays."""
    a = np.abs(x)
    hi = np.clip(np.searchsorted(_GRID, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - _GRID[lo], _GRID[hi] - a
    near = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return np.where(np.isnan(x), np.nan, np.sign(x) * _GRID[near])


def scale_for(amax):
    if amax == 0:
        return 0.0
    k = math.ceil(math.log2(amax / 448)) + 2
    while 2.0 ** (k - 1) * 448 >= amax:
        k -= 1
    return 2.0 ** max(k, -126)


class Pool:
    """K, V as values of their bytes, in 64 bits; scales, means."""

    def __init__(self, K, V, k_scale, v_scale, k_mean):
        self.K, self.V = (VALUES[t.view(torch.uint8).cpu().numpy()] for t in (K, V))
        self.k_scale, self.v_scale, self.k_mean = (t.double().cpu().numpy().copy() for t in (k_scale, v_scale, k_mean))


def rows_of(lens, cu):
    for b, L in enumerate(lens):
        yield b, cu[b], cu[b + 1] - cu[b], L


def append(pool, k, v, table, lens, cu):
    """In place. k, v: 64-bit arrays [T, kv, d]."""
    for b, r, n, L in rows_of(lens, cu):
        n = min(n, table.shape[1] * PAGE - L)
        for j in range(L // PAGE, -(-(L + n) // PAGE) if n else 0):
            page = table[b][j]
            s0, s1 = max(L - j * PAGE, 0), min(L + n - j * PAGE, PAGE)
            if s0 >= s1:
                continue
            for x, buf, scales in ((k, pool.K, pool.k_scale), (v, pool.V, pool.v_scale)):
                for h in range(buf.shape[1]):
                    new = x[r + j * PAGE - L + s0:r + j * PAGE - L + s1, h]
                    new = np.where(np.isfinite(new), new, np.nan)
                    was = scales[page, h] if s0 else 0.0
                    s = max(was, scale_for(np.nanmax(np.abs(new), initial=0.0)))
                    if was < s:
                        buf[page, h, :s0] = round_e4m3(buf[page, h, :s0] * (was / s))
                    buf[page, h, s0:s1] = round_e4m3(new / (s or 1.0))
                    scales[page, h] = s
                    if buf is pool.K and s1 == PAGE:
                        pool.k_mean[page, h] = s * buf[page, h].sum(0) / PAGE


def select(pool, q, table, lens, cu, keep, first, T=None):
    T = q.shape[0]
    kv = pool.K.shape[1]
    G = q.shape[1] // kv
    idx = np.full((T, kv, keep), -1, dtype=np.int32)
    cnt = np.zeros((T, kv), dtype=np.int32)
    for b, r, n, L in rows_of(lens, cu):
        for i in range(n):
            P = -(-max(L - n + i + 1, 0) // PAGE)
            for h in range(kv):
                forced = [j for j in range(P) if j < first or j == P - 1]
                free = [j for j in range(P) if j not in forced]
                score = [max(float(q[r + i, h * G + g] @ pool.k_mean[table[b][j], h]) for g in range(G)) for j in free]
                key = [(-s if s == s else math.inf, j) for s, j in zip(score, free)]
                got = sorted(forced + [j for _, j in sorted(key)[:max(keep - len(forced), 0)]])[:keep]
                idx[r + i, h, :len(got)] = got
                cnt[r + i, h] = len(got)
    return idx, cnt


def attend(pool, q, table, lens, cu, scale, lists=None):
    """(O, lse, A, S): also A = sum of weight * |v| for each output, and S = the largest sum of |scale q k| of a row's
    scores, which bounds of rounding are made of."""
    T, H, d = q.shape
    kv = pool.K.shape[1]
    G = H // kv
    O, A = np.zeros((T, H, d)), np.zeros((T, H, d))
    lse, S = np.full((T, H), -np.inf), np.zeros((T, H))
    for b, r, n, L in rows_of(lens, cu):
        for i in range(n):
            see = max(L - n + i + 1, 0)
            for h in range(kv):
                js = range(-(-see // PAGE)) if lists is None else [j for j in lists[r + i, h] if 0 <= j < -(-see // PAGE)]
                if not len(js):
                    continue
                pg = [table[b][j] for j in js]
                K = np.concatenate([pool.K[p, h, :min(PAGE, see - j * PAGE)] * pool.k_scale[p, h] for p, j in zip(pg, js)])
                V = np.concatenate([pool.V[p, h, :min(PAGE, see - j * PAGE)] * pool.v_scale[p, h] for p, j in zip(pg, js)])
                x = q[r + i, h * G:(h + 1) * G]
                a = scale * x @ K.T
                m = a.max(1, keepdims=True)
                w = np.exp(a - m)
                z = w.sum(1, keepdims=True)
                w /= z
                O[r + i, h * G:(h + 1) * G] = w @ V
                A[r + i, h * G:(h + 1) * G] = w @ np.abs(V)
                lse[r + i, h * G:(h + 1) * G] = (m + np.log(z))[:, 0]
                S[r + i, h * G:(h + 1) * G] = (scale * np.abs(x) @ np.abs(K).T).max(1)
    return O, lse, A, S


def bounds(O, A, S, d, L, bf16):
    """How far (O, lse) may be off. A score is a sum of d exact products in fp32 and two more roundings: off by
    e = (d + 4) 2^-24 S at most, and a weight by twice that; weights and values are summed in fp32, L terms off by
    L 2^-24 at most and 16 more roundings on the way (exp2 is good to 2^-22). bf16 calls round each weight to 8 bits
    of significand, 2^-8, in front of V, and O once more."""
    e = (d + 4) * 2.0 ** -24 * S[..., None]
    rel = 2 * e + (2 * L + 16) * 2.0 ** -24 + 2.0 ** -20
    if bf16:
        return (rel + 2.0 ** -8) * A * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(O) + 1e-38, (e + (L + 64) * 2.0 ** -24)[..., 0]
    return rel * A + 2.0 ** -23 * np.abs(O) + 1e-38, (e + (L + 64) * 2.0 ** -24)[..., 0]
