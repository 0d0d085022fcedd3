"""Float64 NumPy definitions of the operators around the block: 4-bit frozen matrices, dropout from
counters, the LoRA linear on either, the router with its losses over padded batches.  Test
infrastructure only; no code is shared with the package."""
import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


# ---- 4-bit matrices ---------------------------------------------------------------------------

def group_scale(most):
    """Smallest number of six significant bits that is at least most / 6."""
    if not most < 2.0 ** 127:
        return np.nan
    if most < 2.0 ** -100:
        return 0.0
    m, e = np.frexp(most / 6.0)
    return float(np.ldexp(np.ceil(np.ldexp(m, 6)), e - 6))


def nearest_code(w, s):
    """Code (0-7, sign in bit 3) of the level nearest to w / s; a tie goes to the even code."""
    if not s > 0:
        return 0
    d = np.abs(abs(w) - LEVELS * s)
    best = np.flatnonzero(d == d.min())
    c = int(best[0]) if len(best) == 1 else int([b for b in best if b % 2 == 0][0])
    return c + 8 if w < 0 and c else c


def quantize(W, group):
    """codes [n, K] (0-15) and scales [n, groups]; nearest_code for all weights at once."""
    n, K = W.shape
    G = -(-K // group)
    W = W.astype(np.float64)
    padded = np.zeros((n, G * group))
    padded[:, :K] = W
    most = np.abs(padded).reshape(n, G, group).max(2)      # NaN where one is
    scales = np.array([group_scale(m) for m in most.reshape(-1)]).reshape(n, G)
    s = np.repeat(scales, group, axis=1)[:, :K]
    codes, off = np.zeros((n, K), np.uint8), np.full((n, K), np.inf)
    with np.errstate(invalid="ignore"):
        for c in (0, 2, 4, 6, 1, 3, 5, 7):                  # even codes first: a tie stays with them
            d = np.abs(np.abs(W) - LEVELS[c] * s)
            codes, off = np.where(d < off, c, codes).astype(np.uint8), np.minimum(d, off)
        codes[~(s > 0)] = 0
        return np.where((W < 0) & (codes > 0), codes + 8, codes).astype(np.uint8), scales


def values(codes, scales, group):
    v = LEVELS[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    return v * np.repeat(scales, group, axis=1)[:, :codes.shape[1]]


def pack(codes, scales, group):
    """The library's two arrays: bytes, and scales in tile order (float64)."""
    n, K = codes.shape
    nt, kt, per = -(-n // 16), -(-K // 128), 128 // group
    out, sc = np.zeros(nt * kt * 1024, np.uint8), np.zeros(nt * kt * 16 * per)
    i, k = np.arange(n)[:, None], np.arange(K)[None, :]
    b, h, e = k % 128 // 32, k % 32 // 8, k % 8
    at = (i // 16 * kt + k // 128) * 1024 + 16 * (16 * h + i % 16) + 4 * b + e // 2
    np.bitwise_or.at(out, at, codes << (4 * (e % 2)).astype(np.uint8))
    g = np.arange(scales.shape[1])[None, :]
    sc[((i // 16 * kt + g // per) * 16 + i % 16) * per + g % per] = scales
    return out, sc


# ---- dropout ------------------------------------------------------------------------------------

def philox(counter, key, rounds=7):
    """Philox4x32 of one counter (four words) and key (two), in Python integers."""
    c, k = list(counter), list(key)
    for _ in range(rounds):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def dropout_factors(T, width, p, seed, offset):
    """[T, width]: 0 where an element is dropped, else the factor it gets; philox for all blocks at once."""
    thr = int(np.floor(float(np.float32(p)) * 65536.0 + 0.5))
    u = np.uint64
    low, half = u(0xFFFFFFFF), u(32)
    t, c8 = np.meshgrid(np.arange(T, dtype=u), np.arange(-(-width // 8), dtype=u), indexing="ij")
    c = [c8, t, np.full_like(t, u(offset & 0xFFFFFFFF)), np.full_like(t, u(offset >> 32))]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(7):
        a, b = u(0xD2511F53) * c[0], u(0xCD9E8D57) * c[2]
        c = [(b >> half) ^ c[1] ^ u(k[0]), b & low, (a >> half) ^ c[3] ^ u(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    bits = np.stack([w >> u(16 * h) & u(0xFFFF) for w in c for h in (0, 1)], axis=2)
    return np.where(bits.reshape(T, -1)[:, :width] >= u(thr), 65536.0 / (65536.0 - thr), 0.0)


# ---- LoRA linear ----------------------------------------------------------------------------------

def _drop(v, factors):
    return v if factors is None else np.where(factors > 0, v * np.where(factors > 0, factors, 1.0), 0.0)


def linear(x, W, A, B, s, factors=None, dy=None):
    """y, and with dy the gradients; factors as from dropout_factors."""
    x, W, A, B = (np.asarray(v, np.float64) for v in (x, W, A, B))
    xd = _drop(x, factors)
    P = xd @ A.T
    out = {"y": x @ W.T + s * P @ B.T}
    if dy is not None:
        dy = np.asarray(dy, np.float64)
        V = dy @ B
        out["dx"] = dy @ W + _drop(s * V @ A, factors)
        out["dA"], out["dB"] = s * V.T @ xd, s * dy.T @ P
    return out


def linear_sums(x, W, A, B, s, factors=None, dy=None):
    """The same sums over magnitudes: what rounding errors are relative to."""
    x, W, A, B = (np.abs(np.asarray(v, np.float64)) for v in (x, W, A, B))
    return linear(x, W, A, B, abs(s), factors, None if dy is None else np.abs(np.asarray(dy, np.float64)))


# ---- router -----------------------------------------------------------------------------------------

def router(z, mask, k, mode, balance_coeff, z_coeff, d_w=None, d_balance=1.0, d_z=1.0):
    """Token by token; mask None = every token."""
    z = np.asarray(z, np.float64)
    T, N = z.shape
    on = [t for t in range(T) if mask is None or mask[t]]
    n = len(on)
    idx, w = np.full((T, k), -1, np.int32), np.zeros((T, k))
    p, lse = np.zeros((T, N)), np.zeros(T)
    counts, first = np.zeros(N, np.int64), np.zeros(N, np.int64)
    for t in on:
        key = np.where(np.isnan(z[t]), -np.inf, z[t])
        order = sorted(range(N), key=lambda i: (-key[i], i))[:k]
        top = z[t].max()
        with np.errstate(invalid="ignore"):
            ez = np.exp(z[t] - top)
            lse[t] = top + np.log(ez.sum())
            p[t] = ez / ez.sum()
        idx[t], w[t] = order, p[t, order] / p[t, order].sum()
        counts[order] += 1
        first[order[0]] += 1
    F = (first if mode == "top1" else counts / k) / max(n, 1)
    P = sum((p[t] for t in on), np.zeros(N)) / max(n, 1)
    balance = balance_coeff * N * float((F * P).sum())
    zl = z_coeff * sum(lse[t] ** 2 for t in on) / max(n, 1)
    out = dict(loss=np.array([balance + zl, balance, zl]), counts=counts, topk_idx=idx, topk_w=w)
    dz = np.zeros((T, N))
    for t in on:
        dz[t] = p[t] * (d_balance * balance_coeff * N / n * (F - (F * p[t]).sum()) + d_z * z_coeff * 2 / n * lse[t])
        if d_w is not None:
            dz[t, idx[t]] += w[t] * (d_w[t] - (w[t] * d_w[t]).sum())
    out["dlogits"] = dz
    return out
