"""The 4-bit cache, its attention, accumulated weights and eviction from their definitions, in 64 bits, one loop at a time."""
import math

import numpy as np
import torch

# E2M1: code -> magnitude
GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def half_step(dtype):
    """A rounding to this type is off by at most this share of the value."""
    return torch.finfo(dtype).eps / 2


def pack_row(x):
    """x [D] (64 bits) -> codes [D] 0 .. 15, scale bytes [D / 32]."""
    codes, scales = [], []
    for g in np.asarray(x, dtype=np.float64).reshape(-1, 32):
        if not np.isfinite(g).all():
            codes += [0] * 32        # (what they are says nothing)
            scales.append(255)
            continue
        top = np.abs(g).max()
        e = -124
        while e < 125 and top > 7 * 2.0 ** e:
            e += 1
        scales.append(e + 127)
        for v in g:
            y = abs(v) / 2.0 ** e
            d = np.abs(GRID - y)
            best = np.flatnonzero(d == d.min())
            code = int(best[0] if len(best) == 1 or best[0] % 2 == 0 else best[1])   # ties: the even code
            codes.append(code | (8 if math.copysign(1.0, v) < 0 else 0))
    return np.array(codes), np.array(scales)


def unpack(codes, scales):
    """uint8 codes [.., D / 2] and scales [.., D / 32] -> values [.., D] in 64 bits (NaN where the scale is 255)."""
    codes, scales = np.asarray(codes), np.asarray(scales).astype(np.int64)
    n = np.stack((codes & 15, codes >> 4), -1).reshape(codes.shape[:-1] + (-1,)).astype(np.int64)
    v = GRID[n & 7] * np.where(n & 8, -1.0, 1.0)
    e = np.where(scales == 255, np.nan, 2.0 ** (scales - 127.0))
    return v * np.repeat(e, 32, -1)


def attention(q, k, v, kd, vd, parent, n_key, tokens):
    """One KV head of one sequence: q [Mq, G, D], k / v [T, D], kd / vd [M, D], tokens: the attended ones (repeats count).
    -> out [Mq, G, D], lse [Mq, G], the sums of weight * |value|, and sum |q k| / sqrt(D) at its largest per row."""
    Mq, G, D = q.shape
    K, V = k[tokens], v[tokens]
    out, lse, size, reach = np.zeros(q.shape), np.zeros((Mq, G)), np.zeros(q.shape), np.zeros((Mq, G))
    for r in range(Mq):
        path, at = [], r + n_key
        while at >= 0:
            path.append(at)
            at = int(parent[at])
        KK, VV = np.concatenate((K, kd[path])), np.concatenate((V, vd[path]))
        for h in range(G):
            z = KK @ q[r, h] / math.sqrt(D)
            top = z.max()
            p = np.exp(z - top)
            lse[r, h] = top + math.log(p.sum())
            p /= p.sum()
            out[r, h], size[r, h] = p @ VV, p @ np.abs(VV)
            reach[r, h] = (np.abs(KK) @ np.abs(q[r, h])).max() / math.sqrt(D)
    return out, lse, size, reach


def score_error(reach, D):
    """How far a score of fp32 sums over D products may be off, as a share of the weight: each of the sums rounds at most
    D times (2^-24 of at most the sum of magnitudes), the scaling and the exponential a few times more."""
    return reach * (D + 16) * 2.0 ** -24 + 2.0 ** -20


def listed_tokens(L, B, idx=None, cnt=None):
    if idx is None:
        return np.arange(L)
    nb = -(-L // B)
    t = [np.arange(i * B, min((i + 1) * B, L)) for i in np.asarray(idx)[:max(0, int(cnt))] if 0 <= i < nb]
    return np.concatenate(t) if t else np.zeros((0,), dtype=np.int64)


def weights_of(q, k, lse, rows, tokens, T):
    """q [Mq, G, D], lse [Mq, G], rows: those that count (repeats too) -> [T] sums, and the sums of weight * sum |q k| / sqrt(D)."""
    w, off = np.zeros((T,)), np.zeros((T,))
    D = q.shape[2]
    for r in rows:
        for h in range(q.shape[1]):
            if np.isinf(lse[r, h]):      # (a row that attended nothing gives nothing; one of infinite sum weighs nothing)
                continue
            p = np.exp(k[tokens] @ q[r, h] / math.sqrt(D) - lse[r, h])
            reach = np.abs(k[tokens]) @ np.abs(q[r, h]) / math.sqrt(D)
            np.add.at(w, tokens, p)
            np.add.at(off, tokens, p * (score_error(reach, D) + 3 * abs(lse[r, h]) * 2.0 ** -24))
    return w, off


def kept_tokens(w, L, ns, nr, k):
    if L <= ns + nr + k:
        return list(range(L))
    key = lambda t: (math.inf if math.isnan(w[t]) else -w[t] if w[t] != -math.inf else math.inf, math.isnan(w[t]), t)  # noqa: E731
    mid = sorted(range(ns, L - nr), key=key)[:k]
    return list(range(ns)) + sorted(mid) + list(range(L - nr, L))


def cache(sp, batch, Hkv, T, D, B, dtype, layout="bhtd", gap=0, seed=0, lens=None, size=1.0):
    """A packed cache of random rows: the handle, and its values [batch, Hkv, T, D] in 64 bits.  gap: unused rows between heads."""
    gen = np.random.default_rng(seed)
    x = [gen.standard_normal((batch, Hkv, T, D)) * size for _ in "kv"]
    codes, vals = [], []
    for y in x:
        c = gen.integers(0, 256, (batch, Hkv, T, D // 2), dtype=np.uint8)
        s = gen.integers(124, 129, (batch, Hkv, T, D // 32), dtype=np.uint8)
        codes += [c, s]
        vals.append(unpack(c, s) * 1.0)
    lens = [T] * batch if lens is None else lens

    def device(a):
        t = torch.from_numpy(a)
        if layout == "bthd":
            t = t.permute(0, 2, 1, 3)
        t = t.contiguous().cuda()
        if gap:
            big = torch.full((t.shape[0], t.shape[1], t.shape[2] + gap, t.shape[3]), 255, dtype=torch.uint8, device="cuda")
            big[:, :, :t.shape[2]] = t
            t = big[:, :, :t.shape[2]]
        return t
    k, ks, v, vs = (device(a) for a in codes)
    h = sp.PackedKV(k, v, ks, vs, torch.tensor(lens, dtype=torch.int32, device="cuda"), B, layout=layout, dtype=dtype)
    return h, vals[0], vals[1]
