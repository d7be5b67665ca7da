"""Plain references of the operators that decode branches together (numpy, 64 bits and whole
numbers), for the tests."""
import math

import numpy as np

TILE, PAGE, LEVELS = 128, 16, 4


def f64(t):
    return t.detach().double().cpu().numpy()


# ------------------------------------------------------------------- append
def theta_of(geom, layer):
    d = geom.head_dim
    if geom.layer_inv_freq is not None:
        return f64(geom.layer_inv_freq[layer])
    if geom.inv_freq is not None:
        return np.array(geom.inv_freq, np.float64)
    return geom.rope_base ** (-2.0 * np.arange(d // 2) / d)


def normed_rotated(x, weight, eps, pos, geom, layer):
    """(y, size) for one head x [d]: its value and the length of each element's pair."""
    y = x if weight is None else x / math.sqrt((x * x).mean() + eps) * weight
    d, a = len(x), pos * theta_of(geom, layer)
    c, s = np.cos(a), np.sin(a)
    out, size = np.empty(d), np.empty(d)
    u, w = (slice(0, d // 2), slice(d // 2, d)) if geom.rope_style == 0 else (slice(0, d, 2), slice(1, d, 2))
    out[u], out[w] = y[u] * c - y[w] * s, y[u] * s + y[w] * c
    size[u] = size[w] = np.hypot(y[u], y[w])
    return out, size


def append_close(got, ref, size):
    """One rounding to bf16 (2^-8 relative), and fp32's errors relative to the pair's length: a
    head's mean of squares (16 additions in a row and 3 across lanes: 19 2^-24, halved by the
    root), the root (2^-22), two products, the angle (2^-31 of a half turn and one rounding: pi
    2^-25), its cosine and sine (2^-22), three operations of the rotation: below 2^-19."""
    return np.abs(got - ref) <= np.abs(ref) * 2.0 ** -8 + size * 2.0 ** -19 + 2.0 ** -133


# --------------------------------------------------------------------- plan
def plan_nodes(rows, keys, table, num_pages):
    """The nodes [2 n][8] from their definition; keys[i] < 0: entry left alone (its row invalid)."""
    n = len(rows)
    nodes = np.tile(np.array([0, 0, 0, 0, -1, 0, -1, -1]), (2 * n, 1))
    c = [0] * (n + 1)  # c[i + 1]: of boundary i; c[0] = c[n] = 0
    for i in range(n - 1):
        if keys[i] < 0 or keys[i + 1] < 0:
            continue
        t, limit = 0, min(keys[i], keys[i + 1]) // TILE
        while t < limit:
            a = table[rows[i]][8 * t:8 * t + 8]
            b = table[rows[i + 1]][8 * t:8 * t + 8]
            if not ((a == b) & (a >= 0) & (a < num_pages)).all():
                break
            t += 1
        c[i + 1] = t
    run = {}   # a node by its (left, right) columns and count: those of its run

    def bounds(col):
        l = col
        while c[l] >= c[col]:
            l -= 1
        r = col
        while c[r] >= c[col]:
            r += 1
        return l, r

    def first(col):  # the run's first column of this count
        l, r = bounds(col)
        return next(k for k in range(l + 1, r) if c[k] == c[col])

    def above(col):
        l, r = bounds(col)
        up = l if c[l] >= c[r] else r
        return first(up) if c[up] > 0 else 0

    level = {}

    def level_of(col):
        if col not in level:
            up = above(col)
            level[col] = 0 if not up else level_of(up) + 1
        return level[col]

    kept = {col for col in range(1, n) if c[col] > 0 and first(col) == col and level_of(col) < LEVELS}
    for col in kept:
        l, r = bounds(col)
        up = above(col)
        nodes[n + col - 1] = [l, r, c[up] if up else 0, c[col], rows[l], c[col] * TILE,
                              n + up - 1 if up else -1, level[col]]
    for i in range(n):
        nodes[i] = [i, i + 1, 0, 0, -1, keys[i], -1, -1]
        if keys[i] < 0:
            nodes[i, 5] = -1
            continue
        col = i if c[i] >= c[i + 1] else i + 1
        up = first(col) if c[col] > 0 else 0
        while up and up not in kept:
            up = above(up)
        nodes[i] = [i, i + 1, c[up] if up else 0, -(-keys[i] // TILE), rows[i], keys[i],
                    n + up - 1 if up else -1, level[up] + 1 if up else 0]
    del run
    return nodes


# ---------------------------------------------------------------- attention
def attention(q, K, V):
    """(out, lse, A, S) of heads q [Hq][d] over K, V [n][Hkv][d]: A = sum w |v| (the scale of
    the rounding of the weights), S = the largest sum |q k| / sqrt(d)."""
    Hq, d = q.shape
    Hkv = K.shape[1]
    G = Hq // Hkv
    out, A, lse = np.zeros((Hq, d)), np.zeros((Hq, d)), np.full(Hq, -np.inf)
    if not len(K):
        return out, lse, A, 0.0
    S = 0.0
    for h in range(Hq):
        k, v = K[:, h // G], V[:, h // G]
        z = k @ q[h] / math.sqrt(d)
        S = max(S, float((np.abs(k) @ np.abs(q[h])).max()) / math.sqrt(d))
        m = z.max()
        w = np.exp(z - m)
        lse[h] = m + math.log(w.sum())
        w /= w.sum()
        out[h], A[h] = w @ v, w @ np.abs(v)
    return out, lse, A, S


def attention_close(got, lse, ref, S, A, lse_ref):
    """The weights are rounded to bf16 before their product with V (2^-8 each, so 2^-8 A), the
    output once more (2^-8).  A score's fp32 sum of d <= 128 products is off by at most 128
    2^-23 S (additions that cut instead of rounding), the exponential and its argument by 2^-20
    (S + 1): e = S 2^-15 + 2^-19 relative to a weight and absolute on the lse."""
    e = S * 2.0 ** -15 + 2.0 ** -19
    ok = np.abs(got - ref) <= np.abs(ref) * 2.0 ** -8 + A * (2.0 ** -8 + 2 * e) + 2.0 ** -130
    with np.errstate(invalid="ignore"):  # (-infinity from -infinity)
        same = (lse == lse_ref) | (np.abs(lse - lse_ref) <= e + np.abs(lse_ref) * 2.0 ** -22)
    return bool(ok.all()), bool(same.all())


# ----------------------------------------------------------------- sampling
C = [np.float32(x) for x in (0.6931470036506653, 0.24022242426872253, 0.05550733581185341,
                             0.009671512991189957, 0.001326472731307149)]


def weights(x, T):
    """Whole-number weights of the logits x (float32) at temperature T > 0."""
    f = np.float32
    with np.errstate(all="ignore"):
        x = np.where(np.isnan(x), f(-np.inf), x.astype(f))
        M = x.max()
        s = min(f(1.4426950408889634) / f(T), f(1e30))
        z = np.where(x == M, f(0), x - M) * s
        z = np.where(x == -np.inf, f(-np.inf), z)
        live = z >= f(-37)
        j = np.rint(np.where(live, z, f(0)))
        r = np.where(live, z, f(0)) - j
        p = C[4] * r + C[3]
        for c in (C[2], C[1], C[0], f(1)):
            p = p * r + c
        assert p.dtype == f
        m = (p.astype(np.float64) * 2.0 ** 24).astype(np.int64) << 12
        return x, np.where(live, m >> (-j).astype(np.int64), 0)


def share(total, u, top):
    u = np.float32(u)
    u = 0.0 if np.isnan(u) else float(min(max(u, np.float32(0)), np.float32(top)))
    return total * min(int(u * 2.0 ** 24), int(top * 2 ** 24)) >> 24


def sample(x, u, T=1.0, k=0, p=1.0, m=0.0):
    """(token, kept, logprob) of one row, by sorting."""
    greedy = not T > 0
    x, w = weights(np.asarray(x), 1.0 if greedy else T)
    if x.max() == -np.inf:
        return -1, 0, math.nan
    order = [i for i in np.lexsort((np.arange(len(x)), -x.astype(np.float64))) if w[i] > 0]
    if greedy:
        order = order[:1]
    if k > 0:
        order = order[:k]
    if p < 1.0:
        cut, run, end = share(sum(int(w[i]) for i in order), p, 1.0), 0, 0
        while end < len(order) and (run < cut or end == 0):
            run += int(w[order[end]])
            end += 1
        order = order[:end]
    least = int((0.0 if np.isnan(np.float32(m)) else float(min(max(np.float32(m), np.float32(0)), np.float32(1)))) * 2.0 ** 36)
    kept = sorted(i for i in order if w[i] >= least)
    S = sum(int(w[i]) for i in kept)
    at, run = share(S, u, 1.0 - 2.0 ** -24), 0
    for i in kept:
        run += int(w[i])
        if run > at:
            return i, len(kept), math.log(int(w[i]) / S)
    raise AssertionError("nothing drawn")
