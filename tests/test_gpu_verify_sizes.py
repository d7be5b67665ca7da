"""pic_verify_draft at the sizes where its forms change: batches with narrow and wide
clusters, one and several chunks of a row a warp, all tokens at once and level by level.
The rule of test_gpu_verify in whole numbers, by cumulative sums (exact: no tolerance)."""
import numpy as np
import pytest
import torch

from tests.test_gpu_verify import run

pytestmark = pytest.mark.gpu


def draw(p, u):
    w = (np.clip(np.where(np.isnan(p), np.float32(0), p), 0, 1).astype(np.float64) * 2.0 ** 36).astype(np.int64)
    c = np.cumsum(w)
    total, n = int(c[-1]), int(np.float32(u) * np.float32(2 ** 24))
    return int(np.searchsorted(c, total * n >> 24, side="right")) if total else -1


def rule(tokens, n, p, u, q, parent):
    """p: a row of the target's by token; the path, its length and the next token."""
    T = len(tokens)
    if n == 0:
        return [-1] * T, 0, -1
    if q is not None:
        r = next((i for i in range(1, n) if not np.float32(u[i - 1]) * q[i - 1, tokens[i]] < p[i - 1, tokens[i]]), n)
        path = list(range(r))
        x = draw(p[r - 1] - q[r - 1], u[n - 1]) if r < n else -1
        x = draw(p[r - 1], u[n - 1]) if x < 0 else x
    else:
        path = [0]
        while True:
            x = draw(p[path[-1]], u[len(path) - 1])
            child = [c for c in range(path[-1] + 1, n) if parent[c] == path[-1] and tokens[c] == x]
            if not child:
                break
            path.append(child[0])
    return path + [-1] * (T - len(path)), len(path), x


def probs(rng, *shape):
    """Rows with most of their weight on a few entries, as a model's."""
    x = rng.standard_normal(shape, dtype=np.float32) * 2
    x[..., rng.integers(0, shape[-1], 4)] += 10
    e = np.exp(x - x.max(-1, keepdims=True))
    return e / e.sum(-1, keepdims=True)


def check(B, T, V, form, seed, cuda_lib):
    rng = np.random.default_rng(seed)
    p = probs(rng, B, T, V)
    u = rng.random((B, T), dtype=np.float32)
    lens = rng.integers(1, T + 1, B)
    lens[0], lens[B // 2] = T, 0 if B > 2 else T
    tokens, q, parent = np.zeros((B, T), np.int64), None, np.tile(np.arange(T) - 1, (B, 1))
    if form == "sampled":
        q = (probs(rng, B, T - 1, V) + 2 * p[:, :-1]) / np.float32(3)
        for b in range(B):
            for i in range(1, T):
                tokens[b, i] = max(0, draw(q[b, i - 1], rng.random(dtype=np.float32)))
    else:
        if form == "tree":
            parent = np.maximum(0, np.arange(T) - 1 - rng.integers(0, 3, (B, T)))
            parent[:, 0] = -1
        depth = np.zeros((B, T), np.int64)
        for b in range(B):
            for i in range(1, T):  # the target's own draw for two tokens of three
                depth[b, i] = depth[b, parent[b, i]] + 1
                tokens[b, i] = draw(p[b, parent[b, i]], u[b, depth[b, i] - 1]) if rng.random() < 0.67 \
                    else rng.integers(0, V)
    got = run(tokens, lens, p, u, q, parent if form == "tree" else None)
    refused = kept = 0
    for b in range(B):
        want = rule(tokens[b].tolist(), int(lens[b]), p[b], u[b], None if q is None else q[b], parent[b])
        assert (got[0][b], got[1][b], got[2][b]) == want, b
        refused += 0 < want[1] < lens[b]
        kept += want[1] > 1
    assert B < 12 or (kept > 0 and refused > 0)  # both endings are met
    assert cuda_lib.pic_device_status() == (0, 0)


@pytest.mark.parametrize("vocab", [1023, 1025, 50001, 131072, 151936])
@pytest.mark.parametrize("B", [13, 40, 64])
def test_sampled_chains_of_large_batches(cuda_lib, B, vocab):
    check(B, 4, vocab, "sampled", B + vocab, cuda_lib)


@pytest.mark.parametrize("vocab", [131071, 131072, 131073, 151936, 300007])
@pytest.mark.parametrize("B", [1, 5, 12])
def test_sampled_chains_of_small_batches(cuda_lib, B, vocab):
    """Sixteen CTAs a request, one chunk a warp and several."""
    check(B, 5 if B > 1 else 16, vocab, "sampled", B + vocab, cuda_lib)


@pytest.mark.parametrize("form", ["chain", "tree"])
@pytest.mark.parametrize("B,T,vocab", [(13, 13, 1025), (13, 13, 151936), (31, 5, 50001), (64, 3, 131072),
                                       (4, 16, 151936), (12, 8, 131073), (1, 64, 151936),  # wide, by levels
                                       (4, 8, 151936), (19, 8, 50001),                     # all tokens at once
                                       (2, 5, 151936), (1, 12, 300007)])                   # the same, wide
def test_trees(cuda_lib, B, T, vocab, form):
    check(B, T, vocab, form, B + T + vocab, cuda_lib)


@pytest.mark.parametrize("B", [1, 13])
def test_the_largest_vocabulary(cuda_lib, B):
    """2^24 entries, weights spread evenly with one missing at either end."""
    V = 1 << 24
    row = torch.full((V,), 2.0 ** -24, device="cuda")
    row[0] = row[-1] = 0
    u = np.linspace(0, 1 - 2.0 ** -24, B + 1, dtype=np.float32)[1:].reshape(B, 1)
    got = run([[0]] * B, [1] * B, row.expand(B, 1, V), u)
    c = np.arange(V - 2) + 1  # the running sum behind entry c, in units of 2^12
    for b in range(B):
        at = ((V - 2) << 12) * int(u[b, 0] * np.float32(2 ** 24)) >> 24
        assert got[2][b] == 1 + int(np.searchsorted(c << 12, at, side="right"))
    assert cuda_lib.pic_device_status() == (0, 0)
