"""pic_verify_draft against its rule in whole Python numbers (exact: no tolerance),
and the distribution it leaves."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def weights(p):
    p = np.where(np.isnan(p), np.float32(0), p)
    return [int(x) for x in np.clip(p, 0, 1).astype(np.float64) * 2.0 ** 36]


def draw(w, u):
    n = int(min(max(np.float32(0) if np.isnan(u) else np.float32(u) * np.float32(2 ** 24),
                    np.float32(0)), np.float32(2 ** 24 - 1)))
    s = sum(w)
    at, run = s * n >> 24, 0
    for x, v in enumerate(w):
        run += v
        if run > at:
            return x
    return -1


def rule(tokens, n, p, u, q=None, parent=None):
    T, V = len(tokens), p.shape[1]
    pad = lambda x: x + [-1] * (T - len(x))  # noqa: E731
    if n == 0:
        return pad([]), 0, -1
    if q is not None:
        r = n
        for i in range(1, n):
            x = tokens[i]
            with np.errstate(invalid="ignore"):
                if not (0 <= x < V and np.float32(u[i - 1]) * q[i - 1, x] < p[i - 1, x]):
                    r = i
                    break
        w = weights(p[r - 1])
        if r < n:
            with np.errstate(invalid="ignore"):
                rest = weights(p[r - 1] - q[r - 1])
            w = rest if sum(rest) else w
        return pad(list(range(r))), r, draw(w, u[n - 1])
    path = [0]
    while True:
        x = draw(weights(p[path[-1]]), u[len(path) - 1])
        par = [i - 1 for i in range(T)] if parent is None else parent
        child = [c for c in range(path[-1] + 1, n) if par[c] == path[-1] and tokens[c] == x and x >= 0]
        if not child:
            return pad(path), len(path), x
        path.append(child[0])


def run(tokens, lens, p, u, q=None, parent=None):
    import paper_2607_28069_gb300 as pic
    i32 = lambda x: torch.as_tensor(np.asarray(x), dtype=torch.int32).cuda()  # noqa: E731
    B, T = np.asarray(tokens).shape
    path, plen, nxt = (torch.full((B,) + s, 99, dtype=torch.int32, device="cuda")
                       for s in ((T,), (), ()))
    cu = lambda x: x if isinstance(x, torch.Tensor) or x is None else torch.as_tensor(x).cuda()  # noqa: E731
    pic.pic_verify_draft(i32(tokens), i32(lens), cu(p), cu(u), path, plen, nxt, draft_prob=cu(q),
                         parent=None if parent is None else i32(parent))
    return path.cpu().tolist(), plen.cpu().tolist(), nxt.cpu().tolist()


def probs(rng, *shape):
    x = rng.standard_normal(shape) * 3
    x[..., rng.integers(0, shape[-1], 3)] += 8
    e = np.exp(x - x.max(-1, keepdims=True))
    return (e / e.sum(-1, keepdims=True)).astype(np.float32)


@pytest.mark.parametrize("vocab", [1, 2, 31, 1023, 1024, 1025, 8193, 50001])
@pytest.mark.parametrize("form", ["sampled", "chain", "tree"])
def test_rule(cuda_lib, form, vocab):
    rng = np.random.default_rng(vocab)
    B, T = 7, 6 if vocab > 8193 else 40
    p = probs(rng, B, T, vocab)
    u = rng.random((B, T)).astype(np.float32)
    lens = [T, 1, 2, 0, T - 1, 3, T]
    q = parent = None
    if form == "sampled":
        q = probs(rng, B, T - 1, vocab)
        q = ((q + 3 * p[:, :-1]) / 4).astype(np.float32)
        tokens = np.zeros((B, T), np.int64)
        tokens[:, 1:] = (q / rng.exponential(size=q.shape)).argmax(-1)
    else:
        # tokens likely enough to be followed: the draw of another request's row
        parent = np.maximum(0, np.arange(T) - 1 - rng.integers(0, 3, (B, T)))
        parent[:, 0] = -1
        par = parent if form == "tree" else np.tile(np.arange(T) - 1, (B, 1))
        tokens = np.zeros((B, T), np.int64)
        for b in range(B):
            for i in range(1, T):
                tokens[b, i] = p[b, par[b, i]].argsort()[::-1][
                    min(vocab - 1, int((par[b, :i] == par[b, i]).sum()))]
        if form == "chain":
            parent = None
    got = run(tokens, lens, p, u, q, parent)
    for b in range(B):
        want = rule(tokens[b].tolist(), lens[b], p[b], u[b], None if q is None else q[b],
                    None if parent is None else parent[b].tolist())
        assert (got[0][b], got[1][b], got[2][b]) == want, b
    assert cuda_lib.pic_device_status() == (0, 0)


def test_odd_values_and_strides(cuda_lib):
    """NaN, negative, zero and overfull probabilities, numbers at the ends of
    [0, 1), tokens outside the vocabulary, rows with padding behind them."""
    rng = np.random.default_rng(5)
    B, T, V = 8, 4, 2050
    p, q = probs(rng, B, T, V), probs(rng, B, T - 1, V)
    u = rng.random((B, T)).astype(np.float32)
    tokens = rng.integers(0, V, (B, T))
    tokens[0, 1], tokens[1, 1] = V, -1
    p[2, :, ::3] = np.nan
    p[3] = 0
    q[4] = p[4, :-1]          # nothing left where refused
    p[5, :, :] *= 3
    p[5, :, 7] = -2
    u[6], u[7] = 0.0, np.float32(1 - 2 ** -24)
    u[5, T - 1] = 1.0
    u[4, 0] = np.nan          # never accepted
    wide_p = torch.full((B, T, V + 5), 9.0, device="cuda")
    wide_q = torch.full((T - 1, B, V + 3), 9.0, device="cuda").transpose(0, 1)
    wide_p[..., :V] = torch.as_tensor(p).cuda()
    wide_q[..., :V] = torch.as_tensor(q).cuda()
    lens = [T] * B
    for qq in (None, q):
        got = run(tokens, lens, wide_p[..., :V], u, None if qq is None else wide_q[..., :V])
        for b in range(B):
            want = rule(tokens[b].tolist(), T, p[b], u[b], None if qq is None else q[b])
            assert (got[0][b], got[1][b], got[2][b]) == want, (b, qq is None)
    assert cuda_lib.pic_device_status() == (0, 0)


def test_a_bad_length_is_reported(cuda_lib):
    p, u = np.ones((2, 2, 4), np.float32) / 4, np.zeros((2, 2), np.float32)
    got = run([[0, 0], [0, 0]], [3, 1], p, u)
    assert got == ([[-1, -1], [0, -1]], [0, 1], [-1, 0])
    assert cuda_lib.pic_device_status() == (3, 0)


def test_kept_tokens_have_the_targets_distribution(cuda_lib):
    """40000 requests with one draft each from the same q against the same p: the
    token in the draft's place (kept, or the one drawn instead) is distributed as p,
    within five standard deviations per entry."""
    rng = np.random.default_rng(11)
    N, V = 40000, 6
    p1 = np.array([0.4, 0.05, 0.25, 0.0, 0.2, 0.1], np.float32)
    q1 = np.array([0.1, 0.3, 0.2, 0.2, 0.15, 0.05], np.float32)
    tokens = np.zeros((N, 2), np.int64)
    tokens[:, 1] = rng.choice(V, N, p=q1 / q1.sum(dtype=np.float64))
    p = np.tile(p1, (N, 2, 1))
    u = rng.random((N, 2)).astype(np.float32)
    for q in (np.tile(q1, (N, 1, 1)), None):
        path, plen, nxt = run(tokens, [2] * N, p, u, q)
        got = np.where(np.array(plen) == 2, tokens[:, 1], np.array(nxt))
        share = np.bincount(got, minlength=V) / N
        assert np.all(np.abs(share - p1) <= 5 * np.sqrt(p1 * (1 - p1) / N) + 1e-9), share


def test_refusals(cuda_lib):
    import paper_2607_28069_gb300 as pic
    p, u = torch.ones((1, 2, 4), device="cuda"), torch.zeros((1, 2), device="cuda")
    with pytest.raises(ValueError, match="three dimensions"):
        run([[0, 0]], [2], p[0], u)
    with pytest.raises(ValueError, match="contiguous in its last"):
        run([[0, 0]], [2], p.transpose(1, 2).expand(1, 4, 2)[:, :2, :], u)
    with pytest.raises(ValueError, match="draft_prob must be"):
        run([[0, 0]], [2], p, u, q=p)
    with pytest.raises(ValueError, match="needs a chain"):
        run([[0, 0]], [2], p, u, q=p[:, :1], parent=[[-1, 0]])
    with pytest.raises(ValueError, match="must be torch.float32"):
        run([[0, 0]], [2], p.double(), u)
    with pytest.raises(pic.PicError, match="max_draft 65"):
        run([[0] * 65], [2], torch.ones((1, 65, 4), device="cuda"), torch.zeros((1, 65), device="cuda"))


@pytest.mark.parametrize("B", [1, 2, 5])  # 64 and 128 draws at once, 320 level by level
@pytest.mark.parametrize("tree", [False, True])
def test_deep_trees_in_both_forms(cuda_lib, B, tree):
    """Lines of up to 64 accepted tokens, branches, tokens that hang on none or on one that
    is not below them, a row without weight, and lengths that are refused."""
    rng = np.random.default_rng(10 * B + tree)
    T, V = 64, 1500
    p = probs(rng, B, T, V)
    u = rng.random((B, T)).astype(np.float32)
    parent = np.tile(np.arange(T) - 1, (B, 1))
    if tree:
        parent[:, 5::5] -= 1  # every fifth token is a leaf, the line goes on beside it
        parent[:, 44], parent[:, 49], parent[:, 54] = 44, -1, 99
    lens = [T, T - 7, 0, -1, T][:B]
    tokens = rng.integers(0, V, (B, T))
    for b in range(B):  # every token is the target's own draw behind its parent
        depth = [0] * T
        for i in range(1, T):
            if 0 <= parent[b, i] < i:
                depth[i] = depth[parent[b, i]] + 1
                tokens[b, i] = draw(weights(p[b, parent[b, i]]), u[b, depth[i] - 1])
                if tree and i % 5 == 4 and i < 59:
                    tokens[b, i] = (tokens[b, i] + 1) % V  # a leaf that is not taken
        p[b, T - 10 + b] = 0
    got = run(tokens, lens, p, u, None, parent if tree else None)
    seen = 0
    for b in range(B):
        n = lens[b] if 0 <= lens[b] <= T else 0
        want = rule(tokens[b].tolist(), n, p[b], u[b], None, parent[b].tolist() if tree else None)
        assert (got[0][b], got[1][b], got[2][b]) == want, b
        seen = max(seen, want[1])
    assert seen > (40 if tree else 50)
    assert cuda_lib.pic_device_status() == ((3, 3) if B == 5 else (0, 0))
