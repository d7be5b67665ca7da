"""pic_sample against its rule in whole numbers: every filter and mixes of them, ties, infinities,
odd settings, rows of any start and stride."""
import math

import numpy as np
import pytest
import torch

from tests import branch_reference as R

pytestmark = pytest.mark.gpu
NAN, INF = math.nan, math.inf


def f32(x):
    return torch.tensor(np.asarray(x, np.float32), device="cuda")


def run(pic, logits, u, T=None, k=None, p=None, m=None):
    B = logits.shape[0]
    token = torch.full((B,), 77, dtype=torch.int32, device="cuda")
    kept = torch.full((B,), 77, dtype=torch.int32, device="cuda")
    lp = torch.full((B,), 77.0, device="cuda")
    opt = lambda x: None if x is None else f32(x)  # noqa: E731
    pic.pic_sample(logits, f32(u), token, temperature=opt(T),
                   top_k=None if k is None else torch.tensor(k, dtype=torch.int32, device="cuda"),
                   top_p=opt(p), min_p=opt(m), logprob=lp, kept=kept)
    torch.cuda.synchronize()
    return token.tolist(), kept.tolist(), lp.tolist()


def check(pic, logits, u, T=None, k=None, p=None, m=None):
    token, kept, lp = run(pic, logits, u, T, k, p, m)
    x = logits.float().cpu().numpy()
    assert pic.pic_device_status() == (0, 0)
    at = lambda a, b, d: d if a is None else a[b]  # noqa: E731
    for b in range(len(x)):
        want = R.sample(x[b], u[b], at(T, b, 1.0), at(k, b, 0), at(p, b, 1.0), at(m, b, 0.0))
        got = (token[b], kept[b])
        assert got == want[:2], (b, got, want, at(T, b, 1), at(k, b, 0), at(p, b, 1), at(m, b, 0))
        if math.isnan(want[2]):
            assert math.isnan(lp[b])
        else:  # the ratio (2 roundings), the logarithm (2 ulps), of both near 0
            assert abs(lp[b] - want[2]) <= 2.0 ** -22 + abs(want[2]) * 2.0 ** -22


def settings(rng, B):
    pick = lambda a, b, prob: np.where(rng.random(B) < prob, a, b)  # noqa: E731
    T = pick(rng.uniform(0.3, 2.5, B), 1.0, 0.8)
    T = pick(0.0, T, 0.1)
    k = pick(np.exp(rng.uniform(0, 9, B)).astype(int), 0, 0.5).astype(int)
    p = pick(rng.uniform(0, 1, B), 1.0, 0.6)
    m = pick(rng.uniform(0, 0.1, B), 0.0, 0.4)
    return [float(np.float32(x)) for x in T], k.tolist(), [float(np.float32(x)) for x in p], [float(np.float32(x)) for x in m]


@pytest.mark.parametrize("V", [1, 2, 31, 255, 256, 257, 1000, 4097, 12345, 50001, 131072])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_random_rows_and_settings(cuda_lib, V, dtype):
    rng = np.random.default_rng(V)
    B = 10 if V < 20000 else 4
    x = torch.tensor(rng.normal(0, 3, (B, V)), device="cuda").to(dtype)
    u = rng.random(B).astype(np.float32)
    check(cuda_lib, x, u)
    check(cuda_lib, x, u, *settings(rng, B))
    check(cuda_lib, x, u, p=[0.9] * B)
    check(cuda_lib, x, u, k=[1 + b * V // B for b in range(B)])


@pytest.mark.parametrize("B", [1, 12, 13, 39, 70, 161])
def test_batches(cuda_lib, B):
    rng = np.random.default_rng(B)
    x = torch.tensor(rng.normal(0, 2.5, (B, 3001)), device="cuda").float()
    check(cuda_lib, x, rng.random(B).astype(np.float32), *settings(rng, B))


@pytest.mark.parametrize("B", [15, 17, 21])
def test_batches_of_rows_in_more_parts_than_eight(cuda_lib, B):
    rng = np.random.default_rng(B)
    x = torch.tensor(rng.normal(0, 2.5, (B, 50021)), device="cuda").bfloat16()
    check(cuda_lib, x, rng.random(B).astype(np.float32), *settings(rng, B))


def test_long_rows_beyond_shared_memory(cuda_lib):
    """Parts of a row that are read again from memory; a row of 2^24 entries."""
    rng = np.random.default_rng(1)
    x = torch.tensor(rng.normal(0, 2, (20, 400001)), device="cuda").float()
    u = rng.random(20).astype(np.float32)
    T, k, p, m = settings(rng, 20)
    token, kept, lp = run(cuda_lib, x, u, T, k, p, m)
    for b in range(0, 20, 7):
        want = R.sample(x[b].cpu().numpy(), u[b], T[b], k[b], p[b], m[b])
        assert (token[b], kept[b]) == want[:2]
    V = 1 << 24
    x = torch.zeros((1, V), device="cuda")
    for p, want in ((1.0, (1 << 24) // 4), (0.5, (1 << 23) // 4)):
        token, kept, lp = run(cuda_lib, x, [0.25], p=[p])  # equal weights: the count is the place
        assert token == [want] and kept == [int(V * p)] and abs(lp[0] + math.log(V * p)) < 1e-5
    token, kept, _ = run(cuda_lib, x, [0.5], k=[3_000_001])
    assert token == [1_500_000] and kept == [3_000_001]


@pytest.mark.parametrize("V", [300, 5000, 40000, 131072])
def test_ties(cuda_lib, V):
    """Few different logits (hundreds of equal ones at the border), and a crowd of close ones."""
    rng = np.random.default_rng(V)
    B = 6
    u = rng.random(B).astype(np.float32)
    few = torch.tensor(rng.integers(-3, 4, (B, V)), device="cuda").float()
    close = torch.tensor(2.0 + 1e-4 * rng.random((B, V)), device="cuda").float()
    zeros = torch.where(torch.tensor(rng.random((B, V)) < 0.5, device="cuda"), 0.0, -0.0)
    for x in (few, close, zeros, torch.cat([few[:, :V // 2], close[:, V // 2:]], 1)):
        check(cuda_lib, x, u, k=[1, 2, V // 3, V // 2, V - 1, V])
        check(cuda_lib, x, u, p=[0.0, 0.1, 0.5, 0.77, 0.999, 1.0])
        check(cuda_lib, x, u, *settings(rng, B))


def test_infinities_and_nan(cuda_lib):
    rng = np.random.default_rng(0)
    x = rng.normal(0, 2, (9, 3000)).astype(np.float32)
    x[0, 5:] = -INF
    x[1, :] = -INF
    x[2, ::3] = NAN
    x[3, 7], x[3, 2000], x[3, 2999] = INF, INF, NAN
    x[4, :] = NAN
    x[5, 17] = INF
    x[6, :] = INF
    x[7, :] = 3.0e38
    x[7, 9] = -3.0e38
    x[8, :] = -3.4e38
    t = torch.tensor(x, device="cuda")
    u = [0.0, 0.3, 0.5, 0.6, 0.7, 0.8, 0.9, 0.999, 1.0]
    check(cuda_lib, t, u)
    check(cuda_lib, t, u, T=[0.7] * 9, k=[2] * 9)
    check(cuda_lib, t, u, T=[2.0] * 9, p=[0.6] * 9)
    check(cuda_lib, t, u, T=[0.0] * 9, p=[0.6] * 9, m=[0.5] * 9)
    check(cuda_lib, t, u, k=[700] * 9, p=[0.4] * 9, m=[1.0] * 9)


def test_odd_settings(cuda_lib):
    rng = np.random.default_rng(4)
    x = torch.tensor(rng.normal(0, 2, (1, 2500)), device="cuda").float()
    for T in (0.0, -1.0, NAN, INF, 1e-30, 1e-45, 1e30, 0.02):
        for u in (0.0, 0.5, 1.0, 7.0, -3.0, NAN):
            check(cuda_lib, x, [u], T=[T])
    for k in (-5, 0, 1, 2500, 2499, 10 ** 9):
        check(cuda_lib, x, [0.4], k=[k], T=[1.7])
    for p in (-1.0, 0.0, 1e-9, 0.99999, 1.0, 2.0, INF):
        check(cuda_lib, x, [0.9], p=[p], T=[1.7])
    for m in (-1.0, NAN, 0.0, 1e-12, 0.3, 1.0, 5.0):
        check(cuda_lib, x, [0.9], m=[m], T=[3.0])
    assert run(cuda_lib, x, [0.5], p=[NAN]) == run(cuda_lib, x, [0.5])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_of_any_start_and_stride(cuda_lib, dtype):
    rng = np.random.default_rng(9)
    big = torch.tensor(rng.normal(0, 2, (7, 2111)), device="cuda").to(dtype)
    for lo, hi in ((0, 2111), (1, 2000), (3, 1027), (5, 6), (7, 263)):
        x = big[1::2, lo:hi]
        big_before = big.clone()
        check(cuda_lib, x, [0.1, 0.5, 0.9], T=[0.8, 1.0, 1.2], p=[0.7, 0.9, 1.0], k=[0, 40, 3])
        assert torch.equal(big, big_before)
    check(cuda_lib, big[2, :900].expand(4, 900), [0.1, 0.3, 0.6, 0.9], p=[0.8] * 4)  # one row four times
    check(cuda_lib, big[:1, 3:1500], [0.4], p=[0.8])


def test_two_calls_at_once_a_graph_and_no_extras(cuda_lib):
    pic = cuda_lib
    rng = np.random.default_rng(2)
    x = [torch.tensor(rng.normal(0, 2, (16, 30000)), device="cuda").float() for _ in range(2)]
    u = f32(rng.random(16))
    p = f32([0.9] * 16)
    want = []
    for y in x:
        t = torch.zeros(16, dtype=torch.int32, device="cuda")
        pic.pic_sample(y, u, t, top_p=p)
        want.append(t)
    streams = [torch.cuda.Stream() for _ in x]
    torch.cuda.synchronize()
    got = [torch.zeros_like(t) for t in want]
    for _ in range(10):
        for y, s, t in zip(x, streams, got):
            with torch.cuda.stream(s):
                pic.pic_sample(y, u, t, top_p=p)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    g = torch.cuda.CUDAGraph()
    t = torch.zeros(16, dtype=torch.int32, device="cuda")
    with torch.cuda.graph(g):
        pic.pic_sample(x[0], u, t, top_p=p)
    y = x[0].clone()
    x[0].copy_(x[1])
    g.replay()
    assert torch.equal(t, want[1])
    x[0].copy_(y)
    g.replay()
    assert torch.equal(t, want[0]) and pic.pic_device_status() == (0, 0)


def test_draws_follow_the_kept_distribution(cuda_lib):
    """Numbers spread evenly over [0, 1): each kept entry is drawn as often as its weight says."""
    n = 4096
    x = torch.tensor([[2.0, 0.0, 1.0, -1.0, 1.0, -30.0]], device="cuda").expand(n, 6)
    u = (np.arange(n) + 0.5) / n
    token, kept, lp = run(cuda_lib, x, u, p=[0.95] * n)
    assert set(kept) == {4}
    w = np.exp([2.0, 0.0, 1.0, -INF, 1.0, -INF])
    share = np.bincount(token, minlength=6) / n
    assert np.abs(share - w / w.sum()).max() <= 1.5 / n
    assert all(abs(a - math.log(w[t] / w.sum())) < 1e-5 for a, t in zip(lp, token))
