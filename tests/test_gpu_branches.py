"""BranchDecoder: steps over linked contexts and their forks, as a serving loop runs them, with
norms, against a plain model that keeps every row's keys and values in a list."""
import numpy as np
import pytest
import torch

from tests import branch_reference as R
from tests.test_gpu_speculative import contexts, linked

pytestmark = pytest.mark.gpu
HQ, HKV, D = 8, 2, 64


def bf(x):
    return R.f64(torch.as_tensor(np.asarray(x)).to(torch.bfloat16))


def step_inputs(g, layers, n, vocab):
    x = torch.randn((layers, n, 1, HQ + 2 * HKV, D), generator=g, device="cuda").bfloat16()
    logits = 3 * torch.randn((n, vocab), generator=g, device="cuda")
    return x.split([HQ, HKV, HKV], dim=3), logits, torch.rand(n, generator=g, device="cuda")


def run(dec, layers, qkv, logits, u, p):
    dec.begin()
    for layer in range(layers):
        dec.attend(layer, *[(x, layer) for x in qkv])
    dec.sample(logits, u, temperature=torch.full_like(u, 0.8), top_p=torch.full_like(u, p))


def test_steps_forks_and_releases(cuda_lib):
    from paper_2607_28069_gb300.pipeline import BranchDecoder
    L, V = 2, 901
    wl, path = linked(L, spare=60)
    g = torch.Generator(device="cuda").manual_seed(1)
    wq, wk = (1 + torch.randn(D, generator=g, device="cuda") / 4 for _ in range(2))
    wq, wk = wq.bfloat16(), wk.bfloat16()
    dec = BranchDecoder(path, rows=7, max_new=64, q_weight=wq, k_weight=wk)
    geom, rows = dec.geom, contexts(wl) + [None] * 5
    # (the prefill's keys, as the cache holds them)
    for b in range(2):
        at = np.arange(int(dec.ctx_len[b]))
        page = dec.block_table[b].long()[torch.tensor(at // 16, device="cuda")]
        for layer in range(L):
            rows[b][layer] = [R.f64(c[layer][page, :, torch.tensor(at % 16, device="cuda")]) for c in (path.k_cache, path.v_cache)]
    for n in range(24):
        if n == 2:
            dec.fork([0, 1, 0], [2, 4, 3])
            assert dec.in_use == [0, 3, 2, 1, 4]
            for a, z in ((0, 2), (1, 4), (0, 3)):
                rows[z] = [[k.copy(), v.copy()] for k, v in rows[a]]
        if n == 20:
            dec.fork([3, 3], [5, 6])
            assert dec.in_use == [0, 3, 6, 5, 2, 1, 4]
            for z in (5, 6):
                rows[z] = [[k.copy(), v.copy()] for k, v in rows[3]]
        if n == 22:
            dec.release([0, 4])
            assert dec.in_use == [3, 6, 5, 2, 1]
        qkv, logits, u = step_inputs(g, L, len(dec.in_use), V)
        run(dec, L, qkv, logits, u, 0.7)
        assert cuda_lib.pic_device_status() == (0, 0)
        q, k, v = (R.f64(x) for x in qkv)
        for e, r in enumerate(dec.in_use):
            pos = len(rows[r][0][0])
            assert int(dec.ctx_len[r]) == pos + 1
            want = R.sample(logits[e].cpu().numpy(), u[e].item(), 0.8, 0, 0.7)
            assert (int(dec.token[e]), int(dec.kept[e])) == want[:2]
            page = int(dec.block_table[r, pos // 16])
            for layer in range(L):
                qr = np.stack([R.normed_rotated(x, R.f64(wq), 1e-6, pos, geom, layer)[0] for x in q[layer, e, 0]])
                kr = np.stack([R.normed_rotated(x, R.f64(wk), 1e-6, pos, geom, layer)[0] for x in k[layer, e, 0]])
                # the key as the cache holds it: within its rounding, then taken as it is
                got = R.f64(path.k_cache[layer, page, :, pos % 16])
                assert (np.abs(got - kr) <= np.abs(kr) * 2.0 ** -8 + 2.0 ** -17).all()
                K = np.concatenate([rows[r][layer][0], got[None]])
                VV = np.concatenate([rows[r][layer][1], v[layer, e]])
                rows[r][layer] = [K, VV]
                if n % 5 == 2 or n > 20:
                    ref, _, A, S = R.attention(qr, K, VV)
                    out = R.f64(dec.out[layer, e])
                    # the queries' rounding moves a score by at most 2^-8 S, twice for the softmax
                    assert (np.abs(out - ref) <= np.abs(ref) * 2.0 ** -8 + A * (2.0 ** -7 * S + 2.0 ** -7)).all(), (n, r)
    bt = dec.block_table[dec.block_table >= 0].long()
    assert torch.equal(dec.page_refs, torch.bincount(bt, minlength=dec.num_pages).int())


def test_a_captured_step_replays(cuda_lib):
    """Replays on advancing lengths give what the same steps outside a graph give, bit for bit."""
    from paper_2607_28069_gb300.pipeline import BranchDecoder
    got = []
    for captured in (False, True):
        wl, path = linked(2, spare=60)
        dec = BranchDecoder(path, rows=6, max_new=64)
        dec.fork([0, 0, 1, 0], [2, 3, 4, 5])
        g = torch.Generator(device="cuda").manual_seed(3)
        steps = [step_inputs(g, 2, 6, 500) for _ in range(20)]
        qkv, logits, u = step_inputs(g, 2, 6, 500)
        if captured:
            for x, y in zip((*qkv, logits, u), (*steps[0][0], steps[0][1], steps[0][2])):
                x.copy_(y)
            graph = torch.cuda.CUDAGraph()
            torch.cuda.synchronize()
            with torch.cuda.graph(graph):
                run(dec, 2, qkv, logits, u, 0.9)
        rec = []
        for s in steps:
            for x, y in zip((*qkv, logits, u), (*s[0], s[1], s[2])):
                x.copy_(y)
            if captured:
                graph.replay()
            else:
                run(dec, 2, qkv, logits, u, 0.9)
            rec.append([t.clone() for t in (dec.out, dec.token, dec.logprob, dec.kept, dec.ctx_len, dec.block_table)])
        assert cuda_lib.pic_device_status() == (0, 0)
        got.append(rec)
    for a, b in zip(*got):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_a_row_without_a_page_waits(cuda_lib):
    """With no page free, a row at a page's end stays at its length, while others go on; with
    pages again its steps are taken, and no position was passed over (the free pages hold NaN)."""
    from paper_2607_28069_gb300 import DEVICE_CODES
    from paper_2607_28069_gb300.pipeline import BranchDecoder
    wl, path = linked(1, spare=8)
    dec = BranchDecoder(path, max_new=64)
    g = torch.Generator(device="cuda").manual_seed(5)
    free = dec.page_refs == 0
    path.k_cache[:, free] = path.v_cache[:, free] = float("nan")
    dec.page_refs[free] = 1
    waited, geom = torch.zeros(2, dtype=torch.bool, device="cuda"), dec.geom
    for n in range(160):
        if n and bool(waited.all()):
            break
        before = dec.ctx_len.clone()
        room = dec.block_table.gather(1, (before // 16).long()[:, None])[:, 0] >= 0
        qkv, logits, u = step_inputs(g, 1, 2, 300)
        run(dec, 1, qkv, logits, u, 0.7)
        code = cuda_lib.pic_device_status()[0]
        assert DEVICE_CODES[code] == ("ok" if room.all() else "no free page")
        assert torch.equal(dec.ctx_len, before + room.int())
        waited |= ~room
    assert waited.all()
    dec.page_refs[free] = 0
    for n in range(2):
        before = dec.ctx_len.clone()
        qkv, logits, u = step_inputs(g, 1, 2, 300)
        run(dec, 1, qkv, logits, u, 0.7)
        assert cuda_lib.pic_device_status() == (0, 0) and torch.equal(dec.ctx_len, before + 1)
    for e, r in enumerate(dec.in_use):
        at = torch.arange(int(dec.ctx_len[r]), device="cuda")
        page = dec.block_table[r].long()[at // 16]
        K, V = (R.f64(c[0][page, :, at % 16]) for c in (path.k_cache, path.v_cache))
        ref, _, A, S = R.attention(R.f64(dec.q_rot[e, 0]), K, V)
        out = R.f64(dec.out[0, e])
        # (the roundings as in attention_close)
        assert (np.abs(out - ref) <= np.abs(ref) * 2.0 ** -8 + A * (2.0 ** -8 * 1.01 + 2.0 ** -14 * S + 2.0 ** -18)).all()
