"""DraftDecoder: reserve, draft attention, verification, compaction, forks and
releases together, as a serving loop runs them, against a plain model that keeps
every row's keys and values in a list (64-bit attention over bf16 keys; bars as in
test_gpu_draft).  The walk down the drafts has to match exactly."""
import numpy as np
import pytest
import torch

import oracle as O
from paper_2607_28069_gb300.workloads import custom_spec, generate
from tests.helpers import attn_close, f64, oracle_layout, request_inputs, theta_of
from tests.test_gpu_draft import bf16, line_of, rope
from tests.test_gpu_verify import probs, rule

pytestmark = pytest.mark.gpu


def linked(layers=2, spare=40):
    from paper_2607_28069_gb300.pipeline import CacheHitPath
    spec = custom_spec(name="spec", layers=layers, q_heads=8, kv_heads=2, head_dim=64, rope_base=1e4,
                       batch=2, pool_docs=4, docs_per_request=2, doc_len=(20, 90), prefix_len=(3, 17),
                       query_len=9)
    wl = generate(spec, device="cuda", gen_device="cpu")
    wl.num_pages += spare
    path = CacheHitPath(wl)
    path.ttft_pass()
    return wl, path


def contexts(wl):
    """K and V of every request and layer after its prefill, [ctx][Hkv][d] each."""
    theta, got = theta_of(wl.spec), []
    for b in range(wl.spec.batch):
        lay = oracle_layout(wl, b)
        row = []
        for layer in range(wl.spec.layers):
            docs, kd, vd, q, k, v = request_inputs(wl, b, layer)
            K, V = O.dense_context(lay, kd, vd, wl.doc_base_pos.cpu().numpy(), k, v, theta)
            row.append([bf16(K), V])
        got.append(row)
    return got


def i32(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32).cuda()


def inputs(rng, rows, T, layers, vocab, sampled, live):
    s = {}
    r = lambda *sh: torch.as_tensor(rng.standard_normal(sh)).to(torch.bfloat16).cuda()  # noqa: E731
    s["q"], s["k"], s["v"] = r(layers, rows, T, 8, 64), r(layers, rows, T, 2, 64), r(layers, rows, T, 2, 64)
    s["p"] = probs(rng, rows, T, vocab)
    s["u"] = rng.random((rows, T)).astype(np.float32)
    s["len"] = np.where(live, rng.integers(1, T + 1, rows), 0)
    s["draft"] = s["parent"] = None
    s["par"] = np.tile(np.arange(T) - 1, (rows, 1))
    s["tok"] = np.zeros((rows, T), np.int64)
    if sampled:
        s["draft"] = ((probs(rng, rows, T - 1, vocab) + 2 * s["p"][:, :-1]) / 3).astype(np.float32)
        s["tok"][:, 1:] = (s["draft"] / rng.exponential(size=s["draft"].shape)).argmax(-1)
    else:
        s["par"] = np.maximum(0, np.arange(T) - 1 - rng.integers(0, 3, (rows, T)))
        s["par"][:, 0] = -1
        s["parent"] = s["par"]
        for b in range(rows):
            for i in range(1, T):
                rank = int((s["par"][b, 1:i] == s["par"][b, i]).sum())
                s["tok"][b, i] = s["p"][b, s["par"][b, i]].argsort()[::-1][rank]
    return s


def step(dec, s, layers):
    dec.begin()
    par = None if s["parent"] is None else i32(s["parent"])
    for layer in range(layers):
        dec.attend(layer, (s["q"], layer), (s["k"], layer), (s["v"], layer), i32(s["len"]), parent=par)
    cu = lambda x: None if x is None else torch.as_tensor(x).cuda()  # noqa: E731
    dec.accept(i32(s["tok"]), i32(s["len"]), cu(s["p"]), cu(s["u"]), draft_prob=cu(s["draft"]),
               parent=par)


def test_steps_forks_and_releases(cuda_lib):
    from paper_2607_28069_gb300.pipeline import DraftDecoder
    L, T, V = 2, 6, 60
    wl, path = linked(L)
    dec = DraftDecoder(path, T, rows=5, max_new=64)
    rows = contexts(wl) + [None] * 3
    rng = np.random.default_rng(8)
    kept = 0
    for n in range(6):
        if n == 2:  # two branches of request 0, one of request 1
            dec.fork([0, 0, 1], [2, 4, 3])
            for a, z in ((0, 2), (0, 4), (1, 3)):
                rows[z] = [[k.copy(), v.copy()] for k, v in rows[a]]
        if n == 4:  # request 0 ends, its branches go on
            dec.release([0])
            rows[0] = None
        live = np.array([r is not None for r in rows])
        s = inputs(rng, 5, T, L, V, n % 2 == 0, live)
        step(dec, s, L)
        assert cuda_lib.pic_device_status() == (0, 0)
        for b in np.flatnonzero(live):
            m, c = int(s["len"][b]), len(rows[b][0][0])
            want = rule(s["tok"][b].tolist(), m, s["p"][b], s["u"][b],
                        None if s["draft"] is None else s["draft"][b],
                        None if s["parent"] is None else s["par"][b].tolist())
            assert (dec.path_idx[b].tolist(), int(dec.path_len[b]), int(dec.next_token[b])) == want
            line = line_of(s["par"][b], m)
            pos = [c + len(x) - 1 for x in line]
            for layer in range(L):
                kr = bf16(rope(f64(s["k"][layer, b, :m]), pos, 1e4, 0))
                qr = bf16(rope(f64(s["q"][layer, b, :m]), pos, 1e4, 0))
                K = np.concatenate([rows[b][layer][0], kr])
                VV = np.concatenate([rows[b][layer][1], f64(s["v"][layer, b, :m])])
                for i in range(m):
                    at = list(range(c)) + [c + j for j in line[i]]
                    for h in range(8):
                        z = K[at, h // 4] @ qr[i, h] / 8.0
                        w = np.exp(z - z.max())
                        ok, worst, rel = attn_close(f64(dec.out[layer, b, i, h])[None],
                                                    (w @ VV[at, h // 4] / w.sum())[None],
                                                    abs_tol=1e-2, row_rel=1e-2)
                        assert ok, (n, b, layer, i, h, worst, rel)
                keep = list(range(c)) + [c + j for j in want[0][:want[1]]]
                rows[b][layer] = [K[keep], VV[keep]]
            kept += want[1] - 1
            assert int(dec.ctx_len[b]) == c + want[1]
    assert kept > 5  # paths were followed
    # every page has the users that the tables say
    bt = dec.block_table[dec.block_table >= 0].long()
    assert torch.equal(dec.page_refs, torch.bincount(bt, minlength=dec.num_pages).int())
    with pytest.raises(ValueError, match='not in use'):
        dec.fork([2], [4])
    dec.release(range(5))
    assert int(dec.page_refs.sum()) == 0 and cuda_lib.pic_device_status() == (0, 0)


def test_a_captured_step_replays(cuda_lib):
    """A step captured in a CUDA graph: replays on advancing lengths give what the
    same steps outside a graph give, bit for bit."""
    from paper_2607_28069_gb300.pipeline import DraftDecoder
    L, T, V = 1, 5, 40
    rng = np.random.default_rng(2)
    s = inputs(rng, 2, T, L, V, True, np.array([True, True]))
    dev = {k: torch.as_tensor(v).cuda() if v is not None and not isinstance(v, torch.Tensor) else v
           for k, v in s.items()}
    dev["len"], dev["tok"] = i32(s["len"]), i32(s["tok"])

    def run(dec):
        dec.begin()
        dec.attend(0, (s["q"], 0), (s["k"], 0), (s["v"], 0), dev["len"])
        dec.accept(dev["tok"], dev["len"], dev["p"], dev["u"], draft_prob=dev["draft"])

    got = []
    for captured in (False, True):
        wl, path = linked(L)
        dec = DraftDecoder(path, T)
        if captured:
            state = [t.clone() for t in (dec.ctx_len, dec.block_table, dec.page_refs, path.k_cache,
                                         path.v_cache)]
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.stream(side):
                run(dec)
                with torch.cuda.graph(graph, stream=side):
                    run(dec)
            torch.cuda.synchronize()
            for t, old in zip((dec.ctx_len, dec.block_table, dec.page_refs, path.k_cache, path.v_cache),
                              state):
                t.copy_(old)
        outs = []
        for _ in range(4):
            graph.replay() if captured else run(dec)
            outs += [dec.out.clone(), dec.ctx_len.clone(), dec.next_token.clone()]
        got.append(outs + [path.k_cache.clone(), path.v_cache.clone(), dec.block_table.clone()])
    assert cuda_lib.pic_device_status() == (0, 0)
    live = [slice(None)] * len(got[0])
    for i, (a, b) in enumerate(zip(*got)):
        if a.dim() == 5 and a.shape[2] == T:  # rows past a request's drafts are never written
            for r in range(2):
                assert torch.equal(a[:, r, :int(s["len"][r])], b[:, r, :int(s["len"][r])]), i
        else:
            assert torch.equal(a[live[i]], b[live[i]]), i
