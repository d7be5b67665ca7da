"""pic_append_normed against 64 bits: types of geometry, strides, ways to name positions and
rows, the prefill's packed queries, tokens and rows left alone."""
import numpy as np
import pytest
import torch

from tests import branch_reference as R

pytestmark = pytest.mark.gpu
BF = dict(dtype=torch.bfloat16, device="cuda")


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Case:
    def __init__(self, pic, Hq, Hkv, d, B, T, style=0, fused=True, seed=0, rows=None, pages=8, layers=2, **geom):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()  # noqa: E731
        self.pic, self.B, self.T = pic, B, T
        self.geom = pic.Geometry(layers, Hq, Hkv, d, 1e4, rope_style=style, **geom)
        if fused:
            self.q, self.k, self.v = rand(B, T, Hq + 2 * Hkv, d).split([Hq, Hkv, Hkv], dim=2)
        else:
            self.q, self.k, self.v = rand(B, T, Hq, d), rand(B, T, Hkv, d), rand(B, T, Hkv, d)
        self.wq, self.wk = 1 + rand(d) / 4, 1 + rand(d) / 4
        rows = rows or B
        r = np.random.default_rng(seed)
        self.num_pages = rows * pages + 3
        self.table = r.permutation(self.num_pages)[:rows * pages].reshape(rows, pages)
        self.block_table = i32(self.table.tolist())
        shape = (layers, self.num_pages, Hkv, 16, d)
        self.kc, self.vc = torch.full(shape, 7.0, **BF), torch.full(shape, 7.0, **BF)
        self.out = torch.full((B, T, Hq, d), 7.0, **BF)

    def run(self, layer=1, **kw):
        kw = dict(dict(q_weight=self.wq, k_weight=self.wk), **kw)
        if "workspace" not in kw:
            kw["q_out"] = self.out
        self.pic.pic_append_normed(self.geom, layer, self.q, self.k, self.v, self.block_table,
                                   self.num_pages, self.kc, self.vc, **kw)
        torch.cuda.synchronize()

    def check(self, tokens, layer=1, eps=1e-6, wq=True, wk=True):
        """tokens: {(b, t): (row, position)}; all else is as it was."""
        q, k, v = R.f64(self.q), R.f64(self.k), R.f64(self.v)
        wq, wk = R.f64(self.wq) if wq else None, R.f64(self.wk) if wk else None
        out, kc, vc = R.f64(self.out), R.f64(self.kc), R.f64(self.vc)
        left = np.ones(out.shape[:2], bool)
        slots = np.ones(kc.shape[1:2] + (16,), bool)
        for (b, t), (row, pos) in tokens.items():
            left[b, t] = False
            page = self.table[row][pos // 16]
            slots[page, pos % 16] = False
            for h in range(q.shape[2]):
                assert R.append_close(out[b, t, h], *R.normed_rotated(q[b, t, h], wq, eps, pos, self.geom, layer)).all()
            for h in range(k.shape[2]):
                got = kc[layer, page, h, pos % 16]
                assert R.append_close(got, *R.normed_rotated(k[b, t, h], wk, eps, pos, self.geom, layer)).all()
                assert (vc[layer, page, h, pos % 16] == v[b, t, h]).all()
        assert (out[left] == 7).all()
        for c in (kc, vc):
            assert (c[layer].transpose(0, 2, 1, 3)[slots] == 7).all()
            assert (np.delete(c, layer, 0) == 7).all()


GEOMS = [(8, 2, 128), (7, 1, 128), (4, 1, 64), (16, 2, 64), (32, 8, 128), (1, 1, 64), (72, 8, 128), (96, 2, 64)]


@pytest.mark.parametrize("fused", [False, True])
@pytest.mark.parametrize("style", [0, 1])
@pytest.mark.parametrize("heads", GEOMS)
def test_against_64_bits(cuda_lib, heads, style, fused):
    c = Case(cuda_lib, *heads, B=3, T=5, style=style, fused=fused)
    n = [5, 0, 3]
    start = [0, 9, 111]
    pos = [[s + t for t in range(5)] for s in start]
    c.run(num_tokens=i32(n), pos=i32(pos))
    c.check({(b, t): (b, pos[b][t]) for b in range(3) for t in range(n[b])})
    assert cuda_lib.pic_device_status() == (0, 0)


def test_rows_lengths_and_no_norm(cuda_lib):
    c = Case(cuda_lib, 8, 2, 128, B=4, T=1, rows=7)
    row, ctx = [6, 0, 3, 2], [5, 1, 16, 127, 9, 9, 31]
    for wq, wk, eps in ((True, True, 1e-6), (False, True, 0.0), (True, False, 0.5), (False, False, 1e-5)):
        c.kc.fill_(7), c.vc.fill_(7), c.out.fill_(7)
        c.run(layer=0, row=i32(row), ctx_len=i32(ctx), eps=eps, q_weight=c.wq if wq else None,
              k_weight=c.wk if wk else None)
        c.check({(b, 0): (row[b], ctx[row[b]]) for b in range(4)}, layer=0, eps=eps, wq=wq, wk=wk)
    assert cuda_lib.pic_device_status() == (0, 0)


def test_strides_of_every_dimension(cuda_lib):
    c = Case(cuda_lib, 4, 2, 64, B=2, T=3, fused=False)
    g = torch.Generator(device="cuda").manual_seed(5)
    base = torch.randn(4, 3, 5, 2, 72, generator=g, device="cuda").bfloat16()
    c.q = base.permute(2, 3, 1, 0, 4)[1:3].expand(2, 2, 3, 4, 72)[:, 0, :, :, :64]   # heads outermost
    c.k = base[0, 0, 0, 0, :64].expand(2, 3, 2, 64)                                  # broadcast: strides of 0
    c.v = base[:2, :, 0, :, 8:].permute(0, 1, 2, 3)
    pos = [[3, 4, 5], [100, 101, 102]]
    c.run(pos=i32(pos))
    c.check({(b, t): (b, pos[b][t]) for b in range(2) for t in range(3)})


def test_tables_of_frequencies(cuda_lib):
    inv = [1.0 / (3.0 + i) for i in range(32)]
    layer = torch.tensor([inv, [x * 0.37 for x in inv]], dtype=torch.float64, device="cuda")
    for kw in (dict(inv_freq=inv), dict(layer_inv_freq=layer)):
        c = Case(cuda_lib, 4, 1, 64, B=2, T=2, **kw)
        pos = [[0, 1], [126, 127]]
        c.run(pos=i32(pos))
        c.check({(b, t): (b, pos[b][t]) for b in range(2) for t in range(2)})


@pytest.mark.parametrize("B,T", [(1, 700), (40, 33), (1100, 3), (3, 1)])
def test_many_tokens_each_once(cuda_lib, B, T):
    """Shares of requests' tokens (also where one spans several, or takes several rounds)."""
    c = Case(cuda_lib, 4, 1, 64, B=B, T=T, pages=(T + 40) // 16 + 1)
    r = np.random.default_rng(B)
    n = r.integers(0, T + 1, size=B)
    start = r.integers(0, 30, size=B)
    pos = start[:, None] + np.arange(T)
    c.run(num_tokens=i32(n.tolist()), pos=i32(pos.tolist()))
    b, t = np.nonzero(np.arange(T) < n[:, None])
    some = r.permutation(len(b))[:60]
    live = torch.zeros((B, T), dtype=torch.bool, device="cuda")
    live[torch.tensor(b, device="cuda"), torch.tensor(t, device="cuda")] = True
    assert ((c.out != 7).any(-1).any(-1) == live).all()
    written = (c.vc[1] != 7).any(-1).any(1)   # [page][slot]
    want = torch.zeros_like(written)
    want[torch.tensor(c.table[b, pos[b, t] // 16], device="cuda"), torch.tensor(pos[b, t] % 16, device="cuda")] = True
    assert (written == want).all()
    q, k = R.f64(c.q), R.f64(c.k)
    for i in some:
        bb, tt, p = b[i], t[i], pos[b[i], t[i]]
        for h in range(4):
            assert R.append_close(R.f64(c.out[bb, tt, h]), *R.normed_rotated(q[bb, tt, h], R.f64(c.wq), 1e-6, p, c.geom, 1)).all()
        got = R.f64(c.kc[1, c.table[bb, p // 16], 0, p % 16])
        assert R.append_close(got, *R.normed_rotated(k[bb, tt, 0], R.f64(c.wk), 1e-6, p, c.geom, 1)).all()
    assert cuda_lib.pic_device_status() == (0, 0)


def test_what_is_left_alone(cuda_lib):
    """Bad rows, counts, positions and pages; the rest of the batch is served."""
    pic = cuda_lib
    tok = lambda rows, pos: {(b, 0): (rows[b], pos[b]) for b in range(len(rows)) if rows[b] is not None}  # noqa: E731
    c = Case(pic, 4, 1, 64, B=4, T=1)
    c.run(row=i32([0, 4, -1, 2]), ctx_len=i32([3, 4, 5, 6]))
    c.check(tok([0, None, None, 2], [3, 0, 0, 5]))
    assert pic.pic_device_status()[0] == 3
    c = Case(pic, 4, 1, 64, B=4, T=1)
    c.run(row=i32([1, 3, 1, 0]), ctx_len=i32([3, 4, 5, 6]))      # row 1 twice: the second is left alone
    c.check(tok([1, 3, None, 0], [4, 6, 0, 3]))
    assert pic.pic_device_status() == (3, 2)
    c = Case(pic, 4, 1, 64, B=4, T=1)
    c.run(num_tokens=i32([1, 2, -1, 0]), pos=i32([[3], [4], [5], [6]]))
    c.check(tok([0], [3]))
    assert pic.pic_device_status()[0] == 3
    # positions: the queries are written (unrotated), keys and values are not
    c = Case(pic, 4, 1, 64, B=3, T=1)
    c.run(pos=i32([[-1], [128], [127]]))
    assert pic.pic_device_status()[0] in (5, 7)
    for b, p in ((0, 0), (1, 0), (2, 127)):
        assert R.append_close(R.f64(c.out[b, 0, 1]), *R.normed_rotated(R.f64(c.q[b, 0, 1]), R.f64(c.wq), 1e-6, p, c.geom, 1)).all()
    assert int((c.kc != 7).any(-1).sum()) == 1 and int((c.vc != 7).any(-1).sum()) == 1
    # pages
    c = Case(pic, 4, 1, 64, B=2, T=1)
    c.block_table[0, 0] = c.num_pages
    c.run(pos=i32([[3], [4]]))
    assert pic.pic_device_status() == (6, 0) and int((c.vc != 7).any(-1).sum()) == 1


def test_infinite_and_nan_heads_stay_in_their_head(cuda_lib):
    c = Case(cuda_lib, 8, 2, 128, B=1, T=2, fused=False)
    c.q[0, 0, 3, 5], c.k[0, 1, 1, 0] = float("nan"), float("inf")
    c.run(pos=i32([[3, 4]]))
    bad = ~torch.isfinite(c.out.float()).all(-1)
    assert bad.nonzero().tolist() == [[0, 0, 3]]
    page = c.table[0][0]
    bad = ~torch.isfinite(c.kc[1, page].float()).all(-1)
    assert bad.nonzero().tolist() == [[1, 4]]


def test_packed_for_the_prefill(cuda_lib):
    """A Reader's prefill: the append into the workspace, then the attention with NULL
    projections; without norms the same rows as pic_append_inline leaves."""
    pic = cuda_lib
    c = Case(pic, 8, 2, 128, B=2, T=37, pages=4, layers=1)
    n = [37, 11]
    pos = torch.arange(37, device="cuda", dtype=torch.int32).repeat(2, 1).contiguous()
    size = pic.pic_prefill_workspace_size(c.geom, 2, 37, 64, 1)
    ws = [torch.full((size,), 85, dtype=torch.uint8, device="cuda") for _ in range(2)]
    q, k, v = c.q.contiguous(), c.k.contiguous(), c.v.contiguous()
    slots = (c.block_table.repeat_interleave(16, 1).long() * 16 + torch.arange(64, device="cuda") % 16).contiguous()
    kc = [c.kc.clone(), c.kc.clone()]
    pic.pic_append_inline(c.geom, 0, q, k, v, pos, i32(n), slots, c.num_pages, kc[0], c.vc, ws[0])
    pic.pic_append_normed(c.geom, 0, c.q, c.k, c.v, c.block_table, c.num_pages, kc[1], c.vc, workspace=ws[1],
                          num_tokens=i32(n), pos=pos)
    a, b = (w.view(torch.bfloat16).float() for w in ws)
    assert torch.allclose(a, b, rtol=2.0 ** -7, atol=2.0 ** -16, equal_nan=True)
    assert torch.allclose(kc[0].float(), kc[1].float(), rtol=2.0 ** -7, atol=2.0 ** -16)
    out = torch.zeros((2, 37, 8, 128), **BF)
    c.run(layer=0, num_tokens=i32(n), pos=pos, workspace=ws[1])
    ws_a = torch.empty(pic.pic_prefill_workspace_size(c.geom, 2, 37, 64, 0), dtype=torch.uint8, device="cuda")
    ws_a[:size] = ws[1]
    pic.pic_attend_prefill(c.geom, 0, pos, i32(n), 64, c.block_table, c.num_pages, c.kc, c.vc, out, workspace=ws_a)
    torch.cuda.synchronize()
    for b in range(2):
        K = R.f64(c.kc[0, torch.tensor(c.table[b]), :, :]).transpose(0, 2, 1, 3).reshape(-1, 2, 128)
        V = R.f64(c.vc[0, torch.tensor(c.table[b]), :, :]).transpose(0, 2, 1, 3).reshape(-1, 2, 128)
        for t in range(n[b]):
            qr = np.stack([R.normed_rotated(R.f64(c.q[b, t, h]), R.f64(c.wq), 1e-6, t, c.geom, 0)[0] for h in range(8)])
            ref, _, A, S = R.attention(qr, K[:t + 1], V[:t + 1])
            # the queries' own rounding moves a score by at most 2^-8 S, twice for the softmax
            e = 2 * 2.0 ** -8 * S + 2.0 ** -7
            assert (np.abs(R.f64(out[b, t]) - ref) <= np.abs(ref) * 2.0 ** -8 + A * e).all()
    assert pic.pic_device_status() == (0, 0)


def test_two_streams_and_a_graph(cuda_lib):
    c = [Case(cuda_lib, 8, 2, 128, B=5, T=3, seed=s) for s in range(2)]
    pos = i32([[b * 9 + t for t in range(3)] for b in range(5)])
    streams = [torch.cuda.Stream() for _ in c]
    torch.cuda.synchronize()
    for x, s in zip(c, streams):
        with torch.cuda.stream(s):
            x.pic.pic_append_normed(x.geom, 1, x.q, x.k, x.v, x.block_table, x.num_pages, x.kc, x.vc, x.out,
                                    q_weight=x.wq, k_weight=x.wk, pos=pos)
    torch.cuda.synchronize()
    for x in c:
        x.check({(b, t): (b, b * 9 + t) for b in range(5) for t in range(3)})
    x = c[0]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        x.pic.pic_append_normed(x.geom, 1, x.q, x.k, x.v, x.block_table, x.num_pages, x.kc, x.vc, x.out,
                                q_weight=x.wq, k_weight=x.wk, pos=pos)
    pos += 40
    x.kc.fill_(7), x.vc.fill_(7)
    g.replay()
    torch.cuda.synchronize()
    x.check({(b, t): (b, b * 9 + t + 40) for b in range(5) for t in range(3)})


def test_positions_and_offsets_beyond_31_bits_of_elements(cuda_lib):
    """Pages at the end of a cache of more than 2^31 elements, positions of millions."""
    pic = cuda_lib
    geom = pic.Geometry(1, 8, 8, 128, 5e5)
    pages = 140000
    kc, vc = (torch.empty((1, pages, 8, 16, 128), **BF) for _ in range(2))
    assert kc.numel() > 2 ** 31
    table = torch.full((1, 1 << 18), -1, dtype=torch.int32, device="cuda")
    pos = 4_194_301
    table[0, pos // 16] = pages - 1
    q, k, v = (torch.randn((1, 1, 8, 128), device="cuda").bfloat16() for _ in range(3))
    out = torch.empty_like(q)
    pic.pic_append_normed(geom, 0, q, k, v, table, pages, kc, vc, out, pos=i32([[pos]]))
    torch.cuda.synchronize()
    assert pic.pic_device_status() == (0, 0)
    for h in range(8):
        for got, x in ((out[0, 0, h], q), (kc[0, pages - 1, h, pos % 16], k)):
            assert R.append_close(R.f64(got), *R.normed_rotated(R.f64(x[0, 0, h]), None, 0, pos, geom, 0)).all()
        assert torch.equal(vc[0, pages - 1, h, pos % 16], v[0, 0, h])
