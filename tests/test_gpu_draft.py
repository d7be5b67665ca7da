"""pic_attend_draft against a 64-bit softmax over the same bf16 cache, written from
the formulas: chains and trees, one to 64 tokens, contexts that end at, before and
behind page and tile edges (0 cached positions too), ragged batches with empty
requests, GQA groups of 1 to 16 (up to 1024 query rows per kv head), both head
dims and RoPE styles.  Slots and pages behind the drafts hold NaN.

Bars: keys as in the parity tests (bf16 rounding of an fp32 rotation).  Outputs:
the weights are rounded to bf16 (2^-9 of each), the output once more (2^-9 of it),
and a query element now and then rounds the other way than in 64 bits; together
under 1e-2 of a row, and of 1 + |o| per element.  lse: fp32 scores of bf16 queries,
2e-3 as in the decode tests."""
import numpy as np
import pytest
import torch

from tests.helpers import attn_close, f64, kv_tolerance_ok

pytestmark = pytest.mark.gpu


def rope(x, pos, base, style):
    d = x.shape[-1]
    w = np.exp(1j * np.asarray(pos, np.float64)[:, None, None]
               * base ** (-2.0 * np.arange(d // 2) / d))
    if style == 0:
        z = (x[..., :d // 2] + 1j * x[..., d // 2:]) * w
        return np.concatenate([z.real, z.imag], -1)
    z = (x[..., 0::2] + 1j * x[..., 1::2]) * w
    return np.stack([z.real, z.imag], -1).reshape(x.shape)


def bf16(x):
    return torch.as_tensor(x).to(torch.bfloat16).double().numpy()


def line_of(par, n):
    """Ancestors of each token and the token itself."""
    line = []
    for i in range(n):
        line.append((line[par[i]] if par[i] >= 0 else []) + [i])
    return line


def draw(heads, dim, style, ctx, draft, T, tree, layers=2, seed=0, q_scale=1.0, base=5e5):
    import paper_2607_28069_gb300 as pic
    hq, hkv = heads
    B = len(ctx)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda").bfloat16()  # noqa: E731
    pages = max(-(-(c + T) // 16) for c in ctx) + 1
    num = B * pages + 2
    bt = torch.as_tensor(rng.permutation(num)[:B * pages].reshape(B, pages), dtype=torch.int32)
    kc, vc = rnd(layers, num, hkv, 16, dim), rnd(layers, num, hkv, 16, dim)
    # everything that is no cached position of a request is NaN
    used = torch.zeros((num, 16), dtype=torch.bool)
    for b, c in enumerate(ctx):
        t = torch.arange(c)
        used[bt[b, t // 16].long(), t % 16] = True
    for cache in (kc, vc):
        cache.permute(1, 3, 0, 2, 4)[~used.cuda()] = float("nan")
    par = np.full((B, T), -1, np.int64)
    for i in range(1, T):
        par[:, i] = np.maximum(0, i - 1 - rng.integers(0, 4, size=B)) if tree else i - 1
    if tree and T > 4:
        par[:, 4] = -1  # a second root
    dev = lambda x: torch.as_tensor(np.asarray(x), dtype=torch.int32).cuda()  # noqa: E731
    s = dict(geom=pic.Geometry(layers, hq, hkv, dim, base, rope_style=style), layer=layers - 1,
             q=rnd(B, T, hq, dim) * q_scale, k=rnd(B, T, hkv, dim), v=rnd(B, T, hkv, dim),
             ctx=dev(ctx), draft=dev(draft), bt=bt.cuda(), num=num, kc=kc, vc=vc,
             out=torch.full((B, T, hq, dim), 7.0, dtype=torch.bfloat16, device="cuda"),
             lse=torch.full((B, T, hq), 7.0, device="cuda"), parent=dev(par) if tree else None,
             ws=torch.full((pic.pic_draft_workspace_size(pic.Geometry(layers, hq, hkv, dim, base), B,
                                                         T),), 255, dtype=torch.uint8,
                           device="cuda"), par=par, base=base, style=style)
    return s


def call(s, **kw):
    import paper_2607_28069_gb300 as pic
    a = dict(parent=s["parent"], lse=s["lse"], workspace=s["ws"])
    a.update(kw)
    pic.pic_attend_draft(s["geom"], s["layer"], s["q"], s["k"], s["v"], s["ctx"], s["draft"],
                         s["bt"], s["num"], s["kc"], s["vc"], s["out"], **a)


def check(s, ctx, draft, k_before, v_before):
    hq, hkv = s["q"].shape[2], s["k"].shape[2]
    d, G, lay = s["q"].shape[3], hq // hkv, s["layer"]
    kc, vc, bt = s["kc"], s["vc"], s["bt"].cpu().numpy()
    touched = torch.zeros(kc.shape[:2] + (16,), dtype=torch.bool)
    for b, (c, n) in enumerate(zip(ctx, draft)):
        assert bool((s["out"][b, n:] == 7).all()) and bool((s["lse"][b, n:] == 7).all())
        if n == 0:
            continue
        line = line_of(s["par"][b], n)
        pos = [c + len(x) - 1 for x in line]
        t = np.arange(c + n)
        page = bt[b][t // 16]
        touched[lay, page[c:], t[c:] % 16] = True
        K, V = f64(kc[lay])[page, :, t % 16], f64(vc[lay])[page, :, t % 16]
        ok, worst = kv_tolerance_ok(K[c:], rope(f64(s["k"][b, :n]), pos, s["base"], s["style"]))
        assert ok, (b, worst)
        assert np.array_equal(V[c:], f64(s["v"][b, :n]))
        qr = bf16(rope(f64(s["q"][b, :n]), pos, s["base"], s["style"]))
        vis = np.zeros((n, c + n), bool)
        vis[:, :c] = True
        for i in range(n):
            vis[i, [c + j for j in line[i]]] = True
        for h in range(hq):
            z = np.where(vis, qr[:, h] @ K[:, h // G].T / np.sqrt(d), -np.inf)
            m = z.max(-1, keepdims=True)
            w = np.exp(z - m)
            l = w.sum(-1, keepdims=True)
            ok, worst, rel = attn_close(f64(s["out"][b, :n, h]), w @ V[:, h // G] / l, abs_tol=1e-2,
                                        row_rel=1e-2)
            assert ok, (b, h, worst, rel)
            assert np.abs(f64(s["lse"][b, :n, h]) - (m + np.log(l))[:, 0]).max() < 2e-3
    # nothing else in the caches changed, bit for bit
    for new, old in ((kc, k_before), (vc, v_before)):
        same = (new.view(torch.int16) == old.view(torch.int16)).permute(0, 1, 3, 2, 4)
        assert bool(same[~touched.cuda()].all())


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("heads,dim,style", [((4, 4), 128, 0), ((14, 2), 64, 1), ((32, 2), 128, 1),
                                             ((7, 1), 128, 0), ((16, 1), 64, 0)])
@pytest.mark.parametrize("T", [1, 5, 64])
def test_draft_attention(cuda_lib, heads, dim, style, T, tree):
    ctx = [0, 1, 15, 16, 127, 128, 129, 300, 64 * 16]
    draft = [T, max(1, T - 1), T, 1, T, max(1, T // 2), T, 0, T]
    s = draw(heads, dim, style, ctx, draft, T, tree, seed=T + dim)
    before = s["kc"].clone(), s["vc"].clone()
    call(s)
    assert cuda_lib.pic_device_status() == (0, 0)
    check(s, ctx, draft, *before)


@pytest.mark.parametrize("heads,dim", [((8, 1), 128), ((8, 2), 64)])
def test_long_contexts_split_over_many_ctas(cuda_lib, heads, dim):
    """One long context (its tiles over all SMs, up to 152 partial states per
    row) beside a short one, with scores that jump along the context."""
    ctx, draft = [40001, 77], [9, 3]
    s = draw(heads, dim, 0, ctx, draft, 9, True, layers=1, q_scale=4.0)
    # later keys larger: the running maximum grows on the way
    t = torch.arange(40001, device="cuda")
    page = s["bt"][0].long()[t // 16]
    s["kc"][0, page, :, t % 16] *= (1 + 3 * t / 40001)[:, None, None].bfloat16()
    before = s["kc"].clone(), s["vc"].clone()
    call(s)
    assert cuda_lib.pic_device_status() == (0, 0)
    check(s, ctx, draft, *before)


def test_many_requests_and_repeated_calls(cuda_lib):
    """More units than SMs, more requests than a warp; the same call twice gives
    the same bits, on another stream too."""
    rng = np.random.default_rng(3)
    ctx, draft = rng.integers(0, 400, 70).tolist(), rng.integers(0, 5, 70).tolist()
    s = draw((8, 4), 128, 0, ctx, draft, 4, True)
    before = s["kc"].clone(), s["vc"].clone()
    call(s)
    check(s, ctx, draft, *before)
    out, lse = s["out"].clone(), s["lse"].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call(s, stream=side)
    side.synchronize()
    assert torch.equal(out, s["out"]) and torch.equal(lse, s["lse"])
    assert cuda_lib.pic_device_status() == (0, 0)


def test_a_chain_is_decoding_token_by_token(cuda_lib):
    """Drafting a chain gives what decoding its tokens one after the other gives."""
    import paper_2607_28069_gb300 as pic
    ctx, T = [200, 31], 4
    s = draw((8, 2), 128, 0, ctx, [T, T], T, False)
    kc, vc = s["kc"].clone(), s["vc"].clone()
    call(s)
    out = torch.empty((2, 8, 128), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(pic.pic_decode_workspace_size(s["geom"], 2, 256), dtype=torch.uint8,
                     device="cuda")
    for b in range(2):  # decode reads whole pages: no NaN behind the context there
        for cache in (kc, vc):
            t = torch.arange(ctx[b], s["bt"].shape[1] * 16, device="cuda")
            cache.permute(1, 3, 0, 2, 4)[s["bt"][b].long()[t // 16], t % 16] = 0
    for i in range(T):
        pic.pic_attend_decode(s["geom"], 1, s["q"][:, i].contiguous(), s["k"][:, i].contiguous(),
                              s["v"][:, i].contiguous(), s["ctx"], s["bt"], s["num"], kc, vc, out,
                              256, workspace=ws, pos_offset=i)
        ok, worst, rel = attn_close(f64(s["out"][:, i]), f64(out), abs_tol=1e-2, row_rel=1e-2)
        assert ok, (i, worst, rel)
    assert pic.pic_device_status() == (0, 0)


def test_per_layer_frequencies(cuda_lib):
    import paper_2607_28069_gb300 as pic
    ctx, draft = [37, 500], [3, 6]
    s = draw((8, 2), 128, 0, ctx, draft, 6, True, base=1e6)
    i = torch.arange(64, dtype=torch.float64)
    table = torch.stack([1e4 ** (-2 * i / 128), 1e6 ** (-2 * i / 128)]).cuda()
    s["geom"] = pic.Geometry(2, 8, 2, 128, 77.0, layer_inv_freq=table)
    before = s["kc"].clone(), s["vc"].clone()
    call(s)
    assert pic.pic_device_status() == (0, 0)
    check(s, ctx, draft, *before)


def test_device_checks(cuda_lib):
    """A bad length, a table too short, a page outside the cache, a parent behind
    its child: reported, and the other requests served."""
    for name, code in (("length", 3), ("short", 5), ("page", 6), ("parent", 3)):
        ctx, draft = [33, 20], [3, 3]
        s = draw((4, 1), 64, 0, ctx, draft, 3, True)
        if name == "length":
            s["draft"][0] = 4
        elif name == "short":
            s["ctx"][0] = s["bt"].shape[1] * 16 - 2
        elif name == "page":
            s["bt"][0, 2] = s["num"]
        else:
            s["parent"][0, 1] = 2
        before = s["kc"].clone(), s["vc"].clone()
        call(s)
        assert cuda_lib.pic_device_status() == (code, 0), name
        if name in ("length", "short"):
            assert bool((s["out"][0] == 7).all())
            s2 = dict(s, out=s["out"][1:], lse=s["lse"][1:], q=s["q"][1:], k=s["k"][1:],
                      v=s["v"][1:], bt=s["bt"][1:], par=s["par"][1:])
            check(s2, ctx[1:], draft[1:], *before)


@pytest.mark.parametrize("ctx,at", [(100, 1), (100, 5), (9000, 300), (9000, 556)])
def test_a_bad_page_in_the_context_reads_as_zeros(cuda_lib, ctx, at):
    """Anywhere in a CTA's share: reported, and its keys and values count as zeros."""
    s = draw((4, 1), 64, 0, [ctx, 40], [2, 2], 2, False, layers=1)
    good = s["bt"][0, at].item()
    s["kc"][0, good], s["vc"][0, good] = 0, 0
    call(s)
    assert cuda_lib.pic_device_status() == (0, 0)
    out, lse = s["out"].clone(), s["lse"].clone()
    for bad in (-1, s["num"], 2 ** 31 - 1):
        s["bt"][0, at] = bad
        call(s)
        assert cuda_lib.pic_device_status() == (6, 0)
        assert torch.equal(s["out"], out) and torch.equal(s["lse"], lse)


def test_refusals(cuda_lib):
    import paper_2607_28069_gb300 as pic
    s = draw((4, 1), 64, 0, [16], [2], 2, False)
    with pytest.raises(ValueError, match="k_new has the wrong number of elements"):
        call(dict(s, k=s["k"][:, :1].contiguous()))
    with pytest.raises(ValueError, match="k_cache must be"):
        call(dict(s, kc=s["kc"][:1]))
    with pytest.raises(ValueError, match="q must be contiguous"):
        call(dict(s, q=s["q"].transpose(2, 3)))
    with pytest.raises(ValueError, match="workspace is required"):
        call(s, workspace=None)
    with pytest.raises(pic.PicError, match="workspace needs") as e:
        call(s, workspace=s["ws"][:1024])
    assert e.value.status == 4
    big = torch.zeros((1, 65, 4, 64), dtype=torch.bfloat16, device="cuda")
    kv = torch.zeros((1, 65, 1, 64), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(pic.PicError, match="max_draft 65") as e:
        pic.pic_attend_draft(s["geom"], 0, big, kv, kv, s["ctx"], s["draft"], s["bt"], s["num"],
                             s["kc"], s["vc"], big, workspace=s["ws"])
    assert e.value.status == 2
    s["layer"] = 2
    with pytest.raises(pic.PicError, match="layer 2"):
        call(s)


@pytest.mark.parametrize("ctx,at", [(100, 3), (9000, 4801)])
def test_a_nan_in_a_visible_key_shows(cuda_lib, ctx, at):
    """In the rows that see it, whether or not their keys are split over CTAs, and in no
    other row."""
    s = draw((4, 2), 64, 0, [ctx, 40], [3, 2], 3, False, layers=1)
    s["kc"][0, s["bt"][0, at // 16].long(), 1, at % 16, 5] = float("nan")
    call(s)
    bad = torch.zeros((2, 3, 4), dtype=torch.bool)
    bad[0, :, 2:] = True
    assert torch.equal(torch.isnan(s["lse"]).cpu(), bad)
    nan = torch.isnan(s["out"]).cpu()
    assert torch.equal(nan.any(-1), bad) and torch.equal(nan.all(-1), bad)


@pytest.mark.parametrize("heads,dim,ctx,T", [((4, 2), 64, 100, 9), ((4, 1), 128, 9000, 9), ((8, 1), 128, 9080, 64),
                                             ((32, 2), 64, 2040, 40), ((16, 1), 128, 0, 64), ((8, 2), 128, 250, 30)])
def test_infinities_and_nan_of_another_branch_do_not_show(cuda_lib, heads, dim, ctx, T):
    """Drafted values with infinities and NaN: rows that do not see them are, bit for bit,
    those of the same call with zeros in their places; rows that do have them where they
    are, and elsewhere the same bits.  Keys of another branch may be NaN, too."""
    lens = [T, max(1, T - 3), T]
    ctxs = [ctx, 77, 3]
    s = draw(heads, dim, 0, ctxs, lens, T, True, layers=1, seed=T)
    G, hkv = heads[0] // heads[1], heads[1]
    rng = np.random.default_rng(ctx)
    vals = torch.zeros((3, T, hkv, dim))  # what is added to the values
    for b in range(2):  # request 2 stays finite
        for i in rng.choice(lens[b], max(1, T // 6), replace=False):
            h, c = rng.integers(0, hkv), rng.choice(dim, 3, replace=False)
            vals[b, i, h, c[0]], vals[b, i, h, c[1]] = float("inf"), float("-inf")
            vals[b, i, h, c[2]] = float("nan")
    wild = vals != 0
    clean = s["v"].clone()
    clean[wild.cuda()] = 0
    kc, vc = s["kc"].clone(), s["vc"].clone()
    call(dict(s, v=clean))
    out, lse = s["out"].clone(), s["lse"].clone()
    assert bool(torch.isfinite(out.float()).all())
    dirty = clean.clone()
    dirty[wild.cuda()] = vals[wild].bfloat16().cuda()
    s2 = dict(s, v=dirty, kc=kc, vc=vc, out=torch.full_like(out, 7.0), lse=torch.full_like(lse, 7.0))
    call(s2)
    want = out.float().cpu()
    for b in range(3):
        line = line_of(s["par"][b], lens[b])
        for i in range(lens[b]):
            add = vals[b, line[i]].sum(0)  # inf - inf and NaN: NaN
            want[b, i] += add.repeat_interleave(G, 0)
    got = s2["out"].float().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(got, 1.5), torch.nan_to_num(want, 1.5))
    assert torch.equal(s2["lse"], lse)
    # the stored values are what was given
    t = torch.arange(lens[0])
    page = s["bt"].cpu()[0][(ctx + t) // 16].long()
    assert torch.equal(vc[0].cpu()[page, :, (ctx + t) % 16].view(torch.int16), dirty[0, :lens[0]].cpu().view(torch.int16))
    # a key that is NaN shows where it is seen only
    leaf = lens[0] - 1
    k = s["k"].clone()
    k[0, leaf] = float("nan")
    s3 = dict(s, k=k, v=clean, out=torch.full_like(out, 7.0), lse=torch.full_like(lse, 7.0))
    call(s3)
    rest = [i for i in range(lens[0]) if i != leaf]
    assert torch.equal(s3["out"][0, rest], out[0, rest]) and torch.equal(s3["out"][1:], out[1:])
    assert bool(torch.isnan(s3["out"][0, leaf].float()).all())
    assert cuda_lib.pic_device_status() == (0, 0)
