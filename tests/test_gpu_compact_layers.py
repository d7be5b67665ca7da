"""pic_page_compact with frequencies of each layer's own: moved keys against the 64-bit
rotation by their layer's frequencies, in part of the layers too."""
import numpy as np
import pytest
import torch

from tests.helpers import f64, kv_tolerance_ok

pytestmark = pytest.mark.gpu


def turned(x, delta, freq, style):
    """R(delta) of rows x [n][hkv][d]."""
    w = np.exp(1j * delta[:, None, None] * freq)
    d = x.shape[-1]
    if style == 0:
        c = (x[..., :d // 2] + 1j * x[..., d // 2:]) * w
        return np.concatenate([c.real, c.imag], -1)
    c = (x[..., 0::2] + 1j * x[..., 1::2]) * w
    return np.stack([c.real, c.imag], -1).reshape(x.shape)


@pytest.mark.parametrize("dim,hkv,style", [(64, 1, 0), (64, 2, 1), (128, 1, 1), (128, 9, 0)])
@pytest.mark.parametrize("form", ["short", "long"])
@pytest.mark.parametrize("layers", [(0, 13), (5, 12), (12, 13)])
def test_moved_keys_turn_by_their_layer(cuda_lib, dim, hkv, style, form, layers):
    import paper_2607_28069_gb300 as pic
    L, rows, per = 13, 2, 70
    rng = np.random.default_rng(dim + hkv)
    gen = torch.Generator(device="cuda").manual_seed(dim)
    pages = rows * per + 5
    k, v = (torch.randn((L, pages, hkv, 16, dim), generator=gen, device="cuda").bfloat16() for _ in "kv")
    bases = 10.0 ** np.linspace(2, 6, L)
    freq = bases[:, None] ** (-2.0 * np.arange(dim // 2) / dim)
    geom = pic.Geometry(L, hkv, hkv, dim, 77.0, rope_style=style, layer_inv_freq=torch.as_tensor(freq).cuda())
    i32 = lambda x: torch.as_tensor(np.asarray(x), dtype=torch.int32).cuda()  # noqa: E731
    bt = rng.permutation(pages)[:rows * per].reshape(rows, per)
    refs = np.zeros(pages, np.int64)
    refs[bt] = 1
    m, window = (50, 900) if form == "short" else (601, 1000)
    start = [21, 64]
    keep = np.stack([np.sort(rng.choice(window, m, replace=False)) for _ in range(rows)])
    keep[1] = np.sort(np.concatenate([np.arange(30), 30 + rng.choice(window - 30, m - 30, replace=False)]))  # 30 positions stay
    ctx, dbt, drefs, res = i32([1100, 1100]), i32(bt), i32(refs), i32([7, 7])
    k0, v0 = k.cpu(), v.cpu()
    ws = torch.empty(pic.pic_page_compact_workspace_size(geom, rows, m), dtype=torch.uint8, device="cuda")
    lo, hi = layers
    pic.pic_page_compact(geom, i32([0, 1]), i32(keep), i32([m, m]), ctx, dbt, pages, drefs, k, v, res,
                         start=i32(start), rotate=True, workspace=ws, layer_begin=lo, layer_end=hi)
    assert cuda_lib.pic_device_status() == (0, 0) and res.tolist() == [s + m for s in start]
    k1, v1 = k.cpu(), v.cpu()
    want_v, rest = v0.clone(), torch.ones((L, pages, 16), dtype=torch.bool)
    for r in range(rows):
        old, new = start[r] + keep[r], start[r] + np.arange(m)
        a, z = bt[r][old // 16], bt[r][new // 16]
        want_v[lo:hi, z, :, new % 16] = v0[lo:hi, a, :, old % 16]
        rest[lo:hi, z, new % 16] = False
        stay = torch.as_tensor(new == old)
        for layer in range(lo, hi):
            was, got = k0[layer, a, :, old % 16], k1[layer, z, :, new % 16]
            ok, worst = kv_tolerance_ok(f64(got), turned(f64(was), new - old, freq[layer], style))
            assert ok, (layer, r, worst)
            assert torch.equal(got[stay], was[stay])
    assert torch.equal(v1, want_v)
    same = (k1.view(torch.int16) == k0.view(torch.int16)).permute(0, 1, 3, 2, 4)
    assert bool(same[rest].all())
