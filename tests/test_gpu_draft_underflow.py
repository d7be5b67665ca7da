"""An infinity or NaN of a drafted value shows in every row that sees it, also where the
row's keys are split over CTAs and the weight of the part that holds it is below the
smallest number of 32 bits beside another part's."""
import pytest
import torch

from tests.test_gpu_draft import call, draw

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,dim,ctxs,T", [((4, 1), 64, [9000, 40], 3),     # four warps a row in the merge
                                              ((8, 1), 128, [40001, 77], 9),
                                              ((32, 8), 128, [3000] * 4, 5),   # one warp a row
                                              ((16, 16), 64, [2500] * 6, 4)])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan")])
def test_wild_values_under_small_weights(cuda_lib, heads, dim, ctxs, T, value):
    s = draw(heads, dim, 0, ctxs, [T] * len(ctxs), T, False, layers=1)
    # a context key that every query's score is some hundreds above all others for: queries
    # and that key alike in an element whose angle hardly turns (the last frequency)
    e = dim // 2 - 1
    for x in (s["q"], s["k"], s["kc"]):
        x[..., e], x[..., dim - 1] = 0, 0
    s["q"][..., e] = 64
    for b in range(len(ctxs)):
        page = s["bt"][b, 0].long()
        s["kc"][0, page, :, 3, e] = 128
    clean = s["v"].clone()
    call(s)
    out = s["out"].clone()
    assert bool(torch.isfinite(out.float()).all())
    s["v"] = clean
    s["v"][0, 1, -1, 7] = value
    call(s)
    assert cuda_lib.pic_device_status() == (0, 0)
    G = heads[0] // heads[1]
    got, rest = s["out"].float(), torch.ones_like(out, dtype=torch.bool)
    rest[0, 1:, -G:, 7] = False
    assert not bool(torch.isfinite(got[~rest]).any())
    assert torch.equal(torch.nan_to_num(got[~rest], 0.5, 1.5, -1.5),
                       torch.full_like(got[~rest], {float("inf"): 1.5, float("-inf"): -1.5}.get(value, 0.5)))
    assert torch.equal(s["out"][rest], out[rest])
