"""pic_page_reserve, _fork, _compact, _free and _copy against a plain model of the
tables and caches in numpy; whole numbers and copied bits have to be equal, a
re-rotated key within the relocation's bar."""
import numpy as np
import pytest
import torch

from tests.helpers import f64, kv_tolerance_ok

pytestmark = pytest.mark.gpu

PAGE = 16


class Model:
    """The plain model beside the device state."""

    def __init__(self, rows, max_pages, pages, layers=2, heads=(4, 2), dim=64, seed=0, style=0):
        import paper_2607_28069_gb300 as pic
        self.pic = pic
        self.geom = pic.Geometry(layers, heads[0], heads[1], dim, 1e4, rope_style=style)
        self.rows, self.max_pages, self.pages, self.dim, self.style = rows, max_pages, pages, dim, style
        self.bt = np.full((rows, max_pages), -1, np.int64)
        self.ctx = np.zeros(rows, np.int64)
        self.refs = np.zeros(pages, np.int64)
        gen = torch.Generator(device="cuda").manual_seed(seed)
        shape = (layers, pages, heads[1], PAGE, dim)
        self.dk, self.dv = (torch.randn(shape, generator=gen, device="cuda").bfloat16() for _ in "kv")
        self.rng = np.random.default_rng(seed)
        self.up()

    def i32(self, x):
        return torch.as_tensor(np.asarray(x), dtype=torch.int32).cuda()

    def up(self):
        self.dbt, self.dctx, self.drefs = self.i32(self.bt), self.i32(self.ctx), self.i32(self.refs)
        self.k, self.v = self.dk.cpu(), self.dv.cpu()

    def place(self, row, length, spare=0):
        """A context of `length` positions on random free pages."""
        n = -(-(length + spare) // PAGE)
        free = self.rng.permutation(np.flatnonzero(self.refs == 0))[:n]
        self.bt[row, :n] = free
        self.refs[free] = 1
        self.ctx[row] = length

    def check(self, code=(0, 0), keys=True):
        assert self.pic.pic_device_status() == code
        assert np.array_equal(self.dbt.cpu().numpy(), self.bt)
        assert np.array_equal(self.dctx.cpu().numpy(), self.ctx)
        assert np.array_equal(self.drefs.cpu().numpy(), self.refs)
        assert np.array_equal(self.refs, np.bincount(self.bt[self.bt >= 0].ravel(),
                                                     minlength=self.pages)) or code[0] == 6
        if keys:
            assert torch.equal(self.dk.cpu(), self.k)
        assert torch.equal(self.dv.cpu(), self.v)

    def take(self, needs):
        """Pages for each need, in order; None for one that does not fit."""
        free = np.flatnonzero(self.refs == 0).tolist()
        at, got = 0, []
        for n in needs:
            got.append(free[at:at + n] if at + n <= len(free) or n == 0 else None)
            at += n
        return got

    def reserve(self, rows, extra):
        res = self.i32([77] * len(rows))
        self.pic.pic_page_reserve(self.i32(rows), extra, self.dctx, self.dbt, self.pages, self.drefs, res)
        want = [-(-(int(self.ctx[r]) + extra) // PAGE) for r in rows]
        lack = [max(0, w - max(int((self.bt[r] >= 0).sum()), -(-int(self.ctx[r]) // PAGE)))
                for r, w in zip(rows, want)]
        out = []
        for r, w, n, pg in zip(rows, want, lack, self.take(lack)):
            out.append(-1 if pg is None else w)
            if pg:
                self.bt[r, w - n:w] = pg
                self.refs[pg] = 1
        assert res.cpu().tolist() == out
        return out

    def fork(self, src, dst, reserve=0, layers=None):
        res = self.i32([77] * len(src))
        lo, hi = layers or (0, self.geom.num_layers)
        self.pic.pic_page_fork(self.geom, self.i32(src), self.i32(dst), self.dctx, self.dbt, self.pages,
                               self.drefs, self.dk, self.dv, res, reserve=reserve, layer_begin=lo,
                               layer_end=hi)
        full = [int(self.ctx[a]) // PAGE for a in src]
        need = [-(-(int(self.ctx[a]) + reserve) // PAGE) - f for a, f in zip(src, full)]
        out = []
        for a, z, f, n, pg in zip(src, dst, full, need, self.take(need)):
            out.append(-1 if pg is None else int(self.ctx[a]))
            if pg is None:
                continue
            self.bt[z, :f] = self.bt[a, :f]
            self.refs[self.bt[a, :f]] += 1
            self.bt[z, f:f + n] = pg
            self.refs[pg] += 1
            self.ctx[z] = self.ctx[a]
            r = int(self.ctx[a]) % PAGE
            if r:
                for c in (self.k, self.v):
                    c[lo:hi, pg[0], :, :r] = c[lo:hi, self.bt[a, f], :, :r]
        assert res.cpu().tolist() == out
        return out

    def free(self, rows):
        self.pic.pic_page_free(self.i32(rows), self.dbt, self.pages, self.drefs, self.dctx)
        for r in rows:
            np.subtract.at(self.refs, self.bt[r][self.bt[r] >= 0], 1)
            self.bt[r] = -1
            self.ctx[r] = 0

    def compact(self, rows, keep, start=None, reserve=0, rotate=False, layers=None):
        n = len(rows)
        width = max(1, max(len(x) for x in keep))
        kl = np.full((n, width), -5, np.int64)
        for i, x in enumerate(keep):
            kl[i, :len(x)] = x
        res = self.i32([77] * n)
        ws = torch.full((self.pic.pic_page_compact_workspace_size(self.geom, n, width),), 255,
                        dtype=torch.uint8, device="cuda")
        lo, hi = layers or (0, self.geom.num_layers)
        self.pic.pic_page_compact(
            self.geom, self.i32(rows), self.i32(kl), self.i32([len(x) for x in keep]), self.dctx,
            self.dbt, self.pages, self.drefs, self.dk, self.dv, res, workspace=ws,
            start=None if start is None else self.i32(start), reserve=reserve, rotate=rotate,
            layer_begin=lo, layer_end=hi)
        moves = []
        for i, r in enumerate(rows):
            s = int(self.ctx[r]) if start is None else start[i]
            old, new = s + np.asarray(keep[i], np.int64), s + np.arange(len(keep[i]))
            t = self.bt[r]
            if len(old):
                a, z = t[old // PAGE], t[new // PAGE]
                k, v = self.k[lo:hi, a, :, old % PAGE].clone(), self.v[lo:hi, a, :, old % PAGE].clone()
                self.k[lo:hi, z, :, new % PAGE] = k
                self.v[lo:hi, z, :, new % PAGE] = v
                moves.append((z, new, old, lo, hi))
            self.ctx[r] = s + len(old)
            cut = -(-(int(self.ctx[r]) + reserve) // PAGE)
            gone = t[cut:][t[cut:] >= 0]
            self.refs[gone] -= 1
            t[cut:] = -1
        assert res.cpu().tolist() == [int(self.ctx[r]) for r in rows]
        if not rotate:
            return
        for z, new, old, lo, hi in moves:  # the moved keys against 64 bits, then taken over
            x = self.k[lo:hi, z, :, new % PAGE].double().numpy()  # [n][layers][hkv][d]
            d = self.dim
            w = np.exp(1j * (new - old)[:, None, None, None] * 1e4 ** (-2.0 * np.arange(d // 2) / d))
            if self.style == 0:
                c = (x[..., :d // 2] + 1j * x[..., d // 2:]) * w
                x = np.concatenate([c.real, c.imag], -1)
            else:
                c = (x[..., 0::2] + 1j * x[..., 1::2]) * w
                x = np.stack([c.real, c.imag], -1).reshape(x.shape)
            got = self.dk.cpu()[lo:hi, z, :, new % PAGE]
            ok, worst = kv_tolerance_ok(f64(got), x)
            assert ok, worst
            same = torch.as_tensor(new == old)
            assert torch.equal(got[same], self.k[lo:hi, z, :, new % PAGE][same])  # unmoved: no bit changes
            self.k[lo:hi, z, :, new % PAGE] = got


def test_reserve_takes_the_lowest_free_pages(cuda_lib):
    m = Model(5, 40, 5000)
    for r, n in enumerate([0, 1, 16, 17, 100]):
        m.place(r, n)
    m.up()
    assert m.reserve([3, 0, 4, 1, 2], 40) == [4, 3, 9, 3, 4]
    m.check()
    m.reserve([0, 1, 2, 3, 4], 40)  # nothing lacks any more
    m.check()
    m.reserve([2], 500)
    m.check()


def test_reserve_refuses_what_does_not_fit(cuda_lib):
    m = Model(4, 8, 10)
    m.place(0, 30)
    m.place(2, 5)
    m.up()
    # 10 pages, 3 used: 5 for row 1, then 4 are asked for by row 0 and none is left for row 3
    assert m.reserve([1, 0, 3], 80) == [5, -1, -1]
    assert m.pic.pic_device_status()[0] == 10
    m.check()
    assert m.reserve([2], 0) == [1]
    m.check()
    res = m.i32([5, 5, 5])
    m.pic.pic_page_reserve(m.i32([4, -1, 0]), 200, m.dctx, m.dbt, m.pages, m.drefs, res)
    assert res.cpu().tolist() == [-1, -1, -1] and m.pic.pic_device_status()[0] in (3, 5)
    m.check()


@pytest.mark.parametrize("dim,hkv", [(64, 1), (128, 3)])
def test_fork_shares_full_pages_and_copies_the_last(cuda_lib, dim, hkv):
    m = Model(12, 70, 300, layers=3, heads=(hkv, hkv), dim=dim)
    for r, n in enumerate([0, 5, 16, 1003]):
        m.place(r, n, spare=9)
    m.up()
    m.fork([3, 3, 1, 0, 2], [4, 11, 5, 6, 7], reserve=20)
    m.check()
    m.fork([4, 3], [8, 9], layers=(1, 2))  # a branch of a branch, one layer, no room
    m.check()
    m.free([3, 5, 8])
    m.check()
    m.fork([4], [3], reserve=1)
    m.check()


def test_fork_refusals(cuda_lib):
    m = Model(6, 8, 9)
    m.place(0, 50)
    m.place(1, 20)
    m.up()
    # four pages of row 0 (one partial) and two of row 1 leave three: two branches of row 0 with
    # room for 20 take two each, the second does not fit
    assert m.fork([0, 0], [2, 3], reserve=20) == [50, -1]
    assert m.pic.pic_device_status() == (10, 1)
    m.check()
    for src, dst, reserve, code in ((0, 1, 0, 3), (0, 0, 0, 3), (6, 3, 0, 3), (0, -1, 0, 3),
                                    (0, 3, 100, 5)):
        res = m.i32([5])
        m.pic.pic_page_fork(m.geom, m.i32([src]), m.i32([dst]), m.dctx, m.dbt, m.pages, m.drefs, m.dk,
                            m.dv, res, reserve=reserve)
        assert res.item() == -1 and m.pic.pic_device_status() == (code, 0)
        m.check()


def test_free_counts_every_user(cuda_lib):
    m = Model(4, 600, 700)
    m.place(0, 9000)
    m.up()
    m.fork([0, 0], [1, 2])
    m.free([0, 3])
    m.check()
    assert (m.refs > 0).sum() == 562 + 2
    m.free([1, 2])
    m.check()
    assert m.refs.sum() == 0
    m.pic.pic_page_free(m.i32([4]), m.dbt, m.pages, m.drefs, m.dctx)
    assert m.pic.pic_device_status() == (3, 0)
    # a page that nobody uses and a page that is none: reported, counts left alone
    m.dbt[0, 0], m.dbt[1, 0] = 3, 700
    m.pic.pic_page_free(m.i32([0, 1]), m.dbt, m.pages, m.drefs, m.dctx)
    assert m.pic.pic_device_status()[0] == 6
    m.check()


@pytest.mark.parametrize("dim,hkv,style", [(64, 2, 0), (128, 8, 0), (128, 20, 1), (64, 17, 1)])
@pytest.mark.parametrize("rotate", [False, True])
def test_compact(cuda_lib, dim, hkv, style, rotate):
    """Short windows (one CTA's worth) and long ones whose sources and targets
    overlap, kept lists dense, sparse, whole and empty."""
    m = Model(5, 80, 300, layers=2, heads=(hkv, hkv), dim=dim, style=style)
    for r, n in enumerate([0, 37, 160, 1200, 7]):
        m.place(r, n, spare=64)
    m.up()
    m.compact([1, 0, 2], [[0, 2, 3, 9], [5], []], rotate=rotate)
    m.check()
    m.compact([3], [np.sort(m.rng.choice(1150, 700, replace=False)).tolist()], start=[13],
              rotate=rotate)
    m.check()
    m.compact([2, 4], [list(range(100)) + list(range(101, 150)), [0, 1, 2]], start=[3, 4], reserve=40,
              rotate=rotate)
    m.check()
    m.compact([2], [list(range(90, 120))], start=[0], rotate=rotate, layers=(1, 2))
    m.check()
    for n in (16, 17, 32, 33, 63, 64, 65, 80, 81):  # one to five segments, both forms' limits
        m.compact([3], [[0] + list(range(n // 2, n // 2 + n - 1))], start=[100], reserve=300, rotate=rotate)
        m.check()


@pytest.mark.parametrize("dim,hkv,layers", [(64, 1, 21), (64, 2, 14), (64, 3, 13), (128, 1, 11), (128, 2, 9)])
def test_compact_long_lists_of_narrow_rows(cuda_lib, dim, hkv, layers):
    """Several layers a CTA, the last group with fewer, in part of the layers too."""
    m = Model(3, 70, 300, layers=layers, heads=(hkv, hkv), dim=dim)
    for r in range(3):
        m.place(r, 1000)
    m.up()
    m.compact([2, 0, 1], [np.sort(m.rng.choice(990, n, replace=False)).tolist() for n in (800, 33, 640)],
              start=[3, 10, 1], rotate=True)
    m.check()
    m.compact([2], [list(range(1, 700, 2))], start=[50], rotate=False, layers=(2, layers))
    m.check()


def test_compact_many_rows_at_once(cuda_lib):
    m = Model(64, 20, 2000, layers=3, heads=(8, 8), dim=128)
    for r in range(64):
        m.place(r, 3 * r, spare=64)
    m.up()
    keep = [np.sort(m.rng.choice(64, m.rng.integers(1, 65), replace=False)).tolist() for _ in range(64)]
    m.compact(m.rng.permutation(64).tolist(), keep)
    m.check()


def test_compact_refusals_leave_the_row_alone(cuda_lib):
    m = Model(6, 8, 30)
    m.place(0, 60, spare=16)
    m.place(1, 60, spare=16)
    m.up()
    m.fork([0], [2])
    m.check()
    for row, keep, start, code in ((1, [3, 2], 0, 7), (1, [-1, 2], 0, 7), (1, [1, 1], 0, 7),
                                   (1, [0, 79], 70, 5), (1, [0, 100], 0, 6), (6, [0], 0, 3),
                                   (0, [0], -1, 3),
                                   (0, [1], 0, 9),      # into a page that row 2 reads too
                                   (2, [0, 1, 9], 20, 9)):
        res = m.i32([5])
        m.pic.pic_page_compact(m.geom, m.i32([row]), m.i32([keep]), m.i32([len(keep)]), m.dctx, m.dbt,
                               m.pages, m.drefs, m.dk, m.dv, res, start=m.i32([start]))
        assert res.item() == -1, (row, keep)
        assert m.pic.pic_device_status() == (code, 0), (row, keep)
        m.check()
    m.compact([0], [list(range(20))], start=[10])
    m.check()


def test_copy_between_and_within_caches(cuda_lib):
    for dim, hkv in ((64, 1), (64, 3), (128, 8)):
        m = Model(1, 1, 40, layers=3, heads=(hkv, hkv), dim=dim)
        to_k, to_v = (torch.zeros((3, 25, hkv, PAGE, dim), dtype=torch.bfloat16, device="cuda")
                      for _ in "kv")
        m.pic.pic_page_copy(m.geom, m.i32([3, -1, 39, 0, 7]), m.i32([24, -1, 0, 5, 6]), m.dk, m.dv, to_k,
                            to_v, layer_begin=1)
        assert m.pic.pic_device_status() == (0, 0)
        for to, frm in ((to_k, m.dk), (to_v, m.dv)):
            want = torch.zeros_like(to)
            want[1:, [24, 0, 5, 6]] = frm[1:, [3, 39, 0, 7]]
            assert torch.equal(to, want)
        m.pic.pic_page_copy(m.geom, m.i32([1, 2]), m.i32([5, 4]), m.dk, m.dv, m.dk, m.dv)
        m.k[:, [5, 4]], m.v[:, [5, 4]] = m.k[:, [1, 2]], m.v[:, [1, 2]]
        m.check()
        m.pic.pic_page_copy(m.geom, m.i32([1, 40, 2]), m.i32([25, 3, -1]), m.dk, m.dv, to_k, to_v)
        assert m.pic.pic_device_status()[0] == 6
        m.pic.pic_page_copy(m.geom, m.i32([]), m.i32([]), m.dk, m.dv, to_k, to_v)
        m.check()


def test_a_long_run_of_mixed_calls(cuda_lib):
    """Random calls one after the other, the device state against the model after
    each."""
    m = Model(20, 24, 260, layers=2, heads=(2, 2), dim=64, seed=4)
    for r in range(6):
        m.place(r, int(m.rng.integers(1, 200)))
    m.up()
    for step in range(60):
        live = [r for r in range(20) if m.bt[r, 0] >= 0 or m.ctx[r] > 0]
        idle = [r for r in range(20) if m.bt[r, 0] < 0]
        op = step % 4
        if op == 0 and live:
            m.reserve(m.rng.choice(live, min(3, len(live)), replace=False).tolist(), 20)
        elif op == 1 and live and idle:
            n = min(2, len(idle))
            src = [r for r in m.rng.choice(live, n).tolist() if m.ctx[r] < 320]
            m.fork(src, idle[:len(src)], reserve=30)
        elif op == 2:
            rows = [r for r in live if m.ctx[r] < 300 and
                    (m.bt[r] >= 0).sum() * PAGE >= m.ctx[r] + 8 and
                    all(m.refs[m.bt[r, p]] == 1 for p in range(m.ctx[r] // PAGE,
                                                              (m.ctx[r] + 7) // PAGE + 1))]
            if rows:
                m.compact(rows, [[0, 3, 4, 7][:m.rng.integers(1, 5)] for _ in rows], reserve=8)
        elif live and len(live) > 10:
            m.free(m.rng.choice(live, 4, replace=False).tolist())
        status = m.pic.pic_device_status()
        assert status[0] in (0, 10)
        m.check()


def test_refusals_on_the_host(cuda_lib):
    m = Model(2, 4, 10)
    res = m.i32([0])
    with pytest.raises(ValueError, match="page_refs has the wrong number"):
        m.pic.pic_page_reserve(m.i32([0]), 1, m.dctx, m.dbt, 11, m.drefs, res)
    with pytest.raises(ValueError, match="ctx_len must have an entry per row"):
        m.pic.pic_page_free(m.i32([0]), m.dbt, 10, m.drefs, m.dctx[:1])
    with pytest.raises(m.pic.PicError, match="extra -1 is negative"):
        m.pic.pic_page_reserve(m.i32([0]), -1, m.dctx, m.dbt, 10, m.drefs, res)
    with pytest.raises(m.pic.PicError, match="4097 rows"):
        m.pic.pic_page_free(m.i32([0] * 4097), m.dbt, 10, m.drefs, m.dctx)
    with pytest.raises(m.pic.PicError, match="workspace needs") as e:
        m.pic.pic_page_compact(m.geom, m.i32([0]), m.i32([[0] * 65]), m.i32([1]), m.dctx, m.dbt, 10,
                               m.drefs, m.dk, m.dv, res)
    assert e.value.status == 4
    with pytest.raises(m.pic.PicError, match=r"layers \[1, 3\)"):
        m.pic.pic_page_copy(m.geom, m.i32([0]), m.i32([1]), m.dk, m.dv, m.dk, m.dv, 1, 3)
    with pytest.raises(ValueError, match="k_dst must be"):
        m.pic.pic_page_copy(m.geom, m.i32([0]), m.i32([1]), m.dk, m.dv, m.dk[:1], m.dv[:1])


@pytest.mark.parametrize("pages,used", [(32767, 32700), (32768, 32760), (70000, 65530), (140000, 131072)])
@pytest.mark.parametrize("shift", [0, 1])
def test_large_pools(cuda_lib, pages, used, shift):
    """Free pages near the end, and a few scattered ones where `shift` leaves the counts
    unaligned too."""
    import paper_2607_28069_gb300 as pic
    refs = torch.ones(pages + shift, dtype=torch.int32, device="cuda")[shift:]
    refs[used:] = 0
    refs[used + 1:used + 4] = 7
    if shift:
        refs[used // 2] = 0
    free = torch.nonzero(refs == 0)[:8, 0].tolist()  # may be fewer than are asked for
    dev = lambda x: torch.as_tensor(x, dtype=torch.int32).cuda()  # noqa: E731
    bt, ctx = dev([[-1] * 8, [5, 6, 7] + [-1] * 5, [-1] * 8]), dev([0, 33, 0])
    row, res, want = dev([2, 1, 0]), dev([9] * 3), refs.clone()
    pic.pic_page_reserve(row, 40, ctx, bt, pages, refs, res)
    exp = [[-1] * 8, [5, 6, 7] + free[3:5] + [-1] * 3, free[:3] + [-1] * 5]
    if len(free) == 8:
        exp[0] = free[5:] + [-1] * 5
    assert cuda_lib.pic_device_status() == ((0, 0) if len(free) == 8 else (10, 2))
    assert res.tolist() == [3, 5, 3 if len(free) == 8 else -1]
    assert bt.tolist() == exp
    want[torch.as_tensor(free[:8 if len(free) == 8 else 5], device="cuda")] = 1
    assert torch.equal(refs, want)
