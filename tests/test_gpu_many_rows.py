"""pic_page_* with as many rows as a call may list: more than the planning CTA has threads,
and the shared memory of its lists above and below what a launch has by default."""
import os
import subprocess
import sys

import numpy as np
import pytest

from tests.test_gpu_pages import Model

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def model(n, pages):
    """Contexts of 0 to 50 positions in rows 0 .. 8, the others empty."""
    m = Model(n + 9, 8, pages, layers=1, heads=(1, 1), dim=64, seed=n)
    for r, length in enumerate([0, 1, 15, 16, 17, 31, 32, 40, 50]):
        m.place(r, length)
    m.up()
    return m


def checked(m, out):
    """The state, and the status: one of the rows that did not fit, if there are any."""
    status = m.pic.pic_device_status()
    assert status == (0, 0) if -1 not in out else status[0] == 10 and out[status[1]] == -1
    m.check()


def forks(n, short=0):
    """n branches of nine contexts, in any order of rows; the last ones do not fit where
    pages are short."""
    m = model(n, 3 * n + 30 - short)
    dst = 9 + m.rng.permutation(n)
    out = m.fork(m.rng.integers(0, 9, n).tolist(), dst.tolist(), reserve=20)
    assert (-1 in out) == (short > 0)
    checked(m, out)
    m.free(dst.tolist())
    m.check()


def reserves(n, short=0):
    m = model(n, 3 * n + 30 - short)
    rows = m.rng.permutation(n + 9)[:n].tolist()
    m.ctx[9:] = 0
    out = m.reserve(rows, 33)
    assert (-1 in out) == (short > 0)
    checked(m, out)


@pytest.mark.parametrize("n", [1023, 1024, 1025, 2049, 4074, 4096])
def test_forks(cuda_lib, n):
    forks(n)


@pytest.mark.parametrize("n", [4075, 4080, 4095])
def test_forks_in_a_new_process(cuda_lib, n):
    """Before any larger call has asked for more shared memory."""
    run = subprocess.run([sys.executable, "-c", f"from tests.test_gpu_many_rows import forks; forks({n})"],
                         cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stderr[-2000:]


@pytest.mark.parametrize("n", [1025, 4096])
def test_reserves(cuda_lib, n):
    reserves(n)


@pytest.mark.parametrize("what", [forks, reserves])
def test_pages_run_out_behind_the_first_thousand_rows(cuda_lib, what):
    what(2200, short=2200)


@pytest.mark.parametrize("n", [1025, 4096])
def test_compactions(cuda_lib, n):
    m = Model(n, 6, 6 * n, layers=1, heads=(1, 1), dim=64)
    for r in range(n):
        m.place(r, r % 50, spare=20)
    m.up()
    lists = [np.sort(m.rng.choice(20, m.rng.integers(0, 6), replace=False)).tolist() for _ in range(n)]
    m.compact(m.rng.permutation(n).tolist(), lists)
    m.check()
    lists = [list(range(r % 3, int(m.ctx[r]), 2)) for r in range(n)]
    m.compact(list(range(n)), lists, start=[0] * n)
    m.check()
