"""pic_compose with document lists whose offsets fill the shared memory that a launch has by
default: in a new process, before any larger call has asked for more."""
import os
import subprocess
import sys

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def compose(max_docs):
    """Documents of 1 to 3 tokens behind a prefix of 5, 4 query tokens: offsets and length."""
    import torch

    import paper_2607_28069_gb300 as pic
    dev = lambda x, t=torch.int32: torch.as_tensor(np.asarray(x), dtype=t).cuda()  # noqa: E731
    lens = np.arange(max_docs) % 3 + 1
    offs = 5 + np.cumsum(lens) - lens
    ctx = int(5 + lens.sum() + 4)
    pages = -(-ctx // 16)
    out = lambda *s, t=torch.int32: torch.full(s, 77, dtype=t, device="cuda")  # noqa: E731
    doc_offset, doc_delta, inline_pos, ctx_len = out(1, max_docs), out(1, max_docs), out(1, 16), out(1)
    slots, tok = out(1, ctx, t=torch.int64), out(1, ctx, t=torch.int64)
    pic.pic_compose(pic.Geometry(1, 1, 1, 64, 1e4), dev(lens), dev(np.zeros(max_docs)),
                    dev(np.cumsum(lens) - lens, torch.int64), dev(np.arange(max_docs)[None]), dev([max_docs]),
                    dev([5]), dev([4]), dev(np.arange(pages)[None]), pages, ctx, 16, doc_offset, doc_delta,
                    slots, tok, inline_pos, ctx_len)
    assert pic.pic_device_status() == (0, 0)
    assert ctx_len.tolist() == [ctx] and slots[0].tolist() == list(range(ctx))
    assert doc_offset[0].tolist() == offs.tolist()


@pytest.mark.parametrize("max_docs", [2452, 2453, 2456, 2457, 8192])
def test_long_document_lists(cuda_lib, max_docs):
    run = subprocess.run([sys.executable, "-c", f"from tests.test_gpu_compose_docs import compose; compose({max_docs})"],
                         cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stderr[-2000:]
