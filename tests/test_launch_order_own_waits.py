"""Order of waits in the kernels that set something up ahead of a griddepcontrol.wait of their own,
without pdl_entry (no GPU): until that wait they touch none of their parameters, the
descriptors' prefetch and the status word aside, and they let no later launch begin.  (Kernels
whose own body holds the wait; the prefill's attention has it in a function.)"""
import glob
import os
import re

from tests.test_launch_order import CSRC


def kernels(text):
    """(name or line, parameters, body) of every __global__ function in a source."""
    text = re.sub(r"//[^\n]*", "", text)
    for m in re.finditer(r"__global__", text):
        head = re.compile(r"(\w+)\(([\w:<>*&,\s]*)\)\s*\{").search(text, m.end())
        at, depth = head.end(), 1
        while depth:
            depth += {"{": 1, "}": -1}.get(text[at], 0)
            at += 1
        yield head[1], [re.search(r"(\w+)\s*$", x)[1] for x in head[2].split(",") if x.strip()], text[head.end():at - 1]


def ahead_of_wait(params, body):
    """What a kernel with a wait of its own touches too early: a list, None without such a wait."""
    if "griddepcontrol.wait" not in body or "pdl_entry()" in body:
        return None
    early = body[:body.rindex("griddepcontrol.wait")]
    early = re.sub(r"\b(prefetch_tmap|dev_fail|static_assert)\([^;]*;", "", early)
    return [x for x in params if re.search(rf"\b{x}\b", early)] + re.findall(r"griddepcontrol.launch_dependents", early)


def test_kernels_with_a_wait_of_their_own():
    seen = []
    for path in sorted(glob.glob(os.path.join(CSRC, "*.cu"))):
        for name, params, body in kernels(open(path).read()):
            found = ahead_of_wait(params, body)
            assert not found, (path, name, found)
            if found is not None:
                seen.append((os.path.basename(path), name))
    for kernel in (("pic_share_attend.cu", "attend_kernel"), ("pic_draft.cu", "draft_attn_kernel"),
                   ("pic_draft.cu", "draft_merge_kernel"), ("pic_prefill.cu", "combine_kernel"),
                   ("pic_decode.cu", "decode_attn_kernel"), ("pic_decode.cu", "decode_combine_kernel"),
                   ("pic_link.cu", "link_kernel")):
        assert kernel in seen, (kernel, seen)


def test_a_read_ahead_of_the_wait_is_seen():
    """The same source with the plan's first read moved up, and with an early trigger."""
    text = open(os.path.join(CSRC, "pic_share_attend.cu")).read()
    for extra, found in (("Segments sg(p, 0);", ["p"]), ("const int page = p.block_table[0];", ["p"]),
                         ('asm volatile("griddepcontrol.launch_dependents;" ::: "memory");', ["griddepcontrol.launch_dependents"])):
        moved = text.replace("  tc_fence_before();\n  __syncthreads();\n  tc_fence_after();\n",
                             f"  {extra}\n  tc_fence_before();\n  __syncthreads();\n  tc_fence_after();\n", 1)
        assert moved != text
        got = {name: ahead_of_wait(params, body) for name, params, body in kernels(moved)}
        assert got["attend_kernel"] == found and got["merge_kernel"] is None
