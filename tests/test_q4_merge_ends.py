"""The merge of attention over the 4-bit paged cache takes the numbers of a unit's workers from the workspace.  Where a bounded wait of the streaming
kernel gave up, nobody has written them: whatever lies there then may not become an address."""
import os
import re
import subprocess

from paper_2605_23258_b200 import build

HEADER = os.path.join(build.CSRC, "decode_q4.cuh")


def test_which_numbers_are_workers(tmp_path):
    """The kernel's own check, by the compiler: garbage is none, and what passes stays within the workspace's records, one for every unit and worker."""
    source = tmp_path / "ends.cu"
    yes = [(0, 0, 1), (0, 1775, 1776), (1775, 1775, 1776), (3, 40, 1776)]
    no = [(-1, 0, 1776), (0, 1776, 1776), (5, 4, 1776), (0, -1, 1776), (-2147483647 - 1, 2147483647, 1776), (2147483647, -2147483647 - 1, 1776), (0, 2147483647, 1776),
          (2147483647, 2147483647, 1776), (-5, -3, 1776), (0, 0, 0)]
    source.write_text('#include "decode_q4.cuh"\n' + "".join(f"static_assert({'' if ok else '!'}vec::dq4::ends_are_workers({a}, {b}, {n}));\n"
                                                              for ok, cases in ((True, yes), (False, no)) for a, b, n in cases))
    done = subprocess.run([build._nvcc(), *build.NVCC_FLAGS, "-c", str(source), "-o", str(tmp_path / "ends.o")], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert done.returncode == 0, done.stdout


def test_no_address_before_the_check():
    """In the merge, what is read of the ends before the check is the numbers themselves; the check leaves the unit."""
    text = re.sub(r"//[^\n]*", "", open(HEADER).read())
    body = text[text.index("decode_q4_merge("):]
    read, check = body.index("const int2 ends ="), body.index("if (!ends_are_workers(ends.x, ends.y, workers))")
    assert not re.search(r"\bends\b", body[read + len("const int2 ends ="):check])
    left = re.match(r"if \(!ends_are_workers\(ends\.x, ends\.y, workers\)\) \{.*?\n        \}", body[check:], re.S).group(0)
    assert left.rstrip("} \n").endswith("continue;") and "records" not in left
    assert re.search(r"\bends\.", body[check + len(left):])


def test_the_workspace_has_a_record_for_each_of_them():
    """The number of workers that the merge is given is the streaming grid's, and no more than the workspace is made for."""
    text = open(os.path.join(build.CSRC, "decode_q4.cu")).read()
    assert "merge<T, D>(sm_count() * C::WARPS)" in text and "dim3(sm_count()), dim3(C::THREADS)" in text
    assert "C::WARPS <= MOST_WARPS" in text and "((size_t)dm.U + sm_count() * MOST_WARPS)" in text
