"""CPU: the sources that bench.py's stored profiles are tied to are those of the kernels it times."""
import os
import re
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)
import bench as B  # noqa: E402

CSRC = os.path.join("paper_2511_20982_amd", "csrc")


def includes(rel):
    with open(os.path.join(ROOT, rel)) as f:
        names = re.findall(r'^\s*#\s*include\s+"([^"]+)"', f.read(), re.M)
    return [os.path.normpath(os.path.join(os.path.dirname(rel), x)) for x in names if x != "dopd_attn.h"]


def test_every_source_of_the_timed_kernels_is_listed():
    seen, todo = set(), [os.path.join(CSRC, "dopd_attn.hip")]
    while todo:
        rel = todo.pop()
        if rel not in seen:
            seen.add(rel)
            todo += includes(rel)
    assert seen == set(B.KERNEL_SOURCES)


def test_the_library_s_unit_has_nothing_in_front_of_them():
    rel = os.path.join(CSRC, "library.hip")
    with open(os.path.join(ROOT, rel)) as f:
        code = [x.strip() for x in f if x.strip() and not x.startswith("//")]
    assert code[0] == '#include "dopd_attn.hip"'
    assert all(re.fullmatch(r'#include "[\w/.]+"', x) for x in code)
