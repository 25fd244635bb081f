"""Source-level checks of the operators' kernels (no GPU): one that is launched ahead of its
predecessor's end (launch_next), or that lets its successor be (let_next_start), waits for its
predecessor before anything else."""
import os
import re

import pytest

from test_sources import CSRC, _kernel_bodies


def _chained(text):
    """The kernels of a source file that are launched, or let others be, ahead of time."""
    names = set(re.findall(r"\blaunch_next\(\s*(\w+)", text)) - {"void"}
    starts = [m.end() for m in re.finditer(r"__global__", text)]
    for (name, _), start, end in zip(_kernel_bodies(text), starts, starts[1:] + [len(text)]):
        if "let_next_start()" in text[start:end]:
            names.add(name)
    return names


def _early(text):
    """Those of them that do not wait first."""
    first = dict(_kernel_bodies(text))
    return sorted(n for n in _chained(text) if first.get(n) != "grid_dep_wait()")


@pytest.mark.parametrize("fname", ["embedding.cu", "distill.cu", "mx4.cu", "mx4_linear.cu"])
def test_every_chained_kernel_waits_first(fname):
    text = open(os.path.join(CSRC, fname)).read()
    assert _early(text) == []
    if fname == "embedding.cu":
        assert _chained(text) >= {"sort_count_kernel", "sort_scan_kernel", "sort_place_kernel",
                                  "count_heads_kernel", "sum_kernel", "fold_kernel", "join_kernel"}


def test_the_check_sees_a_kernel_that_reads_first():
    text = open(os.path.join(CSRC, "embedding.cu")).read()
    for name, bad in (("join_kernel", "  if (a.n == 0) return;\n"), ("sort_scan_kernel", "")):
        at = text.index("grid_dep_wait();", text.index(name + "("))
        planted = text[:at].rstrip(" ") + bad + text[at + len("grid_dep_wait();"):]
        assert _early(planted) == [name]
