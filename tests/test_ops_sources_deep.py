"""Source-level checks of the kernels for deeper models (no GPU): one that is launched ahead of
its predecessor's end waits for it before anything else, its tensor memory included, which the
predecessor may hold."""
import os
import re

import pytest

from test_sources import CSRC, _kernel_bodies

AHEAD = {"int8_linear.cu": {"tile_kernel"}, "int8_grad_weight.cu": {"weight_kernel", "join_kernel"},
         "norm.cu": {"norm_join_kernel"}, "int8_rows.cu": set()}


def _launched_ahead(text):
    """The kernels that launch_next and launch_next_cluster are given, by name or by a variable."""
    variables = {name: set(re.findall(r"(\w+_kernel)<", value)) for name, value in
                 re.findall(r"const auto (\w+) = ([^;]+_kernel<[^;]+);", text)}
    names = set()
    for m in re.finditer(r"\blaunch_next(?:_cluster)?\(([^;]+);", text):
        first = re.split(r",\s*dim3", m.group(1))[0]
        found = set(re.findall(r"\w+_kernel\b", first))
        names |= found or variables[first.strip()]
    return names


@pytest.mark.parametrize("fname", sorted(AHEAD))
def test_kernels_launched_ahead_wait_first(fname):
    text = open(os.path.join(CSRC, fname)).read()
    assert _launched_ahead(text) == AHEAD[fname]
    assert "let_next_start" not in text
    first = dict(_kernel_bodies(text))
    assert {n: first[n] for n in AHEAD[fname]} == {n: "grid_dep_wait()" for n in AHEAD[fname]}


def test_the_check_sees_a_kernel_that_reads_first():
    text = open(os.path.join(CSRC, "int8_linear.cu")).read()
    at = text.index("grid_dep_wait();")
    planted = text[:at] + "if (a.rows == 0) return;\n  " + text[at:]
    assert dict(_kernel_bodies(planted))["tile_kernel"] == "if (a.rows == 0) return"


def _first_of_its_call(text):
    """The kernels launched ahead before which their call may have launched no other."""
    bodies = re.split(r"\n}\n", text)  # functions, or what is between them
    found = set()
    for body in bodies:
        for m in re.finditer(r"\blaunch_next(?:_cluster)?\((?:(\w+_kernel)|\w+)", body):
            before = body[:m.start()]
            plain = re.search(r"<<<|prepare_operands\(|launch_grad<", before)
            # `plain` is not in a condition, or the launch is the other half of its own
            chosen = re.search(r"first \? launch_cluster\(false,[^;]*$", before)
            conditional = plain and re.search(r"if \(a\.ready\) {[^}]*$", before[:plain.start()])
            if not chosen and (not plain or conditional) and "launch_next" not in before:
                found.add(m.group(1) or "kernel")
    return found


@pytest.mark.parametrize("fname", sorted(AHEAD))
def test_kernels_launched_ahead_follow_one_of_their_call(fname):
    """launch_next's condition: its predecessor on the stream is not the caller's last kernel, of
    which nothing is known."""
    text = open(os.path.join(CSRC, fname)).read()
    # launch_tiles has its operands' kernel launched by its callers
    assert _first_of_its_call(text) <= {"tile_kernel"}
    if fname == "int8_linear.cu":
        for caller in ("launch_linear(", "agnes_int8_linear_grad_input("):
            body = text[text.rindex(caller):]
            assert re.search(r"expand_kernel<<<|prepare_operands\(", body).start() < \
                body.index("launch_product<")
    if fname == "int8_grad_weight.cu":
        assert "const bool first = direct && !a.ready;" in text
