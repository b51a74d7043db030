"""The layer for a few tokens reads its input before its own wait for the kernels before it: what that rests on, in the sources."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "paper_2609_04609_b200", "csrc")


def _read(name):
    with open(os.path.join(CSRC, name)) as f:
        return f.read()


def _statements(source, kernel):
    """What the body of a kernel begins with, comments left out."""
    body = re.sub(r"//[^\n]*", "", source[source.index(kernel + "(const") :])
    body = body[body.index("{") + 1 :]
    return [s.strip() for s in body.split(";")]


def test_the_router_waits_before_it_does_anything_else():
    source = _read("ciera_route.cu")
    for kernel in ("route_few_kernel", "route_kernel"):
        first = [s for s in _statements(source, kernel) if not re.match(r"(constexpr|extern __shared__|__shared__) ", s)][0]
        assert first == "pdl_wait()", kernel
    assert "griddepcontrol" not in source


def test_others_begin_behind_that_wait():
    source = _read("ciera_internal.cuh")
    wait, launch = source.index('"griddepcontrol.wait;"'), source.index('"griddepcontrol.launch_dependents;"')
    assert wait < launch and source.count('"griddepcontrol') == 2
    for name in ("ciera_tokens.cu", "ciera_route.cu", "ciera_product.cuh", "ciera_tensor.cuh", "ciera_pipe.cuh", "ciera_fp4.cuh", "ciera_fp8.cuh"):
        assert "griddepcontrol" not in _read(name), name


def test_what_is_written_meanwhile_is_not_read_as_constant():
    source = _read("ciera_tokens.cu")
    assert not re.search(r"__ldg\(a\.(weights|experts)", source)
    assert not re.search(r"__restrict__ x\b", source)
