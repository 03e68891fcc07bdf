"""The launch plan gives the shapes of the window and tree tests on the GPU to the kernels that those mean."""

import os
import subprocess

import pytest
import q8_span_shapes as sh

from paper_2609_11582_amd import _build


@pytest.fixture(scope="module")
def planned(tmp_path_factory):
    src = os.path.join(os.path.dirname(os.path.abspath(__file__)), "q8_plan_of.cpp")
    exe = str(tmp_path_factory.mktemp("plan") / "q8_plan_of")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", _build.CSRC, src, "-o", exe], check=True)

    def plan(span, shapes):
        lines = [" ".join(map(str, [span, s.H, s.Hq // s.H, s.window, s.sinks, len(s.lens), *s.lens, *s.n])) for s in shapes]
        r = subprocess.run([exe], input="\n".join(lines), capture_output=True, text=True, timeout=60, check=True)
        return [tuple(map(int, x.split()))[:2] for x in r.stdout.splitlines()]
    return plan


@pytest.mark.parametrize("span, shapes", [(1, sh.SPLIT_WINDOWS), (1, sh.HIDDEN_WINDOWS), (2, sh.SPLIT_TREES), (2, sh.HIDDEN_TREES)])
def test_shapes_take_their_kernel(planned, span, shapes):
    assert planned(span, shapes) == [(s.cols, s.most) for s in shapes]
