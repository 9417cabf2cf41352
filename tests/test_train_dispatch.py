"""Rules of the training operators (csrc/dispatch.h), compiled for the host and asked at the sizes on either side of their lines."""
import ctypes as C
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2509_06040_amd", "csrc")
SOURCE = """
#include "dispatch.h"
extern "C" int objective_one_launch(int edges, long long D) { return br::rule::objective_one_launch(edges, D); }
"""


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    d = tmp_path_factory.mktemp("rules")
    (d / "rules.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", CSRC, "-o", str(d / "rules.so"), str(d / "rules.cpp")], check=True)
    return C.CDLL(str(d / "rules.so"))


def test_one_workgroup_takes_only_what_two_launches_are_slower_for(rule):
    """Sets that one workgroup took 12 to 80 us for, where two launches are 11.5 of a stream of calls; and those that it takes 8.4 to 8.8 for."""
    one = lambda edges, D: bool(rule.objective_one_launch(edges, C.c_longlong(D)))
    for edges, D in ((1, 4096), (1, 32768), (8, 4096), (16, 2048), (32, 1024), (33, 64), (64, 64), (128, 256), (512, 64), (1, 1 << 40)):
        assert not one(edges, D), (edges, D)
    for edges, D in ((1, 4), (1, 1024), (8, 1024), (16, 1024), (32, 64), (32, 256), (19, 256), (21, 716), (8, 2048), (10, 2392)):
        assert one(edges, D), (edges, D)
