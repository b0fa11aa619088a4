"""What the gated recurrence counts by (gla_recur_plan.h), on the CPU."""
import ctypes
import os
import subprocess

import pytest

import paper_2405_18428_amd as gla

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2405_18428_amd", "csrc")
SOURCE = r"""
#include "gla_recur_plan.h"
using namespace gla;
extern "C" {
// looks that a wait makes of `tries` tries; -1 if what it has counted is out of line
long long looks(int most, long long tries) {
    RecurLooks l = {most, 0};
    long long made = 0;
    for (long long i = 0; i < tries; ++i) made += l.another();
    return l.made == (most == kRecurNoEnd ? 0 : made) ? made : -1;
}
int no_end() { return kRecurNoEnd; }
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    where = tmp_path_factory.mktemp("plan")
    (where / "plan.cpp").write_text(SOURCE)
    # (a count that overflows ends the process)
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-fsanitize=signed-integer-overflow", "-fsanitize-undefined-trap-on-error", "-shared", "-fPIC", "-I", CSRC, "-o",
                    str(where / "plan.so"), str(where / "plan.cpp")], check=True)
    lib = ctypes.CDLL(str(where / "plan.so"))
    for f in (lib.looks,):
        f.restype = ctypes.c_longlong
    lib.looks.argtypes = [ctypes.c_int, ctypes.c_longlong]
    return lib


@pytest.mark.parametrize("most,tries,made", [(0, 100, 0), (1, 100, 1), (1 << 15, 1 << 20, 1 << 15), (100, 7, 7)])
def test_a_wait_looks_as_often_as_it_may(plan, most, tries, made):
    assert plan.looks(most, tries) == made


def test_a_wait_without_an_end_counts_nothing(plan):
    """More looks than an int can count."""
    assert plan.no_end() < 0 and plan.looks(plan.no_end(), (1 << 31) + 100) == (1 << 31) + 100


# (B, T, D), whether sequences are cut into units, which need a workspace
WALKED = [(1, 256, 64, False), (1, 257, 64, True), (15, 4096, 2048, True), (16, 4096, 2048, False), (16, 257, 2048, False), (255, 1024, 128, True), (256, 1024, 128, False),
          # odd numbers of channels: 64 of them a work-group, not 128
          (7, 1024, 2047, True), (8, 1024, 2047, False), (8, 257, 2047, False), (8, 1025, 2047, True), (255, 1024, 63, True), (261, 1024, 63, False), (64, 4096, 385, True),
          (16, 2048, 2047, True), (1 << 20, 1 << 20, 449, False)]


@pytest.mark.parametrize("B,T,D,units", WALKED)
def test_sequences_that_are_walked(B, T, D, units):
    assert (gla.gla_recur_fwd_workspace_bytes(B, T, D) > 0) == units
