"""Kernels that start before the one in front of them has ended must not read global memory through loads that promise it is
constant while they run: checked on the sources, since a run shows only how one build happens to order them."""
import os
import re

from paper_2502_03805_b200 import build

CONSTANT_LOADS = re.compile(r"__ldg\s*\(|ld\.global(\.\w+)*\.nc|__restrict__")


def included(path, seen):
    """The files of csrc/ that a source file is made of, itself among them."""
    if path not in seen:
        seen.add(path)
        for name in re.findall(r'#include "([\w./]+)"', open(path).read()):
            at = os.path.join(build.CSRC, name)
            if os.path.exists(at):
                included(at, seen)
    return seen


def without_comments(text):
    return re.sub(r"//[^\n]*|/\*.*?\*/", "", text, flags=re.S)


def test_early_kernels_use_no_constant_loads():
    early = os.path.join(build.CSRC, "launch_early.cuh")
    units = [files for files in (included(s, set()) for s in build.sources()) if early in files]
    assert len(units) >= 4                                  # rope, store and load, both decode kernels
    found = {os.path.basename(f): CONSTANT_LOADS.findall(without_comments(open(f).read()))
             for f in sorted(set().union(*units))
             if CONSTANT_LOADS.search(without_comments(open(f).read()))}
    assert not found


def test_early_kernels_wait_before_they_do_anything_else():
    """Every kernel of these files waits; what stands before it are declarations, shared memory and parameter prefetches."""
    for s in build.sources():
        text = open(s).read()
        if '"launch_early.cuh"' not in text and '"paged_decode.cuh"' not in text:
            continue
        bodies = re.split(r"__global__", without_comments(text))[1:]
        assert bodies
        for body in bodies:
            before, wait, _ = body.partition("wait_for_previous_kernel();")
            assert wait, s
            assert not re.search(r"\bp\.\w+(\.\w+)*\[|tma_load|bulk_load|reinterpret_cast<const (u?int|float)", before), s
