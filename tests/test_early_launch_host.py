"""Kernels that are launched while the one before still runs: what that one writes is not read by loads
that take memory for unchanging (read from the sources; a violation shows in no result by itself)."""
import os
import re

from paper_2609_33390_gb300 import build

# the caller's tensors, complete before the first kernel of the call begins
INPUTS = {"cache_evict.cu": ("kf", "vf")}


def bodies(text):
    """Bodies of the kernels of a source."""
    for m in re.finditer(r"__global__[^{;]*\{", text):
        depth, at = 1, m.end()
        while depth:
            depth += {"{": 1, "}": -1}.get(text[at], 0)
            at += 1
        yield text[m.end():at]


def test_early_launched_kernels_read_what_was_just_written_by_coherent_loads():
    found = 0
    for path in build.sources():
        with open(path) as f:
            text = re.sub(r"//[^\n]*", "", f.read())
        for body in bodies(text):
            if "wait_for_previous()" not in body:
                continue
            found += 1
            assert "__ldg(" not in body and "ld.global.nc" not in body, path
            for m in re.finditer(r"\bld_stream_v4\(([^)]*)", body):
                assert re.match(r"\s*(%s)\b" % "|".join(INPUTS.get(os.path.basename(path), ("-",))), m[1]), (path, m[0])
    assert found >= 4
