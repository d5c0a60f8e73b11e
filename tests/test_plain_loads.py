"""Kernels launched programmatically read what an earlier launch writes with plain loads (see test_programmatic_launches):
so do the functions that they call, in every header and source; other loads are named here."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2601_08670_gb300", "csrc")
OTHERS = {
    # block tables of the decode step and the one-layer kernels, embedding rows
    "attention.cu": {"a.block_table + (int64_t)s * a.max_blocks + j", "a.block_table + ptab[i]",
                     "reinterpret_cast<const uint4*>(a.embed + (int64_t)tok * d + e0)"},
    "lm_head.cu": {"wy + i"},  # the unembedding
}


def test_non_coherent_loads_are_the_named_ones():
    files = sorted(glob.glob(os.path.join(CSRC, "*.cu")) + glob.glob(os.path.join(CSRC, "*.cuh")))
    names = {os.path.basename(f) for f in files}
    assert {"paged.cuh", "kv_append.cuh", "kv_append8.cu", "paged_attention.cuh", "paged_attention8.cu", "sample.cuh",
            "sample.cu", "sample_bf16.cu", "attention_tile.cuh", "common.cuh"} <= names
    for path in files:
        src = re.sub(r"//[^\n]*", "", open(path).read())
        assert "__restrict__" not in src and not re.search(r"ld\.global(\.\w+)*\.nc\b", src), path
        loads = set()
        for m in re.finditer(r"__ldg\(", src):
            at, depth = m.end(), 1
            while depth:
                depth += {"(": 1, ")": -1}.get(src[at], 0)
                at += 1
            loads.add(" ".join(src[m.end():at - 1].split()))
        assert loads == OTHERS.get(os.path.basename(path), set()), path
