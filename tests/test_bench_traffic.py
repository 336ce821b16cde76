"""bench.py reports the traffic of the gate/up projection only while the sources that it was
measured on are the ones in use (no GPU)."""
import os
import re

import bench

CSRC = os.path.join(bench.ROOT, "paper_2608_23167_amd", "csrc")


def test_every_source_of_the_projections_counts():
    """gemm.hip and every header of this library that it includes, directly or not."""
    seen, todo = set(), ["gemm.hip"]
    while todo:
        f = todo.pop()
        if f not in seen:
            seen.add(f)
            with open(os.path.join(CSRC, f)) as fh:
                todo += re.findall(r'^#include "(\w+\.h)"', fh.read(), re.M)
    assert set(bench.GEMM_SOURCES) == seen


def test_the_figures_are_those_of_the_current_sources():
    """Otherwise the bench reports null: measure again (profiles/ has the commands)."""
    assert {t["sources_sha256"] for t in bench.TRAFFIC.values()} == {bench.gemm_sources_sha256()}
    assert bench.measured_traffic("llada_gen256", "gemm_gate_up", 32, 2, 1 / 32) > 201326592   # the weights
