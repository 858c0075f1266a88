"""Counters in profiles/ are those of the kernels that are there: the benchmark
reports measured traffic only while a kernel's sources are as they were when
its counters were taken."""
import glob
import os

import pytest

import bench

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
COUNTED = sorted(os.path.basename(f)[:-4] for f in glob.glob(os.path.join(ROOT, "profiles", "*.txt"))
                 if "pmc.kernel_source_sha256" in open(f).read())


def test_there_are_counters():
    assert "k_inc_aniso-8M-d16-k10" in COUNTED


@pytest.mark.parametrize("name", COUNTED)
def test_counters_are_of_the_kernels_that_are_there(name):
    kernel = max((k for k in bench.KERNEL_SOURCES if name.startswith(k + "_")), key=len)
    traffic, source = bench.measured_traffic(kernel, name[len(kernel) + 1:])
    assert traffic is not None and traffic > 0, source
