"""The benchmark reports the GEMM's DRAM traffic from a recorded capture, as long as the kernel's sources are those of the capture."""
import json
import os

from paper_2507_19131_b200 import ncu_summary

import bench


def test_the_record_is_of_the_present_sources():
    """A change of the sources that the kernel is built from needs a new capture (python -m paper_2507_19131_b200.ncu_summary traffic ...)."""
    records = json.load(open(ncu_summary.TRAFFIC_JSON))
    assert records
    for workload, record in records.items():
        assert record["kernel_source_digest"] == ncu_summary.kernel_source_digest(), workload
        assert bench.recorded_traffic(workload) == record


def test_the_row_operators_are_not_part_of_the_gemm_sources():
    csrc = os.path.join(ncu_summary.HERE, "csrc")
    gemm = "".join(open(os.path.join(csrc, f)).read() for f in ncu_summary.GEMM_KERNEL_SOURCES)
    for name in ("Fp8MatmulArgs", "Fp8QuantArgs", "ResNormArgs"):
        assert name not in gemm and name in open(os.path.join(csrc, "row_ops.h")).read()
