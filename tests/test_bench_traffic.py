"""The benchmark's DRAM traffic of a product launch comes from a stored capture, tied to the text of the product kernel's sources."""
import json

import bench


def test_the_capture_on_file_is_of_the_present_product_kernel():
    with open(bench.GEMM_TRAFFIC_JSON) as f:
        stored = json.load(f)
    assert bench.gemm_sources_hash() == stored["sources_sha256_16"]
    traffic, note = bench.gemm_dram_traffic(stored["M"], stored["N"], stored["K"], stored["encoding"])
    assert traffic == stored["dram_bytes_read"] + stored["dram_bytes_write"] and "changed" not in note


def test_another_workload_has_none():
    assert bench.gemm_dram_traffic(16, 16, 16, "awe6") == (None, "the capture on file is of another workload")
