"""The counter summaries that bench.py reports as traffic belong to the kernels as they are."""
import pytest

import bench


@pytest.mark.parametrize("kernel,workload,source", [("flash_attn_kernel", "wan14b", "attention.hip"),
                                                    ("gemm_bf16_ring_kernel", "flux1024", "gemm_bf16.hip")])
def test_traffic_summaries_match_their_sources(kernel, workload, source):
    assert bench.kernel_traffic(kernel, workload, source) > 0
