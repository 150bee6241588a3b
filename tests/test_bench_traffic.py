"""The counter summaries that bench.py reports as traffic belong to the kernels as they are."""
import os
import shutil

import pytest

import bench


@pytest.mark.parametrize("kernel,workload,source", [("flash_attn_kernel", "wan14b", "attention.hip"),
                                                    ("gemm_bf16_ring_kernel", "flux1024", "gemm_bf16.hip")])
def test_traffic_summaries_match_their_sources(kernel, workload, source):
    assert bench.kernel_traffic(kernel, workload, source) > 0


@pytest.mark.parametrize("kernel,workload,source,parts", [
    ("flash_attn_kernel", "wan14b", "attention.hip", ["attention.hip", "attention_tile.h", "common.h"]),
    ("gemm_bf16_ring_kernel", "flux1024", "gemm_bf16.hip", ["gemm_bf16.hip", "gemm_tile.h", "common.h"])])
def test_traffic_summaries_know_the_headers_of_their_kernels(kernel, workload, source, parts, tmp_path, monkeypatch):
    """A change to a file that a kernel's code lies in takes its counters out of use; one to another file does not."""
    csrc = tmp_path / "paper_2608_09231_amd" / "csrc"
    shutil.copytree(os.path.join(bench.ROOT, "paper_2608_09231_amd", "csrc"), csrc)
    shutil.copytree(os.path.join(bench.ROOT, "profiles"), tmp_path / "profiles")
    monkeypatch.setattr(bench, "ROOT", str(tmp_path))
    for name in sorted(os.listdir(csrc)):
        text = (csrc / name).read_bytes()
        (csrc / name).write_bytes(text + b"\n")
        traffic = bench.kernel_traffic(kernel, workload, source)
        assert (traffic is None) == (name in parts), name
        (csrc / name).write_bytes(text)
    assert bench.kernel_traffic(kernel, workload, source) > 0
