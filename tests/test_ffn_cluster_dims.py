"""The gated block's pair kernel, which lives in a header, declares its cluster of two itself, as the
pair kernels of the .cu files do (test_cluster_dims)."""
import glob
import os
import re

from conftest import ROOT


def test_pair_kernels_in_headers_declare_their_cluster():
    found = set()
    for path in glob.glob(os.path.join(ROOT, "paper_2607_03011_gb300", "csrc", "*.cuh")):
        src = re.sub(r"//[^\n]*", "", open(path).read())
        kernels = list(re.finditer(r"__global__\s+void\s+([^;{]*?)(\bk_\w+)\s*\([^;{]*\{", src))
        for k, nxt in zip(kernels, kernels[1:] + [None]):
            body = src[k.end():nxt.start() if nxt else len(src)]
            if "tmem_alloc_pair(" in body:
                found.add(k[2])
                assert "__cluster_dims__(2, 1, 1)" in k[1], k[2]
    assert "k_ffn_gemm" in found
