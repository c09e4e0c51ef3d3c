"""A kernel's allowance of shared memory belongs to the kernel, for all host threads: a
call that sets its own size there can refuse another thread's, which a run shows by chance
alone."""
import os
import re

from paper_2505_23970_gb300 import build as gbuild

from .test_source_cpu import source


def test_only_constants_are_allowed():
    uses = {f: source(f).count("cudaFuncAttributeMaxDynamicSharedMemorySize")
            for f in os.listdir(gbuild.CSRC)}
    assert {f: n for f, n in uses.items() if n} == {"gc_internal.cuh": 1, "kv_copy.cu": 1}
    assert re.search(r"template <size_t kMost, typename\.\.\. P>\s*cudaError_t allow_shared\([^{]*\{"
                     r"[^}]*cudaFuncAttributeMaxDynamicSharedMemorySize,\s*"
                     r"static_cast<int>\(kMost\)", source("gc_internal.cuh"))
    assert re.search(r"const int smem = kStages \* kPiece;\s*cudaError_t ea =\s*"
                     r"cudaFuncSetAttribute\(restore_bulk_kernel, "
                     r"cudaFuncAttributeMaxDynamicSharedMemorySize, smem\)", source("kv_copy.cu"))
