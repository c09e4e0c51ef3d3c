"""A host thread whose first CUDA call is one of the library's."""
import threading

import numpy as np
import pytest

from paper_2505_23970_gb300 import binding as gcb
from paper_2505_23970_gb300 import workloads as wl
from paper_2505_23970_gb300.harness import _i32, bf16_tensor

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["prefill", "prefill_q4", "decode", "decode_q4"])
@pytest.mark.parametrize("d", [64, 128])
def test_a_thread_that_has_made_no_cuda_call(kind, d):
    """(The 4-bit calls over a cache without pages.)"""
    import torch
    B, Hq, Hkv = 5, 8, 2
    pool = gcb.KVPool.create(1, Hkv, d, 16, B)
    pool.planes().copy_(bf16_tensor(wl.normal_bf16(1, 2, (1, 2, B, Hkv, 16, d))))
    q = bf16_tensor(wl.normal_bf16(1, 1, (B, Hq, d)))
    out = torch.zeros_like(q)
    table, none = _i32(np.arange(B)[:, None], "cuda"), _i32(np.full((B, 1), -1), "cuda")
    ones, threes, lens = (_i32(np.full(B, n), "cuda") for n in (1, 3, 4))
    cu = _i32(np.arange(B + 1), "cuda")
    need = max(gcb.gc_paged_decode_workspace_bytes(pool.handle, B, 1, Hq),
               gcb.gc_paged_decode_q4_workspace_bytes(pool.handle, B, 1, Hq, 1))
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    refused = []

    def call():
        prefill = (q, pool.handle, table, threes, ones, out, None, 0, cu, B, 1, Hq, 0.1, B)
        decode = (q, pool.handle, table, lens, out, None, 0, B, 1, Hq, 0.1, ws, need)
        try:
            if kind == "prefill":
                gcb.gc_prefix_prefill_attn(*prefill)
            elif kind == "prefill_q4":
                gcb.gc_prefix_prefill_attn_q4(*prefill, None, none, 0, None, 0)
            elif kind == "decode":
                gcb.gc_paged_decode_attn(*decode)
            else:
                gcb.gc_paged_decode_attn_q4(*decode, None, none, 0, 1)
        except gcb.GcError as e:
            refused.append(str(e))

    call()
    torch.cuda.synchronize()
    want = out.clone()
    assert not refused and float(want.abs().max()) > 0
    out.zero_()
    torch.cuda.synchronize()
    t = threading.Thread(target=call)
    t.start()
    t.join()
    assert not refused, refused
    torch.cuda.synchronize()
    assert torch.equal(out.view(torch.int16), want.view(torch.int16))
    assert pool.check() == gcb.GC_OK
