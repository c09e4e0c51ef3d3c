"""FourBitContext.begin() beside a busy current stream."""
import pytest

from paper_2505_23970_gb300 import binding as gcb
from paper_2505_23970_gb300 import workloads as wl
from paper_2505_23970_gb300.harness import FourBitContext, bf16_tensor

pytestmark = pytest.mark.gpu


def test_memory_that_the_current_stream_still_works_on():
    """Memory freed with work on it still queued on the current stream is not written by a
    prefill on another one: what begin() takes is done with when it returns."""
    import torch
    Hq, Hkv, d, B, n = 8, 2, 128, 4, 500
    c = FourBitContext(Hq, Hkv, d, 16, B, 512, seed=1)
    qkv = bf16_tensor(wl.normal_bf16(1, 1, (B * n, Hq + 2 * Hkv, d)))
    out = torch.empty((B * n, Hq, d), dtype=torch.bfloat16, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    kept, met = [], 0
    for _ in range(5):
        # as large as the q that begin() takes; read long after it has been freed
        old = torch.full((B * n, Hq, d), 3.0, dtype=torch.bfloat16, device="cuda")
        torch.cuda._sleep(200_000_000)
        kept.append(old + 0)
        at = old.data_ptr()
        del old
        c.begin([n] * B)
        met += c._new[3].data_ptr() == at
        c.prefill(qkv, out, 0, side)
        side.synchronize()
        torch.cuda.synchronize()
        assert bool((kept[-1] == 3.0).all())
    assert met, "the allocator never gave the block again"
    assert c.check() == gcb.GC_OK
