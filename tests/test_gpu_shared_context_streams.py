"""SharedContext on a stream that is not torch's current one, and that is still busy when
the calls are made: what they read is as it was then."""
import numpy as np
import pytest

from paper_2505_23970_gb300 import binding as gcb
from paper_2505_23970_gb300 import workloads as wl
from paper_2505_23970_gb300.harness import SharedContext, bf16_bits, bf16_tensor

from ._span import assert_within, attend
from .test_gpu_shared_context import pages_of

pytestmark = pytest.mark.gpu

BUSY = 200_000_000  # clock cycles, about a tenth of a second


def context():
    c = SharedContext(8, 2, 128, 16, [300, 45], [3, 2], 4, [100, 0, 7, 300, 33], seed=3)
    c.pool.planes().fill_(float("nan"))
    return c


def image(c, name):
    n = int((getattr(c, name + "_table") >= 0).sum())
    return bf16_tensor(wl.normal_bf16(7, n, (n, 1, 2, 2, 16, 128)))


def test_restore_behind_a_busy_stream():
    """The page numbers are not given back before the restore has read them."""
    import torch
    c = context()
    s = torch.cuda.Stream()
    images = {"shared": image(c, "shared"), "states": image(c, "state")}
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(BUSY)
    for name, x in images.items():
        c.restore(x, name, s)
    other = [torch.zeros(n, dtype=torch.int32, device="cuda") for n in range(1, 64)]
    assert c.check(s) == gcb.GC_OK
    got = bf16_bits(c.pool.planes())[0]
    for name, table in (("shared", c.shared_table), ("states", c.state_table)):
        want = bf16_bits(images[name])[:, 0].transpose(1, 0, 2, 3, 4)
        assert np.array_equal(got[:, table[table >= 0]], want)
    del other
    c.close()


@pytest.mark.parametrize("as_int", [False, True])
def test_tokens_behind_a_busy_stream(as_int):
    """A token ends behind its steps, not as soon as it is told to."""
    import torch
    c = context()
    s = torch.cuda.Stream()
    c.restore(image(c, "shared"))
    rows = [bf16_tensor(wl.normal_bf16(5, t, (5, 12, 128))) for t in range(3)]
    outs = [torch.full((5, 8, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
            for _ in rows]
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(BUSY)
    qs = []
    for qkv, out in zip(rows, outs):
        c.step(qkv, out, stream=s.cuda_stream if as_int else s)
        with torch.cuda.stream(s):
            qs.append(c.q.clone())
        c.advance()
    assert c.check(s) == gcb.GC_OK
    assert c.own_lens.tolist() == [3] * 5 and c.seq_lens.tolist() == [4] * 5
    planes = c.pool.planes()[0]
    for t, out in enumerate(outs):
        for b in range(5):
            own = pages_of(c.own_table, b, t + 1, 16, planes)
            assert torch.equal(own[1, t], rows[t][b, 10:].double())
            g = int(c.group[b])
            shared = pages_of(c.shared_table, g, int(c.shared_lens[g]), 16, planes)
            want, bound = attend(qs[t][b:b + 1].double(), torch.cat([shared, own], 1), 128 ** -0.5)
            assert_within(out[b:b + 1], want, bound, f"token {t} request {b}")
    c.close()


def test_a_token_in_a_graph():
    """Step and advance are recorded on the stream of the capture."""
    import torch
    c = context()
    c.restore(image(c, "shared"))
    rows = bf16_tensor(wl.normal_bf16(5, 0, (5, 12, 128)))
    out = torch.empty((5, 8, 128), dtype=torch.bfloat16, device="cuda")
    c.step(rows, out)  # (the kernels are loaded)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.step(rows, out, stream=torch.cuda.current_stream())
        c.advance()
    for t in range(3):
        g.replay()
    torch.cuda.synchronize()
    assert c.check() == gcb.GC_OK
    assert c.own_lens.tolist() == [3] * 5
    assert c.positions.tolist() == [303] * 3 + [48] * 2
    c.close()
