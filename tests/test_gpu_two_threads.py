"""Host threads with a pool and a stream each: distinct pools are independent, so a call is
answered whatever sizes the other threads' calls of the same kernel have."""
import ctypes
import os
import subprocess
import threading

import numpy as np
import pytest

from paper_2505_23970_gb300 import binding as gcb
from paper_2505_23970_gb300 import build as gbuild
from paper_2505_23970_gb300 import workloads as wl
from paper_2505_23970_gb300.harness import _i32, bf16_tensor

from . import _q4

pytestmark = pytest.mark.gpu

CALLS = 20000  # of each thread

# The calls come from a loop in C, which no interpreter lock takes apart.
LOOP = r"""
#include "gc.h"
struct Call {
  int32_t kind, batch, width, hq, n4;
  const void* q;
  gc_kv_pool* pool;
  const int32_t *table, *prefix_lens, *new_lens, *cu, *lens, *table4;
  void *out, *ws;
  size_t ws_bytes;
  const void* cache;
  cudaStream_t stream;
  void* call;
};
extern "C" int loop(const Call* c, int n) {
  int refused = 0;
  for (int i = 0; i < n; ++i) {
    gc_status s;
    if (c->kind == 0)
      s = reinterpret_cast<decltype(&gc_prefix_prefill_attn)>(c->call)(
          c->q, c->pool, c->table, c->prefix_lens, c->new_lens, c->out, c->stream, 0, c->cu,
          c->batch, c->width, c->hq, 0.1f, c->batch);
    else if (c->kind == 1)
      s = reinterpret_cast<decltype(&gc_paged_decode_attn)>(c->call)(
          c->q, c->pool, c->table, c->lens, c->out, c->stream, 0, c->batch, c->width, c->hq, 0.1f,
          c->ws, c->ws_bytes);
    else
      s = reinterpret_cast<decltype(&gc_paged_decode_attn_q4)>(c->call)(
          c->q, c->pool, c->table, c->lens, c->out, c->stream, 0, c->batch, c->width, c->hq, 0.1f,
          c->ws, c->ws_bytes, c->cache, c->table4, c->n4, 1);
    refused += s != GC_OK;
  }
  return refused;
}
"""


class Call(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("kind", "batch", "width", "hq", "n4")] + \
        [(n, ctypes.c_void_p) for n in ("q", "pool", "table", "prefix_lens", "new_lens", "cu", "lens",
                                        "table4", "out", "ws")] + \
        [("ws_bytes", ctypes.c_size_t)] + \
        [(n, ctypes.c_void_p) for n in ("cache", "stream", "call")]


@pytest.fixture(scope="module")
def loop(tmp_path_factory):
    at = tmp_path_factory.mktemp("loop")
    (at / "loop.cpp").write_text(LOOP)
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(gbuild.nvcc()))), "include")
    subprocess.run(["g++", "-O1", "-shared", "-fPIC", "-I", gbuild.INCLUDE, "-I", cuda,
                    str(at / "loop.cpp"), "-o", str(at / "loop.so")], check=True)
    lib = ctypes.CDLL(str(at / "loop.so"))
    lib.loop.argtypes = [ctypes.POINTER(Call), ctypes.c_int]
    return lib.loop


class Paged:
    """`batch` requests of 4 tokens, 1 of them new, a page each in a 16-bit pool."""

    def __init__(self, batch, Hq, Hkv, d):
        import torch
        self.pool = gcb.KVPool.create(1, Hkv, d, 16, batch)
        self.pool.planes().copy_(bf16_tensor(wl.normal_bf16(batch, 2, (1, 2, batch, Hkv, 16, d))))
        t = self.tensors = dict(
            q=bf16_tensor(wl.normal_bf16(batch, 1, (batch, Hq, d))),
            table=_i32(np.arange(batch)[:, None], "cuda"), cu=_i32(np.arange(batch + 1), "cuda"),
            prefix_lens=_i32(np.full(batch, 3), "cuda"), new_lens=_i32(np.full(batch, 1), "cuda"),
            lens=_i32(np.full(batch, 4), "cuda"))
        self.out = t["out"] = torch.zeros_like(t["q"])
        self.c = Call(batch=batch, width=1, hq=Hq, pool=self.pool.handle, kind=self.kind)
        self.c.call = ctypes.cast(getattr(gcb.load(), self.entry), ctypes.c_void_p)
        self.more(batch, Hq, Hkv, d)
        for name, x in t.items():
            setattr(self.c, name, x.data_ptr())

    def space(self, need):
        import torch
        self.tensors["ws"] = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
        self.c.ws_bytes = self.tensors["ws"].numel()


class Prefill(Paged):
    kind, entry = 0, "gc_prefix_prefill_attn"

    def more(self, *_):
        pass


class Decode16(Paged):
    kind, entry = 1, "gc_paged_decode_attn"

    def more(self, batch, Hq, Hkv, d):
        self.space(gcb.gc_paged_decode_workspace_bytes(self.pool.handle, batch, 1, Hq))


class Decode4(Paged):
    kind, entry = 2, "gc_paged_decode_attn_q4"

    def more(self, batch, Hq, Hkv, d):
        import torch
        cache = _q4.cache_bytes(wl.normal_bf16(batch, 3, (1, 2, batch, Hkv, 16, d)))
        self.tensors.update(cache=torch.from_numpy(cache).cuda(),
                            table4=self.tensors["table"].flip(0).contiguous())
        self.c.n4 = batch
        self.space(gcb.gc_paged_decode_q4_workspace_bytes(self.pool.handle, batch, 1, Hq, 1))


@pytest.mark.parametrize("kind,Hq,Hkv,d,batches", [
    (Decode4, 8, 1, 128, (1024, 1)), (Decode4, 16, 1, 128, (1024, 1)),
    (Decode4, 4, 1, 64, (1024, 1)), (Decode4, 16, 1, 64, (8192, 1025)),
    (Prefill, 1, 1, 64, (500, 1)), (Prefill, 1, 1, 128, (500, 1)),
    (Decode16, 8, 1, 128, (8192, 7000)), (Decode16, 8, 1, 64, (8192, 7000))])
def test_calls_of_other_sizes_at_the_same_time(loop, kind, Hq, Hkv, d, batches):
    """One thread with the larger batch, two with the smaller one."""
    import torch
    work = [kind(b, Hq, Hkv, d) for b in (batches[0], batches[1], batches[1])]
    want = []
    for w in work:
        assert loop(w.c, 1) == 0
        torch.cuda.synchronize()
        want.append(w.out.clone())
        w.out.zero_()
    torch.cuda.synchronize()
    start, refused = threading.Barrier(len(work)), []

    def run(w):
        stream = torch.cuda.Stream()
        stream.synchronize()
        w.c.stream = stream.cuda_stream
        start.wait()
        refused.append(loop(w.c, CALLS if w.c.batch < 2000 else CALLS // 10))

    threads = [threading.Thread(target=run, args=(w,)) for w in work]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert refused == [0] * len(work)
    for w, x in zip(work, want):
        assert torch.equal(w.out.view(torch.int16), x.view(torch.int16))
        assert w.pool.check() == gcb.GC_OK
