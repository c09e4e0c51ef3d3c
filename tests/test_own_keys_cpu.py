"""What requests' own keys count for where the SMs are divided, compiled from its header:
lengths that the kernels skip count for nothing, and no sum wraps around."""
import numpy as np
import pytest

from .test_host_rules_cpu import INT_MAX, compile_and_run

PROGRAM = """
#include "own_keys.h"
#include <cstdio>
#include <cstdlib>
int main(int n, char** v) {
  const int cap = atoi(v[1]);
  unsigned long long keys = 0;
  int by_warp = 0, valid = 0;
  for (int i = 2; i < n; ++i) {
    const int T = atoi(v[i]);
    if (!gc::own_keys_count(T, cap)) continue;
    keys += static_cast<unsigned long long>(gc::own_keys_cost(T));
    by_warp += gc::own_keys_cost_by_warp(T, 256);
    ++valid;
  }
  printf("%lld %d %d", static_cast<long long>(keys), by_warp, valid);
}"""


@pytest.mark.parametrize("cap", [16, 112, 4096, INT_MAX // 16 * 16])
@pytest.mark.parametrize("lens", [
    [0, 1, 15, 16, 17], [255, 256, 257, 1023, 1024, 1025], [-1, -INT_MAX - 1, 5],
    [INT_MAX] * 9, [INT_MAX - 1023, INT_MAX - 1024, INT_MAX - 255], [INT_MAX // 16 * 16] * 500])
def test_own_keys_are_summed_up(tmp_path, cap, lens):
    used = [t for t in lens if 0 < t <= cap]
    want = [sum(t + int(np.clip(t, 256, 1024)) for t in used), sum(min(t, 256) + 48 for t in used),
            len(used)]
    assert list(map(int, compile_and_run(tmp_path, PROGRAM, cap, *lens))) == want
