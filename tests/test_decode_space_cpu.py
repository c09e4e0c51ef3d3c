"""Room for the partials of decode in shares, compiled from its header: two of every CTA's
(or group's), each of 8 or 16 heads of d columns with a maximum and a sum, whatever the head
dimension and the number of heads."""
import pytest

from .test_host_rules_cpu import compile_and_run

PROGRAM = """
#include "decode_units.h"
#include <cstdio>
#include <cstdlib>
int main(int, char** v) {
  const int d = atoi(v[1]), g = atoi(v[2]), sms = atoi(v[3]), most = atoi(v[4]);
  printf("%d %zu", gc::decode_ctas(d, g <= 8 ? 8 : 16), gc::decode_share_bytes(d, g, sms, most));
}"""

# CTAs on an SM of the kernel's variants (16 warps of 128 registers, 12 of 168, 8 of 255)
CTAS = {(64, 8): 2, (64, 16): 2, (128, 8): 2, (128, 16): 1}


@pytest.mark.parametrize("sms,most", [(152, 448), (1, 448), (300, 448), (152, 100)])
@pytest.mark.parametrize("g", [1, 2, 4, 8, 16])
@pytest.mark.parametrize("d", [64, 128])
def test_every_partial_has_room(tmp_path, d, g, sms, most):
    heads = 8 if g <= 8 else 16
    ctas, size = map(int, compile_and_run(tmp_path, PROGRAM, d, g, sms, most))
    assert ctas == CTAS[d, heads]
    last_cta, slot = min(ctas * sms, most) - 1, 1
    columns = ((last_cta * 2 + slot) * heads + heads) * d * 4
    assert size == columns + ((last_cta * 2 + slot) * heads + heads) * 8
