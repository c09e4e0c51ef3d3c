"""FourBitContext refuses steps that its attention call would refuse, before it takes any
memory (no GPU is needed to see it)."""
import pytest

from paper_2505_23970_gb300.harness import FourBitContext


@pytest.mark.parametrize("Hq,Hkv,tokens", [(64, 8, 3), (64, 8, 4), (16, 1, 2), (8, 8, 17),
                                           (32, 1, 1), (8, 2, 0), (8, 2, -1)])
def test_steps_past_16_rows(Hq, Hkv, tokens):
    with pytest.raises(ValueError, match="16 rows"):
        FourBitContext(Hq, Hkv, 128, 16, 2, 100, tokens)
