"""The ordering rule of dependent kernels' reads (test_source_cpu.py) in every header that
they are made of."""
import os
import re

import pytest

from paper_2505_23970_gb300 import build as gbuild

from .test_source_cpu import source

HEADERS = sorted(f for f in os.listdir(gbuild.CSRC) if f.endswith(".cuh"))


def test_the_headers_of_the_kernels_are_there():
    assert {"decode_mma.cuh", "span.cuh", "gc_internal.cuh", "sm103_ptx.cuh"} <= set(HEADERS)


@pytest.mark.parametrize("name", HEADERS)
@pytest.mark.parametrize("word", ["__ldg", r"ld\.global\.nc", "__restrict__"])
def test_headers_take_no_read_only_loads(name, word):
    assert not re.search(word, source(name))
