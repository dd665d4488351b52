"""The build checks of ``test_build_cpu`` for the attention half's sources:
no packed-fp32 instructions and no scratch traffic in the device code."""

import os

import pytest

import test_build_cpu as T
from paper_2609_38823_amd import build

SOURCES = build.block_sources()


@pytest.mark.parametrize("src", SOURCES, ids=[os.path.basename(s) for s in SOURCES])
def test_device_asm_has_no_packed_fp32(src, tmp_path):
    T.test_device_asm_has_no_packed_fp32(src, tmp_path)
