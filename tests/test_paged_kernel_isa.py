"""The LDS DMA of the paged attention kernels, on the instructions of the library
built here (no GPU needed)."""

import os
import shutil
import subprocess

import pytest

from paper_2607_00501_amd import binding as B
from tests.test_kernel_isa import OBJDUMP, _code_objects


def test_lds_dma_waits_for_m0(tmp_path):
    """One wait state stands between a scalar write of M0 and the LDS DMA that
    reads it; the copies take a scalar base and an offset per lane."""
    if not os.path.exists(B.LIB_PATH) or shutil.which(OBJDUMP) is None:
        pytest.skip("library or llvm-objdump not there")
    with open(B.LIB_PATH, "rb") as f:
        objects = [co for co in _code_objects(f.read()) if b"paged_attn_kernel" in co]
    assert objects
    dma = 0
    for i, co in enumerate(objects):
        path = tmp_path / f"{i}.co"
        path.write_bytes(co)
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", "--no-leading-addr", str(path)],
                              capture_output=True, text=True, check=True).stdout
        before = ""
        for ins in (line.strip() for line in text.splitlines()):
            if ins.startswith("global_load_lds"):
                dma += 1
                assert not (before.startswith("s_") and " m0," in before), f"{before} | {ins}"
                assert " off" not in ins, ins
            before = ins
    assert dma > 0
