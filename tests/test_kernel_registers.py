"""What kernels keep in scratch for want of registers, from the compiler's report (no GPU needed)."""
import os
import re
import subprocess

import pytest

from paper_2606_23419_amd import build as b


def scratch(src, tmp_path):
    """{kernel: bytes of scratch per lane}"""
    r = subprocess.run([b.hipcc(), *b.HIPCC_FLAGS, *b.SOURCE_FLAGS.get(src, []), "-Rpass-analysis=kernel-resource-usage", "--cuda-device-only",
                        "-c", os.path.join(b.CSRC, src), "-o", str(tmp_path / "o")], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    found = re.findall(r"Function Name: (\S+).*?ScratchSize \[bytes/lane\]: (\d+)", r.stderr, re.S)
    assert found
    return {name: int(size) for name, size in found}


def test_norms_stay_in_registers(tmp_path):
    assert set(scratch("norm.hip", tmp_path).values()) == {0}


def test_attention_of_few_rows_over_4_bits(tmp_path):
    """One block of 16 rows a wave, what decoding uses, keeps everything in registers; two blocks of 128 channels do not."""
    got = scratch("attend_rows4.hip", tmp_path)
    assert len(got) == 24
    for name, size in got.items():
        d, _, blocks, _ = map(int, re.findall(r"Li(\d+)E", name))
        assert size <= (124 if d == 128 and blocks == 2 else 0), name


@pytest.mark.parametrize("src", ["attend_tile4.hip"])
def test_attention_of_chunks_over_4_bits(src, tmp_path):
    """128 channels fill the registers; what does not fit is read outside the tiles' loop."""
    got = scratch(src, tmp_path)
    assert len(got) == 8
    for name, size in got.items():
        assert size <= (80 if "ILi128" in name else 0), name
