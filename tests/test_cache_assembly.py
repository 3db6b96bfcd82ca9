"""The compiled code of shared.hip and evict.hip (CPU only): the direct loads to LDS stand
clear of the hazards that the compiler does not look for, no 64-bit shift goes by a wave's
last register, and no kernel keeps registers in memory."""
import os
import re
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2412_00408_amd import build
from test_decode_assembly import _compile, shifts_by_the_last_register
from test_lds_loads import _check


def test_compiled_kernels():
    if not os.path.exists(build.HIPCC):
        pytest.skip("no hipcc")
    files = ["shared.hip", "evict.hip"]
    with ThreadPoolExecutor(len(files)) as ex:
        for f, text in zip(files, ex.map(_compile, files)):
            assert not shifts_by_the_last_register(text)[1], f
            loads = _check([l.split(";")[0].strip() for l in text.splitlines()])
            assert loads >= 100 if f == "shared.hip" else loads == 0, f
            kernels = len(re.findall(r"\.amdhsa_kernel ", text))
            assert re.findall(r"\.vgpr_spill_count: *(\d+)", text) == ["0"] * kernels, f
            assert re.findall(r"\.private_segment_fixed_size: *(\d+)", text) == ["0"] * kernels, f
