"""The compiled code of window.hip, sample.hip and distill.hip (CPU only): no kernel
keeps anything in scratch memory (a build of the sampler that spilled one register
gave wrong sums now and then), and the direct loads to LDS stand clear of the
hazards that the compiler does not look for."""
import os
import re
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2412_00408_amd import build
from test_lds_loads import _check


def _compile(src):
    flags = [f for f in build.FLAGS if f not in ("-Wall", "-fPIC")]
    r = subprocess.run([build.HIPCC, *flags, *build.EXTRA_FLAGS.get(src, []), "--cuda-device-only", "-S",
                        "-o", "-", os.path.join(build.CSRC, src)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    return r.stdout


def test_no_scratch_and_no_load_hazards():
    if not os.path.exists(build.HIPCC):
        pytest.skip("no hipcc")
    files = ["window.hip", "sample.hip", "distill.hip"]
    with ThreadPoolExecutor(len(files)) as ex:
        for f, text in zip(files, ex.map(_compile, files)):
            kernels = re.findall(r"\.name:\s+(_ZN2qk\S+).*?\.private_segment_fixed_size:\s+(\d+)", text,
                                 re.S)
            assert len(kernels) >= 12, f
            assert [k for k in kernels if k[1] != "0"] == [], f
            assert "scratch_" not in text, f
            loads = _check([l.split(";")[0].strip() for l in text.splitlines()])
            assert loads >= 100 if f == "window.hip" else loads == 0, f
