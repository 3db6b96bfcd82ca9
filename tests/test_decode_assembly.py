"""The compiled code of window.hip, sample.hip and distill.hip (CPU only).

A 64-bit shift whose amount lies in the last vector register that the wave has is
not carried out right on this GPU: the amount is read as a pair, whose upper half
does not exist, and comes from v0 instead. A build of the sampler that used all of
its 128 registers shifted some masses by the lane's number. The compiler does not
avoid it, so the compiled code is looked through. The direct loads to LDS have to
stand clear of the hazards that the compiler does not look for either."""
import os
import re
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2412_00408_amd import build
from test_lds_loads import _check

SHIFT = re.compile(r"\bv_(?:lshlrev_b64|lshrrev_b64|ashrrev_i64)\S* v\[\d+:\d+\], v(\d+),")


def shifts_by_the_last_register(text):
    """(64-bit shifts seen, those whose amount is in the last register of the kernel's
    allocation, which is in eights)."""
    seen, bad = 0, []
    for name, regs in re.findall(r"\.amdhsa_kernel (\S+).*?\.amdhsa_next_free_vgpr (\d+)", text, re.S):
        at = text.find("\n%s:" % name)
        body = text[at:text.find(".Lfunc_end", at)]
        last = (int(regs) + 7) // 8 * 8 - 1
        amounts = [int(a) for a in SHIFT.findall(body)]
        seen += len(amounts)
        bad += [name for a in amounts if a == last]
    return seen, bad


def test_the_check_finds_such_a_shift():
    code = "\nk:\n\tv_lshrrev_b64 v[2:3], v%d, v[4:5]\n.Lfunc_end0:\n.amdhsa_kernel k\n.amdhsa_next_free_vgpr %d\n"
    assert shifts_by_the_last_register(code % (127, 128)) == (1, ["k"])
    assert shifts_by_the_last_register(code % (127, 125)) == (1, ["k"])
    assert shifts_by_the_last_register(code % (126, 128)) == (1, [])
    assert shifts_by_the_last_register(code % (127, 129)) == (1, [])


def _compile(src):
    flags = [f for f in build.FLAGS if f not in ("-Wall", "-fPIC")]
    r = subprocess.run([build.HIPCC, *flags, *build.EXTRA_FLAGS.get(src, []), "--cuda-device-only", "-S",
                        "-o", "-", os.path.join(build.CSRC, src)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    return r.stdout


def test_compiled_kernels():
    if not os.path.exists(build.HIPCC):
        pytest.skip("no hipcc")
    files = ["window.hip", "sample.hip", "distill.hip"]
    with ThreadPoolExecutor(len(files)) as ex:
        for f, text in zip(files, ex.map(_compile, files)):
            seen, bad = shifts_by_the_last_register(text)
            assert not bad, (f, bad)
            assert seen > 0 or f != "sample.hip", f
            loads = _check([l.split(";")[0].strip() for l in text.splitlines()])
            assert loads >= 100 if f == "window.hip" else loads == 0, f
