"""The build refuses compiled code that shifts 64 bits by the last register of a kernel's
allocation (CPU only; nothing is run)."""
import os

import pytest

from paper_2412_00408_amd import build

KERNEL = r"""
#include <hip/hip_runtime.h>
__global__ void k(unsigned long long* p) {
  asm volatile("v_lshrrev_b64 v[0:1], v%d, v[2:3]" ::: "v0", "v1", "v2", "v3", "v%d");
}
"""


@pytest.mark.parametrize("amount,refused", [(7, True), (6, False), (15, True), (12, False)])
def test_the_build_looks_through_compiled_code(tmp_path, monkeypatch, amount, refused):
    if not os.path.exists(build.HIPCC):
        pytest.skip("no hipcc")
    monkeypatch.setattr(build, "BUILD_DIR", str(tmp_path))
    src = tmp_path / "shift.hip"
    src.write_text(KERNEL % (amount, amount))
    obj = tmp_path / "shift.hip.o"
    if refused:
        with pytest.raises(RuntimeError, match="64-bit shift"):
            build._compile(str(src))
        assert not obj.exists()
    else:
        assert build._compile(str(src)) == str(obj) and obj.stat().st_size > 0
    assert sorted(p.name for p in tmp_path.iterdir()) == ["shift.hip"] + ([] if refused else ["shift.hip.o"])


def test_a_failed_compilation_is_an_error(tmp_path, monkeypatch):
    if not os.path.exists(build.HIPCC):
        pytest.skip("no hipcc")
    monkeypatch.setattr(build, "BUILD_DIR", str(tmp_path))
    src = tmp_path / "broken.hip"
    src.write_text("not a program")
    with pytest.raises(RuntimeError, match="hipcc failed"):
        build._compile(str(src))
