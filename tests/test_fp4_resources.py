"""The loop of the attention over 4-bit pages keeps everything in registers, and makes nothing but
scaled matrix instructions of its products (CPU only: the assembly of the library's own flags)."""
import os
import shutil
import subprocess

import pytest

from test_attention_resources import _build_script, _innermost_loops, _kernels


def test_loops_without_scratch_memory(tmp_path):
    b = _build_script()
    if shutil.which(b.HIPCC) is None:
        pytest.skip("needs hipcc")
    out = tmp_path / "device.s"
    cmd = [b.HIPCC] + b.COMMON + ["-x", "hip", "--cuda-device-only", "-S", os.path.join(b.CSRC, "attention_fp4.hip"), "-o", str(out)]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    loops = {name: _innermost_loops(lines) for name, lines in _kernels(out.read_text()).items() if "fp4_attention" in name}
    assert len(loops) == 3 and all(loops.values())
    for name, found in loops.items():
        for loop in found:
            assert not any("scratch_" in x or "s_barrier" in x for x in loop), name
            products = [x for x in loop if "v_mfma" in x]
            assert products and all("v_mfma_scale_f32_16x16x128" in x for x in products), name
