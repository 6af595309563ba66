"""The attention's and the weighing's loops keep everything in registers.

A register reloaded from scratch memory inside a loop waits for every copy into
LDS that is in flight (the counter of outstanding loads is one), which costs
the long-context forms a third of their rate without a word from the compiler.  The
sources are compiled to assembly with the library's own flags, and every
innermost loop with matrix instructions is looked through (CPU only)."""
import importlib.util
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _build_script():
    spec = importlib.util.spec_from_file_location("_sc_build", os.path.join(ROOT, "paper_2609_22283_amd", "build.py"))
    b = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(b)
    return b


def _kernels(text):
    """{name: its lines of assembly}"""
    out, lines = {}, None
    for line in text.split("\n"):
        m = re.match(r"^(_Z\w+):", line)
        if m:
            lines = out.setdefault(m.group(1), [])
        elif line.startswith(".Lfunc_end"):
            lines = None
        elif lines is not None:
            lines.append(line)
    return out


def _innermost_loops(lines):
    """The stretches between a label and a branch back to it that hold matrix instructions
    and no smaller such stretch."""
    labels, loops = {}, []
    for i, line in enumerate(lines):
        m = re.match(r"^(\.LBB\w+):", line)
        if m:
            labels[m.group(1)] = i
        m = re.search(r"s_c?branch\w* (\.LBB\w+)", line)
        if m and m.group(1) in labels and any("v_mfma" in x for x in lines[labels[m.group(1)]:i]):
            loops.append((labels[m.group(1)], i))
    return [lines[a:b] for a, b in loops if not any((c, d) != (a, b) and a <= c and d <= b for c, d in loops)]


@pytest.mark.parametrize("source,kernel,least", [
    ("attention.hip", "attn_", 8), ("attention_lse.hip", "attn_", 16), ("weigh.hip", "weigh_", 5)])
def test_loops_without_scratch_memory(source, kernel, least, tmp_path):
    b = _build_script()
    if shutil.which(b.HIPCC) is None:
        pytest.skip("needs hipcc")
    out = tmp_path / "device.s"
    cmd = [b.HIPCC] + b.COMMON + ["-x", "hip", "--cuda-device-only", "-S", os.path.join(b.CSRC, source), "-o", str(out)]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    seen = 0
    for name, lines in _kernels(out.read_text()).items():
        loops = _innermost_loops(lines) if kernel in name else []
        seen += bool(loops)
        for loop in loops:
            assert not any("scratch_" in x for x in loop), name
    assert seen >= least
