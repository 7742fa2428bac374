"""What the kernels' inline assembly tells the compiler, read from the LLVM IR
of the sources (CPU only: nothing runs)."""
import os
import re
import subprocess

from paper_1706_05544_amd import build as b


def test_assembly_that_writes_m0_says_so(tmp_path):
    seen = 0
    for src in b.DEVICE_SOURCES:
        path = os.path.join(b.CSRC, src)
        if "m0" not in open(path).read():
            continue
        out = str(tmp_path / (src + ".ll"))
        # (-O1: the statements' constraints are those of any level)
        cmd = [b._hipcc()] + [c for c in b.COMMON if c != "-O3"] + [
            "-O1", "-x", "hip", "--offload-device-only", "-emit-llvm", "-S",
            path, "-o", out]
        r = subprocess.run(cmd, capture_output=True, text=True)
        assert r.returncode == 0, r.stderr
        for text, constraints in re.findall(
                r'asm (?:sideeffect )?"([^"]*)", "([^"]*)"',
                open(out).read()):
            if re.search(r"s_mov_b32 m0\b", text):
                seen += 1
                assert "~{m0}" in constraints, (src, constraints)
    assert seen
