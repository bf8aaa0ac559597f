"""The amount of shared memory that a kernel may have is the kernel's, not the launch's: two host threads that launch it with different amounts must set the same limit."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2106_06998_b200", "csrc")


def test_every_kernels_limit_is_a_constant():
    found = 0
    for top, _, names in os.walk(CSRC):
        for name in sorted(names):
            if not name.endswith((".cu", ".cuh", ".h")):
                continue
            code = re.sub(r"//[^\n]*", "", open(os.path.join(top, name)).read())
            for m in re.finditer(r"cudaFuncAttributeMaxDynamicSharedMemorySize,\s*((?:[^()]|\([^()]*\))*?)\);", code):
                found += 1
                value = re.sub(r"\(int\)", "", m.group(1)).strip()
                if re.fullmatch(r"(?:G::)?[A-Z_]+(?: - \d+)?|\d+ \* 1024", value):
                    continue
                assert value == "smem", (name, value)                 # (a local: of constants alone)
                local = re.findall(r"const(?:expr)? size_t smem = ([^;]*);", code[:m.start()])[-1]
                assert re.fullmatch(r"[A-Z0-9_ *+()]*", re.sub(r"\(size_t\)|sizeof\(float\)|contract_async_tile_floats<KS, DYS>\(\)", "1", local)), (name, local)
    assert found >= 15
