"""The direct loads of the tree kernel (tree.hip): what test_direct_loads_codegen.py checks for the question kernels, on the
generated code, and that its LDS destinations stay in the 16 bits that M0 has for them."""
import re
import subprocess

import pytest

from test_direct_loads_codegen import CSRC, HIPCC, ROOT


def test_m0_is_only_touched_by_the_direct_loads(tmp_path):
    import os
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not found")
    out = tmp_path / "tree.s"
    cmd = [HIPCC, "--offload-arch=gfx950", "-O3", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-S", "--cuda-device-only", "-o", str(out), os.path.join(CSRC, "tree.hip")]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-2000:]
    code = [l.strip() for l in out.read_text().splitlines()]
    code = [l for l in code if l and not l.startswith((";", ".", "//")) and not l.endswith(":")]
    loads = [i for i, l in enumerate(code) if l.startswith("global_load_lds_dwordx4")]
    assert len(loads) >= 4 * 12
    setters = set()
    for i in loads:
        assert re.match(r"s_nop \d+$", code[i - 1]), code[i - 1]
        assert re.match(r"s_mov_b32 m0,", code[i - 2]), code[i - 2]
        assert not re.search(r"\bs\[\d+:\d+\]", code[i]), "a base address in scalar registers needs more wait states"
        setters.add(i - 2)
    others = [l for i, l in enumerate(code) if re.search(r"\bm0\b", l) and i not in setters]
    assert not others, others[:10]


def test_the_steps_lie_in_the_first_64_kilobytes_of_lds():
    text = open(f"{CSRC}/tree.hip").read()
    body = text[text.index("void tree_rows_kernel"):text.index("static int tree_pieces")]
    assert "__shared__ UnitTable" not in body and body.count("__shared__") == 1  # nothing static in front of the dynamic part
    step = int(re.search(r"kStepBytes = (\d+);", text).group(1))
    assert 2 * step <= 1 << 16
