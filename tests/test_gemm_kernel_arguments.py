"""What the GEMM instances read of their arguments, in the built gfx950 code.

Operands of fewer rows than the output (Params::rows_a, rows_b) belong to the
distillation loss's dz kind alone. A tile's first vector loads wait for the row
counts, so in every other kind those are M and N, which the kernel reads
anyway: a load of rows_a or rows_b there is one more that its start waits for.
"""

import os
import re
import subprocess

from test_build_code_objects import ROOT, _listings, _objects

CSRC = os.path.join(ROOT, "paper_2608_27370_amd", "csrc")
DZ_T = 7                                  # kOutSoftmaxGradT


def _offsets(tmp_path):
    """Byte offsets of the fields of the GEMM kernel's argument structure."""
    src = tmp_path / "params.hip"
    src.write_text('#include "gemm_common.h"\nint bytes = sizeof(puro::gemm_detail::Params);\n')
    r = subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "--offload-arch=gfx950", "--cuda-host-only", "-std=c++17",
                        "-fsyntax-only", "-Xclang", "-fdump-record-layouts", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
                        str(src)], check=True, capture_output=True, text=True)
    body = re.search(r"0 \| struct puro::gemm_detail::Params\n(.*?)\[sizeof", r.stdout, re.S).group(1)
    return {m.group(2): int(m.group(1)) for m in re.finditer(r"^ *(\d+) \|   \S.* (\w+)$", body, re.M)}


def test_only_the_distillation_gradient_reads_its_operands_rows(tmp_path):
    objs = [o for o in _objects() if os.path.basename(o).startswith("gemm_kernel")]
    at = _offsets(tmp_path)
    lo, hi = at["rows_a"], at["rows_b"] + 4
    assert hi == lo + 8 and at["M"] < lo
    words = {"": 1, "x2": 2, "x4": 4, "x8": 8, "x16": 16}
    readers, others = 0, 0
    for obj in objs:
        for name, ins in _listings(obj):
            t = re.search(r"gemm_fp8_kernelI((?:Li\d+E){7})", name)
            if not t:
                continue
            kind = [int(v) for v in re.findall(r"\d+", t.group(1))][6]
            loads = [re.match(r"s_load_dword(x\d+)? \S+ (s\[\d+:\d+\]), 0x([0-9a-f]+)$", i) for i in ins if i.startswith("s_load")]
            assert all(loads), [i for i in ins if i.startswith("s_load")]
            spans = [(int(m.group(3), 16), int(m.group(3), 16) + 4 * words[m.group(1) or ""]) for m in loads]
            hit = any(a < hi and b > lo for a, b in spans)
            if kind == DZ_T:
                readers += 1
                assert hit, name
            else:
                others += 1
                assert not hit, name
    assert readers >= 3 and others > 200
