"""What the compiler makes of single tokens' kernel under a view at every width (no GPU
needed)."""
import os
import re
import subprocess

import pytest

from paper_2608_30963_amd import build as B

SOURCE = """#include "attn_forward_kernels.h"
namespace kvx {{
namespace {{
{}
}}
}}
"""


def _kernels(width, tmp_path):
    """Assembly of forward_few of a width: {symbol: lines}, and {symbol: bytes of scratch
    memory a lane}."""
    try:
        cc = B.hipcc()
    except RuntimeError:
        pytest.skip("hipcc not available")
    src, out = tmp_path / "few.hip", tmp_path / "few.s"
    src.write_text(SOURCE.format("\n".join(
        f"template __global__ void forward_few<{s}, {width}, Cap::{cap}>(AttnView, ForwardPlan);"
        for s in ("bf16_t", "code_i8", "code_e4m3") for cap in ("none", "part", "tanh"))))
    subprocess.run([cc] + B._flags() + ["-S", "--cuda-device-only", str(src), "-o", str(out)],
                   check=True, capture_output=True)
    text = out.read_text()
    body = {m.group(1): text[m.end():text.index("s_endpgm", m.end())].splitlines()
            for m in re.finditer(r"^(_ZN\S*forward_few\S*):", text, re.M)}
    scratch = dict(re.findall(r"\.set (_ZN\S*forward_few\S*)\.private_seg_size, (\d+)", text))
    return body, {k: int(v) for k, v in scratch.items()}


@pytest.mark.parametrize("width", [64, 128, 256])
def test_nothing_is_kept_in_scratch_memory(width, tmp_path):
    """Registers hold all of a wave's work: what is read back from scratch memory is waited
    for, and all copies in flight with it.  Blocks that copy, or that multiply a tile, have
    no wait of the compiler's."""
    body, scratch = _kernels(width, tmp_path)
    assert len(body) == len(scratch) == 9
    assert set(scratch.values()) == {0}, scratch
    for name, lines in body.items():
        blocks, written = [[]], False
        for line in (x.strip() for x in lines):
            if line.startswith((".LBB", "; %bb")):
                blocks.append([])
            written = (written or "ASMSTART" in line) and "ASMEND" not in line
            if line and not line.startswith((";", ".")):
                blocks[-1].append((written, line))
        seen = 0
        for block in blocks:
            copies = any("global_load_lds_dwordx4" in x for _, x in block)
            if not copies and sum("v_mfma" in x for _, x in block) < width // 16:
                continue
            seen += 1
            assert not any(not asm and re.search(r"vmcnt\(\d+\)$", x) for asm, x in block), name
        assert seen >= 4, name
