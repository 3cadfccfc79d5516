"""What the compiler makes of the kernels of serving (no GPU needed)."""
import os
import re
import subprocess

import pytest

from paper_2608_30963_amd import build as B


def _blocks(text, name):
    """(symbol, basic blocks as lists of lines, without what is written out) of kernels."""
    for m in re.finditer(rf"^(_ZN\S*{name}\S*):", text, re.M):
        blocks, written = [[]], False
        for line in text[m.end():text.index("s_endpgm", m.end())].splitlines():
            line = line.strip()
            if line.startswith((".LBB", "; %bb")):
                blocks.append([])
            written = (written or "ASMSTART" in line) and "ASMEND" not in line
            if not written and line and not line.startswith((";", ".")):
                blocks[-1].append(line)
        yield m.group(1), blocks


@pytest.mark.parametrize("coded", [0, 1])
def test_tiles_of_few_rows_do_not_wait_for_copies_in_flight(coded, tmp_path):
    """A load whose branch the compiler has left is waited for where the branches meet, and
    all copies with it: no block with a tile's matrix instructions has such a wait."""
    try:
        cc = B.hipcc()
    except RuntimeError:
        pytest.skip("hipcc not available")
    out = tmp_path / "view.s"
    subprocess.run([cc] + B._flags() + ["-DKVX_ATTN_DP=128", f"-DKVX_ATTN_CODED={coded}", "-S",
                                        "--cuda-device-only", os.path.join(B.CSRC, "attn_view_d.hip"),
                                        "-o", str(out)], check=True, capture_output=True)
    seen = 0
    for name, blocks in _blocks(out.read_text(), "forward_few"):
        for block in blocks:
            if sum("v_mfma" in x for x in block) < 8:
                continue
            seen += 1
            assert not any("vmcnt" in x or "scratch" in x for x in block), name
    assert seen >= 6 * (1 + coded)
