"""What the compiler makes of the decoding kernels (no GPU needed)."""
import os
import re
import subprocess

import pytest

from paper_2608_30963_amd import build as B


def _assembly(unit, dp, tmp_path):
    try:
        cc = B.hipcc()
    except RuntimeError:
        pytest.skip("hipcc not available")
    out = tmp_path / f"{unit}_{dp}.s"
    subprocess.run([cc] + B._flags() + [f"-DKVX_ATTN_DP={dp}", "-S", "--cuda-device-only",
                                        os.path.join(B.CSRC, f"{unit}_d.hip"), "-o", str(out)],
                   check=True, capture_output=True)
    return out.read_text()


def _kernels(text, name):
    """(symbol, basic blocks as lists of lines) of the kernels of a name."""
    for m in re.finditer(rf"^(_ZN\S*{name}\S*):", text, re.M):
        blocks = [[]]
        for line in text[m.end():text.index("s_endpgm", m.end())].splitlines():
            if line.startswith(".LBB"):
                blocks.append([])
            blocks[-1].append(line)
        yield m.group(1), blocks


@pytest.mark.parametrize("dp", [128, 256])
def test_copies_of_single_tokens_do_not_wait_for_each_other(dp, tmp_path):
    """A register that a copy into LDS has to read back from scratch memory makes
    it wait for all copies in flight, which they are there to keep going: less
    than one in eight may."""
    seen = 0
    for name, blocks in _kernels(_assembly("attn_forward", dp, tmp_path), "forward_decode"):
        seen += 1
        copies = reloads = 0
        for b in blocks:
            n = sum("global_load_lds" in x for x in b)
            copies += n
            reloads += sum("scratch_load" in x for x in b) if n else 0
        assert copies >= 32, name
        assert reloads * 8 < copies, (name, reloads, copies)
    assert seen >= 4


def test_written_registers_are_named():
    """Written-out instructions that set M0 or the scalar condition say so: the
    compiler may hold either across them."""
    seen = 0
    for f in sorted(os.listdir(B.CSRC)):
        text = open(os.path.join(B.CSRC, f)).read()
        for m in re.finditer(r"asm volatile\((.*?)\);", text, re.S):
            body = m.group(1)
            for register, written in (("m0", r"s_\w+ m0,"), ("scc", r"s_(add|sub|and|or)_")):
                if re.search(written, body):
                    seen += 1
                    assert f'"{register}"' in body.rsplit(":", 1)[1], (f, body)
    assert seen >= 7
