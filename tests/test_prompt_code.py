"""The generated code of the prompts' attention, whose loads into LDS and products onto
accumulators are inline assembly that the compiler's hazard recogniser does not look into:
the wait states that CDNA4 asks for around them have to be there on every path."""

import os
import re
import subprocess

import pytest

from paper_2505_12398_amd import build as B
from test_lmhead_code import violations

pytestmark = pytest.mark.slow


def of_assembly(found):
    """Hazards of the products that are in assembly: their results are accumulators a[..]; the others
    the compiler knows (it writes and reads vector registers)."""
    write, read = found.split(" -> ")
    if "buffer_load" in read:
        return True
    product = write if write.startswith("v_mfma") else read
    return re.match(r"v_mfma\S+ a\[", product) is not None


def test_prompt_wait_states(tmp_path):
    if not os.path.exists(B.HIPCC):
        pytest.skip("no hipcc")
    out = tmp_path / "prompt.s"
    flags = [f for f in B.FLAGS if f not in ("-shared", "-Wall")] + B.SOURCE_FLAGS["tv_prompt.hip"]
    subprocess.run([B.HIPCC, *flags, "--cuda-device-only", "-S", "-I", B.INCLUDE, "-I", B.CSRC,
                    os.path.join(B.CSRC, "tv_prompt.hip"), "-o", str(out)], check=True,
                   capture_output=True)
    text = out.read_text()
    kernels = re.findall(r"^(_ZN\S*prompt_kernel\S*):\s*;.*?\n(.*?)^\.Lfunc_end", text, re.M | re.S)
    assert len(kernels) == 10          # two types; heads of 64 in three heights, of 128 in two
    for name, body in kernels:
        assert re.search(r"v_mfma_f32_32x32x16_b?f16 a\[", body) and re.search(r"offen lds", body)
        assert [f for f in violations(body) if of_assembly(f)] == [], name
