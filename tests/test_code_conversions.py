"""The packing conversion of 32 binary16 codes to 6-bit floats in the built library (no GPU needed), as tests/test_conversion_operands.py looks at that of
32-bit values: the result has registers of its own, apart from the operand that the conversion still reads."""
import re
import subprocess

from paper_2501_15021_amd import binding as akvq
from test_conversion_operands import OBJDUMP, overlap
from test_kernel_resources import _code_objects

CONVERSION = re.compile(r"v_cvt_scalef32_pk32_fp6_f16 v\[(\d+):(\d+)\], v\[(\d+):(\d+)\]")


def test_no_result_lies_in_the_operand(tmp_path):
    seen = 0
    for i, image in enumerate(_code_objects(open(akvq.LIB_PATH, "rb").read())):
        path = tmp_path / f"{i}.co"
        path.write_bytes(image)
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", str(path)], capture_output=True, text=True, check=True).stdout
        for m in CONVERSION.finditer(text):
            out, codes = (int(m[1]), int(m[2])), (int(m[3]), int(m[4]))
            seen += 1
            assert out[1] - out[0] == 5 and codes[1] - codes[0] == 15 and not overlap(out, codes), m[0]
    assert seen >= 2
