"""The LDS copies of the matrix products, which are written as inline assembly: the distances that test_copy_wait_states.py looks for, in every kernel of theirs."""
import os
import re
import shutil
import subprocess

import pytest

from test_copy_wait_states import OBJDUMP, too_close


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="needs ROCm's llvm-objdump")
def test_copies_keep_their_distances(tmp_path):
    from paper_2012_09849_amd import binding, build
    binding.load_library()
    lib = shutil.copy(build.LIB, tmp_path)
    subprocess.run([OBJDUMP, "--offloading", lib], check=True, capture_output=True, cwd=tmp_path)
    copying = 0
    for code in sorted(tmp_path.glob("*gfx950")):
        text = subprocess.run([OBJDUMP, "-d", "--mcpu=gfx950", str(code)], check=True, capture_output=True, text=True).stdout
        for name, body in re.findall(r"^[0-9a-f]+ <(\S+)>:\n(.*?)(?=^\s*$|\Z)", text, flags=re.S | re.M):
            if "product_kernel" not in name:
                continue
            lines = [line.split("//")[0].strip() for line in body.splitlines()]
            if any(line.startswith("buffer_load") and line.endswith(" lds") for line in lines):
                copying += 1
                assert not too_close(lines), name
    assert copying >= 24                  # three layouts, two types, four or more tilings
