"""The attention kernels' machine code, as the compiler writes it: sums, operands and keys on their way stay in registers, nothing goes through memory of
a thread's own.  (The compiler may reserve such memory for scalars that it then keeps in a vector register's lanes, so the size it
reserves says nothing.)"""

import os
import re
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_1711_07240_amd import build as B

UNITS = [u for u in B._units("") if os.path.basename(u[1]) == "cgbn_attention_inst.hip"]


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    if not os.path.exists(B.HIPCC):
        pytest.skip("no compiler")
    folder = tmp_path_factory.mktemp("attention")

    def compile_one(unit):
        out = folder / (unit[0] + ".s")
        subprocess.run([B.HIPCC] + B.FLAGS + unit[2] + ["--cuda-device-only", "-S", unit[1], "-o", str(out)], check=True, capture_output=True)
        return out.read_text()

    with ThreadPoolExecutor(max_workers=len(UNITS)) as ex:
        return dict(zip((u[0] for u in UNITS), ex.map(compile_one, UNITS)))


@pytest.mark.parametrize("unit", [u[0] for u in UNITS])
def test_nothing_is_spilled_to_memory(assembly, unit):
    code = assembly[unit]
    assert set(re.findall(r"\.vgpr_spill_count:\s*(\d+)", code)) == {"0"}
    assert not re.search(r"^\s*scratch_(load|store)", code, re.M) and len(re.findall("global_load_lds_dwordx4", code)) > 50
