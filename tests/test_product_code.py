"""The matrix products' machine code, as the compiler writes it: what their loads to LDS, which are written out, rely on.

Such a load reads its base address from two scalar registers.  Within five wait states of the vector unit's writing one of them it may read the
old value, and the compiler, which sees to that for its own instructions, does not look into written ones.  The address is
kept by scalar instructions throughout, unless a register is spilled to a vector register's lane and brought back, or a value
taken for one that differs from lane to lane; the kernels must not come to that."""

import os
import re
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_1711_07240_amd import build as B

NEEDED = 5
LOAD = re.compile(r"global_load_lds_dwordx4\s+v\d+,\s*s\[(\d+):(\d+)\]")


def _scalars_written(line):
    """The scalar registers that a vector instruction writes."""
    m = re.match(r"(v_\w+)\s+s(?:(\d+)|\[(\d+):(\d+)\])", line)
    if not m:
        return set()
    return {int(m[2])} if m[2] else set(range(int(m[3]), int(m[4]) + 1))


def _states(line):
    m = re.match(r"s_nop\s+(\d+)", line)
    return int(m[1]) + 1 if m else 1


def unsafe_loads(assembly):
    """Loads whose address a vector instruction wrote fewer than NEEDED wait states before, along the code as it stands."""
    code = [line.split(";")[0].strip() for line in assembly.splitlines()]
    code = [line for line in code if line and not line.startswith(".") and not line.endswith(":")]
    found, loads = [], 0
    for at, line in enumerate(code):
        m = LOAD.match(line)
        if not m:
            continue
        loads += 1
        base, between, back = set(range(int(m[1]), int(m[2]) + 1)), 0, at - 1
        while back >= 0 and between < NEEDED:
            if _scalars_written(code[back]) & base:
                found.append((code[back], line))
                break
            between += _states(code[back])
            back -= 1
    return found, loads


def test_the_check_sees_what_it_looks_for():
    load = "s_mov_b32 m0, s9\n\ts_nop 0\n\tglobal_load_lds_dwordx4 v3, s[10:11]\n"
    for before, bad in (("v_readlane_b32 s11, v40, 3", 1), ("v_readfirstlane_b32 s10, v1", 1), ("v_cmp_gt_u32_e64 s[10:11], v1, v2", 1),
                        ("v_readlane_b32 s12, v40, 3", 0), ("s_add_u32 s10, s10, s4", 0), ("v_readlane_b32 s11, v40, 3\n\ts_nop 2", 0),
                        ("v_readlane_b32 s11, v40, 3\n\ts_nop 1", 1), ("v_readlane_b32 s11, v40, 3\n.LBB0_1:\n\tv_add_u32 v1, v2, v3", 1)):
        found, loads = unsafe_loads(f"\t{before} ; comment\n\t{load}")
        assert len(found) == bad and loads == 1, before


UNITS = [u for u in B._units("") if os.path.basename(u[1]) == "cgbn_gemm_inst.hip"]


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    if not os.path.exists(B.HIPCC):
        pytest.skip("no compiler")
    folder = tmp_path_factory.mktemp("products")

    def compile_one(unit):
        out = folder / (unit[0] + ".s")
        subprocess.run([B.HIPCC] + B.FLAGS + unit[2] + ["--cuda-device-only", "-S", unit[1], "-o", str(out)], check=True, capture_output=True)
        return out.read_text()

    with ThreadPoolExecutor(max_workers=min(len(UNITS), int(os.environ.get("MAX_JOBS", os.cpu_count() or 1)))) as ex:
        return dict(zip((u[0] for u in UNITS), ex.map(compile_one, UNITS)))


@pytest.mark.parametrize("unit", [u[0] for u in UNITS])
def test_no_load_follows_a_vector_write_of_its_address(assembly, unit):
    found, loads = unsafe_loads(assembly[unit])
    assert loads > 50 and not found
    spills = re.findall(r"\.sgpr_spill_count:\s*(\d+)", assembly[unit])
    assert spills and set(spills) == {"0"}
