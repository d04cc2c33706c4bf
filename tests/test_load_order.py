"""Built code: the wavefronts that load for the weight gradient from 8-bit blocks request a k-step's codes behind its rows of dY.  They wait for the
codes only, and take the rows to have landed then.  Read from this repository's own library; no GPU."""
import glob
import os
import shutil
import subprocess

import pytest

from paper_2405_16325_amd.build import LIB_PATH

BIN = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin")
OBJDUMP, READELF = os.path.join(BIN, "llvm-objdump"), os.path.join(BIN, "llvm-readelf")


def late_rows(instructions):
    """Requests of rows (memory to LDS) behind requests of codes (memory to registers) without a branch or barrier between, those of later k-steps."""
    late, codes = [], False
    for text in instructions:
        op = text.split()[0]
        if op.startswith(("s_cbranch", "s_branch", "s_barrier", "s_endpgm")):
            codes = False
        elif op == "buffer_load_dwordx4" and text.split()[-1] == "lds":
            late += [text] if codes else []
        elif op in ("buffer_load_dwordx2", "buffer_load_ubyte"):
            codes = True
    return late


ROWS, CODES, BYTES = "buffer_load_dwordx4 v1, s[8:11], 0 offen lds", "buffer_load_dwordx2 v[2:3], v4, s[4:7], 0 offen", "buffer_load_ubyte v5, v6, s[0:3], 0 offen"


@pytest.mark.parametrize("steps,late", [([ROWS, ROWS, CODES, BYTES], 0), ([ROWS, CODES, ROWS, BYTES], 1), ([CODES, BYTES, ROWS, ROWS], 2),
                                        ([CODES, BYTES, "s_cbranch_scc1 20", ROWS], 0), ([CODES, "s_waitcnt vmcnt(0)", ROWS], 1),
                                        ([ROWS, CODES, "s_barrier", ROWS, CODES], 0), (["buffer_load_dwordx4 v[0:3], v4, s[4:7], 0 offen", CODES], 0)])
def test_the_check_itself(steps, late):
    assert len(late_rows(steps)) == late


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """{symbol: instructions} of the product's kernels that take 8-bit blocks"""
    if not (os.path.exists(OBJDUMP) and os.path.exists(READELF)):
        pytest.skip("no llvm-objdump or llvm-readelf")
    folder = tmp_path_factory.mktemp("code")
    lib = shutil.copy(LIB_PATH, folder / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", lib], check=True, cwd=folder, stdout=subprocess.DEVNULL)
    found = {}
    for part in glob.glob(str(folder / "*gfx950*")):
        symbols = subprocess.run([READELF, "--symbols", "--wide", part], check=True, capture_output=True, text=True).stdout
        names = [n for n in {line.split()[-1] for line in symbols.splitlines() if line.strip()} if "dense_tn_kernel" in n and ("BlocksX" in n or "BlockSlabs" in n) and not n.endswith(".kd")]
        if not names:
            continue
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", "--no-leading-addr", "--disassemble-symbols=" + ",".join(names), part], check=True,
                              capture_output=True, text=True).stdout
        for line in text.splitlines():
            if line.endswith(">:"):
                found[line.split("<")[-1][:-2]] = mine = []
            elif line.startswith("\t") and line.strip():
                mine.append(line.split("//")[0].strip())
    return found


def test_codes_are_requested_behind_rows(kernels):
    assert len(kernels) == 10                                               # five tiles, whole and in slabs
    for name, instructions in kernels.items():
        ops = [i.split()[0] for i in instructions]
        assert "buffer_load_ubyte" in ops and any(i.split()[-1] == "lds" for i in instructions), name
        assert not late_rows(instructions), name
