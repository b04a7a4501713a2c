"""The device code of libgspn.so as it was built: a vector register that a store of more
than 32 bits reads its data from is not written by the instructions right behind the
store, which the hardware has been seen to let through (the stored value is then the new
one in some lanes)."""
import os
import re
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

from paper_2606_00746_amd import LIB_PATH
from paper_2606_00746_amd import build as lib_build

STATES = 16    # wait states that the library's stores have behind them

STORE = re.compile(r"(?:global|buffer|flat)_store_dwordx[234]\s")


def registers(operand):
    m = re.match(r"([va])\[(\d+):(\d+)\]$", operand) or re.match(r"([va])(\d+)$", operand)
    if not m:
        return set()
    lo, hi = int(m.group(2)), int(m.group(m.lastindex))
    return {(m.group(1), i) for i in range(lo, hi + 1)}


def overwritten(lines):
    """(kernel, store, the instruction behind it that writes its data) of a listing."""
    code, kernel, found = [], "", []
    for ln in lines:
        m = re.match(r"[0-9a-f]+ <(.*)>:", ln)
        if m:
            kernel = m.group(1)
            continue
        ins = ln.split("//")[0].strip()
        if ins:
            code.append((kernel, ins))
    for i, (kernel, ins) in enumerate(code):
        if not STORE.match(ins):
            continue
        ops = [o.strip() for o in ins.split(None, 1)[1].split(",")]
        data = registers(ops[0] if ins.startswith("buffer") else ops[1])
        left = STATES
        for k, behind in code[i + 1:i + 1 + STATES]:
            left -= 1 + int(behind.split()[1]) if behind.startswith("s_nop") else 1
            if left < 0 or k != kernel or behind.startswith(("s_endpgm", "s_branch", "s_setpc")):
                break
            if behind.startswith("v_") and registers(behind.split(None, 1)[1].split(",")[0].strip()) & data:
                found.append((kernel, ins, behind))
                break
    return found


def test_the_search_finds_such_a_write():
    listing = """
0000000000001000 <kernel>:
	global_store_dwordx2 v[20:21], v[0:1], off                 // 00: 0
	s_nop 0
	v_or_b32_e32 v{}, 8, v77
	s_nop 7
	v_mov_b32_e32 v2, v3
	s_endpgm
"""
    assert len(overwritten(listing.format(1).splitlines())) == 1
    assert overwritten(listing.format(4).splitlines()) == []
    assert overwritten(listing.format(20).splitlines()) == []     # the address
    assert overwritten(listing.replace("s_nop 0", "s_nop 7\n\ts_nop 7").format(1).splitlines()) == []


def test_no_wide_store_loses_its_data(tmp_path):
    tool = os.path.join(os.path.dirname(os.path.realpath(lib_build.hipcc())), "..", "llvm", "bin", "llvm-objdump")
    tool = tool if os.path.exists(tool) else "/opt/rocm/llvm/bin/llvm-objdump"
    lib = shutil.copy(LIB_PATH, tmp_path)
    subprocess.run([tool, "--offloading", lib], cwd=tmp_path, check=True, capture_output=True)
    objects = sorted(f for f in os.listdir(tmp_path) if "gfx950" in f)
    assert objects

    def listing(f):
        r = subprocess.run([tool, "-d", "--no-show-raw-insn", str(tmp_path / f)], check=True, capture_output=True, text=True)
        return r.stdout.splitlines()

    stores, found = 0, []
    with ThreadPoolExecutor(8) as ex:
        for lines in ex.map(listing, objects):
            stores += sum(1 for ln in lines if STORE.match(ln.strip()))
            found += overwritten(lines)
    assert stores > 1000
    assert not found, found[:5]


def shared_tiles(source):
    """(kernel's mangled name, bytes, alignment) of the [2][2][bytes] arrays of LDS that a
    source declares, as the compiler's front end has them."""
    cmd = [lib_build.hipcc(), *lib_build.HIPCC_FLAGS, *lib_build.SOURCE_FLAGS.get(source, []), "-x", "hip",
           "--offload-device-only", "-Xclang", "-disable-llvm-passes", "-S", "-emit-llvm",
           os.path.join(lib_build.CSRC, source), "-o", "-"]
    out = subprocess.run(cmd, check=True, capture_output=True, text=True).stdout
    found = re.findall(r"^@(\S+) = .*addrspace\(3\) global \[2 x \[2 x \[(\d+) x i8\]\]\] .*align (\d+)", out, re.M)
    return [(name, int(size), int(align)) for name, size, align in found]


def test_tiles_in_lds_begin_at_rows():
    """Attention's tiles of 64 rows are read at addresses formed by exclusive ors inside a
    row: an array of them is aligned to a row, not by luck of what lies ahead of it."""
    with ThreadPoolExecutor(2) as ex:
        tiles = sum(ex.map(shared_tiles, ("attn_fwd.hip", "attn_bwd.hip")), [])
    assert len(tiles) >= 8
    for name, size, align in tiles:
        assert align % (size // 64) == 0, (name, size, align)
