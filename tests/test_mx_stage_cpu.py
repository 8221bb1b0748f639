"""The product's loads into LDS stay inside their matrices: the offset that the
buffer's range check is documented to cover, the lane's own, lies inside for
every live piece of a stage, at that piece, and outside for everything else
(rows past the matrix, stages past the row); the scalar offset, which it does not
cover, is zero."""
import ctypes
import os
import re
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2002_09049_amd", "csrc")


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    so = str(tmp_path_factory.mktemp("host") / "mx_stage.so")
    subprocess.check_call(["g++", "-O2", "-std=c++17", "-shared", "-fPIC", "-I", CSRC,
                           os.path.join(ROOT, "tests", "host", "mx_stage_host.cpp"), "-o", so])
    lib = ctypes.CDLL(so)
    for f, n in ((lib.tile_offset, 6), (lib.slab_offset, 5)):
        f.argtypes = [ctypes.c_int] * n
        f.restype = ctypes.c_uint32
    return lib


def _call_args(text, name):
    """The arguments of every call of a builtin in a source."""
    out = []
    for m in re.finditer(re.escape(name) + r"\(", text):
        depth, arg, args = 1, "", []
        for ch in text[m.end():]:
            depth += ch in "([{"
            depth -= ch in ")]}"
            if depth == 0 or (depth == 1 and ch == ","):
                args.append(arg.strip())
                arg = ""
                if depth == 0:
                    break
            else:
                arg += ch
        out.append(args)
    return out


def test_scalar_offsets_are_zero():
    seen = 0
    for name in sorted(os.listdir(CSRC)):
        if not name.startswith("mx"):
            continue
        text = open(os.path.join(CSRC, name)).read()
        for args in _call_args(text, "__builtin_amdgcn_raw_ptr_buffer_load_lds"):
            assert args[4] == "0", (name, args)
            seen += 1
        for args in _call_args(text, "__builtin_amdgcn_raw_buffer_load_b128"):
            assert args[2] == "0", (name, args)
            seen += 1
    assert seen == 2


@pytest.mark.parametrize("nb", [4, 8, 12, 64, 784, 131072])
@pytest.mark.parametrize("rows,tile_rows", [(1, 64), (15, 64), (16, 128), (63, 64), (64, 64), (130, 256), (255, 256), (256, 256)])
def test_tiles(host, nb, rows, tile_rows):
    row_bytes, records = 16 * nb, rows * 16 * nb
    stages = -(-nb // 4)
    for st in sorted({0, 1, stages - 1, stages, stages + 2} & set(range(stages + 3))):
        for row in range(0, tile_rows, 16):
            loads = tile_rows // 64             # of a wavefront, which has a quarter of the rows
            row0, k = row // 16 // loads * loads * 16, row // 16 % loads
            for lane in range(64):
                at = host.tile_offset(row0, k, lane, row_bytes, st, nb)
                mine = row + lane // 4
                if mine < rows and st < stages:
                    want = mine * row_bytes + st * 64 + ((lane % 4) ^ (lane // 16)) * 16
                    assert at == want and at + 16 <= records
                else:
                    assert at >= records and at + 16 <= 1 << 32


@pytest.mark.parametrize("nb", [4, 12, 16, 20, 64, 784, 131072])
@pytest.mark.parametrize("rows", [1, 3, 4, 15, 16, 17, 63, 64])
def test_slabs(host, nb, rows):
    row_bytes, records = 16 * nb, rows * 16 * nb
    stages = -(-nb // 16)
    for st in sorted({0, stages - 1, stages, stages + 2}):
        for base in range(0, 64, 16):           # the four loads of the tokens; W's is the first
            for row in range(16):
                at = [(host.slab_offset(row, r, row_bytes, st, nb) + base * row_bytes) for r in range(16)]
                assert max(at) < 1 << 32
                inside = np.array(at) < records
                pieces = 16 * st + (np.arange(16) ^ row)
                assert np.array_equal(inside, (pieces < nb) & (base + row < rows))
                want = (base + row) * row_bytes + pieces * 16
                assert np.array_equal(np.array(at)[inside], want[inside])
