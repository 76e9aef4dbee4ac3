"""What the device code tells the compiler, read from the LLVM IR and the assembly of small kernels
compiled here from the library's headers."""
import re
import subprocess
from pathlib import Path

from paper_2206_01299_amd import build as _build

ROOT = Path(__file__).resolve().parent.parent


def _compile(tmp_path, text, *flags):
    src = tmp_path / "probe.hip"
    src.write_text(text)
    r = subprocess.run([_build.HIPCC, *_build.FLAGS, "--cuda-device-only", "-S", *flags, str(src), "-o", "-"],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    return r.stdout


def test_pieces_at_any_element_are_stored_without_a_promise_of_alignment(tmp_path):
    """Rows and groups that are no whole 16-byte pieces start at any element: a store of such a piece may
    promise the element's alignment and no more, and is one instruction all the same."""
    text = """
#include "aqsgd_anygroup.h"
using namespace aqsgd;
extern "C" __global__ void raw(char* p, u32x4_t a, f32x4_t b) { store16(p, a, false); store16(p + 64, b, false); }
extern "C" __global__ void f16(char* p, float x) { float v[8] = {x, x, x, x, x, x, x, x}; store_piece<AQSGD_F16, 8>(p, v); }
extern "C" __global__ void f32(char* p, float x) { float v[4] = {x, x, x, x}; store_piece<AQSGD_F32, 4>(p, v); }
extern "C" __global__ void units(char* p, Raw<AQSGD_F32> r) { store_raw_units(p, p + 100, r, false); }
"""
    ir = _compile(tmp_path, text, "-emit-llvm")
    stores = re.findall(r"store <\d x (\w+)> .*?align (\d+),.*!nontemporal", ir)
    assert len(stores) == 6, ir
    for kind, align in stores:
        assert int(align) <= (4 if kind == "float" else 2), stores
    asm = _compile(tmp_path, text)
    wide = [l for l in asm.splitlines() if re.search(r"global_store_dwordx4 .*\bnt\b", l)]
    assert len(wide) == len(stores), asm


def _bodies(text, opening):
    """(head, body) of every block that a match of `opening` begins; the match ends with the opening brace."""
    for m in re.finditer(opening, text):
        depth, end = 1, m.end()
        while depth:
            depth += {"{": 1, "}": -1}.get(text[end], 0)
            end += 1
        yield m.group(0), text[m.end():end - 1]


def test_loops_with_a_barrier_turn_as_often_for_every_wave_of_a_workgroup():
    """A barrier waits for the whole workgroup, so a loop that has one in it goes by the workgroup's number, never by a team's
    or a lane's: where only some of the teams have a row, the others go along without storing.  Sums over a team of several waves have a
    barrier in them."""
    barrier = re.compile(r"__syncthreads\(|\bteam_(?:sum|sums|top)<|\bworkgroup_sum<")
    own = re.compile(r"\bteam\b|\blane\b|\bslot\b|threadIdx")
    loops = 0
    for name in ("aqsgd_layernorm.h", "aqsgd_layernorm.hip", "aqsgd_grad_norm.hip", "aqsgd_adamw.h"):
        text = re.sub(r"//[^\n]*", "", (_build.CSRC / name).read_text())
        for head, body in _bodies(text, r"__global__[^;{]*\{"):
            kernel = re.search(r"(\w+)\(const", head).group(1)
            for loop, inside in _bodies(body, r"\bfor \([^{;]*;[^{;]*;[^{;]*\) \{"):
                if not barrier.search(inside):
                    continue
                loops += 1
                init, until = loop.replace("(kAlone ? team : 0)", "").split(";")[:2]      # of a wave that is a team, there
                assert not own.search(init) and not own.search(until), f"{kernel}: {loop}"
                for leave in re.finditer(r"^\s*if \(([^{;]*)\) (?:return|continue|break);", inside, re.M):
                    assert "TEAM <= kWave" in leave.group(1) or "kAlone" in leave.group(1) or not re.search(own.pattern + r"|\bhere\b", leave.group(1)), f"{kernel}: {leave.group(0)}"
    assert loops >= 5
