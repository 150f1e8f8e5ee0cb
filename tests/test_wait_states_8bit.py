"""The machine code of libalcop_f8.so, scanned as that of libalcop.so is (test_wait_states.py): its matrix instruction, of 16
passes, has another distance to the first use of its result."""
import os

import pytest

import test_wait_states as w
from paper_2210_16691_amd import build as b

DISTANCE = {"32x32x64": 16 + 4}


def test_the_scan_knows_the_instruction(monkeypatch):
    monkeypatch.setattr(w, "MATRIX_WAIT", DISTANCE)
    matrix, read = "v_mfma_f32_32x32x64_f8f6f4 v[0:15], v[20:27], v[28:35], v[0:15]", "v_add_f32_e32 v40, v15, v15"
    for last, n in ((3, 0), (2, 1)):
        code = [matrix, "s_nop 15", "s_nop %d" % last, read, "s_endpgm"]
        text = "\n".join("\t%s // %012X: 00000000 " % (t, 0x100 + 4 * k) for k, t in enumerate(code))
        seen, bad = w.matrix_violations(text, 0x100)
        assert seen == 1 and len(bad) == n


def test_the_kernels_of_the_8_bit_instruction(tmp_path, monkeypatch):
    if not os.path.exists(w.OBJDUMP):
        pytest.skip("no llvm-objdump")
    monkeypatch.setattr(w, "MATRIX_WAIT", DISTANCE)
    loads = tiles = matrix = 0
    for code in w._code_objects(b.F8_LIB):
        path = str(tmp_path / "code.co")
        open(path, "wb").write(code)
        (n, bad), late, k, (m, early), (_, stores) = w._scan(path)
        assert not bad and not late and not early and not stores, (bad[:2], late[:2], early[:2], stores[:2])
        loads, tiles, matrix = loads + n, tiles + k, matrix + m
    assert tiles >= 18 and matrix >= 18 * 8 and loads > 0
