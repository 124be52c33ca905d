"""The check of tests/test_matrix_wait_states.py for the kernels with matrix instructions of 16-bit operands (build.MATRIX_16_SOURCES).

A product of 16 x 16 over 32 takes four passes, and a straight piece of code gets seven wait states from the compiler between it and a vector or
memory instruction that touches its result."""
import concurrent.futures as cf
import os
import shutil
import subprocess
import sys

import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import test_matrix_wait_states as waits  # noqa: E402

MORE = {"v_mfma_f32_16x16x32_bf16": (7, 7), "v_mfma_f32_16x16x32_f16": (7, 7)}


def test_the_check_knows_the_instructions(monkeypatch):
    monkeypatch.setattr(waits, "NEED", {**waits.NEED, **MORE})
    for op in MORE:
        text = ["k:", f"\t{op} v[0:3], v[8:11], v[12:15], v[0:3]", "\ts_nop 5", "\tv_add_f32_e32 v3, v7, v3", "\ts_endpgm", ".Lfunc_end0:"]
        (_, code, labels), = waits._kernels(text)
        assert waits._too_early(code, labels) == {(op, "v_add_f32_e32", 6)}
        text[2] = "\ts_nop 6"
        (_, code, labels), = waits._kernels(text)
        assert waits._too_early(code, labels) == set()


@pytest.mark.slow
@pytest.mark.timeout(900)
def test_results_of_matrix_instructions_of_16_bits_are_waited_for(tmp_path, monkeypatch):
    if shutil.which("hipcc") is None:
        pytest.skip("hipcc not found")
    from paper_2202_13638_amd import build
    monkeypatch.setattr(waits, "NEED", {**waits.NEED, **MORE})

    def assembly(src):
        out = str(tmp_path / (src + ".s"))
        r = subprocess.run(["hipcc", *build.FLAGS, "--cuda-device-only", "-S", os.path.join(build.CSRC, src), "-o", out],
                           capture_output=True, text=True)
        assert r.returncode == 0, r.stderr
        with open(out) as f:
            return f.readlines()

    with cf.ThreadPoolExecutor(max_workers=6) as ex:
        texts = list(ex.map(assembly, build.MATRIX_16_SOURCES))
    matrix, bad = 0, {}
    for lines in texts:
        for name, code, labels in waits._kernels(lines):
            matrix += sum(op.startswith("v_mfma") for op, _ in code)
            found = waits._too_early(code, labels)
            if found:
                bad[name] = sorted(found)
    assert matrix > 1000
    assert not bad, bad
