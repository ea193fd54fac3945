"""The results of matrix products are in their registers some wait states after the instruction, and the hardware does not check; the compiler, which puts the
states in, has left them out on the way around a branch that is taken.  Here every path behind every product of every kernel is looked at.  CPU only."""
import re
import shutil

import pytest

from tests.test_kernel_resources import compiled, reached

# Wait states until anything but another product may read or overwrite the result: passes and three (products of 32-bit values: and two).
STATES = {"v_mfma_f32_32x32x16_bf16": 11, "v_mfma_f32_16x16x32_bf16": 7, "v_mfma_f32_32x32x2_f32": 18, "v_mfma_f32_16x16x4_f32": 10}


def _registers(operand):
    out = set()
    for kind, first, last in re.findall(r"\b([av])\[(\d+):(\d+)\]", operand):
        out |= {(kind, i) for i in range(int(first), int(last) + 1)}
    return out | {(kind, int(i)) for kind, i in re.findall(r"\b([av])(\d+)\b", operand)}


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
def test_results_of_products_are_waited_for_on_every_path():
    products = 0
    for name, body in compiled()[1].items():
        labels = {operands[0]: i for i, (op, operands) in enumerate(body) if op is None}
        for i, (op, operands) in enumerate(body):
            if op is None or not op.startswith("v_mfma"):
                continue
            products += 1
            result = _registers(operands[0])
            late = [c for c in reached(body, labels, i, STATES[op]) if c[0].startswith(("v_", "ds_", "global_", "buffer_", "flat_", "scratch_"))
                    and not c[0].startswith("v_mfma") and any(_registers(o) & result for o in c[1] if o)]
            assert not late, (name, i, op, operands, late)
    assert products > 20000
