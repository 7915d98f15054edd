"""The tiled 8-bit product issues its matrix instructions as inline assembly with
the accumulators tied to AGPRs, so the compiler's own hazard handling does not
see them.  What the kernel relies on is checked in the assembly that this source
compiles to: inside the k loop nothing but matrix instructions touches an AGPR
and nothing is spilled, accumulators' zeros are not written right before the
first one, no vector instruction writes an operand within two wait states, and
after the last one the pipeline drains before any accumulator is read."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2411_03519_amd import build as b


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    if not (shutil.which(b.HIPCC) or os.path.exists(b.HIPCC)):
        pytest.skip("hipcc not found")
    out = str(tmp_path_factory.mktemp("isa") / "gemm_fp8.s")
    subprocess.run([b.HIPCC, *b.COMMON, *b.DEVICE, "-x", "hip", "--offload-device-only", "-S",
                    os.path.join(b.PKG, "csrc/kernels/gemm_fp8.hip"), "-o", out], check=True, capture_output=True)
    text = open(out).read()
    found = {}
    for m in re.finditer(r"^(_ZN5metro\w*gemm_fp8_tiled_kernel\w*):", text, re.M):
        body = text[m.end():text.index(".Lfunc_end", m.end())]
        found[m.group(1)] = [op for op in (ln.split(";")[0].strip() for ln in body.split("\n")) if re.match(r"[a-z]", op)]
    assert found
    return found


MFMA = re.compile(r"v_mfma_scale_f32_16x16x128_f8f6f4 a\[(\d+):(\d+)\], v\[(\d+):(\d+)\], v\[(\d+):(\d+)\], a\[(\d+):(\d+)\], "
                  r"v(\d+), v(\d+) op_sel_hi:\[0,0,0\]$")


def test_accumulators_stay_in_place(kernels):
    for name, ops in kernels.items():
        mfma = [i for i, op in enumerate(ops) if op.startswith("v_mfma")]
        agpr = [i for i, op in enumerate(ops) if re.search(r"\ba(\[\d|\d)", op) and not op.startswith("v_mfma")]
        inside = [ops[i] for i in agpr if mfma[0] <= i <= mfma[-1]]
        assert not inside, (name, inside[:4])
        assert not [op for op in ops[mfma[0]:mfma[-1]] if op.startswith("scratch_")], name
        reads = {}
        for i in mfma:
            m = MFMA.match(ops[i])
            assert m, (name, ops[i])
            v = list(map(int, m.groups()))
            assert v[0] == v[6] and v[1] == v[7], ops[i]
            reads[i] = set(range(v[2], v[3] + 1)) | set(range(v[4], v[5] + 1)) | {v[8], v[9]}
        # a zero written before the loop is at least 4 instructions old when a matrix instruction adds to it
        first = {}
        for i in reversed(mfma):
            lo, hi = map(int, MFMA.match(ops[i]).groups()[:2])
            first.update((r, i) for r in range(lo, hi + 1))
        for i in agpr:
            if i < mfma[0]:
                m = re.match(r"v_accvgpr_write_b32 a(\d+), 0$", ops[i])
                assert m and first[int(m.group(1))] - i >= 4, (name, ops[i])
        # a vector instruction's result is no operand of a matrix instruction in the next two wait states
        for i in range(mfma[0] - 8, mfma[-1]):
            d = re.match(r"(?!v_mfma|v_cmp)v_\w+ v(?:\[(\d+):(\d+)\]|(\d+))", ops[i])
            if not d:
                continue
            lo, hi = int(d.group(1) or d.group(3)), int(d.group(2) or d.group(3))
            waited, j = 0, i + 1
            while waited < 2 and j < len(ops):
                if j in reads:
                    assert not reads[j] & set(range(lo, hi + 1)), (name, ops[i], ops[j])
                n = re.match(r"s_nop (\d+)", ops[j])
                waited += int(n.group(1)) + 1 if n else 1
                j += 1
        # (zeros of the start may be laid out behind the loop; they branch back to the loads before it)
        after = min(i for i in agpr if i > mfma[-1] and not re.match(r"v_accvgpr_write_b32 a\d+, 0$", ops[i]))
        assert "s_nop 7" in ops[mfma[-1] + 1:after], (name, ops[mfma[-1]:after + 1])
