"""ISA guard (CPU) of the sources whose matrix instructions sum integers: only the
8-bit-to-32-bit-integer kinds, whose sums are exact in any order, and none of the
floating-point forms that the other sources must not hold either."""
import pytest

import test_isa_guard as guard
from paper_2502_19405_amd import build

INTEGER_MFMA = {"v_mfma_i32_32x32x32_i8", "v_mfma_i32_16x16x64_i8"}


@pytest.mark.parametrize("src", build.INTEGER_SOURCES)
def test_only_integer_matrix_instructions(src):
    text = build.disassemble(src)
    used = {m.group(1) for line in guard.instructions(text) for m in [guard.MFMA.match(line)] if m}
    assert used == INTEGER_MFMA, used
    bad = [b for b in guard.scan(text) if not b.startswith("multi-term matrix instruction")]
    assert not bad, bad[:3]


def test_every_source_is_under_a_guard():
    import os
    sources = {f for f in os.listdir(build.CSRC) if f.endswith((".hip", ".cpp"))}
    assert sources == set(build.SOURCES) | set(build.INTEGER_SOURCES)
    assert not set(build.SOURCES) & set(build.INTEGER_SOURCES)
