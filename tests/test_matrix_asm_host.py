"""Inline asm beside matrix instructions that the compiler schedules (no GPU needed).

The compiler puts the waits between a matrix instruction and a vector instruction that writes or reads the same registers by what it knows of both; of an
instruction inside an asm statement it knows nothing.  So the products' sources write no vector instruction by hand: their asm statements hide a value
from the optimiser, wait, or fetch straight into LDS."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2007_14178_amd", "csrc")
SOURCES = sorted(p for name in ("int4_*", "dense_*", "experts_*", "gated_*", "route*") for p in glob.glob(os.path.join(CSRC, name)))


def instructions(source):
    """The instructions of a source's asm statements."""
    for statement in re.finditer(r"\basm\s*(?:volatile\s*)?\(((?:\s*\"(?:[^\"\\]|\\.)*\")+)", source):
        text = "".join(re.findall(r"\"((?:[^\"\\]|\\.)*)\"", statement.group(1)))
        for line in re.split(r"\\n|\\t|;", text):
            if line.strip():
                yield line.strip()


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_no_vector_instruction_by_hand(path):
    for line in instructions(open(path).read()):
        assert re.match(r"s_(nop|waitcnt|barrier)\b", line) or re.match(r"buffer_load_\w+ .*\blds$", line), f"{os.path.basename(path)}: {line}"


def test_the_check_sees_what_it_looks_for():
    assert list(instructions('asm("v_add_u32 %0, %1, %2" : "=v"(a) : "v"(b), "v"(c)); asm volatile("s_nop 0\\n\\ts_barrier" : : : "memory"); asm("" : "+v"(a));')) == [
        "v_add_u32 %0, %1, %2", "s_nop 0", "s_barrier"]
    assert len(SOURCES) > 8


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_shared_memory_read_wide_is_declared_so(path):
    """Shared arrays of bytes, words or floats that are read or written through wider pointers say their alignment; the compiler may place others anywhere."""
    source = open(path).read()
    for name in re.findall(r"__shared__ (?:char|int|float|uint32_t|uint16_t) (\w+)\[", source):
        wide = re.search(r"\((?:const )?(?:f32x4|i32x4|i32x2|uint4|float4) \*\)\s*&?\(?%s\b" % name, source)
        assert not wide, f"{os.path.basename(path)}: {name} is read through a wider pointer"
