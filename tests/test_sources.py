"""What the device sources have to keep to that no compiler tells (CPU)."""
from __future__ import annotations

import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_22648_amd", "csrc")
SOURCES = sorted(glob.glob(os.path.join(CSRC, "*.h*")))


def statements(text):
    """Inline asm statements, whole."""
    return re.findall(r"\basm\b[^;]*?\((?:[^;\"]|\"(?:[^\"\\]|\\.)*\")*\)\s*;", text)


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_loads_to_lds_are_given_their_register(path):
    """A load to LDS takes its place from m0. The compiler reserves that register and takes no note of asm that writes it,
    so that it might keep a value of its own there: the asm asks for it as an operand instead."""
    with open(path) as f:
        asm = statements(f.read())
    for s in asm:
        assert not re.search(r"s_\w+ m0\b", s), s
        if "_load_lds_" in s:
            assert '"{m0}"(' in s and "s_nop 0" in s, s


def test_the_statements_are_found():
    with open(os.path.join(CSRC, "lds_fetch.hpp")) as f:
        assert sum("_load_lds_" in s for s in statements(f.read())) == 5


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_wave_barriers_order_memory(path):
    """A wave barrier alone orders no memory: what lanes exchange through LDS stands between fences of the wave."""
    with open(path) as f:
        text = f.read()
    for m in re.finditer(r"__builtin_amdgcn_wave_barrier\(\);", text):
        assert re.search(r"__builtin_amdgcn_fence\(__ATOMIC_RELEASE, \"\w+\"\);\s*$", text[:m.start()])
        assert re.match(r"\s*__builtin_amdgcn_fence\(__ATOMIC_ACQUIRE, \"\w+\"\);", text[m.end():])


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_arrays_read_in_sixteen_bytes_are_aligned(path):
    """A shared array of single numbers that is read four at a time is declared with the alignment of four."""
    with open(path) as f:
        text = f.read()
    for name in set(re.findall(r"\(const v4[fu]\*\)&(s_\w+)", text)):
        found = re.findall(r"__shared__ ([^;]*\b%s\[[^;]*);" % name, text)
        assert found and all("aligned(16)" in x for x in found), (name, found)
