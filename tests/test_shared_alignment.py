"""Shared memory that kernels read or write as wider types than it is declared with says so in its declaration: an array of words alone is 4-byte aligned."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2512_21571_b200", "csrc")


def test_arrays_that_are_read_as_wider_types_are_aligned():
    for name in sorted(os.listdir(CSRC)):
        if not name.endswith((".cu", ".cuh")):
            continue
        text = open(os.path.join(CSRC, name)).read()
        narrow = re.findall(r"__shared__ (?:uint32_t|float|int|uint16_t|uint8_t|char) ([^;]*);", text)
        for array in {a for of in narrow for a in re.findall(r"(\w+)\[", of)}:
            wide = re.search(r"reinterpret_cast<(?:const |volatile )*(?:u?int[24]|float[24]|ulonglong2) \*>\(\s*&?" + array + r"\b", text)
            assert not wide, (name, array)
