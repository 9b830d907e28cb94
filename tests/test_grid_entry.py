"""Pointers that a kernel reads through are handed to the wait for the launches before it, so that no load through them can be
moved ahead of that wait: read from the sources, for what the compiler may do it does not do today."""
import re

import pytest

from test_waits_source import closing, code

FILES = ["step_kernels.cu", "fp4_kernels.cu", "grad_kernels.cu"]


def structs(text):
    return {m.group(1): text[m.end() - 1:closing(text, m.end() - 1)] for m in re.finditer(r"struct (\w+)[^;{]*\{", text)}


def members(body):
    """Names of the pointers among a struct's members."""
    out = []
    for m in re.finditer(r"^\s*(?:const )?(?:\w+)(?:\s*\*[^;(]*);", body, re.M):
        line = m.group(0)
        if "*" in line and "(" not in line:
            out += re.findall(r"\*\s*(?:const\s+)?(\w+)", line)
    return out


def kernels(text):
    for m in re.finditer(r"__global__ void[^;{]*?(\w+_kernel)\(([^{;]*?)(\w+Params) p\)\s*\{", text, re.S):
        begin = m.end() - 1
        yield m.group(1), m.group(3), text[begin:closing(text, begin)]


def test_the_reading_itself():
    text = "struct AParams {\n  const void *x, *y;\n  float* z;\n  int n;\n};\n__global__ void a_kernel(const AParams p) { enter_grid(p.x); use(p.x); }"
    assert members(structs(text)["AParams"]) == ["x", "y", "z"]
    assert [(n, s) for n, s, _ in kernels(text)] == [("a_kernel", "AParams")]


# what a kernel writes alone, and what is read after a wait of its own
WRITTEN = {"step_kernel": {"r", "n", "stats_y", "stats_r"},
           "step_back_kernel": {"r", "n", "dgate", "dwy", "dby", "dwr", "dbr", "partial", "partial_y"},
           "step_columns_kernel": {"dgate", "dwy", "dby", "dwr", "dbr", "joined"},
           "step_join_kernel": {"dgate", "dwy", "dby", "dwr", "dbr"},
           "quantize_kernel": {"codes", "scales", "values"}, "product_kernel": {"status"}, "few_rows_kernel": {"c", "status"},
           "grad_squares_kernel": {"sum"}, "grad_clip_kernel": {"norm"}}


@pytest.mark.parametrize("name", FILES)
def test_what_is_read_goes_through_the_wait(name):
    text = code(name)
    known = structs(text)
    seen = 0
    for kernel, params, body in kernels(text):
        used = body
        for helper in ("Columns",):  # what it reads and writes for the kernel
            if re.search(rf"\b{helper} c\(", body):
                used += known[helper]
        entered = set(re.findall(r"p\.(\w+)", re.search(r"enter_grid\(([^)]*)\)", body).group(1)))
        pointers = {p for p in members(known[params]) if re.search(rf"\bp\.{p}\b", used)}
        assert pointers - entered <= WRITTEN[kernel], f"{kernel}: {sorted(pointers - entered - WRITTEN[kernel])}"
        assert entered <= pointers, kernel
        seen += 1
    assert seen >= 2
