"""What the kernels' waits rest on and no run on a GPU can show, for there a wait would have to run out: read from the
sources.  A wait in a kernel has a limit, after which a flag is raised; from then on every warp has to come out."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_32197_b200", "csrc")
FILES = sorted(f for f in os.listdir(CSRC) if f.endswith(".cu"))


def code(name):
    """The file without its comments."""
    with open(os.path.join(CSRC, name)) as f:
        text = f.read()
    return re.sub(r"//[^\n]*|/\*.*?\*/", "", text, flags=re.S)


def closing(text, at):
    """Index behind the brace that closes the one at `at`."""
    depth = 0
    for i in range(at, len(text)):
        depth += (text[i] == "{") - (text[i] == "}")
        if depth == 0:
            return i + 1
    raise ValueError("unbalanced braces")


def loops(text):
    """(header, body) of every loop with braces."""
    for m in re.finditer(r"\b(for|while)\s*\(", text):
        at, depth = m.end(), 1
        while depth:
            depth += (text[at] == "(") - (text[at] == ")")
            at += 1
        rest = text[at:]
        if rest.lstrip().startswith("{"):
            begin = at + rest.index("{")
            yield text[m.start():at], text[begin:closing(text, begin)]


def without_inner_loops(body):
    out, at = body[:1], 1
    for header, inner in loops(body[1:]):
        begin = body.find(header + body[body.find(header, at) + len(header):body.find(inner, at)] + inner, at)
        if begin < at:
            continue  # inside a loop that is out already
        out += body[at:begin]
        at = body.find(inner, begin) + len(inner)
    return out + body[at:]


def test_the_reading_itself():
    text = "for (int i = 0; i < f(n); ++i) { a; while (x) { break; } if (y) { b; } }"
    (head, body), (_, inner) = loops(text)
    assert head == "for (int i = 0; i < f(n); ++i)" and inner == "{ break; }"
    assert without_inner_loops(body).split() == "{ a; if (y) { b; } }".split()


@pytest.mark.parametrize("name", FILES)
def test_warps_that_meet_at_a_barrier_all_come(name):
    """A loop in which some of a CTA's warps meet at a named barrier is left at its end alone: a warp that leaves as soon
    as it sees the flag would make those wait for good that looked a moment earlier."""
    for header, body in loops(code(name)):
        own = without_inner_loops(body)
        if re.search(r"bar(rier)?\.sync\s+[1-9%]", own):
            assert not re.search(r"\b(break|return|goto|continue)\b", own), f"{name}: {header}"


def test_results_of_the_products_leave_together():
    """The flag is read once for a warp: its lanes go on to instructions that take all of them."""
    text = code("ffn_kernels.cu")
    at = text.index("while (walk.next()) {")
    results = text[at:closing(text, text.index("{", at))]
    assert "tmem_ld32" in results
    for line in results.splitlines():
        if "*s_abort" in line and "mbar_wait" not in line:
            assert "__any_sync(0xffffffffu, *s_abort" in line, line


def test_no_product_outlives_its_memory():
    """After a wait that ran out nothing more is multiplied, and what was issued is waited for before tensor memory is
    given back and the CTA, with its shared memory, ends."""
    text = code("ffn_kernels.cu")
    waits = re.findall(r"([^;{}]*)mbar_wait_bounded_inline\(full \+ s[^;]*;", text)
    assert len(waits) == 2 and all(w.strip() == "if (!" for w in waits)
    assert len(re.findall(r"mbar_wait_bounded_inline\(full \+ s[^;{}]*\)\) break;", text)) == 2
    for kernel, dealloc in (("void gemm_tiles", "tmem_dealloc_pair"), ("few_kernel(", "tmem_dealloc(")):
        at = text.index(kernel)
        body = text[at:text.index(dealloc, at)]
        assert 0 < body.rindex("mma_commit") < body.index("wait_drained(")


@pytest.mark.parametrize("name", FILES)
def test_tensor_memory_is_taken_before_the_next_launch_may_begin(name):
    """Else a CTA of the next launch could have the columns that this one waits for, and wait for this one's end."""
    text = code(name)
    for m in re.finditer(r"\btmem_alloc(_pair)?\(", text):
        kernel = max(text.rfind("__global__", 0, m.start()), text.rfind("__device__", 0, m.start()))
        begin = text.index("{", kernel)
        body, at = text[begin:closing(text, begin)], m.start() - begin
        first = re.search(r"launch_dependents|enter_grid\(", body)
        assert first is not None and at < first.start(), f"{name}: {text[kernel:begin]}"
