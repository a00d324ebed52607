"""Kernels that let their successor start early (griddepcontrol) must themselves wait before they touch memory: only a
kernel that waits is promised to see what was written before it.  Read from the sources: a race cannot be provoked."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1705_09056_b200", "csrc")


def kernels(text):
    """(name, body) of every __global__ function defined in a source without comments."""
    text = re.sub(r"__launch_bounds__\s*\([^()]*\)", "", text)
    for m in re.finditer(r"__global__[^;{]*?(\w+)\s*\(([^;{]*)\)\s*\{", text):
        depth, i = 1, m.end()
        while depth:
            depth += {"{": 1, "}": -1}.get(text[i], 0)
            i += 1
        yield m.group(1), text[m.end():i - 1]


def sources():
    for f in sorted(os.listdir(CSRC)):
        with open(os.path.join(CSRC, f)) as h:
            yield f, re.sub(r"//[^\n]*|^\s*#[^\n]*", "", re.sub(r"/\*.*?\*/", "", h.read(), flags=re.S), flags=re.M)


def top_level(body):
    """The statements of a function body that are not inside braces, one per element."""
    out, depth, cur = [], 0, ""
    for ch in body:
        if ch == "}":
            depth -= 1
            if depth == 0:
                cur = ""
            continue
        if ch == "{":
            depth += 1
            continue
        if depth == 0:
            cur += ch
            if ch == ";":
                out.append(cur.strip())
                cur = ""
    return out


def test_the_reader_of_sources():
    text = "template <int A>\n__global__ void __launch_bounds__(32)\nf(int a) { x(); if (a) { y(); } if (a) z(); w(); }"
    (name, body), = kernels(text)
    assert name == "f" and top_level(body) == ["x();", "if (a) z();", "w();"]


def test_chained_kernels_wait_before_their_work():
    found = set()
    for f, text in sources():
        for name, body in kernels(text):
            if "chain_next()" not in body:
                continue
            found.add(name)
            steps = top_level(body)
            if "chain_wait();" in steps:
                before = " ".join(steps[:steps.index("chain_wait();")])
                assert not re.search(r"__ld|\breturn\b", before), (f, name)
            else:                                     # an ordinary launch: it starts after everything before it is complete
                assert "chain_wait" not in body, (f, name)
                assert re.search(r"kernel\s*<<<", text) and name == "fp8_weights_kernel", (f, name)
    assert {"fp8_gemm_kernel", "ckpt8_save_kernel", "ckpt8_load_kernel", "delta_kernel", "delta_sum_kernel",
            "gather8_kernel", "fp8_weights_kernel"} <= found
