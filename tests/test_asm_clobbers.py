"""Assembly in the kernels names the special registers that it writes, or leaves them as they were."""
import glob
import os
import re

import pytest

from tests.conftest import ROOT

SOURCES = sorted(glob.glob(os.path.join(ROOT, "paper_2609_34045_amd", "csrc", "*.h*")))
WRITES = {"m0": r"\bs_\w+ m0\b", "vcc": r"\bv_cmp\w* vcc\b|\bs_\w+ vcc\b", "exec": r"\bs_\w+ exec\b|\bv_cmpx",
          "scc": r"\bs_(add|sub|addc|subb|and|or|xor|not|lshl|lshr|ashr|min|max|cmp|bfe|abs|bcnt)\w* "}


def statements(text):
    """Each asm statement with its operands, its instructions apart by blanks."""
    for m in re.finditer(r"\basm\s*(volatile)?\s*\(", text):
        depth, at, quoted = 1, m.end(), False
        while depth:
            c = text[at]
            if c == '"' and text[at - 1] != "\\":
                quoted = not quoted
            depth += 0 if quoted else (c == "(") - (c == ")")
            at += 1
        yield re.sub(r"\\[nt]", " ", text[m.end():at - 1])


def unnamed(s):
    """What a statement writes without telling.  m0, which no list can name, has to be saved first and restored last."""
    written = [r for r, w in WRITES.items() if re.search(w, s) and f'"{r}"' not in s]
    code = " ".join(re.findall(r'"([^"]*)"', s.split(":")[0]))
    if re.match(r"\s*s_mov_b32 (%\d+), m0 .* s_mov_b32 m0, \1\s*$", code):
        written.remove("m0")
    return written


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_written_registers_are_named_or_restored(path):
    with open(path) as f:
        for s in statements(f.read()):
            assert not unnamed(s), s


@pytest.mark.parametrize("code,want", [
    ('asm volatile("s_mov_b32 m0, %0\\n\\ts_add_u32 m0, m0, 4" ::"s"(a[0]) : "memory", "scc");', ["m0"]),
    ('asm volatile("s_mov_b32 %0, m0\\n\\ts_mov_b32 m0, %1\\n\\ts_add_u32 m0, m0, 4\\n\\t" "s_mov_b32 m0, %0" : "=&s"(b) : "s"(a));', ["scc"]),
    ('asm("v_cmp_lt_f32 vcc, %0, %1" ::"v"(a), "v"(b) : "vcc");', [])])
def test_a_register_that_is_not_named_is_found(code, want):
    s, = statements(code)
    assert unnamed(s) == want
