"""Inline assembly of the kernels (no GPU needed): a register that a statement writes
by name is among its clobbers, or the compiler may keep a value of its own there."""
import glob
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STATEMENT = re.compile(r'\basm(?: volatile)?\(("(?:[^"\\]|\\.)*")(.*?)\);', re.DOTALL)
WRITTEN = re.compile(r'(?:"|\\n|\\t)[sv]_\w+ (m0|vcc|exec|[sv]\d+|[sv]\[\d+:\d+\]),')


def unnamed(text):
    """(instructions, register) of those written and not among the clobbers."""
    return [(code, name) for code, rest in STATEMENT.findall(text) for name in WRITTEN.findall(code)
            if f'"{name}"' not in rest.rpartition(":")[2]]


def test_what_the_search_finds():
    assert unnamed('asm("" : "+v"(x)); asm volatile("s_nop 1\\n\\ts_mov_b32 m0, %0" ::"s"(f(a)) : "memory", "m0");') == []
    assert [n for _, n in unnamed('asm volatile("s_nop 1\\n\\ts_mov_b32 m0, %0" ::"s"(f(a)), "v"(b)\n  : "memory");')] == ["m0"]
    assert [n for _, n in unnamed('asm volatile("v_mov_b32 v3, %0" ::"v"(m0));')] == ["v3"]


def test_registers_written_by_name_are_clobbers():
    files = sorted(glob.glob(os.path.join(ROOT, "paper_2606_08761_amd", "**", "*.h*"), recursive=True))
    texts = {f: open(f).read() for f in files}
    assert sum(len(STATEMENT.findall(t)) for t in texts.values()) >= 3
    assert {os.path.basename(f): unnamed(t) for f, t in texts.items() if unnamed(t)} == {}
