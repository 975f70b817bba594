"""What the compiler made of the kernels that bring the next row to LDS while they work on this one.  Runs without a GPU."""
import os
import re
import subprocess

from tests.test_kernel_code import LLVM, code_objects  # noqa: F401  (fixture)


def functions(path, pattern):
    """(name, [(instruction, places it may go on to)]) of the code object's functions that match"""
    text = subprocess.run([os.path.join(LLVM, "llvm-objdump"), "-d", "--no-show-raw-insn", str(path)], capture_output=True, text=True, check=True).stdout
    for func in re.split(r"\n(?=[0-9a-f]{16} <)", text):
        name = re.search(r"<(\S+)>:", func)
        if not name or not re.search(pattern, name[1]):
            continue
        code = [(int(a, 16), i.strip()) for i, a in re.findall(r"^\s+(.+?)\s*// ([0-9A-F]+):", func, re.M)]
        at, out = {a: n for n, (a, _) in enumerate(code)}, []
        for n, (a, ins) in enumerate(code):
            jump = re.match(r"s_(cbranch_\w+|branch) (\d+)", ins)
            go = [] if ins.startswith(("s_endpgm", "s_branch")) else [n + 1]
            if jump:
                words = int(jump[2])
                go.append(at[a + 4 + 4 * (words - (1 << 16) if words >= 1 << 15 else words)])
            out.append((ins, [g for g in go if g < len(code)]))
        yield name[1], out


def reaches(code, start, until, stop):
    """Whether a path from behind `start` comes to an instruction that `until` takes without one that `stop` takes"""
    seen, todo = set(), list(code[start][1])
    while todo:
        n = todo.pop()
        if n in seen or stop(code[n][0]):
            continue
        seen.add(n)
        if until(code[n][0]):
            return True
        todo += code[n][1]
    return False


def test_the_next_row_has_landed_before_it_is_read(code_objects):  # noqa: F811
    """The compiler does not count loads to LDS that are written in assembly.  Between one of them and any read of 16 bytes from LDS lies a wait for all loads, on every path; and between a read and
    the loads that overwrite what it reads, a wait for reads."""
    load = lambda i: i.startswith("buffer_load") and i.endswith("lds")
    read = lambda i: i.startswith("ds_read_b128")
    landed = lambda i: bool(re.match(r"s_waitcnt.*vmcnt\(0\)", i))
    arrived = lambda i: bool(re.match(r"s_waitcnt.*lgkmcnt\(0\)", i))
    kernels = 0
    for path in code_objects:
        for name, code in functions(path, r"logprob_both_kernel"):
            loads, reads = ([n for n, (i, _) in enumerate(code) if f(i)] for f in (load, read))
            ahead = int(re.search(r"Li\d+ELi\d+ELi(\d+)E", name)[1])
            assert len(loads) == ahead and len(reads) == 2 * ahead, (name, len(loads), len(reads))      # the two ways to store
            if not ahead:
                continue
            kernels += 1
            assert any(reaches(code, n, read, lambda i: False) for n in loads) and any(reaches(code, n, load, lambda i: False) for n in reads)
            for n in loads:
                assert not reaches(code, n, read, landed), (name, n)
            for n in reads:
                assert not reaches(code, n, load, arrived), (name, n)
    assert kernels == 2 * 5 * 4
