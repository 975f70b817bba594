"""What the compiler made of the kernels around a training step.  Runs without a GPU."""
import os
import re
import subprocess

from tests.test_kernel_code import LLVM, code_objects, resources  # noqa: F401  (fixtures)


def test_scalar_loads_at_a_register_start_at_the_arguments(code_objects):  # noqa: F811
    """A scalar load drops the low two bits of its base and of its offset before it adds them.  The compiler may split a tensor's place in the list into a base and an offset
    that are no multiples of four by themselves; these kernels' entries are laid out so that it has no reason to, and the base is the arguments' own address."""
    kernels, loads = 0, 0
    for path in code_objects:
        text = subprocess.run([os.path.join(LLVM, "llvm-objdump"), "-d", "--no-show-raw-insn", str(path)], capture_output=True, text=True, check=True).stdout
        for part in re.split(r"^[0-9a-f]+ <(?=\S+>:$)", text, flags=re.M)[1:]:
            name, _, code = part.partition(">:")
            if not re.search(r"(sumsq|clip|adamw)_kernel", name):
                continue
            kernels += 1
            for base in re.findall(r"s_load_dword\w* s\S+, s\[(\d+:\d+)\], s\d+", code):
                loads += 1
                assert base == "0:1", (name, base)
    assert kernels == 2 * (2 + 2 + 4) and loads >= kernels


def test_registers_of_the_log_probability_kernels(resources):  # noqa: F811
    """Eight wavefronts of the walk fit a SIMD; a row in registers is not kept in scratch memory, and its workgroups fit a compute unit as often as they are launched."""
    walk = {n: r for n, r in resources.items() if re.search(r"logprob_kernelI", n)}
    both = {n: r for n, r in resources.items() if re.search(r"logprob_both_kernelI", n)}
    assert len(walk) == 2 * 3 * 8 and len(both) == 2 * (8 * 4 + 2)
    for n, r in walk.items():
        assert r["vgpr_count"] <= 64 and r["vgpr_spill_count"] <= 2, (n, r)
    for n, r in both.items():
        nv = int(re.search(r"Li\d+ELi(\d+)ELi\d+E", n)[1])
        waves = {1: 8, 4: 8, 8: 6, 16: 4}[nv]                            # to a SIMD
        assert r["vgpr_spill_count"] == 0 and waves * ((r["vgpr_count"] + 7) // 8 * 8) <= 512, (n, r)
