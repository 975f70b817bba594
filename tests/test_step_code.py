"""What the compiler made of the kernels over lists of tensors.  Runs without a GPU."""
import os
import re
import subprocess

from tests.test_kernel_code import LLVM, code_objects  # noqa: F401  (fixture)


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
