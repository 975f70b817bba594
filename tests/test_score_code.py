"""What the compiler made of the attention kernels of shaped scores: a register kept in scratch memory inside a loop waits for the tiles in flight, and
a few registers too many halve the wavefronts of a compute unit.  Runs without a GPU."""
import os
import re
import subprocess

from tests.test_kernel_code import LLVM, code_objects, resources  # noqa: F401  (fixtures)


def test_registers_of_the_shaped_score_kernels(resources):  # noqa: F811
    found = {re.sub(r".*?score_(\w+?)_kernelI(.*?)EEEvNS.*", r"\1 \2", n): r for n, r in resources.items() if re.search(r"score_(fwd|dq|dkv|bwd)_kernelI", n)}
    assert len(found) == 14 + 12 + 12 + 8, sorted(found)
    for n, r in found.items():
        # dQ keeps a register or two in scratch across its loop, not in it, capped in the one launch with dK and dV three; the small forward of capped
        # scores keeps two to have four wavefronts to a SIMD
        allowed = 3 if n.startswith("bwd Li128ELi2ELi1ELb1") else 2 if n.startswith("dq Li128") else 2 if n == "fwd Li64ELi512ELi4ELb1" else 0
        assert r["vgpr_spill_count"] <= allowed, (n, r)
    for n in ("fwd Li64ELi256ELi2ELb0", "fwd Li64ELi512ELi4ELb0", "dkv Li64ELi64ELi2ELb0"):
        assert found[n]["vgpr_count"] <= 128, (n, found[n])


def test_nothing_of_attention_is_in_double_precision(code_objects):  # noqa: F811
    """An integer minimum or maximum of two types goes through double precision, where unsigned minus one is four thousand million."""
    kernels, double = 0, []
    for path in code_objects:
        text = subprocess.run([os.path.join(LLVM, "llvm-objdump"), "-d", "--no-show-raw-insn", str(path)], capture_output=True, text=True, check=True).stdout
        for part in re.split(r"^[0-9a-f]+ <(?=\S+>:$)", text, flags=re.M)[1:]:
            name, _, code = part.partition(">:")
            if re.search(r"score(32)?_\w+kernel", name):
                kernels += 1
                double += [(name, line.split("//")[0].strip()) for line in code.splitlines() if "_f64" in line]
    assert kernels >= 14 + 12 + 12 + 8 + 4, kernels
    assert not double, double[:5]
