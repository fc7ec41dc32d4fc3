"""What the compiler made of the kernels of the built library, from their disassembly."""
import os
import re
import shutil
import subprocess

import pytest

import paper_2605_05049_amd as moe
from test_kernel_resources import _code_objects

OBJDUMP = shutil.which("llvm-objdump") or "/opt/rocm/llvm/bin/llvm-objdump"


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """name -> instructions (words of each)."""
    if not os.path.exists(OBJDUMP):
        pytest.skip("no llvm-objdump")
    moe.load_library()
    with open(moe.library_path(), "rb") as f:
        objects = list(_code_objects(f.read()))
    folder, found = tmp_path_factory.mktemp("code"), {}
    for i, elf in enumerate(objects):
        path = folder / f"{i}.elf"
        path.write_bytes(elf)
        name = None
        for line in subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", str(path)], check=True, capture_output=True, text=True).stdout.splitlines():
            at = re.match(r"[0-9a-f]+ <(\w+)>:", line)
            if at:
                name = at.group(1)
                found[name] = []
            elif name and line.startswith("\t"):
                found[name].append(line.split("//")[0].split())
    assert len(found) > 20
    return found


def test_matrix_products_stand_under_no_lane_mask(kernels):
    """A matrix instruction ignores the lane mask, its operands' loads do not: a guard is a scalar branch, or the wavefront's lanes are all on."""
    masked_products, seen = {}, 0
    for name, code in kernels.items():
        masked = False
        for op, *operands in code:
            if "saveexec" in op:
                masked = True
            elif operands and operands[0].startswith("exec"):
                masked = False
            elif op.startswith("v_mfma"):
                seen += 1
                if masked:
                    masked_products[name] = masked_products.get(name, 0) + 1
    assert seen > 1000 and not masked_products


def test_router_of_few_tokens_requests_a_batch_at_once(kernels):
    """The loads of all eight steps of a batch stand before the first wait for one."""
    (code,) = [v for k, v in kernels.items() if "few_router_kernel" in k]
    loads = [i for i, words in enumerate(code) if words[0] == "global_load_dwordx4"]
    waits = [i for i, words in enumerate(code) if any("vmcnt" in w for w in words)]
    assert len(loads) == 16 and loads[-1] < waits[0]
