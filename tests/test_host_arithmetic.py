"""The host side of the layer for a few tokens, built for the CPU alone with checks of its floating-point arithmetic that trap."""
import os
import shutil
import subprocess

import pytest

import paper_2605_05049_amd as moe
from paper_2605_05049_amd import build

STUBS = r"""
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include "moe.h"
// what the launches refer to: nothing is launched here
namespace moe { void prof_begin(const char*, struct ihipStream_t*) {} void prof_end(struct ihipStream_t*) {} }
extern "C" {
int __hipPopCallConfiguration(void*, void*, void*, void*) { abort(); }
int __hipPushCallConfiguration(uint64_t, uint32_t, uint64_t, uint32_t, size_t, void*) { abort(); }
void** __hipRegisterFatBinary(const void*) { static void* handle; return &handle; }
void __hipRegisterFunction() {}
void __hipUnregisterFatBinary(void**) {}
int hipGetLastError() { return 0; }
int hipLaunchKernel() { abort(); }
}
int main() {
  moe_shape s = {0, 0, 0, 0, 0, 0, 1};
  while (scanf("%d %d %d %d %d %d", &s.T, &s.d_model, &s.d_ffn, &s.E, &s.k, &s.E_shared) == 6) {
    printf("%zu\n", moe_layer_few_workspace_bytes(&s));
    fflush(stdout);
  }
}
"""


def test_plans_of_few_tokens(tmp_path):
    """No division by zero and no conversion out of range, for calls without tokens too; and the library's own answers."""
    if not shutil.which(build.HIPCC):
        pytest.skip("no hipcc")
    checks = []
    for c in ("float-divide-by-zero", "float-cast-overflow", "signed-integer-overflow", "integer-divide-by-zero"):
        checks += ["-Xarch_host", f"-fsanitize={c}", "-Xarch_host", f"-fsanitize-trap={c}"]
    (tmp_path / "stubs.cpp").write_text(STUBS)
    include = os.path.join(os.path.dirname(build.PKG_DIR), "include")
    run = lambda *a: subprocess.run(a, check=True, capture_output=True, text=True)  # noqa: E731
    run(build.HIPCC, *build.FLAGS, "--cuda-host-only", *checks, "-c", os.path.join(build.CSRC, "few_tokens.hip"), "-o", str(tmp_path / "few.o"))
    run("g++", "-c", "-I", include, str(tmp_path / "stubs.cpp"), "-o", str(tmp_path / "stubs.o"))
    run("g++", str(tmp_path / "few.o"), str(tmp_path / "stubs.o"), "-Wl,--unresolved-symbols=ignore-all", "-o", str(tmp_path / "plans"))
    shapes = [(T, d, f, E, k, Es) for T in (0, 1, 16, 17, 64) for d, f in ((64, 64), (512, 1024), (4096, 14336), (2 ** 22, 64), (64, 2 ** 22))
              for E, k, Es in ((1, 1, 0), (1, 1, 1023), (8, 2, 0), (64, 6, 2), (1000, 60, 3), (1024, 64, 0))]
    lines = "\n".join(" ".join(map(str, s)) for s in shapes)
    done = subprocess.run([str(tmp_path / "plans")], input=lines, capture_output=True, text=True)
    got = [int(v) for v in done.stdout.split()]
    assert done.returncode == 0, f"trapped at {shapes[len(got)]}"
    assert got == [moe.layer_few_workspace_bytes(moe.Shape(*s)) for s in shapes]
