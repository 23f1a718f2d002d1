"""What the 8-bit product does on the host before its kernels: the driver's entry point is looked up again after a look-up in
vain, and a call that could not be made leaves no error behind for the next one.  (No GPU is used: the library's objects in a
program that answers for the runtime, and whose driver describes nothing.)"""
import os
import subprocess

from paper_2111_00705_b200 import binding as cd
from paper_2111_00705_b200 import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdio>
#include <cstring>
#include <cuda_runtime.h>
#include "cdadam.h"

static int looked, described;
static cudaError_t pending = cudaSuccess;

static int refuse(void *, int, unsigned, void *, const void *, const void *, const void *, const void *, int, int, int, int)
{
    ++described;
    return 1;
}

extern "C" cudaError_t __wrap_cudaGetDriverEntryPointByVersion(const char *, void **fn, unsigned, unsigned long long,
                                                               cudaDriverEntryPointQueryResult *result)
{
    if (++looked < 3) return pending = cudaErrorSystemNotReady;
    *fn = (void *)refuse;
    *result = cudaDriverEntryPointSuccess;
    return cudaSuccess;
}
extern "C" cudaError_t __wrap_cudaGetLastError()
{
    const cudaError_t e = pending;
    pending = cudaSuccess;
    return e;
}

int main()
{
    int8_t *const p = (int8_t *)4096;               // nobody follows it
    for (int i = 0; i < 5; ++i) {
        const int code = cdadam_matmul8(p, 48, (float *)p, p + 4096, 48, (float *)p, nullptr, 4, 6, 40, CDADAM_BF16, CDADAM_F32, p + 8192, 6, nullptr);
        const bool why = strstr(cdadam_last_error(), cudaGetErrorString(cudaErrorSystemNotReady)) != nullptr;
        printf("%d %d %d %d %d\n", code, (int)pending, looked, described, (int)why);
    }
}
"""


def test_a_look_up_in_vain(tmp_path):
    if not os.path.exists(os.path.join(build.OBJ, "matmul8.o")):
        build.build(force=True)
    source, program = tmp_path / "product.cpp", tmp_path / "product"
    source.write_text(PROGRAM)
    cuda = os.path.dirname(os.path.dirname(build._nvcc()))
    subprocess.check_call(["g++", "-std=c++17", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(cuda, "include"), str(source)] +
                          [os.path.join(build.OBJ, s.replace(".cu", ".o")) for s in build.SOURCES] +
                          ["-Wl,--wrap=cudaGetDriverEntryPointByVersion", "-Wl,--wrap=cudaGetLastError", "-L", os.path.join(cuda, "lib64"),
                           "-lcudart_static", "-ldl", "-lrt", "-lpthread", "-o", str(program)])
    out = subprocess.check_output([str(program)], env=dict(os.environ, CUDA_VISIBLE_DEVICES=""), text=True)
    got = [tuple(int(v) for v in line.split()) for line in out.strip().split("\n")]
    # (code, error left behind, look-ups so far, descriptions asked of the driver so far, the message says why)
    e = cd.ERR_CUDA
    assert got == [(e, 0, 1, 0, 1), (e, 0, 2, 0, 1), (e, 0, 3, 1, 0), (e, 0, 3, 2, 0), (e, 0, 3, 3, 0)]
