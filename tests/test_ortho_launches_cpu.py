"""What the launches of the orthogonalised updates say of where vector loads may go, compiled for the host alone: the launches are kept in place of
being made, and every row that a kernel would take four elements at a time is looked at."""
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "..", "paper_2004_08771_amd", "csrc")

MAIN = r"""
#include "ortho.hip"
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

using namespace hb;

// launches in place of the runtime's
static std::vector<std::vector<unsigned char>> seen;
static std::vector<const void *> kernels;
extern "C" {
hipError_t hipLaunchKernel(const void *f, dim3, dim3, void **args, size_t, hipStream_t)
{
    const bool list = f == reinterpret_cast<const void *>(sum_kernel);
    const size_t n = list ? sizeof(List) : sizeof(SmallArgs);
    const unsigned char *const p = static_cast<const unsigned char *>(args[0]);
    const bool has = list || f == reinterpret_cast<const void *>(small_sum_kernel);
    if (has) {
        seen.emplace_back(p, p + n);
        kernels.push_back(f);
    }
    return hipSuccess;
}
hipError_t hipExtLaunchKernel(const void *, dim3, dim3, void **, size_t, hipStream_t, hipEvent_t, hipEvent_t, int) { abort(); }
hipError_t hipFuncSetAttribute(const void *, hipFuncAttribute, int) { return hipSuccess; }
hipError_t hipGetDevice(int *d) { *d = 0; return hipSuccess; }
hipError_t hipGetLastError() { return hipSuccess; }
static struct { dim3 grid, block; size_t lds; hipStream_t stream; } conf;
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, hipStream_t stream)
{
    conf = {grid, block, lds, stream};
    return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *lds, hipStream_t *stream)
{
    *grid = conf.grid; *block = conf.block; *lds = conf.lds; *stream = conf.stream;
    return hipSuccess;
}
void **__hipRegisterFatBinary(const void *) { return nullptr; }
void __hipRegisterFunction(void **, const void *, char *, const char *, unsigned, void *, void *, void *, void *, int *) {}
void __hipUnregisterFatBinary(void **) {}
}

// every row of an operand begins at a boundary of four elements
static bool rows_begin(const void *p, long long ld, int rows, size_t size)
{
    for (int r = 0; r < rows; ++r)
        if ((reinterpret_cast<uintptr_t>(p) + (size_t)r * ld * size) % (4 * size)) return false;
    return true;
}

// rows cols g_tensor base_g ldg base_m ldm muon
int main(int argc, char **argv)
{
    if (argc != 9) return 2;
    int v[8];
    for (int i = 0; i < 8; ++i) v[i] = atoi(argv[i + 1]);
    const OrthoShape shape = {v[0], v[1]};
    const int tensor = v[2];
    const size_t size = tensor == TENSOR_BF16 ? 2 : 4;
    OrthoMatrix o = {};
    o.g = reinterpret_cast<const void *>(0x10000 + size * v[3]);
    o.ldg = v[4];
    o.momentum = reinterpret_cast<float *>(0x4000000 + 4 * (size_t)v[5]);
    o.ldm = v[6];
    o.out = reinterpret_cast<void *>(0x8000000);
    o.ldo = v[1];
    OrthoSteps how = {};
    const float coef[3] = {3.4445f, -4.775f, 2.0315f};
    how.g_tensor = tensor;
    how.steps = 5;
    how.n_coef = 1;
    how.coef = coef;
    how.muon = v[7] != 0;
    if (launch_ortho(&o, &shape, 1, how, reinterpret_cast<void *>(0x10000000), nullptr, PassEvents()) != hipSuccess) return 3;
    if (seen.size() != 1) return 4;
    bool whole_g, whole_m;
    if (kernels[0] == reinterpret_cast<const void *>(sum_kernel)) {
        List l;
        memcpy(static_cast<void *>(&l), seen[0].data(), sizeof(l));
        whole_g = l.mat[0].whole_g;
        whole_m = l.mat[0].whole_m;
    } else {
        SmallArgs l;
        memcpy(static_cast<void *>(&l), seen[0].data(), sizeof(l));
        whole_g = l.mat[0].whole_g;
        whole_m = l.mat[0].whole_m;
    }
    printf("%d %d %d %d\n", whole_g, rows_begin(o.g, o.ldg, v[0], size), whole_m, rows_begin(o.momentum, o.ldm, v[0], 4));
    return 0;
}
"""


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    d = tmp_path_factory.mktemp("launches")
    src, obj, exe = str(d / "main.hip"), str(d / "main.o"), str(d / "main")
    with open(src, "w") as f:
        f.write("#include <vector>\n" + MAIN)
    subprocess.check_call(["hipcc", "-std=c++17", "-O1", "--offload-arch=gfx950", "--offload-host-only", "-Wno-unknown-attributes", "-I", CSRC, "-c", src,
                           "-o", obj])
    # (the device code that a host file refers to is not there, and not needed)
    subprocess.check_call(["g++", obj, "-o", exe, "-no-pie", "-pthread", "-Wl,--unresolved-symbols=ignore-all"])

    def ask(*args):
        got = subprocess.run([exe, *map(str, args)], capture_output=True, text=True, check=True).stdout.split()
        return tuple(v == "1" for v in got)
    return ask


@pytest.mark.parametrize("shape", [(100, 1000), (9000, 20), (16, 1025), (1, 3000), (300, 200)])
@pytest.mark.parametrize("tensor", [0, 1])
@pytest.mark.parametrize("muon", [0, 1])
def test_rows_taken_four_at_a_time_begin_at_boundaries(launches, shape, tensor, muon):
    """Matrices whose sums are launches of their own (several blocks of columns, or more than 128 rows and columns): pitches and beginnings of every remainder."""
    rows, cols = shape
    for base in (0, 1, 2, 4):
        for more in (0, 1, 2, 3, 4):
            for base_m, more_m in ((0, more), (0, 3), (0, 4), (3, 4)):
                whole_g, rows_g, whole_m, rows_m = launches(rows, cols, tensor, base, cols + more, base_m, cols + more_m, muon)
                assert whole_g == rows_g, (shape, tensor, base, more)
                assert whole_m == rows_m, (shape, tensor, base_m, more_m)
