"""Products of 8-bit floats on one device after another, with the HIP runtime's
part played by the test's own program (no GPU needed): a kernel's limit of
dynamic LDS is a device's own, and is set where it is launched."""
import os
import subprocess

from paper_2407_18352_amd import _abi

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")

# The program's definitions take the place of the runtime's for the library too.
PROGRAM = r"""
#include <hip/hip_runtime_api.h>

#include <cstdio>
#include <map>
#include <utility>

#include "hpacmlt.h"

static int device, launches, refused;
static std::map<std::pair<int, const void *>, int> limits;
static struct {
    dim3 grid, block;
    size_t lds;
    hipStream_t stream;
} next;

extern "C" {
hipError_t hipGetDevice(int *d) {
    *d = device;
    return hipSuccess;
}
hipError_t hipGetLastError() { return hipSuccess; }
hipError_t hipPointerGetAttributes(hipPointerAttribute_t *a, const void *) {
    a->type = hipMemoryTypeDevice;
    a->device = device;
    return hipSuccess;
}
hipError_t hipMemGetAddressRange(hipDeviceptr_t *base, size_t *size, hipDeviceptr_t p) {
    *base = p;
    *size = (size_t)1 << 40;
    return hipSuccess;
}
hipError_t hipFuncSetAttribute(const void *f, hipFuncAttribute what, int value) {
    if (what == hipFuncAttributeMaxDynamicSharedMemorySize)
        limits[{device, f}] = value;
    return hipSuccess;
}
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t lds, hipStream_t stream) {
    next = {grid, block, lds, stream};
    return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3 *grid, dim3 *block, size_t *lds, hipStream_t *stream) {
    *grid = next.grid;
    *block = next.block;
    *lds = next.lds;
    *stream = next.stream;
    return hipSuccess;
}
hipError_t hipLaunchKernel(const void *f, dim3, dim3, void **, size_t lds, hipStream_t) {
    ++launches;
    if (lds > 64 * 1024) {
        auto at = limits.find({device, f});
        refused += at == limits.end() || (size_t)at->second < lds;
    }
    return hipSuccess;
}
}

int main() {
    // tiles of 128 x 128, and of 256 x 256
    for (device = 0; device < 3; ++device)
        for (int64_t n : {500, 5000})
            for (int32_t type : {HPACML_F32, HPACML_BF16}) {
                const int64_t k = 1024;
                const hpacmlt_matrix p = {(void *)(1ull << 44), (void *)(2ull << 44), n, k}, q = {(void *)(3ull << 44), (void *)(4ull << 44), n, k};
                if (hpacmlt_product(&p, &q, nullptr, HPACML_ACT_IDENTITY, (void *)(5ull << 44), type, n, 0, (void *)(6ull << 44), (size_t)1 << 40,
                                    nullptr) != HPACML_OK)
                    return 1;
            }
    std::printf("%d %d %d\n", launches >= 12, (int)(limits.size() >= 4), refused);
    return 0;
}
"""


def test_limits_of_lds_on_every_device(tmp_path):
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(PROGRAM)
    lib = os.path.dirname(_abi.LIB_PATH)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wno-unused-result", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROCM, "include"),
                    "-I", os.path.join(ROOT, "include"), str(src), "-rdynamic", "-L", lib, "-lhpacml", "-L", os.path.join(ROCM, "lib"), "-lamdhip64",
                    "-Wl,-rpath," + lib + ":" + os.path.join(ROCM, "lib"), "-o", str(exe)], check=True, capture_output=True, text=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, check=True, timeout=120).stdout.split()
    assert out == ["1", "1", "0"]
