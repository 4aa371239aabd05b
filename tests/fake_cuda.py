"""A source of the library built against a CUDA runtime that launches nothing, for tests of what a call does on the host: it
writes down the launches and the tensor maps in their order and lets one of them fail."""
import ctypes
import os
import subprocess

from paper_2110_04175_gb300 import build as rs_build

RUNTIME = r"""
#include <cuda.h>
#include <cuda_runtime.h>

static int g_launches, g_maps, g_bad_launch, g_bad_map;
static char g_log[256];
static int g_at;
static cudaError_t g_last;

static void note(char c) {
    if (g_at < 255) g_log[g_at++] = c;
    g_log[g_at] = 0;
}
static cudaError_t launch() {
    note('L');
    if (g_launches++ == g_bad_launch) return g_last = cudaErrorLaunchOutOfResources;
    return cudaSuccess;
}
static CUresult encode(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                       const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill) {
    note('M');
    return g_maps++ == g_bad_map ? CUDA_ERROR_INVALID_VALUE : CUDA_SUCCESS;
}

extern "C" {
// Number `bad_launch` and number `bad_map` fail (-1: none).
void fake_start(int bad_launch, int bad_map) {
    g_launches = g_maps = g_at = 0, g_log[0] = 0, g_last = cudaSuccess;
    g_bad_launch = bad_launch, g_bad_map = bad_map;
}
const char* fake_log() { return g_log; }

void** __cudaRegisterFatBinary(void*) {
    static void* one;
    return &one;
}
void __cudaRegisterFatBinaryEnd(void**) {}
void __cudaUnregisterFatBinary(void**) {}
void __cudaRegisterFunction(void**, const char*, char*, const char*, int, uint3*, uint3*, dim3*, dim3*, int*) {}
unsigned __cudaPushCallConfiguration(dim3, dim3, size_t, CUstream_st*) { return 0; }
cudaError_t __cudaPopCallConfiguration(dim3* grid, dim3* block, size_t* shared, void* stream) {
    *grid = *block = dim3(1), *shared = 0, *static_cast<void**>(stream) = nullptr;
    return cudaSuccess;
}
cudaError_t __cudaGetKernel(cudaKernel_t* to, const void* f) {
    *to = reinterpret_cast<cudaKernel_t>(const_cast<void*>(f));
    return cudaSuccess;
}
cudaError_t __cudaLaunchKernel(cudaKernel_t, dim3, dim3, void**, size_t, cudaStream_t) { return launch(); }
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t*, const void*, void**) { return launch(); }
cudaError_t cudaGetLastError() {
    const cudaError_t e = g_last;
    g_last = cudaSuccess;
    return e;
}
cudaError_t cudaGetDevice(int* device) {
    *device = 0;
    return cudaSuccess;
}
cudaError_t cudaDeviceGetAttribute(int* value, cudaDeviceAttr, int) {
    *value = 152;
    return cudaSuccess;
}
cudaError_t cudaFuncSetAttribute(const void*, cudaFuncAttribute, int) { return cudaSuccess; }
cudaError_t cudaGetDriverEntryPointByVersion(const char*, void** f, unsigned, unsigned long long, cudaDriverEntryPointQueryResult* found) {
    *f = reinterpret_cast<void*>(encode);
    if (found) *found = cudaDriverEntryPointSuccess;
    return cudaSuccess;
}
}
"""


def library(folder, source, flags=()):
    """The source's calls on the runtime above (its kernels are compiled, but not for a machine)."""
    nvcc, folder = rs_build.nvcc(), str(folder)
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc))), "include")
    runtime, obj, out = (os.path.join(folder, name) for name in ("runtime.cpp", "source.o", "fake.so"))
    with open(runtime, "w") as f:
        f.write(RUNTIME)
    subprocess.run([nvcc, "-gencode", "arch=compute_103a,code=compute_103a", "-O1", "-std=c++17", "-Xcompiler", "-fPIC",
                    "-I" + rs_build.INCLUDE, "-I" + rs_build.CSRC, *flags, "-c", os.path.join(rs_build.CSRC, source), "-o", obj],
                   check=True)
    # (the symbols of another CUDA runtime in the process must not be taken for these)
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-I" + cuda, runtime, obj, "-Wl,-Bsymbolic", "-o", out], check=True)
    lib = ctypes.CDLL(out)
    lib.fake_log.restype = ctypes.c_char_p
    return lib
