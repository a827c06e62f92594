"""The 8-bit head's entry points in a process that uses several devices, on a
stand-in for the CUDA runtime (no GPU): what holds for one device only (a
kernel's shared-memory limit, the clusters that fit) is set up and asked for on
each, and a call that failed there is tried again."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

from paper_2608_02438_gb300 import binding as X
from paper_2608_02438_gb300 import build as BLD

FAKE = r"""
// The runtime calls of matmul_fp8.cu, matmul_fp8_wide.cu and logits.cu, for 70 devices
// that keep a kernel's attributes each for itself and launch nothing.
#include <cuda.h>
#include <cuda_runtime_api.h>
#include <cstdint>
#include <map>
#include <set>
#include <utility>

static int device, launches, cluster_queries, fail_attributes, clusters_of[70];
static std::map<std::pair<int, const void *>, int> limits;

extern "C" {
void fake_use(int dev) { device = dev; }
int fake_launches() { return launches; }
int fake_cluster_queries() { return cluster_queries; }
void fake_fail_attributes(int n) { fail_attributes = n; }
void fake_clusters(int dev, int n) { clusters_of[dev] = n; }
static unsigned last_cluster;
unsigned fake_last_cluster() { return last_cluster; }

cudaError_t cudaGetDevice(int *dev) { *dev = device; return cudaSuccess; }
cudaError_t cudaGetLastError() { return cudaSuccess; }
cudaError_t cudaFuncSetAttribute(const void *f, cudaFuncAttribute, int value)
{
    if (fail_attributes > 0) { --fail_attributes; return cudaErrorInvalidValue; }
    limits[{device, f}] = value;
    return cudaSuccess;
}
cudaError_t cudaOccupancyMaxActiveClusters(int *n, const void *f, const cudaLaunchConfig_t *c)
{
    ++cluster_queries;
    if (limits[{device, f}] < (int)c->dynamicSmemBytes) return cudaErrorInvalidValue;
    *n = clusters_of[device];
    return cudaSuccess;
}
cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t *c, const void *f, void **)
{
    if (c->dynamicSmemBytes > 48 * 1024 && limits[{device, f}] < (int)c->dynamicSmemBytes) return cudaErrorInvalidValue;
    last_cluster = 1;
    for (unsigned i = 0; i < c->numAttrs; ++i)
        if (c->attrs[i].id == cudaLaunchAttributeClusterDimension) last_cluster = c->attrs[i].val.clusterDim.x;
    ++launches;
    return cudaSuccess;
}
// what the objects' start-up code and unused stubs refer to
void **__cudaRegisterFatBinary(void *) { static void *h; return &h; }
void __cudaRegisterFatBinaryEnd(void **) {}
void __cudaUnregisterFatBinary(void **) {}
void __cudaRegisterFunction() {}
int __cudaPopCallConfiguration() { return 1; }
int __cudaLaunchKernel() { return 1; }
int __cudaGetKernel() { return 1; }
}
namespace xp {
bool tmap_bytes(CUtensorMap *, const void *, uint64_t, uint64_t, uint64_t, uint32_t, uint32_t) { return true; }
bool tmap_bytes_kblocks(CUtensorMap *, const void *, uint64_t, uint64_t, uint64_t, uint32_t, uint32_t) { return true; }
int current_sms() { return 152; }
}
"""


@pytest.fixture
def lib(tmp_path):
    """A fresh library on the stand-in: what the first call sets up is not there yet."""
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    BLD.build()
    src, so = tmp_path / "fake.cpp", tmp_path / f"head_{os.getpid()}.so"
    src.write_text(FAKE)
    objs = [os.path.join(BLD.BUILD, f + ".o") for f in ("matmul_fp8", "matmul_fp8_wide", "logits")]
    inc = os.path.join(os.path.dirname(os.path.dirname(BLD.nvcc())), "include")
    subprocess.run([cxx, "-shared", "-fPIC", "-std=c++17", "-Wl,-Bsymbolic", "-I" + inc, str(src)] + objs + ["-o", str(so)],
                   check=True)
    lib = C.CDLL(str(so))
    lib.xpress_matmul_fp8.argtypes = [C.POINTER(X.XpressMatmulArgs), C.c_void_p, C.c_size_t, C.c_void_p]
    lib.xpress_process_logits.argtypes = [C.POINTER(X.XpressLogitsArgs), C.c_void_p, C.c_size_t, C.c_void_p]
    for dev in range(70):
        lib.fake_clusters(dev, 76)
    return lib


def _matmul(lib, M, N, K):
    # addresses are never followed: nothing is launched
    kb = -(-K // 128)
    g = X.XpressMatmulArgs(M=M, N=N, K=K, out_dtype=X.XPRESS_BF16, a=4096, lda=-(-K // 16) * 16, a_scale=4096, ld_a_scale=kb,
                           w=4096, ldw=-(-K // 16) * 16, w_scale=4096, ld_w_scale=kb, out=4096, ldo=N)
    return lib.xpress_matmul_fp8(g, 4096, 256, None)


def _logits(lib):
    # 600 rows of 151936 with penalties and biases: four slots per thread, 80 KB of counts and biases
    g = X.XpressLogitsArgs(n_seq=600, rows=1, V=151936, dtype=X.XPRESS_BF16, logits=4096, ld=151936, out=4096, ldo=151936,
                           repetition=4096, bias_ids=4096, bias_values=4096, n_bias=4, bias_offsets=4096)
    return lib.xpress_process_logits(g, None, 0, None)


CALLS = [  # few rows (16 and 32 of a tile), K split, many rows: persistent, split over 2, 4 and 8, a single tile of odd rows
    lambda lib: _matmul(lib, 16, 151936, 4096), lambda lib: _matmul(lib, 24, 151936, 4096),
    lambda lib: _matmul(lib, 1, 4096, 4096), lambda lib: _matmul(lib, 2048, 38912, 4096),
    lambda lib: _matmul(lib, 512, 4096, 4096), lambda lib: _matmul(lib, 300, 600, 8192),
    lambda lib: _matmul(lib, 129, 257, 16384), lambda lib: _matmul(lib, 1500, 1501, 400), _logits]


@pytest.mark.parametrize("call", CALLS)
def test_each_device_is_set_up(lib, call):
    for dev in (0, 1, 63, 64, 69, 0, 1):
        lib.fake_use(dev)
        before = lib.fake_launches()
        assert call(lib) == X.XPRESS_OK and lib.fake_launches() > before, f"device {dev}"


@pytest.mark.parametrize("call", [CALLS[0], CALLS[3], _logits])
def test_a_failure_is_not_kept(lib, call):
    lib.fake_fail_attributes(100)
    assert call(lib) == X.XPRESS_ERR_CUDA
    lib.fake_fail_attributes(0)
    assert call(lib) == X.XPRESS_OK


def test_clusters_are_counted_on_each_device(lib):
    lib.fake_clusters(1, 0)                                          # a device that runs no clusters
    sizes = []
    for dev in (0, 1, 0, 1):
        lib.fake_use(dev)
        assert _matmul(lib, 1, 4096, 4096) == X.XPRESS_OK
        sizes.append(lib.fake_last_cluster())
    assert sizes[0] > 1 and sizes == [sizes[0], 1, sizes[0], 1]
    # asked once for each device and cluster size
    lib.fake_use(0)
    n = lib.fake_cluster_queries()
    assert _matmul(lib, 1, 4096, 4096) == X.XPRESS_OK and lib.fake_cluster_queries() == n
