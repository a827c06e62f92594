"""Every compiled variant of the 8-bit head's kernels is one that some call launches:
the kernels that the objects register, against those launched by calls over the entry
points' ranges, on the stand-in for the CUDA runtime (no GPU)."""
import ctypes as C
import itertools
import os
import shutil
import subprocess

import pytest

from paper_2608_02438_gb300 import binding as X
from paper_2608_02438_gb300 import build as BLD
from test_head_devices import FAKE

RECORD = FAKE.replace("void __cudaRegisterFunction() {}", """
void __cudaRegisterFunction(void **, const char *host, char *, const char *name, int, void *, void *, void *, void *, int *)
{
    registered()[host] = name;
}
int fake_registered() { return (int)registered().size(); }
int fake_launched() { return (int)launched().size(); }
const char *fake_never_launched()
{
    static std::string s;
    s.clear();
    for (auto &r : registered())
        if (!launched().count(r.first)) s += r.second + " ";
    return s.c_str();
}
""").replace("++launches;", "++launches; launched().insert(f);").replace(
    "*n = clusters_of[device];", "*n = clusters_of[device] / (int)c->attrs[0].val.clusterDim.x;").replace('extern "C" {\nvoid fake_use', """
#include <string>
static std::map<const void *, std::string> &registered() { static std::map<const void *, std::string> m; return m; }
static std::set<const void *> &launched() { static std::set<const void *> s; return s; }
extern "C" {
void fake_use""")


def _library(tmp_path, *objects):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    BLD.build()
    src, so = tmp_path / "fake.cpp", tmp_path / f"head_{os.getpid()}.so"
    src.write_text(RECORD)
    inc = os.path.join(os.path.dirname(os.path.dirname(BLD.nvcc())), "include")
    subprocess.run([cxx, "-shared", "-fPIC", "-std=c++17", "-Wl,-Bsymbolic", "-I" + inc, str(src)] +
                   [os.path.join(BLD.BUILD, f + ".o") for f in objects] + ["-o", str(so)], check=True)
    lib = C.CDLL(str(so))
    lib.fake_never_launched.restype = C.c_char_p
    for dev in range(70):
        lib.fake_clusters(dev, 152)
    return lib


def _all_launched(lib):
    assert lib.fake_registered() > 0
    assert lib.fake_never_launched() == b""
    assert lib.fake_launched() == lib.fake_registered()


def test_norm(tmp_path):
    lib = _library(tmp_path, "rmsnorm")
    for dt, H, rows, ld in itertools.product((X.XPRESS_F32, X.XPRESS_BF16), (200, 1500, 4096, 8192, 16384, 40000),
                                             (1, 1000), (1 << 16, (1 << 16) + 2, (1 << 16) + 1)):
        a = X.XpressNormArgs(rows=rows, H=H, dtype=dt, eps=1e-6, x=4096, ldx=ld, weight=4096, y=4096, ldy=ld)
        assert lib.xpress_rmsnorm(C.byref(a), None) == X.XPRESS_OK
    _all_launched(lib)


def test_quantize(tmp_path):
    lib = _library(tmp_path, "quant_fp8")
    for dt, ld in itertools.product((X.XPRESS_F32, X.XPRESS_BF16), (256, 257)):
        assert lib.xpress_quantize_weight(C.c_void_p(4096), dt, 300, 200, C.c_int64(ld), C.c_void_p(4096), C.c_int64(256),
                                          C.c_void_p(4096), None) == X.XPRESS_OK
    _all_launched(lib)


def test_matmul(tmp_path):
    lib = _library(tmp_path, "matmul_fp8", "matmul_fp8_wide")
    for M, N, K in ((16, 151936, 4096), (24, 151936, 4096), (1, 4096, 4096), (2048, 38912, 4096), (512, 4096, 4096),
                    (40, 1550, 8192), (40, 5000, 4096), (300, 600, 8192), (400, 5000, 512), (1500, 1501, 400)):
        kb, ld = -(-K // 128), -(-K // 16) * 16
        g = X.XpressMatmulArgs(M=M, N=N, K=K, out_dtype=X.XPRESS_BF16, a=4096, lda=ld, a_scale=4096, ld_a_scale=kb, w=4096,
                               ldw=ld, w_scale=4096, ld_w_scale=kb, out=4096, ldo=N)
        assert lib.xpress_matmul_fp8(C.byref(g), C.c_void_p(4096), C.c_size_t(256), None) == X.XPRESS_OK
    _all_launched(lib)


def test_logits(tmp_path):
    lib = _library(tmp_path, "logits")
    for dt, odd, (n_seq, rows, V, hist) in itertools.product(
            (X.XPRESS_F32, X.XPRESS_BF16), (0, 1),
            ((1, 1, 4096, 10), (300, 3, 4096, 10), (1, 1, 4096, 20000), (1, 300, 4096, 20000), (20, 1, 151936, 10),
             (20, 3, 151936, 10), (600, 1, 151936, 10), (600, 3, 151936, 10))):
        g = X.XpressLogitsArgs(n_seq=n_seq, rows=rows, V=V, dtype=dt, logits=4096, ld=V + odd, out=4096, ldo=V + odd,
                               argmax=4096, repetition=4096, history=4096, n_history=hist * n_seq, history_offsets=4096)
        assert lib.xpress_process_logits(C.byref(g), C.c_void_p(4096), C.c_size_t(1 << 40), None) == X.XPRESS_OK
    _all_launched(lib)
