"""What the library keeps for a device is kept for each device.  No GPU is needed: the host
code is compiled against stand-ins of the CUDA runtime's calls."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2604_20289_gb300", "csrc")
FAKES = r"""
#include <cstdio>
#include <cstdlib>
#include <vector>
static int g_dev = 0, g_fail = 0;
struct Ask { int dev, bytes; };
static std::vector<Ask> g_asked;
extern "C" cudaError_t cudaGetDevice(int *d) { *d = g_dev; return g_dev < 0 ? cudaErrorNoDevice : cudaSuccess; }
static int g_looked = 0, g_sms[64] = {152, 148, 0, 16};
extern "C" cudaError_t cudaDeviceGetAttribute(int *v, cudaDeviceAttr, int d) {
    ++g_looked;
    *v = g_sms[d];
    return g_fail ? cudaErrorInvalidValue : cudaSuccess;
}
static int g_made = 0, g_freed = 0, g_word[8], g_where[8];
extern "C" cudaError_t cudaMalloc(void **p, size_t n) {
    if (g_fail & 1) return cudaErrorMemoryAllocation;
    g_where[g_made] = g_dev;
    *p = &g_word[g_made++];
    return n == 4 ? cudaSuccess : cudaErrorInvalidValue;
}
extern "C" cudaError_t cudaMemset(void *p, int v, size_t n) {
    if (g_fail & 2) return cudaErrorInvalidValue;
    for (size_t i = 0; i < n; ++i) static_cast<char *>(p)[i] = (char)v;
    return cudaSuccess;
}
extern "C" cudaError_t cudaFree(void *) { return ++g_freed, cudaSuccess; }
extern "C" cudaError_t cudaFuncSetAttribute(const void *, cudaFuncAttribute, int v) {
    if (g_fail) return cudaErrorInvalidValue;
    g_asked.push_back({g_dev, v});
    return cudaSuccess;
}
#define EXPECT(x) do { if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); std::exit(1); } } while (0)
"""


def run(tmp_path, body):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no host compiler")
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text('#include "xc_device.h"\n' + FAKES + "int main() {\n" + body + "\n    return 0;\n}\n")
    cuda = os.environ.get("CUDA_HOME", "/usr/local/cuda")
    subprocess.run([cxx, "-std=c++17", "-I", CSRC, "-I", os.path.join(cuda, "include"), str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout


def test_shared_memory_is_asked_for_on_each_device(tmp_path):
    run(tmp_path, r"""
    xc::DeviceSet a{0}, b{0};
    void (*kernel)(int) = nullptr;
    for (int round = 0; round < 2; ++round)
        for (int dev : {0, 3, 63}) {
            g_dev = dev;
            EXPECT(xc::allow_smem(kernel, 100000, a) == cudaSuccess);
        }
    EXPECT(g_asked.size() == 3 && g_asked[0].dev == 0 && g_asked[1].dev == 3 && g_asked[2].dev == 63 && g_asked[1].bytes == 100000);
    EXPECT(xc::allow_smem(kernel, 90000, b) == cudaSuccess && g_asked.size() == 4);   // another kernel
    g_dev = 5;
    g_fail = 1;
    EXPECT(xc::allow_smem(kernel, 100000, a) == cudaErrorInvalidValue);               // not remembered as done
    g_fail = 0;
    EXPECT(xc::allow_smem(kernel, 100000, a) == cudaSuccess && g_asked.back().dev == 5);
    for (int dev : {-1, 64, 1000}) {
        g_dev = dev;
        EXPECT(xc::allow_smem(kernel, 100000, a) != cudaSuccess);
    }
    EXPECT(g_asked.size() == 5);
""")


def test_multiprocessors_are_each_device_s(tmp_path):
    run(tmp_path, r"""
    for (int round = 0; round < 2; ++round) {
        const int devs[] = {0, 1, 3}, want[] = {152, 148, 16};
        for (int i = 0; i < 3; ++i) {
            g_dev = devs[i];
            EXPECT(xc::device_sms() == want[i]);
        }
    }
    EXPECT(g_looked == 3);
    g_dev = 5;
    g_sms[5] = 100;
    g_fail = 1;
    EXPECT(xc::device_sms() == 1);                 // a failure is not remembered
    g_fail = 0;
    EXPECT(xc::device_sms() == 100);
    for (int dev : {-1, 64}) {
        g_dev = dev;
        EXPECT(xc::device_sms() == 1);
    }
""")


def test_the_error_word_is_in_the_device_s_own_memory(tmp_path):
    run(tmp_path, r"""
    for (int &w : g_word) w = 7;
    g_dev = 2;
    int *two = xc::device_error_word();
    g_dev = 0;
    int *zero = xc::device_error_word();
    EXPECT(two != nullptr && zero != nullptr && two != zero && *two == 0 && *zero == 0 && g_where[0] == 2 && g_where[1] == 0);
    g_dev = 2;
    EXPECT(xc::device_error_word() == two && g_made == 2);
    g_dev = 3;
    for (g_fail = 1; g_fail <= 2; ++g_fail) EXPECT(xc::device_error_word() == nullptr);
    EXPECT(g_freed == 1 && g_made == 3);
    g_fail = 0;
    EXPECT(xc::device_error_word() != nullptr && g_made == 4);
    for (int dev : {-1, 64}) {
        g_dev = dev;
        EXPECT(xc::device_error_word() == nullptr);
    }
""")


def test_a_product_s_workspace_is_each_device_s(monkeypatch):
    """Its size follows the multiprocessors."""
    torch = pytest.importorskip("torch")
    from test_devices_host import BF16, F32, I8, Tensor
    if not os.path.exists(os.path.join(ROOT, "paper_2604_20289_gb300", "libxcache.so")):
        from paper_2604_20289_gb300 import build
        build.build()
    from paper_2604_20289_gb300 import xcache as xb
    here, got = [0], []

    class Lib:
        xc_op_linear_i8_workspace_bytes = staticmethod(lambda *a: 1000 + here[0])
        xc_op_linear_i8 = staticmethod(lambda *a: 0)

    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: here[0], raising=False)
    monkeypatch.setattr(xb, "LIB", Lib)
    monkeypatch.setattr(xb, "_I8_BYTES", {})
    monkeypatch.setattr(xb, "_scratch", lambda n, *a: (got.append(n), 1 << 20, n))
    for dev in (0, 1, 0, 1):
        here[0] = dev
        xb.op_linear_i8("bf16", 0, Tensor((40, 64), BF16, dev), Tensor((32, 64), I8, dev), Tensor((32,), F32, dev),
                        Tensor((32,), F32, dev), Tensor((40, 32), BF16, dev), stream=7)
    assert got == [1000, 1001, 1000, 1001]


def sources():
    for name in sorted(os.listdir(CSRC)):
        with open(os.path.join(CSRC, name)) as f:
            yield name, f.read()


def test_no_source_asks_once_for_the_process():
    for name, text in sources():
        assert not re.search(r"static int \*\w+ = nullptr;\s+if", text), name
        assert not re.search(r"static \w+ \*\w+ = nullptr[;,]", text), name     # a pointer to one device's memory
        if name != "xc_device.h":
            assert "cudaFuncSetAttribute" not in text, name
            assert "cudaDevAttrMultiProcessorCount" not in text or name in ("k_gate.cu", "xc_api.cu"), name     # (not kept there)
        assert not re.search(r"static bool \w+ = false", text), name
