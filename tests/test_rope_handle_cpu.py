"""The rope handle's life on a machine with several devices, with the runtime's
calls replaced by ones that keep a log (no GPU needed)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2601_11641_amd", "csrc")
HIP_INCLUDE = "/opt/rocm/include"

RUNTIME = r"""
#include "moddit_internal.h"
#include <cstdarg>
#include <cstdio>
#include <cstdlib>

static int device = 0;                    // the current one
static hipError_t last = hipSuccess;      // what hipGetLastError gives
static size_t room = 1 << 20;             // bytes that an allocation may have
static hipError_t done(hipError_t e) { if (e != hipSuccess) last = e; return e; }

extern "C" {
hipError_t hipGetDevice(int* d) { *d = device; return hipSuccess; }
hipError_t hipSetDevice(int d) { device = d; return hipSuccess; }
hipError_t hipMalloc(void** p, size_t n) {
    if (n > room) return done(hipErrorOutOfMemory);
    *p = std::malloc(n);
    return hipSuccess;
}
hipError_t hipFree(void* p) { std::printf("free on %d\n", device); std::free(p); return hipSuccess; }
hipError_t hipMemcpy(void*, const void*, size_t, hipMemcpyKind) { return hipSuccess; }
hipError_t hipDeviceSynchronize() { std::printf("wait for %d\n", device); return hipSuccess; }
hipError_t hipGetLastError() { hipError_t e = last; last = hipSuccess; return e; }
const char* hipGetErrorString(hipError_t) { return "an error"; }
}

namespace moddit {
mod_status fail(mod_status st, const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    std::vprintf(fmt, ap);
    va_end(ap);
    std::printf("\n");
    return st;
}
mod_status hip_fail(hipError_t, const char* what) { return fail(MOD_ERR_HIP, "%s", what); }
hipError_t launch_rope(const RopeTable&, const Strided&, const Strided&, int, int, int, int, int, int, const int32_t*,
                       bool, hipStream_t) { return hipGetLastError(); }
hipError_t launch_cache_write(const CacheView&, const Strided&, const Strided&, int, int, const int32_t*,
                              const int32_t*, hipStream_t) { std::abort(); }
hipError_t launch_cache_read(const CacheView&, const Strided&, const Strided&, int, int, const int32_t*, const int32_t*,
                             hipStream_t) { std::abort(); }
CacheAttnPlan plan_cache_attn(int, int, int, int, int, int, int, bool) { std::abort(); }
size_t cache_attn_plan_bytes(const CacheAttnPlan&, int) { std::abort(); }
hipError_t launch_cache_attn(const CacheAttnPlan&, const CacheView&, const uint16_t*, int, int, int, const int32_t*,
                             const int32_t*, const int32_t*, float, uint16_t*, float*, void*, hipStream_t) { std::abort(); }
}

int main() {
    mod_rope_params p{64, {16, 24, 24}, 2, 3, 4, 1e4, MOD_ROPE_ADJACENT};
    mod_rope *a = nullptr, *b = nullptr;
    alignas(16) static char x[4096], y[4096];
    mod_shape shape{1, 1, 4, 64, 64, 0, 0};
    @BODY@
    return 0;
}
"""


def run(tmp_path, body):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None or not os.path.exists(os.path.join(HIP_INCLUDE, "hip", "hip_runtime.h")):
        pytest.skip("no C++ compiler or HIP headers")
    src, exe = tmp_path / "handle.cpp", tmp_path / "handle"
    src.write_text(RUNTIME.replace("@BODY@", body))
    subprocess.run([cxx, "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I", HIP_INCLUDE, "-I", CSRC, str(src),
                    os.path.join(CSRC, "capi_cache.cpp"), "-o", str(exe)], check=True)
    return subprocess.run([str(exe)], check=True, capture_output=True, text=True, timeout=60).stdout.splitlines()


def test_destroy_waits_for_the_handles_device(tmp_path):
    """Also while another device is the current one, which it stays."""
    out = run(tmp_path, r"""
    device = 1;
    if (mod_rope_create(&p, &a)) return 1;
    device = 0;
    std::printf("destroy\n");
    if (mod_rope_destroy(a)) return 1;
    std::printf("now on %d\n", device);
    """)
    assert out == ["wait for 1", "destroy", "wait for 1", "free on 1", "now on 0"]


def test_a_failed_allocation_does_not_fail_the_next_call(tmp_path):
    """The runtime keeps an error until it is asked for; a launch asks."""
    out = run(tmp_path, r"""
    if (mod_rope_create(&p, &a)) return 1;
    room = 0;
    if (mod_rope_create(&p, &b) != MOD_ERR_NOMEM || b) return 1;
    std::printf("then %d\n", (int)mod_rope_fwd(a, &shape, x, nullptr, y, nullptr, 0, nullptr, nullptr));
    """)
    assert out[-1] == "then 0"
