"""Which device a logit cap may be set from: the plan's own, whatever the mode and
the cap.  There is no second GPU here, so the planner's source is built against a
runtime that keeps "device" memory on the host and reports the device it is told."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from paper_2608_24658_gb300 import _lib
from paper_2608_24658_gb300 import build as B

FAKE = r"""
#include <cstdlib>
#include <cstring>
#include "internal.h"
namespace parason {
cudaError_t launch_merge(const MergeArgs &, int, int, bool, cudaStream_t) { return cudaErrorNotSupported; }
cudaError_t launch_prefill(const AttnArgs &, const KvMaps &, int, cudaStream_t) { return cudaErrorNotSupported; }
cudaError_t launch_scatter(int32_t *, const int2 *, int32_t, cudaStream_t) { return cudaErrorNotSupported; }
cudaError_t launch_attn_fp8(const AttnArgs &, const KvMaps &, int, cudaStream_t) { return cudaErrorNotSupported; }
cudaError_t launch_attn_bf16(const AttnArgs &, const KvMaps &, int, cudaStream_t) { return cudaErrorNotSupported; }
cudaError_t launch_attn_fp32(const AttnArgs &, const float *, const float *, int, cudaStream_t) {
    return cudaErrorNotSupported;
}
cudaError_t launch_lse_merge(const void *, const float *, const void *, const float *, void *, float *, int64_t, int,
                             int, cudaStream_t) { return cudaErrorNotSupported; }
cudaError_t attn_mma_ctas_per_sm(int, int, int *n) { *n = 1; return cudaSuccess; }
cudaError_t attn_mma_prepare_cap(int, int) { return cudaSuccess; }
cudaError_t prefill_prepare_cap(int) { return cudaSuccess; }
}
static int device = 0;
extern "C" {
void fake_set_device(int d) { device = d; }
cudaError_t cudaGetDevice(int *d) { *d = device; return cudaSuccess; }
cudaError_t cudaDeviceGetAttribute(int *v, cudaDeviceAttr, int) { *v = 152; return cudaSuccess; }
cudaError_t cudaMalloc(void **p, size_t n) { *p = malloc(n); return cudaSuccess; }
cudaError_t cudaFree(void *p) { free(p); return cudaSuccess; }
cudaError_t cudaMemcpy(void *d, const void *s, size_t n, cudaMemcpyKind) { memcpy(d, s, n); return cudaSuccess; }
cudaError_t cudaMemcpyAsync(void *d, const void *s, size_t n, cudaMemcpyKind, cudaStream_t) {
    memcpy(d, s, n);
    return cudaSuccess;
}
cudaError_t cudaMemset(void *d, int v, size_t n) { memset(d, v, n); return cudaSuccess; }
cudaError_t cudaMemsetAsync(void *d, int v, size_t n, cudaStream_t) { memset(d, v, n); return cudaSuccess; }
cudaError_t cudaStreamSynchronize(cudaStream_t) { return cudaSuccess; }
cudaError_t cudaGetLastError() { return cudaSuccess; }
cudaError_t cudaEventCreate(cudaEvent_t *) { return cudaErrorNotSupported; }
cudaError_t cudaEventDestroy(cudaEvent_t) { return cudaSuccess; }
cudaError_t cudaEventElapsedTime(float *, cudaEvent_t, cudaEvent_t) { return cudaErrorNotSupported; }
cudaError_t cudaEventRecord(cudaEvent_t, cudaStream_t) { return cudaErrorNotSupported; }
cudaError_t cudaEventSynchronize(cudaEvent_t) { return cudaErrorNotSupported; }
cudaError_t cudaGetDriverEntryPointByVersion(const char *, void **, unsigned, unsigned long long,
                                             cudaDriverEntryPointQueryResult *) { return cudaErrorNotSupported; }
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    where = tmp_path_factory.mktemp("fake")
    src, out = where / "fake.cpp", where / "libfake.so"
    src.write_text(FAKE)
    subprocess.run(["g++", "-O1", "-std=c++17", "-fPIC", "-shared", "-Wl,-Bsymbolic", "-I", B.INCLUDE, "-I", B.CSRC, "-I",
                    os.path.join(B._cuda_home(), "include"), str(src), os.path.join(B.CSRC, "plan.cpp"), "-o", str(out)],
                   check=True)
    lib = ctypes.CDLL(str(out))
    for name in ("parason_attn_plan", "parason_attn_plan_host", "parason_prefill_plan", "parason_plan_set_logit_cap",
                 "parason_plan_destroy"):
        getattr(lib, name).restype, getattr(lib, name).argtypes = _lib.SIGNATURES[name]
    return lib


def make(lib, mode, fn="parason_attn_plan"):
    cfg = _lib.AttnConfig(8, 2, 128, 16, _lib.MODES[mode], 0.0)
    parent, length, ptr, pages, leaf = (np.array(a, np.int32) for a in ([-1, 0], [40, 20], [0, 3, 5], range(5), [1]))
    plan = ctypes.c_void_p()
    where = 152 if fn.endswith("_host") else None
    st = getattr(lib, fn)(ctypes.byref(cfg), 2, *(a.ctypes.data for a in (parent, length, ptr, pages)), 1,
                          leaf.ctypes.data, 5, where, ctypes.byref(plan))
    assert st == _lib.OK
    return plan


@pytest.mark.parametrize("mode,fn", [("bf16", "parason_attn_plan"), ("fp8", "parason_attn_plan"),
                                     ("fp32", "parason_attn_plan"), ("bf16", "parason_prefill_plan")])
def test_a_cap_is_set_from_the_plans_device(lib, mode, fn):
    lib.fake_set_device(0)
    plan = make(lib, mode, fn)
    for cap in (30.0, 90.0, 0.0):
        lib.fake_set_device(1)
        assert lib.parason_plan_set_logit_cap(plan, cap) == _lib.EINVAL
        lib.fake_set_device(0)
        assert lib.parason_plan_set_logit_cap(plan, cap) == _lib.OK
        assert lib.parason_plan_set_logit_cap(plan, -1.0) == _lib.EINVAL
    lib.parason_plan_destroy(plan)


def test_a_host_plan_has_no_device(lib):
    lib.fake_set_device(1)
    plan = make(lib, "bf16", "parason_attn_plan_host")
    assert lib.parason_plan_set_logit_cap(plan, 30.0) == _lib.OK
    lib.parason_plan_destroy(plan)
    lib.fake_set_device(0)
