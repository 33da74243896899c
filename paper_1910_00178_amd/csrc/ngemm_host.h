// What the host sides of the library share: the context, and the guard that makes its device the current one.
#pragma once
#include "ngemm.h"

#include <hip/hip_runtime.h>
#include <vector>

struct ngemm_ctx {
    uint32_t magic;
    int device;
    int num_cus;
    int num_xcd;             // XCDs (L2 domains) of the device; workgroup ids go round them in turn
    int force_kernel;
    int max_workgroups;      // 0 = one per compute unit
    void *static_scratch;    // device address of this device's copy of `scratch`
    // kernels found fastest by ngemm_tune_u8s8s32, by shape; consulted before the shape heuristic
    struct Tuned {
        int64_t M, N, K;
        int kernel;          // the fastest of NGEMM_KERNEL_*
        bool wavek;          // what only the automatic choice launches (gemm_wavek_kernel, gemm_mid_kernel) was faster still
    };
    std::vector<Tuned> tuned;
};

namespace ngemm {

constexpr uint32_t kCtxMagic = 0x4e47454du;   // "NGEM"

inline bool ctx_ok(const ngemm_ctx *c) { return c && c->magic == kCtxMagic; }

struct DeviceGuard {
    int prev = -1;
    bool ok = false;
    explicit DeviceGuard(int dev)
    {
        if (hipGetDevice(&prev) != hipSuccess) return;
        ok = (prev == dev) || (hipSetDevice(dev) == hipSuccess);
        if (prev == dev) prev = -1;
        // the launches below are checked with hipGetLastError(): drop an error that other code on
        // this thread left behind, so that it is not reported as one of ours
        (void)hipGetLastError();
    }
    ~DeviceGuard()
    {
        if (prev >= 0) (void)hipSetDevice(prev);
    }
};

}  // namespace ngemm
