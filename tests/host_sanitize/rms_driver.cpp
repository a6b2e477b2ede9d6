// The workspace of the RMS norm's backward pass (step_api.cpp): the size for a
// batch serves every smaller one.  The launchers are stand-ins that check the
// partial rows' place.  Nothing here touches a GPU.
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <random>

#include "bk.h"
#include "bk_kernels.h"
#include "step_kernels.h"

namespace {
void need(bool ok, const char* what, int64_t B, int64_t T, int64_t p) {
    if (!ok) {
        std::fprintf(stderr, "check failed: %s (%lld x %lld x %lld)\n", what, (long long)B, (long long)T, (long long)p);
        std::abort();
    }
}
constexpr uintptr_t kWs = 0x700000000000ull;
size_t ws_bytes;
int launches, with_partials;
}  // namespace

extern "C" {
hipError_t hipGetDevice(int*) { return hipErrorUnknown; }
hipError_t hipDeviceGetAttribute(int*, hipDeviceAttribute_t, int) { return hipErrorUnknown; }
}

namespace bk {
bk_status host_fail(bk_status s, const char*, ...) { return s; }
bk_status host_hip_fail(hipError_t, const char*) { return BK_ERR_LAUNCH; }
hipError_t launch_rmsnorm(const RmsArgs&, bool, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_rmsnorm_grad(const RmsGradArgs& a, bool, hipStream_t) {
    ++launches;
    if (a.chunks > 1) {
        ++with_partials;
        need(reinterpret_cast<uintptr_t>(a.part) == kWs && (size_t)a.B * a.chunks * a.p * 4 <= ws_bytes, "partial rows in the workspace",
             a.B, a.T, a.p);
    }
    return hipSuccess;
}
hipError_t launch_ns_small(const NsSmallArgs&, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_ns_thin(const NsThinArgs&, int, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_ns_norm(const NsNormArgs&, int, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_ns_prep(const NsArgs&, int, bool, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_ns_gemm(const NsArgs&, NsOp, bool, NsTile, hipStream_t) { return hipErrorUnknown; }
}  // namespace bk

int main() {
    std::mt19937_64 rng(5);
    const auto at = [](int k) { return reinterpret_cast<void*>((uintptr_t)k << 52); };
    for (int it = 0; it < 600; ++it) {
        const int64_t ps[] = {8, 64, 100, 200, 768, 1025, 2048, 32768};
        const int64_t p = ps[rng() % 8], T = it < 40 ? it : (int64_t)std::exp2((double)(rng() % 1400) / 100);
        const int64_t full = 1 + (int64_t)std::exp2((double)(rng() % 1200) / 100);
        ws_bytes = bk_rmsnorm_grad_workspace_size(full, T, p);
        size_t above = ws_bytes;
        for (int64_t B = full; B >= 1; B -= B > 600 ? 1 + (int64_t)(rng() % 100) : 1) {
            const size_t size = bk_rmsnorm_grad_workspace_size(B, T, p);
            need(size <= above, "a smaller batch asks for no more", B, T, p);
            above = size;
            const bk_status s = bk_rmsnorm_grad(at(1), at(2), static_cast<float*>(at(3)), nullptr, nullptr, BK_BF16, BK_F32, B, T, p, at(4),
                                                static_cast<float*>(at(5)), ws_bytes ? reinterpret_cast<void*>(kWs) : nullptr, ws_bytes,
                                                nullptr);
            need(s == BK_OK, "the full batch's workspace serves a smaller one", B, T, p);
        }
    }
    need(with_partials > 1000 && with_partials < launches, "calls with and without partial rows", launches, with_partials, 0);
    std::printf("ok: %d of %d\n", with_partials, launches);
    return 0;
}
