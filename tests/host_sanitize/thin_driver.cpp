// The rounds of the thin matrices' steps (step_api.cpp), under AddressSanitizer
// and UndefinedBehaviorSanitizer: random polynomials, with the launchers replaced
// by stand-ins that check the plan.  Nothing here touches a GPU.
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "bk.h"
#include "bk_kernels.h"
#include "step_kernels.h"

namespace {
std::mt19937_64 rng(64);
void need(bool ok, const char* what) {
    if (!ok) {
        std::fprintf(stderr, "check failed: %s\n", what);
        std::abort();
    }
}
int launches, most_rounds;
uintptr_t ws_lo, ws_hi;
// The largest factor of a singular value in each step, by sampling.
std::vector<double> gains(const float* coef, int steps) {
    std::vector<double> g;
    double s = 1;
    for (int k = 0; k < steps; ++k) {
        const double a = coef[3 * k], b = coef[3 * k + 1], c = coef[3 * k + 2];
        double factor = 0, next = 0;
        for (int i = 0; i <= 2000; ++i) {
            const double x = s * i / 2000, f = std::fabs(a + x * x * (b + x * x * c));
            factor = std::max(factor, f), next = std::max(next, f * x);
        }
        g.push_back(factor);
        s = next;
    }
    return g;
}
}  // namespace

extern "C" {
hipError_t hipGetDevice(int* d) {
    *d = 0;
    return hipSuccess;
}
hipError_t hipDeviceGetAttribute(int* v, hipDeviceAttribute_t, int) {
    *v = 256;
    return hipSuccess;
}
}

namespace bk {
bk_status host_fail(bk_status s, const char* fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    std::vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    return s;
}
bk_status host_hip_fail(hipError_t, const char*) { return BK_ERR_LAUNCH; }
hipError_t launch_rmsnorm(const RmsArgs&, bool, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_rmsnorm_grad(const RmsGradArgs&, bool, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_ns_small(const NsSmallArgs&, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_ns_norm(const NsNormArgs&, int, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_ns_prep(const NsArgs&, int, bool, hipStream_t) { return hipErrorUnknown; }
hipError_t launch_ns_gemm(const NsArgs&, NsOp, bool, NsTile, hipStream_t) { return hipErrorUnknown; }

int want_steps;
hipError_t launch_ns_thin(const NsThinArgs& a, int, hipStream_t) {
    ++launches;
    need(a.rounds >= 1 && a.rounds <= want_steps && a.end[a.rounds - 1] == want_steps, "the rounds cover the steps");
    most_rounds = std::max(most_rounds, (int)a.rounds);
    const std::vector<double> g = gains(a.coef, want_steps);
    for (int r = 0; r < a.rounds; ++r) {
        const int first = r ? a.end[r - 1] : 0;
        need(a.end[r] > first, "no empty round");
        double all = 1;
        for (int k = first; k < a.end[r]; ++k) all *= std::max(1.0, g[(size_t)k]);
        need(a.end[r] == first + 1 || all <= 512 * 1.001, "a round's gain");
        need(r + 1 == a.rounds || all * std::max(1.0, g[(size_t)a.end[r]]) >= 512 * 0.98, "rounds as long as they may be");
    }
    for (int k = 0; k < a.n; ++k) {
        const int64_t m = std::min(a.L[k].t.d, a.L[k].t.p), m16 = (m + 15) / 16 * 16;
        const uintptr_t p = reinterpret_cast<uintptr_t>(a.ws + a.L[k].gram + a.L[k].chunks * m16 * m16 + 1);
        need(p >= ws_lo && p + (size_t)(a.rounds * m16 * m16) * 4 <= ws_hi, "every round's polynomial in the workspace");
        if (k + 1 < a.n)
            need(p + (size_t)(a.rounds * m16 * m16) * 4 <= reinterpret_cast<uintptr_t>(a.ws + a.L[k + 1].gram), "one after another");
    }
    return hipSuccess;
}
}  // namespace bk

int main() {
    int ok = 0;
    for (int it = 0; it < 3000; ++it) {
        std::vector<bk_matrix> m(1 + rng() % 40);
        uintptr_t at = 0x10000000;
        for (bk_matrix& t : m) {
            t = bk_matrix{};
            t.d = 1 + (int64_t)(rng() % 64), t.p = 2000 + (int64_t)(rng() % 3000);
            if (rng() % 2) std::swap(t.d, t.p);
            t.G = reinterpret_cast<float*>(at), t.O = reinterpret_cast<void*>(at + 4 * 64 * 5000);
            at += 8 * 64 * 5000;
        }
        const int64_t n = (int64_t)m.size();
        const int steps = it < 64 ? it + 1 : 1 + (int)(rng() % 64);
        std::vector<float> coef;
        if (it >= 64)
            for (int k = 0; k < steps; ++k) {
                const float a = 0.5f + (float)(rng() % 100) / 30.f, c = (float)(rng() % 100) / 40.f;
                // b from the extremes: polynomials that stay small, now and then one that does not
                for (float v : {a, -(a + c) + 0.9f - (float)(rng() % 10) / 20.f, c}) coef.push_back(v);
            }
        bk::want_steps = steps;
        const size_t ws = bk_orthogonalize_workspace_size(m.data(), n, BK_NS_F32);
        ws_lo = 0x700000000000ull, ws_hi = ws_lo + ws;
        launches = most_rounds = 0;
        const bk_status s = bk_orthogonalize(m.data(), n, BK_NS_F32, steps, coef.empty() ? nullptr : coef.data(), 1e-7f,
                                             reinterpret_cast<void*>(ws_lo), ws, nullptr);
        need(s == BK_OK || s == BK_ERR_INVALID_VALUE, "status");
        if (s != BK_OK) continue;
        ++ok;
        need(launches == (n + bk::kMaxNsThin - 1) / bk::kMaxNsThin, "batches");
        if (it < 64) need(most_rounds == (steps + 4) / 5, "five of the usual steps to a round");
    }
    need(ok > 500, "calls that run");
    std::printf("ok: %d\n", ok);
    return 0;
}
