// Host side of the operators around the private gradient (include/bk.h): the
// RMS norm with its backward pass, and the orthogonalised updates.  Arguments
// are checked before any HIP call.
#include "bk.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <exception>
#include <vector>

#include "bk_kernels.h"
#include "step_kernels.h"

namespace {

using bk::host_fail;

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
size_t elem_bytes(bk_dtype dt) { return dt == BK_BF16 ? 2 : 4; }
bool is_dtype(int dt) { return dt == BK_F32 || dt == BK_BF16; }
bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// ------------------------------------------------------------------ RMS norm
bk_status check_rms(const char* fn, bk_dtype dt, int64_t B, int64_t T, int64_t p, const void* gamma, bk_dtype gdt) {
    if (!is_dtype(dt)) return host_fail(BK_ERR_INVALID_VALUE, "%s: unknown dtype %d", fn, (int)dt);
    if (gamma && !is_dtype(gdt)) return host_fail(BK_ERR_INVALID_VALUE, "%s: unknown gamma dtype %d", fn, (int)gdt);
    if (B < 0 || T < 0 || p < 1)
        return host_fail(BK_ERR_INVALID_VALUE, "%s: bad size (%lld x %lld rows of %lld columns)", fn, (long long)B,
                         (long long)T, (long long)p);
    int64_t rows;
    if (__builtin_mul_overflow(B, T, &rows))
        return host_fail(BK_ERR_INVALID_VALUE, "%s: size product overflows int64", fn);
    if (rows > INT32_MAX) return host_fail(BK_ERR_NOT_SUPPORTED, "%s: the number of rows must stay below 2^31", fn);
    if (p > bk::kRmsMaxCols)
        return host_fail(BK_ERR_NOT_SUPPORTED, "%s: rows of %lld columns, at most %lld are supported", fn, (long long)p,
                         (long long)bk::kRmsMaxCols);
    if (gamma && !aligned(gamma, elem_bytes(gdt))) return host_fail(BK_ERR_INVALID_VALUE, "%s: gamma misaligned", fn);
    return BK_OK;
}

// Outputs must not overlap anything else; `in_place`: the output may be the
// input that starts where it does (every thread has read what it overwrites).
struct Span {
    const void* t;
    size_t bytes;
    bool out, in_place;
};
template <size_t N>
bool spans_clash(const Span (&v)[N]) {
    for (size_t i = 0; i < N; ++i)
        for (size_t j = 0; j < N; ++j) {
            if (i == j || !v[i].t || !v[j].t || !v[i].out || (v[j].out && j > i)) continue;
            const uintptr_t a = reinterpret_cast<uintptr_t>(v[i].t), b = reinterpret_cast<uintptr_t>(v[j].t);
            if (a < b + v[j].bytes && b < a + v[i].bytes && !(a == b && v[i].in_place && v[j].in_place && !v[j].out))
                return true;
        }
    return false;
}

// Rows of a sample that a workgroup of the backward pass takes: few enough to
// give about 1024 workgroups, and 16 at least, so that the partial sums (4 p
// bytes written and read back for each) stay small next to the rows.  Workgroups
// that hold one row at a time take fewer than 16 until there is one to a CU: bf16
// [16, 64, 2048] 11 us with the joining launch instead of 23, [8, 16, 1100] 8
// instead of 30.  (Those of several rows at once gain nothing and pay for the
// joining: [32, 8, 768] 7.6 instead of 5.4.)
constexpr int64_t kRmsGradGroups = 1024, kRmsGradMinRows = 16, kRmsGradFewGroups = 256;
struct RmsGradPlan {
    int64_t chunk, chunks;
    bool solo;
};
RmsGradPlan rms_grad_plan(int64_t B, int64_t T, int64_t p) {
    const int64_t R = bk::rms_rows_at_once(p);
    if (T < R) return {std::max<int64_t>(T, 1), 1, true};
    const int64_t least = R > 1 ? kRmsGradMinRows : std::min(kRmsGradMinRows, cdiv(B * T, kRmsGradFewGroups));
    const int64_t chunk = cdiv(std::max(least, cdiv(B * T, kRmsGradGroups)), R) * R;
    return {chunk, cdiv(T, chunk), false};
}
size_t rms_grad_ws(int64_t B, int64_t T, int64_t p) {
    const RmsGradPlan g = rms_grad_plan(B, T, p);
    return g.chunks > 1 ? (size_t)B * g.chunks * p * sizeof(float) : 0;
}
// At least rms_grad_ws of B and of every smaller batch, where a workgroup takes
// fewer rows and more partial rows may be needed.  b samples in runs of `most` rows
// or more: b ceil(T / most) partial rows, and b + 1024 at most, as a run has b T /
// 1024 rows or more (from 1024 samples on all T).  Runs that are shorter than 16
// rows have b T / 256 or more: b T, and b + 256 at most, for less than 256 samples.
size_t rms_grad_ws_bound(int64_t B, int64_t T, int64_t p) {
    const int64_t R = bk::rms_rows_at_once(p), most = cdiv(kRmsGradMinRows, R) * R;
    int64_t parts = 0;
    if (T > most) {
        const int64_t b = std::min(B, kRmsGradGroups - 1);
        parts = std::min(b * cdiv(T, most), b + kRmsGradGroups);
    }
    if (R == 1 && T > 1) {
        const int64_t b = std::min(B, kRmsGradFewGroups - 1);
        parts = std::max(parts, std::min(b * T, b + kRmsGradFewGroups));
    }
    return (size_t)parts * p * sizeof(float);
}

// ------------------------------------------------------- orthogonalised updates
constexpr size_t kAlign = 256;
size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
constexpr int64_t kNsMaxSide = 1 << 20, kNsMaxElems = (int64_t)1 << 34;
using bk::kNsMaxSteps;
constexpr int64_t kNsMaxGrid = 1 << 23;        // workgroups of a launch (its threads stay below 2^32)
constexpr float kNsQuintic[3] = {3.4445f, -4.7750f, 2.0315f};

struct NsSize {
    int64_t m, n, mp, np;         // sides, the smaller first, and padded
    int64_t norm_elems, norm_wg, prep_wg;
    size_t bytes;                 // X0, X1, A, Bm
    bool small, thin;             // of these only `thin` uses what follows, and nothing above
    int64_t cols, chunks;         // columns of X for a workgroup, workgroups
};
NsSize ns_size(const bk_matrix& t, bool split) {
    NsSize z{};
    z.m = std::min(t.d, t.p), z.n = std::max(t.d, t.p);
    z.small = bk::ns_is_small(z.m, z.n);
    z.thin = !z.small && z.m <= bk::kNsSmallSide;
    if (z.thin) {
        // at most kNsThinChunks workgroups, each with at least 4 columns for a
        // row of the Gram matrix that it writes
        z.cols = std::max(cdiv(z.m, 16) * 64, cdiv(cdiv(z.n, bk::kNsThinChunks), 16) * 16);
        z.chunks = cdiv(z.n, z.cols);
    }
    if (z.small || z.thin) return z;
    z.mp = cdiv(z.m, bk::kNsPad) * bk::kNsPad, z.np = cdiv(z.n, bk::kNsPad) * bk::kNsPad;
    // at most kNsNormParts partial norms, which every workgroup of the next launch sums
    z.norm_elems = std::max<int64_t>(8, cdiv(cdiv(z.m * z.n, bk::kNsNormParts), 1024)) * 1024;
    z.norm_wg = cdiv(z.m * z.n, z.norm_elems);
    z.prep_wg = (z.mp / 64) * (z.np / 64);
    z.bytes = (split ? 2 : 1) * 2 * (size_t)(2 * z.mp * z.np + 2 * z.mp * z.mp);
    return z;
}

bk_status check_matrices(const char* fn, const bk_matrix* mats, int64_t n, int prec) {
    if (n < 0) return host_fail(BK_ERR_INVALID_VALUE, "%s: negative matrix count", fn);
    if (n > 0 && !mats) return host_fail(BK_ERR_INVALID_VALUE, "%s: NULL matrix array", fn);
    if (prec != BK_NS_F16 && prec != BK_NS_F32) return host_fail(BK_ERR_INVALID_VALUE, "%s: unknown precision %d", fn, prec);
    for (int64_t k = 0; k < n; ++k) {
        const bk_matrix& t = mats[k];
        if (t.d < 0 || t.p < 0)
            return host_fail(BK_ERR_INVALID_VALUE, "%s: matrix %lld: negative size", fn, (long long)k);
        if (t.d > kNsMaxSide || t.p > kNsMaxSide || t.d * t.p > kNsMaxElems)
            return host_fail(BK_ERR_NOT_SUPPORTED, "%s: matrix %lld: %lld x %lld (sides up to 2^20, 2^34 elements)", fn,
                             (long long)k, (long long)t.d, (long long)t.p);
    }
    return BK_OK;
}

// Memory that the call writes must not be read or written under another name.
struct Range {
    uintptr_t lo, hi;
    bool out;
};
bool overlapping(std::vector<Range>& v) {
    std::sort(v.begin(), v.end(), [](const Range& a, const Range& b) { return a.lo < b.lo; });
    uintptr_t end_out = 0, end_any = 0;
    for (const Range& r : v) {
        if (r.lo < (r.out ? end_any : end_out)) return true;
        end_any = std::max(end_any, r.hi);
        if (r.out) end_out = std::max(end_out, r.hi);
    }
    return false;
}

// Compute units of the current device (256 when none can be asked).
int64_t compute_units() {
    int dev = 0, cus = 0;
    if (hipGetDevice(&dev) != hipSuccess || hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus < 1)
        return 256;
    return cus;
}

// The tile shape of a product's launch: a CU takes about 0.15, 0.33, 0.5 and 0.85
// us for a stage of 32 k of a 64 x 64, 128 x 128, 256 x 128 and 256 x 256 tile, so
// the shape with the least of rounds times that.  Larger tiles move less per
// product, smaller ones fill the chip (kernel times, us):
//   A of one 768 x 768        78 / 21 tiles of 64 / 128               6.6 / 10.0
//   A of five odd matrices    340 / 92                                9.8 / 13.2
//   X of the same             871 / 231                              13.4 / 12.0
//   A of 12 x 768 x 768, float32-accurate  936 / 252 / 144 / 72       31 / 29 / 38 / 52
//   X of 4 x 1280 x 5120      1600 / 800 / 400 of 128 / 256 x 128 / 256    83 / 75 / 76
template <typename Count>
bk::NsTile ns_tile(int64_t cus, Count count) {
    constexpr int64_t cost[4] = {15, 33, 50, 85};
    bk::NsTile best = bk::NsTile::T128;
    int64_t least = INT64_MAX;
    for (int t = 0; t < 4; ++t) {
        const int64_t c = cdiv(count((bk::NsTile)t), cus) * cost[t];
        if (c < least) least = c, best = (bk::NsTile)t;
    }
    return best;
}

// Bounds of a step's matrices, from the bound of X's singular values: the
// largest |a + b t + c t^2| over t in [0, s^2], and of |a x + b x^3 + c x^5| over x
// in [0, s].
struct NsBound {
    double poly, next;
};
NsBound ns_bound(double a, double b, double c, double s) {
    auto f = [&](double x) { return std::fabs(x * (a + x * x * (b + x * x * c))); };
    auto g = [&](double t) { return std::fabs(a + t * (b + t * c)); };
    double next = f(s), poly = std::max(g(s * s), g(0));
    const double top = s * s;
    if (c != 0 && -b / (2 * c) > 0 && -b / (2 * c) < top) poly = std::max(poly, g(-b / (2 * c)));
    // 5 c t^2 + 3 b t + a = 0, t = x^2
    double roots[2];
    int nr = 0;
    if (c != 0) {
        const double disc = 9 * b * b - 20 * a * c;
        if (disc >= 0) {
            const double q = std::sqrt(disc);
            roots[nr++] = (-3 * b + q) / (10 * c);
            roots[nr++] = (-3 * b - q) / (10 * c);
        }
    } else if (b != 0) {
        roots[nr++] = -a / (3 * b);
    }
    for (int k = 0; k < nr; ++k)
        if (roots[k] > 0 && roots[k] < top) next = std::max(next, f(std::sqrt(roots[k])));
    return {poly, next};
}
// The power of two that brings `bound` to at most 2^15 (bounds near zero: that
// of 2^-15, so that scales stay far from the ends of float32).
float ns_scale(double bound) { return std::exp2f(std::floor(15 - std::log2(std::max(bound, 0x1p-15)))); }

// The matrices of a call: small ones, thin ones, and the others by the length of
// their first product (its longest tiles start first), in batches of as many as a
// launch's table and grid hold.  One batch runs after the other in the same
// workspace: the table, partial norms, then each matrix's arrays.
const size_t kNsTableBytes = align_up(sizeof(bk::NsTable));
struct NsOrder {
    std::vector<const bk_matrix*> small;
    std::vector<std::pair<const bk_matrix*, NsSize>> thin, rest;
    std::vector<std::pair<size_t, size_t>> batches;       // first, end in `rest`
};
NsOrder ns_order(const bk_matrix* mats, int64_t n, bool split) {
    NsOrder o;
    for (int64_t k = 0; k < n; ++k) {
        if (mats[k].d * mats[k].p == 0) continue;
        const NsSize z = ns_size(mats[k], split);
        if (z.small) o.small.push_back(&mats[k]);
        else if (z.thin) o.thin.emplace_back(&mats[k], z);
        else o.rest.emplace_back(&mats[k], z);
    }
    std::stable_sort(o.rest.begin(), o.rest.end(), [](const auto& x, const auto& y) { return x.second.np > y.second.np; });
    for (size_t k = 0; k < o.rest.size();) {
        const size_t first = k;
        int64_t norm = 0, prep = 0;
        for (; k < o.rest.size() && k - first < (size_t)bk::kMaxNs; ++k) {
            const NsSize& z = o.rest[k].second;
            if (k > first && std::max(norm + z.norm_wg, prep + z.prep_wg) > kNsMaxGrid) break;
            norm += z.norm_wg, prep += z.prep_wg;
        }
        o.batches.emplace_back(first, k);
    }
    return o;
}
size_t ns_ws(const NsOrder& o) {
    size_t most = 0;
    for (size_t k = 0; k < o.thin.size(); k += bk::kMaxNsThin) {
        size_t doubles = 0;
        for (size_t q = k; q < std::min(o.thin.size(), k + bk::kMaxNsThin); ++q)
            doubles += (size_t)bk::ns_thin_doubles(o.thin[q].second.m, o.thin[q].second.chunks);
        most = std::max(most, doubles * sizeof(double));
    }
    for (const auto& [first, last] : o.batches) {
        size_t bytes = 0, parts = 0;
        for (size_t q = first; q < last; ++q) bytes += o.rest[q].second.bytes, parts += (size_t)o.rest[q].second.norm_wg;
        most = std::max(most, kNsTableBytes + align_up(parts * sizeof(double)) + bytes);
    }
    return most;
}

// first[x] .. first[x + 1] - 1: tiles of XCD x, of a launch of `total` tiles of
// which those from L.*begin on cost L.*len each.
void ns_runs(const bk::NsNormArgs& a, int64_t total, int32_t bk::NsMat::*begin, int32_t bk::NsMat::*len, int32_t first[9]) {
    const auto end = [&](int k) { return k + 1 < a.n ? (int64_t)(a.L[k + 1].*begin) : total; };
    int64_t cost = 0, done = 0;
    for (int k = 0; k < a.n; ++k) cost += (end(k) - a.L[k].*begin) * (a.L[k].*len);
    int x = 0;
    for (int k = 0; k < a.n; ++k) {
        const int64_t c = a.L[k].*len, tiles = end(k) - a.L[k].*begin;
        // XCD x starts with the first tile before which x / 8 of the cost lies
        for (; x < 8 && cdiv(x * cost, 8) <= done + (tiles - 1) * c; ++x)
            first[x] = a.L[k].*begin + (int32_t)cdiv(std::max<int64_t>(cdiv(x * cost, 8) - done, 0), c);
        done += tiles * c;
    }
    for (; x <= 8; ++x) first[x] = (int32_t)total;
}

struct NsStep {
    float a, b, c, sx, sa, sb, sx2;
    double gain;                  // the largest factor of a singular value
};

// Rounds of a thin matrix's steps: end[r] is the first step behind round r.  A
// round's polynomials come from one Gram matrix, and their product P is rounded to
// float32, so an error of 2^-53 of an eigenvalue grows by gain^2 in each step (an
// eigenvalue of zero that rounding made negative leaves the polynomials' range
// when it nears 1: 18 of the usual steps, or 48 of 1.5 x - 0.5 x^3, gave NaN for
// updates of low rank), and P's rounding is off by 2^-24 of the product of gains,
// even in directions that have grown to 1 already.  A product of at most 2^9, the
// five usual steps (3.4445^5 = 485), keeps both as small as float32 products of X
// keep theirs: 2^-35 and 2^-15 at most.
constexpr double kNsRoundGain = 512;
int ns_rounds(const NsStep* plan, int64_t steps, uint8_t* end) {
    int rounds = 0;
    double gain = 1;
    for (int64_t k = 0; k < steps; ++k) {
        const double g = std::max(plan[k].gain, 1.0);
        if (k > 0 && gain * g > kNsRoundGain) end[rounds++] = (uint8_t)k, gain = 1;
        gain *= g;
    }
    end[rounds++] = (uint8_t)steps;
    return rounds;
}

bk_status run_ns(const char* fn, const bk_matrix* mats, int64_t n, int prec, bool step, float lr, float beta,
                 bool nesterov, float weight_decay, int64_t steps, const float* coef, float eps, void* ws,
                 size_t ws_bytes, hipStream_t s) {
    bk_status st = check_matrices(fn, mats, n, prec);
    if (st != BK_OK) return st;
    if (!(eps >= 0.f) || std::isinf(eps)) return host_fail(BK_ERR_INVALID_VALUE, "%s: eps must be finite and >= 0", fn);
    if (steps < 1 || steps > kNsMaxSteps)
        return host_fail(BK_ERR_INVALID_VALUE, "%s: %lld steps (1 to %lld)", fn, (long long)steps, (long long)kNsMaxSteps);
    const bool split = prec == BK_NS_F32;
    NsStep plan[kNsMaxSteps];
    double bound = 1.0;
    for (int64_t k = 0; k < steps; ++k) {
        const float* c = coef ? coef + 3 * k : kNsQuintic;
        const NsBound nb = ns_bound(c[0], c[1], c[2], bound);
        if (!(nb.next <= 64) || !(nb.poly <= 4096))
            return host_fail(BK_ERR_INVALID_VALUE, "%s: the polynomial of step %lld leaves [0, 64]", fn, (long long)k);
        plan[k] = {c[0], c[1], c[2], ns_scale(bound), ns_scale(bound * bound), ns_scale(nb.poly), ns_scale(nb.next),
                   nb.poly};
        bound = nb.next;
    }
    std::vector<Range> used;
    used.reserve((size_t)n * 5);
    for (int64_t k = 0; k < n; ++k) {
        const bk_matrix& t = mats[k];
        const int64_t e = t.d * t.p;
        if (e == 0) continue;
        const auto bad = [&](const char* what) {
            return host_fail(BK_ERR_INVALID_VALUE, "%s: matrix %lld: %s", fn, (long long)k, what);
        };
        if (!t.G) return bad("NULL G");
        if (!step && !t.O) return bad("NULL O");
        if (step && !t.O && !t.W) return bad("neither W nor O");
        if (step && t.Wb && !t.W) return bad("Wb without W");
        if (t.O && !is_dtype(t.o_dtype)) return bad("unknown dtype of O");
        const size_t oe = t.O ? elem_bytes((bk_dtype)t.o_dtype) : 1;
        if (!aligned(t.G, 4) || (t.O && !aligned(t.O, oe))) return bad("misaligned pointer");
        const auto add = [&](const void* q, size_t es, bool out) {
            if (q) used.push_back({reinterpret_cast<uintptr_t>(q), reinterpret_cast<uintptr_t>(q) + (size_t)e * es, out});
        };
        add(t.O, oe, true);
        if (t.O != t.G || oe != 4) add(t.G, 4, false);
        if (step) {
            if (!aligned(t.M, 4) || !aligned(t.W, 4) || !aligned(t.Wb, 2)) return bad("misaligned pointer");
            if (!std::isfinite(t.scale)) return bad("scale is not finite");
            add(t.M, 4, true);
            add(t.W, 4, true);
            add(t.Wb, 2, true);
        }
    }
    const NsOrder order = ns_order(mats, n, split);
    const size_t need = ns_ws(order);
    if (need > 0 && ws) used.push_back({reinterpret_cast<uintptr_t>(ws), reinterpret_cast<uintptr_t>(ws) + need, true});
    if (overlapping(used)) return host_fail(BK_ERR_INVALID_VALUE, "%s: tensors overlap", fn);
    if (ws_bytes < need || (need > 0 && !ws))
        return host_fail(BK_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", fn, ws_bytes, need);
    if (need > 0 && !aligned(ws, 16)) return host_fail(BK_ERR_INVALID_VALUE, "%s: workspace not 16-byte aligned", fn);
    const float keep = (float)(1.0 - (double)lr * weight_decay);

    // Small matrices.
    bk::NsSmallArgs sa{};
    sa.steps = (int32_t)steps, sa.nesterov = nesterov, sa.beta = beta, sa.keep = keep, sa.eps = eps;
    for (int64_t q = 0; q < steps; ++q) sa.coef[3 * q] = plan[q].a, sa.coef[3 * q + 1] = plan[q].b, sa.coef[3 * q + 2] = plan[q].c;
    for (size_t k = 0; k < order.small.size(); ++k) {
        const bk_matrix& t = *order.small[k];
        bk::NsSmallMat& L = sa.L[sa.n++];
        L = bk::NsSmallMat{};
        L.G = t.G, L.O = t.O, L.o_bf16 = t.o_dtype == BK_BF16, L.d = (int32_t)t.d, L.p = (int32_t)t.p;
        if (step) L.M = t.M, L.W = t.W, L.Wb = static_cast<uint16_t*>(t.Wb), L.step = (float)((double)lr * t.scale);
        if (sa.n < bk::kMaxNsSmall && k + 1 < order.small.size()) continue;
        const hipError_t e = bk::launch_ns_small(sa, s);
        if (e != hipSuccess) return bk::host_hip_fail(e, "orthogonalisation launch");
        sa.n = 0;
    }

    // Thin ones.
    bk::NsThinArgs ta{};
    ta.rounds = ns_rounds(plan, steps, ta.end), ta.nesterov = nesterov, ta.beta = beta, ta.keep = keep, ta.eps = eps;
    std::copy(sa.coef, sa.coef + 3 * steps, ta.coef);
    ta.ws = static_cast<double*>(ws);
    int64_t wgs = 0, doubles = 0;
    for (size_t k = 0; k < order.thin.size(); ++k) {
        const bk_matrix& t = *order.thin[k].first;
        const NsSize& z = order.thin[k].second;
        bk::NsThinMat& L = ta.L[ta.n++];
        L = bk::NsThinMat{};
        L.t.G = t.G, L.t.O = t.O, L.t.o_bf16 = t.o_dtype == BK_BF16, L.t.d = (int32_t)t.d, L.t.p = (int32_t)t.p;
        if (step)
            L.t.M = t.M, L.t.W = t.W, L.t.Wb = static_cast<uint16_t*>(t.Wb), L.t.step = (float)((double)lr * t.scale);
        L.chunks = (int32_t)z.chunks, L.cols = (int32_t)z.cols, L.begin = (int32_t)wgs, L.gram = doubles;
        wgs += z.chunks;
        doubles += bk::ns_thin_doubles(z.m, z.chunks);
        if (ta.n < bk::kMaxNsThin && k + 1 < order.thin.size()) continue;
        const hipError_t e = bk::launch_ns_thin(ta, (int)wgs, s);
        if (e != hipSuccess) return bk::host_hip_fail(e, "orthogonalisation launch");
        ta.n = 0;
        wgs = doubles = 0;
    }

    bk::NsNormArgs na{};
    bk::NsArgs a{};
    na.table = static_cast<bk::NsTable*>(ws);
    na.part = reinterpret_cast<double*>(static_cast<char*>(ws) + kNsTableBytes);
    a.table = na.table, a.part = na.part;
    na.nesterov = a.nesterov = nesterov, na.beta = a.beta = beta, a.keep = keep, a.eps = eps;
    const int64_t cus = compute_units();
    for (const auto& [first, last] : order.batches) {
        na.n = a.n = (int32_t)(last - first);
        const auto sym_of = [&](const NsSize& z, bk::NsTile t) { return bk::ns_sym_wg(z.mp, t); };
        const auto apply_of = [&](const NsSize& z, bk::NsTile t) { return bk::ns_apply_wg(z.mp, z.np, t); };
        const auto total = [&, first = first, last = last](auto of) {
            return [&, first, last, of](bk::NsTile t) {
                int64_t c = 0;
                for (size_t q = first; q < last; ++q) c += of(order.rest[q].second, t);
                return c;
            };
        };
        const bk::NsTile sym_tile = ns_tile(cus, total(sym_of)), apply_tile = ns_tile(cus, total(apply_of));
        int64_t norm = 0, prep = 0, sym = 0, apply = 0, base = 0, part = 0;
        for (size_t q = first; q < last; ++q) {
            const bk_matrix& t = *order.rest[q].first;
            const NsSize& z = order.rest[q].second;
            bk::NsMat& L = na.L[q - first];
            L = bk::NsMat{};
            L.G = t.G, L.O = t.O, L.o_bf16 = t.o_dtype == BK_BF16;
            if (step) L.M = t.M, L.W = t.W, L.Wb = static_cast<uint16_t*>(t.Wb), L.step = (float)((double)lr * t.scale);
            L.base = base;
            L.d = (int32_t)t.d, L.p = (int32_t)t.p, L.mp = (int32_t)z.mp, L.np = (int32_t)z.np, L.tall = t.d > t.p;
            L.part_off = (int32_t)part, L.norm_elems = (int32_t)z.norm_elems;
            L.norm_wg = (int32_t)norm, L.prep_wg = (int32_t)prep, L.sym_wg = (int32_t)sym, L.apply_wg = (int32_t)apply;
            norm += z.norm_wg, prep += z.prep_wg, sym += sym_of(z, sym_tile), apply += apply_of(z, apply_tile);
            base += (int64_t)z.bytes;
            part += z.norm_wg;
        }
        a.ws = static_cast<char*>(ws) + kNsTableBytes + align_up((size_t)part * sizeof(double));
        a.from = 0;
        a.sx = plan[0].sx;
        hipError_t e = bk::launch_ns_norm(na, (int)norm, s);
        if (e == hipSuccess) e = bk::launch_ns_prep(a, (int)prep, split, s);
        // Runs of tiles for the XCDs, equal in the length of their products: most
        // matrices then are read by one XCD's cache alone.
        int32_t runs[3][9];
        ns_runs(na, sym, &bk::NsMat::sym_wg, &bk::NsMat::np, runs[0]);
        ns_runs(na, sym, &bk::NsMat::sym_wg, &bk::NsMat::mp, runs[1]);
        ns_runs(na, apply, &bk::NsMat::apply_wg, &bk::NsMat::mp, runs[2]);
        const auto product = [&](bk::NsOp op, const int32_t* run, bk::NsTile t) {
            if (e != hipSuccess) return;
            std::copy(run, run + 9, a.xcd);
            e = bk::launch_ns_gemm(a, op, split, t, s);
        };
        for (int64_t q = 0; q < steps; ++q) {
            const NsStep& y = plan[q];
            a.a = y.a, a.b = y.b, a.c = y.c, a.sx = y.sx, a.sa = y.sa, a.sb = y.sb, a.sx2 = y.sx2;
            product(bk::NsOp::Gram, runs[0], sym_tile);
            product(bk::NsOp::Poly, runs[1], sym_tile);
            product(q + 1 < steps ? bk::NsOp::Apply : bk::NsOp::Final, runs[2], apply_tile);
            a.from ^= 1;
        }
        if (e != hipSuccess) return bk::host_hip_fail(e, "orthogonalisation launch");
    }
    return BK_OK;
}

// The lists of a call are its only allocations on the host; no exception leaves
// a C entry.
template <typename F>
bk_status guarded(const char* fn, F f) {
    try {
        return f();
    } catch (const std::exception& e) {
        return host_fail(BK_ERR_NOT_SUPPORTED, "%s: %s", fn, e.what());
    }
}

}  // namespace

extern "C" {

bk_status bk_rmsnorm(const void* x, const void* res, const void* gamma, bk_dtype dt, bk_dtype gamma_dt, int64_t rows,
                     int64_t p, float eps, void* h, void* y, void* xhat, float* rstd, void* q, float* q_scale,
                     int64_t q_group, void* stream) {
    const char* fn = "bk_rmsnorm";
    bk_status st = check_rms(fn, dt, rows, 1, p, gamma, gamma_dt);
    if (st != BK_OK) return st;
    if (!(eps >= 0.f) || std::isinf(eps)) return host_fail(BK_ERR_INVALID_VALUE, "%s: eps must be finite and >= 0", fn);
    if (q && q_group != 0 && q_group != 32 && q_group != 64 && q_group != 128)
        return host_fail(BK_ERR_INVALID_VALUE, "%s: groups of %lld columns (0, 32, 64 or 128)", fn, (long long)q_group);
    if (rows == 0) return BK_OK;
    if (!x) return host_fail(BK_ERR_INVALID_VALUE, "%s: NULL input pointer", fn);
    if (!h && !y && !xhat && !rstd && !q) return host_fail(BK_ERR_INVALID_VALUE, "%s: no output", fn);
    if (!q != !q_scale) return host_fail(BK_ERR_INVALID_VALUE, "%s: q and q_scale go together", fn);
    const size_t es = elem_bytes(dt);
    for (const void* t : {x, res, (const void*)h, (const void*)y, (const void*)xhat})
        if (!aligned(t, es)) return host_fail(BK_ERR_INVALID_VALUE, "%s: misaligned tensor", fn);
    if (!aligned(rstd, 4) || !aligned(q_scale, 4)) return host_fail(BK_ERR_INVALID_VALUE, "%s: misaligned output", fn);
    const size_t n = (size_t)rows * p, scales = (size_t)rows * (q_group ? cdiv(p, q_group) : 1) * 4;
    const Span spans[] = {{x, n * es, false, true},    {res, n * es, false, true}, {gamma, (size_t)p * elem_bytes(gamma_dt), false, false},
                          {h, n * es, true, true},     {y, n * es, true, true},    {xhat, n * es, true, true},
                          {rstd, (size_t)rows * 4, true, false}, {q, n, true, false}, {q_scale, scales, true, false}};
    if (spans_clash(spans)) return host_fail(BK_ERR_INVALID_VALUE, "%s: tensors overlap", fn);
    bk::RmsArgs a{};
    a.x = x, a.res = res, a.gamma = gamma;
    a.h = h, a.y = y, a.xhat = xhat, a.rstd = rstd, a.q = static_cast<uint8_t*>(q), a.q_scale = q_scale;
    a.rows = rows, a.p = (int32_t)p, a.gamma_bf16 = gamma_dt == BK_BF16;
    a.group = q ? (int32_t)q_group : 0;
    a.n_groups = a.group ? (int32_t)cdiv(p, q_group) : 1;
    a.eps = eps;
    const hipError_t e = bk::launch_rmsnorm(a, dt == BK_BF16, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? BK_OK : bk::host_hip_fail(e, "bk_rmsnorm launch");
}

size_t bk_rmsnorm_grad_workspace_size(int64_t B, int64_t T, int64_t p) {
    if (check_rms("bk_rmsnorm_grad_workspace_size", BK_F32, B, T, p, nullptr, BK_F32) != BK_OK || B * T == 0) return 0;
    return rms_grad_ws_bound(B, T, p);
}

bk_status bk_rmsnorm_grad(const void* dy, const void* xhat, const float* rstd, const void* gamma, const void* dres,
                          bk_dtype dt, bk_dtype gamma_dt, int64_t B, int64_t T, int64_t p, void* dx, float* P, void* ws,
                          size_t ws_bytes, void* stream) {
    const char* fn = "bk_rmsnorm_grad";
    bk_status st = check_rms(fn, dt, B, T, p, gamma, gamma_dt);
    if (st != BK_OK) return st;
    if (B == 0) return BK_OK;
    if (!dx && !P) return host_fail(BK_ERR_INVALID_VALUE, "%s: no output", fn);
    if (!aligned(P, 4)) return host_fail(BK_ERR_INVALID_VALUE, "%s: misaligned output", fn);
    if (T > 0) {
        if (!dy || !xhat || !rstd) return host_fail(BK_ERR_INVALID_VALUE, "%s: NULL input pointer", fn);
        const size_t es = elem_bytes(dt);
        for (const void* t : {dy, xhat, dres, (const void*)dx})
            if (!aligned(t, es)) return host_fail(BK_ERR_INVALID_VALUE, "%s: misaligned tensor", fn);
        if (!aligned(rstd, 4)) return host_fail(BK_ERR_INVALID_VALUE, "%s: rstd misaligned", fn);
    } else if (!P) {
        return BK_OK;               // no rows, and no sums asked for
    }
    const RmsGradPlan g = rms_grad_plan(B, T, p);
    const size_t need = P ? rms_grad_ws(B, T, p) : 0;
    if (ws_bytes < need || (need > 0 && !ws))
        return host_fail(BK_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", fn, ws_bytes, need);
    if (!aligned(ws, 4)) return host_fail(BK_ERR_INVALID_VALUE, "%s: misaligned workspace", fn);
    const size_t es = elem_bytes(dt), n = (size_t)B * T * p;
    const Span spans[] = {{dy, n * es, false, true}, {xhat, n * es, false, true}, {dres, n * es, false, true},
                          {rstd, (size_t)B * T * 4, false, false}, {gamma, (size_t)p * elem_bytes(gamma_dt), false, false},
                          {dx, n * es, true, true}, {P, (size_t)B * p * 4, true, false}, {need ? ws : nullptr, need, true, false}};
    if (spans_clash(spans)) return host_fail(BK_ERR_INVALID_VALUE, "%s: tensors overlap", fn);
    bk::RmsGradArgs a{};
    a.dy = dy, a.xhat = xhat, a.rstd = rstd, a.gamma = gamma, a.dres = dres, a.dx = dx, a.P = P;
    a.part = static_cast<float*>(ws);
    a.B = B, a.T = T, a.p = (int32_t)p, a.gamma_bf16 = gamma_dt == BK_BF16;
    a.chunk = (int32_t)g.chunk, a.chunks = (int32_t)g.chunks, a.solo = g.solo;
    const hipError_t e = bk::launch_rmsnorm_grad(a, dt == BK_BF16, static_cast<hipStream_t>(stream));
    return e == hipSuccess ? BK_OK : bk::host_hip_fail(e, "bk_rmsnorm_grad launch");
}

size_t bk_orthogonalize_workspace_size(const bk_matrix* mats, int64_t n, bk_ns_prec prec) {
    size_t bytes = 0;
    const int code = prec;
    guarded("bk_orthogonalize_workspace_size", [&] {
        const bk_status st = check_matrices("bk_orthogonalize_workspace_size", mats, n, code);
        if (st == BK_OK) bytes = ns_ws(ns_order(mats, n, code == BK_NS_F32));
        return st;
    });
    return bytes;
}

bk_status bk_orthogonalize(const bk_matrix* mats, int64_t n, bk_ns_prec prec, int64_t steps, const float* coef,
                           float eps, void* ws, size_t ws_bytes, void* stream) {
    const char* fn = "bk_orthogonalize";
    const int code = prec;
    return guarded(fn, [&] {
        return run_ns(fn, mats, n, code, false, 0.f, 0.f, false, 0.f, steps, coef, eps, ws, ws_bytes,
                      static_cast<hipStream_t>(stream));
    });
}

bk_status bk_muon_step(const bk_matrix* mats, int64_t n, bk_ns_prec prec, float lr, float beta, int nesterov,
                       float weight_decay, int64_t steps, const float* coef, float eps, void* ws, size_t ws_bytes,
                       void* stream) {
    const char* fn = "bk_muon_step";
    if (!std::isfinite(lr) || !std::isfinite(weight_decay) || !(beta >= 0.f && beta <= 1.f))
        return host_fail(BK_ERR_INVALID_VALUE, "%s: lr and weight_decay must be finite, beta in [0, 1]", fn);
    const int code = prec;
    return guarded(fn, [&] {
        return run_ns(fn, mats, n, code, true, lr, beta, nesterov != 0, weight_decay, steps, coef, eps, ws, ws_bytes,
                      static_cast<hipStream_t>(stream));
    });
}

}  // extern "C"
