// Kernel arguments and launchers of the operators on either side of the
// private gradient: the RMS norm with its backward pass, and the Newton-Schulz
// orthogonalisation with the Muon step (internal to libbk; the public
// interface is include/bk.h).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace bk {

// ---- RMS norm ---------------------------------------------------------------
constexpr int64_t kRmsMaxCols = 32768;   // columns the widest kernel holds in registers

struct RmsArgs {
    const void* x;
    const void* res;      // residual, or nullptr
    const void* gamma;    // [p], or nullptr (all ones)
    void* h;              // outputs; nullptr: not wanted
    void* y;
    void* xhat;
    float* rstd;
    uint8_t* q;
    float* q_scale;
    int64_t rows;
    int64_t row0;         // first row of a launch
    int32_t p;
    int32_t gamma_bf16;   // gamma is bf16 (else float32)
    int32_t group;        // columns a scale covers (0: the row)
    int32_t n_groups;     // scales per row
    float eps;
};
hipError_t launch_rmsnorm(const RmsArgs& a, bool bf16, hipStream_t s);

struct RmsGradArgs {
    const void* dy;
    const void* xhat;
    const float* rstd;
    const void* gamma;
    const void* dres;     // gradient of the residual stream, or nullptr
    void* dx;
    float* P;             // [B,p] per-sample gamma gradients, or nullptr
    float* part;          // [B, chunks, p] partial gamma gradients (chunks > 1)
    int64_t B, T;
    int64_t seg0;         // first segment of a launch
    int32_t p;
    int32_t gamma_bf16;
    int32_t chunk;        // rows of a sample that a workgroup (or, with `solo`, a group of threads) takes
    int32_t chunks;       // ceil(T / chunk)
    int32_t solo;         // each group of threads has a sample of its own
};
// Rows a workgroup of the backward kernel works on at once for p columns (a
// multiple of that where there are few workgroups).
constexpr int rms_rows_at_once(int64_t p) { return p <= 64 ? 32 : p <= 128 ? 16 : p <= 256 ? 8 : p <= 1024 ? 4 : 1; }
hipError_t launch_rmsnorm_grad(const RmsGradArgs& a, bool bf16, hipStream_t s);

// ---- Newton-Schulz orthogonalisation, Muon step -------------------------------
// X (m x n, m <= n) is the update or its transpose, rows padded to whole
// multiples of kNsPad with zeros; A = X X^T and Bm = a I + b A + c A^2 are m x m.  All
// are kept as 16-bit floats times a power of two that keeps them below 2^15,
// in the float32-accurate form as two such numbers, the second one what the
// first leaves.
constexpr int kNsPad = 64;
constexpr int64_t kNsNormParts = 4096;   // partial norms of a matrix, at most
struct NsMat {
    const float* G;     // [d,p]
    float* M;           // [d,p] momentum, or nullptr
    float* W;           // [d,p] weights, or nullptr
    uint16_t* Wb;       // [d,p] their bf16 copy, or nullptr
    void* O;            // [d,p] orthogonalised update, or nullptr
    int64_t base;       // bytes from NsArgs::ws to X0, X1, A, Bm
    int32_t d, p;
    int32_t mp, np;     // padded sides, mp <= np
    int32_t tall;       // X = U^T (d > p)
    int32_t o_bf16;     // O is bf16 (else float32)
    float step;         // what multiplies O in the weights' update
    int32_t part_off;   // first norm partial
    int32_t norm_elems; // elements of a partial norm
    int32_t norm_wg, prep_wg, sym_wg, apply_wg;   // first workgroups in the launches
};
constexpr int kMaxNs = 36;
// The first launch of a batch takes its table in the kernel arguments and
// writes it to the workspace, where the others read it: kernel arguments lie in
// host memory, and a search in them costs a round trip for each step.
struct NsTable {
    NsMat L[kMaxNs];
    int32_t prep[kMaxNs], sym[kMaxNs], apply[kMaxNs];   // first workgroups (tiles) of the matrices
};
struct NsNormArgs {
    int32_t n;
    int32_t nesterov;
    float beta;         // momentum
    NsTable* table;
    double* part;       // partial squared norms
    NsMat L[kMaxNs];
};
static_assert(sizeof(NsNormArgs) <= 4096 - 64, "kernel arguments");
struct NsArgs {
    const NsTable* table;
    char* ws;           // the matrices' arrays
    const double* part;
    int32_t n;
    int32_t nesterov;
    float beta;
    float keep;         // 1 - lr weight_decay
    float eps;
    float a, b, c;      // this step's polynomial
    // powers of two: scales of X and of A, Bm in this step, of X after it
    float sx, sa, sb, sx2;
    int32_t from;       // which of X0, X1 holds X
    int32_t xcd[9];     // a product's tiles xcd[x] .. xcd[x + 1] - 1 run on XCD x
};
enum class NsOp { Gram = 0, Poly = 1, Apply = 2, Final = 3 };
enum class NsTile { T64 = 0, T128 = 1, T256x128 = 2, T256 = 3 };
constexpr int ns_tile_m(NsTile t) { return t == NsTile::T64 ? 64 : t == NsTile::T128 ? 128 : 256; }
constexpr int ns_tile_n(NsTile t) { return t == NsTile::T64 ? 64 : t == NsTile::T256 ? 256 : 128; }
// Tiles of a symmetric product on and above the diagonal: column nt of tn has
// the first nt / R + 1 of tm rows of tiles, R = 1 or 2 columns to a row's width.
__host__ __device__ inline int64_t ns_sym_tiles(int64_t tm, int64_t tn, int R) {
    const int64_t full = tn / R;          // whole groups of R columns: 1, 2, ..., full tiles each
    return R * full * (full + 1) / 2 + (tn - R * full) * tm;
}
inline int64_t ns_sym_wg(int64_t mp, NsTile t) {
    const int64_t m = ns_tile_m(t), n = ns_tile_n(t);
    return ns_sym_tiles((mp + m - 1) / m, (mp + n - 1) / n, (int)(m / n));
}
inline int64_t ns_apply_wg(int64_t mp, int64_t np, NsTile t) {
    const int64_t m = ns_tile_m(t), n = ns_tile_n(t);
    return ((mp + m - 1) / m) * ((np + n - 1) / n);
}
// Small matrices: the whole iteration in one workgroup, X in LDS in float32.
struct NsSmallMat {
    const float* G;
    float* M;
    float* W;
    uint16_t* Wb;
    void* O;
    int32_t d, p;
    float step;
    int32_t o_bf16;
};
constexpr int kMaxNsSmall = 56, kNsMaxSteps = 64;
struct NsSmallArgs {
    int32_t n, steps;
    int32_t nesterov;
    float beta, keep, eps;
    float coef[3 * kNsMaxSteps];
    NsSmallMat L[kMaxNsSmall];
};
// Row stride (floats) of X in LDS: a whole number of 16-column tiles, an odd
// multiple of 16 so that four rows' 64-byte pieces lie on distinct banks.
__host__ __device__ inline int64_t ns_small_ld(int64_t n) {
    const int64_t t = (n + 15) / 16;
    return (t | 1) * 16;
}
constexpr int64_t kNsSmallSide = 64, kNsSmallFloats = 27 * 1024;     // m, and m ns_small_ld(n)
inline bool ns_is_small(int64_t m, int64_t n) {
    return m <= kNsSmallSide && n <= kNsSmallFloats && (m + 15) / 16 * 16 * ns_small_ld(n) <= kNsSmallFloats;
}
hipError_t launch_ns_small(const NsSmallArgs& a, hipStream_t s);
// Thin matrices (m <= 64, n too long for LDS): rounds of steps, two launches each
// and one at the end.
struct NsThinMat {
    NsSmallMat t;
    int32_t chunks;     // workgroups along n, `cols` columns of X each (a multiple of 16)
    int32_t cols;
    int32_t begin;      // first workgroup
    int32_t pad;
    int64_t gram;       // doubles from NsThinArgs::ws to the partial Grams [chunks][m16][m16], then 1 / (|U| + eps)
                        // and the rounds' polynomials (float32 [rounds][m16][m16])
};
constexpr int kMaxNsThin = 30, kNsThinChunks = 64;
struct NsThinArgs {
    int32_t n;
    int32_t rounds;                 // at most one to a step
    int32_t nesterov;
    float beta, keep, eps;
    int32_t round, first, last;     // a launch's round, its steps first .. last - 1
    double* ws;
    float coef[3 * kNsMaxSteps];
    NsThinMat L[kMaxNsThin];
    uint8_t end[kNsMaxSteps];       // round r: steps end[r - 1] (0 for the first) .. end[r] - 1 (for the host)
};
static_assert(sizeof(NsThinArgs) <= 4096 - 64 && sizeof(NsSmallArgs) <= 4096 - 64, "kernel arguments");
constexpr int kNsThinFloats = 8192;                     // of X in a workgroup's LDS at a time
__host__ __device__ constexpr int64_t ns_thin_tile(int64_t m) { return kNsThinFloats / ((m + 15) / 16 * 16) / 16 * 16; }   // its columns
inline int64_t ns_thin_doubles(int64_t m, int64_t chunks) {
    const int64_t e = (m + 15) / 16 * 16 * ((m + 15) / 16 * 16);
    return chunks * e + 1 + kNsMaxSteps * (e / 2);
}
// Every round of `a` (whose round, first and last are not read).
hipError_t launch_ns_thin(const NsThinArgs& a, int n_wg, hipStream_t s);
hipError_t launch_ns_norm(const NsNormArgs& a, int n_wg, hipStream_t s);
hipError_t launch_ns_prep(const NsArgs& a, int n_wg, bool split, hipStream_t s);
// The tiles of a.xcd, on 8 times as many workgroups as the largest XCD's run.
hipError_t launch_ns_gemm(const NsArgs& a, NsOp op, bool split, NsTile t, hipStream_t s);

}  // namespace bk
