// Newton-Schulz orthogonalisation of updates, with Muon's momentum before it
// and the weights' update behind it.
//
//   M = beta M + G, U = G + beta M (Nesterov) or M      (no M: U = G)
//   X = U / (|U|_F + eps), transposed if U is taller than wide (m <= n then)
//   steps times:  A = X X^T,  Bm = a I + b A + c A^2,  X <- Bm X
//   O = X (transposed back),  W <- keep W - step O
//
// A and Bm are symmetric: their tiles below the diagonal are mirrored.
//
// The products run on the 16-bit matrix instructions.  bf16 keeps too few bits
// for a chain of fifteen products whose small singular values grow 485-fold
// (O off by 1 to 5% against 64 bits for private gradients of 256 to 768
// columns); fp16 at the same rate keeps 3 more (0.12 to 0.4%; of updates of
// rank r, up to 0.18 / sqrt(r) was seen), and its range
// suffices because every matrix here has a known bound: singular values of X
// are at most 1 at first and the polynomials' largest value later, so that
// powers of two, chosen on the host for each step, keep all entries below 2^15
// and the fp16 quantum at 2^-39 of the bound.  Sums are float32.
//
// SPLIT, the float32-accurate form: a number is v = hi + lo, both fp16: 22
// bits, down to the fp16 quantum, which the powers of two put at 2^-39 of the
// matrix's bound.  A product is hi hi + hi lo + lo hi, three times the matrix
// instructions, summed in one accumulator.
#include "bk_device.h"
#include "step_kernels.h"

#include <algorithm>
#include <type_traits>

namespace bk {
namespace {

typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4_t __attribute__((ext_vector_type(4)));
typedef short v4i16 __attribute__((ext_vector_type(4)));
constexpr uint32_t kOut = 0xFFFFFFF0u;           // buffer offset that loads zeros

// Byte of element (i, j), or of its part z, of a matrix of `rows` rows: columns
// in blocks of 32 (SPLIT: of 16, their high parts before their low parts), a
// block's rows one after another, 64 bytes each.  A stage of a product is then
// made of whole runs of at least 1 KB.
template <bool SPLIT>
__device__ __forceinline__ size_t ns_at(int i, int j, int rows, int z = 0) {
    if constexpr (SPLIT) return (size_t)(j >> 4) * rows * 64 + (size_t)i * 64 + 32 * z + (j & 15) * 2;
    else return (size_t)(j >> 5) * rows * 64 + (size_t)i * 64 + (j & 31) * 2;
}
// Bytes from an element to the one 16 columns on, from a multiple of 32 on.
template <bool SPLIT>
__device__ __forceinline__ size_t ns_next16(int rows) { return SPLIT ? (size_t)rows * 64 : 32; }

// This step's update entry from G and the momentum (already updated).
__device__ __forceinline__ float update_of(float g, float m, bool has_m, int nesterov, float beta) {
    return !has_m ? g : nesterov ? fmaf(beta, m, g) : m;
}

__device__ __forceinline__ double block_sum_double(double v, double* red) {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off, 64);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = red[0] + red[1] + red[2] + red[3];
    return v;
}

// The matrix of workgroup (tile) `wg`: the last k < n <= 64 with begin(k) <= wg,
// begin being non-decreasing from 0 on.  One load for all of them.  `local`: wg's
// place in the matrix.
template <typename Begin>
__device__ __forceinline__ int find_matrix(int n, int wg, int& local, Begin begin) {
    const int lane = threadIdx.x & 63;
    const int b = lane < n ? begin(lane) : INT32_MAX;
    const int k = __builtin_amdgcn_readfirstlane(__popcll(__ballot(b <= wg)) - 1);
    local = wg - __builtin_amdgcn_readlane(b, k);
    return k;
}

// A matrix's entry of the table, by scalar loads (nothing writes the table while
// a kernel reads it).
__device__ __forceinline__ NsMat load_matrix(const NsTable* table, int l) {
    typedef const __attribute__((address_space(4))) uint32_t* scalar_t;
    const scalar_t w = (scalar_t)(uintptr_t)(table->L + l);
    uint32_t v[sizeof(NsMat) / 4];
#pragma unroll
    for (int k = 0; k < (int)sizeof(NsMat) / 4; ++k) v[k] = w[k];
    NsMat m;
    __builtin_memcpy(&m, v, sizeof m);
    return m;
}

// Four columns of row r of a d x p matrix (row stride ld), whatever its
// alignment; what lies past it is left alone (loads: zeros).  The pointers come from the table in
// memory, so the accesses name their address space: flat ones count with LDS (the
// last product of four GPT-2-large blocks took 388 us instead of 358).
template <typename T> using global_t = __attribute__((address_space(1))) T;
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef __bf16 bf16x4_any __attribute__((ext_vector_type(4), aligned(2)));
template <typename E> struct Vec4;
template <> struct Vec4<float> { typedef f32x4_any type; };
template <> struct Vec4<__bf16> { typedef bf16x4_any type; };

__device__ __forceinline__ void load4(const float* t, int r, int c, int d, int p, int ld, float v[4]) {
    const global_t<const float>* at = (const global_t<const float>*)(uintptr_t)(t + (size_t)r * ld + c);
    if (r < d && c + 4 <= p) {
        const f32x4_any w = *(const global_t<const f32x4_any>*)at;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = w[e];
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = r < d && c + e < p ? at[e] : 0.f;
    }
}
template <typename E>
__device__ __forceinline__ void store4(E* t, int r, int c, int d, int p, int ld, const float v[4]) {
    typedef typename Vec4<E>::type V;
    global_t<E>* at = (global_t<E>*)(uintptr_t)(t + (size_t)r * ld + c);
    V w;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = (E)v[e];
    if (r < d && c + 4 <= p) {
        *(global_t<V>*)at = w;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (r < d && c + e < p) at[e] = w[e];
    }
}

// Momentum, and the partial sums of U's squares (in float64: squares of any
// float32 stay in range).  One pass over G and M, bound by HBM: 5.4 TB/s over
// four GPT-2-large blocks (173 us).
__global__ __launch_bounds__(256) void ns_norm_kernel(const NsNormArgs args) {
    __shared__ double red[4];
    if (blockIdx.x == 0) {
        static_assert(sizeof(NsMat) % 4 == 0, "copied by words");
        const uint32_t* from = reinterpret_cast<const uint32_t*>(args.L);
        uint32_t* to = reinterpret_cast<uint32_t*>(args.table->L);
        for (int k = threadIdx.x; k < args.n * (int)sizeof(NsMat) / 4; k += 256) to[k] = from[k];
        if ((int)threadIdx.x < args.n) {
            const NsMat& t = args.L[threadIdx.x];
            args.table->prep[threadIdx.x] = t.prep_wg;
            args.table->sym[threadIdx.x] = t.sym_wg;
            args.table->apply[threadIdx.x] = t.apply_wg;
        }
    }
    int wg;
    const int l = find_matrix(args.n, blockIdx.x, wg, [&](int k) { return args.L[k].norm_wg; });
    const NsMat& L = args.L[l];
    const int64_t n = (int64_t)L.d * L.p, e0 = (int64_t)wg * L.norm_elems;
    double s = 0.0;
#pragma unroll 2
    for (int k = 0; k < L.norm_elems; k += 1024) {
        const int64_t e = e0 + k + threadIdx.x * 4;
        float g[4], m[4];
        if (e + 4 <= n) {
            __builtin_memcpy(g, L.G + e, 16);
            if (L.M) __builtin_memcpy(m, L.M + e, 16);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                g[j] = e + j < n ? L.G[e + j] : 0.f;
                m[j] = L.M && e + j < n ? L.M[e + j] : 0.f;
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (L.M) m[j] = fmaf(args.beta, m[j], g[j]);
            const double u = update_of(g[j], m[j], L.M != nullptr, args.nesterov, args.beta);
            s = fma(u, u, s);
        }
        if (L.M) {
            if (e + 4 <= n) {
                __builtin_memcpy(L.M + e, m, 16);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (e + j < n) L.M[e + j] = m[j];
            }
        }
    }
    s = block_sum_double(s, red);
    if (threadIdx.x == 0) args.part[L.part_off + wg] = s;
}

// X0 from U: one 64 x 64 tile of the padded X to a workgroup.  Reads G and M
// again: 4.6 TB/s over four GPT-2-large blocks (170 us).
template <bool SPLIT>
__global__ __launch_bounds__(256) void ns_prep_kernel(const NsArgs args) {
    __shared__ double red[4];
    __shared__ float tile[64][65];
    int wg;
    const int l = find_matrix(args.n, blockIdx.x, wg, [&](int k) { return args.table->prep[k]; });
    const NsMat L = load_matrix(args.table, l);
    const int tn = L.np / 64;
    const int i0 = wg / tn * 64, j0 = wg % tn * 64;
    const int npart = (int)(((int64_t)L.d * L.p + L.norm_elems - 1) / L.norm_elems);
    double sq = 0.0;
    for (int k = threadIdx.x; k < npart; k += 256) sq += args.part[L.part_off + k];
    const double inv = 1.0 / (sqrt(block_sum_double(sq, red)) + (double)args.eps);

    // Tile of U: rows r0 .., columns c0 .. of G.
    const int r0 = L.tall ? j0 : i0, c0 = L.tall ? i0 : j0;
    const int r = threadIdx.x >> 4, c = (threadIdx.x & 15) * 4;
#pragma unroll
    for (int k = 0; k < 64; k += 16) {
        const int row = r0 + r + k, col = c0 + c;
        float g[4], m[4] = {0.f, 0.f, 0.f, 0.f};
        load4(L.G, row, col, L.d, L.p, L.p, g);
        if (L.M) load4(L.M, row, col, L.d, L.p, L.p, m);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            // what lies past the matrix stays zero whatever the norm is
            const bool in = row < L.d && col + j < L.p;
            const float u = update_of(g[j], m[j], L.M != nullptr, args.nesterov, args.beta);
            const float v = in ? (float)((double)u * inv) * args.sx : 0.f;
            if (L.tall) tile[c + j][r + k] = v;
            else tile[r + k][c + j] = v;
        }
    }
    __syncthreads();
    char* X = args.ws + L.base;
#pragma unroll
    for (int k = 0; k < 64; k += 16) {
        f16x4_t h, q;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float v = tile[r + k][c + j];
            h[j] = (_Float16)v;
            if (SPLIT) q[j] = (_Float16)(v - (float)h[j]);
        }
        __builtin_memcpy(X + ns_at<SPLIT>(i0 + r + k, j0 + c, L.mp), &h, 8);
        if (SPLIT) __builtin_memcpy(X + ns_at<SPLIT>(i0 + r + k, j0 + c, L.mp, 1), &q, 8);
    }
}

// ---------------------------------------------------------------------------
// The products: a TM x TN tile to a workgroup, NX x NY accumulators of 32x32x16
// MFMAs to a wave.  Both operands come by LDS DMA in stages of 32 k (SPLIT: of
// both parts of 16 k) through a ring of three or four buffers.
//
// An operand whose rows run along k is staged as its 64-byte rows, the 16-byte
// piece c of row r at c ^ row_swz(r): the rows that are read together then lie
// on distinct banks.  Apply's X has k as its slow index: blocks of 32 columns,
// 32 rows of 64 bytes each, gathered by the transposing LDS read
// (ds_read_b64_tr_b16), whose 4 rows of 32 columns are 256 bytes in a row.
// SPLIT: blocks of 16 columns, 16 rows each; the halves of an odd block's rows
// are swapped, so that one part of two blocks covers the banks as well.
//
// The MFMA's first operand is the tile's columns: a lane then holds four
// consecutive columns of one row, lane % 32.
//
// A stage is two MFMA steps of 16 k, or three of SPLIT's products.  The
// fragments of a step are read while the step before it multiplies, so that a
// wave's matrix instructions wait for its LDS reads only in the first step.
//
// What it reaches on four GPT-2-large blocks (16 matrices of 1280 rows): X 205 us,
// 980 TFLOP/s; A 126 us, 960 of the tiles that it computes; Bm, with a fifth of
// the work, 49 us; a library's largest fp16 products run at 1140 on this card,
// which is bound by the clock under random data.  With few tiles a launch's fixed
// 4 to 5 us and the latency of a stage take over: one 768 x 768 product takes 6.8
// us, one 333 x 333 5.0.
// ---------------------------------------------------------------------------
constexpr int kBK = 32;

// A 16-byte LDS read serves 16 lanes at a time, not 16 in a row: lanes 0-3,
// 12-15, 20-23 and 24-27 together, then the others of 32 (the counters show
// twice the cycles for a swizzle that is free of conflicts over lanes 0-15 and
// 16-31 alone).  For quads q = r / 4 of rows, q, or 3 - q in the upper half,
// differs over 0, 3, 5, 6 and over 1, 2, 4, 7, and over runs of four too.
__device__ __forceinline__ int row_swz(int r) { return ((r >> 2) ^ -((r >> 4) & 1)) & 3; }

__device__ __forceinline__ uint4 frag_rows(const char* lds, int r0, int kk, int lane) {
    const int r = r0 + (lane & 31), c = 2 * kk + (lane >> 5);
    return *reinterpret_cast<const uint4*>(lds + r * 64 + (c ^ row_swz(r)) * 16);
}
__device__ __forceinline__ uint4 frag_cols(const char* lds, int c0, int kk, int lane) {
    const int grp = lane >> 4, i = lane & 15;
    const char* p = lds + (c0 >> 5) * (kBK * 64) + (16 * kk + 8 * (grp >> 1) + (i >> 2)) * 64 + 32 * (grp & 1) + 8 * (i & 3);
    uint2 h[2];
#pragma unroll
    for (int k = 0; k < 2; ++k)
        h[k] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                             (__attribute__((address_space(3))) v4i16*)(p + 256 * k)));
    return make_uint4(h[0].x, h[0].y, h[1].x, h[1].y);
}
// Part z of 32 columns in two blocks of SPLIT's.
__device__ __forceinline__ uint4 frag_split_cols(const char* lds, int c0, int z, int lane) {
    const int grp = lane >> 4, i = lane & 15, odd = grp & 1;
    const char* p = lds + ((c0 >> 4) + odd) * 1024 + (8 * (grp >> 1) + (i >> 2)) * 64 + 32 * (z ^ odd) + 8 * (i & 3);
    uint2 h[2];
#pragma unroll
    for (int k = 0; k < 2; ++k)
        h[k] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                             (__attribute__((address_space(3))) v4i16*)(p + 256 * k)));
    return make_uint4(h[0].x, h[0].y, h[1].x, h[1].y);
}

// A 32 x 32 block of a 16-bit matrix as an accumulator holds it: two pieces of 8
// columns of one row to a lane, columns 16 k + 8 (lane / 32) + 0 .. 7.  The
// accumulator's lanes l and l + 32 hold 4 columns each of every 8, and swap
// halves of their words.  next: bytes from a row's first 16 columns to the others.
struct Rows16 {
    uint4 p[2];
};
__device__ __forceinline__ Rows16 load_rows16(const char* block, int row, int hi, size_t next) {
    Rows16 r;
#pragma unroll
    for (int k = 0; k < 2; ++k) r.p[k] = *reinterpret_cast<const uint4*>(block + row * 64 + k * next + 16 * hi);
    return r;
}
__device__ __forceinline__ void store_rows16(char* block, int row, int hi, size_t next, const Rows16& r) {
#pragma unroll
    for (int k = 0; k < 2; ++k) *reinterpret_cast<uint4*>(block + row * 64 + k * next + 16 * hi) = r.p[k];
}
__device__ __forceinline__ void swap_halves(uint32_t& a, uint32_t& b) {
    const auto r = __builtin_amdgcn_permlane32_swap(a, b, false, false);
    a = r[0];
    b = r[1];
}
// Values v[16] of the lane's accumulator element order to S parts, and back.
template <int S>
__device__ __forceinline__ void pack_rows16(const float v[16], Rows16 out[S]) {
#pragma unroll
    for (int z = 0; z < S; ++z)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                _Float16 h[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float x = v[8 * k + 2 * j + e];
                    h[e] = (_Float16)x;
                    if (z == 1) h[e] = (_Float16)(x - (float)h[e]);
                }
                __builtin_memcpy(&w[j], h, 4);
            }
            swap_halves(w[0], w[2]);
            swap_halves(w[1], w[3]);
            out[z].p[k] = make_uint4(w[0], w[1], w[2], w[3]);
        }
}
template <int S>
__device__ __forceinline__ void unpack_rows16(const Rows16 in[S], float v[16]) {
#pragma unroll
    for (int z = 0; z < S; ++z)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            uint32_t w[4] = {in[z].p[k].x, in[z].p[k].y, in[z].p[k].z, in[z].p[k].w};
            swap_halves(w[0], w[2]);
            swap_halves(w[1], w[3]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                _Float16 h[2];
                __builtin_memcpy(h, &w[j], 4);
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float& x = v[8 * k + 2 * j + e];
                    x = z == 0 ? (float)h[e] : x + (float)h[e];
                }
            }
        }
}

// One wave's LDS accesses are done in order; this keeps the compiler from
// moving them past each other where lanes read what other lanes wrote.
__device__ __forceinline__ void lds_settle() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// Tile shapes (NsTile): 256 x 256 with eight waves of 128 x 64, one workgroup to
// a CU; 256 x 128 with four of them, and 128 x 128 with four of 64 x 64, two to a
// CU; 64 x 64 with four of 32 x 32.  NB: stages in the ring; KB: blocks of k in a
// stage (SPLIT: one), two where a block has only one MFMA to a wave and step, and
// barriers and LDS latency are most of a stage (SPLIT's have three).
template <NsTile TILE> struct NsCfg;
template <> struct NsCfg<NsTile::T256> {
    static constexpr int TM = 256, TN = 256, WN = 4, waves = 8, NX = 4, NY = 2, NB = 4, KB = 1;
};
template <> struct NsCfg<NsTile::T256x128> {
    static constexpr int TM = 256, TN = 128, WN = 2, waves = 4, NX = 4, NY = 2, NB = 3, KB = 1;
};
template <> struct NsCfg<NsTile::T128> {
    static constexpr int TM = 128, TN = 128, WN = 2, waves = 4, NX = 2, NY = 2, NB = 4, KB = 1;
};
template <> struct NsCfg<NsTile::T64> {
    static constexpr int TM = 64, TN = 64, WN = 2, waves = 4, NX = 1, NY = 1, NB = 4, KB = 2;
};

template <NsOp OP, bool SPLIT, NsTile TILE>
__global__ __launch_bounds__(64 * NsCfg<TILE>::waves, 2) void ns_gemm_kernel(const NsArgs args) {
    using Cfg = NsCfg<TILE>;
    constexpr bool SYM = OP == NsOp::Gram || OP == NsOp::Poly;
    constexpr bool COLS = !SYM;          // the second operand has k as its slow index
    constexpr int TM = Cfg::TM, TN = Cfg::TN, NX = Cfg::NX, NY = Cfg::NY, NB = Cfg::NB;
    constexpr int KB = SPLIT ? 1 : Cfg::KB;
    constexpr int opA_bytes = KB * TM * 64, stage_bytes = KB * (TM + TN) * 64;
    constexpr int DA = KB * TM / 16 / Cfg::waves, DB = KB * TN / 16 / Cfg::waves;     // DMA instructions of a wave and stage
    static_assert(KB == 1 || (TM == kNsPad && TN == kNsPad), "no rows past the matrix, which would be the next block's");
    __shared__ __attribute__((aligned(16))) char lds[NB * stage_bytes];
    // Workgroups go to the 8 XCDs in turn; each XCD has a run of all tiles.
    const int xcd = blockIdx.x & 7, tile = args.xcd[xcd] + (int)(blockIdx.x >> 3);
    if (tile >= args.xcd[xcd + 1]) return;
    int wg;
    const int l = find_matrix(args.n, tile, wg, [&](int k) { return SYM ? args.table->sym[k] : args.table->apply[k]; });
    const NsMat L = load_matrix(args.table, l);
    const int mp = L.mp, np = L.np;
    int mt, nt;
    if constexpr (SYM) {
        // Tiles on and above the diagonal, a column of them after the other:
        // column nt has nt / R + 1, R being TM / TN.
        constexpr int R = TM / TN;
        nt = 0;
        for (mt = wg; mt > nt / R; ++nt) mt -= nt / R + 1;
    } else {
        const int tm = (mp + TM - 1) / TM;
        nt = wg / tm;
        mt = wg - nt * tm;
    }
    const int m0 = mt * TM, n0 = nt * TN;

    constexpr int S = SPLIT ? 2 : 1;
    const size_t xb = (size_t)mp * np * 2, ab = (size_t)mp * mp * 2;
    char* X = args.ws + L.base + (args.from ? S * xb : 0);
    char* Xn = args.ws + L.base + (args.from ? 0 : S * xb);
    char* A = args.ws + L.base + 2 * S * xb;
    char* Bm = A + S * ab;
    const char* opA = OP == NsOp::Gram ? X : OP == NsOp::Poly ? A : Bm;      // rows m0 .. along k
    const char* opB = OP == NsOp::Poly ? A : X;                              // the tile's columns
    const int K = OP == NsOp::Gram ? np : mp;

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / Cfg::WN, wn = wave % Cfg::WN;

    // DMA: a block of an operand's stage is T / 16 instructions of 1 KB; wave w
    // issues numbers w + waves i of each operand.  Rows past the matrix are out
    // of the resource's range, columns past it get kOut.
    constexpr int SK = SPLIT ? kBK / 2 : kBK;         // columns of a block, and k of a stage's blocks
    const uint32_t block = (uint32_t)mp * 64u;        // bytes of a block
    auto row_off = [&](int q) {
        const int r = 16 * q + (lane >> 2), c = (lane & 3) ^ row_swz(r);
        return (uint32_t)(r * 64 + c * 16);
    };
    uint32_t offA[DA], offB[DB];
#pragma unroll
    for (int i = 0; i < DA; ++i) {
        const int q = wave + Cfg::waves * i;
        offA[i] = row_off(q % (TM / 16)) + q / (TM / 16) * block;
    }
#pragma unroll
    for (int i = 0; i < DB; ++i) {
        const int q = (wave + Cfg::waves * i) % (TN / 16), kb = (wave + Cfg::waves * i) / (TN / 16);
        if constexpr (COLS && SPLIT)      // 16 rows of a block of 16 columns
            offB[i] = n0 + 16 * q < np ? q * block + kb * 1024 + (lane >> 2) * 64 + ((lane & 3) ^ 2 * (q & 1)) * 16 : kOut;
        else if constexpr (COLS)          // 16 rows of a block of 32 columns
            offB[i] = n0 + 16 * (q & ~1) < np ? (q >> 1) * block + kb * 2048 + (q & 1) * 1024 + lane * 16 : kOut;
        else
            offB[i] = row_off(q) + kb * block;
    }
    const int nst = K / (SK * KB);
    const uint32_t bytesA = (KB - 1) * block + (uint32_t)min(TM, mp - m0) * 64u;
    const uint32_t bytesB = COLS ? (uint32_t)(min(TN, np - n0) / SK - 1) * block + KB * SK * 64u
                                 : (KB - 1) * block + (uint32_t)min(TN, mp - n0) * 64u;
    const char* baseA = opA + (size_t)m0 * 64;
    const char* baseB = COLS ? opB + (size_t)(n0 / SK) * block : opB + (size_t)n0 * 64;
    // Stage st into the buffer at `buf`; stages past the last one load zeros.
    struct Dma {
        u32x4_t a, b;
        char* buf;
    };
    auto dma_of = [&](int st, char* buf) {
        const bool on = st < nst;
        const char* a = baseA + (size_t)(st * KB) * block;
        const char* b = baseB + (size_t)(st * KB) * (COLS ? SK * 64u : block);
        return Dma{raw_rsrc(a, on ? bytesA : 0u), raw_rsrc(b, on ? bytesB : 0u), buf};
    };
    auto dma_piece = [&](const Dma& d, int i) {
        if (i < DA) dma16_asm(d.a, offA[i], d.buf + (wave + Cfg::waves * i) * 1024);
        else dma16_asm(d.b, offB[i - DA], d.buf + opA_bytes + (wave + Cfg::waves * (i - DA)) * 1024);
    };

    f32x16_t acc[NX][NY];
#pragma unroll
    for (int x = 0; x < NX; ++x)
#pragma unroll
        for (int y = 0; y < NY; ++y)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[x][y][i] = 0.f;

    struct Frags {
        uint4 a[NX], b[NY];
    };
    // Step k of a stage: half (SPLIT: part) k % 2 of block k / 2.
    constexpr int STEPS = 2 * KB;
    auto read = [&](Frags& f, const char* P, int k) {
        const char* Q = P + opA_bytes + (k >> 1) * (TN * 64);
        P += (k >> 1) * (TM * 64);
#pragma unroll
        for (int y = 0; y < NY; ++y)
            f.b[y] = !COLS ? frag_rows(Q, 32 * NY * wn + 32 * y, k & 1, lane)
                     : SPLIT ? frag_split_cols(Q, 32 * NY * wn + 32 * y, k & 1, lane)
                             : frag_cols(Q, 32 * NY * wn + 32 * y, k & 1, lane);
#pragma unroll
        for (int x = 0; x < NX; ++x) f.a[x] = frag_rows(P, 32 * NX * wm + 32 * x, k & 1, lane);
    };
    // A step's MFMAs, `between(k)` behind the k-th of them.
    auto multiply = [&](const Frags& fa, const Frags& fb, auto between) {
#pragma unroll
        for (int x = 0; x < NX; ++x)
#pragma unroll
            for (int y = 0; y < NY; ++y) {
                acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, fb.b[y]),
                                                                   __builtin_bit_cast(f16x8_t, fa.a[x]), acc[x][y], 0, 0, 0);
                between(NY * x + y);
            }
    };
    // The wave's own DMA of the next stage is done, then everyone's.
    auto publish = [&]() {
        wait_vmcnt<(NB - 2) * (DA + DB)>();
        __builtin_amdgcn_sched_barrier(0);
        lds_barrier();
        __builtin_amdgcn_sched_barrier(0);
    };
#pragma unroll
    for (int b = 0; b < NB - 1; ++b) {
        const Dma d = dma_of(b, lds + b * stage_bytes);
#pragma unroll
        for (int i = 0; i < DA + DB; ++i) dma_piece(d, i);
    }
    Frags f0, f2, rest[STEPS - 1];
    publish();
    char *cur = lds, *fill = lds + (NB - 1) * stage_bytes;     // the stage's buffer, and the one before it
    read(f0, cur, 0);
    // On entry `first` holds the stage's first fragments, on return `next` the
    // following stage's.  The buffer that the DMA refills was last read in the
    // stage before, whose reads every wave had finished at the barrier inside
    // that stage (the wait for LDS reads there).
    auto stage = [&](int st, Frags& first, Frags& next) {
        constexpr int PER = (DA + DB + NX * NY - 1) / (NX * NY);      // DMA instructions behind an MFMA
#pragma unroll
        for (int k = 1; k < STEPS; ++k) read(rest[k - 1], cur, k);
        const Dma d = dma_of(st + NB - 1, fill);
        __builtin_amdgcn_sched_barrier(0);
        // The DMA among the MFMAs: issued together, its instructions hold the
        // wave up until the address unit has taken them all.
        multiply(first, first, [&](int k) {
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = PER * k; i < min(PER * (k + 1), DA + DB); ++i) dma_piece(d, i);
            __builtin_amdgcn_sched_barrier(0);
        });
        const auto nothing = [](int) {};
        if constexpr (SPLIT) {
            multiply(first, rest[0], nothing);
        } else {
#pragma unroll
            for (int k = 1; k < STEPS - 1; ++k) multiply(rest[k - 1], rest[k - 1], nothing);
        }
        publish();
        fill = cur;
        cur = cur == lds + (NB - 1) * stage_bytes ? lds : cur + stage_bytes;
        read(next, cur, 0);
        __builtin_amdgcn_sched_barrier(0);
        const Frags& last = rest[STEPS - 2];
        multiply(last, SPLIT ? first : last, nothing);
    };
    if constexpr (SPLIT) {
        for (int st = 0; st < nst; st += 2) {       // K is a multiple of kNsPad
            static_assert(kNsPad % (2 * SK * KB) == 0, "whole pairs of stages");
            stage(st, f0, f2);
            stage(st + 1, f2, f0);
        }
    } else {
        for (int st = 0; st < nst; ++st) stage(st, f0, f0);
    }
#pragma unroll
    for (int x = 0; x < NX; ++x) mfma_settle<NY>(acc[x]);
    // The zero stages behind the last one have landed and every wave has read
    // its last fragments: the ring is free for the epilogue, an equal part of
    // it for each wave.
    wait_vmcnt<0>();
    lds_barrier();

    // Epilogue, one 32 x 32 block after the other: a lane holds row lane % 32,
    // columns 8 q + 4 (lane / 32) + 0 .. 3 for q in 0 .. 3.
    constexpr int wave_lds = NB * stage_bytes / Cfg::waves;
    char* mine = lds + wave * wave_lds;
    const int row = lane & 31, hi = lane >> 5;
    const int i0 = m0 + 32 * NX * wm, j0 = n0 + 32 * NY * wn;      // the wave's rows and columns
    if constexpr (OP != NsOp::Final) {
        char* C = OP == NsOp::Gram ? A : OP == NsOp::Poly ? Bm : Xn;
        const size_t next = ns_next16<SPLIT>(mp);
        const int cols = SYM ? mp : np;
        // v = f acc, for Poly + g A + a on the diagonal
        const float f = OP == NsOp::Gram ? args.sa / (args.sx * args.sx)
                        : OP == NsOp::Poly ? args.c * (args.sb / (args.sa * args.sa)) : args.sx2 / (args.sb * args.sx);
        const float g = args.b * (args.sb / args.sa), diag = args.a * args.sb;
        const bool mirror = SYM && nt / (TM / TN) != mt;      // blocks on the diagonal are whole
#pragma unroll
        for (int x = 0; x < NX; ++x) {
            const int ib = i0 + 32 * x;
            if (ib >= mp) break;
            Rows16 old[NY][S];
            if constexpr (OP == NsOp::Poly) {
#pragma unroll
                for (int y = 0; y < NY; ++y)
                    if (j0 + 32 * y < cols)
#pragma unroll
                        for (int z = 0; z < S; ++z) old[y][z] = load_rows16(A + ns_at<SPLIT>(ib, j0 + 32 * y, mp, z), row, hi, next);
            }
#pragma unroll
            for (int y = 0; y < NY; ++y) {
                const int jb = j0 + 32 * y;
                if (jb >= cols) break;
                float v[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) v[e] = acc[x][y][e] * f;
                if constexpr (OP == NsOp::Poly) {
                    float o[16];
                    unpack_rows16<S>(old[y], o);
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        v[e] = fmaf(o[e], g, v[e]);
                        if (ib + row == jb + acc_row(e, lane)) v[e] += diag;
                    }
                }
                Rows16 out[S];
                pack_rows16<S>(v, out);
#pragma unroll
                for (int z = 0; z < S; ++z) {
                    store_rows16(C + ns_at<SPLIT>(ib, jb, mp, z), row, hi, next, out[z]);
                    if (!mirror) continue;
                    // The block's transpose by way of LDS: written by rows,
                    // read by the transposing read.
                    char* t = mine + 2048 * z;
                    store_rows16(t, row, hi, 32, out[z]);
                    lds_settle();
                    const Rows16 tr = {frag_cols(t, 0, 0, lane), frag_cols(t, 0, 1, lane)};
                    store_rows16(C + ns_at<SPLIT>(jb, ib, mp, z), row, hi, next, tr);
                    lds_settle();
                }
            }
        }
    } else {
        // O and the weights: blocks of 32 rows by the wave's columns (of O
        // transposed if U is tall) pass through LDS in float32, so that a
        // lane's 16 bytes lie beside its neighbours' in whole rows.
        constexpr int NC = 32 * NY;
        constexpr int LDW = NC + 4, LDT = 36;                // floats of an LDS row, wide and tall
        static_assert(32 * LDW * 4 <= wave_lds && NC * LDT * 4 <= wave_lds, "LDS part of a wave");
        float* buf = reinterpret_cast<float*>(mine);
        const float f = 1.0f / (args.sb * args.sx);
        const bool tall = L.tall != 0;
        static_assert(NC == 64 || NC == 32, "pieces of a row");
        const int lg = tall || NC == 32 ? 3 : 4, per = 1 << lg, ld = tall ? LDT : LDW;
        constexpr int N = NC * 32 / 4 / 64;              // pieces of a lane
#pragma unroll
        for (int x = 0; x < NX; ++x) {
            const int ib = i0 + 32 * x;
            if (ib >= mp) break;
            // Rows of O: r0 + .., each `per` pieces of four columns from c0 on.
            const int r0 = tall ? j0 : ib, c0 = tall ? ib : j0;
            const auto at = [&](int k, int& r, int& c) {
                const int piece = k * 64 + lane;
                r = piece >> lg, c = (piece & (per - 1)) * 4;
            };
            // The weights are on their way while the block passes LDS.
            float w[N][4];
            if (L.W)
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    int r, c;
                    at(k, r, c);
                    load4(L.W, r0 + r, c0 + c, L.d, L.p, L.p, w[k]);
                }
#pragma unroll
            for (int y = 0; y < NY; ++y) {
                if (j0 + 32 * y >= np) break;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float v[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = acc[x][y][4 * q + e] * f;
                    const int c = 32 * y + 8 * q + 4 * hi;
                    if (tall) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) buf[(c + e) * LDT + row] = v[e];
                    } else {
                        __builtin_memcpy(buf + row * LDW + c, v, 16);
                    }
                }
            }
            lds_settle();
#pragma unroll
            for (int k = 0; k < N; ++k) {
                int r, c;
                at(k, r, c);
                float v[4];
                __builtin_memcpy(v, buf + r * ld + c, 16);
                if (L.O) {
                    if (L.o_bf16) store4(static_cast<__bf16*>(L.O), r0 + r, c0 + c, L.d, L.p, L.p, v);
                    else store4(static_cast<float*>(L.O), r0 + r, c0 + c, L.d, L.p, L.p, v);
                }
                if (L.W) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[k][e] = fmaf(-L.step, v[e], args.keep * w[k][e]);
                    store4(L.W, r0 + r, c0 + c, L.d, L.p, L.p, w[k]);
                    if (L.Wb) store4(reinterpret_cast<__bf16*>(L.Wb), r0 + r, c0 + c, L.d, L.p, L.p, w[k]);
                }
            }
            lds_settle();
        }
    }
}

// ---------------------------------------------------------------------------
// Small matrices (ns_is_small): a workgroup to a matrix, the whole step in one
// launch.  X, A and Bm stay in LDS in float32, and the products run on the
// float32 matrix instructions (16x16x4): next to the launches that it saves
// (three products a step, each a launch of 4 us or more) their lower rate is
// nothing, and nothing is rounded to 16 bits.  G, M and W pass memory once.  One
// 64 x 96 takes 34 us (6.5 a step: the latency of three dependent products in one
// CU), the general path 105; the Muon step of 48 LoRA factors 768 x 16 25 us and
// 316.
//
// 16x16x4 MFMA: lane l holds row l % 16 of the first operand and column l % 16
// of the second, k = l / 16; of the result column l % 16, rows 4 (l / 16) + 0 .. 3.
// ---------------------------------------------------------------------------
typedef float f32x4_t __attribute__((ext_vector_type(4)));
constexpr int kSmallWaves = 8, kSmallThreads = 64 * kSmallWaves;

// Elements of a small matrix in memory order, four to a thread and turn:
// f(e, count) for each run of 4 (fewer at the end).
template <typename F>
__device__ __forceinline__ void small_runs(int n, F f) {
    for (int e = threadIdx.x * 4; e < n; e += kSmallThreads * 4) f(e, min(4, n - e));
}

// Wait states between the last MFMA and a read of its result (8 passes).
__device__ __forceinline__ void settle4(f32x4_t& a) {
    asm volatile("" : "+v"(a));
    asm volatile("s_nop 15");
    asm volatile("" : "+v"(a));
}

// Tile t of the MT (MT + 1) / 2 on and above the diagonal.
__device__ __forceinline__ void sym_tile(int t, int& ti, int& tj) {
    tj = 0;
    for (ti = t; ti > tj; ++tj) ti -= tj + 1;
}

// X <- Bm X for nt column tiles of 16, a tile to a wave: it reads and writes
// those columns only.
template <int MT, int WAVES>
__device__ __forceinline__ void ns_apply_columns(float* X, const float* Bm, int lda, int nt, int ldx) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, q = lane >> 4;
    f32x4_t f[MT][MT];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int k = 0; k < MT; ++k) f[i][k] = *reinterpret_cast<const f32x4_t*>(Bm + (16 * i + r) * lda + 16 * k + 4 * q);
    for (int t = wave; t < nt; t += WAVES) {
        float* x = X + 16 * t + r;
        f32x4_t acc[MT], v[MT];
#pragma unroll
        for (int k = 0; k < MT; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[k][e] = x[(16 * k + 4 * q + e) * ldx];
#pragma unroll
        for (int i = 0; i < MT; ++i) acc[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < MT; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int i = 0; i < MT; ++i)
                    acc[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(f[i][k][e], v[k][e], acc[i], 0, 0, 0);
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            settle4(acc[i]);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[(16 * i + 4 * q + e) * ldx] = acc[i][e];
        }
    }
}

// MT: row tiles of 16.
template <int MT>
__device__ __forceinline__ void ns_small_steps(const NsSmallArgs& args, float* X, float* A, float* Bm, float* red, int nt,
                                               int ldx) {
    constexpr int lda = 16 * MT + 4;
    // k slices of a tile of A; with more tiles, A and Bm are computed on and above
    // the diagonal and mirrored (one 64 x 96: 37.0 -> 33.9 us).
    constexpr int SL = MT == 1 ? 8 : MT == 2 ? 2 : 1, TILES = SL > 1 ? MT * MT : MT * (MT + 1) / 2;
    const auto tile_of = [](int t, int& ti, int& tj) {
        if constexpr (SL > 1) ti = t / MT, tj = t - ti * MT;
        else sym_tile(t, ti, tj);
    };
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, q = lane >> 4;
    for (int s = 0; s < args.steps; ++s) {
        // A = X X^T: (tile, slice) pairs over the waves.
        for (int t = wave; t < TILES * SL; t += kSmallWaves) {
            const int tile = t / SL, sl = t - tile * SL;
            int ti, tj;
            tile_of(tile, ti, tj);
            const float* a = X + (16 * ti + r) * ldx + 4 * q;
            const float* b = X + (16 * tj + r) * ldx + 4 * q;
            f32x4_t acc = {0.f, 0.f, 0.f, 0.f}, acc2 = acc;
            for (int k = sl; k < nt; k += SL) {
                const f32x4_t u = *reinterpret_cast<const f32x4_t*>(a + 16 * k);
                const f32x4_t v = *reinterpret_cast<const f32x4_t*>(b + 16 * k);
                acc = __builtin_amdgcn_mfma_f32_16x16x4f32(u[0], v[0], acc, 0, 0, 0);
                acc2 = __builtin_amdgcn_mfma_f32_16x16x4f32(u[1], v[1], acc2, 0, 0, 0);
                acc = __builtin_amdgcn_mfma_f32_16x16x4f32(u[2], v[2], acc, 0, 0, 0);
                acc2 = __builtin_amdgcn_mfma_f32_16x16x4f32(u[3], v[3], acc2, 0, 0, 0);
            }
            settle4(acc);
            settle4(acc2);
            acc += acc2;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (SL == 1) A[(16 * ti + 4 * q + e) * lda + 16 * tj + r] = acc[e];
                else red[t * 256 + (4 * q + e) * 16 + r] = acc[e];
            }
            if (SL == 1 && ti != tj) *reinterpret_cast<f32x4_t*>(A + (16 * tj + r) * lda + 16 * ti + 4 * q) = acc;
        }
        __syncthreads();
        if constexpr (SL > 1) {
            for (int e = threadIdx.x; e < MT * MT * 256; e += kSmallThreads) {
                const int tile = e >> 8, in = e & 255;
                float v = 0.f;
#pragma unroll
                for (int k = 0; k < SL; ++k) v += red[(tile * SL + k) * 256 + in];
                A[(16 * (tile / MT) + (in >> 4)) * lda + 16 * (tile % MT) + (in & 15)] = v;
            }
            __syncthreads();
        }
        // Bm = a I + b A + c A^2 (A is symmetric).
        const float ca = args.coef[3 * s], cb = args.coef[3 * s + 1], cc = args.coef[3 * s + 2];
        for (int t = wave; t < TILES; t += kSmallWaves) {
            int ti, tj;
            tile_of(t, ti, tj);
            f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < MT; ++k) {
                const f32x4_t u = *reinterpret_cast<const f32x4_t*>(A + (16 * ti + r) * lda + 16 * k + 4 * q);
                const f32x4_t v = *reinterpret_cast<const f32x4_t*>(A + (16 * tj + r) * lda + 16 * k + 4 * q);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(u[e], v[e], acc, 0, 0, 0);
            }
            settle4(acc);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = 16 * ti + 4 * q + e, j = 16 * tj + r;
                acc[e] = fmaf(cc, acc[e], cb * A[i * lda + j]) + (i == j ? ca : 0.f);
                Bm[i * lda + j] = acc[e];
            }
            if (SL == 1 && ti != tj) *reinterpret_cast<f32x4_t*>(Bm + (16 * tj + r) * lda + 16 * ti + 4 * q) = acc;
        }
        __syncthreads();
        ns_apply_columns<MT, kSmallWaves>(X, Bm, lda, nt, ldx);
        __syncthreads();
    }
}

__global__ __launch_bounds__(kSmallThreads) void ns_small_kernel(const NsSmallArgs args) {
    __shared__ __attribute__((aligned(16))) float X[kNsSmallFloats];
    __shared__ __attribute__((aligned(16))) float A[64 * 68];
    __shared__ __attribute__((aligned(16))) float Bm[64 * 68];
    __shared__ float red[8 * 256];
    __shared__ double dred[kSmallWaves];
    const NsSmallMat& L = args.L[blockIdx.x];
    const int p = L.p, n = L.d * p;
    const bool tall = L.d > p;
    const int m = tall ? p : L.d, nn = tall ? L.d : p;
    const int nt = (nn + 15) / 16, ldx = (int)ns_small_ld(nn), mt = (m + 15) / 16;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // Place of element e = r p + c of U in X.
    auto place = [&](int r, int c) { return tall ? c * ldx + r : r * ldx + c; };

    for (int e = threadIdx.x * 4; e < mt * 16 * ldx; e += kSmallThreads * 4)
        *reinterpret_cast<float4*>(X + e) = make_float4(0.f, 0.f, 0.f, 0.f);
    __syncthreads();
    double sq = 0.0;
    small_runs(n, [&](int e, int count) {
        float g[4] = {0.f, 0.f, 0.f, 0.f}, mm[4] = {0.f, 0.f, 0.f, 0.f};
        if (count == 4) {
            __builtin_memcpy(g, L.G + e, 16);
            if (L.M) __builtin_memcpy(mm, L.M + e, 16);
        } else {
#pragma unroll
            for (int k = 0; k < 3; ++k)
                if (k < count) {
                    g[k] = L.G[e + k];
                    if (L.M) mm[k] = L.M[e + k];
                }
        }
        int r = e / p, c = e - r * p;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (L.M) mm[k] = fmaf(args.beta, mm[k], g[k]);
            const float u = update_of(g[k], mm[k], L.M != nullptr, args.nesterov, args.beta);
            if (k < count) X[place(r, c)] = u;
            sq = fma((double)u, (double)u, sq);
            if (++c == p) c = 0, ++r;
        }
        if (L.M) {
            if (count == 4) {
                __builtin_memcpy(L.M + e, mm, 16);
            } else {
#pragma unroll
                for (int k = 0; k < 3; ++k)
                    if (k < count) L.M[e + k] = mm[k];
            }
        }
    });
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) sq += __shfl_xor(sq, off, 64);
    if (lane == 0) dred[wave] = sq;
    __syncthreads();
    sq = 0.0;
#pragma unroll
    for (int w = 0; w < kSmallWaves; ++w) sq += dred[w];
    const double inv = 1.0 / (sqrt(sq) + (double)args.eps);
    for (int r = wave; r < m; r += kSmallWaves)
        for (int c = lane; c < nn; c += 64) X[r * ldx + c] = (float)((double)X[r * ldx + c] * inv);
    __syncthreads();
    switch (mt) {
        case 1: ns_small_steps<1>(args, X, A, Bm, red, nt, ldx); break;
        case 2: ns_small_steps<2>(args, X, A, Bm, red, nt, ldx); break;
        case 3: ns_small_steps<3>(args, X, A, Bm, red, nt, ldx); break;
        default: ns_small_steps<4>(args, X, A, Bm, red, nt, ldx); break;
    }
    small_runs(n, [&](int e, int count) {
        float v[4], w[4] = {0.f, 0.f, 0.f, 0.f};
        int r = e / p, c = e - r * p;
        if (L.W) {
            if (count == 4) {
                __builtin_memcpy(w, L.W + e, 16);
            } else {
#pragma unroll
                for (int k = 0; k < 3; ++k)
                    if (k < count) w[k] = L.W[e + k];
            }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            v[k] = k < count ? X[place(r, c)] : 0.f;
            if (++c == p) c = 0, ++r;
        }
        auto put = [&](auto* out, const float* x) {
            using E = std::remove_reference_t<decltype(*out)>;
            E t[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) t[k] = (E)x[k];
            if (count == 4) {
                __builtin_memcpy(out + e, t, sizeof t);
            } else {
#pragma unroll
                for (int k = 0; k < 3; ++k)
                    if (k < count) out[e + k] = t[k];
            }
        };
        if (L.O) {
            if (L.o_bf16) put(static_cast<__bf16*>(L.O), v);
            else put(static_cast<float*>(L.O), v);
        }
        if (L.W) {
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = fmaf(-L.step, v[k], args.keep * w[k]);
            put(L.W, w);
            if (L.Wb) put(reinterpret_cast<__bf16*>(L.Wb), w);
        }
    });
}

// ---------------------------------------------------------------------------
// Thin matrices: m <= 64 rows of X, n of any length.  The polynomials of several
// steps (a round) are those of one m x m matrix, A = X X^T / |X|^2, so X is needed
// twice only: for A, and to be multiplied by the product P of the round's Bm,
//   per step  Bm = a I + b A + c A^2,  P <- Bm P,  A <- Bm A Bm.
// The square root of A's rounding error is what small singular values are lost
// in, and they grow 485-fold in five usual steps: in float32 this form loses
// them, in float64 (2^-53 against 485^-2 = 2^-18) it is as good as float32
// products of X itself.  Where further steps would lose that again (the rule is
// the host's), another round begins with the Gram matrix of P X.  P X is not kept:
// each launch multiplies the chunk that it has loaded by the P of all rounds so
// far, which costs the usual one round nothing, and many no memory of X's size.
// Next to 3 launches for each step of the general path: 3 in all for one round,
// two more for each other, and G and M pass memory once a launch over chunks.
// Kernel times: one 16 x 4096 20 us, 24 of them 32, one 48 x 3000 63, one 64 x 3000
// 107 (of them 60 in the polynomials' one workgroup; 10 steps 207, 20 steps 429),
// 24 of them 126; the general path takes 115 for one 65 x 3000 and 172 for 24, in
// the float32-accurate form 210 and 288.
// ---------------------------------------------------------------------------
constexpr int kThinThreads = 256;
constexpr int kThinLds = kNsThinFloats + 64 * 4;      // floats: 16 MT rows of a tile's columns and four more

// Columns of X in LDS at a time, of 16 MT rows.
template <int MT>
constexpr int thin_cols() {
    constexpr int cols = (int)ns_thin_tile(16 * MT);
    static_assert(cols >= 16 && cols % 16 == 0 && 16 * MT * (cols + 4) <= kThinLds, "a tile in LDS");
    return cols;
}

// f(r, c) for runs of four columns (of a row of U) that cover columns j0 ..
// j0 + cols of X, one run to a thread and turn: U's columns, or, tall, its rows.
template <typename F>
__device__ __forceinline__ void thin_runs(const NsSmallMat& L, int j0, int cols, F f) {
    const bool tall = L.d > L.p;
    const int rows = tall ? min(cols, L.d - j0) : L.d, width = tall ? L.p : min(cols, L.p - j0);
    const int per = (width + 3) >> 2;
    for (int k = threadIdx.x; k < rows * per; k += kThinThreads) {
        const int r = k / per, c = (k - r * per) * 4;
        f(tall ? j0 + r : r, tall ? c : j0 + c);
    }
}

// Columns j0 .. of U times `scale` into X (row stride ldx), zeros around them;
// UPDATE: the momentum is brought up to date first.
template <bool UPDATE>
__device__ __forceinline__ void thin_load(const NsThinArgs& args, const NsSmallMat& L, int j0, int cols, int m16, int ldx,
                                          double scale, float* X) {
    for (int e = threadIdx.x * 4; e < m16 * ldx; e += kThinThreads * 4)
        *reinterpret_cast<float4*>(X + e) = make_float4(0.f, 0.f, 0.f, 0.f);
    __syncthreads();
    const bool tall = L.d > L.p;
    const int end = tall ? L.p : min(L.p, j0 + cols);
    thin_runs(L, j0, cols, [&](int r, int c) {
        float g[4], m[4] = {0.f, 0.f, 0.f, 0.f};
        load4(L.G, r, c, L.d, end, L.p, g);
        if (L.M) load4(L.M, r, c, L.d, end, L.p, m);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (UPDATE && L.M) m[e] = fmaf(args.beta, m[e], g[e]);
            const float u = update_of(g[e], m[e], L.M != nullptr, args.nesterov, args.beta);
            const float v = UPDATE ? u : (float)((double)u * scale);
            if (c + e < end) X[tall ? (c + e) * ldx + r - j0 : r * ldx + c + e - j0] = v;
        }
        if (UPDATE && L.M) store4(L.M, r, c, L.d, end, L.p, m);
    });
    __syncthreads();
}

// 16x16x4 float64 MFMA: lane l holds row l % 16 of the first operand and column
// l % 16 of the second, k = l / 16; of the result column l % 16, rows l / 16 + 0,
// 4, 8, 12.  Its 16 passes are settled like the others'.
typedef double f64x4_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ void settle64(f64x4_t& a) {
    asm volatile("" : "+v"(a));
    asm volatile("s_nop 15\n\ts_nop 7");
    asm volatile("" : "+v"(a));
}
// What the polynomials' launch leaves behind the partial Grams: 1 / (|U| + eps),
// and the product P of each round.
__device__ __forceinline__ const double* thin_inv(const NsThinArgs& args, const NsThinMat& L, int m16) {
    return args.ws + L.gram + (size_t)L.chunks * m16 * m16;
}
// P of a round to LDS (a barrier has to follow).
template <int MT>
__device__ __forceinline__ void thin_load_poly(const double* inv, int round, float* P) {
    constexpr int m16 = 16 * MT;
    const float* poly = reinterpret_cast<const float*>(inv + 1) + (size_t)round * m16 * m16;
    for (int e = threadIdx.x; e < m16 * m16; e += kThinThreads) P[e / m16 * (m16 + 4) + e % m16] = poly[e];
}

// Partial Gram matrix of a chunk's columns: every wave the whole of it over a
// quarter of the columns, the waves' sums joined in order.  FIRST: of U, whose
// momentum is brought up to date; else of X after args.round rounds.
template <int MT, bool FIRST>
__device__ __forceinline__ void thin_gram(const NsThinArgs& args, const NsThinMat& L, int chunk, float* X, double* sum,
                                          float* P) {
    constexpr int m16 = 16 * MT, TILES = MT * (MT + 1) / 2, cols = thin_cols<MT>(), ldx = cols + 4;
    const int n = max(L.t.d, L.t.p);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, q = lane >> 4;
    f64x4_t acc[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) acc[t] = f64x4_t{0.0, 0.0, 0.0, 0.0};
    const int end = min(n, (chunk + 1) * L.cols);
    for (int j0 = chunk * L.cols; j0 < end; j0 += cols) {
        const int here = min(cols, end - j0);
        if constexpr (FIRST) {
            thin_load<true>(args, L.t, j0, here, m16, ldx, 1.0, X);
        } else {
            const double* inv = thin_inv(args, L, m16);
            thin_load<false>(args, L.t, j0, here, m16, ldx, inv[0], X);
            for (int r = 0; r < args.round; ++r) {
                thin_load_poly<MT>(inv, r, P);
                __syncthreads();
                ns_apply_columns<MT, kThinThreads / 64>(X, P, m16 + 4, (here + 15) / 16, ldx);
                __syncthreads();
            }
        }
        for (int k = 4 * wave; k < here; k += 16) {          // what follows the columns is zero
            double x[MT];
#pragma unroll
            for (int i = 0; i < MT; ++i) x[i] = (double)X[(16 * i + r) * ldx + k + q];
            int t = 0;
#pragma unroll
            for (int j = 0; j < MT; ++j)
#pragma unroll
                for (int i = 0; i <= j; ++i, ++t) acc[t] = __builtin_amdgcn_mfma_f64_16x16x4f64(x[i], x[j], acc[t], 0, 0, 0);
        }
        __syncthreads();
    }
#pragma unroll
    for (int t = 0; t < TILES; ++t) settle64(acc[t]);
    for (int w = 0; w < kThinThreads / 64; ++w) {
        if (w == wave) {
            int t = 0;
#pragma unroll
            for (int j = 0; j < MT; ++j)
#pragma unroll
                for (int i = 0; i <= j; ++i, ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        double& s = sum[(16 * i + q + 4 * e) * m16 + 16 * j + r];
                        s = w == 0 ? acc[t][e] : s + acc[t][e];
                    }
        }
        __syncthreads();
    }
    double* out = args.ws + L.gram + (size_t)chunk * m16 * m16;
    for (int e = threadIdx.x; e < m16 * m16; e += kThinThreads) {
        const int i = e / m16, j = e % m16;
        out[e] = (i >> 4) <= (j >> 4) ? sum[e] : sum[j * m16 + i];
    }
}

// The chunk of workgroup blockIdx.x.
__device__ __forceinline__ int thin_chunk(const NsThinArgs& args, int& chunk) {
    return find_matrix(args.n, blockIdx.x, chunk, [&](int k) { return args.L[k].begin; });
}

template <bool FIRST>
__global__ __launch_bounds__(kThinThreads) void ns_thin_gram_kernel(const NsThinArgs args) {
    __shared__ __attribute__((aligned(16))) float X[kThinLds];
    __shared__ double sum[64 * 64];
    __shared__ __attribute__((aligned(16))) float P[FIRST ? 4 : 64 * 68];
    int chunk;
    const NsThinMat& L = args.L[thin_chunk(args, chunk)];
    switch ((min(L.t.d, L.t.p) + 15) / 16) {
        case 1: thin_gram<1, FIRST>(args, L, chunk, X, sum, P); break;
        case 2: thin_gram<2, FIRST>(args, L, chunk, X, sum, P); break;
        case 3: thin_gram<3, FIRST>(args, L, chunk, X, sum, P); break;
        default: thin_gram<4, FIRST>(args, L, chunk, X, sum, P); break;
    }
}

// C = A B of symmetric matrices that commute (so B's columns are its rows, and
// C's tiles above the diagonal suffice), or, with `poly`, a I + b A + c A B.
constexpr int kPolyThreads = 512;
template <int MT>
__device__ __forceinline__ void thin_product(const double* A, const double* B, double* C, bool poly, double a, double b, double c) {
    constexpr int ld = 16 * MT + 4, TILES = MT * (MT + 1) / 2, WAVES = kPolyThreads / 64, PER = (TILES + WAVES - 1) / WAVES;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, q = lane >> 4;
    f64x4_t acc[PER];
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        acc[u] = f64x4_t{0.0, 0.0, 0.0, 0.0};
        if (wave + WAVES * u >= TILES) break;
        int ti, tj;
        sym_tile(wave + WAVES * u, ti, tj);
        const double *x = A + (16 * ti + r) * ld + q, *y = B + (16 * tj + r) * ld + q;
#pragma unroll
        for (int k = 0; k < 16 * MT; k += 4) acc[u] = __builtin_amdgcn_mfma_f64_16x16x4f64(x[k], y[k], acc[u], 0, 0, 0);
        settle64(acc[u]);
    }
    __syncthreads();             // C may be A or B
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        if (wave + WAVES * u >= TILES) break;
        int ti, tj;
        sym_tile(wave + WAVES * u, ti, tj);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = 16 * ti + q + 4 * e, j = 16 * tj + r;
            const double v = poly ? fma(c, acc[u][e], b * A[i * ld + j]) + (i == j ? a : 0.0) : acc[u][e];
            C[i * ld + j] = v;
            if (ti != tj) C[j * ld + i] = v;
        }
    }
    __syncthreads();
}

template <int MT>
__device__ __forceinline__ void thin_poly(const NsThinArgs& args, const NsThinMat& L, double* lds) {
    constexpr int m16 = 16 * MT, ld = m16 + 4;
    double *A = lds, *Bm = A + m16 * ld, *P = Bm + m16 * ld;
    double* gram = args.ws + L.gram;
    // The chunks' partial matrices, in order; a thread's elements together, so
    // that their loads overlap (one at a time, 47 chunks of 64 x 64 took 110 us).
    constexpr int PER = (m16 * m16 + kPolyThreads - 1) / kPolyThreads;
    if ((int)threadIdx.x < m16 * m16) {
        double part[PER] = {};
#pragma unroll 4
        for (int k = 0; k < L.chunks; ++k)
#pragma unroll
            for (int e = 0; e < PER; ++e)
                part[e] += gram[(size_t)k * m16 * m16 + min((int)threadIdx.x + e * kPolyThreads, m16 * m16 - 1)];
#pragma unroll
        for (int e = 0; e < PER; ++e) {
            const int at = threadIdx.x + e * kPolyThreads;
            if (at < m16 * m16) A[at / m16 * ld + at % m16] = part[e];
        }
    }
    __syncthreads();
    double* out = gram + (size_t)L.chunks * m16 * m16;
    if (args.round == 0) {
        double sq = 0.0;
        for (int i = 0; i < m16; ++i) sq += A[i * ld + i];
        const double inv = 1.0 / (sqrt(sq) + (double)args.eps);
        __syncthreads();
        for (int e = threadIdx.x; e < m16 * m16; e += kPolyThreads) {
            // U's scale is taken out one factor at a time: its square may be out of range
            const int at = e / m16 * ld + e % m16;
            A[at] = A[at] * inv * inv;
        }
        if (threadIdx.x == 0) out[0] = inv;
        __syncthreads();
    }
    for (int s = args.first; s < args.last; ++s) {
        double* to = s == args.first ? P : Bm;
        thin_product<MT>(A, A, to, true, args.coef[3 * s], args.coef[3 * s + 1], args.coef[3 * s + 2]);
        if (s + 1 < args.last) {
            thin_product<MT>(to, A, A, false, 0.0, 0.0, 0.0);
            thin_product<MT>(to, A, A, false, 0.0, 0.0, 0.0);
        }
        if (s > args.first) thin_product<MT>(Bm, P, P, false, 0.0, 0.0, 0.0);
    }
    float* poly = reinterpret_cast<float*>(out + 1) + (size_t)args.round * m16 * m16;
    for (int e = threadIdx.x; e < m16 * m16; e += kPolyThreads) poly[e] = (float)P[e / m16 * ld + e % m16];
}

__global__ __launch_bounds__(kPolyThreads) void ns_thin_poly_kernel(const NsThinArgs args) {
    __shared__ __attribute__((aligned(16))) double lds[3 * 64 * 68];
    const NsThinMat& L = args.L[blockIdx.x];
    switch ((min(L.t.d, L.t.p) + 15) / 16) {
        case 1: thin_poly<1>(args, L, lds); break;
        case 2: thin_poly<2>(args, L, lds); break;
        case 3: thin_poly<3>(args, L, lds); break;
        default: thin_poly<4>(args, L, lds); break;
    }
}

// ONE: there was one round, whose P stays in LDS.
template <int MT, bool ONE>
__device__ __forceinline__ void thin_apply(const NsThinArgs& args, const NsThinMat& L, int chunk, float* X, float* P) {
    constexpr int m16 = 16 * MT, lda = m16 + 4, cols = thin_cols<MT>(), ldx = cols + 4;
    const int n = max(L.t.d, L.t.p);
    const double* inv = thin_inv(args, L, m16);
    const double scale = inv[0];
    if constexpr (ONE) thin_load_poly<MT>(inv, 0, P);
    const bool tall = L.t.d > L.t.p;
    const int end = min(n, (chunk + 1) * L.cols);
    for (int j0 = chunk * L.cols; j0 < end; j0 += cols) {
        const int here = min(cols, end - j0);
        thin_load<false>(args, L.t, j0, here, m16, ldx, scale, X);
        const int rounds = ONE ? 1 : args.rounds;
        for (int r = 0; r < rounds; ++r) {
            if constexpr (!ONE) {
                thin_load_poly<MT>(inv, r, P);
                __syncthreads();
            }
            ns_apply_columns<MT, kThinThreads / 64>(X, P, lda, (here + 15) / 16, ldx);
            __syncthreads();
        }
        const int stop = tall ? L.t.p : min(L.t.p, j0 + here);
        thin_runs(L.t, j0, here, [&](int r, int c) {
            float v[4], w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = c + e < stop ? X[tall ? (c + e) * ldx + r - j0 : r * ldx + c + e - j0] : 0.f;
            if (L.t.O) {
                if (L.t.o_bf16) store4(static_cast<__bf16*>(L.t.O), r, c, L.t.d, stop, L.t.p, v);
                else store4(static_cast<float*>(L.t.O), r, c, L.t.d, stop, L.t.p, v);
            }
            if (L.t.W) {
                load4(L.t.W, r, c, L.t.d, stop, L.t.p, w);
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = fmaf(-L.t.step, v[e], args.keep * w[e]);
                store4(L.t.W, r, c, L.t.d, stop, L.t.p, w);
                if (L.t.Wb) store4(reinterpret_cast<__bf16*>(L.t.Wb), r, c, L.t.d, stop, L.t.p, w);
            }
        });
        __syncthreads();
    }
}

template <bool ONE>
__global__ __launch_bounds__(kThinThreads) void ns_thin_apply_kernel(const NsThinArgs args) {
    __shared__ __attribute__((aligned(16))) float X[kThinLds];
    __shared__ __attribute__((aligned(16))) float P[64 * 68];
    int chunk;
    const NsThinMat& L = args.L[thin_chunk(args, chunk)];
    switch ((min(L.t.d, L.t.p) + 15) / 16) {
        case 1: thin_apply<1, ONE>(args, L, chunk, X, P); break;
        case 2: thin_apply<2, ONE>(args, L, chunk, X, P); break;
        case 3: thin_apply<3, ONE>(args, L, chunk, X, P); break;
        default: thin_apply<4, ONE>(args, L, chunk, X, P); break;
    }
}

}  // namespace

hipError_t launch_ns_thin(const NsThinArgs& a, int n_wg, hipStream_t s) {
    if (n_wg <= 0) return hipSuccess;
    NsThinArgs b = a;
    for (b.round = 0; b.round < b.rounds; ++b.round) {
        b.first = b.round > 0 ? b.end[b.round - 1] : 0, b.last = b.end[b.round];
        if (b.round == 0) hipLaunchKernelGGL(ns_thin_gram_kernel<true>, dim3(n_wg), dim3(kThinThreads), 0, s, b);
        else hipLaunchKernelGGL(ns_thin_gram_kernel<false>, dim3(n_wg), dim3(kThinThreads), 0, s, b);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(ns_thin_poly_kernel, dim3(b.n), dim3(kPolyThreads), 0, s, b);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (b.rounds == 1) hipLaunchKernelGGL(ns_thin_apply_kernel<true>, dim3(n_wg), dim3(kThinThreads), 0, s, b);
    else hipLaunchKernelGGL(ns_thin_apply_kernel<false>, dim3(n_wg), dim3(kThinThreads), 0, s, b);
    return hipGetLastError();
}

hipError_t launch_ns_small(const NsSmallArgs& a, hipStream_t s) {
    if (a.n <= 0) return hipSuccess;
    hipLaunchKernelGGL(ns_small_kernel, dim3(a.n), dim3(kSmallThreads), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_ns_norm(const NsNormArgs& a, int n_wg, hipStream_t s) {
    if (n_wg <= 0) return hipSuccess;
    hipLaunchKernelGGL(ns_norm_kernel, dim3(n_wg), dim3(256), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_ns_prep(const NsArgs& a, int n_wg, bool split, hipStream_t s) {
    if (n_wg <= 0) return hipSuccess;
    if (split) hipLaunchKernelGGL(ns_prep_kernel<true>, dim3(n_wg), dim3(256), 0, s, a);
    else hipLaunchKernelGGL(ns_prep_kernel<false>, dim3(n_wg), dim3(256), 0, s, a);
    return hipGetLastError();
}

template <NsOp OP, NsTile TILE>
static hipError_t gemm(const NsArgs& a, int n_wg, bool split, hipStream_t s) {
    const dim3 grid(n_wg), block(64 * NsCfg<TILE>::waves);
    if (split) hipLaunchKernelGGL((ns_gemm_kernel<OP, true, TILE>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((ns_gemm_kernel<OP, false, TILE>), grid, block, 0, s, a);
    return hipGetLastError();
}
template <NsOp OP>
static hipError_t gemm(const NsArgs& a, int n_wg, bool split, NsTile t, hipStream_t s) {
    switch (t) {
        case NsTile::T256: return gemm<OP, NsTile::T256>(a, n_wg, split, s);
        case NsTile::T256x128: return gemm<OP, NsTile::T256x128>(a, n_wg, split, s);
        case NsTile::T128: return gemm<OP, NsTile::T128>(a, n_wg, split, s);
        default: return gemm<OP, NsTile::T64>(a, n_wg, split, s);
    }
}

hipError_t launch_ns_gemm(const NsArgs& a, NsOp op, bool split, NsTile t, hipStream_t s) {
    int n_wg = 0;
    for (int x = 0; x < 8; ++x) n_wg = std::max(n_wg, 8 * (a.xcd[x + 1] - a.xcd[x]));
    if (n_wg <= 0) return hipSuccess;
    switch (op) {
        case NsOp::Gram: return gemm<NsOp::Gram>(a, n_wg, split, t, s);
        case NsOp::Poly: return gemm<NsOp::Poly>(a, n_wg, split, t, s);
        case NsOp::Apply: return gemm<NsOp::Apply>(a, n_wg, split, t, s);
        default: return gemm<NsOp::Final>(a, n_wg, split, t, s);
    }
}

}  // namespace bk
