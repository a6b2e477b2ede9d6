// Root-mean-square norm with the residual's addition, and its backward pass.
//
//   h = x + r (rounded to the type, as the residual stream keeps it)
//   s = 1 / sqrt(mean_j h_j^2 + eps),  xhat = h s,  y = gamma * xhat
//   scale_g = max(max_{j in g} |y_j| / 448, 2^-126),  q = e4m3(y / scale_g)
//
//   w = gamma * dy
//   dx = s (w - xhat mean_j(w_j xhat_j)) + dres
//   P_i = sum_t dy_it * xhat_it          (per-sample gradient of gamma)
//
// A row is held in registers by TPR threads, NCH pieces of 8 columns each, so
// that every tensor passes HBM once; sums are float32, in a fixed order.  Rows
// may start at any element: full pieces are 16-byte loads and stores at any
// alignment, only the last piece of a row that is no multiple of 8 columns
// goes by elements.  Bound by HBM for many rows ([16384, 4096] with residual, xhat and
// e4m3 rows: 133 us, 5.6 TB/s; the backward pass of as many 111 us and 5 for the
// partial sums, 4.7 TB/s; a large copy makes 5.0 here), by latency for few
// ([1, 768] 3.5 us; [4096, 768] 9.0 us, 3.5 TB/s).
#include "bk_device.h"
#include "step_kernels.h"

#include <algorithm>

namespace bk {
namespace {

// The 8 values of row[c .. c + 8), zeros past p.
template <typename E>
__device__ __forceinline__ void load_piece(const E* row, int c, int p, float v[8]) {
    if (c + 8 <= p) {
        if constexpr (sizeof(E) == 2) {
            const uint4 w = load16_any(row + c);
            const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[2 * j] = bf16_to_f32(ws[j] & 0xFFFFu);
                v[2 * j + 1] = bf16_to_f32(ws[j] >> 16);
            }
        } else {
            const uint4 a = load16_any(row + c), b = load16_any(row + c + 4);
            const uint32_t ws[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(ws[j]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            v[j] = 0.f;
            if (c + j < p) {
                if constexpr (sizeof(E) == 2) v[j] = bf16_to_f32(reinterpret_cast<const uint16_t*>(row)[c + j]);
                else v[j] = reinterpret_cast<const float*>(row)[c + j];
            }
        }
    }
}

// A row's pieces as they lie in memory (zeros past p), for loads that are to be
// in flight while an earlier row is worked on.
template <typename E, int NCH>
struct RawRow {
    uint4 v[NCH][sizeof(E) / 2];

    template <int TPR>
    __device__ __forceinline__ void load(const E* row, int lane, int p) {
#pragma unroll
        for (int k = 0; k < NCH; ++k) {
            const int c = (k * TPR + lane) * 8;
            if (c + 8 <= p) {
#pragma unroll
                for (int z = 0; z < (int)sizeof(E) / 2; ++z) v[k][z] = load16_any(row + c + 8 / (sizeof(E) / 2) * z);
            } else {
                E t[8] = {};
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (c + j < p) t[j] = row[c + j];
                __builtin_memcpy(v[k], t, sizeof t);
            }
        }
    }
    __device__ __forceinline__ void unpack(int k, float o[8]) const {
        if constexpr (sizeof(E) == 2) {
            const uint32_t w[4] = {v[k][0].x, v[k][0].y, v[k][0].z, v[k][0].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                o[2 * j] = bf16_to_f32(w[j] & 0xFFFFu);
                o[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
            }
        } else {
            __builtin_memcpy(o, v[k], 32);
        }
    }
};

// bf16 of a value that may be infinite or NaN (round to nearest even).
__device__ __forceinline__ uint32_t to_bf16(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }

// v rounded to the type, as it is stored and read back.
template <typename E>
__device__ __forceinline__ float round_to(float v) {
    if constexpr (sizeof(E) == 2) return bf16_to_f32(to_bf16(v));
    else return v;
}

template <typename E>
__device__ __forceinline__ void store_piece(E* row, int c, int p, const float v[8]) {
    if (c >= p) return;
    if (c + 8 <= p) {
        if constexpr (sizeof(E) == 2) {
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = to_bf16(v[2 * j]) | to_bf16(v[2 * j + 1]) << 16;
            __builtin_memcpy(row + c, w, 16);
        } else {
            __builtin_memcpy(row + c, v, 16);
            __builtin_memcpy(row + c + 4, v + 4, 16);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (c + j < p) {
                if constexpr (sizeof(E) == 2) reinterpret_cast<uint16_t*>(row)[c + j] = (uint16_t)to_bf16(v[j]);
                else reinterpret_cast<float*>(row)[c + j] = v[j];
            }
    }
}

__device__ __forceinline__ void load_gamma(const void* gamma, int bf16, int c, int p, float v[8]) {
    if (!gamma) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = 1.f;
    } else if (bf16) {
        load_piece(static_cast<const bf16_t*>(gamma), c, p, v);
    } else {
        load_piece(static_cast<const float*>(gamma), c, p, v);
    }
}

// Sum over the TPR threads of a row, the same in all of them.
// red: TPR / 64 floats; with TPR > 64 the whole workgroup is one row, and red
// must not be the previous call's, which slower waves may still be reading (the
// backward pass alternates between two).
template <int TPR>
__device__ __forceinline__ float row_reduce(float v, float* red) {
#pragma unroll
    for (int off = (TPR < 64 ? TPR : 64) / 2; off >= 1; off >>= 1) v += __shfl_xor(v, off, 64);
    if constexpr (TPR > 64) {
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
        __syncthreads();
        v = red[0];
#pragma unroll
        for (int w = 1; w < TPR / 64; ++w) v += red[w];
    }
    return v;
}

template <int TPR> constexpr int block_of() { return TPR > 64 ? TPR : 256; }

// The largest of |y|, and of |h gamma| in float64.
struct Tops {
    float y;
    double t;
};
__device__ __forceinline__ Tops larger(Tops a, Tops b) { return {fmaxf(a.y, b.y), fmax(a.t, b.t)}; }
// Over runs of 4 to 64 lanes, by the vector unit's own paths (by LDS, whose
// shuffles the groups of a row wait for in turn, [16384, 5120] bf16 in groups of 128
// took 285 us instead of 262).  The mirrored half (row) of lanes that agree already
// in fours (eights) serves as the neighbouring one.
template <typename F>
__device__ __forceinline__ Tops moved(Tops v, F move) {
    const uint64_t t = __builtin_bit_cast(uint64_t, v.t);
    return {__uint_as_float(move(__float_as_uint(v.y))),
            __builtin_bit_cast(double, (uint64_t)move((uint32_t)(t >> 32)) << 32 | move((uint32_t)t))};
}
template <int CTRL>
__device__ __forceinline__ Tops with_lane(Tops v) {
    return larger(v, moved(v, [](uint32_t w) { return (uint32_t)__builtin_amdgcn_mov_dpp((int)w, CTRL, 0xF, 0xF, true); }));
}
__device__ __forceinline__ Tops run_tops(Tops v, int width) {
    v = with_lane<0xB1>(v);                     // lane ^ 1
    v = with_lane<0x4E>(v);                     // lane ^ 2
    if (width >= 8) v = with_lane<0x141>(v);    // 7 - lane of 8
    if (width >= 16) v = with_lane<0x140>(v);   // 15 - lane of 16
    // even rows of 16 (halves) in one result, the odd ones in the other
    if (width >= 32)
        v = larger(moved(v, [](uint32_t w) { return __builtin_amdgcn_permlane16_swap(w, w, false, false)[0]; }),
                   moved(v, [](uint32_t w) { return __builtin_amdgcn_permlane16_swap(w, w, false, false)[1]; }));
    if (width >= 64)
        v = larger(moved(v, [](uint32_t w) { return __builtin_amdgcn_permlane32_swap(w, w, false, false)[0]; }),
                   moved(v, [](uint32_t w) { return __builtin_amdgcn_permlane32_swap(w, w, false, false)[1]; }));
    return v;
}
// Over the TPR threads of a row.
template <int TPR>
__device__ __forceinline__ Tops row_tops(Tops v, Tops* wave) {
    v = run_tops(v, TPR < 64 ? TPR : 64);
    if constexpr (TPR > 64) {
        if ((threadIdx.x & 63) == 0) wave[threadIdx.x >> 6] = v;
        __syncthreads();
        constexpr int waves = TPR / 64, width = waves <= 4 ? 4 : waves <= 8 ? 8 : 16;
        v = run_tops(wave[min((int)threadIdx.x & (width - 1), waves - 1)], width);
    }
    return v;
}

// Q: 8-bit rows are wanted.
template <typename E, int TPR, int NCH, bool Q>
__global__ __launch_bounds__(block_of<TPR>()) void rmsnorm_kernel(const RmsArgs a) {
    constexpr int ROWS = block_of<TPR>() / TPR;
    __shared__ float red[TPR > 64 ? TPR / 64 : 1];
    const int lane = threadIdx.x % TPR;
    const int p = a.p;
    const int64_t row = a.row0 + (int64_t)blockIdx.x * ROWS + threadIdx.x / TPR;
    if (row >= a.rows) return;             // whole rows: with TPR > 64 whole workgroups
    const size_t at = (size_t)row * p;
    const E* x = static_cast<const E*>(a.x) + at;
    float v[NCH][8];
#pragma unroll
    for (int k = 0; k < NCH; ++k) load_piece(x, (k * TPR + lane) * 8, p, v[k]);
    // gamma comes with the row where the registers allow it, not behind the
    // row's reduction ([1, 768] 3.5 us, behind it 3.7).
    constexpr bool EARLY = NCH <= 2;
    float g[EARLY ? NCH : 1][8];
    if constexpr (EARLY)
#pragma unroll
        for (int k = 0; k < NCH; ++k) load_gamma(a.gamma, a.gamma_bf16, (k * TPR + lane) * 8, p, g[k]);
    if (a.res) {
        const E* r = static_cast<const E*>(a.res) + at;
        float w[NCH][8];
#pragma unroll
        for (int k = 0; k < NCH; ++k) load_piece(r, (k * TPR + lane) * 8, p, w[k]);
#pragma unroll
        for (int k = 0; k < NCH; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[k][j] = round_to<E>(v[k][j] + w[k][j]);
    }
    if (a.h) {
        E* h = static_cast<E*>(a.h) + at;
#pragma unroll
        for (int k = 0; k < NCH; ++k) store_piece(h, (k * TPR + lane) * 8, p, v[k]);
    }
    float sq = 0.f;
#pragma unroll
    for (int k = 0; k < NCH; ++k)
#pragma unroll
        for (int j = 0; j < 8; ++j) sq = fmaf(v[k][j], v[k][j], sq);
    sq = row_reduce<TPR>(sq, red);
    const float rstd = 1.0f / sqrtf(sq / (float)p + a.eps);
    if (a.rstd && lane == 0) a.rstd[row] = rstd;
    const auto gamma_of = [&](int k, float w[8]) {
        if constexpr (EARLY) {
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = g[k][j];
        } else {
            load_gamma(a.gamma, a.gamma_bf16, (k * TPR + lane) * 8, p, w);
        }
    };
    if constexpr (!Q) {
#pragma unroll
        for (int k = 0; k < NCH; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[k][j] *= rstd;
        if (a.xhat) {
            E* o = static_cast<E*>(a.xhat) + at;
#pragma unroll
            for (int k = 0; k < NCH; ++k) store_piece(o, (k * TPR + lane) * 8, p, v[k]);
        }
        if (!a.y) return;
#pragma unroll
        for (int k = 0; k < NCH; ++k) {
            float w[8];
            gamma_of(k, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[k][j] *= w[j];
        }
        E* o = static_cast<E*>(a.y) + at;
#pragma unroll
        for (int k = 0; k < NCH; ++k) store_piece(o, (k * TPR + lane) * 8, p, v[k]);
        return;
    }
    // 8-bit rows need h until the end.
    if (a.xhat) {
        E* o = static_cast<E*>(a.xhat) + at;
#pragma unroll
        for (int k = 0; k < NCH; ++k) {
            float n[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) n[j] = v[k][j] * rstd;
            store_piece(o, (k * TPR + lane) * 8, p, n);
        }
    }
    // Threads without columns leave pieces out where a row has many (which also
    // takes fewer registers: [2000, 16384] in groups of 128 75 us, with them 86).
    constexpr bool SKIP = NCH * TPR > 1024;
    Tops m[NCH];
#pragma unroll
    for (int k = 0; k < NCH; ++k) {
        const int c = (k * TPR + lane) * 8;
        m[k] = {0.f, 0.0};
        if (SKIP && c >= p) continue;
        float w[8], y[8];
        gamma_of(k, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = v[k][j] * rstd * w[j];
        if (a.y) store_piece(static_cast<E*>(a.y) + at, c, p, y);
        // (a thread's largest h gamma is that of its largest y, but for magnitudes
        // that lie within 2^-23 of each other)
        float h = 0.f, gh = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const bool take = c + j < p && fabsf(y[j]) > m[k].y;
            m[k].y = take ? fabsf(y[j]) : m[k].y, h = take ? v[k][j] : h, gh = take ? w[j] : gh;
        }
        m[k].t = fabs((double)h * gh);
    }
    // Scales: of the row, or of runs of `group` columns, which are runs of
    // group / 8 threads within one piece.  The quotient y / scale is h gamma 448 /
    // max |h gamma|, for 1 / rms drops out.  It is formed in float64, where h gamma
    // is exact, and rounded to float32 once: quotients between two 8-bit values
    // then go to the even one (of bf16 rows with a bf16 gamma about 1 in 10^4
    // lies there exactly, and float32 sent half of these the other way).  Where
    // y's largest is zero, next to it or infinite, the quotient is y's own.
    __shared__ Tops wave[TPR > 64 ? TPR / 64 : 1];
    const int width = a.group ? min(a.group >> 3, TPR) : TPR;
    if (a.group) {
#pragma unroll
        for (int k = 0; k < NCH; ++k) m[k] = run_tops(m[k], width);
    } else {
#pragma unroll
        for (int k = 1; k < NCH; ++k) m[0] = larger(m[0], m[k]);
        m[0] = row_tops<TPR>(m[0], wave);
#pragma unroll
        for (int k = 1; k < NCH; ++k) m[k] = m[0];
    }
    uint8_t* q = a.q + at;
    float* qs = a.q_scale + (size_t)row * a.n_groups;
#pragma unroll
    for (int k = 0; k < NCH; ++k) {
        const int c = (k * TPR + lane) * 8;
        if (SKIP && c >= p) continue;
        const float exact = m[k].y / 448.0f, scale = fmaxf(exact, 1.17549435e-38f);
        if (c < p && (a.group ? (lane & (width - 1)) == 0 : lane == 0 && k == 0)) qs[a.group ? c / a.group : 0] = scale;
        float w[8], u[8];
        gamma_of(k, w);
        if constexpr (NCH > 2)
            // products formed anew: kept, they cost 16 registers a piece
#pragma unroll
            for (int j = 0; j < 8; ++j) asm volatile("" : "+v"(v[k][j]));
        if (exact > 1.17549435e-38f && exact < INFINITY) {
            // 448 / max |h gamma|: two Newton steps from an approximation
            double to = __builtin_amdgcn_rcp(m[k].t);
#pragma unroll
            for (int j = 0; j < 2; ++j) to = fma(fma(-m[k].t, to, 1.0), to, to);
            to *= 448.0;
#pragma unroll
            for (int j = 0; j < 8; ++j) u[j] = (float)((double)v[k][j] * w[j] * to);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) u[j] = v[k][j] * rstd * w[j] / scale;
        }
        uint32_t b[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            b[j] = __builtin_amdgcn_cvt_pk_fp8_f32(u[4 * j], u[4 * j + 1], 0, false);
            b[j] = __builtin_amdgcn_cvt_pk_fp8_f32(u[4 * j + 2], u[4 * j + 3], b[j], true);
        }
        if (c + 8 <= p) {
            __builtin_memcpy(q + c, b, 8);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (c + j < p) q[c + j] = (uint8_t)(b[j >> 2] >> (8 * (j & 3)));
        }
    }
}

template <typename E, int TPR, int NCH, int BLOCK>
__global__ __launch_bounds__(BLOCK) void rmsnorm_grad_kernel(const RmsGradArgs a) {
    constexpr int ROWS = BLOCK / TPR;
    __shared__ float red[2][TPR > 64 ? TPR / 64 : 1];
    __shared__ float join[ROWS > 1 ? ROWS : 1][ROWS > 1 ? TPR * NCH * 8 : 1];
    const int lane = threadIdx.x % TPR, grp = threadIdx.x / TPR;
    const int p = a.p;
    float g[NCH][8];
#pragma unroll
    for (int k = 0; k < NCH; ++k) load_gamma(a.gamma, a.gamma_bf16, (k * TPR + lane) * 8, p, g[k]);
    int flip = 0;
    // A segment: rows [t0, t1) of sample b, shared by the workgroup's groups of
    // threads, or (solo: samples of few tokens) one segment to each group.
    const int64_t segs = a.B * a.chunks;
    const int64_t seg = a.seg0 + (a.solo ? (int64_t)blockIdx.x * ROWS + grp : (int64_t)blockIdx.x);
    const int64_t b = seg / a.chunks;
    const int64_t t0 = (seg - b * a.chunks) * a.chunk, t1 = seg < segs ? min(a.T, t0 + a.chunk) : t0;
    const int step = a.solo ? 1 : ROWS;
    float pg[NCH][8];
#pragma unroll
    for (int k = 0; k < NCH; ++k)
#pragma unroll
        for (int j = 0; j < 8; ++j) pg[k][j] = 0.f;
    // The next row's dy, xhat and rstd and this row's dres are in flight while
    // this row is reduced: with few workgroups to a CU a row's latency is what
    // a workgroup's rows cost.
    RawRow<E, NCH> dy, xh, dr;
    float rstd = 0.f;
    int64_t t = t0 + (a.solo ? 0 : grp);
    const auto fetch = [&](int64_t row) {
        const size_t at = (size_t)row * p;
        dy.template load<TPR>(static_cast<const E*>(a.dy) + at, lane, p);
        xh.template load<TPR>(static_cast<const E*>(a.xhat) + at, lane, p);
        rstd = a.rstd[row];
    };
    constexpr bool AHEAD = NCH == 1 || TPR == 64;      // the registers allow it
    if (AHEAD && t < t1) fetch(b * a.T + t);
    for (; t < t1; t += step) {
        const int64_t row = b * a.T + t;
        if (!AHEAD) fetch(row);
        const size_t at = (size_t)row * p;
        float w[NCH][8], n[NCH][8];
        float dot = 0.f;
#pragma unroll
        for (int k = 0; k < NCH; ++k) {
            dy.unpack(k, w[k]);
            xh.unpack(k, n[k]);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                pg[k][j] = fmaf(w[k][j], n[k][j], pg[k][j]);
                w[k][j] *= g[k][j];
                dot = fmaf(w[k][j], n[k][j], dot);
            }
        }
        const float rs = rstd;
        if (a.dres && a.dx) dr.template load<TPR>(static_cast<const E*>(a.dres) + at, lane, p);
        if (AHEAD && t + step < t1) fetch(row + step);
        dot = row_reduce<TPR>(dot, red[flip]) / (float)p;
        flip ^= 1;
        if (!a.dx) continue;
#pragma unroll
        for (int k = 0; k < NCH; ++k) {
            const int c = (k * TPR + lane) * 8;
#pragma unroll
            for (int j = 0; j < 8; ++j) w[k][j] = rs * (w[k][j] - n[k][j] * dot);
            if (a.dres) {
                float d[8];
                dr.unpack(k, d);
#pragma unroll
                for (int j = 0; j < 8; ++j) w[k][j] += d[j];
            }
            store_piece(static_cast<E*>(a.dx) + at, c, p, w[k]);
        }
    }
    if (!a.P) return;
    // The groups' sums, joined in order, to P or to the segment's partial row.
    float* out = (a.chunks > 1 ? a.part : a.P) + (size_t)seg * p;
    if (ROWS == 1 || a.solo) {
        if (seg < segs)
#pragma unroll
            for (int k = 0; k < NCH; ++k) store_piece(out, (k * TPR + lane) * 8, p, pg[k]);
        return;
    }
    if constexpr (ROWS > 1) {
#pragma unroll
        for (int k = 0; k < NCH; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) join[grp][(k * TPR + lane) * 8 + j] = pg[k][j];
        __syncthreads();
        for (int c = threadIdx.x; c < p; c += BLOCK) {
            float s = join[0][c];
#pragma unroll
            for (int r = 1; r < ROWS; ++r) s += join[r][c];
            out[c] = s;
        }
    }
}

// P[b] = sum of the sample's partial rows: four runs of them, each in order, and
// then the runs; 64 columns to a workgroup.
__global__ __launch_bounds__(256) void rmsnorm_grad_join_kernel(const float* part, float* P, int chunks, int p,
                                                                int64_t wg0, int col_blocks) {
    __shared__ float runs[4][64];
    const int64_t wg = wg0 + blockIdx.x, b = wg / col_blocks;
    const int run = threadIdx.x >> 6, col = threadIdx.x & 63;
    const int c = (int)(wg - b * col_blocks) * 64 + col;
    const int k0 = run * chunks / 4, k1 = (run + 1) * chunks / 4;
    float s = 0.f;
    if (c < p) {
        const float* q = part + (size_t)b * chunks * p + c;
#pragma unroll 8
        for (int k = k0; k < k1; ++k) s += q[(size_t)k * p];
    }
    runs[run][col] = s;
    __syncthreads();
    if (run == 0 && c < p) P[(size_t)b * p + c] = ((runs[0][col] + runs[1][col]) + runs[2][col]) + runs[3][col];
}

// `wgs` workgroups in launches of at most kMaxGrid (a launch holds fewer than
// 2^32 threads); go(first, count) launches some of them.
constexpr int64_t kMaxGrid = 1 << 20;
template <typename Go>
hipError_t in_launches(int64_t wgs, Go go) {
    for (int64_t at = 0; at < wgs; at += kMaxGrid) {
        go(at, (uint32_t)std::min(wgs - at, kMaxGrid));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename E, bool Q, int TPR, int NCH>
hipError_t forward(const RmsArgs& a, hipStream_t s) {
    constexpr int rows = block_of<TPR>() / TPR;
    return in_launches((a.rows + rows - 1) / rows, [&](int64_t at, uint32_t n) {
        RmsArgs b = a;
        b.row0 = at * rows;
        hipLaunchKernelGGL((rmsnorm_kernel<E, TPR, NCH, Q>), dim3(n), dim3(block_of<TPR>()), 0, s, b);
    });
}
template <typename E, bool Q>
hipError_t forward(const RmsArgs& a, hipStream_t s) {
    const int p = a.p;
    if (p <= 64) return forward<E, Q, 8, 1>(a, s);
    if (p <= 128) return forward<E, Q, 16, 1>(a, s);
    if (p <= 256) return forward<E, Q, 32, 1>(a, s);
    if (p <= 512) return forward<E, Q, 64, 1>(a, s);
    if (p <= 1024) return forward<E, Q, 64, 2>(a, s);
    // A piece to a thread: [1024, 1536] 4.9 us, [16384, 2048] 39 (64 threads of
    // four pieces: 6.4 and 42).
    if (p <= 2048) return forward<E, Q, 256, 1>(a, s);
    // Longer rows: a piece to a thread while they are few and a row's latency
    // counts ([512, 4096] 6.9 us, by 256 threads 7.8); then fewer, busier threads,
    // with less waiting at the reductions ([2048, 4096] 12.2 us, a piece to a thread
    // 13.3; with residual and xhat [16384, 5120] 151 us, a piece to a thread 174, by
    // 256 threads of four pieces 160; in float32 335, 331 and 345).
    const bool few = a.rows <= 512;
    if (p <= 4096) return few ? forward<E, Q, 512, 1>(a, s) : forward<E, Q, 256, 2>(a, s);
    if constexpr (Q) {
        // 8-bit rows, whose quotients want registers and the vector unit: a piece
        // to a thread for many rows too (with residual, xhat and groups of 128
        // [16384, 5120] 192 us, in float32 343; by 256 threads of four pieces 226 and 393).
        if (p <= 6144) return forward<E, Q, 768, 1>(a, s);
        if (p <= 8192) return forward<E, Q, 1024, 1>(a, s);
    } else {
        if (p <= 8192) return few ? forward<E, Q, 1024, 1>(a, s) : forward<E, Q, 512, 2>(a, s);
    }
    if (p <= 16384) return forward<E, Q, 1024, 2>(a, s);
    return forward<E, Q, 1024, 4>(a, s);
}
template <typename E>
hipError_t forward(const RmsArgs& a, hipStream_t s) {
    return a.q ? forward<E, true>(a, s) : forward<E, false>(a, s);
}

template <typename E, int TPR, int NCH, int BLOCK = block_of<TPR>()>
hipError_t backward(const RmsGradArgs& a, hipStream_t s) {
    constexpr int rows = BLOCK / TPR;
    static_assert(rows % rms_rows_at_once(8 * TPR * NCH) == 0, "the host's plan of a sample's rows");
    const int64_t per = a.solo ? rows : 1;
    return in_launches((a.B * a.chunks + per - 1) / per, [&](int64_t at, uint32_t n) {
        RmsGradArgs b = a;
        b.seg0 = at * per;
        hipLaunchKernelGGL((rmsnorm_grad_kernel<E, TPR, NCH, BLOCK>), dim3(n), dim3(BLOCK), 0, s, b);
    });
}
template <typename E>
hipError_t backward(const RmsGradArgs& a, hipStream_t s) {
    const int p = a.p;
    if (p <= 64) return backward<E, 8, 1>(a, s);
    if (p <= 128) return backward<E, 16, 1>(a, s);
    if (p <= 256) return backward<E, 32, 1>(a, s);
    // Where there is a workgroup to a CU at most, it takes as many rows at once as
    // its registers allow, 16 or 8 instead of 4: bf16 [32, 128, 768] 8.3 to 9.3 us
    // instead of 11.8, [16, 33, 300] 5.8 and 9.9, float32 [16, 197, 777] 12.6 and 15.0.  With
    // more, small workgroups fill the CUs better: [8, 1024, 768] 16.3 and 15.0, [2000,
    // 20, 512] 35 and 27.
    const bool few = !a.solo && a.B * a.chunks <= 256;
    if (p > 256 && p <= 512 && few) return backward<E, 64, 1, 1024>(a, s);
    if (p > 512 && p <= 1024 && few) return backward<E, 64, 2, 512>(a, s);
    if (p <= 512) return backward<E, 64, 1>(a, s);
    // Short rows: a wave to a row, several rows at once ([4096, 768] by four waves
    // 11.6 us; by 128 threads of one piece 18.1).  Long ones: a piece to a thread, which leaves
    // the registers to fetch the next row ([16384, 4096] 110 us; by 256 threads of
    // two pieces 124).
    if (p <= 1024) return backward<E, 64, 2>(a, s);
    if (p <= 2048) return backward<E, 256, 1>(a, s);
    if (p <= 4096) return backward<E, 512, 1>(a, s);
    if (p <= 8192) return backward<E, 1024, 1>(a, s);
    if (p <= 16384) return backward<E, 1024, 2>(a, s);
    return backward<E, 1024, 4>(a, s);
}

}  // namespace

hipError_t launch_rmsnorm(const RmsArgs& a, bool bf16, hipStream_t s) {
    return bf16 ? forward<bf16_t>(a, s) : forward<float>(a, s);
}

hipError_t launch_rmsnorm_grad(const RmsGradArgs& a, bool bf16, hipStream_t s) {
    hipError_t e = bf16 ? backward<bf16_t>(a, s) : backward<float>(a, s);
    if (e != hipSuccess || !a.P || a.chunks <= 1) return e;
    const int cb = (a.p + 63) / 64;
    return in_launches(a.B * cb, [&](int64_t at, uint32_t n) {
        hipLaunchKernelGGL(rmsnorm_grad_join_kernel, dim3(n), dim3(256), 0, s, a.part, a.P, a.chunks, a.p, at, cb);
    });
}

}  // namespace bk
