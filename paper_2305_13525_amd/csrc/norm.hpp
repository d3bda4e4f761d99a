// Layer norm for gfx950, forward and backward.
//   forward   s = x + r;  y = (s - mean) rstd gamma + beta
//   backward  h = (s - mean) rstd, g = dy gamma;  dx = r + rstd (g - c1 - h c2), c1 = mean(g), c2 = mean(g h);
//             dgamma = sum over rows of dy h, dbeta = sum over rows of dy
// All of it moves each element once or twice and computes some ten operations on it: bound by memory.
#pragma once
#include "axo_common.hpp"

namespace axo {

// What a call does: all of it on whole rows, or one half of it on a shard's columns of them.
enum NormPhase { NORM_WHOLE = 0, NORM_PART = 1, NORM_APPLY = 2 };

struct NormArgs {
    const void* X; int64_t ldx;
    const void* R; int64_t ldr;  // nullptr: none
    void* S; int64_t lds;        // written where R is
    const bf16_t* gamma;         // nullptr: ones
    const bf16_t* beta;          // nullptr: zeros
    bf16_t* Y; int64_t ldy;
    float2* stats;               // (mean, rstd) per row, or nullptr
    float2* part;                // NORM_PART: (mean, sum of squared deviations) per row, written
    const float2* parts;         // NORM_APPLY: [n_parts x M] of them, read
    int n_parts;
    int M, K;                    // rows, columns here
    float eps;
    int phase;
};

struct NormBwdArgs {
    const bf16_t* dY; int64_t lddy;
    const void* S; int64_t lds;
    const void* R; int64_t ldr;  // nullptr: none
    const bf16_t* gamma;
    const float2* stats;
    float2* sums;                // (sum of g, sum of g h) per row: NORM_PART writes them, NORM_APPLY reads them
    void* dX; int64_t lddx;
    float* dgamma;               // either may be nullptr
    float* dbeta;
    int accumulate;
    float* partial;              // [slices x 2 x K] column sums of row slices
    int slices, rows_per_slice;
    int M, K;                    // rows, columns here
    float per_row;               // 1 / columns of the whole row
    int phase;
};

// Eight consecutive values of a row, the first `valid` (1..8) of them inside the matrix; the others read as zero.
__device__ __forceinline__ void load_chunk(const bf16_t* p, int valid, float (&v)[8]) {
    if (valid >= 8) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < valid ? bf16_bits_to_f32(p[i]) : 0.f;
    }
}
__device__ __forceinline__ void load_chunk(const float* p, int valid, float (&v)[8]) {
    if (valid >= 8) {
        const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[i] = a[i];
            v[4 + i] = b[i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < valid ? p[i] : 0.f;
    }
}
__device__ __forceinline__ void store_chunk(bf16_t* p, int valid, const float (&v)[8]) {
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
    if (valid >= 8) *reinterpret_cast<u32x4*>(p) = w;
    else
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (i < valid) p[i] = (bf16_t)(w[i / 2] >> (i % 2 * 16));
}
__device__ __forceinline__ void store_chunk(float* p, int valid, const float (&v)[8]) {
    if (valid >= 8) {
        *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
        *reinterpret_cast<f32x4*>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
    } else
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (i < valid) p[i] = v[i];
}
// A value as it is stored and read again.
__device__ __forceinline__ float stored(float v, const float*) { return v; }
__device__ __forceinline__ float stored(float v, const bf16_t*) { return __uint_as_float(pack_bf16x2(v, 0.f) << 16); }

// Sums of a workgroup's values, the same in every thread and in a fixed order; `lds`: a float per wave and value.
template <int THREADS, int N>
__device__ __forceinline__ void block_sums(float (&v)[N], float* lds) {
#pragma unroll
    for (int m = 1; m < 64; m <<= 1)
#pragma unroll
        for (int n = 0; n < N; ++n) v[n] += __shfl_xor(v[n], m, 64);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (lane == 0)
#pragma unroll
        for (int n = 0; n < N; ++n) lds[wave * N + n] = v[n];
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n) {
        v[n] = 0.f;
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w) v[n] += lds[w * N + n];
    }
    __syncthreads();
}

// Statistics of a row from those of its n parts of K columns each.  The squared deviations from the parts' own means and those of the
// means themselves add up without cancellation.
__device__ __forceinline__ void join_parts(const NormArgs& g, int row, float& mean, float& rstd) {
    mean = 0.f;
    for (int i = 0; i < g.n_parts; ++i) mean += g.parts[(int64_t)i * g.M + row].x;
    mean /= (float)g.n_parts;
    float m2 = 0.f;
    for (int i = 0; i < g.n_parts; ++i) {
        const float2 q = g.parts[(int64_t)i * g.M + row];
        m2 += q.y + (q.x - mean) * (q.x - mean) * (float)g.K;
    }
    rstd = 1.0f / sqrtf(m2 / ((float)g.K * (float)g.n_parts) + g.eps);
}

// Rows of any length, a workgroup to a row, which it reads once for the mean, once for the deviations and once for the output.
constexpr int NORM_THREADS = 1024;
template <typename T>
__global__ void __launch_bounds__(NORM_THREADS) norm_long_kernel(NormArgs g) {
    __shared__ float lds[NORM_THREADS / 64];
    for (int64_t row = blockIdx.x; row < g.M; row += gridDim.x) {
        const T* x = static_cast<const T*>(g.X) + row * g.ldx;
        float mean = 0.f, rstd = 0.f;
        if (g.R) {
            T* const s = static_cast<T*>(g.S) + row * g.lds;
            for (int64_t c = threadIdx.x * 8; c < g.K; c += NORM_THREADS * 8) {
                const int valid = (int)min((int64_t)8, g.K - c);
                float v[8], r[8];
                load_chunk(x + c, valid, v);
                load_chunk(static_cast<const T*>(g.R) + row * g.ldr + c, valid, r);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] += r[i];
                store_chunk(s + c, valid, v);
            }
            x = s;  // a thread reads back what it wrote itself
        }
        if (g.phase == NORM_APPLY) join_parts(g, (int)row, mean, rstd);
        else {
            float sum[1] = {0.f};
            for (int64_t c = threadIdx.x * 8; c < g.K; c += NORM_THREADS * 8) {
                float v[8];
                load_chunk(x + c, (int)min((int64_t)8, g.K - c), v);
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[0] += v[i];
            }
            block_sums<NORM_THREADS>(sum, lds);
            mean = sum[0] / (float)g.K;
            sum[0] = 0.f;
            for (int64_t c = threadIdx.x * 8; c < g.K; c += NORM_THREADS * 8) {
                const int valid = (int)min((int64_t)8, g.K - c);
                float v[8];
                load_chunk(x + c, valid, v);
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[0] += i < valid ? (v[i] - mean) * (v[i] - mean) : 0.f;
            }
            block_sums<NORM_THREADS>(sum, lds);
            if (g.phase == NORM_PART) {
                if (threadIdx.x == 0) g.part[row] = float2{mean, sum[0]};
                continue;
            }
            rstd = 1.0f / sqrtf(sum[0] / (float)g.K + g.eps);
        }
        if (threadIdx.x == 0 && g.stats) g.stats[row] = float2{mean, rstd};
        for (int64_t c = threadIdx.x * 8; c < g.K; c += NORM_THREADS * 8) {
            const int valid = (int)min((int64_t)8, g.K - c);
            float v[8], w[8];
            load_chunk(x + c, valid, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = (v[i] - mean) * rstd;
            if (g.gamma) {
                load_chunk(g.gamma + c, valid, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] *= w[i];
            }
            if (g.beta) {
                load_chunk(g.beta + c, valid, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] += w[i];
            }
            store_chunk(g.Y + row * g.ldy + c, valid, v);
        }
    }
}

// dX of rows of any length, a workgroup to a row, which it reads once for the two sums and once for the output.
template <typename T>
__global__ void __launch_bounds__(NORM_THREADS) norm_bwd_long_kernel(NormBwdArgs g) {
    __shared__ float lds[2 * NORM_THREADS / 64];
    for (int64_t row = blockIdx.x; row < g.M; row += gridDim.x) {
        const T* const s = static_cast<const T*>(g.S) + row * g.lds;
        const bf16_t* const dy = g.dY + row * g.lddy;
        const float2 st = g.stats[row];
        auto chunk = [&](int64_t c, int valid, float (&h)[8], float (&d)[8]) __attribute__((always_inline)) {  // h and g of the formula
            float w[8];
            load_chunk(s + c, valid, h);
            load_chunk(dy + c, valid, d);
#pragma unroll
            for (int i = 0; i < 8; ++i) h[i] = (h[i] - st.x) * st.y;
            if (!g.gamma) return;
            load_chunk(g.gamma + c, valid, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] *= w[i];
        };
        float c1, c2;
        if (g.phase == NORM_APPLY) {
            c1 = g.sums[row].x;
            c2 = g.sums[row].y;
        } else {
            float sum[2] = {0.f, 0.f};
            for (int64_t c = threadIdx.x * 8; c < g.K; c += NORM_THREADS * 8) {
                const int valid = (int)min((int64_t)8, g.K - c);
                float h[8], d[8];
                chunk(c, valid, h, d);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < valid) {
                        sum[0] += d[i];
                        sum[1] += d[i] * h[i];
                    }
            }
            block_sums<NORM_THREADS>(sum, lds);
            c1 = sum[0];
            c2 = sum[1];
            if (g.phase == NORM_PART) {
                if (threadIdx.x == 0) g.sums[row] = float2{c1, c2};
                continue;
            }
        }
        c1 *= g.per_row;
        c2 *= g.per_row;
        for (int64_t c = threadIdx.x * 8; c < g.K; c += NORM_THREADS * 8) {
            const int valid = (int)min((int64_t)8, g.K - c);
            float h[8], d[8], r[8];
            chunk(c, valid, h, d);
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] = st.y * (d[i] - c1 - h[i] * c2);
            if (g.R) {
                load_chunk(static_cast<const T*>(g.R) + row * g.ldr + c, valid, r);
#pragma unroll
                for (int i = 0; i < 8; ++i) d[i] += r[i];
            }
            store_chunk(static_cast<T*>(g.dX) + row * g.lddx + c, valid, d);
        }
    }
}

// dgamma and dbeta of a strip of 64 columns over a slice of the rows: 8 lanes of 8 columns by 32 rows at a time.  The sums of a slice
// go to `partial`, which norm_join_kernel adds up in ascending order of the slices.
constexpr int NORM_STRIP = 64, NORM_COL_THREADS = 256, NORM_COL_ROWS = NORM_COL_THREADS / (NORM_STRIP / 8);
template <typename T>
__global__ void __launch_bounds__(NORM_COL_THREADS) norm_cols_kernel(NormBwdArgs g) {
    __shared__ float lds[2][NORM_COL_THREADS / 64][NORM_STRIP];
    const int strip = blockIdx.x / g.slices, slice = blockIdx.x % g.slices;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t col = (int64_t)strip * NORM_STRIP + (lane & 7) * 8;
    const int valid = (int)min((int64_t)8, g.K - col);
    float dg[8], db[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) dg[i] = db[i] = 0.f;
    const int64_t end = min((int64_t)g.M, ((int64_t)slice + 1) * g.rows_per_slice);
    if (valid > 0)
        for (int64_t row = (int64_t)slice * g.rows_per_slice + (threadIdx.x >> 3); row < end; row += NORM_COL_ROWS) {
            float x[8], d[8];
            load_chunk(static_cast<const T*>(g.S) + row * g.lds + col, valid, x);
            load_chunk(g.dY + row * g.lddy + col, valid, d);
            const float2 st = g.stats[row];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                dg[i] += d[i] * ((x[i] - st.x) * st.y);
                db[i] += d[i];
            }
        }
#pragma unroll
    for (int m = 8; m < 64; m <<= 1)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            dg[i] += __shfl_xor(dg[i], m, 64);
            db[i] += __shfl_xor(db[i], m, 64);
        }
    if (lane < 8)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            lds[0][wave][lane * 8 + i] = dg[i];
            lds[1][wave][lane * 8 + i] = db[i];
        }
    __syncthreads();
    if (threadIdx.x >= 2 * NORM_STRIP) return;
    const int what = threadIdx.x / NORM_STRIP, c = threadIdx.x % NORM_STRIP;
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < NORM_COL_THREADS / 64; ++w) sum += lds[what][w][c];
    const int64_t at = (int64_t)strip * NORM_STRIP + c;
    if (at < g.K) g.partial[((int64_t)slice * 2 + what) * g.K + at] = sum;
}
__global__ void __launch_bounds__(256) norm_join_kernel(NormBwdArgs g) {
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= 2 * (int64_t)g.K) return;
    float* const out = at < g.K ? g.dgamma : g.dbeta;
    if (!out) return;
    float sum = 0.f;
    for (int s = 0; s < g.slices; ++s) sum += g.partial[(int64_t)s * 2 * g.K + at];
    const int64_t c = at < g.K ? at : at - g.K;
    out[c] = g.accumulate ? out[c] + sum : sum;
}

}  // namespace axo
