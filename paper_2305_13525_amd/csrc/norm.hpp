// Layer norm for gfx950, forward and backward.
//   forward   s = x + r;  y = (s - mean) rstd gamma + beta
//   backward  h = (s - mean) rstd, g = dy gamma;  dx = r + rstd (g - c1 - h c2), c1 = mean(g), c2 = mean(g h);
//             dgamma = sum over rows of dy h, dbeta = sum over rows of dy
// All of it moves each element once or twice and computes some ten operations on it: bound by memory.  Rows are therefore kept in registers between
// their statistics and their outputs, and as many lanes share a row as leave each of them whole 16-byte loads.
// Measured, bf16 with a residual: forward 4096 x 12288 75.8 us (5.3 TB/s; a large copy reaches 4.8), one row of 4096 3.1 us; backward 8192 x 7168 97.7 us with
// dgamma and dbeta (4.8 TB/s), 1001 x 1027 in fp32 9.9 us, two launches of 6.9 and 2.7 to 3.7.  In halves, a shard of 8192 x 3584 of two: statistics with a residual 35 us
// bf16 and 61 fp32 (5.0 and 5.7 TB/s), the other half 33 and 43 (3.6, 4.1); backward 31 and 48 (3.8, 3.6: a second launch), 46 and 75 (5.2, 5.5).  4096 x 1536 of
// eight: 8.3 and 16.7, 17.7 and 19.2 (every lane reads the row's eight pairs, twice, ahead of its output; of 2048 columns 11.5 with two and 13.7 with four), 11.6 and 14.2, 12.1 and 20.0.
#pragma once
#include <type_traits>

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
    float* partial;              // [slices x 2 x partial_cols] column sums of row slices
    int64_t partial_cols;        // K, up to a whole chunk
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

// The sum of a value over groups of LANES lanes, the same in all lanes of a group: inside 16 lanes by the exchanges that an addition takes along, between them through
// the LDS crossbar.
template <int LANES>
__device__ __forceinline__ float lanes_sum(float v) {
    auto with = [](float x, auto ctrl) __attribute__((always_inline)) {
        return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), decltype(ctrl)::value, 0xF, 0xF, true));
    };
    if constexpr (LANES >= 2) v = with(v, std::integral_constant<int, 0xB1>{});    // quad: 1 0 3 2
    if constexpr (LANES >= 4) v = with(v, std::integral_constant<int, 0x4E>{});    // quad: 2 3 0 1
    if constexpr (LANES >= 8) v = with(v, std::integral_constant<int, 0x141>{});   // mirrored halves of 16
    if constexpr (LANES >= 16) v = with(v, std::integral_constant<int, 0x140>{});  // mirrored 16
    const int lane = threadIdx.x & 63;
    if constexpr (LANES >= 32) v += __int_as_float(__builtin_amdgcn_ds_bpermute((lane ^ 16) * 4, __float_as_int(v)));
    if constexpr (LANES >= 64) v += __int_as_float(__builtin_amdgcn_ds_bpermute((lane ^ 32) * 4, __float_as_int(v)));
    return v;
}

// Sums of a workgroup's values, the same in every thread and in a fixed order; `lds`: a float per wave and value.
template <int THREADS, int N>
__device__ __forceinline__ void block_sums(float (&v)[N], float* lds) {
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = lanes_sum<64>(v[n]);
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

// ---- rows that fit the registers of the lanes that share them -----------------------------------
// LANES lanes hold a row, chunk j * LANES + lane of eight values in the lane's j-th of CH chunks, so that lanes beside each other load 16 bytes beside
// each other.  Up to 64 lanes are a part of a wave or a wave, which needs no barrier; more are whole waves of a workgroup.
template <typename T>
struct RawChunk;
template <>
struct RawChunk<bf16_t> {
    u32x4 w;
    __device__ __forceinline__ void load(const bf16_t* p) { w = *reinterpret_cast<const u32x4*>(p); }
    __device__ __forceinline__ float at(int i) const { return __uint_as_float(i % 2 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16); }
    __device__ __forceinline__ void keep(int n) {  // the first n values, zeros behind them
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] &= n >= 2 * i + 2 ? 0xFFFFFFFFu : n == 2 * i + 1 ? 0xFFFFu : 0u;
    }
};
template <>
struct RawChunk<float> {
    f32x4 lo, hi;
    __device__ __forceinline__ void load(const float* p) {
        lo = *reinterpret_cast<const f32x4*>(p);
        hi = *reinterpret_cast<const f32x4*>(p + 4);
    }
    __device__ __forceinline__ float at(int i) const { return i < 4 ? lo[i % 4] : hi[i % 4]; }
    __device__ __forceinline__ void keep(int n) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            lo[i] = n > i ? lo[i] : 0.f;
            hi[i] = n > i + 4 ? hi[i] : 0.f;
        }
    }
};
// What was loaded is taken to be something new from here on: nothing that was formed of it earlier is kept.
__device__ __forceinline__ void pin_chunk(RawChunk<bf16_t>& r) { asm volatile("" : "+v"(r.w)); }
__device__ __forceinline__ void pin_chunk(RawChunk<float>& r) { asm volatile("" : "+v"(r.lo), "+v"(r.hi)); }
// One row that a whole wave works on: a buffer descriptor that ends with it, so that what lies behind the row's end reads as zero and is not written, and lanes need
// no more than the offset of their chunk.  The range check works in dwords: of an odd number of bf16 values the one behind the last is
// read and has to be masked, and the last one is stored on its own.
template <typename T>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t row_buffer(const T* row, int n) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(row), 0, (int)((n * sizeof(T) + 3) & ~(size_t)3), 0x00020000);
}
__device__ __forceinline__ void load_from(__amdgpu_buffer_rsrc_t b, int c, RawChunk<bf16_t>& r) {
    r.w = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(b, c * 2, 0, 0));
}
__device__ __forceinline__ void load_from(__amdgpu_buffer_rsrc_t b, int c, RawChunk<float>& r) {
    r.lo = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(b, c * 4, 0, 0));
    r.hi = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(b, c * 4 + 16, 0, 0));
}

// A lane's chunks of a row.  Where lanes of a wave have different rows a chunk that lies behind its row's end is the first one in its place, and a chunk that the row ends in
// reads on into the row's padding; only the last row may have none (`last`): its last chunk is fetched value by value.  mask() puts zeros in the
// place of what is not the row's.
template <typename T, int LANES, int CH>
struct RowChunks {
    RawChunk<T> raw[CH];
    __device__ __forceinline__ void load(const T* row, int K, int lane, bool last) {
        if constexpr (LANES >= 64) {
            const __amdgpu_buffer_rsrc_t b = row_buffer(row, K);
#pragma unroll
            for (int j = 0; j < CH; ++j) load_from(b, (j * LANES + lane) * 8, raw[j]);
        } else {
            static_assert(CH == 1, "short rows");
            const int c = lane * 8;
            const bool whole = c + 8 <= K || (c < K && !last);
            if (whole || K >= 8) raw[0].load(row + (whole ? c : 0));
            else raw[0] = RawChunk<T>{};
            if (c < K && !whole) {
                float v[8];
                load_chunk(row + c, K - c, v);
                set(raw[0], v);
            }
        }
    }
    static __device__ __forceinline__ void set(RawChunk<bf16_t>& r, const float (&v)[8]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) r.w[i] = __float_as_uint(v[2 * i]) >> 16 | (__float_as_uint(v[2 * i + 1]) & 0xFFFF0000u);
    }
    static __device__ __forceinline__ void set(RawChunk<float>& r, const float (&v)[8]) {
        r.lo = f32x4{v[0], v[1], v[2], v[3]};
        r.hi = f32x4{v[4], v[5], v[6], v[7]};
    }
    __device__ __forceinline__ void mask(int K, int lane) {
        if (LANES >= 64 && (sizeof(T) == 4 || K % 2 == 0)) return;
        asm volatile("" : "+v"(lane));  // in a loop over rows the masks would be kept, four registers a chunk
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int left = K - (j * LANES + lane) * 8;
            if (left < 8) raw[j].keep(left);
        }
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int j = 0; j < CH; ++j) raw[j] = RawChunk<T>{};
    }
};
// Eight values of chunk c of a row.
template <int LANES, typename T>
__device__ __forceinline__ void store_in_row(T* row, int K, int c, const float (&v)[8]) {
    if constexpr (LANES < 64) {
        if (c < K) store_chunk(row + c, K - c, v);
    } else if constexpr (sizeof(T) == 4) {
        const __amdgpu_buffer_rsrc_t b = row_buffer(row, K);
        const f32x4 lo = {v[0], v[1], v[2], v[3]}, hi = {v[4], v[5], v[6], v[7]};
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, lo), b, c * 4, 0, 0);
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, hi), b, c * 4 + 16, 0, 0);
    } else {
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
        __builtin_amdgcn_raw_buffer_store_b128(w, row_buffer(row, K & ~1), c * 2, 0, 0);
        if (K % 2 != 0 && c < K && c + 8 > K) {
            const int d = (K - 1 - c) / 2;
            row[K - 1] = (bf16_t)(d == 0 ? w[0] : d == 1 ? w[1] : d == 2 ? w[2] : w[3]);
        }
    }
}
// Sums over the LANES lanes of a row, the same in all of them.  `lds`: N floats per wave, used by rows of several waves; a caller that comes back without a
// barrier in between alternates between two of them.
template <int LANES, int N>
__device__ __forceinline__ void row_sums(float (&v)[N], float* lds) {
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = lanes_sum<(LANES < 64 ? LANES : 64)>(v[n]);
    if constexpr (LANES > 64) {
        constexpr int WAVES = LANES / 64;
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, first = wave / WAVES * WAVES;
        if (lane == 0)
#pragma unroll
            for (int n = 0; n < N; ++n) lds[wave * N + n] = v[n];
        __syncthreads();
        constexpr int SPAN = WAVES <= 2 ? 2 : WAVES <= 4 ? 4 : WAVES <= 8 ? 8 : 16;
        static_assert(WAVES <= SPAN, "waves of a workgroup");
        const int w = lane % SPAN;
#pragma unroll
        for (int n = 0; n < N; ++n) v[n] = w < WAVES ? lds[(first + w) * N + n] : 0.f;
#pragma unroll
        for (int n = 0; n < N; ++n) v[n] = lanes_sum<SPAN>(v[n]);
    }
}

// Which of a workgroup's rows a thread works on; the compiler is told where that is the same for a whole wave, and addresses rows by scalars then.
template <int LANES>
__device__ __forceinline__ int row_group() {
    return LANES < 64 ? (int)threadIdx.x / LANES : __builtin_amdgcn_readfirstlane((int)threadIdx.x / LANES);
}

// Forward.  The squared deviations are summed up from the registers once the mean is known, which costs a second exchange among the lanes and no memory; x^2 - mean^2
// would cancel where a row's mean is large.
template <typename T, int LANES, int CH>
__global__ void __launch_bounds__(LANES <= 64 ? 256 : LANES) norm_rows_kernel(NormArgs g) {
    constexpr int BLOCK = LANES <= 64 ? 256 : LANES, ROWS = BLOCK / LANES;
    static_assert(LANES <= 64 || ROWS == 1, "rows of several waves meet at barriers");
    __shared__ float lds[2][BLOCK / 64];
    const int lane = threadIdx.x % LANES;
    // (the descriptors of rows are scalars: a row is the same for a whole wave where LANES >= 64)
    for (int64_t row = (int64_t)blockIdx.x * ROWS + row_group<LANES>(); row < g.M; row += (int64_t)gridDim.x * ROWS) {
        const bool last = row == g.M - 1;
        RowChunks<T, LANES, CH> x, r;
        x.load(static_cast<const T*>(g.X) + row * g.ldx, g.K, lane, last);
        if (g.R) r.load(static_cast<const T*>(g.R) + row * g.ldr, g.K, lane, last);
        RowChunks<bf16_t, LANES, CH> gamma, beta;  // the same for all rows, from the caches
        if (g.gamma) gamma.load(g.gamma, g.K, lane, true);
        if (g.beta) beta.load(g.beta, g.K, lane, true);
        x.mask(g.K, lane);
        if (g.R) r.mask(g.K, lane);
        float v[CH][8];
        float sum[1] = {0.f};
#pragma unroll
        for (int j = 0; j < CH; ++j) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[j][i] = x.raw[j].at(i);
            if (g.R) {
                float s[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    s[i] = v[j][i] + r.raw[j].at(i);
                    v[j][i] = stored(s[i], static_cast<const T*>(nullptr));
                }
                store_in_row<LANES>(static_cast<T*>(g.S) + row * g.lds, g.K, (j * LANES + lane) * 8, s);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[0] += v[j][i];
        }
        float mean, rstd;
        if (g.phase == NORM_APPLY) join_parts(g, (int)row, mean, rstd);
        else {
            row_sums<LANES>(sum, lds[0]);
            mean = sum[0] / (float)g.K;
            sum[0] = 0.f;
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                const int left = g.K - (j * LANES + lane) * 8;
                if (left >= 8)
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum[0] += (v[j][i] - mean) * (v[j][i] - mean);
                else
#pragma unroll
                    for (int i = 0; i < 7; ++i) sum[0] += i < left ? (v[j][i] - mean) * (v[j][i] - mean) : 0.f;
            }
            row_sums<LANES>(sum, lds[1]);
            if (g.phase == NORM_PART) {
                if (lane == 0) g.part[row] = float2{mean, sum[0]};
                continue;
            }
            rstd = 1.0f / sqrtf(sum[0] / (float)g.K + g.eps);
        }
        if (lane == 0 && g.stats) g.stats[row] = float2{mean, rstd};
#pragma unroll
        for (int j = 0; j < CH; ++j) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[j][i] = (v[j][i] - mean) * rstd;
                if (g.gamma) v[j][i] *= gamma.raw[j].at(i);
                if (g.beta) v[j][i] += beta.raw[j].at(i);
            }
            store_in_row<LANES>(g.Y + row * g.ldy, g.K, (j * LANES + lane) * 8, v[j]);
        }
    }
}

// Rows of any length, a workgroup to a row, which it reads once for the mean, once for the deviations and once for the output, the second and third time mostly from the
// caches (512 x 40000 bf16 26 us, 3.1 TB/s of what has to be moved).
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

// Backward on rows in registers, one pass over the data: a workgroup of GROUPS rows at a time walks the rows, every lane keeps the sums of its columns of dgamma and
// dbeta as it goes, and the next row's loads are under way while this row's sums meet.  At its end a workgroup adds its groups' columns up through
// LDS, in order, and writes them to `partial`, which norm_join_kernel adds up: no atomics, the same bits every time.  There are no more workgroups than CUs,
// because each leaves two rows of sums (twice as many: 8192 x 4096 54 us and 59, 4096 x 8192 60 and 67).
template <typename T, int LANES, int CH, int GROUPS>
__global__ void __launch_bounds__(LANES * GROUPS) norm_bwd_rows_kernel(NormBwdArgs g) {
    constexpr int BLOCK = LANES * GROUPS;
    constexpr bool AHEAD = sizeof(T) == 2 || LANES * CH < 2048;  // four chunks of fp32 values leave no registers for the next row's
    __shared__ float lds[2][2 * (BLOCK / 64)];
    __shared__ __attribute__((aligned(16))) float cols[GROUPS > 1 ? BLOCK * 8 : 4];
    const int lane = threadIdx.x % LANES, group = row_group<LANES>();
    const bool want_cols = g.phase != NORM_APPLY && (g.dgamma || g.dbeta), want_sums = g.phase != NORM_APPLY;
    float dg[CH][8], db[CH][8];
    RowChunks<bf16_t, LANES, CH> gm;
    if (g.gamma) {
        gm.load(g.gamma, g.K, lane, true);
        gm.mask(g.K, lane);
    }
#pragma unroll
    for (int j = 0; j < CH; ++j) {
#pragma unroll
        for (int i = 0; i < 8; ++i) dg[j][i] = db[j][i] = 0.f;
        if (!g.gamma) gm.raw[j].w = u32x4{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};  // ones
    }
    const int64_t step = (int64_t)gridDim.x * GROUPS;
    RowChunks<T, LANES, CH> x;
    RowChunks<bf16_t, LANES, CH> dy;
    float2 st;
    auto request = [&](int64_t row) __attribute__((always_inline)) {  // rows beyond the last stand for it
        row = min(row, (int64_t)g.M - 1);
        const bool last = row == g.M - 1;
        st = g.stats[row];
        x.load(static_cast<const T*>(g.S) + row * g.lds, g.K, lane, last);
        dy.load(g.dY + row * g.lddy, g.K, lane, last);
    };
    request((int64_t)blockIdx.x * GROUPS + group);
    int turn = 0;
    for (int64_t row0 = (int64_t)blockIdx.x * GROUPS; row0 < g.M; row0 += step, turn ^= 1) {  // as many turns for every group
        const int64_t row = row0 + group;
        const bool here = row < g.M;
        if (!AHEAD && row0 >= step) request(row);
        RowChunks<T, LANES, CH> xs = x;
        RowChunks<bf16_t, LANES, CH> ys = dy;
        const float2 stats = st;
        auto h_of = [&](int j, int i) __attribute__((always_inline)) { return (xs.raw[j].at(i) - stats.x) * stats.y; };
        xs.mask(g.K, lane);
        ys.mask(g.K, lane);  // with dY zero there, a row or a column that is not there adds nothing
        if (!here) ys.clear();
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < CH; ++j) pin_chunk(gm.raw[j]);  // kept as it is loaded, not as eight registers of fp32
#pragma unroll
        for (int j = 0; j < CH; ++j) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float y = ys.raw[j].at(i), h = h_of(j, i), d = y * gm.raw[j].at(i);
                dg[j][i] += y * h;
                db[j][i] += y;
                asm volatile("" : "+v"(dg[j][i]), "+v"(db[j][i]));  // here: put off, they would keep h and y in registers
                sum[0] += d;
                sum[1] += d * h;
            }
        }
        RowChunks<T, LANES, CH> r;
        if (g.R) r.load(static_cast<const T*>(g.R) + min(row, (int64_t)g.M - 1) * g.ldr, g.K, lane, row >= g.M - 1);
        if (AHEAD && row0 + step < g.M) request(row + step);
        if (want_sums) row_sums<LANES>(sum, lds[turn]);
        if (!here) continue;
        if (g.phase == NORM_PART) {
            if (lane == 0) g.sums[row] = float2{sum[0], sum[1]};
            continue;
        }
        if (g.phase == NORM_APPLY) {
            sum[0] = g.sums[row].x;
            sum[1] = g.sums[row].y;
        }
        const float c1 = sum[0] * g.per_row, c2 = sum[1] * g.per_row;
        // h and dy gamma are formed again from what was loaded: kept in fp32 they would be twice to four times the registers
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            pin_chunk(xs.raw[j]);
            pin_chunk(ys.raw[j]);
            pin_chunk(gm.raw[j]);
        }
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            float d[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                d[i] = stats.y * (ys.raw[j].at(i) * gm.raw[j].at(i) - c1 - h_of(j, i) * c2);
                if (g.R) d[i] += r.raw[j].at(i);
            }
            store_in_row<LANES>(static_cast<T*>(g.dX) + row * g.lddx, g.K, (j * LANES + lane) * 8, d);
        }
    }
    if (!want_cols) return;
    constexpr int COLS = LANES * 8;  // of a chunk of all lanes
#pragma unroll
    for (int what = 0; what < 2; ++what) {
        float* const to = g.partial + ((int64_t)blockIdx.x * 2 + what) * g.partial_cols;
        if constexpr (GROUPS > 1) {
            static_assert(CH == 1, "a chunk per lane");
            __syncthreads();
            float* const mine = cols + group * COLS + lane * 8;
            *reinterpret_cast<f32x4*>(mine) = what ? f32x4{db[0][0], db[0][1], db[0][2], db[0][3]} : f32x4{dg[0][0], dg[0][1], dg[0][2], dg[0][3]};
            *reinterpret_cast<f32x4*>(mine + 4) = what ? f32x4{db[0][4], db[0][5], db[0][6], db[0][7]} : f32x4{dg[0][4], dg[0][5], dg[0][6], dg[0][7]};
            __syncthreads();
            for (int c = threadIdx.x; c < COLS && c < g.K; c += BLOCK) {
                float v = 0.f;
#pragma unroll
                for (int q = 0; q < GROUPS; ++q) v += cols[q * COLS + c];
                to[c] = v;
            }
        } else {
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                const int c = (j * LANES + lane) * 8;
                if (c >= g.K) continue;
                const float(&v)[8] = what ? db[j] : dg[j];
                *reinterpret_cast<f32x4*>(to + c) = f32x4{v[0], v[1], v[2], v[3]};
                *reinterpret_cast<f32x4*>(to + c + 4) = f32x4{v[4], v[5], v[6], v[7]};
            }
        }
    }
}

// dX of rows of any length, a workgroup to a row, which it reads once for the two sums and once for the output (512 x 40000 bf16 67 us with the columns' sums, which
// norm_cols_kernel reads the data for again).
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

// dgamma and dbeta of strips of 64 columns over slices of the rows: 8 lanes of 8 columns by 32 rows at a time.  The sums of a slice
// go to `partial`, which norm_join_kernel adds up in ascending order of the slices.
constexpr int NORM_STRIP = 64, NORM_COL_THREADS = 256, NORM_COL_ROWS = NORM_COL_THREADS / (NORM_STRIP / 8);
template <typename T>
__global__ void __launch_bounds__(NORM_COL_THREADS) norm_cols_kernel(NormBwdArgs g) {
    __shared__ float lds[2][NORM_COL_THREADS / 64][NORM_STRIP];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t pieces = ((int64_t)g.K + NORM_STRIP - 1) / NORM_STRIP * g.slices;
    for (int64_t piece = blockIdx.x; piece < pieces; piece += gridDim.x) {
        const int64_t strip = piece / g.slices, slice = piece % g.slices;
        const int64_t col = strip * NORM_STRIP + (lane & 7) * 8;
        const int valid = (int)min((int64_t)8, g.K - col);
        float dg[8], db[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) dg[i] = db[i] = 0.f;
        const int64_t end = min((int64_t)g.M, (slice + 1) * g.rows_per_slice);
        if (valid > 0)
            for (int64_t row = slice * g.rows_per_slice + (threadIdx.x >> 3); row < end; row += NORM_COL_ROWS) {
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
        __syncthreads();  // the last piece's sums have been read
        if (lane < 8)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                lds[0][wave][lane * 8 + i] = dg[i];
                lds[1][wave][lane * 8 + i] = db[i];
            }
        __syncthreads();
        if (threadIdx.x < 2 * NORM_STRIP) {
            const int what = threadIdx.x / NORM_STRIP, c = threadIdx.x % NORM_STRIP;
            float sum = 0.f;
#pragma unroll
            for (int w = 0; w < NORM_COL_THREADS / 64; ++w) sum += lds[what][w][c];
            const int64_t at = strip * NORM_STRIP + c;
            if (at < g.K) g.partial[(slice * 2 + what) * g.partial_cols + at] = sum;
        }
    }
}
// The sums of all slices, added in an order that depends on their number alone: of 32 columns, eight lanes of 16 bytes, a lane to every 128th slice; the lanes of a wave
// meet by exchanges and the waves in LDS.  dgamma and dbeta lie behind each other.  (256 slices of 7168 columns 5.0 to 5.5 us, 2.7 TB/s and more; with a word a
// lane and sums stored a word at a time 64 x 16384 took 25 us as a whole, now 15.)
constexpr int NORM_JOIN_THREADS = 1024, NORM_JOIN_COLS = 32;
__global__ void __launch_bounds__(NORM_JOIN_THREADS) norm_join_kernel(NormBwdArgs g) {
    constexpr int LANES = NORM_JOIN_THREADS * 4 / NORM_JOIN_COLS, WAVES = NORM_JOIN_THREADS / 64;
    __shared__ __attribute__((aligned(16))) float lds[WAVES][NORM_JOIN_COLS];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t both = 2 * g.partial_cols;
    for (int64_t from = (int64_t)blockIdx.x * NORM_JOIN_COLS; from < both; from += (int64_t)gridDim.x * NORM_JOIN_COLS) {
        const int64_t col = from + (lane & 7) * 4;
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
        if (col < both)
            for (int s = threadIdx.x >> 3; s < g.slices; s += LANES) sum += *reinterpret_cast<const f32x4*>(g.partial + s * both + col);
#pragma unroll
        for (int m = 8; m < 64; m <<= 1)
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] += __shfl_xor(sum[i], m, 64);
        __syncthreads();  // the last columns' sums have been read
        if (lane < 8) *reinterpret_cast<f32x4*>(&lds[wave][lane * 4]) = sum;
        __syncthreads();
        const int64_t at = from + threadIdx.x;
        if (threadIdx.x >= NORM_JOIN_COLS || at >= both) continue;
        const bool first = at < g.partial_cols;
        float* const out = first ? g.dgamma : g.dbeta;
        const int64_t c = first ? at : at - g.partial_cols;
        if (!out || c >= g.K) continue;
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) v += lds[w][threadIdx.x];
        out[c] = g.accumulate ? out[c] + v : v;
    }
}

}  // namespace axo
