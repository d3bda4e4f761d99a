// The norms either side of a residual addition, with its gate and scale, for gfx950.
//   forward   ha = (b - mean_a) rstd_a;  z = ha gamma_a + beta_a;  s = x + scale gate z;  y = (s - mean_b) rstd_b gamma_b + beta_b
//   backward  hb = (s - mean_b) rstd_b, g = dy gamma_b;  ds' = ds + rstd_b (g - mean(g) - hb mean(g hb))        dx = ds'
//             q = scale gate gamma_a ds';                db = rstd_a (q - mean(q) - ha mean(q ha))
//             over rows  Y0 = sum dy hb, Y1 = sum dy, S0 = sum ds' ha, S1 = sum ds':
//             dgamma_b = Y0, dbeta_b = Y1, dgamma_a = scale gate S0, dbeta_a = scale gate S1, dgate = scale (gamma_a S0 + beta_a S1)
// A norm is a layer norm, that of the root mean square (mean_ = 0, and mean(g), mean(q) fall away), or none (rstd = 1, ha = b, db = q).
// The four matrices that go in or out are moved once and some thirty operations are done on an element: bound by memory.  Rows stay in registers from their first load
// to their last store, over both norms.
#pragma once
#include "norm.hpp"

namespace axo {

enum NormKind { KIND_NONE = 0, KIND_LAYER = 1, KIND_RMS = 2 };

struct ResnormArgs {
    const bf16_t* B; int64_t ldb;
    const void* X; int64_t ldx;
    void* S; int64_t lds;
    bf16_t* Y; int64_t ldy;
    const bf16_t *gamma_a, *beta_a, *gate, *gamma_b, *beta_b;  // nullptr: ones, zeros
    f32x4* stats;                                              // (mean_a, rstd_a, mean_b, rstd_b) per row, or nullptr
    int M, K, kind_a, kind_b;
    float scale, eps;
};

struct ResnormBwdArgs {
    const bf16_t* dY; int64_t lddy;
    const void* dS; int64_t ldds;  // nullptr: zeros
    const bf16_t* B; int64_t ldb;
    const void* S; int64_t lds;
    void* dX; int64_t lddx;
    bf16_t* dB; int64_t lddb;
    const bf16_t *gamma_a, *beta_a, *gate, *gamma_b;
    const f32x4* stats;
    float *dgamma_a, *dbeta_a, *dgate, *dgamma_b, *dbeta_b;  // any may be nullptr
    float* partial;        // [slices x 4 x partial_cols]: Y0, Y1, S0, S1 of row slices
    float2* means;         // (mean(g), mean(g hb)) per row, or nullptr: for resnorm_cols_kernel, whose
    uint32_t* counters;    // strips have one each
    int64_t partial_cols;  // K, up to a whole chunk
    int slices, rows_per_slice;
    int M, K, kind_a, kind_b, accumulate, want_cols;
    float scale;
};

// Eight values of a vector that all rows share, `other` where there is none.
__device__ __forceinline__ void vector_chunk(const bf16_t* p, int64_t c, int valid, float other, float (&v)[8]) {
    if (p) return load_chunk(p + c, valid, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = other;
}

// A lane's chunks of such a vector.
template <int LANES, int CH>
__device__ __forceinline__ void load_vector(RowChunks<bf16_t, LANES, CH>& to, const bf16_t* p, int K, int lane, uint32_t other) {
    if (p) {
        to.load(p, K, lane, true);
        to.mask(K, lane);
    } else
#pragma unroll
        for (int j = 0; j < CH; ++j) to.raw[j].w = u32x4{other, other, other, other};
}
constexpr uint32_t ONES = 0x3F803F80u;  // two bf16

// Mean and 1 / deviation of a row whose values the lanes hold, zeros behind its end.  The squared deviations are summed up once the mean is known.
template <int LANES, int CH>
__device__ __forceinline__ void row_moments(const float (&v)[CH][8], int K, int lane, int kind, float eps, float (&lds)[2][LANES <= 64 ? 4 : LANES / 64], float& mean, float& rstd) {
    mean = 0.f;
    rstd = 1.f;
    if (kind == KIND_NONE) return;
    float sum[1] = {0.f};
    if (kind == KIND_LAYER) {
#pragma unroll
        for (int j = 0; j < CH; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[0] += v[j][i];
        row_sums<LANES>(sum, lds[0]);
        mean = sum[0] / (float)K;
        sum[0] = 0.f;
    }
#pragma unroll
    for (int j = 0; j < CH; ++j) {
        const int left = K - (j * LANES + lane) * 8;
        if (left >= 8)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[0] += (v[j][i] - mean) * (v[j][i] - mean);
        else
#pragma unroll
            for (int i = 0; i < 7; ++i) sum[0] += i < left ? (v[j][i] - mean) * (v[j][i] - mean) : 0.f;
    }
    row_sums<LANES>(sum, lds[1]);
    rstd = 1.0f / sqrtf(sum[0] / (float)K + eps);
}

// Forward on rows in registers: 4096 x 12288 in bf16, 403 MB, 81 us, 5.0 TB/s, at the rate of a large copy; one row of 4096 3.4 us, a launch and the way from memory and back.
template <typename T, int LANES, int CH>
__global__ void __launch_bounds__(LANES <= 64 ? 256 : LANES) resnorm_rows_kernel(ResnormArgs g) {
    constexpr int BLOCK = LANES <= 64 ? 256 : LANES, ROWS = BLOCK / LANES;
    // two exchanges of each norm, in regions of their own, and rows take turns: between two uses of a region lies the barrier of another
    __shared__ float lds[2][2][2][LANES <= 64 ? 4 : LANES / 64];
    const int lane = threadIdx.x % LANES;
    int turn = 0;
    for (int64_t row = (int64_t)blockIdx.x * ROWS + row_group<LANES>(); row < g.M; row += (int64_t)gridDim.x * ROWS, turn ^= 1) {
        const bool last = row == g.M - 1;
        // The vectors, the same for all rows and from the caches: along with the row, or, of long rows, for which that takes registers away from other rows, once they are wanted.
        constexpr bool LATE = CH > 2, EARLY = CH == 1;
        RowChunks<bf16_t, LANES, CH> b, gamma, beta, gate, gamma_b, beta_b;
        RowChunks<T, LANES, CH> x;
        b.load(g.B + row * g.ldb, g.K, lane, last);
        x.load(static_cast<const T*>(g.X) + row * g.ldx, g.K, lane, last);
        auto first_vectors = [&]() __attribute__((always_inline)) {
            load_vector(gamma, g.gamma_a, g.K, lane, ONES);
            load_vector(beta, g.beta_a, g.K, lane, 0u);
            load_vector(gate, g.gate, g.K, lane, ONES);
        };
        auto second_vectors = [&]() __attribute__((always_inline)) {
            load_vector(gamma_b, g.gamma_b, g.K, lane, ONES);
            load_vector(beta_b, g.beta_b, g.K, lane, 0u);
        };
        if (!LATE) first_vectors();
        if (EARLY) second_vectors();
        b.mask(g.K, lane);
        x.mask(g.K, lane);
        float v[CH][8], mean_a, rstd_a, mean_b, rstd_b;
#pragma unroll
        for (int j = 0; j < CH; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[j][i] = b.raw[j].at(i);
        row_moments<LANES, CH>(v, g.K, lane, g.kind_a, g.eps, lds[turn][0], mean_a, rstd_a);
        if (LATE) first_vectors();
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            const int c = (j * LANES + lane) * 8, left = g.K - c;
            float s[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float h = (v[j][i] - mean_a) * rstd_a;
                s[i] = __builtin_fmaf(g.scale * gate.raw[j].at(i), __builtin_fmaf(h, gamma.raw[j].at(i), beta.raw[j].at(i)), x.raw[j].at(i));
                v[j][i] = stored(s[i], static_cast<const T*>(nullptr));  // the norm is that of what is stored
            }
            if (left < 8)
#pragma unroll
                for (int i = 0; i < 8; ++i) v[j][i] = i < left ? v[j][i] : 0.f;
            store_in_row<LANES>(static_cast<T*>(g.S) + row * g.lds, g.K, c, s);
        }
        if (!EARLY && !LATE) second_vectors();
        row_moments<LANES, CH>(v, g.K, lane, g.kind_b, g.eps, lds[turn][1], mean_b, rstd_b);
        if (LATE) second_vectors();
        if (lane == 0 && g.stats) g.stats[row] = f32x4{mean_a, rstd_a, mean_b, rstd_b};
#pragma unroll
        for (int j = 0; j < CH; ++j) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[j][i] = __builtin_fmaf((v[j][i] - mean_b) * rstd_b, gamma_b.raw[j].at(i), beta_b.raw[j].at(i));
            store_in_row<LANES>(g.Y + row * g.ldy, g.K, (j * LANES + lane) * 8, v[j]);
        }
    }
}

// Rows of any length, a workgroup to a row, read again for each step; a thread reads back the values of S that it wrote itself.
template <typename T>
__global__ void __launch_bounds__(NORM_THREADS) resnorm_long_kernel(ResnormArgs g) {
    __shared__ float lds[NORM_THREADS / 64];
    for (int64_t row = blockIdx.x; row < g.M; row += gridDim.x) {
        auto moments = [&](const auto* from, int kind, float& mean, float& rstd) __attribute__((always_inline)) {
            mean = 0.f;
            rstd = 1.f;
            if (kind == KIND_NONE) return;
            for (int pass = kind == KIND_LAYER ? 0 : 1; pass < 2; ++pass) {
                float sum[1] = {0.f};
                for (int64_t c = threadIdx.x * 8; c < g.K; c += NORM_THREADS * 8) {
                    const int valid = (int)min((int64_t)8, g.K - c);
                    float v[8];
                    load_chunk(from + c, valid, v);
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum[0] += i >= valid ? 0.f : pass ? (v[i] - mean) * (v[i] - mean) : v[i];
                }
                block_sums<NORM_THREADS>(sum, lds);
                if (pass) rstd = 1.0f / sqrtf(sum[0] / (float)g.K + g.eps);
                else mean = sum[0] / (float)g.K;
            }
        };
        const bf16_t* const b = g.B + row * g.ldb;
        T* const s = static_cast<T*>(g.S) + row * g.lds;
        float mean_a, rstd_a, mean_b, rstd_b;
        moments(b, g.kind_a, mean_a, rstd_a);
        for (int64_t c = threadIdx.x * 8; c < g.K; c += NORM_THREADS * 8) {
            const int valid = (int)min((int64_t)8, g.K - c);
            float v[8], x[8], gamma[8], beta[8], gate[8];
            load_chunk(b + c, valid, v);
            load_chunk(static_cast<const T*>(g.X) + row * g.ldx + c, valid, x);
            vector_chunk(g.gamma_a, c, valid, 1.f, gamma);
            vector_chunk(g.beta_a, c, valid, 0.f, beta);
            vector_chunk(g.gate, c, valid, 1.f, gate);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] += g.scale * gate[i] * ((v[i] - mean_a) * rstd_a * gamma[i] + beta[i]);
            store_chunk(s + c, valid, x);
        }
        moments(static_cast<const T*>(s), g.kind_b, mean_b, rstd_b);
        if (threadIdx.x == 0 && g.stats) g.stats[row] = f32x4{mean_a, rstd_a, mean_b, rstd_b};
        for (int64_t c = threadIdx.x * 8; c < g.K; c += NORM_THREADS * 8) {
            const int valid = (int)min((int64_t)8, g.K - c);
            float v[8], gamma[8], beta[8];
            load_chunk(static_cast<const T*>(s) + c, valid, v);
            vector_chunk(g.gamma_b, c, valid, 1.f, gamma);
            vector_chunk(g.beta_b, c, valid, 0.f, beta);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = (v[i] - mean_b) * rstd_b * gamma[i] + beta[i];
            store_chunk(g.Y + row * g.ldy + c, valid, v);
        }
    }
}

// Backward on rows in registers, one pass over the data: a workgroup of GROUPS rows at a time walks the rows, every lane keeps the four sums of its columns as it goes.
// At its end a workgroup adds its groups' columns up through LDS, in order, and writes them to `partial`, which resnorm_join_kernel adds up: no atomics, the same bits
// every time.
// AHEAD: the next row's loads are under way while this one's sums meet.
// 8192 x 7168 in bf16, 705 MB, 131 us, 5.4 TB/s, and the join 7.5; 1001 x 1027 in fp32 12 us and the join 6: two rows in turn to half of the lanes' groups, 129 of 256 lanes at work.
constexpr int RESNORM_LDS_CHUNKS = 4;
template <typename T, int LANES, int CH, int GROUPS, bool AHEAD>
__global__ void __launch_bounds__(LANES * GROUPS) resnorm_bwd_rows_kernel(ResnormBwdArgs g) {
    constexpr int BLOCK = LANES * GROUPS;
    __shared__ float lds[2][2][2 * (BLOCK / 64)];
    __shared__ __attribute__((aligned(16))) float cols[GROUPS > 1 ? BLOCK * 8 : 4];
    const int lane = threadIdx.x % LANES, group = row_group<LANES>();
    const float per_row = 1.0f / (float)g.K;
    // four chunks of four sums each are half of a thread's registers: two of the sums are kept in LDS then, where a lane has places of its own
    constexpr bool IN_LDS = CH == RESNORM_LDS_CHUNKS;
    constexpr int IN_REGS = IN_LDS ? 1 : CH;
    extern __shared__ __attribute__((aligned(16))) float y_sums[];
    auto y_at = [&](int what, int j, int half) __attribute__((always_inline)) { return reinterpret_cast<f32x4*>(y_sums) + ((what * CH + j) * 2 + half) * LANES + lane; };
    float y0[IN_REGS][8], y1[IN_REGS][8], s0[CH][8], s1[CH][8];
#pragma unroll
    for (int j = 0; j < CH; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            y0[j % IN_REGS][i] = y1[j % IN_REGS][i] = s0[j][i] = s1[j][i] = 0.f;
            if (IN_LDS && i < 4) *y_at(i / 2, j, i % 2) = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    RowChunks<bf16_t, LANES, CH> gb, ga, gate;
    load_vector(gb, g.gamma_b, g.K, lane, ONES);
    load_vector(ga, g.gamma_a, g.K, lane, ONES);
    load_vector(gate, g.gate, g.K, lane, ONES);
    const int64_t step = (int64_t)gridDim.x * GROUPS;
    RowChunks<T, LANES, CH> s_next, ds_next;
    RowChunks<bf16_t, LANES, CH> dy_next, b_next;
    f32x4 st_next;
    auto request = [&](int64_t row) __attribute__((always_inline)) {  // rows beyond the last stand for it
        row = min(row, (int64_t)g.M - 1);
        const bool last = row == g.M - 1;
        st_next = g.stats[row];
        s_next.load(static_cast<const T*>(g.S) + row * g.lds, g.K, lane, last);
        dy_next.load(g.dY + row * g.lddy, g.K, lane, last);
        if (g.dS) ds_next.load(static_cast<const T*>(g.dS) + row * g.ldds, g.K, lane, last);
        else ds_next.clear();
        b_next.load(g.B + row * g.ldb, g.K, lane, last);
    };
    if (AHEAD) request((int64_t)blockIdx.x * GROUPS + group);
    int turn = 0;
    for (int64_t row0 = (int64_t)blockIdx.x * GROUPS; row0 < g.M; row0 += step, turn ^= 1) {  // as many turns for every group
        const int64_t row = row0 + group;
        const bool here = row < g.M;
        if (!AHEAD) request(row);
        RowChunks<T, LANES, CH> s = s_next, ds = ds_next;
        RowChunks<bf16_t, LANES, CH> dy = dy_next, b = b_next;
        const f32x4 st = st_next;
        s.mask(g.K, lane);
        dy.mask(g.K, lane);
        ds.mask(g.K, lane);
        b.mask(g.K, lane);
        if (!here) {  // a row that is not there adds nothing
            dy.clear();
            ds.clear();
        }
        auto hb_of = [&](int j, int i) __attribute__((always_inline)) { return (s.raw[j].at(i) - st[2]) * st[3]; };
        auto ha_of = [&](int j, int i) __attribute__((always_inline)) { return (b.raw[j].at(i) - st[0]) * st[1]; };
#pragma unroll
        for (int j = 0; j < CH; ++j) {  // kept as they are loaded, not as eight registers of fp32
            pin_chunk(gb.raw[j]);
            pin_chunk(ga.raw[j]);
            pin_chunk(gate.raw[j]);
        }
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            f32x4 held[4];  // of this chunk: y0's two quads, y1's
            if constexpr (IN_LDS)
#pragma unroll
                for (int q = 0; q < 4; ++q) held[q] = *y_at(q / 2, j, q % 2);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float y = dy.raw[j].at(i), h = hb_of(j, i), d = y * gb.raw[j].at(i);
                if constexpr (IN_LDS) {
                    held[i / 4][i % 4] += y * h;
                    held[2 + i / 4][i % 4] += y;
                } else {
                    y0[j][i] += y * h;
                    y1[j][i] += y;
                    asm volatile("" : "+v"(y0[j][i]), "+v"(y1[j][i]));  // here: put off, they would keep h and y in registers
                }
                sum[0] += d;
                sum[1] += d * h;
            }
            if constexpr (IN_LDS)
#pragma unroll
                for (int q = 0; q < 4; ++q) *y_at(q / 2, j, q % 2) = held[q];
        }
        if (AHEAD && row0 + step < g.M) request(row + step);
        row_sums<LANES>(sum, lds[turn][0]);
        const float c1 = g.kind_b == KIND_LAYER ? sum[0] * per_row : 0.f, c2 = sum[1] * per_row;
        float d[CH][8];  // ds'
        sum[0] = sum[1] = 0.f;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            pin_chunk(s.raw[j]);
            pin_chunk(dy.raw[j]);
            const int left = here ? g.K - (j * LANES + lane) * 8 : 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                d[j][i] = ds.raw[j].at(i) + st[3] * (dy.raw[j].at(i) * gb.raw[j].at(i) - c1 - hb_of(j, i) * c2);
            }
            if (left < 8)
#pragma unroll
                for (int i = 0; i < 8; ++i) d[j][i] = i < left ? d[j][i] : 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float h = ha_of(j, i), q = g.scale * gate.raw[j].at(i) * ga.raw[j].at(i) * d[j][i];
                s0[j][i] += d[j][i] * h;  // zeros, of a row that is not there
                s1[j][i] += d[j][i];
                asm volatile("" : "+v"(s0[j][i]), "+v"(s1[j][i]));
                sum[0] += q;
                sum[1] += q * h;
            }
        }
        if (here)
#pragma unroll
            for (int j = 0; j < CH; ++j) store_in_row<LANES>(static_cast<T*>(g.dX) + row * g.lddx, g.K, (j * LANES + lane) * 8, d[j]);
        if (g.kind_a != KIND_NONE) row_sums<LANES>(sum, lds[turn][1]);
        if (!here) continue;
        const float d1 = g.kind_a == KIND_LAYER ? sum[0] * per_row : 0.f, d2 = g.kind_a != KIND_NONE ? sum[1] * per_row : 0.f;
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            pin_chunk(b.raw[j]);
            pin_chunk(ga.raw[j]);
            pin_chunk(gate.raw[j]);
#pragma unroll
            for (int i = 0; i < 8; ++i) d[j][i] = st[1] * (g.scale * gate.raw[j].at(i) * ga.raw[j].at(i) * d[j][i] - d1 - ha_of(j, i) * d2);
            store_in_row<LANES>(g.dB + row * g.lddb, g.K, (j * LANES + lane) * 8, d[j]);
        }
    }
    if (!g.want_cols) return;
    constexpr int COLS = LANES * 8;  // of a chunk of all lanes
#pragma unroll
    for (int what = 0; what < 4; ++what) {
        float v[CH][8];
#pragma unroll
        for (int j = 0; j < CH; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                v[j][i] = what == 2 ? s0[j][i] : what == 3 ? s1[j][i] : IN_LDS ? (*y_at(what, j, i / 4))[i % 4] : what == 0 ? y0[j % IN_REGS][i] : y1[j % IN_REGS][i];
        float* const to = g.partial + ((int64_t)blockIdx.x * 4 + what) * g.partial_cols;
        if constexpr (GROUPS > 1) {
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                __syncthreads();
                float* const mine = cols + group * COLS + lane * 8;
                *reinterpret_cast<f32x4*>(mine) = f32x4{v[j][0], v[j][1], v[j][2], v[j][3]};
                *reinterpret_cast<f32x4*>(mine + 4) = f32x4{v[j][4], v[j][5], v[j][6], v[j][7]};
                __syncthreads();
                for (int c = threadIdx.x; c < COLS && j * COLS + c < g.K; c += BLOCK) {
                    float sum = 0.f;
#pragma unroll
                    for (int q = 0; q < GROUPS; ++q) sum += cols[q * COLS + c];
                    to[j * COLS + c] = sum;
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < CH; ++j) {
                const int c = (j * LANES + lane) * 8;
                if (c >= g.K) continue;
                *reinterpret_cast<f32x4*>(to + c) = f32x4{v[j][0], v[j][1], v[j][2], v[j][3]};
                *reinterpret_cast<f32x4*>(to + c + 4) = f32x4{v[j][4], v[j][5], v[j][6], v[j][7]};
            }
        }
    }
}

// ds' of eight values of a row of any length, and hb of them.
template <typename T>
__device__ __forceinline__ void resnorm_ds(const ResnormBwdArgs& g, int64_t row, int64_t c, int valid, const f32x4 st, const float2 m, float (&d)[8], float (&y)[8], float (&hb)[8]) {
    float w[8];
    load_chunk(static_cast<const T*>(g.S) + row * g.lds + c, valid, hb);
    load_chunk(g.dY + row * g.lddy + c, valid, y);
    vector_chunk(g.gamma_b, c, valid, 1.f, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        hb[i] = (hb[i] - st[2]) * st[3];
        d[i] = st[3] * (y[i] * w[i] - m.x - hb[i] * m.y);
    }
    if (!g.dS) return;
    load_chunk(static_cast<const T*>(g.dS) + row * g.ldds + c, valid, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) d[i] += w[i];
}

// dX and dB of rows of any length, a workgroup to a row, which it reads three times, and the row's (mean(g), mean(g hb)) for resnorm_cols_kernel.
template <typename T>
__global__ void __launch_bounds__(NORM_THREADS) resnorm_bwd_long_kernel(ResnormBwdArgs g) {
    __shared__ float lds[2 * NORM_THREADS / 64];
    const float per_row = 1.0f / (float)g.K;
    if (g.means) {  // the counters of the resnorm_cols_kernel behind this one
        const int strips = (g.K + NORM_STRIP - 1) / NORM_STRIP;
        for (int i = blockIdx.x * NORM_THREADS + threadIdx.x; i < strips; i += gridDim.x * NORM_THREADS) g.counters[i] = 0u;
    }
    for (int64_t row = blockIdx.x; row < g.M; row += gridDim.x) {
        const f32x4 st = g.stats[row];
        float sum[2] = {0.f, 0.f};
        for (int64_t c = threadIdx.x * 8; c < g.K; c += NORM_THREADS * 8) {
            const int valid = (int)min((int64_t)8, g.K - c);
            float h[8], y[8], w[8];
            load_chunk(static_cast<const T*>(g.S) + row * g.lds + c, valid, h);
            load_chunk(g.dY + row * g.lddy + c, valid, y);
            vector_chunk(g.gamma_b, c, valid, 1.f, w);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < valid) {
                    sum[0] += y[i] * w[i];
                    sum[1] += y[i] * w[i] * ((h[i] - st[2]) * st[3]);
                }
        }
        block_sums<NORM_THREADS>(sum, lds);
        const float2 m = {g.kind_b == KIND_LAYER ? sum[0] * per_row : 0.f, sum[1] * per_row};
        if (threadIdx.x == 0 && g.means) g.means[row] = m;
        // q and ha of a chunk
        auto chunk = [&](int64_t c, int valid, float (&d)[8], float (&q)[8], float (&ha)[8]) __attribute__((always_inline)) {
            float w[8];
            resnorm_ds<T>(g, row, c, valid, st, m, d, q, ha);
            load_chunk(g.B + row * g.ldb + c, valid, ha);
            vector_chunk(g.gate, c, valid, 1.f, q);
            vector_chunk(g.gamma_a, c, valid, 1.f, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                ha[i] = (ha[i] - st[0]) * st[1];
                q[i] = g.scale * q[i] * w[i] * d[i];
            }
        };
        sum[0] = sum[1] = 0.f;
        for (int64_t c = threadIdx.x * 8; c < g.K; c += NORM_THREADS * 8) {
            const int valid = (int)min((int64_t)8, g.K - c);
            float d[8], q[8], ha[8];
            chunk(c, valid, d, q, ha);
            store_chunk(static_cast<T*>(g.dX) + row * g.lddx + c, valid, d);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < valid) {
                    sum[0] += q[i];
                    sum[1] += q[i] * ha[i];
                }
        }
        block_sums<NORM_THREADS>(sum, lds);
        const float d1 = g.kind_a == KIND_LAYER ? sum[0] * per_row : 0.f, d2 = g.kind_a != KIND_NONE ? sum[1] * per_row : 0.f;
        for (int64_t c = threadIdx.x * 8; c < g.K; c += NORM_THREADS * 8) {
            const int valid = (int)min((int64_t)8, g.K - c);
            float d[8], q[8], ha[8];
            chunk(c, valid, d, q, ha);
#pragma unroll
            for (int i = 0; i < 8; ++i) q[i] = st[1] * (q[i] - d1 - ha[i] * d2);
            store_chunk(g.dB + row * g.lddb + c, valid, q);
        }
    }
}

// The gradients of column c from its four sums.
__device__ __forceinline__ void resnorm_gradients(const ResnormBwdArgs& g, int64_t c, const float (&v)[4]) {
    const float gate = g.scale * (g.gate ? bf16_bits_to_f32(g.gate[c]) : 1.f);
    const float gamma = g.gamma_a ? bf16_bits_to_f32(g.gamma_a[c]) : 1.f, beta = g.beta_a ? bf16_bits_to_f32(g.beta_a[c]) : 0.f;
    auto out = [&](float* to, float x) __attribute__((always_inline)) {
        if (to) to[c] = g.accumulate ? to[c] + x : x;
    };
    out(g.dgamma_b, v[0]);
    out(g.dbeta_b, v[1]);
    out(g.dgamma_a, gate * v[2]);
    out(g.dbeta_a, gate * v[3]);
    out(g.dgate, g.scale * (gamma * v[2] + beta * v[3]));
}

// The four column sums of rows whose dX and dB have been formed, and the gradients: strips of 64 columns over slices of the rows, 8 lanes of 8 columns by 32 rows at a
// time, as norm_cols_kernel.  A slice's sums go to the workspace, and whoever comes last of a strip adds them up in the slices' order (as the slices of gated_slim_kernel:
// past the L2, by device-scope accesses).
// It reads the data a second time: for rows that are too long for registers.
template <typename T>
__global__ void __launch_bounds__(NORM_COL_THREADS) resnorm_cols_kernel(ResnormBwdArgs g) {
    __shared__ float lds[4][NORM_COL_THREADS / 64][NORM_STRIP];
    __shared__ uint32_t arrived;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t pieces = ((int64_t)g.K + NORM_STRIP - 1) / NORM_STRIP * g.slices;
    for (int64_t piece = blockIdx.x; piece < pieces; piece += gridDim.x) {
        const int64_t strip = piece / g.slices, slice = piece % g.slices;
        const int64_t col = strip * NORM_STRIP + (lane & 7) * 8;
        const int valid = (int)min((int64_t)8, g.K - col);
        float sum[4][8];
#pragma unroll
        for (int w = 0; w < 4; ++w)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[w][i] = 0.f;
        const int64_t end = min((int64_t)g.M, (slice + 1) * g.rows_per_slice);
        if (valid > 0)
            for (int64_t row = slice * g.rows_per_slice + (threadIdx.x >> 3); row < end; row += NORM_COL_ROWS) {
                const f32x4 st = g.stats[row];
                float d[8], y[8], h[8], b[8];
                resnorm_ds<T>(g, row, col, valid, st, g.means[row], d, y, h);
                load_chunk(g.B + row * g.ldb + col, valid, b);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    sum[0][i] += y[i] * h[i];
                    sum[1][i] += y[i];
                    sum[2][i] += d[i] * ((b[i] - st[0]) * st[1]);
                    sum[3][i] += d[i];
                }
            }
#pragma unroll
        for (int m = 8; m < 64; m <<= 1)
#pragma unroll
            for (int w = 0; w < 4; ++w)
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[w][i] += __shfl_xor(sum[w][i], m, 64);
        __syncthreads();  // the last piece's sums have been read
        if (lane < 8)
#pragma unroll
            for (int w = 0; w < 4; ++w)
#pragma unroll
                for (int i = 0; i < 8; ++i) lds[w][wave][lane * 8 + i] = sum[w][i];
        __syncthreads();
        static_assert(NORM_COL_THREADS == 4 * NORM_STRIP, "a thread for each sum");
        const int what = threadIdx.x / NORM_STRIP, c = threadIdx.x % NORM_STRIP;
        float all = 0.f;
#pragma unroll
        for (int w = 0; w < NORM_COL_THREADS / 64; ++w) all += lds[what][w][c];
        const int64_t at = strip * NORM_STRIP + c;
        if (at < g.K) __hip_atomic_store(g.partial + (slice * 4 + what) * g.partial_cols + at, all, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wave's sums have arrived where all XCDs see them
        __syncthreads();                                  // and those of all waves; lds has been read
        if (threadIdx.x == 0) arrived = __hip_atomic_fetch_add(g.counters + strip, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __syncthreads();
        if (arrived != (uint32_t)(g.slices - 1)) continue;
        all = 0.f;
        if (at < g.K)
            for (int s0 = 0; s0 < g.slices; s0 += 8) {  // eight slices requested at a time
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    v[i] = s0 + i < g.slices ? __hip_atomic_load(g.partial + ((int64_t)(s0 + i) * 4 + what) * g.partial_cols + at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) all += v[i];
            }
        lds[what][0][c] = all;
        __syncthreads();
        if (what == 0 && at < g.K) {
            const float v[4] = {all, lds[1][0][c], lds[2][0][c], lds[3][0][c]};
            resnorm_gradients(g, at, v);
        }
    }
}

// The sums of all slices, added in an order that depends on their number and the columns' alone, and what is formed of them.  A workgroup has 32 columns: 256 threads to each of
// the four sums, eight lanes of 16 bytes by every 32nd slice; the lanes of a wave meet by exchanges and the waves in LDS.  (Eight columns, 32 bytes of a slice's line: 200 x 4000 20.5 us as a
// whole, now 14.3.)
constexpr int RESNORM_JOIN_THREADS = 1024, RESNORM_JOIN_COLS = 32;
__global__ void __launch_bounds__(RESNORM_JOIN_THREADS) resnorm_join_kernel(ResnormBwdArgs g) {
    constexpr int WAVES = RESNORM_JOIN_THREADS / 64 / 4, LANES = RESNORM_JOIN_COLS / 4;  // of a sum; that share a slice
    __shared__ __attribute__((aligned(16))) float lds[4][WAVES][RESNORM_JOIN_COLS];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, what = wave / WAVES;
    for (int64_t from = (int64_t)blockIdx.x * RESNORM_JOIN_COLS; from < g.K; from += (int64_t)gridDim.x * RESNORM_JOIN_COLS) {
        const int64_t col = from + lane % LANES * 4;
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
        if (col < g.partial_cols)
            for (int s = (threadIdx.x & 255) / LANES; s < g.slices; s += 256 / LANES) sum += *reinterpret_cast<const f32x4*>(g.partial + ((int64_t)s * 4 + what) * g.partial_cols + col);
#pragma unroll
        for (int m = LANES; m < 64; m <<= 1)
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] += __shfl_xor(sum[i], m, 64);
        __syncthreads();  // the last columns' sums have been read
        if (lane < LANES) *reinterpret_cast<f32x4*>(&lds[what][wave % WAVES][lane * 4]) = sum;
        __syncthreads();
        const int64_t c = from + threadIdx.x;
        if (threadIdx.x >= RESNORM_JOIN_COLS || c >= g.K) continue;
        float v[4];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            v[w] = 0.f;
#pragma unroll
            for (int i = 0; i < WAVES; ++i) v[w] += lds[w][i][threadIdx.x];
        }
        resnorm_gradients(g, c, v);
    }
}

}  // namespace axo
