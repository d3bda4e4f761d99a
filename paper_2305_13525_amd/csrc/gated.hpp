// The gated feed-forward block for gfx950: H = act(G) * U with G = X Wg + bg, U = X Wu + bu, and its backward pass.
//   dG = dH U act'(G), dU = dH act(G)          dH = dY W^T of the layer behind the block
//   dX = dG Wg^T + dU Wu^T                     one reduction over both products
//   dWg = X^T dG, dWu = X^T dU                 two weight gradients (gemm_tile.hpp, gemm_slim.hpp)
// This file: the element-wise forms and kernels for operands whose spans pass 4 GiB.
#pragma once
#include "axo_common.hpp"
#include "gate.hpp"
#include "gemm_generic.hpp"
#include "gemm_tile.hpp"
#include "norm.hpp"

namespace axo {

// The element-wise forms, eight columns of a row per thread and turn; bound by memory: 8192 x 14336 forward 124 us, backward 206, 5.7 TB/s both.
struct GatedMapArgs {
    const bf16_t *dH, *G, *U;
    bf16_t *H, *dG, *dU;  // H alone, or the other two
    int64_t lddh, ldz, ldout;
    int M, N, gate;
};
constexpr int GATED_MAP_THREADS = 256;
template <bool BACK>
__global__ void __launch_bounds__(GATED_MAP_THREADS) gated_map_kernel(GatedMapArgs g) {
    const int64_t per_row = ((int64_t)g.N + 7) / 8, chunks = per_row * g.M, step = (int64_t)gridDim.x * GATED_MAP_THREADS;
    with_gate(g.gate, [&](auto gate) __attribute__((always_inline)) {
        constexpr int GATE = decltype(gate)::value;
        for (int64_t at = (int64_t)blockIdx.x * GATED_MAP_THREADS + threadIdx.x; at < chunks; at += step) {
            const int64_t row = at / per_row, col = (at - row * per_row) * 8;
            const int valid = (int)min((int64_t)8, g.N - col);
            float v[8], u[8], d[8];
            load_chunk(g.G + row * g.ldz + col, valid, v);
            load_chunk(g.U + row * g.ldz + col, valid, u);
            if (BACK) {
                load_chunk(g.dH + row * g.lddh + col, valid, d);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float2 a = gate_both<GATE>(v[i]);
                    v[i] = d[i] * u[i] * a.y;
                    d[i] *= a.x;
                }
                store_chunk(g.dG + row * g.ldout + col, valid, v);
                store_chunk(g.dU + row * g.ldout + col, valid, d);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = gate_value<GATE>(v[i]) * u[i];
                store_chunk(g.H + row * g.ldout + col, valid, v);
            }
        }
    });
}

// One value of a product with a residual: z = sum + bias.
__device__ __forceinline__ void add_one(const GatedArgs& g, float z, int row, int col) {
    const int64_t at = (int64_t)row * g.ldc + col, from = (int64_t)row * g.ldaux + col;
    const float res = !g.aux ? 0.f : g.wide ? reinterpret_cast<const float*>(g.aux)[from] : bf16_bits_to_f32(g.aux[from]);
    const float y = __builtin_fmaf(g.scale, apply_epilogue(z, 0.f, g.gate), res);
    if (g.wide) reinterpret_cast<float*>(g.C)[at] = y;
    else g.C[at] = f32_to_bf16_bits(y);
    if (g.G) g.G[(int64_t)row * g.ldz + col] = f32_to_bf16_bits(z);
}

// dZ = scale dY act'(Z), element by element, eight columns of a row per thread and turn, as gated_map_kernel; without an activation dZ = scale dY, which
// is then a rounding of the stream's gradient to what the products read.  4000 x 6000 of an fp32 stream, 192 MB, 35 us: 5.5 TB/s.
struct AddMapArgs {
    const void* dY;
    const bf16_t* Z;
    bf16_t* dZ;
    int64_t lddy, ldz, lddz;
    int M, N, epilogue;
    float scale;
};
template <typename T>
__global__ void __launch_bounds__(GATED_MAP_THREADS) add_map_kernel(AddMapArgs g) {
    const int64_t per_row = ((int64_t)g.N + 7) / 8, chunks = per_row * g.M, step = (int64_t)gridDim.x * GATED_MAP_THREADS;
    with_act(g.epilogue, [&](auto act) __attribute__((always_inline)) {
        constexpr int ACT = decltype(act)::value;
        for (int64_t at = (int64_t)blockIdx.x * GATED_MAP_THREADS + threadIdx.x; at < chunks; at += step) {
            const int64_t row = at / per_row, col = (at - row * per_row) * 8;
            const int valid = (int)min((int64_t)8, g.N - col);
            float d[8], z[8];
            load_chunk(static_cast<const T*>(g.dY) + row * g.lddy + col, valid, d);
            if (ACT != EPI_BIAS) load_chunk(g.Z + row * g.ldz + col, valid, z);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                d[i] *= g.scale;
                if (ACT != EPI_BIAS) d[i] *= gate_both<ACT == EPI_BIAS_GELU_TANH ? GATE_GELU_TANH : GATE_GELU_ERF>(z[i]).y;
            }
            store_chunk(g.dZ + row * g.lddz + col, valid, d);
        }
    });
}

// The block's products for any sizes and spans, 64-bit indices, 128 x 128 tiles staged through registers as gemm_generic_kernel: what is left to it are
// empty reductions, operands whose spans pass 4 GiB and outputs of a billion rows or columns, whose 256-row tiles are too many for a launch.  Forward
// 4096 x 8192 x 16384 12.7 ms, an eighth of the tiles' rate.  (FC_ADD, the product with a residual, has the same kernels.)
template <int OP>
__global__ void __launch_bounds__(256) gated_generic_kernel(GatedArgs g) {
    constexpr int LB = OP == GATED_FWD || OP == FC_ADD ? MC : KC, SUMS = OP == GATED_FWD ? 2 : 1;
    __shared__ __attribute__((aligned(16))) bf16_t As[GEN_BM * GEN_LDS_STRIDE];
    __shared__ __attribute__((aligned(16))) bf16_t Bs[SUMS][GEN_BN * GEN_LDS_STRIDE];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wm = wave >> 1, wn = wave & 1;
    const int i0 = blockIdx.y * GEN_BM, j0 = blockIdx.x * GEN_BN;
    f32x16 acc[SUMS][2][2];
#pragma unroll
    for (int s = 0; s < SUMS; ++s)
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[s][a][b][i] = 0.0f;
    auto walk = [&](const bf16_t* A, const bf16_t* B) __attribute__((always_inline)) {
        for (int r0 = 0; r0 < g.R; r0 += GEN_BK) {
            stage_tile<KC>(A, g.lda, i0, g.Mo, r0, g.R, As, tid);
            stage_tile<LB>(B, g.ldb, j0, g.No, r0, g.R, Bs[0], tid);
            if constexpr (OP == GATED_FWD) stage_tile<LB>(g.B2, g.ldb, j0, g.No, r0, g.R, Bs[1], tid);
            __syncthreads();
#pragma unroll
            for (int kk = 0; kk < GEN_BK; kk += 16) {
                const int koff = kk + 8 * (lane >> 5);
                bf16x8 fa[2];
#pragma unroll
                for (int a = 0; a < 2; ++a) fa[a] = *reinterpret_cast<const bf16x8*>(As + (wm * 64 + a * 32 + (lane & 31)) * GEN_LDS_STRIDE + koff);
#pragma unroll
                for (int s = 0; s < SUMS; ++s)
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        const bf16x8 fb = *reinterpret_cast<const bf16x8*>(Bs[s] + (wn * 64 + b * 32 + (lane & 31)) * GEN_LDS_STRIDE + koff);
#pragma unroll
                        for (int a = 0; a < 2; ++a) acc[s][a][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[a], fb, acc[s][a][b], 0, 0, 0);
                    }
            }
            __syncthreads();
        }
    };
    walk(g.A, g.B);
    if constexpr (OP == GATED_DX) walk(g.A2, g.B2);
    if constexpr (OP == FC_ADD) {
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const int col = j0 + wn * 64 + b * 32 + (lane & 31);
                if (col >= g.No) continue;
                const float bias = g.bias ? bf16_bits_to_f32(g.bias[col]) : 0.f;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int row = i0 + wm * 64 + a * 32 + 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3);
                    if (row < g.Mo) add_one(g, acc[0][a][b][e] + bias, row, col);
                }
            }
        return;
    }
    // accumulator element e of a 32x32 tile: row 8*(e/4) + 4*(lane/32) + e%4, column lane%32
    with_gate(g.gate, [&](auto gate) __attribute__((always_inline)) {
        constexpr int GATE = decltype(gate)::value;
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const int col = j0 + wn * 64 + b * 32 + (lane & 31);
                if (col >= g.No) continue;
                const float bg = OP == GATED_FWD && g.bias ? bf16_bits_to_f32(g.bias[col]) : 0.f;
                const float bu = OP == GATED_FWD && g.bias2 ? bf16_bits_to_f32(g.bias2[col]) : 0.f;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int row = i0 + wm * 64 + a * 32 + 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3);
                    if (row >= g.Mo) continue;
                    const int64_t at = (int64_t)row * g.ldc + col;
                    const float v = acc[0][a][b][e];
                    if constexpr (OP == GATED_FWD) {
                        const float gs = v + bg, us = acc[SUMS - 1][a][b][e] + bu;
                        g.C[at] = f32_to_bf16_bits(gate_value<GATE>(gs) * us);
                        if (g.G) {
                            g.G[(int64_t)row * g.ldz + col] = f32_to_bf16_bits(gs);
                            g.U[(int64_t)row * g.ldz + col] = f32_to_bf16_bits(us);
                        }
                    } else if constexpr (OP == GATED_DACT) {
                        const int64_t z = (int64_t)row * g.ldaux + col;
                        const float2 act = gate_both<GATE>(bf16_bits_to_f32(g.aux[z]));
                        g.C[at] = f32_to_bf16_bits(v * bf16_bits_to_f32(g.aux2[z]) * act.y);
                        g.U[at] = f32_to_bf16_bits(v * act.x);
                    } else g.C[at] = f32_to_bf16_bits(v);
                }
            }
    });
}

// ---- the block's products on the tiles of gemm_tile.hpp ---------------------------------------
// The forward's tiles hold as many columns of Wg as of Wu, so a tile of BN columns of the two is one of BN / 2 columns of H, and the operands are read and the
// matrix units fed as for one product of twice the columns.  dX is one product of twice the reduction.
// Bound by the matrix units at large sizes, by the epilogue's memory where the reduction is short.  Measured, 256 x 256 tiles: forward 4096 x 8192 x 16384 with
// G and U kept 1.51 to 1.55 ms, 1440 TFLOP/s (axo_fc_fwd on the same columns 1485); the gradient through the activation 4096 x 8192 x 16384 826 to 844 us, 1300 (axo_fc_dgrad
// 735 us: the rest is G and U read and a second output, which no reduction hides, since all tiles of a round come to their ends together); dX of 4096 x 7168 x 14336
// 1.29 ms, 1310.  1001 x 1027 x 515 forward 10.1 us, through the activation 9.0.
template <int OP>
constexpr int GATED_LB = OP == GATED_FWD || OP == FC_ADD ? MC : KC;
template <int OP>
constexpr int gated_cols(int BN) { return OP == GATED_FWD ? BN / 2 : BN; }  // of the output, in a tile of BN columns of B

// LINES: rows by whole lines on no tiles (0), on the large ones (1), on both (2), as gemm_mixed_kernel.
template <int OP, bool PLAIN, int LINES>
__global__ void __launch_bounds__(TILE_THREADS, 1) gated_mixed_kernel(GatedProduct<OP> g, TileSched sc) {
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    constexpr int LB = GATED_LB<OP>, BIG = gated_cols<OP>(256), HALF = gated_cols<OP>(128);
    const int bid = blockIdx.x;
    start_shift(bid, sc.shift);
    int tm, tn;
    if (bid < sc.n_big) {
        tile_of_index(xcd_run(bid, sc.n_big), sc.tiles_m, sc.big_cols, sc.group_m, tm, tn);
        gemm_tile_body<256, 256, 2, 4, KC, LB, LINES != 0, PLAIN>(g, inside_row<256, KC>(g, tm * 256), inside_col<BIG>(g, tn * BIG), smem);
    } else {
        const int n_small = (int)gridDim.x - sc.n_big;
        tile_of_index(xcd_run(bid - sc.n_big, n_small), sc.tiles_m, sc.small_cols, sc.group_m, tm, tn);
        gemm_ring_body<256, 128, 4, 2, 3, KC, LB, LINES == 2, PLAIN>(g, inside_row<256, KC>(g, tm * 256), inside_col<HALF>(g, sc.big_cols * BIG + tn * HALF), smem, threadIdx.x);
    }
}
template <int OP, bool PLAIN, bool LINES>
__global__ void __launch_bounds__(TILE_THREADS, 1) gated_mid_kernel(GatedProduct<OP> g, int tiles_m, int tiles_n, int group_m) {
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    constexpr int COLS = gated_cols<OP>(128);
    int tm, tn;
    tile_of_index(xcd_run(blockIdx.x, gridDim.x), tiles_m, tiles_n, group_m, tm, tn);
    gemm_ring_body<128, 128, 4, 2, 4, KC, GATED_LB<OP>, LINES, PLAIN>(g, inside_row<128, KC>(g, tm * 128), inside_col<COLS>(g, tn * COLS), smem, threadIdx.x);
}
template <int OP, bool PLAIN, bool LINES>
__global__ void __launch_bounds__(TILE_THREADS, 1) gated_rect_kernel(GatedProduct<OP> g, int tiles_m, int tiles_n, int group_m) {
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    constexpr int COLS = gated_cols<OP>(128);
    int tm, tn;
    tile_of_index(xcd_run(blockIdx.x, gridDim.x), tiles_m, tiles_n, group_m, tm, tn);
    gemm_ring_body<64, 128, 2, 4, 4, KC, GATED_LB<OP>, LINES, PLAIN>(g, inside_row<64, KC>(g, tm * 64), inside_col<COLS>(g, tn * COLS), smem, threadIdx.x);
}
template <int OP, bool PLAIN, bool LINES>
__global__ void __launch_bounds__(256, 2) gated_small_kernel(GatedProduct<OP> g, int tiles_m, int tiles_n, int group_m) {
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    constexpr int COLS = gated_cols<OP>(64);
    int tm, tn;
    tile_of_index(xcd_run(blockIdx.x, gridDim.x), tiles_m, tiles_n, group_m, tm, tn);
    gemm_ring_body<64, 64, 2, 2, LINES ? 5 : 4, KC, GATED_LB<OP>, LINES, PLAIN>(g, inside_row<64, KC>(g, tm * 64), inside_col<COLS>(g, tn * COLS), smem, threadIdx.x);
}

}  // namespace axo
