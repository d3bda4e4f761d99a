// The gated feed-forward block for gfx950: H = act(G) * U with G = X Wg + bg, U = X Wu + bu, and its backward pass.
//   dG = dH U act'(G), dU = dH act(G)          dH = dY W^T of the layer behind the block
//   dX = dG Wg^T + dU Wu^T                     one reduction over both products
//   dWg = X^T dG, dWu = X^T dU                 two weight gradients (gemm_tile.hpp, gemm_slim.hpp)
// This file: the activations, the element-wise forms and kernels for operands whose spans pass 4 GiB.
#pragma once
#include "axo_common.hpp"
#include "gemm_generic.hpp"
#include "norm.hpp"

namespace axo {

enum Gate { GATE_SILU = 0, GATE_GELU_TANH = 1, GATE_GELU_ERF = 2 };

// v sigmoid(v): one exp2 and one reciprocal, as gelu_tanh.  Below v = -87 exp(-v) passes 2^126 and the result is zero (it is smaller than 2^-119).
__device__ __forceinline__ float silu(float v) {
    return v * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(v * -1.4426950408889634f));
}
template <int GATE>
__device__ __forceinline__ float gate_value(float v) {
    return GATE == GATE_SILU ? silu(v) : GATE == GATE_GELU_TANH ? gelu_tanh(v) : gelu_erf(v);
}
// The value and its derivative.
template <int GATE>
__device__ __forceinline__ float2 gate_both(float v) {
    if (GATE == GATE_SILU) {
        const float s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(v * -1.4426950408889634f));
        return float2{v * s, s * __builtin_fmaf(v, 1.0f - s, 1.0f)};
    }
    // beyond 16 the derivative is that of 16 (1 or 0, and nothing overflows on the way); NaN stays NaN
    if (GATE == GATE_GELU_TANH) return float2{gelu_tanh(v), dgelu_tanh(v > 16.0f ? 16.0f : v < -16.0f ? -16.0f : v)};
    return float2{gelu_erf(v), dgelu_erf(v)};
}

// What the kernels of the block take beside a product's arguments.
struct GatedArgs : GemmArgs {
    const bf16_t* A2;     // dU, of dX
    const bf16_t* B2;     // Wu
    const bf16_t* bias2;  // bu
    const bf16_t* aux2;   // U, where aux is G (their pitch: ldaux)
    bf16_t* G;            // outputs beside C: G and U of the forward pass or nullptr, pitch ldz
    bf16_t* U;            // ... dU of the backward pass, where C is dG (pitch ldc)
    int64_t ldz;
    int gate;             // Gate
};

// f of the gate as a compile-time constant.
template <typename F>
__device__ __forceinline__ void with_gate(int gate, F f) {
    if (gate == GATE_SILU) f(std::integral_constant<int, GATE_SILU>{});
    else if (gate == GATE_GELU_TANH) f(std::integral_constant<int, GATE_GELU_TANH>{});
    else f(std::integral_constant<int, GATE_GELU_ERF>{});
}

// H = act(G) * U, eight columns of a row per thread and turn.
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

// The block's products for any sizes and spans, 64-bit indices, 128 x 128 tiles staged through registers as gemm_generic_kernel: what is left to it are
// empty reductions and operands whose spans pass 4 GiB.
enum GatedOp { GATED_FWD = 0, GATED_DACT = 1, GATED_DX = 2 };
template <int OP>
__global__ void __launch_bounds__(256) gated_generic_kernel(GatedArgs g) {
    constexpr int LB = OP == GATED_FWD ? MC : KC, SUMS = OP == GATED_FWD ? 2 : 1;
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

}  // namespace axo
