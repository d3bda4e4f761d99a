// The products of a gated block for few tokens, or outputs so small that tiles of gemm_tile.hpp are few: the waves of a workgroup split the
// reduction of one small tile, as in gemm_slim.hpp, and where that still leaves compute units without work, several workgroups share a tile, each with
// a slice of its reduction.
//
// Such a product reads each weight once and does little with it, so it is bound by memory, and by how much of it is asked for at a time: a
// wave keeps ST chunks of 64 reduction elements under way, in LDS that nobody else touches, and no barrier stands in its loop.
//
// Slices: a workgroup writes its fp32 sums to the workspace and counts itself in on its tile's counter; whoever comes last adds the slices in
// ascending order and finishes the tile, and sets the counter back to zero.  Which workgroup that is depends on timing, what it computes does not.
// All of that goes past the L2 of an XCD by device-scope accesses, without fences (as bias_grad_split_kernel).
// Measured, weights from memory: forward 1 x 8192 x 16384 99 to 101 us, 5.3 TB/s (a large copy 4.8, a stream of reads alone 5.8; on the tiles of gemm_tile.hpp 104); dX of
// 96 x 2048 x 6144 20 us (on those tiles 34), its weights read once from memory and by three tiles from the caches, which is why slices of 128 x 128 tiles, below, take it in 17.
#pragma once
#include "gate.hpp"
#include "gemm_slim.hpp"

namespace axo {

struct GatedSlimSched {
    int tiles_m, tiles_n;
    int slices, chunks;   // slices of a tile's reduction, chunks of 64 in each but the last
    uint32_t* counters;   // one per tile, zero
    float* partial;       // [tile][slice][BM x columns]
};

template <int OP, int BM, int BC, int NW, int ST>
struct GatedSlimCfg {
    static constexpr int PARTS = OP == GATED_FWD ? 2 : 1, COLS = BC * PARTS;  // columns of B
    static constexpr int THREADS = NW * 64;
    static constexpr int STAGE_BYTES = (BM + COLS) * TILE_BK * 2;
    static constexpr int PART_STRIDE = COLS + 4, PART_BYTES = BM * PART_STRIDE * 4;
    static constexpr int WAVE_BYTES = ST * STAGE_BYTES > PART_BYTES ? ST * STAGE_BYTES : PART_BYTES;
    static constexpr int LDS_BYTES = NW * WAVE_BYTES;
    static constexpr int LOADS = STAGE_BYTES / 1024;
    static_assert(BM % 16 == 0 && BC % 32 == 0 && LDS_BYTES <= 160 * 1024 && (ST - 1) * LOADS < 64, "LDS of one CU, loads that a wait can count");
};

// From the sums of four columns of a row to the outputs.  x1, x2: the biases, or G and U.
template <int OP, int PARTS>
__device__ __forceinline__ void gated_finish(const GatedArgs& g, const f32x4 (&sum)[PARTS], const f32x4 x1, const f32x4 x2, int row, int col, int valid) {
    auto store = [&](bf16_t* to, int64_t ld, f32x4 v) __attribute__((always_inline)) {
        GemmArgs h;
        h.C = to;
        h.ldc = ld;
        store_bf16_quad(h, v, row, col, valid);
    };
    if constexpr (OP == GATED_DX || OP == GATED_DW) store(g.C, g.ldc, sum[0]);
    else
        with_gate(g.gate, [&](auto gate) __attribute__((always_inline)) {
            constexpr int GATE = decltype(gate)::value;
            f32x4 v, w;
            if constexpr (OP == GATED_FWD) {
                const f32x4 gs = sum[0] + x1, us = sum[PARTS - 1] + x2;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = gate_value<GATE>(gs[e]) * us[e];
                store(g.C, g.ldc, v);
                if (!g.G) return;
                store(g.G, g.ldz, gs);
                store(g.U, g.ldz, us);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float2 a = gate_both<GATE>(x1[e]);
                    v[e] = sum[0][e] * x2[e] * a.y;
                    w[e] = sum[0][e] * a.x;
                }
                store(g.C, g.ldc, v);
                store(g.U, g.ldc, w);
            }
        });
}

template <int OP, int BM, int BC, int NW, int ST>
__global__ void __launch_bounds__(NW * 64) gated_slim_kernel(GatedProduct<OP> g, GatedSlimSched sc) {
    using C = GatedSlimCfg<OP, BM, BC, NW, ST>;
    constexpr int LB = OP == GATED_FWD ? MC : KC;
    using OA = SlimOperand<BM, KC>;
    using OB = SlimOperand<BC, LB>;
    constexpr int TM = BM / 16, TN = BC / 16, PARTS = C::PARTS;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // the slices of a tile follow each other, the tiles of a column of them, too: what they share of the operands meets in an XCD's L2
    const int id = xcd_run(blockIdx.x, gridDim.x), tile = id / sc.slices, slice = id % sc.slices;
    const int i0 = tile % sc.tiles_m * BM, j0 = tile / sc.tiles_m * BC;
    const int KT = (g.R + TILE_BK - 1) / TILE_BK;  // of one product
    const int first = slice * sc.chunks, end = min((OP == GATED_DX ? 2 : 1) * KT, first + sc.chunks);

    OA oa;
    OB ob;
    oa.init(lane, g.lda);
    ob.init(lane, g.ldb);
    const uint32_t a_bound = operand_bound<KC>(g.lda, min(BM, g.Mo - i0), g.R), b_bound = operand_bound<LB>(g.ldb, min(BC, g.No - j0), g.R);
    u32x4_t a_rsrc[2], b_rsrc[2];
    a_rsrc[0] = tile_rsrc(OA::origin(g.A, g.lda, i0), a_bound);
    b_rsrc[0] = tile_rsrc(OB::origin(g.B, g.ldb, j0), b_bound);
    if constexpr (OP == GATED_DX) a_rsrc[1] = tile_rsrc(OA::origin(g.A2, g.lda, i0), a_bound);
    if constexpr (OP != GATED_DACT) b_rsrc[1] = tile_rsrc(OB::origin(g.B2, g.ldb, j0), b_bound);
    const uint32_t a_step = OA::chunk_step(g.lda), b_step = OB::chunk_step(g.ldb);
    char* const mine = smem + wave * C::WAVE_BYTES;
    const uint32_t mine_lds = (uint32_t)(uintptr_t)(lds_void_ptr)smem + wave * C::WAVE_BYTES;

    // one direct-to-LDS load: 16 bytes per lane to LDS address M0 + 16 * lane (see gemm_tile_body)
    auto load_lds = [](uint32_t lds_dst, uint32_t off, u32x4_t rsrc, uint32_t soff) __attribute__((always_inline)) {
        asm volatile("buffer_load_dwordx4 %0, %1, %2 offen lds"
                     :
                     : "v"(off), "s"(rsrc), "s"(soff), "{m0}"(lds_dst)
                     : "memory");
    };
    auto issue = [&](const int s, const int chunk) __attribute__((always_inline)) {
        const bool second = OP == GATED_DX && chunk >= KT;
        const int at = second ? chunk - KT : chunk;
        const uint32_t a_soff = (uint32_t)at * a_step, b_soff = (uint32_t)at * b_step, dst = mine_lds + s * C::STAGE_BYTES;
        u32x4_t ar = a_rsrc[0], br = b_rsrc[0];
        if constexpr (OP == GATED_DX) {  // the descriptors differ in nothing but their base
            ar[0] = second ? a_rsrc[1][0] : ar[0];
            ar[1] = second ? a_rsrc[1][1] : ar[1];
            br[0] = second ? b_rsrc[1][0] : br[0];
            br[1] = second ? b_rsrc[1][1] : br[1];
        }
#pragma unroll
        for (int j = 0; j < OB::LOADS; ++j) {
            load_lds(dst + OA::BYTES + j * 1024, ob.off[j], br, b_soff);
            if constexpr (PARTS == 2) load_lds(dst + OA::BYTES + OB::BYTES + j * 1024, ob.off[j], b_rsrc[1], b_soff);
        }
#pragma unroll
        for (int j = 0; j < OA::LOADS; ++j) load_lds(dst + j * 1024, oa.off[j], ar, a_soff);
    };

    f32x4 acc[TM][TN * PARTS];
#pragma unroll
    for (int a = 0; a < TM; ++a)
#pragma unroll
        for (int b = 0; b < TN * PARTS; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[a][b][e] = 0.0f;

    // One chunk, held in stage s; the stages of a wave are filled in turn.
    auto chunk_step = [&](auto s_tag, const int chunk) __attribute__((always_inline)) {
        constexpr int s = decltype(s_tag)::value;
        const int later = (end - 1 - chunk) / NW;  // chunks of this wave behind it
        if (later >= ST - 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"((ST - 1) * C::LOADS) : "memory");
        else if (ST > 3 && later == 2) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * C::LOADS) : "memory");
        else if (ST > 2 && later == 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(C::LOADS) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        const char* const stage = mine + s * C::STAGE_BYTES;
        bf16x8 fa[2][TM], fb[2][TN * PARTS];
#pragma unroll
        for (int kq = 0; kq < 2; ++kq) {
#pragma unroll
            for (int a = 0; a < TM; ++a) fa[kq][a] = oa.read(stage, a, kq);
#pragma unroll
            for (int b = 0; b < TN * PARTS; ++b) fb[kq][b] = ob.read(stage + OA::BYTES + b / TN * OB::BYTES, b % TN, kq);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the stage is in registers: refill it
        if (chunk + ST * NW < end) issue(s, chunk + ST * NW);
        const int at = OP == GATED_DX && chunk >= KT ? chunk - KT : chunk;
        if (g.R % TILE_BK != 0 && at == KT - 1) {  // what a KC operand holds behind the end of its rows, in both operands
            const int left = g.R - at * TILE_BK - 8 * (lane >> 4);
#pragma unroll
            for (int kq = 0; kq < 2; ++kq) {
#pragma unroll
                for (int a = 0; a < TM; ++a) fa[kq][a] = first_elements(fa[kq][a], left - kq * 32);
                if constexpr (LB == KC)
#pragma unroll
                    for (int b = 0; b < TN; ++b) fb[kq][b] = first_elements(fb[kq][b], left - kq * 32);
            }
        }
#pragma unroll
        for (int kq = 0; kq < 2; ++kq)
#pragma unroll
            for (int a = 0; a < TM; ++a)
#pragma unroll
                for (int b = 0; b < TN * PARTS; ++b)
                    acc[a][b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[kq][b], fa[kq][a], acc[a][b], 0, 0, 0);
    };
#pragma unroll
    for (int s = 0; s < ST; ++s)
        if (first + wave + s * NW < end) issue(s, first + wave + s * NW);

    // The outputs of a thread, four consecutive columns of a row at a time.  G and U, or the biases, are requested here, so that they arrive during the
    // reduction (the waits of the loop count these loads, too, which makes them no weaker).
    constexpr int QPR = BC / 4, QUADS = BM * QPR, ROUNDS = (QUADS + C::THREADS - 1) / C::THREADS;
    auto quad_row = [&](int i) __attribute__((always_inline)) { return (i * C::THREADS + tid) / QPR; };
    auto quad_col = [&](int i) __attribute__((always_inline)) { return (i * C::THREADS + tid) % QPR * 4; };
    f32x4 x1[ROUNDS], x2[ROUNDS];
    auto extras = [&](const bf16_t* p, f32x4& x, int i) __attribute__((always_inline)) {
        const int row = i0 + quad_row(i), col = j0 + quad_col(i), valid = quad_row(i) < BM && row < g.Mo ? g.No - col : 0;
        x = f32x4{0.f, 0.f, 0.f, 0.f};
        if (p) x = load_bf16x4(OP == GATED_FWD ? p + col : p + (int64_t)row * g.ldaux + col, valid);
    };
    if constexpr (OP != GATED_DX)
#pragma unroll
        for (int i = 0; i < ROUNDS; ++i) {
            extras(OP == GATED_FWD ? g.bias : g.aux, x1[i], i);
            extras(OP == GATED_FWD ? g.bias2 : g.aux2, x2[i], i);
        }

    for (int chunk = first + wave; chunk < end; chunk += ST * NW) {
        chunk_step(IC<0>{}, chunk);
        if (ST > 1 && chunk + NW < end) chunk_step(IC<(ST > 1 ? 1 : 0)>{}, chunk + NW);
        if (ST > 2 && chunk + 2 * NW < end) chunk_step(IC<(ST > 2 ? 2 : 0)>{}, chunk + 2 * NW);
        if (ST > 3 && chunk + 3 * NW < end) chunk_step(IC<(ST > 3 ? 3 : 0)>{}, chunk + 3 * NW);
    }

    // Partial tiles to LDS (each wave inside its own region, whose loads have all landed and been read), then every thread adds the partials of its outputs.
    // acc[a][b][e] is element (a * 16 + lane % 16, b * 16 + 4 * (lane / 16) + e) of the tile.
    const int n_part = min(NW, end - first);
    if (wave < n_part) {
        float* part = reinterpret_cast<float*>(mine);
#pragma unroll
        for (int a = 0; a < TM; ++a)
#pragma unroll
            for (int b = 0; b < TN * PARTS; ++b)
                *reinterpret_cast<f32x4*>(part + (a * 16 + (lane & 15)) * C::PART_STRIDE + b * 16 + 4 * (lane >> 4)) = acc[a][b];
    }
    __syncthreads();
    f32x4 sum[ROUNDS][PARTS];
#pragma unroll
    for (int i = 0; i < ROUNDS; ++i)
#pragma unroll
        for (int q = 0; q < PARTS; ++q) {
            sum[i][q] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (quad_row(i) < BM) {
                const char* const parts = smem + (quad_row(i) * C::PART_STRIDE + q * BC + quad_col(i)) * 4;
                for (int w = 0; w < n_part; ++w) sum[i][q] += *reinterpret_cast<const f32x4*>(parts + w * C::WAVE_BYTES);
            }
        }
    if (sc.slices > 1) {
        constexpr int TILE = BM * C::COLS;
        float* const all = sc.partial + (int64_t)tile * sc.slices * TILE;
        auto place = [&](int i, int q) __attribute__((always_inline)) { return quad_row(i) * C::COLS + q * BC + quad_col(i); };
#pragma unroll
        for (int i = 0; i < ROUNDS; ++i)
#pragma unroll
            for (int q = 0; q < PARTS; ++q)
                if (quad_row(i) < BM && i0 + quad_row(i) < g.Mo)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        __hip_atomic_store(all + (int64_t)slice * TILE + place(i, q) + e, sum[i][q][e], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wave's sums have arrived where all XCDs see them
        __syncthreads();                                  // and those of all waves; the partial tiles in LDS have been read
        uint32_t* const arrived = reinterpret_cast<uint32_t*>(smem);
        if (tid == 0) *arrived = __hip_atomic_fetch_add(sc.counters + tile, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __syncthreads();
        if (*arrived != (uint32_t)(sc.slices - 1)) return;
#pragma unroll
        for (int i = 0; i < ROUNDS; ++i)
#pragma unroll
            for (int q = 0; q < PARTS; ++q) {
                sum[i][q] = f32x4{0.f, 0.f, 0.f, 0.f};
                if (quad_row(i) < BM && i0 + quad_row(i) < g.Mo)
                    for (int k0 = 0; k0 < sc.slices; k0 += 4) {  // four slices requested at a time, added in ascending order
                        f32x4 v[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k)
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                v[k][e] = k0 + k < sc.slices ? __hip_atomic_load(all + (int64_t)(k0 + k) * TILE + place(i, q) + e, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0.f;
#pragma unroll
                        for (int k = 0; k < 4; ++k) sum[i][q] += v[k];
                    }
            }
        if (tid == 0) __hip_atomic_store(sc.counters + tile, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
#pragma unroll
    for (int i = 0; i < ROUNDS; ++i) {
        const int row = i0 + quad_row(i), col = j0 + quad_col(i);
        if (quad_row(i) < BM && row < g.Mo && col < g.No) gated_finish<OP>(g, sum[i], x1[i], x2[i], row, col, min(4, g.No - col));
    }
}

// ---- 128 x 128 tiles whose reductions are cut into slices ----------------------------------------
// For outputs of too few tiles for the CUs and reductions too long for one of them.  What a workgroup computes is a product like any other, on its slice of the operands (of both
// products of dX), and leaves its fp32 sums in the workspace; the tiles of a slice follow each other, so that an XCD's L2 has what they share.  A second launch adds the slices
// in ascending order and has the epilogue: a tile's last workgroup, doing that alone, would read a megabyte or more at a CU's share of the memory (128 x 13952 x 272 through the derivative
// 32 us that way, 15 this).  Measured: forward 1760 x 15131 x 128 28 us (on whole tiles 77), dX of 96 x 2048 x 6144 14 us and 3 for the second launch.
struct GatedSplitSched {
    int tiles_m, tiles_n;
    int slices, chunks;  // of a tile's reduction, steps of 64 in each but the last
    float* partial;      // [tile][slice][128][128]
};
constexpr int SPLIT_TILE = 128 * 128;
// Where a tile's outputs are, and with two weight gradients whose.
template <int OP>
__device__ __forceinline__ void split_tile(const GatedSplitSched& sc, int tile, GatedArgs& g, int& i0, int& j0) {
    int tn = tile / sc.tiles_m;
    if (OP == GATED_DW && tn >= sc.tiles_n / 2) {
        tn -= sc.tiles_n / 2;
        g.B = g.B2;
        g.C = g.U;
    }
    i0 = tile % sc.tiles_m * 128;
    j0 = tn * gated_cols<OP>(128);
}
template <int OP, bool LINES>
__global__ void __launch_bounds__(TILE_THREADS, 1) gated_split_kernel(GatedProduct<OP> product, GatedSplitSched sc) {
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    constexpr int LA = OP == GATED_DW ? MC : KC, LB = OP == GATED_FWD || OP == GATED_DW ? MC : KC;
    const int id = xcd_run(blockIdx.x, gridDim.x), tiles = sc.tiles_m * sc.tiles_n, tile = id % tiles, slice = id / tiles;
    GatedSlice<OP> g;
    static_cast<GatedProduct<OP>&>(g) = product;
    int i0, j0;
    split_tile<OP>(sc, tile, g, i0, j0);
    g.partial = sc.partial + ((int64_t)tile * sc.slices + slice) * SPLIT_TILE;
    const int64_t from = (int64_t)slice * sc.chunks * TILE_BK, a = LA == KC ? from : from * g.lda, b = LB == KC ? from : from * g.ldb;
    g.R = min(sc.chunks * TILE_BK, g.R - (int)from);
    g.A += a;
    g.B += b;
    if constexpr (OP == GATED_DX) g.A2 += a;
    if constexpr (OP == GATED_DX || OP == GATED_FWD) g.B2 += b;
    gemm_ring_body<128, 128, 4, 2, 4, LA, LB, LINES>(g, i0, j0, smem, threadIdx.x);
}
// Four consecutive columns of a row of the outputs to a thread.
constexpr int SPLIT_JOIN_THREADS = 256;
template <int OP>
__global__ void __launch_bounds__(SPLIT_JOIN_THREADS) gated_split_join_kernel(GatedProduct<OP> product, GatedSplitSched sc) {
    constexpr int COLS = gated_cols<OP>(128), QPR = COLS / 4, PARTS = OP == GATED_FWD ? 2 : 1, BLOCKS = 128 * QPR / SPLIT_JOIN_THREADS;  // of a tile
    const int tile = blockIdx.x / BLOCKS, quad = blockIdx.x % BLOCKS * SPLIT_JOIN_THREADS + threadIdx.x, r = quad / QPR, c = quad % QPR * 4;
    GatedArgs g = product;
    int i0, j0;
    split_tile<OP>(sc, tile, g, i0, j0);
    const int row = i0 + r, col = j0 + c, valid = min(4, g.No - col);
    if (row >= g.Mo || valid <= 0) return;
    const float* const from = sc.partial + (int64_t)tile * sc.slices * SPLIT_TILE + r * 128 + c;
    f32x4 sum[PARTS], x1 = {0.f, 0.f, 0.f, 0.f}, x2 = x1;
    if constexpr (OP == GATED_FWD) {
        if (g.bias) x1 = load_bf16x4(g.bias + col, valid);
        if (g.bias2) x2 = load_bf16x4(g.bias2 + col, valid);
    }
    if constexpr (OP == GATED_DACT) {
        x1 = load_bf16x4(g.aux + (int64_t)row * g.ldaux + col, valid);
        x2 = load_bf16x4(g.aux2 + (int64_t)row * g.ldaux + col, valid);
    }
#pragma unroll
    for (int q = 0; q < PARTS; ++q) sum[q] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < sc.slices; s0 += 4) {  // four slices requested at a time
        f32x4 v[4][PARTS];
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int q = 0; q < PARTS; ++q)
                v[s][q] = s0 + s < sc.slices ? *reinterpret_cast<const f32x4*>(from + (int64_t)(s0 + s) * SPLIT_TILE + q * COLS) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int q = 0; q < PARTS; ++q) sum[q] += v[s][q];
    }
    if constexpr (OP == GATED_DW) {
        if (g.epilogue == EPI_ACC_F32) {
            float* const out = reinterpret_cast<float*>(g.C) + (int64_t)row * g.ldc + col;
            if (valid == 4) *reinterpret_cast<f32x4*>(out) += sum[0];
            else
#pragma unroll
                for (int e = 0; e < 3; ++e)
                    if (e < valid) out[e] += sum[0][e];
            return;
        }
    }
    gated_finish<OP>(g, sum, x1, x2, row, col, valid);
}

}  // namespace axo
