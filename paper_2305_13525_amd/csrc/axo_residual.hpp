// Entry points of include/axo_residual.h: the product with a residual and the norms either side of one.  Part of axo_api.hip's translation
// unit, behind axo_block.hpp.
#pragma once
#include "../../include/axo_residual.h"

#include "axo_block.hpp"
#include "resnorm.hpp"

static_assert((int)AXO_NORM_NONE == axo::KIND_NONE && (int)AXO_NORM_LAYER == axo::KIND_LAYER && (int)AXO_NORM_RMS == axo::KIND_RMS, "one numbering");

namespace axo_block {

// ---- norms around a residual addition ---------------------------------------------------------------

template <typename T, int LANES, int CH>
int launch_resnorm_rows(const axo::ResnormArgs& g, hipStream_t st) {
    constexpr int BLOCK = LANES <= 64 ? 256 : LANES, ROWS = BLOCK / LANES;
    hipLaunchKernelGGL((axo::resnorm_rows_kernel<T, LANES, CH>), dim3(at_most(tiles_in(g.M, ROWS), NORM_MOST_BLOCKS)), dim3(BLOCK), 0, st, g);
    return launched();
}
constexpr int RESNORM_MOST_COLS = 16384;  // of rows in registers
template <typename T>
int launch_resnorm_typed(const axo::ResnormArgs& g, hipStream_t st) {
    if (g.K <= 64) return launch_resnorm_rows<T, 8, 1>(g, st);
    if (g.K <= 128) return launch_resnorm_rows<T, 16, 1>(g, st);
    if (g.K <= 256) return launch_resnorm_rows<T, 32, 1>(g, st);
    if (g.K <= 512) return launch_resnorm_rows<T, 64, 1>(g, st);
    if (g.K <= 1024) return launch_resnorm_rows<T, 128, 1>(g, st);
    if (g.K <= 2048) return launch_resnorm_rows<T, 256, 1>(g, st);
    if (g.K <= 4096) return launch_resnorm_rows<T, 512, 1>(g, st);
    if (g.K <= 8192) return launch_resnorm_rows<T, 512, 2>(g, st);
    if (g.K <= 12288) return launch_resnorm_rows<T, 512, 3>(g, st);
    if (g.K <= RESNORM_MOST_COLS) return launch_resnorm_rows<T, 512, 4>(g, st);
    hipLaunchKernelGGL(axo::resnorm_long_kernel<T>, dim3(at_most(g.M, NORM_MOST_BLOCKS)), dim3(axo::NORM_THREADS), 0, st, g);
    return launched();
}

// Whether the column sums of the backward pass come from a second pass over the data (resnorm_cols_kernel), and where that has its rows' means and its counters in the
// workspace, behind the sums of the slices.
bool resnorm_two_passes(int64_t K) { return K > RESNORM_MOST_COLS; }
size_t resnorm_partial_bytes(int64_t M, int64_t K) { return (size_t)std::max<int64_t>(1, std::min<int64_t>(M, NORM_MOST_SLICES)) * 4 * (size_t)norm_partial_cols(K) * sizeof(float); }
size_t resnorm_means_bytes(int64_t M) { return ((size_t)M * sizeof(float2) + 15) / 16 * 16; }
size_t resnorm_workspace(int64_t M, int64_t K) {
    if (K == 0) return 0;
    return resnorm_partial_bytes(M, K) + (resnorm_two_passes(K) ? resnorm_means_bytes(M) + ((size_t)K + 63) / 64 * sizeof(uint32_t) : 0);
}

int launch_resnorm_join(const axo::ResnormBwdArgs& g, hipStream_t st) {
    if (!g.want_cols) return AXO_OK;
    hipLaunchKernelGGL(axo::resnorm_join_kernel, dim3(at_most(tiles_in(g.K, axo::RESNORM_JOIN_COLS), NORM_MOST_BLOCKS)), dim3(axo::RESNORM_JOIN_THREADS), 0, st, g);
    return launched();
}
template <typename T, int LANES, int CH, int GROUPS, bool AHEAD>
int launch_resnorm_bwd_groups(axo::ResnormBwdArgs& g, hipStream_t st) {
    // a workgroup to every row, or pair of long ones, whose sums are much to write and read again (one and two: 200 x 4000 16.2 and 14.3 us, 256 x 4096 17.9 and 15.4; 8 x 4000 8.7 and 10.3,
    // 300 x 512 8.9 and 10.0)
    g.slices = (int)std::min<int64_t>(tiles_in(g.M, GROUPS * (g.K > 2048 && g.M >= 128 ? 2 : 1)), NORM_MOST_SLICES);
    constexpr int lds = CH == axo::RESNORM_LDS_CHUNKS ? 2 * CH * LANES * 8 * (int)sizeof(float) : 0;
    static std::atomic<uint64_t> raised{0};
    if (lds > 0 && !raise_lds_limit(reinterpret_cast<const void*>(axo::resnorm_bwd_rows_kernel<T, LANES, CH, GROUPS, AHEAD>), lds, &raised)) return AXO_ERR_HIP;
    hipLaunchKernelGGL((axo::resnorm_bwd_rows_kernel<T, LANES, CH, GROUPS, AHEAD>), dim3((unsigned)g.slices), dim3(LANES * GROUPS), lds, st, g);
    return launched();
}
template <typename T, int LANES, int CH>
int launch_resnorm_bwd_rows(axo::ResnormBwdArgs& g, hipStream_t st) {
    // the next row's loads ahead, as long as there are registers for them
    return launch_resnorm_bwd_groups<T, LANES, CH, CH == 1 ? 512 / LANES : 1, CH == 1 || (CH == 2 && sizeof(T) == 2)>(g, st);
}
template <typename T>
int launch_resnorm_bwd_typed(axo::ResnormBwdArgs g, hipStream_t st) {
    if (g.M > 0) {
        const int rc = [&] {
            if (g.K <= 64) return launch_resnorm_bwd_rows<T, 8, 1>(g, st);
            if (g.K <= 128) return launch_resnorm_bwd_rows<T, 16, 1>(g, st);
            if (g.K <= 256) return launch_resnorm_bwd_rows<T, 32, 1>(g, st);
            if (g.K <= 512) return launch_resnorm_bwd_rows<T, 64, 1>(g, st);
            if (g.K <= 1024) return launch_resnorm_bwd_rows<T, 128, 1>(g, st);
            if (g.K <= 2048) return launch_resnorm_bwd_rows<T, 256, 1>(g, st);
            if (g.K <= 4096) return launch_resnorm_bwd_rows<T, 512, 1>(g, st);
            if (g.K <= 8192) return launch_resnorm_bwd_rows<T, 512, 2>(g, st);
            if (g.K <= 12288) return launch_resnorm_bwd_rows<T, 512, 3>(g, st);
            if (g.K <= RESNORM_MOST_COLS) return launch_resnorm_bwd_rows<T, 512, 4>(g, st);
            hipLaunchKernelGGL(axo::resnorm_bwd_long_kernel<T>, dim3(at_most(g.M, NORM_MOST_BLOCKS)), dim3(axo::NORM_THREADS), 0, st, g);
            return launched();
        }();
        if (rc) return rc;
    }
    if (!g.want_cols) return AXO_OK;
    if (!g.means) return launch_resnorm_join(g, st);
    if (g.M == 0) {  // sums of nothing
        g.slices = 0;
        return launch_resnorm_join(g, st);
    }
    g.rows_per_slice = norm_slice_rows(g.M);
    g.slices = (int)tiles_in(g.M, g.rows_per_slice);
    hipLaunchKernelGGL(axo::resnorm_cols_kernel<T>, dim3(at_most(tiles_in(g.K, axo::NORM_STRIP) * g.slices, NORM_MOST_BLOCKS)), dim3(axo::NORM_COL_THREADS), 0, st, g);
    return launched();
}

// What both passes check: the problem, and the norms' kinds.
int plan_resnorm(const axo_problem_t* p, int type, int norm_a, float scale, int norm_b, Shard& s) {
    if (const int rc = derive_shard(p, &s)) return rc;
    if (k_axis(p) != 1) return AXO_ERR_BAD_GRID;
    if (!known_type(type) || norm_a < AXO_NORM_NONE || norm_a > AXO_NORM_RMS || norm_b < AXO_NORM_LAYER || norm_b > AXO_NORM_RMS || !std::isfinite(scale)) return AXO_ERR_BAD_ARG;
    return AXO_OK;
}

// ---- product with a residual ----------------------------------------------------------------------------

bool known_epilogue(int epilogue) { return epilogue >= AXO_EPI_NONE && epilogue <= AXO_EPI_BIAS_GELU_ERF; }
bool has_act(int epilogue) { return epilogue == AXO_EPI_BIAS_GELU_TANH || epilogue == AXO_EPI_BIAS_GELU_ERF; }

}  // namespace axo_block

extern "C" {

int axo_resnorm_fwd(const axo_problem_t* p, const void* B, int64_t ldb, const void* X, int64_t ldx, int type, int norm_a, const void* gamma_a, const void* beta_a,
                    const void* gate, float scale, int norm_b, const void* gamma_b, const void* beta_b, float eps, void* S, int64_t lds, void* Y, int64_t ldy,
                    float* stats, void* hip_stream) {
    using namespace axo_block;
    Shard s;
    if (const int rc = plan_resnorm(p, type, norm_a, scale, norm_b, s)) return rc;
    if (!valid_eps(eps)) return AXO_ERR_BAD_ARG;
    const int64_t n = s.M > 0 ? s.Kl : 0;
    if (const int rc = first_error({check_matrix(B, ldb, s.M, s.Kl), check_matrix(X, ldx, s.M, s.Kl), check_matrix(S, lds, s.M, s.Kl), check_matrix(Y, ldy, s.M, s.Kl),
                                    check_vector(gamma_a, n, 16, true), check_vector(beta_a, n, 16, true), check_vector(gate, n, 16, true),
                                    check_vector(gamma_b, n, 16, true), check_vector(beta_b, n, 16, true), check_vector(stats, s.Kl > 0 ? s.M : 0, 16, true)}))
        return rc;
    if (s.M == 0 || s.Kl == 0) return AXO_OK;
    Buffers b;
    b.reads(B, ldb, s.M, s.Kl, 2);
    b.reads(X, ldx, s.M, s.Kl, elem_of(type));
    for (const void* v : {gamma_a, beta_a, gate, gamma_b, beta_b}) b.reads(v, n, 1, n, 2);
    b.writes(S, lds, s.M, s.Kl, elem_of(type));
    b.writes(Y, ldy, s.M, s.Kl, 2);
    b.writes(stats, 4 * s.M, 1, 4 * s.M, 4);
    if (const int rc = b.check()) return rc;
    axo::ResnormArgs g{};
    g.B = static_cast<const bf16_t*>(B); g.ldb = ldb;
    g.X = X; g.ldx = ldx;
    g.S = S; g.lds = lds;
    g.Y = static_cast<bf16_t*>(Y); g.ldy = ldy;
    g.gamma_a = static_cast<const bf16_t*>(gamma_a);
    g.beta_a = static_cast<const bf16_t*>(beta_a);
    g.gate = static_cast<const bf16_t*>(gate);
    g.gamma_b = static_cast<const bf16_t*>(gamma_b);
    g.beta_b = static_cast<const bf16_t*>(beta_b);
    g.stats = reinterpret_cast<axo::f32x4*>(stats);
    g.M = (int)s.M; g.K = (int)s.Kl;
    g.kind_a = norm_a; g.kind_b = norm_b;
    g.scale = scale; g.eps = eps;
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    return type == AXO_TYPE_F32 ? launch_resnorm_typed<float>(g, st) : launch_resnorm_typed<bf16_t>(g, st);
}

int axo_resnorm_bwd(const axo_problem_t* p, const void* dY, int64_t lddy, const void* dS, int64_t ldds, const void* B, int64_t ldb, const void* S, int64_t lds, int type,
                    int norm_a, const void* gamma_a, const void* beta_a, const void* gate, float scale, int norm_b, const void* gamma_b, const float* stats,
                    void* dX, int64_t lddx, void* dB, int64_t lddb, float* dgamma_a, float* dbeta_a, float* dgate, float* dgamma_b, float* dbeta_b, int accumulate,
                    void* ws, size_t ws_bytes, void* hip_stream) {
    using namespace axo_block;
    Shard s;
    if (const int rc = plan_resnorm(p, type, norm_a, scale, norm_b, s)) return rc;
    if (accumulate != 0 && accumulate != 1) return AXO_ERR_BAD_ARG;
    const int64_t n = s.M > 0 ? s.Kl : 0;
    if (const int rc = first_error({check_matrix(dY, lddy, s.M, s.Kl), dS ? check_matrix(dS, ldds, s.M, s.Kl) : AXO_OK, check_matrix(B, ldb, s.M, s.Kl),
                                    check_matrix(S, lds, s.M, s.Kl), check_matrix(dX, lddx, s.M, s.Kl), check_matrix(dB, lddb, s.M, s.Kl),
                                    check_vector(gamma_a, s.Kl, 16, true), check_vector(beta_a, s.Kl, 16, true), check_vector(gate, s.Kl, 16, true),
                                    check_vector(gamma_b, n, 16, true), check_vector(stats, s.Kl > 0 ? s.M : 0, 16, false)}))
        return rc;
    Buffers b;
    b.reads(dY, lddy, s.M, s.Kl, 2);
    if (dS) b.reads(dS, ldds, s.M, s.Kl, elem_of(type));
    b.reads(B, ldb, s.M, s.Kl, 2);
    b.reads(S, lds, s.M, s.Kl, elem_of(type));
    for (const void* v : {gamma_a, beta_a, gate, gamma_b}) b.reads(v, s.Kl, 1, s.Kl, 2);
    b.reads(stats, 4 * s.M, 1, 4 * s.M, 4);
    b.writes(dX, lddx, s.M, s.Kl, elem_of(type));
    b.writes(dB, lddb, s.M, s.Kl, 2);
    axo::ResnormBwdArgs g{};
    for (float* v : {dgamma_a, dbeta_a, dgate, dgamma_b, dbeta_b}) {
        if (const int rc = check_vector(v, s.Kl, 4, true)) return rc;
        b.writes(v, s.Kl, 1, s.Kl, 4);
        g.want_cols |= v != nullptr;
    }
    if (s.Kl == 0) return AXO_OK;
    if (g.want_cols) {
        const size_t need = resnorm_workspace(s.M, s.Kl);
        if (!ws || ws_bytes < need) return AXO_ERR_WORKSPACE;
        if (!aligned16(ws)) return AXO_ERR_MISALIGNED;
        g.partial = static_cast<float*>(ws);
        g.partial_cols = norm_partial_cols(s.Kl);
        if (resnorm_two_passes(s.Kl)) {
            char* const behind = static_cast<char*>(ws) + resnorm_partial_bytes(s.M, s.Kl);
            g.means = reinterpret_cast<float2*>(behind);
            g.counters = reinterpret_cast<uint32_t*>(behind + resnorm_means_bytes(s.M));
        }
        b.writes(ws, (int64_t)need, 1, (int64_t)need, 1);
    }
    if (const int rc = b.check()) return rc;
    g.dY = static_cast<const bf16_t*>(dY); g.lddy = lddy;
    g.dS = dS; g.ldds = ldds;
    g.B = static_cast<const bf16_t*>(B); g.ldb = ldb;
    g.S = S; g.lds = lds;
    g.dX = dX; g.lddx = lddx;
    g.dB = static_cast<bf16_t*>(dB); g.lddb = lddb;
    g.gamma_a = static_cast<const bf16_t*>(gamma_a);
    g.beta_a = static_cast<const bf16_t*>(beta_a);
    g.gate = static_cast<const bf16_t*>(gate);
    g.gamma_b = static_cast<const bf16_t*>(gamma_b);
    g.stats = reinterpret_cast<const axo::f32x4*>(stats);
    g.dgamma_a = dgamma_a; g.dbeta_a = dbeta_a; g.dgate = dgate; g.dgamma_b = dgamma_b; g.dbeta_b = dbeta_b;
    g.M = (int)s.M; g.K = (int)s.Kl;
    g.kind_a = norm_a; g.kind_b = norm_b;
    g.accumulate = accumulate;
    g.scale = scale;
    const hipStream_t st = static_cast<hipStream_t>(hip_stream);
    return type == AXO_TYPE_F32 ? launch_resnorm_bwd_typed<float>(g, st) : launch_resnorm_bwd_typed<bf16_t>(g, st);
}

size_t axo_resnorm_workspace_bytes(const axo_problem_t* p) {
    axo_host::Shard s;
    return axo_host::derive_shard(p, &s) || axo_block::k_axis(p) != 1 ? 0 : axo_block::resnorm_workspace(s.M, s.Kl);
}

int axo_fc_add(const axo_problem_t* p, const void* X, int64_t ldx, const void* W, int64_t ldw, const void* bias, int epilogue, const void* R, int64_t ldr, int type,
               float scale, void* Z, int64_t ldz, void* Y, int64_t ldy, void* ws, size_t ws_bytes, void* hip_stream) {
    using namespace axo_block;
    return guarded([&]() -> int {
        Shard s;
        if (const int rc = derive_shard(p, &s)) return rc;
        if (!known_epilogue(epilogue) || (epilogue != AXO_EPI_NONE && !bias)) return AXO_ERR_BAD_EPILOGUE;
        if (!known_type(type) || !std::isfinite(scale) || (Z && !has_act(epilogue))) return AXO_ERR_BAD_ARG;
        if (has_act(epilogue) && k_axis(p) != 1) return AXO_ERR_BAD_GRID;
        const bool adds = s.k_coord == 0;  // the bias and the residual: on one of the shards whose parts are summed up
        const int64_t n = s.M > 0 ? s.Nl : 0;
        if (const int rc = first_error({check_matrix(X, ldx, s.M, s.Kl), check_matrix(W, ldw, s.Kl, s.Nl), check_matrix(Y, ldy, s.M, s.Nl),
                                        epilogue != AXO_EPI_NONE ? check_vector(bias, n, 16, false) : AXO_OK, adds ? check_matrix(R, ldr, s.M, s.Nl) : AXO_OK,
                                        Z ? check_matrix(Z, ldz, s.M, s.Nl) : AXO_OK}))
            return rc;
        if (n == 0) return AXO_OK;
        Buffers b;
        b.reads(X, ldx, s.M, s.Kl, 2);
        b.reads(W, ldw, s.Kl, s.Nl, 2);
        if (adds) {
            if (epilogue != AXO_EPI_NONE) b.reads(bias, s.Nl, 1, s.Nl, 2);
            b.reads(R, ldr, s.M, s.Nl, elem_of(type));
        }
        b.writes(Y, ldy, s.M, s.Nl, elem_of(type));
        if (Z) b.writes(Z, ldz, s.M, s.Nl, 2);
        const size_t need = gated_plans(s).of[axo::FC_ADD].cut.bytes;
        if (need > 0) {
            if (!ws || ws_bytes < need) return AXO_ERR_WORKSPACE;
            if (!aligned16(ws)) return AXO_ERR_MISALIGNED;
            b.writes(ws, (int64_t)need, 1, (int64_t)need, 1);
        }
        if (const int rc = b.check()) return rc;
        GatedArgs g{};
        g.A = static_cast<const bf16_t*>(X); g.lda = ldx;
        g.B = static_cast<const bf16_t*>(W); g.ldb = ldw;
        g.bias = adds && epilogue != AXO_EPI_NONE ? static_cast<const bf16_t*>(bias) : nullptr;
        g.aux = adds ? static_cast<const bf16_t*>(R) : nullptr; g.ldaux = ldr;
        g.C = static_cast<bf16_t*>(Y); g.ldc = ldy;
        g.G = static_cast<bf16_t*>(Z); g.ldz = ldz;
        g.Mo = (int)s.M; g.No = (int)s.Nl; g.R = (int)s.Kl;
        g.gate = epilogue;
        g.wide = type == AXO_TYPE_F32;
        g.scale = scale;
        return launch_gated<axo::FC_ADD>(g, s, ws, static_cast<hipStream_t>(hip_stream));
    });
}

int axo_fc_add_dact(const axo_problem_t* p, const void* dY, int64_t lddy, int type, const void* Z, int64_t ldz, int epilogue, float scale, void* dZ, int64_t lddz,
                    void* hip_stream) {
    using namespace axo_block;
    Shard s;
    if (const int rc = derive_shard(p, &s)) return rc;
    if (!known_epilogue(epilogue)) return AXO_ERR_BAD_EPILOGUE;
    if (!known_type(type) || !std::isfinite(scale) || (Z && !has_act(epilogue))) return AXO_ERR_BAD_ARG;
    if (has_act(epilogue) && k_axis(p) != 1) return AXO_ERR_BAD_GRID;
    if (const int rc = first_error({check_matrix(dY, lddy, s.M, s.Nl), has_act(epilogue) ? check_matrix(Z, ldz, s.M, s.Nl) : AXO_OK, check_matrix(dZ, lddz, s.M, s.Nl)})) return rc;
    if (s.M == 0 || s.Nl == 0) return AXO_OK;
    Buffers b;
    b.reads(dY, lddy, s.M, s.Nl, elem_of(type));
    if (Z) b.reads(Z, ldz, s.M, s.Nl, 2);
    b.writes(dZ, lddz, s.M, s.Nl, 2);
    if (const int rc = b.check()) return rc;
    axo::AddMapArgs g{};
    g.dY = dY; g.lddy = lddy;
    g.Z = static_cast<const bf16_t*>(Z); g.ldz = ldz;
    g.dZ = static_cast<bf16_t*>(dZ); g.lddz = lddz;
    g.M = (int)s.M; g.N = (int)s.Nl;
    g.epilogue = epilogue;
    g.scale = scale;
    const dim3 grid(at_most((tiles_in(g.N, 8) * g.M + axo::GATED_MAP_THREADS - 1) / axo::GATED_MAP_THREADS, 1 << 20)), block(axo::GATED_MAP_THREADS);
    if (type == AXO_TYPE_F32) hipLaunchKernelGGL(axo::add_map_kernel<float>, grid, block, 0, static_cast<hipStream_t>(hip_stream), g);
    else hipLaunchKernelGGL(axo::add_map_kernel<bf16_t>, grid, block, 0, static_cast<hipStream_t>(hip_stream), g);
    return launched();
}

size_t axo_fc_add_workspace_bytes(const axo_problem_t* p) {
    axo_host::Shard s;
    return axo_host::derive_shard(p, &s) ? 0 : axo_block::gated_plans(s).of[axo::FC_ADD].cut.bytes;
}

}  // extern "C"
