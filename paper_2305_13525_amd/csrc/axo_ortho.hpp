// Entry points of include/axo_update.h: validation, choice of tiles, launches.  Part of axo_api.hip's translation unit, behind axo_block.hpp.
#pragma once
#include "../../include/axo_update.h"

#include <cmath>

#include "axo_host.hpp"
#include "ortho.hpp"

namespace axo_update {

using namespace axo_host;
using axo::bf16_t;

inline int launched() { return hipGetLastError() == hipSuccess ? AXO_OK : AXO_ERR_HIP; }

// Everything that a call takes from its sizes.
struct OrthoPlan {
    int64_t s, l;    // padded
    bool tall;       // more rows than columns
    int exponent;    // X is held as its values times 2^exponent
    bool at_once;    // a step is one launch
    bool rest;       // a step is two, gram and the rest
    axo::SymPlan gram, poly;
    size_t counters, sums, A, Q, X[2], partial, bytes;  // offsets in the workspace
};
int make_plan(const Shard& sh, OrthoPlan* p) {
    const int64_t K = sh.Kl, N = sh.Nl;
    auto padded = [](int64_t n) { return (n + axo::ORTHO_PAD - 1) / axo::ORTHO_PAD * axo::ORTHO_PAD; };
    p->tall = K > N;
    p->s = padded(std::min(K, N));
    p->l = padded(std::max(K, N));
    // byte offsets inside an operand are formed in 32 bits, over its whole padded length
    if ((p->l + 4 * axo::TILE_BK) * p->s * 2 >= (int64_t)0xFFFF0000) return AXO_ERR_BAD_SIZE;
    // about sqrt(K N), whose reciprocal is what the values of X come to; fp16 ends at 2^16, and they reach 2^exponent
    p->exponent = std::min(13, (int)std::floor(0.5 * std::log2((double)K * (double)N)));
    p->gram = axo::sym_plan(p->s, p->l / axo::TILE_BK, NUM_CU);
    p->poly = axo::sym_plan(p->s, p->s / axo::TILE_BK, NUM_CU);
    p->at_once = p->s <= 128 && p->s * p->l <= axo::ORTHO_STEP_MOST;
    p->rest = p->s <= 128 && p->s * p->l <= axo::ORTHO_REST_MOST;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t from = at;
        at += (bytes + 255) / 256 * 256;
        return from;
    };
    auto partials = [](const axo::SymPlan& y) { return (size_t)y.partial_floats() * sizeof(float); };
    p->counters = take((size_t)axo::SYM_MOST_CUT * sizeof(uint32_t));  // where and as many as for any other sizes
    p->sums = take(axo::ORTHO_SUMS * sizeof(double));
    p->A = take((size_t)(p->s * p->s) * 2);
    p->Q = take((size_t)(p->s * p->s) * 2);
    for (size_t& x : p->X) x = take((size_t)(p->s * p->l) * 2);
    p->partial = take(std::max(partials(p->gram), partials(p->poly)));
    p->bytes = at;
    return AXO_OK;
}

// 256 x 128 tiles, and 128 x 128 ones behind them.
struct SymHalfCfg {
    static constexpr int THREADS = axo::TILE_THREADS, LDS_BYTES = std::max(axo::MixSmallCfg::LDS_BYTES, axo::MidCfg::LDS_BYTES);
    static_assert(axo::MixSmallCfg::THREADS == THREADS && axo::MidCfg::THREADS == THREADS, "one launch");
};
template <int SIZE, int LAYOUT, bool SLICED = false>
int launch_sym(const axo::OrthoSym& g, int workgroups, hipStream_t st) {
    using C = std::conditional_t<SIZE == 32, axo::SlimCfg<32, 32, axo::SLIM_WAVES, SLICED ? axo::SLICED_STAGES : 1>, std::conditional_t<SIZE == 64, axo::SmallCfg<false>,
        std::conditional_t<SIZE == 128, axo::MidCfg, std::conditional_t<SIZE == axo::SYM_HALF, SymHalfCfg, axo::MixBigCfg>>>>;
    auto kern = [] {
        if constexpr (SIZE == 32 && SLICED) return axo::ortho_sym_32_sliced_kernel<LAYOUT>;
        else if constexpr (SIZE == 32) return axo::ortho_sym_32_kernel<LAYOUT>;
        else if constexpr (SIZE == 64) return axo::ortho_sym_64_kernel<LAYOUT>;
        else if constexpr (SIZE == 128) return axo::ortho_sym_128_kernel<LAYOUT>;
        else if constexpr (SIZE == axo::SYM_HALF) return axo::ortho_sym_half_kernel<LAYOUT>;
        else return axo::ortho_sym_256_kernel<LAYOUT>;
    }();
    static std::atomic<uint64_t> raised{0};
    if (!raise_lds_limit(reinterpret_cast<const void*>(kern), C::LDS_BYTES, &raised)) return AXO_ERR_HIP;
    hipLaunchKernelGGL(kern, dim3((unsigned)workgroups), dim3(C::THREADS), C::LDS_BYTES, st, g);
    return launched();
}
int launch_sym(axo::OrthoSym g, const axo::SymPlan& y, bool tall, hipStream_t st) {
    g.cut = y.cut;
    g.diagonal = y.diagonal;
    if (y.size == 32 && y.cut.cut > 0) return tall ? launch_sym<32, axo::MC, true>(g, y.workgroups, st) : launch_sym<32, axo::KC, true>(g, y.workgroups, st);
    if (y.size == 32) return tall ? launch_sym<32, axo::MC>(g, y.workgroups, st) : launch_sym<32, axo::KC>(g, y.workgroups, st);
    if (y.size == 64) return tall ? launch_sym<64, axo::MC>(g, y.workgroups, st) : launch_sym<64, axo::KC>(g, y.workgroups, st);
    if (y.size == axo::SYM_HALF) return tall ? launch_sym<axo::SYM_HALF, axo::MC>(g, y.workgroups, st) : launch_sym<axo::SYM_HALF, axo::KC>(g, y.workgroups, st);
    if (y.size == 128) return tall ? launch_sym<128, axo::MC>(g, y.workgroups, st) : launch_sym<128, axo::KC>(g, y.workgroups, st);
    return tall ? launch_sym<256, axo::MC>(g, y.workgroups, st) : launch_sym<256, axo::KC>(g, y.workgroups, st);
}
template <int LB>
int launch_apply(const axo::OrthoApply& g, hipStream_t st) {
    static std::atomic<uint64_t> raised[4]{{0}, {0}, {0}, {0}};
    Tiles tiles = quickest_tiles(g.Mo, g.No, g.R);
    if (tiles == Tiles::tall) tiles = tiles_in(g.Mo, 64) * tiles_in(g.No, 128) <= NUM_CU ? Tiles::wide : Tiles::mid;
    auto go = [&](auto config, auto kern, std::atomic<uint64_t>* up, int rows, int cols) -> int {
        using C = decltype(config);
        if (!raise_lds_limit(reinterpret_cast<const void*>(kern), C::LDS_BYTES, up)) return AXO_ERR_HIP;
        const int tm = (int)tiles_in(g.Mo, rows), tn = (int)tiles_in(g.No, cols);
        hipLaunchKernelGGL(kern, dim3((unsigned)tm * (unsigned)tn), dim3(C::THREADS), C::LDS_BYTES, st, g, tm, tn, std::min(tm, 8));
        return launched();
    };
    if (tiles == Tiles::small) return go(axo::SmallCfg<false>{}, axo::ortho_apply_64_kernel<LB>, &raised[0], 64, 64);
    if (tiles == Tiles::wide) return go(axo::RectCfg<true>{}, axo::ortho_apply_rect_kernel<LB>, &raised[1], 64, 128);
    if (tiles == Tiles::mid) return go(axo::MidCfg{}, axo::ortho_apply_128_kernel<LB>, &raised[2], 128, 128);
    const axo::TileSched sc = plan_columns(g.Mo, g.No, g.R);
    auto kern = axo::ortho_apply_256_kernel<LB>;
    if (!raise_lds_limit(reinterpret_cast<const void*>(kern), axo::MIX_LDS_BYTES, &raised[3])) return AXO_ERR_HIP;
    hipLaunchKernelGGL(kern, dim3(sc.n_big + sc.tiles_m * sc.small_cols), dim3(axo::TILE_THREADS), axo::MIX_LDS_BYTES, st, g, sc);
    return launched();
}

template <int S, int LAYOUT>
int launch_step(const axo::OrthoStep& g, hipStream_t st) {
    using C = std::conditional_t<S == 64, axo::SmallCfg<false>, axo::MidCfg>;
    auto kern = axo::ortho_step_kernel<S, LAYOUT>;
    static std::atomic<uint64_t> raised{0};
    if (!raise_lds_limit(reinterpret_cast<const void*>(kern), C::LDS_BYTES, &raised)) return AXO_ERR_HIP;
    hipLaunchKernelGGL(kern, dim3((unsigned)(g.R / 64)), dim3(C::THREADS), C::LDS_BYTES, st, g);
    return launched();
}
template <int S>
int launch_rest(const axo::OrthoStep& g, const bf16_t* gram, hipStream_t st) {
    using C = std::conditional_t<S == 64, axo::SmallCfg<false>, axo::MidCfg>;
    auto kern = axo::ortho_rest_kernel<S>;
    static std::atomic<uint64_t> raised{0};
    if (!raise_lds_limit(reinterpret_cast<const void*>(kern), C::LDS_BYTES, &raised)) return AXO_ERR_HIP;
    hipLaunchKernelGGL(kern, dim3((unsigned)(g.R / 64)), dim3(C::THREADS), C::LDS_BYTES, st, g, gram);
    return launched();
}
template <typename T>
int launch_load(const axo::OrthoLoadArgs& g, hipStream_t st) {
    hipLaunchKernelGGL(axo::ortho_norm_kernel<T>, dim3(axo::ORTHO_SUMS), dim3(axo::ORTHO_THREADS), 0, st, g);
    if (const int rc = launched()) return rc;
    const int64_t chunks = (int64_t)g.rows * g.cols / 8;
    hipLaunchKernelGGL(axo::ortho_load_kernel<T>, dim3((unsigned)std::min<int64_t>(512, (chunks + axo::ORTHO_THREADS - 1) / axo::ORTHO_THREADS)), dim3(axo::ORTHO_THREADS), 0, st, g);
    return launched();
}

// The quintic whose slope at zero is as large as it can be while what it makes of [0, 1] in a few steps stays around 1.
constexpr float QUINTIC[3] = {3.4445f, -4.7750f, 2.0315f};

int ortho(const OrthoPlan& pl, const axo::OrthoLoadArgs& from, int type, int steps, const float* abc, bf16_t* O, int64_t ldo, char* ws, hipStream_t st) {
    const int s = (int)pl.s, l = (int)pl.l;
    axo::OrthoLoadArgs load = from;
    load.sums = reinterpret_cast<double*>(ws + pl.sums);
    load.rows = pl.tall ? l : s;
    load.cols = pl.tall ? s : l;
    load.scale = std::ldexp(1.0, pl.exponent);
    bf16_t* X[2] = {reinterpret_cast<bf16_t*>(ws + pl.X[0]), reinterpret_cast<bf16_t*>(ws + pl.X[1])};
    load.X = X[0];
    if (const int rc = type == AXO_TYPE_F32 ? launch_load<float>(load, st) : launch_load<bf16_t>(load, st)) return rc;
    bf16_t* const A = reinterpret_cast<bf16_t*>(ws + pl.A);
    bf16_t* const Q = reinterpret_cast<bf16_t*>(ws + pl.Q);
    for (int i = 0; i < steps; ++i) {
        const float* const c = abc ? abc + 3 * i : QUINTIC;
        const bf16_t* const x = X[i % 2];
        axo::OrthoStep whole{};
        if (pl.at_once || pl.rest) {
            axo::OrthoStep& y = whole;
            y.A = y.B = x;
            y.lda = y.ldb = load.cols;
            y.C = X[(i + 1) % 2]; y.ldc = load.cols;
            y.Mo = y.No = s; y.R = l;
            y.alpha = pl.at_once ? (float)std::ldexp(1.0, -2 * pl.exponent) : 1.0f;  // of A, which gram has left with it
            y.a = c[0]; y.b = c[1]; y.c = c[2];
            y.scale = (float)std::ldexp(1.0, -pl.exponent);
            y.K = from.K; y.N = from.N;
            y.tall = pl.tall;
            if (i == steps - 1) {
                y.O = O;
                y.ldo = ldo;
            }
        }
        if (pl.at_once) {
            const axo::OrthoStep& y = whole;
            if (const int rc = s == 64 ? (pl.tall ? launch_step<64, axo::MC>(y, st) : launch_step<64, axo::KC>(y, st))
                                       : (pl.tall ? launch_step<128, axo::MC>(y, st) : launch_step<128, axo::KC>(y, st)))
                return rc;
            continue;
        }
        axo::OrthoSym y{};
        y.A = y.B = x;
        y.lda = y.ldb = load.cols;
        y.C = A; y.ldc = s;
        y.Mo = y.No = s; y.R = l;
        y.alpha = (float)std::ldexp(1.0, -2 * pl.exponent);
        y.partial = reinterpret_cast<float*>(ws + pl.partial);
        y.counters = reinterpret_cast<uint32_t*>(ws + pl.counters);
        if (const int rc = launch_sym(y, pl.gram, pl.tall, st)) return rc;
        if (pl.rest) {
            if (const int rc = s == 64 ? launch_rest<64>(whole, A, st) : launch_rest<128>(whole, A, st)) return rc;
            continue;
        }
        y.A = y.B = A;
        y.lda = y.ldb = s;
        y.C = Q;
        y.R = s;
        y.aux = A; y.ldaux = s;
        y.alpha = c[2]; y.beta = c[1]; y.diag = c[0];
        if (const int rc = launch_sym(y, pl.poly, false, st)) return rc;
        axo::OrthoApply a{};
        a.A = pl.tall ? x : Q;  a.lda = pl.tall ? load.cols : s;
        a.B = pl.tall ? Q : x;  a.ldb = pl.tall ? s : load.cols;
        a.C = X[(i + 1) % 2]; a.ldc = load.cols;
        a.Mo = load.rows; a.No = load.cols; a.R = s;
        a.scale = (float)std::ldexp(1.0, -pl.exponent);
        a.K = from.K; a.N = from.N;
        if (i == steps - 1) {
            a.O = O;
            a.ldo = ldo;
        }
        if (const int rc = pl.tall ? launch_apply<axo::KC>(a, st) : launch_apply<axo::MC>(a, st)) return rc;
    }
    return AXO_OK;
}

// Gradients whose weight is not split.
int check_problem(const axo_problem_t* p, Shard* s) {
    if (const int rc = derive_shard(p, s)) return rc;
    return p->Gx != 1 || p->Gy != 1 ? AXO_ERR_BAD_GRID : AXO_OK;
}

}  // namespace axo_update

extern "C" {

int axo_ortho(const axo_problem_t* p, const void* G, int64_t ldg, int type, int steps, const float* abc, float eps, void* O, int64_t ldo, void* ws, size_t ws_bytes,
              void* hip_stream) {
    using namespace axo_update;
    return guarded([&]() -> int {
        Shard s;
        if (const int rc = check_problem(p, &s)) return rc;
        if (type != AXO_TYPE_BF16 && type != AXO_TYPE_F32) return AXO_ERR_BAD_ARG;
        if (steps < 1 || steps > AXO_ORTHO_MOST_STEPS || !(eps >= 0.0f) || !std::isfinite(eps)) return AXO_ERR_BAD_ARG;
        for (int i = 0; abc && i < 3 * steps; ++i)
            if (!std::isfinite(abc[i])) return AXO_ERR_BAD_ARG;
        if (const int rc = check_matrix(G, ldg, s.Kl, s.Nl)) return rc;
        if (const int rc = check_matrix(O, ldo, s.Kl, s.Nl)) return rc;
        if (s.Kl == 0 || s.Nl == 0) return AXO_OK;
        OrthoPlan plan;
        if (const int rc = make_plan(s, &plan)) return rc;
        if (!ws || ws_bytes < plan.bytes) return AXO_ERR_WORKSPACE;
        if (!aligned16(ws)) return AXO_ERR_MISALIGNED;
        Range g, o, w;
        matrix_range(G, ldg, s.Kl, s.Nl, type == AXO_TYPE_F32 ? 4 : 2, &g);
        matrix_range(O, ldo, s.Kl, s.Nl, 2, &o);
        matrix_range(ws, (int64_t)plan.bytes, 1, (int64_t)plan.bytes, 1, &w);
        if (o.shares_bytes_with(g) || o.shares_bytes_with(w) || w.shares_bytes_with(g)) return AXO_ERR_BAD_ARG;
        axo::OrthoLoadArgs from{};
        from.G = G; from.ldg = ldg;
        from.K = (int)s.Kl; from.N = (int)s.Nl;
        from.eps = eps;
        return ortho(plan, from, type, steps, abc, static_cast<bf16_t*>(O), ldo, static_cast<char*>(ws), static_cast<hipStream_t>(hip_stream));
    });
}

size_t axo_ortho_workspace_bytes(const axo_problem_t* p) {
    axo_host::Shard s;
    axo_update::OrthoPlan plan;
    if (axo_update::check_problem(p, &s) || s.Kl == 0 || s.Nl == 0 || axo_update::make_plan(s, &plan)) return 0;
    return plan.bytes;
}

}  // extern "C"
