// Entry points of include/axo_block.h: validation, choice of kernels, launches.  Part of axo_api.hip's translation unit.
#pragma once
#include "../../include/axo_block.h"

#include <cmath>
#include <initializer_list>

#include "axo_host.hpp"
#include "gated.hpp"
#include "gated_slim.hpp"
#include "last_used.hpp"
#include "norm.hpp"

static_assert((int)AXO_GATED_OP_FWD == axo::GATED_FWD && (int)AXO_GATED_OP_DGRAD_ACT == axo::GATED_DACT && (int)AXO_GATED_OP_DGRAD == axo::GATED_DX && (int)AXO_GATED_OP_WGRAD == axo::GATED_DW, "one numbering");
static_assert((int)AXO_GATE_SILU == axo::GATE_SILU && (int)AXO_GATE_GELU_TANH == axo::GATE_GELU_TANH && (int)AXO_GATE_GELU_ERF == axo::GATE_GELU_ERF, "one numbering");

namespace axo_block {

using namespace axo_host;
using axo::bf16_t;
using axo::GatedArgs;

inline int launched() { return hipGetLastError() == hipSuccess ? AXO_OK : AXO_ERR_HIP; }
// Workgroups of a grid whose workgroups walk over rows or chunks until none are left.
inline unsigned at_most(int64_t blocks, int64_t most) { return (unsigned)std::max<int64_t>(1, std::min(blocks, most)); }

// A call's matrices: what it reads and what it writes.  An output that shares a byte with an input or another output is refused.
struct Buffers {
    Range in[10], out[8];  // of resnorm_bwd, which has most: 9 and 8
    int n_in = 0, n_out = 0;
    void reads(const void* p, int64_t ld, int64_t rows, int64_t cols, int elem) {
        if (matrix_range(p, ld, rows, cols, elem, &in[n_in])) ++n_in;
    }
    void writes(const void* p, int64_t ld, int64_t rows, int64_t cols, int elem) {
        if (matrix_range(p, ld, rows, cols, elem, &out[n_out])) ++n_out;
    }
    int check() const {
        for (int o = 0; o < n_out; ++o) {
            for (int i = 0; i < n_in; ++i)
                if (out[o].shares_bytes_with(in[i])) return AXO_ERR_BAD_ARG;
            for (int q = 0; q < o; ++q)
                if (out[o].shares_bytes_with(out[q])) return AXO_ERR_BAD_ARG;
        }
        return AXO_OK;
    }
};

// A vector argument: n elements, aligned to `align` bytes; NULL where it is optional.
inline int check_vector(const void* p, int64_t n, uintptr_t align, bool optional) {
    if (n == 0) return AXO_OK;
    if (!p) return optional ? AXO_OK : AXO_ERR_NULL_PTR;
    return reinterpret_cast<uintptr_t>(p) % align ? AXO_ERR_MISALIGNED : AXO_OK;
}
inline int first_error(std::initializer_list<int> statuses) {
    for (int rc : statuses)
        if (rc) return rc;
    return AXO_OK;
}

// ---- layer norm ----------------------------------------------------------------------------------

int k_axis(const axo_problem_t* p) { return p->transposed ? p->Gy : p->Gx; }
int elem_of(int type) { return type == AXO_TYPE_F32 ? 4 : 2; }
bool known_type(int type) { return type == AXO_TYPE_BF16 || type == AXO_TYPE_F32; }
bool valid_eps(float eps) { return eps >= 0.0f && std::isfinite(eps); }

// A workgroup to a row or a piece of columns; more of them than this are walked (a grid has fewer than 2^32 threads).
constexpr int64_t NORM_MOST_BLOCKS = 1 << 20;

template <typename T, int LANES, int CH>
int launch_norm_rows(const axo::NormArgs& g, hipStream_t st) {
    constexpr int BLOCK = LANES <= 64 ? 256 : LANES, ROWS = BLOCK / LANES;
    hipLaunchKernelGGL((axo::norm_rows_kernel<T, LANES, CH>), dim3(at_most(tiles_in(g.M, ROWS), NORM_MOST_BLOCKS)), dim3(BLOCK), 0, st, g);
    return launched();
}
// A row is shared by as many lanes as leave each of them 16 to 64 bytes of it; of what holds a row the quickest was taken, bf16 and fp32 with a residual, 2^25 values (us):
//   to 64      8 x 1 chunks 50, 82       64 x 1  205, 265     to 4096   256 x 2  49, 84     512 x 1  49, 85
//   to 256    32 x 1  48, 83             64 x 1   66,  90     to 8192   512 x 2  51, 88     256 x 4  53, 87 (64 rows: 4.4 and 5.2)
//   to 512    64 x 1  48, 83             64 x 2   56,  87     to 12288  512 x 3  53, 88    1024 x 2  66, 102
//   to 1024   64 x 2  50, 83            256 x 1   65,  90     to 16384  512 x 4  57, 99    1024 x 2  62, 95
//   to 2048  256 x 1  48, 83             64 x 4   53,  87     20000    1024 x 3  66, 103   read again from the caches 92, 124
//   32768   1024 x 4  61, 133           read again 79, 126: rows of 64 KB of fp32 and more are
template <typename T>
int launch_norm_typed(const axo::NormArgs& g, hipStream_t st) {
    if (g.K <= 64) return launch_norm_rows<T, 8, 1>(g, st);
    if (g.K <= 128) return launch_norm_rows<T, 16, 1>(g, st);
    if (g.K <= 256) return launch_norm_rows<T, 32, 1>(g, st);
    if (g.K <= 512) return launch_norm_rows<T, 64, 1>(g, st);
    if (g.K <= 1024) return launch_norm_rows<T, 64, 2>(g, st);
    if (g.K <= 2048) return launch_norm_rows<T, 256, 1>(g, st);
    if (g.K <= 4096) return launch_norm_rows<T, 256, 2>(g, st);
    if (g.K <= 8192) return launch_norm_rows<T, 512, 2>(g, st);
    if (g.K <= 12288) return launch_norm_rows<T, 512, 3>(g, st);
    if (g.K <= 16384) return launch_norm_rows<T, 512, 4>(g, st);
    if (g.K <= 24576) return launch_norm_rows<T, 1024, 3>(g, st);
    if constexpr (sizeof(T) == 2)
        if (g.K <= 32768) return launch_norm_rows<T, 1024, 4>(g, st);
    hipLaunchKernelGGL(axo::norm_long_kernel<T>, dim3(at_most(g.M, NORM_MOST_BLOCKS)), dim3(axo::NORM_THREADS), 0, st, g);
    return launched();
}
int launch_norm(const axo::NormArgs& g, int type, hipStream_t st) {
    if (g.M == 0 || g.K == 0) return AXO_OK;
    return type == AXO_TYPE_F32 ? launch_norm_typed<float>(g, st) : launch_norm_typed<bf16_t>(g, st);
}

// The column sums of the backward pass come from so many workgroups at most, each of which leaves two rows of them in the workspace.
constexpr int NORM_MOST_SLICES = 256;
constexpr int NORM_MOST_COLS = 16384;  // of rows in registers
int norm_slice_rows(int64_t M) { return (int)std::max<int64_t>(axo::NORM_COL_ROWS, (M + 255) / 256); }  // of longer ones
int64_t norm_partial_cols(int64_t K) { return (K + 7) / 8 * 8; }
size_t norm_workspace(int64_t M, int64_t K) {
    return (size_t)std::max<int64_t>(1, std::min<int64_t>(M, NORM_MOST_SLICES)) * 2 * (size_t)norm_partial_cols(K) * sizeof(float);
}

int launch_norm_join(const axo::NormBwdArgs& g, hipStream_t st) {
    if (g.phase == axo::NORM_APPLY || (!g.dgamma && !g.dbeta)) return AXO_OK;
    hipLaunchKernelGGL(axo::norm_join_kernel, dim3(at_most((2 * g.partial_cols + axo::NORM_JOIN_COLS - 1) / axo::NORM_JOIN_COLS, NORM_MOST_BLOCKS)),
                       dim3(axo::NORM_JOIN_THREADS), 0, st, g);
    return launched();
}
template <typename T, int LANES, int CH, int GROUPS>
int launch_norm_bwd_groups(axo::NormBwdArgs& g, hipStream_t st) {
    g.slices = (int)std::min<int64_t>(tiles_in(g.M, GROUPS), NORM_MOST_SLICES);
    hipLaunchKernelGGL((axo::norm_bwd_rows_kernel<T, LANES, CH, GROUPS>), dim3((unsigned)g.slices), dim3(LANES * GROUPS), 0, st, g);
    if (const int rc = launched()) return rc;
    return launch_norm_join(g, st);
}
// A workgroup has 512 threads, and of bf16 rows 1024 where there are more rows than workgroups of 512 take at once: the same bytes under way.  2^25 values, 512 and 1024
// threads (us): 64 columns bf16 67, 57, fp32 87, 90; 512 columns 65, 54 and 86, 89; 2048 columns 64, 53 and 86, 90.  (1000 x 64 bf16: 6.9, 8.0.)  Those sizes are bound by
// bandwidth; fp32 rows that take two turns of 512 threads and one of 1024, some thousand of 1027, were not compared.
template <typename T, int LANES, int CH>
int launch_norm_bwd_rows(axo::NormBwdArgs& g, hipStream_t st) {
    constexpr int GROUPS = 512 / LANES;
    if constexpr (sizeof(T) == 2 && CH == 1)
        if (g.M > GROUPS * NORM_MOST_SLICES) return launch_norm_bwd_groups<T, LANES, CH, 2 * GROUPS>(g, st);
    return launch_norm_bwd_groups<T, LANES, CH, GROUPS>(g, st);
}
// Rows of up to 4096 values have a chunk to a lane; of longer ones a lane holds up to four (16384 columns, bf16 and fp32: 512 x 4 65 and 106 us, 1024 x 2 66 and 121, read
// twice 108 and 149).
template <typename T>
int launch_norm_bwd_typed(axo::NormBwdArgs& g, hipStream_t st) {
    if (g.M > 0 && g.K <= NORM_MOST_COLS) {
        if (g.K <= 64) return launch_norm_bwd_rows<T, 8, 1>(g, st);
        if (g.K <= 128) return launch_norm_bwd_rows<T, 16, 1>(g, st);
        if (g.K <= 256) return launch_norm_bwd_rows<T, 32, 1>(g, st);
        if (g.K <= 512) return launch_norm_bwd_rows<T, 64, 1>(g, st);
        if (g.K <= 1024) return launch_norm_bwd_rows<T, 128, 1>(g, st);
        if (g.K <= 2048) return launch_norm_bwd_rows<T, 256, 1>(g, st);
        if (g.K <= 4096) return launch_norm_bwd_rows<T, 512, 1>(g, st);
        if (g.K <= 8192) return launch_norm_bwd_rows<T, 512, 2>(g, st);
        if (g.K <= 12288) return launch_norm_bwd_rows<T, 512, 3>(g, st);
        return launch_norm_bwd_rows<T, 512, 4>(g, st);
    }
    if (g.M > 0) {
        hipLaunchKernelGGL(axo::norm_bwd_long_kernel<T>, dim3(at_most(g.M, NORM_MOST_BLOCKS)), dim3(axo::NORM_THREADS), 0, st, g);
        if (const int rc = launched()) return rc;
    }
    if (g.phase == axo::NORM_APPLY || (!g.dgamma && !g.dbeta)) return AXO_OK;
    g.rows_per_slice = norm_slice_rows(g.M);
    g.slices = (int)std::max<int64_t>(1, tiles_in(g.M, g.rows_per_slice));
    hipLaunchKernelGGL(axo::norm_cols_kernel<T>, dim3(at_most(tiles_in(g.K, axo::NORM_STRIP) * g.slices, NORM_MOST_BLOCKS)), dim3(axo::NORM_COL_THREADS), 0, st, g);
    if (const int rc = launched()) return rc;
    return launch_norm_join(g, st);
}
int launch_norm_bwd(axo::NormBwdArgs g, int type, hipStream_t st) {
    if (g.K == 0) return AXO_OK;
    return type == AXO_TYPE_F32 ? launch_norm_bwd_typed<float>(g, st) : launch_norm_bwd_typed<bf16_t>(g, st);
}

int plan_norm(const axo_problem_t* p, const void* X, int64_t ldx, const void* R, int64_t ldr, int type, void* S, int64_t lds, Buffers& b,
              axo::NormArgs& g) {
    Shard s;
    if (const int rc = derive_shard(p, &s)) return rc;
    if (!known_type(type)) return AXO_ERR_BAD_ARG;
    if (const int rc = check_matrix(X, ldx, s.M, s.Kl)) return rc;
    if (R)
        if (const int rc = first_error({check_matrix(R, ldr, s.M, s.Kl), check_matrix(S, lds, s.M, s.Kl)})) return rc;
    g.X = X; g.ldx = ldx;
    g.R = R; g.ldr = ldr;
    g.S = S; g.lds = lds;
    g.M = (int)s.M; g.K = (int)s.Kl;
    b.reads(X, ldx, s.M, s.Kl, elem_of(type));
    if (R) {
        b.reads(R, ldr, s.M, s.Kl, elem_of(type));
        b.writes(S, lds, s.M, s.Kl, elem_of(type));
    }
    return AXO_OK;
}
int plan_norm_output(const void* gamma, const void* beta, float eps, void* Y, int64_t ldy, float* stats, Buffers& b, axo::NormArgs& g) {
    if (!valid_eps(eps)) return AXO_ERR_BAD_ARG;
    const int64_t n = g.M > 0 ? g.K : 0;
    if (const int rc = first_error({check_matrix(Y, ldy, g.M, g.K), check_vector(gamma, n, 16, true), check_vector(beta, n, 16, true),
                                    check_vector(stats, g.K > 0 ? g.M : 0, 8, true)}))
        return rc;
    g.gamma = static_cast<const bf16_t*>(gamma);
    g.beta = static_cast<const bf16_t*>(beta);
    g.eps = eps;
    g.Y = static_cast<bf16_t*>(Y); g.ldy = ldy;
    g.stats = reinterpret_cast<float2*>(stats);
    b.reads(gamma, g.K, 1, g.K, 2);
    b.reads(beta, g.K, 1, g.K, 2);
    b.writes(Y, ldy, g.M, g.K, 2);
    b.writes(stats, 2 * (int64_t)g.M, 1, 2 * (int64_t)g.M, 4);
    return AXO_OK;
}

int plan_norm_bwd(const axo_problem_t* p, const void* dY, int64_t lddy, const void* S, int64_t lds, int type, const void* gamma,
                  const float* stats, Buffers& b, axo::NormBwdArgs& g) {
    Shard s;
    if (const int rc = derive_shard(p, &s)) return rc;
    if (!known_type(type)) return AXO_ERR_BAD_ARG;
    const bool some = s.M > 0 && s.Kl > 0;
    if (const int rc = first_error({check_matrix(dY, lddy, s.M, s.Kl), check_matrix(S, lds, s.M, s.Kl), check_vector(gamma, some ? s.Kl : 0, 16, true),
                                    check_vector(stats, some ? s.M : 0, 8, false)}))
        return rc;
    g.dY = static_cast<const bf16_t*>(dY); g.lddy = lddy;
    g.S = S; g.lds = lds;
    g.gamma = static_cast<const bf16_t*>(gamma);
    g.stats = reinterpret_cast<const float2*>(stats);
    g.M = (int)s.M; g.K = (int)s.Kl;
    g.per_row = p->K > 0 ? 1.0f / (float)p->K : 0.0f;
    b.reads(dY, lddy, s.M, s.Kl, 2);
    b.reads(S, lds, s.M, s.Kl, elem_of(type));
    b.reads(gamma, s.Kl, 1, s.Kl, 2);
    b.reads(stats, 2 * s.M, 1, 2 * s.M, 4);
    return AXO_OK;
}
int plan_norm_dx(const void* R, int64_t ldr, int type, void* dX, int64_t lddx, Buffers& b, axo::NormBwdArgs& g) {
    if (R)
        if (const int rc = check_matrix(R, ldr, g.M, g.K)) return rc;
    if (const int rc = check_matrix(dX, lddx, g.M, g.K)) return rc;
    g.R = R; g.ldr = ldr;
    g.dX = dX; g.lddx = lddx;
    if (R) b.reads(R, ldr, g.M, g.K, elem_of(type));
    b.writes(dX, lddx, g.M, g.K, elem_of(type));
    return AXO_OK;
}
int plan_norm_columns(float* dgamma, float* dbeta, int accumulate, void* ws, size_t ws_bytes, Buffers& b, axo::NormBwdArgs& g) {
    if (accumulate != 0 && accumulate != 1) return AXO_ERR_BAD_ARG;
    if (const int rc = first_error({check_vector(dgamma, g.K, 4, true), check_vector(dbeta, g.K, 4, true)})) return rc;
    g.dgamma = dgamma;
    g.dbeta = dbeta;
    g.accumulate = accumulate;
    b.writes(dgamma, g.K, 1, g.K, 4);
    b.writes(dbeta, g.K, 1, g.K, 4);
    if ((!dgamma && !dbeta) || g.K == 0) return AXO_OK;
    const size_t need = norm_workspace(g.M, g.K);
    if (need == 0) return AXO_OK;
    if (!ws || ws_bytes < need) return AXO_ERR_WORKSPACE;
    if (!aligned16(ws)) return AXO_ERR_MISALIGNED;
    g.partial = static_cast<float*>(ws);
    g.partial_cols = norm_partial_cols(g.K);
    b.writes(ws, (int64_t)(need / 4), 1, (int64_t)(need / 4), 4);
    return AXO_OK;
}

// ---- gated block -----------------------------------------------------------------------------------

bool known_gate(int gate) { return gate >= AXO_GATE_SILU && gate <= AXO_GATE_GELU_ERF; }

template <int OP>
int launch_gated_generic(const GatedArgs& g, hipStream_t st) {
    const dim3 grid((unsigned)tiles_in(g.No, axo::GEN_BN), (unsigned)tiles_in(g.Mo, axo::GEN_BM));
    if (grid.y > 65535u) return AXO_ERR_BAD_SIZE;
    hipLaunchKernelGGL(axo::gated_generic_kernel<OP>, grid, dim3(256), 0, st, g);
    return launched();
}
// Byte offsets inside an operand of a tile are formed in 32 bits (spans_ok of the products): 256 rows of a KC operand, the walked reduction of an MC one.
template <int OP>
bool gated_spans_ok(const GatedArgs& g) {
    auto fits = [](int64_t elems) { return elems * 2 < (int64_t)0xFFFF0000; };
    const int64_t walked = ((int64_t)g.R + 2 * axo::TILE_BK - 1) / (2 * axo::TILE_BK) * (2 * axo::TILE_BK);
    return fits(256 * g.lda + walked) && fits(axo::GATED_LB<OP> == axo::MC ? walked * g.ldb + 256 : 256 * g.ldb + walked);
}

// Rows of the outputs that straddle cache lines are stored plainly (store_row), but past the caches where the forward pass writes more than they keep for
// a line's other half: whole lines 4096 x 2048 x 4096 through the activation's derivative 73 us plainly and 64 past the caches; straddled 4096 x 2048 x 12296 247 and 271; forward,
// G and U kept, straddled 2048 x 2048 x 6008 87 and 95, 4096 x 2048 x 8200 271 and 241.
template <int OP>
bool gated_plain(const GatedArgs& g) {
    const bool straddles = ((reinterpret_cast<uintptr_t>(g.C) | (uintptr_t)(g.ldc * (OP == axo::FC_ADD && g.wide ? 4 : 2))) & 127) != 0;
    return straddles && (OP != axo::GATED_FWD || (int64_t)g.Mo * g.No * (g.G ? 6 : 2) <= (int64_t)128 << 20);
}

template <typename C, int OP, typename Kernel>
int launch_gated_tiles(Kernel kern, std::atomic<uint64_t>* raised, const GatedArgs& g, int rows, int cols, hipStream_t st) {
    if (!raise_lds_limit(reinterpret_cast<const void*>(kern), C::LDS_BYTES, raised)) return AXO_ERR_HIP;
    axo::GatedProduct<OP> args{g};
    const int tm = (int)tiles_in(g.Mo, rows), tn = (int)tiles_in(g.No, axo::gated_cols<OP>(cols));
    hipLaunchKernelGGL(kern, dim3((unsigned)tm * (unsigned)tn), dim3(C::THREADS), C::LDS_BYTES, st, args, tm, tn, std::min(tm, 8));
    return launched();
}
template <int OP, bool PLAIN, int LINES>
int launch_gated_on(const GatedArgs& g, Tiles tiles, const axo::TileSched& sc, hipStream_t st) {
    static std::atomic<uint64_t> raised[4]{{0}, {0}, {0}, {0}};
    constexpr bool ALL = LINES == 2;
    if constexpr (LINES != 1) {
        if (tiles == Tiles::small) return launch_gated_tiles<axo::SmallCfg<ALL>, OP>(axo::gated_small_kernel<OP, PLAIN, ALL>, &raised[0], g, 64, 64, st);
        if (tiles == Tiles::wide) return launch_gated_tiles<axo::RectCfg<true>, OP>(axo::gated_rect_kernel<OP, PLAIN, ALL>, &raised[1], g, 64, 128, st);
        if (tiles == Tiles::mid) return launch_gated_tiles<axo::MidCfg, OP>(axo::gated_mid_kernel<OP, PLAIN, ALL>, &raised[2], g, 128, 128, st);
    }
    // Forward ring tiles fetch one operand by lines at most and half-width ones none (takes_lines), so there is no forward of kind 2 on 256-row tiles.
    constexpr int MIXED = axo::GATED_LB<OP> == axo::MC && LINES == 2 ? 1 : LINES;
    constexpr int lds = LINES != 0 ? axo::LINES_LDS_BYTES : axo::MIX_LDS_BYTES;
    auto kern = axo::gated_mixed_kernel<OP, PLAIN, MIXED>;
    if (!raise_lds_limit(reinterpret_cast<const void*>(kern), lds, &raised[3])) return AXO_ERR_HIP;
    hipLaunchKernelGGL(kern, dim3(sc.n_big + sc.tiles_m * sc.small_cols), dim3(axo::TILE_THREADS), lds, st, axo::GatedProduct<OP>{g}, sc);
    return launched();
}
// On the tiles of a plan.  Where rows of the inputs are fetched by whole lines those of the outputs mostly straddle lines as well, so there is one kind of
// such kernels, with plain stores, and forward one more.  dX, whose two products may lie differently in their lines, does not do that, and its epilogue looks at the output itself.
template <int OP>
int launch_gated_tiles_of(const GatedArgs& g, Tiles tiles, int cols, int red, hipStream_t st) {
    const axo::TileSched sc = tiles == Tiles::big ? plan_columns(g.Mo, cols, red) : axo::TileSched{};
    if constexpr (OP == axo::GATED_DX) return launch_gated_on<OP, false, 0>(g, tiles, sc, st);
    else {
        axo::GemmArgs as_one = g;
        as_one.No = cols;
        switch (takes_lines_on(as_one, axo::KC, axo::GATED_LB<OP>, tiles, sc)) {
            case 2: return launch_gated_on<OP, true, 2>(g, tiles, sc, st);
            case 1:
                if constexpr (axo::GATED_LB<OP> == axo::MC)
                    if (!gated_plain<OP>(g)) return launch_gated_on<OP, false, 1>(g, tiles, sc, st);
                return launch_gated_on<OP, true, 1>(g, tiles, sc, st);
            default: break;
        }
        return gated_plain<OP>(g) ? launch_gated_on<OP, true, 0>(g, tiles, sc, st) : launch_gated_on<OP, false, 0>(g, tiles, sc, st);
    }
}

// ---- split reductions (gated_slim.hpp) ----
// The workspace: arrival counters of at most so many tiles, and behind them the sums of the slices.
constexpr size_t GATED_COUNTER_BYTES = 8192;
constexpr int64_t GATED_MOST_TILES = GATED_COUNTER_BYTES / sizeof(uint32_t);

// A kind of split-reduction tile, and what a product on it takes in us: `fixed`, and the longest of
//   - a CU's share of the workgroups, each of which costs `each` and takes in its operands at `rate` KB per us, or `alone` where it has the CU to itself;
//   - one wave's chain of chunks, `latency` each, as many under way as it has stages;
//   - the weights, read at `tbs` TB/s;
// and `join` where its reduction is sliced.  Fitted to 14 000 shapes (1 to 800 tokens, widths of 32 to 16384, weights from memory) and for the kind that is left to
// few rows and much weight to 1400 of those; half of the estimates are within 5 to 11 %, nine of ten within 28 %.  Those of the product with a residual to 20 000 (1 to 400 tokens,
// widths of 64 to 16384), each counted by its time: 6 to 8 % and 18 to 21 %.
struct GatedSlim {
    int rows, cols, waves, stages;  // `cols`: of the output
    double fixed, rate, alone, latency, tbs, join, each;
};
constexpr GatedSlim GATED_SLIM[5][4] = {
    {{16, 32, 4, 3, 3.26, 39.4, 67.2, 2.37, 3.78, 2.31, 1.21}, {32, 32, 4, 3, 2.85, 42.6, 64.6, 2.99, 3.14, 3.92, 1.53},
     {16, 64, 2, 4, 3.10, 51.8, 97.2, 2.65, 4.87, 3.79, 2.04}, {16, 128, 2, 2, 4.73, 49.3, 50.0, 3.14, 6.18, 4.74, 0.30}},
    {{16, 32, 4, 3, 4.32, 87.9, 126.6, 0.88, 6.72, 1.20, 0.66}, {32, 32, 4, 3, 3.01, 73.9, 155.4, 1.44, 5.48, 2.59, 1.84}, {}, {}},
    {{16, 32, 4, 3, 4.16, 71.8, 78.6, 1.04, 5.69, 0.71, 0.28}, {32, 32, 4, 3, 3.16, 87.1, 115.1, 1.50, 4.63, 2.34, 1.24}, {}, {}},
    {},
    {{16, 32, 4, 3, 3.20, 46.1, 67.4, 1.47, 4.14, 1.89, 0.62}, {32, 32, 4, 3, 2.03, 50.2, 82.1, 2.28, 3.84, 2.47, 1.96},
     {16, 64, 4, 3, 2.27, 48.8, 87.5, 2.37, 4.95, 2.63, 1.75}, {16, 128, 4, 2, 4.36, 80.0, 89.9, 0.79, 5.91, 2.92, 0.00}}};
// Rows of 256 bytes of either weight (the fourth kind) are for tokens of one tile that read more than the caches hold: there they are the quickest, 1.2 times quicker than 64 x 128
// tiles (1 x 8192 x 16384 97 us, with rows of 128 bytes 109, on those tiles 104; where rows lie a multiple of 4 KiB apart, a column of 128 bytes
// lies in half of each of its DRAM pages).  With less to read they are not.  The product with a residual has one weight and four waves to these tiles: of 1500 shapes up to 16 tokens they
// are the quickest kind from 100 MB on (120 to 140 MB: 1.02 times the best of all, rows of 128 bytes 1.07, 64 x 64 tiles 1.27; 60 to 80 MB 1.10 and 1.02).
constexpr double GATED_WIDE_MB[5] = {200.0, 200.0, 200.0, 200.0, 100.0};
// The same for the tiles of gemm_tile.hpp: what their estimates have to be multiplied with for these products (small, wide, tall, mid, big; medians of the same
// shapes), which read weights from memory and have longer epilogues.  Whatever is estimated quicker is taken: over those shapes the choice is 1.29 (forward), 1.63 and 1.99 times
// quicker than these tiles throughout, 3 to 5 % slower than the best of all, and by more than 5 % slower than these tiles for two or three shapes in a hundred.
// (The last row, of the product with a residual, is no such median: round numbers near the others', which were kept for the choice that they lead to.  Over 1200 drawn products of 1 to 400 tokens
// and widths of 64 to 16384 that is 8 % slower than the best of all, in the geometric mean.)
constexpr double GATED_TILES[5][5] = {{1.06, 1.66, 1.66, 1.21, 1.03}, {0.93, 1.37, 1.37, 1.41, 1.55}, {0.88, 1.47, 1.47, 1.21, 1.08}, {}, {1.0, 1.4, 1.4, 1.2, 1.05}};

// How a product is cut into split-reduction tiles.
struct GatedCut {
    int kind = -1;  // of GATED_SLIM[OP], or -1: not at all
    int64_t tiles_m = 0, tiles_n = 0;
    int slices = 1, chunks = 0;
    size_t bytes = 0;  // of workspace
};
constexpr int GATED_SPLIT = 4;  // the kind of 128 x 128 tiles in slices
// Slices of a reduction: as many as leave every workgroup a CU to itself and sixteen chunks, within 1 to 4 % of the best number over those shapes (two workgroups per CU: 3 to 9 %
// off, eight chunks 3 to 7 %).
int64_t gated_slices(int64_t tiles, int64_t chunks) { return std::max<int64_t>(1, std::min<int64_t>({NUM_CU / tiles, chunks / 16, 16})); }

// Weight matrices of a product.
template <int OP>
constexpr int gated_matrices() { return OP == axo::GATED_DACT || OP == axo::FC_ADD ? 1 : 2; }
// The quickest cut of a product (Mo x No, reductions of R) and the estimate of it.
template <int OP>
GatedCut gated_cut(int Mo, int No, int R, double* us) {
    const int64_t chunks = steps_in(R) * (OP == axo::GATED_DX ? 2 : 1);
    const double weights = 2e-6 * No * (double)R * gated_matrices<OP>();  // MB
    GatedCut best;
    *us = 1e30;
    for (int k = 0; k < 4; ++k) {
        const GatedSlim& m = GATED_SLIM[OP][k];
        if (m.rows == 0 || (m.rows == 16 && Mo > 256) || (k == 3 && (Mo > 16 || weights < GATED_WIDE_MB[OP]))) continue;
        const int64_t tm = tiles_in(Mo, m.rows), tn = tiles_in(No, m.cols), tiles = tm * tn;
        if (tiles > 4000) continue;
        const int cols = m.cols * (OP == axo::GATED_FWD ? 2 : 1);
        const double stage = (m.rows + cols) * 128 / 1024.0;
        const int64_t lds = std::max<int64_t>(m.stages * (m.rows + cols) * 128, m.rows * (cols + 4) * 4) * m.waves;
        const int64_t beside = std::min<int64_t>(8, 160 * 1024 / lds);  // workgroups on a CU
        const int64_t asked = gated_slices(tiles, chunks), per = (chunks + asked - 1) / asked, slices = (chunks + per - 1) / per;
        const int64_t rounds = rounds_of(tiles * slices);
        const double share = rounds * (per * stage / (rounds > 1 ? m.rate : m.alone) + m.each);
        const double chain = (double)((per + m.waves - 1) / m.waves) * m.latency / m.stages * ((rounds + beside - 1) / beside);
        const double t = m.fixed + std::max({share, chain, weights / m.tbs}) + (slices > 1 ? m.join : 0.0);
        if (t >= *us) continue;
        *us = t;
        best.kind = k;
        best.tiles_m = tm;
        best.tiles_n = tn;
        best.slices = (int)slices;
        best.chunks = (int)per;
        best.bytes = slices > 1 ? GATED_COUNTER_BYTES + (size_t)(tiles * slices) * m.rows * cols * sizeof(float) : 0;
    }
    return best;
}
// 128 x 128 tiles in the slices that are estimated to be quickest, all on the CUs at once, and the time of that: two launches, a slice's steps or the operands' way
// from memory, and the sums' way through the workspace.  Taken where that is less than what gated_cut finds and than on whole tiles, to 64 steps by a
// fifth (without that margin beyond: 16 of 70 shapes 3 to 69 % quicker, none slower; with it gone below, 15 to 25 % slower at two slices).  Of 160 drawn
// products with a split, with and without it (us): forward 1760 x 15131 x 128 28 and 77, 128 x 11305 x 1778 25 and 54, through the derivative 512 x 10200 x 512 19 and 27, dX with the weight gradients
// 128 x 2200 x 9344 51 and 80, 5784 x 640 x 752 42 and 115, 4413 x 3952 x 184 62 and 105.
template <int OP>
GatedCut gated_split_cut(int Mo, int No, int R, double* us) {
    GatedCut cut;
    *us = 1e30;
    const int64_t steps = steps_in(R), tm = tiles_in(Mo, 128), tn = tiles_in(No, axo::gated_cols<OP>(128)) * (OP == axo::GATED_DW ? 2 : 1), tiles = tm * tn;
    for (int64_t asked = 2; asked <= 16 && asked * tiles <= NUM_CU; ++asked) {
        const int64_t per = (steps + asked - 1) / asked, slices = (steps + per - 1) / per;
        const double step = OP == axo::GATED_DX ? 0.9 : 0.45;
        const double operands = 2e-6 * R * (OP == axo::GATED_DX ? 2.0 * Mo + 2.0 * No : Mo + (double)gated_matrices<OP>() * No);  // MB
        const double t = 8.5 + std::max(per * step, operands / 5.5) + 0.02 * (double)(tiles * slices);
        if (per < 4 || t >= *us) continue;
        *us = t;
        cut.kind = GATED_SPLIT;
        cut.tiles_m = tm;
        cut.tiles_n = tn;
        cut.slices = (int)slices;
        cut.chunks = (int)per;
        cut.bytes = GATED_COUNTER_BYTES + (size_t)(tiles * slices) * axo::SPLIT_TILE * sizeof(float);
    }
    return cut;
}
static_assert(NUM_CU <= GATED_MOST_TILES, "a counter for every tile that is sliced");

// What a product of a gated block runs on, from its sizes alone.
struct GatedPlan {
    bool general = false;
    Tiles tiles = Tiles::big;
    GatedCut cut;
};
template <int OP>
GatedPlan gated_plan(int Mo, int No, int R) {
    GatedPlan plan;
    if (Mo == 0 || No == 0) return plan;
    // as one product: twice the columns, or twice the reduction
    const int64_t cols = OP == axo::GATED_FWD ? 2 * (int64_t)No : No, red = OP == axo::GATED_DX ? 2 * (int64_t)R : R;
    if (R == 0 || cols > INT32_MAX || red > INT32_MAX || !grid_fits(tiles_in(Mo, 256) * tiles_in((int)cols, 128), axo::TILE_THREADS)) {
        plan.general = true;
        return plan;
    }
    plan.tiles = quickest_tiles(Mo, (int)cols, (int)red);  // 64 x 64 ones where those fit a launch as well, the other small ones for a round of CUs alone
    const double weights = 2e-6 * No * (double)R * gated_matrices<OP>();
    const double tiles_us = std::max(tiles_time(plan.tiles, Mo, (int)cols, (int)red) * GATED_TILES[OP][(int)plan.tiles], 3.0 + weights / 5.0);
    const int64_t small_tiles = tiles_in(Mo, 64) * tiles_in((int)cols, 64);
    const bool round_of_wide = tiles_in(Mo, 64) * tiles_in((int)cols, 128) <= NUM_CU;
    if (plan.tiles == Tiles::tall) plan.tiles = round_of_wide ? Tiles::wide : Tiles::mid;
    // 64 x 64 tiles that leave some CUs two and others one: a 64 x 128 tile for each CU is quicker, from four steps of a reduction on forward and from ten through the
    // activation's derivative, where G and U of a tile wait for its end.  Of 55 such shapes where 64 x 64 tiles were taken, forward 5 to 56 % over four steps (350 x 5928 x 1453 55 us
    // and 37, 1001 x 1027 x 515 12.1 and 10.1) and 0 to -5 % at two; backward 2 to 14 % from ten steps on (700 x 4000 x 1500 26.0 and 22.9), -10 to 3 % below.
    // The product with a residual takes what goes for the forward pass, whose operands lie as its own do; it was not measured for this.
    if (OP != axo::GATED_DX && plan.tiles == Tiles::small && round_of_wide && small_tiles > NUM_CU && steps_in(R) >= (OP == axo::GATED_DACT ? 10 : 4)) plan.tiles = Tiles::wide;
    // Short reductions through the derivative are its reads of G and U and its stores, which go on beside each other where a CU has two tiles: 64 x 64 ones,
    // while there are few of them.  Of 126 shapes with reductions of 32 to 1024: for 128 x 128 tiles, to four steps and two a CU, 42 to 51 % quicker (2638 x 32 x 640 8.6 us and 6.0);
    // for 256 x 256 ones to nine a CU and four steps 0 to 50 % (876 x 192 x 8576 28.6 and 19.1), to six and sixteen steps -1 to 28 %; beyond, 11 % quicker to 27 % slower.
    if (OP == axo::GATED_DACT && ((plan.tiles == Tiles::mid && R <= 256 && small_tiles <= 2 * NUM_CU) ||
                                  (plan.tiles == Tiles::big && R <= 1024 && small_tiles <= (R <= 256 ? 9 : 6) * NUM_CU)))
        plan.tiles = Tiles::small;
    double us = 1e30, split_us;
    GatedCut cut;
    if (Mo <= 2048) cut = gated_cut<OP>(Mo, No, R, &us);  // never quicker beyond
    const GatedCut split = gated_split_cut<OP>(Mo, No, R, &split_us);
    if (split_us < std::min(us, (steps_in(R) < 64 ? 0.8 : 1.0) * tiles_us)) plan.cut = split;
    else if (us < tiles_us) plan.cut = cut;
    return plan;
}

// The same for the two weight gradients (K x N, M tokens), which are split or go the way of axo_fc_wgrad.
GatedPlan gated_wgrad_plan(int K, int N, int M) {
    GatedPlan plan;
    if (K == 0 || N == 0 || M == 0 || N > INT32_MAX / 2) return plan;
    double us;
    const GatedCut split = gated_split_cut<axo::GATED_DW>(K, N, M, &us);
    if (us < pair_time(K, N, M, axo::MC, axo::MC)) plan.cut = split;
    return plan;
}

// The plans of the calls that a problem is passed to, as the block's projections and as the layer behind it, and the largest workspace among them.  A
// plan takes up to a microsecond; a thread keeps those of the last sixteen sizes that it called with.
struct GatedPlans {
    GatedPlan of[5];
    size_t bytes = 0;  // of the first four; the product with a residual has a workspace of its own
};
const GatedPlans& gated_plans(const Shard& s) {
    static thread_local axo::LastUsed<GatedPlans, 16> kept;
    return kept.get(s.M, s.Kl, s.Nl, [&] {
        const int M = (int)s.M, K = (int)s.Kl, N = (int)s.Nl;
        GatedPlans p;
        p.of[axo::GATED_FWD] = gated_plan<axo::GATED_FWD>(M, N, K);
        p.of[axo::GATED_DACT] = gated_plan<axo::GATED_DACT>(M, K, N);
        p.of[axo::GATED_DX] = gated_plan<axo::GATED_DX>(M, K, N);
        p.of[axo::GATED_DW] = gated_wgrad_plan(K, N, M);
        for (const GatedPlan& plan : p.of) p.bytes = std::max(p.bytes, plan.cut.bytes);
        p.of[axo::FC_ADD] = gated_plan<axo::FC_ADD>(M, N, K);
        return p;
    });
}

template <int OP, int KIND>
int launch_gated_slim(const GatedArgs& g, const GatedCut& cut, void* ws, hipStream_t st) {
    constexpr GatedSlim M = GATED_SLIM[OP][KIND];
    if constexpr (M.rows == 0) return AXO_ERR_BAD_ARG;
    else {
        using C = axo::GatedSlimCfg<OP, M.rows, M.cols, M.waves, M.stages>;
        auto kern = axo::gated_slim_kernel<OP, M.rows, M.cols, M.waves, M.stages>;
        static std::atomic<uint64_t> raised{0};
        if (!raise_lds_limit(reinterpret_cast<const void*>(kern), C::LDS_BYTES, &raised)) return AXO_ERR_HIP;
        axo::GatedSlimSched sc{};
        sc.tiles_m = (int)cut.tiles_m;
        sc.tiles_n = (int)cut.tiles_n;
        sc.slices = cut.slices;
        sc.chunks = cut.chunks;
        sc.counters = static_cast<uint32_t*>(ws);
        sc.partial = reinterpret_cast<float*>(static_cast<char*>(ws) + GATED_COUNTER_BYTES);
        hipLaunchKernelGGL(kern, dim3((unsigned)(cut.tiles_m * cut.tiles_n * cut.slices)), dim3(C::THREADS), C::LDS_BYTES, st, axo::GatedProduct<OP>{g}, sc);
        return launched();
    }
}
template <int OP, bool LINES>
int launch_gated_split(const GatedArgs& g, const GatedCut& cut, void* ws, hipStream_t st) {
    auto kern = axo::gated_split_kernel<OP, LINES>;
    static std::atomic<uint64_t> raised{0};
    if (!raise_lds_limit(reinterpret_cast<const void*>(kern), axo::MidCfg::LDS_BYTES, &raised)) return AXO_ERR_HIP;
    const int tiles = (int)(cut.tiles_m * cut.tiles_n);
    const axo::GatedSplitSched sc{(int)cut.tiles_m, (int)cut.tiles_n, cut.slices, cut.chunks, reinterpret_cast<float*>(static_cast<char*>(ws) + GATED_COUNTER_BYTES)};
    hipLaunchKernelGGL(kern, dim3((unsigned)(tiles * cut.slices)), dim3(axo::MidCfg::THREADS), axo::MidCfg::LDS_BYTES, st, axo::GatedProduct<OP>{g}, sc);
    if (const int rc = launched()) return rc;
    const int blocks = 128 * axo::gated_cols<OP>(128) / 4 / axo::SPLIT_JOIN_THREADS;
    hipLaunchKernelGGL(axo::gated_split_join_kernel<OP>, dim3((unsigned)(tiles * blocks)), dim3(axo::SPLIT_JOIN_THREADS), 0, st, axo::GatedProduct<OP>{g}, sc);
    return launched();
}
template <int OP>
int launch_gated(const GatedArgs& g, const Shard& s, void* ws, hipStream_t st) {
    if (g.Mo == 0 || g.No == 0) return AXO_OK;
    const GatedPlan& plan = gated_plans(s).of[OP];
    if (plan.general || !gated_spans_ok<OP>(g)) return launch_gated_generic<OP>(g, st);
    switch (plan.cut.kind) {  // of the sizes alone; kinds that an operation has not are never its plan's
        case 0: return launch_gated_slim<OP, 0>(g, plan.cut, ws, st);
        case 1: return launch_gated_slim<OP, 1>(g, plan.cut, ws, st);
        case 2: return launch_gated_slim<OP, 2>(g, plan.cut, ws, st);
        case 3: return launch_gated_slim<OP, 3>(g, plan.cut, ws, st);
        case GATED_SPLIT:
            if constexpr (OP != axo::GATED_DX) {
                axo::GemmArgs as_one = g;
                if (OP == axo::GATED_FWD) as_one.No *= 2;
                if (takes_lines_on(as_one, axo::KC, axo::GATED_LB<OP>, Tiles::mid, {}) != 0) return launch_gated_split<OP, true>(g, plan.cut, ws, st);
            }
            return launch_gated_split<OP, false>(g, plan.cut, ws, st);
        default: break;
    }
    const int cols = OP == axo::GATED_FWD ? 2 * g.No : g.No, red = OP == axo::GATED_DX ? 2 * g.R : g.R;
    return launch_gated_tiles_of<OP>(g, plan.tiles, cols, red, st);
}

int check_gated_workspace(const Shard& s, const void* ws, size_t ws_bytes, Buffers& b) {
    const size_t need = gated_plans(s).bytes;
    if (need == 0) return AXO_OK;
    if (!ws || ws_bytes < need) return AXO_ERR_WORKSPACE;
    if (!aligned16(ws)) return AXO_ERR_MISALIGNED;
    b.writes(ws, (int64_t)need, 1, (int64_t)need, 1);
    return AXO_OK;
}

int launch_map(const axo::GatedMapArgs& g, bool back, hipStream_t st) {
    if (g.M == 0 || g.N == 0) return AXO_OK;
    const dim3 grid(at_most((tiles_in(g.N, 8) * g.M + axo::GATED_MAP_THREADS - 1) / axo::GATED_MAP_THREADS, 1 << 20)), block(axo::GATED_MAP_THREADS);
    if (back) hipLaunchKernelGGL(axo::gated_map_kernel<true>, grid, block, 0, st, g);
    else hipLaunchKernelGGL(axo::gated_map_kernel<false>, grid, block, 0, st, g);
    return launched();
}

// Two weight gradients.  T: type of the outputs.
template <typename T>
int gated_wgrad(const axo_problem_t* p, const void* X, int64_t ldx, const void* dG, const void* dU, int64_t lddz, T* dWg, T* dWu, int64_t lddw,
                void* ws, size_t ws_bytes, hipStream_t st) {
    constexpr bool F32 = sizeof(T) == 4;
    Shard s;
    if (const int rc = derive_shard(p, &s)) return rc;
    if (const int rc = first_error({check_matrix(X, ldx, s.M, s.Kl), check_matrix(dG, lddz, s.M, s.Nl), check_matrix(dU, lddz, s.M, s.Nl)})) return rc;
    for (const T* w : {dWg, dWu}) {
        if (s.Kl == 0 || s.Nl == 0) break;
        if (!w) return AXO_ERR_NULL_PTR;
        if (lddw < s.Nl) return AXO_ERR_BAD_LD;
        if (!aligned16(w) || lddw % (F32 ? 4 : 8)) return AXO_ERR_MISALIGNED;
    }
    Buffers b;
    b.reads(X, ldx, s.M, s.Kl, 2);
    b.reads(dG, lddz, s.M, s.Nl, 2);
    b.reads(dU, lddz, s.M, s.Nl, 2);
    b.writes(dWg, lddw, s.Kl, s.Nl, sizeof(T));
    b.writes(dWu, lddw, s.Kl, s.Nl, sizeof(T));
    if (const int rc = first_error({check_gated_workspace(s, ws, ws_bytes, b), b.check()})) return rc;
    if (const GatedCut& cut = gated_plans(s).of[axo::GATED_DW].cut; cut.kind == GATED_SPLIT) {
        auto fits = [&](int64_t ld) { return (s.M + axo::TILE_BK) * ld * 2 + 256 < (int64_t)0xFFFF0000; };
        GatedArgs h{};
        h.A = static_cast<const bf16_t*>(X); h.lda = ldx;
        h.B = static_cast<const bf16_t*>(dG); h.B2 = static_cast<const bf16_t*>(dU); h.ldb = lddz;
        h.C = reinterpret_cast<bf16_t*>(dWg); h.U = reinterpret_cast<bf16_t*>(dWu); h.ldc = lddw;
        h.Mo = (int)s.Kl; h.No = (int)s.Nl; h.R = (int)s.M;
        h.epilogue = F32 ? axo::EPI_ACC_F32 : axo::EPI_NONE;
        if (fits(ldx) && fits(lddz)) return launch_gated_split<axo::GATED_DW, false>(h, cut, ws, st);
    }
    axo::GemmArgs g[2]{};
    for (int i = 0; i < 2; ++i) {
        g[i].A = static_cast<const bf16_t*>(X); g[i].lda = ldx;
        g[i].B = static_cast<const bf16_t*>(i ? dU : dG); g[i].ldb = lddz;
        g[i].C = reinterpret_cast<bf16_t*>(i ? dWu : dWg); g[i].ldc = lddw;
        g[i].Mo = (int)s.Kl; g[i].No = (int)s.Nl; g[i].R = (int)s.M;
        g[i].epilogue = F32 ? axo::EPI_ACC_F32 : axo::EPI_NONE;
    }
    return launch_products(g, 2, axo::MC, axo::MC, st);
}

}  // namespace axo_block

extern "C" {

int axo_norm_fwd(const axo_problem_t* p, const void* X, int64_t ldx, const void* R, int64_t ldr, int type, const void* gamma, const void* beta,
                 float eps, void* S, int64_t lds, void* Y, int64_t ldy, float* stats, void* hip_stream) {
    using namespace axo_block;
    axo::NormArgs g{};
    Buffers b;
    if (const int rc = plan_norm(p, X, ldx, R, ldr, type, S, lds, b, g)) return rc;
    if (k_axis(p) != 1) return AXO_ERR_BAD_GRID;
    if (const int rc = plan_norm_output(gamma, beta, eps, Y, ldy, stats, b, g)) return rc;
    if (const int rc = b.check()) return rc;
    g.phase = axo::NORM_WHOLE;
    return launch_norm(g, type, static_cast<hipStream_t>(hip_stream));
}

int axo_norm_part(const axo_problem_t* p, const void* X, int64_t ldx, const void* R, int64_t ldr, int type, void* S, int64_t lds, float* part,
                  void* hip_stream) {
    using namespace axo_block;
    axo::NormArgs g{};
    Buffers b;
    if (const int rc = plan_norm(p, X, ldx, R, ldr, type, S, lds, b, g)) return rc;
    if (const int rc = check_vector(part, g.K > 0 ? g.M : 0, 8, false)) return rc;
    b.writes(part, 2 * (int64_t)g.M, 1, 2 * (int64_t)g.M, 4);
    if (const int rc = b.check()) return rc;
    g.part = reinterpret_cast<float2*>(part);
    g.phase = axo::NORM_PART;
    return launch_norm(g, type, static_cast<hipStream_t>(hip_stream));
}

int axo_norm_apply(const axo_problem_t* p, const void* S, int64_t lds, int type, const float* parts, int n_parts, const void* gamma,
                   const void* beta, float eps, void* Y, int64_t ldy, float* stats, void* hip_stream) {
    using namespace axo_block;
    axo::NormArgs g{};
    Buffers b;
    if (const int rc = plan_norm(p, S, lds, nullptr, 0, type, nullptr, 0, b, g)) return rc;
    if (n_parts != k_axis(p)) return AXO_ERR_BAD_ARG;
    if (const int rc = check_vector(parts, g.K > 0 ? g.M : 0, 8, false)) return rc;
    if (const int rc = plan_norm_output(gamma, beta, eps, Y, ldy, stats, b, g)) return rc;
    b.reads(parts, 2 * (int64_t)g.M * n_parts, 1, 2 * (int64_t)g.M * n_parts, 4);
    if (const int rc = b.check()) return rc;
    g.parts = reinterpret_cast<const float2*>(parts);
    g.n_parts = n_parts;
    g.phase = axo::NORM_APPLY;
    return launch_norm(g, type, static_cast<hipStream_t>(hip_stream));
}

int axo_norm_bwd(const axo_problem_t* p, const void* dY, int64_t lddy, const void* S, int64_t lds, const void* R, int64_t ldr, int type,
                 const void* gamma, const float* stats, void* dX, int64_t lddx, float* dgamma, float* dbeta, int accumulate, void* ws,
                 size_t ws_bytes, void* hip_stream) {
    using namespace axo_block;
    axo::NormBwdArgs g{};
    Buffers b;
    if (const int rc = plan_norm_bwd(p, dY, lddy, S, lds, type, gamma, stats, b, g)) return rc;
    if (k_axis(p) != 1) return AXO_ERR_BAD_GRID;
    if (const int rc = first_error({plan_norm_dx(R, ldr, type, dX, lddx, b, g), plan_norm_columns(dgamma, dbeta, accumulate, ws, ws_bytes, b, g)})) return rc;
    if (const int rc = b.check()) return rc;
    g.phase = axo::NORM_WHOLE;
    return launch_norm_bwd(g, type, static_cast<hipStream_t>(hip_stream));
}

int axo_norm_bwd_part(const axo_problem_t* p, const void* dY, int64_t lddy, const void* S, int64_t lds, int type, const void* gamma,
                      const float* stats, float* sums, float* dgamma, float* dbeta, int accumulate, void* ws, size_t ws_bytes, void* hip_stream) {
    using namespace axo_block;
    axo::NormBwdArgs g{};
    Buffers b;
    if (const int rc = plan_norm_bwd(p, dY, lddy, S, lds, type, gamma, stats, b, g)) return rc;
    if (const int rc = first_error({check_vector(sums, g.K > 0 ? g.M : 0, 8, false), plan_norm_columns(dgamma, dbeta, accumulate, ws, ws_bytes, b, g)})) return rc;
    b.writes(sums, 2 * (int64_t)g.M, 1, 2 * (int64_t)g.M, 4);
    if (const int rc = b.check()) return rc;
    g.sums = reinterpret_cast<float2*>(sums);
    g.phase = axo::NORM_PART;
    return launch_norm_bwd(g, type, static_cast<hipStream_t>(hip_stream));
}

int axo_norm_bwd_apply(const axo_problem_t* p, const void* dY, int64_t lddy, const void* S, int64_t lds, const void* R, int64_t ldr, int type,
                       const void* gamma, const float* stats, const float* sums, void* dX, int64_t lddx, void* hip_stream) {
    using namespace axo_block;
    axo::NormBwdArgs g{};
    Buffers b;
    if (const int rc = plan_norm_bwd(p, dY, lddy, S, lds, type, gamma, stats, b, g)) return rc;
    if (const int rc = first_error({check_vector(sums, g.K > 0 ? g.M : 0, 8, false), plan_norm_dx(R, ldr, type, dX, lddx, b, g)})) return rc;
    b.reads(sums, 2 * (int64_t)g.M, 1, 2 * (int64_t)g.M, 4);
    if (const int rc = b.check()) return rc;
    g.sums = reinterpret_cast<float2*>(const_cast<float*>(sums));
    g.phase = axo::NORM_APPLY;
    return launch_norm_bwd(g, type, static_cast<hipStream_t>(hip_stream));
}

size_t axo_norm_workspace_bytes(const axo_problem_t* p) {
    axo_host::Shard s;
    return axo_host::derive_shard(p, &s) ? 0 : axo_block::norm_workspace(s.M, s.Kl);
}

int axo_gated_fwd(const axo_problem_t* p, const void* X, int64_t ldx, const void* Wg, const void* Wu, int64_t ldw, const void* bg, const void* bu,
                  int gate, void* G, void* U, int64_t ldz, void* H, int64_t ldh, void* ws, size_t ws_bytes, void* hip_stream) {
    using namespace axo_block;
    return guarded([&]() -> int {
        Shard s;
        if (const int rc = derive_shard(p, &s)) return rc;
        if (!known_gate(gate)) return AXO_ERR_BAD_EPILOGUE;
        const bool save = G || U;
        const int64_t n = s.M > 0 ? s.Nl : 0;
        if (const int rc = first_error({check_matrix(X, ldx, s.M, s.Kl), check_matrix(Wg, ldw, s.Kl, s.Nl), check_matrix(Wu, ldw, s.Kl, s.Nl),
                                        check_vector(bg, n, 16, true), check_vector(bu, n, 16, true), check_matrix(H, ldh, s.M, s.Nl)}))
            return rc;
        if (save)
            if (const int rc = first_error({check_matrix(G, ldz, s.M, s.Nl), check_matrix(U, ldz, s.M, s.Nl)})) return rc;
        Buffers b;
        b.reads(X, ldx, s.M, s.Kl, 2);
        b.reads(Wg, ldw, s.Kl, s.Nl, 2);
        b.reads(Wu, ldw, s.Kl, s.Nl, 2);
        b.reads(bg, s.Nl, 1, s.Nl, 2);
        b.reads(bu, s.Nl, 1, s.Nl, 2);
        b.writes(H, ldh, s.M, s.Nl, 2);
        if (save) {
            b.writes(G, ldz, s.M, s.Nl, 2);
            b.writes(U, ldz, s.M, s.Nl, 2);
        }
        if (const int rc = first_error({check_gated_workspace(s, ws, ws_bytes, b), b.check()})) return rc;
        GatedArgs g{};
        g.A = static_cast<const bf16_t*>(X); g.lda = ldx;
        g.B = static_cast<const bf16_t*>(Wg); g.ldb = ldw;
        g.B2 = static_cast<const bf16_t*>(Wu);
        g.bias = s.k_coord == 0 ? static_cast<const bf16_t*>(bg) : nullptr;
        g.bias2 = s.k_coord == 0 ? static_cast<const bf16_t*>(bu) : nullptr;
        g.C = static_cast<bf16_t*>(H); g.ldc = ldh;
        g.G = static_cast<bf16_t*>(G);
        g.U = static_cast<bf16_t*>(U);
        g.ldz = ldz;
        g.Mo = (int)s.M; g.No = (int)s.Nl; g.R = (int)s.Kl;
        g.gate = gate;
        return launch_gated<axo::GATED_FWD>(g, s, ws, static_cast<hipStream_t>(hip_stream));
    });
}

int axo_gated_act(const axo_problem_t* p, const void* G, const void* U, int64_t ldz, int gate, void* H, int64_t ldh, void* hip_stream) {
    using namespace axo_block;
    Shard s;
    if (const int rc = derive_shard(p, &s)) return rc;
    if (!known_gate(gate)) return AXO_ERR_BAD_EPILOGUE;
    if (const int rc = first_error({check_matrix(G, ldz, s.M, s.Kl), check_matrix(U, ldz, s.M, s.Kl), check_matrix(H, ldh, s.M, s.Kl)})) return rc;
    Buffers b;
    b.reads(G, ldz, s.M, s.Kl, 2);
    b.reads(U, ldz, s.M, s.Kl, 2);
    b.writes(H, ldh, s.M, s.Kl, 2);
    if (const int rc = b.check()) return rc;
    axo::GatedMapArgs g{};
    g.G = static_cast<const bf16_t*>(G);
    g.U = static_cast<const bf16_t*>(U);
    g.H = static_cast<bf16_t*>(H);
    g.ldz = ldz;
    g.ldout = ldh;
    g.M = (int)s.M; g.N = (int)s.Kl;
    g.gate = gate;
    return launch_map(g, false, static_cast<hipStream_t>(hip_stream));
}

int axo_gated_dact(const axo_problem_t* p, const void* dH, int64_t lddh, const void* G, const void* U, int64_t ldz, int gate, void* dG, void* dU,
                   int64_t lddz, void* hip_stream) {
    using namespace axo_block;
    Shard s;
    if (const int rc = derive_shard(p, &s)) return rc;
    if (!known_gate(gate)) return AXO_ERR_BAD_EPILOGUE;
    if (const int rc = first_error({check_matrix(dH, lddh, s.M, s.Kl), check_matrix(G, ldz, s.M, s.Kl), check_matrix(U, ldz, s.M, s.Kl),
                                    check_matrix(dG, lddz, s.M, s.Kl), check_matrix(dU, lddz, s.M, s.Kl)}))
        return rc;
    Buffers b;
    b.reads(dH, lddh, s.M, s.Kl, 2);
    b.reads(G, ldz, s.M, s.Kl, 2);
    b.reads(U, ldz, s.M, s.Kl, 2);
    b.writes(dG, lddz, s.M, s.Kl, 2);
    b.writes(dU, lddz, s.M, s.Kl, 2);
    if (const int rc = b.check()) return rc;
    axo::GatedMapArgs g{};
    g.dH = static_cast<const bf16_t*>(dH); g.lddh = lddh;
    g.G = static_cast<const bf16_t*>(G);
    g.U = static_cast<const bf16_t*>(U);
    g.ldz = ldz;
    g.dG = static_cast<bf16_t*>(dG);
    g.dU = static_cast<bf16_t*>(dU);
    g.ldout = lddz;
    g.M = (int)s.M; g.N = (int)s.Kl;
    g.gate = gate;
    return launch_map(g, true, static_cast<hipStream_t>(hip_stream));
}

int axo_gated_dgrad_act(const axo_problem_t* p, const void* dY, int64_t lddy, const void* W, int64_t ldw, const void* G, const void* U, int64_t ldz,
                        int gate, void* dG, void* dU, int64_t lddz, void* ws, size_t ws_bytes, void* hip_stream) {
    using namespace axo_block;
    return guarded([&]() -> int {
        Shard s;
        if (const int rc = derive_shard(p, &s)) return rc;
        if (!known_gate(gate)) return AXO_ERR_BAD_EPILOGUE;
        if (const int rc = first_error({check_matrix(dY, lddy, s.M, s.Nl), check_matrix(W, ldw, s.Kl, s.Nl), check_matrix(G, ldz, s.M, s.Kl),
                                        check_matrix(U, ldz, s.M, s.Kl), check_matrix(dG, lddz, s.M, s.Kl), check_matrix(dU, lddz, s.M, s.Kl)}))
            return rc;
        Buffers b;
        b.reads(dY, lddy, s.M, s.Nl, 2);
        b.reads(W, ldw, s.Kl, s.Nl, 2);
        b.reads(G, ldz, s.M, s.Kl, 2);
        b.reads(U, ldz, s.M, s.Kl, 2);
        b.writes(dG, lddz, s.M, s.Kl, 2);
        b.writes(dU, lddz, s.M, s.Kl, 2);
        if (const int rc = first_error({check_gated_workspace(s, ws, ws_bytes, b), b.check()})) return rc;
        GatedArgs g{};
        g.A = static_cast<const bf16_t*>(dY); g.lda = lddy;
        g.B = static_cast<const bf16_t*>(W); g.ldb = ldw;
        g.C = static_cast<bf16_t*>(dG); g.ldc = lddz;
        g.U = static_cast<bf16_t*>(dU);
        g.aux = static_cast<const bf16_t*>(G); g.ldaux = ldz;
        g.aux2 = static_cast<const bf16_t*>(U);
        g.Mo = (int)s.M; g.No = (int)s.Kl; g.R = (int)s.Nl;
        g.gate = gate;
        return launch_gated<axo::GATED_DACT>(g, s, ws, static_cast<hipStream_t>(hip_stream));
    });
}

int axo_gated_dgrad(const axo_problem_t* p, const void* dG, const void* dU, int64_t lddz, const void* Wg, const void* Wu, int64_t ldw, void* dX,
                    int64_t lddx, void* ws, size_t ws_bytes, void* hip_stream) {
    using namespace axo_block;
    return guarded([&]() -> int {
        Shard s;
        if (const int rc = derive_shard(p, &s)) return rc;
        if (const int rc = first_error({check_matrix(dG, lddz, s.M, s.Nl), check_matrix(dU, lddz, s.M, s.Nl), check_matrix(Wg, ldw, s.Kl, s.Nl),
                                        check_matrix(Wu, ldw, s.Kl, s.Nl), check_matrix(dX, lddx, s.M, s.Kl)}))
            return rc;
        Buffers b;
        b.reads(dG, lddz, s.M, s.Nl, 2);
        b.reads(dU, lddz, s.M, s.Nl, 2);
        b.reads(Wg, ldw, s.Kl, s.Nl, 2);
        b.reads(Wu, ldw, s.Kl, s.Nl, 2);
        b.writes(dX, lddx, s.M, s.Kl, 2);
        if (const int rc = first_error({check_gated_workspace(s, ws, ws_bytes, b), b.check()})) return rc;
        GatedArgs g{};
        g.A = static_cast<const bf16_t*>(dG); g.lda = lddz;
        g.A2 = static_cast<const bf16_t*>(dU);
        g.B = static_cast<const bf16_t*>(Wg); g.ldb = ldw;
        g.B2 = static_cast<const bf16_t*>(Wu);
        g.C = static_cast<bf16_t*>(dX); g.ldc = lddx;
        g.Mo = (int)s.M; g.No = (int)s.Kl; g.R = (int)s.Nl;
        return launch_gated<axo::GATED_DX>(g, s, ws, static_cast<hipStream_t>(hip_stream));
    });
}

int axo_gated_wgrad(const axo_problem_t* p, const void* X, int64_t ldx, const void* dG, const void* dU, int64_t lddz, void* dWg, void* dWu,
                    int64_t lddw, void* ws, size_t ws_bytes, void* hip_stream) {
    using namespace axo_block;
    return guarded([&]() -> int {
        return gated_wgrad(p, X, ldx, dG, dU, lddz, static_cast<bf16_t*>(dWg), static_cast<bf16_t*>(dWu), lddw, ws, ws_bytes, static_cast<hipStream_t>(hip_stream));
    });
}

int axo_gated_wgrad_acc(const axo_problem_t* p, const void* X, int64_t ldx, const void* dG, const void* dU, int64_t lddz, float* dWg, float* dWu,
                        int64_t lddw, void* ws, size_t ws_bytes, void* hip_stream) {
    using namespace axo_block;
    return guarded([&]() -> int { return gated_wgrad(p, X, ldx, dG, dU, lddz, dWg, dWu, lddw, ws, ws_bytes, static_cast<hipStream_t>(hip_stream)); });
}

size_t axo_gated_workspace_bytes(const axo_problem_t* p) {
    axo_host::Shard s;
    return axo_host::derive_shard(p, &s) ? 0 : axo_block::gated_plans(s).bytes;
}

int axo_gated_tiles(const axo_problem_t* p, int op, int* rows, int* cols, int* slices) {
    using namespace axo_block;
    return guarded([&]() -> int {
        Shard s;
        if (const int rc = derive_shard(p, &s)) return rc;
        if (op < AXO_GATED_OP_FWD || op > AXO_GATED_OP_WGRAD) return AXO_ERR_BAD_ARG;
        if (!rows || !cols || !slices) return AXO_ERR_NULL_PTR;
        *rows = *cols = *slices = 0;
        if (s.M == 0 || (op != AXO_GATED_OP_FWD && s.Kl == 0) || ((op == AXO_GATED_OP_FWD || op == AXO_GATED_OP_WGRAD) && s.Nl == 0)) return AXO_OK;
        const GatedPlan& plan = gated_plans(s).of[op];
        if (plan.general) return AXO_OK;
        *slices = plan.cut.slices;
        if (plan.cut.kind == GATED_SPLIT) {
            *rows = 128;
            *cols = op == AXO_GATED_OP_FWD ? 64 : 128;
            return AXO_OK;
        }
        if (op == AXO_GATED_OP_WGRAD) return AXO_OK;
        if (plan.cut.kind >= 0) {
            *rows = GATED_SLIM[op][plan.cut.kind].rows;
            *cols = GATED_SLIM[op][plan.cut.kind].cols;
            return AXO_OK;
        }
        const int wide = plan.tiles == Tiles::small ? 64 : plan.tiles == Tiles::big ? 256 : 128;
        *rows = plan.tiles == Tiles::wide ? 64 : wide;
        *cols = op == AXO_GATED_OP_FWD ? wide / 2 : wide;
        return AXO_OK;
    });
}

}  // extern "C"
