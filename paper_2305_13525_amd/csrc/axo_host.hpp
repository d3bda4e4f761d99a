// Host-side pieces that the entry points share: shard derivation, argument checks, byte ranges of matrices, launch helpers.
#pragma once
#include "../../include/axo.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <new>

#include "gemm_tile.hpp"

namespace axo_host {

struct Shard {
    int64_t M, Kl, Nl, row0, k0, n0;
    int k_coord;  // coordinate along the axis that splits K
};

inline int derive_shard(const axo_problem_t* p, Shard* s) {
    if (!p) return AXO_ERR_NULL_PTR;
    if (p->reserved != 0 || (p->transposed != 0 && p->transposed != 1)) return AXO_ERR_BAD_ARG;
    if (p->Gx < 1 || p->Gy < 1 || p->Gz < 1) return AXO_ERR_BAD_GRID;
    if (p->ix < 0 || p->ix >= p->Gx || p->iy < 0 || p->iy >= p->Gy || p->iz < 0 || p->iz >= p->Gz)
        return AXO_ERR_BAD_COORD;
    if (p->T < 0 || p->K < 0 || p->N < 0) return AXO_ERR_BAD_SIZE;
    // Section 3.2: I is cut over the token axis (Z) and the reduction axis, W over the reduction
    // axis and the output axis.  transposed swaps which of X / Y plays which role.
    const int gk = p->transposed ? p->Gy : p->Gx, ik = p->transposed ? p->iy : p->ix;
    const int gn = p->transposed ? p->Gx : p->Gy, in = p->transposed ? p->ix : p->iy;
    if (p->T % p->Gz != 0 || p->K % gk != 0 || p->N % gn != 0) return AXO_ERR_INDIVISIBLE;
    s->M = p->T / p->Gz;
    s->Kl = p->K / gk;
    s->Nl = p->N / gn;
    if (s->M > INT32_MAX || s->Kl > INT32_MAX || s->Nl > INT32_MAX) return AXO_ERR_BAD_SIZE;
    s->row0 = s->M * p->iz;
    s->k0 = s->Kl * ik;
    s->n0 = s->Nl * in;
    s->k_coord = ik;
    return AXO_OK;
}

inline bool aligned16(const void* q) { return (reinterpret_cast<uintptr_t>(q) & 15u) == 0; }

// One matrix argument: pointer, leading dimension, row length.  A matrix without elements is
// never dereferenced, so nothing about it is checked.
inline int check_matrix(const void* ptr, int64_t ld, int64_t rows, int64_t row_len) {
    if (rows == 0 || row_len == 0) return AXO_OK;
    if (!ptr) return AXO_ERR_NULL_PTR;
    if (ld < row_len) return AXO_ERR_BAD_LD;
    if (!aligned16(ptr) || (ld % 8) != 0) return AXO_ERR_MISALIGNED;
    return AXO_OK;
}

// A launch's threads per grid dimension have to stay below 2^32.  Thin outputs of hundreds of millions of rows or
// columns pass that with the smaller tiles; the choices below then fall through to a kernel that takes them.
inline bool grid_fits(int64_t blocks, int threads) { return blocks <= (int64_t)UINT32_MAX / threads; }
inline int64_t tiles_in(int n, int size) { return ((int64_t)n + size - 1) / size; }

// The tuned kernel covers the output with 256x256 tiles and, to balance tile counts that do not
// fill the last round of CUs, a region of 256x128 tiles.  The CU count is a design constant
// (MI355X: 256 CUs) so that planning needs no device.
constexpr int NUM_CU = 256;

// The tuned kernels' dynamic LDS size is above the default limit, so the limit is raised once per
// kernel and device (`raised` holds one bit per device ordinal; a process rarely sees more than
// 8, and beyond 64 the attribute is simply set on every launch).
inline bool raise_lds_limit(const void* kernel, int bytes, std::atomic<uint64_t>* raised) {
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess) return false;
    const uint64_t bit = dev >= 0 && dev < 64 ? (uint64_t)1 << dev : 0;
    if (bit && (raised->load(std::memory_order_acquire) & bit)) return true;
    if (hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) != hipSuccess)
        return false;
    raised->fetch_or(bit, std::memory_order_release);
    return true;
}

inline int64_t steps_in(int R) { return tiles_in(R, axo::TILE_BK); }
inline int64_t rounds_of(int64_t tiles) { return (tiles + NUM_CU - 1) / NUM_CU; }

// Byte range [lo, hi) that a matrix argument covers (rows x row_len elements of elem bytes, rows
// ld elements apart); empty matrices cover nothing.  The matrix itself is kept beside its range
// for the exact overlap test.
struct Range {
    uintptr_t lo, hi;
    int64_t pitch, rows, width;  // bytes between rows, row count, bytes per row
    static int64_t floor_div(int64_t x, int64_t y) { return x / y - ((x % y != 0) && ((x < 0) != (y < 0)) ? 1 : 0); }
    bool overlaps(const Range& o) const { return lo < o.hi && o.lo < hi; }
    // Do the two matrices share a byte?  (Ranges that overlap need not: two column blocks of one
    // buffer interleave.)  Row r of this matrix covers [a, a + width) relative to the other's
    // base; row q of the other covers [q * pitch, q * pitch + width_o); they meet iff
    // q * pitch < a + width and q * pitch + width_o > a, an interval of q that is clamped to the
    // other's rows.  Only called when the ranges overlap, which no well-formed call makes them do.
    bool shares_bytes_with(const Range& o) const {
        if (!overlaps(o)) return false;
        if (pitch == o.pitch && pitch > 0) {  // rows equally far apart: one interval of t = q - r for all rows
            const int64_t d = (int64_t)(lo - o.lo), t_lo = floor_div(d - o.width, pitch) + 1, t_hi = floor_div(d + width - 1, pitch);
            return std::max<int64_t>(t_lo, 1 - rows) <= std::min<int64_t>(t_hi, o.rows - 1);
        }
        const int64_t op = o.rows > 1 ? o.pitch : (int64_t)(o.hi - o.lo) + 1;  // one row: any positive pitch
        for (int64_t r = 0; r < rows; ++r) {
            const int64_t a = (int64_t)(lo - o.lo) + r * pitch;
            const int64_t q_hi = std::min<int64_t>(floor_div(a + width - 1, op), o.rows - 1);
            const int64_t q_lo = std::max<int64_t>(floor_div(a - o.width, op) + 1, 0);
            if (q_lo <= q_hi) return true;
        }
        return false;
    }
};
inline bool matrix_range(const void* ptr, int64_t ld, int64_t rows, int64_t row_len, int elem, Range* r) {
    if (!ptr || rows <= 0 || row_len <= 0) return false;
    r->lo = reinterpret_cast<uintptr_t>(ptr);
    r->hi = r->lo + (uintptr_t)(((rows - 1) * ld + row_len) * elem);
    r->pitch = ld * elem;
    r->rows = rows;
    r->width = row_len * elem;
    return true;
}

// No exception leaves the library: the planners keep their lists and caches in standard
// containers, whose allocations can fail.
template <typename F>
int guarded(F&& body) noexcept {
    try {
        return body();
    } catch (const std::bad_alloc&) {
        return AXO_ERR_NO_MEMORY;
    } catch (...) {
        return AXO_ERR_BAD_ARG;
    }
}

// Independent products of one kind, in as few launches as a chain's level takes (defined beside the chain's planner).
int launch_products(const axo::GemmArgs* products, int n, int la, int lb, hipStream_t st);
// The tiles of a product on its own, whichever are estimated quickest, from its sizes alone, and how an output of 256-row tiles is cut into columns of whole and of
// half-width ones, start-up shift included (defined beside the planners).
enum class Tiles { small, wide, tall, mid, big };
Tiles quickest_tiles(int Mo, int No, int R);
double tiles_time(Tiles tiles, int Mo, int No, int R);  // estimate in us, operands in the caches
double pair_time(int Mo, int No, int R, int la, int lb);  // two such products in one call
axo::TileSched plan_columns(int Mo, int No, int R);
// Whether a product fetches rows by whole cache lines on those tiles: on none (0), on whole 256-row ones (1), on all (2).
int takes_lines_on(const axo::GemmArgs& g, int la, int lb, Tiles tiles, const axo::TileSched& sc);

}  // namespace axo_host
