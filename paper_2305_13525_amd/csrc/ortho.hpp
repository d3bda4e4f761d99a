// Newton-Schulz iteration for gfx950: an update G is brought to one whose singular values are all about 1,
//   X <- G / (|G| + eps);   `steps` times:  X <- a X + b (X X^T) X + c (X X^T)^2 X = Q X,   Q = a + b A + c A^2,  A = X X^T
// with the Gram matrix A = X^T X and X <- X Q where G has more rows than columns: A and Q are as small as they can be, and symmetric.  The products are
//   gram   A = X X^T        s x s of reductions of l      one half of the tiles, the other half is their mirror image
//   poly   Q of A           s x s of s                    likewise, A read in the epilogue
//   apply  X <- Q X         s x l of s                    tiles of gemm_tile.hpp
// (s the smaller of G's sizes, l the larger), bound by the matrix units.  Nothing is rounded to bf16 on the way: the iteration brings small singular values up, and what
// rounding adds along with them, 1 % of the result with X, A and Q in bf16.  They are held in fp16, which the matrix units take at the same rate, X with a power of two
// that keeps its values off the subnormal numbers (its largest singular value is about 1, so its values are of 1 / sqrt(K N) or more): 0.1 %, and 0.2 % with the last rounding
// to bf16.  Sums are fp32, the norm of G is summed up in fp64, where no square leaves the range.  `a` goes into Q's diagonal, so that X is read once.
// All matrices here are padded with zeros to whole multiples of 64, so that inside no product has an edge within a chunk of eight; the padding stays zero.
#pragma once
#include "axo_common.hpp"
#include "gemm_tile.hpp"
#include "norm.hpp"

namespace axo {

constexpr int ORTHO_PAD = 64;
constexpr int ORTHO_SUMS = 256;  // workgroups that sum up G's squares

struct OrthoLoadArgs {
    const void* G; int64_t ldg;
    double* sums;        // ORTHO_SUMS of them
    bf16_t* X;           // fp16, rows x cols, pitch cols
    int K, N;
    int rows, cols;      // padded
    float eps;
    double scale;        // the power of two
};

// The squares of G, each thread's in turn, then the threads' in a fixed order.
constexpr int ORTHO_THREADS = 512;
__device__ __forceinline__ double ortho_block_sum(double v, double* lds) {
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) v += __shfl_xor(v, m, 64);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    double sum = 0.0;
#pragma unroll
    for (int w = 0; w < ORTHO_THREADS / 64; ++w) sum += lds[w];
    return sum;
}
template <typename T>
__global__ void __launch_bounds__(ORTHO_THREADS) ortho_norm_kernel(OrthoLoadArgs g) {
    __shared__ double lds[ORTHO_THREADS / 64];
    const int64_t per_row = ((int64_t)g.N + 7) / 8, chunks = per_row * g.K, step = (int64_t)gridDim.x * ORTHO_THREADS;
    double sum = 0.0;
    for (int64_t at = (int64_t)blockIdx.x * ORTHO_THREADS + threadIdx.x; at < chunks; at += step) {
        const int64_t row = at / per_row, col = (at - row * per_row) * 8;
        float v[8];
        load_chunk(static_cast<const T*>(g.G) + row * g.ldg + col, (int)min((int64_t)8, g.N - col), v);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += (double)v[i] * (double)v[i];
    }
    sum = ortho_block_sum(sum, lds);
    if (threadIdx.x == 0) g.sums[blockIdx.x] = sum;
}
// Two fp32 values to a packed fp16 pair, to nearest even.
__device__ __forceinline__ uint32_t pack_f16x2(float a, float b) {
    const f16x2 v = {(_Float16)a, (_Float16)b};
    return __builtin_bit_cast(uint32_t, v);
}
// X = G scale / (|G| + eps), zeros around it.  A gradient of zeros stays one.
template <typename T>
__global__ void __launch_bounds__(ORTHO_THREADS) ortho_load_kernel(OrthoLoadArgs g) {
    __shared__ double lds[ORTHO_THREADS / 64];
    const double norm = sqrt(ortho_block_sum(threadIdx.x < ORTHO_SUMS ? g.sums[threadIdx.x] : 0.0, lds)) + (double)g.eps;
    const double factor = norm == 0.0 ? 0.0 : g.scale / norm;
    const int64_t per_row = g.cols / 8, chunks = per_row * g.rows, step = (int64_t)gridDim.x * ORTHO_THREADS;
    for (int64_t at = (int64_t)blockIdx.x * ORTHO_THREADS + threadIdx.x; at < chunks; at += step) {
        const int64_t row = at / per_row, col = (at - row * per_row) * 8;
        u32x4 w = {0u, 0u, 0u, 0u};
        if (row < g.K && col < g.N) {
            float v[8];
            load_chunk(static_cast<const T*>(g.G) + row * g.ldg + col, (int)min((int64_t)8, g.N - col), v);
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = pack_f16x2((float)((double)v[2 * i] * factor), (float)((double)v[2 * i + 1] * factor));
        }
        *reinterpret_cast<u32x4*>(g.X + at * 8) = w;
    }
}

// ---- gram and poly ----------------------------------------------------------------------------
// The tiles on and below the diagonal of a symmetric output, and their mirror images.  Their steps of the reduction are dealt out to the workgroups in equal, contiguous shares, so
// that every workgroup has the same to do whatever the numbers: a share begins and ends inside a tile, and such a tile's sums are written to the workspace; whoever
// comes last adds them up, in the order of the steps, and finishes the tile.  Which workgroup that is depends on timing, what it computes does not, and none waits for
// another.  Those sums go past the L2 of an XCD by device-scope accesses.
struct OrthoSym : GemmArgs {
    static constexpr bool F16 = true, OWN = true;
    float alpha, beta, diag;   // C = alpha sum + beta aux + diag on the diagonal; aux nullptr: none
    float* partial;            // [2 x workgroups][tile]
    uint32_t* counters;        // one per tile, zero
    int steps;                 // of a tile
    int tiles;
    // of the segment at hand
    int tile, from, count;     // steps
    int slot;

    // The workgroup that has unit u of all `tiles * steps`, dealt out to W workgroups: workgroup w begins with unit floor(w U / W).
    __device__ __forceinline__ int64_t units() const { return (int64_t)tiles * steps; }
    __device__ __forceinline__ int64_t first_of(int64_t w) const { return w * units() / gridDim.x; }
    __device__ __forceinline__ int owner_of(int64_t u) const { return (int)(((u + 1) * gridDim.x - 1) / units()); }

    template <typename C, int BM, int BN>
    static __device__ __forceinline__ void finish(const OrthoSym& g, f32x4 (&acc)[C::TM][C::TN], const int i0, const int j0, const int wm, const int wn, const int tid,
                                                  char* smem);
};
// Device-scope accesses of 16 bytes: past the L2, which other XCDs do not see.
constexpr int DEVICE_SCOPE = 16;  // sc1
__device__ __forceinline__ __amdgpu_buffer_rsrc_t partial_buffer(float* p, int bytes) { return __builtin_amdgcn_make_buffer_rsrc(p, 0, bytes, 0x00020000); }

template <typename C, int BM, int BN>
__device__ __forceinline__ void OrthoSym::finish(const OrthoSym& g, f32x4 (&acc)[C::TM][C::TN], const int i0, const int j0, const int wm, const int wn, const int tid,
                                                 char* smem) {
    static_assert(BM == BN, "mirror images");
    constexpr int STRIDE = BN * 2 + 16, CPR = BN / 8, ROUNDS = BM * CPR / C::THREADS, TILE = BM * BN;
    static_assert(2 * BM * STRIDE <= C::LDS_BYTES && BM * CPR % C::THREADS == 0, "both images in the operand buffers");
    const int lane = tid & 63;
    const int row = wm * C::WTM + (lane & 15), col = wn * C::WTN + 4 * (lane >> 4);
    __syncthreads();  // all waves are done reading the operand buffers
    if (g.count < g.steps) {
        // a lane's quads lie behind each other by thread, in rounds: whole lines of the workspace
        auto at = [&](int a, int b) __attribute__((always_inline)) { return ((a * C::TN + b) * C::THREADS + tid) * 16; };
        const __amdgpu_buffer_rsrc_t mine = partial_buffer(g.partial + (int64_t)g.slot * TILE, TILE * 4);
#pragma unroll
        for (int a = 0; a < C::TM; ++a)
#pragma unroll
            for (int b = 0; b < C::TN; ++b) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, acc[a][b]), mine, at(a, b), 0, DEVICE_SCOPE);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wave's sums have arrived where all XCDs see them
        __syncthreads();
        const int64_t first_unit = (int64_t)g.tile * g.steps;
        const int first = g.owner_of(first_unit), last = g.owner_of(first_unit + g.steps - 1);
        uint32_t* const arrived = reinterpret_cast<uint32_t*>(smem);
        if (tid == 0) *arrived = __hip_atomic_fetch_add(g.counters + g.tile, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __syncthreads();
        const bool finishes = *arrived == (uint32_t)(last - first);
        __syncthreads();  // the word has been read
        if (!finishes) return;
        // the first one's share of this tile is the last of its segments, the others' the first of theirs
        const int head = 2 * first + (g.first_of(first) < first_unit ? 1 : 0);
        for (int w = first; w <= last; ++w) {
            const __amdgpu_buffer_rsrc_t part = partial_buffer(g.partial + (int64_t)(w == first ? head : 2 * w) * TILE, TILE * 4);
            f32x4 v[C::TM][C::TN];
#pragma unroll
            for (int a = 0; a < C::TM; ++a)
#pragma unroll
                for (int b = 0; b < C::TN; ++b) v[a][b] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(part, at(a, b), 0, DEVICE_SCOPE));
#pragma unroll
            for (int a = 0; a < C::TM; ++a)
#pragma unroll
                for (int b = 0; b < C::TN; ++b) acc[a][b] = w == first ? v[a][b] : acc[a][b] + v[a][b];
        }
        if (tid == 0) __hip_atomic_store(g.counters + g.tile, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    char* const image = smem + BM * STRIDE;
    const bool mirrored = i0 != j0;
#pragma unroll
    for (int a = 0; a < C::TM; ++a)
#pragma unroll
        for (int b = 0; b < C::TN; ++b) {
            const int r = row + a * 16, c = col + b * 16;
            f32x4 v = acc[a][b] * g.alpha;
            if (g.aux && i0 + r < g.Mo && j0 + c < g.No) {
                const uint2 raw = *reinterpret_cast<const uint2*>(g.aux + (int64_t)(i0 + r) * g.ldaux + j0 + c);
                const f16x2 lo = __builtin_bit_cast(f16x2, raw.x), hi = __builtin_bit_cast(f16x2, raw.y);
                v[0] = __builtin_fmaf(g.beta, (float)lo[0], v[0]);
                v[1] = __builtin_fmaf(g.beta, (float)lo[1], v[1]);
                v[2] = __builtin_fmaf(g.beta, (float)hi[0], v[2]);
                v[3] = __builtin_fmaf(g.beta, (float)hi[1], v[3]);
            }
            if (!mirrored)
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] += r == c + e ? g.diag : 0.f;
            const uint2 packed = {pack_f16x2(v[0], v[1]), pack_f16x2(v[2], v[3])};
            *reinterpret_cast<uint2*>(smem + r * STRIDE + c * 2) = packed;
            if (mirrored) {
                *reinterpret_cast<uint16_t*>(image + c * STRIDE + r * 2) = (uint16_t)packed.x;
                *reinterpret_cast<uint16_t*>(image + (c + 1) * STRIDE + r * 2) = (uint16_t)(packed.x >> 16);
                *reinterpret_cast<uint16_t*>(image + (c + 2) * STRIDE + r * 2) = (uint16_t)packed.y;
                *reinterpret_cast<uint16_t*>(image + (c + 3) * STRIDE + r * 2) = (uint16_t)(packed.y >> 16);
            }
        }
    __syncthreads();
    auto out = [&](const char* from, int r0, int c0) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < ROUNDS; ++i) {
            const int q = i * C::THREADS + tid, r = q / CPR, c = q % CPR * 8;
            if (r0 + r < g.Mo && c0 + c < g.No)
                *reinterpret_cast<u32x4*>(g.C + (int64_t)(r0 + r) * g.ldc + c0 + c) = *reinterpret_cast<const u32x4*>(from + r * STRIDE + c * 2);
        }
    };
    out(smem, i0, j0);
    if (mirrored) out(image, j0, i0);
}

// The tile of an index: rows one behind the other, up to the diagonal.
__device__ __forceinline__ void ortho_tile(int t, int& ti, int& tj) {
    ti = (int)((sqrtf(8.0f * (float)t + 1.0f) - 1.0f) * 0.5f);
    while ((ti + 1) * (ti + 2) / 2 <= t) ++ti;
    while (ti * (ti + 1) / 2 > t) --ti;
    tj = t - ti * (ti + 1) / 2;
}
template <int SIZE, int LAYOUT>
__device__ __forceinline__ void ortho_sym(OrthoSym g, char* smem) {
    const int bid = xcd_run(blockIdx.x, gridDim.x);  // neighbours share rows of tiles
    const int64_t begin = g.first_of(bid), end = g.first_of(bid + 1);
    const bf16_t *const A = g.A, *const B = g.B;
    for (int64_t u = begin; u < end;) {
        g.tile = (int)(u / g.steps);
        g.from = (int)(u - (int64_t)g.tile * g.steps);
        g.count = (int)min((int64_t)(g.steps - g.from), end - u);
        g.slot = 2 * bid + (u > begin ? 1 : 0);
        g.R = g.count * TILE_BK;
        const int64_t skip = (int64_t)g.from * TILE_BK * (LAYOUT == KC ? 1 : g.lda);
        g.A = A + skip;
        g.B = B + skip;
        int ti, tj;
        ortho_tile(g.tile, ti, tj);
        if (u > begin) __syncthreads();  // the tile before has left LDS
        if constexpr (SIZE == 64) gemm_ring_body<64, 64, 2, 2, 4, LAYOUT, LAYOUT>(g, ti * 64, tj * 64, smem, threadIdx.x);
        else gemm_ring_body<128, 128, 4, 2, 4, LAYOUT, LAYOUT>(g, ti * 128, tj * 128, smem, threadIdx.x);
        u += g.count;
    }
}
template <int LAYOUT>
__global__ void __launch_bounds__(256, 2) ortho_sym_64_kernel(OrthoSym g) {
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    ortho_sym<64, LAYOUT>(g, smem);
}
template <int LAYOUT>
__global__ void __launch_bounds__(TILE_THREADS, 1) ortho_sym_128_kernel(OrthoSym g) {
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    ortho_sym<128, LAYOUT>(g, smem);
}

// ---- apply --------------------------------------------------------------------------------------
// A product like any other on the tiles of gemm_tile.hpp; its output X in fp16, or, of the last step, O in bf16 with the power of two taken off, up to O's edges.
struct OrthoApply : GemmArgs {
    static constexpr bool F16 = true, OWN = true;
    bf16_t* O; int64_t ldo;  // nullptr: C is written
    int K, N;                // O's
    float scale;

    template <typename C, int BM, int BN>
    static __device__ __forceinline__ void finish(const OrthoApply& g, f32x4 (&acc)[C::TM][C::TN], const int i0, const int j0, const int wm, const int wn, const int tid,
                                                  char* smem) {
        const int lane = tid & 63, wave = wm * (BN / C::WTN) + wn;
        char* const stage = smem + wave * (C::WTM * C::EPI_STRIDE);
        __syncthreads();  // all waves are done reading the operand buffers
        auto put = [&](auto pack) __attribute__((always_inline)) {
#pragma unroll
            for (int b = 0; b < C::TN; ++b)
#pragma unroll
                for (int a = 0; a < C::TM; ++a)
                    *reinterpret_cast<uint2*>(stage + (a * 16 + (lane & 15)) * C::EPI_STRIDE + (b * 16 + 4 * (lane >> 4)) * 2) =
                        uint2{pack(acc[a][b][0], acc[a][b][1]), pack(acc[a][b][2], acc[a][b][3])};
        };
        if (g.O) put([&](float x, float y) __attribute__((always_inline)) { return pack_bf16x2(x * g.scale, y * g.scale); });
        else put([](float x, float y) __attribute__((always_inline)) { return pack_f16x2(x, y); });
        __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0): the region is private to the wave
        __builtin_amdgcn_wave_barrier();
        constexpr int LPR = C::WTN * 2 / 16, RPP = 64 / LPR, PASSES = C::WTM / RPP;
        u32x4 v[PASSES];
#pragma unroll
        for (int p = 0; p < PASSES; ++p)  // all reads ahead of the first store, as in tile_epilogue
            v[p] = *reinterpret_cast<const u32x4*>(stage + (p * RPP + lane / LPR) * C::EPI_STRIDE + lane % LPR * 16);
        const int row0 = i0 + wm * C::WTM + lane / LPR, col = j0 + wn * C::WTN + lane % LPR * 8;
        const int rows = g.O ? g.K : g.Mo, valid = (g.O ? g.N : g.No) - col;
        bf16_t* const to = g.O ? g.O + (int64_t)row0 * g.ldo + col : g.C + (int64_t)row0 * g.ldc + col;
        const int64_t ld = g.O ? g.ldo : g.ldc;
#pragma unroll
        for (int p = 0; p < PASSES; ++p)
            if (row0 + p * RPP < rows && valid > 0) store_eight<true>(v[p], to + (int64_t)(p * RPP) * ld, false, valid);
    }
};
template <int LB>
__global__ void __launch_bounds__(TILE_THREADS, 1) ortho_apply_256_kernel(OrthoApply g, TileSched sc) {
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int bid = blockIdx.x;
    start_shift(bid, sc.shift);
    int tm, tn;
    if (bid < sc.n_big) {
        tile_of_index(xcd_run(bid, sc.n_big), sc.tiles_m, sc.big_cols, sc.group_m, tm, tn);
        gemm_tile_body<256, 256, 2, 4, KC, LB>(g, inside_row<256, KC>(g, tm * 256), inside_col<256>(g, tn * 256), smem);
    } else {
        const int n_small = (int)gridDim.x - sc.n_big;
        tile_of_index(xcd_run(bid - sc.n_big, n_small), sc.tiles_m, sc.small_cols, sc.group_m, tm, tn);
        gemm_ring_body<256, 128, 4, 2, 3, KC, LB>(g, inside_row<256, KC>(g, tm * 256), inside_col<128>(g, sc.big_cols * 256 + tn * 128), smem, threadIdx.x);
    }
}
template <int LB>
__global__ void __launch_bounds__(TILE_THREADS, 1) ortho_apply_128_kernel(OrthoApply g, int tiles_m, int tiles_n, int group_m) {
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    int tm, tn;
    tile_of_index(xcd_run(blockIdx.x, gridDim.x), tiles_m, tiles_n, group_m, tm, tn);
    gemm_ring_body<128, 128, 4, 2, 4, KC, LB>(g, inside_row<128, KC>(g, tm * 128), inside_col<128>(g, tn * 128), smem, threadIdx.x);
}
template <int LB>
__global__ void __launch_bounds__(TILE_THREADS, 1) ortho_apply_rect_kernel(OrthoApply g, int tiles_m, int tiles_n, int group_m) {
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    int tm, tn;
    tile_of_index(xcd_run(blockIdx.x, gridDim.x), tiles_m, tiles_n, group_m, tm, tn);
    gemm_ring_body<64, 128, 2, 4, 4, KC, LB>(g, inside_row<64, KC>(g, tm * 64), inside_col<128>(g, tn * 128), smem, threadIdx.x);
}
template <int LB>
__global__ void __launch_bounds__(256, 2) ortho_apply_64_kernel(OrthoApply g, int tiles_m, int tiles_n, int group_m) {
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    int tm, tn;
    tile_of_index(xcd_run(blockIdx.x, gridDim.x), tiles_m, tiles_n, group_m, tm, tn);
    gemm_ring_body<64, 64, 2, 2, 4, KC, LB>(g, inside_row<64, KC>(g, tm * 64), inside_col<64>(g, tn * 64), smem, threadIdx.x);
}

}  // namespace axo
