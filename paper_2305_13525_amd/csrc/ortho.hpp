// Newton-Schulz iteration for gfx950: an update G is brought to one whose singular values are all about 1,
//   X <- G / (|G| + eps);   `steps` times:  X <- a X + b (X X^T) X + c (X X^T)^2 X = Q X,   Q = a + b A + c A^2,  A = X X^T
// with the Gram matrix A = X^T X and X <- X Q where G has more rows than columns: A and Q are as small as they can be, and symmetric.  The products are
//   gram   A = X X^T        s x s of reductions of l      one half of the tiles, the other half is their mirror image
//   poly   Q of A           s x s of s                    likewise, A read in the epilogue
//   apply  X <- Q X         s x l of s                    tiles of gemm_tile.hpp
// (s the smaller of G's sizes, l the larger), bound by the matrix units.  Nothing is rounded to bf16 on the way: the iteration brings small singular values up, and what
// rounding adds along with them, of a random G 0.7 to 1.4 % of the result with X, A and Q in bf16.  They are held in fp16, which the matrix units take at the same rate, X with a power of two
// that keeps its values off the subnormal numbers (its largest singular value is about 1, so its values are of 1 / sqrt(K N) or more): 0.1 to 0.2 %, and 0.2 to 0.25 % with the last
// rounding to bf16.  Both grow with the spread of G's singular values, in which X's rounding is more beside the small ones: evenly in their logarithm over a factor of 100, 1.6 to 3.2 % in bf16
// and 0.2 to 0.4 in fp16, of 1000 2.8 to 8.4 and 0.3 to 1.1.
// Sums are fp32, the norm of G is summed up in fp64, where no square leaves the range.  `a` goes into Q's diagonal, so that X is read once.
// All matrices here are padded to whole multiples of 64, so that inside no product has an edge within a chunk of eight.  X's padding and with it A's is zeros; Q's is zeros but for its
// diagonal, where it is `a` throughout.  That the padding of Q X is zeros again is X's doing: a trace or a product of Q with itself would have those `a` in it.
#pragma once
#include "axo_common.hpp"
#include "gemm_slim.hpp"
#include "gemm_tile.hpp"
#include "norm.hpp"
#include "sym_cut.hpp"

namespace axo {

constexpr int ORTHO_PAD = 64;
constexpr int ORTHO_SUMS = 512;  // workgroups that sum up G's squares

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
// ORTHO_AT_ONCE chunks of eight values, `step` chunks of `per_row` to a row apart: whole ones requested together, zeros outside of G.
constexpr int ORTHO_AT_ONCE = 4;
template <typename T>
__device__ __forceinline__ void ortho_chunks(const OrthoLoadArgs& g, uint32_t at0, uint32_t step, uint32_t chunks, uint32_t per_row, float (&v)[ORTHO_AT_ONCE][8]) {
    constexpr int WORDS = sizeof(T) / 2;
    u32x4 raw[ORTHO_AT_ONCE][WORDS];
    int valid[ORTHO_AT_ONCE];
    const T* from[ORTHO_AT_ONCE];
#pragma unroll
    for (int j = 0; j < ORTHO_AT_ONCE; ++j) {
        const uint32_t at = at0 + j * step, row = at / per_row, col = (at - row * per_row) * 8;
        valid[j] = at < chunks && (int)row < g.K ? min(8, g.N - (int)col) : 0;
        from[j] = static_cast<const T*>(g.G) + (int64_t)row * g.ldg + col;
#pragma unroll
        for (int w = 0; w < WORDS; ++w) {
            raw[j][w] = u32x4{0u, 0u, 0u, 0u};
            if (valid[j] == 8) raw[j][w] = reinterpret_cast<const u32x4*>(from[j])[w];
        }
    }
#pragma unroll
    for (int j = 0; j < ORTHO_AT_ONCE; ++j) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t word = WORDS == 1 ? raw[j][0][i / 2] : raw[j][i / 4 % WORDS][i % 4];
            v[j][i] = WORDS == 1 ? bf16_bits_to_f32((bf16_t)(word >> (i % 2 * 16))) : __builtin_bit_cast(float, word);
        }
        if (valid[j] > 0 && valid[j] < 8) load_chunk(from[j], valid[j], v[j]);
    }
}
template <typename T>
__global__ void __launch_bounds__(ORTHO_THREADS) ortho_norm_kernel(OrthoLoadArgs g) {
    __shared__ double lds[ORTHO_THREADS / 64];
    // (fewer than 2^28 chunks, of weights of fewer than 2^31 values)
    const uint32_t per_row = ((uint32_t)g.N + 7) / 8, chunks = per_row * (uint32_t)g.K, step = gridDim.x * ORTHO_THREADS;
    double sum = 0.0;
    for (uint32_t at = blockIdx.x * ORTHO_THREADS + threadIdx.x; at < chunks; at += ORTHO_AT_ONCE * step) {
        float v[ORTHO_AT_ONCE][8];
        ortho_chunks<T>(g, at, step, chunks, per_row, v);
#pragma unroll
        for (int j = 0; j < ORTHO_AT_ONCE; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += (double)v[j][i] * (double)v[j][i];
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
// (Products in fp64 and their conversions bound it: 2048 x 6144 27 us and 10, 4096 x 16384 88 and 46.)
template <typename T>
__global__ void __launch_bounds__(ORTHO_THREADS) ortho_load_kernel(OrthoLoadArgs g) {
    __shared__ double lds[ORTHO_THREADS / 64];
    const double mine = threadIdx.x < ORTHO_SUMS ? g.sums[threadIdx.x] : 0.0;
    const uint32_t per_row = (uint32_t)g.cols / 8, chunks = per_row * (uint32_t)g.rows, step = gridDim.x * ORTHO_THREADS;
    const double norm = sqrt(ortho_block_sum(mine, lds)) + (double)g.eps;
    // scale / norm as a power of two and a number from 1/2 to 1, in that order: no product leaves the range of fp32 that X's does not leave
    int exponent;
    const float factor = (float)frexp(norm == 0.0 ? 0.0 : g.scale / norm, &exponent);
    for (uint32_t at0 = blockIdx.x * ORTHO_THREADS + threadIdx.x; at0 < chunks; at0 += ORTHO_AT_ONCE * step) {
        float v[ORTHO_AT_ONCE][8];
        ortho_chunks<T>(g, at0, step, chunks, per_row, v);
#pragma unroll
        for (int j = 0; j < ORTHO_AT_ONCE; ++j) {
            const uint32_t at = at0 + j * step;
            u32x4 w;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = pack_f16x2(ldexpf(v[j][2 * i], exponent) * factor, ldexpf(v[j][2 * i + 1], exponent) * factor);
            if (at < chunks) *reinterpret_cast<u32x4*>(g.X + (int64_t)at * 8) = w;
        }
    }
}

// ---- gram and poly ----------------------------------------------------------------------------
// The tiles on and below the diagonal of a symmetric output, and their mirror images, dealt out as sym_cut.hpp says.  (With every workgroup's share a contiguous run of
// all tiles' steps, wherever that begins in a tile, 4096 x 4096 with reductions of 16384 took 570 us, 500 TFLOP/s: 256 compute units read 7.8 TB/s of operands from behind
// the caches.)
// What bounds a 128 x 128 tile's step, 0.40 us where the matrix units need 0.21, is the rate at which a CU takes in operands, 32 KB: rings of three to five stages, eight waves that split a step's
// reduction and read a third less from LDS, and tiles dealt out in bands of two to eight rows all take the same time within 2 %.
// A part of a tile leaves its sums in the workspace; whoever comes last adds them up, in the order of the steps, and finishes the tile.  Which workgroup that
// is depends on timing, what it computes does not, and none waits for another.  Those sums go past the L2 of an XCD by device-scope accesses.
struct OrthoSym : GemmArgs {
    static constexpr bool F16 = true, OWN = true;
    float alpha, beta, diag;   // C = alpha sum + beta aux + diag on the diagonal; aux nullptr: none
    float* partial;            // [slots][tile]
    uint32_t* counters;        // one per tile that is cut, zero
    SymCut cut, diagonal;      // of the tiles; of those of SYM_DIAGONAL, behind tiles of SYM_HALF
    SymPart part;              // at hand

    // Quads of outputs (gemm_slim.hpp): the four values of aux, and what becomes of their sums, stored in both places.
    static __device__ __forceinline__ uint2 request(const OrthoSym& g, int row, int col) {
        return g.aux && row < g.Mo && col < g.No ? *reinterpret_cast<const uint2*>(g.aux + (int64_t)row * g.ldaux + col) : uint2{0u, 0u};
    }
    __device__ __forceinline__ f32x4 value(int row, int col, f32x4 sum, uint2 raw) const {
        const f16x2 lo = __builtin_bit_cast(f16x2, raw.x), hi = __builtin_bit_cast(f16x2, raw.y);
        const float x[4] = {(float)lo[0], (float)lo[1], (float)hi[0], (float)hi[1]};
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] = __builtin_fmaf(beta, x[e], sum[e] * alpha) + (row == col + e ? diag : 0.f);
        return sum;
    }
    static __device__ __forceinline__ void quad(const OrthoSym& g, bool mirrored, int row, int col, f32x4 sum, uint2 raw);

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
    constexpr int TILE = BM * BN;
    const int lane = tid & 63, wave = wm * (BN / C::WTN) + wn;
    __syncthreads();  // all waves are done reading the operand buffers
    if (g.part.cut >= 0) {
        // a lane's quads lie behind each other by thread, in rounds: whole lines of the workspace
        auto at = [&](int a, int b) __attribute__((always_inline)) { return ((a * C::TN + b) * C::THREADS + tid) * 16; };
        const __amdgpu_buffer_rsrc_t mine = partial_buffer(g.partial + (int64_t)g.part.slot * TILE, TILE * 4);
#pragma unroll
        for (int a = 0; a < C::TM; ++a)
#pragma unroll
            for (int b = 0; b < C::TN; ++b) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, acc[a][b]), mine, at(a, b), 0, DEVICE_SCOPE);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wave's sums have arrived where all XCDs see them
        __syncthreads();
        uint32_t* const arrived = reinterpret_cast<uint32_t*>(smem);
        if (tid == 0) *arrived = __hip_atomic_fetch_add(g.counters + g.part.cut, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __syncthreads();
        const bool finishes = *arrived == (uint32_t)(g.part.parts - 1);
        __syncthreads();  // the word has been read
        if (!finishes) return;
        for (int part = 0; part < g.part.parts; ++part) {
            const __amdgpu_buffer_rsrc_t from = partial_buffer(g.partial + (int64_t)g.cut.slot_of(g.part.cut, part) * TILE, TILE * 4);
            constexpr int ROWS = C::TM * C::TN > 16 ? 2 : C::TM;  // registers for so many rows of quads at a time
#pragma unroll
            for (int a0 = 0; a0 < C::TM; a0 += ROWS) {
                f32x4 v[ROWS][C::TN];
#pragma unroll
                for (int a = 0; a < ROWS; ++a)
#pragma unroll
                    for (int b = 0; b < C::TN; ++b) v[a][b] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(from, at(a0 + a, b), 0, DEVICE_SCOPE));
#pragma unroll
                for (int a = 0; a < ROWS; ++a)
#pragma unroll
                    for (int b = 0; b < C::TN; ++b) acc[a0 + a][b] = part == 0 ? v[a][b] : acc[a0 + a][b] + v[a][b];
            }
        }
        if (tid == 0) __hip_atomic_store(g.counters + g.part.cut, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    // what becomes of the sums, in place
    const int row0 = i0 + wm * C::WTM, col0 = j0 + wn * C::WTN, r = lane & 15, c = 4 * (lane >> 4);
#pragma unroll
    for (int a = 0; a < C::TM; ++a)
#pragma unroll
        for (int b = 0; b < C::TN; ++b) {
            const int row = row0 + a * 16 + r, col = col0 + b * 16 + c;
            acc[a][b] = g.value(row, col, acc[a][b], request(g, row, col));
        }
    // the wave's part of the tile, and its mirror image, each staged in a region of the wave's own and stored by rows
    constexpr int STRIDE = C::WTN * 2 + 16, IMAGE_STRIDE = C::WTM * 2 + 16;
    constexpr int BYTES = C::WTM * STRIDE > C::WTN * IMAGE_STRIDE ? C::WTM * STRIDE : C::WTN * IMAGE_STRIDE;
    static_assert(C::WAVES * BYTES <= C::LDS_BYTES, "fits the operand buffers");
    char* const stage = smem + wave * BYTES;
    auto out = [&](auto rows_tag, auto cols_tag, int r0, int c0) __attribute__((always_inline)) {
        constexpr int ROWS = decltype(rows_tag)::value, COLS = decltype(cols_tag)::value, LPR = COLS / 8, RPP = 64 / LPR, PASSES = ROWS / RPP;
        __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0): the region is private to the wave
        __builtin_amdgcn_wave_barrier();
        u32x4 v[PASSES];
#pragma unroll
        for (int p = 0; p < PASSES; ++p) v[p] = *reinterpret_cast<const u32x4*>(stage + (p * RPP + lane / LPR) * (COLS * 2 + 16) + lane % LPR * 16);
        const int row = r0 + lane / LPR, col = c0 + lane % LPR * 8;
#pragma unroll
        for (int p = 0; p < PASSES; ++p)
            if (row + p * RPP < g.Mo && col < g.No) *reinterpret_cast<u32x4*>(g.C + (int64_t)(row + p * RPP) * g.ldc + col) = v[p];
        __builtin_amdgcn_wave_barrier();  // LDS operations of a wave complete in order: the next pass may overwrite
    };
#pragma unroll
    for (int a = 0; a < C::TM; ++a)
#pragma unroll
        for (int b = 0; b < C::TN; ++b)
            *reinterpret_cast<uint2*>(stage + (a * 16 + r) * STRIDE + (b * 16 + c) * 2) = uint2{pack_f16x2(acc[a][b][0], acc[a][b][1]), pack_f16x2(acc[a][b][2], acc[a][b][3])};
    out(IC<C::WTM>{}, IC<C::WTN>{}, row0, col0);
    if (row0 < j0 + BN) return;  // on the diagonal, or above it
#pragma unroll
    for (int a = 0; a < C::TM; ++a)
#pragma unroll
        for (int b = 0; b < C::TN; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                *reinterpret_cast<_Float16*>(stage + (b * 16 + c + e) * IMAGE_STRIDE + (a * 16 + r) * 2) = (_Float16)acc[a][b][e];
    out(IC<C::WTN>{}, IC<C::WTM>{}, col0, row0);
}

// (Of 32 x 32 tiles: a part leaves its sums by thread.)
__device__ __forceinline__ void OrthoSym::quad(const OrthoSym& g, bool mirrored, int row, int col, f32x4 sum, uint2 raw) {
    if (g.part.cut >= 0) {
        const __amdgpu_buffer_rsrc_t mine = partial_buffer(g.partial + (int64_t)g.part.slot * 1024, 4096);
        return __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, sum), mine, threadIdx.x * 16, 0, DEVICE_SCOPE);
    }
    const f32x4 v = g.value(row, col, sum, raw);
    *reinterpret_cast<uint2*>(g.C + (int64_t)row * g.ldc + col) = uint2{pack_f16x2(v[0], v[1]), pack_f16x2(v[2], v[3])};
    if (!mirrored) return;
#pragma unroll
    for (int e = 0; e < 4; ++e) *reinterpret_cast<_Float16*>(g.C + (int64_t)(col + e) * g.ldc + row) = (_Float16)v[e];
}

// The tile of an index: rows one behind the other, up to the diagonal.
__device__ __forceinline__ void ortho_tile(int t, int& ti, int& tj) {
    ti = (int)((sqrtf(8.0f * (float)t + 1.0f) - 1.0f) * 0.5f);
    while ((ti + 1) * (ti + 2) / 2 <= t) ++ti;
    while (ti * (ti + 1) / 2 > t) --ti;
    tj = t - ti * (ti + 1) / 2;
}
// Tiles of 256 rows and 128 columns: 2 i + 1 of them in the i-th 256 rows, whose last one has the first half of the diagonal; the other half is left to 128 x 128 tiles.
__device__ __forceinline__ void ortho_half_tile(int t, int& ti, int& tj) {
    ti = (int)sqrtf((float)t);
    while ((ti + 1) * (ti + 1) <= t) ++ti;
    while (ti * ti > t) --ti;
    tj = t - ti * ti;
}
// Of the tiles that `cut` deals out (SIZE: rows), `behind`: not the first ones of the launch.
template <int SIZE, int LAYOUT>
__device__ __forceinline__ void ortho_sym(const OrthoSym& args, const SymCut& cut, char* smem, bool behind = false) {
    SymWalk walk(cut, xcd_run(blockIdx.x, gridDim.x), gridDim.x);  // neighbours share rows of tiles
    OrthoSym g = args;
    g.cut = cut;
    for (bool first = !behind; walk.next(cut, g.part); first = false) {
        g.R = g.part.count * TILE_BK;
        const int64_t skip = (int64_t)g.part.from * TILE_BK * (LAYOUT == KC ? 1 : g.lda);
        g.A = args.A + skip;
        g.B = args.B + skip;
        int ti, tj;
        if constexpr (SIZE == SYM_HALF) ortho_half_tile(g.part.tile, ti, tj);
        else if constexpr (SIZE == SYM_DIAGONAL) tj = ti = 2 * g.part.tile + 1;
        else ortho_tile(g.part.tile, ti, tj);
        if (!first) __syncthreads();  // the tile before has left LDS
        if constexpr (SIZE == 64) gemm_ring_body<64, 64, 2, 2, 4, LAYOUT, LAYOUT>(g, ti * 64, tj * 64, smem, threadIdx.x);
        else if constexpr (SIZE == 128 || SIZE == SYM_DIAGONAL) gemm_ring_body<128, 128, 4, 2, 4, LAYOUT, LAYOUT>(g, ti * 128, tj * 128, smem, threadIdx.x);
        else if constexpr (SIZE == SYM_HALF) gemm_ring_body<256, 128, 4, 2, 3, LAYOUT, LAYOUT>(g, ti * 256, tj * 128, smem, threadIdx.x);
        else gemm_tile_body<256, 256, 2, 4, LAYOUT, LAYOUT>(g, ti * 256, tj * 256, smem);
    }
}
// 32 x 32 tiles whose waves split the reduction, for outputs of few tiles.
template <int LAYOUT>
__global__ void __launch_bounds__(SLIM_WAVES * 64) ortho_sym_32_kernel(OrthoSym g) {
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    int ti, tj;
    ortho_tile(xcd_run(blockIdx.x, gridDim.x), ti, tj);
    g.part.cut = -1;
    slim_tile_body<32, 32, SLIM_WAVES, 1, LAYOUT, LAYOUT>(g, ti * 32, tj * 32, threadIdx.x, smem);
}
// The same, a slice of a tile to a workgroup; a quad of the output to a thread.  Two chunks under way to a wave: an X that is not in the L2 is waited for (128 x 65536, five steps, 183 us, with one 196).
// Before there were slices the update of 64 x 4096 took 87 us and takes 56, 128 x 16384 110 and 94, 256 x 4096 104 and 90.
constexpr int SLICED_STAGES = 2;
template <int LAYOUT>
__global__ void __launch_bounds__(SLIM_WAVES * 64) ortho_sym_32_sliced_kernel(OrthoSym args) {
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    static_assert(SLIM_WAVES * 64 * 4 == 32 * 32, "a quad to a thread");
    OrthoSym g = args;
    SymWalk walk(g.cut, xcd_run(blockIdx.x, gridDim.x), gridDim.x);
    if (!walk.next(g.cut, g.part)) return;
    g.R = g.part.count * TILE_BK;
    const int64_t skip = (int64_t)g.part.from * TILE_BK * (LAYOUT == KC ? 1 : g.lda);
    g.A = args.A + skip;
    g.B = args.B + skip;
    int ti, tj;
    ortho_tile(g.part.tile, ti, tj);
    slim_tile_body<32, 32, SLIM_WAVES, SLICED_STAGES, LAYOUT, LAYOUT>(g, ti * 32, tj * 32, threadIdx.x, smem);
    if (g.part.cut < 0) return;  // the only part of its tile
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // as OrthoSym::finish
    __syncthreads();
    uint32_t* const arrived = reinterpret_cast<uint32_t*>(smem);
    if (threadIdx.x == 0) *arrived = __hip_atomic_fetch_add(g.counters + g.part.cut, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (*arrived != (uint32_t)(g.part.parts - 1)) return;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    for (int part = 0; part < g.part.parts; part += 8) {  // eight requested at a time
        f32x4 v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (part + i < g.part.parts)
                v[i] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(partial_buffer(g.partial + (int64_t)g.cut.slot_of(g.part.cut, part + i) * 1024, 4096),
                                                                                       threadIdx.x * 16, 0, DEVICE_SCOPE));
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += v[i];
    }
    if (threadIdx.x == 0) __hip_atomic_store(g.counters + g.part.cut, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    g.part.cut = -1;
    const int row = ti * 32 + (int)threadIdx.x / 8, col = tj * 32 + (int)threadIdx.x % 8 * 4;
    OrthoSym::quad(g, ti != tj, row, col, sum, OrthoSym::request(g, row, col));
}
template <int LAYOUT>
__global__ void __launch_bounds__(256, 2) ortho_sym_64_kernel(OrthoSym g) {
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    ortho_sym<64, LAYOUT>(g, g.cut, smem);
}
template <int LAYOUT>
__global__ void __launch_bounds__(TILE_THREADS, 1) ortho_sym_128_kernel(OrthoSym g) {
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    ortho_sym<128, LAYOUT>(g, g.cut, smem);
}
template <int LAYOUT>
__global__ void __launch_bounds__(TILE_THREADS, 1) ortho_sym_256_kernel(OrthoSym g) {
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    ortho_sym<256, LAYOUT>(g, g.cut, smem);
}
template <int LAYOUT>
__global__ void __launch_bounds__(TILE_THREADS, 1) ortho_sym_half_kernel(OrthoSym g) {
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    ortho_sym<SYM_HALF, LAYOUT>(g, g.cut, smem);
    ortho_sym<SYM_DIAGONAL, LAYOUT>(g, g.diagonal, smem, true);  // (the tiles ahead of them are all taken whole: the sums in the workspace are the diagonal's)
}

// ---- a step in one launch ----------------------------------------------------------------------
// Where s is at most 128 the three products of a step are too small to be worth a launch each: 3 to 4 us apiece, of which the matrix units work a tenth.  A workgroup here
// has a slab of 64 of the l columns (rows, of a tall X) of the next X, and forms the whole of A for itself, as one tile of S x S; A, Q and the slab of X then go through LDS
// only.  Every workgroup does the same l / 64 steps of A, so this is for X of up to ORTHO_STEP_MOST values; to ORTHO_REST_MOST gram is a launch of its own (ortho_rest_kernel).
// Five steps with three launches each, with two and with one: 128 x 512 65 us, 60 and 48; 128 x 2048 78, 73 and 84; 64 x 4096 73 and 56, 128 x 16384 103 and 94, 128 x 32768 110 and 130.
constexpr int ORTHO_STEP_MOST = 128 * 1024, ORTHO_REST_MOST = 128 * 16384;
struct OrthoStep : GemmArgs {
    static constexpr bool F16 = true, OWN = true;
    float alpha;             // of A
    float a, b, c;           // Q = a + b A + c A^2
    bf16_t* O; int64_t ldo;  // as OrthoApply; C: the next X (pitch ldc)
    int K, N;                // O's
    float scale;
    int tall;                // X is R x S

    template <typename C, int BM, int BN>
    static __device__ __forceinline__ void finish(const OrthoStep& g, f32x4 (&acc)[C::TM][C::TN], int, int, const int wm, const int wn, const int tid, char* smem);
};
// An S x S matrix in LDS as KC operands are read: for each 64 columns, S rows of 128 bytes with their chunks permuted.
template <int S>
__device__ __forceinline__ int image_at(int row, int col) {
    return (col >> 6) * (S * 128) + row * 128 + ((((col >> 3) & 7) ^ swz_kc(row)) << 4) + (col & 7) * 2;
}
template <typename C, int S, int S2>
__device__ __forceinline__ void OrthoStep::finish(const OrthoStep& g, f32x4 (&acc)[C::TM][C::TN], int, int, const int wm, const int wn, const int tid, char* smem) {
    static_assert(S == S2 && C::WAVES * 16 == S, "a wave to 16 rows");
    constexpr int IMAGE = S * S * 2, SLAB_CHUNKS = S * 8 / C::THREADS;
    static_assert(2 * IMAGE + S * 128 <= C::LDS_BYTES, "A, Q and the slab in the operand buffers");
    char *const a_image = smem, *const q_image = smem + IMAGE, *const slab = smem + 2 * IMAGE;
    const int lane = tid & 63, wave = tid >> 6, l0 = blockIdx.x * 64;
    // the slab: S rows of 64 columns, or 64 rows of S; its 16-byte chunks on their way into the layout that their product reads
    u32x4 x[SLAB_CHUNKS];
    int x_at[SLAB_CHUNKS];
#pragma unroll
    for (int i = 0; i < SLAB_CHUNKS; ++i) {
        const int q = i * C::THREADS + tid;
        if (g.tall) {
            const int row = q / (S / 8), chunk = q % (S / 8);
            x[i] = *reinterpret_cast<const u32x4*>(g.A + (int64_t)(l0 + row) * g.lda + chunk * 8);
            x_at[i] = image_at<64>(row, chunk * 8);
        } else {
            const int row = q / 8, chunk = q % 8;
            x[i] = *reinterpret_cast<const u32x4*>(g.A + (int64_t)row * g.lda + l0 + chunk * 8);
            x_at[i] = row * 128 + ((chunk ^ swz_mc<64>(row)) << 4);
        }
    }
    const int r = lane & 15, c4 = 4 * (lane >> 4);
    auto put = [&](char* image, int row, int col, f32x4 v) __attribute__((always_inline)) {
        *reinterpret_cast<uint2*>(image + image_at<S>(row, col)) = uint2{pack_f16x2(v[0], v[1]), pack_f16x2(v[2], v[3])};
    };
    __syncthreads();  // all waves are done reading the operand buffers
#pragma unroll
    for (int a = 0; a < C::TM; ++a)
#pragma unroll
        for (int b = 0; b < C::TN; ++b) {
            acc[a][b] = acc[a][b] * g.alpha;
            put(a_image, wm * C::WTM + a * 16 + r, wn * C::WTN + b * 16 + c4, acc[a][b]);
        }
#pragma unroll
    for (int i = 0; i < SLAB_CHUNKS; ++i) *reinterpret_cast<u32x4*>(slab + x_at[i]) = x[i];
    __syncthreads();
    {
        f32x4 sum[C::TM][C::TN];
        FragAddr<S, KC, C::TM> fa;
        FragAddr<S, KC, C::TN> fb;
        fa.init(wm * C::WTM, lane, 0);
        fb.init(wn * C::WTN, lane, 0);
#pragma unroll
        for (int a = 0; a < C::TM; ++a)
#pragma unroll
            for (int b = 0; b < C::TN; ++b) sum[a][b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < S / 64; ++k)
#pragma unroll
            for (int kq = 0; kq < 2; ++kq) {
                bf16x8 av[C::TM], bv[C::TN];
#pragma unroll
                for (int a = 0; a < C::TM; ++a) av[a] = fa.read(a_image, k, a, kq);
#pragma unroll
                for (int b = 0; b < C::TN; ++b) bv[b] = fb.read(a_image, k, b, kq);
#pragma unroll
                for (int a = 0; a < C::TM; ++a)
#pragma unroll
                    for (int b = 0; b < C::TN; ++b) sum[a][b] = mfma_16x16x32<true>(bv[b], av[a], sum[a][b]);
            }
#pragma unroll
        for (int a = 0; a < C::TM; ++a)
#pragma unroll
            for (int b = 0; b < C::TN; ++b) {
                const int row = wm * C::WTM + a * 16 + r, col = wn * C::WTN + b * 16 + c4;
                f32x4 v = sum[a][b] * g.c;
#pragma unroll
                for (int e = 0; e < 4; ++e)  // A as it is held, in fp16
                    v[e] = __builtin_fmaf(g.b, (float)(_Float16)acc[a][b][e], v[e]) + (row == col + e ? g.a : 0.f);
                put(q_image, row, col, v);
            }
    }
    __syncthreads();
    // 16 rows of Q by the slab, or the slab by 16 columns of Q: four tiles of 16 x 16 to a wave
    f32x4 out[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) out[t] = f32x4{0.f, 0.f, 0.f, 0.f};
    FragAddr<S, KC, 1> fq;
    fq.init(wave * 16, lane, 0);
    if (g.tall) {
        FragAddr<64, KC, 4> fx;
        fx.init(0, lane, 0);
#pragma unroll
        for (int k = 0; k < S / 64; ++k)
#pragma unroll
            for (int kq = 0; kq < 2; ++kq) {
                const bf16x8 q = fq.read(q_image, k, 0, kq);
#pragma unroll
                for (int t = 0; t < 4; ++t) out[t] = mfma_16x16x32<true>(q, fx.read(slab, k, t, kq), out[t]);
            }
    } else {
        FragAddr<64, MC, 4> fx;
        fx.init(0, lane, 0);
#pragma unroll
        for (int k = 0; k < S / 64; ++k)
#pragma unroll
            for (int kq = 0; kq < 2; ++kq) {
                const bf16x8 q = fq.read(q_image, k, 0, kq);
#pragma unroll
                for (int t = 0; t < 4; ++t) out[t] = mfma_16x16x32<true>(fx.read(slab, k, t, kq), q, out[t]);
            }
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const int row = g.tall ? l0 + t * 16 + r : wave * 16 + r, col = g.tall ? wave * 16 + c4 : l0 + t * 16 + c4;
        if (!g.O) {
            *reinterpret_cast<uint2*>(g.C + (int64_t)row * g.ldc + col) = uint2{pack_f16x2(out[t][0], out[t][1]), pack_f16x2(out[t][2], out[t][3])};
            continue;
        }
        GemmArgs to;
        to.C = g.O;
        to.ldc = g.ldo;
        if (row < g.K && col < g.N) store_bf16_quad(to, out[t] * g.scale, row, col, min(4, g.N - col));
    }
}
template <int S, int LAYOUT>
__global__ void __launch_bounds__(S * 4, 1) ortho_step_kernel(OrthoStep g) {
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    if constexpr (S == 64) gemm_ring_body<64, 64, 2, 2, 4, LAYOUT, LAYOUT>(g, 0, 0, smem, threadIdx.x);
    else gemm_ring_body<128, 128, 4, 2, 4, LAYOUT, LAYOUT>(g, 0, 0, smem, threadIdx.x);
}

// The same behind a gram launch, where l is longer: a workgroup reads A instead.
template <int S>
__global__ void __launch_bounds__(S * 4, S == 64 ? 2 : 1) ortho_rest_kernel(OrthoStep g, const bf16_t* gram) {
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    using C = std::conditional_t<S == 64, RingCfg<64, 64, 2, 2, 4>, RingCfg<128, 128, 4, 2, 4>>;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave / 2, wn = wave % 2;
    f32x4 acc[C::TM][C::TN];
#pragma unroll
    for (int a = 0; a < C::TM; ++a)
#pragma unroll
        for (int b = 0; b < C::TN; ++b) {
            const uint2 raw = *reinterpret_cast<const uint2*>(gram + (wm * C::WTM + a * 16 + (lane & 15)) * S + wn * C::WTN + b * 16 + 4 * (lane >> 4));
            const f16x2 lo = __builtin_bit_cast(f16x2, raw.x), hi = __builtin_bit_cast(f16x2, raw.y);
            acc[a][b] = f32x4{(float)lo[0], (float)lo[1], (float)hi[0], (float)hi[1]};
        }
    OrthoStep::finish<C, S, S>(g, acc, 0, 0, wm, wn, threadIdx.x, smem);
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
