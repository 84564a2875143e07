// Matrices made orthogonal by Newton-Schulz products: sage_orthogonalize (include/sage.h).
//
// With m <= n (a taller matrix is worked on as its transpose) and X = G / (||G||_F + eps), a step is three products:
//     A = X X^T  (m^2 n multiplications, half of them by symmetry),  P = a I + b A + c A A  (m^3, half),  X <- P X  (m^2 n).
// It is bound by the matrix cores. A step stretches the small singular values by a, 3.4 with the usual coefficients and 485 in
// five steps, and with them whatever rounding has put into their directions: factors of one bf16 or fp16 part (2^-9, 2^-12) would be seen
// in the result. So every entry is kept as the sum of two fp16 parts, hi + lo, and hi hi + hi lo + lo hi are summed in fp32: three
// products on the fp16 matrix cores for one. Two fp16 parts hold 22 bits and more, as fp32 does, where the low part is a normal
// number; entries are bounded by the largest singular value, whose bound U is known on the host (it follows from the
// coefficients), so that scaling by a power of two to 2^14 / U or more leaves entries of 2^-16 U and above that precision and the rest an
// error of 2^-39 U. (bf16 parts would need three of them, six products.)
//
// Matrices of up to 64 x 512 have one work-group each and one launch for all steps (ortho_small_kernel). The others take a launch for
// each product: by tiles of 256 x 256 (only P X, whose tiles are whole), 128 x 128 or 64 x 64, whichever fills the chip (cut_of).
// 4096 x 4096, five steps: 4.05 ms, 1.02 PFLOP/s of the products that symmetry leaves (the library's plain fp16 product of that size: 1.04).
//
// Layout: 32 columns of a row are 128 bytes, their 32 hi parts and then their 32 lo parts; rows and columns are padded with zeros to
// multiples of the tiles' side. X is kept row by row for A and column by column for P X: the instructions take both factors along the
// summed index.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "logit_rows.h"
#include "rows_meet.h"
#include "sage_internal.h"

namespace sage {
namespace {

typedef _Float16 f16;
typedef f16 f16x4 __attribute__((ext_vector_type(4)));
typedef f16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr int KB = 32;  // columns of a block of 128 bytes

// A padded matrix in parts: element (r, k) is p[r * pitch + (k / 32) * 64 + k % 32] + the one 32 further.
struct Parts {
    f16* p;
    int64_t pitch;  // 2 * padded columns
    int64_t batch;  // from one matrix to the next
};

__device__ __forceinline__ void split(float v, f16& hi, f16& lo) {
    hi = (f16)v;
    lo = (f16)(v - (float)hi);
}

__device__ __forceinline__ void split4(const f32x4& v, f16x4& hi, f16x4& lo) {
    hi = __builtin_convertvector(v, f16x4);
    lo = __builtin_convertvector(v - __builtin_convertvector(hi, f32x4), f16x4);
}

// ---- X: the norm, and the matrix in parts both ways -------------------------------------------------------------

constexpr int NORM_THREADS = 256;

// Sums of squares of groups of rows, in fp64: any fp32 matrix has a norm there. Bound by memory.
template <class T>
__global__ __launch_bounds__(NORM_THREADS) void ortho_norm_kernel(const T* __restrict__ G, int64_t rows, int64_t cols, int64_t ld,
                                                                  int64_t stride, double* __restrict__ partial, int groups) {
    constexpr int VL = RowType<T>::VL;
    __shared__ double part[NORM_THREADS / 64];
    const int group = blockIdx.x % groups;
    const int64_t b = blockIdx.x / groups;
    // a wave has a row at a time (short rows would leave most of a work-group without one)
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    double s = 0.0;
    for (int64_t r = (int64_t)group * 4 + wave; r < rows; r += 4 * groups) {
        const T* row = G + b * stride + r * ld;
#pragma unroll 4
        for (int64_t t = lane * VL; t < cols; t += 64 * VL) {
            float x[VL];
            row_floats(row, t, cols, 0.f, x);
#pragma unroll
            for (int i = 0; i < VL; ++i) s = __builtin_fma((double)x[i], (double)x[i], s);
        }
    }
    for (int d = 32; d >= 1; d >>= 1) s += __shfl_xor(s, d, 64);
    if (lane == 0) part[wave] = s;
    __syncthreads();
    if (threadIdx.x == 0) partial[blockIdx.x] = part[0] + part[1] + part[2] + part[3];
}

// 64 x 64 tiles of scale * G / (norm + eps), row by row into R and column by column into Q; what is outside of G is zero.
template <class T>
__global__ __launch_bounds__(256) void ortho_split_kernel(const T* __restrict__ G, int64_t rows, int64_t cols, int64_t ld, int64_t stride,
                                                          const double* __restrict__ partial, int groups, double eps, double scale,
                                                          Parts R, Parts Q, int tiles_r, int tiles_c) {
    __shared__ float tile[64][65];
    __shared__ double part[4];
    const int64_t b = blockIdx.x / (tiles_r * tiles_c);
    const int at = blockIdx.x % (tiles_r * tiles_c);
    const int64_t r0 = (int64_t)(at / tiles_c) * 64, c0 = (int64_t)(at % tiles_c) * 64;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const T* g = G + b * stride;
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int64_t r = r0 + wave + 4 * i, c = c0 + lane;
        x[i] = r < rows && c < cols ? RowType<T>::widen(g[r * ld + c]) : 0.f;
    }
    double s = tid < groups ? partial[b * groups + tid] : 0.0;
    for (int d = 32; d >= 1; d >>= 1) s += __shfl_xor(s, d, 64);
    if (lane == 0) part[wave] = s;
    __syncthreads();
    s = part[0] + part[1] + part[2] + part[3];
    const double inv = s > 0.0 || s != s ? scale / (sqrt(s) + eps) : 0.0;
#pragma unroll
    for (int i = 0; i < 16; ++i) tile[wave + 4 * i][lane] = (float)((double)x[i] * inv);
    __syncthreads();
    // eight entries of a row, then of a column, at a time: 16 bytes of high parts and 16 of low ones
#pragma unroll
    for (int way = 0; way < 2; ++way) {
        const Parts& to = way ? Q : R;
        const int64_t row0 = way ? c0 : r0, col0 = way ? r0 : c0;
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int row = q * 32 + (tid >> 3), col = (tid & 7) * 8;
            f16x8 hi, lo;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                f16 u, v;
                split(way ? tile[col + e][row] : tile[row][col + e], u, v);
                hi[e] = u;
                lo[e] = v;
            }
            f16* p = to.p + b * to.batch + (row0 + row) * to.pitch + (col0 + (col & 32)) * 2 + (col & 31);
            *(f16x8*)p = hi;
            *(f16x8*)(p + 32) = lo;
        }
    }
}

// ---- the products -----------------------------------------------------------------------------------------------

enum { GRAM, POLY, STEP, LAST };

struct Finish {
    float f;      // of the sum
    float fa;     // of A's entry (POLY)
    float diag;   // added on the diagonal (GRAM, POLY)
    Parts A;      // POLY
    Parts C;      // the result, row by row
    Parts Ct;     // STEP: and column by column
    void* out;    // LAST
    int64_t ld_out, stride_out, rows, cols;
    int out16;
};

// Tile t of a lower triangle: row i, column j <= i.
__device__ __forceinline__ void triangle(int t, int& i, int& j) {
    i = (int)((sqrtf(8.f * (float)t + 1.f) - 1.f) * 0.5f);
    while ((int64_t)i * (i + 1) / 2 > t) --i;
    while ((int64_t)(i + 1) * (i + 2) / 2 <= t) ++i;
    j = t - (int)((int64_t)i * (i + 1) / 2);
}

// 32 x 32 entries of a product from row r0 and column c0 on, by one wave: sums as they are (v[g][e]: row 8 g + 4 h + e of column l32, lane
// l32 + 32 h), scaled, and written in the product's form. mirror: the tile is off the diagonal. lds: 4 KB of the wave's own, in which
// the entries are put in the order of memory: whole lines of 128 bytes are stored.
template <int MODE>
__device__ __forceinline__ void finish(const Finish& fin, int64_t b, int64_t r0, int64_t c0, bool mirror, const f32x4* sum, f16* lds) {
    const int lane = threadIdx.x & 63, l32 = lane & 31, h = lane >> 5;
    f32x4 v[4];
#pragma unroll
    for (int g = 0; g < 4; ++g) v[g] = sum[g] * fin.f;
    if constexpr (MODE == LAST) {
        const int64_t c = c0 + l32;
        if (c < fin.cols) {
#pragma unroll
            for (int g = 0; g < 4; ++g)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int64_t r = r0 + 8 * g + 4 * h + e;
                    if (r < fin.rows) {
                        const int64_t o = b * fin.stride_out + r * fin.ld_out + c;
                        if (fin.out16) ((uint16_t*)fin.out)[o] = RowType<uint16_t>::narrow(v[g][e]);
                        else ((float*)fin.out)[o] = v[g][e];
                    }
                }
        }
    } else {
        if constexpr (MODE == POLY) {  // A is symmetric: its entries at (c, r .. r + 3) are next to each other
            const f16* ap = fin.A.p + b * fin.A.batch + (c0 + l32) * fin.A.pitch + r0 * 2 + 4 * h;
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const f16x4 hi = *(const f16x4*)(ap + 8 * g), lo = *(const f16x4*)(ap + 8 * g + 32);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[g][e] = fmaf(fin.fa, (float)hi[e] + (float)lo[e], v[g][e]);
            }
        }
        if constexpr (MODE == GRAM || MODE == POLY) {
            if (r0 == c0) {
#pragma unroll
                for (int g = 0; g < 4; ++g)
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[g][e] += 8 * g + 4 * h + e == l32 ? fin.diag : 0.f;
            }
        }
        f16x4 hi[4], lo[4];
#pragma unroll
        for (int g = 0; g < 4; ++g) split4(v[g], hi[g], lo[g]);
        // 16 bytes of a line at a time; where they lie in LDS is turned by the row, so that rows meet different banks
        auto store = [&](const Parts& to, int64_t row, int64_t col) __attribute__((always_inline)) {
            f16* p = to.p + b * to.batch + (row + (lane >> 3)) * to.pitch + col * 2 + (lane & 7) * 8;
#pragma unroll
            for (int q = 0; q < 4; ++q) *(u32x4*)(p + (int64_t)(8 * q) * to.pitch) = *(const u32x4*)(lds + (8 * q + (lane >> 3)) * 64 + ((lane & 7) ^ (lane >> 3)) * 8);
        };
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int row = 8 * g + 4 * h + e, turn = (4 * h + e) & 7;
                lds[row * 64 + ((l32 >> 3) ^ turn) * 8 + (l32 & 7)] = hi[g][e];
                lds[row * 64 + ((4 + (l32 >> 3)) ^ turn) * 8 + (l32 & 7)] = lo[g][e];
            }
        store(fin.C, r0, c0);
        // the same values the other way round; a diagonal tile has its own mirror image in it
        if (MODE == STEP || mirror) {
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                *(f16x4*)(lds + l32 * 64 + (g ^ (l32 & 7)) * 8 + 4 * h) = hi[g];
                *(f16x4*)(lds + l32 * 64 + ((4 + g) ^ (l32 & 7)) * 8 + 4 * h) = lo[g];
            }
            store(MODE == STEP ? fin.Ct : fin.C, c0, r0);
        }
    }
}

constexpr int wait_for_loads(int left) { return (left & 15) | (left >> 4) << 14 | 0x0F70; }  // until so many are on their way

// The place of a work-group's tile. Work-groups i and i + 8 run on one XCD and share its L2: each XCD gets a run of consecutive tiles, and
// consecutive tiles go down groups of 8 rows of tiles, column by column, so that those at work together use few rows of either
// factor (nothing but the time depends on it).
__device__ __forceinline__ int tile_in_turn(int block, int blocks) {
    const int x = block & 7, each = blocks >> 3, more = blocks & 7;
    return x * each + min(x, more) + (block >> 3);
}
template <bool SYM>
__device__ __forceinline__ void tile_place(int at, int tiles_r, int tiles_c, int& ti, int& tj) {
    if constexpr (SYM) {  // groups of 8 rows of a lower triangle: 8 g columns of 8, then a triangle of 8; 32 g^2 + 4 g before group g
        int g = (int)((sqrtf(128.f * (float)at + 16.f) - 4.f) * (1.f / 64.f));
        while (32 * g * g + 4 * g > at) --g;
        while (32 * (g + 1) * (g + 1) + 4 * (g + 1) <= at) ++g;
        const int in = at - (32 * g * g + 4 * g), rows = min(8, tiles_r - 8 * g);
        if (in < 8 * g * rows) {
            ti = 8 * g + in % rows;
            tj = in / rows;
        } else {
            triangle(in - 8 * g * rows, ti, tj);
            ti += 8 * g;
            tj += 8 * g;
        }
    } else {
        const int g = at / (8 * tiles_c), in = at - g * 8 * tiles_c, rows = min(8, tiles_r - 8 * g);
        ti = 8 * g + in % rows;
        tj = in / rows;
    }
}

// C = A B^T of padded matrices in parts, both along the summed index: tiles of 32 WR RB x 32 WC CB, WR x WC waves with RB x CB
// instruction tiles of 32 x 32 each. Blocks of 32 of the summed index go straight to LDS, NST - 1 on their way while one is multiplied; a row's
// eight pieces of 16 bytes are stored in an order turned by the row's number, so that the reads of eight rows meet
// different banks. (The loads deposit in lane order: it is their addresses that are turned.) splits > 1: as
// many work-groups have a tile, each a part of the summed index, and leave their sums to
// ortho_join_kernel.
template <int WR, int WC, int RB, int CB, int NST, int MODE>
__global__ __launch_bounds__(WR * WC * 64) void ortho_product_kernel(Parts A, Parts B, int kblocks, int tiles_r, int tiles_c, Finish fin,
                                                                               int tile0, int splits, f32x4* __restrict__ partial) {
    constexpr int TM = 32 * WR * RB, TN = 32 * WC * CB, THREADS = WR * WC * 64;
    constexpr int STAGE = (TM + TN) * 8;  // pieces of 16 bytes
    constexpr int LOADS = STAGE / THREADS;
    static_assert(STAGE % THREADS == 0 && TM * 8 % THREADS == 0, "whole loads");
    static_assert(LOADS * (NST - 1) < 64, "a wait counts up to 63");
    extern __shared__ u32x4 lds[];  // NST * STAGE
    constexpr bool SYM = MODE == GRAM || MODE == POLY;
    const int per = SYM ? tiles_r * (tiles_r + 1) / 2 : tiles_r * tiles_c;
    constexpr bool SPLIT = RB == 2;
    const int unit = tile_in_turn(blockIdx.x, gridDim.x);
    const int tile = tile0 + (SPLIT ? unit / splits : unit), part = SPLIT ? unit % splits : 0;
    const int64_t b = tile / per;
    const int at = tile % per;
    const int first = SPLIT ? kblocks * part / splits : 0;
    if (SPLIT) kblocks = kblocks * (part + 1) / splits - first;
    int ti, tj;
    tile_place<SYM>(at, tiles_r, tiles_c, ti, tj);
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, h = lane >> 5;
    const int wr = wave / WC, wc = wave % WC;

    // (a thread's pieces are in rows THREADS / 8 apart: one offset for each factor, the rest is the same for all threads)
    static_assert(THREADS % 64 == 0, "whole turns of 8 rows");
    const int turned = ((tid & 7) ^ (tid >> 3 & 7)) * 8;
    const uint32_t aoff = (uint32_t)((tid >> 3) * A.pitch) + turned, boff = (uint32_t)((tid >> 3) * B.pitch) + turned;
    const f16* abase = A.p + b * A.batch + (int64_t)ti * TM * A.pitch + (int64_t)first * 64;
    const f16* bbase = B.p + b * B.batch + (int64_t)tj * TN * B.pitch + (int64_t)first * 64;
    auto stage = [&](int kb, int buf) __attribute__((always_inline)) {
#pragma unroll
        for (int q = 0; q < LOADS; ++q) {
            const int row = q * (THREADS / 8);
            const f16* from = row < TM ? abase + (int64_t)row * A.pitch + (int64_t)kb * 64 : bbase + (int64_t)(row - TM) * B.pitch + (int64_t)kb * 64;
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(from + (row < TM ? aoff : boff)),
                                             (__attribute__((address_space(3))) void*)(lds + buf * STAGE + q * THREADS + wave * 64), 16, 0, 0);
        }
    };

    f32x16 acc[RB][CB];
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int j = 0; j < CB; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

    // Factors of half a block: 16 of the summed index
    struct Factors {
        f16x8 a[RB][2], c[CB][2];
    };
    const int arow = wr * 32 * RB + l32, brow = TM + wc * 32 * CB + l32;
    auto read = [&](Factors& f, int buf, int s) __attribute__((always_inline)) {
        const u32x4* st = lds + buf * STAGE;
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const int piece = (4 * p + 2 * s + h) ^ (l32 & 7);
#pragma unroll
            for (int i = 0; i < RB; ++i) f.a[i][p] = __builtin_bit_cast(f16x8, st[(arow + 32 * i) * 8 + piece]);
#pragma unroll
            for (int j = 0; j < CB; ++j) f.c[j][p] = __builtin_bit_cast(f16x8, st[(brow + 32 * j) * 8 + piece]);
        }
        __builtin_amdgcn_sched_barrier(0);  // (the scheduler would put each read next to its use, which then waits for it)
    };
    auto multiply = [&](const Factors& f) __attribute__((always_inline)) {
        constexpr int PA[3] = {1, 0, 0}, PC[3] = {0, 1, 0};
#pragma unroll
        for (int p = 0; p < 3; ++p)
#pragma unroll
            for (int i = 0; i < RB; ++i)
#pragma unroll
                for (int j = 0; j < CB; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f.a[i][PA[p]], f.c[j][PC[p]], acc[i][j], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
    };
    // NST blocks are on their way before the first is used. (Beyond the end the last block is loaded again and not used, so that every turn
    // waits for the same number of loads.)
#pragma unroll
    for (int i = 0; i < NST; ++i) stage(min(i, kblocks - 1), i);
    auto meet = [&](auto wait) __attribute__((always_inline)) {  // the next block has landed; everyone has read the one before it
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(decltype(wait)::value);
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    Factors f0, f1;
    meet(std::integral_constant<int, wait_for_loads(LOADS * (NST - 1))>{});
    read(f0, 0, 0);
    int buf = 0;
    for (int kb = 0; kb < kblocks; ++kb) {
        read(f1, buf, 1);
        multiply(f0);
        meet(std::integral_constant<int, wait_for_loads(LOADS * (NST - 2)) & ~0x0F00>{});  // (and nothing of this block is still being read from LDS)
        stage(min(kb + NST, kblocks - 1), buf);
        buf = buf == NST - 1 ? 0 : buf + 1;
        read(f0, buf, 0);
        multiply(f1);
    }
    __builtin_amdgcn_s_waitcnt(wait_for_loads(0));  // nothing on its way to LDS when the work-group ends or uses LDS otherwise
    if (SPLIT && splits > 1) {
        // the sums of this part of the summed index, in the threads' own order
        f32x4* to = partial + ((int64_t)unit * RB * CB * 4) * THREADS + tid;
#pragma unroll
        for (int i = 0; i < RB; ++i)
#pragma unroll
            for (int j = 0; j < CB; ++j)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    to[((i * CB + j) * 4 + g) * THREADS] = f32x4{acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
        return;
    }
    if constexpr (MODE != LAST) __syncthreads();  // the rings are free
#pragma unroll
    for (int i = 0; i < RB; ++i)
#pragma unroll
        for (int j = 0; j < CB; ++j) {
            f32x4 v[4];
#pragma unroll
            for (int g = 0; g < 4; ++g) v[g] = f32x4{acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
            finish<MODE>(fin, b, (int64_t)ti * TM + (wr * RB + i) * 32, (int64_t)tj * TN + (wc * CB + j) * 32, ti != tj, v,
                         (f16*)lds + wave * 2048);
        }
}

// The same for few tiles: 64 x 64, all of it by each of four waves, which take the blocks of the summed index in turn and add up what
// they have in the end. A wave has its own ring of two blocks and waits for nobody. Bound by LDS: four blocks are 64 KB written there (450 ns
// from an L2) and 64 KB read (390 ns) for matrix instructions of 390 ns; a turn takes 1.0 us. (With a quarter of the tile each, four waves
// read twice as much for a block: X X' of 1000 x 2049 in 21 us instead of 17, P in 14 instead of 12.)
template <int MODE>
__global__ __launch_bounds__(256) void ortho_wave_kernel(Parts A, Parts B, int kblocks, int tiles_r, int tiles_c, Finish fin) {
    constexpr int STAGE = 128 * 8, LOADS = 16, KS = 4;
    extern __shared__ u32x4 lds[];  // KS * 2 * STAGE
    constexpr bool SYM = MODE == GRAM || MODE == POLY;
    const int per = SYM ? tiles_r * (tiles_r + 1) / 2 : tiles_r * tiles_c;
    const int tile = tile_in_turn(blockIdx.x, gridDim.x), at = tile % per;
    const int64_t b = tile / per;
    int ti, tj;
    tile_place<SYM>(at, tiles_r, tiles_c, ti, tj);
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l32 = lane & 31, h = lane >> 5;
    u32x4* const ring = lds + wave * 2 * STAGE;
    const f16* abase = A.p + b * A.batch + (int64_t)ti * 64 * A.pitch;
    const f16* bbase = B.p + b * B.batch + (int64_t)tj * 64 * B.pitch;
    const int turned = ((lane & 7) ^ (lane >> 3)) * 8;
    const uint32_t aoff = (uint32_t)((lane >> 3) * A.pitch) + turned, boff = (uint32_t)((lane >> 3) * B.pitch) + turned;
    auto stage = [&](int kb, int buf) __attribute__((always_inline)) {
        const int64_t at_k = (int64_t)min(kb, kblocks - 1) * 64;  // (beyond the end the last block again, not used)
#pragma unroll
        for (int q = 0; q < LOADS; ++q) {
            const f16* from = q < 8 ? abase + (int64_t)(q * 8) * A.pitch + at_k : bbase + (int64_t)(q * 8 - 64) * B.pitch + at_k;
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(from + (q < 8 ? aoff : boff)),
                                             (__attribute__((address_space(3))) void*)(ring + buf * STAGE + q * 64), 16, 0, 0);
        }
    };
    f32x16 acc[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
    struct Factors {
        f16x8 a[2][2], c[2][2];
    };
    auto read = [&](Factors& f, int buf, int s) __attribute__((always_inline)) {
        const u32x4* st = ring + buf * STAGE + l32 * 8;
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            const int piece = (4 * p + 2 * s + h) ^ (l32 & 7);
#pragma unroll
            for (int i = 0; i < 2; ++i) f.a[i][p] = __builtin_bit_cast(f16x8, st[32 * i * 8 + piece]);
#pragma unroll
            for (int j = 0; j < 2; ++j) f.c[j][p] = __builtin_bit_cast(f16x8, st[(64 + 32 * j) * 8 + piece]);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    auto multiply = [&](const Factors& f) __attribute__((always_inline)) {
        constexpr int PA[3] = {1, 0, 0}, PC[3] = {0, 1, 0};
#pragma unroll
        for (int p = 0; p < 3; ++p)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f.a[i][PA[p]], f.c[j][PC[p]], acc[i][j], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
    };
    auto wait = [&](auto imm) __attribute__((always_inline)) {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(decltype(imm)::value);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    using std::integral_constant;
    Factors f0, f1;
    stage(wave, 0);
    stage(wave + KS, 1);
    wait(integral_constant<int, wait_for_loads(LOADS)>{});
    read(f0, 0, 0);
    int buf = 0;
    for (int kb = wave; kb < kblocks; kb += KS) {
        read(f1, buf, 1);
        multiply(f0);
        wait(integral_constant<int, wait_for_loads(63) & ~0x0F00>{});  // this block has been read from LDS
        stage(kb + 2 * KS, buf);
        wait(integral_constant<int, wait_for_loads(LOADS)>{});  // the next one is there
        buf ^= 1;
        read(f0, buf, 0);
        multiply(f1);
    }
    wait(integral_constant<int, wait_for_loads(0) & ~0x0F00>{});  // nothing on its way to or from LDS
    __syncthreads();
    f32x4* sums = (f32x4*)lds;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                sums[((wave * 4 + 2 * i + j) * 4 + g) * 64 + lane] = f32x4{acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
    __syncthreads();
    const int i = wave >> 1, j = wave & 1;
    f32x4 v[4];
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        v[g] = sums[(wave * 4 + g) * 64 + lane];
#pragma unroll
        for (int q = 1; q < KS; ++q) v[g] += sums[((q * 4 + wave) * 4 + g) * 64 + lane];
    }
    finish<MODE>(fin, b, (int64_t)ti * 64 + i * 32, (int64_t)tj * 64 + j * 32, ti != tj, v, (f16*)(lds + 4096) + wave * 2048);
}

// The sums of the parts added up, in their order, and finished: a wave has one of the RB x CB blocks of one of theirs.
template <int WR, int WC, int RB, int CB, int MODE>
__global__ __launch_bounds__(64) void ortho_join_kernel(const f32x4* __restrict__ partial, int tile0, int splits, int tiles_r, int tiles_c, Finish fin) {
    constexpr int TM = 32 * WR * RB, TN = 32 * WC * CB, WAVES = WR * WC, BLOCKS = RB * CB;
    constexpr bool SYM = MODE == GRAM || MODE == POLY;
    __shared__ u32x4 turn[256];
    const int per = SYM ? tiles_r * (tiles_r + 1) / 2 : tiles_r * tiles_c;
    const int wave = blockIdx.x % WAVES, block = blockIdx.x / WAVES % BLOCKS, mine = blockIdx.x / WAVES / BLOCKS;
    const int tile = tile0 + mine, at = tile % per;
    const int64_t b = tile / per;
    int ti, tj;
    tile_place<SYM>(at, tiles_r, tiles_c, ti, tj);
    const int wr = wave / WC, wc = wave % WC, i = block / CB, j = block % CB;
    const f32x4* from = partial + ((int64_t)mine * splits * BLOCKS * 4 + block * 4) * (WAVES * 64) + wave * 64 + threadIdx.x;
    f32x4 v[4];
#pragma unroll
    for (int g = 0; g < 4; ++g) v[g] = from[g * (WAVES * 64)];
#pragma unroll 4
    for (int q = 1; q < splits; ++q)
#pragma unroll
        for (int g = 0; g < 4; ++g) v[g] += from[((int64_t)q * BLOCKS * 4 + g) * (WAVES * 64)];
    finish<MODE>(fin, b, (int64_t)ti * TM + (wr * RB + i) * 32, (int64_t)tj * TN + (wc * CB + j) * 32, ti != tj, v, (f16*)turn);
}

// ---- small matrices ---------------------------------------------------------------------------------------------

// (64 x 256, five steps: 35 us, 95 with a launch for each product; a step takes 5: 2.2 of matrix instructions, the rest is three
// meetings of the work-group and what each wave does between them on its own; 43 us with 64 columns a wave, which is what more than 256
// columns take: 70 for 64 x 512. Longer rows do not fit in registers.)
constexpr int SMALL_M = 64, SMALL_N = 512, MAX_STEPS = 32;

// What the steps of a call need, for any matrix of it.
struct Steps {
    int count;
    double eps, sx;  // X is kept as sx * X at first
    struct {
        float gram;        // X X^T as it is summed -> A, or straight to P where there is no A A
        float square, linear, diag;  // A A, A and 1 -> P
        float step;        // P X -> the next X, or the result
        int cubic;
    } at[MAX_STEPS];
};

// Up to 64 x 512 (m <= n), all steps by one work-group, which keeps X in registers: each wave has CW blocks of 32 columns of it, once with a lane for a
// row (as X X^T takes it) and once with a lane for a column (as P X takes it). The instruction leaves a lane with four consecutive
// entries along the other side, and two halves of a wave swap registers to make eight of them: P X is formed both ways, X P' and P X, in
// place of a transposition through LDS. A is summed over the waves in LDS.
template <class T, int CW>
__global__ __launch_bounds__(512) void ortho_small_kernel(const T* G, int rows, int cols, int64_t ld, int64_t stride, T* out, int64_t ld_out,
                                                          int64_t stride_out, Steps p) {
    extern __shared__ u32x4 lds[];
    __shared__ double norms[8];
    const int W = blockDim.x >> 6, tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l32 = lane & 31, h = lane >> 5;
    const bool tall = rows > cols;
    const int m = tall ? cols : rows, n = tall ? rows : cols;
    constexpr int XN = 32 * CW;  // columns of a wave, and loads of a lane
    const int c0 = wave * XN, used = (n + XN - 1) / XN;  // waves behind the last column only help with A and P
    const bool mine = wave < used;

    // the wave's 64 rows of XN entries, coalesced; scaled and split they go through LDS to the lanes that have them as factors
    const T* g = G + (int64_t)blockIdx.x * stride;
    float x[XN];
    auto place = [&](int i, int& r, int& c) __attribute__((always_inline)) {
        r = tall ? lane : CW == 2 ? i : 2 * i + h;
        c = tall ? i : CW == 2 ? lane : l32;
    };
#pragma unroll
    for (int i = 0; i < XN; ++i) {
        int r, c;
        place(i, r, c);
        c += c0;
        x[i] = r < m && c < n ? RowType<T>::widen(tall ? g[(int64_t)c * ld + r] : g[(int64_t)r * ld + c]) : 0.f;
    }
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < XN; ++i) s = __builtin_fma((double)x[i], (double)x[i], s);
    for (int d = 32; d >= 1; d >>= 1) s += __shfl_xor(s, d, 64);
    if (lane == 0) norms[wave] = s;
    __syncthreads();
    s = norms[0];
    for (int w = 1; w < used; ++w) s += norms[w];
    // x * inv in fp32, of which inv may be out of range: a power of two first
    const double inv = s > 0.0 || s != s ? p.sx / (sqrt(s) + p.eps) : 0.0;
    const int power = ilogb(inv == 0.0 ? 1.0 : inv);
    const float rest = (float)ldexp(inv, -power);
    uint32_t* xs = (uint32_t*)lds + wave * (64 * (XN + 1));
#pragma unroll
    for (int i = 0; i < XN; ++i) {
        int r, c;
        place(i, r, c);
        f16 hi, lo;
        split(ldexpf(x[i], power) * rest, hi, lo);
        xs[r * (XN + 1) + c] = (uint32_t)__builtin_bit_cast(uint16_t, hi) | (uint32_t)__builtin_bit_cast(uint16_t, lo) << 16;
    }
    auto gather = [&](f16x8* to, int r, int c, int down) __attribute__((always_inline)) {  // eight entries from (r, c) on, along a row or down a column
        u32x4 hi, lo;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            uint32_t u[2];
#pragma unroll
            for (int q = 0; q < 2; ++q) u[q] = xs[(r + (down ? 2 * e + q : 0)) * (XN + 1) + c + (down ? 0 : 2 * e + q)];
            hi[e] = (u[0] & 0xFFFFu) | u[1] << 16;
            lo[e] = u[0] >> 16 | (u[1] & 0xFFFF0000u);
        }
        to[0] = __builtin_bit_cast(f16x8, hi);
        to[1] = __builtin_bit_cast(f16x8, lo);
    };
    f16x8 by_row[2][2 * CW][2], by_col[CW][4][2];  // [32 rows or columns][16 of the others][high, low]
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int k = 0; k < 2 * CW; ++k) gather(by_row[i][k], 32 * i + l32, 16 * k + 8 * h, 0);
#pragma unroll
    for (int j = 0; j < CW; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k) gather(by_col[j][k], 16 * k + 8 * h, 32 * j + l32, 1);
    __syncthreads();

    f32x4* const sums = (f32x4*)lds;               // per wave three blocks of 32 x 32 of X X^T: (0, 0), (1, 0), (1, 1)
    f16* const A = (f16*)(lds + W * 768);          // 64 rows of two blocks of 128 bytes, pieces turned by the row
    f16* const P = A + 64 * 128;
    auto at_part = [&](int r, int c) __attribute__((always_inline)) { return r * 128 + (c >> 5) * 64 + (((c & 31) >> 3 ^ (r & 7)) << 3) + (c & 7); };
    // (the low part is four pieces further, before the turn: one bit of the piece's number)
    auto put = [&](f16* to, int r, int c, const f32x4& v) __attribute__((always_inline)) {  // rows r .. r + 3 of column c, and the mirror image
        f16x4 hi, lo;
        split4(v, hi, lo);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            to[at_part(r + e, c)] = hi[e];
            to[at_part(r + e, c) ^ 32] = lo[e];
        }
        if (r >> 5 != c >> 5) {
            *(f16x4*)(to + at_part(c, r)) = hi;
            *(f16x4*)(to + (at_part(c, r) ^ 32)) = lo;
        }
    };
    auto part = [&](const f16* from, int block, int k, int which) __attribute__((always_inline)) {  // a lane's factor: row 32 block + l32, 16 k + 8 h ..
        return *(const f16x8*)(from + (at_part(32 * block + l32, 16 * k + 8 * h) ^ which * 32));
    };
    // the three products of two parts each, several sums in turn: none waits for its own last
    auto low_high = [&](f32x16& acc, const f16x8* a, const f16x8* b) __attribute__((always_inline)) { acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[1], b[0], acc, 0, 0, 0); };
    auto high_low = [&](f32x16& acc, const f16x8* a, const f16x8* b) __attribute__((always_inline)) { acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[0], b[1], acc, 0, 0, 0); };
    auto high_high = [&](f32x16& acc, const f16x8* a, const f16x8* b) __attribute__((always_inline)) { acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[0], b[0], acc, 0, 0, 0); };
    // entries v[4 g + e] (8 g + 4 h + e along one side, l32 along the other), scaled, as factors of the next products
    auto refill = [&](f16x8 (*to)[2], const f32x16& v, float f) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            f16x4 parts[2][2];
#pragma unroll
            for (int q = 0; q < 2; ++q)
                split4(f32x4{v[8 * k + 4 * q], v[8 * k + 4 * q + 1], v[8 * k + 4 * q + 2], v[8 * k + 4 * q + 3]} * f, parts[0][q], parts[1][q]);
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
                const u32x2 x = __builtin_bit_cast(u32x2, parts[w][0]), y = __builtin_bit_cast(u32x2, parts[w][1]);
                const auto u0 = __builtin_amdgcn_permlane32_swap(x[0], y[0], false, false);
                const auto u1 = __builtin_amdgcn_permlane32_swap(x[1], y[1], false, false);
                to[k][w] = __builtin_bit_cast(f16x8, u32x4{u0[0], u1[0], u0[1], u1[1]});
            }
        }
    };
    const f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};

#pragma unroll 1
    for (int step = 0; step < p.count; ++step) {
        const auto q = p.at[step];
        if (mine) {
            f32x16 acc[3] = {zero, zero, zero};
#pragma unroll
            for (int k = 0; k < 2 * CW; ++k) {
                const auto three = [&](auto one) __attribute__((always_inline)) {
                    one(acc[0], by_row[0][k], by_row[0][k]);
                    one(acc[1], by_row[1][k], by_row[0][k]);
                    one(acc[2], by_row[1][k], by_row[1][k]);
                };
                three(low_high);
                three(high_low);
                three(high_high);
            }
#pragma unroll
            for (int b = 0; b < 3; ++b)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    sums[wave * 768 + (b * 4 + j) * 64 + lane] = f32x4{acc[b][4 * j], acc[b][4 * j + 1], acc[b][4 * j + 2], acc[b][4 * j + 3]};
        }
        __syncthreads();
        for (int i = wave; i < 12; i += W) {
            const int b = i >> 2, j = i & 3, r = (b ? 32 : 0) + 8 * j + 4 * h, c = (b == 2 ? 32 : 0) + l32;
            f32x4 v = sums[i * 64 + lane];
            for (int w = 1; w < used; ++w) v += sums[w * 768 + i * 64 + lane];
            v *= q.gram;
            if (!q.cubic) {
                put(A, r, c, v);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] += r + e == c ? q.diag : 0.f;
                put(P, r, c, v);
            }
        }
        __syncthreads();
        if (!q.cubic) {
            for (int b = wave; b < 3; b += W) {
                f32x16 acc = zero;
                const int rb = b ? 1 : 0, cb = b == 2 ? 1 : 0;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const f16x8 x[2] = {part(A, rb, k, 0), part(A, rb, k, 1)}, y[2] = {part(A, cb, k, 0), part(A, cb, k, 1)};
                    low_high(acc, x, y);
                    high_low(acc, x, y);
                    high_high(acc, x, y);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int r = 32 * rb + 8 * j + 4 * h, c = 32 * cb + l32;
                    const f16x4 hi = *(const f16x4*)(A + at_part(c, r)), lo = *(const f16x4*)(A + (at_part(c, r) ^ 32));
                    f32x4 v;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        v[e] = acc[4 * j + e] * q.square + ((float)hi[e] + (float)lo[e]) * q.linear + (r + e == c ? q.diag : 0.f);
                    put(P, r, c, v);
                }
            }
            __syncthreads();
        }
        const bool last = step + 1 == p.count;
        T* const to = out + (int64_t)blockIdx.x * stride_out;
        if (!mine) continue;
#pragma unroll
        for (int j = 0; j < CW; ++j) {  // 32 columns
            f32x16 down[2] = {zero, zero}, along[2] = {zero, zero};  // P X: a lane has a column; X' P: a lane has a row
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                f16x8 x[2][2];
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int w = 0; w < 2; ++w) x[i][w] = part(P, i, k, w);
                const auto four = [&](auto one, auto other) __attribute__((always_inline)) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        one(down[i], x[i], by_col[j][k]);
                        other(along[i], by_col[j][k], x[i]);
                    }
                };
                four(low_high, high_low);
                four(high_low, low_high);
                four(high_high, high_high);
            }
            if (!last) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    refill(&by_row[i][2 * j], along[i], q.step);
                    refill(&by_col[j][2 * i], down[i], q.step);
                }
            } else {
                // (the form in which a row of the result goes to consecutive lanes)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int c = tall ? 32 * i + l32 : c0 + 32 * j + l32;
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int r = (tall ? c0 + 32 * j : 32 * i) + 8 * (e >> 2) + 4 * h + (e & 3);
                        if (r < rows && c < cols) to[(int64_t)r * ld_out + c] = RowType<T>::narrow((tall ? along[i][e] : down[i][e]) * q.step);
                    }
                }
            }
            // (both at once would need more registers than there are, and P's factors are read again rather than kept)
            __builtin_amdgcn_sched_barrier(0);
            asm volatile("" ::: "memory");
        }
    }
}

// ---- the plan ---------------------------------------------------------------------------------------------------

constexpr int MAX_SIDE = 32768;
// batches are taken in chunks that need no more than 1 GB in all, or one matrix at a time
constexpr int64_t WORK_LIMIT = (1ll << 30) - 512 * 128 * 128 * 4;

template <int MODE>
int64_t tiles_of(int64_t rows, int64_t cols, int64_t side) {
    const int64_t r = rows / side;
    return MODE == GRAM || MODE == POLY ? r * (r + 1) / 2 : r * (cols / side);
}

struct Plan {
    int64_t m, n, M, N;  // the sides, smaller first, and padded
    bool small;          // one work-group each, without work space
    bool huge;           // tiles of 256 x 256
    bool big;            // tiles of 128 x 128, else 64 x 64
    int groups;          // of rows, for the norm
    int64_t x, a;        // halves of X (either way) and of A
    int64_t per;         // bytes of one matrix
    int64_t chunk;       // matrices at a time
    int64_t bytes;       // of the work space
};

int64_t padded(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
int64_t align256(int64_t v) { return (v + 255) / 256 * 256; }

// Tiles of 128 x 128 of X from which on its sides are padded to them (fewer leave most CUs idle, and the padding costs: with 60 and 200 the
// sizes in between take the same time within 3%), and of 256 x 256 for P X, which keep 256 CUs busy once (4096 x 4096: 385 us in tiles of 128,
// 341 so; fewer leave CUs idle, for a tile takes its 341 us alone as well).
constexpr int64_t BIG_FROM = 100;
constexpr int64_t HUGE_FROM = 224;
constexpr int64_t SLOTS = 512;        // work-groups of 128 x 128 at a time, two to a CU
constexpr int SPLIT_BLOCKS = 8;       // blocks of the summed index in a part of it, at least
constexpr int64_t JOIN_BYTES = SLOTS * 128 * 128 * 4;

Plan plan_of(int64_t batch, int64_t rows, int64_t cols) {
    Plan p;
    p.m = std::min(rows, cols);
    p.n = std::max(rows, cols);
    p.small = p.m <= SMALL_M && p.n <= SMALL_N;
    const int64_t tiles = (p.m + 127) / 128 * ((p.n + 127) / 128) * batch;
    p.big = p.m > 64 && tiles >= BIG_FROM;  // (a side of up to 64 would be padded to twice that and more)
    p.huge = p.m > 192 && (p.m + 255) / 256 * ((p.n + 255) / 256) * batch >= HUGE_FROM;
    const int side = p.huge ? 256 : p.big ? 128 : 64;
    p.M = padded(p.m, side);
    p.N = padded(p.n, side);
    p.groups = (int)std::min<int64_t>((rows + 3) / 4, std::max<int64_t>(1, std::min<int64_t>(256, rows * cols / 4096)));
    p.x = 2 * p.M * p.N;
    p.a = 2 * p.M * p.M;
    p.per = (3 * p.x + 2 * p.a) * 2 + align256(8 * p.groups);
    p.chunk = std::max<int64_t>(1, std::min(batch, WORK_LIMIT / p.per));
    p.bytes = p.per * p.chunk + (p.big ? JOIN_BYTES : 0);
    if (p.small) {
        p.chunk = std::min<int64_t>(batch, 1 << 20);  // (a launch has fewer than 2^32 threads)
        p.bytes = 256;  // (nothing of it is used)
    }
    return p;
}

// max |a s + b s^3 + c s^5| (odd) or max |a + b l + c l^2| over [0, top]: at the ends or where the derivative vanishes
double bound_of(double a, double b, double c, double top, bool odd) {
    auto at = [&](double l) { return fabs((odd ? sqrt(l) : 1.0) * (a + l * (b + l * c))); };  // l = s^2
    const double end = odd ? top * top : top;
    double r = std::max(at(0.0), at(end));
    // roots in l of a + 3 b l + 5 c l^2, or of b + 2 c l
    const double A = odd ? 5 * c : 0.0, B = odd ? 3 * b : 2 * c, C = odd ? a : b;
    double root[2] = {-1.0, -1.0};
    if (A != 0.0) {
        const double d = B * B - 4 * A * C;
        if (d >= 0.0) {  // (the root that is a difference of nearly equal numbers, where A is small, is C over the other's numerator)
            const double q = -0.5 * (B + copysign(sqrt(d), B));
            root[0] = q / A;
            if (q != 0.0) root[1] = C / q;
        }
    } else if (B != 0.0) {
        root[0] = -C / B;
    }
    for (double l : root)
        if (l > 0.0 && l < end) r = std::max(r, at(l));
    return r;
}

// the power of two that takes values up to `top` to 2^14 .. 2^15
double scale_for(double top) {
    int e;
    frexp(std::max(top, 0x1p-12), &e);
    return ldexp(1.0, 15 - e);
}

// How a product is cut. Estimates in microseconds, from products of 128 x 1024 (48 of them) to 4096 x 4096: a work-group of
// ortho_wave_kernel, one to a CU, takes 1.0 for four blocks of the summed index and 3 for the rest of a tile of 64 x 64; a tile of
// 128 x 128 takes 1.0 a block when it has a CU to itself, two on one take 1.6, and 4 for the rest. Tiles that are left over when the slots
// have been filled as often as possible may be cut along the summed index, so that they fill them too: joining them takes a launch of
// 6 and 0.03 a part (64 KB written and read). 528 tiles of a 4096 x 4096 product: 275 us as they are, 220 so (512 whole ones
// and 16 in 16 parts); 48 products X X' of 128 x 1024: 18 in tiles of 128, 11 in tiles of 64.
struct Cut {
    bool waves;  // ortho_wave_kernel
    int splits;  // of the tiles that are left over
};

Cut cut_of(int64_t tiles64, int64_t tiles128, int64_t blocks) {
    const double waves = (double)((tiles64 + 255) / 256) * ((double)((blocks + 3) / 4) + 3.0);
    const int64_t rest = tiles128 % SLOTS;
    const double whole = (double)(tiles128 / SLOTS) * (1.6 * (double)blocks + 4.0);
    Cut best{true, 1};
    double least = waves;
    for (int64_t s = 1; s <= (rest ? std::max<int64_t>(1, std::min<int64_t>(SLOTS / rest, blocks / SPLIT_BLOCKS)) : 1); ++s) {
        double t = whole;
        if (rest) t += (rest * s <= SLOTS / 2 ? 1.0 : 1.6) * (double)((blocks + s - 1) / s) + 4.0 + (s > 1 ? 6.0 + 0.03 * (double)(rest * s) : 0.0);
        if (t < least) {
            least = t;
            best = Cut{false, (int)s};
        }
    }
    return best;
}

template <int MODE, int WC, int RB, int NST>
hipError_t product_of(const Parts& A, const Parts& B, int64_t rows, int64_t cols, int64_t k, int64_t batch, const Finish& fin, int64_t slots, int splits,
                      f32x4* partial, hipStream_t st) {
    constexpr int WR = 2, CB = 2, THREADS = WR * WC * 64;
    constexpr int TM = 32 * WR * RB, TN = 32 * WC * CB, BYTES = NST * (TM + TN) * 128;
    const auto kernel = ortho_product_kernel<WR, WC, RB, CB, NST, MODE>;
    if (hipError_t e = ensure_dynamic_lds((const void*)kernel, BYTES); e != hipSuccess) return e;
    const int tr = (int)(rows / TM), tc = (int)(cols / TN), kb = (int)(k / KB);
    const int64_t tiles = tiles_of<MODE>(rows, cols, TM) * batch, rest = tiles % slots;
    const int64_t whole = splits > 1 ? tiles - rest : tiles;
    if (whole) {
        kernel<<<dim3((unsigned)whole), THREADS, BYTES, st>>>(A, B, kb, tr, tc, fin, 0, 1, nullptr);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    if constexpr (RB == 2) {
        if (splits > 1) {
            kernel<<<dim3((unsigned)(rest * splits)), THREADS, BYTES, st>>>(A, B, kb, tr, tc, fin, (int)whole, splits, partial);
            if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
            ortho_join_kernel<WR, WC, RB, CB, MODE>
                <<<dim3((unsigned)(rest * RB * CB * WR * WC)), 64, 0, st>>>(partial, (int)whole, splits, tr, tc, fin);
        }
    }
    return hipGetLastError();
}

template <int MODE>
hipError_t product(const Plan& p, const Parts& A, const Parts& B, int64_t rows, int64_t cols, int64_t k, int64_t batch, const Finish& fin,
                   f32x4* partial, hipStream_t st) {
    // (half of a square is too few tiles of 256 x 256)
    if (p.huge && (MODE == STEP || MODE == LAST)) return product_of<MODE, 4, 4, 2>(A, B, rows, cols, k, batch, fin, 256, 1, nullptr, st);
    if (p.big) {
        const Cut cut = cut_of(tiles_of<MODE>(rows, cols, 64) * batch, tiles_of<MODE>(rows, cols, 128) * batch, k / KB);
        if (!cut.waves) return product_of<MODE, 2, 2, 2>(A, B, rows, cols, k, batch, fin, SLOTS, cut.splits, partial, st);
    }
    const auto kernel = ortho_wave_kernel<MODE>;
    if (hipError_t e = ensure_dynamic_lds((const void*)kernel, 131072); e != hipSuccess) return e;
    kernel<<<dim3((unsigned)(tiles_of<MODE>(rows, cols, 64) * batch)), 256, 131072, st>>>(A, B, (int)(k / KB), (int)(rows / 64), (int)(cols / 64), fin);
    return hipGetLastError();
}

template <class T>
hipError_t run(const Plan& p, const T* G, int64_t batch, int64_t rows, int64_t cols, int64_t ld, int64_t stride, const float* coef, int steps,
               double eps, double scale, T* out, int64_t ld_out, int64_t stride_out, char* work, hipStream_t st) {
    const bool tall = rows > cols;
    if (p.small) {
        Steps q{};
        q.count = steps;
        q.eps = eps;
        double U = 1.0 + 0x1p-10, sx = scale_for(U);
        q.sx = sx;
        for (int s = 0; s < steps; ++s) {
            const double ca = coef[3 * s], cb = coef[3 * s + 1], cc = coef[3 * s + 2];
            const double next = bound_of(ca, cb, cc, U, true) * (1.0 + 0x1p-10);
            const double sa = scale_for(U * U), sp = scale_for(bound_of(ca, cb, cc, U * U, false)), sn = scale_for(next);
            auto& a = q.at[s];
            a.cubic = cc == 0.0;
            a.gram = (float)(a.cubic ? cb * sp / (sx * sx) : sa / (sx * sx));
            a.square = (float)(cc * sp / (sa * sa));
            a.linear = (float)(cb * sp / sa);
            a.diag = (float)(ca * sp);
            a.step = (float)((s + 1 < steps ? sn : scale) / (sp * sx));
            U = next;
            sx = sn;
        }
        // (a few matrices have four waves each, at least, for what is not split over columns)
        const bool wide = p.n > 256;
        const int waves = std::max((int)(p.n + (wide ? 63 : 31)) / (wide ? 64 : 32), batch <= 512 ? 4 : 1);
        const auto bytes = [&](int w) { return std::max(w * 64 * (wide ? 65 : 33) * 4, w * 12288 + 32768); };
        const auto kernel = wide ? ortho_small_kernel<T, 2> : ortho_small_kernel<T, 1>;
        if (hipError_t e = ensure_dynamic_lds((const void*)kernel, bytes(8)); e != hipSuccess) return e;
        kernel<<<dim3((unsigned)batch), waves * 64, bytes(waves), st>>>(G, (int)rows, (int)cols, ld, stride, out, ld_out, stride_out, q);
        return hipGetLastError();
    }
    f16* w = (f16*)work;
    const int64_t c = p.chunk;
    Parts X{w, 2 * p.N, p.x}, Xt[2] = {{w + c * p.x, 2 * p.M, p.x}, {w + 2 * c * p.x, 2 * p.M, p.x}};
    w += 3 * c * p.x;
    const Parts A{w, 2 * p.M, p.a}, P{w + c * p.a, 2 * p.M, p.a};
    double* partial = (double*)(w + 2 * c * p.a);
    f32x4* const join = (f32x4*)(work + c * p.per);

    ortho_norm_kernel<T><<<dim3((unsigned)(p.groups * batch)), NORM_THREADS, 0, st>>>(G, rows, cols, ld, stride, partial, p.groups);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    double U = 1.0 + 0x1p-10;  // of the singular values
    double sx = scale_for(U);
    const int tr = (int)((tall ? p.N : p.M) / 64), tc = (int)((tall ? p.M : p.N) / 64);
    ortho_split_kernel<T><<<dim3((unsigned)((int64_t)tr * tc * batch)), 256, 0, st>>>(G, rows, cols, ld, stride, partial, p.groups, eps, sx,
                                                                                      tall ? Xt[0] : X, tall ? X : Xt[0], tr, tc);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    for (int s = 0; s < steps; ++s) {
        const double ca = coef[3 * s], cb = coef[3 * s + 1], cc = coef[3 * s + 2];
        const double next = bound_of(ca, cb, cc, U, true) * (1.0 + 0x1p-10);
        const double sa = scale_for(U * U), sp = scale_for(bound_of(ca, cb, cc, U * U, false)), sn = scale_for(next);
        Finish f{};
        if (cc != 0.0) {
            f.f = (float)(sa / (sx * sx));
            f.C = A;
            if (hipError_t e = product<GRAM>(p, X, X, p.M, p.M, p.N, batch, f, join, st); e != hipSuccess) return e;
            f.f = (float)(cc * sp / (sa * sa));
            f.fa = (float)(cb * sp / sa);
            f.diag = (float)(ca * sp);
            f.A = A;
            f.C = P;
            if (hipError_t e = product<POLY>(p, A, A, p.M, p.M, p.M, batch, f, join, st); e != hipSuccess) return e;
        } else {
            f.f = (float)(cb * sp / (sx * sx));
            f.diag = (float)(ca * sp);
            f.C = P;
            if (hipError_t e = product<GRAM>(p, X, X, p.M, p.M, p.N, batch, f, join, st); e != hipSuccess) return e;
        }
        const Parts& xt = Xt[s & 1];
        if (s + 1 < steps) {
            f.f = (float)(sn / (sp * sx));
            f.C = X;
            f.Ct = Xt[(s + 1) & 1];
            if (hipError_t e = product<STEP>(p, P, xt, p.M, p.N, p.M, batch, f, join, st); e != hipSuccess) return e;
        } else {
            f.f = (float)(scale / (sp * sx));
            f.out = out;
            f.ld_out = ld_out;
            f.stride_out = stride_out;
            f.rows = rows;
            f.cols = cols;
            f.out16 = sizeof(T) == 2;
            const hipError_t e = tall ? product<LAST>(p, xt, P, p.N, p.M, p.M, batch, f, join, st) : product<LAST>(p, P, xt, p.M, p.N, p.M, batch, f, join, st);
            if (e != hipSuccess) return e;
        }
        U = next;
        sx = sn;
    }
    return hipSuccess;
}

bool sizes_ok(int dtype, int64_t batch, int64_t rows, int64_t cols) {
    return (dtype == SAGE_F32 || dtype == SAGE_BF16) && batch >= 0 && batch <= (1ll << 31) && rows >= 1 && rows <= MAX_SIDE && cols >= 1 &&
           cols <= MAX_SIDE;
}

// matrices whose rows are side by side in rows of ld (the column slices of one matrix); else one is behind the other
bool side_by_side(int64_t batch, int64_t rows, int64_t cols, int64_t ld, int64_t stride) {
    return batch > 1 && rows > 1 && stride >= cols && stride <= ld / (batch - 1) && (batch - 1) * stride + cols <= ld;
}

// rows of `cols` every ld, matrices every stride, none with an element of another, all offsets in 62 bits
bool layout_ok(const void* p, int dtype, int64_t batch, int64_t rows, int64_t cols, int64_t ld, int64_t stride) {
    if (!p || (uintptr_t)p % (dtype == SAGE_BF16 ? 2 : 4) || ld < cols || ld > (1ll << 40)) return false;
    const int64_t one = (rows - 1) * ld + cols;
    return batch <= 1 || side_by_side(batch, rows, cols, ld, stride) || (stride >= one && stride <= (1ll << 59) / batch);
}

}  // namespace
}  // namespace sage

extern "C" int sage_orthogonalize_work(sage_dtype dtype, int64_t batch, int64_t rows, int64_t cols, size_t* bytes) {
    if (!bytes || !sage::sizes_ok(dtype, batch, rows, cols)) return SAGE_ERR_ARG;
    const sage::Plan p = sage::plan_of(batch, rows, cols);
    *bytes = batch ? (size_t)p.bytes : 0;
    return SAGE_OK;
}

extern "C" int sage_orthogonalize(const void* G, sage_dtype dtype, int64_t batch, int64_t rows, int64_t cols, int64_t ld, int64_t stride,
                                  const float* coefficients, int steps, float eps, float scale, void* out, int64_t ld_out,
                                  int64_t stride_out, void* work, size_t work_bytes, void* hip_stream) {
    using namespace sage;
    if (!sizes_ok(dtype, batch, rows, cols) || !coefficients || steps < 1 || steps > MAX_STEPS || !(eps >= 0.f) || !(eps < INFINITY) ||
        !(fabsf(scale) < INFINITY))
        return SAGE_ERR_ARG;
    double U = 1.0 + 0x1p-10;
    for (int s = 0; s < steps; ++s) {
        const float* c = coefficients + 3 * s;
        for (int i = 0; i < 3; ++i)
            if (!(fabsf(c[i]) <= 1024.f)) return SAGE_ERR_ARG;
        U = bound_of(c[0], c[1], c[2], U, true) * (1.0 + 0x1p-10);
        if (!(U <= 1024.0)) return SAGE_ERR_ARG;
    }
    if (batch == 0) return SAGE_OK;
    if (!layout_ok(G, dtype, batch, rows, cols, ld, stride) || !layout_ok(out, dtype, batch, rows, cols, ld_out, stride_out)) return SAGE_ERR_ARG;
    const int64_t es = dtype == SAGE_BF16 ? 2 : 4;
    if (!(G == out && ld == ld_out && (batch == 1 || stride == stride_out))) {
        const uintptr_t g0 = (uintptr_t)G, o0 = (uintptr_t)out;
        const uintptr_t g1 = g0 + es * ((batch > 1 ? (batch - 1) * stride : 0) + (rows - 1) * ld + cols);
        const uintptr_t o1 = o0 + es * ((batch > 1 ? (batch - 1) * stride_out : 0) + (rows - 1) * ld_out + cols);
        const bool alike = (rows == 1 || ld == ld_out) && (batch == 1 || stride == stride_out);  // (else they are taken to meet where their spans do)
        const int64_t d = (int64_t)(o0 - g0), apart = es * (batch > 1 ? stride : (rows - 1) * ld + cols), pitch = es * ld, width = es * cols;
        if (g0 < o1 && o0 < g1 &&
            (!alike || (side_by_side(batch, rows, cols, ld, stride) ? groups_meet(d, pitch, rows, apart, batch, width, width)
                                                                    : groups_meet(d, apart, batch, pitch, rows, width, width))))
            return SAGE_ERR_ARG;
    }
    const Plan p = plan_of(batch, rows, cols);
    if (!work || (uintptr_t)work % 256 || work_bytes < (size_t)p.bytes) return SAGE_ERR_ARG;
    for (int64_t b = 0; b < batch; b += p.chunk) {
        const int64_t n = std::min(p.chunk, batch - b);
        const hipError_t e =
            dtype == SAGE_F32
                ? run<float>(p, (const float*)G + b * stride, n, rows, cols, ld, stride, coefficients, steps, eps, scale,
                             (float*)out + b * stride_out, ld_out, stride_out, (char*)work, (hipStream_t)hip_stream)
                : run<uint16_t>(p, (const uint16_t*)G + b * stride, n, rows, cols, ld, stride, coefficients, steps, eps, scale,
                                (uint16_t*)out + b * stride_out, ld_out, stride_out, (char*)work, (hipStream_t)hip_stream);
        if (e != hipSuccess) {
            (void)hipGetLastError();
            return SAGE_ERR_HIP;
        }
    }
    return SAGE_OK;
}
