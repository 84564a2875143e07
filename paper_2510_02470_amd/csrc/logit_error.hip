// Cross-entropy of rows of logits and its gradient with respect to them: sage_logit_error (include/sage.h).
//
// With m = max z, e_j = exp(z_j - m) and R = the sum of e_j over the classes other than the label y:
//     loss = ln((R + e_y) / e_y) = log1p(R / e_y),   E_j = w e_j / (R + e_y),   E_y = -w R / (R + e_y).
// The label is left out of the sum, because loss and E_y are differences of nearly equal numbers when written with p_y: a
// learnt example has p_y = 1 - 1e-6, of which fp32 keeps one digit of the part that matters.
//
// Bound by memory: a row is read once and its gradient written once. A work-group keeps its row in registers between the two,
// as it was read, and forms the exponentials twice.
#include <algorithm>
#include <type_traits>

#include "logit_rows.h"
#include "sage_internal.h"

namespace sage {
namespace {

// e^(x - m): the difference is exact or rounded once; the product with log2 e is carried to twice the width where WIDE. Without it a
// difference of 16 loses 2^-20, which a bf16 E does not show; the sums always have it, for the loss is fp32 whatever E is (204 us
// for 4096 x 65,536 bf16, 198 without it; 410 and 372 for fp32 logits with a bf16 E).
template <bool WIDE>
__device__ __forceinline__ float exp_diff(float x, float m) {
    const float d = x - m;
    const float L = 1.44269502f, L2 = 1.92596299e-8f;  // log2 e = L + L2
    const float t = d * L;
    const float e = __builtin_amdgcn_exp2f(t);
    if constexpr (!WIDE) return e;
    const float r = fmaf(d, L, -t) + d * L2;
    return t <= -126.f ? 0.f : fmaf(e, r * 0.693147181f, e);  // (r is no number where d is infinite; a NaN stays one)
}

// ln((rest + ey) / ey); where ey is too small for an fp32 the label's distance to the maximum is all that counts beside the sum.
__device__ __forceinline__ float row_loss(float rest, float ey, float zy, float m) {
    if (rest + ey == 0.f) return INFINITY;
    if (ey < 0x1p-100f) return (float)(log((double)rest) + ((double)m - (double)zy));
    return (float)log1p((double)rest / (double)ey);
}

template <class T>
struct ErrorArgs {
    const T* logits;
    int64_t rows;
    int C, parts;
    int64_t ld;
    const int* labels;
    const float* weights;
    int64_t ldE;
    float* loss;
};

// A row's vector from e0 on; what lies behind the end is -inf. whole: it is known not to reach there.
template <class T>
__device__ __forceinline__ u32x4 row_vector(const T* z, int e0, int n, bool whole) {
    constexpr int VL = RowType<T>::VL;
    if (whole || e0 + VL <= n) return load16(z + e0);
    constexpr uint32_t NONE = sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u;
    u32x4 v = {NONE, NONE, NONE, NONE};
#pragma unroll
    for (int i = 0; i < VL; ++i)
        if (e0 + i < n) {
            if constexpr (sizeof(T) == 2) v[i >> 1] = i & 1 ? (v[i >> 1] & 0xFFFFu) | (uint32_t)z[e0 + i] << 16 : (v[i >> 1] & 0xFFFF0000u) | z[e0 + i];
            else v[i] = __float_as_uint(z[e0 + i]);
        }
    return v;
}

// -inf in the label's place, if it is in this vector.
template <class T>
__device__ __forceinline__ void drop_label(u32x4& v, int at) {
    constexpr int VL = RowType<T>::VL;
    if ((unsigned)at >= (unsigned)VL) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 2) {
            if (at == 2 * i) v[i] = (v[i] & 0xFFFF0000u) | 0xFF80u;
            if (at == 2 * i + 1) v[i] = (v[i] & 0xFFFFu) | 0xFF800000u;
        } else {
            if (at == i) v[i] = 0xFF800000u;
        }
    }
}

template <class T, class TE>
__device__ __forceinline__ void write_vector(TE* out, int e0, int n, bool whole, const u32x4& v, float scale, float m) {
    constexpr int VL = RowType<T>::VL;
    constexpr bool WIDE = sizeof(TE) == 4;
    TE h[VL];
#pragma unroll
    for (int i = 0; i < VL; ++i) h[i] = RowType<TE>::narrow(scale * exp_diff<WIDE>(RowType<T>::at(v, i), m));
    if (whole || e0 + VL <= n) {
        __builtin_memcpy(out + e0, h, sizeof(h));
    } else {
#pragma unroll
        for (int i = 0; i < VL; ++i)
            if (e0 + i < n) out[e0 + i] = h[i];
    }
}

// THREADS threads a row, ROWS rows a work-group (rows of one wave each need no barrier, and a launch of many has fewer work-groups to
// hand out: 65,536 rows of 1000 bf16 115 us with 256 threads each, 64 with 4 waves for 4 rows). N > 0: N vectors of 16 bytes a thread, kept in
// registers between reading and writing; 0: a longer row, read a second time. L: as many vectors more in LDS, where registers alone would
// leave room for one work-group to a CU, whose reading and writing then have nothing beside them.
template <class T, class TE, int THREADS, int ROWS, int N, int L>
__global__ __launch_bounds__(THREADS * ROWS) void logit_error_kernel(ErrorArgs<T> a, TE* E) {
    extern __shared__ u32x4 held[];  // L * THREADS
    static_assert(ROWS == 1 || THREADS == 64, "a row of several waves has the work-group's barrier");
    __shared__ float2 wave_part[THREADS / 64];
    constexpr int VL = RowType<T>::VL;
    // a row's work-groups each read all of it and write a part
    const int parts = N == 0 ? a.parts : 1, part = N == 0 ? blockIdx.x % a.parts : 0;
    const int64_t row = N == 0 ? blockIdx.x / a.parts : (int64_t)blockIdx.x * ROWS + (ROWS > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0);
    if (ROWS > 1 && row >= a.rows) return;
    const T* z = a.logits + row * a.ld;
    TE* out = E ? E + row * a.ldE : nullptr;
    const int y = a.labels[row], C = a.C;
    const int tid = ROWS > 1 ? threadIdx.x & 63 : threadIdx.x;
    if (y < 0) {
        if (out)
            for (int j = tid; j < C; j += THREADS) out[j] = 0;
        if (a.loss && tid == 0) a.loss[row] = 0.f;
        return;
    }
    const float zy = y < C ? RowType<T>::widen(z[y]) : __builtin_nanf("");
    const float f = a.weights ? a.weights[row] : 1.f;
    const int turns = (C + THREADS * VL - 1) / (THREADS * VL);
    u32x4 reg[N > 0 ? N : 1];
    // the greatest logit so far and the sum of the exponentials relative to it, together as the vectors arrive; m is finite from the
    // start, so that a difference to it is a number where all logits are -inf
    float m = fmaxf(zy, -3.40282347e38f), rest = 0.f;
    // f(vector, its first element, whether all vectors of the wave are whole); FIRST: the pass that reads, and puts -inf in the label's place
    const int first = __builtin_amdgcn_readfirstlane(tid) * VL;  // of the wave
    auto visit = [&](auto first_pass, auto f) __attribute__((always_inline)) {
        constexpr bool FIRST = decltype(first_pass)::value;
        if constexpr (N > 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int w0 = i * THREADS * VL + first, e0 = (i * THREADS + tid) * VL;
                // (turns mixed with each other, or floats kept from one pass to the next, would need more registers)
                __builtin_amdgcn_sched_barrier(0);
                asm volatile("" : "+v"(reg[i]));
                if (FIRST && (unsigned)(y - w0) < 64u * VL) drop_label<T>(reg[i], y - e0);
                f(reg[i], e0, w0 + 64 * VL <= C);
            }
        }
        if constexpr (L > 0) {
#pragma unroll 1
            for (int i = N; i < turns; ++i) {
                const int w0 = i * THREADS * VL + first, e0 = (i * THREADS + tid) * VL;
                u32x4& v = held[(i - N) * THREADS + tid];
                if (FIRST && (unsigned)(y - w0) < 64u * VL) {
                    u32x4 x = v;
                    drop_label<T>(x, y - e0);
                    v = x;
                }
                f(v, e0, w0 + 64 * VL <= C);
            }
        }
        if constexpr (N == 0) {
            constexpr int AHEAD = 4;  // vectors of a thread that are read together (those behind the end are -inf, and not written)
            const int to = FIRST ? turns : turns * (part + 1) / parts;
#pragma unroll 1
            for (int i = FIRST ? 0 : turns * part / parts; i < to; i += AHEAD) {
                u32x4 v[AHEAD];
#pragma unroll
                for (int k = 0; k < AHEAD; ++k) v[k] = row_vector(z, ((i + k) * THREADS + tid) * VL, C, (i + k) * THREADS * VL + first + 64 * VL <= C);
#pragma unroll
                for (int k = 0; k < AHEAD; ++k) {
                    const int w0 = (i + k) * THREADS * VL + first, e0 = ((i + k) * THREADS + tid) * VL;
                    if (i + k >= to) break;
                    if (FIRST && (unsigned)(y - w0) < 64u * VL) drop_label<T>(v[k], y - e0);
                    f(v[k], e0, w0 + 64 * VL <= C);
                }
            }
        }
    };
    if constexpr (N > 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) reg[i] = row_vector(z, (i * THREADS + tid) * VL, C, i * THREADS * VL + first + 64 * VL <= C);
    }
    if constexpr (L > 0) {
#pragma unroll 4
        for (int i = N; i < turns; ++i) held[(i - N) * THREADS + tid] = row_vector(z, (i * THREADS + tid) * VL, C, i * THREADS * VL + first + 64 * VL <= C);
    }
    visit(std::true_type{}, [&](const u32x4& v, int, bool) __attribute__((always_inline)) {
        float top = m;
#pragma unroll
        for (int i = 0; i < VL; ++i) top = fmaxf(top, RowType<T>::at(v, i));
        float sum = rest * exp_diff<true>(m, top);
#pragma unroll
        for (int i = 0; i < VL; ++i) sum += exp_diff<true>(RowType<T>::at(v, i), top);
        m = top;
        rest = sum;
    });
    // over the wave, then over the work-group
    float top = m;
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
    rest *= exp_diff<true>(m, top);
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) rest += __shfl_xor(rest, d, 64);
    m = top;
    if constexpr (THREADS > 64) {
        if ((tid & 63) == 0) wave_part[tid >> 6] = float2{m, rest};
        __syncthreads();
        float2 w[THREADS / 64];
#pragma unroll
        for (int i = 0; i < THREADS / 64; ++i) w[i] = wave_part[i];
#pragma unroll
        for (int i = 0; i < THREADS / 64; ++i) m = fmaxf(m, w[i].x);
        rest = 0.f;
#pragma unroll
        for (int i = 0; i < THREADS / 64; ++i) rest += w[i].y * exp_diff<true>(w[i].x, m);
    }
    const float ey = exp_diff<true>(zy, m), S = rest + ey;
    if (a.loss && tid == 0 && part == 0) a.loss[row] = row_loss(rest, ey, zy, m);
    if (!out) return;
    const float scale = S == 0.f ? 0.f : f / S;
    visit(std::false_type{}, [&](const u32x4& v, int e0, bool whole) __attribute__((always_inline)) {
        write_vector<T>(out, e0, C, whole, v, scale, m);
    });
    // the label's entry, by the thread that has written its vector: after that one's store
    const int at_turn = y / (THREADS * VL);
    if (y < C && tid == y / VL % THREADS && at_turn >= turns * part / parts && at_turn < turns * (part + 1) / parts) out[y] = RowType<TE>::narrow(-scale * rest);
}

template <int N>
using I = std::integral_constant<int, N>;

template <class T, class TE>
hipError_t launch(const void* z, int64_t rows, int64_t C, int64_t ld, const int* labels, const float* weights, void* E, int64_t ldE,
                  float* loss, hipStream_t st) {
    constexpr int VL = RowType<T>::VL;
    for (int64_t r0 = 0; r0 < rows; r0 += LOGIT_LAUNCH_ROWS) {
        const int64_t n = std::min(rows - r0, LOGIT_LAUNCH_ROWS);
        // long rows that leave CUs idle are written by several work-groups, unless what one writes is what another reads
        const int parts = E && E != z ? (int)std::max<int64_t>(1, std::min<int64_t>(8, 256 / n)) : 1;
        const ErrorArgs<T> a{(const T*)z + r0 * ld, n, (int)C, parts, ld, labels + r0, weights ? weights + r0 : nullptr, ldE, loss ? loss + r0 : nullptr};
        TE* e = E ? (TE*)E + r0 * ldE : nullptr;
        const auto go = [&](auto threads, auto per, auto registers, auto more) {
            constexpr int THREADS = decltype(threads)::value, ROWS = decltype(per)::value, L = decltype(more)::value;
            const auto kernel = logit_error_kernel<T, TE, THREADS, ROWS, decltype(registers)::value, L>;
            if (L > 0)
                if (hipError_t err = ensure_dynamic_lds((const void*)kernel, L * THREADS * 16); err != hipSuccess) return err;
            const int64_t groups = decltype(registers)::value == 0 ? n * parts : (n + ROWS - 1) / ROWS;
            kernel<<<dim3((unsigned)groups), THREADS * ROWS, L * THREADS * 16, st>>>(a, e);
            return hipGetLastError();
        };
        hipError_t err;
        const int64_t vectors = (C + VL - 1) / VL;
        if (vectors <= 64) err = go(I<64>{}, I<4>{}, I<1>{}, I<0>{});
        else if (vectors <= 128) err = go(I<64>{}, I<4>{}, I<2>{}, I<0>{});
        else if (vectors <= 256) err = go(I<64>{}, I<4>{}, I<4>{}, I<0>{});
        else if (vectors <= 512) err = go(I<256>{}, I<1>{}, I<2>{}, I<0>{});
        else if (vectors <= 1024) err = go(I<256>{}, I<1>{}, I<4>{}, I<0>{});
        else if (vectors <= 4096) err = go(I<512>{}, I<1>{}, I<8>{}, I<0>{});
        else if (vectors <= 8192) err = go(I<512>{}, I<1>{}, I<16>{}, I<0>{});
        else if (vectors <= 12800 && rows > 256) err = go(I<512>{}, I<1>{}, I<16>{}, I<9>{});  // two to a CU
        else if (vectors <= 16384) err = go(I<1024>{}, I<1>{}, I<16>{}, I<0>{});
        else err = go(I<1024>{}, I<1>{}, I<0>{}, I<0>{});
        if (err != hipSuccess) return err;
    }
    return hipSuccess;
}

}  // namespace
}  // namespace sage

extern "C" int sage_logit_error(const void* logits, sage_dtype dtype, int64_t rows, int64_t n_classes, int64_t ld, const int32_t* labels,
                                const float* weights, void* E, sage_dtype e_dtype, int64_t ld_e, float* loss, void* hip_stream) {
    if (!sage::logit_rows_ok(logits, dtype, rows, n_classes, ld) || (rows > 0 && !labels)) return SAGE_ERR_ARG;
    if (e_dtype != SAGE_F32 && e_dtype != SAGE_BF16) return SAGE_ERR_ARG;
    if (E && !sage::logit_rows_ok(E, e_dtype, rows, n_classes, ld_e)) return SAGE_ERR_ARG;
    if (E && !(E == logits && e_dtype == dtype && ld_e == ld) &&
        sage::rows_overlap(logits, dtype, ld, E, e_dtype, ld_e, rows, n_classes))
        return SAGE_ERR_ARG;
    if (rows == 0 || (!E && !loss)) return SAGE_OK;
    const hipStream_t st = (hipStream_t)hip_stream;
    const auto go = dtype == SAGE_F32 ? (e_dtype == SAGE_F32 ? sage::launch<float, float> : sage::launch<float, uint16_t>)
                                      : (e_dtype == SAGE_F32 ? sage::launch<uint16_t, float> : sage::launch<uint16_t, uint16_t>);
    const hipError_t e = go(logits, rows, n_classes, ld, labels, weights, E, ld_e, loss, st);
    if (e == hipSuccess) return SAGE_OK;
    (void)hipGetLastError();
    return SAGE_ERR_HIP;
}
