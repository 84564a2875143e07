// A label for every row of logits, drawn with a given random number: sage_sample (include/sage.h).
//
// A class's weight is the whole number rint(2^42 exp((z_j - max z) / T)). Sums of whole numbers do not depend on the order of
// addition, so that the label is a function of the row and its number alone, however a row is cut over threads; a weight is
// off by at most 2^-43 of the greatest, which moves the borders between the classes of a row of 2^20 by less than 2^-23 of
// it at worst and by 2^-33 as such errors fall out. Everything up to the comparison is done in 64 bits.
#include <algorithm>

#include "logit_rows.h"
#include "sage_internal.h"

namespace sage {
namespace {

constexpr int SB = 1024;
constexpr int SWAVES = SB / 64;

// rint(2^42 e^x) for x <= 0: e^x = 2^n e^r with |r| <= ln 2 / 2, and e^r = 1 + r q(r), q of degree 9 through the Chebyshev points
// (relative error 2^-50; q computed for this with rational numbers). Exactly 2^42 at 0.
__device__ __forceinline__ uint64_t weight_of(double x) {
    if (!(x >= -30.0)) return 0;  // (2^42 e^-30 < 1/2)
    constexpr double ROUND = 6755399441055744.0;  // 1.5 * 2^52: added and taken off again it rounds to a whole number
    const double t = __builtin_fma(x, 1.4426950408889634, ROUND);
    const double n = t - ROUND;
    const double r = __builtin_fma(n, -0.6931471805599453, x);
    double q = 0x1.289185613a3d6p-22;
    q = __builtin_fma(q, r, 0x1.72e1150d0c9b6p-19);
    q = __builtin_fma(q, r, 0x1.a019b90d2ae7ap-16);
    q = __builtin_fma(q, r, 0x1.a01994bd214e7p-13);
    q = __builtin_fma(q, r, 0x1.6c16c1788bd90p-10);
    q = __builtin_fma(q, r, 0x1.11111123c1f47p-7);
    q = __builtin_fma(q, r, 0x1.5555555553d63p-5);
    q = __builtin_fma(q, r, 0x1.5555555550d79p-3);
    q = __builtin_fma(q, r, 0x1.0000000000001p-1);
    q = __builtin_fma(q, r, 0x1.0000000000006p+0);
    const double p = __builtin_fma(q, r, 1.0);
    const int e = (int)__double_as_longlong(t) + 42;  // n + 42 >= -1
    const double w = __longlong_as_double(__double_as_longlong(p) + ((int64_t)e << 52));
    return (uint64_t)(__double_as_longlong(w + ROUND) - __double_as_longlong(ROUND));
}

// Floats in their order as unsigned numbers; both zeros are one.
__device__ __forceinline__ uint32_t key_of(float z) {
    const uint32_t u = __float_as_uint(z + 0.f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) {
    return __uint_as_float(key ^ (key >> 31 ? 0x80000000u : 0xFFFFFFFFu));
}

// The classes kept so far: those above a key, and of those at it the ones before an index.
struct Cut {
    uint32_t key;
    int64_t index;
    __device__ bool keeps(uint32_t k, int64_t j) const { return k > key || (k == key && j < index); }
};

template <class T>
struct Row {
    static constexpr int VL = RowType<T>::VL;
    const T* z;
    int64_t n;
    uint64_t* part;  // LDS, SWAVES + 2

    // sum of f(z_j, j)
    template <class F>
    __device__ uint64_t sum(F f) {
        uint64_t s = 0;
        for (int64_t e0 = (int64_t)threadIdx.x * VL; e0 < n; e0 += SB * VL) {
            float x[VL];
            row_floats(z, e0, n, 0.f, x);
#pragma unroll
            for (int i = 0; i < VL; ++i)
                if (e0 + i < n) s += f(x[i], e0 + i);
        }
        __syncthreads();
        return group_reduce<SB>(s, part, [](uint64_t a, uint64_t b) { return a + b; });
    }

    // the first j with f(z_0, 0) + .. + f(z_j, j) > t; n if there is none
    template <class F>
    __device__ int64_t locate(uint64_t t, F f) {
        uint64_t before = 0;
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        for (int64_t c0 = 0; c0 < n; c0 += SB * VL) {
            const int64_t e0 = c0 + (int64_t)threadIdx.x * VL;
            float x[VL];
            row_floats(z, e0, n, 0.f, x);
            uint64_t v[VL], own = 0;
#pragma unroll
            for (int i = 0; i < VL; ++i) {
                v[i] = e0 + i < n ? f(x[i], e0 + i) : 0;
                own += v[i];
            }
            uint64_t incl = own;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const uint64_t o = __shfl_up(incl, d, 64);
                if (lane >= d) incl += o;
            }
            __syncthreads();
            if (lane == 63) part[wave] = incl;
            if (threadIdx.x == 0) part[SWAVES] = (uint64_t)n;
            __syncthreads();
            uint64_t total = 0, mine = before;
            for (int w = 0; w < SWAVES; ++w) {
                if (w < wave) mine += part[w];
                total += part[w];
            }
            mine += incl - own;
            if (before + total > t) {
                if (mine <= t && mine + own > t) {
                    int i = 0;
                    while (i < VL - 1 && mine + v[i] <= t) mine += v[i++];
                    part[SWAVES] = (uint64_t)(e0 + i);
                }
                __syncthreads();
                return (int64_t)part[SWAVES];
            }
            before += total;
        }
        return n;
    }

    // the greatest key c for which the f of the keys >= c sum to `need` or more, and the sum of those above it
    template <class F>
    __device__ uint32_t key_reaching(uint64_t need, F f, uint64_t& above) {
        uint32_t lo = 0;  // reaches
        uint64_t hi = 1ull << 32;
        above = 0;
        while (hi - lo > 1) {
            const uint32_t mid = (uint32_t)((lo + hi) >> 1);
            const uint64_t s = sum([&](float x, int64_t j) { return key_of(x) >= mid ? f(x, j) : 0ull; });
            if (s >= need) {
                lo = mid;
            } else {
                hi = mid;
                above = s;
            }
        }
        return lo;
    }
};

template <class T>
__global__ __launch_bounds__(SB) void sample_kernel(const T* __restrict__ logits, int64_t C, int64_t ld, const float* __restrict__ u_rows,
                                                    sage_sampling how, int* __restrict__ labels, float* __restrict__ logp) {
    __shared__ uint64_t part[SWAVES + 2];
    __shared__ float fpart[SWAVES];
    const int64_t row = blockIdx.x;
    Row<T> r{logits + row * ld, C, part};
    const float T32 = how.temperature_rows ? how.temperature_rows[row] : how.temperature;
    const float P32 = how.top_p_rows ? how.top_p_rows[row] : how.top_p;
    const float M32 = how.min_p_rows ? how.min_p_rows[row] : how.min_p;
    const int K = how.top_k_rows ? how.top_k_rows[row] : how.top_k;

    float m = -INFINITY;
    uint64_t bad = 0;
    for (int64_t e0 = (int64_t)threadIdx.x * r.VL; e0 < C; e0 += SB * r.VL) {
        float x[RowType<T>::VL];
        row_floats(r.z, e0, C, -INFINITY, x);
#pragma unroll
        for (int i = 0; i < RowType<T>::VL; ++i) {
            m = fmaxf(m, x[i]);
            bad += x[i] != x[i];
        }
    }
    m = group_reduce<SB>(m, fpart, [](float a, float b) { return fmaxf(a, b); });
    bad = group_reduce<SB>(bad, part, [](uint64_t a, uint64_t b) { return a + b; });
    if (bad || !(fabsf(m) < INFINITY)) {
        if (threadIdx.x == 0) {
            labels[row] = -1;
            if (logp) logp[row] = __builtin_nanf("");
        }
        return;
    }
    if (!(T32 > 0.f)) {
        const uint32_t top = key_of(m);
        const int64_t j = r.locate(0, [&](float x, int64_t) { return key_of(x) == top ? 1ull : 0ull; });
        if (threadIdx.x == 0) {
            labels[row] = (int)j;
            if (logp) logp[row] = 0.f;
        }
        return;
    }
    const double Td = T32, inv = 1.0 / Td, md = m;
    auto weight = [&](float x) { return weight_of(((double)x - md) * inv); };
    Cut cut{0, C};  // (no float has key 0 or below but NaNs)
    if (K > 0 && K < C) {
        uint64_t above;
        auto one = [](float, int64_t) { return 1ull; };
        cut.key = r.key_reaching((uint64_t)K, one, above);
        cut.index = 1 + r.locate(K - above - 1, [&](float x, int64_t) { return key_of(x) == cut.key ? 1ull : 0ull; });
    }
    auto kept_weight = [&](float x, int64_t j) { return cut.keeps(key_of(x), j) ? weight(x) : 0ull; };
    if (P32 < 1.f) {
        const uint64_t S = r.sum(kept_weight);
        const double q = ceil((double)P32 * (double)S);
        const uint64_t need = q >= 1.0 ? (uint64_t)q : 1;
        uint64_t above;
        const uint32_t key = r.key_reaching(need, kept_weight, above);
        const uint64_t w = weight(value_of(key));
        const uint64_t count = (need - above + w - 1) / w;  // w > 0: that key made the sum reach
        const int64_t end = 1 + r.locate(count - 1, [&](float x, int64_t j) { return key_of(x) == key && cut.keeps(key, j) ? 1ull : 0ull; });
        cut = Cut{key, end};
    }
    double border = -INFINITY;  // z - m of the least class that min-p keeps
    if (M32 > 0.f) border = Td * log((double)fminf(M32, 1.f));
    auto drawn = [&](float x, int64_t j) { return (double)x - md >= border ? kept_weight(x, j) : 0ull; };
    const uint64_t S = r.sum(drawn);
    const float u = u_rows[row];
    uint64_t t = u > 0.f ? (uint64_t)((double)fminf(u, 1.f) * (double)S) : 0;
    if (t >= S) t = S - 1;
    const int64_t j = r.locate(t, drawn);
    if (threadIdx.x == 0) {
        labels[row] = (int)j;
        if (logp) logp[row] = (float)(((double)RowType<T>::widen(r.z[j]) - md) * inv - log((double)S * 0x1p-42));
    }
}

}  // namespace

bool logit_rows_ok(const void* p, int dtype, int64_t rows, int64_t C, int64_t ld) {
    if (dtype != SAGE_F32 && dtype != SAGE_BF16) return false;
    if (rows < 0 || C < 1 || C > SAGE_MAX_CLASSES || ld < C || ld > (INT64_MAX >> 24)) return false;
    if (rows == 0) return true;
    return p && (uintptr_t)p % (dtype == SAGE_BF16 ? 2 : 4) == 0 && ld <= (INT64_MAX >> 3) / rows;
}

bool rows_overlap(const void* a, int da, int64_t lda, const void* b, int db, int64_t ldb, int64_t rows, int64_t C) {
    if (rows == 0) return false;
    const uintptr_t a0 = (uintptr_t)a, b0 = (uintptr_t)b;
    const uintptr_t a1 = a0 + ((uint64_t)(rows - 1) * lda + C) * (da == SAGE_BF16 ? 2 : 4);
    const uintptr_t b1 = b0 + ((uint64_t)(rows - 1) * ldb + C) * (db == SAGE_BF16 ? 2 : 4);
    return a0 < b1 && b0 < a1;
}

}  // namespace sage

extern "C" int sage_sample(const void* logits, sage_dtype dtype, int64_t rows, int64_t n_classes, int64_t ld, const float* u,
                           const sage_sampling* how, int32_t* labels, float* logp, void* hip_stream) {
    if (!sage::logit_rows_ok(logits, dtype, rows, n_classes, ld) || (rows > 0 && (!u || !labels))) return SAGE_ERR_ARG;
    if (rows == 0) return SAGE_OK;
    sage_sampling h = how ? *how : sage_sampling{1.f, 0, 1.f, 0.f, nullptr, nullptr, nullptr, nullptr};
    const hipStream_t st = (hipStream_t)hip_stream;
    for (int64_t r0 = 0; r0 < rows; r0 += sage::LOGIT_LAUNCH_ROWS) {
        const dim3 grid((unsigned)std::min(rows - r0, sage::LOGIT_LAUNCH_ROWS));
        float* lp = logp ? logp + r0 : nullptr;
        if (dtype == SAGE_F32)
            sage::sample_kernel<float><<<grid, sage::SB, 0, st>>>((const float*)logits + r0 * ld, n_classes, ld, u + r0, h, labels + r0, lp);
        else
            sage::sample_kernel<uint16_t><<<grid, sage::SB, 0, st>>>((const uint16_t*)logits + r0 * ld, n_classes, ld, u + r0, h, labels + r0, lp);
        if (hipGetLastError() != hipSuccess) return SAGE_ERR_HIP;
        if (h.temperature_rows) h.temperature_rows += grid.x;
        if (h.top_k_rows) h.top_k_rows += grid.x;
        if (h.top_p_rows) h.top_p_rows += grid.x;
        if (h.min_p_rows) h.min_p_rows += grid.x;
    }
    return SAGE_OK;
}
