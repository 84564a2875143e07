// A label for every row of logits, drawn with a given random number: sage_sample (include/sage.h).
//
// A class's weight is the whole number rint(2^42 exp((z_j - max z) / T)). Sums of whole numbers do not depend on the order of
// addition, so that the label is a function of the row and its number alone, however a row is cut over threads; a weight is
// off by at most 2^-43 of the greatest, which moves the borders between the classes of a row of 2^20 by less than 2^-23 of
// it at worst and by 2^-33 as such errors fall out. Everything up to the comparison is done in 64 bits.
#include <algorithm>
#include <type_traits>

#include "logit_rows.h"
#include "sage_internal.h"

namespace sage {
namespace {

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
// The classes kept so far: those above a key, and of those at it the ones before an index.
struct Cut {
    uint32_t key;
    int index;
    __device__ bool keeps(uint32_t k, int j) const { return k > key || (k == key && j < index); }
};

// What the THREADS threads of a row share.
template <int THREADS>
struct Shared {
    static constexpr int W = THREADS / 64;
    static constexpr int BITS = THREADS == 64 ? 8 : THREADS == 256 ? 10 : 11, BINS = 1 << BITS;  // of a histogram
    static constexpr int LIST = THREADS == 64 ? 128 : THREADS == 256 ? 512 : 1024;  // classes that are put in order one by one
    static constexpr int SEGS = THREADS == 1024 ? SAGE_MAX_CLASSES / 256 : 16 * W;  // pieces of 64 vectors of the longest row
    uint64_t hist[BINS > SEGS ? BINS : SEGS];  // a histogram, or the sums of segments
    uint64_t part[W];
    float fpart[2 * W];
    uint64_t lkey[LIST];  // key and place of a listed class, one number in their common order; and its weight
    uint64_t lw[LIST];
    uint64_t found[2];
    unsigned listed;
    uint64_t answer;
};

// A row as THREADS threads see it: vector i of a thread holds elements (i THREADS + thread) VL .. + VL - 1, those behind the row's
// end being -inf. STAGED: kept in LDS by load(), else read again for every pass (one vector on its way while one is worked on).
template <class T, int THREADS, bool STAGED>
struct Row {
    static constexpr int VL = RowType<T>::VL;
    static constexpr uint32_t NONE = sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u;  // -inf
    const T* z;
    int n, tid, count;  // count: vectors of a thread
    u32x4* lds;         // count * THREADS

    __device__ u32x4 fetch(int e0) const {
        if (e0 + VL <= n) return load16(z + e0);
        u32x4 v = {NONE, NONE, NONE, NONE};
        if (e0 < n) {
            if constexpr (sizeof(T) == 2) {
#pragma unroll
                for (int i = 0; i < VL; ++i)
                    if (e0 + i < n) v[i >> 1] = i & 1 ? (v[i >> 1] & 0xFFFFu) | (uint32_t)z[e0 + i] << 16 : (v[i >> 1] & 0xFFFF0000u) | z[e0 + i];
            } else {
#pragma unroll
                for (int i = 0; i < VL; ++i)
                    if (e0 + i < n) v[i] = __float_as_uint(z[e0 + i]);
            }
        }
        return v;
    }
    // f(i, first element, vector), in the order of i; first: the pass that reads the row
    template <bool FIRST = false, class F>
    __device__ __forceinline__ void visit(F f) const {
        if constexpr (STAGED && !FIRST) {
#pragma unroll 1
            for (int i = 0; i < count; ++i) f(i, (i * THREADS + tid) * VL, lds[i * THREADS + tid]);
        } else {
            u32x4 v = fetch(tid * VL);
#pragma unroll 1
            for (int i = 0; i < count; ++i) {
                const u32x4 next = fetch(i + 1 < count ? ((i + 1) * THREADS + tid) * VL : n);
                if constexpr (STAGED) lds[i * THREADS + tid] = v;
                f(i, (i * THREADS + tid) * VL, v);
                v = next;
            }
        }
    }
    // f(value, element) for each element
    template <bool FIRST = false, class F>
    __device__ __forceinline__ void each(F f) const {
        visit<FIRST>([&](int, int e0, const u32x4& v) __attribute__((always_inline)) {
#pragma unroll
            for (int k = 0; k < VL; ++k) f(RowType<T>::at(v, k), e0 + k);
        });
    }
};

__device__ __forceinline__ uint64_t wave_sum(uint64_t v) {
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d, 64);
    return v;
}
__device__ __forceinline__ uint64_t wave_scan(uint64_t v, int lane) {  // sums up to and with each lane
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint64_t o = __shfl_up(v, d, 64);
        if (lane >= d) v += o;
    }
    return v;
}

// The first of `count` sums in LDS up to which they come to more than t: found[0] its number, found[1] the sum of those
// before it. t < 0 (as an unsigned number, -1): nothing is looked for. Returns the sum of all.
template <int THREADS>
__device__ uint64_t find_sum(Shared<THREADS>& S, int count, int tid, uint64_t* t_of_total, const float* u) {
    const int per = (count + THREADS - 1) / THREADS;
    uint64_t own = 0;
    for (int i = 0; i < per; ++i)
        if (tid * per + i < count) own += S.hist[tid * per + i];
    const uint64_t incl = wave_scan(own, tid & 63);
    uint64_t before = incl - own, total = incl;
    if constexpr (THREADS > 64) {
        if ((tid & 63) == 63) S.part[tid >> 6] = incl;
        __syncthreads();
        total = 0;
        for (int w = 0; w < THREADS / 64; ++w) {
            if (w < tid >> 6) before += S.part[w];
            total += S.part[w];
        }
    } else {
        total = __shfl(incl, 63, 64);
    }
    if (u) {  // t from the total: a random number's place in it
        const float x = *u;
        uint64_t t = x > 0.f ? (uint64_t)((double)fminf(x, 1.f) * (double)total) : 0;
        *t_of_total = t >= total ? total - 1 : t;
    }
    const uint64_t t = *t_of_total;
    if (before <= t && before + own > t) {
        int i = tid * per;
        while (before + S.hist[i] <= t) before += S.hist[i++];
        S.found[0] = (uint64_t)i;
        S.found[1] = before;
    }
    __syncthreads();
    return total;
}

// The first element up to which f(value, element) sum to more than t, or to more than u's share of their sum, which is returned
// (the sum in `total`). f is 0 for what lies behind the row's end.
template <class T, int THREADS, bool STAGED, class F>
__device__ int locate(const Row<T, THREADS, STAGED>& r, Shared<THREADS>& S, uint64_t t, const float* u, uint64_t& total, F f) {
    constexpr int VL = RowType<T>::VL, W = THREADS / 64;
    const int lane = r.tid & 63, wave = r.tid >> 6;
    __syncthreads();
    r.visit([&](int i, int e0, const u32x4& v) __attribute__((always_inline)) {
        uint64_t own = 0;
#pragma unroll
        for (int k = 0; k < VL; ++k) own += f(RowType<T>::at(v, k), e0 + k);
        const uint64_t s = __any(own != 0) ? wave_sum(own) : 0;
        if (lane == 0) S.hist[i * W + wave] = s;
    });
    __syncthreads();
    total = find_sum<THREADS>(S, r.count * W, r.tid, &t, u);
    const int seg = (int)S.found[0];
    if (wave == seg % W) {
        const uint64_t base = S.found[1];
        const int e0 = (seg * 64 + lane) * VL;
        const u32x4 v = r.fetch(e0);
        uint64_t w[VL], own = 0;
#pragma unroll
        for (int k = 0; k < VL; ++k) {
            w[k] = f(RowType<T>::at(v, k), e0 + k);
            own += w[k];
        }
        uint64_t before = base + wave_scan(own, lane) - own;
        if (before <= t && before + own > t) {
            int at = 0;
#pragma unroll
            for (int k = 0; k < VL - 1; ++k) {  // (no indexing of registers)
                if (at == k && before + w[k] <= t) {
                    before += w[k];
                    ++at;
                }
            }
            S.answer = (uint64_t)(e0 + at);
        }
    }
    __syncthreads();
    return (int)S.answer;
}

// One more histogram of f over the members of a set: bin_of(value) in [0, Shared::BINS), lower bins first in the order, or -1. Finds the bin in
// which the sum from the front passes t; below: the sum before it (S.found).
template <class T, int THREADS, bool STAGED, class B, class F>
__device__ void histogram(const Row<T, THREADS, STAGED>& r, Shared<THREADS>& S, uint64_t t, B bin_of, F f) {
    __syncthreads();
    for (int i = r.tid; i < S.BINS; i += THREADS) S.hist[i] = 0;
    __syncthreads();
    r.each([&](float x, int j) __attribute__((always_inline)) {
        const int b = bin_of(x, j);
        if (b >= 0) {
            const uint64_t w = f(x, j);
            if (w) atomicAdd((unsigned long long*)&S.hist[b], (unsigned long long)w);
        }
    });
    __syncthreads();
    find_sum<THREADS>(S, S.BINS, r.tid, &t, nullptr);
}

// The shortest front part of the order (value descending, place ascending) whose f sum to more than t, as a cut. The sum of all f is more
// than t. A histogram over the distance to the maximum (equal parts of `range`) leaves one bin; its members are put in order
// one by one, or, if they are many, told apart by more histograms over their keys first.
template <class T, int THREADS, bool STAGED, class F>
__device__ Cut front(const Row<T, THREADS, STAGED>& r, Shared<THREADS>& S, uint64_t t, float m, float range, F f) {
    constexpr float LAST = (float)(Shared<THREADS>::BINS - 1);
    constexpr int LIST = Shared<THREADS>::LIST, BITS = Shared<THREADS>::BITS;
    const float scale = LAST / range;  // (may be infinite or 0: bins 0 and, for what is not the maximum, the last)
    auto bin = [&](float x) __attribute__((always_inline)) {
        const float d = m - x;
        return d > 0.f ? (int)fminf(d * scale, LAST) : 0;
    };
    histogram(r, S, t, [&](float x, int) __attribute__((always_inline)) { return bin(x); }, f);
    const int at = (int)S.found[0];
    uint64_t above = S.found[1];
    uint32_t prefix = 0;
    int shift = 32;  // keys of the set agree with prefix from this bit on
    auto member = [&](float x) __attribute__((always_inline)) {
        return bin(x) == at && (shift == 32 || key_of(x) >> shift == prefix);
    };
    for (;;) {
        __syncthreads();
        if (r.tid == 0) S.listed = 0;
        __syncthreads();
        r.each([&](float x, int j) __attribute__((always_inline)) {
            if (member(x)) {
                const uint64_t w = f(x, j);
                if (w) {
                    const unsigned p = atomicAdd(&S.listed, 1u);
                    if (p < LIST) {
                        S.lkey[p] = (uint64_t)key_of(x) << 32 | (uint32_t)~j;  // greater: earlier in the order
                        S.lw[p] = w;
                    }
                }
            }
        });
        __syncthreads();
        const int count = (int)S.listed;
        if (count <= LIST) {
            // the last of the front is the one before which they sum to t or less and with which to more
            for (int i = r.tid; i < count; i += THREADS) {
                const uint64_t key = S.lkey[i];
                uint64_t before = above;
                for (int k = 0; k < count; ++k)
                    if (S.lkey[k] > key) before += S.lw[k];
                if (before <= t && before + S.lw[i] > t) S.answer = key;
            }
            __syncthreads();
            return Cut{(uint32_t)(S.answer >> 32), (int)~(uint32_t)S.answer + 1};
        }
        if (shift == 0) {  // many equal values: their f are equal too, and the first of them are meant
            uint64_t total;
            const int last = locate(r, S, t - above, nullptr, total, [&](float x, int j) { return member(x) ? f(x, j) : 0ull; });
            return Cut{prefix, last + 1};
        }
        const int step = shift < BITS ? shift : BITS;
        const int low = shift - step;
        auto sub = [&](float x, int) __attribute__((always_inline)) {
            return member(x) ? (1 << step) - 1 - (int)(key_of(x) >> low & ((1u << step) - 1)) : -1;
        };
        histogram(r, S, t - above, sub, f);
        above += S.found[1];
        const uint32_t digit = (1u << step) - 1 - (uint32_t)S.found[0];
        prefix = prefix << step | digit;
        shift = low;
    }
}

template <class T, int THREADS, bool STAGED>
__global__ __launch_bounds__(THREADS) void sample_kernel(const T* __restrict__ logits, int C, int64_t ld, const float* __restrict__ u_rows,
                                                         sage_sampling how, int* __restrict__ labels, float* __restrict__ logp) {
    __shared__ Shared<THREADS> S;
    constexpr int VL = RowType<T>::VL;
    const int64_t row = blockIdx.x;
    extern __shared__ u32x4 staged[];
    const Row<T, THREADS, STAGED> r{logits + row * ld, C, (int)threadIdx.x, (C + THREADS * VL - 1) / (THREADS * VL), staged};
    const float T32 = how.temperature_rows ? how.temperature_rows[row] : how.temperature;
    const float P32 = how.top_p_rows ? how.top_p_rows[row] : how.top_p;
    const float M32 = how.min_p_rows ? how.min_p_rows[row] : how.min_p;
    const int K = how.top_k_rows ? how.top_k_rows[row] : how.top_k;

    float m = -INFINITY, low = INFINITY;  // greatest, and least finite
    bool nan = false;
    r.template each<true>([&](float x, int) __attribute__((always_inline)) {
        m = fmaxf(m, x);
        low = x > -INFINITY ? fminf(low, x) : low;
        nan |= x != x;
    });
    if (nan) m = INFINITY;  // either is no distribution
    m = group_reduce<THREADS>(m, S.fpart, [](float a, float b) { return fmaxf(a, b); });
    low = group_reduce<THREADS>(low, S.fpart + THREADS / 64, [](float a, float b) { return fminf(a, b); });
    if (!(fabsf(m) < INFINITY)) {
        if (r.tid == 0) {
            labels[row] = -1;
            if (logp) logp[row] = __builtin_nanf("");
        }
        return;
    }
    uint64_t total;
    if (!(T32 > 0.f)) {
        const int j = locate(r, S, 0, nullptr, total, [&](float x, int) { return x == m ? 1ull : 0ull; });
        if (r.tid == 0) {
            labels[row] = j;
            if (logp) logp[row] = 0.f;
        }
        return;
    }
    const double Td = T32, inv = 1.0 / Td, md = m;
    const float spread = fminf(m - low, 3e38f);
    auto weight = [&](float x) __attribute__((always_inline)) { return weight_of(((double)x - md) * inv); };
    Cut cut{0, 0};  // (no value has key 0)
    if (K > 0 && K < C)
        cut = front(r, S, (uint64_t)K - 1, m, fminf(spread, 64.f), [&](float, int j) __attribute__((always_inline)) { return j < C ? 1ull : 0ull; });
    auto kept_weight = [&](float x, int j) __attribute__((always_inline)) { return cut.keeps(key_of(x), j) ? weight(x) : 0ull; };
    if (P32 < 1.f) {
        uint64_t s = 0;
        r.each([&](float x, int j) __attribute__((always_inline)) { s += kept_weight(x, j); });
        __syncthreads();
        s = group_reduce<THREADS>(s, S.part, [](uint64_t a, uint64_t b) { return a + b; });
        const double q = ceil((double)P32 * (double)s);
        cut = front(r, S, q >= 1.0 ? (uint64_t)q - 1 : 0, m, fminf(spread, 30.f * T32), kept_weight);
    }
    double border = -INFINITY;  // z - m of the least class that min-p keeps
    if (M32 > 0.f) border = Td * log((double)fminf(M32, 1.f));
    const int j = locate(r, S, 0, u_rows + row, total, [&](float x, int k) __attribute__((always_inline)) {
        return (double)x - md >= border ? kept_weight(x, k) : 0ull;
    });
    if (r.tid == 0) {
        labels[row] = j;
        if (logp) logp[row] = (float)(((double)RowType<T>::widen(r.z[j]) - md) * inv - log((double)total * 0x1p-42));
    }
}

template <class T>
hipError_t launch_sample(const void* logits, int64_t rows, int C, int64_t ld, const float* u, sage_sampling h, int* labels, float* logp,
                         hipStream_t st) {
    constexpr int VL = RowType<T>::VL;
    for (int64_t r0 = 0; r0 < rows; r0 += LOGIT_LAUNCH_ROWS) {
        const dim3 grid((unsigned)std::min(rows - r0, LOGIT_LAUNCH_ROWS));
        const T* z = (const T*)logits + r0 * ld;
        float* lp = logp ? logp + r0 : nullptr;
        const auto go = [&](auto threads, auto staged) {
            constexpr int N = decltype(threads)::value;
            constexpr bool ST = decltype(staged)::value;
            const size_t lds = ST ? (size_t)((C + N * VL - 1) / (N * VL)) * N * 16 : 0;
            const auto kernel = sample_kernel<T, N, ST>;
            if (lds > 32768)
                if (hipError_t e = ensure_dynamic_lds((const void*)kernel, 65536); e != hipSuccess) return e;
            kernel<<<grid, N, lds, st>>>(z, C, ld, u + r0, h, labels + r0, lp);
            return hipGetLastError();
        };
        hipError_t e;
        using std::integral_constant;
        if (C <= 64 * 4 * VL) e = go(integral_constant<int, 64>{}, std::true_type{});
        else if (C <= 256 * 4 * VL) e = go(integral_constant<int, 256>{}, std::true_type{});
        else if (C <= 1024 * 4 * VL) e = go(integral_constant<int, 1024>{}, std::true_type{});
        else e = go(integral_constant<int, 1024>{}, std::false_type{});
        if (e != hipSuccess) return e;
        if (h.temperature_rows) h.temperature_rows += grid.x;
        if (h.top_k_rows) h.top_k_rows += grid.x;
        if (h.top_p_rows) h.top_p_rows += grid.x;
        if (h.min_p_rows) h.min_p_rows += grid.x;
    }
    return hipSuccess;
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
    const sage_sampling h = how ? *how : sage_sampling{1.f, 0, 1.f, 0.f, nullptr, nullptr, nullptr, nullptr};
    const auto go = dtype == SAGE_F32 ? sage::launch_sample<float> : sage::launch_sample<uint16_t>;
    if (go(logits, rows, (int)n_classes, ld, u, h, labels, logp, (hipStream_t)hip_stream) == hipSuccess) return SAGE_OK;
    (void)hipGetLastError();
    return SAGE_ERR_HIP;
}
