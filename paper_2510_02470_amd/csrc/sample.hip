// A label for every row of logits, drawn with a given random number: sage_sample (include/sage.h).
//
// A class's weight is the whole number rint(2^42 exp((z_j - max z) / T)). Sums of whole numbers do not depend on the order of
// addition, so that the label is a function of the row and its number alone, however a row is cut over threads; a weight is
// off by at most 2^-43 of the greatest, which moves the borders between the classes of a row of 2^20 by less than 2^-23 of
// it at worst and by 2^-33 as such errors fall out. Everything up to the comparison is done in 64 bits.
//
// A row has one work-group (a wave up to 256 vectors of 16 bytes, four up to 1024, sixteen up to 4096, from LDS; longer rows are read again
// by every pass, 8 waves twice on a CU, or 16 where there are no more than 256 rows). Passes: the maximum; for top-k a histogram of the
// distance to it, and a list of all that is in the K-th's bin and above, on which the rest is done; for top-p without it an approximate
// histogram of weights and one exact pass; otherwise one exact pass. An exact pass is bound by 64-bit arithmetic: 18 such instructions
// and about as many others a class, 30 us for a row of 131,072 on a CU, where a reading takes 10. So long bf16 rows without top-k are
// counted by value, in two passes (draw_by_value). 1024 rows of 131,072 bf16, the same ones again and again: the greatest 81 us, top-k 50 135,
// plain 122 (214 by classes), top-p 0.9 135 (410), 142 on other rows each time; 37 rows of 50,021 bf16 26 and 33 (31 and 52). A row that has
// to be left to the other passes costs 7% more.
#include <algorithm>
#include <type_traits>

#include "logit_rows.h"
#include "rows_meet.h"
#include "sage_internal.h"
#include "wave_ops.h"

namespace sage {
namespace {

// rint(2^42 e^x) for x <= 0: e^x = 2^n e^r with |r| <= ln 2 / 2, and e^r = 1 + r q(r), q of degree 9 through the Chebyshev points
// (relative error 2^-50; q computed for this with rational numbers). Exactly 2^42 at 0; 0 below -30, and for NaN (-inf at an infinite
// temperature). weight_bits is the weight and the bits of ROUND, which a sum takes off once.
constexpr double ROUND = 6755399441055744.0;  // 1.5 * 2^52: added and taken off again it rounds to a whole number
constexpr uint64_t ROUND_BITS = 0x4338000000000000ull;
__device__ __forceinline__ double fma_s(double a, double b, double c) {  // c in scalar registers (the compiler copies it to vector ones)
    double d;
    asm("v_fma_f64 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "s"(c));
    return d;
}
__device__ __forceinline__ uint64_t weight_bits(double x) {
    x = fmax(x, -31.0);  // 2^42 e^-31 rounds to 0
    const double t = __builtin_fma(x, 1.4426950408889634, ROUND);
    const double n = t - ROUND;
    const double r = __builtin_fma(n, -0.6931471805599453, x);
    double q = fma_s(0x1.289185613a3d6p-22, r, 0x1.72e1150d0c9b6p-19);
    q = fma_s(q, r, 0x1.a019b90d2ae7ap-16);
    q = fma_s(q, r, 0x1.a01994bd214e7p-13);
    q = fma_s(q, r, 0x1.6c16c1788bd90p-10);
    q = fma_s(q, r, 0x1.11111123c1f47p-7);
    q = fma_s(q, r, 0x1.5555555553d63p-5);
    q = fma_s(q, r, 0x1.5555555550d79p-3);
    q = fma_s(q, r, 0x1.0000000000001p-1);
    q = fma_s(q, r, 0x1.0000000000006p+0);
    const double p = __builtin_fma(q, r, 1.0);
    const uint64_t pb = (uint64_t)__double_as_longlong(p);
    const uint32_t hi = (uint32_t)(pb >> 32) + (((uint32_t)__double_as_longlong(t) + 42u) << 20);  // times 2^(n + 42), n >= -45
    const double w = __longlong_as_double((long long)((uint64_t)hi << 32 | (uint32_t)pb));
    return (uint64_t)__double_as_longlong(w + ROUND);
}
__device__ __forceinline__ uint64_t weight_of(double x) { return weight_bits(x) - ROUND_BITS; }

// Floats in their order as unsigned numbers; both zeros are one.
__device__ __forceinline__ uint32_t key_of(float z) {
    const uint32_t u = __float_as_uint(z + 0.f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) {
    return __uint_as_float(key ^ (key >> 31 ? 0x80000000u : 0xFFFFFFFFu));
}

// The classes kept so far: those above a value, and of those at it the ones before a place.
struct Cut {
    float value;
    int place;
    __device__ __forceinline__ bool keeps(float x, int j) const { return (x > value) | ((x == value) & (j < place)); }  // (| and &: no branches)
};
__device__ __forceinline__ Cut cut_after(uint64_t listed) {  // the last that is kept, as listed
    return Cut{value_of((uint32_t)(listed >> 32)), (int)~(uint32_t)listed + 1};
}

constexpr int U = 2;  // vectors of a thread that are read together

// What the THREADS threads of a row share.
template <int THREADS>
struct Shared {
    static constexpr int W = THREADS / 64;
    static constexpr int BITS = THREADS == 64 ? 8 : THREADS == 256 ? 10 : 11, BINS = 1 << BITS;  // of a histogram
    static constexpr int LIST = THREADS == 64 ? 128 : THREADS == 256 ? 512 : 1024;  // classes that are put in order one by one
    static constexpr int SEGS = THREADS >= 512 ? SAGE_MAX_CLASSES / (256 * U) : 16 * W;  // pieces of 64 * U vectors of the longest row
    uint64_t hist[BINS];  // a histogram (of counts, weights, or approximate weights)
    uint64_t seg[SEGS];   // sums of segments
    uint64_t part[W];
    float fpart[2 * W];
    union {
        struct {
            uint64_t lkey[LIST], skey[LIST];  // of listed classes key and place, one number in their common order
            uint64_t lw[LIST], sw[LIST];      // and weight
        };
        uint64_t table[4 * LIST + 2];  // weights by value (draw_by_value)
    };
    uint64_t found[2];
    unsigned listed, few;
    uint64_t answer;
};

__device__ __forceinline__ uint64_t mask_of(bool b) { return b ? ~0ull : 0ull; }


// A row as THREADS threads see it. A segment is 64 * U vectors, of which lane l of a wave has vectors l, 64 + l, ..; waves take
// segments in turn. Elements behind the row's end are -inf. STAGED: the first pass leaves the row in LDS, else it is read again by
// every pass (one segment on its way while one is worked on).
template <class T, int THREADS, bool STAGED>
struct Row {
    static constexpr int VL = RowType<T>::VL, W = THREADS / 64;
    static constexpr uint32_t NONE = sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u;  // -inf
    const T* z;
    int n, tid, count;  // count: segments of a wave
    u32x4* lds;         // count * THREADS * U

    __device__ __forceinline__ u32x4 fetch(int e0) const {
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
    __device__ __forceinline__ int place(int i, int u) const { return (((i * W + (tid >> 6)) * U + u) * 64 + (tid & 63)) * VL; }  // first element
    __device__ int segment_of(int j) const { return j / (64 * U * VL); }
    __device__ __forceinline__ void fetch_segment(int i, u32x4* v) const {
        if (((i * W + (tid >> 6)) + 1) * (U * 64 * VL) <= n) {  // (the same for the whole wave)
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = load16(z + place(i, u));
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = fetch(place(i, u));
        }
    }
    // f(segment of the wave, vectors), the last one if it says false; first: the pass that reads the row
    template <bool FIRST = false, class F>
    __device__ __forceinline__ void visit(F f) const {
        if constexpr (STAGED && !FIRST) {
#pragma unroll 1
            for (int i = 0; i < count; ++i) {
                u32x4 v[U];
#pragma unroll
                for (int u = 0; u < U; ++u) v[u] = lds[(i * U + u) * THREADS + tid];
                f(i, v);
            }
        } else {
            u32x4 v[U];
            fetch_segment(0, v);
#pragma unroll 1
            for (int i = 0; i < count; ++i) {
                u32x4 next[U];
                if (i + 1 < count) fetch_segment(i + 1, next);
                if constexpr (STAGED) {
#pragma unroll
                    for (int u = 0; u < U; ++u) lds[(i * U + u) * THREADS + tid] = v[u];
                }
                if constexpr (std::is_same<decltype(f(i, v)), bool>::value) {
                    if (!f(i, v)) break;
                } else {
                    f(i, v);
                }
#pragma unroll
                for (int u = 0; u < U; ++u) v[u] = next[u];
            }
        }
    }
    // f(value, element) for each element
    template <bool FIRST = false, class F>
    __device__ __forceinline__ void each(F f) const {
        visit<FIRST>([&](int i, const u32x4* v) __attribute__((always_inline)) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
#pragma unroll
                for (int k = 0; k < VL; ++k) {
                    if (k % 4 == 0) __builtin_amdgcn_sched_barrier(0);  // (more of them mixed would need more registers than there are)
                    f(RowType<T>::at(v[u], k), place(i, u) + k);
                }
            }
        });
    }
};

template <int CTRL>
__device__ __forceinline__ uint64_t dpp_move_u64(uint64_t v) {
    const uint32_t lo = (uint32_t)__builtin_amdgcn_mov_dpp((int)(uint32_t)v, CTRL, 0xF, 0xF, false);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_mov_dpp((int)(uint32_t)(v >> 32), CTRL, 0xF, 0xF, false);
    return (uint64_t)hi << 32 | lo;
}
template <int D>
__device__ __forceinline__ uint64_t add_swapped(uint64_t v) {
    const unsigned lo = (unsigned)v, hi = (unsigned)(v >> 32);
    const auto l = D == 16 ? __builtin_amdgcn_permlane16_swap(lo, lo, false, false) : __builtin_amdgcn_permlane32_swap(lo, lo, false, false);
    const auto h = D == 16 ? __builtin_amdgcn_permlane16_swap(hi, hi, false, false) : __builtin_amdgcn_permlane32_swap(hi, hi, false, false);
    return ((uint64_t)h[0] << 32 | l[0]) + ((uint64_t)h[1] << 32 | l[1]);
}
__device__ __forceinline__ uint64_t wave_sum(uint64_t v) {  // the same in every lane
    v += dpp_move_u64<DPP_XOR1>(v);
    v += dpp_move_u64<DPP_XOR2>(v);
    v += dpp_move_u64<DPP_HALF_MIRROR>(v);
    v += dpp_move_u64<DPP_MIRROR>(v);
    return add_swapped<32>(add_swapped<16>(v));
}
template <class A>
__device__ __forceinline__ A wave_scan(A v, int lane) {  // sums up to and with each lane
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const A o = __shfl_up(v, d, 64);
        if (lane >= d) v += o;
    }
    return v;
}
// (Waves may still be reading S.part when others return: whoever writes it, this or find_sum, has them all meet first.)
template <int THREADS>
__device__ __forceinline__ uint64_t group_sum(uint64_t v, Shared<THREADS>& S) {
    v = wave_sum(v);
    if constexpr (THREADS > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) S.part[threadIdx.x >> 6] = v;
        __syncthreads();
        v = S.part[0];
#pragma unroll
        for (int w = 1; w < THREADS / 64; ++w) v += S.part[w];
    }
    return v;
}

// What a random number takes of a sum.
__device__ __forceinline__ uint64_t share_of(float u, uint64_t total) {
    const uint64_t t = u > 0.f ? (uint64_t)((double)fminf(u, 1.f) * (double)total) : 0;
    return t >= total ? total - 1 : t;
}

// The first of `count` sums (sums[i], of LDS) up to which they come to more than t = want(their total): its number, and in S.found the
// sum of those before it and its own. The work-group meets first: the sums may just have been written, and what this
// writes may still be read.
template <int THREADS, class E, class F>
__device__ __forceinline__ int find_sum(Shared<THREADS>& S, E sums, int count, int tid, uint64_t& total, F want) {
    const int per = (count + THREADS - 1) / THREADS;
    uint64_t own = 0;
    __syncthreads();
    for (int i = 0; i < per; ++i)
        if (tid * per + i < count) own += sums[tid * per + i];
    const uint64_t incl = wave_scan(own, tid & 63);
    uint64_t before = incl - own;
    if (tid == 0) S.listed = 0;  // (none, should rounding leave the total out of reach)
    if constexpr (THREADS > 64) {
        if ((tid & 63) == 63) S.part[tid >> 6] = incl;
        __syncthreads();
        total = 0;
        uint64_t front = 0;
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w) {
            front = w < tid >> 6 ? front + S.part[w] : front;
            total += S.part[w];
        }
        before += front;
    } else {
        __syncthreads();
        total = __shfl(incl, 63, 64);
    }
    const uint64_t t = want(total);
    if (before <= t && before + own > t) {
        int i = tid * per;
        while (i < tid * per + per - 1 && i < count - 1 && before + sums[i] <= t) before += sums[i++];
        S.listed = (unsigned)i;
        S.found[0] = before;
        S.found[1] = sums[i];
    }
    __syncthreads();
    return (int)S.listed;
}

// The element of a segment at which the sum of f (value, element) passes t, `before` being the sum before the segment.
template <class T, int THREADS, bool STAGED, class F>
__device__ __forceinline__ int locate_at(const Row<T, THREADS, STAGED>& r, Shared<THREADS>& S, int seg, uint64_t before, uint64_t t, F f) {
    constexpr int VL = RowType<T>::VL, W = THREADS / 64;
    const int lane = r.tid & 63, wave = r.tid >> 6;
    if (wave == seg % W) {
        bool done = false;
#pragma unroll 1
        for (int q = 0; q < U; ++q) {
            const int e0 = ((seg * U + q) * 64 + lane) * VL;
            const u32x4 v = r.fetch(e0);
            uint64_t w[VL], own = 0;
#pragma unroll
            for (int k = 0; k < VL; ++k) {
                w[k] = f(RowType<T>::at(v, k), e0 + k);
                own += w[k];
            }
            const uint64_t incl = wave_scan(own, lane);
            uint64_t mine = before + incl - own;
            if (!done && mine <= t && mine + own > t) {
                int at = 0;
#pragma unroll
                for (int k = 0; k < VL - 1; ++k) {  // (no indexing of registers)
                    if (at == k && mine + w[k] <= t) {
                        mine += w[k];
                        ++at;
                    }
                }
                S.answer = (uint64_t)(e0 + at);
            }
            before += __shfl(incl, 63, 64);
            done = before > t;
        }
    }
    __syncthreads();
    return (int)S.answer;
}

// With the sums of segments in LDS: the element at which the sum of f (value, element) passes t, the sum of all being total.
template <class T, int THREADS, bool STAGED, class F>
__device__ __forceinline__ int locate_in(const Row<T, THREADS, STAGED>& r, Shared<THREADS>& S, uint64_t& total, const float* u, uint64_t t0, F f) {
    const int seg = find_sum<THREADS>(S, (const uint64_t*)S.seg, r.count * r.W, r.tid, total,
                                      [&](uint64_t all) { return u ? share_of(*u, all) : t0; });
    return locate_at(r, S, seg, S.found[0], u ? share_of(*u, total) : t0, f);
}

// The same from the row alone. keeps(value, element): whether it counts at all; f(value, element): what it counts if so, a whole number.
template <class T, int THREADS, bool STAGED, class K, class F>
__device__ __forceinline__ int locate(const Row<T, THREADS, STAGED>& r, Shared<THREADS>& S, uint64_t& total, const float* u, uint64_t t0, K keeps, F f) {
    constexpr int VL = RowType<T>::VL, W = THREADS / 64;
    __syncthreads();
    r.visit([&](int i, const u32x4* v) __attribute__((always_inline)) {
        uint64_t own = 0;
#pragma unroll
        for (int q = 0; q < U; ++q) {
            __builtin_amdgcn_sched_barrier(0);
            bool any = false;
#pragma unroll
            for (int k = 0; k < VL; ++k) any |= keeps(RowType<T>::at(v[q], k), r.place(i, q) + k);
            if (__any(any)) {
#pragma unroll
                for (int k = 0; k < VL; ++k) {
                    if (k % 4 == 0) __builtin_amdgcn_sched_barrier(0);
                    const float x = RowType<T>::at(v[q], k);
                    const uint64_t w = f(x, r.place(i, q) + k);
                    own += w & mask_of(keeps(x, r.place(i, q) + k));
                }
            }
        }
        const uint64_t s = wave_sum(own);
        if ((r.tid & 63) == 0) S.seg[i * W + (r.tid >> 6)] = s;
    });
    return locate_in(r, S, total, u, t0, [&](float x, int j) __attribute__((always_inline)) { return f(x, j) & mask_of(keeps(x, j)); });
}

// The bins of a histogram: equal parts of the distance to the maximum, everything beyond `range` in the last.
struct Bins {
    float m, scale, last;
    // (a range of 0 would make 0 * infinity of the maximum's distance)
    __device__ Bins(float m_, float range, int bins) : m(m_), scale(fminf((float)(bins - 1) / range, 1e30f)), last((float)(bins - 1)) {}
    __device__ __forceinline__ int operator()(float x) const { return (int)fminf((m - x) * scale, last); }
};

// The least value whose bin is at most b (bins fall with the value).
__device__ __forceinline__ float least_of_bin(const Bins& bins, int b) {
    uint32_t lo = key_of(-INFINITY), hi = key_of(bins.m);  // hi: in bin 0
    if (b < 0) return INFINITY;
    while (lo < hi) {
        const uint32_t mid = lo + (hi - lo) / 2;
        if (bins(value_of(mid)) <= b) hi = mid;
        else lo = mid + 1;
    }
    return value_of(lo);
}

template <int THREADS>
__device__ __forceinline__ void clear_histogram(Shared<THREADS>& S, int tid) {
    __syncthreads();
    for (int i = tid; i < S.BINS; i += THREADS) S.hist[i] = 0;
    __syncthreads();
}

// Classes whose bin is at most `bin` (or just it), as long as there is room: how many there are.
template <class T, int THREADS, bool STAGED, class M, class F>
__device__ __forceinline__ int collect(const Row<T, THREADS, STAGED>& r, Shared<THREADS>& S, M member, F f) {
    __syncthreads();
    if (r.tid == 0) S.listed = 0;
    __syncthreads();
    r.each([&](float x, int j) __attribute__((always_inline)) {
        if (member(x, j)) {
            const uint64_t w = f(x, j);
            if (w) {
                const unsigned p = atomicAdd(&S.listed, 1u);
                if (p < Shared<THREADS>::LIST) {
                    S.lkey[p] = (uint64_t)key_of(x) << 32 | (uint32_t)~j;  // greater: earlier in the order
                    S.lw[p] = w;
                }
            }
        }
    });
    __syncthreads();
    return (int)S.listed;
}

// The shortest front part of the order (value descending, place ascending) whose f sum to more than t, as a cut; the sum of all f is more
// than t. For any f and any row: a histogram over the distance to the maximum leaves one bin; its members are put in order
// one by one, or, if they are many, told apart by more histograms over their keys first.
template <class T, int THREADS, bool STAGED, class F>
__device__ __forceinline__ Cut front(const Row<T, THREADS, STAGED>& r, Shared<THREADS>& S, uint64_t t, const Bins& bins, F f) {
    constexpr int LIST = Shared<THREADS>::LIST, BITS = Shared<THREADS>::BITS;
    uint32_t prefix = 0;
    int shift = 33;  // keys of the set agree with prefix from bit `shift` on; 33: the set is everything, 32: a bin of values
    float from = INFINITY, least = -INFINITY;
    uint64_t above = 0;
    auto member = [&](float x) __attribute__((always_inline)) {
        return (x < from) & (x >= least) & (shift >= 32 || key_of(x) >> (shift & 31) == prefix);
    };
    for (;;) {
        const int step = shift < BITS ? shift : BITS, low = shift - step;
        clear_histogram(S, r.tid);
        r.each([&](float x, int j) __attribute__((always_inline)) {
            if (member(x)) {
                const uint64_t w = f(x, j);
                const int b = shift == 33 ? bins(x) : (1 << step) - 1 - (int)(key_of(x) >> low & ((1u << step) - 1));
                if (w) atomicAdd((unsigned long long*)&S.hist[b], (unsigned long long)w);
            }
        });
        uint64_t total;
        const int b = find_sum<THREADS>(S, (const uint64_t*)S.hist, S.BINS, r.tid, total, [&](uint64_t) { return t - above; });
        above += S.found[0];
        if (shift == 33) {
            from = least_of_bin(bins, b - 1);
            least = least_of_bin(bins, b);
            shift = 32;
        } else {
            prefix = prefix << step | ((1u << step) - 1 - (uint32_t)b);
            shift = low;
        }
        const int count = collect(r, S, [&](float x, int) __attribute__((always_inline)) { return member(x); }, f);
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
            return cut_after(S.answer);
        }
        if (shift == 0) {  // many equal values: their f are equal too, and the first of them are meant
            const int last = locate(r, S, total, nullptr, t - above, [&](float x, int) __attribute__((always_inline)) { return member(x); }, f);
            return Cut{value_of(prefix), last + 1};
        }
    }
}

// Of the members of the list (member(i)), in falling order of key(i), the one up to which f(i) sum to more than t, `above` being the sum
// before the first of them: its key. They are few as a rule (of one bin, or of one segment): each looks at all others.
template <int THREADS, class M, class K, class F>
__device__ __forceinline__ uint64_t passing(Shared<THREADS>& S, int count, int tid, uint64_t above, uint64_t t, M member, K key, F f) {
    __syncthreads();
    if (tid == 0) S.few = 0;
    __syncthreads();
    for (int i = tid; i < count; i += THREADS)
        if (member(i)) {
            const unsigned p = atomicAdd(&S.few, 1u);
            S.skey[p] = key(i);
            S.sw[p] = f(i);
        }
    __syncthreads();
    const int few = (int)S.few;
    for (int i = tid; i < few; i += THREADS) {
        const uint64_t mine = S.skey[i];
        uint64_t before = above;
#pragma unroll 8
        for (int k = 0; k < few; ++k) before += S.skey[k] > mine ? S.sw[k] : 0;
        if (before <= t && before + S.sw[i] > t) S.answer = mine;
    }
    __syncthreads();
    return S.answer;
}

// The listed classes (those of bins up to b, in which the K-th of the order is, `before` of them in the bins before it) reduced by top-k,
// top-p and min-p, and the draw.
template <class T, int THREADS, bool STAGED>
__device__ __forceinline__ int draw_listed(const Row<T, THREADS, STAGED>& r, Shared<THREADS>& S, int count, int K, const Bins& bins, int b,
                                           uint64_t before, float P, double border, double md, float u, uint64_t& total) {
    const int tid = r.tid;
    auto value = [&](int i) __attribute__((always_inline)) { return value_of((uint32_t)(S.lkey[i] >> 32)); };
    auto key = [&](int i) __attribute__((always_inline)) { return S.lkey[i]; };
    auto weight = [&](int i) __attribute__((always_inline)) { return S.lw[i]; };
    uint64_t last = passing(S, count, tid, before, (uint64_t)K - 1, [&](int i) __attribute__((always_inline)) { return bins(value(i)) == b; }, key,
                            [](int) { return 1ull; });
    if (P < 1.f) {
        clear_histogram(S, tid);
        for (int i = tid; i < count; i += THREADS)
            if (S.lkey[i] >= last) atomicAdd((unsigned long long*)&S.hist[bins(value(i))], (unsigned long long)S.lw[i]);
        uint64_t t = 0;
        const int at = find_sum<THREADS>(S, (const uint64_t*)S.hist, S.BINS, tid, total, [&](uint64_t all) {
            const double q = ceil((double)P * (double)all);
            return t = q >= 1.0 ? (uint64_t)q - 1 : 0;
        });
        const uint64_t above = S.found[0], top_k = last;
        last = passing(S, count, tid, above, t,
                       [&](int i) __attribute__((always_inline)) { return (S.lkey[i] >= top_k) & (bins(value(i)) == at); }, key, weight);
    }
    // the draw: the segments' sums, and the classes of one segment by their places
    auto kept = [&](int i) __attribute__((always_inline)) { return (S.lkey[i] >= last) & ((double)value(i) - md >= border); };
    auto place = [&](int i) __attribute__((always_inline)) { return (int)~(uint32_t)S.lkey[i]; };
    __syncthreads();
    for (int i = tid; i < r.count * r.W; i += THREADS) S.seg[i] = 0;
    __syncthreads();
    for (int i = tid; i < count; i += THREADS)
        if (kept(i)) atomicAdd((unsigned long long*)&S.seg[r.segment_of(place(i))], (unsigned long long)S.lw[i]);
    const int seg = find_sum<THREADS>(S, (const uint64_t*)S.seg, r.count * r.W, tid, total, [&](uint64_t all) { return share_of(u, all); });
    const uint64_t base = S.found[0];
    return (int)~(uint32_t)passing(S, count, tid, base, share_of(u, total),
                                   [&](int i) __attribute__((always_inline)) { return kept(i) & (r.segment_of(place(i)) == seg); },
                                   [&](int i) __attribute__((always_inline)) { return (uint64_t)(uint32_t)S.lkey[i]; }, weight);
}

// ---- long bf16 rows without top-k -------------------------------------------------------------------------------

// A bf16 of magnitude 2^-9 to 2^7 is one of 4096 values, and a long row has few of them, each many times. One pass counts them; weights,
// the border of top-p and what min-p leaves are found from values and counts (with 4096 exponentials instead of one for every class), and
// a second pass adds up a table's entries: 8 instructions a class and a reading of LDS instead of 36. Smaller magnitudes, one in a
// thousand, are listed; a row with more of them, or with greater ones that matter, is left to the other passes. Both passes treat a class like
// any other and see to what is not counted once a vector or afterwards: 135 us for 1024 rows of 131,072 with top-p, 157 with branches for
// each class.
constexpr int VALUES = 4096, HALF = VALUES / 2, MAX_TINY = 1024;
constexpr unsigned VALUES_FROM = 118u << 7;  // 2^-9

__device__ __forceinline__ unsigned bits_of(const u32x4& v, int k) { return k & 1 ? v[k >> 1] >> 16 : v[k >> 1] & 0xFFFFu; }
__device__ __forceinline__ unsigned above_of(const u32x4& v, int k) { return (bits_of(v, k) & 0x7FFFu) - VALUES_FROM; }
__device__ __forceinline__ int number_of(const u32x4& v, int k, unsigned above) {  // in rising order; -1 and VALUES for above = HALF
    return HALF + (int)(above ^ (unsigned)((int)(k & 1 ? v[k >> 1] : v[k >> 1] << 16) >> 31));
}
__device__ __forceinline__ unsigned value_bits(int i) { return i < HALF ? 0x8000u + VALUES_FROM + (HALF - 1 - i) : VALUES_FROM + (i - HALF); }
__device__ __forceinline__ float bf16_value(unsigned bits) { return __uint_as_float(bits << 16); }

// The sums of the values in falling order, those of small magnitude as one in the middle.
struct ValueSums {
    const uint32_t* counts;
    const uint64_t* table;
    uint64_t tiny;
    __device__ __forceinline__ uint64_t operator[](int i) const {
        if (i == HALF) return tiny;
        const int n = VALUES - 1 - i + (i > HALF);
        return counts[n] * table[n];
    }
};
// Sums of a segment: of weights below, of classes at the border from this bit on (1024 classes of up to 2^42).
constexpr int AT_BORDER = 53;
struct BorderCounts {
    const uint64_t* seg;
    __device__ __forceinline__ uint64_t operator[](int i) const { return seg[i] >> AT_BORDER; }
};

// The label, m and the total; or -1: a row for the other passes.
template <class T, int THREADS, bool STAGED>
__device__ __forceinline__ int draw_by_value(const Row<T, THREADS, STAGED>& r, Shared<THREADS>& S, double inv, float P, double border, float u,
                                             float& m, uint64_t& total) {
    constexpr int VL = RowType<T>::VL, W = THREADS / 64, SEGMENTS = SAGE_MAX_CLASSES / (64 * U * VL);
    static_assert(VL == 8 && 64 * U * VL <= 1024 && Shared<THREADS>::BINS * 2 >= VALUES && Shared<THREADS>::LIST * 4 >= VALUES, "room in LDS");
    static_assert(SEGMENTS + MAX_TINY <= Shared<THREADS>::SEGS, "room behind the segments");
    const int tid = r.tid;
    uint32_t* const counts = (uint32_t*)S.hist;
    uint64_t* const tiny = S.seg + SEGMENTS;    // place and bits
    uint64_t* const table = S.table + 1;        // (at its ends 0, for what is not counted)
    if (tid == 0) S.few = 0;
    clear_histogram(S, tid);
    float low = -INFINITY;  // greatest of the values below all counted ones
    bool other = false;     // NaN, or above all counted ones
    r.template visit<true>([&](int i, const u32x4* v) __attribute__((always_inline)) {
#pragma unroll
        for (int q = 0; q < U; ++q) {
            unsigned most = 0;
#pragma unroll
            for (int k = 0; k < VL; ++k) {
                if (k % 4 == 0) __builtin_amdgcn_sched_barrier(0);
                const unsigned above = above_of(v[q], k);
                if (above < (unsigned)HALF) atomicAdd(&counts[number_of(v[q], k, above)], 1u);
                most = max(most, above);
            }
            if (most >= (unsigned)HALF) {
#pragma unroll
                for (int k = 0; k < VL; ++k) {
                    const unsigned h = bits_of(v[q], k), above = above_of(v[q], k);
                    if ((int)above < 0) {
                        const unsigned p = atomicAdd(&S.few, 1u);
                        if (p < (unsigned)MAX_TINY) tiny[p] = (uint64_t)(r.place(i, q) + k) << 16 | h;
                    } else if (above >= (unsigned)HALF) {
                        if (h >> 15 && h <= 0xFF80u) low = fmaxf(low, bf16_value(h));
                        else other = true;
                    }
                }
            }
        }
        return (int)__builtin_amdgcn_readfirstlane(*(volatile unsigned*)&S.few) <= MAX_TINY;
    });
    low = group_reduce<THREADS>(other ? INFINITY : low, S.fpart, [](float a, float b) { return fmaxf(a, b); });
    constexpr int PER = VALUES / THREADS;
    float first = -1.f;
#pragma unroll
    for (int i = 0; i < PER; ++i)
        if (counts[tid * PER + i]) first = (float)(tid * PER + i);
    first = group_reduce<THREADS>(first, S.fpart + W, [](float a, float b) { return fmaxf(a, b); });
    const int few = (int)S.few;
    if (low == INFINITY || first < 0.f || few > (first >= (float)HALF ? MAX_TINY : 0)) return -1;
    m = bf16_value(value_bits((int)first));
    const double md = m;
    if (((double)low - md) * inv > -29.9) return -1;  // (below -43 ln 2 there is no weight)
    auto weight = [&](float x) __attribute__((always_inline)) { return weight_of(((double)x - md) * inv); };
    for (int i = tid; i < VALUES; i += THREADS) table[i] = counts[i] ? weight(bf16_value(value_bits(i))) : 0;
    if (tid == 0) table[-1] = table[VALUES] = 0;
    uint64_t tiny_sum = 0;
    for (int i = tid; i < few; i += THREADS) tiny_sum += weight(bf16_value((unsigned)tiny[i] & 0xFFFFu));
    tiny_sum = group_sum<THREADS>(tiny_sum, S);  // (the table is there too)
    int last = -1;             // the last value that top-p keeps any of
    uint64_t kept = 0, at_last = 0;  // so many, if not all of it, of this weight
    if (P < 1.f) {
        uint64_t t = 0;
        const int at = find_sum<THREADS>(S, ValueSums{counts, table, tiny_sum}, VALUES + 1, tid, total, [&](uint64_t all) {
            const double q = ceil((double)P * (double)all);
            return t = q >= 1.0 ? (uint64_t)q - 1 : 0;
        });
        if (at == HALF) return -1;
        last = VALUES - 1 - at + (at > HALF);
        at_last = table[last];
        kept = (t - S.found[0]) / at_last + 1;
        if (kept >= counts[last]) kept = 0;
    }
    const float value = last >= 0 ? bf16_value(value_bits(last)) : -INFINITY;
    __syncthreads();
    // what is left of the table; a value kept in part is counted
    for (int i = tid; i < VALUES; i += THREADS) {
        if (i == last && kept) table[i] = 1ull << AT_BORDER;
        else if (i < last || (double)bf16_value(value_bits(i)) - md < border) table[i] = 0;
    }
    if ((double)value - md < border) at_last = 0;
    auto drawn = [&](float x) __attribute__((always_inline)) { return weight(x) & mask_of((double)x - md >= border); };
    __syncthreads();
    r.visit([&](int i, const u32x4* v) __attribute__((always_inline)) {
        uint64_t own = 0;
#pragma unroll
        for (int q = 0; q < U; ++q) {
#pragma unroll
            for (int k = 0; k < VL; ++k) {
                if (k % 4 == 0) __builtin_amdgcn_sched_barrier(0);
                own += table[number_of(v[q], k, min(above_of(v[q], k), (unsigned)HALF))];
            }
        }
        const uint64_t s = wave_sum(own);
        if ((tid & 63) == 0) S.seg[i * W + (tid >> 6)] = s;
    });
    __syncthreads();
    if (last < HALF)
        for (int i = tid; i < few; i += THREADS)
            atomicAdd((unsigned long long*)&S.seg[r.segment_of((int)(tiny[i] >> 16))], (unsigned long long)drawn(bf16_value((unsigned)tiny[i] & 0xFFFFu)));
    Cut cut{value, 0x7FFFFFFF};
    if (kept) {
        const int seg = find_sum<THREADS>(S, BorderCounts{S.seg}, r.count * W, tid, total, [&](uint64_t) { return kept - 1; });
        const uint64_t before = S.found[0];
        cut.place = 1 + locate_at(r, S, seg, before, kept - 1, [&](float x, int) __attribute__((always_inline)) { return x == value ? 1ull : 0ull; });
        for (int i = tid; i < r.count * W; i += THREADS) {
            const uint64_t s = S.seg[i], n = i < seg ? s >> AT_BORDER : i == seg ? kept - before : 0;
            S.seg[i] = (s & ((1ull << AT_BORDER) - 1)) + n * at_last;
        }
    }
    return locate_in(r, S, total, &u, 0, [&](float x, int e) __attribute__((always_inline)) { return drawn(x) & mask_of(cut.keeps(x, e)); });
}

template <class T, int THREADS, bool STAGED>
__global__ __launch_bounds__(THREADS, THREADS == 512 ? 4 : 1) void sample_kernel(const T* __restrict__ logits, int C, int64_t ld, const float* __restrict__ u_rows,
                                                         sage_sampling how, int* __restrict__ labels, float* __restrict__ logp) {
    __shared__ Shared<THREADS> S;
    constexpr int VL = RowType<T>::VL, W = THREADS / 64, LIST = Shared<THREADS>::LIST;
    extern __shared__ u32x4 staged[];
    const int64_t row = blockIdx.x;
    const Row<T, THREADS, STAGED> r{logits + row * ld, C, (int)threadIdx.x, (C + THREADS * U * VL - 1) / (THREADS * U * VL), staged};
    const float T32 = how.temperature_rows ? how.temperature_rows[row] : how.temperature;
    const float P32 = how.top_p_rows ? how.top_p_rows[row] : how.top_p;
    const float M32 = how.min_p_rows ? how.min_p_rows[row] : how.min_p;
    const int K = how.top_k_rows ? how.top_k_rows[row] : how.top_k;
    const float u = u_rows[row];

    auto done = [&](int j, float m, double inv, uint64_t total) __attribute__((always_inline)) {
        if (r.tid != 0) return;
        j = (int)min((unsigned)j, (unsigned)C - 1);  // (logits that change between the passes may leave no class: nothing is read behind the row)
        labels[row] = j;
        if (logp) logp[row] = (float)(((double)RowType<T>::widen(r.z[j]) - (double)m) * inv - log((double)total * 0x1p-42));
    };
    const double inv = 1.0 / (double)T32;
    double border = -INFINITY;  // z - m of the least class that min-p keeps; never above 0: the greatest class stays
    if (M32 > 0.f) border = M32 < 1.f ? (double)T32 * log((double)M32) : 0.0;  // (an infinite temperature times ln 1 is no number)
    if constexpr (sizeof(T) == 2 && THREADS >= 512) {
        // (short rows without top-p take as long either way: 1024 of 16,384 51 us by classes and 54 by values, of 32,768 79 and 67)
        if (T32 > 0.f && !(K > 0 && K < C) && (P32 < 1.f || C > 16384)) {
            float m;
            uint64_t total = 0;
            const int j = draw_by_value(r, S, inv, P32, border, u, m, total);
            if (j >= 0) return done(j, m, inv, total);
            __syncthreads();
        }
    }
    float m = -INFINITY, low = INFINITY;  // greatest, and least finite
    bool nan = false;
    r.template each<true>([&](float x, int) __attribute__((always_inline)) {
        m = fmaxf(m, x);
        low = x > -INFINITY ? fminf(low, x) : low;
        nan |= x != x;
    });
    if (nan) m = INFINITY;  // either is no distribution
    m = group_reduce<THREADS>(m, S.fpart, [](float a, float b) { return fmaxf(a, b); });
    low = group_reduce<THREADS>(low, S.fpart + W, [](float a, float b) { return fminf(a, b); });
    if (!(fabsf(m) < INFINITY)) {
        if (r.tid == 0) {
            labels[row] = -1;
            if (logp) logp[row] = __builtin_nanf("");
        }
        return;
    }
    uint64_t total = 0;
    int j = -1;
    if (!(T32 > 0.f)) {
        j = locate(r, S, total, nullptr, 0, [&](float x, int) __attribute__((always_inline)) { return x == m; }, [](float, int) { return 1ull; });
        if (r.tid == 0) {
            labels[row] = j;
            if (logp) logp[row] = 0.f;
        }
        return;
    }
    const double md = m;
    const float spread = fminf(m - low, 3e38f);
    auto bits = [&](float x) __attribute__((always_inline)) { return weight_bits(((double)x - md) * inv); };
    auto weight = [&](float x, int) __attribute__((always_inline)) { return bits(x) - ROUND_BITS; };
    Cut cut{-INFINITY, 0};  // (-inf has no weight)
    if (K > 0 && K < C) {
        // the bin that the K-th is in; if all up to it can be listed, the rest is done on the list
        const Bins kbins(m, fminf(spread, 64.f), S.BINS);
        uint32_t* counts = (uint32_t*)S.hist;
        clear_histogram(S, r.tid);
        r.each([&](float x, int) __attribute__((always_inline)) {
            if (x > -INFINITY) atomicAdd(&counts[kbins(x)], 1u);  // (masked classes, all in one bin, would wait for each other)
        });
        uint64_t all;
        const int b = find_sum<THREADS>(S, (const uint32_t*)counts, S.BINS, r.tid, all, [&](uint64_t) { return (uint64_t)K - 1; });
        const uint64_t before = S.found[0], through = before + S.found[1];
        if (all <= (uint64_t)K) {
            // every class that has a weight is among the first K
        } else if (through <= LIST) {
            const float least = least_of_bin(kbins, b);
            const int count = collect(r, S, [&](float x, int) __attribute__((always_inline)) { return (x >= least) & (x > -INFINITY); },
                                      [&](float x, int e) __attribute__((always_inline)) { return weight(x, e) | 1ull << 63; });
            for (int i = r.tid; i < count; i += THREADS) S.lw[i] &= ~(1ull << 63);  // (without a weight they count for top-k all the same)
            __syncthreads();
            j = draw_listed(r, S, count, K, kbins, b, before, P32, border, md, u, total);
        } else {
            cut = front(r, S, (uint64_t)K - 1, kbins, [&](float x, int) __attribute__((always_inline)) { return x > -INFINITY ? 1ull : 0ull; });
        }
    }
    const Bins bins(m, fminf(spread, 30.f * T32), S.BINS);
    const bool cut_before = cut.place > 0;  // a top-k of more than the list holds: any row, any order of the cuts
    if (cut_before && P32 < 1.f) {
        uint64_t sum = 0;
        r.each([&](float x, int e) __attribute__((always_inline)) { sum += weight(x, e) & mask_of(cut.keeps(x, e)); });
        sum = group_sum<THREADS>(sum, S);
        const double q = ceil((double)P32 * (double)sum);
        const Cut k_cut = cut;
        cut = front(r, S, q >= 1.0 ? (uint64_t)q - 1 : 0, bins,
                    [&](float x, int e) __attribute__((always_inline)) { return weight(x, e) & mask_of(k_cut.keeps(x, e)); });
    }
    if (j < 0 && P32 < 1.f && !cut_before) {
        // An approximate histogram says in which bin the border is likely to be. One exact pass then has the sum of all, for each segment the
        // sum of what is in the bins before, and a list of the bin itself, whose kept members are added to the segments one by one.
        const float c2 = (float)(inv * 1.4426950408889634);
        clear_histogram(S, r.tid);
        r.each([&](float x, int) __attribute__((always_inline)) {
            // (whole numbers: adding floats in LDS takes ten times as long)
            const uint32_t w = (uint32_t)__builtin_amdgcn_exp2f(fmaf(x - m, c2, 31.f));
            if (w) atomicAdd((unsigned long long*)&S.hist[bins(x)], (unsigned long long)w);
        });
        const int b = find_sum<THREADS>(S, (const uint64_t*)S.hist, S.BINS, r.tid, total, [&](uint64_t all) { return share_of(P32, all); });
        __syncthreads();
        if (r.tid == 0) S.listed = 0;
        __syncthreads();
        const float from = least_of_bin(bins, b - 1), least = least_of_bin(bins, b);
        uint64_t sum = 0, before = 0;
        r.visit([&](int i, const u32x4* v) __attribute__((always_inline)) {
            uint64_t own = 0;
#pragma unroll
            for (int q = 0; q < U; ++q) {
#pragma unroll
                for (int k = 0; k < VL; ++k) {
                    if (k % 4 == 0) __builtin_amdgcn_sched_barrier(0);
                    const float x = RowType<T>::at(v[q], k);
                    const int e = r.place(i, q) + k;
                    const uint64_t w = bits(x) - ROUND_BITS;
                    sum += w;
                    own += w & mask_of(x >= from);
                    if ((x < from) & (x >= least) & (w != 0)) {
                        const unsigned p = atomicAdd(&S.listed, 1u);
                        if (p < LIST) {
                            S.lkey[p] = (uint64_t)key_of(x) << 32 | (uint32_t)~e;
                            S.lw[p] = w;
                        }
                    }
                }
            }
            before += own;
            const uint64_t s = wave_sum(own);
            if ((r.tid & 63) == 0) S.seg[i * W + (r.tid >> 6)] = s;
        });
        sum = group_sum<THREADS>(sum, S);
        before = group_sum<THREADS>(before, S);
        const double q = ceil((double)P32 * (double)sum);
        const uint64_t need = q >= 1.0 ? (uint64_t)q : 1;
        const int listed = (int)S.listed;
        uint64_t listed_sum = 0;
        if (listed <= LIST) {
            for (int i = r.tid; i < listed; i += THREADS) listed_sum += S.lw[i];
            listed_sum = group_sum<THREADS>(listed_sum, S);
        }
        if (before < need && before + listed_sum >= need) {
            for (int i = r.tid; i < listed; i += THREADS) {
                const uint64_t key = S.lkey[i];
                uint64_t ahead = before;
#pragma unroll 8
                for (int k = 0; k < listed; ++k) ahead += S.lkey[k] > key ? S.lw[k] : 0;
                if (ahead < need) {
                    atomicAdd((unsigned long long*)&S.seg[r.segment_of((int)~(uint32_t)key)], (unsigned long long)S.lw[i]);
                    if (ahead + S.lw[i] >= need) S.answer = key;
                }
            }
            __syncthreads();
            cut = cut_after(S.answer);
            __syncthreads();
            if ((double)cut.value - md >= border)  // (else min-p keeps less)
                j = locate_in(r, S, total, &u, 0, [&](float x, int e) __attribute__((always_inline)) { return weight(x, e) & mask_of(cut.keeps(x, e)); });
        } else {
            cut = front(r, S, need - 1, bins, weight);
        }
    }
    if (j < 0)
        j = locate(r, S, total, &u, 0,
                   [&](float x, int e) __attribute__((always_inline)) { return ((double)x - md >= border) & cut.keeps(x, e) & (e < C); }, weight);
    done(j, m, inv, total);
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
            const size_t lds = ST ? (size_t)((C + N * U * VL - 1) / (N * U * VL)) * N * U * 16 : 0;
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
        else if (rows <= 256) e = go(integral_constant<int, 1024>{}, std::false_type{});  // a CU has one of them, if any
        else e = go(integral_constant<int, 512>{}, std::false_type{});
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
    const int64_t ea = da == SAGE_BF16 ? 2 : 4, eb = db == SAGE_BF16 ? 2 : 4;
    const uintptr_t a1 = a0 + ((rows - 1) * lda + C) * ea, b1 = b0 + ((rows - 1) * ldb + C) * eb;
    if (a0 >= b1 || b0 >= a1) return false;
    // (rows of other distances are taken to meet where their spans do)
    return rows == 1 || lda * ea != ldb * eb || rows_meet((int64_t)(b0 - a0), lda * ea, rows, C * ea, C * eb);
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
