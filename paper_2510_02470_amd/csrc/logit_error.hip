// Cross-entropy of rows of logits and its gradient with respect to them: sage_logit_error (include/sage.h).
//
// With m = max z, e_j = exp(z_j - m) and R = the sum of e_j over the classes other than the label y:
//     loss = ln((R + e_y) / e_y) = log1p(R / e_y),   E_j = w e_j / (R + e_y),   E_y = -w R / (R + e_y).
// The label is left out of the sum, because loss and E_y are differences of nearly equal numbers when written with p_y: a
// learnt example has p_y = 1 - 1e-6, of which fp32 keeps one digit of the part that matters.
#include <algorithm>

#include "logit_rows.h"
#include "sage_internal.h"

namespace sage {
namespace {

constexpr int EB = 1024;

// e^(x - m): the difference is exact or rounded once; the product with log2 e is carried to twice the width.
__device__ __forceinline__ float exp_diff(float x, float m) {
    const float d = x - m;
    const float L = 1.44269502f, L2 = 1.92596299e-8f;  // log2 e = L + L2
    const float t = d * L;
    const float r = fmaf(d, L, -t) + d * L2;
    const float e = __builtin_amdgcn_exp2f(t);
    return t <= -126.f ? 0.f : fmaf(e, r * 0.693147181f, e);  // (r is no number where d is infinite; a NaN stays one)
}

// ln((rest + ey) / ey); where ey is too small for an fp32 the label's distance to the maximum is all that counts beside the sum.
__device__ __forceinline__ float row_loss(float rest, float ey, float zy, float m) {
    if (rest + ey == 0.f) return INFINITY;
    if (ey < 0x1p-100f) return (float)(log((double)rest) + ((double)m - (double)zy));
    return (float)log1p((double)rest / (double)ey);
}

// One work-group a row: maximum, sum, and the row again for the answer.
template <class T, class TE>
__global__ __launch_bounds__(EB) void logit_error_kernel(const T* logits, int64_t C, int64_t ld, const int* __restrict__ labels,
                                                         const float* __restrict__ weights, TE* E, int64_t ldE, float* __restrict__ loss) {
    __shared__ float part[2][EB / 64];
    const int64_t row = blockIdx.x;
    const T* z = logits + row * ld;
    TE* out = E ? E + row * ldE : nullptr;
    const int y = labels[row];
    const int tid = threadIdx.x;
    if (y < 0) {
        if (out)
            for (int64_t j = tid; j < C; j += EB) out[j] = 0;
        if (loss && tid == 0) loss[row] = 0.f;
        return;
    }
    constexpr int VL = RowType<T>::VL;
    const bool known = y < C;
    const float zy = known ? RowType<T>::widen(z[y]) : __builtin_nanf("");
    float m = zy;
    for (int64_t e0 = (int64_t)tid * VL; e0 < C; e0 += EB * VL) {
        float x[VL];
        row_floats(z, e0, C, -INFINITY, x);
#pragma unroll
        for (int i = 0; i < VL; ++i) m = fmaxf(m, x[i]);
    }
    m = group_reduce<EB>(m, part[0], [](float a, float b) { return fmaxf(a, b); });
    if (m == -INFINITY) m = 0.f;  // no class is possible: every e is 0
    float rest = 0.f;
    for (int64_t e0 = (int64_t)tid * VL; e0 < C; e0 += EB * VL) {
        float x[VL];
        row_floats(z, e0, C, -INFINITY, x);
#pragma unroll
        for (int i = 0; i < VL; ++i) rest += e0 + i == y ? 0.f : exp_diff(x[i], m);
    }
    rest = group_reduce<EB>(rest, part[1], [](float a, float b) { return a + b; });
    const float ey = exp_diff(zy, m), S = rest + ey;
    if (loss && tid == 0) loss[row] = row_loss(rest, ey, zy, m);
    if (!out) return;
    const float f = weights ? weights[row] : 1.f;
    const float scale = S == 0.f ? 0.f : f / S;
    for (int64_t e0 = (int64_t)tid * VL; e0 < C; e0 += EB * VL) {
        float x[VL];
        row_floats(z, e0, C, -INFINITY, x);
#pragma unroll
        for (int i = 0; i < VL; ++i)
            if (e0 + i < C) out[e0 + i] = RowType<TE>::narrow(e0 + i == y ? -scale * rest : scale * exp_diff(x[i], m));
    }
}

}  // namespace

template <class T, class TE>
static hipError_t launch(const void* z, int64_t rows, int64_t C, int64_t ld, const int* labels, const float* weights, void* E,
                         int64_t ldE, float* loss, hipStream_t st) {
    for (int64_t r0 = 0; r0 < rows; r0 += LOGIT_LAUNCH_ROWS) {
        const dim3 grid((unsigned)std::min(rows - r0, LOGIT_LAUNCH_ROWS));
        logit_error_kernel<T, TE><<<grid, EB, 0, st>>>((const T*)z + r0 * ld, C, ld, labels + r0, weights ? weights + r0 : nullptr,
                                                       E ? (TE*)E + r0 * ldE : nullptr, ldE, loss ? loss + r0 : nullptr);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
}

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
