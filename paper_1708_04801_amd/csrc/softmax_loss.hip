// Softmax cross-entropy of a batch of scores, with its gradient:
//   loss_i = r_i (log sum_c exp(z_ic) - z_it),   grad_ic = scale r_i (exp(z_ic - m_i) / s_i - [c = t]),   m_i the row's maximum, s_i = sum_c exp(z_ic - m_i).
#include "row_softmax.h"

namespace wpsgd {

struct LossOfRow {
    static constexpr bool kOneWave = false, kWideSum = false;
    double scale;
    float *loss;
    __device__ bool counts(int64_t, int64_t label, float r) const { return !(label < 0 || r == 0.0f); }
    __device__ void absent(int64_t row) const { loss[row] = 0.0f; }
    __device__ float make(int64_t row, float r, const RowState &x, bool writes) const
    {
        if (writes) loss[row] = x.unknown ? __builtin_nanf("") : x.empty ? __builtin_inff() : (x.m - x.z_label + logf(x.s)) * r;
        return (float)(scale * (double)r);
    }
};

}  // namespace wpsgd

using namespace wpsgd;

extern "C" {

int wpsgd_softmax_loss(const void *Z, int64_t n, int64_t classes, int64_t ld, wpsgd_dtype dtype, const int64_t *labels, const float *row_weights, double scale,
                       float *loss, void *grad, int64_t ld_grad, void *stream)
{
    const int rc = check_scores(Z, n, classes, ld, dtype, grad, ld_grad);
    if (rc != WPSGD_OK || n == 0) return rc;
    if (!labels || !loss || !(scale - scale == 0.0)) return WPSGD_INVALID_ARG;
    const RowArgs a{Z, n, classes, ld, labels, row_weights, grad, ld_grad, 0};
    const LossOfRow op{scale, loss};
    hipStream_t s = static_cast<hipStream_t>(stream);
    const hipError_t e = dtype == WPSGD_F32 ? launch_rows_softmax<float>(a, op, s) : launch_rows_softmax<uint16_t>(a, op, s);
    return e == hipSuccess ? WPSGD_OK : hip_fail(e);
}

}  // extern "C"
