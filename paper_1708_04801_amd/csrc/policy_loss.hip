// Clipped policy loss of one drawn class a for each row of scores, with its gradient.  With l = z_a - log sum_c exp(z_c), rho = exp(l - old), A the row's advantage:
//   loss = r (-min(rho A, clip(rho, low, high) A) + kl (exp(ref - l) - (ref - l) - 1)),
//   d loss / d l = r (-[rho A <= clip(rho) A] rho A - kl (exp(ref - l) - 1)),   d l / d z_c = [c = a] - softmax(z)_c.
// One pass over the scores (row_softmax.h).  What a row makes of l is formed in fp64 by one wave: the ratio is compared with borders, and near 1 the KL term is a
// difference of nearly equal numbers; so are the sums of exponentials, which costs nothing where memory is the bound.  8192 x 65536 bfloat16 reads and writes 1 GiB each in 391 us,
// 5.5 TB/s; 1023 x 32001 takes 26, 5.1; 64 x 1000 fp32 3.9, a launch and one wave's logarithm and exponentials.
#include "row_softmax.h"

namespace wpsgd {

struct PolicyOfRow {
    static constexpr bool kOneWave = true, kWideSum = true;
    const float *old_log, *ref_log, *advantage;
    double low, high, kl, scale;
    float *loss, *log_prob;
    __device__ bool counts(int64_t, int64_t label, float r) const { return !(label < 0 || r == 0.0f); }
    __device__ void absent(int64_t row) const
    {
        loss[row] = 0.0f;
        if (log_prob) log_prob[row] = 0.0f;
    }
    __device__ float make(int64_t row, float r, const RowState &x, bool writes) const
    {
        constexpr double kInf = __builtin_inf();
        const double l = x.unknown ? __builtin_nan("") : x.empty ? -kInf : ((double)x.z_label - (double)x.m) - log(x.sum);
        const bool lost = l == -kInf;                                             // drawn, and now without probability: a ratio of 0, no gradient
        const double A = advantage[row];
        const double ratio = lost ? 0.0 : old_log ? exp(l - (double)old_log[row]) : l == l ? 1.0 : l;
        const double free = A == 0.0 && ratio == kInf ? 0.0 : ratio * A;
        const double held = fmin(fmax(ratio, low), high) * A;
        // (a NaN is no larger than anything, and stays)
        double made = free > held ? -held : -free, by_log = free > held ? 0.0 : -free;
        if (kl != 0.0) {
            const double ref = ref_log[row], gap = lost && ref == -kInf ? 0.0 : ref - l, more = expm1(gap);
            made += kl * (gap == kInf ? kInf : more - gap);
            by_log -= kl * more;
        }
        const float result = (float)((double)r * made);
        if (writes) {
            loss[row] = result;
            if (log_prob) log_prob[row] = (float)l;
        }
        // (an infinite loss shows; an infinite factor would make NaN of every class of probability 0)
        return lost || fabsf(result) == __builtin_inff() ? 0.0f : (float)(-scale * (double)r * by_log);
    }
};

}  // namespace wpsgd

using namespace wpsgd;

extern "C" int wpsgd_policy_loss(const void *Z, int64_t n, int64_t classes, int64_t ld, wpsgd_dtype dtype, const int64_t *drawn, const float *old_log,
                                 const float *ref_log, const float *advantage, const float *row_weights, double clip_low, double clip_high, double kl,
                                 double scale, float *loss, float *log_prob, void *grad, int64_t ld_grad, void *stream)
{
    if (!(clip_low >= 0.0 && clip_low <= 1.0) || !(clip_high >= 0.0) || !(kl >= 0.0) || !(kl - kl == 0.0) || !(scale - scale == 0.0)) return WPSGD_INVALID_ARG;
    const int rc = check_scores(Z, n, classes, ld, dtype, grad, ld_grad);
    if (rc != WPSGD_OK || n == 0) return rc;
    if (!drawn || !advantage || !loss || (kl != 0.0 && !ref_log)) return WPSGD_INVALID_ARG;
    const RowArgs a{Z, n, classes, ld, drawn, row_weights, grad, ld_grad, 0};
    const PolicyOfRow op{old_log, ref_log, advantage, 1.0 - clip_low, 1.0 + clip_high, kl, scale, loss, log_prob};
    hipStream_t s = static_cast<hipStream_t>(stream);
    const hipError_t e = dtype == WPSGD_F32 ? launch_rows_softmax<float>(a, op, s) : launch_rows_softmax<uint16_t>(a, op, s);
    return e == hipSuccess ? WPSGD_OK : hip_fail(e);
}
