// Rotary frequencies (host-only arithmetic in double precision; no device is touched).
#include <math.h>
#include <stdint.h>

#include "aaf_kv.h"

extern "C" int aaf_kv_rope_freqs(int32_t rot_dim, double base, int32_t scaling, const aaf_kv_rope_scaling *s,
                                 double *inv_freq_host, float *mscale_out) {
    if (rot_dim < 2 || rot_dim % 2 || !(base > 1.0) || base - base != 0.0 || !inv_freq_host) return AAF_ERR_INVALID_ARG;
    const double pi = 3.14159265358979323846;
    if (scaling != AAF_ROPE_NONE) {
        if (!s || s->struct_size != sizeof(aaf_kv_rope_scaling) || !(s->factor >= 1.0) || s->factor - s->factor != 0.0)
            return AAF_ERR_INVALID_ARG;
        if (scaling == AAF_ROPE_WAVELENGTH &&
            !(s->orig_context > 0.0 && s->low > 0.0 && s->high > s->low && s->high - s->high == 0.0 && s->orig_context - s->orig_context == 0.0))
            return AAF_ERR_INVALID_ARG;
        if (scaling == AAF_ROPE_RAMP &&
            !(s->orig_context > 0.0 && s->low > 0.0 && s->high > s->low && s->high - s->high == 0.0 && s->orig_context - s->orig_context == 0.0))
            return AAF_ERR_INVALID_ARG;
    }
    if (scaling < AAF_ROPE_NONE || scaling > AAF_ROPE_RAMP) return AAF_ERR_INVALID_ARG;
    if (scaling == AAF_ROPE_BASE) {  // the base grows so that the slowest pair is stretched by the factor
        if (rot_dim < 4) return AAF_ERR_INVALID_ARG;
        base *= pow(s->factor, (double)rot_dim / (rot_dim - 2));
    }
    // pair index at which a frequency makes `turns` turns over the original context
    auto index_of = [&](double turns) { return rot_dim * log(s->orig_context / (turns * 2.0 * pi)) / (2.0 * log(base)); };
    double lo = 0.0, hi = 0.0;
    if (scaling == AAF_ROPE_RAMP) {
        lo = fmax(floor(index_of(s->high)), 0.0);
        hi = fmin(ceil(index_of(s->low)), rot_dim - 1.0);
        if (hi <= lo) hi = lo + 0.001;
    }
    for (int i = 0; i < rot_dim / 2; ++i) {
        double f = pow(base, -2.0 * i / rot_dim);
        if (scaling == AAF_ROPE_LINEAR) {
            f /= s->factor;
        } else if (scaling == AAF_ROPE_WAVELENGTH) {
            // turns over the original context: many keep the frequency, few divide it, between them a linear blend
            const double turns = s->orig_context * f / (2.0 * pi);
            const double keep = fmin(1.0, fmax(0.0, (turns - s->low) / (s->high - s->low)));
            f = (1.0 - keep) * f / s->factor + keep * f;
        } else if (scaling == AAF_ROPE_RAMP) {
            const double slow = fmin(1.0, fmax(0.0, (i - lo) / (hi - lo)));
            f = slow * f / s->factor + (1.0 - slow) * f;
        }
        inv_freq_host[i] = f;
    }
    if (mscale_out) *mscale_out = scaling == AAF_ROPE_RAMP ? (float)(0.1 * log(s->factor) + 1.0) : 1.0f;
    return AAF_OK;
}
