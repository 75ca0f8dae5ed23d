// C entry points of the rotary positions: host checks, the frequencies, then the
// launch of rotary.hip.
#include <limits.h>
#include <math.h>

#include "rotary.hpp"

using namespace readme;

namespace {

inline readme_status st_of(hipError_t e) { return e == hipSuccess ? README_OK : README_ERR_HIP; }
inline bool al(const void* p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

constexpr int kMaxHeadDim = 512;
constexpr double kPi = 3.14159265358979323846;

bool rot_ok(int32_t rot, int32_t D) { return rot % 16 == 0 && rot >= 16 && rot <= D; }

}  // namespace

namespace readme {

readme_status rotary_check_sizes(int32_t D, int32_t rot, readme_rotary_layout layout,
                                 int32_t inverse, float amplitude) {
    if (layout != README_ROTARY_HALF && layout != README_ROTARY_PAIRS) return README_ERR_UNSUPPORTED;
    if (D % 16 != 0 || D < 16 || D > kMaxHeadDim || !rot_ok(rot, D)) return README_ERR_UNSUPPORTED;
    if (inverse < 0 || inverse > 1 || !isfinite(amplitude)) return README_ERR_ARG;
    return README_OK;
}

}  // namespace readme

extern "C" {

readme_status readme_rotary_freqs(int32_t rot, double theta, int32_t scaling, double factor,
                                  double trained_len, double low, double high, double* freqs) {
    if (!rot_ok(rot, kMaxHeadDim)) return README_ERR_UNSUPPORTED;
    if (scaling < README_ROTARY_PLAIN || scaling > README_ROTARY_BANDED) return README_ERR_UNSUPPORTED;
    auto positive = [](double v) { return v > 0.0 && isfinite(v); };
    if (!freqs || !positive(theta) || !positive(factor)) return README_ERR_ARG;
    if (scaling == README_ROTARY_BANDED &&
        (!positive(trained_len) || !isfinite(low) || !isfinite(high) || !(low < high)))
        return README_ERR_ARG;
    for (int32_t i = 0; i < rot / 2; ++i) {
        double f = pow(theta, -2.0 * i / rot);
        if (scaling == README_ROTARY_LINEAR) {
            f /= factor;
        } else if (scaling == README_ROTARY_BANDED) {
            const double n = trained_len * f / (2.0 * kPi);
            const double g = fmin(1.0, fmax(0.0, (n - low) / (high - low)));
            f *= g + (1.0 - g) / factor;
        }
        freqs[i] = f;
    }
    return README_OK;
}

readme_status readme_rotary(readme_dtype dt, int64_t T, int32_t H, int32_t D, int32_t rot,
                            readme_rotary_layout layout, int32_t inverse, float amplitude,
                            const int32_t* pos, const double* freqs, const void* x, int64_t ld_x,
                            void* y, int64_t ld_y, void* stream) {
    if (dt != README_F32 && dt != README_BF16) return README_ERR_UNSUPPORTED;
    if (T < 0 || H < 0) return README_ERR_ARG;
    const readme_status st = rotary_check_sizes(D, rot, layout, inverse, amplitude);
    if (st != README_OK) return st;
    if (H > 65535 || T > (1ll << 31) / (D / 16)) return README_ERR_UNSUPPORTED;
    if (T == 0 || H == 0) return README_OK;
    const int64_t width = (int64_t)H * D, es = (int64_t)dtype_size(dt);
    if (!pos || !freqs || !x || !y) return README_ERR_ARG;
    if (!al(pos, 4) || !al(freqs, 8) || !al(x, 16) || !al(y, 16)) return README_ERR_ARG;
    if (ld_x < width || ld_y < width || ld_x * es % 16 != 0 || ld_y * es % 16 != 0)
        return README_ERR_ARG;
    if (x == y && ld_x != ld_y) return README_ERR_ARG;
    RotaryArgs a;
    a.pos = pos;
    a.freqs = freqs;
    a.amplitude = amplitude;
    a.rot = rot;
    a.layout = layout;
    a.inverse = inverse;
    return st_of(launch_rotary(dt, T, H, D, a, x, ld_x, y, ld_y, reinterpret_cast<hipStream_t>(stream)));
}

}  // extern "C"
