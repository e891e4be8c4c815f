// Launchers behind lsh_residual.h.  Arguments are already validated
// (residual_api.cpp); every launcher only enqueues work on `stream`.
#pragma once

#include "launch_cache.h"

namespace lsh {

struct ResidualArgs {
    int64_t T, f_stride, gate_stride;  // strides filled in
    int D, layer, post, pre, gate;     // gate: 0 none, 1 linear, 2 sigmoid
    float alpha, eps;
    const float *scale, *post_g, *post_b, *pre_g, *pre_b;  // null: 1 or 0
};
struct ResidualGrads {
    float *dx, *df, *dgate;
    float* cols[5];  // dscale, dpost_g, dpost_b, dpre_g, dpre_b; null: not wanted
};
// Waves of a row, at 512 columns a wave.
inline int residual_waves(int D) {
    int w = 1;
    while (512 * w < D) w *= 2;
    return w;
}
// Workgroups (of four waves, or of those of a row) that the chip's 256 CUs hold at
// once: those that fit a CU whole, by the waves that a SIMD holds with each kernel's
// registers.  BwdPlain: neither scale nor biases.
enum ResidualPass { kResidualFwd, kResidualBwd, kResidualBwdPlain };
inline int residual_resident(ResidualPass pass, int D) {
    const int waves = residual_waves(D);
    const int simd = pass == kResidualFwd ? (waves == 1 ? 5 : 4) : pass == kResidualBwdPlain || waves == 16 ? 4 : 3;
    return 256 * (4 * simd / (waves > 4 ? waves : 4));
}

bool residual_fits(const ResidualArgs& a);
size_t residual_workspace_bytes(const ResidualArgs& a);
hipError_t launch_residual_fwd(const ResidualArgs& a, bool f32, const float* x, const void* f, const void* gate,
                               float* y, void* z, hipStream_t stream);
hipError_t launch_residual_bwd(const ResidualArgs& a, bool f32, const float* y, const void* f, const void* gate,
                               const float* dy, const float* dz, const ResidualGrads& g, void* workspace,
                               hipStream_t stream);

}  // namespace lsh
