// Device helpers of the per-head norm and the position rotation (lsh_qk.h):
// eight lanes hold a head's 64 values, eight each.
#pragma once

#include "common.h"

namespace lsh {

constexpr int kMaxTokens = 16;  // whose angles a workgroup holds at a time

// Of a workgroup's tokens: the angles of their pairs, and where their rows go.
struct Angles {
    alignas(16) float c[kMaxTokens][32];  // read four at a time
    alignas(16) float s[kMaxTokens][32];
    int b[kMaxTokens], l[kMaxTokens];  // batch entry and position in it (L > 0)
};

// Revolutions a position: an angle's frequency / (2 pi), in fp64.
__device__ __forceinline__ double revolutions(float freq) { return (double)freq * 0.15915494309189535; }

// The angle of pair p of token t, reduced in fp64 so that only the fraction of a
// revolution reaches fp32.  Its rounding there, up to 2^-25 half turns, would turn by
// more than the roundings of sine and cosine: what it leaves turns them on.
__device__ __forceinline__ void form_angle(Angles& A, int t, int p, double pos, double f) {
    double rev = pos * f;
    rev = 2.0 * (rev - rint(rev));
    const float half = (float)rev, rest = (float)(rev - (double)half) * 3.14159265f;
    float s, c;
    sincospif(half, &s, &c);
    A.c[t][p] = fmaf(-s, rest, c);
    A.s[t][p] = fmaf(c, rest, s);
}

// A lane's eight dimensions (8 l ..) turned by the angles of token t (by their
// negatives for sign = -1).  All eight lanes of the group take part.
template <bool INTER>
__device__ __forceinline__ void turn(float* y, const Angles& A, int t, int l, int rot, float sign) {
    if constexpr (INTER) {
        if (8 * l >= rot) return;
        const f32x4 c = *reinterpret_cast<const f32x4*>(&A.c[t][4 * l]);
        const f32x4 s = *reinterpret_cast<const f32x4*>(&A.s[t][4 * l]);
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const float a = y[2 * p], b = y[2 * p + 1], sn = sign * s[p];
            y[2 * p] = a * c[p] - b * sn;
            y[2 * p + 1] = a * sn + b * c[p];
        }
    } else {
        const int hl = rot >> 4;  // lanes in half of the turned dimensions
        const bool low = l < hl, in = l < 2 * hl;
        float z[8];
        if (hl == 4) {  // lane l ^ 4: the banks of four lanes trade places by moves within their row
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int x = __float_as_int(y[e]);
                const int up = __builtin_amdgcn_update_dpp(x, x, 0x104, 0xF, 0x5, false);  // banks 0, 2: from l + 4
                z[e] = __int_as_float(__builtin_amdgcn_update_dpp(up, x, 0x114, 0xF, 0xA, false));  // 1, 3: from l - 4
            }
        } else if (hl == 2) {  // lane l ^ 2
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] = dpp_f32<kDppXor2>(y[e]);
        } else {
            const int other = (threadIdx.x & 63) + (in ? (low ? hl : -hl) : 0);
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] = __shfl(y[e], other);
        }
        if (!in) return;
        const int p0 = 8 * (low ? l : l - hl);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float sn = low ? -sign * A.s[t][p0 + e] : sign * A.s[t][p0 + e];
            y[e] = y[e] * A.c[t][p0 + e] + z[e] * sn;
        }
    }
}

__device__ __forceinline__ float inv_rms(const float* x, float eps) {
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) ss = fmaf(x[e], x[e], ss);
    const float ms = group8_sum(ss) * (1.f / kHeadDim) + eps;
    const bool tiny = ms < 0x1p-100f;  // the instruction takes subnormals as 0
    const float r = __builtin_amdgcn_rsqf(tiny ? ms * 0x1p80f : ms) * (tiny ? 0x1p40f : 1.f);  // within 2^-22 of it
    return ms == 0.f ? 0.f : r;
}

}  // namespace lsh
