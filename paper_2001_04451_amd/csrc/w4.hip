// Products with weights of 4 bits (lsh_w4.h), and the weights' own passes:
// quantise, lay out, read back.
//
// Rows times weights: a 16 x 16 x 32 product on the matrix cores takes 8 codes
// of a lane as 8 bf16 values.  E2M1 codes come with their scale, exactly.  INT4
// codes are read as e4m3 bytes: those of 0 .. 15 stand for c 2^-9, subnormals
// and the first normals alike, so one conversion with a scale of 2^9 gives c
// itself; the group's sum of products is scaled afterwards in fp32,
//   s (sum a c - z sum a),
// with sum a from a product with ones, which lands where the sum of a c does.
#include "common.h"
#include "launch_w4.h"

namespace lsh {
namespace {

struct W4Args {
    W4Shape s;
    W4Call c;
    const char *codes, *scales;
    const uint8_t* zeros;
};

__device__ __forceinline__ bf16x8 from_pairs(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return as_bf16x8(u32x4{a, b, c, d});
}
__device__ __forceinline__ uint32_t fp8_pair(uint32_t w, bool high) {
    return high ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 512.f, true))
                : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 512.f, false));
}
// A word's eight codes as they are: the low halves of its bytes are inputs 0 .. 3.
__device__ __forceinline__ bf16x8 int4_codes(uint32_t w) {
    const uint32_t lo = w & 0x0F0F0F0Fu, hi = (w >> 4) & 0x0F0F0F0Fu;
    return from_pairs(fp8_pair(lo, false), fp8_pair(lo, true), fp8_pair(hi, false), fp8_pair(hi, true));
}
// A word's eight e2m1 codes, in order, times 2^(byte - 127) (255: NaN).
__device__ __forceinline__ bf16x8 e2m1_values(uint32_t w, uint32_t byte) {
    const float s = __uint_as_float(byte << 23);
    return from_pairs(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3)));
}

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Scales (as fp32) and zero points of a lane's output in one tile.
template <int PT>
struct Scales {
    float s[PT], z[PT];
    __device__ __forceinline__ void load(const W4Args& g, int64_t tile, int n) {
        const int64_t at = (tile * 16 + n) * PT;
        const uint16_t* p = reinterpret_cast<const uint16_t*>(g.scales) + at;
#pragma unroll
        for (int i = 0; i < PT; ++i) s[i] = bf16_bits_to_f32(p[i]);
#pragma unroll
        for (int i = 0; i < PT; ++i) z[i] = g.zeros ? (float)g.zeros[at + i] : 8.f;
    }
};

__device__ __forceinline__ void put(const W4Args& g, int64_t m, int n, float v) {
    if (m >= g.c.M || n >= g.s.N) return;
    const int64_t at = m * g.s.N + n;
    if (g.c.bias) v += g.c.bias[n];
    if (g.c.out_f32)
        g.c.out_f32[at] = fmaf(g.c.sign, v, g.c.resid ? g.c.resid[at] : 0.f);
    else
        g.c.out_bf16[at] = (uint16_t)f32_to_bf16_bits(g.c.relu && v < 0.f ? 0.f : v);
}

constexpr int kWaves = 8;

// A workgroup takes 16 outputs of 16 MT rows; its waves take the tiles of 128
// inputs in turn and add up in LDS.
template <bool E2M1, int PT, int MT>
__global__ __launch_bounds__(64 * kWaves) void w4_rows_kernel(W4Args g) {
    __shared__ float sums[kWaves][MT][16][16];  // [wave][row tile][row][output]
    const int lane = lane_id(), wave = threadIdx.x >> 6, n = lane & 15, q = lane >> 4;
    const int64_t m0 = (int64_t)blockIdx.y * (16 * MT);
    const int tiles_k = (int)g.s.tiles_k;
    const int64_t row_tile = (int64_t)blockIdx.x * tiles_k;
    const uint16_t* x[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) x[t] = g.c.a + min(m0 + 16 * t + n, g.c.M - 1) * g.c.a_stride + 8 * q;
    const bf16x8 ones = from_pairs(0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u);
    const f32x4 none = {0.f, 0.f, 0.f, 0.f};
    f32x4 acc[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) acc[t] = none;
    for (int b = wave; b < tiles_k; b += kWaves) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(g.codes + (row_tile + b) * 1024 + 16 * lane);
        const int steps = min(4, (g.s.K - 128 * b) / 32);
        if constexpr (E2M1) {
            const uint32_t bytes = *reinterpret_cast<const uint32_t*>(g.scales + ((row_tile + b) * 16 + n) * 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (i >= steps) break;
                const bf16x8 v = e2m1_values(w[i], (bytes >> (8 * i)) & 255u);
#pragma unroll
                for (int t = 0; t < MT; ++t)
                    acc[t] = mfma16(*reinterpret_cast<const bf16x8*>(x[t] + 128 * b + 32 * i), v, acc[t]);
            }
        } else {
            Scales<PT> sc;
            sc.load(g, row_tile + b, n);
#pragma unroll
            for (int p = 0; p < PT; ++p) {
                constexpr int kSteps = 4 / PT;
                f32x4 part[MT], sum[MT];
#pragma unroll
                for (int t = 0; t < MT; ++t) part[t] = sum[t] = none;
#pragma unroll
                for (int j = 0; j < kSteps; ++j) {
                    const int i = p * kSteps + j;
                    if (i >= steps) break;
                    const bf16x8 v = int4_codes(w[i]);
#pragma unroll
                    for (int t = 0; t < MT; ++t) {
                        const bf16x8 xv = *reinterpret_cast<const bf16x8*>(x[t] + 128 * b + 32 * i);
                        part[t] = mfma16(xv, v, part[t]);
                        sum[t] = mfma16(xv, ones, sum[t]);
                    }
                }
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        acc[t][e] = fmaf(sc.s[p], fmaf(-sc.z[p], sum[t][e], part[t][e]), acc[t][e]);
            }
        }
    }
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) sums[wave][t][4 * q + e][n] = acc[t][e];
    __syncthreads();
    for (int i = threadIdx.x; i < MT * 256; i += 64 * kWaves) {
        const int t = i >> 8, r = (i >> 4) & 15, c = i & 15;
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) v += sums[w][t][r][c];
        put(g, m0 + 16 * t + r, (int)(blockIdx.x * 16) + c, v);
    }
}

// ---------------------------------------------------------------------------
// The weights' own passes.  A workgroup takes a tile of 16 outputs x 128 inputs,
// a thread 8 inputs of one output: thread 16 r + j inputs 8 j .. + 7 of output r,
// whose word is word j / 4 of piece 16 (j % 4) + r.

struct Spot {
    int64_t tile;
    int n, k, word, pair;  // output, first input, word of the tile (of 256), row r
    bool in;
};
__device__ __forceinline__ Spot spot_of(const W4Shape& s) {
    const int r = threadIdx.x >> 4, j = threadIdx.x & 15;
    const int64_t tn = blockIdx.x / s.tiles_k, tk = blockIdx.x - tn * s.tiles_k;
    Spot p;
    p.tile = blockIdx.x;
    p.n = (int)(16 * tn) + r;
    p.k = (int)(128 * tk) + 8 * j;
    p.word = (16 * (j & 3) + r) * 4 + (j >> 2);
    p.pair = r;
    p.in = p.n < s.N && p.k < s.K;
    return p;
}
__device__ __forceinline__ uint32_t word_of(const uint32_t* code, bool e2m1) {
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) w |= code[e] << (e2m1 ? 4 * e : (e < 4 ? 8 * e : 8 * (e - 4) + 4));
    return w;
}
__device__ __forceinline__ uint32_t code_at(uint32_t w, int e, bool e2m1) {
    return (w >> (e2m1 ? 4 * e : (e < 4 ? 8 * e : 8 * (e - 4) + 4))) & 15u;
}

// Over the aligned group of 2^k lanes (4, 8 or 16) that holds a group's values.
template <typename F>
__device__ __forceinline__ float group_fold(float x, int lanes, F f) {
    for (int o = 1; o < lanes; o <<= 1) x = f(x, __shfl_xor(x, o));
    return x;
}

// The smallest bf16 value s with steps * s >= reach (finite), as its bits: one
// of four from just below the rounded quotient on, compared exactly in fp64.
__device__ __forceinline__ uint32_t scale_for(double reach, double steps) {
    uint32_t b = __float_as_uint((float)(reach / steps)) >> 16;
    b = b > 0 ? b - 1 : 0;
#pragma unroll
    for (int i = 0; i < 3; ++i)
        if (steps * (double)bf16_bits_to_f32(b) < reach) ++b;
    return b;
}

template <bool F32>
__global__ __launch_bounds__(256) void w4_quantize_kernel(W4Shape s, const void* __restrict__ w,
                                                          char* __restrict__ packed) {
    __shared__ uint32_t words[256];
    const Spot p = spot_of(s);
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = 0.f;
    if (p.in) {
        const int64_t at = (int64_t)p.n * s.K + p.k;
        if constexpr (F32) {
            const f32x4* src = reinterpret_cast<const f32x4*>(static_cast<const float*>(w) + at);
            const f32x4 lo = src[0], hi = src[1];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = lo[e], x[4 + e] = hi[e];
        } else {
            const u32x4 v = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(w) + at);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x[2 * e] = __uint_as_float(v[e] << 16);
                x[2 * e + 1] = __uint_as_float(v[e] & 0xFFFF0000u);
            }
        }
    }
    float lo = 0.f, hi = 0.f, bad = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        lo = fminf(lo, x[e]);
        hi = fmaxf(hi, x[e]);
        if (!(fabsf(x[e]) < __builtin_inff())) bad = 1.f;
    }
    const int lanes = s.group / 8;
    lo = group_fold(lo, lanes, [](float a, float b) { return fminf(a, b); });
    hi = group_fold(hi, lanes, [](float a, float b) { return fmaxf(a, b); });
    bad = group_fold(bad, lanes, [](float a, float b) { return fmaxf(a, b); });
    const int j = threadIdx.x & 15, per = s.per_tile(), at = ((int)p.pair) * per + j / lanes;
    char* const scales = packed + s.codes_size() + p.tile * (16 * per * (int64_t)s.scale_bytes());
    uint8_t* const zeros = reinterpret_cast<uint8_t*>(packed + s.codes_size() + s.scales_size()) + p.tile * 16 * per;
    uint32_t code[8];
    if (s.e2m1) {
        // the smallest exponent that brings the largest magnitude to 6 = 1.5 * 2^2 or below
        const uint32_t big = __float_as_uint(fmaxf(hi, -lo));
        const int byte = bad > 0.f ? 255 : max((int)(big >> 23) - 2 + ((big & 0x7FFFFFu) > 0x400000u ? 1 : 0), 0);
        uint32_t c = 0;
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = bad > 0.f ? 0.f : ldexpf(x[e], 127 - byte);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[0], y[1], 1.f, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[2], y[3], 1.f, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[4], y[5], 1.f, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[6], y[7], 1.f, 3);
        words[p.word] = c;
        if (j % lanes == 0) scales[at] = (char)(uint8_t)(p.in ? byte : 0);
    } else {
        const double reach = s.zeros ? (double)hi - (double)lo : (double)fmaxf(hi, -lo);
        uint32_t bits = scale_for(bad > 0.f ? 0. : reach, s.zeros ? 15. : 7.);
        const double by = bits ? (double)bf16_bits_to_f32(bits) : 1.;
        const double z = s.zeros ? fmin(rint(-(double)lo / by), 15.) : 8.;
#pragma unroll
        for (int e = 0; e < 8; ++e)  // quotients in fp64: values next to a border fall on their side of it
            code[e] = bad > 0.f ? 0u : (uint32_t)fmin(fmax(rint((double)x[e] / by) + z, 0.), 15.);
        if (bad > 0.f) bits = 0x7FC0u;
        words[p.word] = p.in ? word_of(code, false) : 0u;
        if (j % lanes == 0) {
            reinterpret_cast<uint16_t*>(scales)[at] = (uint16_t)(p.in ? bits : 0u);
            if (s.zeros) zeros[at] = (uint8_t)(p.in && !(bad > 0.f) ? (uint32_t)z : 0u);
        }
    }
    __syncthreads();
    reinterpret_cast<uint32_t*>(packed + p.tile * 1024)[threadIdx.x] = words[threadIdx.x];
}

__global__ __launch_bounds__(256) void w4_pack_kernel(W4Shape s, const uint8_t* __restrict__ codes,
                                                      const void* __restrict__ scales,
                                                      const uint8_t* __restrict__ zeros, char* __restrict__ packed) {
    __shared__ uint32_t words[256];
    const Spot p = spot_of(s);
    uint32_t w = 0;
    if (p.in) w = *reinterpret_cast<const uint32_t*>(codes + ((int64_t)p.n * s.K + p.k) / 2);
    if (!s.e2m1) {
        uint32_t code[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) code[e] = code_at(w, e, true);
        w = word_of(code, false);
    }
    words[p.word] = w;
    const int j = threadIdx.x & 15, per = s.per_tile();
    if (j < per) {
        const int groups = (s.K + s.group - 1) / s.group, k = p.k - 8 * j + j * s.group;  // the group's first input
        const bool in = p.n < s.N && k < s.K;
        const int64_t from = in ? (int64_t)p.n * groups + k / s.group : 0, to = (p.tile * 16 + p.pair) * per + j;
        char* const sc = packed + s.codes_size();
        if (s.e2m1)
            sc[to] = in ? static_cast<const char*>(scales)[from] : 0;
        else
            reinterpret_cast<uint16_t*>(sc)[to] = in ? static_cast<const uint16_t*>(scales)[from] : 0;
        if (s.zeros) (packed + s.codes_size() + s.scales_size())[to] = in ? (char)(zeros[from] & 15) : 0;
    }
    __syncthreads();
    reinterpret_cast<uint32_t*>(packed + p.tile * 1024)[threadIdx.x] = words[threadIdx.x];
}

template <bool F32>
__global__ __launch_bounds__(256) void w4_unpack_kernel(W4Shape s, const char* __restrict__ packed,
                                                        void* __restrict__ out) {
    const Spot p = spot_of(s);
    if (!p.in) return;
    const uint32_t w = reinterpret_cast<const uint32_t*>(packed + p.tile * 1024)[p.word];
    const int j = threadIdx.x & 15, per = s.per_tile();
    const int64_t at = (p.tile * 16 + p.pair) * per + j / (s.group / 8);
    const char* const sc = packed + s.codes_size();
    float v[8];
    if (s.e2m1) {
        const uint32_t byte = (uint8_t)sc[at];
        const float lowest[8] = {0.f, 0.5f, 1.f, 1.5f, 2.f, 3.f, 4.f, 6.f};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t c = code_at(w, e, true);
            const float a = byte == 255 ? __builtin_nanf("") : ldexpf(lowest[c & 7], (int)byte - 127);
            v[e] = c & 8 ? -a : a;
        }
    } else {
        const float scale = bf16_bits_to_f32(reinterpret_cast<const uint16_t*>(sc)[at]);
        const float z = s.zeros ? (float)(uint8_t)(packed + s.codes_size() + s.scales_size())[at] : 8.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = scale * ((float)code_at(w, e, false) - z);
    }
    const int64_t to = (int64_t)p.n * s.K + p.k;
    if constexpr (F32) {
        f32x4* dst = reinterpret_cast<f32x4*>(static_cast<float*>(out) + to);
        dst[0] = f32x4{v[0], v[1], v[2], v[3]};
        dst[1] = f32x4{v[4], v[5], v[6], v[7]};
    } else {
        u32x4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = pack_bf16x2(v[2 * e], v[2 * e + 1]);
        *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(out) + to) = y;
    }
}

template <int MT, typename Go>
void by_weights(const W4Shape& s, Go go) {
    if (s.e2m1)
        go(w4_rows_kernel<true, 4, MT>);
    else if (s.group == 32)
        go(w4_rows_kernel<false, 4, MT>);
    else if (s.group == 64)
        go(w4_rows_kernel<false, 2, MT>);
    else
        go(w4_rows_kernel<false, 1, MT>);
}

unsigned tiles(const W4Shape& s) { return (unsigned)(s.tiles_n * s.tiles_k); }

}  // namespace

hipError_t launch_w4_quantize(const W4Shape& s, bool f32, const void* w, char* packed, hipStream_t stream) {
    if (f32)
        w4_quantize_kernel<true><<<tiles(s), 256, 0, stream>>>(s, w, packed);
    else
        w4_quantize_kernel<false><<<tiles(s), 256, 0, stream>>>(s, w, packed);
    return hipGetLastError();
}

hipError_t launch_w4_pack(const W4Shape& s, const uint8_t* codes, const void* scales, const uint8_t* zeros,
                          char* packed, hipStream_t stream) {
    w4_pack_kernel<<<tiles(s), 256, 0, stream>>>(s, codes, scales, zeros, packed);
    return hipGetLastError();
}

hipError_t launch_w4_unpack(const W4Shape& s, bool f32, const char* packed, void* w, hipStream_t stream) {
    if (f32)
        w4_unpack_kernel<true><<<tiles(s), 256, 0, stream>>>(s, packed, w);
    else
        w4_unpack_kernel<false><<<tiles(s), 256, 0, stream>>>(s, packed, w);
    return hipGetLastError();
}

bool w4_fits(const W4Shape& s, int64_t M) { return s.tiles_n < (int64_t)1 << 22 && (M + 63) / 64 < 65536; }

size_t w4_workspace_bytes(const W4Shape&, int64_t) { return 0; }

hipError_t launch_linear_w4(const W4Shape& s, const W4Call& c, void*, hipStream_t stream) {
    const W4Args g{s, c, c.packed, c.packed + s.codes_size(),
                   s.zeros ? reinterpret_cast<const uint8_t*>(c.packed + s.codes_size() + s.scales_size()) : nullptr};
    auto go = [&](int mt) {
        return [&g, mt, stream](auto kernel) {
            const dim3 grid((unsigned)g.s.tiles_n, (unsigned)((g.c.M + 16 * mt - 1) / (16 * mt)));
            kernel<<<grid, 64 * kWaves, 0, stream>>>(g);
        };
    };
    if (c.M <= 16)
        by_weights<1>(s, go(1));
    else if (c.M <= 32)
        by_weights<2>(s, go(2));
    else
        by_weights<4>(s, go(4));
    return hipGetLastError();
}

}  // namespace lsh
