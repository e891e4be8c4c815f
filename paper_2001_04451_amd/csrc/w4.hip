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
#include "attn_common.h"
#include "launch_w4.h"

#include <type_traits>

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

__device__ __forceinline__ bf16x8 all_of(uint32_t bf16) {
    const uint32_t p = bf16 | bf16 << 16;
    return from_pairs(p, p, p, p);
}
constexpr f32x4 kNone = {0.f, 0.f, 0.f, 0.f};

// A lane's piece of a tile's codes; with E2M1 the scale bytes of its output.
template <bool E2M1>
struct Codes {
    u32x4 w;
    uint32_t bytes;
    __device__ __forceinline__ void load(const W4Args& g, int64_t tile, int lane) {
        w = *reinterpret_cast<const u32x4*>(g.codes + tile * 1024 + 16 * lane);
        if constexpr (E2M1) bytes = *reinterpret_cast<const uint32_t*>(g.scales + tile * 64 + 4 * (lane & 15));
    }
    // Step i's eight weights, scaled (E2M1) or as codes.
    __device__ __forceinline__ bf16x8 step(int i) const {
        if constexpr (E2M1)
            return e2m1_values(w[i], (bytes >> (8 * i)) & 255u);
        else
            return int4_codes(w[i]);
    }
};

// INT4's scales and zero points.  Products take the weights first, so that a lane
// ends up with outputs 4 q .. + 3 of row l % 16 (q = l / 16): the scales of these.
__device__ __forceinline__ f32x4 four_bf16(uint2 s) {
    return f32x4{__uint_as_float(s.x << 16), __uint_as_float(s.x & 0xFFFF0000u), __uint_as_float(s.y << 16),
                 __uint_as_float(s.y & 0xFFFF0000u)};
}
__device__ __forceinline__ f32x4 four_bytes(uint32_t z) {
    return f32x4{(float)(z & 255u), (float)((z >> 8) & 255u), (float)((z >> 16) & 255u), (float)(z >> 24)};
}
template <int BYTES>
struct Bytes {  // from memory aligned to them, or to 16
    uint32_t w[BYTES / 4];
    __device__ __forceinline__ void load(const void* p) {
        if constexpr (BYTES % 16 == 0) {
#pragma unroll
            for (int i = 0; i < BYTES / 16; ++i) {
                const u32x4 v = reinterpret_cast<const u32x4*>(p)[i];
#pragma unroll
                for (int e = 0; e < 4; ++e) w[4 * i + e] = v[e];
            }
        } else if constexpr (BYTES == 8) {
            const uint2 v = *static_cast<const uint2*>(p);
            w[0] = v.x, w[1] = v.y;
        } else {
            w[0] = *static_cast<const uint32_t*>(p);
        }
    }
};
template <bool ZEROS, int PT>
struct Scales {
    Bytes<8 * PT> s;
    Bytes<ZEROS ? 4 * PT : 0> z;
    __device__ __forceinline__ void load(const W4Args& g, int64_t tile, int lane) {
        s.load(g.scales + (tile * 4 + (lane >> 4)) * (8 * PT));
        if constexpr (ZEROS) z.load(g.zeros + (tile * 4 + (lane >> 4)) * (4 * PT));
    }
    __device__ __forceinline__ f32x4 scale(int p) const { return four_bf16(make_uint2(s.w[2 * p], s.w[2 * p + 1])); }
    __device__ __forceinline__ f32x4 zero(int p) const {
        if constexpr (ZEROS) return four_bytes(z.w[p]);
        return f32x4{8.f, 8.f, 8.f, 8.f};
    }
};
struct NoScales {
    __device__ __forceinline__ void load(const W4Args&, int64_t, int) {}
};

// Four outputs n .. n + 3 of row m.
__device__ __forceinline__ void put4(const W4Args& g, int64_t m, int n, f32x4 v) {
    const int N = g.s.N;
    if (m >= g.c.M || n >= N) return;
    const int64_t at = m * N + n;
    if ((N & 3) == 0) {  // then n + 3 < N and the four are aligned
        if (g.c.bias) v += *reinterpret_cast<const f32x4*>(g.c.bias + n);
        if (g.c.out_f32) {
            f32x4 r = g.c.resid ? *reinterpret_cast<const f32x4*>(g.c.resid + at) : kNone;
#pragma unroll
            for (int e = 0; e < 4; ++e) r[e] = fmaf(g.c.sign, v[e], r[e]);
            *reinterpret_cast<f32x4*>(g.c.out_f32 + at) = r;
        } else {
            if (g.c.relu)
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = v[e] < 0.f ? 0.f : v[e];
            *reinterpret_cast<uint2*>(g.c.out_bf16 + at) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (n + e >= N) break;
        float x = v[e] + (g.c.bias ? g.c.bias[n + e] : 0.f);
        if (g.c.out_f32)
            g.c.out_f32[at + e] = fmaf(g.c.sign, x, g.c.resid ? g.c.resid[at + e] : 0.f);
        else
            g.c.out_bf16[at + e] = (uint16_t)f32_to_bf16_bits(g.c.relu && x < 0.f ? 0.f : x);
    }
}

// Outputs n + 4 q .. + 3 and 16 further of row m to bf16, N a multiple of 8: the four
// lanes of a row trade them for n + 8 q .. + 7, so that the row's 64 bytes leave in
// one store.
__device__ __forceinline__ void put_pair(const W4Args& g, int64_t m, int n, int q, f32x4 a, f32x4 b) {
    const int N = g.s.N;
    if (g.c.bias) {
        if (n + 4 * q < N) a += *reinterpret_cast<const f32x4*>(g.c.bias + n + 4 * q);
        if (n + 16 + 4 * q < N) b += *reinterpret_cast<const f32x4*>(g.c.bias + n + 16 + 4 * q);
    }
    if (g.c.relu)
#pragma unroll
        for (int e = 0; e < 4; ++e) a[e] = a[e] < 0.f ? 0.f : a[e], b[e] = b[e] < 0.f ? 0.f : b[e];
    u32x4 out;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const auto half = __builtin_amdgcn_permlane32_swap(pack_bf16x2(a[2 * e], a[2 * e + 1]),
                                                           pack_bf16x2(b[2 * e], b[2 * e + 1]), false, false);
        const auto row = __builtin_amdgcn_permlane16_swap(half[0], half[1], false, false);
        out[e] = row[0];
        out[2 + e] = row[1];
    }
    if (m < g.c.M && n + 8 * q < N) *reinterpret_cast<u32x4*>(g.c.out_bf16 + m * N + n + 8 * q) = out;
}

// ---------------------------------------------------------------------------
// Few rows.  A workgroup takes 16 NT outputs of 16 MT rows; its waves take the
// tiles of 128 inputs in turn, the codes of AHEAD of them on their way, and add
// up in LDS.  Where the rows are short (STAGED) they pass through LDS once, while
// the first codes are on their way; else a wave loads them tile by tile.
// HBM-bound where the matrix is large: one row by 16384 x 16384 26 us in int4 (5.2
// TB/s), 24 in e2m1 (5.9), by 32000 x 4096 16 and 15; by 4096 x 1024 3.0, of which the
// launch is 2.5.
constexpr size_t kStaged = 34 * 1024;  // bytes of rows, at most
__host__ __device__ constexpr int64_t staged_stride(int K) { return K + 32; }  // rows start 16 banks apart

template <bool E2M1, bool ZEROS, int PT, int MT, int NT, bool STAGED>
__global__ __launch_bounds__(512) void w4_rows_kernel(W4Args g) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    float* const sums = reinterpret_cast<float*>(smem);  // [wave][output tile][row tile][row][output]
    constexpr int AHEAD = NT == 1 ? (!E2M1 && PT == 4 ? 2 : 4) : (NT == 2 ? 2 : 1);
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int q = lane >> 4, K = g.s.K;
    const int64_t m0 = (int64_t)blockIdx.y * (16 * MT);
    const int tiles_k = (int)g.s.tiles_k, whole = K / 128;
    int64_t tile[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) tile[j] = min((int64_t)blockIdx.x * NT + j, g.s.tiles_n - 1) * tiles_k;
    struct Block {
        Codes<E2M1> w[NT];
        std::conditional_t<E2M1, NoScales, Scales<ZEROS, PT>> s[NT];
    } blocks[AHEAD];
    auto load = [&](Block& b, int k) {
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            b.w[j].load(g, tile[j] + k, lane);
            b.s[j].load(g, tile[j] + k, lane);
        }
    };
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
        if (wave + u * waves < whole) load(blocks[u], wave + u * waves);
    // Rows past M repeat the last one: their lanes' values meet their own results alone,
    // which are not stored.
    const uint16_t* x[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int64_t m = min(m0 + 16 * t + (lane & 15), g.c.M - 1);
        if constexpr (STAGED)
            x[t] = reinterpret_cast<const uint16_t*>(smem) + (m - m0) * staged_stride(K) + 8 * q;
        else
            x[t] = g.c.a + m * g.c.a_stride + 8 * q;
    }
    if constexpr (STAGED) {
        const int pieces = K / 8, all = (int)min((int64_t)16 * MT, g.c.M - m0) * pieces;
#pragma unroll 4
        for (int i = threadIdx.x; i < all; i += blockDim.x) {
            const int r = i / pieces, p = i - r * pieces;
            *reinterpret_cast<u32x4*>(smem + 2 * (r * staged_stride(K) + 8 * p)) =
                *reinterpret_cast<const u32x4*>(g.c.a + (m0 + r) * g.c.a_stride + 8 * p);
        }
        __syncthreads();
    }
    f32x4 acc[NT][MT];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int t = 0; t < MT; ++t) acc[j][t] = kNone;
    // `last`: a tile that ends inside; steps past K take rows of zeros (their codes are 0)
    auto add = [&](const Block& b, int k, auto last) {
        bf16x8 xv[4][MT];
#pragma unroll
        for (int t = 0; t < MT; ++t) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                xv[i][t] = !decltype(last)::value || 128 * k + 32 * i < K
                               ? *reinterpret_cast<const bf16x8*>(x[t] + 128 * k + 32 * i)
                               : all_of(0);
        }
        if constexpr (E2M1) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    const bf16x8 v = b.w[j].step(i);
#pragma unroll
                    for (int t = 0; t < MT; ++t) acc[j][t] = mfma16(v, xv[i][t], acc[j][t]);
                }
        } else {
            const bf16x8 ones = all_of(0x3F80u);
#pragma unroll
            for (int p = 0; p < PT; ++p) {
                f32x4 part[NT][MT], sum[MT];
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    sum[t] = kNone;
#pragma unroll
                    for (int j = 0; j < NT; ++j) part[j][t] = kNone;
                }
#pragma unroll
                for (int i = p * (4 / PT); i < (p + 1) * (4 / PT); ++i) {
#pragma unroll
                    for (int t = 0; t < MT; ++t) sum[t] = mfma16(ones, xv[i][t], sum[t]);
#pragma unroll
                    for (int j = 0; j < NT; ++j) {
                        const bf16x8 v = b.w[j].step(i);
#pragma unroll
                        for (int t = 0; t < MT; ++t) part[j][t] = mfma16(v, xv[i][t], part[j][t]);
                    }
                }
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    const f32x4 s = b.s[j].scale(p), z = b.s[j].zero(p);
#pragma unroll
                    for (int t = 0; t < MT; ++t)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            acc[j][t][e] = fmaf(s[e], fmaf(-z[e], sum[t][e], part[j][t][e]), acc[j][t][e]);
                }
                if constexpr (MT > 1) __builtin_amdgcn_sched_barrier(0);  // no group's products before the last one's: spills
            }
        }
    };
    for (int k = wave; k < whole; k += AHEAD * waves) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int at = k + u * waves;
            if (at >= whole) break;
            add(blocks[u], at, std::false_type{});
            if (at + AHEAD * waves < whole) load(blocks[u], at + AHEAD * waves);
        }
    }
    if (whole < tiles_k && wave == whole % waves) {
        load(blocks[0], whole);
        add(blocks[0], whole, std::true_type{});
    }
    if constexpr (STAGED) __syncthreads();  // the rows have been read
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int t = 0; t < MT; ++t)
            *reinterpret_cast<f32x4*>(sums + (((wave * NT + j) * MT + t) * 16 + (lane & 15)) * 16 + 4 * q) = acc[j][t];
    __syncthreads();
    for (int i = threadIdx.x; i < NT * MT * 64; i += blockDim.x) {
        const int c = 4 * (i & 3), row = (i >> 2) % (16 * MT), j = (i >> 2) / (16 * MT);
        if (m0 + row >= g.c.M) continue;
        f32x4 v = *reinterpret_cast<const f32x4*>(sums + (j * MT * 16 + row) * 16 + c);
        for (int w = 1; w < waves; ++w)
            v += *reinterpret_cast<const f32x4*>(sums + ((w * NT + j) * MT * 16 + row) * 16 + c);
        put4(g, m0 + row, (int)((blockIdx.x * NT + j) * 16) + c, v);
    }
}

// ---------------------------------------------------------------------------
// Many rows.  A workgroup of 2 x WN waves computes 32 MI rows x 16 NI WN outputs, a
// wave 16 MI x 16 NI.  Rows, codes and scales pass through a ring of LDS stages of
// 128 inputs, copied there by buffer loads that the kernel counts by hand; codes
// are widened in the registers of the waves that use them.  A call with few tiles
// splits its inputs over workgroups, whose sums a second kernel joins in order.
// 2048 x 4096 x 4096: int4 70 us (0.98 PFLOP/s), e2m1 56 (1.23; a bf16 product of
// 8192^3 by the library reaches 1.39); 2048 x 4096 x 1024 23 and 19.  Bound by the
// copies (8.8 TB/s out of L2, a workgroup a CU) with the first stages' and the
// epilogue's latency; int4 issues a quarter more products for the sums of rows.
constexpr int kMostSplits = 8;
__host__ __device__ constexpr int partial_width(int N) { return (N + 3) & ~3; }

template <int MI, int NI, int WN>
struct Wide {
    static constexpr int TM = 32 * MI, TN = 16 * NI * WN, kWaves = 2 * WN;
    static constexpr int STAGES = MI == 1 ? 4 : 3;
    static constexpr int kRowBytes = TM * 256;                    // two halves of 64 inputs, rows of 128 bytes each
    static constexpr int kScales = kRowBytes + TN * 64;           // behind them the codes,
    static constexpr int kScaleBytes = TN > 128 ? TN * 8 : 1024;  // scales (as of groups of 32)
    static constexpr int kZeros = kScales + kScaleBytes;
    static constexpr int kStage = kZeros + 1024;                  // and zero points
    static constexpr int kCopies = TM / 4 / kWaves;               // of 1 KB of rows, a wave and stage,
    static constexpr int kCodes = TN / 16 / kWaves;               // and of codes
    static constexpr int kLoads = kCopies + kCodes;
    static constexpr size_t kLds = STAGES * kStage;
};

// raw_buffer() in scalar registers.
__device__ __forceinline__ u32x4 buffer_of(const void* p, uint64_t bytes) {
    u32x4 b = raw_buffer(p, bytes);
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = __builtin_amdgcn_readfirstlane(b[i]);
    return b;
}

template <bool E2M1, bool ZEROS, int PT, int MI, int NI, int WN>
__global__ __launch_bounds__(128 * WN, 2) void w4_wide_kernel(W4Args g, int splits, float* __restrict__ partial) {
    using S = Wide<MI, NI, WN>;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4;
    const int wm = wave & 1, wn = wave >> 1, tiles_k = (int)g.s.tiles_k;
    const int split = (int)(blockIdx.x % (unsigned)splits), block = (int)(blockIdx.x / (unsigned)splits);
    const int k0 = (int)((int64_t)tiles_k * split / splits), k1 = (int)((int64_t)tiles_k * (split + 1) / splits);
    // Tile of this workgroup (workgroup b runs on XCD b % 8): an XCD takes a run of
    // the walk along the rows, so that its rows and weights meet in its L2.
    const int nm = (int)((g.c.M + S::TM - 1) / S::TM), nn = (g.s.N + S::TN - 1) / S::TN;
    int tm, tn;
    {
        const int tiles = nm * nn, xcd = block % 8;
        const int i = xcd * (tiles / 8) + min(xcd, tiles % 8) + block / 8;
        tn = i / nm;
        tm = i - tn * nm;
    }
    const int64_t m0 = (int64_t)tm * S::TM;
    const int n0 = tn * S::TN;
    const uint16_t* const base = g.c.a + m0 * g.c.a_stride;
    const u32x4 buf = buffer_of(base, ((uint64_t)(g.c.M - 1 - m0) * g.c.a_stride + g.s.K) * 2);
    static_assert(S::TM / 8 % S::kCopies == 0, "a wave's runs lie in one half");
    const int run = wave * S::kCopies;
    W4RowCopies<S::TM, S::kCopies> from(lane, run, g.c.M - 1 - m0, (uint32_t)g.c.a_stride * 2);
    const uint32_t lds0 = lds_addr(smem);
    const int64_t tile0 = n0 / 16;
    // Scales, 32 PT bytes a tile (E2M1 64), and zero points, 16 PT: a copy each of
    // 64 lanes (two where the tiles have more); lanes past the last tile repeat it.
    constexpr int kScaleLanes = E2M1 ? 4 : 2 * PT, kTiles = S::TN / 16;
    constexpr int kScaleCopies = (kTiles * kScaleLanes + 63) / 64;
    static_assert(kTiles * PT <= 64 && kScaleCopies * 1024 <= S::kScaleBytes && kScaleCopies < S::kWaves, "");
    const int sl = lane + 64 * min(wave, kScaleCopies - 1);
    const int st = min(sl / kScaleLanes, kTiles - 1), zt = min(lane / PT, kTiles - 1);
    const uint32_t scale_off = (uint32_t)(min(tile0 + st, g.s.tiles_n - 1) * tiles_k * (16 * kScaleLanes)) +
                               16 * (sl % kScaleLanes);
    const uint32_t zero_off = (uint32_t)(min(tile0 + zt, g.s.tiles_n - 1) * tiles_k * (16 * PT)) + 16 * (lane % PT);
    const u32x4 scale_buf = buffer_of(g.scales, g.s.scales_size());
    const u32x4 zero_buf = buffer_of(g.zeros, ZEROS ? g.s.zeros_size() : 0);
    const bool extra = wave < kScaleCopies || (ZEROS && wave == kScaleCopies);  // this wave's stages have a copy more
    u32x4 code_buf[S::kCodes];  // of its tiles
#pragma unroll
    for (int j = 0; j < S::kCodes; ++j)
        code_buf[j] = buffer_of(g.codes + min(tile0 + wave * S::kCodes + j, g.s.tiles_n - 1) * tiles_k * 1024,
                                (uint64_t)tiles_k * 1024);
    auto copy = [&](int k, int slot) {
        const uint32_t to = lds0 + slot * S::kStage;
        if (128 * k + 128 > g.s.K) from.shorten((uint32_t)(g.s.K - 128 * k) * 2);  // the last tile, once
#pragma unroll
        for (int j = 0; j < S::kCopies; ++j)
            buffer_to_lds(buf, from.at[j], (uint32_t)k * 256u, to + (run + j) * 1024);
#pragma unroll
        for (int j = 0; j < S::kCodes; ++j)
            buffer_to_lds(code_buf[j], 16 * lane, (uint32_t)k * 1024u, to + S::kRowBytes + (wave * S::kCodes + j) * 1024);
        if (wave < kScaleCopies)
            buffer_to_lds(scale_buf, scale_off, (uint32_t)k * (16 * kScaleLanes), to + S::kScales + wave * 1024);
        else if (ZEROS && wave == kScaleCopies)
            buffer_to_lds(zero_buf, zero_off, (uint32_t)k * (16 * PT), to + S::kZeros);
    };
    auto scale = [&](int slot, int i, int p) {
        return four_bf16(*reinterpret_cast<const uint2*>(smem + slot * S::kStage + S::kScales +
                                                         ((wn * NI + i) * 4 + q) * (8 * PT) + 8 * p));
    };
    auto zero = [&](int slot, int i, int p) {
        return four_bytes(*reinterpret_cast<const uint32_t*>(smem + slot * S::kStage + S::kZeros +
                                                             ((wn * NI + i) * 4 + q) * (4 * PT) + 4 * p));
    };
    auto codes = [&](int slot, int i) {
        const char* const at = smem + slot * S::kStage;
        Codes<E2M1> c;
        c.w = *reinterpret_cast<const u32x4*>(at + S::kRowBytes + (wn * NI + i) * 1024 + 16 * lane);
        if constexpr (E2M1)
            c.bytes = *reinterpret_cast<const uint32_t*>(at + S::kScales + (wn * NI + i) * 64 + 4 * (lane & 15));
        return c;
    };
    // rows 16 t + l % 16 of the wave's, piece 4 (i % 2) + q of half i / 2
    const uint32_t row = wm * (S::TM / 2) + (lane & 15);
    auto rows = [&](int slot, int i, int t) {
        const uint32_t at = slot * S::kStage + (i >> 1) * (S::TM * 128) + (row + 16 * t) * 128 +
                            16 * ((4 * (i & 1) + q) ^ (row & 7));
        return *reinterpret_cast<const bf16x8*>(smem + at);
    };
    f32x4 acc[NI][MI];
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int t = 0; t < MI; ++t) acc[i][t] = kNone;
    constexpr int kSteps = E2M1 ? 1 : 4 / PT;  // products of 32 inputs between two scalings
    // Small tiles: every product's chain apart, for there is little else to hide
    // their latency; large ones start a tile's chain from its zero points' part, an
    // output tile after the other, for their registers.
    constexpr bool APART = MI <= 2 || E2M1;
    // `last`: the tile may end inside; steps past K take rows of zeros (their codes are 0)
    auto add = [&](int k, int slot, auto last) {
        Codes<E2M1> cur[NI];  // small tiles: all at once
        if constexpr (APART)
#pragma unroll
            for (int i = 0; i < NI; ++i) cur[i] = codes(slot, i);
#pragma unroll
        for (int p = 0; p < 4 / kSteps; ++p) {
            bf16x8 x[kSteps][MI];
#pragma unroll
            for (int j = 0; j < kSteps; ++j)
#pragma unroll
                for (int t = 0; t < MI; ++t) {
                    x[j][t] = rows(slot, p * kSteps + j, t);
                    if (decltype(last)::value && 128 * k + 32 * (p * kSteps + j) >= g.s.K) x[j][t] = all_of(0);
                }
            if constexpr (E2M1) {
#pragma unroll
                for (int i = 0; i < NI; ++i) {
                    const bf16x8 v = cur[i].step(p);
#pragma unroll
                    for (int t = 0; t < MI; ++t) acc[i][t] = mfma16(v, x[0][t], acc[i][t]);
                }
            } else {
                const bf16x8 ones = all_of(ZEROS || APART ? 0x3F80u : 0xC100u);  // 1 or -8
                f32x4 sum[MI];
#pragma unroll
                for (int t = 0; t < MI; ++t) sum[t] = kNone;
#pragma unroll
                for (int j = 0; j < kSteps; ++j)
#pragma unroll
                    for (int t = 0; t < MI; ++t) sum[t] = mfma16(ones, x[j][t], sum[t]);
                if constexpr (APART) {
                    f32x4 part[NI][MI];
#pragma unroll
                    for (int i = 0; i < NI; ++i)
#pragma unroll
                        for (int t = 0; t < MI; ++t) part[i][t] = kNone;
#pragma unroll
                    for (int j = 0; j < kSteps; ++j)
#pragma unroll
                        for (int i = 0; i < NI; ++i) {
                            const bf16x8 v = cur[i].step(p * kSteps + j);
#pragma unroll
                            for (int t = 0; t < MI; ++t) part[i][t] = mfma16(v, x[j][t], part[i][t]);
                        }
#pragma unroll
                    for (int i = 0; i < NI; ++i) {
                        const f32x4 s = scale(slot, i, p), z = ZEROS ? zero(slot, i, p) : f32x4{8.f, 8.f, 8.f, 8.f};
#pragma unroll
                        for (int t = 0; t < MI; ++t)
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                acc[i][t][e] = fmaf(s[e], fmaf(-z[e], sum[t][e], part[i][t][e]), acc[i][t][e]);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < NI; ++i) {
                        f32x4 part[MI];
                        const Codes<E2M1> own = codes(slot, i);
                        const f32x4 s = scale(slot, i, p);
                        if constexpr (ZEROS) {
                            const f32x4 z = zero(slot, i, p);
#pragma unroll
                            for (int t = 0; t < MI; ++t)
#pragma unroll
                                for (int e = 0; e < 4; ++e) part[t][e] = -z[e] * sum[t][e];
                        } else {
#pragma unroll
                            for (int t = 0; t < MI; ++t) part[t] = sum[t];
                        }
#pragma unroll
                        for (int j = 0; j < kSteps; ++j) {
                            const bf16x8 v = own.step(p * kSteps + j);
#pragma unroll
                            for (int t = 0; t < MI; ++t) part[t] = mfma16(v, x[j][t], part[t]);
                        }
#pragma unroll
                        for (int t = 0; t < MI; ++t)
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[i][t][e] = fmaf(s[e], part[t][e], acc[i][t][e]);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
            }
        }
    };
    constexpr int kAhead = S::STAGES - 1;  // stages on their way: all but the one that is being read
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
        if (k0 + u < k1) copy(k0 + u, u);
    int slot = 0;
    auto stage = [&](int k, auto last) {
        if (k + kAhead - 1 >= k1)
            wait_loads<0>();
        else if (extra)
            wait_loads<(kAhead - 1) * (S::kLoads + 1)>();
        else
            wait_loads<(kAhead - 1) * S::kLoads>();
        barrier();  // this stage is there, and everyone has read the last one
        if (k + kAhead < k1) copy(k + kAhead, slot == 0 ? S::STAGES - 1 : slot - 1);
        add(k, slot, last);
        slot = slot + 1 == S::STAGES ? 0 : slot + 1;
    };
    // the tile that ends inside apart: two forms in one loop move the accumulators between them
    const int whole = min(k1, g.s.K / 128);
    for (int k = k0; k < whole; ++k) stage(k, std::false_type{});
    if (whole < k1) stage(whole, std::true_type{});
    if (splits == 1 && g.c.out_bf16 && (g.s.N & 7) == 0) {
#pragma unroll
        for (int t = 0; t < MI; ++t)
#pragma unroll
            for (int i = 0; i < NI; i += 2)
                put_pair(g, m0 + row + 16 * t, n0 + 16 * (wn * NI + i), q, acc[i][t], acc[i + 1][t]);
        return;
    }
#pragma unroll
    for (int t = 0; t < MI; ++t)
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int64_t m = m0 + row + 16 * t;
            const int n = n0 + 16 * (wn * NI + i) + 4 * q;
            if (splits == 1)
                put4(g, m, n, acc[i][t]);
            else if (m < g.c.M && n < g.s.N)
                *reinterpret_cast<f32x4*>(partial + (split * g.c.M + m) * partial_width(g.s.N) + n) = acc[i][t];
        }
}

// The splits' parts of four outputs added in order.
__global__ __launch_bounds__(256) void w4_join_kernel(W4Args g, int splits, const float* __restrict__ partial) {
    const int width = partial_width(g.s.N);
    const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4, all = g.c.M * width;
    if (at >= all) return;
    f32x4 part[kMostSplits];  // their loads in flight together
#pragma unroll
    for (int s = 0; s < kMostSplits; ++s)
        part[s] = s < splits ? *reinterpret_cast<const f32x4*>(partial + s * all + at) : kNone;
    f32x4 v = part[0];
#pragma unroll
    for (int s = 1; s < kMostSplits; ++s) v += part[s];
    const int64_t m = at / width;
    put4(g, m, (int)(at - m * width), v);
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
constexpr int kGridY = 32768;  // rows of tiles in the grid's second dimension
__device__ __forceinline__ Spot spot_of(const W4Shape& s) {
    const int r = threadIdx.x >> 4, j = threadIdx.x & 15;
    const int64_t tn = (int64_t)blockIdx.z * kGridY + blockIdx.y;
    Spot p;
    p.tile = tn * s.tiles_k + blockIdx.x;
    p.n = (int)(16 * tn) + r;
    p.k = (int)(128 * blockIdx.x) + 8 * j;
    p.word = (16 * (j & 3) + r) * 4 + (j >> 2);
    p.pair = r;
    p.in = p.n < s.N && p.k < s.K;
    return p;
}
// Where a tile's scale (and zero point) of output r's group j lies.
__device__ __forceinline__ int scale_place(const W4Shape& s, int r, int j) {
    return s.e2m1 ? r * s.per_tile() + j : (r >> 2) * 4 * s.per_tile() + 4 * j + (r & 3);
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

// Over the aligned group of LANES lanes that holds a group's values, by moves within
// a row of sixteen.
template <int LANES, typename F>
__device__ __forceinline__ float group_fold(float x, F f) {
    x = f(x, dpp_f32<kDppXor1>(x));
    x = f(x, dpp_f32<kDppXor2>(x));
    if constexpr (LANES > 4) x = f(x, dpp_f32<kDppHalfMirror>(x));
    if constexpr (LANES > 8) x = f(x, dpp_f32<kDppMirror>(x));
    return x;
}

// The smallest bf16 value s with steps * s >= hi - lo (finite), as its bits: one of
// four from just below the rounded quotient on, compared exactly in fp64.
__device__ __forceinline__ uint32_t scale_for(float hi, float lo, float steps) {
    const double reach = (double)hi - (double)lo;
    uint32_t b = __float_as_uint((float)(reach * (1. / (double)steps))) >> 16;  // reach itself may pass fp32's range
    b = b > 0 ? b - 1 : 0;
#pragma unroll
    for (int i = 0; i < 3; ++i)
        if ((double)steps * (double)bf16_bits_to_f32(b) < reach) ++b;
    return b;
}

// x / s to the nearest whole number, ties to even, for a bf16 s > 0 and |x| <= 15.5
// s, from a whole number at most one away: by the remainder, which one fused
// operation gives exactly (n s has 12 bits, and x - n s no more than x's at s).
__device__ __forceinline__ float put_right(float n, float x, float s) {
    const float r = 2.f * fmaf(-n, s, x), off = fabsf(r);
    return n + (off > s || (off == s && ((int)n & 1)) ? copysignf(1.f, r) : 0.f);
}

// HBM-bound but for short calls: 16384 x 4096 in fp32 to int4 with zero points 67 us
// (302 MB, 4.5 TB/s); 106 with quotients in fp64, 86 with put_right() for every value.
template <bool F32, bool E2M1, bool ZEROS, int PT>
__global__ __launch_bounds__(256) void w4_quantize_kernel(W4Shape s, const void* __restrict__ w,
                                                          char* __restrict__ packed) {
    constexpr int LANES = 16 / PT;  // of a group
    __shared__ uint32_t words[256];
    const Spot p = spot_of(s);
    if (p.n - (int)(threadIdx.x >> 4) >= s.N) return;  // a row of tiles past the last: the same for the workgroup
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = 0.f;
    if (p.in) load8<F32>(w, (int64_t)p.n * s.K + p.k, x);
    float lo = 0.f, hi = 0.f, big = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if constexpr (ZEROS) lo = fminf(lo, x[e]);
        if constexpr (ZEROS) hi = fmaxf(hi, x[e]);
        // magnitudes as bits: those of infinities and NaN are the largest, and as floats fmaxf drops NaN
        big = __uint_as_float(max(__float_as_uint(big), __float_as_uint(x[e]) & 0x7FFFFFFFu));
    }
    auto most = [](float a, float b) { return __uint_as_float(max(__float_as_uint(a), __float_as_uint(b))); };
    if constexpr (ZEROS) {
        lo = group_fold<LANES>(lo, [](float a, float b) { return fminf(a, b); });
        hi = group_fold<LANES>(hi, [](float a, float b) { return fmaxf(a, b); });
    }
    big = group_fold<LANES>(big, most);
    const bool bad = __float_as_uint(big) >= 0x7F800000u;
    const int j = threadIdx.x & 15, at = scale_place(s, p.pair, j / LANES);
    char* const scales = packed + s.codes_size() + p.tile * (16 * PT * (E2M1 ? 1 : 2));
    uint8_t* const zeros = reinterpret_cast<uint8_t*>(packed + s.codes_size() + s.scales_size()) + p.tile * 16 * PT;
    uint32_t word = 0;
    if constexpr (E2M1) {
        // the smallest exponent that brings the largest magnitude to 6 = 1.5 * 2^2 or below
        const uint32_t bits = __float_as_uint(big);
        const int byte = bad ? 255 : max((int)(bits >> 23) - 2 + ((bits & 0x7FFFFFu) > 0x400000u ? 1 : 0), 0);
        float y[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = ldexpf(x[e], 127 - byte);
        word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, y[0], y[1], 1.f, 0);
        word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, y[2], y[3], 1.f, 1);
        word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, y[4], y[5], 1.f, 2);
        word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, y[6], y[7], 1.f, 3);
        if (j % LANES == 0) scales[at] = (char)(uint8_t)(p.in ? byte : 0);
    } else {
        if (bad) lo = hi = big = 0.f;
        const uint32_t bits = ZEROS ? scale_for(hi, lo, 15.f) : scale_for(big, 0.f, 7.f);
        float by = bits ? bf16_bits_to_f32(bits) : 1.f;
        const float lift = by < 0x1p-100f ? 0x1p60f : 1.f;  // exact, and 1 / by stays within fp32
        by *= lift;
        const float inv = 1.f / by;
        const float z = ZEROS ? fminf(put_right(rintf(-lo * lift * inv), -lo * lift, by), 15.f) : 8.f;
        float n[8], far = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            x[e] *= lift;
            const float quot = x[e] * inv;  // within 2^-18 of the exact one
            n[e] = rintf(quot);
            far = fmaxf(far, fabsf(quot - n[e]));
        }
        if (__any(far > 0.49999f))  // a border may lie between
#pragma unroll
            for (int e = 0; e < 8; ++e) n[e] = put_right(n[e], x[e], by);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            word |= (uint32_t)fminf(fmaxf(n[e] + z, 0.f), 15.f) << (e < 4 ? 8 * e : 8 * (e - 4) + 4);
        if (j % LANES == 0) {
            reinterpret_cast<uint16_t*>(scales)[at] = (uint16_t)(!p.in ? 0u : bad ? 0x7FC0u : bits);
            if constexpr (ZEROS) zeros[at] = (uint8_t)(p.in ? (uint32_t)z : 0u);
        }
    }
    words[p.word] = p.in && !bad ? word : 0u;
    __syncthreads();
    reinterpret_cast<uint32_t*>(packed + p.tile * 1024)[threadIdx.x] = words[threadIdx.x];
}

__global__ __launch_bounds__(256) void w4_pack_kernel(W4Shape s, const uint8_t* __restrict__ codes,
                                                      const void* __restrict__ scales,
                                                      const uint8_t* __restrict__ zeros, char* __restrict__ packed) {
    __shared__ uint32_t words[256];
    const Spot p = spot_of(s);
    if (p.n - (int)(threadIdx.x >> 4) >= s.N) return;  // a row of tiles past the last: the same for the workgroup
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
        const int64_t from = in ? (int64_t)p.n * groups + k / s.group : 0;
        const int64_t to = p.tile * 16 * per + scale_place(s, p.pair, j);
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
    const int64_t at = p.tile * 16 * per + scale_place(s, p.pair, (8 * j) / s.group);
    const char* const sc = packed + s.codes_size();
    float v[8];
    if (s.e2m1) {
        const uint32_t byte = (uint8_t)sc[at];
        typedef float f32x2 __attribute__((ext_vector_type(2)));
        const f32x2 pairs[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 1),
                                __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 3)};
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] = byte == 255 ? __builtin_nanf("") : ldexpf(pairs[e >> 1][e & 1], (int)byte - 127);
    } else {
        const float scale = bf16_bits_to_f32(reinterpret_cast<const uint16_t*>(sc)[at]);
        const float z = s.zeros ? (float)(uint8_t)(packed + s.codes_size() + s.scales_size())[at] : 8.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = scale * ((float)code_at(w, e, false) - z);
    }
    store8<F32>(out, (int64_t)p.n * s.K + p.k, v);
}

template <typename Go>
void by_weights(const W4Shape& s, Go go) {
    using std::integral_constant;
    auto with = [&](auto pt) { s.zeros ? go(std::false_type{}, std::true_type{}, pt) : go(std::false_type{}, std::false_type{}, pt); };
    if (s.e2m1)
        go(std::true_type{}, std::false_type{}, integral_constant<int, 4>{});
    else if (s.group == 32)
        with(integral_constant<int, 4>{});
    else if (s.group == 64)
        with(integral_constant<int, 2>{});
    else
        with(integral_constant<int, 1>{});
}

dim3 tile_grid(const W4Shape& s) {
    const int64_t y = std::min<int64_t>(s.tiles_n, kGridY);
    return dim3((unsigned)s.tiles_k, (unsigned)y, (unsigned)((s.tiles_n + kGridY - 1) / kGridY));
}

}  // namespace

hipError_t launch_w4_quantize(const W4Shape& s, bool f32, const void* w, char* packed, hipStream_t stream) {
    by_weights(s, [&](auto e2m1, auto zeros, auto pt) {
        constexpr bool E2M1 = decltype(e2m1)::value, ZEROS = decltype(zeros)::value;
        constexpr int PT = decltype(pt)::value;
        if (f32)
            w4_quantize_kernel<true, E2M1, ZEROS, PT><<<tile_grid(s), 256, 0, stream>>>(s, w, packed);
        else
            w4_quantize_kernel<false, E2M1, ZEROS, PT><<<tile_grid(s), 256, 0, stream>>>(s, w, packed);
    });
    return hipGetLastError();
}

hipError_t launch_w4_pack(const W4Shape& s, const uint8_t* codes, const void* scales, const uint8_t* zeros,
                          char* packed, hipStream_t stream) {
    w4_pack_kernel<<<tile_grid(s), 256, 0, stream>>>(s, codes, scales, zeros, packed);
    return hipGetLastError();
}

hipError_t launch_w4_unpack(const W4Shape& s, bool f32, const char* packed, void* w, hipStream_t stream) {
    if (f32)
        w4_unpack_kernel<true><<<tile_grid(s), 256, 0, stream>>>(s, packed, w);
    else
        w4_unpack_kernel<false><<<tile_grid(s), 256, 0, stream>>>(s, packed, w);
    return hipGetLastError();
}

namespace {

// Which kernel a call takes, by its sizes alone (us of both sides, int4 with groups
// of 128 unless said; weights out of the caches).
//   Up to 16 rows: the rows kernel, 16 outputs a workgroup, from 512 tiles of
//   outputs on 32 and from 1024 on 64: reading the rows once a workgroup is what
//   bounds wider calls (L2 gives all CUs together 8.8 TB/s).  16 x 4096 x 4096 (16
//   outputs / 32 / 64) 7.4 / 7.5 / 8.6, 16 x 8192 x 4096 11.6 / 8.1 / 8.8, 16 x
//   16384 x 4096 19.5 / 12.7 / 9.7, 1 x 8192 x 4096 6.8 / 6.3 / 7.7, 1 x 32000 x
//   4096 22.5 / 17.6 / 16.0.
//   Up to 32 rows the same (32 x 16384 x 4096 33 / 20 / 13.6), but with groups of
//   32, whose scales leave no registers for 64 outputs (23 / 40 at 32 / 64, with
//   zero points 23 / 88).
//   Up to 64 rows the same where there is little to split: 64 x 4096 x 1024 6.6
//   against the wide kernel's 6.8 (e2m1 6.5 and 5.8, groups of 32 with zero points
//   6.9 and 8.7), 40 rows of it 5.5 and 6.8 (5.6 and 5.8, 5.9 and 8.7), but 64 x 4096
//   x 4096 18.1 and 14.3.
//   Beyond: the wide kernel, in the largest tiles that make a workgroup for every
//   CU (and are not mostly past N): 2048 x 4096 x 1024 in tiles of 128 x 256 23.2,
//   64 x 128 28.5, 64 x 64 35; 1024 x 4096 x 1024 20.8 / 16.3 / 18.9.  With fewer
//   tiles of 64 x 64 than that, long sums are split until there are 512 workgroups
//   (128 x 4096 x 4096 unsplit 24.0, in four 17.4; 512 x 1024 x 4096 24.1 / 17.1);
//   short ones take tiles of 32 x 64 (128 x 4096 x 1024 8.1 / 7.0, split in two 9.8).
//   From 8192 inputs on the largest tiles are split into up to four where that makes
//   192 to 256 workgroups of them: 512 x 8192 x 8192 93 -> 80 (e2m1 68 -> 65), 1000 x
//   2048 x 8192 61 -> 47 (44 -> 40), 800 x 2048 x 16384 110 -> 77 (80 -> 62); with 288
//   workgroups 300 x 8192 x 8192 89 -> 100, with 4096 inputs 512 x 4096 32 -> 34, half
//   empty 64 x 16384 x 8192 37 -> 45; unsplit 1500 x 4096 x 8192 145 -> 131, but in
//   groups of 32 with zero points 210 -> 241.
//   What the rule does not look at: how far the largest tiles' last round fills the
//   chip (257 to 511 of them take as long as 512) and how much of them lies past M.
//   There it is behind tiles of 64 x 128: 2048 x 5120 x 5120 164 and 155, 2048 x 4112
//   x 4096 132 and 116, 1024 x 9216 x 4096 132 and 115, 520 x 16384 x 4096 132 and
//   112, 64 x 131072 x 4096 141 and 103 (e2m1 116 and 79).
enum Kernel { kRows, kWide32x64, kWide64x64, kWide64x128, kWide128x256 };
struct Plan {
    Kernel kernel;
    int splits;
};
Plan plan_of(const W4Shape& s, int64_t M) {
    if (M <= 32 || (M <= 64 && s.tiles_k <= 8 && s.tiles_n <= 256)) return {kRows, 1};
    auto tiles = [&](int tm, int tn) { return ((M + tm - 1) / tm) * ((s.N + tn - 1) / tn); };
    if (tiles(128, 256) >= 256 && s.N > 128) return {kWide128x256, 1};
    const int64_t large = tiles(128, 256), part = std::min<int64_t>(256 / large, 4);
    if (M > 64 && s.N > 128 && large * part >= 192 && s.tiles_k >= std::max<int64_t>(64, 16 * part) &&
        (part > 1 || s.e2m1 || s.group > 32))
        return {kWide128x256, (int)part};
    if (tiles(64, 128) >= 256 && s.N > 64) return {kWide64x128, 1};
    const int64_t t = tiles(64, 64);
    if (s.tiles_k <= 8) return {t >= 256 ? kWide64x64 : kWide32x64, 1};
    const int64_t splits = std::min<int64_t>({512 / t, s.tiles_k / 4, kMostSplits});
    return {kWide64x64, (int)std::max<int64_t>(splits, 1)};
}

// Whether the rows kernel stages its rows: long ones that fit, where a wave goes
// round often enough (1 x 16384 x 16384 26 us; tile by tile, 16, 32 or 64 outputs a
// workgroup, 34 / 27 / 28; 1 x 4096 x 16384 10.1 and 11.2, but 16 x 4096 x 1024 4.1
// and 3.7, 4 x 4096 x 4096 6.0 and 5.5).
bool stages_rows(const W4Shape& s, int64_t M) {
    return s.tiles_k >= 96 && (size_t)M * staged_stride(s.K) * 2 <= kStaged;
}

template <bool E2M1, bool ZEROS, int PT, int MT, int NT>
void launch_rows(const W4Args& g, hipStream_t stream) {
    const int waves = g.s.tiles_k >= 8 ? 8 : 4;
    const dim3 grid((unsigned)((g.s.tiles_n + NT - 1) / NT), (unsigned)((g.c.M + 16 * MT - 1) / (16 * MT)));
    const size_t sums = (size_t)waves * NT * MT * 1024;
    if constexpr (MT == 1 && NT == 1) {
        if (stages_rows(g.s, g.c.M)) {
            const size_t rows = (size_t)g.c.M * staged_stride(g.s.K) * 2;
            w4_rows_kernel<E2M1, ZEROS, PT, MT, NT, true><<<grid, 64 * waves, std::max(rows, sums), stream>>>(g);
            return;
        }
    }
    w4_rows_kernel<E2M1, ZEROS, PT, MT, NT, false><<<grid, 64 * waves, sums, stream>>>(g);
}

template <bool E2M1, bool ZEROS, int PT, int MI, int NI, int WN>
void launch_wide(const W4Args& g, int splits, float* partial, hipStream_t stream) {
    using S = Wide<MI, NI, WN>;
    auto* k = &w4_wide_kernel<E2M1, ZEROS, PT, MI, NI, WN>;
    if (S::kLds > 64 * 1024)
        (void)hipFuncSetAttribute(reinterpret_cast<const void*>(k), hipFuncAttributeMaxDynamicSharedMemorySize,
                                  (int)S::kLds);
    const int64_t tiles = ((g.c.M + S::TM - 1) / S::TM) * ((g.s.N + S::TN - 1) / S::TN);
    k<<<(unsigned)(tiles * splits), 128 * WN, S::kLds, stream>>>(g, splits, partial);
    if (splits > 1)
        w4_join_kernel<<<(unsigned)((g.c.M * partial_width(g.s.N) / 4 + 255) / 256), 256, 0, stream>>>(g, splits, partial);
}

}  // namespace

size_t w4_workspace_bytes(const W4Shape& s, int64_t M) {
    const int splits = plan_of(s, M).splits;
    return splits > 1 ? align256((size_t)M * partial_width(s.N) * 4 * splits) : 0;
}

hipError_t launch_linear_w4(const W4Shape& s, const W4Call& c, void* workspace, hipStream_t stream) {
    const W4Args g{s, c, c.packed, c.packed + s.codes_size(),
                   s.zeros ? reinterpret_cast<const uint8_t*>(c.packed + s.codes_size() + s.scales_size()) : nullptr};
    // a tile's rows are within 32-bit offsets of its first
    const Plan plan = c.a_stride < 1 << 24 ? plan_of(s, c.M) : Plan{kRows, 1};
    by_weights(s, [&](auto e2m1, auto zeros, auto pt) {
        constexpr bool E2M1 = decltype(e2m1)::value, ZEROS = decltype(zeros)::value;
        constexpr int PT = decltype(pt)::value;
        float* const partial = static_cast<float*>(workspace);
        switch (plan.kernel) {
            case kWide32x64: return launch_wide<E2M1, ZEROS, PT, 1, 2, 2>(g, plan.splits, partial, stream);
            case kWide64x64: return launch_wide<E2M1, ZEROS, PT, 2, 2, 2>(g, plan.splits, partial, stream);
            case kWide64x128: return launch_wide<E2M1, ZEROS, PT, 2, 2, 4>(g, plan.splits, partial, stream);
            case kWide128x256: return launch_wide<E2M1, ZEROS, PT, 4, 4, 4>(g, plan.splits, partial, stream);
            case kRows: break;
        }
        if (c.M <= 16) {
            if (s.tiles_n >= 1024 && !stages_rows(s, c.M))
                launch_rows<E2M1, ZEROS, PT, 1, 4>(g, stream);
            else if (s.tiles_n >= 512 && !stages_rows(s, c.M))
                launch_rows<E2M1, ZEROS, PT, 1, 2>(g, stream);
            else
                launch_rows<E2M1, ZEROS, PT, 1, 1>(g, stream);
        } else if (c.M <= 32) {
            constexpr int kMost = PT == 4 && !E2M1 ? 2 : 4;
            if (s.tiles_n >= 1024)
                launch_rows<E2M1, ZEROS, PT, 2, kMost>(g, stream);
            else if (s.tiles_n >= 512)
                launch_rows<E2M1, ZEROS, PT, 2, 2>(g, stream);
            else
                launch_rows<E2M1, ZEROS, PT, 2, 1>(g, stream);
        } else {  // also many rows at a stride that a tile's 32-bit offsets do not span
            launch_rows<E2M1, ZEROS, PT, 4, 1>(g, stream);
        }
    });
    return hipGetLastError();
}

}  // namespace lsh
