// The step between two blocks (lsh_residual.h): a block's output normed, gated
// and added to the residual stream, and the stream normed for the next block.
//
// A thread holds eight consecutive values of a row, so a row takes 1, 2, 4, 8 or
// 16 waves and each value is read once, in 16-byte pieces; mean and deviation
// are taken in two steps from registers.  A workgroup walks over rows and keeps
// its threads' weights, and in the backward their columns' sums, in registers.
// HBM-bound: 65,536 rows of 1024 (bf16, gate, both norms) forward 182 us (0.94 GB,
// 5.2 TB/s), backward 357 (1.88 GB, 5.3; 429 with 162 registers and workgroups that
// came in two rounds); 5997 fp32 rows of 1000 with all weights 25 and 41 (4.8 and 4.7
// TB/s).  16 rows of 4096 4.4 us: the launch, one trip to memory and two barriers.
#include "common.h"
#include "launch_residual.h"

namespace lsh {
namespace {

// Eight weights of a thread's columns; `other` where there are none.
__device__ __forceinline__ void weights8(const float* w, int c, bool on, float other, float* x) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = other;
    if (w && on) load8<true>(w, c, x);
}

__device__ __forceinline__ float wave_sum(float x) {
    x = group8_sum(x);
    x += dpp_f32<kDppMirror>(x);  // the other eight lanes of a row of sixteen
    return sum_xor32(sum_xor16(x));
}

// Sums over the WAVES waves of a row, the same in all of them; rows of a
// workgroup side by side.  Two places in turn, so that one barrier is enough.
template <int WAVES, int ROWS>
struct RowSums {
    float (*lds)[ROWS][2][WAVES];  // [2]
    int turn = 0, row, wave;
    __device__ __forceinline__ void two(float& a, float& b) {
        a = wave_sum(a);
        b = wave_sum(b);
        if constexpr (WAVES > 1) {
            if ((threadIdx.x & 63) == 0) {
                lds[turn][row][0][wave] = a;
                lds[turn][row][1][wave] = b;
            }
            __syncthreads();
            a = b = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                a += lds[turn][row][0][w];
                b += lds[turn][row][1][w];
            }
            turn ^= 1;
        }
    }
};

// 1 / sqrt(ms), 0 for 0.
__device__ __forceinline__ float inv_dev(float ms) {
    const bool tiny = ms < 0x1p-100f;  // the instruction takes subnormals as 0
    const float m = tiny ? ms * 0x1p80f : ms;
    float r = __builtin_amdgcn_rsqf(m);          // within 2^-22
    r = fmaf(0.5f * r, fmaf(-m * r, r, 1.f), r);  // one Newton step: the error of a row's factor is common to all its values
    r *= tiny ? 0x1p40f : 1.f;
    return ms == 0.f ? 0.f : (ms < __builtin_inff() ? r : 1.f / ms);
}

// gate' and its slope, each without cancellation.
__device__ __forceinline__ void gate_of(int kind, float g, float& v, float& slope) {
    if (kind == 2) {
        const float e = expf(-fabsf(g)), r = 1.f / (1.f + e), er = e * r;
        v = g >= 0.f ? r : er;
        slope = r * er;
        if (g != g) v = slope = g;
    } else {
        v = kind == 1 ? g : 1.f;
        slope = 1.f;
    }
}

template <int WAVES>
constexpr int kThreads = WAVES < 4 ? 256 : 64 * WAVES;
template <int WAVES>
constexpr int kRows = kThreads<WAVES> / (64 * WAVES);  // of a workgroup

// A thread's place: eight columns of one of its workgroup's rows.
template <int WAVES>
struct Place {
    int row, wave, col;
    bool on;
    __device__ __forceinline__ explicit Place(int D) {
        const int w = threadIdx.x >> 6;
        row = w / WAVES;
        wave = w - row * WAVES;
        col = 8 * (wave * 64 + (int)(threadIdx.x & 63));
        on = col < D;
        if (!on) col = 0;
    }
};

// The mean (layer norms) and 1 / deviation of up to two rows at once.
template <int WAVES>
__device__ __forceinline__ void stats(const ResidualArgs& a, RowSums<WAVES, kRows<WAVES>>& sums, bool on,
                                      const float* p, const float* q, float& mp, float& rp, float& mq, float& rq) {
    float s = 0.f, t = 0.f;
    mp = mq = 0.f;
    const float inv = 1.f / (float)a.D;
    if (a.layer) {
        if (on)
#pragma unroll
            for (int e = 0; e < 8; ++e) s += p[e], t += q[e];
        sums.two(s, t);
        mp = s * inv;
        mq = t * inv;
        s = t = 0.f;
    }
    if (on)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float d = p[e] - mp, f = q[e] - mq;
            s = fmaf(d, d, s);
            t = fmaf(f, f, t);
        }
    sums.two(s, t);
    rp = inv_dev(s * inv + a.eps);
    rq = inv_dev(t * inv + a.eps);
}

template <bool F32, int WAVES>
__global__ __launch_bounds__(kThreads<WAVES>) void residual_fwd_kernel(ResidualArgs a, const float* __restrict__ x,
                                                                       const void* __restrict__ f,
                                                                       const void* __restrict__ gate,
                                                                       float* __restrict__ y, void* __restrict__ z) {
    __shared__ float lds[2][kRows<WAVES>][2][WAVES];
    const Place<WAVES> p(a.D);
    RowSums<WAVES, kRows<WAVES>> sums{lds, 0, p.row, p.wave};
    float sc[8], pg[8], pb[8], rg[8], rb[8];
    weights8(a.scale, p.col, p.on, 1.f, sc);
    weights8(a.post_g, p.col, p.on, 1.f, pg);
    weights8(a.post_b, p.col, p.on, 0.f, pb);
    weights8(a.pre_g, p.col, p.on, 1.f, rg);
    weights8(a.pre_b, p.col, p.on, 0.f, rb);
    for (int64_t r0 = (int64_t)blockIdx.x * kRows<WAVES>; r0 < a.T; r0 += (int64_t)gridDim.x * kRows<WAVES>) {
        const int64_t t = min(r0 + p.row, a.T - 1);
        const bool mine = p.on && r0 + p.row < a.T;
        float v[8], u[8], g[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = u[e] = g[e] = 0.f;
        if (f) load8<F32>(f, t * a.f_stride + p.col, u);
        if (x) load8<true>(x, t * a.D + p.col, v);
        if (gate) load8<F32>(gate, t * a.gate_stride + p.col, g);
        float m0, r, m1, r1;
        if (a.post) {
            stats<WAVES>(a, sums, p.on, u, u, m0, r, m1, r1);
#pragma unroll
            for (int e = 0; e < 8; ++e) u[e] = fmaf((u[e] - m0) * r, pg[e], pb[e]);
        }
        if (f) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float gv, slope;
                gate_of(a.gate, g[e], gv, slope);
                v[e] = fmaf(a.alpha * sc[e] * gv, u[e], v[e]);
            }
        }
        if (y && mine) store8<true>(y, t * a.D + p.col, v);
        if (a.pre) {
            stats<WAVES>(a, sums, p.on, v, v, m0, r, m1, r1);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = fmaf((v[e] - m0) * r, rg[e], rb[e]);
            if (mine) store8<F32>(z, t * a.D + p.col, v);
        }
    }
}

// norm'(d) of a row, in place.
template <int WAVES>
__device__ __forceinline__ void norm_back(const ResidualArgs& a, RowSums<WAVES, kRows<WAVES>>& sums, bool on,
                                          const float* n, float r, float* d) {
    float s = 0.f, t = 0.f;
    if (on)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            s = fmaf(d[e], n[e], s);
            t += d[e];
        }
    sums.two(s, t);
    s *= 1.f / (float)a.D;
    t = a.layer ? t * (1.f / (float)a.D) : 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) d[e] = r * (d[e] - t - n[e] * s);
}

// partial: [workgroup][5][D].  PLAIN: neither scale nor biases, whose sums and
// weights then take no registers: four waves a SIMD in place of three.  Sixteen waves
// a row leave 128 registers, so that with scale or biases 51 (fp32) or 43 of them go
// through scratch: 4096 bf16 rows of 8192 207 us, PLAIN 150, at much the same bytes.
template <bool F32, bool PLAIN, int WAVES>
__global__ __launch_bounds__(kThreads<WAVES>, PLAIN || WAVES == 16 ? 4 : 3) void residual_bwd_kernel(
    ResidualArgs a, const float* __restrict__ y, const void* __restrict__ f, const void* __restrict__ gate,
    const float* __restrict__ dy, const float* __restrict__ dz, ResidualGrads g, float* __restrict__ partial) {
    constexpr int ROWS = kRows<WAVES>;
    __shared__ float lds[2][ROWS][2][WAVES];
    __shared__ __attribute__((aligned(16))) float cols[ROWS > 1 ? ROWS : 1][ROWS > 1 ? 512 * WAVES : 1];
    const Place<WAVES> p(a.D);
    RowSums<WAVES, ROWS> sums{lds, 0, p.row, p.wave};
    float sc[8], pg[8], pb[8], rg[8], col[5][8];
    weights8(PLAIN ? nullptr : a.scale, p.col, p.on, 1.f, sc);
    weights8(a.post_g, p.col, p.on, 1.f, pg);
    weights8(PLAIN ? nullptr : a.post_b, p.col, p.on, 0.f, pb);
    weights8(a.pre_g, p.col, p.on, 1.f, rg);
#pragma unroll
    for (int i = 0; i < 5; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) col[i][e] = 0.f;
    for (int64_t r0 = (int64_t)blockIdx.x * ROWS; r0 < a.T; r0 += (int64_t)gridDim.x * ROWS) {
        const int64_t t = min(r0 + p.row, a.T - 1), at = t * a.D + p.col;
        const bool mine = p.on && r0 + p.row < a.T;
        float v[8], u[8], h[8], dv[8], dw[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = u[e] = h[e] = dv[e] = dw[e] = 0.f;
        if (a.pre) {
            load8<true>(y, at, v);
            load8<true>(dz, at, dw);
        }
        if (f) load8<F32>(f, t * a.f_stride + p.col, u);
        if (gate) load8<F32>(gate, t * a.gate_stride + p.col, h);
        if (dy) load8<true>(dy, at, dv);
        float mv = 0.f, rv = 0.f, mu = 0.f, ru = 0.f;
        if (a.pre || a.post) stats<WAVES>(a, sums, p.on, v, u, mv, rv, mu, ru);
        if (a.pre) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[e] = (v[e] - mv) * rv;
                if (mine) {
                    col[3][e] = fmaf(dw[e], v[e], col[3][e]);
                    if constexpr (!PLAIN) col[4][e] += dw[e];
                }
                dw[e] *= rg[e];
            }
            norm_back<WAVES>(a, sums, p.on, v, rv, dw);
#pragma unroll
            for (int e = 0; e < 8; ++e) dv[e] += dw[e];
        }
        if (mine) store8<true>(g.dx, at, dv);
        if (!f) continue;
        float n[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            n[e] = a.post ? (u[e] - mu) * ru : 0.f;
            const float uu = a.post ? fmaf(n[e], pg[e], pb[e]) : u[e];
            float gv, slope;
            gate_of(a.gate, h[e], gv, slope);
            const float dm = dv[e] * uu * a.alpha;
            h[e] = dm * sc[e] * slope;
            dv[e] *= a.alpha * sc[e] * gv;
            if (mine) {
                col[1][e] = fmaf(dv[e], n[e], col[1][e]);
                if constexpr (!PLAIN) {
                    col[0][e] = fmaf(dm, gv, col[0][e]);
                    col[2][e] += dv[e];
                }
            }
            dv[e] *= a.post ? pg[e] : 1.f;
        }
        if (gate && mine) store8<true>(g.dgate, at, h);
        if (a.post) norm_back<WAVES>(a, sums, p.on, n, ru, dv);
        if (mine) store8<true>(g.df, at, dv);
    }
    float* const out = partial + (int64_t)blockIdx.x * 5 * a.D;
#pragma unroll
    for (int i = 0; i < 5; ++i) {
        if ((PLAIN && i != 1 && i != 3) || !g.cols[i]) continue;  // uniform
        if constexpr (ROWS == 1) {
            if (p.on) store8<true>(out, (int64_t)i * a.D + p.col, col[i]);
        } else {
            __syncthreads();
            if (p.on) store8<true>(&cols[p.row][0], p.col, col[i]);
            __syncthreads();
            for (int c = threadIdx.x; c < a.D; c += kThreads<WAVES>) {
                float s = 0.f;
#pragma unroll
                for (int r = 0; r < ROWS; ++r) s += cols[r][c];
                out[(int64_t)i * a.D + c] = s;
            }
        }
    }
}

// One workgroup for 32 columns of one weight: its workgroups' partial sums added in
// fp64, in 32 interleaved runs and then those in halves.
constexpr int kRuns = 32, kRunCols = 32;
__global__ __launch_bounds__(kRuns* kRunCols) void residual_cols_kernel(const float* __restrict__ partial, int parts,
                                                                        int D, ResidualGrads g) {
    __shared__ double run[kRuns][kRunCols];
    const int i = blockIdx.y, d = threadIdx.x % kRunCols, s = threadIdx.x / kRunCols;
    const int c = (int)blockIdx.x * kRunCols + d;
    float* const to = i == 0 ? g.cols[0] : i == 1 ? g.cols[1] : i == 2 ? g.cols[2] : i == 3 ? g.cols[3] : g.cols[4];
    if (!to) return;  // uniform
    double z = 0;
#pragma unroll 8
    for (int p = s; p < parts; p += kRuns) z += partial[((int64_t)p * 5 + i) * D + min(c, D - 1)];
    run[s][d] = z;
    for (int h = kRuns / 2; h > 0; h /= 2) {
        __syncthreads();
        if (s < h) run[s][d] += run[s + h][d];
    }
    if (s == 0 && c < D) to[c] = (float)run[0][d];
}

int rows_of(int D) { return std::max(1, 4 / residual_waves(D)); }
// Workgroups: as many as are resident at once, at most, so that no second round of a
// few of them follows.  65,536 rows of 256 forward 51 us (60 with 2048 workgroups in
// place of 1280), of 1024 181 to 184 (2048 in place of 1024 the same, 1280 233), 8192
// rows of 4096 with all weights backward 196 (245 with 384 in place of 256).
int64_t groups(const ResidualArgs& a, ResidualPass pass) {
    return std::min<int64_t>((a.T + rows_of(a.D) - 1) / rows_of(a.D), residual_resident(pass, a.D));
}
bool is_plain(const ResidualArgs& a) { return !a.scale && !a.post_b && !a.pre_b; }

template <typename Go>
void by_width(int D, Go go) {
    switch (residual_waves(D)) {
        case 1: go(std::integral_constant<int, 1>{}); break;
        case 2: go(std::integral_constant<int, 2>{}); break;
        case 4: go(std::integral_constant<int, 4>{}); break;
        case 8: go(std::integral_constant<int, 8>{}); break;
        default: go(std::integral_constant<int, 16>{});
    }
}

}  // namespace

bool residual_fits(const ResidualArgs&) { return true; }  // the grids are bounded by the chip's size

size_t residual_workspace_bytes(const ResidualArgs& a) {
    return align256((size_t)groups(a, kResidualBwdPlain) * 5 * a.D * sizeof(float));  // the more of both
}

hipError_t launch_residual_fwd(const ResidualArgs& a, bool f32, const float* x, const void* f, const void* gate,
                               float* y, void* z, hipStream_t stream) {
    by_width(a.D, [&](auto w) {
        constexpr int W = decltype(w)::value;
        const unsigned grid = (unsigned)groups(a, kResidualFwd);
        if (f32)
            residual_fwd_kernel<true, W><<<grid, kThreads<W>, 0, stream>>>(a, x, f, gate, y, z);
        else
            residual_fwd_kernel<false, W><<<grid, kThreads<W>, 0, stream>>>(a, x, f, gate, y, z);
    });
    return hipGetLastError();
}

hipError_t launch_residual_bwd(const ResidualArgs& a, bool f32, const float* y, const void* f, const void* gate,
                               const float* dy, const float* dz, const ResidualGrads& g, void* workspace,
                               hipStream_t stream) {
    float* const partial = static_cast<float*>(workspace);
    const bool plain = is_plain(a);
    const unsigned grid = (unsigned)groups(a, plain ? kResidualBwdPlain : kResidualBwd);
    by_width(a.D, [&](auto w) {
        constexpr int W = decltype(w)::value;
        auto go = [&](auto kernel) { kernel<<<grid, kThreads<W>, 0, stream>>>(a, y, f, gate, dy, dz, g, partial); };
        if (f32)
            plain ? go(residual_bwd_kernel<true, true, W>) : go(residual_bwd_kernel<true, false, W>);
        else
            plain ? go(residual_bwd_kernel<false, true, W>) : go(residual_bwd_kernel<false, false, W>);
    });
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    bool any = false;
    for (const float* c : g.cols) any = any || c;
    if (!any) return hipSuccess;
    residual_cols_kernel<<<dim3((unsigned)((a.D + kRunCols - 1) / kRunCols), 5), kRuns * kRunCols, 0, stream>>>(partial, (int)grid, a.D, g);
    return hipGetLastError();
}

}  // namespace lsh
