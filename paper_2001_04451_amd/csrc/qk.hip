// Per-head norm and position rotation of projected rows, and its backward:
//   y = Rot(pos) (g * x r),  r = 1 / sqrt(mean x^2 + eps);
//   u = Rot(-pos) dy,  w = g * u,  dx = r (w - x r^2 mean(w x)),  dg = sum u * x r.
//
// gfx950 design.  Eight lanes hold a head's 64 values, eight each, so its sums
// are DPP reductions and its rows leave in 16-byte pieces.  The angles depend
// on the token alone: a workgroup forms those of its tokens once, in LDS, and
// all heads share them.  Each is pos * (freq / 2 pi) in fp64, reduced there, so
// only the fraction of a revolution reaches fp32.  A pair's other value is in
// the same lane (interleaved) or a lane shift away (halves, rot a multiple of
// 16).  The backward is held to 128 registers: four waves a SIMD, where three
// took 315 us.
// HBM-bound: 8 x 32K tokens of 8 heads in bf16 107 us forward (5.0 TB/s; a
// 2 GiB copy reaches 4.8 on this card), 282 backward with the 7 of its second
// kernel (4.9 in the first); with per-row divisions and one row's loads at a
// time both took 5-15% more.  64 tokens of 16 heads 3.9 us.
#include "launch_cache.h"
#include "qk_common.h"

namespace lsh {
namespace {

constexpr int kGroups = 32;     // eight-lane groups of a workgroup
constexpr int kAtOnce = 2;      // rows of a group whose loads are under way

struct QkArgs {
    int64_t T, L, x_stride, dx_stride;
    int Hq, Hk, rot;
    uint32_t h_magic;  // row / (Hq + Hk) as a product (more than one head)
    float eps;
};

__device__ __forceinline__ void form_angles(Angles& A, int64_t t0, int tokens, int pairs, const QkArgs& a,
                                            const float* __restrict__ freq, const int32_t* __restrict__ pos) {
    const uint32_t L = (uint32_t)a.L, b0 = L ? (uint32_t)t0 / L : 0, l0 = L ? (uint32_t)t0 % L : (uint32_t)t0;  // T < 2^31
    const int p = threadIdx.x & 31;  // a thread keeps to one pair
    const double f = p < pairs ? revolutions(freq[p]) : 0.;
    for (int t = threadIdx.x >> 5; t < tokens; t += (int)(blockDim.x >> 5)) {
        uint32_t b = b0, l = l0 + (uint32_t)t;
        if (L >= kMaxTokens) {  // one batch entry's end at most lies among the tokens
            if (l >= L) l -= L, ++b;
        } else if (L > 0) {
            b += l / L;
            l %= L;
        }
        if (p == 0) {
            A.b[t] = (int)b;
            A.l[t] = (int)l;
        }
        if (p >= pairs) continue;
        form_angle(A, t, p, pos ? (double)pos[t0 + t] : (double)l, f);
    }
}

// Where head h (of H) of the workgroup's token t0 + t starts in q, k and their gradients.
__device__ __forceinline__ int64_t out_row(const QkArgs& a, const Angles& A, int64_t t0, int t, int h, int H) {
    if (a.L > 0) return (((int64_t)A.b[t] * H + h) * a.L + A.l[t]) * kHeadDim;
    return ((t0 + t) * H + h) * kHeadDim;
}

// The rows (tokens times heads) of a workgroup's tokens, kAtOnce a group at a
// time: their loads are under way while the angles are formed.
template <bool F32, bool INTER, bool PER_HEAD>
__global__ __launch_bounds__(256) void qk_fwd_kernel(QkArgs a, int tokens_wg, const void* __restrict__ x,
                                                     const float* __restrict__ gq, const float* __restrict__ gk,
                                                     const float* __restrict__ freq, const int32_t* __restrict__ pos,
                                                     void* __restrict__ q, void* __restrict__ k) {
    __shared__ Angles A;
    const int64_t t0 = (int64_t)blockIdx.x * tokens_wg;
    const int tokens = (int)min((int64_t)tokens_wg, a.T - t0);
    const int l = threadIdx.x & 7, group = threadIdx.x >> 3, H = a.Hq + a.Hk, rows = tokens * H;
    float gs[2][8];
    if constexpr (!PER_HEAD) {
        load8<true>(gq, 8 * l, gs[0]);
        load8<true>(a.Hk ? gk : gq, 8 * l, gs[1]);
    }
    for (int r0 = 0; r0 < rows; r0 += kGroups * kAtOnce) {
        float v[kAtOnce][8];
        int t[kAtOnce], h[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            if (r0 + kGroups * u >= rows) break;
            const int r = min(r0 + kGroups * u + group, rows - 1);  // idle groups redo the last row
            t[u] = H == 1 ? r : (int)__umulhi((uint32_t)r, a.h_magic);
            h[u] = r - t[u] * H;
            load8<F32>(x, (t0 + t[u]) * a.x_stride + h[u] * kHeadDim + 8 * l, v[u]);
        }
        if (r0 == 0) {
            form_angles(A, t0, tokens, a.rot >> 1, a, freq, pos);
            __syncthreads();
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            if (r0 + kGroups * u >= rows) break;
            const bool key = h[u] >= a.Hq;
            const int hh = key ? h[u] - a.Hq : h[u];
            float g[8];
            if constexpr (PER_HEAD) {
                load8<true>(key ? gk : gq, hh * kHeadDim + 8 * l, g);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) g[e] = gs[0][e];
                if (a.Hk > 0)
#pragma unroll
                    for (int e = 0; e < 8; ++e) g[e] = key ? gs[1][e] : gs[0][e];
            }
            const float inv = inv_rms(v[u], a.eps);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[u][e] = v[u][e] * inv * g[e];
            turn<INTER>(v[u], A, t[u], l, a.rot, 1.f);
            if (r0 + kGroups * u + group < rows)
                store8<F32>(key ? k : q, out_row(a, A, t0, t[u], hh, key ? a.Hk : a.Hq) + 8 * l, v[u]);
        }
    }
}

// A workgroup takes a run of tokens; an eight-lane group keeps to one head
// (of up to 32 at a time) so that its part of the gain's gradient stays in
// registers.  partial: [workgroup][gain row][64].
template <bool F32, bool INTER, bool PER_HEAD>
__global__ __launch_bounds__(256, 4) void qk_bwd_kernel(QkArgs a, const void* __restrict__ x,
                                                        const float* __restrict__ gq, const float* __restrict__ gk,
                                                        const float* __restrict__ freq,
                                                        const int32_t* __restrict__ pos,
                                                        const float* __restrict__ dq, const float* __restrict__ dk,
                                                        float* __restrict__ dx, float* __restrict__ partial,
                                                        int gain_rows) {
    __shared__ Angles both[2];  // of the batch at hand and of the next
    __shared__ __attribute__((aligned(16))) float sums[kGroups][kHeadDim];
    const int l = threadIdx.x & 7, group = threadIdx.x >> 3, H = a.Hq + a.Hk;
    const int64_t ta = a.T * blockIdx.x / gridDim.x, tb = a.T * (blockIdx.x + 1) / gridDim.x;
    float* mine = partial + (int64_t)blockIdx.x * gain_rows * kHeadDim;
    float shared_sum = 0.f;  // thread d + 64 (0 queries, 1 keys): without gain_per_head
    const int nh = min(H, kGroups), tpar = kGroups / nh;
    for (int h0 = 0; h0 < H; h0 += nh) {
        const int h = h0 + group % nh, slot = group / nh;
        const bool on = slot < tpar && h < H;
        const int hc = min(h, H - 1);
        const bool key = hc >= a.Hq;
        const int hh = key ? hc - a.Hq : hc, Hx = key ? a.Hk : a.Hq;
        const float* const dy = key ? dk : dq;
        float g[8], dg[8];
        load8<true>(key ? gk : gq, (PER_HEAD ? hh * kHeadDim : 0) + 8 * l, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) dg[e] = 0.f;
        auto batch = [&](int64_t t0) { return (int)min((int64_t)kMaxTokens, tb - t0); };
        form_angles(both[0], ta, batch(ta), a.rot >> 1, a, freq, pos);
        __syncthreads();
        for (int64_t t0 = ta, i0 = 0; t0 < tb; t0 += kMaxTokens, ++i0) {
            const Angles& A = both[i0 & 1];
            const int tokens = batch(t0);
            for (int s0 = 0; s0 < tokens; s0 += tpar * kAtOnce) {
                float v[kAtOnce][8], u[kAtOnce][8];
#pragma unroll
                for (int i = 0; i < kAtOnce; ++i) {
                    const int t = min(s0 + tpar * i + slot, tokens - 1);
                    load8<F32>(x, (t0 + t) * a.x_stride + hc * kHeadDim + 8 * l, v[i]);
                    load8<true>(dy, out_row(a, A, t0, t, hh, Hx) + 8 * l, u[i]);
                }
                // the next batch's angles, while this one's rows are on their way
                if (s0 == 0 && t0 + kMaxTokens < tb)
                    form_angles(both[(i0 + 1) & 1], t0 + kMaxTokens, batch(t0 + kMaxTokens), a.rot >> 1, a, freq, pos);
#pragma unroll
                for (int i = 0; i < kAtOnce; ++i) {
                    const int t = min(s0 + tpar * i + slot, tokens - 1);
                    const bool take = on && s0 + tpar * i + slot < tokens;
                    turn<INTER>(u[i], A, t, l, a.rot, -1.f);
                    const float inv = inv_rms(v[i], a.eps);
                    float dot = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        v[i][e] *= inv;  // x r
                        if (take) dg[e] = fmaf(u[i][e], v[i][e], dg[e]);
                        u[i][e] *= g[e];
                        dot = fmaf(u[i][e], v[i][e], dot);
                    }
                    dot = group8_sum(dot) * (1.f / kHeadDim);
#pragma unroll
                    for (int e = 0; e < 8; ++e) u[i][e] = inv * (u[i][e] - v[i][e] * dot);
                    if (take) store8<true>(dx, (t0 + t) * a.dx_stride + hc * kHeadDim + 8 * l, u[i]);
                }
            }
            __syncthreads();  // the next batch's angles are there, this one's read (and the sums of the last heads)
        }
        store8<true>(&sums[group][0], 8 * l, dg);  // zeros where !on
        __syncthreads();
        if constexpr (PER_HEAD) {
            for (int i = threadIdx.x; i < nh * kHeadDim; i += blockDim.x) {
                const int hn = i >> 6, d = i & 63;
                if (h0 + hn >= H) continue;
                float z = 0.f;
                for (int s = 0; s < tpar; ++s) z += sums[s * nh + hn][d];
                mine[(h0 + hn) * kHeadDim + d] = z;
            }
        } else if (threadIdx.x < 2 * kHeadDim) {
            const int d = threadIdx.x & 63;
            for (int s = 0; s < tpar * nh; ++s)
                if ((h0 + s % nh >= a.Hq) == (threadIdx.x >= kHeadDim)) shared_sum += sums[s][d];
        }
    }
    if (!PER_HEAD && threadIdx.x < gain_rows * kHeadDim) mine[threadIdx.x] = shared_sum;
}

// One gain row a workgroup: its workgroups' partial sums added in fp64, in
// sixteen interleaved runs and then those in order.
__global__ __launch_bounds__(1024) void qk_gain_kernel(const float* __restrict__ partial, int parts, int gain_rows,
                                                       int q_rows, float* __restrict__ dgq,
                                                       float* __restrict__ dgk) {
    __shared__ double run[16][kHeadDim];
    const int d = threadIdx.x & 63, s = threadIdx.x >> 6, row = blockIdx.x;
    double z = 0;
#pragma unroll 8
    for (int p = s; p < parts; p += 16) z += partial[((int64_t)p * gain_rows + row) * kHeadDim + d];
    run[s][d] = z;
    __syncthreads();
    if (s == 0) {
        for (int i = 1; i < 16; ++i) z += run[i][d];
        (row < q_rows ? dgq + row * kHeadDim : dgk + (row - q_rows) * kHeadDim)[d] = (float)z;
    }
}

// Workgroups of the backward: four a CU, of four tokens at least.
int64_t bwd_parts(int64_t T) { return std::min<int64_t>((T + 3) / 4, 1024); }
int gain_rows(const QkShape& s) { return s.per_head ? s.Hq + s.Hk : (s.Hk ? 2 : 1); }

QkArgs args_of(const QkShape& s) {
    // row * ceil(2^32 / H) >> 32 is row / H for rows below 2^22 and H up to 1024
    const uint64_t H = (uint64_t)s.Hq + s.Hk;
    const uint32_t magic = H > 1 ? (uint32_t)((((uint64_t)1 << 32) + H - 1) / H) : 0;
    return {s.T, s.L, s.x_stride, s.dx_stride, s.Hq, s.Hk, s.rot, magic, s.eps};
}

}  // namespace

bool qk_fits(const QkShape& s) { return (s.T + kMaxTokens - 1) / kMaxTokens <= kMaxWorkgroups; }

size_t qk_workspace_bytes(const QkShape& s) {
    return align256((size_t)bwd_parts(s.T) * gain_rows(s) * kHeadDim * sizeof(float));
}

hipError_t launch_qk_fwd(const QkShape& s, bool f32, const void* x, const float* gq, const float* gk,
                         const float* freq, const int32_t* pos, void* q, void* k, hipStream_t stream) {
    // As many tokens a workgroup (sharing its angles) as leave four workgroups a CU.
    int tokens = kMaxTokens;
    while (tokens > 1 && (s.T + tokens - 1) / tokens < 1024) tokens /= 2;
    auto go = [&](auto kernel) {
        kernel<<<(unsigned)((s.T + tokens - 1) / tokens), 256, 0, stream>>>(args_of(s), tokens, x, gq, gk, freq, pos, q,
                                                                           k);
    };
    if (s.per_head) {
        if (f32)
            s.interleaved ? go(qk_fwd_kernel<true, true, true>) : go(qk_fwd_kernel<true, false, true>);
        else
            s.interleaved ? go(qk_fwd_kernel<false, true, true>) : go(qk_fwd_kernel<false, false, true>);
    } else {
        if (f32)
            s.interleaved ? go(qk_fwd_kernel<true, true, false>) : go(qk_fwd_kernel<true, false, false>);
        else
            s.interleaved ? go(qk_fwd_kernel<false, true, false>) : go(qk_fwd_kernel<false, false, false>);
    }
    return hipGetLastError();
}

hipError_t launch_qk_bwd(const QkShape& s, bool f32, const void* x, const float* gq, const float* gk,
                         const float* freq, const int32_t* pos, const float* dq, const float* dk, float* dx,
                         float* dgq, float* dgk, void* workspace, hipStream_t stream) {
    const int64_t parts = bwd_parts(s.T);
    const int rows = gain_rows(s);
    float* partial = static_cast<float*>(workspace);
    auto go = [&](auto kernel) {
        kernel<<<(unsigned)parts, 256, 0, stream>>>(args_of(s), x, gq, gk, freq, pos, dq, dk, dx, partial, rows);
    };
    if (s.per_head) {
        if (f32)
            s.interleaved ? go(qk_bwd_kernel<true, true, true>) : go(qk_bwd_kernel<true, false, true>);
        else
            s.interleaved ? go(qk_bwd_kernel<false, true, true>) : go(qk_bwd_kernel<false, false, true>);
    } else {
        if (f32)
            s.interleaved ? go(qk_bwd_kernel<true, true, false>) : go(qk_bwd_kernel<true, false, false>);
        else
            s.interleaved ? go(qk_bwd_kernel<false, true, false>) : go(qk_bwd_kernel<false, false, false>);
    }
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    qk_gain_kernel<<<(unsigned)rows, 1024, 0, stream>>>(partial, (int)parts, rows, s.per_head ? s.Hq : 1, dgq, dgk);
    return hipGetLastError();
}

}  // namespace lsh
