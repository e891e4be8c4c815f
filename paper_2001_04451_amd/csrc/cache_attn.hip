// Attention of new tokens over their sequences' cached rows (lsh_cache.h):
//   o_i = sum_j w_ij v_j / sum_j w_ij,  w_ij = exp2(z_ij - m_i),  z_ij = scale log2(e) q_i.k_j,
// with the offset m_i (near the running maximum), the sum and the output kept in fp32 over one pass.
//
// gfx950 design.  The rows of a sequence and key head are its new tokens times
// the H / Hkv query heads that share the key head.  A work item is a tile of
// these rows and a run of keys; runs are split so that items are alike in
// length however ragged the batch is, and a second kernel joins the parts of
// rows that were split.  The split is made by every workgroup for itself from
// `first` and `length` (find_item), or for many sequences by a kernel before
// (cache_plan_kernel), so that nothing is planned on the host and a captured
// call serves any lengths.
// Both kinds of tile form S^T = K Q^T and O^T = V^T P^T on the matrix cores
// with 16 rows of queries as the columns (mfma_f32_16x16x32_bf16), so a lane's
// scores of four keys of two 16-key tiles are, packed to bf16, its operand of
// the second product, and V^T comes from LDS rows by the transposing read.
// Codes are turned to bf16 with their block's scale on the way (exact).  The
// weights are rounded to bf16, as the matrix cores take them; the output is
// divided by the sum of the rounded ones (one more product, with ones), so
// they sum to one, and the log-partition takes the fp32 sum.  Tiles of 16 and
// 64 rows, but for large prompts (Plan::two), add the product with what the
// rounding left (a second bf16 number a weight), so that the output has little
// more than the rounding of its own: of 16 heads over 1K keys 0.0017 of its
// norm off, where the rounded weights alone leave 0.0024.  In tiles of 128 rows
// that would cost 2-12% (512 tokens over 4K, 16 heads 30.5 / 34 us), in those
// of 256 the registers that the accumulators of a second product need.
//   narrow  16 rows (decoding, a few tokens): each of four waves walks its own
//           keys, K rows straight from memory into operand registers, V rows
//           through an LDS area of its own; the waves are joined at the end.
//           Bound by HBM: 64 sequences of up to 16K, 16 heads, e4m3, 127 us
//           (5.1 TB/s); one of 64K in bf16 45 us (6.0 TB/s), 52 with its join.
//           Grouped 4-bit caches are bound by the conversions and exp instead
//           (32 of 32K, 8 query heads a key head: 46 us with the join; with one
//           number a weight 40).
//   wide    64 QT rows (chunks): the four waves share blocks of 64 keys staged
//           in LDS, double-buffered.  Bound by exp and the other vector
//           instructions, which fill 59% of a SIMD's time, and by how far two
//           waves overlap them with the matrix cores (37%): 2K tokens over
//           32K, 16 heads, e4m3, 329 us with its join (0.81 PFLOP/s; a library
//           matrix product of 8192^3 reaches 1.12 on this card).
#include "attn_common.h"
#include "cache_common.h"

namespace lsh {
namespace {

constexpr int kSwz = 1;  // LDS row layout (attn_common.h): 16-row operand reads
constexpr int kNarrowRows = 16;
constexpr bf16x8 kOnes8 = {(__bf16)1.0f, (__bf16)1.0f, (__bf16)1.0f, (__bf16)1.0f,
                           (__bf16)1.0f, (__bf16)1.0f, (__bf16)1.0f, (__bf16)1.0f};
constexpr float kNegInf = -__builtin_inff();
// The offset that weights are taken against follows the running maximum only
// when that has risen by more than this (in log2): weights stay below 2^16,
// sums far within fp32, and neither the four lanes of a query nor the sums so
// far need to be brought into line at every step.  Each row's offset moves by
// that row's maximum alone, so that keys hidden from it do not touch even its
// rounding.
constexpr float kSlack = 16.f;
// No running maximum is taken where normalised keys keep every logit (log2)
// within this: weights are within 2^-30 and 2^30 then, and fp32 holds the sums
// of 2^30 of them times values of up to 2^60.
constexpr float kFree = 30.f;

// How the keys are split: rows in (lo, hi] belong to this kernel, in tiles of
// `rows`; parts are multiples of `step` keys.  Up to `target` items a head,
// but parts of fewer than `longer` keys only to have `few` items a head, and
// none of fewer than `shorter`: each part costs a workgroup's start and its
// results' way through memory.
struct Split {
    int rows, lo, hi, step, shorter, longer, few, target;
};

struct Item {
    int seq, tile, part, parts, keys;  // keys a part
    int n_rows;                        // of the sequence and head
    int64_t first, pos0;               // row of its first new token, and that token's position
    int slot;                          // of the partial results, where parts > 1
};

__device__ __forceinline__ int cache_cap(const CacheArgs& a) { return a.max_pages << a.page_log2; }

// What a sequence brings: its rows of this kernel's kind and its cached keys.
__device__ __forceinline__ void seq_work(const CacheArgs& a, const Split& sp, int s, int& tiles, int& keys, int& rows) {
    tiles = keys = rows = 0;
    if (s >= a.n_seq) return;
    const int64_t f0 = min(max((int64_t)a.first[s], (int64_t)0), a.T);
    const int64_t f1 = min(max((int64_t)a.first[s + 1], f0), a.T);
    rows = (int)(f1 - f0) * (a.H / a.Hkv);
    if (rows <= sp.lo || rows > sp.hi) return;
    tiles = (rows + sp.rows - 1) / sp.rows;
    keys = min(max(a.length[s], 0), cache_cap(a));
}

// Sums over lanes 0 .. own, by moves within rows of sixteen and then from row
// to row (no LDS round trips).
__device__ __forceinline__ int wave_scan(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false);  // from 1, 2, 4, 8 lanes below in the row
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);  // last lane of row 0 into row 1, 2 into 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);  // lane 31 into rows 2 and 3
    return x;
}
__device__ __forceinline__ float wave_sum(float x) {  // the same in every lane
    x = group8_sum(x);
    return sum_xor32(sum_xor16(x + dpp_f32<kDppMirror>(x)));
}

// Keys of a part, at most: C >= keys of all tiles / target, so that there are
// at most target + tiles items, and at most 2 target of them in sequences that
// are split (a tile of keys > C makes at most 2 keys / C parts).
__device__ __forceinline__ int part_keys(const Split& sp, float work) {
    const float few = fminf(fmaxf(work / (float)sp.few, (float)sp.shorter), (float)sp.longer);
    return (int)fminf(fmaxf(work * 1.0001f / (float)sp.target, few), 1073741824.f) + 1;
}
__device__ __forceinline__ int parts_of(int tiles, int keys, int C) {
    return tiles ? max(1, (int)(((uint32_t)keys + (uint32_t)C - 1u) / (uint32_t)C)) : 0;
}

// The split of many sequences, made once a call: of each sequence the number of
// items up to its last, its first slot and its parts a tile.  One workgroup a
// kind of tile.
__global__ __launch_bounds__(1024) void cache_plan_kernel(CacheArgs a, Split narrow, Split wide, int4* narrow_plan,
                                                          int4* wide_plan) {
    __shared__ float works[16];
    __shared__ int2 sums[16];
    const Split sp = blockIdx.x ? wide : narrow;
    int4* const plan = blockIdx.x ? wide_plan : narrow_plan;
    if (!plan) return;
    const int lane = lane_id(), wave = threadIdx.x >> 6;
    int tiles, keys, rows;
    float work = 0.f;
    for (int s = threadIdx.x; s < a.n_seq; s += 1024) {
        seq_work(a, sp, s, tiles, keys, rows);
        work += (float)tiles * (float)keys;
    }
    work = wave_sum(work);
    if (lane == 0) works[wave] = work;
    __syncthreads();
    work = 0.f;
    for (int w = 0; w < 16; ++w) work += works[w];
    const int C = part_keys(sp, work);
    int2 base = make_int2(0, 0);
    for (int s0 = 0; s0 < a.n_seq; s0 += 1024) {
        const int s = s0 + (int)threadIdx.x;
        seq_work(a, sp, s, tiles, keys, rows);
        const int parts = parts_of(tiles, keys, C), items = tiles * parts, split = parts > 1 ? items : 0;
        int2 sum = make_int2(wave_scan(items), wave_scan(split));
        __syncthreads();  // the last round's sums are read
        if (lane == 63) sums[wave] = sum;
        __syncthreads();
        int2 all = make_int2(0, 0);
        for (int w = 0; w < 16; ++w) {
            if (w < wave) sum.x += sums[w].x, sum.y += sums[w].y;
            all.x += sums[w].x, all.y += sums[w].y;
        }
        if (s < a.n_seq) plan[s] = make_int4(base.x + sum.x, base.y + sum.y - split, parts, 0);
        base.x += all.x, base.y += all.y;
    }
}

// Item number `item` of the split, the same for all lanes; false past the
// last.  Without a plan every workgroup adds the sequences up for itself.
__device__ bool find_item(const CacheArgs& a, const Split& sp, const int4* __restrict__ plan, int item, Item& it) {
    const int lane = lane_id();
    int tiles, keys, rows, at, slot;
    if (plan) {
        int base = 0, count = a.n_seq;  // the first sequence whose items end behind `item`: 64 at a time
        for (;;) {
            const int step = (count + 63) >> 6, end = min((lane + 1) * step, count);
            const int n = __popcll(__ballot(lane * step < count && plan[base + end - 1].x <= item));
            if (n * step >= count) return false;
            base += n * step;
            count = min(step, count - n * step);
            if (count == 1) break;
        }
        const int4 p = plan[base];
        seq_work(a, sp, base, tiles, keys, rows);
        it.seq = base;
        it.parts = __builtin_amdgcn_readfirstlane(p.z);
        at = item - __builtin_amdgcn_readfirstlane(p.x - tiles * p.z);
        slot = __builtin_amdgcn_readfirstlane(p.y);
        tiles = __builtin_amdgcn_readfirstlane(tiles);
        keys = __builtin_amdgcn_readfirstlane(keys);
        rows = __builtin_amdgcn_readfirstlane(rows);
    } else {
        float work = 0.f;  // the same in every workgroup: the same sums in the same order
        for (int s0 = 0; s0 < a.n_seq; s0 += 64) {
            seq_work(a, sp, s0 + lane, tiles, keys, rows);
            work += (float)tiles * (float)keys;
        }
        const int C = part_keys(sp, wave_sum(work));
        int base = 0, slots = 0, s0 = 0;
        for (;; s0 += 64) {
            if (s0 >= a.n_seq) return false;
            if (a.n_seq > 64) seq_work(a, sp, s0 + lane, tiles, keys, rows);
            const int parts = parts_of(tiles, keys, C), items = tiles * parts, split = parts > 1 ? items : 0;
            const int sum = wave_scan(items), sum2 = wave_scan(split);
            const uint64_t mine = __ballot(item - base < sum);
            if (mine) {
                const int l = __builtin_ctzll(mine);
                it.seq = s0 + l;
                it.parts = __builtin_amdgcn_readlane(parts, l);
                at = item - base - __builtin_amdgcn_readlane(sum - items, l);
                slot = slots + __builtin_amdgcn_readlane(sum2 - split, l);
                tiles = __builtin_amdgcn_readlane(tiles, l);
                keys = __builtin_amdgcn_readlane(keys, l);
                rows = __builtin_amdgcn_readlane(rows, l);
                break;
            }
            base += __builtin_amdgcn_readlane(sum, 63);
            slots += __builtin_amdgcn_readlane(sum2, 63);
        }
    }
    // the same in all lanes: into scalar registers
    auto scalar = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
    it.seq = scalar(it.seq);
    it.parts = scalar(it.parts);
    at = scalar(at);
    const int back = scalar(at / it.parts);  // the last tile, whose rows see the most, first
    it.part = at - back * it.parts;
    it.tile = scalar(tiles) - 1 - back;
    const int keys_part = scalar((keys + it.parts - 1) / it.parts);  // alike parts, in whole steps
    it.keys = scalar((keys_part + sp.step - 1) / sp.step * sp.step);
    it.n_rows = scalar(rows);
    it.slot = scalar(slot) + it.tile * it.parts + it.part;
    it.first = min(max((int64_t)scalar(a.first[it.seq]), (int64_t)0), a.T);
    it.pos0 = (int64_t)scalar(a.length[it.seq]) - scalar(a.first[it.seq + 1]) + it.first;
    return true;
}

// Row r of the item's sequence and head: query head within the group, token,
// and the number of cached positions from 0 on that it may see (with shared
// QK without its own, which counts only where there is no other).
struct QueryRow {
    int token, group, limit;
};
__device__ __forceinline__ QueryRow query_row(const CacheArgs& a, const Item& it, int r, int G, int shared) {
    QueryRow q;
    q.token = r / G;
    q.group = r - q.token * G;
    const int64_t n = it.pos0 + q.token + (shared ? 0 : 1);
    q.limit = r < it.n_rows ? (int)min(max(n, (int64_t)0), (int64_t)cache_cap(a)) : 0;
    return q;
}

// The limit of a row that is the same for all lanes, in a scalar register.
__device__ __forceinline__ int row_limit(const CacheArgs& a, const Item& it, int r, int G, int shared) {
    return __builtin_amdgcn_readfirstlane(query_row(a, it, r, G, shared).limit);
}

// The query of row r (of the last row, past it).
__device__ __forceinline__ const uint16_t* query_at(const CacheArgs& a, const Item& it, const uint16_t* __restrict__ q,
                                                    int head, int G, int r) {
    const int rc = min(r, it.n_rows - 1), token = rc / G;
    return q + (it.first + token) * a.q_stride + (head * G + rc - token * G) * kHeadDim;
}

// Tiles of 16 positions, tile0 .. tile0 + 63 of a sequence and head, one a
// lane: the number of the 16-slot run that holds it, or -1 for none (no slot,
// or not before position `end`).
__device__ __forceinline__ int tile_runs(const CacheArgs& a, int seq, int head, int tile, int end) {
    if (tile * 16 >= end) return -1;  // end <= cache_cap: the table has an entry
    const int shift = a.page_log2 - 4;
    const int32_t page = a.table[(int64_t)seq * a.max_pages + (tile >> shift)];
    if (page < 0 || page >= a.n_pages) return -1;
    return (int)((((int64_t)page * a.Hkv + head) << shift) + (tile & ((1 << shift) - 1)));
}

// Partial results of split rows, in the workspace.
struct Parts {
    float* o;       // [slot][Hkv][tile rows][64]: sum of weights times values
    f32x4* stat;    // [slot][Hkv][tile rows]: offset (log2), sum of weights, sum of the weights as rounded
    int2* of_seq;   // [n_seq]: parts a tile, first slot
    int slots;      // enough for any `first` that does not decrease; the rest of others is left out
    const int4* plan;  // of cache_plan_kernel, or null
};

// Value d of a cached row.
template <CacheType TYPE>
__device__ __forceinline__ float cached(const char* base, const uint8_t* scale, int64_t slot, int d) {
    if constexpr (TYPE == kCacheBf16) {
        return bf16_bits_to_f32(reinterpret_cast<const uint16_t*>(base)[slot * 64 + d]);
    } else {
        const int byte = scale[2 * slot + (d >> 5)];
        float x;
        if constexpr (TYPE == kCacheE4m3)
            x = __builtin_amdgcn_cvt_f32_fp8((uint32_t) reinterpret_cast<const uint8_t*>(base)[slot * 64 + d], 0);
        else
            x = pair_to_f32<TYPE, 0>((uint32_t) reinterpret_cast<const uint8_t*>(base)[slot * 32 + (d >> 1)])[d & 1];
        return byte == 255 ? __builtin_nanf("") : ldexpf(x, byte - 127);
    }
}

// Four dimensions of a finished row (d0 .. d0+3): out and, by the caller that
// has d0 = 0, lse.  A row without keys has its own key left (shared QK), or
// nothing.
template <CacheType TYPE>
__device__ void finish_row(const CacheArgs& a, const uint16_t* __restrict__ q, uint16_t* __restrict__ out,
                           float* __restrict__ lse, int64_t t, int h, int seq, int64_t pos, int d0, f32x4 o, float m,
                           float l, float rounded) {
    float z = (m + __log2f(l)) * kLn2;
    if (l == 0.f) {
        o = f32x4{};
        z = kNegInf;
        const int64_t self = a.shared ? slot_of(a, seq, pos, h) : -1;
        if (self >= 0) {
            float dot = 0.f;
            for (int d = 0; d < kHeadDim; ++d)
                dot = fmaf(bf16_bits_to_f32(q[t * a.q_stride + h * kHeadDim + d]),
                           cached<TYPE>(a.k, a.k_scale, self, d), dot);
            z = dot * a.scale * a.k_inv[self] - a.self_mask;
            for (int e = 0; e < 4; ++e) o[e] = cached<TYPE>(a.v, a.v_scale, self, d0 + e);
        }
    } else {
        o *= 1.f / rounded;
    }
    const int64_t row = t * a.H + h;
    *reinterpret_cast<uint2*>(out + row * kHeadDim + d0) = make_uint2(pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3]));
    if (lse && d0 == 0) lse[row] = z;
}

// ---- values that are not finite ----
// 0 times infinity is NaN, so such a value must not enter the products of a
// tile in which some rows do not see its key.  There it is blanked in the
// operand, and after the walk added to the rows that do see it: a positive
// weight times such a value is the value, and a logit of -inf makes it NaN.

// The operand without its non-finite values; found is set where it had one.
__device__ __forceinline__ bf16x8 blank(bf16x8 vt, uint32_t& found) {
    u32x4 w = __builtin_bit_cast(u32x4, vt);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        // a half's exponent is all ones: adding one to it carries into the half's top bit
        const uint32_t odd = (((w[i] & 0x7F807F80u) + 0x00800080u) & 0x80008000u) >> 15;
        found |= odd;
        w[i] &= ~(odd * 0xFFFFu);
    }
    return as_bf16x8(w);
}
// o (dimensions 16 dt + 4 g + e of a row whose query is at q) with the
// non-finite values of the positions from .. to - 1 that it sees (rare, and slow).
template <CacheType TYPE>
__device__ __forceinline__ void add_odd(const CacheArgs& a, int seq, int head, int from, int to, int limit, int g,
                                        const uint16_t* __restrict__ q, f32x4 (&o)[4]) {
#pragma unroll 1
    for (int key = from; key < min(to, limit); ++key) {
        const int64_t slot = slot_of(a, seq, key, head);
        if (slot < 0) continue;
        f32x4 x[4];
        bool odd = false;
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float v = cached<TYPE>(a.v, a.v_scale, slot, 16 * dt + 4 * g + e);
                const bool finite = fabsf(v) < __builtin_inff();
                x[dt][e] = finite ? 0.f : v;
                odd |= !finite;
            }
        if (!odd) continue;
        float z = 0.f;
#pragma unroll 1
        for (int d = 0; d < kHeadDim; ++d) z = fmaf(bf16_bits_to_f32(q[d]), cached<TYPE>(a.k, a.k_scale, slot, d), z);
        const bool none = z * a.scale == kNegInf;
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[dt][e] += none && x[dt][e] != 0.f ? __builtin_nanf("") : x[dt][e];
    }
}

// The compiler must not move a lane's LDS reads across other lanes' writes of the same wave.
__device__ __forceinline__ void wave_lds_order() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

template <bool B>
struct Tag {
    static constexpr bool value = B;
};

// ---- narrow ----

// 16-key tiles that a wave takes a step (its loads under way), and workgroups
// a CU.  Two tiles and three workgroups keep the walk out of scratch: 64
// sequences of e4m3 / one of 64K in bf16 132 / 52 us, with four workgroups 159
// / 102, with four tiles 157 / 81.
constexpr int kTiles = 2;
constexpr int kNarrowOcc = 3;
constexpr int kNarrowStep = 4 * 16 * kTiles;  // of the four waves

// One 16-key tile as loaded: K rows in operand order (lane: row lane % 16,
// group g = lane / 16), V rows in memory order.
template <CacheType TYPE>
struct RawTile {
    static constexpr int kPieces = TYPE == kCacheBf16 ? 2 : 1;
    u32x4 k[kPieces], v[kPieces];
    uint32_t ks, vs;
};

template <CacheType TYPE>
__device__ __forceinline__ void load_tile(const CacheArgs& a, int run, RawTile<TYPE>& r) {
    const int lane = lane_id(), n = lane & 15, g = lane >> 4;
    const int64_t row0 = (int64_t)run * 16;
    const char* k = a.k + row0 * kRowBytes<TYPE>;
    const char* v = a.v + row0 * kRowBytes<TYPE>;
    if constexpr (TYPE == kCacheBf16) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            r.k[i] = *reinterpret_cast<const u32x4*>(k + n * 128 + 64 * i + 16 * g);
            r.v[i] = *reinterpret_cast<const u32x4*>(v + 1024 * i + 16 * lane);
        }
    } else {
        if constexpr (TYPE == kCacheE4m3) {
            r.k[0] = *reinterpret_cast<const u32x4*>(k + n * 64 + 16 * g);
            r.v[0] = *reinterpret_cast<const u32x4*>(v + 16 * lane);
        } else {
            const uint2 x = *reinterpret_cast<const uint2*>(k + n * 32 + 8 * g);
            const uint2 y = *reinterpret_cast<const uint2*>(v + 8 * lane);
            r.k[0] = u32x4{x.x, x.y, 0u, 0u};
            r.v[0] = u32x4{y.x, y.y, 0u, 0u};
        }
        r.ks = a.k_scale[2 * (row0 + n) + (g >> 1)];
        r.vs = a.v_scale[2 * (row0 + (lane >> 2)) + ((lane >> 1) & 1)];
    }
}

// Sixteen codes (a lane's quarter of a row) as two operands of eight bf16.
template <CacheType TYPE>
__device__ __forceinline__ void widen16(u32x4 c, uint32_t byte, bf16x8* x) {
    const float s = scale_of(byte);
    if constexpr (TYPE == kCacheE4m3) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
            x[h] = as_bf16x8(u32x4{pair_to_bf16<TYPE, 0>(c[2 * h], s), pair_to_bf16<TYPE, 1>(c[2 * h], s),
                                   pair_to_bf16<TYPE, 0>(c[2 * h + 1], s), pair_to_bf16<TYPE, 1>(c[2 * h + 1], s)});
    } else {
#pragma unroll
        for (int h = 0; h < 2; ++h)
            x[h] = as_bf16x8(u32x4{pair_to_bf16<TYPE, 0>(c[h], s), pair_to_bf16<TYPE, 1>(c[h], s),
                                   pair_to_bf16<TYPE, 2>(c[h], s), pair_to_bf16<TYPE, 3>(c[h], s)});
    }
}

struct NarrowShared {
    char Vs[4][16 * kTiles * 128];
    float invs[4][16 * kTiles];  // k_inv of the step's keys
    f32x4 stats[4][kNarrowRows];
};

// What rounding to bf16 leaves of two weights, as bf16 (16 bits of a weight in all).
struct Minus {
    uint32_t lo = 0x0000BF80u, hi = 0xBF800000u;  // (-1, 0) and (0, -1)
    // In registers: as operands of their own, the first was taken for a -1 of 32 bits.
    __device__ __forceinline__ Minus() { asm("" : "+s"(lo), "+s"(hi)); }
    __device__ __forceinline__ uint32_t rest(float p0, float p1, uint32_t w) const {  // w: p0 and p1 rounded
        const bf16x2 w2 = __builtin_bit_cast(bf16x2, w);  // the differences are exact
        return pack_bf16x2(__builtin_amdgcn_fdot2_f32_bf16(w2, __builtin_bit_cast(bf16x2, lo), p0, false),
                           __builtin_amdgcn_fdot2_f32_bf16(w2, __builtin_bit_cast(bf16x2, hi), p1, false));
    }
};
// The products with the weights as rounded and with their rests together.  An
// infinite value times a rest may be NaN or of the other sign; times the
// weight as rounded it is what counts.
__device__ __forceinline__ f32x4 with_rest(f32x4 o, f32x4 rest) {
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += fabsf(rest[e]) < __builtin_inff() ? rest[e] : 0.f;
    return o;
}

template <CacheType TYPE, bool SHARED>
__device__ __forceinline__ void narrow_tile(const CacheArgs& a, const Split& sp, const Parts& parts,
                                            const uint16_t* __restrict__ q, uint16_t* __restrict__ out,
                                            float* __restrict__ lse, uint32_t block, NarrowShared& S) {
    constexpr int NT = kTiles, kStep = 16 * NT;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = lane & 15, g = lane >> 4;
    const int G = a.H / a.Hkv, head = block % (unsigned)a.Hkv;
    Item it;
    if (!find_item(a, sp, parts.plan, (int)(block / (unsigned)a.Hkv), it)) return;
    if (it.tile == 0 && it.part == 0 && head == 0 && tid == 0)
        parts.of_seq[it.seq] = make_int2(it.parts, it.slot);  // slot of tile 0, part 0
    if (it.parts > 1 && it.slot >= parts.slots) return;
    const int r0 = it.tile * kNarrowRows;
    const QueryRow row = query_row(a, it, r0 + n, G, SHARED);
    const int last = min(r0 + kNarrowRows, it.n_rows) - 1;
    const int most = row_limit(a, it, last, G, SHARED);  // of any row of the tile
    const int least = row_limit(a, it, r0, G, SHARED);
    const int k0 = it.part * it.keys, k1 = min(k0 + it.keys, most);

    // The queries' operand: the dimensions of K's in the same order.
    // A negative scale turns the queries round, which is exact, so that the
    // largest logit is the largest product.
    bf16x8 qop[2];
    const uint16_t* const qrow = query_at(a, it, q, head, G, r0 + n);
    float qq = 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        u32x4 x = *reinterpret_cast<const u32x4*>(qrow + (TYPE == kCacheBf16 ? 32 * i + 8 * g : 16 * g + 8 * i));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (a.scale < 0.f) x[e] ^= 0x80008000u;
            const float lo = __uint_as_float(x[e] << 16), hi = __uint_as_float(x[e] & 0xFFFF0000u);
            qq = fmaf(lo, lo, fmaf(hi, hi, qq));
        }
        qop[i] = as_bf16x8(x);
    }
    const float scale_log2e = fabsf(a.scale) * kLog2e;
    const bool fast = SHARED && __all(scale_log2e * sqrtf(sum_xor32(sum_xor16(qq))) <= kFree);

    float m = fast ? 0.f : kNegInf, l = 0.f;  // l: this lane's keys
    f32x4 o[4] = {}, rest[4] = {};
    const Minus minus;
    uint32_t odd = 0;            // a non-finite value was blanked,
    int edge0 = 0x7FFFFFFF;      // at this position or later
    const int per = ((k1 - k0 + 4 * kStep - 1) / (4 * kStep)) * kStep;  // keys a wave
    const int w0 = k0 + wave * per, w1 = min(w0 + per, k1);
    const int steps = w0 < w1 ? (w1 - w0 + kStep - 1) / kStep : 0;
    char* const V = S.Vs[wave];

    constexpr int kRun = 64 / NT;  // steps that the runs of a wave's lanes last
    int runs = steps ? tile_runs(a, it.seq, head, w0 / 16 + lane, w1) : -1, runs_next = -1;
    RawTile<TYPE> raw[NT];
    float inv = 0.f;    // k_inv of key `lane` of the step
    uint32_t gone = 0;  // bit t: tile t of the step has no slots
    auto fetch = [&](int st) {
        if (st % kRun == 0) {
            if (st) runs = runs_next;
            if (st + kRun < steps) runs_next = tile_runs(a, it.seq, head, w0 / 16 + NT * (st + kRun) + lane, w1);
        }
        gone = 0;
        int mine = 0;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int run = __builtin_amdgcn_readlane(runs, (NT * st + t) & 63);
            gone |= run < 0 ? 1u << t : 0u;
            load_tile<TYPE>(a, max(run, 0), raw[t]);
            if (t == 0 || lane >= 16 * t) mine = max(run, 0);
        }
        if constexpr (SHARED) inv = a.k_inv[(int64_t)mine * 16 + n];
    };
    int st = 0;
    // EDGE: keys of the step may be hidden from some or all rows.
    auto step = [&](auto fast_tag, auto edge_tag) {
        constexpr bool FAST = decltype(fast_tag)::value, EDGE = decltype(edge_tag)::value;
        const int key0 = w0 + st * kStep;
        const bool differ = EDGE && least != most;
        if (differ) edge0 = min(edge0, key0);
        wave_lds_order();  // the last step's reads of V before this step's writes
        f32x4 z[NT];
        if (SHARED && lane < kStep) S.invs[wave][lane] = scale_log2e * inv;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            bf16x8 kop[2];
            u32x4 vrow[2];
            if constexpr (TYPE == kCacheBf16) {
#pragma unroll
                for (int i = 0; i < 2; ++i) kop[i] = as_bf16x8(raw[t].k[i]), vrow[i] = raw[t].v[i];
            } else {
                bf16x8 x[2];
                widen16<TYPE>(raw[t].k[0], raw[t].ks, kop);
                widen16<TYPE>(raw[t].v[0], raw[t].vs, x);
                vrow[0] = __builtin_bit_cast(u32x4, x[0]), vrow[1] = __builtin_bit_cast(u32x4, x[1]);
            }
            z[t] = mfma16x16x32(kop[0], qop[0], f32x4{});
            z[t] = mfma16x16x32(kop[1], qop[1], z[t]);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = TYPE == kCacheBf16 ? 8 * i + (lane >> 3) : lane >> 2;
                const int piece = TYPE == kCacheBf16 ? lane & 7 : 2 * (lane & 3) + i;
                if (EDGE && ((gone >> t & 1) || key0 + 16 * t + r >= w1)) vrow[i] = u32x4{};
                *reinterpret_cast<u32x4*>(V + row_piece_offset<kSwz>(16 * t + r, piece)) = vrow[i];
            }
        }
        const uint32_t hidden = gone;
        if (st + 1 < steps) fetch(st + 1);  // into the registers just used up
        wave_lds_order();
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            if constexpr (SHARED) z[t] *= *reinterpret_cast<const f32x4*>(&S.invs[wave][16 * t + 4 * g]);
            if constexpr (EDGE)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int key = key0 + 16 * t + 4 * g + j;
                    z[t][j] = !(hidden >> t & 1) && key < min(row.limit, w1) ? z[t][j] : kNegInf;
                }
        }
        const float c = SHARED ? 1.f : scale_log2e;  // what z still lacks
        float off = 0.f;
        if constexpr (!FAST) {
            float mt = kNegInf;
#pragma unroll
            for (int t = 0; t < NT; ++t)
                mt = fmaxf(fmaxf(mt, fmaxf(z[t][0], z[t][1])), fmaxf(z[t][2], z[t][3]));
            if constexpr (!SHARED) mt = mt > kNegInf ? mt * c : mt;
            if (__any(mt > m + kSlack)) {
                mt = max_xor32(max_xor16(mt));
                const float m1 = mt > m + kSlack ? mt : m;  // for each row by itself (kSlack)
                const float corr = m1 > kNegInf ? __builtin_amdgcn_exp2f(m - m1) : 1.f;
                l *= corr;
#pragma unroll
                for (int dt = 0; dt < 4; ++dt) o[dt] *= corr, rest[dt] *= corr;
                m = m1;
            }
            off = m > kNegInf ? m : 0.f;
        }
#pragma unroll
        for (int t = 0; t < NT; t += 2) {
            u32x4 pw, pr;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                f32x4& p = z[t + i];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if constexpr (EDGE && !SHARED)  // the scale of 0 leaves a hidden key hidden
                        p[j] = p[j] == kNegInf ? 0.f : __builtin_amdgcn_exp2f(fmaf(p[j], c, -off));
                    else
                        p[j] = __builtin_amdgcn_exp2f(SHARED ? p[j] - off : fmaf(p[j], c, -off));
                }
                l += (p[0] + p[1]) + (p[2] + p[3]);
#pragma unroll
                for (int j = 0; j < 4; j += 2) {
                    const uint32_t w = pack_bf16x2(p[j], p[j + 1]);
                    pw[2 * i + j / 2] = w;
                    pr[2 * i + j / 2] = minus.rest(p[j], p[j + 1], w);
                }
            }
#pragma unroll
            for (int dt = 0; dt < 4; ++dt) {
                bf16x8 vt = cat4(vt_read(V + vt_offset<kSwz>(16 * t, 16 * dt, lane)),
                                 vt_read(V + vt_offset<kSwz>(16 * t + 16, 16 * dt, lane)));
                if (EDGE && differ) vt = blank(vt, odd);
                o[dt] = mfma16x16x32(vt, as_bf16x8(pw), o[dt]);
                rest[dt] = mfma16x16x32(vt, as_bf16x8(pr), rest[dt]);
            }
        }
        ++st;
    };
    if (steps) fetch(0);
    const int whole = max(min(least, w1) - w0, 0) / kStep;
    auto walk = [&](auto fast_tag) {
        while (st < whole && !gone) step(fast_tag, Tag<false>{});
    };
    if (fast)
        walk(Tag<true>{});
    else
        walk(Tag<false>{});
    while (st < steps) step(Tag<false>{}, Tag<true>{});
    l = sum_xor32(sum_xor16(l));
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) o[dt] = with_rest(o[dt], rest[dt]);
    if (__any(odd)) add_odd<TYPE>(a, it.seq, head, edge0, w1, row.limit, g, qrow, o);

    // Join the four waves: thread takes row tid / 16 and four dimensions.
    __syncthreads();
    float* const O = reinterpret_cast<float*>(S.Vs[wave]);  // [row][64]
#pragma unroll
    for (int dt = 0; dt < 4; ++dt) *reinterpret_cast<f32x4*>(O + n * kHeadDim + 16 * dt + 4 * g) = o[dt];
    if (g == 0) S.stats[wave][n] = f32x4{m, l, l, 0.f};
    __syncthreads();
    const int r = tid >> 4, d0 = 4 * (tid & 15);
    if (r0 + r >= it.n_rows) return;
    f32x4 ws[4];
    float top = kNegInf;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        ws[w] = S.stats[w][r];
        if (ws[w][1] != 0.f) top = fmaxf(top, ws[w][0]);
    }
    f32x4 sum = {}, stat = {top, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if (ws[w][1] == 0.f) continue;  // no keys there
        const float f = __builtin_amdgcn_exp2f(ws[w][0] - top);
        sum += f * *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(S.Vs[w]) + r * kHeadDim + d0);
        stat[1] += f * ws[w][1];
        stat[2] += f * ws[w][2];
    }
    if (it.parts > 1) {
        const int64_t at = ((int64_t)it.slot * a.Hkv + head) * sp.rows + r;
        *reinterpret_cast<f32x4*>(parts.o + at * kHeadDim + d0) = sum;
        if (d0 == 0) parts.stat[at] = stat;
        return;
    }
    const QueryRow mine = query_row(a, it, r0 + r, G, SHARED);
    finish_row<TYPE>(a, q, out, lse, it.first + mine.token, head * G + mine.group, it.seq, it.pos0 + mine.token, d0, sum,
                     stat[0], stat[1], stat[2]);
}

// ---- wide ----

template <CacheType TYPE>
struct WideShared {
    char Ks[2][64 * 128];
    char Vs[2][64 * 128];
    float inv[2][4][64];  // k_inv of a tile's rows in the first 16 of each 64
    int hole[2][4];       // tile without slots
    // a tile's codes and scales as copied: K's and V's
    char raw[4][TYPE == kCacheBf16 ? 16 : 2 * 16 * kRowBytes<TYPE>];
    uint32_t scales[4][TYPE == kCacheBf16 ? 4 : 64];
};

struct Weights {
    bf16x8 rounded, rest;  // (Minus)
};

template <CacheType TYPE, bool SHARED, int QT, bool TWO>
__device__ __forceinline__ void wide_tile(const CacheArgs& a, const Split& sp, const Parts& parts,
                                          const uint16_t* __restrict__ q, uint16_t* __restrict__ out,
                                          float* __restrict__ lse, int items, int sets, uint32_t block,
                                          WideShared<TYPE>& S) {
    constexpr int kRows = 64 * QT;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = lane & 15, g = lane >> 4;
    const int G = a.H / a.Hkv;
    // Each XCD keeps to its own heads (or kXcds / sets XCDs share some), whose rows its L2 then serves.
    const int xcd = (int)(block % kXcds), heads = a.Hkv / sets;
    const int64_t turn = (int64_t)(block / kXcds) * (kXcds / sets) + xcd / sets;
    const int head = (int)(turn % heads) * sets + xcd % sets;
    if (turn / heads >= items) return;
    Item it;
    if (!find_item(a, sp, parts.plan, (int)(turn / heads), it)) return;
    if (it.tile == 0 && it.part == 0 && head == 0 && tid == 0)
        parts.of_seq[it.seq] = make_int2(it.parts, it.slot);  // slot of tile 0, part 0
    if (it.parts > 1 && it.slot >= parts.slots) return;
    const int r0 = it.tile * kRows, rw = r0 + 16 * QT * wave;
    const int most = row_limit(a, it, min(r0 + kRows, it.n_rows) - 1, G, SHARED);
    const int k0 = it.part * it.keys, k1 = min(k0 + it.keys, most);
    const bool active = __builtin_amdgcn_readfirstlane(rw) < it.n_rows;
    // what this wave's rows see: all of them the first `least` keys, none more than `mine`
    const int mine = active ? row_limit(a, it, min(rw + 16 * QT, it.n_rows) - 1, G, SHARED) : 0;
    const int least = active ? row_limit(a, it, rw, G, SHARED) : 0;
    const float scale_log2e = fabsf(a.scale) * kLog2e;  // a negative scale turns the queries round, which is exact

    bf16x8 qop[QT][2];
    uint32_t past = 0;  // byte qt: what row 16 qt + n of the wave sees beyond `least` (at most 63 positions)
    float biggest = 0.f;
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
        past |= (uint32_t)max(query_row(a, it, rw + 16 * qt + n, G, SHARED).limit - least, 0) << (8 * qt);
        const uint16_t* at = query_at(a, it, q, head, G, rw + 16 * qt + n);
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            u32x4 x = *reinterpret_cast<const u32x4*>(at + 32 * i + 8 * g);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (a.scale < 0.f) x[e] ^= 0x80008000u;
                const float lo = __uint_as_float(x[e] << 16), hi = __uint_as_float(x[e] & 0xFFFF0000u);
                ss = fmaf(lo, lo, fmaf(hi, hi, ss));
            }
            qop[qt][i] = as_bf16x8(x);
        }
        ss = sum_xor32(sum_xor16(ss));
        biggest = fmaxf(biggest, ss);
    }

    float m[QT], l[QT];
    static_assert(!TWO || QT == 1);
    const Minus minus;
    f32x4 o[QT][4], rounded[QT], rest[4] = {};
    uint32_t odd = 0;  // a non-finite value was blanked
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
        m[qt] = kNegInf;
        l[qt] = 0.f;
        rounded[qt] = f32x4{};
#pragma unroll
        for (int dt = 0; dt < 4; ++dt) o[qt][dt] = f32x4{};
    }

    // Staging: wave w brings the block's 16-key tile w by copies to LDS, bf16
    // rows to their places, codes to an area of the wave's own, from where they
    // are widened once the block before is done with: nothing of it lives in
    // registers meanwhile.
    const int blocks = k0 < k1 ? (k1 - k0 + 63) / 64 : 0;
    int runs = -1, run = -1;
    auto fetch = [&](int kb, int b) {
        if ((kb & 63) == 0) runs = tile_runs(a, it.seq, head, k0 / 16 + 4 * (kb + lane) + wave, k1);
        run = __builtin_amdgcn_readlane(runs, kb & 63);
        if (run < 0) return;
        const int64_t row0 = (int64_t)run * 16;
        if constexpr (SHARED) copy4_to_lds(a.k_inv + row0 + n, S.inv[b][wave]);
        if constexpr (TYPE == kCacheBf16) {
            // rows at k1 and past it repeat the last one before it
            const int here = k1 - (k0 + kb * 64 + 16 * wave);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = 8 * i + (lane >> 3);
                const int64_t off = (row0 + min(r, here - 1)) * 128 + swz<kSwz>(16 * wave + r, lane & 7) * 16;
                copy16_to_lds(a.k + off, S.Ks[b] + (16 * wave + 8 * i) * 128);
                copy16_to_lds(a.v + off, S.Vs[b] + (16 * wave + 8 * i) * 128);
            }
        } else {
            if constexpr (TYPE == kCacheE4m3) {
                copy16_to_lds(a.k + row0 * 64 + 16 * lane, S.raw[wave]);
                copy16_to_lds(a.v + row0 * 64 + 16 * lane, S.raw[wave] + 1024);
            } else {
                copy16_to_lds((lane < 32 ? a.k : a.v) + row0 * 32 + 16 * (lane & 31), S.raw[wave]);
            }
            copy4_to_lds((lane & 8 ? a.v_scale : a.k_scale) + 2 * row0 + 4 * (lane & 7), S.scales[wave]);
        }
    };
    auto place = [&](int kb, int b) {  // what fetch(kb) brought, into buffer b
        if (lane == 0) S.hole[b][wave] = run < 0;
        if (TYPE != kCacheBf16 && run >= 0) {
            __builtin_amdgcn_s_waitcnt(0);
            const int r = lane >> 2;
            const bool gone = k0 + kb * 64 + 16 * wave + r >= k1;
            const uint8_t* scale = reinterpret_cast<const uint8_t*>(S.scales[wave]) + 2 * r + ((lane >> 1) & 1);
#pragma unroll
            for (int v = 0; v < 2; ++v) {
                u32x4 c{};
                if constexpr (TYPE == kCacheE4m3) {
                    c = *reinterpret_cast<const u32x4*>(S.raw[wave] + 1024 * v + 16 * lane);
                } else {
                    const uint2 x = *reinterpret_cast<const uint2*>(S.raw[wave] + 512 * v + 8 * lane);
                    c[0] = x.x, c[1] = x.y;
                }
                bf16x8 x[2];
                widen16<TYPE == kCacheBf16 ? kCacheE4m3 : TYPE>(c, scale[32 * v], x);
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    *reinterpret_cast<u32x4*>((v ? S.Vs[b] : S.Ks[b]) + row_piece_offset<kSwz>(16 * wave + r, 2 * (lane & 3) + i)) =
                        v && gone ? u32x4{} : __builtin_bit_cast(u32x4, x[i]);
            }
        }
        if (run < 0) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                *reinterpret_cast<u32x4*>(S.Ks[b] + (16 * wave + 8 * i) * 128 + 16 * lane) = u32x4{};
                *reinterpret_cast<u32x4*>(S.Vs[b] + (16 * wave + 8 * i) * 128 + 16 * lane) = u32x4{};
            }
        }
    };

    // The pieces of a block's work for keys 32 kp .. +31 (two 16-key tiles) and
    // the wave's query tile qt.
    auto load_k = [&](int b, int kp, bf16x8 (&kop)[2][2], f32x4 (&cf)[2]) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int r = 32 * kp + 16 * t;
            kop[t][0] = as_bf16x8(lds_piece<kSwz>(S.Ks[b], r + n, g));
            kop[t][1] = as_bf16x8(lds_piece<kSwz>(S.Ks[b], r + n, 4 + g));
            if constexpr (SHARED) cf[t] = scale_log2e * *reinterpret_cast<const f32x4*>(&S.inv[b][2 * kp + t][4 * g]);
        }
    };
    auto load_v = [&](int b, int kp, int dt) {
        return cat4(vt_read(S.Vs[b] + vt_offset<kSwz>(32 * kp, 16 * dt, lane)),
                    vt_read(S.Vs[b] + vt_offset<kSwz>(32 * kp + 16, 16 * dt, lane)));
    };
    auto scores = [&](int qt, const bf16x8 (&kop)[2][2], f32x4 (&z)[2]) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            z[t] = mfma16x16x32(kop[t][0], qop[qt][0], f32x4{});
            z[t] = mfma16x16x32(kop[t][1], qop[qt][1], z[t]);
        }
    };
    // z: products, with shared QK times their keys' factors, -inf where hidden.
    auto weights = [&](int qt, f32x4 (&z)[2], auto fast_tag, auto edge_tag) {
        constexpr bool FAST = decltype(fast_tag)::value, EDGE = decltype(edge_tag)::value;
        float off = 0.f;
        if constexpr (!FAST) {
            float mt = fmaxf(fmaxf(fmaxf(z[0][0], z[0][1]), fmaxf(z[0][2], z[0][3])),
                             fmaxf(fmaxf(z[1][0], z[1][1]), fmaxf(z[1][2], z[1][3])));
            if constexpr (!SHARED) mt = mt > kNegInf ? mt * scale_log2e : mt;
            if (__any(mt > m[qt] + kSlack)) {
                mt = max_xor32(max_xor16(mt));
                const float m1 = mt > m[qt] + kSlack ? mt : m[qt];  // for each row by itself (kSlack)
                const float corr = m1 > kNegInf ? __builtin_amdgcn_exp2f(m[qt] - m1) : 1.f;
                l[qt] *= corr;
                if constexpr (!TWO) rounded[qt] *= corr;
                if constexpr (TWO)
#pragma unroll
                    for (int dt = 0; dt < 4; ++dt) rest[dt] *= corr;
#pragma unroll
                for (int dt = 0; dt < 4; ++dt) o[qt][dt] *= corr;
                m[qt] = m1;
            }
            off = m[qt] > kNegInf ? m[qt] : 0.f;
        }
        u32x4 pw, pr = {};
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            f32x4 p = z[t];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (EDGE && !SHARED)  // a scale of 0 leaves a hidden key hidden
                    p[j] = p[j] == kNegInf ? 0.f : __builtin_amdgcn_exp2f(fmaf(p[j], scale_log2e, -off));
                else
                    p[j] = __builtin_amdgcn_exp2f(FAST ? p[j] : SHARED ? p[j] - off : fmaf(p[j], scale_log2e, -off));
            }
            l[qt] += (p[0] + p[1]) + (p[2] + p[3]);
#pragma unroll
            for (int j = 0; j < 4; j += 2) {
                const uint32_t w = pack_bf16x2(p[j], p[j + 1]);
                pw[2 * t + j / 2] = w;
                if constexpr (TWO) pr[2 * t + j / 2] = minus.rest(p[j], p[j + 1], w);
            }
        }
        return Weights{as_bf16x8(pw), as_bf16x8(pr)};
    };
    auto count = [&](int qt, const Weights& p) {
        if constexpr (!TWO) rounded[qt] = mfma16x16x32(kOnes8, p.rounded, rounded[qt]);
    };
    auto product = [&](int qt, int dt, bf16x8 vt, const Weights& p) {
        o[qt][dt] = mfma16x16x32(vt, p.rounded, o[qt][dt]);
        if constexpr (TWO) rest[dt] = mfma16x16x32(vt, p.rest, rest[dt]);
    };

    // A block that the wave's rows see in full, as a pipeline over units of 32
    // keys and 16 queries: while a unit's weights are formed, the matrix cores
    // take the next one's scores and the last one's values.
    auto attend_whole = [&](int b, auto fast_tag) {
        constexpr int kUnits = 2 * QT;
        bf16x8 kop[2][2], vt[4];
        Weights pk[2];
        f32x4 cf[2], cf_next[2], z[2][2];
        load_k(b, 0, kop, cf);
        scores(0, kop, z[0]);
        if constexpr (QT == 1) {
            load_k(b, 1, kop, cf_next);
        }
#pragma unroll
        for (int u = 0; u < kUnits; ++u) {
            if (u == 0 || u == QT + 1)
#pragma unroll
                for (int dt = 0; dt < 4; ++dt) vt[dt] = load_v(b, u / QT, dt);
            if (u + 1 < kUnits) scores((u + 1) % QT, kop, z[(u + 1) & 1]);
            if (u + 2 == QT) load_k(b, 1, kop, cf_next);  // the last scores of these keys are on their way
            if (u == QT) cf[0] = cf_next[0], cf[1] = cf_next[1];
            auto values = [&] {
                const int qt = (u - 1) % QT;
                count(qt, pk[(u - 1) & 1]);
#pragma unroll
                for (int dt = 0; dt < 4; ++dt) product(qt, dt, vt[dt], pk[(u - 1) & 1]);
            };
            if (QT == 1 && u > 0) values();  // a new maximum rescales this very tile's sums
            if constexpr (SHARED) z[u & 1][0] *= cf[0], z[u & 1][1] *= cf[1];
            pk[u & 1] = weights(u % QT, z[u & 1], fast_tag, Tag<false>{});
            if (QT > 1 && u > 0) values();
            __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (QT == 1)
#pragma unroll
            for (int dt = 0; dt < 4; ++dt) vt[dt] = load_v(b, 1, dt);
        count(QT - 1, pk[1]);
#pragma unroll
        for (int dt = 0; dt < 4; ++dt) product(QT - 1, dt, vt[dt], pk[1]);
    };
    // Any block: every key is tested against every row.
    auto attend_edge = [&](int b, int key0, uint32_t hole) {
#pragma unroll 1
        for (int kp = 0; kp < 2; ++kp) {
            bf16x8 kop[2][2];
            Weights pk[QT];
            f32x4 cf[2];
            load_k(b, kp, kop, cf);
#pragma unroll
            for (int qt = 0; qt < QT; ++qt) {
                f32x4 z[2];
                scores(qt, kop, z);
                const int end = min(least + (int)(past >> (8 * qt) & 255), k1);
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    if constexpr (SHARED) z[t] *= cf[t];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int key = key0 + 32 * kp + 16 * t + 4 * g + j;
                        z[t][j] = key < end && !(hole >> (2 * kp + t) & 1) ? z[t][j] : kNegInf;
                    }
                }
                pk[qt] = weights(qt, z, Tag<false>{}, Tag<true>{});
                count(qt, pk[qt]);
            }
#pragma unroll
            for (int dt = 0; dt < 4; ++dt) {
                const bf16x8 vt = blank(load_v(b, kp, dt), odd);
#pragma unroll
                for (int qt = 0; qt < QT; ++qt) product(qt, dt, vt, pk[qt]);
            }
        }
    };

    // for the whole workgroup: normalised keys bound a logit by the query's length
    const bool fast = SHARED && __syncthreads_and(scale_log2e * sqrtf(biggest) <= kFree);
    if (fast)
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) m[qt] = 0.f;
    if (blocks) {
        fetch(0, 0);
        place(0, 0);
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
    }
    int kb = 0;
    auto hole = [&] {
        const int4 none = *reinterpret_cast<const int4*>(S.hole[kb & 1]);
        return (uint32_t)__builtin_amdgcn_readfirstlane(none.x | none.y << 1 | none.z << 2 | none.w << 3);
    };
    auto step = [&](auto use) {
        const int b = kb & 1;
        if (kb + 1 < blocks) fetch(kb + 1, b ^ 1);
        use(b, k0 + kb * 64);
        if (kb + 1 < blocks) place(kb + 1, b ^ 1);
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
        ++kb;
    };
    // First the blocks that all rows of the workgroup see in full, up to the
    // first hole; then the others, whose keys are tested one by one.  Loops of
    // their own: the choice within one cost 30 registers.
    const int whole = min(blocks, max(row_limit(a, it, r0, G, SHARED) - k0, 0) / 64);
    auto walk = [&](auto fast_tag) {
        while (kb < whole && !hole())
            step([&](int b, int) {
                if (active) attend_whole(b, fast_tag);
            });
    };
    if (fast)
        walk(Tag<true>{});
    else
        walk(Tag<false>{});
    const int edge0 = k0 + kb * 64;
    while (kb < blocks)
        step([&](int b, int key0) {
            if (key0 < mine) attend_edge(b, key0, hole());
        });
    if (!active) return;

#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
        const float sum = sum_xor32(sum_xor16(l[qt])), top = m[qt];
        if constexpr (TWO) {
            rounded[qt][0] = sum;
#pragma unroll
            for (int dt = 0; dt < 4; ++dt) o[qt][dt] = with_rest(o[qt][dt], rest[dt]);
        }
        const int r = 16 * QT * wave + 16 * qt + n;
        if (__any(odd))
            add_odd<TYPE>(a, it.seq, head, edge0, k1, least + (int)(past >> (8 * qt) & 255), g,
                          query_at(a, it, q, head, G, rw + 16 * qt + n), o[qt]);
        if (r0 + r >= it.n_rows) continue;
        if (it.parts > 1) {
            const int64_t at = ((int64_t)it.slot * a.Hkv + head) * sp.rows + r;
#pragma unroll
            for (int dt = 0; dt < 4; ++dt)
                *reinterpret_cast<f32x4*>(parts.o + at * kHeadDim + 16 * dt + 4 * g) = o[qt][dt];
            if (g == 0) parts.stat[at] = f32x4{top, sum, rounded[qt][0], 0.f};
            continue;
        }
        const QueryRow at = query_row(a, it, r0 + r, G, SHARED);
        const int64_t t = it.first + at.token, where = t * a.H + head * G + at.group;
        if (sum == 0.f) {
#pragma unroll 1
            for (int dt = 0; dt < 4; ++dt)
                finish_row<TYPE>(a, q, out, lse, t, head * G + at.group, it.seq, it.pos0 + at.token, 16 * dt + 4 * g,
                                 f32x4{}, 0.f, 0.f, 0.f);
            continue;
        }
        const float over = 1.f / rounded[qt][0];
#pragma unroll
        for (int dt = 0; dt < 4; ++dt)
            *reinterpret_cast<uint2*>(out + where * kHeadDim + 16 * dt + 4 * g) =
                make_uint2(pack_bf16x2(o[qt][dt][0] * over, o[qt][dt][1] * over),
                           pack_bf16x2(o[qt][dt][2] * over, o[qt][dt][3] * over));
        if (lse && g == 0) lse[where] = (top + __log2f(sum)) * kLn2;
    }
}

// ---- the kernels ----

template <CacheType TYPE, bool SHARED>
__global__ __launch_bounds__(256, kNarrowOcc) void cache_narrow_kernel(CacheArgs a, Split sp, Parts parts,
                                                                       const uint16_t* __restrict__ q,
                                                                       uint16_t* __restrict__ out,
                                                                       float* __restrict__ lse) {
    __shared__ __attribute__((aligned(16))) NarrowShared S;
    narrow_tile<TYPE, SHARED>(a, sp, parts, q, out, lse, blockIdx.x, S);
}

// Chunks, and beside them decoding sequences, in one grid, the chunks' tiles first.
// TWO: weights as two numbers, as narrow tiles have them.
template <CacheType TYPE, bool SHARED, int QT, int OCC, bool TWO>
__global__ __launch_bounds__(256, OCC) void cache_wide_kernel(CacheArgs a, Split narrow, Split wide, Parts np, Parts wp,
                                                              const uint16_t* __restrict__ q,
                                                              uint16_t* __restrict__ out, float* __restrict__ lse,
                                                              int items, int sets, uint32_t wide_blocks) {
    constexpr size_t kBytes = sizeof(WideShared<TYPE>) > sizeof(NarrowShared) ? sizeof(WideShared<TYPE>) : sizeof(NarrowShared);
    __shared__ __attribute__((aligned(16))) char mem[kBytes];
    if (blockIdx.x < wide_blocks)
        wide_tile<TYPE, SHARED, QT, TWO>(a, wide, wp, q, out, lse, items, sets, blockIdx.x,
                                         *reinterpret_cast<WideShared<TYPE>*>(mem));
    else
        narrow_tile<TYPE, SHARED>(a, narrow, np, q, out, lse, blockIdx.x - wide_blocks,
                                                         *reinterpret_cast<NarrowShared*>(mem));
}

// ---- joining split rows ----

// LANES lanes a (token, query head), 16, 64 or 256: a lane takes four
// dimensions of every LANES / 16-th part, and the lanes are added in a fixed
// order, so the result does not depend on which part came first.
template <CacheType TYPE, int LANES>
__global__ __launch_bounds__(256) void cache_join_kernel(CacheArgs a, Split narrow, Split wide, bool any_wide, Parts np,
                                                         Parts wp, const uint16_t* __restrict__ q,
                                                         uint16_t* __restrict__ out, float* __restrict__ lse) {
    constexpr int kSub = LANES / 16;  // lanes that share dimensions
    __shared__ f32x4 sums[4][16];
    __shared__ f32x4 stats[4];
    const int wave = threadIdx.x >> 6, lane = lane_id();
    const int64_t item = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
    const int64_t t = item / a.H, t0 = (item - (LANES == 16 ? lane >> 4 : 0)) / a.H;  // of the wave's first row
    const int h = (int)(item - t * a.H), G = a.H / a.Hkv, head = h / G;
    // rows leave whole (with LANES = 256 the workgroup)
    if (t0 >= a.T) return;
    int s = max(seq_of(a.first, a.n_seq, t0), 0);
    if (LANES == 16) s = seq_from(a.first, a.n_seq, s, t);
    if (t >= a.T || t < a.first[s] || t >= a.first[s + 1]) return;
    const int64_t f0 = max((int64_t)a.first[s], (int64_t)0), f1 = min((int64_t)a.first[s + 1], a.T);
    const int rows = (int)(f1 - f0) * G;
    const bool is_narrow = rows <= wide.lo || !any_wide;
    const Split sp = is_narrow ? narrow : wide;
    const Parts p = is_narrow ? np : wp;
    const int2 of = p.of_seq[s];
    const int r = (int)(t - f0) * G + h % G, tile = r / sp.rows;
    if (of.x <= 1 || of.y < 0 || of.y + ((int64_t)tile + 1) * of.x > p.slots) return;
    const int64_t at0 = ((int64_t)(of.y + tile * of.x) * a.Hkv + head) * sp.rows + r % sp.rows;
    const int64_t step = (int64_t)a.Hkv * sp.rows;
    const int d0 = 4 * (lane & 15);
    f32x4 stat = {kNegInf, 0.f, 0.f, 0.f}, o = {};
    auto add = [&](f32x4 st, f32x4 x) {
        const bool some = st[1] != 0.f;  // keys there (x is not written otherwise)
        const float m1 = some ? fmaxf(stat[0], st[0]) : stat[0];
        const float fa = stat[1] != 0.f ? __builtin_amdgcn_exp2f(stat[0] - m1) : 0.f;
        const float fb = some ? __builtin_amdgcn_exp2f(st[0] - m1) : 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = o[e] * fa + (some ? x[e] * fb : 0.f);
        stat = f32x4{m1, stat[1] * fa + st[1] * fb, stat[2] * fa + (some ? st[2] * fb : 0.f), 0.f};
    };
    constexpr int kAtOnce = 4;  // loads under way
    for (int i = (threadIdx.x % LANES) >> 4; i < of.x; i += kSub * kAtOnce) {
        f32x4 st[kAtOnce], x[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const int64_t at = at0 + min(i + kSub * u, of.x - 1) * step;
            st[u] = p.stat[at];
            x[u] = *reinterpret_cast<const f32x4*>(p.o + at * kHeadDim + d0);
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u)
            if (i + kSub * u < of.x) add(st[u], x[u]);
    }
    if constexpr (LANES > 16) {  // the four lanes of a wave that share dimensions
        const float top = max_xor32(max_xor16(stat[0]));
        const float f = stat[1] != 0.f ? __builtin_amdgcn_exp2f(stat[0] - top) : 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = sum_xor32(sum_xor16(o[e] * f));
        stat = f32x4{top, sum_xor32(sum_xor16(stat[1] * f)), sum_xor32(sum_xor16(stat[2] * f)), 0.f};
    }
    if constexpr (LANES > 64) {
        if (lane < 16) sums[wave][lane] = o;
        if (lane == 0) stats[wave] = stat;
        __syncthreads();
        if (threadIdx.x >= 16) return;
        for (int w = 1; w < 4; ++w) add(stats[w], sums[w][lane]);
    }
    if (LANES == 16 || lane < 16)
        finish_row<TYPE>(a, q, out, lse, t, h, s, (int64_t)a.length[s] - a.first[s + 1] + t, d0, o, stat[0], stat[1],
                         stat[2]);
}

// The kernels and splits of a call.
struct Plan {
    bool narrow, wide, two, join, planned;
    int qt;
    Split n, w;
    int64_t n_items, w_items;  // a head, at most
    size_t n_slots, w_slots, bytes;
    int sets, lanes;              // of wide_tile; of the join, a row
    int64_t n_wg, w_wg, join_wg;  // workgroups
};

Plan plan_of(const CacheArgs& a, int max_new) {
    const int64_t G = a.H / a.Hkv, rows = a.T * G, cap = (int64_t)a.max_pages << a.page_log2;
    const int64_t most = (max_new > 0 ? std::min<int64_t>(max_new, a.T) : a.T) * G;  // rows of a sequence, if the hint holds
    constexpr int kAll = 0x7FFFFFFF;
    Plan p{};
    p.narrow = most <= kNarrowRows || a.n_seq > 1;
    p.wide = most > kNarrowRows;
    // Larger tiles read K and V from LDS less often, but leave fewer of them and
    // need more parts to fill the chip.  Measured, 256 / 128 / 64 rows a tile
    // (us): 2K tokens over 32K, 16 heads (2^30 pairs) 331 / 581 / 680; 256 over
    // 64K (2^28) 116 / 122 / 166; 512 over 4K (2^25) 40 / 31 / 38; 24 over 1K, 8
    // heads 13.2 / 11.4 / 10.7.
    const int64_t pairs = a.T * a.H * cap;
    const bool prompt = cap < 2 * most / G;
    if (prompt)  // a whole prompt, half of whose pairs are hidden: parts do not even its tiles out, more tiles do
        p.qt = a.T * a.H >= 512 * 256 ? 4 : 1;  // 16 heads of 8K 206 / 207 / 233, of 4K 107 / 78 / 76, of 2K 51 / 41 / 35
    else
        p.qt = most > 128 && pairs >= 1 << 27 ? 4 : most > 64 && pairs >= 1 << 24 ? 2 : 1;
    // Weights as one number / as two in tiles of 64 rows (us): chunks wait for
    // memory (24 tokens over 1K, 8 heads 10.4 / 10.6; 48 over 16K, 16 heads 24.4
    // / 25.0; 64 over 64K 56.1 / 57.0) and small prompts for launches (512 tokens
    // of 16 heads 19.4 / 20.0; 1000 28.7 / 29.6), but larger ones for the matrix
    // cores (1024 19.1 / 20.9; 2048 32.4 / 35.6; 4096 71 / 84).
    p.two = p.qt == 1 && !(prompt && pairs >= 1 << 24);
    auto a_head = [&](int items) { return (items + a.Hkv - 1) / a.Hkv; };
    // with a sequence and head for every CU, short parts are not needed, and short caches no join
    const int shorter = a.n_seq * (int64_t)a.Hkv >= 256 ? 4 * kNarrowStep : kNarrowStep;
    p.n = {kNarrowRows, 0, p.wide ? kNarrowRows : kAll, kNarrowStep, shorter, 4 * kNarrowStep, a_head(256), a_head(2048)};
    p.w = {64 * p.qt, p.narrow ? kNarrowRows : 0, kAll, 64, 64, 128, a_head(128), a_head(p.qt == 1 ? 768 : 512)};
    // With a tile for every CU only those are split that have twice the keys of
    // the others, of a single sequence none (16 heads of a 2K prompt: 45 -> 41
    // us without parts and without the kernel that joins them).
    if (a.T * a.H >= 256 * p.w.rows) {
        p.w.few = p.w.target = (int)std::max<int64_t>(rows / p.w.rows / 2, 1);
        if (a.n_seq == 1) p.w.shorter = p.w.longer = (int)cap;
    }
    const int64_t seqs = std::min<int64_t>(a.n_seq, a.T);
    if (!p.wide && seqs * a.Hkv >= 2048) p.n.target = (int)(seqs + 1) / 2;  // decoding, likewise
    p.planned = a.n_seq > 128;
    size_t off = align256((size_t)a.n_seq * sizeof(int2)) + (p.planned ? 2 * align256((size_t)a.n_seq * sizeof(int4)) : 0);
    auto size = [&](const Split& s, int64_t tiles, int64_t& items, size_t& slots) {
        const int64_t parts = (cap + s.shorter - 1) / s.shorter;  // of a tile, at most
        items = std::min<int64_t>(s.target, tiles * (parts - 1)) + tiles;
        slots = parts > 1 ? (size_t)std::min<int64_t>(2 * (int64_t)s.target, tiles * parts) : 0;
        off += align256(slots * a.Hkv * s.rows * kHeadDim * sizeof(float)) + align256(slots * a.Hkv * s.rows * sizeof(f32x4));
    };
    if (p.narrow) size(p.n, p.wide ? seqs : rows / kNarrowRows + seqs, p.n_items, p.n_slots);
    if (p.wide) size(p.w, rows / p.w.rows + seqs, p.w_items, p.w_slots);
    p.join = p.n_slots + p.w_slots > 0;
    p.bytes = off;
    p.sets = kXcds;
    while (a.Hkv % p.sets != 0) p.sets /= 2;
    const int64_t turns = p.w_items * (a.Hkv / p.sets), per = kXcds / p.sets;
    p.w_wg = (turns + per - 1) / per * kXcds, p.n_wg = p.n_items * a.Hkv;
    // Few rows have many parts each, many rows few.
    p.lanes = a.T * a.H <= 1024 ? 256 : a.T * a.H <= 16384 ? 64 : 16;
    p.join_wg = p.join ? (a.T * a.H * p.lanes + 255) / 256 : 0;
    return p;
}

template <CacheType TYPE, bool SHARED>
hipError_t launch(const CacheArgs& a, const Plan& p, const uint16_t* q, uint16_t* out, float* lse, void* workspace,
                  hipStream_t stream) {
    char* at = static_cast<char*>(workspace) + align256((size_t)a.n_seq * sizeof(int2));
    auto plan = [&](bool used) {
        int4* r = used && p.planned ? reinterpret_cast<int4*>(at) : nullptr;
        if (p.planned) at += align256((size_t)a.n_seq * sizeof(int4));
        return r;
    };
    int4* const n_plan = plan(p.narrow);
    int4* const w_plan = plan(p.wide);
    auto carve = [&](size_t slots, const Split& s, const int4* of) {
        Parts r;
        r.plan = of;
        r.of_seq = static_cast<int2*>(workspace);
        r.slots = (int)slots;
        r.o = reinterpret_cast<float*>(at);
        at += align256(slots * a.Hkv * s.rows * kHeadDim * sizeof(float));
        r.stat = reinterpret_cast<f32x4*>(at);
        at += align256(slots * a.Hkv * s.rows * sizeof(f32x4));
        return r;
    };
    const Parts np = carve(p.n_slots, p.n, n_plan), wp = carve(p.w_slots, p.w, w_plan);
    if (p.planned) {
        cache_plan_kernel<<<2, 1024, 0, stream>>>(a, p.n, p.w, n_plan, w_plan);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    const unsigned wide = (unsigned)p.w_wg, narrow = (unsigned)p.n_wg;
    if (p.wide) {
        auto go = [&](auto kernel) {
            kernel<<<wide + narrow, 256, 0, stream>>>(a, p.n, p.w, np, wp, q, out, lse, (int)p.w_items, p.sets, wide);
        };
        switch (p.qt) {
            case 4: go(cache_wide_kernel<TYPE, SHARED, 4, 2, false>); break;
            case 2: go(cache_wide_kernel<TYPE, SHARED, 2, 2, false>); break;
            default:
                if (p.two)
                    go(cache_wide_kernel<TYPE, SHARED, 1, 3, true>);
                else
                    go(cache_wide_kernel<TYPE, SHARED, 1, 3, false>);
        }
    } else {
        cache_narrow_kernel<TYPE, SHARED><<<narrow, 256, 0, stream>>>(a, p.n, np, q, out, lse);
    }
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    if (p.join) {
        auto go = [&](auto kernel) {
            kernel<<<(unsigned)p.join_wg, 256, 0, stream>>>(a, p.n, p.w, p.wide, np, wp, q, out, lse);
        };
        switch (p.lanes) {
            case 256: go(cache_join_kernel<TYPE, 256>); break;
            case 64: go(cache_join_kernel<TYPE, 64>); break;
            default: go(cache_join_kernel<TYPE, 16>);
        }
    }
    return hipGetLastError();
}

}  // namespace

bool cache_attn_fits(const CacheArgs& a, int max_new) {
    const Plan p = plan_of(a, max_new);
    return p.w_wg + p.n_wg <= kMaxWorkgroups && p.join_wg <= kMaxWorkgroups;
}

size_t cache_attn_workspace_bytes(const CacheArgs& a, int max_new) { return plan_of(a, max_new).bytes; }

hipError_t launch_cache_attn(const CacheArgs& a, CacheType type, int max_new, const uint16_t* q, uint16_t* out,
                             float* lse, void* workspace, hipStream_t stream) {
    const Plan p = plan_of(a, max_new);
    auto go = [&](auto one, auto other) { return (a.shared ? one : other)(a, p, q, out, lse, workspace, stream); };
    switch (type) {
        case kCacheBf16: return go(launch<kCacheBf16, true>, launch<kCacheBf16, false>);
        case kCacheE4m3: return go(launch<kCacheE4m3, true>, launch<kCacheE4m3, false>);
        default: return go(launch<kCacheE2m1, true>, launch<kCacheE2m1, false>);
    }
}

}  // namespace lsh
