// Token eviction by accumulated attention weight: per (layer, sequence, KV head) the heaviest tokens stay, and their K and V
// rows and masses are closed up.
//
// Selection (select_kernel, a CTA, or where there are few of them a cluster of CTAs, per (layer, sequence, KV head)).  The masses'
// order as unsigned keys (key_of); the key of the quota-th heaviest candidate is found digit by digit, 11, 11 and 10 bits,
// counting keys per digit value in shared memory (added up over the cluster's shared memories); keys above it stay, and of
// those equal to it the first ones.  A last pass in the order of positions numbers the kept tokens.  The first digit has
// sign, exponent and two bits of the fraction, so that masses that differ by powers of two - attention weights do - spread
// over the counters, and few are left with the limit's first digit: these are listed in the pass that counts the kept
// tokens, and the other digits are found from the list.  The masses stay in shared memory for the passes if they fit.
// Of few tokens, one per thread, each is compared with every other instead.
//
// Rows (move_kernel).  A kept row is read and written once, 8 * head_dim bytes for K and V together: memory-bound, in pieces of a row
// (2 * head_dim bytes) at scattered places.  Whole rows are moved by neighbouring lanes, rows in the order of their
// positions by neighbouring warps, so that the memory sees its pages' accesses together.  To other slots every CTA takes a
// range of rows.  In place a kept row's new position never lies behind its old one: a CTA that goes up in batches, each read
// completely before it is written, never overwrites a row that it has yet to read.  Where there are few slabs a cluster
// shares one, batch by batch.
//
// One kernel or two.  Where an item's rows are few batches, or there are items enough to keep the memory busy with one CTA each,
// the CTA that selected the rows moves them too (FUSED; the rule stands in llms_evict_tokens): some CTAs select while
// others move.
//
// Measured, a B200: 32 layers x 32 heads of 128 channels, 4096 -> 2048 tokens in place 364 us (2.19 GB, 6.0 TB/s: bound by the
// memory); 32 x 8 heads, 32768 -> 8192 to other slots 374 us, of which 44 select; 1 layer x 4 heads, 256 -> 128: 6.4 us, a
// chain of comparisons and rounds.
#include <algorithm>

#include <cooperative_groups.h>

#include "paged.cuh"

namespace llms {

namespace cg = cooperative_groups;

constexpr int kSliceTokens = 16384;               // masses that a CTA holds in shared memory; of longer sequences it reads them again,
constexpr int kSliceTokensShared = 40960;         // but a cluster's CTAs hold theirs (with four sets of counters and the longest list 224 KiB)
constexpr int kBins = 2048;
constexpr int kMoveThreads = 256;
__host__ __device__ constexpr int in_flight(bool cluster) { return cluster ? 8 : 4; }   // 16-byte vectors of a thread
constexpr int kMaxCluster = 8;
// Up to so many tokens each candidate is compared with every other: 4 items, 256 -> 16 tokens 6.8 us by digits, 5.8; 88 -> 3 tokens
// 6.6 and 4.1
constexpr int kPairTokens = 256;
constexpr int kFusedMostThreads = 512;            // of a CTA that selects and moves: 64 registers a thread

struct EvictArgs {
    const float *mass;
    float *mass_out;
    uint16_t *kv;
    const int32_t *table, *dst_table, *lens;
    int32_t *kept, *new_lens;
    int64_t stride_l, stride_s, stride_h, mass_stride;
    int table_stride, dst_stride, n_seqs, max_len, L, Hkv, d, chunk_len, n_slots, budget, recent;
    int list_room;                                // keys with the limit's first digit that are listed
    int in_smem, select_shift, warps_shift;       // the masses fit into shared memory; log2 of the CTAs per (layer, sequence, KV head)
                                                  // and of the warps per CTA
    Divisor by_chunk, by_parts, by_vec;
    int parts, batches;                           // move: CTAs per slab; batches of rows a CTA takes (0: all, in place)
};

// What a mass is ranked by: NaN as -inf, -0 as +0.
__device__ __forceinline__ float rank_value(float m) { return fmaxf(m, -INFINITY) + 0.0f; }
// The order of these values as unsigned keys, 0x007fffff (-inf) to 0xff800000 (+inf), and back.
__device__ __forceinline__ uint32_t key_of(float v)
{
    const uint32_t u = __float_as_uint(v);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key ^ (((int32_t)key >> 31) ? 0x80000000u : 0xffffffffu)); }

__device__ __forceinline__ int slot_row(const EvictArgs &a, const int32_t *row, int t)
{
    const int chunk = a.by_chunk(t), slot = __ldg(row + chunk);
    return (unsigned)slot < (unsigned)a.n_slots ? slot * a.chunk_len + (t - chunk * a.chunk_len) : -1;
}

// The places of rows j0 .. j0 + n - 1 of the m kept ones: old and new row; a new row of -1: nothing to move.
__device__ __forceinline__ void look_up_rows(const EvictArgs &a, int2 *rows, const int32_t *kept, const int32_t *from, const int32_t *to, int j0, int n,
                                             int m, int tid, int threads)
{
    for (int i = tid; i < n; i += threads) {
        const int j = j0 + i;
        int2 x = make_int2(-1, -1);
        if (j < m) {
            x.x = slot_row(a, from, __ldcg(kept + j));
            x.y = slot_row(a, to, j);
            if (x.x < 0 || x.x == x.y) x.y = -1;
        }
        rows[i] = x;
    }
}

template <bool CLUSTER, bool FUSED>
__global__ void __launch_bounds__(FUSED ? kFusedMostThreads : 1024, 2) select_kernel(const EvictArgs a)
{
    // counters, one set per digit in a cluster (other CTAs may still read the last one) and one for the sums; list; masses
    extern __shared__ uint4 smem_select[];
    uint32_t *hist = reinterpret_cast<uint32_t *>(smem_select);
    uint32_t *const sums = hist + (CLUSTER ? 3 * kBins : 0);
    uint2 *list = reinterpret_cast<uint2 *>(sums + kBins);                     // key, token
    float *slice = reinterpret_cast<float *>(list + a.list_room);
    __shared__ uint32_t warp_sum[32], warp_eq[32], warp_add[2][32], s_digit, s_need, s_bin, s_listed, s_counts[2];
    const int threads = blockDim.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n_warps = threads >> 5;
    const int parts = CLUSTER ? 1 << a.select_shift : 1, part = CLUSTER ? blockIdx.x & (parts - 1) : 0;
    const int h = CLUSTER ? blockIdx.x >> a.select_shift : blockIdx.x, b = blockIdx.y, l = blockIdx.z;
    const int64_t row = ((int64_t)l * a.n_seqs + b) * a.Hkv + h;
    const float *mass = a.mass + row * a.mass_stride;
    float *mass_out = a.mass_out + row * a.mass_stride;
    int32_t *kept = a.kept + row * a.budget;
    const bool no_digits = !CLUSTER && a.max_len <= min(threads, kPairTokens);
    if (!no_digits)
        for (int i = tid; i < (CLUSTER ? 3 : 1) * kBins / 4; i += threads) smem_select[i] = make_uint4(0, 0, 0, 0);
    grid_dependency_wait();
    grid_launch_dependents();
    const int len = __ldg(a.lens + b);
    const bool bad = len < 0 || len > a.max_len;
    const int n = bad ? 0 : len, m = min(a.budget, n), recent = min(a.recent, m), cand = n - recent, quota = m - recent;
    // this CTA's tokens, from t0 on, and how many of them are candidates
    const int share = CLUSTER ? (((n + parts - 1) >> a.select_shift) + 3) & ~3 : n, t0 = CLUSTER ? min(n, part * share) : 0, count = min(n, t0 + share) - t0;
    // (none if they all stay).  Values above the limit's stay, and the first `need` ones equal to it
    const int mine = quota >= cand ? 0 : max(0, min(count, cand - t0));
    const bool pairs = !CLUSTER && a.in_smem && n <= min(threads, kPairTokens);
    const bool ranked = quota > 0 && quota < cand && !pairs;
    uint32_t limit = 0, need = ranked ? quota : 0;
    const float *from = a.in_smem ? slice : mass;
    // four neighbouring masses (what lies behind the last one is -inf and counts nowhere)
    const bool wide = a.in_smem || (reinterpret_cast<uintptr_t>(mass) & 15) == 0;                // t0 is a multiple of four
    auto four = [&](const float *src, int i, bool vector) {
        if (vector && i + 4 <= count) return *reinterpret_cast<const float4 *>(src + i);
        return make_float4(i < count ? src[i] : -INFINITY, i + 1 < count ? src[i + 1] : -INFINITY, i + 2 < count ? src[i + 2] : -INFINITY,
                           i + 3 < count ? src[i + 3] : -INFINITY);
    };
    // a warp's own tokens, for the passes in the order of positions
    const int warp_shift = a.warps_shift, each_warp = (((count + n_warps - 1) >> warp_shift) + 127) & ~127, w0 = min(count, warp * each_warp), w1 = min(count, w0 + each_warp);
    uint32_t n_gt = 0, n_eq = 0;                  // of the warp's tokens: above the limit, equal to it
    if (tid == 0) s_listed = 0;
    if (tid < 32) warp_add[0][tid] = warp_add[1][tid] = 0;
    __syncthreads();                              // hist is cleared
    const bool aligned_rows = (reinterpret_cast<uintptr_t>(mass) & 15) == 0;
#pragma unroll 2
    for (int i = 4 * tid; i < count; i += 4 * threads) {
        const float4 x = four(mass + t0, i, aligned_rows);
        if (a.in_smem) *reinterpret_cast<float4 *>(slice + i) = x;
        if (ranked) {
            const float w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (i + j < mine) atomicAdd(&hist[key_of(rank_value(w[j])) >> 21], 1u);
        }
    }
    __syncthreads();
    bool listed = false;
    if (ranked) {
#pragma unroll 1
        for (int shift = 21; ; shift = max(0, shift - 11)) {
            // from the highest value down: thread t has 2048 / threads neighbouring ones
            const int each = kBins >> (5 + a.warps_shift), top = kBins - 1 - tid * each;
            uint32_t sum = 0;
            if constexpr (CLUSTER) {
                cg::this_cluster().sync();
                for (int i = 0; i < each; ++i) {
                    uint32_t c = 0;
                    for (int p = 0; p < parts; ++p) c += cg::this_cluster().map_shared_rank(hist, p)[top - i];
                    sums[top - i] = c;
                    sum += c;
                }
            } else if (each >= 4) {
                for (int i = 0; i < each / 4; ++i) {
                    const uint4 x = smem_select[top / 4 - i];
                    sum += x.x + x.y + x.z + x.w;
                }
            } else {
                for (int i = 0; i < each; ++i) sum += hist[top - i];
            }
            uint32_t upto = sum;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const uint32_t up = __shfl_up_sync(0xffffffffu, upto, d);
                if (lane >= d) upto += up;
            }
            if (lane == 31) warp_sum[warp] = upto;
            __syncthreads();
            upto += __reduce_add_sync(0xffffffffu, lane < warp ? warp_sum[lane] : 0u);
            uint32_t above = upto - sum;          // keys with higher values
            if (above < need && upto >= need) {
                int i = 0;
                while (above + sums[top - i] < need) above += sums[top - i++];
                s_digit = top - i;
                s_need = need - above;
                s_bin = sums[top - i];
            }
            __syncthreads();
            limit |= s_digit << shift;
            need = s_need;
            if (shift == 0) break;
            if constexpr (CLUSTER) {
                hist += kBins;
            } else {
                for (int i = tid; i < kBins / 4; i += threads) smem_select[i] = make_uint4(0, 0, 0, 0);
                __syncthreads();
            }
            const uint32_t want = limit >> shift;
            if (shift == 21) {
                listed = s_bin <= (uint32_t)a.list_room;                       // the whole cluster's: the same for all its CTAs
                if (listed) {
                    // values from `low` on have the limit's digit, from `high` on a higher one (none if that is no number)
                    const float high = value_of((want + 1) << 21), low = want << 21 < 0x007fffffu ? -INFINITY : value_of(want << 21);
#pragma unroll 2
                    for (int i = w0 + 4 * lane; i < w1; i += 128) {
                        const float4 x = four(from, i, wide);
                        const float w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float v = fmaxf(w[j], -INFINITY);
                            const bool above = i + j >= mine || v >= high;
                            n_gt += above && i + j < w1;
                            if (!above && v >= low) list[atomicAdd(&s_listed, 1u)] = make_uint2(key_of(v + 0.0f), i + j);
                        }
                    }
                    __syncthreads();
                }
            }
            const int next = max(0, shift - 11), bits = shift - next;          // 11, then 10
            if (listed) {
                for (int i = tid; i < (int)s_listed; i += threads) {
                    const uint32_t k = list[i].x;
                    if (k >> shift == want) atomicAdd(&hist[(k >> next) & ((1u << bits) - 1u)], 1u);
                }
            } else {
#pragma unroll 8
                for (int i = tid; i < mine; i += threads) {
                    const uint32_t k = key_of(rank_value(from[i]));
                    if (k >> shift == want) atomicAdd(&hist[(k >> next) & ((1u << bits) - 1u)], 1u);
                }
            }
            __syncthreads();
        }
    }
    const float border = ranked ? value_of(limit) : INFINITY;                  // nothing to rank: no candidate stays
    auto stays = [&](int i, float w, bool &gt, bool &eq) {                     // token t0 + i
        const float v = fmaxf(w, -INFINITY);
        gt = i >= mine || v > border;
        eq = !gt && v == border;
    };
    if (pairs) {
        // a token per thread: it stays if fewer than `quota` candidates come before it.  Those of the warps before come before it
        // if they are as heavy, those of the warps behind if they are heavier
        const float w = tid < n ? slice[tid] : 0.0f, v = fmaxf(w, -INFINITY);
        const int own = warp * 32;
        int before = 0;
        bool stay = tid < n;
        if (quota < cand && own < cand) {
#pragma unroll 2
            for (int j = 0; j < own; j += 4) {
                const float4 x = *reinterpret_cast<const float4 *>(slice + j);
                before += (fmaxf(x.x, -INFINITY) >= v) + (fmaxf(x.y, -INFINITY) >= v) + (fmaxf(x.z, -INFINITY) >= v) + (fmaxf(x.w, -INFINITY) >= v);
            }
#pragma unroll 8
            for (int j = 0; j < 32; ++j) {
                const float x = __shfl_sync(0xffffffffu, v, j);
                before += own + j < cand && (j < lane ? x >= v : x > v);
            }
            for (int j = own + 32; j < cand; ++j) before += fmaxf(slice[j], -INFINITY) > v;
            stay = stay && (tid >= cand || before < quota);
        }
        const uint32_t ballot = __ballot_sync(0xffffffffu, stay);
        if (lane == 0) warp_sum[warp] = __popc(ballot);
        __syncthreads();
        const int to = __reduce_add_sync(0xffffffffu, lane < warp ? warp_sum[lane] : 0u) + __popc(ballot & ((1u << lane) - 1u));
        if (stay) {
            kept[to] = tid;
            mass_out[to] = w;
        }
    } else if (CLUSTER || a.in_smem || a.mass != a.mass_out) {
        // a warp takes neighbouring tokens, 32 at a time: it counts its ones, then numbers them in the order of positions
        if (listed) {
            for (int i = tid; i < (int)s_listed; i += threads) {
                const uint2 x = list[i];
                if (x.x >= limit) atomicAdd(&warp_add[x.x == limit][x.y / (uint32_t)each_warp], 1u);
            }
        } else {
            for (int i = w0 + 4 * lane; i < w1; i += 128) {
                const float4 x = four(from, i, wide);
                const float w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    bool gt, eq;
                    stays(i + j, w[j], gt, eq);
                    n_gt += gt && i + j < w1;
                    n_eq += eq && i + j < w1;
                }
            }
        }
        __syncthreads();
        uint32_t g = n_gt, e = n_eq;
        g = __reduce_add_sync(0xffffffffu, g);
        e = __reduce_add_sync(0xffffffffu, e);
        if (lane == 0) {
            warp_sum[warp] = g + warp_add[0][warp];
            warp_eq[warp] = e + warp_add[1][warp];
        }
        __syncthreads();
        const uint32_t all_g = lane < n_warps ? warp_sum[lane] : 0u, all_e = lane < n_warps ? warp_eq[lane] : 0u;
        g = __reduce_add_sync(0xffffffffu, lane < warp ? all_g : 0u);
        e = __reduce_add_sync(0xffffffffu, lane < warp ? all_e : 0u);
        if constexpr (CLUSTER) {
            if (warp == 0) {
                const uint32_t cta_g = __reduce_add_sync(0xffffffffu, all_g), cta_e = __reduce_add_sync(0xffffffffu, all_e);
                if (lane == 0) {
                    s_counts[0] = cta_g;
                    s_counts[1] = cta_e;
                }
            }
            cg::this_cluster().sync();            // every mass of the sequence has been read: mass_out may be the same array
            for (int p = 0; p < part; ++p) {
                const uint32_t *c = cg::this_cluster().map_shared_rank(&s_counts[0], p);
                g += c[0];
                e += c[1];
            }
        }
        uint32_t first = g + min(e, need);        // where the warp's first token goes that stays
#pragma unroll 1
        for (int i0 = w0; i0 < w1; i0 += 128) {
            const int i = i0 + 4 * lane;
            const float4 x = four(from, i, wide);
            const float w[4] = {x.x, x.y, x.z, x.w};
            uint32_t gts = 0, eqs = 0;            // bit j: token i + j is above the limit, equal to it
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                bool gt, eq;
                stays(i + j, w[j], gt, eq);
                gts |= (gt && i + j < w1 ? 1u : 0u) << j;
                eqs |= (eq && i + j < w1 ? 1u : 0u) << j;
            }
            if (__any_sync(0xffffffffu, eqs)) {   // few tokens are equal to the limit: those that stay join the others
                uint32_t upto = __popc(eqs);
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const uint32_t up = __shfl_up_sync(0xffffffffu, upto, d);
                    if (lane >= d) upto += up;
                }
                uint32_t e_me = e + upto - __popc(eqs);
                e += __shfl_sync(0xffffffffu, upto, 31);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (eqs >> j & 1) gts |= (e_me++ < need ? 1u : 0u) << j;
            }
            uint32_t upto = __popc(gts);
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const uint32_t up = __shfl_up_sync(0xffffffffu, upto, d);
                if (lane >= d) upto += up;
            }
            uint32_t to = first + upto - __popc(gts);
            first += __shfl_sync(0xffffffffu, upto, 31);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (gts >> j & 1) {
                    kept[to] = t0 + i + j;
                    mass_out[to++] = w[j];
                }
        }
        if constexpr (CLUSTER) cg::this_cluster().sync();                      // nobody reads this CTA's counts any more
    } else {
        // a token per thread, tile by tile: what is written lies at or before the tokens that have been read, so mass_out may be
        // the same array
        const uint32_t below = (1u << lane) - 1u;
        uint32_t g = 0, e = 0;
#pragma unroll 1
        for (int i0 = 0; i0 < n; i0 += threads) {
            const int t = i0 + tid;
            bool gt = false, eq = false;
            float w = 0.0f;
            if (t < n) {
                w = mass[t];
                stays(t, w, gt, eq);
            }
            const uint32_t bg = __ballot_sync(0xffffffffu, gt), be = __ballot_sync(0xffffffffu, eq);
            __syncthreads();                      // the sums of the tile before have been read
            if (lane == 0) {
                warp_sum[warp] = __popc(bg);
                warp_eq[warp] = __popc(be);
            }
            __syncthreads();
            const uint32_t wg = lane < n_warps ? warp_sum[lane] : 0u, we = lane < n_warps ? warp_eq[lane] : 0u;
            const uint32_t e_me = e + __reduce_add_sync(0xffffffffu, lane < warp ? we : 0u) + __popc(be & below);
            const uint32_t to = g + __reduce_add_sync(0xffffffffu, lane < warp ? wg : 0u) + __popc(bg & below) + min(e_me, need);
            if (gt || (eq && e_me < need)) {
                kept[to] = t;
                mass_out[to] = w;
            }
            g += __reduce_add_sync(0xffffffffu, wg);
            e += __reduce_add_sync(0xffffffffu, we);
        }
        __syncthreads();
    }
    for (int j = m + part * threads + tid; j < a.budget; j += parts * threads) kept[j] = -1;
    for (int t = m + part * threads + tid; t < n; t += parts * threads) mass_out[t] = 0.0f;
    if (tid == 0 && part == 0 && l == 0 && h == 0) a.new_lens[b] = bad ? -1 : m;
    if constexpr (FUSED) {
        // half of the threads move the K rows, half the V rows, in batches as move_kernel's
        const bool in_place = a.dst_table == nullptr;
        if (bad || (in_place && m == n)) return;
        constexpr int kInFlight = in_flight(false);
        const int vec = a.d / 8, per_half = threads / 2, at_once = a.by_vec(per_half), batch = at_once * kInFlight;
        const int half = tid >= per_half, r = a.by_vec(tid - half * per_half), c = tid - half * per_half - r * vec;
        const bool live = r < at_once;
        const int32_t *table = a.table + (int64_t)b * a.table_stride, *to = in_place ? table : a.dst_table + (int64_t)b * a.dst_stride;
        uint4 *slab = reinterpret_cast<uint4 *>(a.kv + l * a.stride_l + half * a.stride_s + h * a.stride_h) + c;
        int2 *rows = reinterpret_cast<int2 *>(hist);                           // of these rows and of the next ones, in the counters' place
        __syncthreads();                          // kept is complete, the counters are done with
        look_up_rows(a, rows, kept, table, to, 0, batch, m, tid, threads);
        __syncthreads();
#pragma unroll 1
        for (int j0 = 0, k = 0; j0 < m; j0 += batch, k ^= 1) {
            uint4 v[kInFlight];
            int d[kInFlight];
#pragma unroll
            for (int u = 0; u < kInFlight; ++u) {
                const int2 x = live ? rows[k * batch + u * at_once + r] : make_int2(-1, -1);
                d[u] = x.y;
                if (x.y >= 0) v[u] = __ldcg(slab + (int64_t)x.x * vec);
            }
            if (j0 + batch < m) look_up_rows(a, rows + (k ^ 1) * batch, kept, table, to, j0 + batch, batch, m, tid, threads);
            __syncthreads();
#pragma unroll
            for (int u = 0; u < kInFlight; ++u)
                if (d[u] >= 0) slab[(int64_t)d[u] * vec] = v[u];
        }
    }
}

// A slab (K or V of a KV head) of one sequence; its CTAs take batches of rows in turn.
template <bool IN_PLACE, bool CLUSTER>
__global__ void __launch_bounds__(kMoveThreads, 4) move_kernel(const EvictArgs a)
{
    constexpr int kInFlight = in_flight(CLUSTER), kMostRows = kMoveThreads / 2 * kInFlight;                   // of a batch: rows have at least two vectors
    __shared__ int2 rows[2][kMostRows];           // old and new row, of this batch and the next; a new row of -1: nothing to move
    const int vec = a.d / 8, at_once = a.by_vec(kMoveThreads), batch = at_once * kInFlight, tid = threadIdx.x;
    const int r = a.by_vec(tid), c = tid - r * vec;
    const bool live = r < at_once;
    const int slab_of = a.by_parts(blockIdx.x), part = blockIdx.x - slab_of * a.parts;
    const int half = slab_of & 1, h = slab_of >> 1, b = blockIdx.y, l = blockIdx.z;
    const int32_t *kept = a.kept + (((int64_t)l * a.n_seqs + b) * a.Hkv + h) * a.budget;
    const int32_t *from = a.table + (int64_t)b * a.table_stride;
    const int32_t *to = IN_PLACE ? from : a.dst_table + (int64_t)b * a.dst_stride;
    uint4 *slab = reinterpret_cast<uint4 *>(a.kv + l * a.stride_l + half * a.stride_s + h * a.stride_h) + c;
    grid_dependency_wait();
    grid_launch_dependents();
    const int n = __ldg(a.lens + b);
    if (n < 0 || n > a.max_len) return;
    const int m = min(a.budget, n);
    if (IN_PLACE && m == n) return;               // every row stays where it is
    const int first = IN_PLACE ? part * batch : part * a.batches * batch, step = IN_PLACE ? a.parts * batch : batch;
    const int rounds = IN_PLACE ? (m + step - 1) / step : min(a.batches, max(0, m - first + batch - 1) / batch);
    auto look_up = [&](int k) { look_up_rows(a, rows[k & 1], kept, from, to, first + k * step, batch, m, tid, kMoveThreads); };
    if (rounds > 0) look_up(0);
    __syncthreads();
#pragma unroll 1
    for (int k = 0; k < rounds; ++k) {            // in a cluster every CTA goes through every round
        uint4 v[kInFlight];
        int d[kInFlight];
#pragma unroll
        for (int u = 0; u < kInFlight; ++u) {
            const int2 x = live ? rows[k & 1][u * at_once + r] : make_int2(-1, -1);
            d[u] = x.y;
            if (x.y >= 0) v[u] = __ldcg(slab + (int64_t)x.x * vec);
        }
        if (k + 1 < rounds) look_up(k + 1);       // while the vectors are on their way
        if constexpr (CLUSTER) cg::this_cluster().sync();
        else __syncthreads();
#pragma unroll
        for (int u = 0; u < kInFlight; ++u)
            if (d[u] >= 0) slab[(int64_t)d[u] * vec] = v[u];
    }
}

}  // namespace llms

using namespace llms;

extern "C" int llms_evict_tokens(const llms_kv_desc *desc, void *kv, const float *mass, int64_t mass_stride,
                                 const int32_t *chunk_table, int table_stride, const int32_t *lens, int n_seqs, int max_len,
                                 int budget, int recent, const int32_t *dst_table, int dst_stride, float *mass_out,
                                 int32_t *kept, int32_t *new_lens, void *stream)
{
    const int rc = check_paged(desc, n_seqs, max_len);
    if (rc) return rc;
    if (budget < 1 || recent < 0 || recent > budget) return LLMS_ERR_INVALID_ARG;
    if (n_seqs == 0) return LLMS_OK;
    if (!kv || !mass || !chunk_table || !lens || !mass_out || !kept || !new_lens || new_lens == lens) return LLMS_ERR_INVALID_ARG;
    if (table_stride < 1 || (int64_t)table_stride * desc->chunk_len < max_len || mass_stride < max_len) return LLMS_ERR_INVALID_ARG;
    const int most = budget < max_len ? budget : max_len;
    if (dst_table && (dst_stride < 1 || (int64_t)dst_stride * desc->chunk_len < most)) return LLMS_ERR_INVALID_ARG;
    if (dst_table == chunk_table) {               // the sequences' own chunks; of one sequence the strides mean nothing
        if (n_seqs > 1 && dst_stride != table_stride) return LLMS_ERR_INVALID_ARG;
        dst_table = nullptr;
    }
    if (!aligned(kv, 16)) return LLMS_ERR_MISALIGNED;
    if (!aligned(mass, 4) || !aligned(mass_out, 4) || !aligned(chunk_table, 4) || !aligned(lens, 4) || !aligned(dst_table, 4) ||
        !aligned(kept, 4) || !aligned(new_lens, 4))
        return LLMS_ERR_MISALIGNED;
    const int64_t items = (int64_t)desc->n_layers * n_seqs * desc->n_kv_heads;
    if (items > 0x7fffffff / 64 || desc->n_layers > 65535) return LLMS_ERR_UNSUPPORTED;
    EvictArgs a{};
    a.mass = mass; a.mass_out = mass_out;
    a.kv = static_cast<uint16_t *>(kv);
    a.table = chunk_table; a.dst_table = dst_table; a.lens = lens;
    a.kept = kept; a.new_lens = new_lens;
    a.stride_l = desc->stride_l; a.stride_s = desc->stride_s; a.stride_h = desc->stride_h; a.mass_stride = mass_stride;
    a.table_stride = table_stride; a.dst_stride = dst_stride;
    a.n_seqs = n_seqs; a.max_len = max_len; a.L = desc->n_layers; a.Hkv = desc->n_kv_heads; a.d = desc->head_dim;
    a.chunk_len = desc->chunk_len; a.n_slots = n_chunks(*desc);
    a.by_chunk = Divisor(a.chunk_len);
    a.by_vec = Divisor(a.d / 8);
    a.budget = budget; a.recent = recent;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    // Selection: as many threads as fit the GPU at once, but no fewer than 128 to a CTA and two masses to a thread
    const int64_t room = (int64_t)sm_count() * 2048;
    int threads = 1024;
    while (threads > 128 && (items * threads > room || threads * 2 > max_len)) threads /= 2;
    int parts = 1;
    while (parts < kMaxCluster && items * threads * parts * 2 <= room && parts * threads * 4 <= max_len) parts *= 2;
    int share = ((max_len + parts - 1) / parts + 3) & ~3;
    if (share > kSliceTokensShared) parts = 1, share = max_len;
    // One kernel instead of two.  Where an item's rows make few batches it saves a launch (2 layers x 8 heads: 256 -> 96 tokens
    // 9.8 -> 9.2 us, but 256 -> 128, four batches, 9.9 -> 10.3).  With more items some CTAs select while others move; what holds
    // against it is that an item's move has one CTA only, with a selection's shared memory.  256 items, 2000 -> 1000 tokens, 16
    // batches: 58 -> 54 us, 4096 -> 2048: 101 -> 102; 160 items: 43 -> 46.  More CTAs than the GPU takes at once, 1024 items,
    // 4096 -> 2048: 422 -> 362; 16384 -> 4096, with two CTAs per SM: 816 -> 997.  512 threads if they all run at once: 256
    // items, 1024 -> 512 tokens: 37 us with 256, 32 with 512; 512 items: 56 and 60.  128 for more than run at
    // once and little to keep: 3024 items, 600 -> 100 tokens 88 us with 256, 84 with 128; 256 -> 16: 54 and 36; 600 -> 250: 151 and
    // 148, but 2048 ragged ones of up to 1024 -> 512 tokens 58 and 62.  64 threads: 3024 items, 32 -> 8: 12.6 us with 128, 9.9 with 64
    const int resident = sm_count() * 1024;       // threads
    int fused_threads = threads >= 512 && items * 512 <= resident ? 512 : 256;
    if (items * 256 > resident && most <= 256) fused_threads = max_len <= 64 ? 64 : 128;
    const int fused_batch = fused_threads / 2 / (a.d / 8) * in_flight(false);
    const int fused_batches = (most + fused_batch - 1) / fused_batch;
    a.in_smem = parts > 1 || max_len <= kSliceTokens;
    a.list_room = std::min(4096, std::max(256, (share / 8 + 1) & ~1));
    const size_t smem = (parts > 1 ? 4 : 1) * kBins * 4 + (size_t)a.list_room * 8 + (a.in_smem ? round_up((uint64_t)share * 4, 16) : 0);
    static_assert(kFusedMostThreads / 4 * in_flight(false) * 2 * sizeof(int2) <= kBins * 4);       // two batches' rows, of at least two vectors
    const bool fused = parts == 1 && (fused_batches <= 3 || (items >= sm_count() * 3 / 2 && fused_batches <= 16) ||
                                      (items > sm_count() * 4 && smem <= 56 * 1024));
    if (fused) threads = fused_threads;
    const bool shared = parts > 1;
    while ((1 << a.select_shift) < parts) ++a.select_shift;
    while ((32 << a.warps_shift) < threads) ++a.warps_shift;
    void (*select)(EvictArgs) = shared ? select_kernel<true, false> : (fused ? select_kernel<false, true> : select_kernel<false, false>);
    cudaError_t (*allow)() = shared ? allow_shared_memory<select_kernel<true, false>>
                                    : (fused ? allow_shared_memory<select_kernel<false, true>> : allow_shared_memory<select_kernel<false, false>>);
    LLMS_CUDA_TRY(allow());
    LLMS_CUDA_TRY(launch_dependent_cluster(select, dim3(a.Hkv * parts, n_seqs, a.L), dim3(threads), smem, parts, st, a));
    if (fused) return LLMS_OK;

    const int fill_ctas = 2 * sm_count();         // in place, a slab is shared by a cluster until there are so many CTAs (see move_kernel)
    const int batch = kMoveThreads / (a.d / 8) * in_flight(false), most_batches = (most + batch - 1) / batch;
    void (*kernel)(EvictArgs);
    if (dst_table) {
        a.batches = 4;
        a.parts = (most_batches + a.batches - 1) / a.batches;
        kernel = move_kernel<false, false>;
    } else {
        a.parts = 1;
        while (a.parts < kMaxCluster && items * 2 * a.parts < fill_ctas && a.parts < most_batches) a.parts *= 2;
        kernel = a.parts > 1 ? move_kernel<true, true> : move_kernel<true, false>;
    }
    if ((int64_t)a.Hkv * 2 * a.parts > 0x7fffffff) return LLMS_ERR_UNSUPPORTED;
    a.by_parts = Divisor(a.parts);
    LLMS_CUDA_TRY(launch_dependent_cluster(kernel, dim3(a.Hkv * 2 * a.parts, n_seqs, a.L), dim3(kMoveThreads), 0, dst_table ? 1 : a.parts, st, a));
    return LLMS_OK;
}
