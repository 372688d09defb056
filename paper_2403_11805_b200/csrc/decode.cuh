// What the kernels that attend to a paged cache share: the batch's tiles and how they are handed out, online softmax, joining of
// partial results, weights.  decode.cu has the mathematics and the split.
#pragma once

#include <math.h>

#include <algorithm>

#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include "paged.cuh"
#include "tma.cuh"

namespace llms {

namespace cg = cooperative_groups;

constexpr int kTile = 16;                         // tokens per tile: the 16 side of an MMA
constexpr int kQuerySlots = 2;                    // items whose query rows a warp holds: the current one's, the next one's
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// Weights are taken against a reference that follows the running maximum in steps: it moves only when a logit exceeds it by more
// than kSlack (in units of log2), so most tiles need no maximum over the warp's lanes and no rescaling.
// For the product with V a weight goes into the MMA as kLift times its value, as a sum of two 16-bit values hi + lo.  hi is cut
// off a little below the weight, so that lo is not 0 (of weights above 2^-30 of the reference in fp16, of any that is not 0 in bf16):
// a value of V that is infinite then gives an infinity, not 0 * inf.  The lift (a power of two, taken back exactly at the end) keeps kLift * 2^kSlack in fp16's range.  hi + lo is off by less than
// 2^-20 (fp16) or 2^-15.6 (bf16) of the weight; one 16-bit value alone would add an error as large as the rounding of the
// output itself.  fp16's smallest step makes it 2^-31 of the reference at least: weights below 2^-11 of it have fewer bits, those
// below 2^-31 none (4000 of them together less than half a step of an fp16 output next to values of its size).
constexpr float kSlack = 8.0f, kLift = 64.0f;

struct DecodeArgs {
    const uint16_t *q, *k_new, *v_new;
    uint16_t *k, *v, *out;                        // K and V of the layer: base of KV head 0
    const int32_t *table, *lens;
    float *lse, *row_lse;                         // caller's (may be NULL), natural; workspace's, in units of log2
    const float *mass_in;
    float *mass_out;
    float *logits;                                // workspace: v of every (sequence, KV head, token, query head), for the masses
    float *part;                                  // workspace: two partial results per run (rows x (cols + 4): O, m, l): of the item
                                                  // that began before the run, of the one that goes on behind it
    int2 *span;                                   // workspace: per item the first and the last run that have tiles of it;
                                                  // (-1, 0): one run has them all
    int32_t *open;                                // workspace: per run the item that begins in it and goes on behind it, or -1
    int64_t q_stride, new_stride, stride_h, mass_stride;
    int table_stride, n_seqs, max_len, window, Hkv, Hq, group, d, chunk_len, n_slots;
    int blocks;                                   // blocks of query rows per KV head
    int piece_shift;                              // log2 of the tokens per TMA box: the largest power of two up to 16 that divides chunk_len
    Divisor by_chunk, by_blocks, by_per_seq, by_mass_x, by_hkv, by_group;
    int rows;                                     // query rows kept per partial result
    int runs, grid_runs, few_tiles;               // runs; runs at most (CTAs of the main kernel), which up to few_tiles tiles are cut into
    int q_bytes;                                  // of an item's query rows
    int whole_tile;                               // one TMA copy takes K and V of a tile
    int item_shift;                               // a cluster per item: log2 of its CTAs
    float scale_log2;
};

// A sequence's tokens as tiles: the first tile is the one that the window begins in.
struct SeqTiles {
    int len, first, tile0, n;                     // tokens; first token seen; its tile; tiles (0 for an empty or invalid row)
};
template <int TILE = kTile>
__device__ __forceinline__ SeqTiles seq_tiles(const DecodeArgs &a, int len)
{
    SeqTiles s;
    s.len = len < 0 || len > a.max_len ? 0 : len;
    s.first = a.window > 0 && s.len > a.window ? s.len - a.window : 0;
    s.tile0 = s.first / TILE;
    s.n = (s.len + TILE - 1) / TILE - s.tile0;
    return s;
}

// The runs that the batch's tiles are cut into: the first `longer` ones have a tile more than the others.
constexpr int kMinTiles = 2;                      // tiles that a run has at least (but for the last ones of a small batch)
struct Runs {
    int n, tiles, longer;
    __device__ __forceinline__ Runs(const DecodeArgs &a, int total)
    {
        n = max(1, min(total <= a.few_tiles ? a.grid_runs : a.runs, total / kMinTiles));
        tiles = (int)((unsigned)total / (unsigned)n);
        longer = total - n * tiles;
    }
    __device__ __forceinline__ int begin(int i) const { return i * tiles + min(i, longer); }
    __device__ __forceinline__ int of(int tile) const                         // the run that has a tile
    {
        const int border = longer * (tiles + 1);
        return tile < border ? (int)((unsigned)tile / (unsigned)(tiles + 1)) : longer + (int)((unsigned)(tile - border) / (unsigned)max(tiles, 1));
    }
};

// Wait for the phase of the given parity to complete, all lanes of a warp together; false when it did not within the limit.
__device__ __forceinline__ bool warp_wait(unsigned long long *bar, uint32_t parity)
{
    const uint32_t addr = smem_u32(bar);
    uint32_t done = 0;
    for (uint32_t i = 0; i < kSpinLimit; ++i) {
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.b32 %0, 1, 0, p;\n\t}"
                     : "=r"(done) : "r"(addr), "r"(parity) : "memory");
        if (done) break;
        if (i > 32) __nanosleep(64);
    }
    return __all_sync(0xffffffffu, done);
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, unsigned long long *bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 :: "r"(dst), "l"(src), "r"(bytes), "r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x)
{
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
template <bool BF>
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    if constexpr (BF)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// (lo, hi) as a pair of 16-bit values, lo in the low half; cut off towards zero or rounded to nearest
template <bool BF>
__device__ __forceinline__ uint32_t pack_cut(float lo, float hi)
{
    uint32_t r;
    if constexpr (BF) asm("cvt.rz.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rz.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
template <bool BF>
__device__ __forceinline__ uint32_t pack_round(float lo, float hi)
{
    uint32_t r;
    if constexpr (BF) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
template <bool BF>
__device__ __forceinline__ float2 unpack(uint32_t x)
{
    if constexpr (BF) return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
    const __half2 h = *reinterpret_cast<const __half2 *>(&x);
    return __half22float2(h);
}

// A channel of the output: its weighted sum times the inverse of the weights' sum.  A row of no weight at all is 0 even where a value is
// infinite or NaN, whose product with a weight of 0 has made the sum NaN.
__device__ __forceinline__ float channel(float acc, float inv) { return inv == 0.0f ? 0.0f : acc * inv; }

// Four channels of a finished row (16-bit values), and with the first ones the row's log-sum.
template <bool BF>
__device__ __forceinline__ void finish_row(const DecodeArgs &a, int64_t row, int c, const float (&acc)[4], float top, float sum)
{
    const float inv = sum == 0.0f ? 0.0f : (1.0f / kLift) / sum;
    if (c < a.d) {
        const uint2 x = make_uint2(pack_round<BF>(channel(acc[0], inv), channel(acc[1], inv)), pack_round<BF>(channel(acc[2], inv), channel(acc[3], inv)));
        *reinterpret_cast<uint2 *>(a.out + row * a.d + c) = x;
    }
    if (c == 0) {
        const float lg = sum == 0.0f ? -INFINITY : top + log2f(sum);
        a.row_lse[row] = lg;
        if (a.lse) a.lse[row] = lg * kLn2;
    }
}

template <int DB> struct DecodeCols {
    static constexpr int kCols = DB * 64;                     // channels, rounded up to whole blocks of 64
    static constexpr int kPitch = kCols + 4;                  // floats per row of a partial result: O, then m and l
};

constexpr int kItemWarps = 4;

// In a cluster, the first of n tiles that its warp number i takes.
template <int W>
__device__ __forceinline__ int part_begin(const DecodeArgs &a, int n, int i) { return (n * i) >> (a.item_shift + (W == 4 ? 2 : 0)); }

__device__ __forceinline__ void lse_add(float &top, float &sum, float m, float l)   // (top, sum) joined with (m, l)
{
    const float t = fmaxf(top, m), ref = t == -INFINITY ? 0.0f : t;
    sum = __fmaf_rn(sum, exp2_fast(top - ref), l * exp2_fast(m - ref));
    top = t;
}

// Rows without tokens: zeros, or NaN where the length is invalid.
template <bool BF>
__device__ __forceinline__ void fill_empty(const DecodeArgs &a, int64_t row, int rows, bool bad, int tid, int threads)
{
    const uint32_t x = bad ? (BF ? 0x7fc07fc0u : 0x7e007e00u) : 0u;
    uint4 *to = reinterpret_cast<uint4 *>(a.out + row * a.d);
#pragma unroll 1
    for (int i = tid; i < rows * (a.d / 8); i += threads) to[i] = make_uint4(x, x, x, x);
#pragma unroll 1
    for (int i = tid; i < rows; i += threads)
        if (a.lse) a.lse[row + i] = bad ? NAN : -INFINITY;
}

// The end of an item that a cluster has: the warps' pieces joined, each CTA taking an equal share of the row elements, and the
// weights of the warp's own tokens [16 w0, 16 w1).
template <bool BF, int DB, int NT>
__device__ __forceinline__ void join_item(const DecodeArgs &a, unsigned char *rings, int warp_bytes, int w0, int w1)
{
    using S = DecodeCols<DB>;
    constexpr int W = kItemWarps, kThreads = W * 32;
    __shared__ float s_factor[8 * NT * W], s_lse[W][8 * NT];
    __shared__ float2 s_joined[8 * NT];
    __shared__ int s_piece;
    cg::cluster_group cluster = cg::this_cluster();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int ctas = 1 << a.item_shift, part = blockIdx.x & (ctas - 1), item = blockIdx.x >> a.item_shift;
    const int per_seq = a.Hkv * a.blocks, b = a.by_per_seq(item), hb = item - b * per_seq, h = a.by_blocks(hb), row0 = (hb - h * a.blocks) * 8 * NT;
    const int have = min(a.rows, a.group - row0), len = __ldg(a.lens + b);
    const int64_t first_row = (int64_t)b * a.Hq + h * a.group + row0;
    const SeqTiles s = seq_tiles(a, len);
    if (s.n == 0) {
        if (part == 0) fill_empty<BF>(a, first_row, have, len != 0, tid, kThreads);
        return;
    }
    // the CTA's own pieces first, into the first live warp's place; then, through the cluster's shared memory, the CTAs' pieces
    auto local = [&](int w) { return reinterpret_cast<float *>(rings + w * warp_bytes); };
    const int mine0 = part * W;
    int first = 0;
    while (first < W && part_begin<W>(a, s.n, mine0 + first) == part_begin<W>(a, s.n, mine0 + first + 1)) ++first;
    __syncthreads();
    if (first < W - 1) {
#pragma unroll 1
        for (int e = tid; e < have * W; e += kThreads) {       // factor of every piece's row
            const int r = e / W, w = e - r * W;
            float top = -INFINITY, m = -INFINITY, sum = 0.0f;
#pragma unroll
            for (int i = 0; i < W; ++i) {
                if (part_begin<W>(a, s.n, mine0 + i) == part_begin<W>(a, s.n, mine0 + i + 1)) continue;
                const float2 ml = *reinterpret_cast<const float2 *>(local(i) + r * S::kPitch + S::kCols);
                lse_add(top, sum, ml.x, ml.y);
                if (i == w) m = ml.x;
            }
            s_factor[r * W + w] = exp2_fast(m - (top == -INFINITY ? 0.0f : top));
            if (w == 0) s_joined[r] = make_float2(top, sum);
        }
        __syncthreads();
#pragma unroll 1
        for (int e = tid; e < have * (S::kCols / 4); e += kThreads) {
            const int r = e / (S::kCols / 4), c = (e - r * (S::kCols / 4)) * 4;
            float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
            for (int i = 0; i < W; ++i) {
                if (part_begin<W>(a, s.n, mine0 + i) == part_begin<W>(a, s.n, mine0 + i + 1)) continue;
                const float f = s_factor[r * W + i];
                const float4 v = *reinterpret_cast<const float4 *>(local(i) + r * S::kPitch + c);
                acc.x = __fmaf_rn(f, v.x, acc.x);
                acc.y = __fmaf_rn(f, v.y, acc.y);
                acc.z = __fmaf_rn(f, v.z, acc.z);
                acc.w = __fmaf_rn(f, v.w, acc.w);
            }
            *reinterpret_cast<float4 *>(local(first) + r * S::kPitch + c) = acc;   // only this thread reads or writes these elements
        }
        __syncthreads();
        for (int r = tid; r < have; r += kThreads) *reinterpret_cast<float2 *>(local(first) + r * S::kPitch + S::kCols) = s_joined[r];
    }
    if (tid == 0) s_piece = first < W ? first * warp_bytes : -1;
    cluster.sync();
    int at_cta[8];                                            // where a CTA's piece lies, -1: it has none
#pragma unroll
    for (int i = 0; i < 8; ++i) at_cta[i] = i < ctas ? *cluster.map_shared_rank(&s_piece, i) : -1;
    auto piece = [&](int i) -> const float * { return reinterpret_cast<const float *>(cluster.map_shared_rank(rings, i) + at_cta[i]); };
    const int share = (a.rows * (S::kCols / 4)) >> a.item_shift;               // groups of four channels that this CTA joins
#pragma unroll 1
    for (int e = part * share + tid; e < (part + 1) * share; e += kThreads) {
        const int r = e / (S::kCols / 4), c = (e - r * (S::kCols / 4)) * 4;
        if (r >= have) continue;
        float2 ml[8];
        float4 v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            ml[i] = make_float2(-INFINITY, 0.0f);
            v[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (at_cta[i] >= 0) {
                ml[i] = *reinterpret_cast<const float2 *>(piece(i) + r * S::kPitch + S::kCols);
                v[i] = *reinterpret_cast<const float4 *>(piece(i) + r * S::kPitch + c);
            }
        }
        float top = -INFINITY, sum = 0.0f, acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < 8; ++i) top = fmaxf(top, ml[i].x);
        const float ref = top == -INFINITY ? 0.0f : top;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float w = exp2_fast(ml[i].x - ref);
            sum = __fmaf_rn(w, ml[i].y, sum);
            acc[0] = __fmaf_rn(w, v[i].x, acc[0]);
            acc[1] = __fmaf_rn(w, v[i].y, acc[1]);
            acc[2] = __fmaf_rn(w, v[i].z, acc[2]);
            acc[3] = __fmaf_rn(w, v[i].w, acc[3]);
        }
        finish_row<BF>(a, first_row + r, c, acc, top, sum);
    }
    if (a.mass_out) {                                         // (only where an item has all query heads of its KV head)
        for (int r = lane; r < have; r += 32) {
            float top = -INFINITY, sum = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (at_cta[i] >= 0) {
                    const float2 ml = *reinterpret_cast<const float2 *>(piece(i) + r * S::kPitch + S::kCols);
                    lse_add(top, sum, ml.x, ml.y);
                }
            s_lse[warp][r] = sum == 0.0f ? -INFINITY : top + log2f(sum);
        }
        __syncwarp();
        const int64_t at = (int64_t)b * a.Hkv + h;
        const float *v = a.logits + at * a.max_len * a.group, *in = a.mass_in ? a.mass_in + at * a.mass_stride : nullptr;
        float *out = a.mass_out + at * a.mass_stride;
        const int t1 = min(s.len, (s.tile0 + w1) * kTile);
        constexpr int kAtOnce = 4;                            // tokens of a lane whose loads are under way together
        auto put = [&](int t0, int end, int step, auto weight) {               // tokens t0, t0 + step, ...
#pragma unroll 1
            for (int t = t0; t < end; t += kAtOnce * step) {
                float w[kAtOnce];
#pragma unroll
                for (int i = 0; i < kAtOnce; ++i) {
                    const int u = t + i * step;
                    w[i] = u < end ? weight(u) : 0.0f;
                    if (in && u < end) w[i] = in[u] + w[i];
                }
#pragma unroll
                for (int i = 0; i < kAtOnce; ++i)
                    if (t + i * step < end) out[t + i * step] = w[i];
            }
        };
        auto one = [&](float x, int r) { return s_lse[warp][r] == -INFINITY ? 0.0f : exp2_fast(x - s_lse[warp][r]); };
        put(max(s.first, (s.tile0 + w0) * kTile) + lane, t1, 32, [&](int t) {
            const float *x = v + (int64_t)t * a.group;
            float w = 0.0f;
            if ((have & 3) == 0) {                            // (have is the group here)
                for (int r = 0; r < have; r += 4) {
                    const float4 y = *reinterpret_cast<const float4 *>(x + r);
                    w += (one(y.x, r) + one(y.y, r + 1)) + (one(y.z, r + 2) + one(y.w, r + 3));
                }
            } else {
                for (int r = 0; r < have; ++r) w += one(x[r], r);
            }
            return w;
        });
        if (in != out) put(part * kThreads + tid, s.first, ctas * kThreads, [&](int) { return 0.0f; });   // before the window
    }
    cluster.sync();                                           // nobody reads this CTA's pieces any more
}

// The tiles [w0, w1) of a warp, and a sequence at or before the first of them with the number of its first tile.
template <bool ITEM, int W>
__device__ __forceinline__ void find_tiles(const DecodeArgs &a, int warp, int lane, int &w0, int &w1, int &f_seq, int &f_base, int &total, SeqTiles &f_s)
{
    const int run = blockIdx.x, per_seq = a.Hkv * a.blocks;
    total = 0;
    if constexpr (ITEM) {
        // the item of the cluster, its tiles numbered from 0, and this warp's part of them
        const int item = run >> a.item_shift, me = (run & ((1 << a.item_shift) - 1)) * W + warp;
        f_seq = a.by_per_seq(item);
        f_s = seq_tiles(a, __ldg(a.lens + f_seq));
        f_base = -(item - f_seq * per_seq) * f_s.n;
        w0 = part_begin<W>(a, f_s.n, me);
        w1 = part_begin<W>(a, f_s.n, me + 1);
    } else {
        // tiles of the batch, and the sequence that this run begins in: a lane adds up neighbouring sequences
        const int each = (a.n_seqs + 31) / 32;
        int incl = 0;
        for (int b = lane * each; b < min(a.n_seqs, (lane + 1) * each); ++b) incl += seq_tiles(a, __ldg(a.lens + b)).n * per_seq;
        const int own = incl;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int up = __shfl_up_sync(0xffffffffu, incl, d);
            if (lane >= d) incl += up;
        }
        total = __shfl_sync(0xffffffffu, incl, 31);
        const Runs cut(a, total);
        w0 = run < cut.n ? cut.begin(run) : 0;
        w1 = run < cut.n ? cut.begin(run + 1) : 0;
        const int holder = max(0, __ffs(__ballot_sync(0xffffffffu, incl > w0)) - 1);
        f_seq = holder * each;
        f_base = __shfl_sync(0xffffffffu, incl - own, holder);
        f_s = seq_tiles(a, __ldg(a.lens + f_seq));
    }
}

// Items that span runs are joined, block (x, y) taking kJoinCols groups of four channels of the y-th part of item x (by_item) or of
// the item that is open at the end of run x, in SLICES over the runs that have pieces of it.  The other blocks: the weights
// of kMassTokens tokens per thread.
constexpr int kJoinCols = 16, kMassTokens = 2;
struct FinishArgs {
    int by_item, joins, join_y, cols, mass_x;
};

template <bool BF, int SLICES>
__global__ void __launch_bounds__(SLICES * kJoinCols) finish_kernel(const DecodeArgs a, const FinishArgs f)
{
    constexpr int kThreads = SLICES * kJoinCols;
    __shared__ float4 s_acc[kThreads];
    __shared__ float2 s_ml[SLICES];
    __shared__ float s_lse[64];
    grid_dependency_wait();
    grid_launch_dependents();
    const int per_seq = a.Hkv * a.blocks, pitch = f.cols + 4, block_rows = a.group > 8 ? 16 : 8;
    const int64_t stride = (int64_t)a.rows * pitch;
    if ((int)blockIdx.x < f.joins) {
        const int x = blockIdx.x / f.join_y, y = blockIdx.x - x * f.join_y;
        const int item = f.by_item ? x : a.open[x];
        if (item < 0) return;
        const int b = a.by_per_seq(item), hb = item - b * per_seq, h = a.by_blocks(hb), rb = hb - h * a.blocks;
        const int2 span = a.span[item];
        if (f.by_item && seq_tiles(a, __ldg(a.lens + b)).n == 0) return;   // its span was never written
        if (span.x < 0) return;
        const int slice = threadIdx.x / kJoinCols, e = y * kJoinCols + threadIdx.x % kJoinCols;
        const int r = e / (f.cols / 4), c = (e - r * (f.cols / 4)) * 4;     // one row per block: cols / 4 is a multiple of kJoinCols
        if (rb * block_rows + r >= a.group) return;
        float top = -INFINITY, sum = 0.0f, acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        const float *from = a.part + (int64_t)r * pitch;
#pragma unroll 4
        for (int i = span.x + slice; i <= span.y; i += SLICES) {
            // the first run's last piece, then the following runs' first ones
            const float *at = from + ((int64_t)i * 2 + (i == span.x)) * stride;
            const float2 ml = __ldcg(reinterpret_cast<const float2 *>(at + f.cols));
            const float4 v = __ldcg(reinterpret_cast<const float4 *>(at + c));
            const float t = fmaxf(top, ml.x), ref = t == -INFINITY ? 0.0f : t;
            const float keep = exp2_fast(top - ref), w = exp2_fast(ml.x - ref);
            top = t;
            sum = __fmaf_rn(sum, keep, w * ml.y);
            acc[0] = __fmaf_rn(acc[0], keep, w * v.x);
            acc[1] = __fmaf_rn(acc[1], keep, w * v.y);
            acc[2] = __fmaf_rn(acc[2], keep, w * v.z);
            acc[3] = __fmaf_rn(acc[3], keep, w * v.w);
        }
        s_acc[threadIdx.x] = make_float4(acc[0], acc[1], acc[2], acc[3]);
        if (threadIdx.x % kJoinCols == 0) s_ml[slice] = make_float2(top, sum);
        __syncthreads();
        if (slice) return;
        const int n = min(SLICES, span.y - span.x + 1);
        for (int i = 1; i < n; ++i) top = fmaxf(top, s_ml[i].x);
        const float ref = top == -INFINITY ? 0.0f : top;
        sum = acc[0] = acc[1] = acc[2] = acc[3] = 0.0f;
#pragma unroll 4
        for (int i = 0; i < n; ++i) {
            const float2 ml = s_ml[i];
            const float4 v = s_acc[i * kJoinCols + threadIdx.x];
            const float w = exp2_fast(ml.x - ref);
            sum = __fmaf_rn(w, ml.y, sum);
            acc[0] = __fmaf_rn(w, v.x, acc[0]);
            acc[1] = __fmaf_rn(w, v.y, acc[1]);
            acc[2] = __fmaf_rn(w, v.z, acc[2]);
            acc[3] = __fmaf_rn(w, v.w, acc[3]);
        }
        finish_row<BF>(a, (int64_t)b * a.Hq + h * a.group + rb * block_rows + r, c, acc, top, sum);
        return;
    }
    // weights: 2^(v - lse) over the query heads of the KV head
    const int x = blockIdx.x - f.joins;
    const int bh = a.by_mass_x(x), b = a.by_hkv(bh), h = bh - b * a.Hkv, t0 = (x - bh * f.mass_x) * kThreads * kMassTokens, len = __ldg(a.lens + b);
    if (len > a.max_len || t0 >= len) return;
    const int first = a.window > 0 && len > a.window ? len - a.window : 0;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t at = (int64_t)b * a.Hkv + h;
    const float *v = a.logits + at * a.max_len * a.group;
    float w[kMassTokens], before[kMassTokens];                // added once, at the end: one rounding at the size of the mass
    float4 early[kMassTokens];                                // the logits, where a token has four: asked for before the log-sums
    int t[kMassTokens];
    const bool four = a.group == 4;
#pragma unroll
    for (int j = 0; j < kMassTokens; ++j) {
        t[j] = t0 + j * kThreads + threadIdx.x;
        w[j] = 0.0f;
        before[j] = a.mass_in && t[j] < len ? a.mass_in[at * a.mass_stride + t[j]] : 0.0f;
        if (four && t[j] < len && t[j] >= first) early[j] = __ldcg(reinterpret_cast<const float4 *>(v) + t[j]);
    }
    for (int g0 = 0; g0 < a.group; g0 += 64) {
        const int n_g = min(64, a.group - g0);
        for (int g = warp; g < n_g; g += kThreads / 32) {
            const int rb = (g0 + g) / block_rows, r = g0 + g - rb * block_rows;
            const int2 span = a.span[b * per_seq + h * a.blocks + rb];
            float lse;
            if (span.x < 0) {
                lse = a.row_lse[at * a.group + g0 + g];
            } else {                                          // the joining blocks run at the same time: again from the pieces
                float top = -INFINITY, sum = 0.0f;
                const float *from = a.part + (int64_t)r * pitch + f.cols;
#pragma unroll 4
                for (int i = span.x + lane; i <= span.y; i += 32) {
                    const float2 ml = __ldcg(reinterpret_cast<const float2 *>(from + ((int64_t)i * 2 + (i == span.x)) * stride));
                    lse_add(top, sum, ml.x, ml.y);
                }
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const float m2 = __shfl_xor_sync(0xffffffffu, top, d), l2 = __shfl_xor_sync(0xffffffffu, sum, d);
                    lse_add(top, sum, m2, l2);
                }
                lse = sum == 0.0f ? -INFINITY : top + log2f(sum);
            }
            if (lane == 0) s_lse[g] = lse;
        }
        __syncthreads();
        auto weight = [&](float x, float lse) { return lse == -INFINITY ? 0.0f : exp2_fast(x - lse); };
        if (four) {
#pragma unroll
            for (int j = 0; j < kMassTokens; ++j)
                if (t[j] < len && t[j] >= first)
                    w[j] = (weight(early[j].x, s_lse[0]) + weight(early[j].y, s_lse[1])) + (weight(early[j].z, s_lse[2]) + weight(early[j].w, s_lse[3]));
        } else {
            for (int g = 0; g < n_g; ++g)
#pragma unroll
                for (int j = 0; j < kMassTokens; ++j)
                    if (t[j] < len && t[j] >= first) w[j] += weight(__ldcg(v + (int64_t)t[j] * a.group + g0 + g), s_lse[g]);
        }
        __syncthreads();
    }
#pragma unroll
    for (int j = 0; j < kMassTokens; ++j)
        if (t[j] < len) a.mass_out[at * a.mass_stride + t[j]] = before[j] + w[j];
}

template <bool BF>
int launch_finish(DecodeArgs &a, FinishArgs f, cudaStream_t st)
{
    // few items: a block per item and part of its row, the slices as many as its pieces call for; more items than runs: a block
    // per run, whose open item has pieces in few other runs
    const int n_items = a.n_seqs * a.Hkv * a.blocks, slices = a.grid_runs >= 128 * n_items ? 64 : (a.grid_runs >= 16 * n_items ? 16 : 4);
    f.by_item = n_items <= a.grid_runs;
    f.join_y = a.rows * (f.cols / 4) / kJoinCols;
    f.joins = std::min(n_items, a.grid_runs) * f.join_y;
    const int tokens = slices * kJoinCols * kMassTokens;
    f.mass_x = (a.max_len + tokens - 1) / tokens;
    a.by_mass_x = Divisor(f.mass_x);
    const dim3 grid(f.joins + (a.mass_out ? f.mass_x * a.Hkv * a.n_seqs : 0)), block(slices * kJoinCols);
    LLMS_CUDA_TRY(launch_dependent(slices == 64 ? finish_kernel<BF, 64> : (slices == 16 ? finish_kernel<BF, 16> : finish_kernel<BF, 4>),
                                   grid, block, 0, st, a, f));
    return LLMS_OK;
}

constexpr int kRounds = 4, kRunTiles = 16;
struct DecodeLayout {
    int blocks_of_64, mode, rows, blocks;
    int runs, grid_runs, few_tiles;
    uint64_t off_lse, off_span, off_open, off_part, off_logits, total;
};

// warps: per SM, as many as it takes to keep the memory busy
inline DecodeLayout decode_layout(const llms_kv_desc &d, int n_seqs, int max_len, bool with_mass, int warps, int tile = kTile)
{
    DecodeLayout t;
    const int group = d.n_q_heads / d.n_kv_heads;
    t.blocks_of_64 = (d.head_dim + 63) / 64;
    t.mode = group <= 4 ? 0 : (group <= 8 ? 1 : 2);
    t.rows = std::min(group, t.mode == 2 ? 16 : 8);
    t.blocks = (group + 15) / 16;
    t.off_lse = 0;
    // Runs: one for each of the warps that it takes to keep the memory busy (with more tiles on their way at once the memory gets
    // slower), or a small multiple of that where a run then still has kRunTiles tiles: the warps that get done early take
    // the next ones.  A batch of many items whose tiles come to less than six a run is cut finer (few items: their many
    // pieces would cost more in finish_kernel).  max_len is a bound; the device knows better (struct Runs)
    const uint64_t most_tiles = (uint64_t)n_seqs * d.n_kv_heads * t.blocks * (((uint64_t)max_len + tile - 1) / tile);
    const uint64_t room = (uint64_t)sm_count() * warps;
    const uint64_t rounds = std::min<uint64_t>(kRounds, std::max<uint64_t>(1, most_tiles / (room * kRunTiles)));
    const uint64_t finest = std::max<uint64_t>(1, most_tiles / kMinTiles);
    t.few_tiles = (int)(6 * room);
    t.runs = (int)std::min<uint64_t>(room * rounds, finest);
    const bool many_items = (uint64_t)n_seqs * d.n_kv_heads * t.blocks * 4 >= room;
    t.grid_runs = many_items ? (int)std::max<uint64_t>(t.runs, std::min<uint64_t>(2 * room, finest)) : t.runs;
    t.off_span = round_up((uint64_t)n_seqs * d.n_q_heads * 4, 256);
    t.off_open = t.off_span + round_up((uint64_t)n_seqs * d.n_kv_heads * t.blocks * 8, 256);
    t.off_part = t.off_open + round_up((uint64_t)t.grid_runs * 4, 256);
    t.off_logits = t.off_part + round_up((uint64_t)t.grid_runs * 2 * t.rows * (t.blocks_of_64 * 64 + 4) * 4, 256);
    t.total = t.off_logits + (with_mass ? round_up((uint64_t)n_seqs * d.n_q_heads * (uint64_t)max_len * 4, 256) : 0);
    return t;
}

// What follows from the shapes and from where the workspace's parts lie.
inline void set_decode_shape(DecodeArgs &a, const llms_kv_desc &d, const DecodeLayout &lay, uint8_t *ws, float scale)
{
    a.row_lse = reinterpret_cast<float *>(ws + lay.off_lse);
    a.span = reinterpret_cast<int2 *>(ws + lay.off_span);
    a.open = reinterpret_cast<int32_t *>(ws + lay.off_open);
    a.part = reinterpret_cast<float *>(ws + lay.off_part);
    a.Hkv = d.n_kv_heads; a.Hq = d.n_q_heads; a.group = a.Hq / a.Hkv; a.d = d.head_dim;
    a.chunk_len = d.chunk_len; a.n_slots = n_chunks(d);
    a.blocks = lay.blocks; a.rows = lay.rows;
    a.by_chunk = Divisor(a.chunk_len);
    a.by_blocks = Divisor(a.blocks);
    a.by_per_seq = Divisor(a.Hkv * a.blocks);
    a.by_hkv = Divisor(a.Hkv);
    a.by_group = Divisor(a.group);
    a.scale_log2 = scale * kLog2e;
    a.runs = lay.runs; a.grid_runs = lay.grid_runs; a.few_tiles = lay.few_tiles;
    a.q_bytes = a.rows * a.d * 2;
}

// CTAs of a cluster per item, or 0: runs.  As many CTAs as leave a warp one tile, up to eight and up to kItemRounds rounds of the
// GPU (per_sm: CTAs that an SM has room for); not if a warp is left with more than four tiles, in a batch (whose sequences are
// seldom all as long as max_len) eight.
constexpr int kItemRounds = 2;
inline int decode_item_ctas(const DecodeArgs &a, int per_sm, int rounds = kItemRounds, int tile = kTile, int warps = kItemWarps)
{
    if (a.mass_out && a.blocks > 1) return 0;                 // a token's weight is made of several items' logits
    const int seen = a.window > 0 ? (int)std::min<int64_t>(a.max_len, (int64_t)a.window + tile - 1) : a.max_len, tiles = (seen + tile - 1) / tile;
    const int64_t n_items = (int64_t)a.n_seqs * a.Hkv * a.blocks, room = (int64_t)sm_count() * per_sm * rounds;
    int ctas = 1;
    while (ctas < 8 && ctas * warps < tiles && n_items * ctas * 2 <= room) ctas *= 2;
    return n_items * ctas <= room && tiles <= ctas * warps * (a.n_seqs > 1 ? 8 : 4) ? ctas : 0;
}

}  // namespace llms
