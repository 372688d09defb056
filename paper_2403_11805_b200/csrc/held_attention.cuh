// Attention of one new token per sequence over a pool held at 8 or 4 bits, one layer per call: the kernel.
//
// Mathematics.  As for the fp16 pool (decode.cu), with K_t = z_t + s_t k_t and V_t = z'_t + s'_t v_t, k_t and v_t whole numbers below 2^bits,
// s and z the scale and zero-point of a token's group of channels.  Both products are taken on the codes:
//     <q, K_t> = sum over groups  s_t <q, k_t> + z_t sum q,        sum_t p_t V_t = sum_t (p_t s'_t) v_t + sum_t p_t z'_t.
// A code enters an fp16 MMA as it lies in its word: bits 0 .. 9 of an fp16 whose upper bits are 0 are a subnormal number, the code times
// 2^-24 (or 2^-20, four bits further up), exactly.  So a mask, for half of the codes a shift too, makes a pair of operands, the products
// are exact, and the powers of two are taken back in the sums.
//
// Bound.  A quarter (half) of the fp16 pool's bytes for the same arithmetic: at 4 bits and 128 channels an SM has some 80 cycles per 16
// tokens at the copy bandwidth, in which its four schedulers issue at most 320 instructions; 16 tokens take 250, half of
// them logical ones that hold their pipe for two cycles.  Large batches take the same time without their copies, with 55% of the
// issue slots and half of that pipe busy: the fixed latencies of a warp's chain of instructions bound them, at four warps per scheduler.
// The latencies of length, table, tile and join bound small calls.
//
// Split.  As for the fp16 pool: runs of tiles, one per warp, or a cluster per item for small calls.  A tile of the pool is one run of bytes,
// copied by a warp's own lanes (cp.async: a third of the instructions that one lane's bulk copies and their barriers took), and
// its codes lie in the order of the MMAs' operands, so that they go from shared memory into masks and MMAs.  The
// parts of a cluster's warps are stored into the shared memory of the CTA that joins them: one barrier, no reads across.
//
// Measured, a B200: 16 contexts of 4096 tokens, 32 heads of 128 channels at 4 bits 64 us (286 MB, 4.5 TB/s; 164 us in the fp16 pool); one
// grouped-query context of 32768 tokens 19.8 us; one context of 4096 tokens 10.3; one of 256 tokens, 4 heads of 64, 4.1.
// Warps per SM (us for 12, 16, 20, the last at 96 registers with spills): that batch 68, 64, 64; 64 contexts 226, 216, 220; 64
// contexts of 8 heads with four query rows 82, 78, 86.
#pragma once

#include "decode.cuh"
#include "held.cuh"

namespace llms {

struct HeldFeed {
    uint8_t *held;                                // of the layer
    int tiles, bf16, stage_bytes;                 // tiles per KV head; type of the rows; shared memory of a stage
};

// A kernel's tile is 32 tokens, two tiles of the pool: what a tile costs besides its arithmetic - waiting, asking for the next copies,
// looking for a larger maximum - then counts half.
constexpr int kHeldTile = 32;
// By a tile's bytes: warps per CTA of a cluster; warps per SM for runs, and stages of a warp's ring.  Many tiles: enough warps to keep
// the arithmetic busy, and copies one tile ahead.  Few tiles (DEEP; clusters too): each warp has few, and a trip through the
// loop is shorter than a copy's way, so that copies further ahead count more than warps.
__host__ __device__ constexpr int held_item_warps(uint64_t bytes) { return bytes <= 2304 ? 8 : 4; }
constexpr int kRunWarps = 4;                      // per CTA, for runs: each has its own, but the SM's four schedulers get equally many
__host__ __device__ constexpr int held_room(uint64_t bytes, bool deep) { return deep ? (bytes <= 4608 ? 8 : 4) : (bytes <= 2304 ? 16 : (bytes <= 4608 ? 12 : 4)); }
__host__ __device__ constexpr int held_stages(uint64_t bytes, bool deep) { return deep ? (bytes <= 2304 ? 4 : (bytes <= 4608 ? 3 : 2)) : 2; }
constexpr int kAhead = 16;                        // tiles that a warp looks up at once

// Shared memory of a warp: a ring of stages, each a tile and behind it the query rows of the item that begins with it, the newest token's
// rows of K and V if the tile has its place, and the tile of the pool that they go to.  In a cluster a CTA has behind its
// warps' rings the places that all warps of the cluster put their parts of its channels into.
inline int held_stage_bytes(uint64_t tile_bytes, int rows, int d) { return (int)((2 * tile_bytes + rows * d * 2 + d * 4 + 16 + 15) & ~15ull); }
inline size_t held_item_smem(uint64_t tile_bytes, int rows, int d, int ctas)
{
    const int warps = held_item_warps(tile_bytes);
    return (size_t)warps * held_stages(tile_bytes, true) * held_stage_bytes(tile_bytes, rows, d) + (size_t)ctas * warps * rows * (d / ctas + 2) * 4;
}
// Of the channels of an output row, N lie side by side in a lane; a CTA of a cluster has 1 / ctas of these groups.
template <typename S>
struct HeldParts {
    static constexpr int N = 16 / S::BITS, kGroups = S::D / N, kWarps = held_item_warps(S::kTileBytes);
};

// c += a b, or c = a b.  Not volatile: the compiler may move them, so that the two halves of a tile fill each other's gaps.
__device__ __forceinline__ void mma_add(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_set(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.0f));
}
__device__ __forceinline__ void copy16(uint32_t dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" :: "n"(N) : "memory"); }

template <int N>
__device__ __forceinline__ void lds(uint32_t (&x)[N], const void *p)
{
    if constexpr (N == 4) *reinterpret_cast<uint4 *>(x) = *reinterpret_cast<const uint4 *>(p);
    else if constexpr (N == 2) *reinterpret_cast<uint2 *>(x) = *reinterpret_cast<const uint2 *>(p);
    else x[0] = *reinterpret_cast<const uint32_t *>(p);
}

// The newest token's row of K or V, quantised by a warp: a lane has every 32nd word of codes.
template <typename S>
struct FreshRow {
    static constexpr int kWords = S::D * S::BITS / 32, kPer = (kWords + 31) / 32, kPairs = 16 / S::BITS;
    static constexpr int kGroupWords = kWords / S::GPR;
    uint32_t x[kPer][kPairs];                     // the row's channels; then a word of codes and the group's parameters
    __device__ __forceinline__ void load(const uint16_t *row, int lane)
    {
#pragma unroll
        for (int m = 0; m < kPer; ++m)
            if (lane + 32 * m < kWords) {
                const uint32_t *from = reinterpret_cast<const uint32_t *>(row) + (lane + 32 * m) * kPairs;
                if constexpr (kPairs == 4) *reinterpret_cast<uint4 *>(x[m]) = *reinterpret_cast<const uint4 *>(from);
                else *reinterpret_cast<uint2 *>(x[m]) = *reinterpret_cast<const uint2 *>(from);
            } else {
#pragma unroll
                for (int c = 0; c < kPairs; ++c) x[m][c] = 0u;
            }
    }
    __device__ __forceinline__ void quantise(bool bf16)
    {
        __half2 r[kPer];
#pragma unroll
        for (int m = 0; m < kPer; ++m) {
            GroupRange range;
#pragma unroll
            for (int c = 0; c < kPairs; ++c) {
                const __half2 v = bf16 ? to_half2<true>(x[m][c]) : to_half2<false>(x[m][c]);
                x[m][c] = half2_bits(v);
                range.add(v);
            }
            r[m] = range.own();
#pragma unroll
            for (int d = 1; d < (kGroupWords < 32 ? kGroupWords : 32); d <<= 1)
                r[m] = __hmin2_nan(r[m], as_half2(__shfl_xor_sync(0xffffffffu, half2_bits(r[m]), d)));
        }
        if constexpr (kGroupWords > 32)
#pragma unroll
            for (int m = 1; m < kPer; ++m) r[0] = r[m] = __hmin2_nan(r[0], r[m]);
#pragma unroll
        for (int m = 0; m < kPer; ++m) {
            GroupRule rule;
            rule.template set<S::kTop>(kGroupWords > 32 ? r[kPer - 1] : r[m]);
            uint32_t word = 0;
#pragma unroll
            for (int c = 0; c < kPairs; ++c) {
                const float2 v = __half22float2(as_half2(x[m][c]));
                word |= (__float_as_uint(rule.template stepped<S::kTop>(v.x)) & S::kTop) << (2 * c * S::BITS);
                word |= (__float_as_uint(rule.template stepped<S::kTop>(v.y)) & S::kTop) << ((2 * c + 1) * S::BITS);
            }
            x[m][0] = word;
            x[m][1] = rule.params;
        }
    }
    // to a tile's codes of K (half 0) or V and its parameters; t: place in the tile
    __device__ __forceinline__ void store(uint8_t *tile, int half, int t, int lane) const
    {
#pragma unroll
        for (int m = 0; m < kPer; ++m) {
            const int n = lane + 32 * m;
            if (n >= kWords) continue;
            if (half == 0) {
                reinterpret_cast<uint32_t *>(tile)[S::place(t >> 3, n >> 2, (t & 7) * 4 + (n & 3))] = x[m][0];
            } else {
                uint32_t *codes = reinterpret_cast<uint32_t *>(tile + S::kCodes);
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int unit = 2 * n + u;
                    reinterpret_cast<uint16_t *>(codes + S::place(t >> 3, unit >> 3, (unit & 7) * 4 + ((t & 7) >> 1)))[t & 1] = (uint16_t)(x[m][0] >> (16 * u));
                }
            }
            if (n % kGroupWords == 0) reinterpret_cast<uint32_t *>(tile + 2 * S::kCodes + half * S::kParams)[t * S::GPR + n / kGroupWords] = x[m][1];
        }
    }
};

__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t cluster_addr(const void *p, int rank)
{
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_u32(p)), "r"(rank));
    return r;
}
template <int N>
__device__ __forceinline__ void cluster_store(uint32_t addr, const float (&v)[N])
{
    if constexpr (N == 4) asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" :: "r"(addr), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]) : "memory");
    else asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" :: "r"(addr), "f"(v[0]), "f"(v[1]) : "memory");
}

// N channels of an output row.
template <int N>
__device__ __forceinline__ void store_channels(uint16_t *to, const float (&v)[N], float inv, bool bf16)
{
    uint32_t x[N / 2];
#pragma unroll
    for (int n = 0; n < N; n += 2)
        x[n / 2] = bf16 ? pack_round<true>(channel(v[n], inv), channel(v[n + 1], inv)) : pack_round<false>(channel(v[n], inv), channel(v[n + 1], inv));
    if constexpr (N == 4) *reinterpret_cast<uint2 *>(to) = make_uint2(x[0], x[1]);
    else *reinterpret_cast<uint32_t *>(to) = x[0];
}

// The newest token's rows of K and V (side by side in shared memory), quantised into a tile in shared memory and, unless `pool` is NULL,
// into the pool.
template <typename S>
__device__ __noinline__ void append_token(const uint16_t *rows, bool bf16, uint8_t *tile, uint8_t *pool, int t)
{
    const int lane = threadIdx.x & 31;
    FreshRow<S> row[2];
#pragma unroll
    for (int half = 0; half < 2; ++half) row[half].load(rows + half * S::D, lane);
#pragma unroll
    for (int half = 0; half < 2; ++half) row[half].quantise(bf16);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        row[half].store(tile, half, t, lane);
        if (pool) row[half].store(pool, half, t, lane);
    }
}

// The end of an item that a cluster has: its warps' parts of this CTA's channels, joined.  A group of channels has `lanes` lanes, each
// of which takes every lanes-th warp's part.
template <typename S>
__device__ __forceinline__ void join_parts(const DecodeArgs &a, bool bf16, const float *parts, int seq, int row0, int h, int have, int live)
{
    constexpr int N = HeldParts<S>::N, kWarps = HeldParts<S>::kWarps, kThreads = kWarps * 32;
    const int ctas = 1 << a.item_shift, each = HeldParts<S>::kGroups >> a.item_shift, warps = ctas * kWarps, groups = have * each;
    const float2 *const ml = reinterpret_cast<const float2 *>(parts + (size_t)warps * a.rows * each * N);
    int lanes = 1;
    while (lanes < 32 && lanes < live && groups * lanes * 2 <= kThreads) lanes *= 2;
    const int me = threadIdx.x & (lanes - 1);
#pragma unroll 1
    for (int e = threadIdx.x / lanes; e - (int)(threadIdx.x / lanes) < groups; e += kThreads / lanes) {     // all lanes of a warp take part
        const int r = min(e, groups - 1) / each, c = min(e, groups - 1) - r * each;
        float top = -INFINITY, sum = 0.0f, acc[N];
#pragma unroll
        for (int n = 0; n < N; ++n) acc[n] = 0.0f;
        for (int p = me; p < live; p += lanes) top = fmaxf(top, ml[p * a.rows + r].x);
        for (int d = 1; d < lanes; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
        const float ref = top == -INFINITY ? 0.0f : top;
#pragma unroll 1
        for (int p = me; p < live; p += lanes) {
            const float2 x = ml[p * a.rows + r];
            float v[N];
            lds(reinterpret_cast<uint32_t (&)[N]>(v), parts + ((size_t)(p * a.rows + r) * each + c) * N);
            const float w = exp2_fast(x.x - ref);
            sum = __fmaf_rn(w, x.y, sum);
#pragma unroll
            for (int n = 0; n < N; ++n) acc[n] = __fmaf_rn(w, v[n], acc[n]);
        }
#pragma unroll 1
        for (int d = 1; d < lanes; d <<= 1) {
            sum += __shfl_xor_sync(0xffffffffu, sum, d);
#pragma unroll
            for (int n = 0; n < N; ++n) acc[n] += __shfl_xor_sync(0xffffffffu, acc[n], d);
        }
        if (me || e >= groups) continue;
        const int64_t row = (int64_t)seq * a.Hq + h * a.group + row0 + r;
        const int group = cluster_rank() * each + c;
        store_channels(a.out + row * S::D + group * N, acc, sum == 0.0f ? 0.0f : (1.0f / kLift) / sum, bf16);
        if (group == 0 && a.lse) a.lse[row] = sum == 0.0f ? -INFINITY : (top + log2f(sum)) * kLn2;
    }
}

// How the batch is cut into runs: into equal numbers of slots.  An item has a slot per tile and kItemSlots in front of them for what it costs
// to begin and end one (query rows, first maxima, the newest token, results: about as much as five tiles), so that a run through
// many short items is not the one that all wait for.
constexpr int kItemSlots = 5;
struct HeldCut {
    int w0, w1;                                   // the run's tiles, in the batch's numbering
    int seq = 0, base = 0, slot = 0;              // the sequence of the first one, the numbers of its first tile and of its first slot
    int total;                                    // slots
    SeqTiles s{};                                 // (a run behind the last slot has no tiles, and none of these)
    __device__ __forceinline__ HeldCut(const DecodeArgs &a, int run, int lane)
    {
        const int per_seq = a.Hkv * a.blocks, each = (a.n_seqs + 31) / 32;
        int tiles = 0, items = 0;                 // of this lane's sequences; then with those of the lanes before
#pragma unroll 1
        for (int b = lane * each; b < min(a.n_seqs, (lane + 1) * each); ++b) {
            const int n = seq_tiles<kHeldTile>(a, __ldg(a.lens + b)).n;
            tiles += n * per_seq;
            items += n ? per_seq : 0;
        }
        const int own_tiles = tiles, own_items = items;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int t = __shfl_up_sync(0xffffffffu, tiles, d), i = __shfl_up_sync(0xffffffffu, items, d);
            if (lane >= d) {
                tiles += t;
                items += i;
            }
        }
        const int all_tiles = __shfl_sync(0xffffffffu, tiles, 31), slots = tiles + items * kItemSlots;
        total = __shfl_sync(0xffffffffu, slots, 31);
        const Runs cut(a, total);
        w0 = w1 = 0;
#pragma unroll 1
        for (int end = 1; end >= 0; --end) {      // where the run ends, then where it begins
            const int at = run < cut.n ? cut.begin(run + end) : total;
            if (at >= total) {
                w0 = all_tiles;
            } else {
                const int holder = __ffs(__ballot_sync(0xffffffffu, slots > at)) - 1;
                seq = holder * each;
                base = __shfl_sync(0xffffffffu, tiles - own_tiles, holder);
                slot = __shfl_sync(0xffffffffu, slots - own_tiles - own_items * kItemSlots, holder);
                for (;;) {
                    s = seq_tiles<kHeldTile>(a, __ldg(a.lens + seq));
                    if (s.n && slot + per_seq * (s.n + kItemSlots) > at) break;
                    base += per_seq * s.n;
                    slot += s.n ? per_seq * (s.n + kItemSlots) : 0;
                    ++seq;
                }
                const int hb = (int)((unsigned)(at - slot) / (unsigned)(s.n + kItemSlots));
                w0 = base + hb * s.n + max(0, at - slot - hb * (s.n + kItemSlots) - kItemSlots);
            }
            if (end) w1 = w0;
        }
    }
};

// What a warp needs at the borders of items only, in shared memory: the registers are for the loop.
struct HeldPlace {
    int seq, hb, first_tile, first_idx, len, first, tile0, n, slot;       // of the item at hand: its tile first_tile is the run's tile first_idx
    int f_seq, f_base, f_len, f_first, f_tile0, f_n;                      // of the look-ups
};

// MODE: up to 4, 8 or 16 query rows (see decode_kernel), or 3: one.  One row stands in all eight columns of the MMAs, of which a lane then
// needs one instead of two: half the arithmetic on logits and weights.
template <typename S, int MODE, bool ITEM, bool DEEP, int kMinCtas>
__global__ void __launch_bounds__((ITEM ? HeldParts<S>::kWarps : kRunWarps) * 32, kMinCtas) held_attention_kernel(const DecodeArgs a, const HeldFeed f)
{
    constexpr int NT = MODE == 2 ? 2 : 1;                     // column groups of eight query rows
    constexpr bool kTwin = MODE == 0 || MODE == 3;
    constexpr int NC = MODE == 3 ? 1 : 2;                     // query rows of a lane's columns
    constexpr int kStages = held_stages(S::kTileBytes, DEEP);
    constexpr int kCols = DecodeCols<(S::D + 63) / 64>::kCols, kPitch = DecodeCols<(S::D + 63) / 64>::kPitch;
    constexpr int MT = S::D / 16, GPR = S::GPR;               // 16-channel tiles of the output; groups per row
    constexpr bool k4 = S::BITS == 4;
    // Codes of 4 bits are moved up by two places: an MMA keeps its sums to 24 bits or so below the operands' exponents, and a subnormal
    // operand's exponent is that of its top place, however few of the ten places it fills (moved up, results come four times nearer)
    constexpr uint32_t kLow = k4 ? 0x003c003cu : 0x00ff00ffu, kHigh = 0x03c003c0u;
    constexpr int kUp = k4 ? 2 : 0, kDown = 8 - kUp;
    constexpr float kUnit = k4 ? 0x1p22f : 0x1p24f, kMiddle = (float)S::kTop / 2;             // (in the high places 16 times the low ones')
    constexpr int W = ITEM ? HeldParts<S>::kWarps : kRunWarps, N = HeldParts<S>::N;
    extern __shared__ __align__(128) unsigned char smem_held[];
    __shared__ int4 s_feed[W][kAhead];                        // tiles looked up: the two tiles of the pool; sequence; query rows, first
                                                              // query row << 8, 64 or 32: the newest token's row goes into
                                                              // the first, second half, 128: a half lies outside the pool
    __shared__ HeldPlace s_place[W];
    const int lane = threadIdx.x & 31, warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), run = ITEM ? blockIdx.x : blockIdx.x * W + warp, g = lane >> 2, j = lane & 3;
    unsigned char *const ring = smem_held + warp * kStages * f.stage_bytes;
    if constexpr (ITEM) cluster_arrive();                     // this CTA has begun: the others may store into its shared memory
    grid_dependency_wait();
    grid_launch_dependents();

    // tiles of this warp: [w0, w1) of the batch's, or every step-th of the cluster's item, numbered 0 .. w1 - 1
    const int per_seq = a.Hkv * a.blocks;
    int w0, w1, f_seq, f_base, total = 0, me = 0;             // (a sequence, and its first tile)
    constexpr int kWarpShift = W == 8 ? 3 : 2;
    const int step_shift = ITEM ? a.item_shift + kWarpShift : 0, step = 1 << step_shift;
    SeqTiles f_s;
    int early_slot = -1;                                      // in a cluster, where the first tiles do not hang on the length
    int c_seq, c_hb, c_tile, c_slot = 0;                      // where the arithmetic is (c_slot: of the sequence)
    if constexpr (ITEM) {
        const int item = run >> a.item_shift;
        me = cluster_rank() * W + warp;
        f_seq = a.by_per_seq(item);
        f_base = item - f_seq * per_seq;                      // the item in its sequence
        const int tok = (me + (lane >> 1) * step) * kHeldTile + (lane & 1) * 16;
        if (a.window == 0 && tok < a.max_len) early_slot = __ldg(a.table + (int64_t)f_seq * a.table_stride + a.by_chunk(tok));
        f_s = seq_tiles<kHeldTile>(a, __ldg(a.lens + f_seq));
        w0 = 0;
        w1 = max(0, f_s.n - me + step - 1) >> step_shift;
        c_hb = f_base;
        c_tile = me;
    } else {
        if (run >= a.runs) return;
        const HeldCut cut(a, run, lane);
        w0 = cut.w0, w1 = cut.w1, f_seq = cut.seq, f_base = cut.base, f_s = cut.s, c_slot = cut.slot, total = cut.total;
        c_hb = w0 < w1 ? (int)((unsigned)(w0 - f_base) / (unsigned)f_s.n) : 0;
        c_tile = w0 - f_base - c_hb * f_s.n;
    }
    HeldPlace &place = s_place[warp];
    place.seq = place.f_seq = c_seq = f_seq;                  // (every lane writes the same)
    place.hb = c_hb;
    place.first_tile = c_tile;
    place.first_idx = w0;
    place.len = place.f_len = f_s.len;
    place.first = place.f_first = f_s.first;
    place.tile0 = place.f_tile0 = f_s.tile0;
    place.n = place.f_n = f_s.n;
    place.slot = c_slot;
    place.f_base = f_base;
    __syncwarp();
    int open_item = -1;                                       // the item that begins in this run and goes on behind it

    if (w0 < w1) {
        // ---- feeding: lane i looks up half i % 2 of the tile i / 2 behind `base`
        auto look_up = [&](int base) {
            const int idx = base + (lane >> 1), last = min(base + kAhead, w1) - 1;
            int f_seq = place.f_seq, f_base = place.f_base;
            SeqTiles f_s{place.f_len, place.f_first, place.f_tile0, place.f_n};
            int x = 0, seq = 0, what = 0;                     // (halves that nobody sees or outside the pool: any tile of it will do)
            auto entry = [&](int hb, int tile, bool with_q, bool early) {
                const int tok = (f_s.tile0 + tile) * kHeldTile + (lane & 1) * 16;
                const int h = a.by_blocks(hb), r0 = (hb - h * a.blocks) * 8 * NT, chunk = a.by_chunk(tok);
                if (tok < f_s.len && tok + 16 > f_s.first) {
                    const int slot = early ? early_slot : __ldg(a.table + (int64_t)f_seq * a.table_stride + chunk);
                    const bool inside = (unsigned)slot < (unsigned)a.n_slots;
                    x = inside ? h * f.tiles + slot * (a.chunk_len >> 4) + ((tok - chunk * a.chunk_len) >> 4) : -1;
                    what = inside ? 0 : 128;
                    if (a.k_new && tok + 16 >= f_s.len) what |= lane & 1 ? 32 : 64;
                }
                seq = f_seq;
                what |= (h * a.group + r0) << 8;
                if (with_q) what |= min(a.rows, a.group - r0);
            };
            if constexpr (ITEM) {
                if (idx <= last) entry(f_base, me + idx * step, idx == 0, a.window == 0 && base == 0);
            } else {
                for (;;) {
                    if (idx >= f_base && idx <= last && idx < f_base + f_s.n * per_seq) {
                        const int hb = (int)((unsigned)(idx - f_base) / (unsigned)f_s.n), tile = idx - f_base - hb * f_s.n;
                        entry(hb, tile, idx == w0 || tile == 0, false);
                    }
                    if (last < f_base + f_s.n * per_seq) break;
                    f_base += f_s.n * per_seq;                // on to the next sequence
                    f_s = seq_tiles<kHeldTile>(a, __ldg(a.lens + ++f_seq));
                }
                __syncwarp();
                place.f_seq = f_seq;
                place.f_base = f_base;
                place.f_len = f_s.len;
                place.f_first = f_s.first;
                place.f_tile0 = f_s.tile0;
                place.f_n = f_s.n;
            }
            const int x1 = __shfl_down_sync(0xffffffffu, x, 1), other = __shfl_down_sync(0xffffffffu, what, 1) & (128 | 32);
            __syncwarp();
            if ((lane & 1) == 0) s_feed[warp][lane >> 1] = make_int4(x, x1, seq, what | other);
            __syncwarp();
        };
        constexpr int kVectors = S::kTileBytes / 16;
        const uint32_t lane_addr = smem_u32(ring) + lane * 16;
        const uint8_t *const lane_held = f.held + lane * 16;
        const int ring_bytes = kStages * f.stage_bytes, fresh_at = 2 * S::kTileBytes + a.rows * S::D * 2;
        int next = w0, in = 0, at = 0;                        // the next tile to ask for; offsets of its stage and of the current one's
        uint32_t poisoned = 0;                                // bit i: a half of the i-th tile from here lies outside the pool

        // ---- the arithmetic's state
        uint32_t qf[NT][S::W][k4 ? 4 : 2];
        float o[NT][MT][4], ref[NT][NC], limit[NT][NC], l[NT][NC], zero_sum[NT][GPR][NC], w_sum[NT][GPR][NC], fac[NT][NC], q_sum[NT][GPR][NC];
        float lift = 1.0f, scale_limit = -1.0f;               // what V's scales are multiplied with; the largest one that this suits
        int left = 0, odd_first = 0, odd_last = 0;            // tiles of the item in this run; what `left` is at its first and last tile if
                                                              // those may hold places nobody sees or the newest token (else -1)
        const float middle = kTwin && (lane & 2) ? 0.0f : -kMiddle / kUnit;                // of the columns of whole weights
        bool begins = true, started = false;                  // the item's first tile here is next; the item has had a tile

        // a group of copies per trip (an empty one behind the last tile); the first trips only ask
#pragma unroll 1
        for (int idx = w0 - (kStages - 1); idx < w1; ++idx) {
            if (next < w1) {
                const int n = (next - w0) & (kAhead - 1);
                if (n == 0) look_up(next);
                const int4 feed = s_feed[warp][n];
#pragma unroll
                for (int u = 0; u < 2; ++u) {                 // every lane copies every 32nd vector
                    const uint8_t *from = lane_held + (int64_t)max(u ? feed.y : feed.x, 0) * S::kTileBytes;
                    const uint32_t to = lane_addr + in + u * S::kTileBytes;
#pragma unroll
                    for (int i = 0; i < kVectors / 32; ++i) copy16(to + i * 512, from + i * 512);
                    if (kVectors % 32 && lane < kVectors % 32) copy16(to + kVectors / 32 * 512, from + kVectors / 32 * 512);
                }
                if (feed.w & 128) poisoned |= 1u << (kStages - 1);
                if (feed.w & 31) {
                    const uint16_t *from = a.q + feed.z * a.q_stride + (int64_t)(feed.w >> 8) * S::D;
#pragma unroll 1
                    for (int c = lane; c < (feed.w & 31) * (S::D / 8); c += 32) copy16(lane_addr + in + 2 * S::kTileBytes + (c - lane) * 16, from + c * 8);
                }
                if (feed.w & (64 | 32)) {                     // the newest token's rows of K and V, and where they go (-1: nowhere)
                    const int64_t row = feed.z * a.new_stride + (int64_t)a.by_group(feed.w >> 8) * S::D;
#pragma unroll 1
                    for (int c = lane; c < S::D / 4; c += 32)
                        copy16(lane_addr + in + fresh_at + (c - lane) * 16, (c < S::D / 8 ? a.k_new + c * 8 : a.v_new + (c - S::D / 8) * 8) + row);
                    if (lane == 0) *reinterpret_cast<int *>(ring + in + fresh_at + S::D * 4) = feed.w & 32 ? feed.y : feed.x;
                }
                ++next;
                in = in + f.stage_bytes == ring_bytes ? 0 : in + f.stage_bytes;
            }
            copies_commit();
            if (idx < w0) {
                poisoned >>= 1;
                continue;
            }
            copies_wait<kStages - 1>();
            __syncwarp();
            unsigned char *const mem = ring + at;
            if (begins) {
                const int c_hb = place.hb, row0 = (c_hb - a.by_blocks(c_hb) * a.blocks) * 8 * NT, have = min(a.rows, a.group - row0);
                // query rows as the MMA's second operand, channels in the order that K's codes come in; columns beyond the item's rows
                // repeat others (nobody reads their results).  bfloat16 rows become fp16 times a power of two, exactly but for
                // values below 2^-29 of the row's largest.  fac: what a logit in these units is multiplied with; q_sum: sum q per
                // group, a product with ones
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const int r = nt * 8 + (g & (kTwin ? 3 : 7));
                    const unsigned char *row = mem + 2 * S::kTileBytes + min(r, have - 1) * S::D * 2;
                    uint32_t x[S::W][k4 ? 4 : 2];
#pragma unroll
                    for (int w = 0; w < S::W; ++w) lds(x[w], row + (4 * w + j) * (k4 ? 16 : 8));
#pragma unroll
                    for (int i = 0; i < NC; ++i) fac[nt][i] = a.scale_log2;
                    if (f.bf16) {
                        uint32_t most = 0;
#pragma unroll
                        for (int w = 0; w < S::W; ++w)
#pragma unroll
                            for (int c = 0; c < (k4 ? 4 : 2); ++c) most = __vmaxu2(most, x[w][c] & 0x7fff7fffu);
                        most = max(most & 0xffffu, most >> 16);
                        most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
                        most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
                        // the largest value comes to lie in [2^14, 2^15) (an infinity or a NaN stays one)
                        const int shift = min(14 + 127 - min((int)(most >> 7), 254), 126);
                        const float up = __uint_as_float((uint32_t)(127 + shift) << 23), down = __uint_as_float((uint32_t)(127 - shift) << 23);
#pragma unroll
                        for (int w = 0; w < S::W; ++w)
#pragma unroll
                            for (int c = 0; c < (k4 ? 4 : 2); ++c) {
                                const float2 v = unpack<true>(x[w][c]);
                                x[w][c] = pack_round<false>(v.x * up, v.y * up);
                            }
#pragma unroll
                        for (int i = 0; i < NC; ++i) fac[nt][i] *= __shfl_sync(0xffffffffu, down, (2 * j + i) * 4);   // from a lane that has row 2 j + i
                    }
#pragma unroll
                    for (int grp = 0; grp < GPR; ++grp) {
                        float sums[4];
#pragma unroll
                        for (int w = grp * S::kGroupWords; w < (grp + 1) * S::kGroupWords; ++w) {
                            const uint32_t ones[4] = {0x3c003c00u, 0x3c003c00u, 0x3c003c00u, 0x3c003c00u};
                            if (w == grp * S::kGroupWords) mma_set(sums, ones, x[w][0], x[w][1]);
                            else mma_add(sums, ones, x[w][0], x[w][1]);
                            if constexpr (k4) mma_add(sums, ones, x[w][2], x[w][3]);
                        }
#pragma unroll
                        for (int i = 0; i < NC; ++i) {
                            q_sum[nt][grp][i] = sums[i];
                            zero_sum[nt][grp][i] = w_sum[nt][grp][i] = 0.0f;
                            if (!isfinite(sums[i])) fac[nt][i] = NAN;
                        }
                    }
#pragma unroll
                    for (int w = 0; w < S::W; ++w) {
                        if constexpr (k4) {
                            qf[nt][w][0] = __byte_perm(x[w][0], x[w][2], 0x5410);     // channels 0, 4; 2, 6; 1, 5; 3, 7 of a word
                            qf[nt][w][1] = __byte_perm(x[w][1], x[w][3], 0x5410);
                            qf[nt][w][2] = __byte_perm(x[w][0], x[w][2], 0x7632);
                            qf[nt][w][3] = __byte_perm(x[w][1], x[w][3], 0x7632);
                        } else {
                            qf[nt][w][0] = __byte_perm(x[w][0], x[w][1], 0x5410);     // channels 0, 2; 1, 3
                            qf[nt][w][1] = __byte_perm(x[w][0], x[w][1], 0x7632);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < NC; ++i) {
                        ref[nt][i] = l[nt][i] = 0.0f;
                        limit[nt][i] = -INFINITY;             // reference + kSlack; -inf: no logit yet
                    }
#pragma unroll
                    for (int t = 0; t < MT; ++t)
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[nt][t][i] = 0.0f;
                }
                lift = 1.0f;
                scale_limit = -1.0f;
                left = ITEM ? w1 : min(place.n - place.first_tile, w1 - idx);
                const int behind = ITEM ? (place.n - 1 - me) & (step - 1) : place.n - place.first_tile - left;   // 0: the item's last tile is this warp's
                odd_first = place.first_tile == 0 && place.first % kHeldTile ? left : -1;
                odd_last = behind == 0 && (a.k_new || place.len % kHeldTile) ? 1 : -1;
                begins = started = false;
            }
            // a tile that holds places nobody sees, the newest token, or a slot outside the pool
            const bool poison = poisoned & 1, special = poison || left == odd_last || left == odd_first;
            int tok0 = 0;
            if (special) {
                // parameters of rows that are not seen are cleared: whatever codes lie there are 0 then.  The newest token's row: what the
                // caller gave, here and in the pool
                tok0 = (place.tile0 + place.first_tile + (idx - place.first_idx) * step) * kHeldTile;
                if (tok0 + lane < place.first || tok0 + lane >= place.len)
#pragma unroll
                    for (int n = 0; n < 2 * GPR; ++n)
                        reinterpret_cast<uint32_t *>(mem + (lane >> 4) * S::kTileBytes + 2 * S::kCodes + n / GPR * S::kParams)[(lane & 15) * GPR + n % GPR] = 0u;
                if (a.k_new && tok0 + kHeldTile >= place.len) {
                    const int t = place.len - 1 - tok0, to = *reinterpret_cast<const int *>(mem + fresh_at + S::D * 4);
                    const bool store = (unsigned)to < (unsigned)(a.Hkv * f.tiles) && place.hb == a.by_blocks(place.hb) * a.blocks;
                    append_token<S>(reinterpret_cast<const uint16_t *>(mem + fresh_at), f.bf16, mem + (t >> 4) * S::kTileBytes,
                                    store ? f.held + (int64_t)to * S::kTileBytes : nullptr, t & 15);
                }
                __syncwarp();
            }

            // logits: tokens x query rows, for each half of the tile
            float s[2][NT][2 * NC];
            bool over = false;
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint32_t *const codes = reinterpret_cast<const uint32_t *>(mem + u * S::kTileBytes);
                const __half2 *const rule = reinterpret_cast<const __half2 *>(mem + u * S::kTileBytes + 2 * S::kCodes);
#pragma unroll
                for (int grp = 0; grp < GPR; ++grp) {
                    float c0[NT][4], c1[NT][4];               // 4 bits: codes of low and of high places; 8 bits: two chains
                    constexpr int VW = S::VW < S::kGroupWords ? S::VW : S::kGroupWords;
#pragma unroll
                    for (int v = 0; v < S::kGroupWords; v += VW) {
                        uint32_t x0[VW], x1[VW];              // words of tokens g and 8 + g
                        lds(x0, codes + S::place(0, grp * S::kGroupWords + v, lane));
                        lds(x1, codes + S::place(1, grp * S::kGroupWords + v, lane));
#pragma unroll
                        for (int n = 0; n < VW; ++n) {
                            const int w = grp * S::kGroupWords + v + n;
                            const uint32_t z0 = x0[n] << kUp, z1 = x1[n] << kUp, y0 = x0[n] >> kDown, y1 = x1[n] >> kDown;
                            const uint32_t low[4] = {z0 & kLow, z1 & kLow, y0 & kLow, y1 & kLow};
                            const uint32_t high[4] = {z0 & kHigh, z1 & kHigh, y0 & kHigh, y1 & kHigh};
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) {
                                float (&c)[4] = k4 || (v + n) % 2 == 0 ? c0[nt] : c1[nt];
                                if (v + n < (k4 ? 1 : 2)) mma_set(c, low, qf[nt][w][0], qf[nt][w][1]);
                                else mma_add(c, low, qf[nt][w][0], qf[nt][w][1]);
                                if constexpr (k4) {
                                    if (v + n == 0) mma_set(c1[nt], high, qf[nt][w][2], qf[nt][w][3]);
                                    else mma_add(c1[nt], high, qf[nt][w][2], qf[nt][w][3]);
                                }
                            }
                        }
                    }
                    const float2 r0 = __half22float2(rule[g * GPR + grp]), r1 = __half22float2(rule[(8 + g) * GPR + grp]);
                    const float m0 = r0.x * (k4 ? kUnit / 16 : kUnit), m1 = r1.x * (k4 ? kUnit / 16 : kUnit);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int i = 0; i < 2 * NC; ++i) {
                            const int hh = i / NC, n = 2 * hh + i % NC;          // token g or 8 + g; the fragment's register
                            const float c = k4 ? __fmaf_rn(c0[nt][n], 16.0f, c1[nt][n]) : c0[nt][n] + c1[nt][n];
                            const float v = __fmaf_rn(c, hh ? m1 : m0, (hh ? r1.y : r0.y) * q_sum[nt][grp][i % NC]);
                            s[u][nt][i] = grp == 0 ? v : s[u][nt][i] + v;
                        }
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 2 * NC; ++i) s[u][nt][i] *= fac[nt][i % NC];
            }
            if (special) {
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int i = 0; i < 2 * NC; ++i) {
                            const int t = tok0 + u * 16 + g + i / NC * 8;
                            if (poison) s[u][nt][i] = NAN;
                            if (t < place.first || t >= place.len) s[u][nt][i] = -INFINITY;
                        }
            }
            float2 v_rule[2][GPR][2];                         // V's scales and the values of the middle code, of this lane's tokens
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const __half2 *const rule = reinterpret_cast<const __half2 *>(mem + u * S::kTileBytes + 2 * S::kCodes + S::kParams);
#pragma unroll
                for (int grp = 0; grp < GPR; ++grp)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        v_rule[u][grp][i] = __half22float2(rule[(8 * i + g) * GPR + grp]);
                        v_rule[u][grp][i].y = __fmaf_rn(v_rule[u][grp][i].x, kMiddle, v_rule[u][grp][i].y);
                        over |= v_rule[u][grp][i].x > scale_limit;
                    }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 2 * NC; ++i) over |= s[u][nt][i] > limit[nt][i % NC];
            }
            if (__any_sync(0xffffffffu, over)) {              // the references move up to the maxima
                float keep[NT][NC], change = 1.0f;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < NC; ++i) {
                        float top = fmaxf(fmaxf(s[0][nt][i], s[0][nt][i + NC]), fmaxf(s[1][nt][i], s[1][nt][i + NC]));
#pragma unroll
                        for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                        keep[nt][i] = 1.0f;
                        if (top > limit[nt][i] - kSlack) {
                            keep[nt][i] = limit[nt][i] == -INFINITY ? 0.0f : exp2_fast(ref[nt][i] - top);
                            ref[nt][i] = top;
                            limit[nt][i] = top + kSlack;
                        }
                    }
                float top = 0.0f;
#pragma unroll
                for (int grp = 0; grp < GPR; ++grp)
                    top = fmaxf(top, fmaxf(fmaxf(v_rule[0][grp][0].x, v_rule[0][grp][1].x), fmaxf(v_rule[1][grp][0].x, v_rule[1][grp][1].x)));
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                if (top > scale_limit) {
                    // the scale's power of two becomes 32: with weights up to 2^kSlack and scales up to four times that power of two the
                    // product stays below 2^15
                    const uint32_t power = __float_as_uint(top) & 0x7f800000u;
                    const float to = top > 0.0f ? __uint_as_float((259u << 23) - power) : 1.0f;
                    change = to / lift;
                    lift = to;
                    scale_limit = 4.0f * __uint_as_float(power);
                }
                if (started) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int i = 0; i < NC; ++i) {
                            l[nt][i] *= keep[nt][i];
#pragma unroll
                            for (int grp = 0; grp < GPR; ++grp) {
                                zero_sum[nt][grp][i] *= keep[nt][i];
                                w_sum[nt][grp][i] *= keep[nt][i] * change;
                            }
                        }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int t = 0; t < MT; ++t)
#pragma unroll
                            for (int i = 0; i < 4; ++i) o[nt][t][i] *= keep[nt][i % NC] * change;
                }
            }
            started = true;
            // weights, and the product with V
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint32_t *const codes = reinterpret_cast<const uint32_t *>(mem + u * S::kTileBytes + S::kCodes);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                    for (int i = 0; i < 2 * NC; ++i) s[u][nt][i] = exp2_fast(s[u][nt][i] - ref[nt][i % NC]);
#pragma unroll
                    for (int i = 0; i < NC; ++i) l[nt][i] += s[u][nt][i] + s[u][nt][i + NC];
                }
#pragma unroll
                for (int grp = 0; grp < GPR; ++grp) {
                    uint32_t p_hi[NT][2], p_lo[NT][2];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int hh = 0; hh < 2; ++hh) {
                            const float m = v_rule[u][grp][hh].x * lift;
                            float p[NC];
#pragma unroll
                            for (int i = 0; i < NC; ++i) {
                                const float w = s[u][nt][hh * NC + i];
                                zero_sum[nt][grp][i] = __fmaf_rn(w, v_rule[u][grp][hh].y, zero_sum[nt][grp][i]);
                                p[i] = w * m;
                                w_sum[nt][grp][i] += p[i];
                            }
                            if constexpr (kTwin) {
                                // the first four columns get the weights cut off to fp16, the others what was cut off, to nearest (cut off
                                // again it would be too small on average, which adds up over the tokens)
#pragma unroll
                                for (int i = 0; i < NC; ++i) {
                                    const float hi = __uint_as_float(__float_as_uint(p[i]) & 0xffffe000u);
                                    p[i] = lane & 2 ? p[i] - hi : hi;
                                }
                                p_hi[nt][hh] = transpose8x8(pack_round<false>(p[0], p[NC - 1]));
                            } else {
                                const uint32_t hi = pack_round<false>(p[0], p[1]);
                                const float2 back = unpack<false>(hi);
                                p_hi[nt][hh] = transpose8x8(hi);
                                p_lo[nt][hh] = transpose8x8(pack_round<false>(p[0] - back.x, p[1] - back.y));
                            }
                        }
                    constexpr int VW = S::VW < S::kGroupWords ? S::VW : S::kGroupWords;
#pragma unroll
                    for (int v = 0; v < S::kGroupWords; v += VW) {
                        uint32_t x0[VW], x1[VW];              // words of tokens 2 j, 2 j + 1 and 8 + 2 j, 9 + 2 j
                        lds(x0, codes + S::place(0, grp * S::kGroupWords + v, lane));
                        lds(x1, codes + S::place(1, grp * S::kGroupWords + v, lane));
#pragma unroll
                        for (int n = 0; n < VW; ++n) {
                            const int w = grp * S::kGroupWords + v + n;
                            const uint32_t z0 = x0[n] << kUp, z1 = x1[n] << kUp, y0 = x0[n] >> kDown, y1 = x1[n] >> kDown;
                            if constexpr (k4) {
                                const uint32_t f0[4] = {z0 & kLow, z0 & kHigh, z1 & kLow, z1 & kHigh};
                                const uint32_t f1[4] = {y0 & kLow, y0 & kHigh, y1 & kLow, y1 & kHigh};
#pragma unroll
                                for (int nt = 0; nt < NT; ++nt) {
                                    mma_add(o[nt][2 * w], f0, p_hi[nt][0], p_hi[nt][1]);
                                    mma_add(o[nt][2 * w + 1], f1, p_hi[nt][0], p_hi[nt][1]);
                                    if constexpr (!kTwin) {
                                        mma_add(o[nt][2 * w], f0, p_lo[nt][0], p_lo[nt][1]);
                                        mma_add(o[nt][2 * w + 1], f1, p_lo[nt][0], p_lo[nt][1]);
                                    }
                                }
                            } else {
                                const uint32_t f0[4] = {z0 & kLow, y0 & kLow, z1 & kLow, y1 & kLow};
#pragma unroll
                                for (int nt = 0; nt < NT; ++nt) {
                                    mma_add(o[nt][w], f0, p_hi[nt][0], p_hi[nt][1]);
                                    if constexpr (!kTwin) mma_add(o[nt][w], f0, p_lo[nt][0], p_lo[nt][1]);
                                }
                            }
                        }
                    }
                }
            }
            // The sums over codes are held about the middle code: taken as they are they grow with the number of tokens while the result does
            // not, and an MMA cuts its sums off.  Every few tiles, and at the end, the middle is taken out of what has come in (a batch
            // of 16 contexts of 4096 tokens: 1.01 times the error that the rounding of the output has, at the end only 1.03; no time)
            if (left == 1 || (left & 3) == 0) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int grp = 0; grp < GPR; ++grp) {
                        float low[NC];
#pragma unroll
                        for (int i = 0; i < NC; ++i) {
#pragma unroll
                            for (int d = 4; d < 32; d <<= 1) w_sum[nt][grp][i] += __shfl_xor_sync(0xffffffffu, w_sum[nt][grp][i], d);
                            low[i] = w_sum[nt][grp][i] * middle;
                            w_sum[nt][grp][i] = 0.0f;
                        }
#pragma unroll
                        for (int t = grp * (MT / GPR); t < (grp + 1) * (MT / GPR); ++t)
#pragma unroll
                            for (int i = 0; i < 4; ++i) o[nt][t][i] = __fmaf_rn(low[i % NC], k4 && i >= 2 ? 16.0f : 1.0f, o[nt][t][i]);
                    }
            }
            __syncwarp();                                     // the stage may be filled again
            poisoned >>= 1;
            at = at + f.stage_bytes == ring_bytes ? 0 : at + f.stage_bytes;
            if (--left) continue;

            // the end of the item, or of this warp's run.  Sums in units of kLift, as finish_row takes them; N neighbouring channels of a
            // row lie in a lane
            const int c_seq = place.seq, c_hb = place.hb, h = a.by_blocks(c_hb), row0 = (c_hb - h * a.blocks) * 8 * NT, have = min(a.rows, a.group - row0);
            const int tile_end = place.first_tile + idx + 1 - place.first_idx;
            const bool item_ends = !ITEM && tile_end == place.n, began = !ITEM && place.first_tile == 0, whole = item_ends && began;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < NC; ++i)
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) {
                        l[nt][i] += __shfl_xor_sync(0xffffffffu, l[nt][i], d);
#pragma unroll
                        for (int grp = 0; grp < GPR; ++grp) zero_sum[nt][grp][i] += __shfl_xor_sync(0xffffffffu, zero_sum[nt][grp][i], d);
                    }
            if constexpr (kTwin) {
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[0][t][i] += __shfl_xor_sync(0xffffffffu, o[0][t][i], 2);
            }
            const float unit0 = kLift * kUnit * __uint_as_float((254u << 23) - __float_as_uint(lift)), unit1 = k4 ? unit0 * 0x1p-4f : unit0;
            // where a partial result goes: a place of the workspace, or the places of the cluster's CTAs
            float *part = a.part + ((int64_t)run * 2 + (began ? 1 : 0)) * a.rows * kPitch;
            const float *const parts = reinterpret_cast<const float *>(smem_held + W * kStages * f.stage_bytes);
            const int each = HeldParts<S>::kGroups >> a.item_shift;
            if constexpr (ITEM) cluster_wait();               // the other CTAs have begun
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < NC; ++i) {
                    const int r = nt * 8 + 2 * j + i;
                    if (r >= have) continue;
                    const int64_t row = (int64_t)c_seq * a.Hq + h * a.group + row0 + r;
                    const float inv = l[nt][i] == 0.0f ? 0.0f : (1.0f / kLift) / l[nt][i];
#pragma unroll
                    for (int w = 0; w < S::W; ++w) {
                        const float z = zero_sum[nt][w / S::kGroupWords][i] * kLift;
                        float v[N];
#pragma unroll
                        for (int c = 0; c < N; c += 2) {
                            const float *acc = o[nt][k4 ? 2 * w + c / 2 : w];
                            v[c] = __fmaf_rn(acc[i], unit0, z);
                            v[c + 1] = __fmaf_rn(acc[i + 2], unit1, z);
                        }
                        const int group = 8 * w + g;
                        if constexpr (ITEM) {
                            const int cta = (group << a.item_shift) / HeldParts<S>::kGroups;
                            cluster_store(cluster_addr(parts + ((size_t)(me * a.rows + r) * each + group - cta * each) * N, cta), v);
                        } else if (whole) {
                            store_channels(a.out + row * S::D + group * N, v, inv, f.bf16);
                        } else if constexpr (N == 4) {
                            *reinterpret_cast<float4 *>(part + r * kPitch + group * N) = make_float4(v[0], v[1], v[2], v[3]);
                        } else {
                            *reinterpret_cast<float2 *>(part + r * kPitch + group * N) = make_float2(v[0], v[1]);
                        }
                    }
                    const float ml[2] = {limit[nt][i] == -INFINITY ? -INFINITY : ref[nt][i], l[nt][i]};
                    if constexpr (ITEM) {
                        // (lane g stores it to CTA g)
                        if (g < 1 << a.item_shift) cluster_store(cluster_addr(parts + (size_t)step * a.rows * each * N + (me * a.rows + r) * 2, g), ml);
                    } else if (g == 0) {
                        if (!whole) *reinterpret_cast<float2 *>(part + r * kPitch + kCols) = make_float2(ml[0], ml[1]);
                        else if (a.lse) a.lse[row] = l[nt][i] == 0.0f ? -INFINITY : (ref[nt][i] + log2f(l[nt][i])) * kLn2;
                    }
                }
            if constexpr (!ITEM) {
                const int item = c_seq * per_seq + c_hb;
                if (began) {                                  // the item begins here: say who has its tiles
                    if (!item_ends) open_item = item;
                    if (lane == 0) a.span[item] = item_ends ? make_int2(-1, 0) : make_int2(run, Runs(a, total).of(place.slot + (c_hb + 1) * (place.n + kItemSlots) - 1));
                }
                begins = true;
                __syncwarp();
                place.first_tile = 0;
                place.first_idx = idx + 1;
                if (idx + 1 < w1) {
                    if (c_hb + 1 < per_seq) {
                        place.hb = c_hb + 1;
                    } else {
                        place.hb = 0;
                        place.slot += per_seq * (place.n + kItemSlots);
                        int seq = c_seq;
                        SeqTiles s;
                        do s = seq_tiles<kHeldTile>(a, __ldg(a.lens + ++seq));
                        while (s.n == 0);
                        place.seq = seq;
                        place.len = s.len;
                        place.first = s.first;
                        place.tile0 = s.tile0;
                        place.n = s.n;
                    }
                }
                __syncwarp();
            }
        }
    } else if constexpr (ITEM) {
        cluster_wait();
    }
    if constexpr (ITEM) {
        cluster_arrive();
        cluster_wait();                                       // every warp's part has arrived
        const int h = a.by_blocks(c_hb), row0 = (c_hb - h * a.blocks) * 8 * NT, have = min(a.rows, a.group - row0);
        if (f_s.n) {
            join_parts<S>(a, f.bf16, reinterpret_cast<const float *>(smem_held + W * kStages * f.stage_bytes), c_seq, row0, h, have, min(f_s.n, step));
        } else if (cluster_rank() == 0) {
            const int64_t row = (int64_t)c_seq * a.Hq + h * a.group + row0;
            if (f.bf16) fill_empty<true>(a, row, have, __ldg(a.lens + c_seq) != 0, threadIdx.x, W * 32);
            else fill_empty<false>(a, row, have, __ldg(a.lens + c_seq) != 0, threadIdx.x, W * 32);
        }
        return;
    }
    if (lane == 0) a.open[run] = open_item;

    // rows of the batch without tokens
    for (int b = run; b < a.n_seqs; b += a.runs) {
        const int len = __ldg(a.lens + b);
        if (seq_tiles<kHeldTile>(a, len).n) continue;
        if (f.bf16) fill_empty<true>(a, (int64_t)b * a.Hq, a.Hq, len != 0, lane, 32);
        else fill_empty<false>(a, (int64_t)b * a.Hq, a.Hq, len != 0, lane, 32);
    }
}

template <typename S, int MODE, bool ITEM, bool DEEP>
int launch_held_form(const DecodeArgs &a, const HeldFeed &f, int item_ctas, cudaStream_t st)
{
    // registers: as many warps as held_room says, where there are few query rows
    constexpr int kMin = (MODE == 0 || MODE == 3) && !ITEM ? held_room(S::kTileBytes, DEEP) / kRunWarps : 1;
    constexpr auto kernel = held_attention_kernel<S, MODE, ITEM, DEEP, kMin>;
    LLMS_CUDA_TRY(allow_shared_memory<kernel>());
    if constexpr (ITEM)
        LLMS_CUDA_TRY(launch_dependent_cluster(kernel, dim3(a.n_seqs * a.Hkv * a.blocks * item_ctas), dim3(HeldParts<S>::kWarps * 32),
                                               held_item_smem(S::kTileBytes, a.rows, S::D, item_ctas), item_ctas, st, a, f));
    else
        LLMS_CUDA_TRY(launch_dependent(kernel, dim3((a.runs + kRunWarps - 1) / kRunWarps), dim3(kRunWarps * 32),
                                       (size_t)kRunWarps * held_stages(S::kTileBytes, DEEP) * f.stage_bytes, st, a, f));
    return LLMS_OK;
}

template <typename S, int MODE>
int launch_held_mode(const DecodeArgs &a, HeldFeed f, int item_ctas, bool deep, cudaStream_t st)
{
    f.stage_bytes = held_stage_bytes(S::kTileBytes, a.rows, S::D);
    if (item_ctas) return launch_held_form<S, MODE, true, true>(a, f, item_ctas, st);
    if (deep) return launch_held_form<S, MODE, false, true>(a, f, 0, st);
    return launch_held_form<S, MODE, false, false>(a, f, 0, st);
}

// Instantiated per head_dim in files of their own (held_attention_<head_dim>.cu).
template <int D>
int launch_held_attention(int bits, int groups, int mode, const DecodeArgs &a, const HeldFeed &f, int item_ctas, bool deep, cudaStream_t st);

template <typename S>
int launch_held_shape(int mode, const DecodeArgs &a, const HeldFeed &f, int item_ctas, bool deep, cudaStream_t st)
{
    if (mode == 0) return a.group == 1 ? launch_held_mode<S, 3>(a, f, item_ctas, deep, st) : launch_held_mode<S, 0>(a, f, item_ctas, deep, st);
    return mode == 1 ? launch_held_mode<S, 1>(a, f, item_ctas, deep, st) : launch_held_mode<S, 2>(a, f, item_ctas, deep, st);
}

}  // namespace llms
