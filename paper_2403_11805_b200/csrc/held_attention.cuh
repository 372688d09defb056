// Attention of one new token per sequence over a pool held at 8 or 4 bits, one layer per call: the kernel.
//
// Mathematics.  As for the fp16 pool (decode.cu), with K_t = z_t + s_t k_t and V_t = z'_t + s'_t v_t, k_t and v_t whole numbers below 2^bits,
// s and z the scale and zero-point of a token's group of channels.  Both products are taken on the codes:
//     <q, K_t> = sum over groups  s_t <q, k_t> + z_t sum q,        sum_t p_t V_t = sum_t (p_t s'_t) v_t + sum_t p_t z'_t.
// A code enters an fp16 MMA as it lies in its word: bits 0 .. 9 of an fp16 whose upper bits are 0 are a subnormal number, the code times
// 2^-24 (or 2^-20, four bits further up), exactly.  So a mask, for half of the codes a shift too, makes a pair of operands, the products
// are exact, and the powers of two are taken back in the sums.
//
// Bound.  A quarter (half) of the fp16 pool's bytes for the same arithmetic: at 4 bits and 128 channels an SM has some 95 cycles per
// tile of 2176 bytes at the copy bandwidth, and a tile takes about 200 instructions of a warp.  So both count: the
// instructions must be few, and enough warps must be there to fill each other's gaps.
//
// Split.  As for the fp16 pool: runs of 16-token tiles, one per warp, or a cluster per item for small calls.  A tile is one
// run of bytes in the pool and comes as one copy; its codes lie in the order of the MMAs' operands.
#pragma once

#include "decode.cuh"
#include "held.cuh"

namespace llms {

struct HeldFeed {
    uint8_t *held;                                // of the layer
    int tiles, bf16, warp_bytes;                  // tiles per KV head; type of the rows; shared memory of a warp
};

template <typename S, int MODE>
struct HeldWarp {
    static constexpr int kStages = S::kTileBytes <= 2304 ? 4 : (S::kTileBytes <= 4608 ? 3 : 2);
    static constexpr int DB = (S::D + 63) / 64;
    // ring, and query rows of two items; a partial result takes the ring's place in a cluster
    static int bytes(int rows, bool item)
    {
        const int ring = kStages * S::kTileBytes + kQuerySlots * rows * S::D * 2, part = item ? rows * DecodeCols<DB>::kPitch * 4 : 0;
        return (std::max(ring, part) + 127) & ~127;
    }
};

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
                if constexpr (kPairs == 4) *reinterpret_cast<uint4 *>(x[m]) = __ldg(reinterpret_cast<const uint4 *>(from));
                else *reinterpret_cast<uint2 *>(x[m]) = __ldg(reinterpret_cast<const uint2 *>(from));
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

// MODE: up to 4, 8 or 16 query rows (see decode_kernel).
template <typename S, int MODE, bool ITEM>
__global__ void __launch_bounds__(ITEM ? kItemWarps * 32 : 32) held_attention_kernel(const DecodeArgs a, const HeldFeed f)
{
    constexpr int NT = MODE == 2 ? 2 : 1;                     // column groups of eight query rows
    constexpr bool kTwin = MODE == 0;
    using HW = HeldWarp<S, MODE>;
    constexpr int DB = HW::DB, kStages = HW::kStages, kPitch = DecodeCols<DB>::kPitch, kCols = DecodeCols<DB>::kCols;
    constexpr int MT = S::D / 16, GPR = S::GPR;               // 16-channel tiles of the output; groups per row
    constexpr bool k4 = S::BITS == 4;
    constexpr uint32_t kLow = k4 ? 0x000f000fu : 0x00ff00ffu, kHigh = 0x00f000f0u;
    constexpr int W = ITEM ? kItemWarps : 1;
    extern __shared__ __align__(128) unsigned char smem_held[];
    const int lane = threadIdx.x & 31, warp = ITEM ? threadIdx.x >> 5 : 0, run = blockIdx.x, g = lane >> 2, j = lane & 3;
    unsigned char *const ring = smem_held + warp * f.warp_bytes;
    const uint32_t ring_addr = smem_u32(ring), q_addr = ring_addr + kStages * S::kTileBytes;
    __shared__ unsigned long long s_full[W][kStages];
    unsigned long long *const full = s_full[warp];

    if (lane == 0) {
#pragma unroll
        for (int s = 0; s < kStages; ++s) mbar_init(&full[s], 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    grid_dependency_wait();
    grid_launch_dependents();

    const int per_seq = a.Hkv * a.blocks;
    int w0, w1, f_seq, f_base, total;                         // tiles of this warp; a sequence, and its first tile
    SeqTiles f_s;
    find_tiles<ITEM, W>(a, warp, lane, w0, w1, f_seq, f_base, total, f_s);
    const Runs runs(a, total);
    int open_item = -1;                                       // the item that begins in this run and goes on behind it

    if (w0 < w1) {
        auto skip = [&](int idx) {                            // on to the sequence that has tile idx
            while (f_base + f_s.n * per_seq <= idx) {
                f_base += f_s.n * per_seq;
                f_s = seq_tiles(a, __ldg(a.lens + ++f_seq));
            }
        };
        skip(w0);
        int c_seq = f_seq, c_hb = (w0 - f_base) / f_s.n, c_tile = w0 - f_base - c_hb * f_s.n;   // where the arithmetic is
        SeqTiles c_s = f_s;

        // ---- feeding: lane i looks up the tile i behind `base`
        int f_slot, f_row, f_q;                                               // slot, row in its chunk, sequence
        bool f_need;
        uint32_t f_h, f_qb;                                                   // KV head (and first query row << 16); bytes of query rows,
                                                                              // which come with the first tile of an item
        auto look_up = [&](int base) {
            const int idx = base + lane, last = min(base + 32, w1) - 1;
            f_need = false;
            f_slot = -1;
            f_row = 0;
            f_h = f_qb = 0;
            for (;;) {
                if (idx >= f_base && idx <= last && idx < f_base + f_s.n * per_seq) {
                    const int hb = (idx - f_base) / f_s.n, tile = idx - f_base - hb * f_s.n, tok = (f_s.tile0 + tile) * kTile;
                    f_need = true;
                    f_h = a.by_blocks(hb);
                    const int chunk = a.by_chunk(tok);
                    f_row = tok - chunk * a.chunk_len;
                    f_slot = __ldg(a.table + (int64_t)f_seq * a.table_stride + chunk);
                    if (idx == w0 || tile == 0) {
                        const int r0 = (hb - f_h * a.blocks) * 8 * NT;
                        f_qb = min(a.rows, a.group - r0) * S::D * 2;
                        f_q = f_seq;
                        f_h |= (uint32_t)r0 << 16;
                    }
                }
                if (last < f_base + f_s.n * per_seq) break;
                skip(f_base + f_s.n * per_seq);
            }
        };
        int base = w0, issued = w0, stage_in = 0, q_issued = 0, q_read = 0;
        uint32_t ok_mask = 0, q_mask = 0, poisoned = 0;                       // poisoned: stages whose tile's slot lies outside the pool
        const uint8_t *f_from = nullptr;
        bool fetched = false;                                                 // the masks belong to the look-up at `base`
        auto issue = [&] {
            if (!fetched) {
                const bool inside = f_need && (unsigned)f_slot < (unsigned)a.n_slots;
                ok_mask = __ballot_sync(0xffffffffu, inside);
                q_mask = __ballot_sync(0xffffffffu, f_qb != 0);
                f_from = f.held + ((int64_t)(f_h & 0xffff) * f.tiles + (((int64_t)f_slot * a.chunk_len + f_row) >> 4)) * S::kTileBytes;
                fetched = true;
            }
            const int lead = issued - base;
            const bool with_q = q_mask >> lead & 1;
            if (with_q && q_issued - q_read >= kQuerySlots) return;           // its query rows have no place yet
            const bool there = ok_mask >> lead & 1;
            unsigned long long *bar = &full[stage_in];
            poisoned = (poisoned & ~(1u << stage_in)) | (there ? 0u : 1u << stage_in);
            if (lane == lead) {
                mbar_expect_tx(bar, (there ? S::kTileBytes : 0) + f_qb);
                if (there) bulk_load(ring_addr + stage_in * S::kTileBytes, f_from, S::kTileBytes, bar);
                if (f_qb)
                    bulk_load(q_addr + (q_issued % kQuerySlots) * a.q_bytes,
                              a.q + f_q * a.q_stride + (int64_t)((f_h & 0xffff) * a.group + (f_h >> 16)) * S::D, f_qb, bar);
            }
            q_issued += with_q;
            ++issued;
            stage_in = stage_in + 1 == kStages ? 0 : stage_in + 1;
            if (issued - base == 32 && issued < w1) {
                base = issued;
                fetched = false;
                look_up(base);
            }
        };
        look_up(base);
#pragma unroll 1
        for (int s = 0; s < kStages && issued < w1; ++s) issue();

        // ---- the arithmetic
        int stage = 0, phase = 0, done = w0;
        bool lost = false;                                    // a copy did not arrive: no more are asked for, those on their way are
                                                              // still waited for, and what has not arrived counts as NaN
#pragma unroll 1
        for (int idx = w0; idx < w1;) {                       // the items that this run has tiles of
            const int h = a.by_blocks(c_hb), rb = c_hb - h * a.blocks;
            const int row0 = rb * 8 * NT, have = min(a.rows, a.group - row0);     // query rows of this item
            const int tile_end = min(c_s.n, c_tile + w1 - idx);
            const bool item_ends = tile_end == c_s.n;
            // the newest token's rows, for the item's last tile
            FreshRow<S> fresh_k, fresh_v;
            int fresh_slot = -1;
            const bool append = a.k_new && item_ends;
            if (append) {
                fresh_k.load(a.k_new + c_seq * a.new_stride + (int64_t)h * S::D, lane);
                fresh_v.load(a.v_new + c_seq * a.new_stride + (int64_t)h * S::D, lane);
                fresh_slot = __ldg(a.table + (int64_t)c_seq * a.table_stride + a.by_chunk(c_s.len - 1));
            }
            bool good = idx < issued && warp_wait(&full[stage], phase);
            lost |= !good;
            // query rows as the MMA's second operand, channels in the order that K's codes come in; columns beyond the item's rows repeat
            // others (nobody reads their results).  bfloat16 rows become fp16 times a power of two, exactly but for values
            // below 2^-29 of the row's largest.  fac: what a logit in these units is multiplied with; q_sum: sum q per group
            uint32_t qf[NT][S::W][k4 ? 4 : 2];
            float o[NT][MT][4], ref[NT][2], limit[NT][2], l[NT][2], zero_sum[NT][GPR][2], fac[NT][2], q_sum[NT][GPR][2];
            float lift = 1.0f, scale_limit = -1.0f;           // what V's scales are multiplied with; the largest one that this suits
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const int r = nt * 8 + (g & (kTwin ? 3 : 7));
                const unsigned char *row = ring + kStages * S::kTileBytes + (q_read % kQuerySlots) * a.q_bytes + min(r, have - 1) * S::D * 2;
                uint32_t most = 0, x[S::W][k4 ? 4 : 2];
#pragma unroll
                for (int w = 0; w < S::W; ++w) {
                    lds(x[w], row + (4 * w + j) * (k4 ? 16 : 8));
#pragma unroll
                    for (int c = 0; c < (k4 ? 4 : 2); ++c) most = __vmaxu2(most, x[w][c] & 0x7fff7fffu);
                }
                most = max(most & 0xffffu, most >> 16);
                most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
                most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
                float own = a.scale_log2;
                if (f.bf16) {
                    // the largest value comes to lie in [2^14, 2^15)
                    const int e = min((int)(most >> 7) - 127, 127), shift = min(14 - e, 126);
                    const float up = __uint_as_float((uint32_t)(127 + shift) << 23);
                    own *= __uint_as_float((uint32_t)(127 - shift) << 23);
#pragma unroll
                    for (int w = 0; w < S::W; ++w)
#pragma unroll
                        for (int c = 0; c < (k4 ? 4 : 2); ++c) {
                            const float2 v = unpack<true>(x[w][c]);
                            x[w][c] = pack_round<false>(v.x * up, v.y * up);
                        }
                }
                if (most >= (f.bf16 ? 0x7f80u : 0x7c00u)) own = NAN;
                float sums[GPR];
#pragma unroll
                for (int grp = 0; grp < GPR; ++grp) {
                    sums[grp] = 0.0f;
#pragma unroll
                    for (int w = grp * S::kGroupWords; w < (grp + 1) * S::kGroupWords; ++w)
#pragma unroll
                        for (int c = 0; c < (k4 ? 4 : 2); ++c) {
                            const float2 v = unpack<false>(x[w][c]);
                            sums[grp] += v.x + v.y;
                        }
                    sums[grp] += __shfl_xor_sync(0xffffffffu, sums[grp], 1);
                    sums[grp] += __shfl_xor_sync(0xffffffffu, sums[grp], 2);
                }
#pragma unroll
                for (int w = 0; w < S::W; ++w) {
                    if constexpr (k4) {
                        qf[nt][w][0] = __byte_perm(x[w][0], x[w][2], 0x5410);         // channels 0, 4; 2, 6; 1, 5; 3, 7 of a word
                        qf[nt][w][1] = __byte_perm(x[w][1], x[w][3], 0x5410);
                        qf[nt][w][2] = __byte_perm(x[w][0], x[w][2], 0x7632);
                        qf[nt][w][3] = __byte_perm(x[w][1], x[w][3], 0x7632);
                    } else {
                        qf[nt][w][0] = __byte_perm(x[w][0], x[w][1], 0x5410);         // channels 0, 2; 1, 3
                        qf[nt][w][1] = __byte_perm(x[w][0], x[w][1], 0x7632);
                    }
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int from = (2 * j + i) * 4;         // a lane that has row 2 j + i
                    fac[nt][i] = __shfl_sync(0xffffffffu, own, from);
#pragma unroll
                    for (int grp = 0; grp < GPR; ++grp) {
                        q_sum[nt][grp][i] = __shfl_sync(0xffffffffu, sums[grp], from);
                        zero_sum[nt][grp][i] = 0.0f;
                    }
                    ref[nt][i] = 0.0f;
                    limit[nt][i] = -INFINITY;                 // reference + kSlack; -inf: no logit yet
                    l[nt][i] = 0.0f;
                }
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[nt][t][i] = 0.0f;
            }
            __syncwarp();
            ++q_read;
            const int tile_begin = c_tile;

#pragma unroll 1
            for (int tile = tile_begin; tile < tile_end; ++tile) {
                if (tile != tile_begin) {
                    good = done < issued && warp_wait(&full[stage], phase);
                    lost |= !good;
                }
                const int tok0 = (c_s.tile0 + tile) * kTile;
                unsigned char *const mem = ring + stage * S::kTileBytes;
                const bool poison = !good || (poisoned >> stage & 1);
                // tiles that hold places nobody sees, the newest token, or a slot outside the pool
                const bool special = poison || tok0 < c_s.first || tok0 + kTile > c_s.len || (append && tile + 1 == c_s.n);
                if (special) {
                    // parameters of rows that are not seen are cleared: whatever codes lie there are 0 then.  The newest token's row: what
                    // the caller gave, here and in the pool
                    const int t = tok0 + (lane & 15);
                    if (t < c_s.first || t >= c_s.len)
#pragma unroll
                        for (int grp = 0; grp < GPR; ++grp)
                            reinterpret_cast<uint32_t *>(mem + 2 * S::kCodes + (lane >> 4) * S::kParams)[(lane & 15) * GPR + grp] = 0u;
                    if (append && tile + 1 == c_s.n) {
                        fresh_k.quantise(f.bf16);
                        fresh_v.quantise(f.bf16);
                        const int at = c_s.len - 1 - tok0;
                        __syncwarp();
                        fresh_k.store(mem, 0, at, lane);
                        fresh_v.store(mem, 1, at, lane);
                        if ((unsigned)fresh_slot < (unsigned)a.n_slots && rb == 0) {
                            const int row = c_s.len - 1 - a.by_chunk(c_s.len - 1) * a.chunk_len;
                            uint8_t *to = f.held + ((int64_t)h * f.tiles + (((int64_t)fresh_slot * a.chunk_len + row) >> 4)) * S::kTileBytes;
                            fresh_k.store(to, 0, at, lane);
                            fresh_v.store(to, 1, at, lane);
                        }
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // before a copy fills this stage again
                    __syncwarp();
                }
                const __half2 *const k_rule = reinterpret_cast<const __half2 *>(mem + 2 * S::kCodes);
                const __half2 *const v_rule = reinterpret_cast<const __half2 *>(mem + 2 * S::kCodes + S::kParams);

                // logits: tokens x query rows
                float s[NT][4];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[nt][i] = 0.0f;
                uint32_t x0[S::W], x1[S::W];                  // words of tokens g and 8 + g
#pragma unroll
                for (int w = 0; w < S::W; w += S::VW) {
                    lds(reinterpret_cast<uint32_t (&)[S::VW]>(x0[w]), reinterpret_cast<const uint32_t *>(mem) + S::place(0, w, lane));
                    lds(reinterpret_cast<uint32_t (&)[S::VW]>(x1[w]), reinterpret_cast<const uint32_t *>(mem) + S::place(1, w, lane));
                }
#pragma unroll
                for (int grp = 0; grp < GPR; ++grp) {
                    float c0[NT][4], c1[NT][4];               // 4 bits: codes of low and of high places; 8 bits: two chains
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int i = 0; i < 4; ++i) c0[nt][i] = c1[nt][i] = 0.0f;
#pragma unroll
                    for (int w = grp * S::kGroupWords; w < (grp + 1) * S::kGroupWords; ++w) {
                        const uint32_t y0 = x0[w] >> 8, y1 = x1[w] >> 8;
                        const uint32_t low[4] = {x0[w] & kLow, x1[w] & kLow, y0 & kLow, y1 & kLow};
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) mma<false>(k4 || w % 2 == 0 ? c0[nt] : c1[nt], low, qf[nt][w][0], qf[nt][w][1]);
                        if constexpr (k4) {
                            const uint32_t high[4] = {x0[w] & kHigh, x1[w] & kHigh, y0 & kHigh, y1 & kHigh};
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) mma<false>(c1[nt], high, qf[nt][w][2], qf[nt][w][3]);
                        }
                    }
                    const float2 r0 = __half22float2(k_rule[g * GPR + grp]), r1 = __half22float2(k_rule[(8 + g) * GPR + grp]);
                    constexpr float kUnit = k4 ? 0x1p20f : 0x1p24f;
                    const float m0 = r0.x * kUnit, m1 = r1.x * kUnit;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float c = k4 ? __fmaf_rn(c0[nt][i], 16.0f, c1[nt][i]) : c0[nt][i] + c1[nt][i];
                            const float z = (i < 2 ? r0.y : r1.y) * q_sum[nt][grp][i & 1];
                            s[nt][i] = grp == 0 ? __fmaf_rn(c, i < 2 ? m0 : m1, z) : s[nt][i] + __fmaf_rn(c, i < 2 ? m0 : m1, z);
                        }
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[nt][i] *= fac[nt][i & 1];
                if (special) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int t = tok0 + g + (i >> 1) * 8;
                            if (poison) s[nt][i] = NAN;
                            if (t < c_s.first || t >= c_s.len) s[nt][i] = -INFINITY;
                        }
                }
                // V's words and parameters
                float v_scale[GPR][2], v_zero[GPR][2];
                bool over = false;
#pragma unroll
                for (int grp = 0; grp < GPR; ++grp)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float2 r = __half22float2(v_rule[(8 * i + g) * GPR + grp]);
                        v_scale[grp][i] = r.x;
                        v_zero[grp][i] = r.y;
                        over |= r.x > scale_limit;
                    }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) over |= s[nt][i] > limit[nt][i & 1];
                if (__any_sync(0xffffffffu, over)) {          // the references move up to the maxima
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            float top = fmaxf(s[nt][i], s[nt][i + 2]);
#pragma unroll
                            for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                            if (top > limit[nt][i] - kSlack) {
                                const float keep = limit[nt][i] == -INFINITY ? 0.0f : exp2_fast(ref[nt][i] - top);
                                ref[nt][i] = top;
                                limit[nt][i] = top + kSlack;
                                l[nt][i] *= keep;
#pragma unroll
                                for (int grp = 0; grp < GPR; ++grp) zero_sum[nt][grp][i] *= keep;
#pragma unroll
                                for (int t = 0; t < MT; ++t) {
                                    o[nt][t][i] *= keep;
                                    o[nt][t][i + 2] *= keep;
                                }
                            }
                        }
                    float top = 0.0f;
#pragma unroll
                    for (int grp = 0; grp < GPR; ++grp) top = fmaxf(top, fmaxf(v_scale[grp][0], v_scale[grp][1]));
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                    if (top > scale_limit) {
                        // the scale's power of two becomes 16: with weights up to 2^kSlack and scales up to eight times that power of two
                        // the product stays below 2^15
                        const uint32_t power = __float_as_uint(top) & 0x7f800000u;
                        const float next = top > 0.0f ? __uint_as_float((258u << 23) - power) : 1.0f, change = next / lift;
                        lift = next;
                        scale_limit = 8.0f * __uint_as_float(power);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int t = 0; t < MT; ++t)
#pragma unroll
                                for (int i = 0; i < 4; ++i) o[nt][t][i] *= change;
                    }
                }
                // weights
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[nt][i] = exp2_fast(s[nt][i] - ref[nt][i & 1]);
#pragma unroll
                    for (int i = 0; i < 2; ++i) l[nt][i] += s[nt][i] + s[nt][i + 2];
                }
#pragma unroll
                for (int w = 0; w < S::W; w += S::VW) {       // words of tokens 2 j, 2 j + 1 and 8 + 2 j, 9 + 2 j
                    lds(reinterpret_cast<uint32_t (&)[S::VW]>(x0[w]), reinterpret_cast<const uint32_t *>(mem + S::kCodes) + S::place(0, w, lane));
                    lds(reinterpret_cast<uint32_t (&)[S::VW]>(x1[w]), reinterpret_cast<const uint32_t *>(mem + S::kCodes) + S::place(1, w, lane));
                }
#pragma unroll
                for (int grp = 0; grp < GPR; ++grp) {
                    uint32_t p_hi[NT][2], p_lo[NT][2];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const float m = v_scale[grp][i] * lift, p0 = s[nt][2 * i] * m, p1 = s[nt][2 * i + 1] * m;
                            zero_sum[nt][grp][0] = __fmaf_rn(s[nt][2 * i], v_zero[grp][i], zero_sum[nt][grp][0]);
                            zero_sum[nt][grp][1] = __fmaf_rn(s[nt][2 * i + 1], v_zero[grp][i], zero_sum[nt][grp][1]);
                            const uint32_t hi = pack_round<false>(p0, p1);
                            const float2 back = unpack<false>(hi);
                            const uint32_t lo = pack_round<false>(p0 - back.x, p1 - back.y);
                            p_hi[nt][i] = transpose8x8(kTwin && (lane & 2) ? lo : hi);
                            if constexpr (!kTwin) p_lo[nt][i] = transpose8x8(lo);
                        }
#pragma unroll
                    for (int w = grp * S::kGroupWords; w < (grp + 1) * S::kGroupWords; ++w) {
                        const uint32_t y0 = x0[w] >> 8, y1 = x1[w] >> 8;
                        if constexpr (k4) {
                            const uint32_t f0[4] = {x0[w] & kLow, x0[w] & kHigh, x1[w] & kLow, x1[w] & kHigh};
                            const uint32_t f1[4] = {y0 & kLow, y0 & kHigh, y1 & kLow, y1 & kHigh};
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) {
                                mma<false>(o[nt][2 * w], f0, p_hi[nt][0], p_hi[nt][1]);
                                mma<false>(o[nt][2 * w + 1], f1, p_hi[nt][0], p_hi[nt][1]);
                                if constexpr (!kTwin) {
                                    mma<false>(o[nt][2 * w], f0, p_lo[nt][0], p_lo[nt][1]);
                                    mma<false>(o[nt][2 * w + 1], f1, p_lo[nt][0], p_lo[nt][1]);
                                }
                            }
                        } else {
                            const uint32_t f0[4] = {x0[w] & kLow, y0 & kLow, x1[w] & kLow, y1 & kLow};
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) {
                                mma<false>(o[nt][w], f0, p_hi[nt][0], p_hi[nt][1]);
                                if constexpr (!kTwin) mma<false>(o[nt][w], f0, p_lo[nt][0], p_lo[nt][1]);
                            }
                        }
                    }
                }
                __syncwarp();
                ++done;
#pragma unroll 1
                for (int s = 0; s < 2 && !lost && issued < w1 && issued < done + kStages; ++s) issue();      // two: one may have had to wait
                if (++stage == kStages) {
                    stage = 0;
                    phase ^= 1;
                }
            }

            // the end of the item, or of this warp's run
            const int item_begin = idx - tile_begin;
            idx += tile_end - tile_begin;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) {
                        l[nt][i] += __shfl_xor_sync(0xffffffffu, l[nt][i], d);
#pragma unroll
                        for (int grp = 0; grp < GPR; ++grp) zero_sum[nt][grp][i] += __shfl_xor_sync(0xffffffffu, zero_sum[nt][grp][i], d);
                    }
                }
            if constexpr (kTwin) {
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[0][t][i] += __shfl_xor_sync(0xffffffffu, o[0][t][i], 2);
            }
            // sums in units of kLift, as finish_row takes them; four (8 bits: two) neighbouring channels of a row lie in a lane
            constexpr int N = k4 ? 4 : 2;
            const float unit0 = kLift * 0x1p24f / lift, unit1 = k4 ? kLift * 0x1p20f / lift : unit0;
            const bool whole = !ITEM && item_ends && tile_begin == 0;
            float *part = ITEM ? reinterpret_cast<float *>(ring) : a.part + ((int64_t)run * 2 + (tile_begin > 0 ? 0 : 1)) * a.rows * kPitch;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int r = nt * 8 + 2 * j + i;
                    const int64_t row = (int64_t)c_seq * a.Hq + h * a.group + row0 + r;
                    const float inv = l[nt][i] == 0.0f ? 0.0f : (1.0f / kLift) / l[nt][i];
                    if (r >= (whole ? have : a.rows)) continue;
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
                        const int c = (8 * w + g) * N;
                        if (whole) {
                            uint32_t out[N / 2];
#pragma unroll
                            for (int n = 0; n < N; n += 2)
                                out[n / 2] = f.bf16 ? pack_round<true>(channel(v[n], inv), channel(v[n + 1], inv))
                                                    : pack_round<false>(channel(v[n], inv), channel(v[n + 1], inv));
                            uint16_t *to = a.out + row * S::D + c;
                            if constexpr (N == 4) *reinterpret_cast<uint2 *>(to) = make_uint2(out[0], out[1]);
                            else *reinterpret_cast<uint32_t *>(to) = out[0];
                        } else {
                            float *to = part + r * kPitch + c;
                            if constexpr (N == 4) *reinterpret_cast<float4 *>(to) = make_float4(v[0], v[1], v[2], v[3]);
                            else *reinterpret_cast<float2 *>(to) = make_float2(v[0], v[1]);
                        }
                    }
                    if (g == 0) {
                        if (whole) {
                            const float lg = l[nt][i] == 0.0f ? -INFINITY : ref[nt][i] + log2f(l[nt][i]);
                            if (a.lse) a.lse[row] = lg * kLn2;
                        } else {
                            *reinterpret_cast<float2 *>(part + r * kPitch + kCols) =
                                make_float2(limit[nt][i] == -INFINITY ? -INFINITY : ref[nt][i], l[nt][i]);
                        }
                    }
                }
            const int item = c_seq * per_seq + c_hb;
            if (!ITEM && tile_begin == 0) {                   // the item begins here: say who has its tiles
                if (!item_ends) open_item = item;
                if (lane == 0) a.span[item] = item_ends ? make_int2(-1, 0) : make_int2(run, runs.of(item_begin + c_s.n - 1));
            }
            if (!ITEM && idx < w1) {
                c_tile = 0;
                if (++c_hb == per_seq) {
                    c_hb = 0;
                    do c_s = seq_tiles(a, __ldg(a.lens + ++c_seq));
                    while (c_s.n == 0);
                }
            }
        }
    }
    if constexpr (ITEM) {
        if (f.bf16) join_item<true, DB, NT>(a, smem_held, f.warp_bytes, w0, w1);
        else join_item<false, DB, NT>(a, smem_held, f.warp_bytes, w0, w1);
        return;
    }
    if (lane == 0) a.open[run] = open_item;

    // rows of the batch without tokens
    for (int b = run; b < a.n_seqs; b += gridDim.x) {
        const int len = __ldg(a.lens + b);
        if (seq_tiles(a, len).n) continue;
        if (f.bf16) fill_empty<true>(a, (int64_t)b * a.Hq, a.Hq, len != 0, lane, 32);
        else fill_empty<false>(a, (int64_t)b * a.Hq, a.Hq, len != 0, lane, 32);
    }
}

template <typename S, int MODE>
int launch_held_mode(const DecodeArgs &a, HeldFeed f, int item_ctas, cudaStream_t st)
{
    f.warp_bytes = HeldWarp<S, MODE>::bytes(a.rows, item_ctas != 0);
    const size_t smem = (size_t)f.warp_bytes * (item_ctas ? kItemWarps : 1);
    if (item_ctas) {
        LLMS_CUDA_TRY((allow_shared_memory<held_attention_kernel<S, MODE, true>>()));
        LLMS_CUDA_TRY(launch_dependent_cluster(held_attention_kernel<S, MODE, true>, dim3(a.n_seqs * a.Hkv * a.blocks * item_ctas), dim3(kItemWarps * 32),
                                               smem, item_ctas, st, a, f));
    } else {
        LLMS_CUDA_TRY((allow_shared_memory<held_attention_kernel<S, MODE, false>>()));
        LLMS_CUDA_TRY(launch_dependent(held_attention_kernel<S, MODE, false>, dim3(a.grid_runs), dim3(32), smem, st, a, f));
    }
    return LLMS_OK;
}

// Instantiated per head_dim in files of their own (held_attention_<head_dim>.cu).
template <int D>
int launch_held_attention(int bits, int groups, int mode, const DecodeArgs &a, const HeldFeed &f, int item_ctas, cudaStream_t st);

template <typename S>
int launch_held_shape(int mode, const DecodeArgs &a, const HeldFeed &f, int item_ctas, cudaStream_t st)
{
    if (mode == 0) return launch_held_mode<S, 0>(a, f, item_ctas, st);
    return mode == 1 ? launch_held_mode<S, 1>(a, f, item_ctas, st) : launch_held_mode<S, 2>(a, f, item_ctas, st);
}

}  // namespace llms
