// What the kernels that attend to a paged cache share (decode.cu, held_attention.cuh): operands, the batch's tiles and runs of them, conversions,
// how a row ends, the workspace and when a call has clusters.  decode.cu has the mathematics and the split.
#pragma once

#include <math.h>

#include <algorithm>

#include <cuda_bf16.h>

#include "paged.cuh"
#include "tma.cuh"

namespace llms {

constexpr int kTile = 16;                         // tokens per tile: the 16 side of an MMA
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

__device__ __forceinline__ uint32_t transpose8x8(uint32_t x)
{
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// (lo, hi) as a pair of 16-bit values, lo in the low half, each rounded to nearest
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

// CTAs of a cluster per item, or 0: runs.  As many CTAs as leave a warp one tile, up to eight and up to `rounds` rounds of the
// GPU (per_sm: CTAs that an SM has room for); not if a warp is left with more than four tiles, in a batch (whose sequences are
// seldom all as long as max_len) eight.
inline int decode_item_ctas(const DecodeArgs &a, int per_sm, int rounds, int tile, int warps)
{
    if (a.mass_out && a.blocks > 1) return 0;                 // a token's weight is made of several items' logits
    const int seen = a.window > 0 ? (int)std::min<int64_t>(a.max_len, (int64_t)a.window + tile - 1) : a.max_len, tiles = (seen + tile - 1) / tile;
    const int64_t n_items = (int64_t)a.n_seqs * a.Hkv * a.blocks, room = (int64_t)sm_count() * per_sm * rounds;
    int ctas = 1;
    while (ctas < 8 && ctas * warps < tiles && n_items * ctas * 2 <= room) ctas *= 2;
    return n_items * ctas <= room && tiles <= ctas * warps * (a.n_seqs > 1 ? 8 : 4) ? ctas : 0;
}

}  // namespace llms
