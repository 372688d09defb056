// Attention of one new token per sequence over the paged cache (a pool of chunk slots), one layer per call.
//
// Mathematics.  With logits in units of log2 (v = scale * log2(e) * <q, k>), a run of tokens leaves, per query head, the
// triple (m, l, O) = (max v, sum 2^(v - m), sum 2^(v - m) V); two runs join as m = max, l and O scaled by 2^(m_i - m) and
// added, in any split of the tokens.  out = O / l, lse = ln 2 * (m + log2 l), weight of a token = 2^(v - m) / l.
//
// Bound.  Every K and V element is used for 2 multiply-adds per query head that reads it: 1 flop per byte and query head of
// the group, so with groups of 1 to some tens the read of K and V from HBM bounds it, not the arithmetic.  Warp-level MMAs
// with eight query rows (m16n8k16, tokens or channels on the 16 side) keep that arithmetic far below the memory time;
// a tcgen05 MMA has at least 64 rows and would multiply mostly padding.
//
// Split.  The work is the sequence of all 16-token tiles of all (sequence, KV head) items of the batch.  It is cut into equal
// runs, one per CTA, and each into equal runs per warp, whatever the sequences' lengths: the lengths are known on the
// device only, and equal runs balance ragged batches and long single contexts alike.  A warp feeds itself: its lane 0
// (with chunks shorter than a tile, a lane per piece of the tile) asks for tiles a ring of stages ahead by TMA, 64
// channels x 16 tokens at a time, 128-byte swizzled; nothing is exchanged between warps until their runs end.  An item that
// lies in one warp's run is finished by it; the pieces of the others are joined in shared memory at the end of the CTA,
// and where an item spans CTAs, from the workspace by join_kernel.  All sums have a fixed order: repeated calls agree
// bit for bit.
#include <math.h>

#include <algorithm>

#include <cuda_bf16.h>

#include "llms_internal.cuh"
#include "tma.cuh"

namespace llms {

constexpr int kTile = 16;                         // tokens per tile: the 16 side of an MMA
constexpr int kMaxStages = 8;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// For the product with V a weight 2^(v - m) goes into the MMA as kLift times its value, as a sum of two 16-bit values
// hi + lo.  hi is cut off a little below the weight, so that lo is never 0: a value of V that is infinite then gives an
// infinity, not 0 * inf.  The lift (a power of two, taken back exactly at the end) keeps lo a normal fp16 number for
// weights down to 2^-26 of the largest.  Together the two carry 21 (fp16) or 16 (bf16) bits; one 16-bit value alone would
// add an error as large as the rounding of the output itself.
constexpr float kLift = 16384.0f;

struct DecodeArgs {
    const uint16_t *q, *k_new, *v_new;
    uint16_t *k, *v, *out;                        // K and V of the layer: base of KV head 0
    const int32_t *table, *lens;
    float *lse, *row_lse;                         // caller's (may be NULL), natural; workspace's, in units of log2
    const float *mass_in;
    float *mass_out;
    float *logits;                                // workspace: v of every (sequence, KV head, token, query head), for the masses
    float *part;                                  // workspace: two partial results per CTA
    int32_t *plan;                                // workspace: first tile of every sequence, then the tiles of the batch
    int64_t q_stride, new_stride, stride_h, mass_stride;
    int table_stride, n_seqs, max_len, window, Hkv, Hq, group, d, chunk_len, n_slots;
    int blocks;                                   // blocks of query rows per KV head
    int piece;                                    // tokens per TMA box: the largest power of two up to 16 that divides chunk_len
    int stages, rows, ctas;                       // ring stages, query rows kept per partial result, CTAs of the main kernel
    int min_tiles;                                // a CTA takes at least this many tiles
    float scale_log2;
};

// A sequence's tokens as tiles: the first tile is the one that the window begins in.
struct SeqTiles {
    int len, first, tile0, n;                     // tokens; first token seen; its tile; tiles (0 for an empty or invalid row)
};
__device__ __forceinline__ SeqTiles seq_tiles(const DecodeArgs &a, int len)
{
    SeqTiles s;
    s.len = len < 0 || len > a.max_len ? 0 : len;
    s.first = a.window > 0 && s.len > a.window ? s.len - a.window : 0;
    s.tile0 = s.first / kTile;
    s.n = (s.len + kTile - 1) / kTile - s.tile0;
    return s;
}

// CTAs that share the batch's tiles, and who has which
__device__ __forceinline__ int working_ctas(const DecodeArgs &a, int total) { return min(a.ctas, max(1, total / a.min_tiles)); }
__device__ __forceinline__ int run_begin(int total, int parts, int i) { return (int)((int64_t)total * i / parts); }
__device__ __forceinline__ int run_of(int total, int parts, int tile) { return (int)((((int64_t)tile + 1) * parts - 1) / total); }

// Where in the batch a tile lies; advanced tile by tile.
struct Cursor {
    SeqTiles s;
    int b, hb, tile;                              // sequence, KV head * blocks + block of query rows, tile of the item
    __device__ __forceinline__ void start(const DecodeArgs &a, const int32_t *plan, int idx)
    {
        int lo = 0, hi = a.n_seqs - 1;            // the last sequence that begins at or before idx
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (plan[mid] <= idx) lo = mid;
            else hi = mid - 1;
        }
        b = lo;
        s = seq_tiles(a, __ldg(a.lens + b));
        const int r = idx - plan[b];
        hb = r / s.n;
        tile = r - hb * s.n;
    }
    __device__ __forceinline__ void next(const DecodeArgs &a)
    {
        if (++tile < s.n) return;
        tile = 0;
        if (++hb < a.Hkv * a.blocks) return;
        hb = 0;
        do {
            if (++b >= a.n_seqs) return;
            s = seq_tiles(a, __ldg(a.lens + b));
        } while (s.n == 0);
    }
};

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap *map, int c0, int c1, int c2, unsigned long long *bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 :: "r"(dst), "l"(map), "r"(smem_u32(bar)), "r"(c0), "r"(c1), "r"(c2) : "memory");
}
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_trans(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
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

template <int DB> struct DecodeShape {
    static constexpr int kWarps = DB <= 2 ? 8 : 4;            // warps x stages x tile fill the SM's shared memory
    static constexpr int kHalf = DB * kTile * 128;            // K (or V) of a tile
    static constexpr int kStage = 2 * kHalf;
    static constexpr int kCols = DB * 64;                     // channels, rounded up to whole boxes
    static constexpr int kPitch = kCols + 4;                  // floats per row of a piece in shared memory
};

// Shared memory: [1 KiB alignment][warps x stages x tile][first pieces][barriers, piece table][plan].  A warp leaves the piece
// that its run begins with in its own place of the first-piece area, and the one that its run ends with in its own part of
// the ring, which has run dry by then.
// A piece: [rows][kPitch] floats, O in the first kCols columns of a row, then m and l.
template <int DB>
__host__ __device__ constexpr size_t piece_floats(int rows) { return (size_t)rows * DecodeShape<DB>::kPitch; }

struct WarpSlots {
    unsigned long long full[kMaxStages];
};

template <bool BF, int DB, int NT>
__global__ void __launch_bounds__(DecodeShape<DB>::kWarps * 32, 1)
decode_kernel(const DecodeArgs a, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v)
{
    using S = DecodeShape<DB>;
    constexpr int W = S::kWarps, KS = DB * 4;                 // k-steps over the channels; also 16-channel tiles of the output
    extern __shared__ unsigned char smem_raw[];
    unsigned char *ring = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const size_t ring_bytes = (size_t)W * a.stages * S::kStage;
    float *first_pieces = reinterpret_cast<float *>(ring + ring_bytes);
    WarpSlots *slots = reinterpret_cast<WarpSlots *>(first_pieces + (size_t)W * piece_floats<DB>(a.rows));
    int32_t *plan = reinterpret_cast<int32_t *>(slots + W);   // n_seqs + 1
    __shared__ int piece_item[2 * W], piece_at[2 * W];        // item of every piece left behind (-1: none) and its first tile
    __shared__ int warp_sum[W];
    __shared__ uint32_t gave_up;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    unsigned long long *full = slots[warp].full;
    if (lane == 0) {
        for (int s = 0; s < a.stages; ++s) mbar_init(&full[s], 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        piece_item[2 * warp] = piece_item[2 * warp + 1] = -1;
    }
    if (threadIdx.x == 0) gave_up = 0;

    // tiles before every sequence
    const int per_seq = a.Hkv * a.blocks;
    {
        int base = 0;
        for (int b0 = 0; b0 < a.n_seqs; b0 += W * 32) {
            const int b = b0 + threadIdx.x;
            int v = b < a.n_seqs ? seq_tiles(a, __ldg(a.lens + b)).n * per_seq : 0;
            int incl = v;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int up = __shfl_up_sync(0xffffffffu, incl, d);
                if (lane >= d) incl += up;
            }
            if (lane == 31) warp_sum[warp] = incl;
            __syncthreads();
            int before = base;
            for (int w = 0; w < W; ++w) {
                if (w < warp) before += warp_sum[w];
                base += warp_sum[w];
            }
            if (b < a.n_seqs) plan[b] = before + incl - v;
            __syncthreads();
        }
        if (threadIdx.x == 0) plan[a.n_seqs] = base;
        __syncthreads();
    }
    const int total = plan[a.n_seqs];
    if (blockIdx.x == 0)
        for (int b = threadIdx.x; b <= a.n_seqs; b += W * 32) a.plan[b] = plan[b];

    // rows of the batch without tokens: zeros, or NaN where the length is invalid
    for (int b = blockIdx.x; b < a.n_seqs; b += gridDim.x) {
        if (plan[b + 1] != plan[b]) continue;
        const bool bad = __ldg(a.lens + b) != 0;
        const uint16_t fill = bad ? (uint16_t)(BF ? 0x7fc0 : 0x7e00) : (uint16_t)0;
        for (int i = threadIdx.x; i < a.Hq * a.d; i += W * 32) a.out[(int64_t)b * a.Hq * a.d + i] = fill;
        for (int i = threadIdx.x; i < a.Hq; i += W * 32) {
            const float l = bad ? NAN : -INFINITY;
            a.row_lse[(int64_t)b * a.Hq + i] = l;
            if (a.lse) a.lse[(int64_t)b * a.Hq + i] = l;
        }
    }

    const int C = working_ctas(a, total), cta = blockIdx.x;
    const int run0 = cta < C ? run_begin(total, C, cta) : total, run1 = cta < C ? run_begin(total, C, cta + 1) : total;
    const int w0 = run0 + run_begin(run1 - run0, W, warp), w1 = run0 + run_begin(run1 - run0, W, warp + 1);

    if (w0 < w1) {
        unsigned char *my_ring = ring + (size_t)warp * a.stages * S::kStage;
        const uint32_t ring_addr = smem_u32(my_ring);
        // ---- feeding: lane i asks for piece i of a tile
        Cursor pc;
        pc.start(a, plan, w0);
        int issued = w0, stage_in = 0;
        uint32_t poisoned = 0;                                // stages whose tile has a slot outside the pool
        const int n_pieces = kTile / a.piece;
        int p_tok, p_slot = 0;
        bool p_need;
        auto look_up = [&] {                                  // slot of this lane's piece of the tile that is asked for next
            p_tok = (pc.s.tile0 + pc.tile) * kTile + lane * a.piece;
            p_need = lane < n_pieces && p_tok < pc.s.len && p_tok + a.piece > pc.s.first;
            if (p_need) p_slot = __ldg(a.table + (int64_t)pc.b * a.table_stride + p_tok / a.chunk_len);
        };
        auto issue = [&] {
            const bool inside = p_need && (unsigned)p_slot < (unsigned)a.n_slots;
            const uint32_t ok = __ballot_sync(0xffffffffu, inside), bad = __ballot_sync(0xffffffffu, p_need && !inside);
            unsigned long long *bar = &full[stage_in];
            poisoned = (poisoned & ~(1u << stage_in)) | (bad ? 1u << stage_in : 0u);
            if (lane == 0) mbar_expect_tx(bar, __popc(ok) * a.piece * 128 * DB * 2);
            __syncwarp();
            if (inside) {
                const int row = p_slot * a.chunk_len + p_tok % a.chunk_len, h = pc.hb / a.blocks;
                const uint32_t dst = ring_addr + stage_in * S::kStage + lane * a.piece * 128;
#pragma unroll
                for (int i = 0; i < DB; ++i) {
                    tma_load_3d(dst + i * kTile * 128, &map_k, i * 64, row, h, bar);
                    tma_load_3d(dst + S::kHalf + i * kTile * 128, &map_v, i * 64, row, h, bar);
                }
            }
            ++issued;
            stage_in = stage_in + 1 == a.stages ? 0 : stage_in + 1;
            if (issued < w1) {
                pc.next(a);
                look_up();
            }
        };
        look_up();
        for (int s = 0; s < a.stages && issued < w1; ++s) issue();

        // ---- the arithmetic
        Cursor cc;
        cc.start(a, plan, w0);
        uint32_t qf[KS][NT][2];
        float o[KS][NT][4];
        float m[NT][2], l[NT][2];
        int stage = 0, phase = 0;
        bool fresh = true;
        // addresses inside a tile: K as stored (rows = tokens), V transposed (rows = channels)
        const int k_row = lane & 15, v_row = (lane & 7) + ((lane >> 4) << 3);
        const uint32_t k_base = k_row * 128, v_base = v_row * 128;
        const uint32_t k_c = lane >> 4, v_c = (lane >> 3) & 1, k_x = k_row & 7, v_x = v_row & 7;

        for (int idx = w0; idx < w1; ++idx) {
            const int h = cc.hb / a.blocks, rb = cc.hb - h * a.blocks;
            if (fresh) {
                fresh = false;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const int r = rb * 8 * NT + nt * 8 + (lane >> 2);
                    const uint16_t *q = a.q + cc.b * a.q_stride + (int64_t)(h * a.group + r) * a.d + (lane & 3) * 2;
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const int c = ks * 16 + i * 8;
                            qf[ks][nt][i] = r < a.group && c + (lane & 3) * 2 < a.d ? __ldg(reinterpret_cast<const uint32_t *>(q + c)) : 0u;
                        }
                    m[nt][0] = m[nt][1] = -INFINITY;
                    l[nt][0] = l[nt][1] = 0.0f;
#pragma unroll
                    for (int t = 0; t < KS; ++t)
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[t][nt][i] = 0.0f;
                }
            }
            const int tok0 = (cc.s.tile0 + cc.tile) * kTile;
            const uint32_t k_tile = ring_addr + stage * S::kStage, v_tile = k_tile + S::kHalf;
            const bool poison = !mbar_wait(&full[stage], phase, &gave_up) || (poisoned >> stage & 1);

            const bool newest = a.k_new && tok0 + kTile >= cc.s.len;
            const bool edge = tok0 < cc.s.first || tok0 + kTile > cc.s.len;
            if (newest || edge) {
                // rows that are not seen: V is cleared, so that 0 * (whatever lies there) is 0.  The newest token's row:
                // what the caller gave, here and in the pool
                unsigned char *v_mem = my_ring + stage * S::kStage + S::kHalf;
                if (edge)
                    for (int i = lane; i < DB * kTile * 8; i += 32) {
                        const int t = tok0 + (i >> 3) % kTile;
                        if (t < cc.s.first || t >= cc.s.len) *reinterpret_cast<uint4 *>(v_mem + i * 16) = make_uint4(0, 0, 0, 0);
                    }
                if (newest) {
                    const int t = cc.s.len - 1, r = t - tok0;
                    const int slot = __ldg(a.table + (int64_t)cc.b * a.table_stride + t / a.chunk_len);
                    const bool inside = (unsigned)slot < (unsigned)a.n_slots;
                    const int64_t at = (int64_t)h * a.stride_h + ((int64_t)slot * a.chunk_len + t % a.chunk_len) * a.d;
                    const int64_t from = cc.b * a.new_stride + (int64_t)h * a.d;
                    for (int c = lane; c < a.d / 8; c += 32) {
                        const uint4 kn = __ldg(reinterpret_cast<const uint4 *>(a.k_new + from) + c);
                        const uint4 vn = __ldg(reinterpret_cast<const uint4 *>(a.v_new + from) + c);
                        unsigned char *mem = v_mem + (c >> 3) * kTile * 128 + r * 128 + (((c & 7) ^ (r & 7)) << 4);
                        *reinterpret_cast<uint4 *>(mem - S::kHalf) = kn;
                        *reinterpret_cast<uint4 *>(mem) = vn;
                        if (inside && rb == 0) {
                            reinterpret_cast<uint4 *>(a.k + at)[c] = kn;
                            reinterpret_cast<uint4 *>(a.v + at)[c] = vn;
                        }
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // before TMA fills this stage again
                __syncwarp();
            }

            // logits: tokens x query rows, two chains of accumulators
            float s[NT][4], s2[NT][4];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[nt][i] = s2[nt][i] = 0.0f;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                uint32_t f[4];
                const uint32_t c = (ks & 3) * 2 + k_c;
                ldsm4(f, k_tile + (ks >> 2) * kTile * 128 + k_base + ((c ^ k_x) << 4));
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) mma<BF>(ks & 1 ? s2[nt] : s[nt], f, qf[ks][nt][0], qf[ks][nt][1]);
            }
            uint32_t p_hi[NT][2], p_lo[NT][2];
            bool moved = false;
            float keep[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                float v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[i] = (s[nt][i] + s2[nt][i]) * a.scale_log2;
                    if (poison) v[i] = NAN;
                }
                if (edge) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int t = tok0 + (lane >> 2) + (i >> 1) * 8;
                        if (t < cc.s.first || t >= cc.s.len) v[i] = -INFINITY;
                    }
                }
                if (a.logits) {
                    const int r0 = rb * 8 * NT + nt * 8 + (lane & 3) * 2;
                    float *to = a.logits + (((int64_t)cc.b * a.Hkv + h) * a.max_len + tok0) * a.group + r0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int t = (lane >> 2) + (i >> 1) * 8;
                        if (r0 + (i & 1) < a.group && tok0 + t < cc.s.len) to[(int64_t)t * a.group + (i & 1)] = v[i];
                    }
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float top = fmaxf(v[i], v[i + 2]);
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                    top = fmaxf(top, m[nt][i]);
                    const float ref = top == -INFINITY ? 0.0f : top;
                    keep[nt][i] = top == m[nt][i] ? 1.0f : exp2_fast(m[nt][i] - ref);
                    moved |= top != m[nt][i];
                    m[nt][i] = top;
                    v[i] = exp2_fast(v[i] - ref);
                    v[i + 2] = exp2_fast(v[i + 2] - ref);
                    l[nt][i] = __fmaf_rn(l[nt][i], keep[nt][i], v[i] + v[i + 2]);
                }
                constexpr float kCut = kLift * (BF ? 1.0f - 1.0f / 512.0f : 1.0f - 1.0f / 4096.0f);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint32_t hi = pack_cut<BF>(v[2 * i] * kCut, v[2 * i + 1] * kCut);
                    const float2 back = unpack<BF>(hi);
                    const uint32_t lo = pack_round<BF>(__fmaf_rn(v[2 * i], kLift, -back.x), __fmaf_rn(v[2 * i + 1], kLift, -back.y));
                    p_hi[nt][i] = transpose8x8(hi);
                    p_lo[nt][i] = transpose8x8(lo);
                }
            }
            if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
                for (int t = 0; t < KS; ++t)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[t][nt][i] *= keep[nt][i & 1];
            }
#pragma unroll
            for (int t = 0; t < KS; ++t) {
                uint32_t f[4];
                const uint32_t c = (t & 3) * 2 + v_c;
                ldsm4_trans(f, v_tile + (t >> 2) * kTile * 128 + v_base + ((c ^ v_x) << 4));
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    mma<BF>(o[t][nt], f, p_hi[nt][0], p_hi[nt][1]);
                    mma<BF>(o[t][nt], f, p_lo[nt][0], p_lo[nt][1]);
                }
            }
            __syncwarp();
            if (issued < w1) issue();
            if (++stage == a.stages) {
                stage = 0;
                phase ^= 1;
            }

            // the end of the item, or of this warp's run
            const bool item_ends = cc.tile + 1 == cc.s.n;
            if (item_ends || idx + 1 == w1) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int d = 4; d < 32; d <<= 1) l[nt][i] += __shfl_xor_sync(0xffffffffu, l[nt][i], d);
                const int item_begin = idx - cc.tile;
                if (item_ends && item_begin >= w0) {
                    // complete: to the output, two channels of a row per lane
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        float inv[2];
#pragma unroll
                        for (int i = 0; i < 2; ++i) inv[i] = l[nt][i] == 0.0f ? 0.0f : (1.0f / kLift) / l[nt][i];
                        const int r = rb * 8 * NT + nt * 8 + (lane >> 2);
                        uint16_t *to = a.out + ((int64_t)cc.b * a.Hq + h * a.group + r) * a.d + (lane & 3) * 2;
#pragma unroll
                        for (int t = 0; t < KS; ++t)
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                const uint32_t x = transpose8x8(pack_round<BF>(o[t][nt][2 * i] * inv[0], o[t][nt][2 * i + 1] * inv[1]));
                                if (r < a.group && t * 16 + i * 8 + (lane & 3) * 2 < a.d) *reinterpret_cast<uint32_t *>(to + t * 16 + i * 8) = x;
                            }
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const int r2 = rb * 8 * NT + nt * 8 + (lane & 3) * 2 + i;
                            if (lane < 4 && r2 < a.group) {
                                const int64_t at = (int64_t)cc.b * a.Hq + h * a.group + r2;
                                const float lg = l[nt][i] == 0.0f ? -INFINITY : m[nt][i] + log2f(l[nt][i]);
                                a.row_lse[at] = lg;
                                if (a.lse) a.lse[at] = lg * kLn2;
                            }
                        }
                    }
                } else {
                    // a piece: the run's last one, unless the item ends here (then it began before the run)
                    const int which = item_ends ? 0 : 1;
                    float *to = which == 0 ? first_pieces + warp * piece_floats<DB>(a.rows) : reinterpret_cast<float *>(my_ring);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int r = nt * 8 + (lane & 3) * 2 + (i & 1);
                            if (r < a.rows) {
#pragma unroll
                                for (int t = 0; t < KS; ++t) to[r * S::kPitch + t * 16 + (i >> 1) * 8 + (lane >> 2)] = o[t][nt][i];
                                if (lane < 4 && i < 2) {
                                    to[r * S::kPitch + S::kCols] = m[nt][i];
                                    to[r * S::kPitch + S::kCols + 1] = l[nt][i];
                                }
                            }
                        }
                    if (lane == 0) {
                        piece_item[2 * warp + which] = cc.b * per_seq + cc.hb;
                        piece_at[2 * warp + which] = item_begin;
                    }
                }
                fresh = true;
            }
            cc.next(a);
        }
    }
    __syncthreads();
    grid_launch_dependents();

    // ---- the pieces that the warps left: runs of pieces of one item, joined; all threads share the elements
    const int row_elems = S::kCols;
    for (int p = 0; p < 2 * W;) {
        const int item = piece_item[p];
        if (item < 0) {
            ++p;
            continue;
        }
        int end = p + 1;
        while (end < 2 * W && (piece_item[end] == item || piece_item[end] < 0)) ++end;
        const int b = item / per_seq, hb = item - b * per_seq, h = hb / a.blocks, rb = hb - h * a.blocks;
        const int begin = piece_at[p], finish = begin + (plan[b + 1] - plan[b]) / per_seq;
        const bool whole = begin >= run0 && finish <= run1;
        float *part = a.part + ((int64_t)cta * 2 + (begin < run0 ? 0 : 1)) * a.rows * (S::kCols + 2);
        for (int e = threadIdx.x; e < a.rows * row_elems; e += W * 32) {
            const int r = e / row_elems, c = e - r * row_elems;
            if (rb * 8 * NT + r >= a.group) continue;
            float top = -INFINITY;
            for (int i = p; i < end; ++i) {
                if (piece_item[i] < 0) continue;
                const float *at = i & 1 ? reinterpret_cast<const float *>(ring + (size_t)(i >> 1) * a.stages * S::kStage)
                                        : first_pieces + (i >> 1) * piece_floats<DB>(a.rows);
                top = fmaxf(top, at[r * S::kPitch + S::kCols]);
            }
            const float ref = top == -INFINITY ? 0.0f : top;
            float sum = 0.0f, acc = 0.0f;
            for (int i = p; i < end; ++i) {
                if (piece_item[i] < 0) continue;
                const float *at = i & 1 ? reinterpret_cast<const float *>(ring + (size_t)(i >> 1) * a.stages * S::kStage)
                                        : first_pieces + (i >> 1) * piece_floats<DB>(a.rows);
                const float f = exp2_fast(at[r * S::kPitch + S::kCols] - ref);
                sum = __fmaf_rn(f, at[r * S::kPitch + S::kCols + 1], sum);
                acc = __fmaf_rn(f, at[r * S::kPitch + c], acc);
            }
            if (whole) {
                const int64_t row = (int64_t)b * a.Hq + h * a.group + rb * 8 * NT + r;
                if (c < a.d) {
                    const float x = sum == 0.0f ? 0.0f : acc * (1.0f / kLift) / sum;
                    a.out[row * a.d + c] = (uint16_t)pack_round<BF>(x, x);
                }
                if (c == 0) {
                    const float lg = sum == 0.0f ? -INFINITY : top + log2f(sum);
                    a.row_lse[row] = lg;
                    if (a.lse) a.lse[row] = lg * kLn2;
                }
            } else {
                part[(int64_t)r * (S::kCols + 2) + c] = acc;
                if (c < 2) part[(int64_t)r * (S::kCols + 2) + S::kCols + c] = c == 0 ? top : sum;
            }
        }
        p = end;
    }
}

// Items that span CTAs: block (c, r) joins query row r of the item that begins in CTA c's run and goes on behind it (if one
// does), threads over channels and, where there are many pieces, over them.
constexpr int kJoinThreads = 256;
template <bool BF>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const DecodeArgs a, int cols)
{
    __shared__ float s_acc[kJoinThreads], s_top[kJoinThreads / 32], s_sum[kJoinThreads / 32];
    grid_dependency_wait();
    const int per_seq = a.Hkv * a.blocks, c0 = blockIdx.x, r = blockIdx.y;
    const int total = a.plan[a.n_seqs], C = working_ctas(a, total);
    if (c0 + 1 >= C) return;
    const int begin_run = run_begin(total, C, c0), border = run_begin(total, C, c0 + 1);
    Cursor last;                                              // the run's last tile
    last.start(a, a.plan, border - 1);
    const int b = last.b, h = last.hb / a.blocks, rb = last.hb - h * a.blocks, row_in_group = rb * a.rows + r;
    const int begin = border - 1 - last.tile, tiles = last.s.n;
    if (begin < begin_run || begin + tiles <= border || row_in_group >= a.group) return;
    const int c1 = run_of(total, C, begin + tiles - 1);
    const int64_t stride = (int64_t)a.rows * (cols + 2);
    const float *base = a.part + (int64_t)r * (cols + 2);
    // first CTA's last piece, then the following CTAs' first pieces
    auto at = [&](int c) { return base + ((int64_t)c * 2 + (c == c0 ? 1 : 0)) * stride; };
    float top = -INFINITY;
    for (int c = c0 + threadIdx.x; c <= c1; c += kJoinThreads) top = fmaxf(top, at(c)[cols]);
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    if ((threadIdx.x & 31) == 0) s_top[threadIdx.x >> 5] = top;
    __syncthreads();
    for (int w = 0; w < kJoinThreads / 32; ++w) top = fmaxf(top, s_top[w]);
    const float ref = top == -INFINITY ? 0.0f : top;
    float sum = 0.0f;
    for (int c = c0 + threadIdx.x; c <= c1; c += kJoinThreads) sum = __fmaf_rn(exp2_fast(at(c)[cols] - ref), at(c)[cols + 1], sum);
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    if ((threadIdx.x & 31) == 0) s_sum[threadIdx.x >> 5] = sum;
    __syncthreads();
    sum = 0.0f;
    for (int w = 0; w < kJoinThreads / 32; ++w) sum += s_sum[w];
    const int slices = kJoinThreads / cols, slice = threadIdx.x / cols, col = threadIdx.x - slice * cols;
    float acc = 0.0f;
    if (slice < slices)
        for (int c = c0 + slice; c <= c1; c += slices) acc = __fmaf_rn(exp2_fast(at(c)[cols] - ref), at(c)[col], acc);
    s_acc[threadIdx.x] = acc;
    __syncthreads();
    const int64_t row = (int64_t)b * a.Hq + h * a.group + row_in_group;
    if (slice == 0 && col < a.d) {
        for (int i = 1; i < slices; ++i) acc += s_acc[i * cols + col];
        const float x = sum == 0.0f ? 0.0f : acc * (1.0f / kLift) / sum;
        a.out[row * a.d + col] = (uint16_t)pack_round<BF>(x, x);
    }
    if (threadIdx.x == 0) {
        const float lg = sum == 0.0f ? -INFINITY : top + log2f(sum);
        a.row_lse[row] = lg;
        if (a.lse) a.lse[row] = lg * kLn2;
    }
}

// Weights of all tokens: the logits left by the main kernel against the rows' log-sums.
__global__ void __launch_bounds__(256) mass_kernel(const DecodeArgs a)
{
    grid_dependency_wait();
    const int b = blockIdx.z, h = blockIdx.y, n = __ldg(a.lens + b), t = blockIdx.x * 256 + threadIdx.x;
    if (n > a.max_len || t >= n) return;
    const int first = a.window > 0 && n > a.window ? n - a.window : 0;
    const int64_t at = (int64_t)b * a.Hkv + h;
    float w = 0.0f;
    if (t >= first) {
        const float *v = a.logits + (at * a.max_len + t) * a.group, *l = a.row_lse + at * a.group;
        for (int g = 0; g < a.group; ++g) {
            const float lg = l[g];
            w += lg == -INFINITY ? 0.0f : exp2_fast(v[g] - lg);
        }
    }
    a.mass_out[at * a.mass_stride + t] = (a.mass_in ? a.mass_in[at * a.mass_stride + t] : 0.0f) + w;
}

struct DecodeLayout {
    int blocks_of_64, nt, rows, blocks;
    uint64_t off_lse, off_plan, off_part, off_logits, total;
};

static DecodeLayout decode_layout(const llms_kv_desc &d, int n_seqs, int max_len, bool with_mass)
{
    DecodeLayout t;
    const int group = d.n_q_heads / d.n_kv_heads;
    t.blocks_of_64 = (d.head_dim + 63) / 64;
    t.nt = group > 8 ? 2 : 1;
    t.rows = std::min(group, 8 * t.nt);
    t.blocks = (group + 8 * t.nt - 1) / (8 * t.nt);
    t.off_lse = 0;
    t.off_plan = round_up((uint64_t)n_seqs * d.n_q_heads * 4, 256);
    t.off_part = t.off_plan + round_up((uint64_t)(n_seqs + 1) * 4, 256);
    t.off_logits = t.off_part + round_up((uint64_t)sm_count() * 2 * t.rows * (t.blocks_of_64 * 64 + 2) * 4, 256);
    t.total = t.off_logits + (with_mass ? round_up((uint64_t)n_seqs * d.n_q_heads * (uint64_t)max_len * 4, 256) : 0);
    return t;
}

// A layer's K or V half as (channel, token, KV head), boxes of 64 channels x `piece` tokens; channels past head_dim read as 0
static bool encode_half(CUtensorMap *map, const void *base, bool bf16, const llms_kv_desc &d, int piece)
{
    const cuuint64_t dims[3] = {(cuuint64_t)d.head_dim, (cuuint64_t)d.n_tokens, (cuuint64_t)d.n_kv_heads};
    const cuuint64_t head = d.n_kv_heads == 1 ? (cuuint64_t)d.n_tokens * d.head_dim : (cuuint64_t)d.stride_h;
    const cuuint64_t strides[2] = {(cuuint64_t)d.head_dim * 2, head * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)piece, 1}, elem[3] = {1, 1, 1};
    return tensor_map_encoder()(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void *>(base),
                                dims, strides, box, elem, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                                CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <bool BF, int DB, int NT>
static int launch_decode(DecodeArgs &a, const CUtensorMap &map_k, const CUtensorMap &map_v, cudaStream_t st)
{
    using S = DecodeShape<DB>;
    const size_t fixed = 1024 + S::kWarps * (piece_floats<DB>(a.rows) * 4 + sizeof(WarpSlots)) + round_up((uint64_t)(a.n_seqs + 1) * 4, 16);
    const size_t most = 226 * 1024;
    a.stages = (int)std::min<size_t>(kMaxStages, (most - fixed) / (S::kWarps * S::kStage));
    a.min_tiles = S::kWarps;
    const size_t smem = fixed + (size_t)S::kWarps * a.stages * S::kStage;
    LLMS_CUDA_TRY(cudaFuncSetAttribute(decode_kernel<BF, DB, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    decode_kernel<BF, DB, NT><<<a.ctas, S::kWarps * 32, smem, st>>>(a, map_k, map_v);
    LLMS_CUDA_TRY(cudaGetLastError());
    return LLMS_OK;
}

template <bool BF>
static int launch_decode_shape(DecodeArgs &a, int db, int nt, const CUtensorMap &mk, const CUtensorMap &mv, cudaStream_t st)
{
    switch (db * 2 + nt - 1) {
    case 2: return launch_decode<BF, 1, 1>(a, mk, mv, st);
    case 3: return launch_decode<BF, 1, 2>(a, mk, mv, st);
    case 4: return launch_decode<BF, 2, 1>(a, mk, mv, st);
    case 5: return launch_decode<BF, 2, 2>(a, mk, mv, st);
    case 6: return launch_decode<BF, 3, 1>(a, mk, mv, st);
    case 7: return launch_decode<BF, 3, 2>(a, mk, mv, st);
    case 8: return launch_decode<BF, 4, 1>(a, mk, mv, st);
    case 9: return launch_decode<BF, 4, 2>(a, mk, mv, st);
    default: return LLMS_ERR_UNSUPPORTED;
    }
}

}  // namespace llms

using namespace llms;

extern "C" int llms_decode_workspace_bytes(const llms_kv_desc *desc, int n_seqs, int max_len, int with_mass, uint64_t *nbytes)
{
    const int rc = check_paged(desc, n_seqs, max_len);
    if (rc) return rc;
    if (!nbytes) return LLMS_ERR_INVALID_ARG;
    *nbytes = decode_layout(*desc, n_seqs, max_len, with_mass != 0).total;
    return LLMS_OK;
}

extern "C" int llms_decode_attention(const llms_kv_desc *desc, int dtype, int layer, void *kv, const void *q, int64_t q_stride,
                                     const void *k_new, const void *v_new, int64_t new_stride, const int32_t *chunk_table,
                                     int table_stride, const int32_t *lens, int n_seqs, int max_len, int window, float scale,
                                     void *out, float *lse, const float *mass_in, float *mass_out, int64_t mass_stride,
                                     void *workspace, uint64_t workspace_bytes, void *stream)
{
    int rc = check_paged(desc, n_seqs, max_len);
    if (rc) return rc;
    if (dtype != LLMS_F16 && dtype != LLMS_BF16) return LLMS_ERR_INVALID_ARG;
    if (layer < 0 || layer >= desc->n_layers || window < 0 || !isfinite(scale)) return LLMS_ERR_INVALID_ARG;
    if (n_seqs == 0) return LLMS_OK;
    if (!kv || !q || !chunk_table || !lens || !out || !workspace) return LLMS_ERR_INVALID_ARG;
    if ((k_new == nullptr) != (v_new == nullptr) || (mass_in && !mass_out)) return LLMS_ERR_INVALID_ARG;
    if (table_stride < 1 || (int64_t)table_stride * desc->chunk_len < max_len) return LLMS_ERR_INVALID_ARG;
    if (q_stride < (int64_t)desc->n_q_heads * desc->head_dim) return LLMS_ERR_INVALID_ARG;
    if (k_new && new_stride < (int64_t)desc->n_kv_heads * desc->head_dim) return LLMS_ERR_INVALID_ARG;
    if (mass_out && mass_stride < max_len) return LLMS_ERR_INVALID_ARG;
    if (!aligned(kv, 16) || !aligned(q, 16) || !aligned(out, 16) || q_stride % 8 || !aligned(workspace, 256)) return LLMS_ERR_MISALIGNED;
    if (k_new && (!aligned(k_new, 16) || !aligned(v_new, 16) || new_stride % 8)) return LLMS_ERR_MISALIGNED;
    if (!aligned(chunk_table, 4) || !aligned(lens, 4) || !aligned(lse, 4) || !aligned(mass_in, 4) || !aligned(mass_out, 4)) return LLMS_ERR_MISALIGNED;
    const DecodeLayout lay = decode_layout(*desc, n_seqs, max_len, mass_out != nullptr);
    if (workspace_bytes < lay.total) return LLMS_ERR_BUF_TOO_SMALL;
    if (!tensor_map_encoder()) return LLMS_ERR_UNSUPPORTED;

    DecodeArgs a{};
    a.q = static_cast<const uint16_t *>(q);
    a.k_new = static_cast<const uint16_t *>(k_new);
    a.v_new = static_cast<const uint16_t *>(v_new);
    a.k = static_cast<uint16_t *>(kv) + layer * desc->stride_l;
    a.v = a.k + desc->stride_s;
    a.out = static_cast<uint16_t *>(out);
    a.table = chunk_table; a.lens = lens;
    a.lse = lse;
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    a.row_lse = reinterpret_cast<float *>(ws + lay.off_lse);
    a.plan = reinterpret_cast<int32_t *>(ws + lay.off_plan);
    a.part = reinterpret_cast<float *>(ws + lay.off_part);
    a.logits = mass_out ? reinterpret_cast<float *>(ws + lay.off_logits) : nullptr;
    a.mass_in = mass_in; a.mass_out = mass_out;
    a.q_stride = q_stride; a.new_stride = new_stride; a.stride_h = desc->stride_h; a.mass_stride = mass_stride;
    a.table_stride = table_stride; a.n_seqs = n_seqs; a.max_len = max_len; a.window = window;
    a.Hkv = desc->n_kv_heads; a.Hq = desc->n_q_heads; a.group = a.Hq / a.Hkv; a.d = desc->head_dim;
    a.chunk_len = desc->chunk_len; a.n_slots = n_chunks(*desc);
    a.blocks = lay.blocks; a.rows = lay.rows;
    a.piece = 1;
    while (a.piece < kTile && a.chunk_len % (a.piece * 2) == 0) a.piece *= 2;
    a.scale_log2 = scale * kLog2e;
    a.ctas = sm_count();
    const bool bf16 = dtype == LLMS_BF16;
    CUtensorMap map_k, map_v;
    if (!encode_half(&map_k, a.k, bf16, *desc, a.piece) || !encode_half(&map_v, a.v, bf16, *desc, a.piece)) return LLMS_ERR_UNSUPPORTED;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    rc = bf16 ? launch_decode_shape<true>(a, lay.blocks_of_64, lay.nt, map_k, map_v, st)
              : launch_decode_shape<false>(a, lay.blocks_of_64, lay.nt, map_k, map_v, st);
    if (rc) return rc;
    const dim3 join_grid(a.ctas, a.rows);
    LLMS_CUDA_TRY(launch_dependent(bf16 ? join_kernel<true> : join_kernel<false>, join_grid, dim3(kJoinThreads), 0, st, a, lay.blocks_of_64 * 64));
    if (mass_out) LLMS_CUDA_TRY(launch_dependent(mass_kernel, dim3((max_len + 255) / 256, a.Hkv, n_seqs), dim3(256), 0, st, a));
    return LLMS_OK;
}
