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
// Split.  The work is the sequence of all 16-token tiles of all items (sequence, KV head, up to 16 query heads of it) of the
// batch.  It is cut into equal runs, one per warp, whatever the sequences' lengths: the lengths are known on the device only,
// and equal runs balance ragged batches and long single contexts alike.  A CTA is one warp: nothing is exchanged between
// warps, so none waits for another, and the hardware hands the next run to whichever SM has room (SMs stream at different
// speeds; a fixed split over resident warps left the fastest idle for a third of the time).  A warp feeds itself: its lanes
// look the slots of up to 32 tiles up at once and ask for the tiles by TMA a ring of stages ahead, 128-byte swizzled; with an
// item's first tile come its query rows.  An item that lies in one run is finished by its warp; the pieces of the others go to
// the workspace, where finish_kernel joins them; it also turns the logits into the tokens' weights.  All sums have a fixed
// order: repeated calls agree bit for bit.
//
// Small calls (ITEM) have a cluster of up to eight CTAs of four warps per item instead: its warps take equal parts of the item's
// tiles, join their pieces through the cluster's shared memory and make the weights themselves, so that one kernel
// does it all.
//
// Measured, a B200: 16 contexts of 4096 tokens, 32 heads of 128 channels 164 us (1.075 GB, 6.5 TB/s, the copy bandwidth); one
// grouped-query context of 32768 tokens (8 KV heads of 4 query heads) with weights 34.4 us, of which 8 are finish_kernel's;
// one context of 256 tokens, 4 heads of 64 (ITEM) 5.3 us.
#include <cooperative_groups.h>

#include "decode.cuh"

namespace llms {

namespace cg = cooperative_groups;

constexpr int kQuerySlots = 2;                    // items whose query rows a warp holds: the current one's, the next one's

__device__ __forceinline__ void tma_load_5d(uint32_t dst, const CUtensorMap *map, int c0, int c1, int c2, int c3, int c4, unsigned long long *bar)
{
    asm volatile("cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], [%2];"
                 :: "r"(dst), "l"(map), "r"(smem_u32(bar)), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(c4) : "memory");
}
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
// (lo, hi) as a pair of 16-bit values, lo in the low half, cut off towards zero
template <bool BF>
__device__ __forceinline__ uint32_t pack_cut(float lo, float hi)
{
    uint32_t r;
    if constexpr (BF) asm("cvt.rz.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rz.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
template <int DB> struct DecodeShape : DecodeCols<DB> {
    static constexpr int kStages = DB == 1 ? 4 : 2;
    static constexpr int kHalf = DB * kTile * 128;            // K (or V) of a tile
    static constexpr int kStage = 2 * kHalf;
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

// Bytes of a warp's ring and query rows.
template <int DB>
__host__ __device__ inline int warp_smem(int q_bytes)
{
    return (DecodeShape<DB>::kStages * DecodeShape<DB>::kStage + kQuerySlots * q_bytes + 1023) & ~1023;
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

// Shared memory: [1 KiB alignment][stages x tile][query rows of two items].
//
// MODE: up to 4, 8 or 16 query rows.  With up to 4 the MMA's eight columns hold every row twice: the second copy's lanes
// turn their weights into the lo parts, so hi and lo take one MMA together and the copies' results are added at the end.
template <bool BF, int DB, int MODE, bool ITEM>
__global__ void __launch_bounds__(ITEM ? kItemWarps * 32 : 32) decode_kernel(const DecodeArgs a, const __grid_constant__ CUtensorMap map)
{
    constexpr int NT = MODE == 2 ? 2 : 1;                     // column groups of eight query rows
    constexpr bool kTwin = MODE == 0;
    using S = DecodeShape<DB>;
    constexpr int KS = DB * 4;                                // k-steps over the channels; also 16-channel tiles of the output
    extern __shared__ unsigned char smem_raw[];
    constexpr int W = ITEM ? kItemWarps : 1;
    const int lane = threadIdx.x & 31, warp = ITEM ? threadIdx.x >> 5 : 0, run = blockIdx.x;
    const int warp_bytes = warp_smem<DB>(a.q_bytes);
    unsigned char *const rings = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    unsigned char *const ring = rings + warp * warp_bytes;
    const uint32_t ring_addr = smem_u32(ring), q_addr = ring_addr + S::kStages * S::kStage;
    __shared__ unsigned long long s_full[W][S::kStages];
    unsigned long long *const full = s_full[warp];

    if (lane == 0) {
#pragma unroll
        for (int s = 0; s < S::kStages; ++s) mbar_init(&full[s], 1);
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

        // ---- feeding: lane i looks up piece i % n_pieces of the tile i / n_pieces behind `base`
        const int n_shift = 4 - a.piece_shift, n_pieces = 1 << n_shift, ahead = 32 >> n_shift;   // pieces per tile, tiles per look-up
        int f_row, f_slot, f_q;                                               // row in its chunk, slot, sequence
        bool f_need;
        uint32_t f_h, f_qb;                                                   // KV head (and first query row << 16); bytes of query rows,
                                                                              // which come with the first tile of an item
        auto look_up = [&](int base) {
            const int idx = base + (lane >> n_shift), last = min(base + ahead, w1) - 1;
            f_need = false;
            f_slot = -1;
            f_qb = 0;
            for (;;) {
                if (idx >= f_base && idx <= last && idx < f_base + f_s.n * per_seq) {
                    const int hb = (idx - f_base) / f_s.n, tile = idx - f_base - hb * f_s.n;
                    const int tok = (f_s.tile0 + tile) * kTile + ((lane & (n_pieces - 1)) << a.piece_shift);
                    f_need = tok < f_s.len && tok + (1 << a.piece_shift) > f_s.first;
                    f_h = a.by_blocks(hb);
                    const int chunk = a.by_chunk(tok);
                    f_row = tok - chunk * a.chunk_len;
                    if (f_need) f_slot = __ldg(a.table + (int64_t)f_seq * a.table_stride + chunk);
                    if ((idx == w0 || tile == 0) && (lane & (n_pieces - 1)) == 0) {
                        const int r0 = (hb - f_h * a.blocks) * 8 * NT;
                        f_qb = min(a.rows, a.group - r0) * a.d * 2;
                        f_q = f_seq;
                        f_h |= (uint32_t)r0 << 16;
                    }
                }
                if (last < f_base + f_s.n * per_seq) break;
                skip(f_base + f_s.n * per_seq);
            }
        };
        int base = w0, issued = w0, stage_in = 0, q_issued = 0, q_read = 0;
        uint32_t ok_mask = 0, bad_mask = 0, q_mask = 0, poisoned = 0;         // poisoned: stages whose tile has a slot outside the pool
        bool fetched = false;                                                 // the masks belong to the look-up at `base`
        auto issue = [&] {
            if (!fetched) {
                const bool inside = f_need && (unsigned)f_slot < (unsigned)a.n_slots;
                ok_mask = __ballot_sync(0xffffffffu, inside);
                bad_mask = __ballot_sync(0xffffffffu, f_need && !inside);
                q_mask = __ballot_sync(0xffffffffu, f_qb != 0);
                fetched = true;
            }
            const int lead = (issued - base) << n_shift;
            const bool with_q = q_mask >> lead & 1;
            if (with_q && q_issued - q_read >= kQuerySlots) return;           // its query rows have no place yet
            const uint32_t mine = ((1u << n_pieces) - 1u) << lead;
            unsigned long long *bar = &full[stage_in];
            poisoned = (poisoned & ~(1u << stage_in)) | (bad_mask & mine ? 1u << stage_in : 0u);
            if (lane == lead) mbar_expect_tx(bar, (__popc(ok_mask & mine) << a.piece_shift) * 128 * DB * 2 + f_qb);
            __syncwarp();
            if (mine >> lane & 1) {
                if (ok_mask >> lane & 1) {
                    const int row = f_slot * a.chunk_len + f_row, h = f_h & 0xffff;
                    const uint32_t dst = ring_addr + stage_in * S::kStage + ((lane - lead) << a.piece_shift) * 128;
                    if (a.whole_tile) {
                        tma_load_5d(dst, &map, 0, row, 0, h, 0, bar);
                    } else {
#pragma unroll
                        for (int i = 0; i < DB; ++i) {
                            tma_load_5d(dst + i * kTile * 128, &map, i * 64, row, 0, h, 0, bar);
                            tma_load_5d(dst + S::kHalf + i * kTile * 128, &map, i * 64, row, 0, h, 1, bar);
                        }
                    }
                }
                if (f_qb)
                    bulk_load(q_addr + (q_issued % kQuerySlots) * a.q_bytes,
                              a.q + f_q * a.q_stride + (int64_t)((f_h & 0xffff) * a.group + (f_h >> 16)) * a.d, f_qb, bar);
            }
            q_issued += with_q;
            ++issued;
            stage_in = stage_in + 1 == S::kStages ? 0 : stage_in + 1;
            if (issued - base == ahead && issued < w1) {
                base = issued;
                fetched = false;
                look_up(base);
            }
        };
        look_up(base);
#pragma unroll 1
        for (int s = 0; s < S::kStages && issued < w1; ++s) issue();

        // ---- the arithmetic
        int stage = 0, phase = 0, done = w0;
        bool lost = false;                                    // a copy did not arrive: no more are asked for, those on their way are
                                                              // still waited for, and what has not arrived counts as NaN
        // addresses inside a tile: K as stored (rows = tokens), V transposed (rows = channels)
        const int k_row = lane & 15, v_row = (lane & 7) + ((lane >> 4) << 3);
        const uint32_t k_base = ring_addr + k_row * 128, v_base = ring_addr + S::kHalf + v_row * 128;
        const uint32_t k_c = lane >> 4, v_c = (lane >> 3) & 1, k_x = k_row & 7, v_x = v_row & 7;

#pragma unroll 1
        for (int idx = w0; idx < w1;) {                       // the items that this run has tiles of
            const int h = a.by_blocks(c_hb), rb = c_hb - h * a.blocks;
            const int row0 = rb * 8 * NT, have = min(a.rows, a.group - row0);     // query rows of this item
            const int tile_end = min(c_s.n, c_tile + w1 - idx);
            const bool item_ends = tile_end == c_s.n;
            // the newest token's row, for the item's last tile: lanes hold 16 bytes each of K (first) and V
            uint4 fresh[DB <= 2 ? 1 : 2];
            int fresh_slot = -1;
            const bool append = a.k_new && item_ends;
            if (append) {
#pragma unroll
                for (int i = 0; i < (DB <= 2 ? 1 : 2); ++i) {
                    const int c = lane + i * 32, half = a.d / 8;
                    const uint16_t *from = c < half ? a.k_new : a.v_new;
                    if (c < 2 * half) fresh[i] = __ldg(reinterpret_cast<const uint4 *>(from + c_seq * a.new_stride + (int64_t)h * a.d) + (c < half ? c : c - half));
                }
                fresh_slot = __ldg(a.table + (int64_t)c_seq * a.table_stride + a.by_chunk(c_s.len - 1));
            }
            bool good = idx < issued && warp_wait(&full[stage], phase);
            lost |= !good;
            // query rows as the MMA's second operand; columns beyond the item's rows repeat others (nobody reads their
            // results), channels behind head_dim are 0 like K's there
            uint32_t qf[KS][NT][2];
            float o[KS][NT][4], ref[NT][2], limit[NT][2], l[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const int r = nt * 8 + (lane & (kTwin ? 3 : 7));
                const uint32_t row = q_addr + (q_read % kQuerySlots) * a.q_bytes + min(r, have - 1) * a.d * 2;
#pragma unroll
                for (int ks = 0; ks < KS; ks += 2) {
                    uint32_t f[4];
                    const int c = ks * 16 + (lane >> 3) * 8;
                    ldsm4(f, row + (c < a.d ? c * 2 : 0));
                    qf[ks][nt][0] = ks * 16 < a.d ? f[0] : 0u;
                    qf[ks][nt][1] = ks * 16 < a.d ? f[1] : 0u;
                    qf[ks + 1][nt][0] = ks * 16 + 16 < a.d ? f[2] : 0u;
                    qf[ks + 1][nt][1] = ks * 16 + 16 < a.d ? f[3] : 0u;
                }
                ref[nt][0] = ref[nt][1] = 0.0f;
                limit[nt][0] = limit[nt][1] = -INFINITY;      // reference + kSlack; -inf: no logit yet
                l[nt][0] = l[nt][1] = 0.0f;
#pragma unroll
                for (int t = 0; t < KS; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[t][nt][i] = 0.0f;
            }
            __syncwarp();
            ++q_read;
            float *logits = nullptr;
            if (a.logits) logits = a.logits + ((int64_t)c_seq * a.Hkv + h) * a.max_len * a.group + row0 + (lane & 3) * 2;
            const int tile_begin = c_tile;

#pragma unroll 1
            for (int tile = tile_begin; tile < tile_end; ++tile) {
                if (tile != tile_begin) {
                    good = done < issued && warp_wait(&full[stage], phase);
                    lost |= !good;
                }
                const int tok0 = (c_s.tile0 + tile) * kTile;
                const uint32_t at = stage * S::kStage;
                const bool poison = !good || (poisoned >> stage & 1);
                // tiles that hold places nobody sees, the newest token, or a slot outside the pool
                const bool special = poison || tok0 < c_s.first || tok0 + kTile > c_s.len || (append && tile + 1 == c_s.n);
                if (special) {
                    // rows that are not seen: V is cleared, so that 0 * (whatever lies there) is 0.  The newest token's row:
                    // what the caller gave, here and in the pool
                    unsigned char *mem = ring + at;
#pragma unroll 1
                    for (int i = lane; i < DB * kTile * 8; i += 32) {
                        const int t = tok0 + (i >> 3) % kTile;
                        if (t < c_s.first || t >= c_s.len) *reinterpret_cast<uint4 *>(mem + S::kHalf + i * 16) = make_uint4(0, 0, 0, 0);
                    }
                    if (append && tile + 1 == c_s.n) {
                        const int t = c_s.len - 1, r = t - tok0;
                        const bool inside = (unsigned)fresh_slot < (unsigned)a.n_slots && rb == 0;
                        const int64_t to = (int64_t)h * a.stride_h + ((int64_t)fresh_slot * a.chunk_len + (t - a.by_chunk(t) * a.chunk_len)) * a.d;
#pragma unroll
                        for (int i = 0; i < (DB <= 2 ? 1 : 2); ++i) {
                            const int half = a.d / 8, cv = lane + i * 32, c = cv < half ? cv : cv - half;
                            if (cv < 2 * half) {
                                *reinterpret_cast<uint4 *>(mem + (cv < half ? 0 : S::kHalf) + (c >> 3) * kTile * 128 + r * 128 + (((c & 7) ^ (r & 7)) << 4)) = fresh[i];
                                if (inside) reinterpret_cast<uint4 *>((cv < half ? a.k : a.v) + to)[c] = fresh[i];
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
                    ldsm4(f, k_base + at + (ks >> 2) * kTile * 128 + ((((ks & 3) * 2 + k_c) ^ k_x) << 4));
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma<BF>(ks & 1 ? s2[nt] : s[nt], f, qf[ks][nt][0], qf[ks][nt][1]);
                }
                bool over = false;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[nt][i] = (s[nt][i] + s2[nt][i]) * a.scale_log2;
                if (special) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int t = tok0 + (lane >> 2) + (i >> 1) * 8;
                            if (poison) s[nt][i] = NAN;
                            if (t < c_s.first || t >= c_s.len) s[nt][i] = -INFINITY;
                        }
                }
                if (logits) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int i = 0; i < 4; i += 2) {
                            const int t = tok0 + (lane >> 2) + i * 4, r = nt * 8 + (lane & 3) * 2;
                            float *to = logits + (int64_t)t * a.group + nt * 8;
                            if (t >= c_s.len || r >= have) continue;
                            if ((a.group & 1) == 0) {
                                *reinterpret_cast<float2 *>(to) = make_float2(s[nt][i], s[nt][i + 1]);
                            } else {
                                to[0] = s[nt][i];
                                if (r + 1 < have) to[1] = s[nt][i + 1];
                            }
                        }
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
                                for (int t = 0; t < KS; ++t) {
                                    o[t][nt][i] *= keep;
                                    o[t][nt][i + 2] *= keep;
                                }
                            }
                        }
                }
                constexpr float kCut = kLift * (BF ? 1.0f - 1.0f / 512.0f : 1.0f - 1.0f / 4096.0f);
                uint32_t p_hi[NT][2], p_lo[NT][2];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[nt][i] = exp2_fast(s[nt][i] - ref[nt][i & 1]);
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        l[nt][i] += s[nt][i] + s[nt][i + 2];
                        const uint32_t hi = pack_cut<BF>(s[nt][2 * i] * kCut, s[nt][2 * i + 1] * kCut);
                        const float2 back = unpack<BF>(hi);
                        const uint32_t lo = pack_round<BF>(__fmaf_rn(s[nt][2 * i], kLift, -back.x), __fmaf_rn(s[nt][2 * i + 1], kLift, -back.y));
                        p_hi[nt][i] = transpose8x8(kTwin && (lane & 2) ? lo : hi);
                        if constexpr (!kTwin) p_lo[nt][i] = transpose8x8(lo);
                    }
                }
#pragma unroll
                for (int t = 0; t < KS; ++t) {
                    uint32_t f[4];
                    ldsm4_trans(f, v_base + at + (t >> 2) * kTile * 128 + ((((t & 3) * 2 + v_c) ^ v_x) << 4));
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        mma<BF>(o[t][nt], f, p_hi[nt][0], p_hi[nt][1]);
                        if constexpr (!kTwin) mma<BF>(o[t][nt], f, p_lo[nt][0], p_lo[nt][1]);
                    }
                }
                __syncwarp();
                ++done;
#pragma unroll 1
                for (int s = 0; s < 2 && !lost && issued < w1 && issued < done + S::kStages; ++s) issue();   // two: one may have had to wait
                if (++stage == S::kStages) {
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
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) l[nt][i] += __shfl_xor_sync(0xffffffffu, l[nt][i], d);
            if constexpr (kTwin) {
#pragma unroll
                for (int t = 0; t < KS; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[t][0][i] += __shfl_xor_sync(0xffffffffu, o[t][0][i], 2);
            }
            if (!ITEM && item_ends && tile_begin == 0) {
                // complete: to the output, two channels of a row per lane
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    float inv[2];
#pragma unroll
                    for (int i = 0; i < 2; ++i) inv[i] = l[nt][i] == 0.0f ? 0.0f : (1.0f / kLift) / l[nt][i];
                    const int r = nt * 8 + (lane >> 2);
                    uint16_t *to = a.out + ((int64_t)c_seq * a.Hq + h * a.group + row0 + r) * a.d + (lane & 3) * 2;
#pragma unroll
                    for (int t = 0; t < KS; ++t)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const uint32_t x = transpose8x8(pack_round<BF>(channel(o[t][nt][2 * i], inv[0]), channel(o[t][nt][2 * i + 1], inv[1])));
                            if (r < have && t * 16 + i * 8 + (lane & 3) * 2 < a.d) *reinterpret_cast<uint32_t *>(to + t * 16 + i * 8) = x;
                        }
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int r2 = nt * 8 + (lane & 3) * 2 + i;
                        if (lane < 4 && r2 < have) {
                            const int64_t row = (int64_t)c_seq * a.Hq + h * a.group + row0 + r2;
                            const float lg = l[nt][i] == 0.0f ? -INFINITY : ref[nt][i] + log2f(l[nt][i]);
                            a.row_lse[row] = lg;
                            if (a.lse) a.lse[row] = lg * kLn2;
                        }
                    }
                }
            } else {
                // a piece: of an item that began before this run, or of one that goes on behind it; in a cluster, of the item (where
                // the ring was, which has run dry)
                float *to = ITEM ? reinterpret_cast<float *>(ring) : a.part + ((int64_t)run * 2 + (tile_begin > 0 ? 0 : 1)) * a.rows * S::kPitch;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int r = nt * 8 + (lane & 3) * 2 + (i & 1);
                        if (r < a.rows) {
#pragma unroll
                            for (int t = 0; t < KS; ++t) to[r * S::kPitch + t * 16 + (i >> 1) * 8 + (lane >> 2)] = o[t][nt][i];
                            if (lane < 4 && i < 2)
                                *reinterpret_cast<float2 *>(to + r * S::kPitch + S::kCols) =
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
        join_item<BF, DB, NT>(a, rings, warp_bytes, w0, w1);
        return;
    }
    if (lane == 0) a.open[run] = open_item;

    // rows of the batch without tokens
    for (int b = run; b < a.n_seqs; b += gridDim.x) {
        const int len = __ldg(a.lens + b);
        if (seq_tiles(a, len).n == 0) fill_empty<BF>(a, (int64_t)b * a.Hq, a.Hq, len != 0, lane, 32);
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
static int launch_finish(DecodeArgs &a, FinishArgs f, cudaStream_t st)
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

// A layer as (channel, token, block of 64 channels, KV head, K or V), boxes of 64 channels x `piece` tokens.  Where head_dim is a
// multiple of 64 a box has all blocks, of K and of V: one copy per piece.  Elsewhere the channels stay one dimension, so
// that those past head_dim read as 0, and a box has 64 of them.
static bool encode_layer(CUtensorMap *map, const void *base, bool bf16, const llms_kv_desc &d, int piece, bool whole)
{
    const cuuint64_t head = d.n_kv_heads == 1 ? (cuuint64_t)d.n_tokens * d.head_dim : (cuuint64_t)d.stride_h;
    const cuuint32_t n_blocks = whole ? d.head_dim / 64 : 1;
    const cuuint64_t dims[5] = {whole ? 64 : (cuuint64_t)d.head_dim, (cuuint64_t)d.n_tokens, n_blocks, (cuuint64_t)d.n_kv_heads, 2};
    const cuuint64_t strides[4] = {(cuuint64_t)d.head_dim * 2, 128, head * 2, (cuuint64_t)d.stride_s * 2};
    const cuuint32_t box[5] = {64, (cuuint32_t)piece, n_blocks, 1, whole ? 2u : 1u}, elem[5] = {1, 1, 1, 1, 1};
    return encode_tensor_map(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 5, const_cast<void *>(base), dims,
                             strides, box, elem, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
}

template <bool BF, int DB, int MODE>
static int launch_decode(DecodeArgs &a, int item_ctas, const CUtensorMap &map, cudaStream_t st)
{
    const int n_items = a.n_seqs * a.Hkv * a.blocks;
    const size_t per_warp = warp_smem<DB>(a.q_bytes), smem = 1024 + per_warp * (item_ctas ? kItemWarps : 1);
    if (item_ctas) {
        LLMS_CUDA_TRY((allow_shared_memory<decode_kernel<BF, DB, MODE, true>>()));
        LLMS_CUDA_TRY(launch_dependent_cluster(decode_kernel<BF, DB, MODE, true>, dim3(n_items * item_ctas), dim3(kItemWarps * 32), smem, item_ctas, st,
                                               a, map));
    } else {
        LLMS_CUDA_TRY((allow_shared_memory<decode_kernel<BF, DB, MODE, false>>()));
        LLMS_CUDA_TRY(launch_dependent(decode_kernel<BF, DB, MODE, false>, dim3(a.grid_runs), dim3(32), smem, st, a, map));
    }
    return LLMS_OK;
}

// By blocks of 64 channels: warps per SM that keep the memory busy, and CTAs that an SM has room for with up to four query rows.
// Rows take shared memory too: of 16 rows of 64 channels and of 8 or 16 of 128 two CTAs fit, of 8 or 16 of 192 one, so that their
// rounds may be more than kItemRounds.  Measured (us, clusters / runs): one 256-token context 5.3 / 7.2, eight ragged contexts of up
// to 1024 tokens and 32 heads 12.1 / 13.2, one of 4096 tokens and 32 heads (eight tiles a warp) 21.6 / 20.4; a launch less on the
// host, 2.2 us.  kItemRounds: rounds of the GPU that a call's clusters may take
constexpr int kRoom[4] = {8, 5, 4, 3}, kPerSm[4] = {3, 3, 2, 1}, kItemRounds = 2;

static DecodeLayout layout_of(const llms_kv_desc &d, int n_seqs, int max_len, bool with_mass)
{
    return decode_layout(d, n_seqs, max_len, with_mass, kRoom[(d.head_dim + 63) / 64 - 1]);
}

template <bool BF>
static int launch_decode_shape(DecodeArgs &a, int db, int mode, int item_ctas, const CUtensorMap &map, cudaStream_t st)
{
    switch (db * 3 + mode) {
    case 3: return launch_decode<BF, 1, 0>(a, item_ctas, map, st);
    case 4: return launch_decode<BF, 1, 1>(a, item_ctas, map, st);
    case 5: return launch_decode<BF, 1, 2>(a, item_ctas, map, st);
    case 6: return launch_decode<BF, 2, 0>(a, item_ctas, map, st);
    case 7: return launch_decode<BF, 2, 1>(a, item_ctas, map, st);
    case 8: return launch_decode<BF, 2, 2>(a, item_ctas, map, st);
    case 9: return launch_decode<BF, 3, 0>(a, item_ctas, map, st);
    case 10: return launch_decode<BF, 3, 1>(a, item_ctas, map, st);
    case 11: return launch_decode<BF, 3, 2>(a, item_ctas, map, st);
    case 12: return launch_decode<BF, 4, 0>(a, item_ctas, map, st);
    case 13: return launch_decode<BF, 4, 1>(a, item_ctas, map, st);
    case 14: return launch_decode<BF, 4, 2>(a, item_ctas, map, st);
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
    *nbytes = layout_of(*desc, n_seqs, max_len, with_mass != 0).total;
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
    const DecodeLayout lay = layout_of(*desc, n_seqs, max_len, mass_out != nullptr);
    if (workspace_bytes < lay.total) return LLMS_ERR_BUF_TOO_SMALL;

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
    a.logits = mass_out ? reinterpret_cast<float *>(ws + lay.off_logits) : nullptr;
    a.mass_in = mass_in; a.mass_out = mass_out;
    a.q_stride = q_stride; a.new_stride = new_stride; a.stride_h = desc->stride_h; a.mass_stride = mass_stride;
    a.table_stride = table_stride; a.n_seqs = n_seqs; a.max_len = max_len; a.window = window;
    set_decode_shape(a, *desc, lay, ws, scale);
    while (a.piece_shift < 4 && a.chunk_len % (2 << a.piece_shift) == 0) ++a.piece_shift;
    const bool bf16 = dtype == LLMS_BF16;
    CUtensorMap map;
    // a box may not hold more than one piece of a tile if K and V, or the blocks, are to lie a whole tile apart
    a.whole_tile = a.d % 64 == 0 && a.piece_shift == 4;
    if (!encode_layer(&map, a.k, bf16, *desc, 1 << a.piece_shift, a.whole_tile)) return LLMS_ERR_UNSUPPORTED;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int item_ctas = decode_item_ctas(a, kPerSm[lay.blocks_of_64 - 1], kItemRounds, kTile, kItemWarps);
    while ((1 << a.item_shift) < item_ctas) ++a.item_shift;
    rc = bf16 ? launch_decode_shape<true>(a, lay.blocks_of_64, lay.mode, item_ctas, map, st)
              : launch_decode_shape<false>(a, lay.blocks_of_64, lay.mode, item_ctas, map, st);
    if (rc || item_ctas) return rc;
    FinishArgs f{};
    f.cols = lay.blocks_of_64 * 64;
    return bf16 ? launch_finish<true>(a, f, st) : launch_finish<false>(a, f, st);
}
