// Attention of one new token per sequence over a pool held at 8 or 4 bits, one layer per call: the entry points.
#include "held_attention.cuh"

namespace llms {

// Warps per SM for runs, as many as their shared memory allows.
static int held_warps(const llms_kv_desc &d, int bits, bool deep)
{
    const uint64_t tile = held_tile_bytes(d, bits);
    const int rows = std::min(d.n_q_heads / d.n_kv_heads, 16);
    const int cta = kRunWarps * (held_stages(tile, deep) * held_stage_bytes(tile, rows, d.head_dim) + 320) + 1024;
    return std::max(1, std::min<int>(held_room(tile, deep) / kRunWarps, 228 * 1024 / cta)) * kRunWarps;
}

// Runs: one per warp that there is room for, or up to kHeldRounds if each then still has kHeldRunTiles tiles (the warps that get done early
// take the next ones).  With up to kFewTiles tiles for each of DEEP's warps, runs are DEEP.
constexpr int kHeldRounds = 4, kHeldRunTiles = 12, kFewTiles = 32;
struct HeldLayout : DecodeLayout {
    bool deep;
};
static HeldLayout held_layout(const llms_kv_desc &d, int bits, int n_seqs, int max_len, int window)
{
    HeldLayout t;
    static_cast<DecodeLayout &>(t) = decode_layout(d, n_seqs, max_len, false, 1, kHeldTile);
    const uint64_t seen = window > 0 ? std::min<uint64_t>(max_len, (uint64_t)window + kHeldTile - 1) : max_len;
    const uint64_t tiles = (uint64_t)n_seqs * d.n_kv_heads * t.blocks * ((seen + kHeldTile - 1) / kHeldTile);
    const uint64_t deep_room = (uint64_t)sm_count() * held_warps(d, bits, true), room = (uint64_t)sm_count() * held_warps(d, bits, false);
    t.deep = tiles <= deep_room * kFewTiles;
    const uint64_t rounds = t.deep ? 1 : std::min<uint64_t>(kHeldRounds, std::max<uint64_t>(1, tiles / (room * kHeldRunTiles)));
    t.runs = (int)std::min<uint64_t>(t.deep ? deep_room : room * rounds, std::max<uint64_t>(1, tiles / kMinTiles));
    t.few_tiles = 0;
    // (the workspace is the same whatever the window: for as many runs as any needs)
    t.grid_runs = (int)std::max(deep_room, room * kHeldRounds);
    t.off_part = t.off_open + round_up((uint64_t)t.grid_runs * 4, 256);
    t.total = t.off_logits = t.off_part + round_up((uint64_t)t.grid_runs * 2 * t.rows * (t.blocks_of_64 * 64 + 4) * 4, 256);
    t.grid_runs = t.runs;
    return t;
}

// Items that span runs are joined: a CTA per query row of an item (by_item), or of the item that is open at the end of a run.  A group of
// four channels has a thread in each of the CTA's slices, which take the runs' pieces in turn; their loads are under way
// together, so that the time is two ways to L2 and back.
constexpr int kFinishThreads = 256, kFinishLoads = 8;

template <bool BF>
__global__ void __launch_bounds__(kFinishThreads) held_finish_kernel(const DecodeArgs a, int by_item, int cols, Divisor by_rows)
{
    __shared__ float4 s_acc[kFinishThreads];
    __shared__ float2 s_ml[kFinishThreads / 16];
    const int x = by_rows(blockIdx.x), r = blockIdx.x - x * a.rows, per_seq = a.Hkv * a.blocks;
    // (the lengths are older than the kernel before, which has begun: they need not be waited for.  No CTA ends before the wait: the
    // kernel behind this one waits for this one only)
    const bool empty = by_item && seq_tiles<kHeldTile>(a, __ldg(a.lens + a.by_per_seq(x))).n == 0;
    grid_dependency_wait();
    grid_launch_dependents();
    const int item = by_item ? x : __ldcg(a.open + x);
    if (empty || item < 0) return;
    const int2 span = __ldcg(a.span + item);
    const int b = a.by_per_seq(item), hb = item - b * per_seq, h = a.by_blocks(hb), rb = hb - h * a.blocks;
    const int row = rb * (a.group > 8 ? 16 : 8) + r;          // of the KV head's
    if (row >= a.group || span.x < 0) return;
    const int groups = cols / 4, slices = kFinishThreads / groups, slice = threadIdx.x / groups, c = (threadIdx.x - slice * groups) * 4, pitch = cols + 4;
    const float *const from = a.part + (int64_t)r * pitch;
    const int64_t stride = (int64_t)a.rows * pitch;
    float top = -INFINITY, sum = 0.0f, acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
    for (int i0 = span.x + slice; i0 <= span.y; i0 += slices * kFinishLoads) {
        float2 ml[kFinishLoads];
        float4 v[kFinishLoads];
#pragma unroll
        for (int u = 0; u < kFinishLoads; ++u) {
            // the first run's last piece, then the following runs' first ones
            const int i = i0 + u * slices;
            const float *at = from + ((int64_t)i * 2 + (i == span.x)) * stride;
            ml[u] = make_float2(-INFINITY, 0.0f);
            if (i <= span.y) {
                ml[u] = __ldcg(reinterpret_cast<const float2 *>(at + cols));
                v[u] = __ldcg(reinterpret_cast<const float4 *>(at + c));
            }
        }
        float most = top;
#pragma unroll
        for (int u = 0; u < kFinishLoads; ++u) most = fmaxf(most, ml[u].x);
        const float ref = most == -INFINITY ? 0.0f : most, keep = exp2_fast(top - ref);
        top = most;
        sum *= keep;
#pragma unroll
        for (int n = 0; n < 4; ++n) acc[n] *= keep;
#pragma unroll
        for (int u = 0; u < kFinishLoads; ++u) {
            if (i0 + u * slices > span.y) break;
            const float w = exp2_fast(ml[u].x - ref);
            sum = __fmaf_rn(w, ml[u].y, sum);
            acc[0] = __fmaf_rn(w, v[u].x, acc[0]);
            acc[1] = __fmaf_rn(w, v[u].y, acc[1]);
            acc[2] = __fmaf_rn(w, v[u].z, acc[2]);
            acc[3] = __fmaf_rn(w, v[u].w, acc[3]);
        }
    }
    s_acc[threadIdx.x] = make_float4(acc[0], acc[1], acc[2], acc[3]);
    if (c == 0) s_ml[slice] = make_float2(top, sum);
    __syncthreads();
    if (slice) return;
    const int n = min(slices, span.y - span.x + 1);
    for (int i = 1; i < n; ++i) top = fmaxf(top, s_ml[i].x);
    const float ref = top == -INFINITY ? 0.0f : top;
    sum = acc[0] = acc[1] = acc[2] = acc[3] = 0.0f;
#pragma unroll 4
    for (int i = 0; i < n; ++i) {
        const float2 ml = s_ml[i];
        const float4 v = s_acc[i * groups + threadIdx.x];
        const float w = exp2_fast(ml.x - ref);
        sum = __fmaf_rn(w, ml.y, sum);
        acc[0] = __fmaf_rn(w, v.x, acc[0]);
        acc[1] = __fmaf_rn(w, v.y, acc[1]);
        acc[2] = __fmaf_rn(w, v.z, acc[2]);
        acc[3] = __fmaf_rn(w, v.w, acc[3]);
    }
    finish_row<BF>(a, (int64_t)b * a.Hq + h * a.group + row, c, acc, top, sum);
}

static int launch_held_finish(const DecodeArgs &a, bool bf16, int cols, cudaStream_t st)
{
    const int n_items = a.n_seqs * a.Hkv * a.blocks, by_item = n_items <= a.grid_runs;
    LLMS_CUDA_TRY(launch_dependent(bf16 ? held_finish_kernel<true> : held_finish_kernel<false>, dim3(std::min(n_items, a.grid_runs) * a.rows),
                                   dim3(kFinishThreads), 0, st, a, by_item, cols, Divisor(a.rows)));
    return LLMS_OK;
}

// CTAs of a cluster per item, or 0: runs.
static int held_item_ctas(const DecodeArgs &a, uint64_t tile_bytes)
{
    const int ctas = decode_item_ctas(a, 1, 1, kHeldTile, held_item_warps(tile_bytes));
    return ctas && held_item_smem(tile_bytes, a.rows, a.d, ctas) <= 220 * 1024 ? ctas : 0;
}

}  // namespace llms

using namespace llms;

extern "C" int llms_held_workspace_bytes(const llms_kv_desc *desc, int bits, int n_seqs, int max_len, uint64_t *nbytes)
{
    const int rc = check_held(desc, bits, n_seqs, max_len);
    if (rc) return rc;
    if (!nbytes) return LLMS_ERR_INVALID_ARG;
    *nbytes = held_layout(*desc, bits, n_seqs, max_len, 0).total;
    return LLMS_OK;
}

extern "C" int llms_held_attention(const llms_kv_desc *desc, int bits, int dtype, int layer, void *held, uint64_t held_size, const void *q,
                                   int64_t q_stride, const void *k_new, const void *v_new, int64_t new_stride, const int32_t *chunk_table, int table_stride,
                                   const int32_t *lens, int n_seqs, int max_len, int window, float scale, void *out, float *lse,
                                   void *workspace, uint64_t workspace_bytes, void *stream)
{
    int rc = check_held(desc, bits, n_seqs, max_len);
    if (rc) return rc;
    if (dtype != LLMS_F16 && dtype != LLMS_BF16) return LLMS_ERR_INVALID_ARG;
    if (layer < 0 || layer >= desc->n_layers || window < 0 || !isfinite(scale)) return LLMS_ERR_INVALID_ARG;
    if (n_seqs == 0) return LLMS_OK;
    if (!held || !q || !chunk_table || !lens || !out || !workspace || (k_new == nullptr) != (v_new == nullptr)) return LLMS_ERR_INVALID_ARG;
    if (table_stride < 1 || (int64_t)table_stride * desc->chunk_len < max_len) return LLMS_ERR_INVALID_ARG;
    if (q_stride < (int64_t)desc->n_q_heads * desc->head_dim) return LLMS_ERR_INVALID_ARG;
    if (k_new && new_stride < (int64_t)desc->n_kv_heads * desc->head_dim) return LLMS_ERR_INVALID_ARG;
    if (!aligned(held, 16) || !aligned(q, 16) || !aligned(out, 16) || q_stride % 8 || !aligned(workspace, 256)) return LLMS_ERR_MISALIGNED;
    if (k_new && (!aligned(k_new, 16) || !aligned(v_new, 16) || new_stride % 8)) return LLMS_ERR_MISALIGNED;
    if (!aligned(chunk_table, 4) || !aligned(lens, 4) || !aligned(lse, 4)) return LLMS_ERR_MISALIGNED;
    const HeldLayout lay = held_layout(*desc, bits, n_seqs, max_len, window);
    if (workspace_bytes < lay.total || held_size < held_pool_bytes(*desc, bits)) return LLMS_ERR_BUF_TOO_SMALL;

    DecodeArgs a{};
    a.q = static_cast<const uint16_t *>(q);
    a.k_new = static_cast<const uint16_t *>(k_new);
    a.v_new = static_cast<const uint16_t *>(v_new);
    a.out = static_cast<uint16_t *>(out);
    a.table = chunk_table; a.lens = lens;
    a.lse = lse;
    a.q_stride = q_stride; a.new_stride = new_stride;
    a.table_stride = table_stride; a.n_seqs = n_seqs; a.max_len = max_len; a.window = window;
    uint8_t *ws = static_cast<uint8_t *>(workspace);
    set_decode_shape(a, *desc, lay, ws, scale);
    // the kernel counts an item's tiles and kItemSlots more in 32 bits
    if (((uint64_t)max_len / kHeldTile + 1 + kItemSlots) * n_seqs * a.Hkv * a.blocks > 0x7fffffff) return LLMS_ERR_UNSUPPORTED;
    HeldFeed f{};
    f.tiles = held_tiles(*desc);
    f.held = static_cast<uint8_t *>(held) + (uint64_t)layer * a.Hkv * f.tiles * held_tile_bytes(*desc, bits);
    f.bf16 = dtype == LLMS_BF16;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int item_ctas = held_item_ctas(a, held_tile_bytes(*desc, bits)), groups = a.d / desc->group_size;
    while ((1 << a.item_shift) < item_ctas) ++a.item_shift;
    switch (a.d) {
    case 64: rc = launch_held_attention<64>(bits, groups, lay.mode, a, f, item_ctas, lay.deep, st); break;
    case 96: rc = launch_held_attention<96>(bits, groups, lay.mode, a, f, item_ctas, lay.deep, st); break;
    case 128: rc = launch_held_attention<128>(bits, groups, lay.mode, a, f, item_ctas, lay.deep, st); break;
    default: rc = launch_held_attention<256>(bits, groups, lay.mode, a, f, item_ctas, lay.deep, st);
    }
    if (rc || item_ctas) return rc;
    return launch_held_finish(a, f.bf16, lay.blocks_of_64 * 64, st);
}
