// Attention of one new token per sequence over a pool held at 8 or 4 bits, one layer per call: the entry points.
#include "held_attention.cuh"

namespace llms {

// By a tile's bytes: warps per SM that keep the memory busy, and CTAs of a cluster that an SM has room for.
static int held_room(const llms_kv_desc &d, int bits)
{
    const uint64_t bytes = held_tile_bytes(d, bits);
    return bytes <= 2304 ? 16 : (bytes <= 4608 ? 10 : 6);
}
static int held_per_sm(const llms_kv_desc &d, int bits)
{
    const uint64_t bytes = held_tile_bytes(d, bits);
    return bytes <= 2304 ? 4 : (bytes <= 4608 ? 3 : 2);
}

}  // namespace llms

using namespace llms;

extern "C" int llms_held_workspace_bytes(const llms_kv_desc *desc, int bits, int n_seqs, int max_len, uint64_t *nbytes)
{
    const int rc = check_held(desc, bits, n_seqs, max_len);
    if (rc) return rc;
    if (!nbytes) return LLMS_ERR_INVALID_ARG;
    *nbytes = decode_layout(*desc, n_seqs, max_len, false, held_room(*desc, bits)).total;
    return LLMS_OK;
}

extern "C" int llms_held_attention(const llms_kv_desc *desc, int bits, int dtype, int layer, void *held, const void *q, int64_t q_stride,
                                   const void *k_new, const void *v_new, int64_t new_stride, const int32_t *chunk_table, int table_stride,
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
    const DecodeLayout lay = decode_layout(*desc, n_seqs, max_len, false, held_room(*desc, bits));
    if (workspace_bytes < lay.total) return LLMS_ERR_BUF_TOO_SMALL;

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
    HeldFeed f{};
    f.tiles = held_tiles(*desc);
    f.held = static_cast<uint8_t *>(held) + (uint64_t)layer * a.Hkv * f.tiles * held_tile_bytes(*desc, bits);
    f.bf16 = dtype == LLMS_BF16;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int item_ctas = decode_item_ctas(a, held_per_sm(*desc, bits)), groups = a.d / desc->group_size;
    while ((1 << a.item_shift) < item_ctas) ++a.item_shift;
    switch (a.d) {
    case 64: rc = launch_held_attention<64>(bits, groups, lay.mode, a, f, item_ctas, st); break;
    case 96: rc = launch_held_attention<96>(bits, groups, lay.mode, a, f, item_ctas, st); break;
    case 128: rc = launch_held_attention<128>(bits, groups, lay.mode, a, f, item_ctas, st); break;
    default: rc = launch_held_attention<256>(bits, groups, lay.mode, a, f, item_ctas, st);
    }
    if (rc || item_ctas) return rc;
    FinishArgs fin{};
    fin.cols = lay.blocks_of_64 * 64;
    return f.bf16 ? launch_finish<true>(a, fin, st) : launch_finish<false>(a, fin, st);
}
