// Attention of one new token per sequence over a pool held at 8 or 4 bits, one layer per call.
#include <math.h>

#include "held.cuh"

namespace llms {

struct HeldAttentionArgs {
    const uint8_t *held;                          // of the layer
    const uint16_t *q;
    uint16_t *out;
    const int32_t *table, *lens;
    float *lse;
    int64_t q_stride;
    int table_stride, n_seqs, max_len, window, H, Hq, group, chunk_len, n_slots, tiles;
    float scale;
};

// A warp per query head of a sequence; a lane has every 32nd channel.
template <typename S, bool BF>
__global__ void __launch_bounds__(32) held_attention_kernel(const HeldAttentionArgs a)
{
    grid_dependency_wait();
    grid_launch_dependents();
    constexpr int N = S::D / 32;
    const int b = blockIdx.x / a.Hq, hq = blockIdx.x - b * a.Hq, h = hq / a.group, lane = threadIdx.x;
    const int given = __ldg(a.lens + b), len = given < 0 || given > a.max_len ? 0 : given;
    float q[N], acc[N], top = -INFINITY, sum = 0.0f;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const uint16_t x = a.q[b * a.q_stride + (int64_t)hq * S::D + n * 32 + lane];
        q[n] = BF ? __uint_as_float((uint32_t)x << 16) : __half2float(__ushort_as_half(x));
        acc[n] = 0.0f;
    }
    bool lost = given != len;
#pragma unroll
    for (int n = 0; n < N; ++n) lost |= len > 0 && !isfinite(q[n]);
    lost = __any_sync(0xffffffffu, lost);
    for (int t = a.window > 0 ? max(0, len - a.window) : 0; t < len; ++t) {
        const int chunk = t / a.chunk_len, slot = __ldg(a.table + (int64_t)b * a.table_stride + chunk);
        if ((unsigned)slot >= (unsigned)a.n_slots) {
            lost = true;
            continue;
        }
        const int64_t row = (int64_t)slot * a.chunk_len + (t - chunk * a.chunk_len);
        const int r = (int)(row & 15);
        const uint8_t *tile = a.held + ((int64_t)h * a.tiles + (row >> 4)) * S::kTileBytes;
        auto value = [&](int half, int c) {
            constexpr int kWord = 32 / S::BITS, kUnit = 16 / S::BITS;
            const int u = c / kUnit, word = c / kWord;
            const int at = half ? S::place(r / 8, u / 8, (u % 8) * 4 + (r % 8) / 2) * 4 + (r & 1) * 2 : S::place(r / 8, word / 4, (r % 8) * 4 + word % 4) * 4;
            const uint32_t bits = half ? *reinterpret_cast<const uint16_t *>(tile + S::kCodes + at) : *reinterpret_cast<const uint32_t *>(tile + at);
            const uint32_t code = (bits >> (c % (half ? kUnit : kWord) * S::BITS)) & S::kTop;
            const float2 p = __half22float2(*reinterpret_cast<const __half2 *>(tile + 2 * S::kCodes + half * S::kParams + (r * S::GPR + c / S::kGroup) * 4));
            return __fmaf_rn((float)code, p.x, p.y);
        };
        float s = 0.0f;
#pragma unroll
        for (int n = 0; n < N; ++n) s = __fmaf_rn(q[n], value(0, n * 32 + lane), s);
#pragma unroll
        for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
        s *= a.scale;
        const float m = fmaxf(top, s), ref = m == -INFINITY ? 0.0f : m, keep = expf(top - ref), w = expf(s - ref);
        top = m;
        sum = sum * keep + w;
#pragma unroll
        for (int n = 0; n < N; ++n) acc[n] = __fmaf_rn(w, value(1, n * 32 + lane), acc[n] * keep);
    }
    const int64_t row = (int64_t)b * a.Hq + hq;
#pragma unroll
    for (int n = 0; n < N; ++n) {
        const float x = lost ? NAN : (sum == 0.0f ? 0.0f : acc[n] / sum);
        a.out[row * S::D + n * 32 + lane] = BF ? __bfloat16_as_ushort(__float2bfloat16_rn(x)) : __half_as_ushort(__float2half_rn(x));
    }
    if (lane == 0 && a.lse) a.lse[row] = lost ? NAN : (sum == 0.0f ? -INFINITY : top + logf(sum));
}

}  // namespace llms

using namespace llms;

extern "C" int llms_held_workspace_bytes(const llms_kv_desc *desc, int bits, int n_seqs, int max_len, uint64_t *nbytes)
{
    const int rc = check_held(desc, bits, n_seqs, max_len);
    if (rc) return rc;
    if (!nbytes) return LLMS_ERR_INVALID_ARG;
    *nbytes = 256;
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
    uint64_t need;
    llms_held_workspace_bytes(desc, bits, n_seqs, max_len, &need);
    if (workspace_bytes < need) return LLMS_ERR_BUF_TOO_SMALL;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    HeldAttentionArgs a{};
    a.H = desc->n_kv_heads; a.Hq = desc->n_q_heads; a.group = a.Hq / a.H;
    a.tiles = held_tiles(*desc);
    uint8_t *base = static_cast<uint8_t *>(held) + (uint64_t)layer * a.H * a.tiles * held_tile_bytes(*desc, bits);
    a.held = base;
    a.q = static_cast<const uint16_t *>(q); a.out = static_cast<uint16_t *>(out);
    a.table = chunk_table; a.lens = lens; a.lse = lse; a.q_stride = q_stride;
    a.table_stride = table_stride; a.n_seqs = n_seqs; a.max_len = max_len; a.window = window;
    a.chunk_len = desc->chunk_len; a.n_slots = n_chunks(*desc); a.scale = scale;
    if (k_new) {
        HeldRows r{};
        r.held = base; r.table = chunk_table; r.lens = lens;
        r.k = static_cast<const uint16_t *>(k_new); r.v = static_cast<const uint16_t *>(v_new);
        r.row_stride = new_stride;
        r.table_stride = table_stride; r.n_seqs = r.n_rows = r.spans = n_seqs; r.max_len = max_len; r.H = a.H;
        r.chunk_len = a.chunk_len; r.n_slots = a.n_slots; r.tiles = a.tiles;
        r.by_chunk = Divisor(a.chunk_len); r.by_heads = Divisor(a.H);
        if ((rc = launch_held_write(*desc, bits, dtype, r, st))) return rc;
    }
    return with_held_shape(*desc, bits, [&](auto s) {
        using S = decltype(s);
        LLMS_CUDA_TRY(launch_dependent(dtype == LLMS_BF16 ? held_attention_kernel<S, true> : held_attention_kernel<S, false>, dim3(n_seqs * a.Hq),
                                       dim3(32), 0, st, a));
        return LLMS_OK;
    });
}
