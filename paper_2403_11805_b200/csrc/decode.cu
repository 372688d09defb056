// Attention of one new token per sequence over the paged cache (a pool of chunk slots), one layer per call.
#include <math.h>

#include <cuda_bf16.h>

#include "llms_internal.cuh"

namespace llms {

struct DecodeArgs {
    const uint16_t *q, *k_new, *v_new;
    uint16_t *k, *v, *out;                     // K and V of the layer: base of KV head 0
    const int32_t *table, *lens;
    float *lse, *row_lse;                      // caller's (may be NULL), workspace's
    const float *mass_in;
    float *mass_out;
    int64_t q_stride, new_stride, stride_h, mass_stride;
    int table_stride, n_seqs, max_len, window, Hkv, Hq, group, d, chunk_len, n_slots;
    float scale;
};

template <bool BF>
__device__ __forceinline__ float widen(uint16_t x)
{
    if constexpr (BF) return __uint_as_float((uint32_t)x << 16);
    return __half2float(__ushort_as_half(x));
}
template <bool BF>
__device__ __forceinline__ uint16_t narrow(float x)
{
    if constexpr (BF) return __bfloat16_as_ushort(__float2bfloat16_rn(x));
    return __half_as_ushort(__float2half_rn(x));
}

// Row of the slab that token t of sequence b lies in, -1 for a slot outside the pool.
__device__ __forceinline__ int64_t token_row(const DecodeArgs &a, int b, int t)
{
    const int slot = __ldg(a.table + (int64_t)b * a.table_stride + t / a.chunk_len);
    return (unsigned)slot < (unsigned)a.n_slots ? (int64_t)slot * a.chunk_len + t % a.chunk_len : -1;
}

__global__ void append_kernel(const DecodeArgs a)
{
    const int b = blockIdx.y, h = blockIdx.x, n = a.lens[b];
    if (n < 1 || n > a.max_len) return;
    const int64_t row = token_row(a, b, n - 1);
    if (row < 0) return;
    for (int c = threadIdx.x; c < a.d; c += blockDim.x) {
        a.k[h * a.stride_h + row * a.d + c] = a.k_new[b * a.new_stride + h * a.d + c];
        a.v[h * a.stride_h + row * a.d + c] = a.v_new[b * a.new_stride + h * a.d + c];
    }
}

// One warp per (sequence, query head): lanes hold channels, tokens one after another.
template <bool BF>
__global__ void decode_simple_kernel(const DecodeArgs a)
{
    const int b = blockIdx.y, g = blockIdx.x, h = g / a.group, lane = threadIdx.x;
    const int n = a.lens[b];
    const bool bad = n < 0 || n > a.max_len;
    float q[8], acc[8];
    for (int i = 0; i < 8; ++i) {
        const int c = lane + 32 * i;
        q[i] = c < a.d ? widen<BF>(a.q[b * a.q_stride + (int64_t)g * a.d + c]) : 0.0f;
        acc[i] = 0.0f;
    }
    float m = -INFINITY, z = 0.0f;
    const int first = a.window > 0 && n > a.window ? n - a.window : 0;
    for (int t = bad ? n : first; t < n; ++t) {
        const int64_t row = token_row(a, b, t);
        float s = 0.0f;
        for (int i = 0; i < 8; ++i) {
            const int c = lane + 32 * i;
            if (c < a.d && row >= 0) s = fmaf(q[i], widen<BF>(a.k[h * a.stride_h + row * a.d + c]), s);
        }
        for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
        s = row >= 0 ? s * a.scale : NAN;
        const float m2 = fmaxf(m, s), ref = m2 == -INFINITY ? 0.0f : m2;
        const float old = expf(m - ref), p = expf(s - ref);
        z = fmaf(z, old, p);
        for (int i = 0; i < 8; ++i) {
            const int c = lane + 32 * i;
            if (c < a.d && row >= 0) acc[i] = fmaf(p, widen<BF>(a.v[h * a.stride_h + row * a.d + c]), acc[i] * old);
        }
        m = m2;
    }
    const int64_t o = (int64_t)b * a.Hq + g;
    const float inv = bad ? NAN : (z == 0.0f ? 0.0f : 1.0f / z);
    for (int i = 0; i < 8; ++i) {
        const int c = lane + 32 * i;
        if (c < a.d) a.out[o * a.d + c] = narrow<BF>(inv == 0.0f ? 0.0f : acc[i] * inv);
    }
    if (lane == 0) {
        const float l = bad ? NAN : (z == 0.0f ? -INFINITY : m + logf(z));
        a.row_lse[o] = l;
        if (a.lse) a.lse[o] = l;
    }
}

// One warp per (sequence, KV head, token)
template <bool BF>
__global__ void mass_simple_kernel(const DecodeArgs a)
{
    const int b = blockIdx.z, h = blockIdx.y, n = a.lens[b], lane = threadIdx.x & 31;
    const int t = blockIdx.x * (blockDim.x / 32) + threadIdx.x / 32;
    if (n > a.max_len || t >= n) return;
    float w = 0.0f;
    if (a.window == 0 || t >= n - a.window) {
        const int64_t row = token_row(a, b, t);
        for (int j = 0; j < a.group; ++j) {
            const int g = h * a.group + j;
            float s = 0.0f;
            for (int c = lane; c < a.d && row >= 0; c += 32)
                s = fmaf(widen<BF>(a.q[b * a.q_stride + (int64_t)g * a.d + c]), widen<BF>(a.k[h * a.stride_h + row * a.d + c]), s);
            for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
            s = row >= 0 ? s * a.scale : NAN;
            const float l = a.row_lse[(int64_t)b * a.Hq + g];
            w += l == -INFINITY ? 0.0f : expf(s - l);
        }
    }
    const int64_t i = ((int64_t)b * a.Hkv + h) * a.mass_stride + t;
    if (lane == 0) a.mass_out[i] = (a.mass_in ? a.mass_in[i] : 0.0f) + w;
}

static int check_decode(const llms_kv_desc *d, int n_seqs, int max_len)
{
    const int rc = check_paged(d, n_seqs, max_len);
    if (rc) return rc;
    return LLMS_OK;
}

static uint64_t decode_ws_bytes(const llms_kv_desc &d, int n_seqs)
{
    return round_up((uint64_t)n_seqs * d.n_q_heads * 4, 256);
}

}  // namespace llms

using namespace llms;

extern "C" int llms_decode_workspace_bytes(const llms_kv_desc *desc, int n_seqs, int max_len, int with_mass, uint64_t *nbytes)
{
    (void)with_mass;
    const int rc = check_decode(desc, n_seqs, max_len);
    if (rc) return rc;
    if (!nbytes) return LLMS_ERR_INVALID_ARG;
    *nbytes = decode_ws_bytes(*desc, n_seqs);
    return LLMS_OK;
}

extern "C" int llms_decode_attention(const llms_kv_desc *desc, int dtype, int layer, void *kv, const void *q, int64_t q_stride,
                                     const void *k_new, const void *v_new, int64_t new_stride, const int32_t *chunk_table,
                                     int table_stride, const int32_t *lens, int n_seqs, int max_len, int window, float scale,
                                     void *out, float *lse, const float *mass_in, float *mass_out, int64_t mass_stride,
                                     void *workspace, uint64_t workspace_bytes, void *stream)
{
    int rc = check_decode(desc, n_seqs, max_len);
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
    if (workspace_bytes < decode_ws_bytes(*desc, n_seqs)) return LLMS_ERR_BUF_TOO_SMALL;

    DecodeArgs a{};
    a.q = static_cast<const uint16_t *>(q);
    a.k_new = static_cast<const uint16_t *>(k_new);
    a.v_new = static_cast<const uint16_t *>(v_new);
    a.k = static_cast<uint16_t *>(kv) + layer * desc->stride_l;
    a.v = a.k + desc->stride_s;
    a.out = static_cast<uint16_t *>(out);
    a.table = chunk_table; a.lens = lens;
    a.lse = lse; a.row_lse = static_cast<float *>(workspace);
    a.mass_in = mass_in; a.mass_out = mass_out;
    a.q_stride = q_stride; a.new_stride = new_stride; a.stride_h = desc->stride_h; a.mass_stride = mass_stride;
    a.table_stride = table_stride; a.n_seqs = n_seqs; a.max_len = max_len; a.window = window;
    a.Hkv = desc->n_kv_heads; a.Hq = desc->n_q_heads; a.group = a.Hq / a.Hkv; a.d = desc->head_dim;
    a.chunk_len = desc->chunk_len; a.n_slots = n_chunks(*desc);
    a.scale = scale;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (k_new) append_kernel<<<dim3(a.Hkv, n_seqs), 64, 0, st>>>(a);
    if (dtype == LLMS_BF16) decode_simple_kernel<true><<<dim3(a.Hq, n_seqs), 32, 0, st>>>(a);
    else decode_simple_kernel<false><<<dim3(a.Hq, n_seqs), 32, 0, st>>>(a);
    if (mass_out) {
        const dim3 grid((max_len + 7) / 8, a.Hkv, n_seqs);
        if (dtype == LLMS_BF16) mass_simple_kernel<true><<<grid, 256, 0, st>>>(a);
        else mass_simple_kernel<false><<<grid, 256, 0, st>>>(a);
    }
    LLMS_CUDA_TRY(cudaGetLastError());
    return LLMS_OK;
}
