// Token eviction by accumulated attention weight: per (layer, sequence, KV head) the heaviest tokens are selected, then
// their K and V rows are closed up.
#include "llms_internal.cuh"

namespace llms {

struct EvictArgs {
    const float *mass;
    float *mass_out;
    uint16_t *kv;
    const int32_t *table, *dst_table, *lens;
    int32_t *kept, *new_lens;
    int64_t stride_l, stride_s, stride_h, mass_stride;
    int table_stride, dst_stride, n_seqs, max_len, L, Hkv, d, chunk_len, n_slots, budget, recent;
};

constexpr int kSelectThreads = 1024;

// Order of the masses as an unsigned key: larger mass, larger key; NaN and -inf are both 0 and lie below every other
// value, -0 equals +0.
__device__ __forceinline__ uint32_t mass_key(float m)
{
    if (isnan(m) || m == -INFINITY) return 0u;
    const uint32_t u = m == 0.0f ? 0u : __float_as_uint(m);
    return (u >> 31) ? ~u : (u | 0x80000000u);
}

// Select: one CTA per (KV head, sequence, layer).  The key of the quota-th heaviest candidate is found digit by digit
// (four passes of 256 bins), then one pass in the order of positions numbers the kept tokens.
__global__ void __launch_bounds__(kSelectThreads) select_kernel(const EvictArgs a)
{
    __shared__ uint32_t hist[256];
    __shared__ uint32_t warp_gt[32], warp_eq[32];
    __shared__ uint32_t s_prefix, s_need;
    const int h = blockIdx.x, b = blockIdx.y, l = blockIdx.z, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int len = a.lens[b];
    const int64_t row = ((int64_t)l * a.n_seqs + b) * a.Hkv + h;
    const float *mass = a.mass + row * a.mass_stride;
    float *mass_out = a.mass_out + row * a.mass_stride;
    int32_t *kept = a.kept + row * a.budget;
    const bool bad = len < 0 || len > a.max_len;
    const int n = bad ? 0 : len, m = min(a.budget, n), recent = min(a.recent, m);
    const int cand = n - recent, quota = m - recent;
    uint32_t limit = 0, need = quota;             // keys above `limit` stay, and the first `need` ones equal to it
    if (quota > 0 && quota < cand) {
        uint32_t prefix = 0;
        for (int shift = 24; shift >= 0; shift -= 8) {
            for (int i = threadIdx.x; i < 256; i += kSelectThreads) hist[i] = 0;
            __syncthreads();
            const uint32_t mask = shift == 24 ? 0u : 0xffffffffu << (shift + 8);
            for (int t = threadIdx.x; t < cand; t += kSelectThreads) {
                const uint32_t k = mass_key(mass[t]);
                if ((k & mask) == prefix) atomicAdd(&hist[(k >> shift) & 255u], 1u);
            }
            __syncthreads();
            if (threadIdx.x == 0) {
                int bin = 255;
                while (bin > 0 && hist[bin] < need) need -= hist[bin--];
                s_prefix = prefix | ((uint32_t)bin << shift);
                s_need = need;
            }
            __syncthreads();
            prefix = s_prefix;
            need = s_need;
        }
        limit = prefix;
    }
    uint32_t gt_base = 0, eq_base = 0;
    for (int t0 = 0; t0 < n; t0 += kSelectThreads) {
        const int t = t0 + threadIdx.x;
        float w = 0.0f;
        bool gt = false, eq = false;
        if (t < n) {
            w = mass[t];
            const uint32_t k = mass_key(w);
            gt = t >= cand || (quota > 0 && k > limit) || quota >= cand;
            eq = !gt && quota > 0 && k == limit;
        }
        const uint32_t bg = __ballot_sync(0xffffffffu, gt), be = __ballot_sync(0xffffffffu, eq);
        if (lane == 0) {
            warp_gt[warp] = __popc(bg);
            warp_eq[warp] = __popc(be);
        }
        __syncthreads();                          // also: every mass of this tile has been read
        uint32_t gt_before = gt_base + __popc(bg & ((1u << lane) - 1)), eq_before = eq_base + __popc(be & ((1u << lane) - 1));
        for (int w2 = 0; w2 < 32; ++w2) {
            const uint32_t g = warp_gt[w2], e = warp_eq[w2];
            if (w2 < warp) {
                gt_before += g;
                eq_before += e;
            }
            gt_base += g;
            eq_base += e;
        }
        if (gt || (eq && eq_before < need)) {
            const uint32_t j = gt_before + min(eq_before, need);
            kept[j] = t;
            mass_out[j] = w;
        }
        __syncthreads();
    }
    for (int j = m + threadIdx.x; j < a.budget; j += kSelectThreads) kept[j] = -1;
    for (int t = m + threadIdx.x; t < n; t += kSelectThreads) mass_out[t] = 0.0f;
    if (threadIdx.x == 0 && l == 0 && h == 0) a.new_lens[b] = bad ? -1 : m;
}

__device__ __forceinline__ int64_t slot_row(const int32_t *row, int chunk_len, int n_slots, int t)
{
    const int slot = __ldg(row + t / chunk_len);
    return (unsigned)slot < (unsigned)n_slots ? (int64_t)slot * chunk_len + t % chunk_len : -1;
}

// Move: one CTA per (K or V of a KV head, sequence, layer).  A kept row's new position never lies behind its old one, so
// going up in tiles of rows, each read completely before it is written, is safe in place.
__global__ void __launch_bounds__(256) move_kernel(const EvictArgs a)
{
    const int h = blockIdx.x >> 1, s = blockIdx.x & 1, b = blockIdx.y, l = blockIdx.z;
    const int32_t *kept = a.kept + (((int64_t)l * a.n_seqs + b) * a.Hkv + h) * a.budget;
    uint4 *base = reinterpret_cast<uint4 *>(a.kv + l * a.stride_l + s * a.stride_s + h * a.stride_h);
    const int vec = a.d / 8;
    const int m = a.new_lens[b];
    const int32_t *src_tab = a.table + (int64_t)b * a.table_stride;
    const int32_t *dst_tab = a.dst_table ? a.dst_table + (int64_t)b * a.dst_stride : src_tab;
    const int rows_at_once = 256 / vec;
    const int r = threadIdx.x / vec, c = threadIdx.x % vec;
    for (int j0 = 0; j0 < m; j0 += rows_at_once) {
        const int j = j0 + r;
        uint4 v;
        int64_t src = -1, dst = -1;
        if (r < rows_at_once && j < m) {
            src = slot_row(src_tab, a.chunk_len, a.n_slots, kept[j]);
            dst = slot_row(dst_tab, a.chunk_len, a.n_slots, j);
            if (src >= 0) v = base[src * vec + c];
        }
        __syncthreads();
        if (src >= 0 && dst >= 0 && src != dst) base[dst * vec + c] = v;
    }
}

}  // namespace llms

using namespace llms;

extern "C" int llms_evict_tokens(const llms_kv_desc *desc, void *kv, const float *mass, int64_t mass_stride,
                                 const int32_t *chunk_table, int table_stride, const int32_t *lens, int n_seqs, int max_len,
                                 int budget, int recent, const int32_t *dst_table, int dst_stride, float *mass_out,
                                 int32_t *kept, int32_t *new_lens, void *stream)
{
    const int rc = check_paged(desc, n_seqs, max_len);
    if (rc) return rc;
    if (budget < 1 || recent < 0 || recent > budget) return LLMS_ERR_INVALID_ARG;
    if (n_seqs == 0) return LLMS_OK;
    if (!kv || !mass || !chunk_table || !lens || !mass_out || !kept || !new_lens || new_lens == lens) return LLMS_ERR_INVALID_ARG;
    if (table_stride < 1 || (int64_t)table_stride * desc->chunk_len < max_len || mass_stride < max_len) return LLMS_ERR_INVALID_ARG;
    const int most = budget < max_len ? budget : max_len;
    if (dst_table && (dst_stride < 1 || (int64_t)dst_stride * desc->chunk_len < most)) return LLMS_ERR_INVALID_ARG;
    if (!aligned(kv, 16)) return LLMS_ERR_MISALIGNED;
    if (!aligned(mass, 4) || !aligned(mass_out, 4) || !aligned(chunk_table, 4) || !aligned(lens, 4) || !aligned(dst_table, 4) ||
        !aligned(kept, 4) || !aligned(new_lens, 4))
        return LLMS_ERR_MISALIGNED;
    if (desc->n_layers > 65535) return LLMS_ERR_UNSUPPORTED;
    EvictArgs a{};
    a.mass = mass; a.mass_out = mass_out;
    a.kv = static_cast<uint16_t *>(kv);
    a.table = chunk_table; a.dst_table = dst_table; a.lens = lens;
    a.kept = kept; a.new_lens = new_lens;
    a.stride_l = desc->stride_l; a.stride_s = desc->stride_s; a.stride_h = desc->stride_h; a.mass_stride = mass_stride;
    a.table_stride = table_stride; a.dst_stride = dst_stride;
    a.n_seqs = n_seqs; a.max_len = max_len; a.L = desc->n_layers; a.Hkv = desc->n_kv_heads; a.d = desc->head_dim;
    a.chunk_len = desc->chunk_len; a.n_slots = n_chunks(*desc);
    a.budget = budget; a.recent = recent;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    select_kernel<<<dim3(a.Hkv, n_seqs, a.L), kSelectThreads, 0, st>>>(a);
    LLMS_CUDA_TRY(cudaGetLastError());
    move_kernel<<<dim3(a.Hkv * 2, n_seqs, a.L), 256, 0, st>>>(a);
    LLMS_CUDA_TRY(cudaGetLastError());
    return LLMS_OK;
}
