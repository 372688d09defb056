// Quantising K and V rows into a pool held at 8 or 4 bits, and reading rows back out of it.
//
// Mathematics.  Per group of channels of a token: zero = min x, scale = fp16((max x - min x) / (2^b - 1)), code = rint((x - zero) / scale);
// the group stands for zero + code * scale.
//
// Bound.  Every element is read and written once (2 bytes one way, b / 8 and its share of the parameters the other), with some ten
// instructions in between: memory-bound.
//
// Split.  A warp takes K or V of one KV head's 16 tokens of one sequence: a tile of the pool, in whose order of codes its lanes hold the
// channels from the start, so that a whole tile is written (or read) in full vectors and nothing is exchanged but the ranges
// of the groups.  A sequence's rows may begin and end inside a tile: the other tokens' codes in it are left as they are.
// Neighbouring warps take the heads of the same tokens, whose rows lie side by side.
#include <algorithm>

#include "held.cuh"

namespace llms {

constexpr int kHeldWarps = 4;                     // per CTA

// The span of up to 16 rows that a warp has: the rows of a sequence's tokens in one tile.
struct HeldSpan {
    int first, end;                               // tokens [first, end) of the tile's 16 have a row
    int64_t row0;                                 // row of the tile's first token, whether it has one or not
    int64_t tile;                                 // in the pool (per KV head), or -1: the tokens lie nowhere
    __device__ __forceinline__ bool has(int i) const { return i >= first && i < end; }
};

// Spans are numbered so that sequence b's begin at first_row[b] / 16 + 2 b: rows [f, f') touch at most (f' - f) / 16 + 2 tiles.
// (64 bits: whatever first_row holds, no row outside the array is touched.)
__device__ __forceinline__ bool find_span(const HeldRows &a, int span, HeldSpan &s)
{
    int b = span;
    int64_t f = span, n = 1, begin = span;
    if (a.first_row) {
        int lo = -1, hi = a.n_seqs;               // the last sequence that begins at or before this span
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if ((int64_t)(__ldg(a.first_row + mid) >> 4) + 2 * mid <= span) lo = mid;
            else hi = mid;
        }
        if (lo < 0) return false;
        b = lo;
        f = __ldg(a.first_row + b);
        n = __ldg(a.first_row + b + 1) - f;
        begin = (f >> 4) + 2 * b;
    }
    int64_t len = __ldg(a.lens + b);
    if (n <= 0 || (!a.first_row && len == 0)) return false;
    const bool valid = len <= a.max_len && n <= len;
    if (!valid) len = n;                          // its rows are still told from others
    const int64_t begin_token = len - n, t0 = ((begin_token >> 4) + (span - begin)) * 16;
    if (t0 >= len) return false;
    s.row0 = f + t0 - begin_token;
    s.first = (int)max(max((int64_t)0, begin_token - t0), min((int64_t)16, -s.row0));
    s.end = (int)min(min((int64_t)16, len - t0), max((int64_t)0, a.n_rows - s.row0));
    s.tile = -1;
    if (valid) {
        const int chunk = a.by_chunk((int)t0), slot = __ldg(a.table + (int64_t)b * a.table_stride + chunk);
        if ((unsigned)slot < (unsigned)a.n_slots) s.tile = ((int64_t)slot * a.chunk_len + ((int)t0 - chunk * a.chunk_len)) / 16;
    }
    return s.first < s.end;
}

template <int N> struct Words;
template <> struct Words<1> { using T = uint32_t; };
template <> struct Words<2> { using T = uint2; };
template <> struct Words<4> { using T = uint4; };

// N words from or to an address that is aligned to them.
template <int N>
__device__ __forceinline__ void load_words(uint32_t (&x)[N], const void *p)
{
    using T = typename Words<N>::T;
    *reinterpret_cast<T *>(x) = __ldg(reinterpret_cast<const T *>(p));
}
template <int N>
__device__ __forceinline__ void load_words_if(bool there, uint32_t (&x)[N], const void *p)
{
    if (there) {
        load_words(x, p);
    } else {
#pragma unroll
        for (int c = 0; c < N; ++c) x[c] = 0u;
    }
}
template <int N>
__device__ __forceinline__ void store_words(void *p, const uint32_t (&x)[N])
{
    using T = typename Words<N>::T;
    *reinterpret_cast<T *>(p) = *reinterpret_cast<const T *>(x);
}

// Sum over c of (0x4b400000 << c * bits): what the upper bits of `n` stepped values add up to in a word of codes.
template <int BITS>
__host__ __device__ constexpr uint32_t magic_sum(int n)
{
    uint32_t s = 0;
    for (int c = 0; c < n; ++c) s += 0x4b400000u << (c * BITS);
    return s;
}

// N neighbouring channels (pairs x) of a token: their codes as N * BITS bits, and the values that they stand for.
template <typename S, bool BF, int N>
__device__ __forceinline__ uint32_t encode(const GroupRule &rule, const uint32_t (&x)[N / 2], uint32_t (&seen)[N / 2])
{
    uint32_t word = 0u - magic_sum<S::BITS>(N);
#pragma unroll
    for (int c = 0; c < N; c += 2) {
        const float2 v = __half22float2(as_half2(x[c / 2]));
        const float a = rule.template stepped<S::kTop>(v.x), b = rule.template stepped<S::kTop>(v.y);
        word += (__float_as_uint(a) << (c * S::BITS)) + (__float_as_uint(b) << ((c + 1) * S::BITS));
        seen[c / 2] = to_row<BF>(rule.value(a), rule.value(b));
    }
    return word;
}

template <typename S, bool BF>
__global__ void __launch_bounds__(kHeldWarps * 32) held_write_kernel(const HeldRows a)
{
    grid_dependency_wait();
    grid_launch_dependents();
    const int lane = threadIdx.x & 31, unit = blockIdx.x * kHeldWarps + (threadIdx.x >> 5), half = unit & 1;
    const int span = a.by_heads(unit >> 1), h = (unit >> 1) - span * a.H;
    HeldSpan s;
    if (span >= a.spans || !find_span(a, span, s)) return;
    uint8_t *tile = s.tile < 0 ? nullptr : a.held + ((int64_t)h * a.tiles + s.tile) * S::kTileBytes;
    const int g = lane >> 2, j = lane & 3;
    constexpr int kWordChannels = 32 / S::BITS, kUnitChannels = 16 / S::BITS;
    const uint16_t *from = (half ? a.v : a.k) + (int64_t)h * S::D;
    uint16_t *seen_at = half ? a.v_out : a.k_out;
    if (seen_at) seen_at += (int64_t)h * S::D;

    if (half == 0) {
        uint32_t x[2][S::W][kWordChannels / 2];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int w = 0; w < S::W; ++w)
                load_words_if(s.has(8 * i + g), x[i][w], from + (s.row0 + 8 * i + g) * a.row_stride + (4 * w + j) * kWordChannels);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int t = 8 * i + g;
            const bool has = s.has(t);
#pragma unroll
            for (int grp = 0; grp < S::GPR; ++grp) {
                GroupRange range;
#pragma unroll
                for (int w = grp * S::kGroupWords; w < (grp + 1) * S::kGroupWords; ++w)
#pragma unroll
                    for (int c = 0; c < kWordChannels / 2; ++c) {
                        const __half2 v = to_half2<BF>(x[i][w][c]);
                        x[i][w][c] = half2_bits(v);
                        range.add(v);
                    }
                __half2 r = range.own();
#pragma unroll
                for (int d = 1; d < 4; d <<= 1) r = __hmin2_nan(r, as_half2(__shfl_xor_sync(0xffffffffu, half2_bits(r), d)));
                GroupRule rule;
                rule.set<S::kTop>(r);
                if (!tile) rule.zero = NAN, rule.scale = 0.0f;                 // nothing is held of it
#pragma unroll
                for (int w = grp * S::kGroupWords; w < (grp + 1) * S::kGroupWords; ++w) {
                    uint32_t seen[kWordChannels / 2];
                    const uint32_t word = encode<S, BF, kWordChannels>(rule, x[i][w], seen);
                    if (seen_at && has) store_words(seen_at + (s.row0 + t) * a.out_stride + (4 * w + j) * kWordChannels, seen);
                    x[i][w][0] = word;
                }
                if (tile && has && j == 0) reinterpret_cast<uint32_t *>(tile + 2 * S::kCodes)[t * S::GPR + grp] = rule.params;
            }
            if (tile && has) {
#pragma unroll
                for (int w = 0; w < S::W; w += S::VW) {
                    uint32_t v[S::VW];
#pragma unroll
                    for (int n = 0; n < S::VW; ++n) v[n] = x[i][w + n][0];
                    store_words(reinterpret_cast<uint32_t *>(tile) + S::place(i, w, lane), v);
                }
            }
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int t = 8 * i + 2 * j;
        uint32_t x[2][S::W][kUnitChannels / 2], word[S::W];
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int w = 0; w < S::W; ++w)
                load_words_if(s.has(t + e), x[e][w], from + (s.row0 + t + e) * a.row_stride + (8 * w + g) * kUnitChannels);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const bool has = s.has(t + e);
#pragma unroll
            for (int grp = 0; grp < S::GPR; ++grp) {
                GroupRange range;
#pragma unroll
                for (int w = grp * S::kGroupWords; w < (grp + 1) * S::kGroupWords; ++w)
#pragma unroll
                    for (int c = 0; c < kUnitChannels / 2; ++c) {
                        const __half2 v = to_half2<BF>(x[e][w][c]);
                        x[e][w][c] = half2_bits(v);
                        range.add(v);
                    }
                __half2 r = range.own();
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) r = __hmin2_nan(r, as_half2(__shfl_xor_sync(0xffffffffu, half2_bits(r), d)));
                GroupRule rule;
                rule.set<S::kTop>(r);
                if (!tile) rule.zero = NAN, rule.scale = 0.0f;
#pragma unroll
                for (int w = grp * S::kGroupWords; w < (grp + 1) * S::kGroupWords; ++w) {
                    uint32_t seen[kUnitChannels / 2];
                    const uint32_t bits = encode<S, BF, kUnitChannels>(rule, x[e][w], seen) & 0xffffu;
                    if (seen_at && has) store_words(seen_at + (s.row0 + t + e) * a.out_stride + (8 * w + g) * kUnitChannels, seen);
                    word[w] = e ? word[w] | bits << 16 : bits;
                }
                if (tile && has && g == 0) reinterpret_cast<uint32_t *>(tile + 2 * S::kCodes + S::kParams)[(t + e) * S::GPR + grp] = rule.params;
            }
        }
        uint32_t *codes = reinterpret_cast<uint32_t *>(tile + S::kCodes);
        if (tile && s.has(t) && s.has(t + 1)) {
#pragma unroll
            for (int w = 0; w < S::W; w += S::VW) {
                uint32_t v[S::VW];
#pragma unroll
                for (int n = 0; n < S::VW; ++n) v[n] = word[w + n];
                store_words(codes + S::place(i, w, lane), v);
            }
        } else if (tile && (s.has(t) || s.has(t + 1))) {      // the other token's half of the words stays
            const int e = s.has(t) ? 0 : 1;
#pragma unroll
            for (int w = 0; w < S::W; ++w) reinterpret_cast<uint16_t *>(codes + S::place(i, w, lane))[e] = (uint16_t)(word[w] >> (16 * e));
        }
    }
}

// N neighbouring channels out of N * BITS bits.
template <typename S, bool BF, int N>
__device__ __forceinline__ void decode(uint32_t word, float scale, float zero, uint32_t (&row)[N / 2])
{
#pragma unroll
    for (int c = 0; c < N; c += 2) {
        const float a = (float)((word >> (c * S::BITS)) & S::kTop), b = (float)((word >> ((c + 1) * S::BITS)) & S::kTop);
        row[c / 2] = to_row<BF>(__fmaf_rn(a, scale, zero), __fmaf_rn(b, scale, zero));
    }
}

template <typename S, bool BF>
__global__ void __launch_bounds__(kHeldWarps * 32) held_read_kernel(const HeldRows a)
{
    grid_dependency_wait();
    grid_launch_dependents();
    const int lane = threadIdx.x & 31, unit = blockIdx.x * kHeldWarps + (threadIdx.x >> 5), half = unit & 1;
    const int span = a.by_heads(unit >> 1), h = (unit >> 1) - span * a.H;
    HeldSpan s;
    if (span >= a.spans || !find_span(a, span, s)) return;
    const uint8_t *tile = s.tile < 0 ? nullptr : a.held + ((int64_t)h * a.tiles + s.tile) * S::kTileBytes;
    const int g = lane >> 2, j = lane & 3;
    constexpr int kWordChannels = 32 / S::BITS, kUnitChannels = 16 / S::BITS;
    uint16_t *to = (half ? a.v_out : a.k_out) + (int64_t)h * S::D;
    uint32_t x[2][S::W], p[2][2][S::GPR];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int w = 0; w < S::W; w += S::VW) {
            uint32_t v[S::VW] = {};
            if (tile) load_words(v, reinterpret_cast<const uint32_t *>(tile + half * S::kCodes) + S::place(i, w, lane));
#pragma unroll
            for (int n = 0; n < S::VW; ++n) x[i][w + n] = v[n];
        }
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int grp = 0; grp < S::GPR; ++grp) {
                const int t = half ? 8 * i + 2 * j + e : 8 * i + g;
                p[i][e][grp] = tile ? __ldg(reinterpret_cast<const uint32_t *>(tile + 2 * S::kCodes + half * S::kParams) + t * S::GPR + grp) : kNanHalf << 16;
            }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int w = 0; w < S::W; ++w) {
            const int grp = w / S::kGroupWords;
            if (half == 0) {
                const int t = 8 * i + g;
                const float2 rule = __half22float2(as_half2(p[i][0][grp]));
                uint32_t row[kWordChannels / 2];
                decode<S, BF, kWordChannels>(x[i][w], rule.x, rule.y, row);
                if (s.has(t)) store_words(to + (s.row0 + t) * a.out_stride + (4 * w + j) * kWordChannels, row);
            } else {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int t = 8 * i + 2 * j + e;
                    const float2 rule = __half22float2(as_half2(p[i][e][grp]));
                    uint32_t row[kUnitChannels / 2];
                    decode<S, BF, kUnitChannels>(x[i][w] >> (16 * e), rule.x, rule.y, row);
                    if (s.has(t)) store_words(to + (s.row0 + t) * a.out_stride + (8 * w + g) * kUnitChannels, row);
                }
            }
        }
}

static int64_t held_ctas(const HeldRows &a) { return ((int64_t)a.spans * a.H * 2 + kHeldWarps - 1) / kHeldWarps; }

int launch_held_write(const llms_kv_desc &d, int bits, int dtype, const HeldRows &a, cudaStream_t st)
{
    return with_held_shape(d, bits, [&](auto s) {
        using S = decltype(s);
        LLMS_CUDA_TRY(launch_dependent(dtype == LLMS_BF16 ? held_write_kernel<S, true> : held_write_kernel<S, false>, dim3((unsigned)held_ctas(a)),
                                       dim3(kHeldWarps * 32), 0, st, a));
        return LLMS_OK;
    });
}

static int launch_held_read(const llms_kv_desc &d, int bits, int dtype, const HeldRows &a, cudaStream_t st)
{
    return with_held_shape(d, bits, [&](auto s) {
        using S = decltype(s);
        LLMS_CUDA_TRY(launch_dependent(dtype == LLMS_BF16 ? held_read_kernel<S, true> : held_read_kernel<S, false>, dim3((unsigned)held_ctas(a)),
                                       dim3(kHeldWarps * 32), 0, st, a));
        return LLMS_OK;
    });
}

int check_held(const llms_kv_desc *d, int bits, int n_seqs, int max_len)
{
    const int rc = check_paged(d, n_seqs, max_len);
    if (rc) return rc;
    if (n_chunks(*d) < 1) return LLMS_ERR_INVALID_ARG;
    if (max_len > 0x7fffff00) return LLMS_ERR_UNSUPPORTED;    // positions are counted up to a tile further, in 32 bits
    if (check_bits(bits)) return LLMS_ERR_BAD_BITS;
    if (bits != 4 && bits != 8) return LLMS_ERR_UNSUPPORTED;
    if (d->quant_mode != 0 || d->chunk_len % 16) return LLMS_ERR_UNSUPPORTED;
    if (d->head_dim != 64 && d->head_dim != 96 && d->head_dim != 128 && d->head_dim != 256) return LLMS_ERR_UNSUPPORTED;
    if (d->group_size < 32 || !is_pow2(d->group_size) || d->head_dim / d->group_size > 4) return LLMS_ERR_UNSUPPORTED;
    if ((int64_t)d->n_kv_heads * held_tiles(*d) > 0x7fffffff) return LLMS_ERR_UNSUPPORTED;       // a layer's tiles are numbered in 32 bits
    return LLMS_OK;
}

// What a write and a read have in common: checks, and the operands as the kernels take them.
static int check_rows(const llms_kv_desc *desc, int bits, int dtype, int layer, const void *held, int n_rows, const int32_t *first_row,
                      const int32_t *chunk_table, int table_stride, const int32_t *lens, int n_seqs, int max_len, HeldRows &a)
{
    const int rc = check_held(desc, bits, n_seqs, max_len);
    if (rc) return rc;
    if (dtype != LLMS_F16 && dtype != LLMS_BF16) return LLMS_ERR_INVALID_ARG;
    if (layer < 0 || layer >= desc->n_layers || n_rows < 0 || (!first_row && n_rows != n_seqs)) return LLMS_ERR_INVALID_ARG;
    if (n_seqs == 0 || n_rows == 0) return LLMS_OK;
    if (!held || !chunk_table || !lens) return LLMS_ERR_INVALID_ARG;
    if (table_stride < 1 || (int64_t)table_stride * desc->chunk_len < max_len) return LLMS_ERR_INVALID_ARG;
    if (!aligned(held, 16) || !aligned(chunk_table, 4) || !aligned(lens, 4) || !aligned(first_row, 4)) return LLMS_ERR_MISALIGNED;
    a.H = desc->n_kv_heads;
    a.tiles = held_tiles(*desc);
    a.held = static_cast<uint8_t *>(const_cast<void *>(held)) + (uint64_t)layer * a.H * a.tiles * held_tile_bytes(*desc, bits);
    a.table = chunk_table; a.lens = lens; a.first_row = first_row;
    a.table_stride = table_stride; a.n_seqs = n_seqs; a.n_rows = n_rows; a.max_len = max_len;
    a.chunk_len = desc->chunk_len; a.n_slots = n_chunks(*desc);
    a.spans = first_row ? n_rows / 16 + 2 * n_seqs : n_seqs;
    a.by_chunk = Divisor(a.chunk_len);
    a.by_heads = Divisor(a.H);
    if ((int64_t)a.spans * a.H * 2 > 0x7fffff00) return LLMS_ERR_UNSUPPORTED;
    return LLMS_OK;
}

static int check_row_pair(const llms_kv_desc &d, const void *k, const void *v, int64_t stride)
{
    if (!k || !v || stride < (int64_t)d.n_kv_heads * d.head_dim) return LLMS_ERR_INVALID_ARG;
    return !aligned(k, 16) || !aligned(v, 16) || stride % 8 ? LLMS_ERR_MISALIGNED : LLMS_OK;
}

}  // namespace llms

using namespace llms;

extern "C" int llms_held_bytes(const llms_kv_desc *desc, int bits, uint64_t *nbytes)
{
    const int rc = check_held(desc, bits, 0, 1);
    if (rc) return rc;
    if (!nbytes) return LLMS_ERR_INVALID_ARG;
    *nbytes = (uint64_t)desc->n_layers * desc->n_kv_heads * held_tiles(*desc) * held_tile_bytes(*desc, bits);
    return LLMS_OK;
}

extern "C" int llms_held_write(const llms_kv_desc *desc, int bits, int dtype, int layer, void *held, const void *k, const void *v,
                               int64_t row_stride, int n_rows, const int32_t *first_row, const int32_t *chunk_table, int table_stride,
                               const int32_t *lens, int n_seqs, int max_len, void *k_seen, void *v_seen, int64_t seen_stride, void *stream)
{
    HeldRows a{};
    int rc = check_rows(desc, bits, dtype, layer, held, n_rows, first_row, chunk_table, table_stride, lens, n_seqs, max_len, a);
    if (rc || n_seqs == 0 || n_rows == 0) return rc;
    if ((rc = check_row_pair(*desc, k, v, row_stride))) return rc;
    if ((k_seen == nullptr) != (v_seen == nullptr)) return LLMS_ERR_INVALID_ARG;
    if (k_seen && (rc = check_row_pair(*desc, k_seen, v_seen, seen_stride))) return rc;
    a.k = static_cast<const uint16_t *>(k); a.v = static_cast<const uint16_t *>(v);
    a.k_out = static_cast<uint16_t *>(k_seen); a.v_out = static_cast<uint16_t *>(v_seen);
    a.row_stride = row_stride; a.out_stride = seen_stride;
    return launch_held_write(*desc, bits, dtype, a, static_cast<cudaStream_t>(stream));
}

extern "C" int llms_held_read(const llms_kv_desc *desc, int bits, int dtype, int layer, const void *held, const int32_t *chunk_table,
                              int table_stride, const int32_t *lens, int n_seqs, int max_len, const int32_t *first_row, int n_rows,
                              void *k_out, void *v_out, int64_t out_stride, void *stream)
{
    HeldRows a{};
    int rc = check_rows(desc, bits, dtype, layer, held, n_rows, first_row, chunk_table, table_stride, lens, n_seqs, max_len, a);
    if (rc || n_seqs == 0 || n_rows == 0) return rc;
    if ((rc = check_row_pair(*desc, k_out, v_out, out_stride))) return rc;
    a.k_out = static_cast<uint16_t *>(k_out); a.v_out = static_cast<uint16_t *>(v_out);
    a.out_stride = out_stride;
    return launch_held_read(*desc, bits, dtype, a, static_cast<cudaStream_t>(stream));
}
