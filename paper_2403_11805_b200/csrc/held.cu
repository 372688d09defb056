// Quantising K and V rows into a pool held at 8 or 4 bits, and reading rows back out of it.
//
// Mathematics.  Per group of channels of a token: zero = min x, scale = fp16((max x - min x) * r) with r next to 1 / (2^b - 1), code =
// rint((x - zero) * (1 / scale)); the group stands for zero + code * scale.
//
// Bound.  Every element is read and written once (2 bytes one way, b / 8 and its share of the parameters the other), with some ten
// instructions in between.  Memory would bound it; what does is how many loads are under way, which for a write are the rows that
// 96 registers and five warps per scheduler hold (2.3 stalled cycles per instruction on loads, 60% of the issue slots busy).
//
// Split.  A warp takes K and V of one KV head's 16 tokens of one sequence: a tile of the pool, in whose order of codes its lanes hold the
// channels from the start, so that a whole tile is written (or read) in full vectors and nothing is exchanged but the ranges
// of the groups.  All its loads are under way before the first value is used.  A sequence's rows may begin and end inside
// a tile: the other tokens' codes in it are left as they are.  Neighbouring warps take the heads of the same tokens, whose
// rows lie side by side.
//
// Measured, a B200, 4 bits: a prompt of 32768 tokens, 8 heads of 128 channels, written in 35 us (170 MB, 4.8 TB/s; 11
// instructions per channel); 4096 tokens of 32 heads read in 16.3 us (85 MB, 5.2 TB/s); one token for each of
// 32 sequences, one head of 256 channels at 8 bits, 4.3 us.  K and V in warps of their own: 55 and 22 us.
#include <algorithm>
#include <type_traits>

#include "held.cuh"

namespace llms {

constexpr int kHeldWarps = 4;                     // per CTA

// The span of up to 16 rows that a warp has: the rows of a sequence's tokens in one tile.
struct HeldSpan {
    int first, end;                               // tokens [first, end) of the tile's 16 have a row
    int64_t row0;                                 // row of the tile's first token, whether it has one or not
    int64_t tile;                                 // in the pool (per KV head), or -1: the tokens lie nowhere
    __device__ __forceinline__ bool has(int i) const { return i >= first && i < end; }
    // whether one of tokens 8 i .. 8 i + 7 has a row; one with the parity e
    __device__ __forceinline__ bool any(int i) const { return end > 8 * i && first < 8 * i + 8; }
    __device__ __forceinline__ bool any(int i, int e) const
    {
        const int lo = max(first, 8 * i), n = min(end, 8 * i + 8) - lo;
        return n > 1 || (n == 1 && (lo & 1) == e);
    }
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

// N words from or to an address that is aligned to them.  WRITTEN: the kernel stores to that memory too (rows whose held values
// take their place), so that the load must not be one of memory that stays as it is.
template <bool WRITTEN, int N>
__device__ __forceinline__ void load_words_if(bool there, uint32_t (&x)[N], const void *p)
{
    using T = typename Words<N>::T;
    if (there) {
        if constexpr (WRITTEN) *reinterpret_cast<T *>(x) = *reinterpret_cast<const T *>(p);
        else *reinterpret_cast<T *>(x) = __ldg(reinterpret_cast<const T *>(p));
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

// fp32(x) + c with one rounding; x are fp16 bits.
__device__ __forceinline__ float add_half(uint32_t x, float c)
{
    float d;
    asm("add.rn.f32.f16 %0, %1, %2;" : "=f"(d) : "h"((unsigned short)x), "f"(c));
    return d;
}
// fp32(x) * fp32(y) + c with one rounding; x and y are fp16 bits.
__device__ __forceinline__ float fma_half(uint32_t x, uint32_t y, float c)
{
    float d;
    asm("fma.rn.f32.f16 %0, %1, %2, %3;" : "=f"(d) : "h"((unsigned short)x), "h"((unsigned short)y), "f"(c));
    return d;
}
// Two products, each rounded.
__device__ __forceinline__ float2 mul_pair(float2 x, float2 y)
{
    float2 d;
    asm("{\n\t.reg .b64 a, b;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmul.rn.f32x2 a, a, b;\n\tmov.b64 {%0, %1}, a;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(x.x), "f"(x.y), "f"(y.x), "f"(y.y));
    return d;
}

// N neighbouring channels (pairs x, fp16) of a token: their codes as N * BITS bits, and the values that they stand for.  PLAIN: every
// group of the warp has finite values and a scale that is 0 or no subnormal number: then no code can pass the largest (the
// scale is off by 2^-11 at most, the codes by less than half), and a scale of 0 needs no case of its own.
template <typename S, bool BF, bool SEEN, bool PLAIN, int N>
__device__ __forceinline__ uint32_t encode(const GroupRule &rule, const uint32_t (&x)[N / 2], uint32_t (&seen)[N / 2])
{
    uint32_t word = 0u - magic_sum<S::BITS>(N);
#pragma unroll
    for (int c = 0; c < N; c += 2) {
        float2 v;
        if constexpr (PLAIN) {
            v = mul_pair(make_float2(add_half(x[c / 2], -rule.zero), add_half(x[c / 2] >> 16, -rule.zero)), make_float2(rule.inverse, rule.inverse));
            v.x = __fadd_rn(v.x, 12582912.0f);
            v.y = __fadd_rn(v.y, 12582912.0f);
        } else {
            v = __half22float2(as_half2(x[c / 2]));
            v.x = rule.template stepped<S::kTop>(v.x);
            v.y = rule.template stepped<S::kTop>(v.y);
        }
        word += (__float_as_uint(v.x) << (c * S::BITS)) + (__float_as_uint(v.y) << ((c + 1) * S::BITS));
        if constexpr (SEEN) seen[c / 2] = to_row<BF>(rule.value(v.x), rule.value(v.y));
    }
    return word;
}

// The channels of one token that a lane has in words [0, W) (pairs x), which become their codes; ranges are exchanged with the
// lanes that differ in the bits of MASK.
template <typename S, bool BF, bool SEEN, int N, int FIRST, int LAST>
__device__ __forceinline__ void encode_token(uint32_t (&x)[S::W][N / 2], uint32_t (&code)[S::W], bool has, bool stored, uint32_t *params, bool writes_params,
                                             uint16_t *seen_at, int seen_step)
{
#pragma unroll
    for (int grp = 0; grp < S::GPR; ++grp) {
        GroupRange range;
#pragma unroll
        for (int w = grp * S::kGroupWords; w < (grp + 1) * S::kGroupWords; ++w)
#pragma unroll
            for (int c = 0; c < N / 2; ++c) {
                const __half2 v = to_half2<BF>(x[w][c]);
                x[w][c] = half2_bits(v);
                range.add(v);
            }
        __half2 r = range.own();
#pragma unroll
        for (int d = FIRST; d < LAST; d <<= 1) r = __hmin2_nan(r, as_half2(__shfl_xor_sync(0xffffffffu, half2_bits(r), d)));
        GroupRule rule;
        rule.set<S::kTop>(r);
        if (!stored) rule.zero = NAN, rule.scale = 0.0f;      // nothing is held of it
        const bool plain = rule.zero == rule.zero && (rule.scale == 0.0f || rule.scale >= 0x1p-14f);
        auto all_words = [&](auto is_plain) {
#pragma unroll
            for (int w = grp * S::kGroupWords; w < (grp + 1) * S::kGroupWords; ++w) {
                uint32_t seen[N / 2];
                code[w] = encode<S, BF, SEEN, decltype(is_plain)::value, N>(rule, x[w], seen);
                if (SEEN && has) store_words(seen_at + w * seen_step, seen);
            }
        };
        if (__all_sync(0xffffffffu, plain)) all_words(std::true_type());
        else all_words(std::false_type());
        if (writes_params) params[grp] = rule.params;
    }
}

template <typename S, bool BF, bool SEEN>
__global__ void __launch_bounds__(kHeldWarps * 32) held_write_kernel(const HeldRows a)
{
    grid_dependency_wait();
    grid_launch_dependents();
    const int lane = threadIdx.x & 31, unit = blockIdx.x * kHeldWarps + __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);
    const int span = a.by_heads(unit), h = unit - span * a.H;
    HeldSpan s;
    if (span >= a.spans || !find_span(a, span, s)) return;
    const bool stored = s.tile >= 0;                          // (else no pointer into the tile is used)
    uint8_t *const tile = a.held + ((int64_t)h * a.tiles + max(s.tile, (int64_t)0)) * S::kTileBytes;
    const int g = lane >> 2, j = lane & 3;
    constexpr int kWordChannels = 32 / S::BITS, kUnitChannels = 16 / S::BITS;
    uint32_t k[2][S::W][kWordChannels / 2], v[2][2][S::W][kUnitChannels / 2];  // tokens 8 i + g of K; 8 i + 2 j + e of V
    const uint16_t *const k_from = a.k + (int64_t)h * S::D + j * kWordChannels, *const v_from = a.v + (int64_t)h * S::D + g * kUnitChannels;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int w = 0; w < S::W; ++w) load_words_if<SEEN>(s.has(8 * i + g), k[i][w], k_from + (s.row0 + 8 * i + g) * a.row_stride + w * 4 * kWordChannels);
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int w = 0; w < S::W; ++w) {
                const int t = 8 * i + 2 * j + e;
                load_words_if<SEEN>(s.has(t), v[i][e][w], v_from + (s.row0 + t) * a.row_stride + w * 8 * kUnitChannels);
            }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int t = 8 * i + g;
        const bool has = s.has(t);
        uint32_t code[S::W];
        if (!s.any(i)) continue;                              // (one new token: most of the tile is somebody else's)
        encode_token<S, BF, SEEN, kWordChannels, 1, 4>(k[i], code, has, stored, reinterpret_cast<uint32_t *>(tile + 2 * S::kCodes) + t * S::GPR,
                                                       stored && has && j == 0,
                                                       SEEN ? a.k_out + (s.row0 + t) * a.out_stride + (int64_t)h * S::D + j * kWordChannels : nullptr,
                                                       4 * kWordChannels);
        if (stored && has) {
#pragma unroll
            for (int w = 0; w < S::W; w += S::VW) {
                uint32_t x[S::VW];
#pragma unroll
                for (int n = 0; n < S::VW; ++n) x[n] = code[w + n];
                store_words(reinterpret_cast<uint32_t *>(tile) + S::place(i, w, lane), x);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        uint32_t code[2][S::W];
        const int t = 8 * i + 2 * j;
#pragma unroll
        for (int e = 0; e < 2; ++e)
            if (s.any(i, e)) encode_token<S, BF, SEEN, kUnitChannels, 4, 32>(v[i][e], code[e], s.has(t + e), stored,
                                                            reinterpret_cast<uint32_t *>(tile + 2 * S::kCodes + S::kParams) + (t + e) * S::GPR,
                                                            stored && s.has(t + e) && g == 0,
                                                            SEEN ? a.v_out + (s.row0 + t + e) * a.out_stride + (int64_t)h * S::D + g * kUnitChannels : nullptr,
                                                            8 * kUnitChannels);
        uint32_t *codes = reinterpret_cast<uint32_t *>(tile + S::kCodes);
        if (stored && s.has(t) && s.has(t + 1)) {
#pragma unroll
            for (int w = 0; w < S::W; w += S::VW) {
                uint32_t x[S::VW];
#pragma unroll
                for (int n = 0; n < S::VW; ++n) x[n] = __byte_perm(code[0][w + n], code[1][w + n], 0x5410);
                store_words(codes + S::place(i, w, lane), x);
            }
        } else if (stored && (s.has(t) || s.has(t + 1))) {      // the other token's half of the words stays
            const int e = s.has(t) ? 0 : 1;
#pragma unroll
            for (int w = 0; w < S::W; ++w) reinterpret_cast<uint16_t *>(codes + S::place(i, w, lane))[e] = (uint16_t)(e ? code[1][w] : code[0][w]);
        }
    }
}

// N neighbouring channels out of N * BITS bits; scale in fp16 bits.
template <typename S, bool BF, int N>
__device__ __forceinline__ void decode(uint32_t word, uint32_t scale, float zero, uint32_t (&row)[N / 2])
{
#pragma unroll
    for (int c = 0; c < N; c += 2) {
        // the code in the low bits of 1024 is 1024 + code; what is left behind 1024 is exact
        const uint32_t q = c ? word >> (c * S::BITS) : word;
        const uint32_t pair = S::BITS == 4 ? ((q & 0xfu) | ((q << 12 & 0xf0000u) | 0x64006400u)) : __byte_perm(q, 0x64006400u, 0x5150);
        const uint32_t code = half2_bits(__hsub2(as_half2(pair), as_half2(0x64006400u)));
        row[c / 2] = to_row<BF>(fma_half(code, scale, zero), fma_half(code >> 16, scale, zero));
    }
}

template <typename S, bool BF>
__global__ void __launch_bounds__(kHeldWarps * 32) held_read_kernel(const HeldRows a)
{
    grid_dependency_wait();
    grid_launch_dependents();
    const int lane = threadIdx.x & 31, unit = blockIdx.x * kHeldWarps + __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0);
    const int span = a.by_heads(unit), h = unit - span * a.H;
    HeldSpan s;
    if (span >= a.spans || !find_span(a, span, s)) return;
    // (an address, 0 if the tokens lie nowhere: what is added to it then is no pointer)
    const uintptr_t tile = s.tile < 0 ? 0 : reinterpret_cast<uintptr_t>(a.held + ((int64_t)h * a.tiles + s.tile) * S::kTileBytes);
    const int g = lane >> 2, j = lane & 3;
    constexpr int kWordChannels = 32 / S::BITS, kUnitChannels = 16 / S::BITS;
    uint32_t x[2][2][S::W], k_rule[2][S::GPR], v_rule[2][2][S::GPR];           // [K, V][i]; of tokens 8 i + g; of tokens 8 i + 2 j + e
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int w = 0; w < S::W; w += S::VW) {
                uint32_t v[S::VW];
                load_words_if<false>(tile != 0, v, reinterpret_cast<const uint32_t *>(tile + half * S::kCodes + S::place(i, w, lane) * 4));
#pragma unroll
                for (int n = 0; n < S::VW; ++n) x[half][i][w + n] = v[n];
            }
    auto rule_of = [&](int i) { return tile ? __ldg(reinterpret_cast<const uint32_t *>(tile + 2 * S::kCodes + i * 4)) : kNanHalf << 16; };
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int grp = 0; grp < S::GPR; ++grp) {
            k_rule[i][grp] = rule_of((8 * i + g) * S::GPR + grp);
#pragma unroll
            for (int e = 0; e < 2; ++e) v_rule[i][e][grp] = rule_of((16 + 8 * i + 2 * j + e) * S::GPR + grp);
        }
    uint16_t *const k_to = a.k_out + (int64_t)h * S::D + j * kWordChannels, *const v_to = a.v_out + (int64_t)h * S::D + g * kUnitChannels;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int w = 0; w < S::W; ++w) {
            const int t = 8 * i + g;
            const uint32_t rule = k_rule[i][w / S::kGroupWords];
            uint32_t row[kWordChannels / 2];
            if (!s.any(i)) continue;
            decode<S, BF, kWordChannels>(x[0][i][w], rule, __high2float(as_half2(rule)), row);
            if (s.has(t)) store_words(k_to + (s.row0 + t) * a.out_stride + w * 4 * kWordChannels, row);
        }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int w = 0; w < S::W; ++w) {
                const int t = 8 * i + 2 * j + e;
                const uint32_t rule = v_rule[i][e][w / S::kGroupWords];
                uint32_t row[kUnitChannels / 2];
                if (!s.any(i, e)) continue;
                decode<S, BF, kUnitChannels>(x[1][i][w] >> (16 * e), rule, __high2float(as_half2(rule)), row);
                if (s.has(t)) store_words(v_to + (s.row0 + t) * a.out_stride + w * 8 * kUnitChannels, row);
            }
}

static int64_t held_ctas(const HeldRows &a) { return ((int64_t)a.spans * a.H + kHeldWarps - 1) / kHeldWarps; }

static int launch_held_write(const llms_kv_desc &d, int bits, int dtype, const HeldRows &a, cudaStream_t st)
{
    return with_held_shape(d, bits, [&](auto s) {
        using S = decltype(s);
        const auto kernel = dtype == LLMS_BF16 ? (a.k_out ? held_write_kernel<S, true, true> : held_write_kernel<S, true, false>)
                                               : (a.k_out ? held_write_kernel<S, false, true> : held_write_kernel<S, false, false>);
        LLMS_CUDA_TRY(launch_dependent(kernel, dim3((unsigned)held_ctas(a)), dim3(kHeldWarps * 32), 0, st, a));
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
static int check_rows(const llms_kv_desc *desc, int bits, int dtype, int layer, const void *held, uint64_t held_size, int n_rows, const int32_t *first_row,
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
    if (held_size < held_pool_bytes(*desc, bits)) return LLMS_ERR_BUF_TOO_SMALL;
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
    *nbytes = held_pool_bytes(*desc, bits);
    return LLMS_OK;
}

extern "C" int llms_held_write(const llms_kv_desc *desc, int bits, int dtype, int layer, void *held, uint64_t held_size, const void *k, const void *v,
                               int64_t row_stride, int n_rows, const int32_t *first_row, const int32_t *chunk_table, int table_stride,
                               const int32_t *lens, int n_seqs, int max_len, void *k_seen, void *v_seen, int64_t seen_stride, void *stream)
{
    HeldRows a{};
    int rc = check_rows(desc, bits, dtype, layer, held, held_size, n_rows, first_row, chunk_table, table_stride, lens, n_seqs, max_len, a);
    if (rc || n_seqs == 0 || n_rows == 0) return rc;
    if ((rc = check_row_pair(*desc, k, v, row_stride))) return rc;
    if ((k_seen == nullptr) != (v_seen == nullptr)) return LLMS_ERR_INVALID_ARG;
    if (k_seen && (rc = check_row_pair(*desc, k_seen, v_seen, seen_stride))) return rc;
    a.k = static_cast<const uint16_t *>(k); a.v = static_cast<const uint16_t *>(v);
    a.k_out = static_cast<uint16_t *>(k_seen); a.v_out = static_cast<uint16_t *>(v_seen);
    a.row_stride = row_stride; a.out_stride = seen_stride;
    return launch_held_write(*desc, bits, dtype, a, static_cast<cudaStream_t>(stream));
}

extern "C" int llms_held_read(const llms_kv_desc *desc, int bits, int dtype, int layer, const void *held, uint64_t held_size,
                              const int32_t *chunk_table, int table_stride, const int32_t *lens, int n_seqs, int max_len, const int32_t *first_row, int n_rows,
                              void *k_out, void *v_out, int64_t out_stride, void *stream)
{
    HeldRows a{};
    int rc = check_rows(desc, bits, dtype, layer, held, held_size, n_rows, first_row, chunk_table, table_stride, lens, n_seqs, max_len, a);
    if (rc || n_seqs == 0 || n_rows == 0) return rc;
    if ((rc = check_row_pair(*desc, k_out, v_out, out_stride))) return rc;
    a.k_out = static_cast<uint16_t *>(k_out); a.v_out = static_cast<uint16_t *>(v_out);
    a.out_stride = out_stride;
    return launch_held_read(*desc, bits, dtype, a, static_cast<cudaStream_t>(stream));
}
