// The format of a pool whose K and V are held at 8 or 4 bits, shared by the calls that write it, read it and attend to it.
//
// A tile is 16 tokens of a chunk slot, K and V of one KV head: one run of bytes, so that a tile comes into shared memory as
// one copy.  Codes lie in the order in which the lanes of a warp want them as operands of m16n8k16 MMAs, so that a lane reads them
// with its widest loads and without bank conflicts: with lane = 4 g + j (g < 8, j < 4), i < 2 and W words of 32 bits,
//     K: word (w, j) of token 8 i + g: 32 / bits channels from (4 w + j) * 32 / bits on.  A row of the MMA is a token;
//     V: 16-bit unit (w, g) of tokens 8 i + 2 j + e (e < 2, in the low and the high half of a word): 16 / bits channels from
//        (8 w + g) * 16 / bits on.  A row of the MMA is a channel, and two tokens share a register.
// Words w of a lane lie together VW at a time: [i][w / VW][lane][w % VW].
#pragma once

#include <cuda_bf16.h>

#include "paged.cuh"

namespace llms {

template <int D_, int BITS_, int GPR_>
struct HeldShape {
    static constexpr int D = D_, BITS = BITS_, GPR = GPR_;            // channels, bits of a code, groups of channels per row
    static constexpr int W = D * BITS / 128;
    static constexpr int VW = W % 4 == 0 ? 4 : (W % 2 == 0 ? 2 : 1);
    static constexpr int kGroup = D / GPR, kGroupWords = W / GPR;
    static constexpr int kTop = (1 << BITS) - 1;
    static constexpr int kCodes = 2 * D * BITS, kParams = 64 * GPR;   // bytes of a tile's K (or V)
    static constexpr int kTileBytes = 2 * (kCodes + kParams);
    // words from the start of a tile's codes
    __host__ __device__ static constexpr int place(int i, int w, int lane) { return ((i * (W / VW) + w / VW) * 32 + lane) * VW + w % VW; }
};

inline uint64_t held_tile_bytes(const llms_kv_desc &d, int bits) { return 2 * (2 * (uint64_t)d.head_dim * bits + 64 * (d.head_dim / d.group_size)); }
inline int held_tiles(const llms_kv_desc &d) { return n_chunks(d) * (d.chunk_len / 16); }   // per (layer, KV head)

inline uint64_t held_pool_bytes(const llms_kv_desc &d, int bits) { return (uint64_t)d.n_layers * d.n_kv_heads * held_tiles(d) * held_tile_bytes(d, bits); }

// Checks of shape that all calls on a held pool make.
int check_held(const llms_kv_desc *d, int bits, int n_seqs, int max_len);

// Calls f(HeldShape) for the shape of a checked descriptor.
template <typename F>
int with_held_shape(const llms_kv_desc &d, int bits, F &&f)
{
    const int gpr = d.head_dim / d.group_size;
    if (bits == 4) {
        if (d.head_dim == 64) return gpr == 1 ? f(HeldShape<64, 4, 1>()) : f(HeldShape<64, 4, 2>());
        if (d.head_dim == 96) return f(HeldShape<96, 4, 3>());
        if (d.head_dim == 128) return gpr == 1 ? f(HeldShape<128, 4, 1>()) : (gpr == 2 ? f(HeldShape<128, 4, 2>()) : f(HeldShape<128, 4, 4>()));
        return gpr == 1 ? f(HeldShape<256, 4, 1>()) : (gpr == 2 ? f(HeldShape<256, 4, 2>()) : f(HeldShape<256, 4, 4>()));
    }
    if (d.head_dim == 64) return gpr == 1 ? f(HeldShape<64, 8, 1>()) : f(HeldShape<64, 8, 2>());
    if (d.head_dim == 96) return f(HeldShape<96, 8, 3>());
    if (d.head_dim == 128) return gpr == 1 ? f(HeldShape<128, 8, 1>()) : (gpr == 2 ? f(HeldShape<128, 8, 2>()) : f(HeldShape<128, 8, 4>()));
    return gpr == 1 ? f(HeldShape<256, 8, 1>()) : (gpr == 2 ? f(HeldShape<256, 8, 2>()) : f(HeldShape<256, 8, 4>()));
}

struct HeldRows {                                 // operands of a write or read
    uint8_t *held;                                // of the layer
    const int32_t *table, *lens, *first_row;
    const uint16_t *k, *v;                        // write: the rows
    uint16_t *k_out, *v_out;                      // read: the rows; write: the values held, or NULL
    int64_t row_stride, out_stride;
    int table_stride, n_seqs, n_rows, max_len, H, chunk_len, n_slots, tiles, spans;   // spans: groups of up to 16 rows, per KV head
    Divisor by_chunk, by_heads;
};

#ifdef __CUDACC__

__device__ __forceinline__ uint32_t half2_bits(__half2 x) { return *reinterpret_cast<uint32_t *>(&x); }
__device__ __forceinline__ __half2 as_half2(uint32_t x) { return *reinterpret_cast<__half2 *>(&x); }
constexpr uint32_t kNanHalf = 0x7e00u;

// A pair of a row's values as fp16: bfloat16 to nearest, saturated, its infinities and NaN as NaN.
template <bool BF>
__device__ __forceinline__ __half2 to_half2(uint32_t x)
{
    if constexpr (!BF) return as_half2(x);
    const float a = __uint_as_float(x << 16), b = __uint_as_float(x & 0xffff0000u);
    uint32_t r;
    asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    if ((x & 0x7f80u) == 0x7f80u) r = (r & 0xffff0000u) | kNanHalf;
    if ((x & 0x7f800000u) == 0x7f800000u) r = (r & 0xffffu) | (kNanHalf << 16);
    return as_half2(r);
}
// A pair of held values in a row's type, each rounded once (fp16: saturated; NaN stays).
template <bool BF>
__device__ __forceinline__ uint32_t to_row(float a, float b)
{
    uint32_t r;
    if constexpr (BF) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    else asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    return r;
}

// The smallest value and the negated largest one of a group, as far as one lane has it; a NaN or an infinity ends as one.
struct GroupRange {
    __half2 low, high;
    __device__ __forceinline__ GroupRange() : low(as_half2(0x7c007c00u)), high(as_half2(0xfc00fc00u)) {}
    __device__ __forceinline__ void add(__half2 x)
    {
        low = __hmin2_nan(low, x);
        high = __hmax2_nan(high, x);
    }
    __device__ __forceinline__ __half2 own() const
    {
        return __halves2half2(__hmin_nan(__low2half(low), __high2half(low)), __hneg(__hmax_nan(__low2half(high), __high2half(high))));
    }
};

// Scale and zero-point of a group and what its codes are made with: binary32, to nearest, nothing fused.  The scale is a product with
// the binary32 number next to 1 / TOP, which lies above 1 / TOP for 15 and 255.  So where the quotient, which the swap records take,
// lies half-way between two fp16 numbers the scale is the upper of the two, and a record's the even one; elsewhere they are the same.
struct GroupRule {
    float zero, inverse, scale;                   // a group with an infinity or a NaN: zero is NaN, all codes are 0
    uint32_t params;                              // (scale, zero) in fp16
    template <int TOP>
    __device__ __forceinline__ void set(__half2 range)
    {
        const float low = __half2float(__low2half(range)), high = -__half2float(__high2half(range));
        const bool finite = isfinite(low) && isfinite(high);
        const __half s = finite ? __float2half_rn(__fmul_rn(fabsf(__fsub_rn(high, low)), 1.0f / TOP)) : __ushort_as_half(0);
        zero = finite ? __fadd_rn(low, 0.0f) : NAN;
        scale = __half2float(s);
        inverse = scale == 0.0f ? 0.0f : __frcp_rn(scale);
        params = (uint32_t)__half_as_ushort(s) | (finite ? (uint32_t)__half_as_ushort(__float2half_rn(zero)) : kNanHalf) << 16;
    }
    // 1.5 * 2^23 + the code of a value: the code lies in the low bits.
    template <int TOP>
    __device__ __forceinline__ float stepped(float x) const
    {
        const float y = inverse == 0.0f ? 0.0f : fminf(__fmul_rn(__fsub_rn(x, zero), inverse), (float)TOP);
        return __fadd_rn(y, 12582912.0f);
    }
    __device__ __forceinline__ float value(float stepped) const { return __fmaf_rn(__fsub_rn(stepped, 12582912.0f), scale, zero); }
};

#endif

}  // namespace llms
