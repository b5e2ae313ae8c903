// Tokens as whole numbers with a scale each, for a wave or a workgroup: a kernel of its own (q8.hip) and a part of one (q8_few.hip).
//     scale = max |v| / 127     q = v / scale, rounded to the nearest whole number, halves to the even one
// The quotient is the exact one: a product with 1 / scale can land on the other side of a half, so where it comes near one (1e-4 either side; its own
// error is below 2e-5) the remainder v - q scale, which fp32 holds exactly there, decides.
#pragma once
#include "kernels.h"
#include "row_common.h"

namespace lobra {
namespace rows {

// (Magnitudes whose scale is no normal number count as zeros: the scale is 0, and every q.)
struct Quantiser {
    float scale, inv;
};
__device__ __forceinline__ Quantiser quantiser(float amax)       // amax: finite, >= 0
{
    Quantiser z;
    z.scale = amax >= 127.f * 0x1p-126f ? amax / 127.f : 0.f;
    z.inv = z.scale > 0.f ? 1.f / z.scale : 0.f;
    return z;
}

// q of N values at a time, as bytes.  A product plus 1.5 x 2^23 is the nearest whole number (halves to the even one) in the lowest bits of a float.
template <int N> __device__ __forceinline__ void quantise(const Quantiser& z, const float (&v)[N], uint32_t (&b)[N / 4])
{
    constexpr float kWhole = 12582912.f;
    float t[N], far = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        t[i] = fmaf(v[i], z.inv, kWhole);
        far = fmaxf(far, fabsf(fmaf(v[i], z.inv, kWhole - t[i])));
    }
    if (far > 0.4999f) {                             // (a packet in some hundreds)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float q = t[i] - kWhole, r = fmaf(-q, z.scale, v[i]), over = fabsf(r) - 0.5f * z.scale;
            if (over > 0.f || (over == 0.f && (int32_t(q) & 1))) t[i] += copysignf(1.f, r);
        }
    }
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        const uint32_t lo = __builtin_amdgcn_perm(__float_as_uint(t[4 * i + 1]), __float_as_uint(t[4 * i]), 0x0c0c0400u),
                       hi = __builtin_amdgcn_perm(__float_as_uint(t[4 * i + 3]), __float_as_uint(t[4 * i + 2]), 0x04000c0cu);
        b[i] = lo | hi;
    }
}

// The largest magnitude of eight bf16 as bits, two in a word (NaN and infinity: 0x7f80 and above), joined with m.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ u16x2 amax_bits(u32x4 p, u16x2 m)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, p[i] & 0x7fff7fffu));
    return m;
}
// (NaN counts as infinity: a maximum would drop it)
__device__ __forceinline__ float amax_value(u16x2 m)
{
    const uint32_t b = max(uint32_t(m[0]), uint32_t(m[1])) << 16;
    return __uint_as_float(b > 0x7f800000u ? 0x7f800000u : b);
}

__device__ __forceinline__ void store_packet(const Quantiser& z, u32x4 p, bool finite, uint8_t* out)
{
    float v[8];
    uint32_t b[2] = {0u, 0u};
    if (finite) {
        Packet<uint16_t>::widen(p, v);
        quantise<8>(z, v, b);
    }
    *reinterpret_cast<uint64_t*>(out) = uint64_t(b[1]) << 32 | b[0];
}

// Row row0, or with W = 1 the wave's of the four from there on.  W waves have a row, whose packets stay in registers between the maximum and the quotients, H a
// lane (what does not fit is read again).  part: four floats of LDS (W = 4).  Bound: memory, and some six VALU instructions an element next to it; few
// rows: the round trip.
// TILED: q as a wave reads it for the matrix instruction, [block of 16 rows][step of 64 k][lane: 16 k of a row][16], instead of row by row.
template <int W, int H, bool TILED = false>
__device__ __forceinline__ void quantise_rows(int32_t T, int32_t d, int32_t pitch, const uint16_t* __restrict__ x, uint8_t* __restrict__ q,
                                              float* __restrict__ scale, int32_t row0, [[maybe_unused]] float* part)
{
    const int32_t wave = __builtin_amdgcn_readfirstlane(int32_t(threadIdx.x >> 6)), row = row0 + wave / W;
    if (W == 1 && row >= T) return;
    constexpr int32_t step = 64 * W;
    const int32_t t = int32_t(threadIdx.x) % step;
    const u32x4* p = reinterpret_cast<const u32x4*>(x + size_t(row) * d);
    uint8_t* const out = q + (TILED ? size_t(row >> 4) * 16 * pitch + (row & 15) * 16 : size_t(row) * pitch);
    auto place = [&](int32_t i) { return out + (TILED ? (i >> 3) * 1024 + (i >> 1 & 3) * 256 + (i & 1) * 8 : 8 * i); };
    const int32_t packets = d / 8, all = pitch / 8;
    const u32x4 none = {0u, 0u, 0u, 0u};
    u32x4 held[H];
#pragma unroll
    for (int c = 0; c < H; ++c) held[c] = t + step * c < packets ? p[t + step * c] : none;
    u16x2 m = {0, 0};
#pragma unroll
    for (int c = 0; c < H; ++c) m = amax_bits(held[c], m);
    for (int32_t i = t + step * H; i < packets; i += step) m = amax_bits(p[i], m);
    float amax = wave_max(amax_value(m));
    if constexpr (W > 1) {
        static_assert(W == 4, "a row per workgroup");
        if ((threadIdx.x & 63) == 0) part[wave] = amax;
        __syncthreads();
        amax = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
    }
    const bool finite = amax < INFINITY;
    const Quantiser z = quantiser(finite ? amax : 0.f);
#pragma unroll
    for (int c = 0; c < H; ++c)
        if (t + step * c < all) store_packet(z, held[c], finite, place(t + step * c));
    for (int32_t i = t + step * H; i < all; i += step) store_packet(z, i < packets ? p[i] : none, finite, place(i));
    if (t == 0) scale[row] = finite ? z.scale : NAN;
}

}  // namespace rows
}  // namespace lobra
