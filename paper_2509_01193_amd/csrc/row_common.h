// Pieces of the kernels that stream rows of fp32 or bf16 elements (log probabilities, norms, activations): 16-byte packets and the sums
// over a wave or a workgroup.
#pragma once
#include <hip/hip_runtime.h>
#include <cstdint>

#include "device_common.h"

namespace lobra {
namespace rows {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// Elements of a 16-byte packet, and the way between a packet and fp32.  (To bf16: to nearest even, NaN stays NaN.)
template <typename E> struct Packet;
template <> struct Packet<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ void widen(u32x4 p, float (&v)[N])
    {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = __uint_as_float(p[i]);
    }
    static __device__ __forceinline__ u32x4 narrow(const float (&v)[N])
    {
        u32x4 p;
#pragma unroll
        for (int i = 0; i < N; ++i) p[i] = __float_as_uint(v[i]);
        return p;
    }
};
template <> struct Packet<uint16_t> {
    static constexpr int N = 8;
    static __device__ __forceinline__ void widen(u32x4 p, float (&v)[N])
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(p[i] << 16);
            v[2 * i + 1] = __uint_as_float(p[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ u32x4 narrow(const float (&v)[N])
    {
        union { bf16x8 b; u32x4 u; } c;
#pragma unroll
        for (int i = 0; i < N; ++i) c.b[i] = (__bf16)v[i];
        return c.u;
    }
};

__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) v += __shfl_xor(v, m);
    return v;
}

__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) v = fmaxf(v, __shfl_xor(v, m));
    return v;
}

// A row of n elements that may start anywhere: `head` elements up to the first 16-byte boundary, `packets` whole packets, `tail`
// elements.  Nothing outside the row is read or written.
struct RowShape {
    int32_t head, packets, tail;
};
template <typename E> __device__ __forceinline__ RowShape row_shape(const E* row, int32_t n)
{
    constexpr int32_t N = Packet<E>::N;
    const int32_t off = int32_t((reinterpret_cast<uintptr_t>(row) & 15u) / sizeof(E));
    RowShape s;
    s.head = min(off ? N - off : 0, n);
    s.packets = (n - s.head) / N;
    s.tail = n - s.head - s.packets * N;
    return s;
}

}  // namespace rows
}  // namespace lobra
