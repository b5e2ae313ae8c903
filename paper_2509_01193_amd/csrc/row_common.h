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
    static __device__ __forceinline__ float element(u32x4 p, int i) { return __uint_as_float(p[i]); }
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
    static __device__ __forceinline__ float element(u32x4 p, int i) { return __uint_as_float(i & 1 ? p[i >> 1] & 0xffff0000u : p[i >> 1] << 16); }
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

// Joins of a value over the 64 lanes of a wave, the result in all of them: along the rows of 16 lanes, then row 0 into 1 and 2 into 3,
// then 1 into 2 and 3.  Data-parallel moves take a few cycles each, where a shuffle goes through the LDS unit.  Every lane has to be
// active.  `none`: what joins without effect.
template <int CTRL, int ROWS> __device__ __forceinline__ float lanes_moved(float v, float none)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(none), __float_as_int(v), CTRL, ROWS, 0xf, false));
}
template <typename F> __device__ __forceinline__ float wave_join(float v, float none, F&& f)
{
    v = f(v, lanes_moved<0x111, 0xf>(v, none));      // row_shr 1, 2, 4, 8
    v = f(v, lanes_moved<0x112, 0xf>(v, none));
    v = f(v, lanes_moved<0x114, 0xf>(v, none));
    v = f(v, lanes_moved<0x118, 0xf>(v, none));
    v = f(v, lanes_moved<0x142, 0xa>(v, none));      // row_bcast 15: lane 15 of a row to the next one
    v = f(v, lanes_moved<0x143, 0xc>(v, none));      // row_bcast 31
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}
// The sum of the first 16 lanes, in all lanes.
__device__ __forceinline__ float row_sum(float v)
{
    v += lanes_moved<0x111, 0xf>(v, 0.f);
    v += lanes_moved<0x112, 0xf>(v, 0.f);
    v += lanes_moved<0x114, 0xf>(v, 0.f);
    v += lanes_moved<0x118, 0xf>(v, 0.f);
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 15));
}
__device__ __forceinline__ float wave_sum(float v)
{
    return wave_join(v, 0.f, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ float wave_max(float v)
{
    return wave_join(v, -INFINITY, [](float a, float b) { return fmaxf(a, b); });
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
