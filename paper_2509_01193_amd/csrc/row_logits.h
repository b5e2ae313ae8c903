// Pieces of the kernels that go over rows of logits (log probabilities, a teacher's tokens, beams): sums of exponentials with a running maximum, and
// logits as numbers that order.
#pragma once
#include "row_common.h"

namespace lobra {
namespace rows {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kFar = -1e30f;            // below every difference that matters: exp is 0, and 0 times it is 0

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// m, S and U of some elements (U in units of log2: sum of 2^x x with x = (z - m) log2 e; here and below log2 e / temperature where one is given)
struct Stat {
    float m, s, u;
};

template <bool ENT> __device__ __forceinline__ void rescale(Stat& a, float m, float c = kLog2e)
{
    const float x = fmaxf((a.m - (m == -INFINITY ? 0.f : m)) * c, kFar);        // (a.m = -inf: s and u are 0)
    const float f = exp2_fast(x);
    if (ENT) a.u = f * (a.u + a.s * x);
    a.s *= f;
    a.m = m;
}

// (the more elements at a time, the less often m grows: nearly every time some lane's does)
template <bool ENT, int N> __device__ __forceinline__ void take(Stat& a, const float (&z)[N], float scale = kLog2e)
{
    float c = z[0];
#pragma unroll
    for (int i = 1; i < N; ++i) c = fmaxf(c, z[i]);
    if (c > a.m) rescale<ENT>(a, c, scale);
    const float ref = a.m == -INFINITY ? 0.f : a.m;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float x = (z[i] - ref) * scale;       // (NaN where z is NaN or m = +inf: s stays NaN from here on)
        const float e = exp2_fast(x);
        a.s += e;
        if (ENT) a.u = fmaf(e, fmaxf(x, kFar), a.u);
    }
}

template <typename E> __device__ __forceinline__ float element(const E* p, int32_t i) { return Elem<E>::load(p, size_t(i)); }

// A packet of -inf, which adds nothing.
template <typename E> __device__ __forceinline__ u32x4 nothing()
{
    const uint32_t w = sizeof(E) == 4 ? 0xff800000u : 0xff80ff80u;
    return u32x4{w, w, w, w};
}

// The statistics of the elements that this thread looks at: batches of U packets, the next one on its way while one is worked on, the
// last one filled up with -inf.  (One by one, what is left behind the whole batches - up to a quarter of a row - would wait for memory U
// times more.)
// left_out(z, first): the values of the packet that begins at element `first` of the row, or of a single element, which may take some out (-inf).
// left_out.begin() runs when the first loads are on their way.
struct NoneLeftOut {
    __device__ __forceinline__ void begin() const {}
    template <int N> __device__ __forceinline__ void operator()(float (&)[N], int32_t, int = 0) const {}
};
template <typename E, int NT, bool ENT, typename F = NoneLeftOut>
__device__ __forceinline__ Stat row_stat(const E* row, const RowShape& sh, float scale = kLog2e, F&& left_out = F())
{
    constexpr int N = Packet<E>::N, U = 4;
    Stat a{-INFINITY, 0.f, 0.f};
    const u32x4* p = reinterpret_cast<const u32x4*>(row + sh.head);
    const int32_t t = threadIdx.x;
    auto fetch = [&](u32x4 (&q)[U], int32_t first) {
        if (first + U * NT <= sh.packets) {           // (uniform)
#pragma unroll
            for (int c = 0; c < U; ++c) q[c] = p[first + c * NT + t];
        } else {
#pragma unroll
            for (int c = 0; c < U; ++c) q[c] = first + c * NT + t < sh.packets ? p[first + c * NT + t] : nothing<E>();
        }
    };
    u32x4 q[U], next[U];
    if (sh.packets > 0) fetch(q, 0);
    // the elements in front of the first packet and behind the last one: fewer than 2 N, a thread each
    const bool has_edge = t < sh.head + sh.tail;
    E edge = E(0);
    if (has_edge) edge = row[t < sh.head ? t : t + sh.packets * N];
    left_out.begin();
    for (int32_t first = 0; first < sh.packets; first += U * NT) {
        if (first + U * NT < sh.packets) fetch(next, first + U * NT);
        float z[U * N];
#pragma unroll
        for (int c = 0; c < U; ++c)
#pragma unroll
            for (int e = 0; e < N; ++e) z[c * N + e] = Packet<E>::element(q[c], e);
#pragma unroll
        for (int c = 0; c < U; ++c) left_out(z, sh.head + (first + c * NT + t) * N, c * N);
        take<ENT>(a, z, scale);
#pragma unroll
        for (int c = 0; c < U; ++c) q[c] = next[c];
    }
    if (has_edge) {
        float z[1] = {Elem<E>::load(&edge, 0)};
        left_out(z, t < sh.head ? t : t + sh.packets * N);
        take<ENT>(a, z, scale);
    }
    return a;
}

// A logit and its index as one number that orders by value, the lowest index first among equals.
__device__ __forceinline__ uint64_t order_key(float z, int32_t index)
{
    const uint32_t b = __float_as_uint(z + 0.f);       // (-0 is 0)
    return (uint64_t(b & 0x80000000u ? ~b : b | 0x80000000u) << 32) | uint32_t(~index);
}
__device__ __forceinline__ float key_value(uint64_t key)
{
    const uint32_t b = uint32_t(key >> 32);
    return __uint_as_float(b & 0x80000000u ? b & 0x7fffffffu : ~b);
}
__device__ __forceinline__ int32_t key_index(uint64_t key) { return int32_t(~uint32_t(key)); }

}  // namespace rows
}  // namespace lobra
