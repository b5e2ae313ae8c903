// The gated feed-forward block's activation: h = a(g) u, and backward dg = dh u a'(g), du = dh a(g), of [g | u] [T][2 f].
//     silu: a = g q, a' = q (1 + g (1 - q)) with q = 1 / (1 + exp(-g))
//     gelu: a = g (1 + th) / 2, a' = (1 + th) / 2 + g (1 - th^2) / 2 c (1 + 3 k g^2), th = tanh(c (g + k g^3))
// f is a multiple of 8, so that rows of all three tensors keep 16-byte packets.
// Roundings (bf16): h starts here from [g | u] as stored, which is off by up to 2^-8 of each; the forms that hold the fp32 projections do not use this
// kernel.  [dg | du] is rounded because the products that read it (dx, dA, dB) take bf16 operands.  Error of h from here, and of dA and dB rounded to
// bf16 (2-norms, of the result's): 0.0030, where the rounding of the result alone leaves 0.0017.
// Bound: memory.  Measured: backward of 16384 x 2 x 11008 bf16 335 us (of 1804 MB, 5.4 TB/s), of 8190 x 2 x 1376 20.  A pass that derives and
// projects (G of [dg | du]) per token block reads two tensors less but reaches 3.9 TB/s like the projection's own: 475 us against 335 + 184
// there, nothing gained at 1376 columns, 10 - 25 % lost where segments have 3 to 20 tokens; not kept.
#include "activation.h"
#include "kernels.h"
#include "row_common.h"

namespace lobra {

using namespace rows;

namespace {

constexpr int NT = 256;

// Packet k of T fp (fp packets to a row): a thread takes every stride-th, whose row and column follow without a division
// (stride = srow fp + scol).
template <typename E, int ACT, bool BACK>
__global__ __launch_bounds__(NT)
void gated_kernel(int64_t packets, int32_t fp, int64_t srow, int32_t scol, const E* gu, const E* __restrict__ dh, E* out)
{
    constexpr int N = Packet<E>::N;
    const size_t f = size_t(fp) * N;
    int64_t k = int64_t(blockIdx.x) * NT + threadIdx.x;
    int64_t row = k / fp;
    int32_t col = int32_t(k - row * fp);
    for (; k < packets; k += int64_t(gridDim.x) * NT) {
        const size_t at = size_t(row) * (2 * f) + size_t(col) * N, ah = size_t(k) * N;
        float g[N], u[N], d[N];
        Packet<E>::widen(*reinterpret_cast<const u32x4*>(gu + at), g);
        Packet<E>::widen(*reinterpret_cast<const u32x4*>(gu + at + f), u);
        if (BACK) {
            Packet<E>::widen(*reinterpret_cast<const u32x4*>(dh + ah), d);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                float da;
                const float a = activate<ACT>(g[e], da);
                g[e] = d[e] * u[e] * da;
                u[e] = d[e] * a;
            }
            *reinterpret_cast<u32x4*>(out + at) = Packet<E>::narrow(g);
            *reinterpret_cast<u32x4*>(out + at + f) = Packet<E>::narrow(u);
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) g[e] = activate<ACT>(g[e]) * u[e];
            *reinterpret_cast<u32x4*>(out + ah) = Packet<E>::narrow(g);
        }
        row += srow;
        col += scol;
        if (col >= fp) {
            col -= fp;
            ++row;
        }
    }
}

// The sums of a split product, in order of the splits, activated before any rounding: 8 columns of a row per thread, in workgroups of a wave (few
// tokens or columns make few of them).  Instead of the launches that add and the one that activates, product included, us: 192 x 4096 x 2 x 1376,
// two products, 40.5 / 37.0; 400 x 4096 x 2 x 256 22.7 / 21.9, 192 18.7 / 19.1.
template <int ACT>
__global__ __launch_bounds__(64)
void gated_sums_kernel(int64_t packets, int32_t fp, const float* __restrict__ g, const float* __restrict__ u, int64_t ld, int64_t stride, int32_t n,
                       uint16_t* __restrict__ gu, uint16_t* __restrict__ h)
{
    constexpr int V = 4;                              // sums on their way at a time
    const int64_t k = int64_t(blockIdx.x) * 64 + threadIdx.x;
    if (k >= packets) return;
    const int64_t row = k / fp;
    const int32_t col = int32_t(k - row * fp) * 8;
    const float *pg = g + row * ld + col, *pu = u + row * ld + col;
    float a[8], b[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) a[e] = b[e] = 0.f;
    for (int32_t s = 0; s < n; s += V) {
        f32x4 v[V][4];
#pragma unroll
        for (int c = 0; c < V; ++c) {
            const int64_t at = int64_t(min(s + c, n - 1)) * stride;
            v[c][0] = *reinterpret_cast<const f32x4*>(pg + at);
            v[c][1] = *reinterpret_cast<const f32x4*>(pg + at + 4);
            v[c][2] = *reinterpret_cast<const f32x4*>(pu + at);
            v[c][3] = *reinterpret_cast<const f32x4*>(pu + at + 4);
        }
#pragma unroll
        for (int c = 0; c < V; ++c) {
            if (s + c >= n) break;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                a[e] += v[c][0][e];
                a[4 + e] += v[c][1][e];
                b[e] += v[c][2][e];
                b[4 + e] += v[c][3][e];
            }
        }
    }
    if (gu) {
        uint16_t* o = gu + size_t(row) * (16 * size_t(fp)) + col;
        *reinterpret_cast<u32x4*>(o) = Packet<uint16_t>::narrow(a);
        *reinterpret_cast<u32x4*>(o + 8 * size_t(fp)) = Packet<uint16_t>::narrow(b);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) a[e] = activate<ACT>(a[e]) * b[e];
    *reinterpret_cast<u32x4*>(h + size_t(k) * 8) = Packet<uint16_t>::narrow(a);
}

template <typename E, bool BACK>
hipError_t launch(int act, int64_t T, int32_t f, const void* gu, const void* dh, void* out, hipStream_t st)
{
    const int32_t fp = f / Packet<E>::N;
    const int64_t packets = T * fp, most = 256 * 16, blocks = (packets + NT - 1) / NT;
    const dim3 grid(uint32_t(blocks < most ? blocks : most));
    const int64_t stride = int64_t(grid.x) * NT, srow = stride / fp;
    const int32_t scol = int32_t(stride - srow * fp);
    const E *a = static_cast<const E*>(gu), *b = static_cast<const E*>(dh);
    E* o = static_cast<E*>(out);
    if (act == LOBRA_ACT_SILU) gated_kernel<E, LOBRA_ACT_SILU, BACK><<<grid, NT, 0, st>>>(packets, fp, srow, scol, a, b, o);
    else gated_kernel<E, LOBRA_ACT_GELU_TANH, BACK><<<grid, NT, 0, st>>>(packets, fp, srow, scol, a, b, o);
    return hipGetLastError();
}

}  // namespace

hipError_t gated_activate(int dtype, int act, int64_t T, int32_t f, const void* gu, void* h, hipStream_t st)
{
    return dtype == LOBRA_F32 ? launch<float, false>(act, T, f, gu, nullptr, h, st) : launch<uint16_t, false>(act, T, f, gu, nullptr, h, st);
}

hipError_t gated_sums(int act, int64_t T, int32_t f, const float* g, const float* u, int64_t ld, int64_t stride, int32_t n, void* gu, void* h,
                      hipStream_t st)
{
    const int32_t fp = f / 8;
    const int64_t packets = T * fp;                   // (a split product's sums are at most 12 MiB)
    const dim3 grid(uint32_t((packets + 63) / 64));
    uint16_t *o = static_cast<uint16_t*>(gu), *p = static_cast<uint16_t*>(h);
    if (act == LOBRA_ACT_SILU) gated_sums_kernel<LOBRA_ACT_SILU><<<grid, 64, 0, st>>>(packets, fp, g, u, ld, stride, n, o, p);
    else gated_sums_kernel<LOBRA_ACT_GELU_TANH><<<grid, 64, 0, st>>>(packets, fp, g, u, ld, stride, n, o, p);
    return hipGetLastError();
}

hipError_t gated_derive(int dtype, int act, int64_t T, int32_t f, const void* gu, const void* dh, void* dgu, hipStream_t st)
{
    return dtype == LOBRA_F32 ? launch<float, true>(act, T, f, gu, dh, dgu, st) : launch<uint16_t, true>(act, T, f, gu, dh, dgu, st);
}

}  // namespace lobra
