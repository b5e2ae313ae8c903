// A frozen base in 8-bit integers: tokens (q8_rows.h) and channels as whole numbers with a scale each, and the way back.
#include "kernels.h"
#include "q8_rows.h"
#include "row_common.h"

namespace lobra {

using namespace rows;

namespace {

template <int W, int H>
__global__ __launch_bounds__(256) void q8_rows_kernel(int32_t T, int32_t d, int32_t pitch, const uint16_t* __restrict__ x, uint8_t* __restrict__ q,
                                                      float* __restrict__ scale)
{
    __shared__ float part[4];
    quantise_rows<W, H>(T, d, pitch, x, q, scale, int32_t(blockIdx.x) * (4 / W), part);
}

// 64 columns per workgroup, a lane each; its 16 waves share the rows, 16 neighbouring ones at a time, so that a lane's 16 values are 16 neighbouring
// bytes of its column's row of q.  Done once per weight: 4096 x 11008 bf16 183 us, fp32 78; 4096 x 4096 177 and 61;
// 11008 x 4096 478 and 155 (with four waves a workgroup 617 for the first).  Bound: round trips; a column's 16 waves wait for each batch of 16 rows.
constexpr int kWeightWaves = 16;
template <typename E>
__global__ __launch_bounds__(64 * kWeightWaves) void q8_weight_kernel(int32_t d_in, int32_t d_out, int32_t pitch, int64_t ldw, const E* __restrict__ W,
                                                                     uint8_t* __restrict__ q, float* __restrict__ scale)
{
    __shared__ float part[kWeightWaves][64];
    const int32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t col = int64_t(blockIdx.x) * 64 + lane;
    const bool in = col < d_out;
    float m = 0.f;
    auto rows = [&](int32_t k0, float (&v)[16]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = in && k0 + i < d_in ? Elem<E>::load(W, size_t(k0 + i) * ldw + col) : 0.f;
    };
    for (int32_t k0 = 16 * wave; k0 < d_in; k0 += 16 * kWeightWaves) {
        float v[16];
        rows(k0, v);
#pragma unroll
        for (int i = 0; i < 16; ++i) m = fabsf(v[i]) < INFINITY ? fmaxf(m, fabsf(v[i])) : INFINITY;
    }
    part[wave][lane] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWeightWaves; ++w) m = fmaxf(m, part[w][lane]);
    if (!in) return;
    const bool finite = m < INFINITY;
    const Quantiser z = quantiser(finite ? m : 0.f);
    for (int32_t k0 = 16 * wave; k0 < pitch; k0 += 16 * kWeightWaves) {
        float v[16];
        uint32_t b[4] = {0u, 0u, 0u, 0u};
        rows(k0, v);
        if (finite) quantise<16>(z, v, b);
        *reinterpret_cast<u32x4*>(q + size_t(col) * pitch + k0) = u32x4{b[0], b[1], b[2], b[3]};
    }
    if (wave == 0) scale[col] = finite ? z.scale : NAN;
}

// W [d_in][d_out] = q scale, rounded once to bf16 (backward multiplies in bf16).  A block of 64 x 64 through LDS: 64 bytes of each row of q are
// read, whole 128-byte lines of W written.  Bound: memory, 4096 x 4096 13 us (3.9 TB/s).
__global__ __launch_bounds__(256) void q8_dequantise_kernel(int32_t d_in, int32_t d_out, int32_t pitch, const uint8_t* __restrict__ q,
                                                            const float* __restrict__ scale, uint16_t* __restrict__ W)
{
    __shared__ __attribute__((aligned(16))) uint8_t tile[64][80];
    const int32_t t = threadIdx.x, n0 = int32_t(blockIdx.x) * 64, k0 = int32_t(blockIdx.y) * 64;
    {
        const int32_t n = t >> 2, c = 16 * (t & 3);
        if (n0 + n < d_out) *reinterpret_cast<u32x4*>(&tile[n][c]) = *reinterpret_cast<const u32x4*>(q + size_t(n0 + n) * pitch + k0 + c);
    }
    __syncthreads();
    const int32_t n = 8 * (t & 7);
    if (n0 + n >= d_out) return;                     // (d_out is a multiple of 8)
    float s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] = scale[n0 + n + e];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int32_t k = (t >> 3) + 32 * h;
        if (k0 + k >= d_in) continue;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = float(int32_t(int8_t(tile[n + e][k]))) * s[e];
        *reinterpret_cast<u32x4*>(W + size_t(k0 + k) * d_out + n0 + n) = Packet<uint16_t>::narrow(v);
    }
}

// (a launch holds less than 2^32 threads)
constexpr int64_t kRowsPerLaunch = 1 << 22;

}  // namespace

hipError_t q8_rows(int64_t T, int32_t d, const void* x, void* q, float* scale, hipStream_t st)
{
    const int32_t pitch = int32_t(q8_pitch(d));
    for (int64_t r = 0; r < T; r += kRowsPerLaunch) {
        const int32_t n = int32_t(T - r < kRowsPerLaunch ? T - r : kRowsPerLaunch);
        const auto go = [&](auto kernel, int32_t rows) {
            kernel<<<dim3(uint32_t((n + rows - 1) / rows)), 256, 0, st>>>(n, d, pitch, static_cast<const uint16_t*>(x) + r * d, static_cast<uint8_t*>(q) + r * pitch,
                                                                         scale + r);
        };
        // a wave per row where a workgroup has less than two packets a thread and there are enough rows (us, a row per wave / workgroup: 16384 x 256
        // 12.6 / 20.6, x 1024 17.0 / 23.1, x 2048 22.3 / 28.0, x 4096 37.9 / 36.0, 8190 x 4096 23.4 / 21.8, 40 x 2048 6.9 / 6.1)
        if (d <= 2048 && n > 1024) go(q8_rows_kernel<1, 8>, 4);
        else d <= 8192 ? go(q8_rows_kernel<4, 4>, 1) : go(q8_rows_kernel<4, 8>, 1);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t q8_weight(int dtype, int32_t d_in, int32_t d_out, int64_t ldw, const void* W, void* q, float* scale, hipStream_t st)
{
    const dim3 grid(uint32_t((int64_t(d_out) + 63) / 64));
    const int32_t pitch = int32_t(q8_pitch(d_in));
    if (dtype == LOBRA_F32)
        q8_weight_kernel<float><<<grid, 64 * kWeightWaves, 0, st>>>(d_in, d_out, pitch, ldw, static_cast<const float*>(W), static_cast<uint8_t*>(q), scale);
    else
        q8_weight_kernel<uint16_t><<<grid, 64 * kWeightWaves, 0, st>>>(d_in, d_out, pitch, ldw, static_cast<const uint16_t*>(W), static_cast<uint8_t*>(q), scale);
    return hipGetLastError();
}

hipError_t q8_dequantise(int32_t d_in, int32_t d_out, const void* q, const float* scale, void* W, hipStream_t st)
{
    const dim3 grid(uint32_t((d_out + 63) / 64), uint32_t((d_in + 63) / 64));
    q8_dequantise_kernel<<<grid, 256, 0, st>>>(d_in, d_out, int32_t(q8_pitch(d_in)), static_cast<const uint8_t*>(q), scale, static_cast<uint16_t*>(W));
    return hipGetLastError();
}

}  // namespace lobra
