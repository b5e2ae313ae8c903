// The layer on a base in 8-bit integers for few tokens (decoding), in two launches: tokens quantised and projected; then the product, which adds the
// adapter term and writes y.
//
// The product reads W once and does next to nothing with it, so what counts is that all of W is on its way at once and that no sum goes through
// memory.  A workgroup has 16 columns, its eight waves share K in pieces of 256, two of them on their way, and the waves' whole sums meet in LDS.
// A lane of the matrix instruction holds 16 k of a column of its own; read like that, each load touches 64 bytes of 16 lines, so four whole lines of
// each of four columns are read instead and turned in LDS.  The tokens (a few hundred KB) come from the L2, as the instruction takes them.
// The projection of a token has a workgroup per quarter of K, since one alone streams the 128 KiB of a rank-16 adapter at K = 4096 for longer than the
// product takes; the quarters' fp32 sums are added where they are used.
//
// us, the tiled product (q8.hip, gemm_tile_q8.hip) / these; one-token segments, K x N:
//     rank  tokens   1            16           40           64
//     16    4096 x 4096     13.6 /  9.6  15.3 / 10.9  15.4 / 13.3  16.6 / 15.5
//     16    4096 x 8192     15.9 / 12.4  18.3 / 14.9  18.9 / 20.8
//     16    4096 x 11008    16.7 / 16.7  18.8 / 19.8  20.2 / 27.3
//     64    4096 x 4096     16.9 / 14.3  18.3 / 18.6 (8 tokens)    19.5 / 22.6
//     16    64 tokens: 1376 x 4096 14.0 / 10.5, 512 x 512 10.9 / 9.3, 11008 x 4096 29.7 / 26.4; 32 tokens: 2048 x 2048 12.3 / 9.0
//     128   8 tokens: 1024 x 1024 15.8 / 19.4
// So not where the columns are more than two workgroups' for every compute unit, each of which takes the tokens from the L2 once more, nor for wide
// adapters, whose ranks are added one by one.
// 40 x 4096 x 4096 otherwise: W read 64 bytes of a line at a time 15.7, three pieces of W on their way 13.8, tokens row by row 0.7 more, 32 columns a
// workgroup half as much again.
#include "gemm_common.h"
#include "kernels.h"
#include "q8_rows.h"

namespace lobra {

using namespace gemm;

namespace {

constexpr int kParts = 4;                            // of K, for the projection
constexpr int kWaves = 8;

__host__ __device__ inline int32_t few_pitch(int32_t r_max) { return (r_max + 3) / 4 * 4; }

// P[part][row][rho] = s_t sum over a quarter of k of x[row][k] A[rho][k], four ranks at a time per wave.
__device__ __forceinline__ void project(const PlanDev& pd, const uint16_t* __restrict__ x, const uint16_t* __restrict__ A, const float* __restrict__ s,
                                        float* __restrict__ P, int32_t row, int32_t part)
{
    const int32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(int32_t(threadIdx.x >> 6));
    const int32_t task = wave_segment(pd, row).task;
    if (task < 0) return;
    const int32_t r0 = pd.rank_off[task], r = pd.rank_off[task + 1] - r0, d = pd.d_in, packets = d / 8, per = (packets + kParts - 1) / kParts;
    const int32_t end = min((part + 1) * per, packets);
    const float st = s[task];
    const u32x4* const xp = reinterpret_cast<const u32x4*>(x + size_t(row) * d);
    const int32_t pitch = few_pitch(pd.r_max);
    float* const out = P + (size_t(part) * pd.T + row) * pitch;
    for (int32_t p0 = 4 * wave; p0 < r; p0 += 16) {
        float acc[4] = {0.f, 0.f, 0.f, 0.f};
        const u32x4* ap[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) ap[q] = reinterpret_cast<const u32x4*>(A + size_t(r0 + min(p0 + q, r - 1)) * d);
#pragma unroll 2
        for (int32_t i = part * per + lane; i < end; i += 64) {
            float xv[8], av[8];
            rows::Packet<uint16_t>::widen(__builtin_bit_cast(rows::u32x4, xp[i]), xv);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                rows::Packet<uint16_t>::widen(__builtin_bit_cast(rows::u32x4, ap[q][i]), av);
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[q] = fmaf(xv[e], av[e], acc[q]);
            }
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float v = rows::wave_sum(acc[q]);
            if (lane == 0 && p0 + q < pitch) out[p0 + q] = p0 + q < r ? st * v : 0.f;
        }
    }
}

// Workgroups 0 .. T - 1 quantise a token each, the others project a quarter of one.
template <int H>
__global__ __launch_bounds__(256) void q8_few_rows_kernel(PlanDev pd, const uint16_t* __restrict__ x, const uint16_t* __restrict__ A,
                                                          const float* __restrict__ s, int32_t pitch, uint8_t* __restrict__ q, float* __restrict__ scale,
                                                          float* __restrict__ P)
{
    __shared__ float part[4];
    const int32_t wg = int32_t(blockIdx.x);
    if (wg < pd.T) rows::quantise_rows<4, H, true>(pd.T, pd.d_in, pitch, x, q, scale, wg, part);
    else project(pd, x, A, s, P, (wg - pd.T) / kParts, (wg - pd.T) % kParts);
}

// y = z_scale w_scale (Z W^T) + P B_t, 16 columns a workgroup, NBT blocks of 16 tokens.  Result layout of the MFMA: lane (j, kg) has columns 4 kg .. + 3 of token j.
template <int NBT>
__global__ __launch_bounds__(64 * kWaves)
void q8_few_kernel(PlanDev pd, const uint8_t* __restrict__ Z, const float* __restrict__ z_scale, const uint8_t* __restrict__ W,
                   const float* __restrict__ w_scale, const float* __restrict__ P, const uint16_t* __restrict__ B, uint16_t* __restrict__ y, int32_t pitch)
{
    constexpr int U = kQ8Pad / 64;                   // steps of 64 k to a piece of K
    static_assert(NBT <= kWaves && NBT <= 4, "a wave ends a block of tokens, and its sums lie where it has turned W");
    __shared__ i32x4 own[kWaves][256];               // a wave's: 256 k of 16 columns, chunk c of column r at 16 r + (c ^ r); then its sums [block][lane]
    const int32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(int32_t(threadIdx.x >> 6));
    const int32_t j = lane & 15, kg = lane >> 4, T = pd.T, N = pd.d_out, col0 = int32_t(blockIdx.x) * 16;
    const int32_t pieces = pitch / kQ8Pad, first = pieces * wave / kWaves, last = pieces * (wave + 1) / kWaves;
    const uint8_t* wp[U];                            // four columns a load, whole lines of each
#pragma unroll
    for (int i = 0; i < U; ++i) wp[i] = W + size_t(min(col0 + 4 * i + (lane >> 4), N - 1)) * pitch + 16 * j;
    const uint8_t* zp[NBT];
#pragma unroll
    for (int b = 0; b < NBT; ++b) zp[b] = Z + size_t(b) * 16 * pitch + 16 * lane;        // (rows beyond T: whatever is there, which goes nowhere)
    i32x4 acc[NBT];
#pragma unroll
    for (int b = 0; b < NBT; ++b) acc[b] = i32x4{0, 0, 0, 0};
    // the wave ends the block of 16 tokens of its number.  A segment per lane (no more of them than tokens): its end, its task's first rank row and rank, on
    // their way before anything else
    const bool ends = wave < NBT;                    // (uniform)
    int32_t end = 0x7fffffff, seg_r0 = 0, seg_r = 0;
    if (ends && P && lane < pd.nseg) {
        end = pd.cseg_off[lane + 1];
        seg_r0 = cseg_rank(pd)[lane];
        seg_r = cseg_rank(pd)[pd.nseg + lane];
    }
    i32x4 w[U], z[U][NBT], wn[U], zn[U][NBT];
    auto load = [&](int32_t g, i32x4 (&wv)[U], i32x4 (&zv)[U][NBT]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < U; ++i) wv[i] = __builtin_nontemporal_load(reinterpret_cast<const i32x4*>(wp[i] + g * kQ8Pad));
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int b = 0; b < NBT; ++b) zv[u][b] = *reinterpret_cast<const i32x4*>(zp[b] + (g * U + u) * 1024);
    };
    if (first < last) load(first, w, z);
    for (int32_t g = first; g < last; ++g) {
        if (g + 1 < last) load(g + 1, wn, zn);
        // (the wave's own part of LDS, whose operations are carried out in order)
#pragma unroll
        for (int i = 0; i < U; ++i) own[wave][16 * (4 * i + (lane >> 4)) + (j ^ (4 * i + (lane >> 4)))] = w[i];
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int u = 0; u < U; ++u) w[u] = own[wave][16 * j + ((4 * u + kg) ^ j)];
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int b = 0; b < NBT; ++b) acc[b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[u], z[u][b], acc[b], 0, 0, 0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            w[u] = wn[u];
#pragma unroll
            for (int b = 0; b < NBT; ++b) z[u][b] = zn[u][b];
        }
    }
#pragma unroll
    for (int b = 0; b < NBT; ++b) own[wave][64 * b + lane] = acc[b];
    // the adapter term of the wave's block, while the others arrive
    const int32_t row = 16 * wave + j, col = col0 + 4 * kg;
    float up[4] = {0.f, 0.f, 0.f, 0.f};
    const bool mine = ends && row < T && col < N;
    if (ends && P) {
        int32_t seg = 0;                             // how many segments end in front of the lane's token
#pragma unroll
        for (int t = 0; t < 16; ++t) {
            const int32_t n = __popcll(__ballot(end <= 16 * wave + t));
            seg = j == t ? n : seg;
        }
        const int32_t r0 = __shfl(seg_r0, seg), stacked = __shfl(seg_r, seg), r = mine ? stacked / pd.n_proj : 0;
        if (r > 0) {
            const int32_t pj = col / pd.dg, pp = few_pitch(pd.r_max);
            const float* const p = P + size_t(row) * pp + pj * r;
            const uint16_t* const m = B + size_t(r0 + pj * r) * pd.dg + (col - pj * pd.dg);
            const size_t part = size_t(T) * pp;
            auto add = [&](float v, uint64_t b) __attribute__((always_inline)) {
                const uint32_t lo = uint32_t(b), hi = uint32_t(b >> 32);
                up[0] = fmaf(v, __uint_as_float(lo << 16), up[0]);
                up[1] = fmaf(v, __uint_as_float(lo & 0xffff0000u), up[1]);
                up[2] = fmaf(v, __uint_as_float(hi << 16), up[2]);
                up[3] = fmaf(v, __uint_as_float(hi & 0xffff0000u), up[3]);
            };
            if (pd.n_proj == 1) {                    // four ranks at a time (P is zero up to the next multiple of four)
#pragma unroll 4
                for (int32_t i = 0; i < r; i += 4) {
                    f32x4 v[kParts];
                    uint64_t b[4];
#pragma unroll
                    for (int q = 0; q < kParts; ++q) v[q] = *reinterpret_cast<const f32x4*>(p + q * part + i);
#pragma unroll
                    for (int q = 0; q < 4; ++q) b[q] = *reinterpret_cast<const uint64_t*>(m + size_t(min(i + q, r - 1)) * pd.dg);
                    const f32x4 sum = (v[0] + v[1]) + (v[2] + v[3]);
#pragma unroll
                    for (int q = 0; q < 4; ++q) add(sum[q], i + q < r ? b[q] : 0);
                }
            } else {
#pragma unroll 4
                for (int32_t i = 0; i < r; ++i)
                    add((p[i] + p[part + i]) + (p[2 * part + i] + p[3 * part + i]), *reinterpret_cast<const uint64_t*>(m + size_t(i) * pd.dg));
            }
        }
    }
    __syncthreads();
    if (!mine) return;
    i32x4 sum = own[0][64 * wave + lane];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) sum = sum + own[w][64 * wave + lane];
    const float zs = z_scale[row];
    const f32x4 ws = *reinterpret_cast<const f32x4*>(w_scale + col);
    bf16x4 o;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        // (a large scale of a channel last: nothing on the way leaves the range, see near_scale; the sum with the adapter's term is one rounding)
        const bool far = ws[v] > 0x1p96f;
        o[v] = (__bf16)(float(sum[v]) * (far ? zs : ws[v]) * (far ? ws[v] : zs) + up[v]);
    }
    *reinterpret_cast<bf16x4*>(y + size_t(row) * N + col) = o;
}

}  // namespace

size_t q8_few_bytes(int64_t T, int32_t r_max) { return size_t(kParts) * size_t(T) * size_t(few_pitch(r_max)) * sizeof(float); }

hipError_t q8_few_rows(const PlanDev& pd, const void* x, const void* A, const float* s, void* q, float* scale, float* P, hipStream_t st)
{
    const int32_t pitch = int32_t(q8_pitch(pd.d_in));
    const dim3 grid(uint32_t(pd.T * (P ? 1 + kParts : 1)));
#define LOBRA_ROWS(H) \
    q8_few_rows_kernel<H><<<grid, 256, 0, st>>>(pd, static_cast<const uint16_t*>(x), static_cast<const uint16_t*>(A), s, pitch, static_cast<uint8_t*>(q), scale, P)
    if (pd.d_in <= 8192) LOBRA_ROWS(4);
    else LOBRA_ROWS(8);
#undef LOBRA_ROWS
    return hipGetLastError();
}

hipError_t q8_few(const PlanDev& pd, const void* Z, const float* z_scale, const void* W, const float* w_scale, const float* P, const void* B, void* y,
                  hipStream_t st)
{
    static_assert(kQ8FewTokens <= 64, "four blocks of 16 tokens");
    if (pd.T < 1 || pd.T > kQ8FewTokens || pd.nseg > 64) return hipErrorInvalidValue;
    const dim3 grid(uint32_t((pd.d_out + 15) / 16));
#define LOBRA_FEW(NBT) \
    q8_few_kernel<NBT><<<grid, 64 * kWaves, 0, st>>>(pd, static_cast<const uint8_t*>(Z), z_scale, static_cast<const uint8_t*>(W), w_scale, P, \
                                                    static_cast<const uint16_t*>(B), static_cast<uint16_t*>(y), int32_t(q8_pitch(pd.d_in)))
    if (pd.T <= 16) LOBRA_FEW(1);
    else if (pd.T <= 32) LOBRA_FEW(2);
    else if (pd.T <= 48) LOBRA_FEW(3);
    else LOBRA_FEW(4);
#undef LOBRA_FEW
    return hipGetLastError();
}

}  // namespace lobra
