// The gated feed-forward block's forward pass for up to 64 tokens, fp32: the products of x with gate and up weights cut along K to fill the
// chip, the adapters' down projections in the same launch, and a second launch that adds up, activates and
// multiplies.
//     [g | u] = x W + s_t (A_t x) B_t   h = a(g) u
//
// Bound: the bytes of W for wide layers, launches and memory round trips for narrow ones (a product per projection, the adapters' term and the
// activation apart are four launches that wait for each other).  A workgroup has 64 gate and the 64 matching up columns of a range of K; its four
// waves take 16 k of it in turns, straight from memory into the matrix instructions: lane (j, kg) reads 4 columns from column 4 j on of the rows
// k = 4 kg + i, i = 0 .. 3, and 4 k from k = 4 kg on of token j (rows of x begin at any element), so that instruction i multiplies the same k of
// both.  The waves' sums meet in LDS.  Four blocks of 16 tokens take 256 registers, two workgroups to a compute unit, and 68 bytes a lane of scratch
// memory.
// Measured against the layer's products and an activation (8 tasks of rank 16, us, here / those): 4096 x 2 x 11008 with 4, 28, 64 tokens 77 / 137
// (of 361 MB, 4.7 TB/s), 95 / 168, 166 / 211; 919 x 2 x 256 11 / 35, 14 / 45, 18 / 46; 326 x 2 x 1408 9 / 27, 12 / 36, 18 / 37.
#include "activation.h"
#include "gemm_common.h"
#include "kernels.h"
#include "row_common.h"

namespace lobra {

using namespace gemm;

namespace {

constexpr int COLS = 64, NW = 4, STEP = 16;          // columns of a tile (of gate and of up), waves, k of a wave's turn
constexpr int ROUND = NW * STEP;

typedef float AnyFloats __attribute__((ext_vector_type(4), aligned(4)));         // (global memory is read in 16 bytes from any multiple of 4)

struct Cut {
    int32_t tiles, splits, per;                      // column tiles, parts of K, k of a part (a multiple of ROUND)
};

// H[token][row] = s_t (A_t x)[row]: four rank rows of a token at a time, item `wave` of every `waves`, K over a wave's lanes
__device__ __forceinline__ void project(const PlanDev& pd, const float* x, const float* A, const float* s, float* H, int32_t K, int32_t wave, int32_t waves)
{
    constexpr int ROWS = 4;                          // (stacked ranks are multiples of 16)
    const int lane = threadIdx.x & 63;
    const int32_t groups = pd.r_max / ROWS;
    for (int32_t n = wave; n < pd.T * groups; n += waves) {
        const int32_t token = n / groups, row = (n - token * groups) * ROWS;
        const int32_t task = wave_segment(pd, token).task;
        if (task < 0) continue;
        const int32_t r0 = pd.rank_off[task];
        if (row >= pd.rank_off[task + 1] - r0) continue;
        const float *xr = x + size_t(token) * K, *ar = A + size_t(r0 + row) * K;
        float sum[ROWS] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int32_t k = 4 * lane; k + 3 < K; k += 256) {
            const AnyFloats p = *reinterpret_cast<const AnyFloats*>(xr + k);
#pragma unroll
            for (int c = 0; c < ROWS; ++c) {
                const AnyFloats q = *reinterpret_cast<const AnyFloats*>(ar + size_t(c) * K + k);
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[c] = fmaf(p[e], q[e], sum[c]);
            }
        }
        const int32_t last = (K & ~3) + lane;
        if (last < K)
#pragma unroll
            for (int c = 0; c < ROWS; ++c) sum[c] = fmaf(xr[last], ar[size_t(c) * K + last], sum[c]);
        const float st = s[task];
#pragma unroll
        for (int c = 0; c < ROWS; ++c) {
            const float v = st * rows::wave_sum(sum[c]);
            if (lane == c) H[size_t(token) * pd.r_max + row + c] = v;
        }
    }
}

// TB blocks of 16 tokens
constexpr int resident(int tb) { return tb == 1 ? 4 : tb == 2 ? 3 : 2; }           // workgroups of a compute unit
template <int TB>
__global__ __launch_bounds__(64 * NW, resident(TB))
void gated_few_kernel(PlanDev pd, const float* __restrict__ x, const float* __restrict__ W, const float* __restrict__ A, const float* __restrict__ s,
                      float* __restrict__ part, float* __restrict__ H, int32_t K, int32_t f, Cut cut)
{
    __shared__ f32x4 sums[2][8 * TB][64];
    const int32_t id = blockIdx.x, T = pd.T;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, j = lane & 15, kg = lane >> 4;
    if (id >= cut.tiles * cut.splits) {              // (only with adapters)
        const int32_t first = cut.tiles * cut.splits;
        project(pd, x, A, s, H, K, (id - first) * NW + wave, (int32_t(gridDim.x) - first) * NW);
        return;
    }
    const int32_t split = id / cut.tiles, tile = id - split * cut.tiles;
    const int32_t k0 = split * cut.per, k1 = min(k0 + cut.per, K), c0 = tile * COLS;
    const size_t ldw = 2 * size_t(f);
    const float* wp = W + min(c0 + 4 * j, f - 4);    // (columns that are not there repeat the last ones and are not stored)
    const float* xp[TB];
#pragma unroll
    for (int b = 0; b < TB; ++b) xp[b] = x + size_t(min(16 * b + j, T - 1)) * K;
    f32x4 acc[TB][2][4];                             // [half][e]: columns 4 (4 kg + v) + e of token j
#pragma unroll
    for (int b = 0; b < TB; ++b)
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[b][half][e] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto turn = [&](int32_t k, bool whole) __attribute__((always_inline)) {
        const int32_t kk = k + 4 * kg;               // this lane's first k
        f32x4 w[2][4], z[TB];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float* p = wp + size_t(whole ? kk + i : min(kk + i, K - 1)) * ldw;
            w[0][i] = *reinterpret_cast<const f32x4*>(p);
            w[1][i] = *reinterpret_cast<const f32x4*>(p + f);
        }
#pragma unroll
        for (int b = 0; b < TB; ++b) {
            if (whole) {
                z[b] = *reinterpret_cast<const AnyFloats*>(xp[b] + kk);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) z[b][i] = xp[b][min(kk + i, K - 1)];
            }
        }
        if (!whole)                                  // k beyond K: nothing of either operand
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool in = kk + i < K;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    w[0][i][e] = in ? w[0][i][e] : 0.f;
                    w[1][i][e] = in ? w[1][i][e] : 0.f;
                }
#pragma unroll
                for (int b = 0; b < TB; ++b) z[b][i] = in ? z[b][i] : 0.f;
            }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int b = 0; b < TB; ++b)
#pragma unroll
                for (int half = 0; half < 2; ++half)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        acc[b][half][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(w[half][i][e], z[b][i], acc[b][half][e], 0, 0, 0);
    };
    int32_t k = k0 + wave * STEP;
#pragma unroll 2
    for (; k + STEP <= k1; k += ROUND) turn(k, true);
    if (k < k1) turn(k, false);                      // (only at the end of K: parts are whole rounds)
    // waves 2 and 3 hand their sums to 0 and 1, then 1 to 0
#pragma unroll
    for (int far = 2; far > 0; far >>= 1) {
        if (far == 1) __syncthreads();
        if (wave >= far && wave < 2 * far)
#pragma unroll
            for (int b = 0; b < TB; ++b)
#pragma unroll
                for (int half = 0; half < 2; ++half)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sums[wave - far][(b * 2 + half) * 4 + e][lane] = acc[b][half][e];
        __syncthreads();
        if (wave < far)
#pragma unroll
            for (int b = 0; b < TB; ++b)
#pragma unroll
                for (int half = 0; half < 2; ++half)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[b][half][e] = acc[b][half][e] + sums[wave][(b * 2 + half) * 4 + e][lane];
    }
    if (wave != 0) return;
    // lane (j, kg): columns 16 kg .. + 15 of token j of a block
    float* dst = part + size_t(id) * 2 * size_t(T) * COLS + 16 * kg;
#pragma unroll
    for (int b = 0; b < TB; ++b)
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int32_t i = 16 * b + j;
            if (i >= T) continue;
#pragma unroll
            for (int v = 0; v < 4; ++v)
                *reinterpret_cast<f32x4*>(dst + (size_t(half) * T + i) * COLS + 4 * v) =
                    f32x4{acc[b][half][0][v], acc[b][half][1][v], acc[b][half][2][v], acc[b][half][3][v]};
        }
}

// Sum of the parts, adapter term, activation and product: a thread has 4 columns of a token.
template <int ACT>
__global__ __launch_bounds__(64)
void gated_few_finish_kernel(PlanDev pd, const float* __restrict__ part, const float* __restrict__ H, const float* __restrict__ B, int32_t f, Cut cut,
                             float* __restrict__ gu, float* __restrict__ h)
{
    const int32_t col = (int32_t(blockIdx.x) * 64 + int32_t(threadIdx.x)) * 4, i = blockIdx.y, T = pd.T;
    const int32_t task = H ? wave_segment(pd, i).task : -1;
    if (col >= f) return;
    const int32_t tile = col / COLS;
    const float* at = part + (size_t(tile) * 2 * T + i) * COLS + col % COLS;
    const size_t stride = size_t(cut.tiles) * 2 * size_t(T) * COLS;
    f32x4 g = {0.f, 0.f, 0.f, 0.f}, u = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int32_t n = 0; n < cut.splits; ++n) {
        g = g + *reinterpret_cast<const f32x4*>(at + n * stride);
        u = u + *reinterpret_cast<const f32x4*>(at + n * stride + size_t(T) * COLS);
    }
    if (task >= 0) {
        const int32_t r0 = pd.rank_off[task], r = (pd.rank_off[task + 1] - r0) / 2;
        const float *hv = H + size_t(i) * pd.r_max, *bg = B + size_t(r0) * f + col, *bu = bg + size_t(r) * f;
#pragma unroll 8
        for (int32_t k = 0; k < r; ++k) {
            g = g + hv[k] * *reinterpret_cast<const f32x4*>(bg + size_t(k) * f);
            u = u + hv[r + k] * *reinterpret_cast<const f32x4*>(bu + size_t(k) * f);
        }
    }
    if (gu) {
        *reinterpret_cast<f32x4*>(gu + size_t(i) * 2 * f + col) = g;
        *reinterpret_cast<f32x4*>(gu + size_t(i) * 2 * f + f + col) = u;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) g[e] = activate<ACT>(g[e]) * u[e];
    *reinterpret_cast<f32x4*>(h + size_t(i) * f + col) = g;
}

int token_blocks(int64_t T) { return int((T + 15) / 16); }

// The parts of K that take the least: rounds of resident workgroups, each at the bytes of W of its part, and the sums' way to memory and back.
Cut make_cut(int64_t T, int32_t K, int32_t f)
{
    Cut c;
    c.tiles = (f + COLS - 1) / COLS;
    const int32_t rounds = (K + ROUND - 1) / ROUND;
    const int64_t slots = 256 * resident(token_blocks(T));
    double least = 0.;
    for (int32_t n = 1; n <= rounds && n <= 64; ++n) {
        const int32_t per = (rounds + n - 1) / n, splits = (rounds + per - 1) / per;
        const int64_t wgs = int64_t(c.tiles) * splits;
        const double cost = double((wgs + slots - 1) / slots) * slots * per * ROUND * 2 * COLS * 4 + double(wgs) * T * 2 * COLS * 8;
        if (n == 1 || cost < least) least = cost, c.per = per * ROUND, c.splits = splits;
    }
    return c;
}
size_t align256(size_t v) { return (v + 255) / 256 * 256; }
size_t part_bytes(const Cut& c, int64_t T) { return align256(size_t(c.splits) * c.tiles * 2 * size_t(T) * COLS * 4); }

}  // namespace

size_t gated_few_ws_bytes(int64_t T, int32_t K, int32_t f, int32_t r_max)
{
    return part_bytes(make_cut(T, K, f), T) + align256(size_t(T) * size_t(r_max) * 4);
}

hipError_t gated_few_product(const PlanDev& pd, const float* x, const float* W, const float* A, const float* s, void* ws, bool adapters, hipStream_t st)
{
    const int32_t K = pd.d_in, f = pd.dg;
    const Cut c = make_cut(pd.T, K, f);
    float* part = static_cast<float*>(ws);
    float* H = adapters ? reinterpret_cast<float*>(static_cast<char*>(ws) + part_bytes(c, pd.T)) : nullptr;
    const int32_t items = H ? pd.T * (pd.r_max / 4) : 0, projections = (items + NW - 1) / NW;
    const dim3 grid(uint32_t(c.tiles * c.splits + (projections < 256 ? projections : 256)));
    switch (token_blocks(pd.T)) {
    case 1: gated_few_kernel<1><<<grid, 64 * NW, 0, st>>>(pd, x, W, A, s, part, H, K, f, c); break;
    case 2: gated_few_kernel<2><<<grid, 64 * NW, 0, st>>>(pd, x, W, A, s, part, H, K, f, c); break;
    case 3: gated_few_kernel<3><<<grid, 64 * NW, 0, st>>>(pd, x, W, A, s, part, H, K, f, c); break;
    default: gated_few_kernel<4><<<grid, 64 * NW, 0, st>>>(pd, x, W, A, s, part, H, K, f, c); break;
    }
    return hipGetLastError();
}

hipError_t gated_few_finish(const PlanDev& pd, int act, const float* B, const void* ws, bool adapters, float* gu, float* h, hipStream_t st)
{
    const int32_t f = pd.dg;
    const Cut c = make_cut(pd.T, pd.d_in, f);
    const float* part = static_cast<const float*>(ws);
    const float* H = adapters ? reinterpret_cast<const float*>(static_cast<const char*>(ws) + part_bytes(c, pd.T)) : nullptr;
    const dim3 grid(uint32_t((f / 4 + 63) / 64), uint32_t(pd.T));
    if (act == LOBRA_ACT_SILU) gated_few_finish_kernel<LOBRA_ACT_SILU><<<grid, 64, 0, st>>>(pd, part, H, B, f, c, gu, h);
    else gated_few_finish_kernel<LOBRA_ACT_GELU_TANH><<<grid, 64, 0, st>>>(pd, part, H, B, f, c, gu, h);
    return hipGetLastError();
}

}  // namespace lobra
