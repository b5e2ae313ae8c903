// The gated feed-forward block's forward pass for few tokens (decoding), bf16: the product of up to 64 rows of x with gate and up weights
// as one stream over W, the adapters' down projections in the same launch, and a second launch that adds up, activates and multiplies.
//     [g | u] = x W + s_t (A_t x) B_t   h = a(g) u
//
// Bound: the bytes of W.  Every workgroup streams 64 gate and the 64 matching up columns of W (whole 128-byte lines of it) through an
// LDS ring of direct copies, several K tiles of 64 in flight, and multiplies them with the x of the same k, which all workgroups read from
// the L2.  Where there are fewer column tiles than compute units K is split among workgroups.  The fp32 sums go to scratch (T 2 f 4 bytes
// per split), so that activation, adapters and the sum of the splits see what no rounding has touched; the kernel that does this takes
// the place of the one that would activate [g | u].
// A token's projections H = s_t A_t x, 32 rank rows a workgroup, are independent of the product and need few workgroups: they run
// beside it, in front of the grid.
#include <atomic>

#include "activation.h"
#include "gemm_common.h"
#include "kernels.h"
#include "row_common.h"

namespace lobra {

using namespace gemm;

namespace {

constexpr int KT = 64;                        // k of a tile
constexpr int COLS = 64;                      // gate columns (and up columns) of a workgroup
constexpr int W_BYTES = KT * 2 * COLS * 2;    // 16 KiB: 64 k rows of 128 columns
constexpr int GROUP = 32;                     // rank rows of a projection item
constexpr int LDS_MOST = 144 * 1024;

// TB blocks of 16 tokens; D tiles in the ring
template <int TB> struct Ring {
    static constexpr int X_BYTES = TB * 16 * KT * 2, STAGE = W_BYTES + X_BYTES;
    static constexpr int D = LDS_MOST / STAGE < 8 ? LDS_MOST / STAGE : 8;
    static constexpr int XC = TB < 2 ? 1 : TB / 2;       // x copies per wave (one block: waves 2 and 3 repeat those of 0 and 1)
    static constexpr int NC = 4 + XC;                    // copies per wave and tile
};

// s_t A_t x of one token, 32 rank rows: 8 per wave, K over the lanes
__device__ __forceinline__ void project(const PlanDev& pd, const uint16_t* x, const uint16_t* A, const float* s, float* H, int32_t K, int32_t token,
                                        int32_t group)
{
    const int32_t task = pd.cseg_task[segment_of_row(pd, token)];
    if (task < 0) return;
    const int32_t r0 = pd.rank_off[task], r = pd.rank_off[task + 1] - r0;
    const int lane = threadIdx.x & 63;
    const int32_t first = group * GROUP + __builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6)) * 8;
    if (first >= r) return;
    float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const uint16_t* xr = x + size_t(token) * K;
    for (int32_t k = lane * 8; k < K; k += 512) {
        rows::u32x4 q[8];
        float xv[8];
        rows::Packet<uint16_t>::widen(*reinterpret_cast<const rows::u32x4*>(xr + k), xv);
#pragma unroll
        for (int c = 0; c < 8; ++c)
            q[c] = *reinterpret_cast<const rows::u32x4*>(A + size_t(r0 + min(first + c, r - 1)) * K + k);
#pragma unroll
        for (int c = 0; c < 8; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[c] = fmaf(xv[e], rows::Packet<uint16_t>::element(q[c], e), sum[c]);
    }
    const float st = s[task];
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        const float v = st * rows::wave_sum(sum[c]);
        if (lane == c && first + c < r) H[size_t(token) * pd.r_max + first + c] = v;
    }
}

template <int TB>
__global__ __launch_bounds__(256)
void gated_skinny_kernel(PlanDev pd, const uint16_t* __restrict__ x, const uint16_t* __restrict__ W, const uint16_t* __restrict__ A,
                         const float* __restrict__ s, float* __restrict__ part, float* __restrict__ H, int32_t K, int32_t f, int32_t tiles,
                         int32_t kper, int32_t items, int32_t groups)
{
    typedef Ring<TB> R;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    if (int32_t(blockIdx.x) < items) {
        project(pd, x, A, s, H, K, int32_t(blockIdx.x) / groups, int32_t(blockIdx.x) % groups);
        return;
    }
    const int32_t id = int32_t(blockIdx.x) - items, split = id / tiles, c0 = (id - split * tiles) * COLS;
    const int32_t T = pd.T, k0 = split * kper, k1 = min(K, k0 + kper), steps = (k1 - k0 + KT - 1) / KT;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int j = lane & 15, kg = lane >> 4;
    const uint32_t lds0 = uint32_t(uintptr_t((__attribute__((address_space(3))) unsigned char*)lds));
    const size_t ldw = 2 * size_t(f);

    // Copies of tile t.  W: copy c holds k rows 4 c .. + 3, 16 chunks of 8 columns each, gate's then up's; chunk n of row k at
    // n ^ kn_swz(k).  x: copy c holds tokens 8 c .. + 7, 8 chunks of 8 k each; chunk n of token i at n ^ swz_row(i).  Rows, columns and
    // tokens that are not there repeat the last one; what they add is cleared or not stored.
    auto copy = [&](int32_t t) __attribute__((always_inline)) {
        const int32_t kt = k0 + t * KT;
        const uint32_t stage = lds0 + uint32_t(t % R::D) * R::STAGE;
        const unsigned char* wp = reinterpret_cast<const unsigned char*>(W + size_t(kt) * ldw);
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            const int c = wave + 4 * m, row = 4 * c + (lane >> 4), n = (lane & 15) ^ kn_swz(row);
            const int32_t col = min(c0 + 8 * (n & 7), f - 8) + (n >> 3) * f;
            dma16(stage + c * 1024, wp, (uint32_t(min(row, K - 1 - kt)) * uint32_t(ldw) + uint32_t(col)) * 2u);
        }
        const unsigned char* xp = reinterpret_cast<const unsigned char*>(x + kt);
#pragma unroll
        for (int m = 0; m < R::XC; ++m) {
            const int c = TB < 2 ? (wave & 1) : wave + 4 * m, i = 8 * c + (lane >> 3), n = (lane & 7) ^ swz_row(i);
            dma16(stage + W_BYTES + c * 1024, xp, (uint32_t(min(i, T - 1)) * uint32_t(K) + uint32_t(min(8 * n, K - 8 - kt))) * 2u);
        }
    };

    f32x4 acc[TB][2];
#pragma unroll
    for (int b = 0; b < TB; ++b) acc[b][0] = acc[b][1] = f32x4{0.f, 0.f, 0.f, 0.f};
    const bf16x8 zero = as_bf16x8(u32x4{0u, 0u, 0u, 0u});
    for (int32_t t = 0; t < min(steps, R::D - 1); ++t) copy(t);
    for (int32_t t = 0; t < steps; ++t) {
        // tile t has landed when only the copies of the tiles behind it are on their way
        const int32_t behind = min(steps - 1 - t, R::D - 2);
        static_for<0, R::D - 1>([&](auto n) {
            if (behind == decltype(n)::value) wait_vmcnt<decltype(n)::value * R::NC>();
        });
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();                // (and everybody has read tile t - 1)
        asm volatile("" ::: "memory");
        if (t + R::D - 1 < steps) copy(t + R::D - 1);
        const unsigned char* ws = lds + (t % R::D) * R::STAGE;
        const unsigned char* xs = ws + W_BYTES;
        const int32_t left = K - (k0 + t * KT);
#pragma unroll
        for (int ks = 0; ks < KT / 32; ++ks) {
            const int krow = 32 * ks + 8 * kg + (j >> 2);
            bf16x8 wf[2], xf[TB];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int n = COLS * half + 16 * wave + 4 * (j & 3);
                wf[half] = tr_pair(ws + krow * 256 + ((n >> 3) ^ kn_swz(krow)) * 16 + (n & 7) * 2, 256);
            }
#pragma unroll
            for (int b = 0; b < TB; ++b) {
                const int i = 16 * b + j;
                xf[b] = *reinterpret_cast<const bf16x8*>(xs + i * (KT * 2) + ((4 * ks + kg) ^ swz_row(i)) * 16);
            }
            if (32 * ks + 32 > left) {               // (uniform) k beyond K: cleared in both operands
                const bool in = 32 * ks + 8 * kg < left;
#pragma unroll
                for (int half = 0; half < 2; ++half) wf[half] = in ? wf[half] : zero;
#pragma unroll
                for (int b = 0; b < TB; ++b) xf[b] = in ? xf[b] : zero;
            }
#pragma unroll
            for (int b = 0; b < TB; ++b)
#pragma unroll
                for (int half = 0; half < 2; ++half)
                    acc[b][half] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[half], xf[b], acc[b][half], 0, 0, 0);
        }
    }
    // lane (j, kg): columns 16 wave + 4 kg .. + 3 of token j of a block
    const int32_t col = c0 + 16 * wave + 4 * kg;
    if (col >= f) return;
#pragma unroll
    for (int b = 0; b < TB; ++b) {
        const int32_t i = 16 * b + j;
        if (i >= T) continue;
        float* dst = part + (size_t(split) * T + i) * ldw + col;
        *reinterpret_cast<f32x4*>(dst) = acc[b][0];
        *reinterpret_cast<f32x4*>(dst + f) = acc[b][1];
    }
}

// Sum of the splits, adapter term, activation and product: a thread has 8 columns of a token.
template <int ACT>
__global__ __launch_bounds__(256)
void gated_skinny_finish_kernel(PlanDev pd, const float* __restrict__ part, const float* __restrict__ H, const uint16_t* __restrict__ B, int32_t f,
                                int32_t splits, uint16_t* __restrict__ gu, uint16_t* __restrict__ h)
{
    const int32_t col = (int32_t(blockIdx.x) * 256 + int32_t(threadIdx.x)) * 8, i = blockIdx.y, T = pd.T;
    if (col >= f) return;
    const size_t ldw = 2 * size_t(f);
    float g[8], u[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) g[e] = u[e] = 0.f;
    for (int32_t k = 0; k < splits; ++k) {
        const f32x4* p = reinterpret_cast<const f32x4*>(part + (size_t(k) * T + i) * ldw + col);
        const f32x4* q = reinterpret_cast<const f32x4*>(part + (size_t(k) * T + i) * ldw + f + col);
        const f32x4 a = p[0], b = p[1], c = q[0], d = q[1];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            g[e] += a[e];
            g[4 + e] += b[e];
            u[e] += c[e];
            u[4 + e] += d[e];
        }
    }
    const int32_t task = H ? pd.cseg_task[segment_of_row(pd, i)] : -1;
    if (task >= 0) {
        const int32_t r0 = pd.rank_off[task], r = (pd.rank_off[task + 1] - r0) / 2;
        const float* hv = H + size_t(i) * pd.r_max;
        const uint16_t* b0 = B + size_t(r0) * f + col;
#pragma unroll 4
        for (int32_t k = 0; k < r; ++k) {
            float bg[8], bu[8];
            rows::Packet<uint16_t>::widen(*reinterpret_cast<const rows::u32x4*>(b0 + size_t(k) * f), bg);
            rows::Packet<uint16_t>::widen(*reinterpret_cast<const rows::u32x4*>(b0 + size_t(r + k) * f), bu);
            const float hg = hv[k], hu = hv[r + k];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                g[e] = fmaf(hg, bg[e], g[e]);
                u[e] = fmaf(hu, bu[e], u[e]);
            }
        }
    }
    if (gu) {
        *reinterpret_cast<rows::u32x4*>(gu + size_t(i) * ldw + col) = rows::Packet<uint16_t>::narrow(g);
        *reinterpret_cast<rows::u32x4*>(gu + size_t(i) * ldw + f + col) = rows::Packet<uint16_t>::narrow(u);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) g[e] = activate<ACT>(g[e]) * u[e];
    *reinterpret_cast<rows::u32x4*>(h + size_t(i) * f + col) = rows::Packet<uint16_t>::narrow(g);
}

struct Cut {
    int32_t tiles, splits, kper, groups, items;
};
// A workgroup per compute unit: what the projections' workgroups leave of 256 is split among the column tiles, four K tiles each at least.
Cut cut(int64_t T, int32_t K, int32_t f, int32_t r_max)
{
    Cut c;
    c.tiles = (f + COLS - 1) / COLS;
    c.groups = (r_max + GROUP - 1) / GROUP;
    c.items = int32_t(T) * c.groups;
    const int32_t room = (c.items < 128 ? 256 - c.items : 128) / c.tiles, most = K / (4 * KT);
    int32_t s = room < most ? room : most;
    s = s < 1 ? 1 : s > 16 ? 16 : s;
    c.kper = ((K + s - 1) / s + KT - 1) / KT * KT;
    c.splits = (K + c.kper - 1) / c.kper;
    return c;
}

template <int TB>
hipError_t launch(const PlanDev& pd, const Cut& c, const uint16_t* x, const uint16_t* W, const uint16_t* A, const float* s, float* part, float* H,
                  int32_t K, int32_t f, hipStream_t st)
{
    typedef Ring<TB> R;
    constexpr int bytes = R::D * R::STAGE;
    // once per device: more dynamic LDS than the default limit
    static std::atomic<bool> ready[64];
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    if (dev < 0 || dev >= 64) return hipErrorInvalidDevice;
    if (!ready[dev].load(std::memory_order_acquire)) {
        e = hipFuncSetAttribute(reinterpret_cast<const void*>(&gated_skinny_kernel<TB>), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e != hipSuccess) return e;
        ready[dev].store(true, std::memory_order_release);
    }
    const int32_t items = H ? c.items : 0;
    gated_skinny_kernel<TB><<<dim3(uint32_t(items + c.tiles * c.splits)), 256, bytes, st>>>(pd, x, W, A, s, part, H, K, f, c.tiles, c.kper, items,
                                                                                           c.groups);
    return hipGetLastError();
}

size_t align256(size_t v) { return (v + 255) / 256 * 256; }

}  // namespace

size_t gated_skinny_ws_bytes(int64_t T, int32_t K, int32_t f, int32_t r_max)
{
    return align256(size_t(cut(T, K, f, r_max).splits) * size_t(T) * 2 * size_t(f) * 4) + align256(size_t(T) * size_t(r_max) * 4);
}

hipError_t gated_skinny_product(const PlanDev& pd, const void* x, const void* W, const void* A, const float* s, void* ws, bool adapters, hipStream_t st)
{
    const int32_t K = pd.d_in, f = pd.dg;
    const Cut c = cut(pd.T, K, f, pd.r_max);
    float* part = static_cast<float*>(ws);
    float* H = adapters ? reinterpret_cast<float*>(static_cast<char*>(ws) + align256(size_t(c.splits) * size_t(pd.T) * 2 * size_t(f) * 4)) : nullptr;
    const uint16_t *xp = static_cast<const uint16_t*>(x), *wp = static_cast<const uint16_t*>(W), *ap = static_cast<const uint16_t*>(A);
    return pd.T <= 16 ? launch<1>(pd, c, xp, wp, ap, s, part, H, K, f, st) : pd.T <= 32 ? launch<2>(pd, c, xp, wp, ap, s, part, H, K, f, st)
                                                                                      : launch<4>(pd, c, xp, wp, ap, s, part, H, K, f, st);
}

hipError_t gated_skinny_finish(const PlanDev& pd, int act, const void* B, const void* ws, bool adapters, void* gu, void* h, hipStream_t st)
{
    const int32_t f = pd.dg;
    const Cut c = cut(pd.T, pd.d_in, f, pd.r_max);
    const float* part = static_cast<const float*>(ws);
    const float* H = adapters ? reinterpret_cast<const float*>(static_cast<const char*>(ws) + align256(size_t(c.splits) * size_t(pd.T) * 2 * size_t(f) * 4)) : nullptr;
    const dim3 grid(uint32_t((f / 8 + 255) / 256), uint32_t(pd.T));
    const uint16_t* b = static_cast<const uint16_t*>(B);
    uint16_t *g = static_cast<uint16_t*>(gu), *o = static_cast<uint16_t*>(h);
    if (act == LOBRA_ACT_SILU) gated_skinny_finish_kernel<LOBRA_ACT_SILU><<<grid, 256, 0, st>>>(pd, part, H, b, f, c.splits, g, o);
    else gated_skinny_finish_kernel<LOBRA_ACT_GELU_TANH><<<grid, 256, 0, st>>>(pd, part, H, b, f, c.splits, g, o);
    return hipGetLastError();
}

}  // namespace lobra
