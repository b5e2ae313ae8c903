// The gated feed-forward block's forward pass for few tokens (decoding), bf16: the product of up to 128 rows of x with gate and up weights
// as one stream over W, the adapters' down projections in the same launch, and a second launch that adds up, activates and multiplies.
//     [g | u] = x W + s_t (A_t x) B_t   h = a(g) u
//
// Bound: the bytes of W.  A column tile is 128 gate and the 128 matching up columns (256 contiguous bytes of W: a plain read of the same W
// in pieces of 128, 256 and 512 bytes reaches 5.3, 6.0 and 6.4 TB/s); its K tiles of 64 go through an LDS ring of direct copies, several
// of them in flight, and meet the x of the same k, which all workgroups read from the L2.  All K tiles of all column tiles are one list
// that is dealt evenly to a workgroup per compute unit, and a workgroup writes its fp32 sums where its part of a column tile ends (to
// slot workgroup + tile, which no two parts share).  Activation, adapters and the sum of the parts thus see what no rounding has touched;
// the kernel that does this takes the place of the one that would activate [g | u].
// The projections H = s_t A_t x are dealt to the same workgroups' waves, four rank rows of a token at a time, while their first K
// tiles are on their way.  (Workgroups of their own in front of the grid hold up the stream of a compute unit each: 6 us of 44.)
// Measured (4096 x 2 x 11008, 8 tasks of rank 16, us): 40 tokens 36 .. 38 (180 MB, 5.0 TB/s) and 7.5; W copied as data that is read again 5 more.
// Against the layer's product and an activation behind it (both launches / those): 65 tokens 51 / 67, 128 tokens 63 / 74; 128 tokens of 4096 x 2 x
// 1376 30 / 41, of 1024 x 2 x 2816 23 / 23.  More tokens leave the ring less than two tiles on their way.
#include <atomic>

#include "activation.h"
#include "gemm_common.h"
#include "kernels.h"
#include "row_common.h"

namespace lobra {

using namespace gemm;

namespace {

constexpr int KT = 64;                        // k of a tile
constexpr int COLS = 128;                     // gate columns (and up columns) of a column tile
constexpr int W_BYTES = KT * 2 * COLS * 2;    // 32 KiB: 64 k rows of 256 columns
constexpr int LDS_MOST = 160 * 1024;
constexpr int NW = 8;                         // waves

// TB blocks of 16 tokens; D tiles in the ring
template <int TB> struct Ring {
    static constexpr int X_BYTES = TB * 16 * KT * 2, STAGE = W_BYTES + X_BYTES;
    static constexpr int D = LDS_MOST / STAGE;
    static constexpr int XC = (2 * TB + NW - 1) / NW, NC = 4 + XC;         // copies per wave and tile: of x (2 TB copies of 8 tokens: waves left over
                                                                           // repeat some), and with those of W
};

// Task of a token, looked up by a whole wave: no more segments than tokens, two per lane.  (A chain of two reads less than segment_of_row,
// which walks the table.)
static_assert(kSkinnyTokens <= 128, "two segments a lane");
__device__ __forceinline__ int32_t token_task(const PlanDev& pd, int32_t token)
{
    const int lane = threadIdx.x & 63;
    const int32_t a = min(lane, pd.nseg - 1), b = min(64 + lane, pd.nseg - 1);
    const int32_t enda = pd.cseg_off[a + 1], endb = pd.cseg_off[b + 1], taska = pd.cseg_task[a], taskb = pd.cseg_task[b];
    const int k = __popcll(__ballot(lane < pd.nseg && enda <= token)) + __popcll(__ballot(64 + lane < pd.nseg && endb <= token));
    return k < 64 ? __builtin_amdgcn_readlane(taska, k) : __builtin_amdgcn_readlane(taskb, k - 64);
}

// H[token][row] = s_t (A_t x)[row]: ROWS rank rows of a token at a time, item `wave` of every `waves`, K over a wave's lanes
__device__ __forceinline__ void project(const PlanDev& pd, const uint16_t* x, const uint16_t* A, const float* s, float* H, int32_t K, int32_t wave,
                                        int32_t waves)
{
    constexpr int ROWS = 4;                          // (stacked ranks are multiples of 16)
    const int lane = threadIdx.x & 63;
    const int32_t groups = pd.r_max / ROWS;
    for (int32_t n = wave; n < pd.T * groups; n += waves) {
        const int32_t token = n / groups, row = (n - token * groups) * ROWS;
        const int32_t task = token_task(pd, token);
        if (task < 0) continue;
        const int32_t r0 = pd.rank_off[task];
        if (row >= pd.rank_off[task + 1] - r0) continue;
        const uint16_t *xr = x + size_t(token) * K, *ar = A + size_t(r0 + row) * K;
        float sum[ROWS] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 2
        for (int32_t k = lane * 8; k < K; k += 512) {
            rows::u32x4 q[ROWS];
            const rows::u32x4 p = *reinterpret_cast<const rows::u32x4*>(xr + k);
#pragma unroll
            for (int c = 0; c < ROWS; ++c) q[c] = *reinterpret_cast<const rows::u32x4*>(ar + size_t(c) * K + k);
#pragma unroll
            for (int c = 0; c < ROWS; ++c)
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[c] = fmaf(rows::Packet<uint16_t>::element(p, e), rows::Packet<uint16_t>::element(q[c], e), sum[c]);
        }
        const float st = s[task];
#pragma unroll
        for (int c = 0; c < ROWS; ++c) {
            const float v = st * rows::wave_sum(sum[c]);
            if (lane == c) H[size_t(token) * pd.r_max + row + c] = v;
        }
    }
}

// The list of K tiles and how it is dealt.
struct Cut {
    int32_t tiles, ks, per, streams;                     // column tiles, K tiles of one, K tiles of a workgroup, workgroups
};

template <int TB>
__global__ __launch_bounds__(64 * NW)
void gated_skinny_kernel(PlanDev pd, const uint16_t* __restrict__ x, const uint16_t* __restrict__ W, const uint16_t* __restrict__ A,
                         const float* __restrict__ s, float* __restrict__ part, float* __restrict__ H, int32_t K, int32_t f, Cut cut)
{
    typedef Ring<TB> R;
    extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
    const int32_t id = blockIdx.x, first = id * cut.per, steps = min(cut.per, cut.tiles * cut.ks - first);      // (steps <= 0: projections alone)
    const int32_t T = pd.T;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int j = lane & 15, kg = lane >> 4;
    const uint32_t lds0 = uint32_t(uintptr_t((__attribute__((address_space(3))) unsigned char*)lds));
    const size_t ldw = 2 * size_t(f);
    struct Cursor {
        int32_t tile, kt, stage;                     // column tile, K tile of it, place in the ring
    };
    auto advance = [&](Cursor& c) __attribute__((always_inline)) {
        c.stage = c.stage + 1 == R::D ? 0 : c.stage + 1;
        if (++c.kt == cut.ks) {
            c.kt = 0;
            ++c.tile;
        }
    };

    // Copies of a K tile.  W: copy c holds k rows 2 c and 2 c + 1, 32 chunks of 8 columns each, gate's then up's; chunk n of row k at
    // n ^ kn_swz(k).  x: copy c holds tokens 8 c .. + 7, 8 chunks of 8 k each; chunk n of token i at n ^ swz_row(i).  Rows, columns and
    // tokens that are not there repeat the last one; what they add is cleared or not stored.
    uint32_t wvo[4], xvo[R::XC];                     // a whole tile's offsets from its first row and column, and from its first k
#pragma unroll
    for (int m = 0; m < 4; ++m) {
        const int row = 2 * (wave + NW * m) + (lane >> 5), n = (lane & 31) ^ kn_swz(row);
        wvo[m] = (uint32_t(row) * uint32_t(ldw) + uint32_t(8 * (n & 15)) + uint32_t(n >> 4) * uint32_t(f)) * 2u;
    }
    int xc[R::XC], xn[R::XC];
#pragma unroll
    for (int m = 0; m < R::XC; ++m) {
        xc[m] = (wave + NW * m) % (2 * TB);
        const int xi = 8 * xc[m] + (lane >> 3);
        xn[m] = (lane & 7) ^ swz_row(xi);
        xvo[m] = (uint32_t(min(xi, T - 1)) * uint32_t(K) + uint32_t(8 * xn[m])) * 2u;
    }
    auto copy = [&](const Cursor& u) __attribute__((always_inline)) {
        const int32_t kt = u.kt * KT, c0 = u.tile * COLS;
        const uint32_t stage = lds0 + uint32_t(u.stage) * R::STAGE;
        const unsigned char* wp = reinterpret_cast<const unsigned char*>(W + size_t(kt) * ldw + c0);
        const unsigned char* xp = reinterpret_cast<const unsigned char*>(x + kt);
        if (kt + KT <= K && c0 + COLS <= f) {        // (uniform)
#pragma unroll
            for (int m = 0; m < 4; ++m) dma16_once(stage + (wave + NW * m) * 1024, wp, wvo[m]);
#pragma unroll
            for (int m = 0; m < R::XC; ++m) dma16(stage + W_BYTES + xc[m] * 1024, xp, xvo[m]);
            return;
        }
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            const int c = wave + NW * m, row = 2 * c + (lane >> 5), n = (lane & 31) ^ kn_swz(row);
            const int32_t col = min(8 * (n & 15), f - 8 - c0) + (n >> 4) * f;
            dma16_once(stage + c * 1024, wp, (uint32_t(min(row, K - 1 - kt)) * uint32_t(ldw) + uint32_t(col)) * 2u);
        }
#pragma unroll
        for (int m = 0; m < R::XC; ++m) dma16(stage + W_BYTES + xc[m] * 1024, xp, xvo[m] - 2u * uint32_t(8 * xn[m] - min(8 * xn[m], K - 8 - kt)));
    };

    // wave w: columns 16 w .. + 15 of gate and of up
    f32x4 acc[TB][2];
#pragma unroll
    for (int b = 0; b < TB; ++b) acc[b][0] = acc[b][1] = f32x4{0.f, 0.f, 0.f, 0.f};
    const bf16x8 zero = as_bf16x8(u32x4{0u, 0u, 0u, 0u});
    Cursor at{first / cut.ks, 0, 0}, ahead;
    at.kt = first - at.tile * cut.ks;
    ahead = at;
    for (int32_t t = 0; t < min(steps, R::D - 1); ++t) {
        copy(ahead);
        advance(ahead);
    }
    if (H) project(pd, x, A, s, H, K, id * NW + wave, int32_t(gridDim.x) * NW);
    for (int32_t t = 0; t < steps; ++t) {
        // tile t has landed when only the copies of the tiles behind it are on their way (and what is stored behind those)
        const int32_t behind = min(steps - 1 - t, R::D - 2);
        static_for<0, R::D - 1>([&](auto n) {
            if (behind == decltype(n)::value) wait_vmcnt<decltype(n)::value * R::NC>();
        });
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();                // (and everybody has read tile t - 1)
        asm volatile("" ::: "memory");
        if (t + R::D - 1 < steps) {
            copy(ahead);
            advance(ahead);
        }
        const unsigned char* ws = lds + at.stage * R::STAGE;
        const unsigned char* xs = ws + W_BYTES;
        const int32_t left = K - at.kt * KT;
#pragma unroll
        for (int ks = 0; ks < KT / 32; ++ks) {
            const int krow = 32 * ks + 8 * kg + (j >> 2);
            bf16x8 wf[2], xf[TB];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int n = COLS * half + 16 * wave + 4 * (j & 3);
                wf[half] = tr_pair(ws + krow * 512 + ((n >> 3) ^ kn_swz(krow)) * 16 + (n & 7) * 2, 512);
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
        // the end of this workgroup's part of a column tile
        if (at.kt + 1 == cut.ks || t + 1 == steps) {
            // lane (j, kg): columns 16 wave + 4 kg .. + 3 of token j of a block
            float* dst = part + size_t(id + at.tile) * 2 * size_t(T) * COLS + 16 * wave + 4 * kg;
#pragma unroll
            for (int b = 0; b < TB; ++b)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int32_t i = 16 * b + j;
                    if (i < T) *reinterpret_cast<f32x4*>(dst + (size_t(half) * T + i) * COLS) = acc[b][half];
                    acc[b][half] = f32x4{0.f, 0.f, 0.f, 0.f};
                }
        }
        advance(at);
    }
}

// Sum of the parts, adapter term, activation and product: a thread has 8 columns of a token.
template <int ACT>
__global__ __launch_bounds__(256)
void gated_skinny_finish_kernel(PlanDev pd, const float* __restrict__ part, const float* __restrict__ H, const uint16_t* __restrict__ B, int32_t f,
                                Cut cut, uint16_t* __restrict__ gu, uint16_t* __restrict__ h)
{
    const int32_t col = (int32_t(blockIdx.x) * 256 + int32_t(threadIdx.x)) * 8, i = blockIdx.y, T = pd.T;
    const int32_t task = H ? token_task(pd, i) : -1;
    if (col >= f) return;
    const size_t ldw = 2 * size_t(f);
    float g[8], u[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) g[e] = u[e] = 0.f;
    // the parts of this column tile: of workgroups w0 .. w1, four at a time
    const int32_t tile = col / COLS, w0 = tile * cut.ks / cut.per, w1 = ((tile + 1) * cut.ks - 1) / cut.per;
    const float* at = part + (size_t(tile) * 2 * T + i) * COLS + col % COLS;
    constexpr int V = 4;
    f32x4 v[V][4];
    auto fetch_parts = [&](int32_t w) __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < V; ++c) {
            const float* p = at + size_t(min(w + c, w1)) * 2 * size_t(T) * COLS;
            const float* q = p + size_t(T) * COLS;
            v[c][0] = *reinterpret_cast<const f32x4*>(p);
            v[c][1] = *reinterpret_cast<const f32x4*>(p + 4);
            v[c][2] = *reinterpret_cast<const f32x4*>(q);
            v[c][3] = *reinterpret_cast<const f32x4*>(q + 4);
        }
    };
    fetch_parts(w0);
    // U ranks' rows of B are on their way at a time (ranks are multiples of U: every stacked rank is one of 8 n_proj)
    constexpr int U = 8;
    const int32_t r0 = task >= 0 ? pd.rank_off[task] : 0, r = task >= 0 ? (pd.rank_off[task + 1] - r0) / 2 : 0;
    const float* hv = H + size_t(i) * pd.r_max;
    const uint16_t* b0 = B + size_t(r0) * f + col;
    rows::u32x4 bg[U], bu[U];
    auto fetch = [&](int32_t k) __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < U; ++c) {
            bg[c] = *reinterpret_cast<const rows::u32x4*>(b0 + size_t(k + c) * f);
            bu[c] = *reinterpret_cast<const rows::u32x4*>(b0 + size_t(r + k + c) * f);
        }
    };
    if (r > 0) fetch(0);
    for (int32_t w = w0; w <= w1; w += V) {
        if (w > w0) fetch_parts(w);
#pragma unroll
        for (int c = 0; c < V; ++c) {
            if (w + c > w1) break;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                g[e] += v[c][0][e];
                g[4 + e] += v[c][1][e];
                u[e] += v[c][2][e];
                u[4 + e] += v[c][3][e];
            }
        }
    }
    for (int32_t k = 0; k < r; k += U) {
        if (k > 0) fetch(k);
#pragma unroll
        for (int c = 0; c < U; ++c) {
            const float hg = hv[k + c], hu = hv[r + k + c];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                g[e] = fmaf(hg, rows::Packet<uint16_t>::element(bg[c], e), g[e]);
                u[e] = fmaf(hu, rows::Packet<uint16_t>::element(bu[c], e), u[e]);
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

Cut make_cut(int32_t K, int32_t f)
{
    Cut c;
    c.tiles = (f + COLS - 1) / COLS;
    c.ks = (K + KT - 1) / KT;
    // a workgroup per compute unit, of four K tiles at least
    const int32_t total = c.tiles * c.ks;
    c.per = (total + 255) / 256;
    c.per = c.per < 4 ? 4 : c.per;
    c.streams = (total + c.per - 1) / c.per;
    return c;
}
size_t part_bytes(const Cut& c, int64_t T) { return size_t(c.streams + c.tiles) * 2 * size_t(T) * COLS * 4; }

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
    gated_skinny_kernel<TB><<<dim3(uint32_t(H ? 256 : c.streams)), 64 * NW, bytes, st>>>(pd, x, W, A, s, part, H, K, f, c);
    return hipGetLastError();
}

size_t align256(size_t v) { return (v + 255) / 256 * 256; }

}  // namespace

size_t gated_skinny_ws_bytes(int64_t T, int32_t K, int32_t f, int32_t r_max)
{
    return align256(part_bytes(make_cut(K, f), T)) + align256(size_t(T) * size_t(r_max) * 4);
}

hipError_t gated_skinny_product(const PlanDev& pd, const void* x, const void* W, const void* A, const float* s, void* ws, bool adapters, hipStream_t st)
{
    const int32_t K = pd.d_in, f = pd.dg;
    const Cut c = make_cut(K, f);
    float* part = static_cast<float*>(ws);
    float* H = adapters ? reinterpret_cast<float*>(static_cast<char*>(ws) + align256(part_bytes(c, pd.T))) : nullptr;
    const uint16_t *xp = static_cast<const uint16_t*>(x), *wp = static_cast<const uint16_t*>(W), *ap = static_cast<const uint16_t*>(A);
    switch ((pd.T + 15) / 16) {
    case 1: return launch<1>(pd, c, xp, wp, ap, s, part, H, K, f, st);
    case 2: return launch<2>(pd, c, xp, wp, ap, s, part, H, K, f, st);
    case 3: return launch<3>(pd, c, xp, wp, ap, s, part, H, K, f, st);
    case 4: return launch<4>(pd, c, xp, wp, ap, s, part, H, K, f, st);
    case 5:
    case 6: return launch<6>(pd, c, xp, wp, ap, s, part, H, K, f, st);
    default: return launch<8>(pd, c, xp, wp, ap, s, part, H, K, f, st);
    }
}

hipError_t gated_skinny_finish(const PlanDev& pd, int act, const void* B, const void* ws, bool adapters, void* gu, void* h, hipStream_t st)
{
    const int32_t f = pd.dg;
    const Cut c = make_cut(pd.d_in, f);
    const float* part = static_cast<const float*>(ws);
    const float* H = adapters ? reinterpret_cast<const float*>(static_cast<const char*>(ws) + align256(part_bytes(c, pd.T))) : nullptr;
    const dim3 grid(uint32_t((f / 8 + 255) / 256), uint32_t(pd.T));
    const uint16_t* b = static_cast<const uint16_t*>(B);
    uint16_t *g = static_cast<uint16_t*>(gu), *o = static_cast<uint16_t*>(h);
    if (act == LOBRA_ACT_SILU) gated_skinny_finish_kernel<LOBRA_ACT_SILU><<<grid, 256, 0, st>>>(pd, part, H, b, f, c, g, o);
    else gated_skinny_finish_kernel<LOBRA_ACT_GELU_TANH><<<grid, 256, 0, st>>>(pd, part, H, b, f, c, g, o);
    return hipGetLastError();
}

}  // namespace lobra
