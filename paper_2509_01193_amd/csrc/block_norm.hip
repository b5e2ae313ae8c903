// Norms after one residual block and before the next, with the block's gate and residual scale, in one pass.
//     n = 1 / rms(b)   r' = r + alpha gate_t w_post b n   m = 1 / rms(r')   x = w_pre r' m
// Backward, with bh = b n, rh = r' m, u = w_pre dx, q = alpha gate_t w_post:
//     g = dr' + m (u - rh mean(u rh))            -> dr
//     db = n (q g - bh mean(q g bh))             (no post norm: db = alpha gate_t g)
//     dgate_t = alpha w_post sum_t g bh   dw_post = alpha sum gate_t g bh   dw_pre = sum dx rh
// The two means of backward are one reduction: with s1 = sum u rh, s2 = sum q bh (dr' + m u), s3 = sum q bh rh, mean(u rh) = s1 / d and
// mean(q g bh) = (s2 - m s1 / d s3) / d.
// Forward, a row lives in the registers of a team of threads - a wave, or a workgroup of up to 1024 - from its read to its write.  Backward's teams
// take neighbouring rows and keep the sums over tokens from row to row; they write them out where their rows end, the gate's also where a
// segment ends (slot: team + segment, which no two runs share; the slots' tasks stand beside them), and a second launch adds them in order.
// A row, the next one, gains, gate and sums are more than the 128 registers that 16 waves a compute unit leave to each; what does not fit is in
// scratch memory, bytes a lane with sums: bf16 32 - 36 at one packet a lane (teams of up to 512), 356 at two (d > 8192); fp32 104 - 116 at two (d >
// 4096), 604 - 616 at four (d > 8192; without sums 136 - 176).  (The first were not timed apart; the widest are what bounds the pass.)
// Bound: memory, 4 T d elements forward and 6 T d backward.  Measured, us: 16384 x 4096 bf16 forward 102 .. 114 (of 537 MB, 5.0 TB/s), backward
// 161 .. 178 (805 MB, 4.7 TB/s) and its sums' launch 7; 2999 x 1025 fp32, out of the caches, 15, 22 and 5; 40 x 4096 forward 4.  Widths between those
// of whole teams leave lanes idle: bf16 forward, TB/s, 2560 3.9, 4096 4.7, 5120 4.1, 6144 4.3, 8192 4.9; backward with sums 3.8, 4.5, 4.6, 4.6, 4.7.
// Scratch memory, backward with / without sums: bf16 4096 x 12288 574 / 125, 4096 x 16384 618 / 153; fp32 4096 x 8192 191 / 149, 2048 x 16384 571 / 245.
#include <algorithm>

#include "kernels.h"
#include "row_common.h"

namespace lobra {

using namespace rows;

namespace {

typedef u32x4 AnyPacket __attribute__((aligned(4)));       // (global memory is read and written in 16 bytes from any multiple of 4)

// A 16-byte packet of a row of d elements, of which `left` are left from the packet's first one on.  RAGGED: rows whose width is no multiple of a
// packet (fp32): packets begin at any element, and the row's last one is read and written element by element.
template <typename E, bool RAGGED> struct Piece {
    static constexpr int N = Packet<E>::N;
    template <bool ONCE> static __device__ __forceinline__ u32x4 fetch_row(const E* p, int32_t left)
    {
        if (RAGGED && left < N) {
            u32x4 q = zero();
#pragma unroll
            for (int e = 0; e < N - 1; ++e)
                if (e < left) q[e] = __float_as_uint(Elem<E>::load(p, size_t(e)));
            return q;
        }
        if constexpr (RAGGED) return ONCE ? __builtin_nontemporal_load(reinterpret_cast<const AnyPacket*>(p)) : *reinterpret_cast<const AnyPacket*>(p);
        else return ONCE ? __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p)) : *reinterpret_cast<const u32x4*>(p);
    }
    static __device__ __forceinline__ u32x4 fetch(const E* p, int32_t left) { return fetch_row<false>(p, left); }
    static __device__ __forceinline__ void widen(u32x4 r, float (&v)[N]) { Packet<E>::widen(r, v); }
    static __device__ __forceinline__ float widen(u32x4 r, int i) { return Packet<E>::element(r, i); }
    static __device__ __forceinline__ u32x4 zero() { return u32x4{0u, 0u, 0u, 0u}; }
    static __device__ __forceinline__ void load(const E* p, float (&v)[N], int32_t left) { widen(fetch(p, left), v); }
    template <bool ONCE> static __device__ __forceinline__ void store_row(E* p, const float (&v)[N], int32_t left)
    {
        if (RAGGED && left < N) {
#pragma unroll
            for (int e = 0; e < N - 1; ++e)
                if (e < left) Elem<E>::store(p, size_t(e), v[e]);
            return;
        }
        const u32x4 q = Packet<E>::narrow(v);
        if constexpr (RAGGED) {
            if (ONCE) __builtin_nontemporal_store(q, reinterpret_cast<AnyPacket*>(p));
            else *reinterpret_cast<AnyPacket*>(p) = q;
        } else {
            if (ONCE) __builtin_nontemporal_store(q, reinterpret_cast<u32x4*>(p));
            else *reinterpret_cast<u32x4*>(p) = q;
        }
    }
    static __device__ __forceinline__ void store(E* p, const float (&v)[N], int32_t left) { store_row<false>(p, v, left); }
};
// v as the element type holds it
template <typename E> __device__ __forceinline__ float rounded(float v);
template <> __device__ __forceinline__ float rounded<float>(float v) { return v; }
template <> __device__ __forceinline__ float rounded<uint16_t>(float v) { return float((__bf16)v); }

// Sums over a team of NT threads (64: a wave).  lds: one array of K NT / 64 floats per call site and parity of the row.
template <int NT, int K> __device__ __forceinline__ void team_sum(float (&v)[K], float* lds)
{
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = wave_sum(v[k]);
    if constexpr (NT > 64) {
        const int w = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < K; ++k) lds[w * K + k] = v[k];
        __syncthreads();
        const int o = threadIdx.x & 15;               // (up to 16 waves: a wave's sum per lane of a row of 16)
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = row_sum(o < NT / 64 ? lds[o * K + k] : 0.f);
    }
}

template <typename E> struct NormArgs {
    const E *r, *b, *w_post, *gate, *w_pre;
    E *r_out, *x;
    float *rstd_post, *rstd_pre;
    int32_t d;
    float eps, alpha;
    bool post;
};

// I packets of N elements per thread hold a row of up to NT I N; BT / NT teams per workgroup, a row each, from row0 on.
template <typename E, bool RAGGED, int NT, int I>
__global__ __launch_bounds__(NT < 256 ? 256 : NT)
void block_norm_fwd_kernel(PlanDev pd, NormArgs<E> a, int32_t row0)
{
    typedef Piece<E, RAGGED> P;
    constexpr int BT = NT < 256 ? 256 : NT, N = P::N;
    __shared__ float lds[2][NT / 64];
    const int64_t at = row0 + int64_t(xcd_contiguous(int32_t(blockIdx.x), int32_t(gridDim.x))) * (BT / NT) + int32_t(threadIdx.x) / NT;
    if (at >= pd.T) return;                           // (whole waves; with NT > 64 a workgroup has one row)
    const int32_t row = int32_t(at), t = threadIdx.x % NT;
    const size_t base = size_t(row) * a.d;
    float v[I][N], bv[I][N];
    float sums[1];
#pragma unroll
    for (int i = 0; i < I; ++i) {
        const int32_t c = (t + i * NT) * N;
        if (c < a.d) {
            P::load(a.r + base + c, v[i], a.d - c);
            if (a.b) P::load(a.b + base + c, bv[i], a.d - c);
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) v[i][e] = bv[i][e] = 0.f;
        }
    }
    if (a.b) {
        float n = 1.f;
        if (a.post) {
            sums[0] = 0.f;
#pragma unroll
            for (int i = 0; i < I; ++i)
#pragma unroll
                for (int e = 0; e < N; ++e) sums[0] = fmaf(bv[i][e], bv[i][e], sums[0]);
            team_sum<NT, 1>(sums, lds[0]);
            n = 1.f / sqrtf(sums[0] / float(a.d) + a.eps);
            if (t == 0 && a.rstd_post) a.rstd_post[row] = n;
        }
        const int32_t task = a.gate ? wave_segment(pd, row).task : -1;
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int32_t c = (t + i * NT) * N;
            if (c >= a.d) continue;
            float k[N];
#pragma unroll
            for (int e = 0; e < N; ++e) k[e] = a.alpha;
            if (a.post) {
                float w[N];
                P::load(a.w_post + c, w, a.d - c);
#pragma unroll
                for (int e = 0; e < N; ++e) k[e] *= w[e] * n;
            }
            if (task >= 0) {
                float w[N];
                P::load(a.gate + size_t(task) * a.d + c, w, a.d - c);
#pragma unroll
                for (int e = 0; e < N; ++e) k[e] *= w[e];
            }
#pragma unroll
            for (int e = 0; e < N; ++e) v[i][e] = rounded<E>(fmaf(k[e], bv[i][e], v[i][e]));
            P::store(a.r_out + base + c, v[i], a.d - c);
        }
    }
    if (!a.w_pre) return;
    sums[0] = 0.f;
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
        for (int e = 0; e < N; ++e) sums[0] = fmaf(v[i][e], v[i][e], sums[0]);
    team_sum<NT, 1>(sums, lds[1]);
    const float m = 1.f / sqrtf(sums[0] / float(a.d) + a.eps);
    if (t == 0 && a.rstd_pre) a.rstd_pre[row] = m;
#pragma unroll
    for (int i = 0; i < I; ++i) {
        const int32_t c = (t + i * NT) * N;
        if (c >= a.d) continue;
        float w[N];
        P::load(a.w_pre + c, w, a.d - c);
#pragma unroll
        for (int e = 0; e < N; ++e) w[e] = w[e] * (v[i][e] * m);
        P::store(a.x + base + c, w, a.d - c);
    }
}

template <typename E> struct NormGradArgs {
    const E *r_out, *b, *w_post, *gate, *w_pre, *dr_out, *dx;
    const float *rstd_post, *rstd_pre;
    E *dr, *db;
    float *part_gate, *part_post, *part_pre;          // [teams + nseg][d], [teams][d], [teams][d], or NULL
    int32_t* slot_task;                               // [teams + nseg]: whose a slot of part_gate is
    int32_t d, rows;                                  // rows: of a team
    float alpha;
    bool post;
};

// A team's rows one after the other.  SUMS: the sums over tokens are wanted.  sum_run = sum g bh of a run of rows of one segment (without
// gates: of all rows): at its end it goes to the gate's partial sums and, times alpha gate_t, into sum_post.
// ONCE: the rows are more than the caches hold and are read and written past them.
template <typename E, bool RAGGED, int NT, int I, bool SUMS, bool ONCE>
__global__ __launch_bounds__(NT < 256 ? 256 : NT, I == 1 ? 4 : 1)
void block_norm_bwd_kernel(PlanDev pd, NormGradArgs<E> a)
{
    typedef Piece<E, RAGGED> P;
    constexpr int BT = NT < 256 ? 256 : NT, N = P::N;
    __shared__ float lds[2][3 * (NT / 64)];
    const int32_t team = xcd_contiguous(int32_t(blockIdx.x), int32_t(gridDim.x)) * (BT / NT) + int32_t(threadIdx.x) / NT, t = threadIdx.x % NT;
    const int64_t first = int64_t(team) * a.rows;
    if (first >= pd.T) return;                        // (whole waves, or the whole workgroup)
    const int32_t row0 = int32_t(first), row1 = int32_t(first + a.rows < pd.T ? first + a.rows : pd.T);
    constexpr int IS = SUMS ? I : 1;
    float sum_run[IS][N], sum_post[IS][N], sum_pre[IS][N];
#pragma unroll
    for (int i = 0; i < IS; ++i)
#pragma unroll
        for (int e = 0; e < N; ++e) sum_run[i][e] = sum_post[i][e] = sum_pre[i][e] = 0.f;
    const bool gated = a.gate != nullptr;             // the rows' tasks matter
    const Segment own = gated ? wave_segment(pd, row0) : Segment{0, -1};
    int32_t seg = own.seg, task = own.task, seg_end = gated ? pd.cseg_off[seg + 1] : row1;
    // (a segment that begins with a team's first row leaves a slot between its run and the one before)
    if (SUMS && a.part_gate && t == 0 && team > 0 && pd.cseg_off[seg] == row0) a.slot_task[team + seg - 1] = -1;
    // gains and the task's gate stay in registers as they are in memory, and a row is fetched while the one before is worked on
    u32x4 w_post[I], w_pre[I], w_gate[I];
    auto end_run = [&]() {
        if constexpr (SUMS) {
            if (a.part_gate && t == 0) a.slot_task[team + seg] = task;
#pragma unroll
            for (int i = 0; i < I; ++i) {
                const int32_t c = (t + i * NT) * N;
                if (c >= a.d) continue;
                float k[N];
                P::widen(w_gate[i], k);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    if (RAGGED && c + e >= a.d) break;
                    if (task < 0) k[e] = 1.f;
                    if (a.part_gate) a.part_gate[(size_t(team) + seg) * a.d + c + e] = sum_run[i][e];
                    sum_post[i][e] = fmaf(a.alpha * k[e], sum_run[i][e], sum_post[i][e]);
                    sum_run[i][e] = 0.f;
                }
            }
        }
    };
    struct Row {
        u32x4 dx[I], r[I], dr[I], b[I];
        float n, m;
    };
    auto fetch_gate = [&]() {
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int32_t c = (t + i * NT) * N;
            w_gate[i] = c < a.d && task >= 0 ? P::fetch(a.gate + size_t(task) * a.d + c, a.d - c) : P::zero();
        }
    };
    auto fetch_row = [&](Row& f, int32_t row) {
        const size_t base = size_t(row) * a.d;
        f.n = a.post ? a.rstd_post[row] : 1.f;
        f.m = a.dx ? a.rstd_pre[row] : 0.f;
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int32_t c = (t + i * NT) * N;
            const bool in = c < a.d;
            f.dx[i] = in && a.dx ? P::template fetch_row<ONCE>(a.dx + base + c, a.d - c) : P::zero();
            f.r[i] = in && a.dx ? P::template fetch_row<ONCE>(a.r_out + base + c, a.d - c) : P::zero();
            f.dr[i] = in && a.dr_out ? P::template fetch_row<ONCE>(a.dr_out + base + c, a.d - c) : P::zero();
            f.b[i] = in && a.b ? P::template fetch_row<ONCE>(a.b + base + c, a.d - c) : P::zero();
        }
    };
#pragma unroll
    for (int i = 0; i < I; ++i) {
        const int32_t c = (t + i * NT) * N;
        w_post[i] = c < a.d && a.post ? P::fetch(a.w_post + c, a.d - c) : P::zero();
        w_pre[i] = c < a.d && a.dx ? P::fetch(a.w_pre + c, a.d - c) : P::zero();
    }
    fetch_gate();
    // an element's terms, from how they are in memory: g without the term of its mean
    struct Terms {
        float dx, rh, bh, q, u, g;
    };
    auto expand = [&](const Row& f, int i, int e) __attribute__((always_inline)) {
        Terms k;
        k.dx = P::widen(f.dx[i], e);
        k.rh = f.m * P::widen(f.r[i], e);
        k.bh = f.n * P::widen(f.b[i], e);
        k.u = P::widen(w_pre[i], e) * k.dx;
        k.g = fmaf(f.m, k.u, P::widen(f.dr[i], e));
        k.q = a.alpha;
        if (a.post) k.q *= P::widen(w_post[i], e);
        if (task >= 0) k.q *= P::widen(w_gate[i], e);
        return k;
    };
    constexpr bool AHEAD = I == 1;       // (the next row does not fit next to larger ones)
    Row cur, next;
    fetch_row(cur, row0);
    const float inv_d = 1.f / float(a.d);
    for (int32_t row = row0; row < row1; ++row) {
        if (row >= seg_end) {                         // (no segment is empty)
            end_run();
            ++seg;
            seg_end = pd.cseg_off[seg + 1];
            task = pd.cseg_task[seg];
            fetch_gate();
        }
        if (AHEAD && row + 1 < row1) fetch_row(next, row + 1);
        float sums[3] = {0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < I; ++i) {
            asm volatile("" : "+v"(w_post[i]), "+v"(w_pre[i]), "+v"(w_gate[i]));        // (they are not widened in front of the loop)
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const Terms k = expand(cur, i, e);
                const float qb = k.q * k.bh;
                sums[0] = fmaf(k.u, k.rh, sums[0]);
                sums[1] = fmaf(qb, k.g, sums[1]);
                sums[2] = fmaf(qb, k.rh, sums[2]);
            }
        }
        team_sum<NT, 3>(sums, lds[row & 1]);
        const float mean = sums[0] * inv_d, c1 = cur.m * mean, c2 = (sums[1] - c1 * sums[2]) * inv_d;
        const size_t base = size_t(row) * a.d;
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int32_t c = (t + i * NT) * N;
            // (opaque to the optimiser: the terms are worked out once more instead of waiting in 48 registers for the sums, which would
            //  halve the waves of a compute unit)
            asm volatile("" : "+v"(cur.dx[i]), "+v"(cur.r[i]), "+v"(cur.dr[i]), "+v"(cur.b[i]), "+v"(w_post[i]), "+v"(w_pre[i]), "+v"(w_gate[i]));
            float g[N], out[N];
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const Terms k = expand(cur, i, e);
                g[e] = fmaf(-c1, k.rh, k.g);
                if constexpr (SUMS) {
                    sum_run[i][e] = fmaf(g[e], k.bh, sum_run[i][e]);
                    sum_pre[i][e] = fmaf(k.dx, k.rh, sum_pre[i][e]);
                }
                out[e] = k.q * g[e];
                if (a.post) out[e] = cur.n * fmaf(-k.bh, c2, out[e]);
            }
            if (c < a.d) {
                P::template store_row<ONCE>(a.dr + base + c, g, a.d - c);
                if (a.b) P::template store_row<ONCE>(a.db + base + c, out, a.d - c);
            }
        }
        if (AHEAD) cur = next;
        else if (row + 1 < row1) fetch_row(cur, row + 1);
    }
    if constexpr (SUMS) {
        end_run();
#pragma unroll
        for (int i = 0; i < I; ++i) {
            const int32_t c = (t + i * NT) * N;
            if (c >= a.d) continue;
#pragma unroll
            for (int e = 0; e < N; ++e) {
                if (RAGGED && c + e >= a.d) break;
                if (a.part_post) a.part_post[size_t(team) * a.d + c + e] = sum_post[i][e];
                if (a.part_pre) a.part_pre[size_t(team) * a.d + c + e] = sum_pre[i][e];
            }
        }
    }
}

// Adds the partial sums up, in order: first + y = 0 and 1: the gains', over the teams; first + y = 2 + t: task t's gate's, over its slots,
// which are gathered 1024 slots at a time.  COLS columns by 1024 / COLS lanes.
template <typename E, int COLS>
__global__ __launch_bounds__(1024)
void block_norm_sum_kernel(const float* __restrict__ part_gate, const float* __restrict__ part_post, const float* __restrict__ part_pre,
                           const int32_t* __restrict__ slot_task, int32_t d, int32_t teams, int32_t slots, float alpha, const E* __restrict__ w_post,
                           float* __restrict__ dgate, float* __restrict__ dw_post, float* __restrict__ dw_pre, int accumulate, int32_t first)
{
    constexpr int LANES = 1024 / COLS;
    __shared__ float lds[16][COLS];
    __shared__ int32_t own[1024];                     // the task's slots among 1024
    __shared__ int32_t found[16];
    const int32_t tid = threadIdx.x, wave = tid >> 6;
    const int32_t col = int32_t(blockIdx.x) * COLS + tid % COLS, lane = tid / COLS;
    const int32_t what = first + int32_t(blockIdx.y);
    float* out = what == 0 ? dw_post : what == 1 ? dw_pre : dgate;
    if (!out) return;                                 // (uniform)
    float s = 0.f;
    bool any = true;
    if (what < 2) {
        const float* p = what == 0 ? part_post : part_pre;
        if (col < d)
#pragma unroll 8
            for (int32_t k = lane; k < teams; k += LANES) s += p[size_t(k) * d + col];
    } else {
        any = false;
        for (int32_t base = 0; base < slots; base += 1024) {
            const bool mine = base + tid < slots && slot_task[base + tid] == what - 2;
            const uint64_t mask = __ballot(mine);
            if ((tid & 63) == 0) found[wave] = __popcll(mask);
            __syncthreads();
            int32_t at = 0, n = 0;
#pragma unroll
            for (int w = 0; w < 16; ++w) {
                at += w < wave ? found[w] : 0;
                n += found[w];
            }
            if (mine) own[at + __popcll(mask & ((uint64_t(1) << (tid & 63)) - 1))] = base + tid;
            __syncthreads();
            any = any || n > 0;
            if (col < d)
#pragma unroll 8
                for (int32_t q = lane; q < n; q += LANES) s += part_gate[size_t(own[q]) * d + col];
            __syncthreads();
        }
        out += size_t(what - 2) * d;
    }
#pragma unroll
    for (int m = COLS; m < 64; m <<= 1) s += __shfl_xor(s, m);
    if ((tid & 63) < COLS) lds[wave][tid % COLS] = s;
    __syncthreads();
    if (tid >= COLS || col >= d) return;
    s = 0.f;
#pragma unroll
    for (int w = 0; w < 16; ++w) s += lds[w][tid];
    if (what >= 2) s *= w_post ? alpha * Elem<E>::load(w_post, size_t(col)) : alpha;
    if (accumulate) {
        if (any) out[col] += s;
    } else {
        out[col] = s;
    }
}

// How rows are dealt to threads: a wave holds a row of up to two packets a lane; wider ones take workgroups.
struct Deal {
    int32_t nt, i;           // threads of a team, packets per thread
    bool ragged;
};
Deal deal(int dtype, int32_t d)
{
    const int32_t per = dtype == LOBRA_F32 ? 4 : 8, packets = (d + per - 1) / per;
    const bool ragged = d % per != 0;                // (bf16 widths are multiples of 8)
    if (packets <= 64) return {64, 1, ragged};
    if (packets <= 128) return {64, 2, ragged};
    if (packets <= 256) return {256, 1, ragged};
    if (packets <= 512) return {512, 1, ragged};
    if (packets <= 1024) return {1024, 1, ragged};
    if (packets <= 2048) return {1024, 2, ragged};
    return {1024, 4, ragged};
}

// Columns of a workgroup of the sum: a line's 64, or 16 of narrow rows, which would make too few workgroups of 64 (us of both launches, 64 /
// 16: 12527 x 128 27 / 25, 9181 x 64 25 / 22, 8000 x 1024 37 / 37, 261 x 1920 22 / 25, 4000 x 4096 58 / 65).
constexpr int32_t kNarrow = 1024;

// Rows of a team of the backward kernel: what makes some 16 waves per compute unit.  With sums over tokens, which a team writes once (T /
// rows fp32 rows per sum next to T rows of six bf16 ones) and the second launch reads, at least eight where that leaves 256 teams, fewer
// where it does not: a team's rows are a chain (us with at least 8 / 4 / 2 / 1: 261 x 1920 22 / 17 / 15 / 16, 1000 x 4096 35 / 31 / 37 /
// 37, 2000 x 4096 40 / 45 / 45 / 45; without sums 13 / 8 / 5 / 4, 19 / 14 / 12 / 12, 23 / 21 / 21 / 21).
int32_t team_rows(const Deal& dl, int64_t T, bool sums)
{
    const int64_t teams = 4096 / (dl.nt / 64), rows = (T + teams - 1) / teams;
    const int64_t least = sums ? std::min<int64_t>(8, (T + 255) / 256) : 1;
    return int32_t(std::max<int64_t>(std::max<int64_t>(rows, least), 1));
}

template <typename E, bool RAGGED, int NT, int I> struct Launch {
    static void fwd(const PlanDev& pd, const NormArgs<E>& a, hipStream_t st)
    {
        constexpr int BT = NT < 256 ? 256 : NT;
        constexpr int64_t most = int64_t(1) << 21;    // rows of a launch, which holds less than 2^32 threads
        for (int64_t row0 = 0; row0 < pd.T; row0 += most) {
            const int64_t rows = pd.T - row0 < most ? pd.T - row0 : most;
            block_norm_fwd_kernel<E, RAGGED, NT, I><<<dim3(uint32_t((rows + BT / NT - 1) / (BT / NT))), BT, 0, st>>>(pd, a, int32_t(row0));
        }
    }
    static void bwd(const PlanDev& pd, const NormGradArgs<E>& a, bool sums, int32_t teams, hipStream_t st)
    {
        constexpr int BT = NT < 256 ? 256 : NT;
        const dim3 grid(uint32_t((teams + BT / NT - 1) / (BT / NT)));
        // six tensors beyond the 256 MB infinity cache (us, plain / past the caches: 16384 x 4096 bf16, 805 MB, with the forward pass in
        // front of it 313 / 275; 2999 x 1025 fp32, 74 MB, 26 / 33)
        const bool once = size_t(pd.T) * size_t(a.d) * sizeof(E) * 6 > (size_t(256) << 20);
        if (sums) {
            if (once) block_norm_bwd_kernel<E, RAGGED, NT, I, true, true><<<grid, BT, 0, st>>>(pd, a);
            else block_norm_bwd_kernel<E, RAGGED, NT, I, true, false><<<grid, BT, 0, st>>>(pd, a);
        } else {
            if (once) block_norm_bwd_kernel<E, RAGGED, NT, I, false, true><<<grid, BT, 0, st>>>(pd, a);
            else block_norm_bwd_kernel<E, RAGGED, NT, I, false, false><<<grid, BT, 0, st>>>(pd, a);
        }
    }
};

// f(Launch<...>) of the deal
template <typename E, bool RAGGED, typename F> void with_team(const Deal& dl, F&& f)
{
    if (dl.nt == 64) {
        if (dl.i == 1) f(Launch<E, RAGGED, 64, 1>{});
        else f(Launch<E, RAGGED, 64, 2>{});
    } else if (dl.nt == 256) f(Launch<E, RAGGED, 256, 1>{});
    else if (dl.nt == 512) f(Launch<E, RAGGED, 512, 1>{});
    else if (dl.i == 1) f(Launch<E, RAGGED, 1024, 1>{});
    else if (dl.i == 2) f(Launch<E, RAGGED, 1024, 2>{});
    else if constexpr (Packet<E>::N == 4) f(Launch<E, RAGGED, 1024, 4>{});
}
template <typename E, typename F> void with_deal(const Deal& dl, F&& f)
{
    if constexpr (Packet<E>::N == 4) {
        if (dl.ragged) return with_team<E, true>(dl, f);
    }
    with_team<E, false>(dl, f);
}

template <typename E>
hipError_t fwd(const PlanDev& pd, int dtype, const BlockNorm& bn, const void* r, const void* b, void* r_out, void* x, float* rstd_post,
               float* rstd_pre, hipStream_t st)
{
    NormArgs<E> a;
    a.r = static_cast<const E*>(r);
    a.b = bn.block ? static_cast<const E*>(b) : nullptr;
    a.w_post = static_cast<const E*>(bn.w_post);
    a.gate = bn.block ? static_cast<const E*>(bn.gate) : nullptr;
    a.w_pre = static_cast<const E*>(bn.w_pre);
    a.r_out = static_cast<E*>(r_out);
    a.x = static_cast<E*>(x);
    a.rstd_post = rstd_post;
    a.rstd_pre = rstd_pre;
    a.d = pd.d_in;
    a.eps = bn.eps;
    a.alpha = bn.alpha;
    a.post = bn.post;
    with_deal<E>(deal(dtype, pd.d_in), [&](auto l) { l.fwd(pd, a, st); });
    return hipGetLastError();
}

template <typename E>
hipError_t bwd(const PlanDev& pd, int dtype, const BlockNorm& bn, const void* r_out, const void* b, const float* rstd_post, const float* rstd_pre,
               const void* dr_out, const void* dx, void* dr, void* db, float* dgate, float* dw_post, float* dw_pre, bool accumulate, float* part,
               hipStream_t st)
{
    const Deal dl = deal(dtype, pd.d_in);
    const bool sums = dgate || dw_post || dw_pre;
    const int32_t rows = team_rows(dl, pd.T, sums), teams = int32_t((int64_t(pd.T) + rows - 1) / rows);
    NormGradArgs<E> a;
    a.r_out = static_cast<const E*>(r_out);
    a.b = bn.block ? static_cast<const E*>(b) : nullptr;
    a.w_post = static_cast<const E*>(bn.w_post);
    a.gate = bn.block ? static_cast<const E*>(bn.gate) : nullptr;
    a.w_pre = static_cast<const E*>(bn.w_pre);
    a.dr_out = static_cast<const E*>(dr_out);
    a.dx = static_cast<const E*>(dx);
    a.rstd_post = rstd_post;
    a.rstd_pre = rstd_pre;
    a.dr = static_cast<E*>(dr);
    a.db = static_cast<E*>(db);
    const size_t row = size_t(pd.d_in);
    a.part_gate = dgate ? part : nullptr;
    a.part_post = dw_post ? part + size_t(teams + pd.nseg) * row : nullptr;
    a.part_pre = dw_pre ? part + size_t(2 * size_t(teams) + pd.nseg) * row : nullptr;
    a.slot_task = reinterpret_cast<int32_t*>(part + (size_t(3) * size_t(teams) + size_t(pd.nseg)) * row);
    a.d = pd.d_in;
    a.rows = rows;
    a.alpha = bn.alpha;
    a.post = bn.post;
    if (pd.T > 0) with_deal<E>(dl, [&](auto l) { l.bwd(pd, a, sums, teams, st); });
    const int32_t outs = !sums ? 0 : dgate ? 2 + pd.n_tasks : 2, most = 1 << 15;         // (a grid's y is below 2^16)
    const bool narrow = pd.d_in <= kNarrow;
    const int32_t cols = narrow ? 16 : 64;
    for (int32_t first = 0; first < outs; first += most)
        (narrow ? block_norm_sum_kernel<E, 16> : block_norm_sum_kernel<E, 64>)
            <<<dim3(uint32_t((pd.d_in + cols - 1) / cols), uint32_t(outs - first < most ? outs - first : most)), 1024, 0, st>>>(
                a.part_gate, a.part_post, a.part_pre, a.slot_task, pd.d_in, teams, teams + pd.nseg - 1, bn.alpha, bn.post ? a.w_post : nullptr,
                dgate, dw_post, dw_pre, accumulate ? 1 : 0, first);
    return hipGetLastError();
}

}  // namespace

size_t block_norm_part_bytes(int64_t T, int32_t d, int32_t nseg, int dtype)
{
    const int64_t rows = team_rows(deal(dtype, d), T, true), teams = (T + rows - 1) / rows;
    return (size_t(3 * teams) + size_t(nseg)) * size_t(d) * sizeof(float) + size_t(teams + nseg) * sizeof(int32_t);
}

hipError_t block_norm_fwd(const PlanDev& pd, int dtype, const BlockNorm& bn, const void* r, const void* b, void* r_out, void* x,
                          float* rstd_post, float* rstd_pre, hipStream_t st)
{
    return dtype == LOBRA_F32 ? fwd<float>(pd, dtype, bn, r, b, r_out, x, rstd_post, rstd_pre, st)
                              : fwd<uint16_t>(pd, dtype, bn, r, b, r_out, x, rstd_post, rstd_pre, st);
}

hipError_t block_norm_bwd(const PlanDev& pd, int dtype, const BlockNorm& bn, const void* r_out, const void* b, const float* rstd_post,
                          const float* rstd_pre, const void* dr_out, const void* dx, void* dr, void* db, float* dgate, float* dw_post,
                          float* dw_pre, bool accumulate, float* part, hipStream_t st)
{
    return dtype == LOBRA_F32
        ? bwd<float>(pd, dtype, bn, r_out, b, rstd_post, rstd_pre, dr_out, dx, dr, db, dgate, dw_post, dw_pre, accumulate, part, st)
        : bwd<uint16_t>(pd, dtype, bn, r_out, b, rstd_post, rstd_pre, dr_out, dx, dr, db, dgate, dw_post, dw_pre, accumulate, part, st);
}

}  // namespace lobra
