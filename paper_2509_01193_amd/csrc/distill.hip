// The loss of rows of logits against the likeliest tokens of a teacher, and its gradient.
//
// With c = 1 / temperature, m the row's largest logit, S = sum exp(c (z - m)): ln p_j = c (z_j - m) - ln S, and
//     loss = sum_j q_j (ln q_j - ln p_j)  over the listed tokens        dz_j = dloss c (p_j sum q - q_j [listed])
// and with a tail, R = the tokens that are not listed, q_r = 1 - sum q, p_r = sum of p over R:
//     loss += q_r (ln q_r - ln p_r)                                     dz_j -= dloss c q_r (p_j / p_r) [j in R],  sum q + q_r for sum q
// Forward reads a row once, keeping sums as the log probabilities do (row_logits.h).  With a tail what is listed stays out of the sums and joins
// them at the end: p_r as a difference would lose all its digits where the student is sure of the list.  A table of bits in LDS says which
// elements are listed, a byte (bf16) to a packet.  The list itself, up to 128 tokens, is a thread's business each, in fp64: it costs a row next to nothing.
// Backward writes every element as if it were not listed, and then the listed ones.
// Bound: memory.  Forward / backward, us: 8190 x 32000 bf16, 20 listed, 119 / 156 (backward leaves the rows without a teacher unread), 4096 x 128000 with a tail and 64 listed
// 193 / 415 (5.4 and 5.0 TB/s), 1000 x 50257 fp32 with a tail 54 / 72; 48 x 32000 6.0 / 4.7, where a row is three rounds to memory and the list in fp64.
#include "kernels.h"
#include "row_common.h"
#include "row_logits.h"

namespace lobra {

using namespace rows;

namespace {

constexpr int kMost = LOBRA_MAX_TEACHER;
constexpr int kTableBits = 1 << 18;                  // 32 KiB; longer rows fold onto it
constexpr double kNoTail = 0x1p-20;                  // 1 - sum q below this is the rounding of the log probabilities

__device__ __forceinline__ double wave_sum64(double v)
{
#pragma unroll
    for (int x = 32; x > 0; x >>= 1) v += __shfl_xor(v, x);
    return v;
}

// (bare: loads in flight stay there)
__device__ __forceinline__ void lds_barrier()
{
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// A place of the row's list: a thread's own, read behind the first loads of the row.
template <typename E> struct Place {
    const E* row;
    const int32_t* ids;
    const float* ls;
    int32_t V, k;
    int32_t id = -1;
    float l = -INFINITY, z = 0.f;
    __device__ __forceinline__ void read()
    {
        const int32_t t = threadIdx.x;
        if (t >= k) return;
        id = ids[t];
        l = ls[t];
        if (l == INFINITY) l = NAN;
        if (uint32_t(id) >= uint32_t(V)) id = -1, l = -INFINITY;
        else z = element(row, id);
    }
};
template <typename E> struct NoneListed {
    Place<E>& mine;
    __device__ __forceinline__ void begin() const { mine.read(); }
    template <int N> __device__ __forceinline__ void operator()(float (&)[N], int32_t, int = 0) const {}
};

// How often a token stands in the list (kMost ids, -1 in empty places), read four ids at a time: nearly always once.  219 x 1408 with 128 places, forward
// and backward, us: place by place 27.8, so 12.5.
__device__ __forceinline__ int32_t times_listed(const int32_t* ids, int32_t k, int32_t id)
{
    int32_t n = 0;
#pragma unroll 4
    for (int32_t i = 0; i < k; i += 4) {
        const int4 v = *reinterpret_cast<const int4*>(ids + i);
        n += int32_t(v.x == id) + int32_t(v.y == id) + int32_t(v.z == id) + int32_t(v.w == id);
    }
    return n;
}

// Elements listed in a row, as bits.  Bit 0 of a packet's is bit 0 of a group of N (the elements in front of the first packet end a group of their own).
template <typename E, int NT> struct ListedBits {
    static constexpr int N = Packet<E>::N;
    Place<E>& mine;
    uint32_t* table;
    int32_t* id;
    int32_t shift, mask, k;
    bool folded;
    __device__ __forceinline__ void begin() const
    {
        const int32_t t = threadIdx.x;
        for (int32_t i = t; i < (mask + 1) / 128; i += NT) reinterpret_cast<u32x4*>(table)[i] = u32x4{0u, 0u, 0u, 0u};
        lds_barrier();
        mine.read();
        if (t < kMost) id[t] = mine.id;
        if (mine.id >= 0) {
            const int32_t bit = (mine.id + shift) & mask;
            atomicOr(&table[bit >> 5], 1u << (bit & 31));
        }
        lds_barrier();
    }
    template <int M> __device__ __forceinline__ void operator()(float (&z)[M], int32_t first, int at = 0) const
    {
        const int32_t bit = (first + shift) & mask;
        constexpr int n = M == 1 ? 1 : N;
        uint32_t hits = table[bit >> 5] >> (bit & 31) & ((1u << n) - 1);
        if (hits == 0) return;
        if (folded) {                                // (perhaps another element's)
            uint32_t sure = 0;
            for (int32_t i = 0; i < k; ++i) {
                const uint32_t d = uint32_t(id[i]) - uint32_t(first);
                if (id[i] >= 0 && d < uint32_t(n)) sure |= 1u << d;
            }
            hits &= sure;
        }
#pragma unroll
        for (int e = 0; e < n; ++e) z[at + e] = hits >> e & 1 ? -INFINITY : z[at + e];
    }
};

template <typename E, int NT, bool TAIL>
__global__ __launch_bounds__(NT)
void distill_fwd_kernel(const E* __restrict__ logits, int64_t ld, int32_t V, int32_t k, float temperature, const float* __restrict__ teacher_logp,
                        const int32_t* __restrict__ teacher_id, float* __restrict__ loss, float4* __restrict__ stat, int32_t table_bits)
{
    constexpr int W = NT / 64, N = Packet<E>::N;
    static_assert(NT >= kMost, "a thread per place of the list");
    extern __shared__ __attribute__((aligned(16))) uint32_t table[];
    __shared__ Stat part[W];
    __shared__ __attribute__((aligned(16))) int32_t ids[kMost];      // -1: an empty place
    __shared__ double join[3][kMost / 64];
    __shared__ float top[2][kMost / 64];
    __shared__ bool any[kMost / 64];
    const size_t r = size_t(xcd_contiguous(int32_t(blockIdx.x), int32_t(gridDim.x)));
    const E* row = logits + r * size_t(ld);
    const RowShape sh = row_shape(row, V);
    const int32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const float c = 1.f / temperature, scale = c * kLog2e;
    const int32_t shift = sh.head ? N - sh.head : 0;
    Place<E> mine{row, teacher_id + r * size_t(k), teacher_logp + r * size_t(k), V, k};
    Stat a;
    if constexpr (TAIL) a = row_stat<E, NT, false>(row, sh, scale, ListedBits<E, NT>{mine, table, ids, shift, table_bits - 1, k, V + N > table_bits});
    else a = row_stat<E, NT, false>(row, sh, scale, NoneListed<E>{mine});
    const float l = mine.l, zj = mine.z;
    const int32_t id = mine.id;
    rescale<false>(a, wave_max(a.m), scale);
    a.s = wave_sum(a.s);
    if (lane == 0) part[wave] = a;
    // the teacher's own sum, or that of its probabilities; the largest logit of the list
    if (wave < kMost / 64) {
        const float lm = wave_max(l == l ? l : INFINITY), zm = wave_max(id >= 0 ? zj : -INFINITY);
        const bool some = __ballot(id >= 0) != 0;
        if (lane == 0) top[0][wave] = lm, top[1][wave] = zm, any[wave] = some;
    }
    __syncthreads();
    // the list's waves are left (a barrier waits for the surviving waves only)
    const int32_t lists = (k + 63) / 64;
    if (wave >= lists) return;
    float m = part[0].m, s = 0.f;
#pragma unroll
    for (int w = 1; w < W; ++w) m = fmaxf(m, part[w].m);
#pragma unroll
    for (int w = 0; w < W; ++w) {
        Stat b = part[w];
        rescale<false>(b, m, scale);
        s += b.s;
    }
    const double rest_m = double(m), rest_s = double(s), cd = 1. / double(temperature);
    double M = rest_m, S = rest_s, ln_q = double(l);
    const float lm = fmaxf(top[0][0], top[0][1]);
    const bool teacher = (any[0] || any[1]) && (TAIL || lm > -INFINITY);
    double ex = 0., own = 0.;                        // exp(c (z - M)) of a listed token; what the teacher's sum takes
    if (TAIL) {
        const float zm = fmaxf(top[1][0], top[1][1]);
        M = fmax(rest_m, double(zm));
        bool first = id >= 0;
        if (first && times_listed(ids, k, id) > 1)
            for (int32_t i = 0; i < tid; ++i) first = first && ids[i] != id;
        if (first) ex = zj == -INFINITY ? 0. : exp((double(zj) - M) * cd);        // (NaN, also where nothing else is left)
        own = id >= 0 ? exp(ln_q) : 0.;
    } else {
        own = id >= 0 ? exp((ln_q - double(lm)) * cd) : 0.;
    }
    ex = wave_sum64(ex);
    double own_sum = wave_sum64(own);
    if (lists > 1) {                                 // (uniform)
        if (lane == 0) join[0][wave] = ex, join[1][wave] = own_sum;
        __syncthreads();
        ex = join[0][0] + join[0][1];
        own_sum = join[1][0] + join[1][1];
    }
    double q = own, tl = 0., ln_own = 0.;            // tl: the teacher's ln of the sum, in units of l
    if (TAIL) {
        S = (rest_s > 0. ? rest_s * exp((rest_m - M) * cd) : rest_s) + ex;
    } else {
        q = own / own_sum;
        ln_own = log(own_sum);
        tl = double(lm) + ln_own / cd;
        ln_q = (ln_q - double(lm)) * cd - ln_own;
    }
    const double ln_s = log(S);
    // (a probability of 0 adds nothing, NaN everything)
    double term = id >= 0 && !(q == 0.) ? q * (ln_q - ((double(zj) - M) * cd - ln_s)) : 0.;
    double total = wave_sum64(term);
    if (lists > 1) {
        if (lane == 0) join[2][wave] = total;
        __syncthreads();
        total = join[2][0] + join[2][1];
    }
    if (tid != 0) return;
    // What backward starts from, as two numbers each: ln of a sum next to a huge logit is nothing even in 64 bits, so the lower one takes it by itself.
    const double lse = S == 0. ? -INFINITY : M + ln_s / cd;
    float4 v;
    v.x = float(lse);
    v.y = S == 0. ? 0.f : float((M - double(v.x)) + ln_s / cd);
    if (TAIL) {
        double qr = 1. - own_sum;
        if (!(qr > kNoTail)) qr = 0.;
        if (qr > 0. && teacher) {
            const double ln_pr = rest_s == 0. ? -INFINITY : (rest_m - M) * cd + log(rest_s) - ln_s;
            total += qr * (log(qr) - ln_pr);
        }
        // in backward the tail's p_j / p_r q_r is exp(c (z_j - t)); +inf: there is none, and the sum of the list's q in its place
        const double ln_t = (log(rest_s) - log(qr)) / cd, t = qr > 0. && rest_s > 0. ? rest_m + ln_t : INFINITY;
        v.z = float(t);
        v.w = qr > 0. ? (rest_s > 0. ? float((rest_m - double(v.z)) + ln_t) : 1.f) : float(own_sum);
    } else {
        v.z = float(tl);
        v.w = float((double(lm) - double(v.z)) + ln_own / cd);
    }
    if (S == 0.) total = own_sum == own_sum ? INFINITY : NAN;       // (nothing but -inf: whatever the teacher likes has p = 0)
    if (total != total) v.x = NAN;                   // (its gradient is NaN too, and not that of a row of nothing)
    if (!teacher) total = 0., v = make_float4(-INFINITY, 0.f, 0.f, 0.f);
    if (loss) loss[r] = float(total);
    if (stat) stat[r] = v;
}

// Workgroup (row, part): packets part * NT + ... with a stride of all parts.  In place (dlogits = logits) every thread writes what it has
// read itself, and the threads of the list read their logits before that.  A row without any weight is not read.
// The last rows come first: they are what forward has left in the 256 MB infinity cache, and gradients that would fill it anyway (once: logits of
// 128 MB and more) go past the caches.  Forward and backward, us: 8190 x 32000 bf16 290, either alone 288 and 287, both 275; 4096 x 128000 643, 641,
// 614, 604; 1000 x 50257 fp32 145, 145, 127, 127.
template <typename E, int NT, bool TAIL, bool ADD, bool ONCE>
__global__ __launch_bounds__(NT)
void distill_bwd_kernel(const E* logits, int64_t ld, int32_t V, int32_t k, float temperature, const float* __restrict__ teacher_logp,
                        const int32_t* __restrict__ teacher_id, const float4* __restrict__ stat, const float* __restrict__ dloss, E* dlogits)
{
    constexpr int N = Packet<E>::N;
    static_assert(NT >= kMost, "a thread per place of the list");
    __shared__ __attribute__((aligned(16))) int32_t ids[kMost];      // -1: an empty place
    __shared__ float qs[kMost];
    const size_t r = size_t(xcd_contiguous(int32_t(gridDim.x - 1 - blockIdx.x), int32_t(gridDim.x)));
    const E* row = logits + r * size_t(ld);
    E* out = dlogits + r * size_t(ld);
    const RowShape sh = row_shape(row, V);            // (logits and dlogits are aligned alike: both bases to 16 bytes)
    const float4 st = stat[r];
    const float c = 1.f / temperature, scale = c * kLog2e, w = dloss[r] * c;
    const int32_t t = threadIdx.x, stride = NT * int32_t(gridDim.y), first = blockIdx.y * NT + t;
    const u32x4* src = reinterpret_cast<const u32x4*>(row + sh.head);
    u32x4* dst = reinterpret_cast<u32x4*>(out + sh.head);
    if (dloss[r] == 0.f || st.x == -INFINITY) {       // (uniform)
        if (ADD) return;
        for (int32_t i = first; i < sh.packets; i += stride) dst[i] = u32x4{0u, 0u, 0u, 0u};
        if (blockIdx.y == 0 && t < sh.head + sh.tail) Elem<E>::store(out, size_t(t < sh.head ? t : t + sh.packets * N), 0.f);
        return;
    }
    // the tokens of the list that lie in this workgroup's packets: logit and gradient so far, before anything is written
    int32_t id = -1;
    float l = 0.f, zj = 0.f, had = 0.f;
    bool mine = false;
    if (t < k) {
        id = teacher_id[r * size_t(k) + t];
        l = teacher_logp[r * size_t(k) + t];
        if (uint32_t(id) >= uint32_t(V)) id = -1;
        if (id >= 0) {
            const int32_t p = (id - sh.head) / N;
            const bool edge = id < sh.head || p >= sh.packets;
            mine = int32_t(edge ? 0 : p / NT % int32_t(gridDim.y)) == int32_t(blockIdx.y);
            if (mine) {
                zj = element(row, id);
                if (ADD) had = Elem<E>::load(out, size_t(id));
            }
        }
        qs[t] = l == INFINITY ? NAN : TAIL ? float(exp(double(l))) : float(exp((double(l) - double(st.z) - double(st.w)) * double(c)));
    }
    if (t < kMost) ids[t] = id;
    const float rest = -scale * st.y;
    const float sum_q = TAIL ? (st.z == INFINITY ? st.w : 1.f) : st.z == st.z ? 1.f : NAN;        // (a teacher of NaN)
    // the tail as a multiple of p, where that is not near the ends of fp32's range (else an exponential of its own)
    const float ratio_log = TAIL ? ((st.x - st.z) + (st.y - st.w)) * scale : 0.f;
    const bool by_ratio = !TAIL || fabsf(ratio_log) < 60.f || st.z == INFINITY;
    const float keep = TAIL && st.z != INFINITY && by_ratio ? sum_q - exp2_fast(ratio_log) : sum_q;
    const float rest_t = TAIL && !by_ratio ? -scale * st.w : 0.f;
    auto gradient = [&](float z) {
        const float p = exp2_fast(fmaf(z - st.x, scale, rest));
        if (by_ratio) return w * keep * p;           // (uniform)
        return w * (sum_q * p - exp2_fast(fmaf(z - st.z, scale, rest_t)));
    };
    __syncthreads();
    float gj = 0.f;
    if (mine) {
        float q = qs[t];
        if (times_listed(ids, k, id) > 1) {
            q = 0.f;
            for (int32_t i = 0; i < k; ++i) {
                const bool same = ids[i] == id;
                if (same && i < t) mine = false;     // an earlier place writes it
                q += same ? qs[i] : 0.f;
            }
        }
        gj = had + w * (sum_q * exp2_fast(fmaf(zj - st.x, scale, rest)) - q);
    }
    for (int32_t i = first; i < sh.packets; i += stride) {
        float z[N], g[N];
        Packet<E>::widen(src[i], z);
        if (ADD) {
            float o[N];
            Packet<E>::widen(dst[i], o);
#pragma unroll
            for (int e = 0; e < N; ++e) g[e] = o[e] + gradient(z[e]);
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) g[e] = gradient(z[e]);
        }
        if constexpr (ONCE) __builtin_nontemporal_store(Packet<E>::narrow(g), dst + i);
        else dst[i] = Packet<E>::narrow(g);
    }
    if (blockIdx.y == 0 && t < sh.head + sh.tail) {
        const int32_t at = t < sh.head ? t : t + sh.packets * N;
        Elem<E>::store(out, size_t(at), (ADD ? Elem<E>::load(out, size_t(at)) : 0.f) + gradient(element(row, at)));
    }
    __syncthreads();
    if (mine) Elem<E>::store(out, size_t(id), gj);
}

template <typename E, int NT>
void launch_fwd(const DistillShape& s, const E* logits, const float* tl, const int32_t* ti, float* loss, float4* stat, hipStream_t st)
{
    const dim3 grid(uint32_t(s.T));
    if (s.tail) {
        int32_t bits = 1024;
        while (bits < s.V + Packet<E>::N && bits < kTableBits) bits *= 2;
        distill_fwd_kernel<E, NT, true><<<grid, NT, size_t(bits / 8), st>>>(logits, s.ld, s.V, s.top_k, s.temperature, tl, ti, loss, stat, bits);
    } else {
        distill_fwd_kernel<E, NT, false><<<grid, NT, 0, st>>>(logits, s.ld, s.V, s.top_k, s.temperature, tl, ti, loss, stat, 0);
    }
}

template <typename E>
hipError_t fwd(const DistillShape& s, const E* logits, const float* tl, const int32_t* ti, float* loss, float4* stat, hipStream_t st)
{
    const int32_t packets = s.V / Packet<E>::N;
    if (packets <= 512) launch_fwd<E, 128>(s, logits, tl, ti, loss, stat, st);
    else if (packets <= 2048) launch_fwd<E, 256>(s, logits, tl, ti, loss, stat, st);
    else launch_fwd<E, 512>(s, logits, tl, ti, loss, stat, st);
    return hipGetLastError();
}

template <typename E>
hipError_t bwd(const DistillShape& s, const E* logits, const float* tl, const int32_t* ti, const float4* stat, const float* dloss, E* dlogits, bool add,
               hipStream_t st)
{
    constexpr int NT = 256;
    // a workgroup per row where there are enough rows, else several, of at least four packets a thread
    const int64_t most = (int64_t(s.V) / Packet<E>::N + 4 * NT - 1) / (4 * NT), wanted = (2048 + s.T - 1) / s.T;
    const dim3 grid(uint32_t(s.T), uint32_t(wanted < most ? wanted : most > 0 ? most : 1));
    const bool once = s.T * s.V * int64_t(sizeof(E)) >= int64_t(128) << 20;
#define LOBRA_DISTILL(tail, acc) \
    (once ? distill_bwd_kernel<E, NT, tail, acc, true> : distill_bwd_kernel<E, NT, tail, acc, false>)<<<grid, NT, 0, st>>>( \
        logits, s.ld, s.V, s.top_k, s.temperature, tl, ti, stat, dloss, dlogits)
    if (s.tail) {
        if (add) LOBRA_DISTILL(true, true);
        else LOBRA_DISTILL(true, false);
    } else if (add) LOBRA_DISTILL(false, true);
    else LOBRA_DISTILL(false, false);
#undef LOBRA_DISTILL
    return hipGetLastError();
}

// (a launch holds less than 2^32 threads)
constexpr int64_t kRowsPerLaunch = 1 << 22;
template <typename F> hipError_t by_rows(const DistillShape& shape, F&& f)
{
    for (int64_t r = 0; r < shape.T; r += kRowsPerLaunch) {
        DistillShape s = shape;
        s.T = shape.T - r < kRowsPerLaunch ? shape.T - r : kRowsPerLaunch;
        const hipError_t e = f(s, r);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t distill_fwd(const DistillShape& shape, const void* logits, const float* teacher_logp, const int32_t* teacher_id, float* loss, float* stat,
                       hipStream_t st)
{
    return by_rows(shape, [&](const DistillShape& s, int64_t r) {
        const float* tl = teacher_logp + r * s.top_k;
        const int32_t* ti = teacher_id + r * s.top_k;
        float4* v = stat ? reinterpret_cast<float4*>(stat) + r : nullptr;
        float* lo = loss ? loss + r : nullptr;
        return s.dtype == LOBRA_F32 ? fwd(s, static_cast<const float*>(logits) + r * s.ld, tl, ti, lo, v, st)
                                    : fwd(s, static_cast<const uint16_t*>(logits) + r * s.ld, tl, ti, lo, v, st);
    });
}

hipError_t distill_bwd(const DistillShape& shape, const void* logits, const float* teacher_logp, const int32_t* teacher_id, const float* stat,
                       const float* dloss, void* dlogits, bool accumulate, hipStream_t st)
{
    return by_rows(shape, [&](const DistillShape& s, int64_t r) {
        const float* tl = teacher_logp + r * s.top_k;
        const int32_t* ti = teacher_id + r * s.top_k;
        const float4* v = reinterpret_cast<const float4*>(stat) + r;
        const int64_t off = r * s.ld;
        return s.dtype == LOBRA_F32
                   ? bwd(s, static_cast<const float*>(logits) + off, tl, ti, v, dloss + r, static_cast<float*>(dlogits) + off, accumulate, st)
                   : bwd(s, static_cast<const uint16_t*>(logits) + off, tl, ti, v, dloss + r, static_cast<uint16_t*>(dlogits) + off, accumulate, st);
    });
}

}  // namespace lobra
