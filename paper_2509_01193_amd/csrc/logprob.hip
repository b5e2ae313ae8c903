// Log probabilities of given tokens under rows of logits, entropy and the likeliest alternatives, and the gradient of the logits
// (the loss of a training step; what serving reports).
//
// With m = max z, S = sum exp(z - m), U = sum exp(z - m) (z - m) of a row:
//     lse = m + ln S      logp = (z_target - m) - ln S      entropy = ln S - U / S
// and with p = exp(z - lse)    dz = dlogp (1[target] - p) - dentropy p ((z - lse) + entropy).
//
// Forward reads a row once: every thread keeps m, S, U of the elements it has seen and corrects S and U when its m grows; they are
// joined over the workgroup at the end.  The row's own maximum is the reference (not a multiple of it in the log2 domain, which would
// save an instruction): differences of equal logits are 0 at any magnitude, so that rows of the type's lowest value are uniform ones.
// A workgroup per row; nothing is split over workgroups, since a launch that joins costs more than what a row of 256 KiB takes.
// Bound: memory; per element some ten VALU slots, four of them the exponential, where the memory's rate leaves 13 to a bf16 element.  A row alone
// is bound by these on its compute unit.  Measured, us: 8190 x 32000 bf16 forward 89 (of 524 MB, 5.9 TB/s; right behind a backward pass, whose
// gradients are still on their way to memory, 124), backward 206 (of 1048 MB, 5.1 TB/s), over the logits 151; 4096 x 128000 with entropy and 8
// alternatives 186; 40 x 32000 with 20 of them 9; one row of 32000 5, of 256000 20, with 32 alternatives 8 and 27.
#include "kernels.h"
#include "row_common.h"

namespace lobra {

using namespace rows;

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kFar = -1e30f;            // below every difference that matters: exp is 0, and 0 times it is 0
constexpr int kCandidates = 1024;         // logits that may be among the largest: 8 KiB of LDS

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// m, S and U of some elements (U in units of log2: sum of 2^x x with x = (z - m) log2 e)
struct Stat {
    float m, s, u;
};

template <bool ENT> __device__ __forceinline__ void rescale(Stat& a, float m)
{
    const float x = fmaxf((a.m - (m == -INFINITY ? 0.f : m)) * kLog2e, kFar);        // (a.m = -inf: s and u are 0)
    const float f = exp2_fast(x);
    if (ENT) a.u = f * (a.u + a.s * x);
    a.s *= f;
    a.m = m;
}

// (the more elements at a time, the less often m grows: nearly every time some lane's does)
template <bool ENT, int N> __device__ __forceinline__ void take(Stat& a, const float (&z)[N])
{
    float c = z[0];
#pragma unroll
    for (int i = 1; i < N; ++i) c = fmaxf(c, z[i]);
    if (c > a.m) rescale<ENT>(a, c);
    const float ref = a.m == -INFINITY ? 0.f : a.m;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float x = (z[i] - ref) * kLog2e;       // (NaN where z is NaN or m = +inf: s stays NaN from here on)
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
template <typename E, int NT, bool ENT> __device__ __forceinline__ Stat row_stat(const E* row, const RowShape& sh)
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
    for (int32_t first = 0; first < sh.packets; first += U * NT) {
        if (first + U * NT < sh.packets) fetch(next, first + U * NT);
        float z[U * N];
#pragma unroll
        for (int c = 0; c < U; ++c)
#pragma unroll
            for (int e = 0; e < N; ++e) z[c * N + e] = Packet<E>::element(q[c], e);
        take<ENT>(a, z);
#pragma unroll
        for (int c = 0; c < U; ++c) q[c] = next[c];
    }
    if (has_edge) {
        const float z[1] = {Elem<E>::load(&edge, 0)};
        take<ENT>(a, z);
    }
    return a;
}

// f(first index, values) over the elements of the row that this thread looks at, in ascending order of index within the whole packets
template <typename E, int NT, typename F> __device__ __forceinline__ void each(const E* row, const RowShape& sh, F&& f)
{
    constexpr int N = Packet<E>::N;
    const u32x4* p = reinterpret_cast<const u32x4*>(row + sh.head);
    int32_t i = threadIdx.x;
    for (; i + 3 * NT < sh.packets; i += 4 * NT) {
        u32x4 q[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) q[c] = p[i + c * NT];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            float z[N];
            Packet<E>::widen(q[c], z);
            f(sh.head + (i + c * NT) * N, z);
        }
    }
    for (; i < sh.packets; i += NT) {
        float z[N];
        Packet<E>::widen(p[i], z);
        f(sh.head + i * N, z);
    }
    // the elements in front of the first packet and behind the last one: fewer than 2 N, a thread each
    const int32_t e = threadIdx.x;
    if (e < sh.head + sh.tail) {
        const int32_t at = e < sh.head ? e : e + sh.packets * N;
        float z[1] = {element(row, at)};
        f(at, z);
    }
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

// The top_k largest of a row, all of whose threads know m and ln S.
// 64 groups of threads have a maximum each; the top_k-th largest of these, tau, has at least top_k logits at or above it, and what is
// not below tau was seen by a few threads only.  All threads together look at these threads' packets again (they are in the caches) and
// put what is not below tau on a list, whose members find their place by counting who is larger.  (Each thread looking at its own packets
// again keeps its wave busy with nearly the whole row: 4096 x 128000, 8 alternatives, 250 us instead of 188.)  Rows with more
// candidates than the list holds (thousands of equal logits) take the largest top_k times over.
template <typename E, int NT>
__device__ void alternatives(const E* row, const RowShape& sh, int32_t V, float mine, float m, float ln_s, int32_t k, float* top_logp,
                             int32_t* top_id)
{
    __shared__ uint64_t list[kCandidates];
    __shared__ float group_max[64];
    __shared__ float tau_s;
    __shared__ int32_t count, seers;
    __shared__ int32_t seer[NT];
    constexpr int G = NT / 64;
    const int32_t tid = threadIdx.x, lane = tid & 63;
    float g = mine;
#pragma unroll
    for (int x = 1; x < G; x <<= 1) g = fmaxf(g, __shfl_xor(g, x));
    if (tid % G == 0) group_max[tid / G] = g;
    if (tid == 0) count = seers = 0;
    __syncthreads();
    if (tid < 64) {
        // whoever has k - 1 others in front of it (a short loop: code that runs once is fetched about as slowly as it is long)
        const float v = group_max[lane];
        int32_t in_front = 0;
#pragma unroll 8
        for (int32_t o = 0; o < 64; ++o) {
            const float other = group_max[o];
            in_front += other > v || (other == v && o < lane) ? 1 : 0;
        }
        if (in_front == k - 1) tau_s = v;
    }
    __syncthreads();
    const float tau = tau_s;
    auto write = [&](int32_t place, uint64_t key) {
        const float v = key_value(key);
        if (top_logp) top_logp[place] = m == -INFINITY ? -INFINITY : (v - m) - ln_s;
        if (top_id) top_id[place] = key_index(key);
    };
    if (mine >= tau && mine > -INFINITY) seer[atomicAdd(&seers, 1)] = tid;
    __syncthreads();
    auto consider = [&](float z, int32_t at) {
        if (z >= tau && z > -INFINITY) {
            const int32_t n = atomicAdd(&count, 1);
            if (n < kCandidates) list[n] = order_key(z, at);
        }
    };
    {
        constexpr int N = Packet<E>::N;
        const u32x4* p = reinterpret_cast<const u32x4*>(row + sh.head);
        const int32_t of = seers, total = of * ((sh.packets + NT - 1) / NT);
        for (int32_t j = tid; j < total; j += NT) {
            const int32_t step = j / of, i = step * NT + seer[j - step * of];
            if (i >= sh.packets) continue;
            const u32x4 q = p[i];
            uint32_t hits = 0;
#pragma unroll
            for (int e = 0; e < N; ++e) hits |= Packet<E>::element(q, e) >= tau ? 1u << e : 0u;
            for (; hits; hits &= hits - 1) {
                const int32_t at = sh.head + i * N + __builtin_ctz(hits);
                consider(element(row, at), at);
            }
        }
        if (tid < sh.head + sh.tail) {
            const int32_t at = tid < sh.head ? tid : tid + sh.packets * N;
            consider(element(row, at), at);
        }
    }
    __syncthreads();
    const int32_t n = count;
    int32_t filled = min(n, k);
    if (n <= kCandidates) {
        for (int32_t c = tid; c < n; c += NT) {
            const uint64_t key = list[c];
            int32_t rank = 0;
#pragma unroll 4
            for (int32_t o = 0; o < n; ++o) rank += list[o] > key ? 1 : 0;
            if (rank < k) write(rank, key);
        }
    } else {
        uint64_t last = ~uint64_t(0);
        for (int32_t r = 0; r < k; ++r) {
            uint64_t best = 0;
            each<E, NT>(row, sh, [&](int32_t at, const auto& z) {
#pragma unroll
                for (int i = 0; i < int(sizeof(z) / sizeof(float)); ++i)
                    if (z[i] >= tau) {
                        const uint64_t key = order_key(z[i], at + i);
                        best = key < last && key > best ? key : best;
                    }
            });
#pragma unroll
            for (int x = 32; x > 0; x >>= 1) {
                const uint64_t o = __shfl_xor((unsigned long long)best, x);
                best = o > best ? o : best;
            }
            __syncthreads();                          // (the round before has been read)
            if (lane == 0) list[tid / 64] = best;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < G; ++w) best = list[w] > best ? list[w] : best;
            if (tid == 0) write(r, best);
            last = best;
        }
    }
    // barred tokens (-inf) in order of index where nothing else is left, then nothing
    if (filled < k && tid < 64) {
        for (int32_t base = 0; base < V && filled < k; base += 64) {
            const bool hit = base + lane < V && element(row, base + lane) == -INFINITY;
            const uint64_t mask = __ballot(hit);
            const int32_t place = filled + __popcll(mask & ((uint64_t(1) << lane) - 1));
            if (hit && place < k) write(place, order_key(-INFINITY, base + lane));
            filled += __popcll(mask);
        }
        if (lane >= filled && lane < k) {
            if (top_logp) top_logp[lane] = -INFINITY;
            if (top_id) top_id[lane] = -1;
        }
    }
}

template <typename E, int NT, bool ENT, bool TOP>
__global__ __launch_bounds__(NT)
void logprob_fwd_kernel(const E* __restrict__ logits, int64_t ld, int32_t V, const int32_t* __restrict__ target, LogprobOut out, int32_t top_k)
{
    __shared__ Stat part[NT / 64];
    const size_t r = size_t(xcd_contiguous(int32_t(blockIdx.x), int32_t(gridDim.x)));
    const E* row = logits + r * size_t(ld);
    const RowShape sh = row_shape(row, V);
    const int32_t tid = threadIdx.x;
    const int32_t tgt = target ? target[r] : -1;
    const bool has = tgt >= 0 && tgt < V;
    Stat a = row_stat<E, NT, ENT>(row, sh);
    const float zt = has ? element(row, tgt) : 0.f;
    const float mine = a.m;
    rescale<ENT>(a, wave_max(a.m));
    a.s = wave_sum(a.s);
    if (ENT) a.u = wave_sum(a.u);
    if ((tid & 63) == 0) part[tid >> 6] = a;
    __syncthreads();
    float m = part[0].m;
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) m = fmaxf(m, part[w].m);
    float s = 0.f, u = 0.f;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
        Stat b = part[w];
        rescale<ENT>(b, m);
        s += b.s;
        u += b.u;
    }
    const float ln_s = logf(s);
    if (tid == 0) {
        // (s = 0: nothing but -inf)
        const float sum = s == 0.f ? -INFINITY : m + ln_s;
        if (out.lse) out.lse[r] = sum;
        if (out.lse_rest) out.lse_rest[r] = s == 0.f ? 0.f : fabsf(m) >= fabsf(ln_s) ? (m - sum) + ln_s : (ln_s - sum) + m;
        if (out.logp) out.logp[r] = !has ? 0.f : s == 0.f ? -INFINITY : (zt - m) - ln_s;
        if (ENT) out.entropy[r] = s == 0.f ? 0.f : ln_s - kLn2 * (u / s);
    }
    if (TOP) alternatives<E, NT>(row, sh, V, mine, m, ln_s, top_k, out.top_logp ? out.top_logp + r * size_t(top_k) : nullptr,
                                 out.top_id ? out.top_id + r * size_t(top_k) : nullptr);
}

// Workgroup (row, part): packets part * NT + ... with a stride of all parts.  In place (dlogits = logits) every thread writes what it has
// read itself.  A row without any weight is not read.
template <typename E, int NT, bool ENT>
__global__ __launch_bounds__(NT)
void logprob_bwd_kernel(const E* logits, int64_t ld, int32_t V, const int32_t* __restrict__ target, LogprobGrad in, E* dlogits)
{
    constexpr int N = Packet<E>::N;
    const size_t r = size_t(xcd_contiguous(int32_t(blockIdx.x), int32_t(gridDim.x)));
    const E* row = logits + r * size_t(ld);
    E* out = dlogits + r * size_t(ld);
    const RowShape sh = row_shape(row, V);            // (logits and dlogits are aligned alike: both bases to 16 bytes)
    const int32_t tgt = target ? target[r] : -1;
    const bool has = tgt >= 0 && tgt < V;
    const float w = has && in.dlogp ? in.dlogp[r] : 0.f, v = ENT ? in.dentropy[r] : 0.f, l = in.lse[r], h = ENT ? in.entropy[r] : 0.f;
    const float rest = in.lse_rest ? -kLog2e * in.lse_rest[r] : 0.f;
    const bool zero = (w == 0.f && v == 0.f) || l == -INFINITY;
    auto gradient = [&](float z, int32_t at) {
        const float x = fmaf(z - l, kLog2e, rest), p = exp2_fast(x);         // x = log2 p
        const float g = ENT ? p * (-w - v * fmaf(fmaxf(x, kFar), kLn2, h)) : -w * p;
        return at == tgt && has ? g + w : g;
    };
    const u32x4* src = reinterpret_cast<const u32x4*>(row + sh.head);
    u32x4* dst = reinterpret_cast<u32x4*>(out + sh.head);
    const int32_t t = threadIdx.x, stride = NT * int32_t(gridDim.y), first = blockIdx.y * NT + t;
    if (zero) {
        for (int32_t i = first; i < sh.packets; i += stride) dst[i] = u32x4{0u, 0u, 0u, 0u};
    } else {
        for (int32_t i = first; i < sh.packets; i += stride) {
            float z[N], g[N];
            Packet<E>::widen(src[i], z);
#pragma unroll
            for (int c = 0; c < N; ++c) g[c] = gradient(z[c], sh.head + i * N + c);
            dst[i] = Packet<E>::narrow(g);
        }
    }
    if (blockIdx.y == 0 && t < sh.head + sh.tail) {
        const int32_t at = t < sh.head ? t : t + sh.packets * N;
        Elem<E>::store(out, size_t(at), zero ? 0.f : gradient(element(row, at), at));
    }
}

template <typename E, int NT, bool ENT>
void launch_fwd(const LogprobShape& s, const E* logits, const int32_t* target, const LogprobOut& out, hipStream_t st)
{
    const dim3 grid(uint32_t(s.T));
    if (s.top_k > 0 && (out.top_logp || out.top_id))
        logprob_fwd_kernel<E, NT, ENT, true><<<grid, NT, 0, st>>>(logits, s.ld, s.V, target, out, s.top_k);
    else
        logprob_fwd_kernel<E, NT, ENT, false><<<grid, NT, 0, st>>>(logits, s.ld, s.V, target, out, 0);
}

template <typename E> hipError_t fwd(const LogprobShape& s, const E* logits, const int32_t* target, const LogprobOut& out, hipStream_t st)
{
    // four to eight packets a thread: more threads than that wait for each other at a row's end longer than they read, fewer have too little
    // on the way (forward alone, us, with 64 / 128 / 256 / 512 threads: 16000 x 1000 10 / 15 / 25 / 47, x 4000 25 / 24 / 32 / 62, 8000 x
    // 16000 50 / 48 / 45 / 45, 4096 x 128000 with 8 alternatives 315 / 261 / 214 / 195, 1 x 32000 with 20 28 / 16 / 11 / 9.5)
    const int32_t packets = s.V / Packet<E>::N;
    if (out.entropy) {
        if (packets <= 256) launch_fwd<E, 64, true>(s, logits, target, out, st);
        else if (packets <= 512) launch_fwd<E, 128, true>(s, logits, target, out, st);
        else if (packets <= 2048) launch_fwd<E, 256, true>(s, logits, target, out, st);
        else launch_fwd<E, 512, true>(s, logits, target, out, st);
    } else {
        if (packets <= 256) launch_fwd<E, 64, false>(s, logits, target, out, st);
        else if (packets <= 512) launch_fwd<E, 128, false>(s, logits, target, out, st);
        else if (packets <= 2048) launch_fwd<E, 256, false>(s, logits, target, out, st);
        else launch_fwd<E, 512, false>(s, logits, target, out, st);
    }
    return hipGetLastError();
}

template <typename E>
hipError_t bwd(const LogprobShape& s, const E* logits, const int32_t* target, const LogprobGrad& in, E* dlogits, hipStream_t st)
{
    constexpr int NT = 256;
    // a workgroup per row where there are enough rows, else several, of at least four packets a thread
    const int64_t most = (int64_t(s.V) / Packet<E>::N + 4 * NT - 1) / (4 * NT), wanted = (2048 + s.T - 1) / s.T;
    const dim3 grid(uint32_t(s.T), uint32_t(wanted < most ? wanted : most > 0 ? most : 1));
    if (in.dentropy) logprob_bwd_kernel<E, NT, true><<<grid, NT, 0, st>>>(logits, s.ld, s.V, target, in, dlogits);
    else logprob_bwd_kernel<E, NT, false><<<grid, NT, 0, st>>>(logits, s.ld, s.V, target, in, dlogits);
    return hipGetLastError();
}

// (a launch holds less than 2^32 threads)
constexpr int64_t kRowsPerLaunch = 1 << 22;

// f(the shape of a run of rows, first row)
template <typename F> hipError_t by_rows(const LogprobShape& shape, F&& f)
{
    for (int64_t r = 0; r < shape.T; r += kRowsPerLaunch) {
        LogprobShape s = shape;
        s.T = shape.T - r < kRowsPerLaunch ? shape.T - r : kRowsPerLaunch;
        const hipError_t e = f(s, r);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}
template <typename P> P* at(P* p, int64_t i) { return p ? p + i : p; }

}  // namespace

hipError_t logprob_fwd(const LogprobShape& shape, const void* logits, const int32_t* target, const LogprobOut& out, hipStream_t st)
{
    return by_rows(shape, [&](const LogprobShape& s, int64_t r) {
        const LogprobOut o{at(out.logp, r), at(out.lse, r), at(out.lse_rest, r), at(out.entropy, r), at(out.top_logp, r * s.top_k),
                           at(out.top_id, r * s.top_k)};
        return s.dtype == LOBRA_F32 ? fwd(s, static_cast<const float*>(logits) + r * s.ld, at(target, r), o, st)
                                    : fwd(s, static_cast<const uint16_t*>(logits) + r * s.ld, at(target, r), o, st);
    });
}

hipError_t logprob_bwd(const LogprobShape& shape, const void* logits, const int32_t* target, const LogprobGrad& in, void* dlogits, hipStream_t st)
{
    return by_rows(shape, [&](const LogprobShape& s, int64_t r) {
        const LogprobGrad g{at(in.lse, r), at(in.lse_rest, r), at(in.entropy, r), at(in.dlogp, r), at(in.dentropy, r)};
        const int64_t off = r * s.ld;
        return s.dtype == LOBRA_F32 ? bwd(s, static_cast<const float*>(logits) + off, at(target, r), g, static_cast<float*>(dlogits) + off, st)
                                    : bwd(s, static_cast<const uint16_t*>(logits) + off, at(target, r), g, static_cast<uint16_t*>(dlogits) + off, st);
    });
}

}  // namespace lobra
