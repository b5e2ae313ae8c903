// A step of beam search: the best continuations of every request over its beams and the vocabulary, and the reordering of what is kept per
// sequence.
//
// Selection.  Beam b of score s continued by token j has the value (s - lse_b) + z_j, lse_b = ln sum exp(z_b).  A beam's own best continuations
// are its largest logits, so a part of a row hands on its n largest logits, the lowest index first among equals, and its sum; a workgroup per
// request then makes lse and values, in fp64, and orders what is left.  A logit is read once: a part's 16 KB stay in registers from the sum to
// the choice.  Rows are cut into parts by index, wherever they begin in memory, so that beams of equal logits have equal sums bit for bit, and
// what is equal in the formula is equal here.
// Reordering.  A thread has the same 16 bytes of all rows of a request: it has read every row it needs before it writes one, which is all
// that reordering in place takes.
#include "kernels.h"
#include "row_common.h"
#include "row_logits.h"

namespace lobra {

using namespace rows;

namespace {

constexpr int kThreads = 256;
// Bytes of a row that a workgroup works on at a time.  64 x 8 x 128000, the choice of a step, us: bf16 with 8 KB 51, 16 KB 43, 32 KB 53 (512 threads 46);
// fp32 8 KB 79, 16 KB 59, 32 KB 70, 64 KB 58; 5 x 5 x 50257 fp32 with its states 13.3, 14.3, 15.4.
constexpr int kPartBytes = 16384;
template <typename E> constexpr int kPart = kPartBytes / int(sizeof(E));
constexpr int kPackets = 128;             // 16 bytes each of a part's logits that may hold one of the best
static_assert(LOBRA_MAX_VOCAB <= 1 << 24 && LOBRA_MAX_TOP <= 256, "a token's and a beam's bits in a continuation's place");
constexpr int kList = 512;                // of a part's logits, or a request's continuations, that may be among the best

// 16 bytes of a row that may begin at any element.
template <typename E> struct Loose;
template <> struct Loose<float> { typedef u32x4 __attribute__((aligned(4))) type; };
template <> struct Loose<uint16_t> { typedef u32x4 __attribute__((aligned(2))) type; };

template <typename E> __device__ __forceinline__ void put(u32x4& q, int e, E v)
{
    if constexpr (sizeof(E) == 4) q[e] = __float_as_uint(v);
    else q[e >> 1] = e & 1 ? (q[e >> 1] & 0xffffu) | uint32_t(v) << 16 : (q[e >> 1] & 0xffff0000u) | uint32_t(v);
}

// A number that at least k (<= 64) of 64 numbers reach, a lane's each, and few more than k: the largest whose order's lower 16 bits are clear (all
// that bf16 has).  Every lane of the wave has to be active; all get it.  (Bit by bit, a ballot each: a tenth of the instructions of counting in front.)
__device__ __forceinline__ uint32_t float_order(float z)
{
    const uint32_t b = __float_as_uint(z + 0.f);       // (-0 is 0)
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ uint32_t reached_by(uint32_t order, int32_t k)
{
    uint32_t t = 0;
#pragma unroll
    for (int bit = 31; bit >= 16; --bit) {
        const uint32_t c = t | 1u << bit;
        if (__popcll(__ballot(order >= c)) >= k) t = c;
    }
    return t;
}

// Whether a beam's logits are looked at.
__device__ __forceinline__ bool looked_at(float score, const int32_t* done, size_t row) { return score > -INFINITY && !(done && done[row] != 0); }

// Part blockIdx.x % parts of row blockIdx.x / parts: keys [n] (0: none left) in order, {max, sum exp(z - max)}.
// 64 groups of four threads have a maximum each; what the n-th largest of these (or a little less) reaches, n logits at least, goes on a list and
// finds its place there by counting who is larger.  Parts with more of them than the list holds (equal logits) take the largest n times over.
// Bound: neither is full, VALUs busy for 63 % and 2.8 TB/s, since a workgroup computes when its loads are there and has no others on their way: 512 x 128000 bf16 of which a
// tenth is done 38 to 44 us, four rows of 32000 5.1.
template <typename E>
__global__ __launch_bounds__(kThreads)
void beam_part_kernel(BeamShape sh, const E* __restrict__ logits, const float* __restrict__ score, const int32_t* __restrict__ done, int32_t parts,
                      bool at_once, uint64_t* __restrict__ keys, float2* __restrict__ sums)
{
    constexpr int N = Packet<E>::N, U = kPart<E> / (kThreads * N), W = kThreads / 64;
    __shared__ uint64_t list[kList];
    __shared__ float group_max[64];
    __shared__ Stat stat[W];
    __shared__ u32x4 packet[kPackets];
    __shared__ int32_t packet_at[kPackets], packets, count;
    const int32_t tid = threadIdx.x, lane = tid & 63, n = sh.n_out;
    const int32_t row = int32_t(blockIdx.x) / parts, base = (int32_t(blockIdx.x) - row * parts) * kPart<E>, len = min(kPart<E>, sh.V - base);
    // (at_once: the logits are fetched before it is known whether they are looked at, a round trip less; many parts find out first)
    if (!at_once && !looked_at(score[row], done, size_t(row))) return;
    const E* p = logits + size_t(row) * size_t(sh.ld) + base;
    u32x4 q[U];
    if (len == kPart<E>) {                            // (uniform)
#pragma unroll
        for (int c = 0; c < U; ++c) q[c] = *reinterpret_cast<const typename Loose<E>::type*>(p + (c * kThreads + tid) * N);
    } else
#pragma unroll
    for (int c = 0; c < U; ++c) {
        const int32_t at = (c * kThreads + tid) * N;
        if (at + N <= len) {
            q[c] = *reinterpret_cast<const typename Loose<E>::type*>(p + at);
        } else {                                     // (the row's last packet, then nothing)
            q[c] = nothing<E>();
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (at + e < len) put<E>(q[c], e, p[at + e]);
        }
    }
    if (at_once && !looked_at(score[row], done, size_t(row))) return;
    if (tid == 0) count = packets = 0;
    // (widened twice, so that 32 elements wait in 16 registers: twice the workgroups on a compute unit)
    float most[U];                                   // of each packet
    Stat a{-INFINITY, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < U; ++c) {
        most[c] = Packet<E>::element(q[c], 0);
#pragma unroll
        for (int e = 1; e < N; ++e) most[c] = fmaxf(most[c], Packet<E>::element(q[c], e));
        a.m = fmaxf(a.m, most[c]);
        asm volatile("" : "+v"(q[c]));
    }
    const float ref = a.m == -INFINITY ? 0.f : a.m;
#pragma unroll
    for (int c = 0; c < U; ++c)
#pragma unroll
        for (int e = 0; e < N; ++e) a.s += exp2_fast((Packet<E>::element(q[c], e) - ref) * kLog2e);
    const float mine = a.m;
    {
        float g = mine;
#pragma unroll
        for (int x = 1; x < kThreads / 64; x <<= 1) g = fmaxf(g, __shfl_xor(g, x));
        if (tid % (kThreads / 64) == 0) group_max[tid / (kThreads / 64)] = g;
    }
    rescale<false>(a, wave_max(a.m), kLog2e);
    a.s = wave_sum(a.s);
    if (lane == 0) stat[tid >> 6] = a;
    __syncthreads();
    const uint32_t tau = reached_by(float_order(group_max[lane]), n);       // (-inf: 0x007f....; its bits below are clear in tau)
    if (tid == 0) {
        float m = stat[0].m, s = 0.f;
#pragma unroll
        for (int w = 1; w < W; ++w) m = fmaxf(m, stat[w].m);
#pragma unroll
        for (int w = 0; w < W; ++w) {
            Stat b = stat[w];
            rescale<false>(b, m, kLog2e);
            s += b.s;
        }
        sums[blockIdx.x] = make_float2(m, s);
    }
    // the packets that reach tau, then their elements, one a thread (looking through every thread's packets is four times the code)
#pragma unroll
    for (int c = 0; c < U; ++c)
        if (most[c] > -INFINITY && float_order(most[c]) >= tau) {
            const int32_t o = atomicAdd(&packets, 1);
            if (o < kPackets) packet[o] = q[c], packet_at[o] = (c * kThreads + tid) * N;
        }
    __syncthreads();
    const int32_t some = packets;
    if (some <= kPackets)
        for (int32_t i = tid; i < some * N; i += kThreads) {
            const uint32_t w = reinterpret_cast<const uint32_t*>(packet)[sizeof(E) == 4 ? i : i >> 1];
            const float z = __uint_as_float(sizeof(E) == 4 ? w : i & 1 ? w & 0xffff0000u : w << 16);
            if (z > -INFINITY && float_order(z) >= tau) {
                const int32_t o = atomicAdd(&count, 1);
                if (o < kList) list[o] = order_key(z, base + packet_at[i / N] + i % N);
            }
        }
    __syncthreads();
    const int32_t found = some <= kPackets ? count : kList + 1;
    uint64_t* const out = keys + size_t(blockIdx.x) * n;
    if (found <= kList) {
        for (int32_t c = tid; c < found; c += kThreads) {
            const uint64_t key = list[c];
            int32_t place = 0;
#pragma unroll 4
            for (int32_t o = 0; o < found; ++o) place += list[o] > key ? 1 : 0;
            if (place < n) out[place] = key;
        }
        if (tid >= found && tid < n) out[tid] = 0;   // (n <= 32)
        return;
    }
    uint64_t last = ~uint64_t(0);
    for (int32_t r = 0; r < n; ++r) {
        uint64_t best = 0;
        // (from memory once more: from the registers they would all be keys there, and those are few)
        for (int32_t i = tid; i < len; i += kThreads) {
            const float z = element(p, i);
            const uint64_t key = z > -INFINITY ? order_key(z, base + i) : 0;
            best = key < last && key > best ? key : best;
        }
#pragma unroll
        for (int x = 32; x > 0; x >>= 1) {
            const uint64_t o = __shfl_xor((unsigned long long)best, x);
            best = o > best ? o : best;
        }
        __syncthreads();                             // (the round before has been read)
        if (lane == 0) list[tid >> 6] = best;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < W; ++w) best = list[w] > best ? list[w] : best;
        if (tid == 0) out[r] = best;
        last = best;
    }
}

// A continuation as two numbers: its value's order, and beam, logit and token, the lower the better: 8 bits of beam, the logit's order from the largest down, 24 bits of
// token (of a beam that is done: of no token).  Within a beam the logits' order is the values', also where those are equal in 64 bits because the score is far larger than
// a logit, so that what a part hands on is what the request wants of it.
struct Next {
    uint64_t order, place;
    __device__ __forceinline__ bool operator>(const Next& o) const { return order > o.order || (order == o.order && place < o.place); }
};
__device__ __forceinline__ uint64_t double_order(double v)
{
    const uint64_t b = uint64_t(__double_as_longlong(v + 0.));
    return b >> 63 ? ~b : b | uint64_t(1) << 63;
}
__device__ __forceinline__ double order_value(uint64_t o)
{
    return __longlong_as_double((long long)(o >> 63 ? o & ~(uint64_t(1) << 63) : ~o));
}

// A workgroup per request: 16 lanes per beam for its lse, then the continuations as the logits in a part, by the upper halves of their orders.
// Bound: round trips and fp64 logarithms, 4 us for a request of four beams, 6.4 for 64 of eight beams with 16 parts each.
__global__ __launch_bounds__(kThreads)
void beam_merge_kernel(BeamShape sh, const float* score, const int32_t* __restrict__ done, int32_t done_token, int32_t parts,
                       const uint64_t* __restrict__ keys, const float2* __restrict__ sums, float* out_score, int32_t* __restrict__ out_beam,
                       int32_t* __restrict__ out_token)
{
    constexpr int W = kThreads / 64, G = 16, H = 4, kNear = 1024;        // H: continuations that a thread keeps
    __shared__ double offset[LOBRA_MAX_TOP];         // s - lse; of a beam that is done: s
    __shared__ int32_t kind[LOBRA_MAX_TOP];          // 0: no continuations, 1: its logits, 2: done
    __shared__ Next list[kList];
    __shared__ uint32_t group_max[64];
    __shared__ int32_t count, bins[kThreads], chosen[2], near[kNear], near_parts;
    static_assert(kThreads == 256, "a bin per thread");
    const int32_t tid = threadIdx.x, lane = tid & 63, n = sh.n_out;
    const size_t row0 = size_t(blockIdx.x) * sh.beams;
    const int32_t per = parts * n, total = sh.beams * per;
    const uint64_t* const k0 = keys + row0 * per;
    uint64_t held[H];
#pragma unroll
    for (int h = 0; h < H; ++h) held[h] = tid + h * kThreads < total ? k0[tid + h * kThreads] : 0;       // (of beams without any: not looked at)
    if (tid == 0) count = 0;
    for (int32_t b = tid / G; b < sh.beams; b += kThreads / G) {
        const float2* part = sums + (row0 + b) * parts;
        const float s = score[row0 + b];
        const bool logits = looked_at(s, done, row0 + b);
        float2 v = tid % G < parts ? part[tid % G] : make_float2(-INFINITY, 0.f);        // (perhaps never written)
        double l = 0.;
        if (logits) {
            float m = v.x;
            for (int32_t i = tid % G + G; i < parts; i += G) m = fmaxf(m, part[i].x);
#pragma unroll
            for (int x = 1; x < G; x <<= 1) m = fmaxf(m, __shfl_xor(m, x));
            double sum = 0.;
            for (int32_t i = tid % G; i < parts; i += G) {
                if (i >= G) v = part[i];
                sum += v.y > 0.f ? double(v.y) * exp(double(v.x) - double(m)) : double(v.y);        // (NaN stays NaN)
            }
#pragma unroll
            for (int x = 1; x < G; x <<= 1) sum += __shfl_xor(sum, x);
            l = double(m) + log(sum);
        }
        if (tid % G == 0) {
            kind[b] = logits ? (l > -INFINITY && l < INFINITY ? 1 : 0) : s > -INFINITY ? 2 : 0;
            offset[b] = double(s) - l;
        }
    }
    __syncthreads();
    auto value = [&](int32_t i, uint64_t key) {      // continuation i; order 0: there is none
        const int32_t beam = i / per, k = kind[beam];
        const double o = offset[beam];
        if (k == 1 && key != 0)
            return Next{double_order(o + double(key_value(key))), uint64_t(beam) << 56 | uint64_t(~uint32_t(key >> 32)) << 24 | uint32_t(key_index(key))};
        if (k == 2 && i == beam * per) return Next{double_order(o), uint64_t(beam) << 56};
        return Next{0, 0};
    };
    Next mine[H];
    uint32_t best = 0;
#pragma unroll
    for (int h = 0; h < H; ++h) {
        const int32_t i = tid + h * kThreads;
        mine[h] = i < total ? value(i, held[h]) : Next{0, 0};
        best = max(best, uint32_t(mine[h].order >> 32));
    }
#pragma unroll 4
    for (int32_t i = tid + H * kThreads; i < total; i += kThreads) best = max(best, uint32_t(value(i, k0[i]).order >> 32));
    uint32_t g = best;
#pragma unroll
    for (int x = 1; x < kThreads / 64; x <<= 1) g = max(g, uint32_t(__shfl_xor(int(g), x)));
    if (tid % (kThreads / 64) == 0) group_max[tid / (kThreads / 64)] = g;
    __syncthreads();
    const uint32_t tau = reached_by(group_max[lane], n);
    auto consider = [&](const Next& c) {
        if (c.order == 0 || uint32_t(c.order >> 32) < tau) return;
        const int32_t o = atomicAdd(&count, 1);
        if (o < kList) list[o] = c;
    };
#pragma unroll
    for (int h = 0; h < H; ++h) consider(mine[h]);
    for (int32_t i = tid + H * kThreads; i < total; i += kThreads) consider(value(i, k0[i]));
    __syncthreads();
    int32_t found = count;
    if (found > kList) {                             // (uniform)
        // What a group's maximum says is little where one beam is far ahead and a part hands on many: the upper half of the n-th largest order itself, eight bits at
        // a time from counts, over the parts whose first reaches tau.  (5 x 16 beams x 112768 fp32, 32 continuations, us: the best one 32 times over 608, so 139
        // over all parts, 91.)
        if (tid == 0) near_parts = 0;
        __syncthreads();
        for (int32_t l = tid; l < sh.beams * parts; l += kThreads) {
            const uint64_t order = value(l * n, k0[l * n]).order;
            if (order == 0 || uint32_t(order >> 32) < tau) continue;
            const int32_t o = atomicAdd(&near_parts, 1);
            if (o < kNear) near[o] = l;
        }
        __syncthreads();
        const bool few = near_parts <= kNear;        // (uniform)
        const int32_t all = few ? near_parts * n : total;
        auto candidate = [&](int32_t i) {
            const int32_t at = few ? near[i / n] * n + i % n : i;
            return value(at, k0[at]);
        };
        uint32_t nth = 0;
        int32_t want = n;                            // of those whose upper bits are nth's
        for (int32_t shift = 24; shift >= 0; shift -= 8) {
            bins[tid] = 0;
            __syncthreads();
#pragma unroll 4
            for (int32_t i = tid; i < all; i += kThreads) {
                const uint64_t order = candidate(i).order;
                const uint32_t up = uint32_t(order >> 32);
                if (order != 0 && (uint64_t(up ^ nth) >> (shift + 8)) == 0) atomicAdd(&bins[up >> shift & 255], 1);
            }
            __syncthreads();
            int32_t above = 0;                       // in the bins over the thread's
#pragma unroll 8
            for (int32_t b = tid + 1; b < kThreads; ++b) above += bins[b];
            if (above < want && above + bins[tid] >= want) chosen[0] = tid, chosen[1] = want - above;
            __syncthreads();
            nth |= uint32_t(chosen[0]) << shift;
            want = chosen[1];
        }
        if (tid == 0) count = 0;
        __syncthreads();
#pragma unroll 4
        for (int32_t i = tid; i < all; i += kThreads) {
            const Next c = candidate(i);
            if (c.order != 0 && uint32_t(c.order >> 32) >= nth) {
                const int32_t o = atomicAdd(&count, 1);
                if (o < kList) list[o] = c;
            }
        }
        __syncthreads();
        found = count;
    }
    auto write = [&](int32_t place, const Next& c) {
        const size_t o = size_t(blockIdx.x) * n + place;
        out_score[o] = c.order ? float(order_value(c.order)) : -INFINITY;
        const int32_t beam = int32_t(c.place >> 56);
        out_beam[o] = c.order ? beam : -1;
        out_token[o] = !c.order ? -1 : kind[beam] == 2 ? done_token : int32_t(c.place & 0xffffff);
    };
    if (found <= kList) {
        for (int32_t c = tid; c < found; c += kThreads) {
            const Next x = list[c];
            int32_t place = 0;
#pragma unroll 8
            for (int32_t o = 0; o < found; ++o) place += list[o] > x ? 1 : 0;
            if (place < n) write(place, x);
        }
        if (tid >= found && tid < n) write(tid, Next{0, 0});
        return;
    }
    // more of nearly the same value than the list holds (orders with the upper half of the n-th): the best n times over
    Next last{~uint64_t(0), 0};
    for (int32_t r = 0; r < n; ++r) {
        Next top{0, 0};
        for (int32_t i = tid; i < total; i += kThreads) {
            const Next c = value(i, k0[i]);
            if (c.order && last > c && c > top) top = c;
        }
#pragma unroll
        for (int x = 32; x > 0; x >>= 1) {
            const Next o{uint64_t(__shfl_xor((unsigned long long)top.order, x)), uint64_t(__shfl_xor((unsigned long long)top.place, x))};
            if (o > top) top = o;
        }
        __syncthreads();
        if (lane == 0) list[tid / 64] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < W; ++w)
            if (list[w] > top) top = list[w];
        if (tid == 0) write(r, top);
        last = top;
    }
}

// ---- reordering ---------------------------------------------------------------------------------------------------------------
// Bound: memory.  4 tensors of 512 rows of up to 262 KB, 8 beams, half of each used on average, out of place: 68 us; a row that several beams go on from comes
// from memory once.
constexpr int kStates = 64;                          // tensors of a launch
struct StateTable {
    const char* src[kStates];
    char* dst[kStates];
    int64_t row_bytes[kStates], unit[kStates];
};
static_assert(sizeof(StateTable) + 64 <= 4096, "the arguments of a launch");

// Units of type U; blockIdx = (256 units of a row, request, tensor).  B: at least the beams.  IN_PLACE: a thread has read all rows before it writes one;
// else four at a time.
template <typename U, int B, bool IN_PLACE>
__global__ __launch_bounds__(256)
void beam_reorder_kernel(StateTable tab, int64_t first_block, int32_t first_req, int32_t beams, const int32_t* __restrict__ parent, int64_t parent_ld,
                         const int32_t* __restrict__ used)
{
    const int32_t s = blockIdx.z;
    const int64_t req = int64_t(first_req) + blockIdx.y, row = tab.row_bytes[s];
    int64_t bytes = row;
    if (used) {
        const int32_t u = used[req];
        const int64_t most = tab.unit[s] > 0 ? row / tab.unit[s] : 0;
        bytes = u < 0 ? 0 : u >= most ? row : u * tab.unit[s];
    }
    const int64_t base = (first_block + blockIdx.x) * 256 * int64_t(sizeof(U)), left = bytes - base;
    if (left <= 0) return;
    const int32_t* const from = parent + req * parent_ld;
    const char* const src = tab.src[s] + req * beams * row + base;
    char* const dst = tab.dst[s] + req * beams * row + base;
    // n bytes from `off` on, of every beam
    auto move = [&](auto unit, uint32_t off) __attribute__((always_inline)) {
        typedef decltype(unit) T;
        if constexpr (IN_PLACE) {
            T v[B];
#pragma unroll
            for (int i = 0; i < B; ++i) {
                const int32_t of = i < beams ? from[i] : -1;
                if (of >= 0 && of < beams && of != i) v[i] = *reinterpret_cast<const T*>(src + of * row + off);
                // (a join the optimiser cannot see through: it made a path of its own of every combination of rows that move, 222 registers for eight)
                if constexpr (sizeof(T) >= 4) asm volatile("" : "+v"(v[i]));
            }
#pragma unroll
            for (int i = 0; i < B; ++i) {
                const int32_t of = i < beams ? from[i] : -1;
                if (of >= 0 && of < beams && of != i) *reinterpret_cast<T*>(dst + i * row + off) = v[i];
            }
        } else {
            for (int32_t i0 = 0; i0 < beams; i0 += 4) {
                T v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int32_t of = i0 + i < beams ? from[i0 + i] : -1;
                    if (of >= 0 && of < beams) v[i] = *reinterpret_cast<const T*>(src + of * row + off);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int32_t of = i0 + i < beams ? from[i0 + i] : -1;
                    if (of >= 0 && of < beams) *reinterpret_cast<T*>(dst + (i0 + i) * row + off) = v[i];
                }
            }
        }
    };
    const uint32_t mine = threadIdx.x * uint32_t(sizeof(U));
    if (int64_t(mine) + int64_t(sizeof(U)) <= left) {
        move(U{}, mine);
    } else if (sizeof(U) > 1 && mine < left) {       // the end of what is used lies within the unit (a row itself is whole ones)
#pragma unroll 1
        for (uint32_t e = mine; e < left; ++e) move(uint8_t{}, e);
    }
}

template <typename U, bool IN_PLACE>
hipError_t launch_reorder(const StateTable& tab, dim3 grid, int64_t first_block, int32_t first_req, int32_t beams, const int32_t* parent,
                          int64_t parent_ld, const int32_t* used, hipStream_t st)
{
#define LOBRA_REORDER(B) beam_reorder_kernel<U, B, IN_PLACE><<<grid, 256, 0, st>>>(tab, first_block, first_req, beams, parent, parent_ld, used)
    if (!IN_PLACE || beams <= 4) LOBRA_REORDER(4);
    else if (beams <= 8) LOBRA_REORDER(IN_PLACE ? 8 : 4);
    else if (beams <= 16) LOBRA_REORDER(IN_PLACE ? 16 : 4);
    else LOBRA_REORDER(IN_PLACE ? 32 : 4);
#undef LOBRA_REORDER
    return hipGetLastError();
}

}  // namespace

int32_t beam_parts(int32_t dtype, int32_t V)
{
    const int32_t part = dtype == LOBRA_F32 ? kPart<float> : kPart<uint16_t>;
    return (V - 1) / part + 1;
}

hipError_t beam_select(const BeamShape& s, const void* logits, const float* score, const int32_t* done, int32_t done_token, float* out_score,
                       int32_t* out_beam, int32_t* out_token, uint64_t* keys, float* sums, hipStream_t st)
{
    const int32_t parts = beam_parts(s.dtype, s.V);
    const dim3 grid(uint32_t(s.n_req) * uint32_t(s.beams) * uint32_t(parts));
    const bool at_once = grid.x <= 1024;
    if (s.dtype == LOBRA_F32)
        beam_part_kernel<float><<<grid, kThreads, 0, st>>>(s, static_cast<const float*>(logits), score, done, parts, at_once, keys, reinterpret_cast<float2*>(sums));
    else
        beam_part_kernel<uint16_t><<<grid, kThreads, 0, st>>>(s, static_cast<const uint16_t*>(logits), score, done, parts, at_once, keys, reinterpret_cast<float2*>(sums));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    beam_merge_kernel<<<dim3(uint32_t(s.n_req)), kThreads, 0, st>>>(s, score, done, done_token, parts, keys, reinterpret_cast<const float2*>(sums), out_score,
                                                                  out_beam, out_token);
    return hipGetLastError();
}

hipError_t beam_reorder(const lobra_beam_state* states, int32_t n_states, int32_t n_req, int32_t beams, const int32_t* parent, int64_t parent_ld,
                        const int32_t* used, hipStream_t st)
{
    for (int32_t i0 = 0; i0 < n_states;) {
        // runs of tensors whose rows are whole units of the same size, all in place or none
        StateTable tab;
        int32_t n = 0;
        int64_t most = 0;
        uint64_t unit = 0;
        bool in_place = false;
        for (; i0 < n_states && n < kStates; ++i0) {
            const lobra_beam_state& a = states[i0];
            const uint64_t bits = reinterpret_cast<uintptr_t>(a.src) | reinterpret_cast<uintptr_t>(a.dst) | uint64_t(a.row_bytes);
            const uint64_t own = bits % 16 == 0 ? 16 : bits % 4 == 0 ? 4 : bits % 2 == 0 ? 2 : 1;
            if (a.row_bytes == 0) continue;
            if (n > 0 && (own != unit || in_place != (a.src == a.dst))) break;
            unit = own;
            in_place = a.src == a.dst;
            tab.src[n] = static_cast<const char*>(a.src);
            tab.dst[n] = static_cast<char*>(a.dst);
            tab.row_bytes[n] = a.row_bytes;
            tab.unit[n] = a.unit_bytes;
            most = a.row_bytes > most ? a.row_bytes : most;
            ++n;
        }
        if (n == 0) break;
        // (a launch holds less than 2^32 threads)
        const int64_t all = (most / int64_t(unit) + 255) / 256;
        constexpr int64_t kBlocks = 1 << 17, kWorkgroups = 1 << 23;
        for (int64_t b = 0; b < all; b += kBlocks) {
            const int64_t blocks = all - b < kBlocks ? all - b : kBlocks, fit = kWorkgroups / (blocks * n), step = fit < 1 ? 1 : fit < 32768 ? fit : 32768;
            for (int64_t r = 0; r < n_req; r += step) {
                const dim3 grid(uint32_t(blocks), uint32_t(n_req - r < step ? n_req - r : step), uint32_t(n));
                const auto go = [&](auto u) {
                    typedef decltype(u) U;
                    return in_place ? launch_reorder<U, true>(tab, grid, b, int32_t(r), beams, parent, parent_ld, used, st)
                                    : launch_reorder<U, false>(tab, grid, b, int32_t(r), beams, parent, parent_ld, used, st);
                };
                const hipError_t e = unit == 16 ? go(u32x4{}) : unit == 4 ? go(uint32_t{}) : unit == 2 ? go(uint16_t{}) : go(uint8_t{});
                if (e != hipSuccess) return e;
            }
        }
    }
    return hipSuccess;
}

}  // namespace lobra
