// A step of beam search: the best continuations of every request over its beams and the vocabulary, and the reordering of what is kept per
// sequence.
//
// Selection.  Beam b of score s continued by token j has the value (s - lse_b) + z_j, lse_b = ln sum exp(z_b).  A beam's own best continuations
// are its largest logits, so a part of a row hands on its n largest logits, the lowest index first among equals, and its sum; a workgroup per
// request then makes lse and values, in fp64, and orders what is left.  A logit is read once: a part's 8192 stay in registers from the sum to
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
constexpr int kPart = 8192;               // elements of a row to a workgroup
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
// 64 groups of four threads have a maximum each; the n-th largest of these has at least n logits at or above it, which go on a list and find
// their place there by counting who is larger.  Parts with more of them than the list holds (equal logits) take the largest n times over.
template <typename E>
__global__ __launch_bounds__(kThreads)
void beam_part_kernel(BeamShape sh, const E* __restrict__ logits, const float* __restrict__ score, const int32_t* __restrict__ done, int32_t parts,
                      uint64_t* __restrict__ keys, float2* __restrict__ sums)
{
    constexpr int N = Packet<E>::N, U = kPart / (kThreads * N), W = kThreads / 64;
    __shared__ uint64_t list[kList];
    __shared__ float group_max[64];
    __shared__ Stat stat[W];
    __shared__ int32_t count;
    const int32_t row = int32_t(blockIdx.x) / parts, part = int32_t(blockIdx.x) - row * parts;
    if (!looked_at(score[row], done, size_t(row))) return;
    const int32_t tid = threadIdx.x, lane = tid & 63, base = part * kPart, n = sh.n_out;
    const int32_t len = min(kPart, sh.V - base);
    const E* p = logits + size_t(row) * size_t(sh.ld) + base;
    u32x4 q[U];
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
    if (tid == 0) count = 0;
    Stat a{-INFINITY, 0.f, 0.f};
    float most[U];                                   // of each packet
    {
        float z[U * N];
#pragma unroll
        for (int c = 0; c < U; ++c) {
#pragma unroll
            for (int e = 0; e < N; ++e) z[c * N + e] = Packet<E>::element(q[c], e);
            most[c] = z[c * N];
#pragma unroll
            for (int e = 1; e < N; ++e) most[c] = fmaxf(most[c], z[c * N + e]);
        }
        take<false>(a, z, kLog2e);
    }
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
    // packet by packet, of those in which any lane of the wave has one
#pragma unroll
    for (int c = 0; c < U; ++c) {
        if (!(most[c] > -INFINITY && float_order(most[c]) >= tau)) continue;
        uint32_t hits = 0;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float z = Packet<E>::element(q[c], e);
            hits |= z > -INFINITY && float_order(z) >= tau ? 1u << e : 0u;
        }
        for (; hits; hits &= hits - 1) {
            const int e = __builtin_ctz(hits);
            float z = 0.f;
#pragma unroll
            for (int i = 0; i < N; ++i) z = i == e ? Packet<E>::element(q[c], i) : z;
            const int32_t o = atomicAdd(&count, 1);
            if (o < kList) list[o] = order_key(z, base + (c * kThreads + tid) * N + e);
        }
    }
    __syncthreads();
    const int32_t found = count;
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
#pragma unroll
        for (int c = 0; c < U; ++c)
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float z = Packet<E>::element(q[c], e);
                const uint64_t key = z > -INFINITY ? order_key(z, base + (c * kThreads + tid) * N + e) : 0;
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

// A continuation: larger first, then the lower beam, then the lower token.
struct Next {
    double v;
    int32_t beam, token;
};
__device__ __forceinline__ bool in_front(const Next& a, const Next& b)
{
    if (a.v != b.v) return a.v > b.v;
    return a.beam != b.beam ? a.beam < b.beam : a.token < b.token;
}

// A workgroup per request.
__global__ __launch_bounds__(kThreads)
void beam_merge_kernel(BeamShape sh, const float* score, const int32_t* __restrict__ done, int32_t done_token, int32_t parts,
                       const uint64_t* __restrict__ keys, const float2* __restrict__ sums, float* out_score, int32_t* __restrict__ out_beam,
                       int32_t* __restrict__ out_token)
{
    constexpr int W = kThreads / 64;
    __shared__ double offset[LOBRA_MAX_TOP];         // s - lse; -inf: no continuations
    __shared__ int32_t kind[LOBRA_MAX_TOP];          // 0: none, 1: its logits, 2: done
    __shared__ Next list[kList];
    __shared__ uint32_t group_max[64];
    __shared__ int32_t count;
    const int32_t tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = sh.n_out;
    const size_t row0 = size_t(blockIdx.x) * sh.beams;
    for (int32_t b = wave; b < sh.beams; b += W) {   // a wave per beam
        const float s = score[row0 + b];
        if (!looked_at(s, done, row0 + b)) {
            if (lane == 0) kind[b] = s > -INFINITY ? 2 : 0, offset[b] = double(s);
            continue;
        }
        const float2* part = sums + (row0 + b) * parts;
        float m = -INFINITY;
        for (int32_t i = lane; i < parts; i += 64) m = fmaxf(m, part[i].x);
        m = wave_max(m);
        double sum = 0;
        for (int32_t i = lane; i < parts; i += 64) {
            const float2 v = part[i];
            sum += v.y > 0.f ? double(v.y) * exp(double(v.x) - double(m)) : double(v.y);        // (NaN stays NaN)
        }
#pragma unroll
        for (int x = 32; x > 0; x >>= 1) sum += __shfl_xor(sum, x);
        const double l = double(m) + log(sum);
        if (lane == 0) kind[b] = l > -INFINITY && l < INFINITY ? 1 : 0, offset[b] = double(s) - l;
    }
    if (tid == 0) count = 0;
    __syncthreads();
    const int32_t per = parts * n, total = sh.beams * per;
    const uint64_t* const k0 = keys + row0 * per;
    auto value = [&](int32_t i, Next& c) {           // continuation i, false: there is none
        c.beam = i / per;
        const int32_t j = i - c.beam * per;
        if (kind[c.beam] != 1) {
            c.v = offset[c.beam];
            c.token = done_token;
            return kind[c.beam] == 2 && j == 0;
        }
        const uint64_t key = k0[i];
        c.v = offset[c.beam] + double(key_value(key));
        c.token = key_index(key);
        return key != 0;
    };
    // (as in a part: values by their order in fp32, rounded down, so that none is above what it stands for)
    auto order = [](double v) { return float_order(__double2float_rd(v)); };
    uint32_t best = 0;
    for (int32_t i = tid; i < total; i += kThreads) {
        Next c;
        if (value(i, c)) best = max(best, order(c.v));
    }
    uint32_t g = best;
#pragma unroll
    for (int x = 1; x < kThreads / 64; x <<= 1) g = max(g, uint32_t(__shfl_xor(int(g), x)));
    if (tid % (kThreads / 64) == 0) group_max[tid / (kThreads / 64)] = g;
    __syncthreads();
    const uint32_t tau = reached_by(group_max[lane], n);
    if (best >= tau && best > 0)
        for (int32_t i = tid; i < total; i += kThreads) {
            Next c;
            if (value(i, c) && order(c.v) >= tau) {
                const int32_t o = atomicAdd(&count, 1);
                if (o < kList) list[o] = c;
            }
        }
    __syncthreads();
    const int32_t found = count;
    auto write = [&](int32_t place, const Next& c) {
        const size_t o = size_t(blockIdx.x) * n + place;
        out_score[o] = float(c.v);
        out_beam[o] = c.beam;
        out_token[o] = c.token;
    };
    const Next nobody{-INFINITY, -1, -1};
    if (found <= kList) {
        for (int32_t c = tid; c < found; c += kThreads) {
            const Next mine = list[c];
            int32_t place = 0;
            for (int32_t o = 0; o < found; ++o) place += in_front(list[o], mine) ? 1 : 0;
            if (place < n) write(place, mine);
        }
        if (tid >= found && tid < n) write(tid, nobody);
        return;
    }
    // more of equal value than the list holds: the best n times over
    Next last{INFINITY, -1, -1};
    for (int32_t r = 0; r < n; ++r) {
        Next top = nobody;
        for (int32_t i = tid; i < total; i += kThreads) {
            Next c;
            if (value(i, c) && in_front(last, c) && (top.beam < 0 || in_front(c, top))) top = c;
        }
#pragma unroll
        for (int x = 32; x > 0; x >>= 1) {
            const Next o{__shfl_xor(top.v, x), __shfl_xor(top.beam, x), __shfl_xor(top.token, x)};
            if (o.beam >= 0 && (top.beam < 0 || in_front(o, top))) top = o;
        }
        __syncthreads();
        if (lane == 0) list[wave] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < W; ++w)
            if (list[w].beam >= 0 && (top.beam < 0 || in_front(list[w], top))) top = list[w];
        if (tid == 0) write(r, top);
        last = top;
    }
}

// ---- reordering ---------------------------------------------------------------------------------------------------------------
constexpr int kStates = 64;                          // tensors of a launch
struct StateTable {
    const char* src[kStates];
    char* dst[kStates];
    int64_t row_bytes[kStates], unit[kStates];
};
static_assert(sizeof(StateTable) + 64 <= 4096, "the arguments of a launch");

// Units of type U; blockIdx = (columns of a row, request, tensor).  B: at least the beams.
template <typename U, int B>
__global__ __launch_bounds__(256)
void beam_reorder_kernel(StateTable tab, int32_t first_req, int32_t beams, const int32_t* __restrict__ parent, int64_t parent_ld,
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
    const int32_t* const from = parent + req * parent_ld;
    int32_t of[B];
#pragma unroll
    for (int i = 0; i < B; ++i) of[i] = i < beams ? from[i] : -1;
    const bool in_place = tab.src[s] == tab.dst[s];
    const char* const src = tab.src[s] + req * beams * row;
    char* const dst = tab.dst[s] + req * beams * row;
    for (int64_t at = (int64_t(blockIdx.x) * 256 + threadIdx.x) * int64_t(sizeof(U)); at < bytes; at += int64_t(gridDim.x) * 256 * int64_t(sizeof(U))) {
        U v[B];
#pragma unroll
        for (int i = 0; i < B; ++i)
            if (of[i] >= 0 && of[i] < beams && !(in_place && of[i] == i)) v[i] = *reinterpret_cast<const U*>(src + of[i] * row + at);
#pragma unroll
        for (int i = 0; i < B; ++i) {
            if (of[i] < 0 || of[i] >= beams || (in_place && of[i] == i)) continue;
            if (sizeof(U) == 1 || at + int64_t(sizeof(U)) <= bytes) {
                *reinterpret_cast<U*>(dst + i * row + at) = v[i];
            } else {                                 // the end of what is used lies within the unit (a row itself is whole units)
                const unsigned char* b = reinterpret_cast<const unsigned char*>(&v[i]);
#pragma unroll
                for (int e = 0; e < int(sizeof(U)); ++e)
                    if (at + e < bytes) dst[i * row + at + e] = char(b[e]);
            }
        }
    }
}

template <typename U>
hipError_t launch_reorder(const StateTable& tab, dim3 grid, int32_t first_req, int32_t beams, const int32_t* parent, int64_t parent_ld, const int32_t* used,
                          hipStream_t st)
{
    if (beams <= 2) beam_reorder_kernel<U, 2><<<grid, 256, 0, st>>>(tab, first_req, beams, parent, parent_ld, used);
    else if (beams <= 4) beam_reorder_kernel<U, 4><<<grid, 256, 0, st>>>(tab, first_req, beams, parent, parent_ld, used);
    else if (beams <= 8) beam_reorder_kernel<U, 8><<<grid, 256, 0, st>>>(tab, first_req, beams, parent, parent_ld, used);
    else if (beams <= 16) beam_reorder_kernel<U, 16><<<grid, 256, 0, st>>>(tab, first_req, beams, parent, parent_ld, used);
    else beam_reorder_kernel<U, 32><<<grid, 256, 0, st>>>(tab, first_req, beams, parent, parent_ld, used);
    return hipGetLastError();
}

}  // namespace

int32_t beam_parts(int32_t V) { return (V + kPart - 1) / kPart; }

hipError_t beam_select(const BeamShape& s, const void* logits, const float* score, const int32_t* done, int32_t done_token, float* out_score,
                       int32_t* out_beam, int32_t* out_token, uint64_t* keys, float* sums, hipStream_t st)
{
    const int32_t parts = beam_parts(s.V);
    const dim3 grid(uint32_t(s.n_req) * uint32_t(s.beams) * uint32_t(parts));
    if (s.dtype == LOBRA_F32)
        beam_part_kernel<float><<<grid, kThreads, 0, st>>>(s, static_cast<const float*>(logits), score, done, parts, keys, reinterpret_cast<float2*>(sums));
    else
        beam_part_kernel<uint16_t><<<grid, kThreads, 0, st>>>(s, static_cast<const uint16_t*>(logits), score, done, parts, keys, reinterpret_cast<float2*>(sums));
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
        // runs of tensors whose rows are whole units of the same size
        StateTable tab;
        int32_t n = 0;
        int64_t most = 0;
        uint64_t unit = 0;
        for (; i0 < n_states && n < kStates; ++i0) {
            const lobra_beam_state& a = states[i0];
            const uint64_t bits = reinterpret_cast<uintptr_t>(a.src) | reinterpret_cast<uintptr_t>(a.dst) | uint64_t(a.row_bytes);
            const uint64_t own = bits % 16 == 0 ? 16 : bits % 4 == 0 ? 4 : 1;
            if (a.row_bytes == 0) continue;
            if (n > 0 && own != unit) break;
            unit = own;
            tab.src[n] = static_cast<const char*>(a.src);
            tab.dst[n] = static_cast<char*>(a.dst);
            tab.row_bytes[n] = a.row_bytes;
            tab.unit[n] = a.unit_bytes;
            most = a.row_bytes > most ? a.row_bytes : most;
            ++n;
        }
        if (n == 0) break;
        const int64_t units = most / int64_t(unit);
        constexpr int32_t kRequests = 32768;         // of a launch
        for (int32_t r = 0; r < n_req; r += kRequests) {
            const uint32_t reqs = uint32_t(n_req - r < kRequests ? n_req - r : kRequests);
            // some 16 workgroups per compute unit and no more: what is left of a row they take in strides
            const int64_t all = (units + 255) / 256, wanted = int64_t(4096) / (int64_t(reqs) * n) + 1;
            const dim3 grid(uint32_t(all < wanted ? all : wanted), reqs, uint32_t(n));
            const hipError_t e = unit == 16 ? launch_reorder<u32x4>(tab, grid, r, beams, parent, parent_ld, used, st)
                                 : unit == 4 ? launch_reorder<uint32_t>(tab, grid, r, beams, parent, parent_ld, used, st)
                                             : launch_reorder<uint8_t>(tab, grid, r, beams, parent, parent_ld, used, st);
            if (e != hipSuccess) return e;
        }
    }
    return hipSuccess;
}

}  // namespace lobra
