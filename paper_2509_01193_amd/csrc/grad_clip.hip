// Norms of the tasks' gradients over many tensors, and the factors that clip them.
//     S_t = sum over the pieces of task t of g^2      norm_t = |grad_scale_t| sqrt(S_t)      clip_scale_t = grad_scale_t min(1, max_t / norm_t)
// Every piece of a tensor - consecutive elements of one task - is a workgroup's, which writes its sum; a second launch adds a task's sums in
// order.  The Adam step takes the factors as they are; where the clipped gradients themselves are wanted the second launch writes them too, or
// of many pieces a third.
// Squares and sums are fp64 (a conversion and one FMA per 4 bytes read): fp32 squares overflow from 1.8e19 on and vanish below 1e-23.
// Bound: memory, one read of all gradients (640 MB, 448 tensors: 95 us, 6.7 TB/s; through the caches 110; the sums' launch 4.7), with clipped
// gradients a second one and their write (470 MB, 448 x 64 x 4096: 73 without, 255 with, 1.41 GB at 5.5 TB/s).
#include "kernels.h"
#include "row_common.h"

namespace lobra {

using namespace rows;

namespace {

constexpr int NT = 256;

__device__ __forceinline__ double block_sum(double v, double* lds)
{
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) v += __shfl_xor(v, m);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    double s = 0.;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) s += lds[w];
    __syncthreads();
    return s;
}

// ONCE: the gradients are more than the caches hold and are read past them.
template <bool ONCE>
__global__ __launch_bounds__(NT)
void grad_squares_kernel(const GradPiece* __restrict__ pieces, double* __restrict__ partial)
{
    __shared__ double lds[NT / 64];
    const GradPiece pc = pieces[blockIdx.x];
    const RowShape sh = row_shape(pc.grad, pc.n);
    const f32x4* p = reinterpret_cast<const f32x4*>(pc.grad + sh.head);
    const int32_t t = threadIdx.x;
    double a[4] = {0., 0., 0., 0.};
    auto add = [&](f32x4 v) {
#pragma unroll
        for (int c = 0; c < 4; ++c) a[c] = fma(double(v[c]), double(v[c]), a[c]);
    };
    int32_t i = t;
    for (; i + 7 * NT < sh.packets; i += 8 * NT) {
        f32x4 v[8];
#pragma unroll
        for (int c = 0; c < 8; ++c) v[c] = ONCE ? __builtin_nontemporal_load(p + i + c * NT) : p[i + c * NT];
#pragma unroll
        for (int c = 0; c < 8; ++c) add(v[c]);
    }
    for (; i < sh.packets; i += NT) add(p[i]);
    if (t < sh.head + sh.tail) {
        const double v = pc.grad[t < sh.head ? t : t + 4 * sh.packets];
        a[0] = fma(v, v, a[0]);
    }
    const double s = block_sum((a[0] + a[1]) + (a[2] + a[3]), lds);
    if (t == 0) partial[blockIdx.x] = s;
}

struct Clip {
    const GradPiece* pieces;
    const double* partial;
    const int32_t* task_piece;                       // [n_tasks + 1]
    int32_t n_pieces, n_tasks;
    const float* max_norm;
    const float* grad_scale;
    bool joint;
};

// The norm of task t (joint: of all), by all threads of a workgroup.
__device__ __forceinline__ double task_norm(const Clip& a, int32_t t, double* lds)
{
    auto scale = [&](int32_t k) { return a.grad_scale ? double(a.grad_scale[k]) : 1.; };
    const int32_t end = a.joint ? a.n_pieces : a.task_piece[t + 1];
    double s = 0.;
    for (int32_t i = (a.joint ? 0 : a.task_piece[t]) + int32_t(threadIdx.x); i < end; i += NT) {
        const double f = a.joint ? scale(a.pieces[i].task) : 1.;
        s = fma(f * f, a.partial[i], s);
    }
    const double f = a.joint ? 1. : scale(t);
    return sqrt(f * f * block_sum(s, lds));
}
__device__ __forceinline__ bool is_finite(double norm) { return norm <= double(3.402823466e38f); }       // (a norm that fp32 does not hold is none)
__device__ __forceinline__ float clip_factor(const Clip& a, int32_t t, double norm)
{
    const float gs = a.grad_scale ? a.grad_scale[t] : 1.f, most = a.max_norm ? a.max_norm[t] : -1.f;
    if (!is_finite(norm)) return 0.f;
    return most >= 0.f && norm > double(most) ? float(double(gs) * (double(most) / norm)) : gs;
}
// What task t's caller is told, by one thread.
__device__ __forceinline__ void report(const Clip& a, int32_t t, double n, const int32_t* step, float* norm, float* clip_scale, int32_t* step_out,
                                       float* scale)
{
    const float c = clip_factor(a, t, n);
    if (scale) scale[t] = c;
    if (norm) norm[t] = float(n);
    if (clip_scale) clip_scale[t] = c;
    if (step_out) step_out[t] = is_finite(n) ? step[t] : 0;
}

// Workgroup t: task t's norm and factor.  joint: one workgroup, all tasks' (clip_scale may be grad_scale, which nobody else reads any more
// by then).
__global__ __launch_bounds__(NT)
void grad_factor_kernel(Clip a, const int32_t* step, float* __restrict__ norm, float* clip_scale, int32_t* step_out, float* __restrict__ scale)
{
    __shared__ double lds[NT / 64];
    const double n = task_norm(a, int32_t(blockIdx.x), lds);
    if (a.joint)
        for (int32_t t = threadIdx.x; t < a.n_tasks; t += NT) report(a, t, n, step, norm, clip_scale, step_out, scale);
    else if (threadIdx.x == 0)
        report(a, int32_t(blockIdx.x), n, step, norm, clip_scale, step_out, scale);
}

__device__ __forceinline__ void scale_piece(const GradPiece& pc, float f)
{
    const RowShape sh = row_shape(pc.grad, pc.n);           // (out is aligned as grad is)
    const f32x4* p = reinterpret_cast<const f32x4*>(pc.grad + sh.head);
    f32x4* q = reinterpret_cast<f32x4*>(pc.out + sh.head);
    const int32_t t = threadIdx.x;
    const f32x4 none = {0.f, 0.f, 0.f, 0.f};
    int32_t i = t;
    if (f == 0.f) {
        for (; i < sh.packets; i += NT) q[i] = none;
    } else if (!(f == 1.f && pc.out == pc.grad)) {
        for (; i + 3 * NT < sh.packets; i += 4 * NT) {
            f32x4 v[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) v[c] = p[i + c * NT];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
#pragma unroll
                for (int e = 0; e < 4; ++e) v[c][e] *= f;
                q[i + c * NT] = v[c];
            }
        }
        for (; i < sh.packets; i += NT) {
            f32x4 v = p[i];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] *= f;
            q[i] = v;
        }
    }
    if (t < sh.head + sh.tail) {
        const int32_t at = t < sh.head ? t : t + 4 * sh.packets;
        pc.out[at] = f == 0.f ? 0.f : pc.grad[at] * f;
    }
}

__global__ __launch_bounds__(NT)
void grad_scale_kernel(const GradPiece* __restrict__ pieces, const float* __restrict__ scale)
{
    const GradPiece pc = pieces[blockIdx.x];
    if (pc.out) scale_piece(pc, scale[pc.task]);
}

// Both in one launch, of few pieces: every workgroup of a piece works its task's factor out itself (all alike: in the same order); those
// behind them, one per task, report it.  Nothing that is written is read here (clip_scale is not grad_scale).
__global__ __launch_bounds__(NT)
void grad_factor_scale_kernel(Clip a, const int32_t* step, float* __restrict__ norm, float* __restrict__ clip_scale, int32_t* step_out)
{
    __shared__ double lds[NT / 64];
    const int32_t id = blockIdx.x;
    if (id >= a.n_pieces) {
        const int32_t t = id - a.n_pieces;
        const double n = task_norm(a, t, lds);
        if (threadIdx.x == 0) report(a, t, n, step, norm, clip_scale, step_out, nullptr);
        return;
    }
    const GradPiece pc = a.pieces[id];
    if (pc.out) scale_piece(pc, clip_factor(a, pc.task, task_norm(a, pc.task, lds)));
}

// Up to so many pieces (and tasks) the factors and the scaling are one launch, which reads n_pieces^2 / n_tasks partial sums (us, apart / in one:
// 2 x 64 x 4096 of 4 tasks 10.8 / 8.0, from a graph 7.4 / 6.3; 14 x 64 x 4096 of 8 tasks, 1796 partial sums, 10.7 / 9.8; 5826 of them 348 / 347).
constexpr int32_t kOneLaunchPieces = 2048;

}  // namespace

hipError_t grad_clip(const GradPiece* pieces, const int32_t* task_piece, int32_t n_pieces, int32_t n_tasks, bool any_out, bool once, const float* max_norm,
                     const float* grad_scale, const int32_t* step, float* norm, float* clip_scale, int32_t* step_out, bool joint,
                     double* partial, float* scale, hipStream_t st)
{
    if (n_pieces > 0) (once ? grad_squares_kernel<true> : grad_squares_kernel<false>)<<<dim3(uint32_t(n_pieces)), NT, 0, st>>>(pieces, partial);
    const Clip a{pieces, partial, task_piece, n_pieces, n_tasks, max_norm, grad_scale, joint};
    if (any_out && n_pieces + n_tasks <= kOneLaunchPieces && clip_scale != grad_scale) {
        grad_factor_scale_kernel<<<dim3(uint32_t(n_pieces + n_tasks)), NT, 0, st>>>(a, step, norm, clip_scale, step_out);
    } else {
        grad_factor_kernel<<<dim3(joint ? 1u : uint32_t(n_tasks)), NT, 0, st>>>(a, step, norm, clip_scale, step_out, scale);
        if (any_out && n_pieces > 0) grad_scale_kernel<<<dim3(uint32_t(n_pieces)), NT, 0, st>>>(pieces, scale);
    }
    return hipGetLastError();
}

}  // namespace lobra
