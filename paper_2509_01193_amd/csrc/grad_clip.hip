// Norms of the tasks' gradients over many tensors, and the factors that clip them.
//     S_t = sum over the pieces of task t of g^2      norm_t = |grad_scale_t| sqrt(S_t)      clip_scale_t = grad_scale_t min(1, max_t / norm_t)
// Every piece of a tensor - consecutive elements of one task - is a workgroup's, which writes its sum; a second launch adds a task's sums in
// order.  Where the clipped gradients themselves are wanted a third one writes them; the Adam step takes the factors instead.
// Squares and sums are fp64 (a conversion and one FMA per 4 bytes read): fp32 squares overflow from 1.8e19 on and vanish below 1e-23.
// Bound: memory, one read of all gradients (640 MB, 448 tensors: 95 us, 6.7 TB/s; through the caches 110; the sums' launch 4.7).
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

// Workgroup t: task t's sum, norm and factor.  joint: one workgroup, the sum of all (clip_scale may be grad_scale, which nobody
// else reads any more by then).
__global__ __launch_bounds__(NT)
void grad_factor_kernel(const GradPiece* __restrict__ pieces, const double* __restrict__ partial, const int32_t* __restrict__ task_piece, int32_t n_tasks,
                        const float* __restrict__ max_norm, const float* grad_scale, const int32_t* step, float* __restrict__ norm, float* clip_scale,
                        int32_t* step_out, int joint, float* __restrict__ scale)
{
    __shared__ double lds[NT / 64];
    auto factor = [&](int32_t k) { return grad_scale ? double(grad_scale[k]) : 1.; };
    const int32_t own = joint ? 0 : int32_t(blockIdx.x), end = task_piece[joint ? n_tasks : own + 1];
    double s = 0.;
    for (int32_t i = task_piece[own] + int32_t(threadIdx.x); i < end; i += NT) {
        const double f = joint ? factor(pieces[i].task) : 1.;
        s = fma(f * f, partial[i], s);
    }
    const double f = joint ? 1. : factor(own), square = f * f * block_sum(s, lds);
    if (!joint && threadIdx.x != 0) return;
    const double n = sqrt(square);
    const bool finite = n <= double(3.402823466e38f);       // (a norm that fp32 does not hold is none)
    for (int32_t t = joint ? int32_t(threadIdx.x) : int32_t(blockIdx.x); t < n_tasks; t += joint ? NT : n_tasks) {
        const float gs = grad_scale ? grad_scale[t] : 1.f, most = max_norm ? max_norm[t] : -1.f;
        float c = gs;
        if (most >= 0.f && n > double(most)) c = float(double(gs) * (double(most) / n));
        if (!finite) c = 0.f;
        scale[t] = c;
        if (norm) norm[t] = float(n);
        if (clip_scale) clip_scale[t] = c;
        if (step_out) step_out[t] = finite ? step[t] : 0;
    }
}

__global__ __launch_bounds__(NT)
void grad_scale_kernel(const GradPiece* __restrict__ pieces, const float* __restrict__ scale)
{
    const GradPiece pc = pieces[blockIdx.x];
    if (!pc.out) return;
    const float f = scale[pc.task];
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

}  // namespace

hipError_t grad_clip(const GradPiece* pieces, const int32_t* task_piece, int32_t n_pieces, int32_t n_tasks, bool any_out, bool once, const float* max_norm,
                     const float* grad_scale, const int32_t* step, float* norm, float* clip_scale, int32_t* step_out, bool joint,
                     double* partial, float* scale, hipStream_t st)
{
    if (n_pieces > 0) (once ? grad_squares_kernel<true> : grad_squares_kernel<false>)<<<dim3(uint32_t(n_pieces)), NT, 0, st>>>(pieces, partial);
    grad_factor_kernel<<<dim3(joint ? 1u : uint32_t(n_tasks)), NT, 0, st>>>(pieces, partial, task_piece, n_tasks, max_norm, grad_scale, step, norm, clip_scale, step_out,
                                                              joint ? 1 : 0, scale);
    if (any_out && n_pieces > 0) grad_scale_kernel<<<dim3(uint32_t(n_pieces)), NT, 0, st>>>(pieces, scale);
    return hipGetLastError();
}

}  // namespace lobra
