// extern "C" entry points of the steps around the LoRA linears: the gated feed-forward block, the norms around a residual block, log
// probabilities, gradient norms and clipping.  Argument checks on the host, then launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <new>
#include <vector>

#include "api_common.h"

using namespace lobra;

namespace {

inline bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
inline size_t align256(size_t v) { return (v + 255) / 256 * 256; }

// ---- gated feed-forward block ------------------------------------------------------------------------------------------------

// The plan is one of gate and up projection, and the activation is known.
lobra_status gated_check(const Plan& p, int32_t act)
{
    if (p.n_proj != 2 || (act != LOBRA_ACT_SILU && act != LOBRA_ACT_GELU_TANH)) return LOBRA_ERR_SHAPE;
    return LOBRA_OK;
}

// Bytes in front of the layer's own workspace for [g | u] where the caller does not keep it.
size_t gated_scratch(const Plan& p)
{
    return align256(size_t(p.desc.T) * size_t(p.desc.d_out) * (p.desc.dtype == LOBRA_F32 ? 4 : 2));
}

// Few tokens (decoding) have kernels of their own, which keep no projected activations.
bool gated_is_skinny(const Plan& p) { return p.desc.T > 0 && p.desc.T <= (p.mfma ? kSkinnyTokens : p.desc.dtype == LOBRA_F32 ? kFewTokens : 0); }
size_t gated_skinny_bytes(const Plan& p)
{
    return (p.mfma ? gated_skinny_ws_bytes : gated_few_ws_bytes)(p.desc.T, p.desc.d_in, p.dg, p.tb.empty() ? 0 : p.r_max);
}

// (The forms below that project in a launch of their own hand the projected activations s_t A_t x on as the layer does, rounded to bf16: operands of
// the matrix instructions in the up projection and in dB.  The few-token kernels keep them in fp32.)
// A layer product whose K is split leaves its fp32 sums to the activation, if the workspace has room for those of both projections.
size_t gated_sums_bytes(const Plan& p) { return p.mfma && p.desc.T > 0 ? p.fwd_part * (p.fwd_group > 0 ? 1 : 2) : 0; }

// ---- norms ----------------------------------------------------------------------------------------------------------------

lobra_status block_norm_check(const Plan& p, const lobra_block_norm_config* cfg)
{
    if (!cfg) return LOBRA_ERR_NULL;
    if (!(cfg->eps >= 0.f) || !std::isfinite(cfg->eps) || !std::isfinite(cfg->alpha) || p.desc.d_in > LOBRA_MAX_NORM_WIDTH) return LOBRA_ERR_SHAPE;
    return LOBRA_OK;
}

// ---- log probabilities --------------------------------------------------------------------------------------------------------

lobra_status logprob_shape(const lobra_logprob_desc* d, LogprobShape* s)
{
    if (!d) return LOBRA_ERR_NULL;
    if (d->dtype != LOBRA_F32 && d->dtype != LOBRA_BF16) return LOBRA_ERR_DTYPE;
    const int64_t ld = d->ld == 0 ? d->V : d->ld;
    if (d->V < 1 || d->V > LOBRA_MAX_VOCAB || d->T < 0 || d->T >= (int64_t(1) << 31) || ld < d->V || d->top_k < 0 || d->top_k > LOBRA_MAX_TOP)
        return LOBRA_ERR_SHAPE;
    if (d->T > 0 && ld >= (int64_t(1) << 60) / d->T) return LOBRA_ERR_SHAPE;
    *s = LogprobShape{d->dtype, d->V, d->top_k, d->T, ld};
    return LOBRA_OK;
}

}  // namespace

// The tensors of a set, cut into pieces of one task each.
struct lobra_grad_set {
    std::vector<unsigned char> blob;         // what the device has: the pieces, then task_piece [n_tasks + 1]
    size_t o_task_piece = 0;
    int32_t n_pieces = 0, n_tasks = 0;
    bool any_out = false, once = false;      // once: more than the 256 MB infinity cache holds
    int device = -1;
    void* dev = nullptr;
    bool owns = false;
};

namespace {

// Elements of a piece: some eight workgroups per compute unit, of a few loads a thread at least, and not so large that the last
// ones are alone.
int64_t piece_elements(int64_t total)
{
    const int64_t n = (total / 2048 + 1023) / 1024 * 1024;
    return std::min<int64_t>(std::max<int64_t>(n, 2048), 32768);
}

lobra_status make_set(const lobra_grad_tensor* tensors, int32_t n_tensors, int32_t n_tasks, lobra_grad_set** out)
{
    if (n_tensors < 0 || n_tasks < 0 || n_tasks >= 1 << 23) return LOBRA_ERR_SHAPE;
    if (n_tensors > 0 && !tensors) return LOBRA_ERR_NULL;
    int64_t total = 0;
    for (int32_t i = 0; i < n_tensors; ++i) {
        const lobra_grad_tensor& g = tensors[i];
        if (!g.rank_off) return LOBRA_ERR_NULL;
        if (g.D < 1 || g.D > LOBRA_MAX_WIDTH) return LOBRA_ERR_SHAPE;
        if (g.rank_off[0] != 0) return LOBRA_ERR_RANK;
        for (int32_t t = 0; t < n_tasks; ++t)
            if (g.rank_off[t + 1] < g.rank_off[t]) return LOBRA_ERR_RANK;
        const int64_t n = int64_t(g.rank_off[n_tasks]) * g.D;
        if (n >= int64_t(1) << 40) return LOBRA_ERR_SHAPE;
        if (n > 0 && !g.grad) return LOBRA_ERR_NULL;
        if (!aligned16(g.grad) || !aligned16(g.out)) return LOBRA_ERR_ALIGN;
        if ((total += n) >= int64_t(1) << 56) return LOBRA_ERR_SHAPE;
    }
    const int64_t per = piece_elements(total);
    if (total / per + int64_t(n_tensors) * n_tasks >= int64_t(1) << 23) return LOBRA_ERR_SHAPE;     // (a launch holds less than 2^32 threads)
    lobra_grad_set* s = new (std::nothrow) lobra_grad_set();
    if (!s) return LOBRA_ERR_NOMEM;
    s->once = size_t(total) * sizeof(float) > (size_t(256) << 20);
    try {
        std::vector<GradPiece> pieces;
        std::vector<int32_t> task_piece(size_t(n_tasks) + 1, 0);
        for (int32_t t = 0; t < n_tasks; ++t) {
            for (int32_t i = 0; i < n_tensors; ++i) {
                const lobra_grad_tensor& g = tensors[i];
                const int64_t end = int64_t(g.rank_off[t + 1]) * g.D;
                for (int64_t at = int64_t(g.rank_off[t]) * g.D; at < end;) {
                    const int64_t next = std::min(end, (at / per + 1) * per);       // (pieces begin at multiples of `per`: aligned)
                    pieces.push_back(GradPiece{g.grad + at, g.out ? g.out + at : nullptr, int32_t(next - at), t});
                    at = next;
                }
                s->any_out = s->any_out || g.out;
            }
            task_piece[size_t(t) + 1] = int32_t(pieces.size());
        }
        s->n_pieces = int32_t(pieces.size());
        s->n_tasks = n_tasks;
        s->o_task_piece = pieces.size() * sizeof(GradPiece);
        s->blob.resize(s->o_task_piece + task_piece.size() * sizeof(int32_t));
        if (!pieces.empty()) std::memcpy(s->blob.data(), pieces.data(), s->o_task_piece);
        std::memcpy(s->blob.data() + s->o_task_piece, task_piece.data(), task_piece.size() * sizeof(int32_t));
    } catch (const std::bad_alloc&) {
        delete s;
        return LOBRA_ERR_NOMEM;
    }
    *out = s;
    return LOBRA_OK;
}

// Partial sums, then the tasks' factors.
size_t clip_ws_bytes(const lobra_grad_set& s)
{
    return align256(size_t(s.n_pieces) * sizeof(double)) + size_t(s.n_tasks) * sizeof(float);
}

}  // namespace

extern "C" {

lobra_status lobra_mlora_gated_workspace_bytes(const lobra_mlora_plan* plan, int32_t save_gu, size_t* fwd_bytes)
{
    if (!plan) return LOBRA_ERR_PLAN;
    if (!fwd_bytes) return LOBRA_ERR_NULL;
    if (plan->n_proj != 2) return LOBRA_ERR_SHAPE;
    *fwd_bytes = (save_gu || plan->gated_persistent ? 0 : gated_scratch(*plan)) + plan->fwd_ws_bytes;
    if (gated_is_skinny(*plan)) *fwd_bytes = std::max(*fwd_bytes, gated_skinny_bytes(*plan));
    if (!plan->gated_persistent && gated_sums_bytes(*plan) > 0) *fwd_bytes = std::max(*fwd_bytes, gated_sums_bytes(*plan) + plan->p_layout.total);
    return LOBRA_OK;
}

lobra_status lobra_mlora_gated_fwd(const lobra_mlora_plan* plan, int32_t act, const void* x, const void* W, const void* A, const void* B,
                                   const float* s, void* gu, void* h, void* h_save, void* ws, size_t ws_bytes, void* hip_stream)
{
    lobra_status rs = runnable(plan);
    if (rs != LOBRA_OK) return rs;
    const Plan& p = *plan;
    if ((rs = gated_check(p, act)) != LOBRA_OK) return rs;
    if (p.desc.T == 0) return LOBRA_OK;
    if (!h) return LOBRA_ERR_NULL;
    if (!aligned16(h) || !aligned16(gu) || !aligned16(ws)) return LOBRA_ERR_ALIGN;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const bool adapters = !p.tb.empty();
    if (gated_is_skinny(p) && !h_save) {
        if (!x || !W || (adapters && (!A || !B || !s))) return LOBRA_ERR_NULL;
        if (!aligned16(x) || !aligned16(W) || !aligned16(A) || !aligned16(B)) return LOBRA_ERR_ALIGN;
        if (!ws || ws_bytes < gated_skinny_bytes(p)) return LOBRA_ERR_WORKSPACE;
        PlanDev pd = device_view(p);
        if (!adapters) pd.r_max = 0;
        if (p.mfma) {
            LOBRA_LAUNCH(p, st, LOBRA_K_SHRINK_GEMM, gated_skinny_product(pd, x, W, A, s, ws, adapters, st));
            LOBRA_LAUNCH(p, st, LOBRA_K_GATED, gated_skinny_finish(pd, act, B, ws, adapters, gu, h, st));
        } else {
            const auto floats = [](const void* q) { return static_cast<const float*>(q); };
            LOBRA_LAUNCH(p, st, LOBRA_K_SHRINK_GEMM, gated_few_product(pd, floats(x), floats(W), floats(A), s, ws, adapters, st));
            LOBRA_LAUNCH(p, st, LOBRA_K_GATED, gated_few_finish(pd, act, floats(B), ws, adapters, static_cast<float*>(gu), static_cast<float*>(h), st));
        }
        return LOBRA_OK;
    }
    if (p.gated_persistent) {
        if ((rs = plan_fwd_check(p, x, W, A, B, s, h, h_save, ws, ws_bytes)) != LOBRA_OK) return rs;
        const PlanDev pd = device_view(p);
        char* const hb = static_cast<char*>(h_save ? h_save : ws);
        if (adapters)
            LOBRA_LAUNCH(p, st, LOBRA_K_SHRINK,
                         shrink_mfma(pd, x, A, s, hb + p.p_layout.p_tok, hb + p.p_layout.p_blk, pd.d_in, pd.d_in, 1, 0, st));
        LOBRA_LAUNCH(p, st, LOBRA_K_GATED, gemm_persistent_gated(pd, act, x, W, adapters ? hb + p.p_layout.p_tok : nullptr, B, gu, h, st));
        return LOBRA_OK;
    }
    const size_t sums = gated_sums_bytes(p);
    if (sums > 0 && ws && ws_bytes >= sums + (h_save ? 0 : p.p_layout.total)) {
        if ((rs = plan_fwd_check(p, x, W, A, B, s, h, h_save, ws, ws_bytes)) != LOBRA_OK) return rs;
        const PlanDev pd = device_view(p);
        char* const hb = h_save ? static_cast<char*>(h_save) : static_cast<char*>(ws) + sums;
        const char* const P = adapters ? hb + p.p_layout.p_tok : nullptr;
        if (adapters)
            LOBRA_LAUNCH(p, st, LOBRA_K_SHRINK, shrink_mfma(pd, x, A, s, hb + p.p_layout.p_tok, hb + p.p_layout.p_blk, pd.d_in, pd.d_in, 1, 0, st));
        const int32_t N = p.fwd_group > 0 ? pd.d_out : pd.dg;
        const int32_t n = choose_gemm(pd.T, pd.d_in, N, p.fwd_group, adapters ? pd.nseg : 0, pd.r_max / 2, std::min(p.fwd_part, kMaxPartBytes)).splits +
                          (adapters ? 1 : 0);
        float *const g = static_cast<float*>(ws), *const u = p.fwd_group > 0 ? g + pd.dg : reinterpret_cast<float*>(static_cast<char*>(ws) + p.fwd_part);
        if (p.fwd_group > 0)
            LOBRA_LAUNCH(p, st, LOBRA_K_GEMM, gemm_mfma(pd, false, x, W, P, B, nullptr, pd.d_in, N, pd.d_out, st, pd.d_out, 2, -1, g, p.fwd_part));
        else
            for (int32_t j = 0; j < 2; ++j)
                LOBRA_LAUNCH(p, st, LOBRA_K_GEMM,
                             gemm_mfma(pd, false, x, static_cast<const char*>(W) + size_t(j) * pd.dg * 2, P, B, nullptr, pd.d_in, N, pd.d_out, st, pd.d_out, 2,
                                       j, j == 0 ? g : u, p.fwd_part));
        LOBRA_LAUNCH(p, st, LOBRA_K_GATED, gated_sums(act, pd.T, pd.dg, g, u, N, int64_t(pd.T) * N, n, gu, h, st));
        return LOBRA_OK;
    }
    const size_t own = gu ? 0 : gated_scratch(p);
    if (own > 0 && (!ws || ws_bytes < own)) return LOBRA_ERR_WORKSPACE;
    void* const y = gu ? gu : ws;
    char* const rest = ws ? static_cast<char*>(ws) + own : nullptr;
    if ((rs = lobra_mlora_plan_fwd(plan, x, W, A, B, s, y, h_save, rest, ws_bytes - own, hip_stream)) != LOBRA_OK) return rs;
    LOBRA_LAUNCH(p, st, LOBRA_K_GATED, gated_activate(p.desc.dtype, act, p.desc.T, p.dg, y, h, st));
    return LOBRA_OK;
}

lobra_status lobra_mlora_gated_bwd(const lobra_mlora_plan* plan, int32_t act, const void* x, const void* W, const void* A, const void* B,
                                   const float* s, const void* gu, const void* dh, const void* h_saved, void* dgu, void* dx, float* dA, float* dB,
                                   uint32_t flags, void* ws, size_t ws_bytes, void* hip_stream)
{
    lobra_status rs = runnable(plan);
    if (rs != LOBRA_OK) return rs;
    const Plan& p = *plan;
    if ((rs = gated_check(p, act)) != LOBRA_OK) return rs;
    if (p.desc.T > 0) {
        if (!gu || !dh || !dgu) return LOBRA_ERR_NULL;
        if (!aligned16(gu) || !aligned16(dh) || !aligned16(dgu)) return LOBRA_ERR_ALIGN;
    }
    if ((rs = plan_bwd_check(p, x, W, A, B, s, dgu, h_saved, dx, dA, dB, flags, ws, ws_bytes)) != LOBRA_OK) return rs;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (p.desc.T > 0) LOBRA_LAUNCH(p, st, LOBRA_K_GATED, gated_derive(p.desc.dtype, act, p.desc.T, p.dg, gu, dh, dgu, st));
    return lobra_mlora_plan_bwd(plan, x, W, A, B, s, dgu, h_saved, dx, dA, dB, flags, ws, ws_bytes, hip_stream);
}

lobra_status lobra_mlora_block_norm_workspace_bytes(const lobra_mlora_plan* plan, size_t* bwd_bytes)
{
    if (!plan) return LOBRA_ERR_PLAN;
    if (!bwd_bytes) return LOBRA_ERR_NULL;
    if (plan->desc.d_in > LOBRA_MAX_NORM_WIDTH) return LOBRA_ERR_SHAPE;
    *bwd_bytes = block_norm_part_bytes(plan->desc.T, plan->desc.d_in, int32_t(plan->cseg_task.size()), plan->desc.dtype);
    return LOBRA_OK;
}

lobra_status lobra_mlora_block_norm_fwd(const lobra_mlora_plan* plan, const lobra_block_norm_config* cfg, const void* r, const void* b,
                                        const void* w_post, const void* gate, const void* w_pre, void* r_out, void* x, float* rstd_post,
                                        float* rstd_pre, void* hip_stream)
{
    lobra_status rs = runnable(plan);
    if (rs != LOBRA_OK) return rs;
    const Plan& p = *plan;
    if ((rs = block_norm_check(p, cfg)) != LOBRA_OK) return rs;
    if (p.desc.T == 0) return LOBRA_OK;
    if (!r || (b && !r_out) || (w_pre && !x)) return LOBRA_ERR_NULL;
    for (const void* q : {r, b, w_post, gate, w_pre, static_cast<const void*>(r_out), static_cast<const void*>(x)})
        if (!aligned16(q)) return LOBRA_ERR_ALIGN;
    if (!aligned4(rstd_post) || !aligned4(rstd_pre)) return LOBRA_ERR_ALIGN;
    if (!b && !w_pre) return LOBRA_OK;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const PlanDev pd = device_view(p);
    const BlockNorm bn{cfg->eps, cfg->alpha, w_post, gate, w_pre, b && w_post, b != nullptr};
    LOBRA_LAUNCH(p, st, LOBRA_K_BLOCK_NORM, block_norm_fwd(pd, p.desc.dtype, bn, r, b, r_out, x, rstd_post, rstd_pre, st));
    return LOBRA_OK;
}

lobra_status lobra_mlora_block_norm_bwd(const lobra_mlora_plan* plan, const lobra_block_norm_config* cfg, const void* r_out, const void* b,
                                        const void* w_post, const void* gate, const void* w_pre, const float* rstd_post, const float* rstd_pre,
                                        const void* dr_out, const void* dx, void* dr, void* db, float* dgate, float* dw_post, float* dw_pre,
                                        uint32_t flags, void* ws, size_t ws_bytes, void* hip_stream)
{
    lobra_status rs = runnable(plan);
    if (rs != LOBRA_OK) return rs;
    const Plan& p = *plan;
    if ((rs = block_norm_check(p, cfg)) != LOBRA_OK) return rs;
    const bool post = b && w_post;
    // what has no norm, or no gate, has no gradient of it (an empty batch's tensors have no address: it says nothing of them)
    const bool block = b || p.desc.T == 0, normed = dx || p.desc.T == 0;
    if ((dgate && (!gate || !block)) || (dw_post && (!w_post || !block)) || (dw_pre && (!w_pre || !normed))) return LOBRA_ERR_NULL;
    if (p.desc.T > 0) {
        if (!dr || (b && !db) || (dx && (!w_pre || !r_out || !rstd_pre)) || (post && !rstd_post)) return LOBRA_ERR_NULL;
    }
    for (const void* q : {r_out, b, w_post, gate, w_pre, dr_out, dx, static_cast<const void*>(dr), static_cast<const void*>(db),
                          static_cast<const void*>(dgate), static_cast<const void*>(dw_post), static_cast<const void*>(dw_pre),
                          static_cast<const void*>(ws)})
        if (!aligned16(q)) return LOBRA_ERR_ALIGN;
    if (!aligned4(rstd_post) || !aligned4(rstd_pre)) return LOBRA_ERR_ALIGN;
    const size_t need = dgate || dw_post || dw_pre ? block_norm_part_bytes(p.desc.T, p.desc.d_in, int32_t(p.cseg_task.size()), p.desc.dtype) : 0;
    if (need > 0 && (!ws || ws_bytes < need)) return LOBRA_ERR_WORKSPACE;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const PlanDev pd = device_view(p);
    const BlockNorm bn{cfg->eps, cfg->alpha, w_post, gate, w_pre, post, b != nullptr};
    LOBRA_LAUNCH(p, st, LOBRA_K_BLOCK_NORM,
                 block_norm_bwd(pd, p.desc.dtype, bn, r_out, b, rstd_post, rstd_pre, dr_out, dx, dr, db, dgate, dw_post, dw_pre,
                                (flags & LOBRA_FLAG_ACCUMULATE_GRADS) != 0, static_cast<float*>(ws), st));
    return LOBRA_OK;
}

lobra_status lobra_token_logprob_fwd(const lobra_logprob_desc* desc, const void* logits, const int32_t* target, float* logp, float* lse,
                                     float* lse_rest, float* entropy, float* top_logp, int32_t* top_id, void* hip_stream)
{
    LogprobShape s;
    const lobra_status rs = logprob_shape(desc, &s);
    if (rs != LOBRA_OK) return rs;
    if (s.T == 0) return LOBRA_OK;
    if (!logits) return LOBRA_ERR_NULL;
    if (!aligned16(logits)) return LOBRA_ERR_ALIGN;
    for (const void* q : {static_cast<const void*>(target), static_cast<const void*>(logp), static_cast<const void*>(lse),
                          static_cast<const void*>(lse_rest), static_cast<const void*>(entropy), static_cast<const void*>(top_logp), static_cast<const void*>(top_id)})
        if (!aligned4(q)) return LOBRA_ERR_ALIGN;
    LOBRA_HIP(logprob_fwd(s, logits, target, LogprobOut{logp, lse, lse_rest, entropy, top_logp, top_id}, static_cast<hipStream_t>(hip_stream)));
    return LOBRA_OK;
}

lobra_status lobra_token_logprob_bwd(const lobra_logprob_desc* desc, const void* logits, const int32_t* target, const float* lse,
                                     const float* lse_rest, const float* entropy, const float* dlogp, const float* dentropy, void* dlogits,
                                     void* hip_stream)
{
    LogprobShape s;
    const lobra_status rs = logprob_shape(desc, &s);
    if (rs != LOBRA_OK) return rs;
    if (s.T == 0) return LOBRA_OK;
    if (!logits || !lse || !dlogits || (dentropy && !entropy)) return LOBRA_ERR_NULL;
    if (!aligned16(logits) || !aligned16(dlogits)) return LOBRA_ERR_ALIGN;
    for (const void* q : {static_cast<const void*>(target), static_cast<const void*>(lse), static_cast<const void*>(lse_rest),
                          static_cast<const void*>(entropy),
                          static_cast<const void*>(dlogp), static_cast<const void*>(dentropy)})
        if (!aligned4(q)) return LOBRA_ERR_ALIGN;
    LOBRA_HIP(logprob_bwd(s, logits, target, LogprobGrad{lse, lse_rest, entropy, dlogp, dentropy}, dlogits, static_cast<hipStream_t>(hip_stream)));
    return LOBRA_OK;
}

lobra_status lobra_grad_set_device_bytes(const lobra_grad_tensor* tensors, int32_t n_tensors, int32_t n_tasks, size_t* bytes)
{
    if (!bytes) return LOBRA_ERR_NULL;
    lobra_grad_set* s = nullptr;
    const lobra_status rs = make_set(tensors, n_tensors, n_tasks, &s);
    if (rs != LOBRA_OK) return rs;
    *bytes = s->blob.size();
    delete s;
    return LOBRA_OK;
}

lobra_status lobra_grad_set_create(const lobra_grad_tensor* tensors, int32_t n_tensors, int32_t n_tasks, lobra_grad_set** out)
{
    if (!out) return LOBRA_ERR_NULL;
    lobra_grad_set* s = nullptr;
    lobra_status rs = make_set(tensors, n_tensors, n_tasks, &s);
    if (rs != LOBRA_OK) return rs;
    if (hipGetDevice(&s->device) != hipSuccess) rs = LOBRA_ERR_HIP;
    else if (hipMalloc(&s->dev, s->blob.size()) != hipSuccess) rs = LOBRA_ERR_NOMEM;
    else if (hipMemcpy(s->dev, s->blob.data(), s->blob.size(), hipMemcpyHostToDevice) != hipSuccess) {
        (void)hipFree(s->dev);
        rs = LOBRA_ERR_HIP;
    }
    if (rs != LOBRA_OK) {
        delete s;
        return rs;
    }
    s->owns = true;
    *out = s;
    return LOBRA_OK;
}

lobra_status lobra_grad_set_init(const lobra_grad_tensor* tensors, int32_t n_tensors, int32_t n_tasks, void* device_mem, size_t device_bytes,
                                 void* hip_stream, lobra_grad_set** out)
{
    if (!out) return LOBRA_ERR_NULL;
    lobra_grad_set* s = nullptr;
    lobra_status rs = make_set(tensors, n_tensors, n_tasks, &s);
    if (rs != LOBRA_OK) return rs;
    if (!device_mem || device_bytes < s->blob.size()) rs = LOBRA_ERR_WORKSPACE;
    else if (!aligned16(device_mem)) rs = LOBRA_ERR_ALIGN;
    else if (hipGetDevice(&s->device) != hipSuccess) rs = LOBRA_ERR_HIP;
    // the source of the copy is the set's own host image, which lives as long as the set
    else if (hipMemcpyAsync(device_mem, s->blob.data(), s->blob.size(), hipMemcpyHostToDevice, static_cast<hipStream_t>(hip_stream)) != hipSuccess)
        rs = LOBRA_ERR_HIP;
    if (rs != LOBRA_OK) {
        delete s;
        return rs;
    }
    s->dev = device_mem;
    *out = s;
    return LOBRA_OK;
}

lobra_status lobra_grad_set_destroy(lobra_grad_set* set)
{
    if (!set) return LOBRA_OK;
    const lobra_status rs = set->owns && hipFree(set->dev) != hipSuccess ? LOBRA_ERR_HIP : LOBRA_OK;
    delete set;
    return rs;
}

lobra_status lobra_grad_set_workspace_bytes(const lobra_grad_set* set, size_t* bytes)
{
    if (!set) return LOBRA_ERR_PLAN;
    if (!bytes) return LOBRA_ERR_NULL;
    *bytes = clip_ws_bytes(*set);
    return LOBRA_OK;
}

lobra_status lobra_grad_clip(const lobra_grad_set* set, const float* max_norm, const float* grad_scale, const int32_t* step, float* norm,
                             float* clip_scale, int32_t* step_out, uint32_t flags, void* ws, size_t ws_bytes, void* hip_stream)
{
    if (!set || !set->dev) return LOBRA_ERR_PLAN;
    int dev = -1;
    LOBRA_HIP(hipGetDevice(&dev));
    if (dev != set->device) return LOBRA_ERR_PLAN;
    if (set->n_tasks == 0) return LOBRA_OK;
    if ((step == nullptr) != (step_out == nullptr)) return LOBRA_ERR_NULL;
    for (const void* q : {static_cast<const void*>(max_norm), static_cast<const void*>(grad_scale), static_cast<const void*>(step),
                          static_cast<const void*>(norm), static_cast<const void*>(clip_scale), static_cast<const void*>(step_out)})
        if (!aligned4(q)) return LOBRA_ERR_ALIGN;
    if (!aligned16(ws)) return LOBRA_ERR_ALIGN;
    if (!ws || ws_bytes < clip_ws_bytes(*set)) return LOBRA_ERR_WORKSPACE;
    const char* d = static_cast<const char*>(set->dev);
    double* partial = static_cast<double*>(ws);
    float* scale = reinterpret_cast<float*>(static_cast<char*>(ws) + align256(size_t(set->n_pieces) * sizeof(double)));
    LOBRA_HIP(grad_clip(reinterpret_cast<const GradPiece*>(d), reinterpret_cast<const int32_t*>(d + set->o_task_piece), set->n_pieces, set->n_tasks,
                        set->any_out, set->once, max_norm, grad_scale, step, norm, clip_scale, step_out, (flags & LOBRA_FLAG_JOINT_NORM) != 0, partial, scale,
                        static_cast<hipStream_t>(hip_stream)));
    return LOBRA_OK;
}

}  // extern "C"
