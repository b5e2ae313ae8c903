// extern "C" entry points of the layer on a base in 8-bit integers.  Argument checks on the host, then launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "api_common.h"

using namespace lobra;

namespace {

inline size_t align256(size_t v) { return (v + 255) / 256 * 256; }

// What the layer needs of a plan to run on an 8-bit base.
lobra_status q8_plan(const Plan& p)
{
    if (p.desc.dtype != LOBRA_BF16 || !p.mfma) return LOBRA_ERR_DTYPE;
    if (p.desc.d_in > LOBRA_MAX_QUANT_IN) return LOBRA_ERR_SHAPE;
    return LOBRA_OK;
}

// A product of all projections in one launch where no tile straddles two, else one of each.
struct Q8Product {
    int32_t K, N, launches, proj;        // K in pairs; the first projection, or -1: all
    GemmChoice choice;
    bool beside = false;                 // the projection of x runs in the product's launch
};
Q8Product q8_product(const Plan& p)
{
    const bool adapters = !p.tb.empty();
    const int32_t K = int32_t(q8_pitch(p.desc.d_in) / 2), nseg = adapters ? int32_t(p.cseg_task.size()) : 0;
    const auto choose = [&](int32_t N, int32_t group) { return choose_q8(p.desc.T, K, N, group, nseg, kMaxPartBytes); };
    Q8Product one{K, p.desc.d_out, 1, p.n_proj > 1 ? -1 : 0, choose(p.desc.d_out, p.n_proj > 1 ? p.dg : 0)};
    if (p.n_proj > 1) {
        const Q8Product each{K, p.dg, p.n_proj, 0, choose(p.dg, 0)};
        if (one.choice.tile < 0 || float(p.n_proj) * (each.choice.cost + 3.f) < one.choice.cost) return each;
    } else if (adapters) {
        int32_t halves = 1;
        for (const TokenBlock& b : p.tb) halves = std::max(halves, (b.nrows + 15) / 16);
        const GemmChoice c = choose_q8_beside(p.desc.T, K, p.desc.d_out, nseg, p.r_max, int64_t(p.tb.size()), halves, p.desc.d_in);
        if (c.tile >= 0) one.choice = c, one.beside = true;
    }
    return one;
}

// Few tokens have kernels of their own, which keep no projected activations (which are better: q8_few.hip).
bool q8_is_few(const Plan& p)
{
    return p.desc.T > 0 && p.desc.T <= kQ8FewTokens && p.desc.d_out <= kQ8FewColumns * (p.desc.T <= 16 ? 2 : 1) && p.r_max <= kQ8FewRank;
}

// The forward workspace: quantised tokens, their scales, a split product's sums, projected activations.
struct Q8Layout {
    size_t scale, part, h, total;
};
Q8Layout q8_layout(const Plan& p, const Q8Product& g, bool h_saved)
{
    Q8Layout l;
    // (few tokens: in blocks of 16)
    l.scale = align256(size_t(q8_is_few(p) ? (p.desc.T + 15) / 16 * 16 : p.desc.T) * size_t(q8_pitch(p.desc.d_in)));
    l.part = l.scale + align256(size_t(p.desc.T) * sizeof(float));
    l.h = l.part + (g.choice.splits > 1 || g.beside ? align256(size_t(g.choice.splits + 1) * size_t(p.desc.T) * size_t(g.N) * sizeof(float)) : 0);
    l.total = l.h + (h_saved || p.tb.empty() ? 0 : p.p_layout.total);
    return l;
}

size_t q8_fwd_bytes(const Plan& p, const Q8Layout& l, bool h_saved)
{
    return h_saved || !q8_is_few(p) || p.tb.empty() ? l.total : std::max(l.total, l.part + q8_few_bytes(p.desc.T, p.r_max));
}

size_t q8_weight_bytes(const Plan& p) { return align256(size_t(p.desc.d_in) * size_t(p.desc.d_out) * 2); }

}  // namespace

extern "C" {

int64_t lobra_quant_pitch(int32_t d_in) { return d_in < 1 ? 0 : q8_pitch(d_in); }

lobra_status lobra_quantise_weight(int32_t dtype, int32_t d_in, int32_t d_out, int64_t ldw, const void* W, int8_t* Wq, float* w_scale,
                                      void* hip_stream)
{
    if (dtype != LOBRA_F32 && dtype != LOBRA_BF16) return LOBRA_ERR_DTYPE;
    if (ldw == 0) ldw = d_out;
    if (d_in < 1 || d_in > LOBRA_MAX_QUANT_IN || d_out < 1 || d_out > LOBRA_MAX_WIDTH || ldw < d_out || ldw >= int64_t(1) << 40) return LOBRA_ERR_SHAPE;
    if (!W || !Wq || !w_scale) return LOBRA_ERR_NULL;
    if (!aligned16(W) || !aligned16(Wq) || !aligned16(w_scale)) return LOBRA_ERR_ALIGN;
    LOBRA_HIP(q8_weight(dtype, d_in, d_out, ldw, W, Wq, w_scale, static_cast<hipStream_t>(hip_stream)));
    return LOBRA_OK;
}

lobra_status lobra_mlora_quant_workspace_bytes(const lobra_mlora_plan* plan, size_t* fwd_bytes, size_t* bwd_bytes)
{
    if (!plan) return LOBRA_ERR_PLAN;
    const lobra_status rs = q8_plan(*plan);
    if (rs != LOBRA_OK) return rs;
    if (fwd_bytes) *fwd_bytes = plan->desc.T == 0 ? 0 : q8_fwd_bytes(*plan, q8_layout(*plan, q8_product(*plan), false), false);
    if (bwd_bytes) *bwd_bytes = q8_weight_bytes(*plan) + plan->bwd_ws_bytes;
    return LOBRA_OK;
}

lobra_status lobra_mlora_quant_fwd(const lobra_mlora_plan* plan, const void* x, const int8_t* Wq, const float* w_scale, const void* A, const void* B,
                                const float* s, void* y, void* h_save, void* ws, size_t ws_bytes, void* hip_stream)
{
    lobra_status rs = runnable(plan);
    if (rs != LOBRA_OK) return rs;
    const Plan& p = *plan;
    if ((rs = q8_plan(p)) != LOBRA_OK) return rs;
    if (p.desc.T == 0) return LOBRA_OK;
    if (!w_scale) return LOBRA_ERR_NULL;
    const Q8Product g = q8_product(p);
    const Q8Layout l = q8_layout(p, g, h_save != nullptr);
    if ((rs = plan_fwd_check(p, x, Wq, A, B, s, y, h_save, ws, ws_bytes)) != LOBRA_OK) return rs;
    if (!aligned16(w_scale)) return LOBRA_ERR_ALIGN;
    const bool few = q8_is_few(p) && !h_save;
    if (!ws || ws_bytes < q8_fwd_bytes(p, l, h_save != nullptr)) return LOBRA_ERR_WORKSPACE;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const PlanDev pd = device_view(p);
    const bool adapters = !p.tb.empty();
    char* const wsb = static_cast<char*>(ws);
    float* const x_scale = reinterpret_cast<float*>(wsb + l.scale);
    float* const part = reinterpret_cast<float*>(wsb + l.part);
    char* const hb = h_save ? static_cast<char*>(h_save) : wsb + l.h;
    if (few) {
        float* const P = adapters ? part : nullptr;
        LOBRA_LAUNCH(p, st, adapters ? LOBRA_K_SHRINK : LOBRA_K_QUANT, q8_few_rows(pd, x, A, s, wsb, x_scale, P, st));
        LOBRA_LAUNCH(p, st, LOBRA_K_GEMM, q8_few(pd, wsb, x_scale, Wq, w_scale, P, B, y, st));
        return LOBRA_OK;
    }
    LOBRA_LAUNCH(p, st, LOBRA_K_QUANT, q8_rows(p.desc.T, pd.d_in, x, wsb, x_scale, st));
    if (g.beside) {
        LOBRA_LAUNCH(p, st, LOBRA_K_SHRINK_GEMM,
                     gemm_tile_q8_beside(pd, g.choice, wsb, x_scale, Wq, w_scale, x, A, s, hb + p.p_layout.p_tok, hb + p.p_layout.p_blk, B, y, g.K, g.N,
                                         p.has_row_table(), st, part));
        return LOBRA_OK;
    }
    if (adapters)
        LOBRA_LAUNCH(p, st, LOBRA_K_SHRINK, shrink_mfma(pd, x, A, s, hb + p.p_layout.p_tok, hb + p.p_layout.p_blk, pd.d_in, pd.d_in, 1, 0, st));
    const char* const P = adapters ? hb + p.p_layout.p_tok : nullptr;
    for (int32_t j = 0; j < g.launches; ++j) {
        const int8_t* const Wj = Wq + size_t(j) * pd.dg * size_t(2 * g.K);
        char* const yj = static_cast<char*>(y) + size_t(j) * pd.dg * 2;
        const int32_t proj = g.proj < 0 ? -1 : j;
        if (g.choice.tile == kPersistentTile)
            LOBRA_LAUNCH(p, st, LOBRA_K_GEMM, gemm_persistent_q8(pd, wsb, x_scale, Wj, w_scale + size_t(j) * pd.dg, P, B, yj, g.K, g.N, pd.d_out, p.n_proj, proj, st));
        else
            LOBRA_LAUNCH(p, st, LOBRA_K_GEMM,
                         gemm_tile_q8(pd, g.choice, wsb, x_scale, Wj, w_scale + size_t(j) * pd.dg, P, B, yj, g.K, g.N, pd.d_out, p.n_proj, proj, st, part));
    }
    return LOBRA_OK;
}

lobra_status lobra_mlora_quant_bwd(const lobra_mlora_plan* plan, const void* x, const int8_t* Wq, const float* w_scale, const void* A, const void* B,
                                const float* s, const void* dy, const void* h_saved, void* dx, float* dA, float* dB, uint32_t flags, void* ws,
                                size_t ws_bytes, void* hip_stream)
{
    lobra_status rs = runnable(plan);
    if (rs != LOBRA_OK) return rs;
    const Plan& p = *plan;
    if ((rs = q8_plan(p)) != LOBRA_OK) return rs;
    const bool want_dx = !(flags & LOBRA_FLAG_NO_DX);
    const size_t own = want_dx ? q8_weight_bytes(p) : 0;             // (only dx takes the weight)
    if (p.desc.T > 0 && !w_scale) return LOBRA_ERR_NULL;
    if (!aligned16(w_scale)) return LOBRA_ERR_ALIGN;
    char* const rest = ws ? static_cast<char*>(ws) + own : nullptr;
    const size_t left = ws && ws_bytes > own ? ws_bytes - own : 0;
    if ((rs = plan_bwd_check(p, x, Wq, A, B, s, dy, h_saved, dx, dA, dB, flags, rest, left)) != LOBRA_OK) return rs;
    if (p.desc.T > 0 && own > 0 && (!ws || ws_bytes < own)) return LOBRA_ERR_WORKSPACE;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (p.desc.T > 0 && want_dx)
        LOBRA_LAUNCH(p, st, LOBRA_K_QUANT, q8_dequantise(p.desc.d_in, p.desc.d_out, Wq, w_scale, ws, st));
    return lobra_mlora_plan_bwd(plan, x, want_dx ? ws : Wq, A, B, s, dy, h_saved, dx, dA, dB, flags, rest, left, hip_stream);
}

}  // extern "C"
