// What the translation units with extern "C" entry points share: the device view of a plan, the check that a plan can run here, and
// the launch macros.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "kernels.h"
#include "lobra_mlora.h"
#include "plan.h"

namespace lobra {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline PlanDev device_view(const Plan& p)
{
    const int32_t* b = static_cast<const int32_t*>(p.dev_blob);
    PlanDev d;
    d.cseg_off = b + p.o_cseg_off;
    d.cseg_task = b + p.o_cseg_task;
    d.rowblk_seg = b + p.o_rowblk;
    d.tb = reinterpret_cast<const TokenBlock*>(b + p.o_tb);
    d.chunks = reinterpret_cast<const GradChunk*>(b + p.o_chunks);
    d.task_chunk_off = b + p.o_task_chunk;
    d.rank_off = b + p.o_rank_off;
    d.task_tb_off = b + p.o_task_tb;
    d.sb_off = b + p.o_sb;
    d.tb_order = p.tb_order.empty() ? nullptr : b + p.o_tb_order;
    d.sb_order = p.sb_order.empty() || p.shrink_group == 1 ? nullptr : b + p.o_sb_order;
    d.fb_wg_run_off = p.fused_db ? b + p.o_fb_wg : nullptr;
    d.fb_run_row = p.fused_db ? b + p.o_fb_run : nullptr;
    d.fb_cnt = p.fused_db ? b + p.o_fb_cnt : nullptr;
    d.fb_task_row0 = p.fused_db ? b + p.o_fb_row0 : nullptr;
    d.gemm_tile_seg = b + p.o_tile_seg;
    d.T = int32_t(p.desc.T);
    d.d_in = p.desc.d_in;
    d.d_out = p.desc.d_out;
    d.n_tasks = p.desc.n_tasks;
    d.nseg = int32_t(p.cseg_task.size());
    d.ntb = int32_t(p.tb.size());
    d.nchunks = int32_t(p.chunks.size());
    d.r_max = p.r_max;
    d.r_pad = p.r_pad;
    d.R_tot = p.R_tot;
    d.nsb = int32_t(p.sb_off.size()) - 1;
    d.shrink_group = p.shrink_group;
    d.n_proj = p.n_proj;
    d.dg = p.dg;
    return d;
}

// A plan can run only on the device it was uploaded to.
inline lobra_status runnable(const lobra_mlora_plan* plan)
{
    if (!plan) return LOBRA_ERR_PLAN;
    if (!plan->dev_blob) return LOBRA_ERR_PLAN;
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess) return LOBRA_ERR_HIP;
    if (dev != plan->device) return LOBRA_ERR_PLAN;
    return LOBRA_OK;
}

#define LOBRA_HIP(expr)                                   \
    do {                                                  \
        if ((expr) != hipSuccess) return LOBRA_ERR_HIP;   \
    } while (0)

// One kernel launch, bracketed by the plan's trace events when a trace is attached.
#define LOBRA_LAUNCH(plan_ref, stream, kernel_id, expr)                                          \
    do {                                                                                         \
        const Plan& tp_ = (plan_ref);                                                            \
        const int32_t ti_ = tp_.trace_events ? tp_.trace_next++ : -1;                            \
        const bool tr_ = ti_ >= 0 && ti_ < tp_.trace_pairs;                                      \
        if (tp_.trace_count) *tp_.trace_count = tp_.trace_next;                                  \
        if (tr_) {                                                                               \
            if (tp_.trace_ids) tp_.trace_ids[ti_] = (kernel_id);                                 \
            LOBRA_HIP(hipEventRecord(static_cast<hipEvent_t>(tp_.trace_events[2 * ti_]), stream)); \
        }                                                                                        \
        LOBRA_HIP(expr);                                                                         \
        if (tr_)                                                                                 \
            LOBRA_HIP(hipEventRecord(static_cast<hipEvent_t>(tp_.trace_events[2 * ti_ + 1]), stream)); \
    } while (0)

// Argument checks of a forward call on plan p (everything except the plan itself): host only.
inline lobra_status plan_fwd_check(const Plan& p, const void* x, const void* W, const void* A, const void* B, const float* s,
                                   const void* y, const void* h_save, const void* ws, size_t ws_bytes)
{
    const bool adapters = !p.tb.empty();
    if (!x || !W || !y) return LOBRA_ERR_NULL;
    if (adapters && (!A || !B || !s)) return LOBRA_ERR_NULL;
    if (!aligned16(x) || !aligned16(W) || !aligned16(y) || !aligned16(A) || !aligned16(B) ||
        !aligned16(h_save) || !aligned16(ws))
        return LOBRA_ERR_ALIGN;
    // the workspace holds, without h_save, the projected activations, and in front of them, if there is room, a split base product's sums
    const size_t need = h_save ? 0 : p.p_layout.total;
    if (adapters && need > 0 && (!ws || ws_bytes < need)) return LOBRA_ERR_WORKSPACE;
    return LOBRA_OK;
}

// Argument checks of a backward call on plan p (everything except the plan itself): host only.
inline lobra_status plan_bwd_check(const Plan& p, const void* x, const void* W, const void* A, const void* B, const float* s,
                                   const void* dy, const void* h_saved, const void* dx, const float* dA, const float* dB,
                                   uint32_t flags, const void* ws, size_t ws_bytes)
{
    const bool adapters = !p.tb.empty();
    const bool want_dx = !(flags & LOBRA_FLAG_NO_DX);
    if (p.R_tot > 0 && (!dA || !dB)) return LOBRA_ERR_NULL;
    if (p.desc.T > 0) {
        if (!W || !dy) return LOBRA_ERR_NULL;
        if (want_dx && !dx) return LOBRA_ERR_NULL;
        if (adapters && (!x || !A || !B || !s)) return LOBRA_ERR_NULL;
    }
    if (!aligned16(x) || !aligned16(W) || !aligned16(A) || !aligned16(B) || !aligned16(dy) ||
        !aligned16(h_saved) || !aligned16(dx) || !aligned16(dA) || !aligned16(dB) || !aligned16(ws))
        return LOBRA_ERR_ALIGN;
    if (p.bwd_need > 0 && adapters && (!ws || ws_bytes < p.bwd_need)) return LOBRA_ERR_WORKSPACE;
    return LOBRA_OK;
}

}  // namespace lobra
