// extern "C" entry points of the operators on rows of logits beyond their log probabilities: a teacher's likeliest tokens, beam search.  Argument
// checks on the host, then launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "api_common.h"

using namespace lobra;

namespace {

inline bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

lobra_status distill_shape(const lobra_distill_desc* d, DistillShape* s)
{
    if (!d) return LOBRA_ERR_NULL;
    if (d->dtype != LOBRA_F32 && d->dtype != LOBRA_BF16) return LOBRA_ERR_DTYPE;
    const int64_t ld = d->ld == 0 ? d->V : d->ld;
    if (d->V < 1 || d->V > LOBRA_MAX_VOCAB || d->T < 0 || d->T >= (int64_t(1) << 31) || ld < d->V || d->top_k < 1 || d->top_k > LOBRA_MAX_TEACHER)
        return LOBRA_ERR_SHAPE;
    if ((d->tail != 0 && d->tail != 1) || !(d->temperature > 0.f) || !std::isfinite(d->temperature) || !std::isfinite(1.f / d->temperature * 1.4426950408889634f))
        return LOBRA_ERR_SHAPE;
    if (d->T > 0 && ld >= (int64_t(1) << 60) / d->T) return LOBRA_ERR_SHAPE;
    *s = DistillShape{d->dtype, d->V, d->top_k, d->tail != 0, d->T, ld, d->temperature};
    return LOBRA_OK;
}

lobra_status beam_shape(const lobra_beam_desc* d, BeamShape* s)
{
    if (!d) return LOBRA_ERR_NULL;
    if (d->dtype != LOBRA_F32 && d->dtype != LOBRA_BF16) return LOBRA_ERR_DTYPE;
    const int64_t ld = d->ld == 0 ? d->V : d->ld;
    if (d->V < 1 || d->V > LOBRA_MAX_VOCAB || ld < d->V || d->n_req < 0 || d->beams < 1 || d->beams > LOBRA_MAX_TOP || d->n_out < 1 ||
        d->n_out > LOBRA_MAX_TOP)
        return LOBRA_ERR_SHAPE;
    const int64_t rows = int64_t(d->n_req) * d->beams;
    if (rows >= int64_t(1) << 24 || rows * beam_parts(d->dtype, d->V) >= int64_t(1) << 24) return LOBRA_ERR_SHAPE;     // (a launch holds less than 2^32 threads)
    if (rows > 0 && ld >= (int64_t(1) << 60) / rows) return LOBRA_ERR_SHAPE;
    *s = BeamShape{d->dtype, d->V, ld, d->n_req, d->beams, d->n_out};
    return LOBRA_OK;
}

// What is read beside the states.
struct Bytes {
    const void* at;
    uintptr_t n;
};

// Whether a tensor of the list writes what another one reads or writes (they run side by side), or something of `beside`.  What kAtATime tensors read and write is sorted by address, with the
// furthest end of all that begins no later, and of what is written among it; every tensor behind them is looked up there.  No memory is taken.  (160 tensors, the
// keys and values of 80 layers, 4 us in place, 7 apart, and pair by pair 21; 1000 of them 43 and 131, and 744.)
constexpr int32_t kAtATime = 256;
template <int N> bool states_meet(const lobra_beam_state* states, int32_t n, int64_t rows, const Bytes (&beside)[N])
{
    struct Range {
        uintptr_t at, end, written_end;
        bool meets(uintptr_t from, bool written) const { return (written ? end : written_end) > from; }
    } r[2 * kAtATime];
    // f(first byte, the one behind the last, whether it is written) for what tensor i reads and writes; false: enough
    const auto of = [&](int32_t i, auto&& f) {
        const lobra_beam_state& t = states[i];
        const uintptr_t bytes = uintptr_t(t.row_bytes) * uintptr_t(rows), a = reinterpret_cast<uintptr_t>(t.src), b = reinterpret_cast<uintptr_t>(t.dst);
        return bytes == 0 || (f(b, b + bytes, true) && (a == b || f(a, a + bytes, false)));
    };
    for (int32_t i0 = 0; i0 < n; i0 += kAtATime) {
        const int32_t i1 = std::min(n, i0 + kAtATime);
        Range* last = r;
        for (int32_t i = i0; i < i1; ++i)
            of(i, [&](uintptr_t at, uintptr_t end, bool written) {
                *last++ = Range{at, end, written ? end : 0};
                return true;
            });
        std::sort(r, last, [](const Range& x, const Range& y) { return x.at < y.at; });
        for (Range* p = r + 1; p < last; ++p) {
            if (p[-1].meets(p->at, p->written_end > 0)) return true;
            p->end = std::max(p->end, p[-1].end);
            p->written_end = std::max(p->written_end, p[-1].written_end);
        }
        const auto apart = [&](uintptr_t at, uintptr_t end, bool written) {
            const Range* const behind = std::lower_bound(r, last, end, [](const Range& x, uintptr_t v) { return x.at < v; });
            return behind == r || !behind[-1].meets(at, written);
        };
        for (int32_t i = i1; i < n; ++i)
            if (!of(i, apart)) return true;
        for (const Bytes& b : beside)
            if (const uintptr_t at = reinterpret_cast<uintptr_t>(b.at); at && !apart(at, at + b.n, false)) return true;
    }
    return false;
}

// Every part's largest logits, then its sums.
size_t beam_key_bytes(const BeamShape& s) { return size_t(s.n_req) * s.beams * beam_parts(s.dtype, s.V) * s.n_out * sizeof(uint64_t); }
size_t beam_ws_bytes(const BeamShape& s) { return beam_key_bytes(s) + size_t(s.n_req) * s.beams * beam_parts(s.dtype, s.V) * 2 * sizeof(float); }

}  // namespace

extern "C" {

lobra_status lobra_token_distill_fwd(const lobra_distill_desc* desc, const void* logits, const float* teacher_logp, const int32_t* teacher_id, float* loss,
                                     float* stat, void* hip_stream)
{
    DistillShape s;
    const lobra_status rs = distill_shape(desc, &s);
    if (rs != LOBRA_OK) return rs;
    if (s.T == 0) return LOBRA_OK;
    if (!logits || !teacher_logp || !teacher_id) return LOBRA_ERR_NULL;
    if (!aligned16(logits) || !aligned16(stat) || !aligned4(teacher_logp) || !aligned4(teacher_id) || !aligned4(loss)) return LOBRA_ERR_ALIGN;
    if (!loss && !stat) return LOBRA_OK;
    LOBRA_HIP(distill_fwd(s, logits, teacher_logp, teacher_id, loss, stat, static_cast<hipStream_t>(hip_stream)));
    return LOBRA_OK;
}

lobra_status lobra_token_distill_bwd(const lobra_distill_desc* desc, const void* logits, const float* teacher_logp, const int32_t* teacher_id,
                                     const float* stat, const float* dloss, void* dlogits, uint32_t flags, void* hip_stream)
{
    DistillShape s;
    const lobra_status rs = distill_shape(desc, &s);
    if (rs != LOBRA_OK) return rs;
    if (s.T == 0) return LOBRA_OK;
    if (!logits || !teacher_logp || !teacher_id || !stat || !dloss || !dlogits) return LOBRA_ERR_NULL;
    if (!aligned16(logits) || !aligned16(dlogits) || !aligned16(stat) || !aligned4(teacher_logp) || !aligned4(teacher_id) || !aligned4(dloss))
        return LOBRA_ERR_ALIGN;
    const bool add = (flags & LOBRA_FLAG_ACCUMULATE_GRADS) != 0;
    if (add && logits == dlogits) return LOBRA_ERR_SHAPE;
    LOBRA_HIP(distill_bwd(s, logits, teacher_logp, teacher_id, stat, dloss, dlogits, add, static_cast<hipStream_t>(hip_stream)));
    return LOBRA_OK;
}

lobra_status lobra_beam_workspace_bytes(const lobra_beam_desc* desc, size_t* bytes)
{
    BeamShape s;
    const lobra_status rs = beam_shape(desc, &s);
    if (rs != LOBRA_OK) return rs;
    if (!bytes) return LOBRA_ERR_NULL;
    *bytes = beam_ws_bytes(s);
    return LOBRA_OK;
}

lobra_status lobra_beam_select(const lobra_beam_desc* desc, const void* logits, const float* score, const int32_t* done, int32_t done_token,
                               float* out_score, int32_t* out_beam, int32_t* out_token, void* ws, size_t ws_bytes, void* hip_stream)
{
    BeamShape s;
    const lobra_status rs = beam_shape(desc, &s);
    if (rs != LOBRA_OK) return rs;
    if (s.n_req == 0) return LOBRA_OK;
    if (!logits || !score || !out_score || !out_beam || !out_token) return LOBRA_ERR_NULL;
    if (!aligned16(logits) || !aligned16(ws)) return LOBRA_ERR_ALIGN;
    for (const void* q : {static_cast<const void*>(score), static_cast<const void*>(done), static_cast<const void*>(out_score),
                          static_cast<const void*>(out_beam), static_cast<const void*>(out_token)})
        if (!aligned4(q)) return LOBRA_ERR_ALIGN;
    if (out_score == score && s.n_out != s.beams) return LOBRA_ERR_SHAPE;
    if (!ws || ws_bytes < beam_ws_bytes(s)) return LOBRA_ERR_WORKSPACE;
    LOBRA_HIP(beam_select(s, logits, score, done, done_token, out_score, out_beam, out_token, static_cast<uint64_t*>(ws),
                          reinterpret_cast<float*>(static_cast<char*>(ws) + beam_key_bytes(s)), static_cast<hipStream_t>(hip_stream)));
    return LOBRA_OK;
}

lobra_status lobra_beam_reorder(const lobra_beam_state* states, int32_t n_states, int32_t n_req, int32_t beams, const int32_t* parent, int64_t parent_ld,
                                const int32_t* used, void* hip_stream)
{
    if (n_states < 0 || n_req < 0 || beams < 1 || beams > LOBRA_MAX_TOP || parent_ld < beams || parent_ld >= int64_t(1) << 40) return LOBRA_ERR_SHAPE;
    const int64_t rows = int64_t(n_req) * beams;
    if (rows >= int64_t(1) << 24) return LOBRA_ERR_SHAPE;
    if (n_states > 0 && !states) return LOBRA_ERR_NULL;
    bool any = false;
    for (int32_t i = 0; i < n_states; ++i) {
        const lobra_beam_state& t = states[i];
        if (t.row_bytes < 0 || t.unit_bytes < 0 || (rows > 0 && t.row_bytes >= (int64_t(1) << 60) / rows)) return LOBRA_ERR_SHAPE;
        const int64_t bytes = t.row_bytes * rows;
        if (bytes == 0) continue;
        any = true;
        if (!t.src || !t.dst) return LOBRA_ERR_NULL;
        const uintptr_t a = reinterpret_cast<uintptr_t>(t.src), b = reinterpret_cast<uintptr_t>(t.dst);
        if (a != b && (a < b ? b - a : a - b) < uintptr_t(bytes)) return LOBRA_ERR_SHAPE;
    }
    if (!any) return LOBRA_OK;
    const bool given = parent && aligned4(parent) && aligned4(used);          // (else refused below)
    const Bytes parents{given ? parent : nullptr, uintptr_t((n_req - 1) * parent_ld + beams) * sizeof(int32_t)},
        lengths{given ? used : nullptr, uintptr_t(n_req) * sizeof(int32_t)};
    if (states_meet(states, n_states, rows, {parents, lengths})) return LOBRA_ERR_SHAPE;
    if (!parent) return LOBRA_ERR_NULL;
    if (!aligned4(parent) || !aligned4(used)) return LOBRA_ERR_ALIGN;
    LOBRA_HIP(beam_reorder(states, n_states, n_req, beams, parent, parent_ld, used, static_cast<hipStream_t>(hip_stream)));
    return LOBRA_OK;
}

}  // extern "C"
