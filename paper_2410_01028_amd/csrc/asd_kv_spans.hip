// Host side of the attention with a window and of the attention of sequences that begin with the same tokens (asd.h).
#include "asd_kv_host.h"
#include "asd_kv_plan.h"
#include "asd_kv_spans.h"

namespace {

const char* attend_fault(const asd_kv_shape* s, const asd_kv_batch* b, const void* q, int64_t q_stride, const void* out, int64_t out_stride, float scale) {
    const char* why = shape_fault(s);
    if (!why) why = batch_fault(s, b);
    if (!why && (!q || !out)) why = "q and out must be device pointers";
    if (!why) why = rows_fault(s, q, q_stride, s->n_heads);
    if (!why) why = rows_fault(s, out, out_stride, s->n_heads);
    const float c2 = (float)((double)scale * 1.4426950408889634074);      // log2(e)
    if (!why && !(scale > 0.f && std::isfinite(c2))) why = "scale must be a positive number, scale * log2(e) too";
    return why;
}
const char* window_fault(int32_t window, int32_t sinks) {
    if (window < 1) return "window must be positive";
    if (sinks < 0) return "sinks must be 0 or more";
    return nullptr;
}
const char* groups_fault(const asd_kv_groups* g) {
    if (!g) return "groups is NULL";
    if (!g->group_start || !g->shared_len) return "group_start and shared_len must be device pointers";
    if (((uintptr_t)g->group_start | (uintptr_t)g->shared_len) % 4) return "the groups' arrays must be 4-byte aligned";
    if (g->n_groups < 1 || g->n_groups > 65536) return "n_groups must be in 1..65536";
    return nullptr;
}
int room(const char* what, size_t need, const void* workspace, size_t bytes) {
    if (need && (!workspace || (uintptr_t)workspace % 256)) return refuse(ASD_E_INVAL, "%s: workspace must be 256-byte aligned", what);
    if (bytes < need) return refuse(ASD_E_NOMEM, "%s: workspace too small: %zu bytes given, %zu needed", what, bytes, need);
    return ASD_OK;
}
void attend_args(KvAttendArgs* a, const asd_kv_shape* s, const asd_kv_batch* b, const void* q, int64_t q_stride, void* out, int64_t out_stride, float scale) {
    a->kv = kv_args(s, b);
    a->q = q; a->out = out; a->q_stride = q_stride; a->out_stride = out_stride;
    a->c2 = (float)((double)scale * 1.4426950408889634074);
}

int32_t at_most(int32_t x, int32_t most) { return x < most ? x : most; }
// the notes on the rows that may be joined, in front of the partial sums
size_t notes_bytes(const AttendPlan& p) { return (64 + (size_t)p.join_blocks * sizeof(KvNote) + 255) / 256 * 256; }
AttendPlan window_plan(const asd_kv_shape* s, const asd_kv_batch* b, int32_t window, int32_t sinks) {
    const int64_t cap = kv_args(s, b).cap, chunks = (cap + 63) / 64, group = s->n_heads / s->n_kv_heads;
    return attend_plan(s, b, [=](int rows) {           // as kv_window_chunks
        const int64_t most = rows % group ? (rows + group - 2) / group + 1 : rows / group, tokens = most < b->max_new ? most : b->max_new;
        const int64_t n = ((int64_t)at_most(sinks, (int32_t)cap) + 63) / 64 + (at_most(window, (int32_t)cap) + tokens + 125) / 64;
        return n < chunks ? n : chunks;
    }, PLAN_EVEN);
}
// Groups either way: `apart`, the shared keys read once for the rows of all sequences of a group, and each sequence's own; or, with `own` alone, each
// sequence's tiles walk both.
struct SharedPlan {
    bool apart;
    AttendPlan front, own;
    size_t front_at, own_at, bytes;                     // (the notes lie in front)
};
SharedPlan shared_plan(const asd_kv_shape* s, const asd_kv_batch* b, const asd_kv_groups* g) {
    SharedPlan p{};
    const int64_t chunks = (kv_args(s, b).cap + 63) / 64, group = s->n_heads / s->n_kv_heads;
    // Apart every row's parts are joined, and own keys are items of a wave each.  Worth it where the sequences' tiles are not full by themselves (64 rows on average) and, walking both, would
    // read much more than there is (64 / 8 heads, 8 bits, one token of 64 sequences behind 4000 shared ones and up to 300 own: 36 us, walking both 63; of 4 behind 1000: 14.7 and 13.1;
    // 130 rows of 24 sequences: 309 and 272).  The bounds do not say what is shared.  Where it is little beside the own keys the two are nearly even, and causal attention over tables that
    // hold the common pages is ahead: 50, 500, 2000 shared tokens, one token of 16 sequences with up to 4000 of their own 30, 30, 30 us, walking both 27, 28, 38, causal 27, 27, 34; of 64
    // with up to 8000 116, 115, 128 and 116, 115, 123, causal 106, 109, 117.  1024 sequences with up to 200 of their own in 256 groups of 1000: 485 and 550, causal 332 (in 32 groups 292, 479, 302).
    const int64_t cap = kv_args(s, b).cap, read = b->n_seqs * cap * (int64_t)(asd_kv_page_bytes(s) / s->page_tokens);
    p.apart = b->n_seqs / 2 >= g->n_groups && b->n_rows * group <= 64 * (int64_t)b->n_seqs && ((cap >= 512 && read >= 40 << 20) || read >= 256 << 20);
    if (!p.apart) {
        p.own = attend_plan(s, b, [=](int) { return chunks + 1; }, PLAN_BOTH);      // (the chunk in which the shared tokens end comes twice)
        p.bytes = p.own.join ? notes_bytes(p.own) + p.own.bytes : 0;
        p.own_at = notes_bytes(p.own);
        return p;
    }
    asd_kv_batch rows = *b;                             // a group is one sequence to its shared keys
    rows.n_seqs = g->n_groups;
    rows.max_new = (b->n_rows + g->n_groups - 1) / g->n_groups;      // (on average: a rule's, no bound)
    p.front = attend_plan(s, &rows, [=](int) { return chunks; }, PLAN_FRONT);
    p.own = attend_plan(s, b, [=](int) { return chunks; }, PLAN_WAVE);
    // every tile has a place, cut or not
    for (AttendPlan* x : {&p.front, &p.own}) {
        x->o_bytes = ((size_t)x->grid * 16 * x->nt * s->head_dim * 4 + 255) / 256 * 256;
        x->bytes = (x->o_bytes + (size_t)x->grid * 16 * x->nt * 8 + 255) / 256 * 256;
    }
    p.front_at = notes_bytes(p.own);
    p.own_at = p.front_at + p.front.bytes;
    p.bytes = p.own_at + p.own.bytes;
    return p;
}

}  // namespace

extern "C" {

size_t asd_kv_attend_window_workspace(const asd_kv_shape* s, const asd_kv_batch* b, int32_t window, int32_t sinks) {
    if (shape_fault(s) || batch_fault(s, b) || window_fault(window, sinks)) return 0;
    const AttendPlan p = window_plan(s, b, window, sinks);
    return p.join ? notes_bytes(p) + p.bytes : 0;
}

int asd_kv_attend_window(const asd_kv_shape* s, const asd_kv_batch* b, int32_t window, int32_t sinks, const void* q, int64_t q_stride, void* out,
                         int64_t out_stride, float scale, void* workspace, size_t workspace_bytes, void* hip_stream) {
    static const char* const name = "asd_kv_attend_window";
    const char* why = attend_fault(s, b, q, q_stride, out, out_stride, scale);
    if (!why) why = window_fault(window, sinks);
    if (why) return refuse(ASD_E_INVAL, "%s: %s", name, why);
    const AttendPlan p = window_plan(s, b, window, sinks);
    if (const int rc = room(name, p.join ? notes_bytes(p) + p.bytes : 0, workspace, workspace_bytes)) return rc;
    if (p.grid > MOST_GROUPS || p.join_blocks > MOST_GROUPS) return refuse(ASD_E_INVAL, "%s: the batch is too large", name);
    KvWindowArgs a{};
    attend_args(&a, s, b, q, q_stride, out, out_stride, scale);
    KvNotes* notes = (KvNotes*)workspace;
    a.o_part = (float*)((char*)workspace + notes_bytes(p)); a.ml_part = (float*)((char*)a.o_part + p.o_bytes);
    a.target = p.target; a.cut = p.join; a.tail = p.tail; a.min_run = p.min_run; a.tile_rows = 16 * p.nt;
    a.window = at_most(window, a.kv.cap); a.sinks = at_most(sinks, a.kv.cap);
    const hipStream_t stream = (hipStream_t)hip_stream;
    by_shape(s, [&](auto t, auto c, auto h) {
        using T = decltype(t);
        using C = decltype(c);
        constexpr bool bf16 = T::KE == 8, q8 = sizeof(typename C::elem) == 1;
        if (p.nt == 1) kv_window_kernel<T, C, h.value, 1><<<(unsigned)p.grid, 256, 0, stream>>>(a, notes);
        if constexpr (bf16 != q8) { if (p.nt == 2) kv_window_kernel<T, C, h.value, 2><<<(unsigned)p.grid, 256, 0, stream>>>(a, notes); }
        if constexpr (bf16 && h.value >= 64) { if (p.nt == 8) kv_window_rows_kernel<C, h.value, 2, 4><<<(unsigned)p.grid, 256, 0, stream>>>(a, notes); }
        if (p.join) kv_parts_kernel<T, h.value><<<(unsigned)p.join_blocks, 256, 0, stream>>>(a, notes, nullptr, nullptr, 16);
    });
    return launched(name);
}

size_t asd_kv_attend_shared_workspace(const asd_kv_shape* s, const asd_kv_batch* b, const asd_kv_groups* g) {
    if (shape_fault(s) || batch_fault(s, b) || groups_fault(g)) return 0;
    return shared_plan(s, b, g).bytes;
}

int asd_kv_attend_shared(const asd_kv_shape* s, const asd_kv_batch* b, const asd_kv_groups* g, const void* q, int64_t q_stride, void* out,
                         int64_t out_stride, float scale, void* workspace, size_t workspace_bytes, void* hip_stream) {
    static const char* const name = "asd_kv_attend_shared";
    const char* why = attend_fault(s, b, q, q_stride, out, out_stride, scale);
    if (!why) why = groups_fault(g);
    if (why) return refuse(ASD_E_INVAL, "%s: %s", name, why);
    const SharedPlan p = shared_plan(s, b, g);
    if (const int rc = room(name, p.bytes, workspace, workspace_bytes)) return rc;
    if (p.front.grid + p.own.grid > MOST_GROUPS || p.own.join_blocks > MOST_GROUPS) return refuse(ASD_E_INVAL, "%s: the batch is too large", name);
    KvSharedArgs a{};
    attend_args(&a, s, b, q, q_stride, out, out_stride, scale);
    a.group_start = g->group_start; a.shared_len = g->shared_len; a.n_groups = g->n_groups;
    KvNotes* notes = (KvNotes*)workspace;
    a.front_o = (float*)((char*)workspace + p.front_at); a.front_ml = (float*)((char*)a.front_o + p.front.o_bytes);
    a.o_part = (float*)((char*)workspace + p.own_at); a.ml_part = (float*)((char*)a.o_part + p.own.o_bytes);
    a.front_target = p.front.target; a.front_min_run = p.front.min_run; a.front_cut = p.front.join; a.front_rows = 16 * p.front.nt; a.front_grid = (int32_t)p.front.grid;
    a.target = p.own.target; a.cut = p.own.join; a.tail = p.own.tail; a.min_run = p.own.min_run; a.tile_rows = 16 * p.own.nt;
    const hipStream_t stream = (hipStream_t)hip_stream;
    by_shape(s, [&](auto t, auto c, auto h) {
        using T = decltype(t);
        using C = decltype(c);
        constexpr bool bf16 = T::KE == 8, q8 = sizeof(typename C::elem) == 1;
        if (p.apart) {
            const unsigned grid = (unsigned)(p.front.grid + (p.own.grid + 3) / 4);
            if (p.front.nt == 1) kv_apart_kernel<T, C, h.value, 1><<<grid, 256, 0, stream>>>(a, notes);
            if constexpr (bf16 != q8) { if (p.front.nt == 2) kv_apart_kernel<T, C, h.value, 2><<<grid, 256, 0, stream>>>(a, notes); }
            if constexpr (bf16 && h.value >= 64) { if (p.front.nt == 8) kv_apart_kernel<T, C, h.value, 8><<<grid, 256, 0, stream>>>(a, notes); }
        } else {
            const unsigned grid = (unsigned)p.own.grid;
            if (p.own.nt == 1) kv_both_kernel<T, C, h.value, 1><<<grid, 256, 0, stream>>>(a, notes);
            if constexpr (bf16 != q8) { if (p.own.nt == 2) kv_both_kernel<T, C, h.value, 2><<<grid, 256, 0, stream>>>(a, notes); }
            if constexpr (bf16 && h.value >= 64) { if (p.own.nt == 8) kv_both_rows_kernel<C, h.value, 2, 4><<<grid, 256, 0, stream>>>(a, notes); }
        }
        if (p.apart || p.own.join) kv_parts_kernel<T, h.value><<<(unsigned)p.own.join_blocks, 256, 0, stream>>>(a, notes, a.front_o, a.front_ml, a.front_rows);
    });
    return launched(name);
}

}  // extern "C"
