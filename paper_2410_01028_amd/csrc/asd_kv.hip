// Host side of the operators over a paged cache of several sequences: argument checks, launch rules, the C ABI of asd.h.
#include "asd_kv_host.h"
#include "asd_kv_attend.h"
#include "asd_kv_plan.h"

// ---------------------------------------------------------------- rotary tables
// (cos, sin) of pos * frequency, in double; frequencies theta^(-2j / rot), changed for contexts longer than the trained one
// (turns of frequency f over the trained length: r = trained * f / 2 pi):
//   ASD_ROPE_LINEAR  f / factor
//   ASD_ROPE_BANDS   f where r >= high, f / factor where r <= low, in between mixed by (r - low) / (high - low)
//   ASD_ROPE_RAMP    mixed by the pair's index between the indexes that make `high` and `low` turns (rounded outwards), values times `gain`
struct RopeArgs { double theta, factor, low, high, trained, gain; int32_t rot, kind, positions; };
__global__ __launch_bounds__(256) void kv_rope_kernel(const RopeArgs a, float* out) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int hr = a.rot / 2;
    if (i >= (int64_t)a.positions * hr) return;
    const int j = (int)(i % hr), pos = (int)(i / hr);
    const double two_pi = 6.283185307179586476925;
    double f = pow(a.theta, -2.0 * j / a.rot);
    if (a.kind == ASD_ROPE_LINEAR) f /= a.factor;
    if (a.kind == ASD_ROPE_BANDS) {
        const double keep = fmin(1.0, fmax(0.0, (a.trained * f / two_pi - a.low) / (a.high - a.low)));
        f = keep * f + (1.0 - keep) * f / a.factor;
    }
    if (a.kind == ASD_ROPE_RAMP) {
        auto index = [&](double turns) { return a.rot * log(a.trained / (turns * two_pi)) / (2.0 * log(a.theta)); };
        const double lo = fmax(0.0, floor(index(a.high))), hi = fmin(a.rot - 1.0, ceil(index(a.low)));
        const double keep = 1.0 - fmin(1.0, fmax(0.0, (j - lo) / fmax(hi - lo, 1e-3)));
        f = keep * f + (1.0 - keep) * f / a.factor;
    }
    out[2 * i] = (float)(cos(pos * f) * a.gain);
    out[2 * i + 1] = (float)(sin(pos * f) * a.gain);
}

extern "C" {

size_t asd_kv_page_bytes(const asd_kv_shape* s) {
    if (shape_fault(s)) return 0;
    const int es = s->kv_dtype == ASD_DT_FP8 ? 1 : s->kv_dtype == ASD_DT_BF16 ? 2 : 4;
    return (size_t)s->n_kv_heads * (s->page_tokens / 64) * (128 * (size_t)s->head_dim * es + (es == 1 ? 128 : 0));
}

int asd_kv_append(const asd_kv_shape* s, const asd_kv_batch* b, const asd_kv_prep* p, const void* q, int64_t q_stride, const void* k,
                  int64_t k_stride, const void* v, int64_t v_stride, void* q_out, int64_t out_stride, void* hip_stream) {
    const char* why = shape_fault(s);
    if (!why) why = batch_fault(s, b);
    if (!why && !p) why = "prep is NULL";
    if (!why && (!k || !v)) why = "k and v must be device pointers";
    if (!why && !q != !q_out) why = "q and q_out go together";
    if (!why) why = rows_fault(s, k, k_stride, s->n_kv_heads);
    if (!why) why = rows_fault(s, v, v_stride, s->n_kv_heads);
    if (!why && q) why = rows_fault(s, q, q_stride, s->n_heads);
    if (!why && q) why = rows_fault(s, q_out, out_stride, s->n_heads);
    if (!why && (p->rot_dim < 0 || p->rot_dim > s->head_dim || p->rot_dim % (s->dtype == ASD_DT_BF16 ? 16 : 8))) why = "rot_dim must be a multiple of 16 (fp32 rows: 8) in 0..head_dim";
    if (!why && p->rot_dim && (!p->rope || (uintptr_t)p->rope % 16 || p->rope_positions < 1)) why = "rope must be a 16-byte aligned table of at least one position";
    if (!why && ((uintptr_t)p->q_gain | (uintptr_t)p->k_gain) % 16) why = "gains must be 16-byte aligned";
    if (!why && (p->q_gain || p->k_gain) && !(p->eps >= 0.f && std::isfinite(p->eps))) why = "eps must be a number >= 0";
    if (why) return refuse(ASD_E_INVAL, "asd_kv_append: %s", why);
    KvAppendArgs a{};
    a.kv = kv_args(s, b);
    a.q = q; a.k = k; a.v = v; a.q_out = q_out;
    a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride; a.out_stride = out_stride;
    a.q_gain = p->q_gain; a.k_gain = p->k_gain; a.rope = p->rope; a.eps = p->eps;
    a.rope_positions = p->rope_positions; a.rot = p->rot_dim;
    // Tiles of 64 tokens, whole chunks, where there are enough of them to fill the card (6900 tokens of 32 + 32 heads, with the rows read back:
    // 107 us, with tiles of 16 120 us; 20 tokens of 256 sequences 72 against 112); else tiles of 16, four times the workgroups.  (Rows are counted,
    // not tiles: one token of each of 1024 sequences gets tiles of 64, too, and takes 176 us, with tiles of 16 158; into bf16 pages 159 and 127.)
    const int64_t seqs = b->n_seqs < b->n_rows ? b->n_seqs : b->n_rows;
    const int tok = (int64_t)b->n_rows * s->n_kv_heads / 64 >= 2 * (int64_t)units() ? 64 : 16;
    const int most = b->max_new < tok ? b->max_new : tok;           // tokens of a tile
    const int pairs = APPEND_SLOTS(tok, s->head_dim * (s->kv_dtype == ASD_DT_FP8 ? 1 : s->kv_dtype == ASD_DT_BF16 ? 2 : 4));
    a.kv_heads_per = pairs / most < s->n_kv_heads ? pairs / most : s->n_kv_heads;
    if (a.kv_heads_per > 8) a.kv_heads_per = 8;
    a.q_heads_per = s->n_heads < 8 ? s->n_heads : 8;
    a.kv_blocks = (s->n_kv_heads + a.kv_heads_per - 1) / a.kv_heads_per;
    const int q_blocks = q ? (s->n_heads + a.q_heads_per - 1) / a.q_heads_per : 0;
    // tiles at positions divisible by tok: rows / tok and two more at a sequence's ends, but no more than it has rows
    const int64_t loose = b->n_rows / tok + 2 * seqs;
    a.blocks = 2 * a.kv_blocks + q_blocks;
    const int64_t grid = (loose < b->n_rows ? loose : b->n_rows) * a.blocks;
    if (grid > MOST_GROUPS) return refuse(ASD_E_INVAL, "asd_kv_append: the batch is too large");
    by_shape(s, [&](auto t, auto c, auto h) {
        auto go = [&](auto tiles, auto inter) { kv_append_kernel<decltype(t), decltype(c), h.value, tiles.value, inter.value><<<(unsigned)grid, 256, 0, (hipStream_t)hip_stream>>>(a); };
        auto turned = [&](auto tiles) { if (p->interleaved && p->rot_dim) go(tiles, std::true_type{}); else go(tiles, std::false_type{}); };
        if (tok == 64) turned(std::integral_constant<int, 64>{}); else turned(std::integral_constant<int, 16>{});
    });
    return launched("asd_kv_append");
}

size_t asd_kv_attend_workspace(const asd_kv_shape* s, const asd_kv_batch* b) {
    if (shape_fault(s) || batch_fault(s, b)) return 0;
    return attend_plan(s, b, whole_lengths(s, b)).bytes;
}

int asd_kv_attend(const asd_kv_shape* s, const asd_kv_batch* b, const void* q, int64_t q_stride, void* out, int64_t out_stride, float scale,
                  void* workspace, size_t workspace_bytes, void* hip_stream) {
    const char* why = shape_fault(s);
    if (!why) why = batch_fault(s, b);
    if (!why && (!q || !out)) why = "q and out must be device pointers";
    if (!why) why = rows_fault(s, q, q_stride, s->n_heads);
    if (!why) why = rows_fault(s, out, out_stride, s->n_heads);
    const float c2 = (float)((double)scale * 1.4426950408889634074);      // log2(e)
    if (!why && !(scale > 0.f && std::isfinite(c2))) why = "scale must be a positive number, scale * log2(e) too";
    if (why) return refuse(ASD_E_INVAL, "asd_kv_attend: %s", why);
    const AttendPlan p = attend_plan(s, b, whole_lengths(s, b));
    if (p.bytes && (!workspace || (uintptr_t)workspace % 256)) return refuse(ASD_E_INVAL, "asd_kv_attend: workspace must be 256-byte aligned");
    if (workspace_bytes < p.bytes) return refuse(ASD_E_NOMEM, "asd_kv_attend: workspace too small: %zu bytes given, %zu needed", workspace_bytes, p.bytes);
    if (p.grid > MOST_GROUPS) return refuse(ASD_E_INVAL, "asd_kv_attend: the batch is too large");
    KvAttendArgs a{};
    a.kv = kv_args(s, b);
    a.q = q; a.out = out; a.q_stride = q_stride; a.out_stride = out_stride;
    a.c2 = c2;
    a.o_part = (float*)workspace; a.ml_part = (float*)((char*)workspace + p.o_bytes);
    a.target = p.target; a.cut = p.join; a.min_run = p.min_run;
    const hipStream_t stream = (hipStream_t)hip_stream;
    const dim3 join_grid((unsigned)((int64_t)p.max_tiles * s->n_kv_heads), p.nt);
    auto go = [&](auto t, auto c, auto h, auto nt) {
        kv_attend_kernel<decltype(t), decltype(c), h.value, nt.value><<<(unsigned)p.grid, 256, 0, stream>>>(a);
        if (p.join) kv_join_kernel<decltype(t), h.value, nt.value><<<join_grid, 256, 0, stream>>>(a);
    };
    by_shape(s, [&](auto t, auto c, auto h) {
        using T = decltype(t);
        using C = decltype(c);
        constexpr bool bf16 = T::KE == 8, q8 = sizeof(typename C::elem) == 1;
        if (p.nt == 1) go(t, c, h, std::integral_constant<int, 1>{});
        if constexpr (bf16 != q8) { if (p.nt == 2) go(t, c, h, std::integral_constant<int, 2>{}); }
        if constexpr (bf16 && h.value >= 64) {
            if (p.nt == 8) {
                kv_rows_kernel<C, h.value, 2, 4><<<(unsigned)p.grid, 256, 0, stream>>>(a);
                if (p.join) kv_join_kernel<T, h.value, 8><<<join_grid, 256, 0, stream>>>(a);
            }
        }
    });
    return launched("asd_kv_attend");
}

int asd_kv_read(const asd_kv_shape* s, const asd_kv_batch* b, void* k_out, int64_t k_stride, void* v_out, int64_t v_stride, void* hip_stream) {
    const char* why = shape_fault(s);
    if (!why) why = batch_fault(s, b);
    if (!why && k_out) why = rows_fault(s, k_out, k_stride, s->n_kv_heads);
    if (!why && v_out) why = rows_fault(s, v_out, v_stride, s->n_kv_heads);
    if (why) return refuse(ASD_E_INVAL, "asd_kv_read: %s", why);
    if (!k_out && !v_out) return ASD_OK;
    KvReadArgs a{};
    a.kv = kv_args(s, b);
    a.k_out = k_out; a.v_out = v_out; a.k_stride = k_stride; a.v_stride = v_stride;
    const int64_t seqs = b->n_seqs < b->n_rows ? b->n_seqs : b->n_rows, loose = b->n_rows / 64 + 2 * seqs;
    const int64_t most = loose < b->n_rows ? loose : b->n_rows;
    if (most > MOST_GROUPS) return refuse(ASD_E_INVAL, "asd_kv_read: the batch is too large");
    const dim3 grid((unsigned)most, s->n_kv_heads, 2);
    by_shape(s, [&](auto t, auto c, auto h) { kv_read_kernel<decltype(t), decltype(c), h.value><<<grid, 256, 0, (hipStream_t)hip_stream>>>(a); });
    return launched("asd_kv_read");
}

int asd_rope_table(const asd_rope* r, int32_t positions, float* table, void* hip_stream) {
    const char* why = nullptr;
    if (!r || !table || (uintptr_t)table % 16) why = "rope and table (16-byte aligned) must be given";
    else if (r->kind < ASD_ROPE_PLAIN || r->kind > ASD_ROPE_RAMP) why = "unknown kind";
    else if (r->rot_dim < 8 || r->rot_dim % 8 || r->rot_dim > 128) why = "rot_dim must be a multiple of 8 in 8..128";
    else if (positions < 1 || positions > 1 << 24) why = "positions must be in 1..2^24";
    else if (!(r->theta > 1.0) || !std::isfinite(r->theta)) why = "theta must be above 1";
    else if (r->kind != ASD_ROPE_PLAIN && (!(r->factor >= 1.0) || !std::isfinite(r->factor))) why = "factor must be at least 1";
    else if (r->kind >= ASD_ROPE_BANDS && !(r->low > 0.0 && r->high > r->low && std::isfinite(r->high) && r->trained >= 1.0 && std::isfinite(r->trained))) why = "0 < low < high and trained >= 1 are needed";
    else if (!(r->gain >= 0.0) || !std::isfinite(r->gain)) why = "gain must be a number >= 0";
    if (why) return refuse(ASD_E_INVAL, "asd_rope_table: %s", why);
    const RopeArgs a{r->theta, r->factor, r->low, r->high, r->trained, r->gain == 0.0 ? 1.0 : r->gain, r->rot_dim, r->kind, positions};
    kv_rope_kernel<<<(unsigned)(((int64_t)positions * (r->rot_dim / 2) + 255) / 256), 256, 0, (hipStream_t)hip_stream>>>(a, table);
    return launched("asd_rope_table");
}

}  // extern "C"
