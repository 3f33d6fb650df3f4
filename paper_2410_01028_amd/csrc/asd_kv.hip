// Host side of the operators over a paged cache of several sequences: argument checks, launch rules, the C ABI of asd.h.
#include "../../include/asd.h"
#include "asd_kv.h"

#include <cmath>
#include <cstdarg>
#include <cstdio>

__attribute__((visibility("hidden"))) void asd_note_error(const char* message);

namespace {

int refuse(int code, const char* fmt, ...) {
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    try { asd_note_error(buf); } catch (...) {}
    return code;
}

const char* shape_fault(const asd_kv_shape* s) {
    if (!s) return "shape is NULL";
    if (s->n_heads < 1 || s->n_kv_heads < 1 || s->n_heads % s->n_kv_heads) return "n_heads must be a positive multiple of n_kv_heads";
    if (s->n_heads > 4096) return "more than 4096 heads";
    if (s->head_dim != 32 && s->head_dim != 64 && s->head_dim != 128) return "head_dim must be 32, 64 or 128";
    if (s->page_tokens < 64 || s->page_tokens % 64 || s->page_tokens > 1 << 24) return "page_tokens must be a positive multiple of 64";
    if (s->dtype != ASD_DT_F32 && s->dtype != ASD_DT_BF16) return "dtype must be ASD_DT_F32 or ASD_DT_BF16";
    if (s->kv_dtype != s->dtype && s->kv_dtype != ASD_DT_FP8) return "kv_dtype must be dtype or ASD_DT_FP8";
    return nullptr;
}

const char* batch_fault(const asd_kv_shape* s, const asd_kv_batch* b) {
    if (!b) return "batch is NULL";
    if (!b->pages || (uintptr_t)b->pages % 16) return "pages must be a device pointer, 16-byte aligned";
    if (!b->page_table || !b->row_start || !b->kv_len) return "page_table, row_start and kv_len must be device pointers";
    if (((uintptr_t)b->page_table | (uintptr_t)b->row_start | (uintptr_t)b->kv_len | (uintptr_t)b->status) % 4) return "the batch's arrays must be 4-byte aligned";
    if (b->n_pages < 1 || b->table_stride < 1) return "n_pages and table_stride must be positive";
    if (b->n_seqs < 1 || b->n_seqs > 65536) return "n_seqs must be in 1..65536";
    if (b->n_rows < 1 || (int64_t)b->n_rows * s->n_heads >= (int64_t)1 << 31) return "n_rows must be positive, and n_rows * n_heads below 2^31";
    if (b->max_new < 1 || b->max_new > b->n_rows) return "max_new must be in 1..n_rows";
    if (b->max_len < 1 || b->max_len > 1 << 24) return "max_len must be in 1..2^24";
    return nullptr;
}

// a buffer of rows: pointer, stride from row to row, heads of a row
const char* rows_fault(const asd_kv_shape* s, const void* p, int64_t stride, int heads) {
    const int es = s->dtype == ASD_DT_BF16 ? 2 : 4;
    if ((uintptr_t)p % 16 || stride * es % 16) return "row pointers and strides must be multiples of 16 bytes";
    if (stride < (int64_t)heads * s->head_dim || stride > (int64_t)1 << 40) return "a row stride is smaller than a row";
    return nullptr;
}

KvArgs kv_args(const asd_kv_shape* s, const asd_kv_batch* b) {
    KvArgs a{};
    a.pages = (char*)b->pages; a.table = b->page_table; a.row_start = b->row_start; a.kv_len = b->kv_len; a.status = b->status;
    a.n_pages = b->n_pages; a.table_stride = b->table_stride; a.n_seqs = b->n_seqs; a.n_rows = b->n_rows; a.max_new = b->max_new;
    const int64_t reach = (int64_t)b->table_stride * s->page_tokens;
    a.cap = (int32_t)(reach < b->max_len ? reach : b->max_len);
    a.n_h = s->n_heads; a.n_kv = s->n_kv_heads; a.group = s->n_heads / s->n_kv_heads; a.page_tokens = s->page_tokens;
    return a;
}

// f<row type, cache type, head dim>() for the shape
template <class F> void by_shape(const asd_kv_shape* s, F f) {
    auto dim = [&](auto t, auto c) {
        if (s->head_dim == 32) f(t, c, std::integral_constant<int, 32>{});
        else if (s->head_dim == 64) f(t, c, std::integral_constant<int, 64>{});
        else f(t, c, std::integral_constant<int, 128>{});
    };
    const bool q8 = s->kv_dtype == ASD_DT_FP8;
    if (s->dtype == ASD_DT_BF16) { if (q8) dim(BF16{}, FP8{}); else dim(BF16{}, BF16{}); }
    else { if (q8) dim(F32{}, FP8{}); else dim(F32{}, F32{}); }
}

int launched(const char* what) {
    const hipError_t r = hipGetLastError();
    return r == hipSuccess ? ASD_OK : refuse(ASD_E_HIP, "%s: %s", what, hipGetErrorString(r));
}

int units() {
    static const int n = [] {
        int dev = 0, v = 0;
        return hipGetDevice(&dev) == hipSuccess && hipDeviceGetAttribute(&v, hipDeviceAttributeMultiprocessorCount, dev) == hipSuccess && v > 0 ? v : 256;
    }();
    return n;
}

// Workgroups of 256 that a launch can have: its threads are counted in 32 bits
constexpr int64_t MOST_GROUPS = ((int64_t)1 << 32) / 256 - 1;

// How asd_kv_attend runs a batch of these bounds
struct AttendPlan {
    int nt;                        // 16-row column blocks of a tile
    bool rows;                     // kv_rows_kernel
    int32_t target, max_tiles, min_run;
    int64_t grid;                  // most work items
    bool join;                     // some sequence's keys may be cut
    size_t o_bytes, bytes;
};
AttendPlan attend_plan(const asd_kv_shape* s, const asd_kv_batch* b) {
    AttendPlan p{};
    const int group = s->n_heads / s->n_kv_heads;
    const int64_t rows = (int64_t)b->max_new * group, chunks = (kv_args(s, b).cap + 63) / 64;
    const bool bf16 = s->dtype == ASD_DT_BF16, q8 = s->kv_dtype == ASD_DT_FP8;
    const int64_t seqs = b->n_seqs < b->n_rows ? b->n_seqs : b->n_rows;
    auto tiles = [&](int nt) { return (int64_t)b->n_rows * group / (16 * nt) + seqs; };      // the most that there can be
    // Which kernel.  kv_attend_kernel's workgroups are many and short, its tiles read a sequence's pages again for every 16 rows (mostly from L2);
    // kv_rows_kernel reads them once for 128 rows, with a step's cost whether they are all in use or not.  Up to 32 rows (new tokens x heads of a group)
    // the first one, whatever the lengths (64 sequences of 4 new tokens, 4000 in all, 64 / 8 heads x 128: 8 bits 131 us against 171, bf16 pages 191
    // against 217).  Above, the second one where the first has more than two rounds of workgroups (16 sequences of 40 new tokens, 128 in all, 32 / 32
    // heads: 13 us against 23, 14 against 25) or more than 64 chunks per compute unit (two sequences of 100 new tokens, 32 / 32 heads, 4000 in all:
    // 42 against 62, 41 against 71; with 1000 in all 33 against 17, 29 against 19).
    const int64_t work = tiles(1) * s->n_kv_heads;
    p.rows = bf16 && s->head_dim >= 64 && rows > 32 && (work > 4 * (int64_t)units() || work * chunks > 64 * (int64_t)units());
    // 16 rows to a tile; 32 where a fragment's second use is worth more than twice the workgroups: bf16 pages of some length (64 sequences of 3 new tokens,
    // 4000 in all, 64 / 8 heads x 128: 187 us against 269; 8 bits 142 against 135), and codes widened for fp32 products in a batch that fills the card
    // (four prompts of 500, 32 / 32 heads x 128: 186 against 224; with 8 / 8 heads, just below the border, the rule's 63 against 57).
    p.nt = rows <= 16 ? 1 : bf16 ? (!q8 && chunks >= 8 ? 2 : 1) : (q8 && (int64_t)b->n_rows * s->n_heads / 32 >= 2 * units() ? 2 : 1);
    if (p.rows) p.nt = 8;
    p.max_tiles = (int32_t)tiles(p.nt);
    // Keys are cut into about four items per compute unit (48 sequences of 500 to 8192 tokens: 90 us, with two 100, with eight 97), but not
    // into runs of fewer than 16 chunks (with 8, five rows of eight sequences of 1031 tokens take 19.1 us, not 16.9), and not where
    // kv_rows_kernel's tiles are as many by themselves: full ones, or, as long as none is long, ones that a token alone may have.  (64 / 8 heads x 128,
    // 8 bits, 128 tokens behind 400, 512 rows behind 3488 and a token behind 4000: 164 us, cut 177; behind 8192: 245 and 178; behind 60000: 1493
    // and 221.  128 tokens behind 400 .. 8192 and the 512 rows: 402 and 428, behind 400 .. 16384 734 and 703)
    p.min_run = 16;
    p.target = 4 * units();
    const int64_t whole = (int64_t)p.max_tiles * s->n_kv_heads, full = (int64_t)b->n_rows * group / (16 * p.nt) * s->n_kv_heads;
    const int64_t most = (chunks + p.min_run / 2) / p.min_run;      // runs of the longest sequence
    p.join = most > 1 && !(p.rows && (full >= p.target || (whole >= p.target && chunks < 128)));
    p.grid = p.join ? whole + p.target : whole;
    if (p.join && whole * most < p.grid) p.grid = whole * most;
    if (p.join) {
        p.o_bytes = ((size_t)p.grid * 16 * p.nt * s->head_dim * 4 + 255) / 256 * 256;
        p.bytes = p.o_bytes + (size_t)p.grid * 16 * p.nt * 8;
    }
    return p;
}

}  // namespace

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
    return attend_plan(s, b).bytes;
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
    const AttendPlan p = attend_plan(s, b);
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
