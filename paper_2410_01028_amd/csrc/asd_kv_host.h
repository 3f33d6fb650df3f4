// What the host sides of the operators over a paged cache share: refusals, argument checks, launches by type and width.
#pragma once
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

}  // namespace
