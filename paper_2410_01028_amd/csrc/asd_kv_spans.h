// Two more forms of attention over a paged cache of several sequences: with a sliding window and first tokens that stay visible
// (asd_kv_attend_window), and for groups of sequences that begin with the same tokens (asd_kv_attend_shared).  The work on a tile is
// kv_few_rows and kv_many_rows (asd_kv_attend.h); here is which tiles and runs of keys there are.
#pragma once
#include "asd_kv_attend.h"

// tiles of `rows` rows
__device__ __forceinline__ int kv_tiles_of(const KvArgs& a, const KvSeq& v, int rows) { return (int)(((uint32_t)v.n * a.group + rows - 1) / (uint32_t)rows); }
// the run of all entries of x, bad ones as they are mended: no more items than the plan has room for, whatever `chunks` says
template <class Lanes, class F> __device__ __forceinline__ int kv_run_all(const KvAttendArgs& a, Lanes x, int lane, int rows, F chunks) {
    if (!a.cut) return 1 << 28;
    int64_t t = 0;
    for (int s0 = 0;;) {
        t += (int64_t)kv_tiles_of(a.kv, x.v, rows) * chunks(x.v);
        s0 += 64;
        if (s0 >= x.entries(a.kv)) break;
        x.load(a.kv, s0, lane, false);
    }
    return kv_run_of(a, wave_sum(t));
}
// items of the entries in front of entry n
template <class Lanes, class F> __device__ __forceinline__ int64_t kv_items_before(const KvArgs& a, Lanes x, int n, int lane, F count) {
    int64_t t = 0;
    for (int s0 = 0; s0 < n; s0 += 64) {
        if (s0) x.load(a, s0, lane, false);
        t += s0 + lane < n ? count(x.v) : 0;
    }
    return wave_sum(t);
}
// item `local` of an entry: its run, tile and KV head.  last_first: the tiles that see most come first
__device__ __forceinline__ void kv_place_item(KvItem& it, int local, int64_t first, int n_tiles, int n_kv, bool last_first) {
    const int tile = local / n_kv % n_tiles;
    it.kvh = local % n_kv; it.tile = last_first ? n_tiles - 1 - tile : tile; it.split = local / n_kv / n_tiles;
    it.part = first + (int64_t)(it.split * n_tiles + it.tile) * n_kv + it.kvh;
}

// ---------------------------------------------------------------- a sliding window and the first tokens
// The chunks that the tiles of R rows of a sequence walk at most: those of the first tokens, and those from the first row's window on to the last row
__device__ __forceinline__ int kv_window_chunks(const KvWindowArgs& a, const KvSeq& v, int R) {
    const int whole = (v.len + 63) / 64, sink = (a.sinks + 63) / 64, group = a.kv.group;
    if ((int64_t)v.n * group <= R) {                    // one tile: as it is
        const int first = max(v.len - v.n - a.window + 1, 0) / 64;
        return sink < first ? whole - first + sink : whole;
    }
    const int tokens = min(v.n, R % group ? (R + group - 2) / group + 1 : R / group);
    return min(whole, sink + (a.window + tokens + 125) / 64);
}
template <int R, class F> __device__ __forceinline__ bool kv_window_item(const KvWindowArgs& a, KvItem& it, F) {
    const int lane = threadIdx.x & 63, n_kv = a.kv.n_kv;
    int local;
    int64_t first;
    const bool check = blockIdx.x == 0 && threadIdx.x < 64;
    KvLanes all;
    all.load(a.kv, 0, lane, check);
    auto chunks = [&](const KvSeq& v) { return kv_window_chunks(a, v, R); };
    const int run = kv_run_all(a, all, lane, R, chunks);
    if (!kv_find(a.kv, all, blockIdx.x, lane, check, [&](const KvSeq& v) { return kv_tiles_of(a.kv, v, R) * kv_splits(chunks(v), run) * n_kv; }, &it.seq, &local, &first, &it.s)) return false;
    const int n_splits = kv_splits(chunks(it.s), run);
    kv_place_item(it, local, first, kv_tiles_of(a.kv, it.s, R), n_kv, F::value);
    it.per = kv_per_split(chunks(it.s), n_splits);
    it.whole = n_splits == 1;
    return true;
}
template <class A, class C, int H, int NT>
__global__ __launch_bounds__(256, A::KE == 4 ? 1 : 2) void kv_window_kernel(const KvWindowArgs a) {
    __shared__ KvFewLds<H> lds;
    KvItem it;
    if (kv_window_item<16 * NT>(a, it, std::false_type{})) kv_few_rows<A, C, H, NT, KV_WINDOW>(a, it, lds);
}
template <class C, int H, int NT, int NW>
__global__ __launch_bounds__(64 * NW, 2) void kv_window_rows_kernel(const KvWindowArgs a) {
    __shared__ u32x4 mem[KV_RING<C, H>];
    KvItem it;
    if (kv_window_item<16 * NT * NW>(a, it, std::true_type{})) kv_many_rows<C, H, NT, NW, KV_WINDOW>(a, it, mem);
}
template <class A, int H>
__global__ __launch_bounds__(256) void kv_window_join_kernel(const KvWindowArgs a) {
    const int lane = threadIdx.x & 63, n_kv = a.kv.n_kv, group = a.kv.group, R = a.tile_rows;
    int seq, local;
    int64_t first;
    KvSeq s;
    KvLanes all;
    all.load(a.kv, 0, lane, false);
    auto chunks = [&](const KvSeq& v) { return kv_window_chunks(a, v, R); };
    const int run = kv_run_all(a, all, lane, R, chunks);
    // 16 rows of a cut sequence and KV head
    if (!kv_find(a.kv, all, blockIdx.x, lane, false, [&](const KvSeq& v) { return kv_splits(chunks(v), run) > 1 ? kv_tiles_of(a.kv, v, 16) * n_kv : 0; }, &seq, &local, &first, &s)) return;
    const int64_t item0 = kv_items_before(a.kv, all, seq, lane, [&](const KvSeq& v) { return (int64_t)kv_tiles_of(a.kv, v, R) * kv_splits(chunks(v), run) * n_kv; });
    const int n_splits = kv_splits(chunks(s), run), n_tiles = kv_tiles_of(a.kv, s, R), kvh = local % n_kv, row0 = local / n_kv * 16;
    const int64_t step = (int64_t)n_tiles * n_kv * R, at = (item0 + (int64_t)(row0 / R) * n_kv + kvh) * R + row0 % R;
    kv_join_rows<A, H>(a, s, kvh, row0, min(s.n * group - row0, 16), n_splits, [&](int i, int r) { const int64_t p = at + r + i * step; return KvPartial{a.o_part + p * H, a.ml_part + p * 2}; });
}

// ---------------------------------------------------------------- sequences that begin with the same tokens
// The keys that a group shares are read once for the rows of all its sequences: these lie one behind the other, so that a group is to its shared keys what a
// sequence is to its own, all rows seeing all of them.  The keys behind them are each sequence's own.  Every row's sums come in two
// parts at least, put together in a launch of their own.
struct KvSharedArgs : KvAttendArgs {                    // (o_part .. cut: of the own keys)
    const int32_t *group_start, *shared_len;
    int32_t n_groups;
    int32_t front_target, front_cut, front_rows;
    float *front_o, *front_ml;
    __device__ __forceinline__ KvAttendArgs front() const {
        KvAttendArgs f = *this;
        f.o_part = front_o; f.ml_part = front_ml; f.target = front_target; f.cut = front_cut;
        return f;
    }
};
// the largest of the lanes in front of this one, and of what came before (top, which takes them all in)
__device__ __forceinline__ int kv_max_before(int x, int& top, int lane) {
    x = wave_max_upto(x);
    const int t = __shfl_up(x, 1), before = lane ? max(top, t) : top;
    top = max(top, from_lane(x, 63));
    return before;
}
// A wave's view of the groups, 64 at a time: sequences f0 .. f1 - 1, their rows (v.r0, v.n) and the tokens that they share (v.len).  As with the rows: no
// sequence belongs to two groups, one that begins in front of an earlier one's end has none (nor one whose rows do).  f0 never descends.
struct KvGroupLanes {
    const KvSharedArgs* a;
    KvSeq v;
    int f0, f1, top_f = 0, top_h = 0;
    __device__ __forceinline__ KvGroupLanes(const KvSharedArgs& args) : a(&args) {}
    __device__ __forceinline__ int entries(const KvArgs&) const { return a->n_groups; }
    __device__ __forceinline__ void load(const KvArgs& kv, int g0, int lane, bool check) {
        const int g = g0 + lane;
        const bool on = g < a->n_groups;
        const int s0 = on ? a->group_start[g] : 0, s1 = on ? a->group_start[g + 1] : 0, len = on ? a->shared_len[g] : 0;
        const int before = kv_max_before(min(max(s1, 0), kv.n_seqs), top_f, lane);
        const bool order = s0 >= before && s1 >= s0 && s1 <= kv.n_seqs;
        f0 = !on ? 0x7fffffff : order ? s0 : before;
        f1 = on && order ? s1 : f0;
        v = KvSeq{0, 0, min(max(len, 0), kv.cap)};
        int end = 0;
        if (f1 > f0) { v.r0 = min(max(kv.row_start[f0], 0), kv.n_rows); end = min(max(kv.row_start[f1], 0), kv.n_rows); }
        v.n = v.r0 >= kv_max_before(end, top_h, lane) ? max(end - v.r0, 0) : 0;
        if (check && on && (!order || v.len != len)) kv_flag(kv, ASD_KV_BAD_GROUP);
    }
};
// The sequences, with the first key of their own (v.low): 0 where a sequence is in no group, or has a new row that does not lie behind the shared tokens
struct KvOwnLanes : KvLanes {
    KvGroupLanes groups;                                // (the first 64)
    __device__ __forceinline__ KvOwnLanes(const KvGroupLanes& g) : groups(g) {}
    __device__ __forceinline__ void load(const KvArgs& kv, int s0, int lane, bool check) {
        KvLanes::load(kv, s0, lane, check);
        const int s = s0 + lane, n = groups.entries(kv);
        KvGroupLanes g = groups;
        for (int g0 = 0;;) {
            int at = 0;                                 // the last one that begins at s or in front of it
            if (n > 1)
#pragma unroll
                for (int step = 32; step > 0; step >>= 1) if (__shfl(g.f0, at + step) <= s) at += step;
            const int f0 = __shfl(g.f0, at), f1 = __shfl(g.f1, at), r0 = __shfl(g.v.r0, at), rows = __shfl(g.v.n, at), len = __shfl(g.v.len, at);
            if (s >= f0 && s < f1 && v.n > 0 && v.r0 >= r0 && v.r0 + v.n <= r0 + rows && v.len - v.n >= len) v.low = len;
            g0 += 64;
            if (g0 >= n) break;
            g.load(kv, g0, lane, false);
        }
    }
};
__device__ __forceinline__ int kv_front_chunks(const KvSeq& v) { return (v.len + 63) / 64; }
__device__ __forceinline__ int kv_own_chunks(const KvSeq& v) { return (v.len + 63) / 64 - v.low / 64; }
// work item `item` of the shared keys
template <int R, class F> __device__ __forceinline__ bool kv_front_item(const KvSharedArgs& a, int64_t item, KvItem& it, F) {
    const int lane = threadIdx.x & 63, n_kv = a.kv.n_kv;
    int local, group;
    int64_t first;
    const bool check = item == 0 && threadIdx.x < 64;
    KvGroupLanes all(a);
    all.load(a.kv, 0, lane, check);
    const int run = kv_run_all(a.front(), all, lane, R, kv_front_chunks);
    auto count = [&](const KvSeq& v) { return v.len > 0 ? kv_tiles_of(a.kv, v, R) * kv_splits(kv_front_chunks(v), run) * n_kv : 0; };
    if (!kv_find(a.kv, all, item, lane, check, count, &group, &local, &first, &it.s)) return false;
    it.seq = a.group_start[group];
    kv_place_item(it, local, first, kv_tiles_of(a.kv, it.s, R), n_kv, F::value);
    it.per = kv_per_split(kv_front_chunks(it.s), kv_splits(kv_front_chunks(it.s), run));
    it.whole = false;
    return true;
}
// work item `item` of the own keys
template <int R, class F> __device__ __forceinline__ bool kv_own_item(const KvSharedArgs& a, int64_t item, KvItem& it, F) {
    const int lane = threadIdx.x & 63, n_kv = a.kv.n_kv;
    int local;
    int64_t first;
    const bool check = item == 0 && threadIdx.x < 64;
    KvGroupLanes groups(a);
    groups.load(a.kv, 0, lane, false);
    KvOwnLanes all(groups);
    all.load(a.kv, 0, lane, check);
    const int run = kv_run_all(a, all, lane, R, kv_own_chunks);
    auto count = [&](const KvSeq& v) { return kv_tiles_of(a.kv, v, R) * kv_splits(kv_own_chunks(v), run) * n_kv; };
    if (!kv_find(a.kv, all, item, lane, check, count, &it.seq, &local, &first, &it.s)) return false;
    const int n_splits = kv_splits(kv_own_chunks(it.s), run);
    kv_place_item(it, local, first, kv_tiles_of(a.kv, it.s, R), n_kv, F::value);
    it.per = kv_per_split(kv_own_chunks(it.s), n_splits);
    it.whole = n_splits == 1 && it.s.low == 0;
    return true;
}
template <class A, class C, int H, int NT>
__global__ __launch_bounds__(256, A::KE == 4 ? 1 : 2) void kv_front_kernel(const KvSharedArgs a) {
    __shared__ KvFewLds<H> lds;
    KvItem it;
    if (kv_front_item<16 * NT>(a, blockIdx.x, it, std::false_type{})) kv_few_rows<A, C, H, NT, KV_SHARED>(a.front(), it, lds);
}
template <class A, class C, int H, int NT>
__global__ __launch_bounds__(256, A::KE == 4 ? 1 : 2) void kv_own_kernel(const KvSharedArgs a) {
    __shared__ KvFewLds<H> lds;
    KvItem it;
    if (kv_own_item<16 * NT>(a, blockIdx.x, it, std::false_type{})) kv_few_rows<A, C, H, NT, KV_OWN>(a, it, lds);
}
template <class C, int H, int NT, int NW>
__global__ __launch_bounds__(64 * NW, 2) void kv_front_rows_kernel(const KvSharedArgs a) {
    __shared__ u32x4 mem[KV_RING<C, H>];
    KvItem it;
    if (kv_front_item<16 * NT * NW>(a, blockIdx.x, it, std::false_type{})) kv_many_rows<C, H, NT, NW, KV_SHARED>(a.front(), it, mem);
}
template <class C, int H, int NT, int NW>
__global__ __launch_bounds__(64 * NW, 2) void kv_own_rows_kernel(const KvSharedArgs a) {
    __shared__ u32x4 mem[KV_RING<C, H>];
    KvItem it;
    if (kv_own_item<16 * NT * NW>(a, blockIdx.x, it, std::true_type{})) kv_many_rows<C, H, NT, NW, KV_OWN>(a, it, mem);
}
// Puts the parts of every row together
template <class A, int H>
__global__ __launch_bounds__(256) void kv_shared_join_kernel(const KvSharedArgs a) {
    const int lane = threadIdx.x & 63, n_kv = a.kv.n_kv, rows_each = a.kv.group, R = a.tile_rows, FR = a.front_rows;
    int seq, local;
    int64_t first;
    KvSeq s;
    KvGroupLanes groups(a);
    groups.load(a.kv, 0, lane, false);
    KvOwnLanes all(groups);
    all.load(a.kv, 0, lane, false);
    const int run = kv_run_all(a, all, lane, R, kv_own_chunks);
    // 16 rows of a sequence with more than one part and KV head
    if (!kv_find(a.kv, all, blockIdx.x, lane, false, [&](const KvSeq& v) { return kv_splits(kv_own_chunks(v), run) > 1 || v.low > 0 ? kv_tiles_of(a.kv, v, 16) * n_kv : 0; },
                 &seq, &local, &first, &s)) return;
    const int64_t item0 = kv_items_before(a.kv, all, seq, lane, [&](const KvSeq& v) { return (int64_t)kv_tiles_of(a.kv, v, R) * kv_splits(kv_own_chunks(v), run) * n_kv; });
    const int n_own = kv_splits(kv_own_chunks(s), run), n_tiles = kv_tiles_of(a.kv, s, R), kvh = local % n_kv, row0 = local / n_kv * 16;
    const int64_t step = (int64_t)n_tiles * n_kv * R, at = (item0 + (int64_t)(row0 / R) * n_kv + kvh) * R + row0 % R;
    // the group of the sequence, its first item, and the sequence's first row among the group's
    int n_front = 0, front_tiles = 0;
    int64_t front0 = 0, front_row = 0;
    if (s.low > 0) {
        const int front_run = kv_run_all(a.front(), groups, lane, FR, kv_front_chunks);
        for (int g0 = 0;;) {
            const int64_t c = groups.v.len > 0 ? (int64_t)kv_tiles_of(a.kv, groups.v, FR) * kv_splits(kv_front_chunks(groups.v), front_run) * n_kv : 0;
            const unsigned long long mine = __ballot(seq >= groups.f0 && seq < groups.f1);
            const int l = uniform(mine ? __ffsll(mine) - 1 : 64);
            front0 += wave_sum(lane < l ? c : 0);
            if (mine) {
                const KvSeq g{from_lane(groups.v.r0, l), from_lane(groups.v.n, l), from_lane(groups.v.len, l)};
                n_front = kv_splits(kv_front_chunks(g), front_run);
                front_tiles = kv_tiles_of(a.kv, g, FR);
                front_row = (int64_t)(s.r0 - g.r0) * rows_each + row0;
                break;
            }
            g0 += 64;
            if (g0 >= a.n_groups) break;
            groups.load(a.kv, g0, lane, false);
        }
    }
    kv_join_rows<A, H>(a, s, kvh, row0, min(s.n * rows_each - row0, 16), n_own + n_front, [&](int i, int r) {
        const float *o = a.o_part, *ml = a.ml_part;
        int64_t p = at + r + i * step;
        if (i >= n_own) {
            const int64_t row = front_row + r;
            p = (front0 + ((int64_t)(i - n_own) * front_tiles + row / FR) * n_kv + kvh) * FR + row % FR;
            o = a.front_o; ml = a.front_ml;
        }
        return KvPartial{o + p * H, ml + p * 2};
    });
}
