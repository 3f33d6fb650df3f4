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

// What the join of 16 rows for a KV head has to know, written by the work item that has their first run: the join itself then looks nothing up but this (with the
// search for its rows and runs, as kv_join_kernel has it, 64 sequences in two parts took 20 us).
struct KvNote {
    int32_t r0, row0, left, kvh;                        // the sequence's first row, the first of these rows x heads, how many
    int32_t n_own, own, own_step, own_row;              // runs; the item of the first, to the next; the first row's place in it
    int32_t n_front, front, front_step, front_row;      // the same of the shared keys; the first row's place among the group's
};
struct KvNotes {
    int32_t n, pad[15];
    KvNote at[1];
};
// The join: 4 to 6 us, of them 2 for the launch and the note, then one look at all of a row's sums (64 sequences x 64 heads in nine to eleven parts, 20 MB: 5.9 us)
template <class A, int H>
__global__ __launch_bounds__(256) void kv_parts_kernel(const KvAttendArgs a, const KvNotes* notes, const float* front_o, const float* front_ml, int front_rows) {
    const int n = notes->n;
    const KvNote k = notes->at[blockIdx.x];             // (the notes have room for every block)
    if ((int)blockIdx.x >= n || k.left == 0) return;
    const KvSeq s{uniform(k.r0), 0, 0};
    kv_join_rows<A, H>(a, s, uniform(k.kvh), uniform(k.row0), uniform(k.left), uniform(k.n_own + k.n_front), [&](int i, int r) {
        if (i < k.n_own) {
            const int64_t p = (int64_t)(k.own + i * k.own_step) * a.tile_rows + k.own_row + r;
            return KvPartial{a.o_part + p * H, a.ml_part + p * 2};
        }
        const uint32_t row = (uint32_t)(k.front_row + r), tile = row / (uint32_t)front_rows;
        const int64_t p = (int64_t)(k.front + (i - k.n_own) * k.front_step + (int)tile * a.kv.n_kv) * front_rows + row % (uint32_t)front_rows;
        return KvPartial{front_o + p * H, front_ml + p * 2};
    });
}
// The notes on a tile's rows, by one wave of its first run; k: what concerns all of them.  before: 16-row blocks of the sequences in front that are joined
__device__ __forceinline__ void kv_write_notes(KvNotes* notes, const KvAttendArgs& a, const KvItem& it, int n_tiles, int64_t before, int lane, KvNote k) {
    const int row = it.tile * a.tile_rows + lane * 16, left = it.s.n * a.kv.group - row;
    if (lane * 16 >= a.tile_rows || left <= 0) return;
    k.r0 = it.s.r0; k.row0 = row; k.left = min(left, 16); k.kvh = it.kvh;
    k.own = (int)it.part; k.own_step = n_tiles * a.kv.n_kv; k.own_row = lane * 16;
    k.front_row += row;
    notes->at[(before + row / 16) * a.kv.n_kv + it.kvh] = k;
}

// how many there are
template <class Lanes, class F> __device__ __forceinline__ void kv_count_notes(KvNotes* notes, const KvArgs& a, const Lanes& all, int lane, F joined) {
    const int64_t n = kv_items_before(a, all, a.n_seqs, lane, joined);
    if (lane == 0) notes->n = (int)(n * a.n_kv);
}

// Item `item` where only the last round's tiles are cut (attend_plan): of all tiles and KV heads those that fill whole rounds of a.target come first, whole, then the others
// in k runs each.  The notes on the latter lie tile by tile.
template <int R, class Lanes, class F> __device__ __forceinline__ bool kv_tail_item(const KvAttendArgs& a, KvNotes* notes, const Lanes& all, int64_t item, int lane, bool check, KvItem& it, F chunks) {
    const int n_kv = a.kv.n_kv;
    auto tiles = [&](const KvSeq& v) { return kv_tiles_of(a.kv, v, R) * n_kv; };
    const int total = (int)kv_items_before(a.kv, all, all.entries(a.kv), lane, tiles), rest = total % a.target, full = total - rest;
    const int k = rest ? max(1, min(a.target / rest, a.tail)) : 1;
    if (check && a.tail > 1 && lane == 0) notes->n = k > 1 ? rest * (R / 16) : 0;
    const int over = max((int)item - full, 0), th = min((int)item, full) + over / k;
    int local;
    int64_t first;
    if (!kv_find(a.kv, all, th, lane, check, tiles, &it.seq, &local, &first, &it.s)) return false;
    kv_place_item(it, local, 0, kv_tiles_of(a.kv, it.s, R), n_kv, true);
    it.split = over % k;
    it.per = kv_per_split(chunks(it.s), th < full ? 1 : k);
    it.whole = th < full || k == 1;
    it.part = over;
    if (!it.whole && it.split == 0 && threadIdx.x >= 192 && lane < R / 16) {
        const int row = it.tile * R + lane * 16;
        notes->at[(th - full) * (R / 16) + lane] = KvNote{it.s.r0, row, max(min(it.s.n * a.kv.group - row, 16), 0), it.kvh, k, over, 1, lane * 16};
    }
    return true;
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
template <int R, class F> __device__ __forceinline__ bool kv_window_item(const KvWindowArgs& a, KvNotes* notes, KvItem& it, F) {
    const int lane = threadIdx.x & 63, n_kv = a.kv.n_kv;
    int local;
    int64_t first;
    const bool check = blockIdx.x == 0 && threadIdx.x < 64;
    KvLanes all;
    all.load(a.kv, 0, lane, check);
    auto chunks = [&](const KvSeq& v) { return kv_window_chunks(a, v, R); };
    if (F::value && a.tail) return kv_tail_item<R>(a, notes, all, blockIdx.x, lane, check, it, chunks);
    const int run = kv_run_all(a, all, lane, R, chunks);
    auto joined = [&](const KvSeq& v) { return kv_splits(chunks(v), run) > 1 ? kv_tiles_of(a.kv, v, 16) : 0; };
    if (check && a.cut) kv_count_notes(notes, a.kv, all, lane, joined);
    if (!kv_find(a.kv, all, blockIdx.x, lane, check, [&](const KvSeq& v) { return kv_tiles_of(a.kv, v, R) * kv_splits(chunks(v), run) * n_kv; }, &it.seq, &local, &first, &it.s)) return false;
    const int n_splits = kv_splits(chunks(it.s), run), n_tiles = kv_tiles_of(a.kv, it.s, R);
    kv_place_item(it, local, first, n_tiles, n_kv, F::value);
    it.per = kv_per_split(chunks(it.s), n_splits);
    it.whole = n_splits == 1;
    if (!it.whole && it.split == 0 && threadIdx.x >= 192) kv_write_notes(notes, a, it, n_tiles, kv_items_before(a.kv, all, it.seq, lane, joined), lane, KvNote{.n_own = n_splits});
    return true;
}
// A tile walks the chunks of the first tokens, then those from its first row's window on; in between nothing is read.  Bound as kv_few_rows and kv_many_rows are:
// one token of 48 sequences, window 1024, 64 / 8 heads x 128, 8 bits: 27 us, 3.8 TB/s with launch and look-ups (bf16 pages 5.0); one prompt of 16384 tokens, window 4096, 32
// heads, bf16 pages: 968 TFLOP/s, window 256: 322 TFLOP/s, where five of a tile's eight steps have an edge.
template <class A, class C, int H, int NT>
__global__ __launch_bounds__(256, A::KE == 4 ? 1 : 2) void kv_window_kernel(const KvWindowArgs a, KvNotes* notes) {
    __shared__ KvFewLds<H> lds;
    KvItem it;
    if (kv_window_item<16 * NT>(a, notes, it, std::false_type{})) kv_few_rows<A, C, H, NT, KV_WINDOW, 4>(a, it, lds);
}
template <class C, int H, int NT, int NW>
__global__ __launch_bounds__(64 * NW, 2) void kv_window_rows_kernel(const KvWindowArgs a, KvNotes* notes) {
    __shared__ u32x4 mem[KV_RING<C, H>];
    KvItem it;
    if (kv_window_item<16 * NT * NW>(a, notes, it, std::true_type{})) kv_many_rows<C, H, NT, NW, KV_WINDOW>(a, it, mem);
}
// ---------------------------------------------------------------- sequences that begin with the same tokens
// The keys that a group shares are read once for the rows of all its sequences: these lie one behind the other, so that a group is to its shared keys what a
// sequence is to its own, all rows seeing all of them.  The keys behind them are each sequence's own.  Every row's sums come in two
// parts at least, put together in a launch of their own.
struct KvSharedArgs : KvAttendArgs {                    // (o_part .. cut: of the own keys)
    const int32_t *group_start, *shared_len;
    int32_t n_groups;
    int32_t front_target, front_min_run, front_cut, front_rows, front_grid;
    float *front_o, *front_ml;
    __device__ __forceinline__ KvAttendArgs front() const {
        KvAttendArgs f = *this;
        f.o_part = front_o; f.ml_part = front_ml; f.target = front_target; f.min_run = front_min_run; f.cut = front_cut;
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
    int s0, s1, len;                                    // what the arrays say
    __device__ __forceinline__ KvGroupLanes(const KvSharedArgs& args) : a(&args) {}
    __device__ __forceinline__ int entries(const KvArgs&) const { return a->n_groups; }
    __device__ __forceinline__ void ask(int g0, int lane) {
        const int g = min(g0 + lane, a->n_groups - 1);
        s0 = a->group_start[g]; s1 = a->group_start[g + 1]; len = a->shared_len[g];
    }
    // begin(s), tokens(s), of all lanes at once: row_start[s], kv_len[s]
    template <class F, class G> __device__ __forceinline__ void take(const KvArgs& kv, int g0, int lane, bool check, F begin, G tokens) {
        const bool on = g0 + lane < a->n_groups;
        const int before = kv_max_before(on ? min(max(s1, 0), kv.n_seqs) : 0, top_f, lane);
        const bool order = s0 >= before && s1 >= s0 && s1 <= kv.n_seqs;
        f0 = !on ? 0x7fffffff : order ? s0 : before;
        f1 = on && order ? s1 : f0;
        const int shared = min(max(len, 0), kv.cap), r0 = begin(f1 > f0 ? f0 : 0), r1 = begin(f1 > f0 ? f1 : 0), held = tokens(f1 > f0 ? f0 : 0);
        v = KvSeq{f1 > f0 ? min(max(r0, 0), kv.n_rows) : 0, 0, held < shared ? 0 : shared};      // (the first one has to hold them)
        const int end = f1 > f0 ? min(max(r1, 0), kv.n_rows) : 0;
        v.n = v.r0 >= kv_max_before(end, top_h, lane) ? max(end - v.r0, 0) : 0;
        if (check && on && (!order || shared != len)) kv_flag(kv, ASD_KV_BAD_GROUP);
    }
    __device__ __forceinline__ void load(const KvArgs& kv, int g0, int lane, bool check) {
        ask(g0, lane);
        take(kv, g0, lane, check, [&](int s) { return kv.row_start[s]; }, [&](int s) { return kv.kv_len[s]; });
    }
    // the first 64; with up to 64 sequences their beginnings are asked for along with the groups
    __device__ __forceinline__ void begin(const KvArgs& kv, int lane, bool check) {
        ask(0, lane);
        if (kv.n_seqs > 64) return take(kv, 0, lane, check, [&](int s) { return kv.row_start[s]; }, [&](int s) { return kv.kv_len[s]; });
        const int s = min(lane, kv.n_seqs - 1), r0 = kv.row_start[s], r1 = kv.row_start[s + 1], n = kv.kv_len[s];
        take(kv, 0, lane, check, [&](int at) { const int x = __shfl(r0, min(at, 63)), y = __shfl(r1, max(at - 1, 0)); return at < kv.n_seqs ? x : y; }, [&](int at) { return __shfl(n, at); });
    }
};
// The sequences, with the first key of their own (v.low): 0 where a sequence is in no group, or has a new row that does not lie behind the shared tokens, or
// where the group's first sequence does not hold them
struct KvOwnLanes : KvLanes {
    KvGroupLanes groups;                                // 64 of them, from g0 on
    int g0 = 0;
    __device__ __forceinline__ KvOwnLanes(const KvGroupLanes& first) : groups(first) {}
    __device__ __forceinline__ void load(const KvArgs& kv, int s0, int lane, bool check) {
        KvLanes::load(kv, s0, lane, check);
        const int s = s0 + lane, n = groups.entries(kv);
        for (;;) {
            int at = 0;                                 // the last one that begins at s or in front of it
            if (n > 1)
#pragma unroll
                for (int step = 32; step > 0; step >>= 1) if (__shfl(groups.f0, at + step) <= s) at += step;
            const int f0 = __shfl(groups.f0, at), f1 = __shfl(groups.f1, at), r0 = __shfl(groups.v.r0, at), rows = __shfl(groups.v.n, at), len = __shfl(groups.v.len, at);
            if (s >= f0 && s < f1 && v.n > 0 && v.r0 >= r0 && v.r0 + v.n <= r0 + rows && v.len - v.n >= len) { v.low = len; v.lead = f0; }
            // Later groups begin at the end of these or behind it: where that is behind the sequences at hand, they wait for the next ones, so that a walk over all
            // sequences is one over all groups too, whatever there are of either.
            if (groups.top_f > s0 + 63 || g0 + 64 >= n) break;
            g0 += 64;
            groups.load(kv, g0, lane, false);
        }
    }
};
__device__ __forceinline__ int kv_front_chunks(const KvSeq& v) { return (v.len + 63) / 64; }
__device__ __forceinline__ int kv_own_chunks(const KvSeq& v) { return (v.len + 63) / 64 - v.low / 64; }
__device__ __forceinline__ int kv_both_chunks(const KvSeq& v) { return (v.len + 63) / 64 + (v.low % 64 != 0); }
__device__ __forceinline__ int kv_front_items(const KvSharedArgs& a, const KvSeq& v, int rows, int run) {
    return v.len > 0 ? kv_tiles_of(a.kv, v, rows) * kv_splits(kv_front_chunks(v), run) * a.kv.n_kv : 0;
}
// work item `item` of the shared keys
template <int R, class F> __device__ __forceinline__ bool kv_front_item(const KvSharedArgs& a, int64_t item, KvItem& it, F) {
    const int lane = threadIdx.x & 63, n_kv = a.kv.n_kv;
    int local, group;
    int64_t first;
    const bool check = item == 0 && threadIdx.x < 64;
    KvGroupLanes all(a);
    all.begin(a.kv, lane, check);
    const int run = kv_run_all(a.front(), all, lane, R, kv_front_chunks);
    auto count = [&](const KvSeq& v) { return kv_front_items(a, v, R, run); };
    if (!kv_find(a.kv, all, item, lane, check, count, &group, &local, &first, &it.s)) return false;
    it.seq = a.group_start[group];
    kv_place_item(it, local, first, kv_tiles_of(a.kv, it.s, R), n_kv, F::value);
    it.per = kv_per_split(kv_front_chunks(it.s), kv_splits(kv_front_chunks(it.s), run));
    it.whole = false;
    return true;
}
// where the sums of the sequence's rows over the shared keys are
__device__ __forceinline__ void kv_front_note(const KvSharedArgs& a, KvGroupLanes groups, const KvItem& it, int lane, KvNote& k) {
    const int n_kv = a.kv.n_kv, R = a.front_rows, run = kv_run_all(a.front(), groups, lane, R, kv_front_chunks);
    int64_t before = 0;
    for (int g0 = 0; g0 < a.n_groups; g0 += 64) {
        if (g0) groups.load(a.kv, g0, lane, false);
        const int c = kv_front_items(a, groups.v, R, run);
        const unsigned long long mine = __ballot(groups.f0 == it.s.lead && groups.f1 > groups.f0);
        const int l = uniform(mine ? __ffsll(mine) - 1 : 64);
        before += wave_sum(lane < l ? c : 0);
        if (!mine) continue;
        const KvSeq g{from_lane(groups.v.r0, l), from_lane(groups.v.n, l), from_lane(groups.v.len, l)};
        k.n_front = kv_splits(kv_front_chunks(g), run);
        k.front = (int)before + it.kvh;
        k.front_step = kv_tiles_of(a.kv, g, R) * n_kv;
        k.front_row = (it.s.r0 - g.r0) * a.kv.group;
        return;
    }
}
// work item `item` of the own keys; BOTH: of all keys of a sequence, the shared ones in front
template <int R, bool BOTH, class F> __device__ __forceinline__ bool kv_own_item(const KvSharedArgs& a, KvNotes* notes, int64_t item, KvItem& it, F) {
    const int lane = threadIdx.x & 63, n_kv = a.kv.n_kv;
    int local;
    int64_t first;
    const bool check = item == 0 && threadIdx.x < 64;
    KvGroupLanes groups(a);
    groups.begin(a.kv, lane, BOTH && check);
    KvOwnLanes all(groups);
    all.load(a.kv, 0, lane, check);
    auto chunks = [](const KvSeq& v) { return BOTH ? kv_both_chunks(v) : kv_own_chunks(v); };
    if (BOTH && check && a.n_groups > 64) for (int g0 = 64; g0 < a.n_groups; g0 += 64) groups.load(a.kv, g0, lane, true);
    if (F::value && a.tail) return kv_tail_item<R>(a, notes, all, item, lane, check, it, chunks);
    const int run = kv_run_all(a, all, lane, R, chunks);
    auto count = [&](const KvSeq& v) { return kv_tiles_of(a.kv, v, R) * kv_splits(chunks(v), run) * n_kv; };
    // (Apart, all rows are joined: one that shares nothing may lie in a tile of those that do, whose queries must not change while the tile is at work: `out` may be `q`.)
    auto joined = [&](const KvSeq& v) { return !BOTH || kv_splits(chunks(v), run) > 1 ? kv_tiles_of(a.kv, v, 16) : 0; };
    if (check && (!BOTH || a.cut)) kv_count_notes(notes, a.kv, all, lane, joined);
    if (!kv_find(a.kv, all, item, lane, check, count, &it.seq, &local, &first, &it.s)) return false;
    const int n_splits = kv_splits(chunks(it.s), run), n_tiles = kv_tiles_of(a.kv, it.s, R);
    kv_place_item(it, local, first, n_tiles, n_kv, F::value);
    it.per = kv_per_split(chunks(it.s), n_splits);
    it.whole = BOTH && n_splits == 1;
    if (!it.whole && it.split == 0 && (!BOTH || threadIdx.x >= 192)) {     // (own items are a wave's each)
        KvNote k{.n_own = n_splits};
        if (!BOTH && it.s.low > 0) kv_front_note(a, groups, it, lane, k);
        kv_write_notes(notes, a, it, n_tiles, kv_items_before(a.kv, all, it.seq, lane, joined), lane, k);
    }
    return true;
}
// Both parts in one launch, the shared keys' items first: tiles of 16 * FNT rows (128: FNT = 8), the own ones of 16, a wave each.  64 answers to 8005 shared tokens, 64 / 8
// heads x 128, 8 bits: 37.5 us: 256 workgroups of 16 steps over the shared keys, one to a compute unit, 33 to 37 us; the own keys (up to 300 each) end after 22 beside them.
// In two launches the two took 37 and 20.  Shorter runs of the shared keys take the place that the own ones have beside them (runs of 8 chunks: 29 us, the own keys then
// until 40).  16 samples of 2048 tokens and up to 512 of their own, 32 heads, bf16 pages: 20 us, 84 MB.
template <class A, class C, int H, int FNT>
__global__ __launch_bounds__(256, A::KE == 4 ? 1 : 2) void kv_apart_kernel(const KvSharedArgs a, KvNotes* notes) {
    using Ring = u32x4[KV_RING<C, H>];
    constexpr size_t RING = FNT == 8 ? sizeof(Ring) : 0;
    __shared__ __align__(16) char mem[RING > sizeof(KvFewLds<H>) ? RING : sizeof(KvFewLds<H>)];
    KvItem it;
    if (blockIdx.x >= (unsigned)a.front_grid) {
        const int64_t item = (int64_t)(blockIdx.x - a.front_grid) * 4 + uniform(threadIdx.x >> 6);
        if (kv_own_item<16, false>(a, notes, item, it, std::false_type{})) kv_few_rows<A, C, H, 1, KV_OWN, 1>(a, it, *(KvFewLds<H>*)mem);
    } else if (kv_front_item<16 * FNT>(a, blockIdx.x, it, std::false_type{})) {
        if constexpr (FNT == 8) kv_many_rows<C, H, 2, 4, KV_SHARED>(a.front(), it, *(Ring*)mem);
        else kv_few_rows<A, C, H, FNT, KV_SHARED, 4>(a.front(), it, *(KvFewLds<H>*)mem);
    }
}
// All keys of a sequence, the shared ones through the page table of the group's first: causal attention, but for the chunk in which the shared tokens end, which comes twice.
// 24 questions of up to 130 tokens behind three system prompts of 2756 to 4000, 64 / 8 heads x 128: 8 bits 270 us, 753 TFLOP/s, bf16 pages 238, 857 TFLOP/s.
template <class A, class C, int H, int NT>
__global__ __launch_bounds__(256, A::KE == 4 ? 1 : 2) void kv_both_kernel(const KvSharedArgs a, KvNotes* notes) {
    __shared__ KvFewLds<H> lds;
    KvItem it;
    if (kv_own_item<16 * NT, true>(a, notes, blockIdx.x, it, std::false_type{})) kv_few_rows<A, C, H, NT, KV_BOTH, 4>(a, it, lds);
}
template <class C, int H, int NT, int NW>
__global__ __launch_bounds__(64 * NW, 2) void kv_both_rows_kernel(const KvSharedArgs a, KvNotes* notes) {
    __shared__ u32x4 mem[KV_RING<C, H>];
    KvItem it;
    if (kv_own_item<16 * NT * NW, true>(a, notes, blockIdx.x, it, std::true_type{})) kv_many_rows<C, H, NT, NW, KV_BOTH>(a, it, mem);
}
