// Attention of new rows over a paged cache of several sequences (the pages: asd_kv.h).
#pragma once
#include "asd_kv.h"

// ---------------------------------------------------------------- attention of the new rows
struct KvAttendArgs {
    KvArgs kv;
    const void* q;
    void* out;
    int64_t q_stride, out_stride;
    float c2;                       // scale * log2(e)
    float *o_part, *ml_part;        // [item][rows of a tile][H] unnormalised sums; [item][rows][2] (maximum, sum)
    int32_t target;                 // work items to cut the batch into
    int32_t min_run;                // chunks that are worth a run
    int32_t cut;                    // 0: every tile's keys stay together
    int32_t tail;                   // > 0: those of the last round's tiles are cut, into this many runs at most (asd_kv_spans.h)
    int32_t tile_rows;              // rows of a tile
};
// What the rows of a tile see.  KV_ALL: the keys 0 .. position of their sequence.  KV_WINDOW: of those the last `window` and the first `sinks`.  Sequences that
// share their first keys: KV_SHARED those (the rows of all sequences of a group, each sees them all), KV_OWN the keys low .. position behind them, KV_BOTH
// both, the keys 0 .. low - 1 through the table of the group's first sequence.
enum { KV_ALL = 0, KV_WINDOW = 1, KV_SHARED = 2, KV_OWN = 3, KV_BOTH = 4 };
struct KvWindowArgs : KvAttendArgs { int32_t window, sinks; };
// A work item: a tile of a sequence's rows for one KV head against one of the runs that its chunks are cut into
struct KvItem {
    int seq;                        // whose page table (KV_BOTH: s.lead's for the keys below s.low)
    KvSeq s;
    int kvh, tile, split, per;      // per: chunks of a run
    bool whole;                     // nothing else belongs to the tile's rows: the results go to `out`
    int64_t part;                   // else: its place among the partial sums
    // the same in scalar registers (left to itself the compiler keeps what comes through the structure in 16 vector registers)
    __device__ __forceinline__ KvItem scalar() const {
        return KvItem{uniform(seq), KvSeq{uniform(s.r0), uniform(s.n), uniform(s.len), uniform(s.low), uniform(s.lead)}, uniform(kvh), uniform(tile), uniform(split), uniform(per), uniform(whole) != 0,
                      (int64_t)((uint64_t)(uint32_t)uniform((int)part) | (uint64_t)(uint32_t)uniform((int)(part >> 32)) << 32)};
    }
};
// The chunks (units) that a tile walks, numbered without those that no row sees: the `first` ones (of the first tokens; of the shared ones), then those behind `skip`
// others (-1: the chunk in which the shared tokens end comes twice, through either table)
struct KvSteps {
    int first = 0, skip = 0;
    __device__ __forceinline__ int at(int i) const { return i >= first ? i + skip : i; }
};
template <int SEES, class Args> __device__ __forceinline__ KvSteps kv_steps(const Args& a, int low, int keys) {      // low: first key of the tile's window; keys of a step
    KvSteps t;
    if constexpr (SEES == KV_WINDOW) {
        const int first = max(low, 0) / keys, n = (a.sinks + keys - 1) / keys;
        if (n < first) t = KvSteps{n, first - n};
    }
    if constexpr (SEES == KV_OWN) t.skip = low / keys;
    if constexpr (SEES == KV_BOTH) { t.first = (low + keys - 1) / keys; t.skip = low / keys - t.first; }
    return t;
}
// The pages of 64 entries of a table from `base` on, in a wave's lanes (-1: no page of the pool)
struct KvPages {
    int base = -64, page = 0;
    __device__ __forceinline__ void load(const KvArgs& a, int seq, int from, int lane) {
        base = from;
        page = from + lane < a.table_stride ? a.table[(size_t)seq * a.table_stride + from + lane] : -1;
        if ((unsigned)page >= (unsigned)a.n_pages) page = -1;
    }
    __device__ __forceinline__ int at(int i) const { return __builtin_amdgcn_readlane(page, i - base); }
};
// How a batch is cut.  The rows of a sequence and KV head are its new tokens x the heads of the group; a tile is 16 * NT of
// them.  With `cut`, all tiles' key ranges are cut into runs of `run` chunks, the same for every sequence, so that about `target` items come out
// whatever the lengths are: one long conversation among short ones is spread over the card.  (attend_plan in asd_kv_plan.h says which batches are cut.)
template <int NT> __device__ __forceinline__ int kv_tiles(const KvArgs& a, const KvSeq& v) { return (int)(((uint32_t)v.n * a.group + 16 * NT - 1) / (16 * NT)); }      // (n_rows * n_h is below 2^31)
__device__ __forceinline__ int kv_run_of(const KvAttendArgs& a, int64_t t) {      // t: chunks of all tiles of a KV head
    const int run = (int)fminf((float)(t * a.kv.n_kv) / (float)a.target, 1e8f) + 1;
    return uniform(max(run, a.min_run));
}
// chunks(sequence): the chunks that its tiles walk at most
template <int NT, class F> __device__ __forceinline__ int kv_run(const KvAttendArgs& a, const KvLanes& all, int lane, F chunks) {
    if (!a.cut) return 1 << 28;
    auto units = [&](const KvSeq& v) { return (int64_t)kv_tiles<NT>(a.kv, v) * chunks(v); };
    int64_t t = units(all.v);
    for (int s = lane + 64; s < a.kv.n_seqs; s += 64) t += units(kv_seq(a.kv, s));      // (of bad ones no less than they have: longer runs)
    return kv_run_of(a, a.kv.n_seqs > 1 ? wave_sum(t) : t);
}
// runs of a sequence, of equal length: its chunks / run, to the nearest
__device__ __forceinline__ int kv_splits(int chunks, int run) { return max(1, (int)((uint32_t)(chunks + run / 2) / (uint32_t)run)); }
__device__ __forceinline__ int kv_per_split(int chunks, int n_splits) { return (int)((uint32_t)(chunks + n_splits - 1) / (uint32_t)n_splits); }

// ---- V that is not finite at a key that some rows of a tile do not see: 0 times it is not 0.  In the chunks where that can be (edge
// chunks: not all rows of the tile see all keys) such values are taken out of the products, and what a row sees of them is added to
// its sums when they have been stored (infinities and NaN may be added in any order).  Rare, so that path is a plain loop over memory.
// the top bits of a word's elements of a V^T piece that are not finite
template <class C> __device__ __forceinline__ uint32_t kv_odd(uint32_t v) {
    if constexpr (sizeof(typename C::elem) == 4) return (v & 0x7f800000u) == 0x7f800000u ? 0x80000000u : 0u;
    else if constexpr (sizeof(typename C::elem) == 2) return ~(((v & 0x7f807f80u) ^ 0x7f807f80u) + 0x7fff7fffu) & 0x80008000u;      // (no carry leaves a half)
    else return ((v & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
}
// the word without them
template <class C> __device__ __forceinline__ uint32_t kv_clean(uint32_t v) {
    constexpr int B = 8 * (int)sizeof(typename C::elem) - 1;
    const uint32_t t = kv_odd<C>(v);
    return v & ~((t - (t >> B)) | t);
}
// their sum over the keys key0 .. last at one dim (0: there are none), without those below `low` that are not among the first `sinks` and without main0 .. main1 - 1
template <class C, int H> __device__ float kv_odd_sum(const KvArgs& a, int seq, int kvh, int key0, int last, int dim, int low = 0, int sinks = 0, int main0 = 0, int main1 = 0) {
    float sum = 0.f;
    for (int key = key0; key <= last; ++key) {
        if (key >= main0 && key < main1) { key = main1 - 1; continue; }
        if (key < low && key >= sinks) continue;
        const char* p = kv_chunk<C, H>(a, seq, key / 64, kvh);
        if (!p) continue;
        const typename C::elem v = *(const typename C::elem*)(p + KvLayout<C, H>::v_off(key % 64, dim));
        float f;
        if constexpr (sizeof(v) == 1) f = (v & 0x7f) == 0x7f ? __uint_as_float(0x7fc00000u) : 0.f;
        else f = C::to_f32(v);
        if (!finite(f)) sum += f;
    }
    return sum;
}
// the bits of word x of a lane's V^T piece ks whose keys are among the first n_keys of the chunk
template <class C> __device__ __forceinline__ uint32_t kv_kept(int n_keys, int ks, int g, int x) {
    constexpr int EB = 8 * (int)sizeof(typename C::elem), PER = 32 / EB;      // bits of an element, elements of a word
    const int left = n_keys - (ks * 4 * C::KE + g * C::KE + x * PER);
    return left >= PER ? 0xffffffffu : left <= 0 ? 0u : (1u << (left * EB & 31)) - 1u;
}

// Units of a chunk: one step of V^T pieces each, so that a wave's share is small where the work of a key is large (fp32 products) and a
// unit takes no more registers than it must (bf16: one sequence of 8192 tokens 32.8 us with whole chunks, 29.4 with halves)
#define KV_UNITS(C) (16 / C::KE)
template <int H> struct alignas(16) KvFewLds {
    float o[4][16][H], ml[4][16][2];
    int odd;
};
// 16 * NT rows against a run of chunks, in units: the keys of one step of V^T pieces (16 fp32, 32 bf16, 64 codes).  W waves (4, or 1: each has an item of its own), wave w
// the units w, w + W, ... of the run with a running maximum and sum per row, merged through LDS at the end.  Scores S[key][row] = K q^T and the output O[dim][row] = V^T P are matrix-core products with the rows as
// columns (see asd_attn.h); a unit's fragments go from memory into registers ahead of their use: memory-bound while the rows are few.
// 8 bits: K is widened with its scale, V without: V's scales go into the probabilities, one value per key.
// One token of 48 sequences of 500 to 8192 tokens, 64 / 8 heads x 128, 8 bits: 84 us, with the join 5.6 TB/s.  A batch too small for memory to
// bound it waits for its loads, 1.7 us for each unit of a wave: five rows of eight sequences of up to 1031 tokens, 40 heads, 16 us.  Around them about 5 us: a launch,
// 1.7 us until a wave knows its item (lengths, sums over them), 1 for the pages, 2 for the merge.
// With a window (KV_WINDOW) that is all that is left of the length: the 48 sequences with the last 1024 tokens and the first 4 27 us (bf16 pages 40, 5.0 TB/s).
// A wave to an item (W = 1) leaves the merge and its LDS out, for short runs beside other work (the own keys of sequences that share the others).
template <class A, class C, int H, int NT, int SEES, int W, class Args> __device__ __forceinline__ void kv_few_rows(const Args& a, const KvItem& item, KvFewLds<H>& sh) {
    using L = KvLayout<C, H>;
    using E = typename A::elem;
    constexpr int AE = A::KE, KK = L::KK, HP = L::HP, US = KK / AE, QS = HP * US;      // operand steps of a K piece, of a row
    constexpr int HT = L::HT, KST = L::KST, VS = L::KV / AE;                           // ... of a V^T piece
    constexpr int UPC = KV_UNITS(C), UK = 64 / UPC, KT = 4 / UPC, KSU = KST / UPC, PS = KSU * VS;      // units of a chunk; keys, score tiles, V^T pieces, steps of a unit
    const int tid = threadIdx.x, lane = tid & 63, w = W == 1 ? 0 : uniform(tid >> 6), g = lane >> 4, m = lane & 15;
    const KvItem it = item.scalar();
    const int seq = it.seq, kvh = it.kvh, tile = it.tile, split = it.split, per = it.per, n_kv = a.kv.n_kv;
    const KvSeq s = it.s;
    if (W > 1 && tid == 0) sh.odd = 0;
    const int rows = s.n * a.kv.group, base = s.len - s.n;
    // last keys of the tile's last and first row; first keys of their windows (KV_OWN: of all rows)
    const int last = SEES == KV_SHARED ? s.len - 1 : base + (min((tile + 1) * NT * 16, rows) - 1) / a.kv.group;
    const int from = SEES == KV_SHARED ? s.len - 1 : base + tile * NT * 16 / a.kv.group;
    int window = 0, sinks = 0, low = 0, low_last = 0;
    if constexpr (SEES == KV_WINDOW) { window = a.window; sinks = a.sinks; low = from - window + 1; low_last = last - window + 1; }
    if constexpr (SEES >= KV_OWN) low = low_last = s.low;
    const KvSteps steps = kv_steps<SEES>(a, low, UK);
    const int u_begin = split * per * UPC, u_end = min((last + UK) / UK - steps.skip, (split + 1) * per * UPC);      // (nothing to do where last is negative)
    // The pages lie in the wave's lanes, those of the first steps apart from the others: a look-up in memory per unit would wait
    // for every fragment asked for before it.  (Asked for ahead of the queries, which nothing waits for before the first scores.)
    constexpr bool TWO = SEES == KV_WINDOW || SEES == KV_BOTH;
    const int cpp = a.kv.page_tokens / 64, first_seq = SEES == KV_BOTH ? s.lead : seq, u_first = u_begin + w;
    KvPages pages, first_pages;
    if (u_first < u_end) {
        if (TWO && u_first < steps.first) {
            first_pages.load(a.kv, first_seq, u_first / UPC / cpp, lane);
            if (u_end > steps.first) pages.load(a.kv, seq, (steps.first + steps.skip) / UPC / cpp, lane);
        } else {
            pages.load(a.kv, seq, steps.at(u_first) / UPC / cpp, lane);
        }
    }
    int pos[NT];                                        // last key of this lane's rows (-1: no such row, or none)
    u32x4 qf[NT][QS];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int row = (tile * NT + t) * 16 + m, token = row / a.kv.group, head = kvh * a.kv.group + row % a.kv.group;
        const bool on = row < rows;
        pos[t] = on ? SEES == KV_SHARED ? s.len - 1 : base + token : -1;
        const E* qp = (const E*)a.q + (s.r0 + (int64_t)token) * a.q_stride + head * H;
#pragma unroll
        for (int i = 0; i < QS; ++i) qf[t][i] = on ? *(const u32x4*)(qp + i / US * 4 * KK + g * KK + i % US * AE) : u32x4{0u, 0u, 0u, 0u};
    }
    auto hidden = [&](int key, int t, bool first) {      // first: of the first steps
        bool h = key > pos[t];
        if constexpr (SEES == KV_WINDOW) h = h || (key <= pos[t] - window && key >= sinks);
        if constexpr (SEES == KV_OWN) h = h || key < low;
        if constexpr (SEES == KV_BOTH) h = h || (key < low) != first;
        return h;
    };

    f32x4 o[NT][HT];
    float mx[NT], l[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        mx[t] = -INFINITY; l[t] = 0.f;
#pragma unroll
        for (int ht = 0; ht < HT; ++ht) o[t][ht] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    struct Unit { u32x4 k[KT][HP], v[HT][KSU], ke, ve; };
    auto ask_k = [&](Unit& f, const char* p) {
#pragma unroll
        for (int kt = 0; kt < KT; ++kt)
#pragma unroll
            for (int hp = 0; hp < HP; ++hp) {
                if constexpr (KK * sizeof(typename C::elem) == 16) f.k[kt][hp] = __builtin_nontemporal_load((const u32x4*)(p + ((kt * HP + hp) * 64 + lane) * 16));
                else { const uint64_t x = __builtin_nontemporal_load((const uint64_t*)(p + ((kt * HP + hp) * 64 + lane) * 8)); f.k[kt][hp] = u32x4{(uint32_t)x, (uint32_t)(x >> 32), 0u, 0u}; }
            }
        if constexpr (L::Q8) f.ke = *(const u32x4*)(p + 2 * L::K_BYTES + 16 * (m >> 2));
    };
    auto ask_v = [&](Unit& f, const char* p) {
#pragma unroll
        for (int ht = 0; ht < HT; ++ht)
#pragma unroll
            for (int ks = 0; ks < KSU; ++ks) f.v[ht][ks] = __builtin_nontemporal_load((const u32x4*)(p + ((ht * KST + ks) * 64 + lane) * 16));
        if constexpr (L::Q8) f.ve = *(const u32x4*)(p + L::K_BYTES + 64 + 16 * g);
    };
    // the first unit from u on that has a page, and where it is; one without counts as hidden
    const char *at_k = nullptr, *at_v = nullptr;
    auto next = [&](int u) {
        for (; u < u_end; u += W) {
            const int r = steps.at(u), c = r / UPC, i = c / cpp;
            int page;
            if (TWO && u < steps.first) {
                if (i - first_pages.base >= 64) first_pages.load(a.kv, first_seq, i, lane);
                page = first_pages.at(i);
            } else {
                if (i - pages.base >= 64) pages.load(a.kv, seq, i, lane);
                page = pages.at(i);
            }
            const char* p = a.kv.pages + (((size_t)max(page, 0) * n_kv + kvh) * cpp + c % cpp) * L::CHUNK;
            at_k = p + r % UPC * KT * HP * 64 * KK * sizeof(typename C::elem);
            at_v = p + L::K_BYTES + r % UPC * KSU * 1024;
            if (page >= 0) break;
            if (lane == 0) kv_flag(a.kv, ASD_KV_BAD_PAGE);
        }
        return u;
    };
    bool odd = false;
    auto work = [&](Unit& f, const int u, auto after_scores) {
        const int key0 = steps.at(u) * UK;
        const bool first = TWO && u < steps.first;
        f32x4 sc[NT][KT];
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
            float scale = 1.f;
            if constexpr (L::Q8) scale = q8_scale((f.ke[kt] >> (8 * (m & 3))) & 255u);
#pragma unroll
            for (int t = 0; t < NT; ++t) sc[t][kt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < QS; ++i) {
                const u32x4 x = kv_operand<A, C>(f.k[kt][i / US], i % US, scale);
#pragma unroll
                for (int t = 0; t < NT; ++t) mma16<A>(sc[t][kt], x, qf[t][i]);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        after_scores();
        __builtin_amdgcn_sched_barrier(0);
        // some rows do not see all of the unit; some of its keys are behind the sequence's end
        bool edge = key0 + UK - 1 > from;
        if constexpr (SEES == KV_WINDOW || SEES == KV_OWN) edge = edge || (key0 < low_last && key0 + UK > sinks);
        if constexpr (SEES == KV_BOTH) edge = edge || (first ? key0 + UK > low : key0 < low);
        float vs[KT][4];
        if constexpr (L::Q8)
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                for (int j = 0; j < 4; ++j) vs[kt][j] = q8_scale((f.ve[kt] >> (8 * j)) & 255u);
        u32x4 pf[NT][PS];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            if (edge) {
#pragma unroll
                for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (hidden(key0 + score_key<C>(kt, 4 * g + j), t, first)) sc[t][kt][j] = -INFINITY;
            }
            float cm = sc[t][0][0];
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                for (int j = 0; j < 4; ++j) cm = fmaxf(cm, sc[t][kt][j]);
            cm = groups_max(cm);
            const float mn = fmaxf(mx[t], cm), ref = mn == -INFINITY ? 0.f : mn;      // nothing seen yet: all weights are 0
            const float alpha = __builtin_amdgcn_exp2f((mx[t] - ref) * a.c2);
            mx[t] = mn;
            l[t] *= alpha;
#pragma unroll
            for (int ht = 0; ht < HT; ++ht) { o[t][ht][0] *= alpha; o[t][ht][1] *= alpha; o[t][ht][2] *= alpha; o[t][ht][3] *= alpha; }
            float pr[KT][4];
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float e = __builtin_amdgcn_exp2f((sc[t][kt][j] - ref) * a.c2);
                    l[t] += e;
                    pr[kt][j] = e;
                    if constexpr (L::Q8) {
                        pr[kt][j] = e * vs[kt][j];
                        // (an unwritten scale may be anything)
                        if (edge && hidden(key0 + score_key<C>(kt, 4 * g + j), t, first)) pr[kt][j] = 0.f;
                    }
                }
            // the probabilities as operands: lane group g holds, in order, the keys of its V^T pieces
#pragma unroll
            for (int i = 0; i < PS; ++i) {
                if constexpr (AE == 8) {
                    // bf16, as V is: each weight is off by at most 2^-8 of itself, and the sum of weights is taken unrounded
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const int e = 2 * x, kt = 2 * i + e / 4;
                        pf[t][i][x] = bf16_pair(pr[kt][e & 3], pr[kt][(e & 3) + 1]);
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) pf[t][i][j] = __float_as_uint(pr[i][j]);
                }
            }
        }
        if (edge) {
            // what is behind the end, or no row sees, is cleared: 0 times whatever lies there must be 0
            int cut = 0, n_keys = s.len - key0;
            if constexpr (SEES == KV_OWN) cut = low - key0;
            if constexpr (SEES == KV_BOTH) { if (first) n_keys = low - key0; else cut = low - key0; }
            if constexpr (SEES == KV_WINDOW) {
                if (key0 >= sinks) cut = low - key0;
                if (key0 + UK <= low) n_keys = min(n_keys, sinks - key0);
            }
            if (n_keys < UK || cut > 0) {
#pragma unroll
                for (int ks = 0; ks < KSU; ++ks)
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        uint32_t keep = kv_kept<C>(n_keys, ks, g, x);
                        if constexpr (SEES != KV_ALL && SEES != KV_SHARED) keep &= ~kv_kept<C>(cut, ks, g, x);
#pragma unroll
                        for (int ht = 0; ht < HT; ++ht) f.v[ht][ks][x] &= keep;
                    }
            }
            uint32_t hit = 0;
#pragma unroll
            for (int ht = 0; ht < HT; ++ht)
#pragma unroll
                for (int ks = 0; ks < KSU; ++ks)
#pragma unroll
                    for (int x = 0; x < 4; ++x) hit |= kv_odd<C>(f.v[ht][ks][x]);
            if (__any(hit != 0)) {
                odd = true;
#pragma unroll
                for (int ht = 0; ht < HT; ++ht)
#pragma unroll
                    for (int ks = 0; ks < KSU; ++ks)
#pragma unroll
                        for (int x = 0; x < 4; ++x) f.v[ht][ks][x] = kv_clean<C>(f.v[ht][ks][x]);
            }
        }
#pragma unroll
        for (int ht = 0; ht < HT; ++ht)
#pragma unroll
            for (int i = 0; i < PS; ++i) {
                const u32x4 v = kv_operand<A, C>(f.v[ht][i / VS], i % VS, 1.f);
#pragma unroll
                for (int t = 0; t < NT; ++t) mma16<A>(o[t][ht], v, pf[t][i]);
            }
    };
    int unit = next(u_begin + w);
    // One token against bf16 pages: two units in registers, all of the next on its way while one is worked on (one sequence of 8192 tokens,
    // 32 heads: 29.4 -> 28.6 us).  Codes and fp32 rows take more registers per unit or more time per key: with two units, 48 sequences
    // of 8-bit pages took 103 us and not 90, a small fp32 batch 10.6 and not 9.5
    if constexpr (NT == 1 && sizeof(typename C::elem) == 2) {
        Unit f0, f1;
        auto ask = [&](Unit& f) { ask_k(f, at_k); ask_v(f, at_v); };
        auto turn = [&](Unit& now, Unit& then) {
            const int un = next(unit + W);
            if (un < u_end) ask(then);
            __builtin_amdgcn_sched_barrier(0);
            work(now, unit, [] {});
            unit = un;
        };
        if (unit < u_end) ask(f0);
        while (unit < u_end) {
            turn(f0, f1);
            if (unit >= u_end) break;
            turn(f1, f0);
        }
    } else {                                            // one: the next K behind the scores, the next V behind the output
        Unit f;
        if (unit < u_end) { ask_k(f, at_k); ask_v(f, at_v); }
        while (unit < u_end) {
            const int un = next(unit + W);
            work(f, unit, [&] { if (un < u_end) ask_k(f, at_k); });
            __builtin_amdgcn_sched_barrier(0);
            if (un < u_end) ask_v(f, at_v);
            __builtin_amdgcn_sched_barrier(0);
            unit = un;
        }
    }

    // four dims of row r of column block t, unnormalised: the row's maximum and sum of weights; found: something was taken out of V
    auto put = [&](int t, int r, int d, float (&v)[4], float top, float sum, float inv, bool found) {
        const int row = (tile * NT + t) * 16 + r, token = row / a.kv.group, head = kvh * a.kv.group + row % a.kv.group;
        if (row >= rows) return;
        if (found) {                                     // what the row sees among the item's keys, but for units that all rows see
            const int end = SEES == KV_SHARED ? from : base + token, row_low = SEES == KV_WINDOW ? end - window + 1 : low;
            const int main0 = (max(low_last, 0) + UK - 1) / UK * UK, main1 = (from + 1) / UK * UK;
            const int first_key = steps.at(max(u_begin, steps.first)) * UK, last_key = min(end, (u_end + steps.skip) * UK - 1);
            for (int j = 0; j < 4; ++j) {
                v[j] += kv_odd_sum<C, H>(a.kv, seq, kvh, first_key, last_key, d + j, row_low, sinks, main0, main1);
                if (TWO && u_begin < steps.first)
                    v[j] += kv_odd_sum<C, H>(a.kv, first_seq, kvh, u_begin * UK, min(min(end, (SEES == KV_BOTH ? low : sinks) - 1), u_end * UK - 1), d + j, 0, 0, 0, (SEES == KV_BOTH ? low : sinks) / UK * UK);
            }
        }
        if (it.whole) {
            v[0] *= inv; v[1] *= inv; v[2] *= inv; v[3] *= inv;
            store4<A>((E*)a.out + (s.r0 + (int64_t)token) * a.out_stride + head * H + d, v);
        } else {
            const size_t at = (size_t)it.part * (16 * NT) + t * 16 + r;
            *(float4*)(a.o_part + at * H + d) = float4{v[0], v[1], v[2], v[3]};
            if (d == 0) { a.ml_part[at * 2] = top; a.ml_part[at * 2 + 1] = sum; }
        }
    };
    if constexpr (W == 1) {                              // an item to each wave: nothing to merge
        const bool found = __any(odd);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const float sum = groups_sum(l[t]), inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
            for (int ht = 0; ht < HT; ++ht) {
                float v[4] = {o[t][ht][0], o[t][ht][1], o[t][ht][2], o[t][ht][3]};
                put(t, m, ht * 16 + 4 * g, v, mx[t], sum, inv, found);
            }
        }
        return;
    }
    // ---- the waves' results, 16 rows at a time, wave order
    __syncthreads();                                    // (sh.odd is cleared)
    if (odd && lane == 0) sh.odd = 1;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        if (t) __syncthreads();
        l[t] = groups_sum(l[t]);
        if (g == 0) { sh.ml[w][m][0] = mx[t]; sh.ml[w][m][1] = l[t]; }
#pragma unroll
        for (int ht = 0; ht < HT; ++ht) *(f32x4*)&sh.o[w][m][ht * 16 + 4 * g] = o[t][ht];
        __syncthreads();
        const int r = tid & 15;
        float top = -INFINITY, sum = 0.f, wt[4];
#pragma unroll
        for (int ww = 0; ww < 4; ++ww) top = fmaxf(top, sh.ml[ww][r][0]);
        const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (int ww = 0; ww < 4; ++ww) { wt[ww] = __builtin_amdgcn_exp2f((sh.ml[ww][r][0] - ref) * a.c2); sum += sh.ml[ww][r][1] * wt[ww]; }
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        for (int d = (tid >> 4) * 4; d < H; d += 64) {
            float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ww = 0; ww < 4; ++ww) {
                const f32x4 x = *(const f32x4*)&sh.o[ww][r][d];
                v[0] += x[0] * wt[ww]; v[1] += x[1] * wt[ww]; v[2] += x[2] * wt[ww]; v[3] += x[3] * wt[ww];
            }
            put(t, r, d, v, top, sum, inv, sh.odd != 0);
        }
    }
}

template <class A, class C, int H, int NT>
__global__ __launch_bounds__(256, A::KE == 4 ? 1 : 2) void kv_attend_kernel(const KvAttendArgs a) {
    __shared__ KvFewLds<H> lds;
    const int lane = threadIdx.x & 63;
    KvItem it;
    int local;
    int64_t first;
    const bool check = blockIdx.x == 0 && threadIdx.x < 64;
    KvLanes all;
    all.load(a.kv, 0, lane, check);
    auto chunks = [](const KvSeq& v) { return (v.len + 63) / 64; };
    const int run = kv_run<NT>(a, all, lane, chunks), n_kv = a.kv.n_kv;
    if (!kv_find(a.kv, all, blockIdx.x, lane, check, [&](const KvSeq& v) { return kv_tiles<NT>(a.kv, v) * kv_splits(chunks(v), run) * n_kv; }, &it.seq, &local, &first, &it.s)) return;
    const int n_tiles = kv_tiles<NT>(a.kv, it.s), n_splits = kv_splits(chunks(it.s), run);
    it.kvh = local % n_kv; it.tile = local / n_kv % n_tiles; it.split = local / n_kv / n_tiles;
    it.per = kv_per_split(chunks(it.s), n_splits);
    it.whole = n_splits == 1;
    it.part = blockIdx.x;
    kv_few_rows<A, C, H, NT, KV_ALL, 4>(a, it, lds);
}

// Many rows (bf16): NW waves with 16 * NT rows each walk a run of chunks together, their fragments in LDS once for all of them.  They come by
// direct loads into a ring of five half-chunks (K, V^T, K, ..): one barrier per chunk c, behind which K and V^T of c have landed
// and the slots of c - 1 may be asked for anew (V^T of c + 1, K of c + 2).  A SIMD has two waves.
// (Prompts of 1035 to 2048 tokens, 32 heads x 128, bf16 pages, took 160 us so at the step when four waves of 16 rows took 199 and two waves with the
// next product's fragments in registers 200, both spilling.)  Bound by products, exponentials (in 8 bits the widening, too, which each wave does for itself) and the
// fragments' way out of LDS, each of them about 2000 cycles of a compute unit for a step of two workgroups (bf16 pages), which takes 2900 (8 bits 3400 to 4000; one
// workgroup alone 3300): the vector unit issues in 48 to 53 % of the busy cycles (8 bits 73 to 76), the matrix cores are at work in 33 to 38.  And by what each tile takes
// once, about 10000 cycles in front (its item, the page table, queries, first fragments) and 4000 behind; a step with an edge takes 5000: the chunk's V^T is looked
// through, and rows are masked on the side on which some see less.  (7600 with a mask of three comparisons per score and V^T written back always, behind a barrier of its own:
// prompts of 4096, 3575, 2070 and 4062 tokens, window 1024: 325 us, 281 to 300 so.)
// The prompts above now take 134 to 137 us (8-bit pages 154), 750 TFLOP/s, one of 8192 tokens 1058 TFLOP/s (967); 512 rows behind 8195 tokens and 260 behind 2665 in 8
// bits, 64 / 8 heads, 209 us with the join, with a window of 2048 92 us.
template <class C, int H> constexpr int KV_RING = 5 * KvLayout<C, H>::K_BYTES / 16 + (KvLayout<C, H>::Q8 ? 4 * 8 : 0);       // (bf16 at head dim 128: two of them are a unit's whole LDS)
template <class C, int H, int NT, int NW, int SEES, class Args> __device__ __forceinline__ void kv_many_rows(const Args& a, const KvItem& item, u32x4 (&mem)[KV_RING<C, H>]) {
    static_assert(SEES != KV_OWN, "own keys behind shared ones, apart from them, are kv_few_rows'");
    using A = BF16;
    using L = KvLayout<C, H>;
    constexpr int AE = A::KE, KK = L::KK, HP = L::HP, US = KK / AE, QS = HP * US, HT = L::HT, KST = L::KST, VS = L::KV / AE, PS = KST * VS;
    constexpr int HF = L::K_BYTES / 1024, LH = HF / NW, SLOTS = 5, SC = 4, X = L::Q8 ? 1 : 0, RT = NW * NT;      // fragments of a half, requests per wave and half; chunks' scales; 16-row blocks of a tile
    static_assert(HF % NW == 0 && HF == 4 * HP && HF == HT * KST, "every wave asks for the same number of fragments");
    const int tid = threadIdx.x, lane = tid & 63, w = uniform(tid >> 6), g = lane >> 4, m = lane & 15;
    const KvItem it = item.scalar();
    const int seq = it.seq, kvh = it.kvh, tile = it.tile, per = it.per, n_kv = a.kv.n_kv;
    const KvSeq s = it.s;
    const int rows = s.n * a.kv.group, base = s.len - s.n, row0 = (tile * NW + w) * NT * 16;
    // last key of row `row`'s token
    auto reach = [&](int row) { return SEES == KV_SHARED ? s.len - 1 : base + row / a.kv.group; };
    const int from = reach(tile * RT * 16), last = reach(min((tile + 1) * 16 * RT, rows) - 1);                 // ... of the workgroup's first and last row
    const int my_from = reach(row0), my_last = row0 < rows ? reach(min(row0 + 16 * NT, rows) - 1) : -1;           // ... of this wave's
    int window = 0, sinks = 0, low = 0, low_last = 0, my_low = 0, my_low_last = 0;                               // first keys of those rows' windows (KV_BOTH: of all rows)
    if constexpr (SEES == KV_WINDOW) {
        window = a.window; sinks = a.sinks;
        low = from - window + 1; low_last = last - window + 1; my_low = my_from - window + 1; my_low_last = my_last - window + 1;
    }
    if constexpr (SEES == KV_BOTH) low = low_last = my_low = my_low_last = s.low;
    // Steps of one chunk: those of the workgroup's run, those that all its rows see whole
    const KvSteps steps = kv_steps<SEES>(a, low, 64);
    const int c0 = it.split * per, c_end = min((last + 64) / 64 - steps.skip, c0 + per);
    const int main0 = max((max(low_last, 0) + 63) / 64 - steps.skip, c0), main1 = min(c_end, (from + 1) / 64 - steps.skip);
    const int first_main = SEES == KV_BOTH ? min(low / 64, c_end) : SEES == KV_WINDOW && steps.first ? min(sinks / 64, c_end) : 0;      // ... and the first ones
    // The page of the chunk asked for next: the table's entries lie in the wave's lanes, those of the first steps apart from the others.  (Asked for ahead of the
    // queries: the first chunk's request waits for them alone.)
    constexpr bool TWO = SEES == KV_WINDOW || SEES == KV_BOTH;
    const int cpp = a.kv.page_tokens / 64, r0 = steps.at(c0), first_seq = SEES == KV_BOTH ? s.lead : seq;
    int page_i = r0 / cpp, in_page = r0 % cpp;
    KvPages pages, later;
    if (c_end > c0) {
        pages.load(a.kv, TWO && c0 < steps.first ? first_seq : seq, page_i, lane);
        if constexpr (TWO) if (c0 < steps.first && c_end > steps.first) later.load(a.kv, seq, (steps.first + steps.skip) / cpp, lane);
    }
    int pos[NT];
    u32x4 qf[NT][QS];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int row = row0 + t * 16 + m, token = row / a.kv.group, head = kvh * a.kv.group + row % a.kv.group;
        const bool on = row < rows;
        pos[t] = on ? SEES == KV_SHARED ? s.len - 1 : base + token : -1;
        const uint16_t* qp = (const uint16_t*)a.q + (s.r0 + (int64_t)token) * a.q_stride + head * H;
#pragma unroll
        for (int i = 0; i < QS; ++i) qf[t][i] = on ? *(const u32x4*)(qp + i / US * 4 * KK + g * KK + i % US * AE) : u32x4{0u, 0u, 0u, 0u};
    }
    f32x4 o[NT][HT];
    float mx[NT], l[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        mx[t] = -INFINITY; l[t] = 0.f;
#pragma unroll
        for (int ht = 0; ht < HT; ++ht) o[t][ht] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    bool odd = false;                                    // this lane has taken a value out of V
    if (c_end > c0) {
        uint32_t gone = 0;                               // bit c % 32: the chunk of step c has no page
        bool lost = false;
        int asked = c0;                                  // chunk whose K is asked for next
        const char* src = nullptr;                       // the chunk whose K was asked for last; n_bytes 0: nowhere, zeros come back
        int n_bytes = 0, slot_k = 0, slot_v = 1;
        auto half = [&](const char* from_, const int n, const int slot) {
            // (a descriptor in scalar registers: the loads would be issued lane by lane otherwise)
            from_ = (const char*)((uint64_t)(uint32_t)uniform((int)(uintptr_t)from_) | (uint64_t)(uint32_t)uniform((int)((uintptr_t)from_ >> 32)) << 32);
            const uint32_t bytes = (uint32_t)uniform(n);
#pragma unroll
            for (int q = 0; q < LH; ++q) frag_to_lds(from_ + (w + NW * q) * 1024, bytes, mem + slot * HF * 64 + (w + NW * q) * 64, lane);
        };
        auto ask_k = [&]() {                             // past the end: nothing, the requests are only counted
            if (asked < c_end) {
                const int page = pages.at(page_i);
                src = a.kv.pages + (((size_t)max(page, 0) * n_kv + kvh) * cpp + in_page) * L::CHUNK;
                n_bytes = page >= 0 ? -1 : 0;
                gone = page >= 0 ? gone & ~(1u << (asked & 31)) : gone | 1u << (asked & 31);
                lost |= page < 0;
                if (++in_page == cpp) { in_page = 0; ++page_i; }
                if constexpr (TWO) if (asked + 1 == steps.first) {
                    page_i = (steps.first + steps.skip) / cpp; in_page = (steps.first + steps.skip) % cpp;
                    pages = later;
                }
            } else {
                n_bytes = 0;
            }
            half(src, n_bytes, slot_k);
            if constexpr (L::Q8)
                if (lane < 8) frag_to_lds(src + 2 * L::K_BYTES, (uint32_t)uniform(n_bytes & 128), mem + SLOTS * HF * 64 + asked % SC * 8, lane);
            ++asked;
            slot_k = slot_k + 2 >= SLOTS ? slot_k + 2 - SLOTS : slot_k + 2;
        };
        auto ask_v = [&](const char* p, const int n) {
            half(p + L::K_BYTES, n, slot_v);
            slot_v = slot_v + 2 >= SLOTS ? slot_v + 2 - SLOTS : slot_v + 2;
        };
        int use_k = 0, use_v = 1;                        // slots of the chunk at hand
        ask_k(); ask_v(src, n_bytes); ask_k();           // K, V^T of the first chunk, K of the next
        wait_vm<3 * LH + 2 * X, true>();                 // the queries are there: from here on only the ring's requests count
        auto turn = [&]() {
            if (page_i - pages.base >= 62) {             // (once in 62 pages: the ring runs dry for a moment)
                pages.load(a.kv, TWO && asked < steps.first ? first_seq : seq, page_i, lane);
                wait_vm<0, false>();
            }
            wait_vm<LH + X, true>();                     // the K of the next chunk may still be on its way
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
        };
        auto ask = [&]() { ask_v(src, n_bytes); ask_k(); };      // V^T of the next chunk, K of the one behind it
        // the written keys that belong to step c: first_key .. last_key - 1
        auto first_key = [&](int c) { return SEES == KV_BOTH && c >= steps.first ? low : 0; };
        auto last_key = [&](int c) { return SEES == KV_BOTH && c < steps.first ? low : s.len; };
        auto cleaned = [&]() {
            asm volatile("" ::: "memory");
            wait_vm<63, true>();                         // (the ring's requests go on)
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
        };
        // step c, chunk r: one that this wave has products for; edge: some of its rows do not see all of it
        auto work = [&](const int c, const int r, auto is_edge) {
            constexpr bool edge = decltype(is_edge)::value;
            const u32x4 *kp = mem + use_k * HF * 64 + lane, *vp = mem + use_v * HF * 64 + lane;
            f32x4 sc[NT][4];
            const uint8_t* ex = (const uint8_t*)(mem + SLOTS * HF * 64 + c % SC * 8);
            u32x4 ke{}, ve{};
            if constexpr (L::Q8) { ke = *(const u32x4*)(ex + 16 * (m >> 2)); ve = *(const u32x4*)(ex + 64 + 16 * g); }
            // The four score tiles side by side, so that no product waits for the one before it, and the fragments of a step
            // are read while the step before it runs; so too the output tiles below, two at a time (the fences keep that order)
            u32x4 f[2][4];
            __builtin_amdgcn_s_setprio(1);               // products ahead of what else the other wave has to issue
#pragma unroll
            for (int kt = 0; kt < 4; ++kt) f[0][kt] = kp[kt * HP * 64];
#pragma unroll
            for (int hp = 0; hp < HP; ++hp) {
#pragma unroll
                for (int kt = 0; kt < 4; ++kt)
                    if (hp + 1 < HP) f[(hp + 1) & 1][kt] = kp[(kt * HP + hp + 1) * 64];
                    else if (!edge) f[(hp + 1) & 1][kt] = vp[kt * 64];
#pragma unroll
                for (int u = 0; u < US; ++u)
#pragma unroll
                    for (int kt = 0; kt < 4; ++kt) {
                        float scale = 1.f;
                        if constexpr (L::Q8) scale = q8_scale((ke[kt] >> (8 * (m & 3))) & 255u);
                        const u32x4 x = kv_operand<A, C>(f[hp & 1][kt], u, scale);
#pragma unroll
                        for (int t = 0; t < NT; ++t) {
                            if (hp == 0 && u == 0) sc[t][kt] = f32x4{0.f, 0.f, 0.f, 0.f};
                            mma16<A>(sc[t][kt], x, qf[t][hp * US + u]);
                        }
                    }
                __builtin_amdgcn_sched_barrier(0);
            }
            __builtin_amdgcn_s_setprio(0);
            ask();
            float vs[4][4];
            if constexpr (L::Q8)
#pragma unroll
                for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t e = (ve[kt] >> (8 * j)) & 255u;
                        vs[kt][j] = q8_scale(edge ? min(e, 254u) : e);      // (a key that no row sees may have any scale: its weight, 0, times a finite one is 0; written ones are below)
                    }
            if constexpr (edge) {
                // Masks by the places of a row's first and last key in the chunk, and only on the side on which some row of the wave does not see all of it (a lane's
                // keys: those of lane group 0, at constants, and `at` on)
                const bool first = TWO && c < steps.first;
                const int at = r * 64 + score_key<C>(0, 4 * g), end = first ? (SEES == KV_WINDOW ? sinks : low) - 1 : 0x7fffffff;
                if (r * 64 + 63 > min(my_from, end)) {
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        const int most = min(pos[t], end) - at;
#pragma unroll
                        for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                            for (int j = 0; j < 4; ++j) if (score_key<C>(kt, j) > most) sc[t][kt][j] = -INFINITY;
                    }
                }
                if constexpr (SEES == KV_WINDOW || SEES == KV_BOTH) if (!first && r * 64 < my_low_last) {
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        const int least = (SEES == KV_WINDOW ? pos[t] - window + 1 : low) - at, after = SEES == KV_WINDOW ? max(sinks - at, -64) : -64;      // (hidden: after .. least - 1)
                        const uint32_t gap = (uint32_t)max(least - after, 0);
#pragma unroll
                        for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                            for (int j = 0; j < 4; ++j) if ((uint32_t)(score_key<C>(kt, j) - after) < gap) sc[t][kt][j] = -INFINITY;
                    }
                }
            }
            u32x4 pf[NT][PS];
            // The reference of a row's exponents need not be its maximum: it moves only when a weight would pass 2^8 (one branch for all column blocks, so that their chains run
            // side by side)
            float cm[NT];
            bool past = false;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                cm[t] = sc[t][0][0];
#pragma unroll
                for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                    for (int j = 0; j < 4; ++j) cm[t] = fmaxf(cm[t], sc[t][kt][j]);
                cm[t] = groups_max(cm[t]);
                past = past || (cm[t] - mx[t]) * a.c2 > 8.f;
            }
            if (__any(past)) {
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    if (!__any((cm[t] - mx[t]) * a.c2 > 8.f)) continue;
                    const float mn = fmaxf(mx[t], cm[t]), alpha = mn == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((mx[t] - mn) * a.c2);
                    mx[t] = mn;
                    l[t] *= alpha;
#pragma unroll
                    for (int ht = 0; ht < HT; ++ht) { o[t][ht][0] *= alpha; o[t][ht][1] *= alpha; o[t][ht][2] *= alpha; o[t][ht][3] *= alpha; }
                }
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const float off = mx[t] == -INFINITY ? 0.f : -mx[t] * a.c2;
                float sum[2] = {0.f, 0.f};
#pragma unroll
                for (int kt = 0; kt < 4; ++kt) {
                    float e[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) { e[j] = __builtin_amdgcn_exp2f(fmaf(sc[t][kt][j], a.c2, off)); sum[j & 1] += e[j]; }
                    if constexpr (L::Q8)
#pragma unroll
                        for (int j = 0; j < 4; ++j) e[j] *= vs[kt][j];
                    pf[t][kt / 2][kt % 2 * 2] = bf16_pair(e[0], e[1]);      // as V is: see kv_few_rows
                    pf[t][kt / 2][kt % 2 * 2 + 1] = bf16_pair(e[2], e[3]);
                }
                l[t] += sum[0] + sum[1];
            }
            if constexpr (edge) {
                cleaned();
#pragma unroll
                for (int j = 0; j < 4; ++j) f[HP & 1][j] = vp[j * 64];
            }
            __builtin_amdgcn_s_setprio(1);
            constexpr int HG = 4 / KST;                  // output tiles of a step
#pragma unroll
            for (int q = 0; q < HF / 4; ++q) {
                u32x4 (&now)[4] = f[(HP + q) & 1];
                if (q + 1 < HF / 4) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) f[(HP + q + 1) & 1][j] = vp[(q * 4 + 4 + j) * 64];
                }
#pragma unroll
                for (int ks = 0; ks < KST; ++ks)
#pragma unroll
                    for (int u = 0; u < VS; ++u)
#pragma unroll
                        for (int h = 0; h < HG; ++h) {
                            const u32x4 v = kv_operand<A, C>(now[h * KST + ks], u, 1.f);
#pragma unroll
                            for (int t = 0; t < NT; ++t) mma16<A>(o[t][q * HG + h], v, pf[t][ks * VS + u]);
                        }
                __builtin_amdgcn_sched_barrier(0);
            }
            __builtin_amdgcn_s_setprio(0);
        };
        // A chunk with an edge: keys behind the end and values that are not finite leave V^T (see kv_clean) before its products; each wave cleans what it has
        // asked for, behind `cleaned` it has been done
        auto clean = [&](const int c, const int r) {
            const int n_keys = last_key(c) - r * 64, cut = first_key(c) - r * 64;
            const bool part = n_keys < 64 || cut > 0;
            u32x4* p = mem + (use_v * HF + w) * 64 + lane;
            u32x4 f[LH];
            uint32_t hit = 0;
#pragma unroll
            for (int q = 0; q < LH; ++q) f[q] = p[NW * q * 64];
            if (part)
#pragma unroll
                for (int q = 0; q < LH; ++q)
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        f[q][x] &= kv_kept<C>(n_keys, (w + NW * q) % KST, g, x);
                        if constexpr (SEES == KV_BOTH) f[q][x] &= ~kv_kept<C>(cut, (w + NW * q) % KST, g, x);
                    }
#pragma unroll
            for (int q = 0; q < LH; ++q)
#pragma unroll
                for (int x = 0; x < 4; ++x) hit |= kv_odd<C>(f[q][x]);
            if (part || __any(hit != 0))
#pragma unroll
                for (int q = 0; q < LH; ++q) {
#pragma unroll
                    for (int x = 0; x < 4; ++x) f[q][x] = kv_clean<C>(f[q][x]);
                    p[NW * q * 64] = f[q];
                }
            odd |= hit != 0;
        };
        auto done = [&]() {
            use_k = use_k + 2 >= SLOTS ? use_k + 2 - SLOTS : use_k + 2;
            use_v = use_v + 2 >= SLOTS ? use_v + 2 - SLOTS : use_v + 2;
        };
        // Chunks that all rows of the workgroup see run in a loop of their own, without masks; those with an edge, or without a page, one by one
        int c = c0;
        for (;;) {
            for (const int stop = c < first_main ? first_main : c >= main0 ? main1 : c; c < stop && gone == 0; ++c) {
                turn();
                work(c, steps.at(c), std::false_type{});
                done();
            }
            if (c >= c_end) break;
            turn();
            const int r = steps.at(c);
            if (c >= first_main && (c < main0 || c >= main1)) clean(c, r);       // (beside a missing page: what all rows see goes through the products)
            bool mine = r * 64 <= my_last;
            if constexpr (SEES == KV_WINDOW) mine = mine && (r * 64 + 63 >= my_low || r * 64 < sinks);
            if (mine && !((gone >> (c & 31)) & 1u)) work(c, r, std::true_type{}); else { ask(); cleaned(); }
            done();
            gone &= ~(1u << (c & 31));
            ++c;
        }
        if (lost && tid == 0) kv_flag(a.kv, ASD_KV_BAD_PAGE);
        wait_vm<0, true>();                              // no request may outlive the workgroup's LDS
        __syncthreads();
        int* any = (int*)mem;                            // the ring is free: what one lane has taken out concerns all
        const bool found = __any(odd);
        if (lane == 0) any[w] = found;
        __syncthreads();
        odd = any[lane % NW] != 0;
        odd = __any(odd);
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const float z = groups_sum(l[t]);
        const int row = row0 + t * 16 + m, token = row / a.kv.group, head = kvh * a.kv.group + row % a.kv.group;
        if (row >= rows) continue;
        const size_t at = (size_t)it.part * (16 * RT) + row - tile * 16 * RT;
        uint16_t* out = (uint16_t*)a.out + (s.r0 + (int64_t)token) * a.out_stride + head * H;
        if (it.whole) {
            const float inv = z == 0.f ? 0.f : 1.f / z;
#pragma unroll
            for (int ht = 0; ht < HT; ++ht) {
                const float v[4] = {o[t][ht][0] * inv, o[t][ht][1] * inv, o[t][ht][2] * inv, o[t][ht][3] * inv};
                store4<A>(out + ht * 16 + 4 * g, v);
            }
        } else {
#pragma unroll
            for (int ht = 0; ht < HT; ++ht) *(f32x4*)(a.o_part + at * H + ht * 16 + 4 * g) = o[t][ht];
            if (g == 0) { a.ml_part[at * 2] = mx[t]; a.ml_part[at * 2 + 1] = z; }
        }
        if (odd) {                                       // (each lane changes what it has stored)
            for (int d = 0; d < H / 4; ++d) {
                const int dim = d / 4 * 16 + 4 * g + d % 4;
                float x = kv_odd_sum<C, H>(a.kv, seq, kvh, steps.at(max(c0, steps.first)) * 64, min(pos[t], (c_end + steps.skip) * 64 - 1), dim,
                                           SEES == KV_WINDOW ? pos[t] - window + 1 : low, sinks, (main0 + steps.skip) * 64, (main1 + steps.skip) * 64);
                if ((SEES == KV_WINDOW || SEES == KV_BOTH) && c0 < steps.first)
                    x += kv_odd_sum<C, H>(a.kv, SEES == KV_BOTH ? s.lead : seq, kvh, c0 * 64, min(min(pos[t], (SEES == KV_BOTH ? low : sinks) - 1), c_end * 64 - 1), dim, 0, 0, 0, first_main * 64);
                if (finite(x)) continue;                 // (nothing of its own row's to add)
                if (it.whole) out[dim] = BF16::from_f32(BF16::to_f32(out[dim]) + x); else a.o_part[at * H + dim] += x;
            }
        }
    }
}

template <class C, int H, int NT, int NW>
__global__ __launch_bounds__(64 * NW, 2) void kv_rows_kernel(const KvAttendArgs a) {
    constexpr int RT = NW * NT;
    __shared__ u32x4 mem[KV_RING<C, H>];
    const int lane = threadIdx.x & 63;
    KvItem it;
    int local;
    int64_t first;
    const bool check = blockIdx.x == 0 && threadIdx.x < 64;
    KvLanes all;
    all.load(a.kv, 0, lane, check);
    auto chunks = [](const KvSeq& v) { return (v.len + 63) / 64; };
    const int run = kv_run<RT>(a, all, lane, chunks), n_kv = a.kv.n_kv;
    if (!kv_find(a.kv, all, blockIdx.x, lane, check, [&](const KvSeq& v) { return kv_tiles<RT>(a.kv, v) * kv_splits(chunks(v), run) * n_kv; }, &it.seq, &local, &first, &it.s)) return;
    const int n_tiles = kv_tiles<RT>(a.kv, it.s), n_splits = kv_splits(chunks(it.s), run);
    it.kvh = local % n_kv; it.tile = n_tiles - 1 - local / n_kv % n_tiles; it.split = local / n_kv / n_tiles;      // longest first
    it.per = kv_per_split(chunks(it.s), n_splits);
    it.whole = n_splits == 1;
    it.part = first + (int64_t)(it.split * n_tiles + it.tile) * n_kv + it.kvh;
    kv_many_rows<C, H, NT, NW, KV_ALL>(a, it, mem);
}

// Joins the runs of tiles whose keys were cut: a workgroup per tile, KV head and 16 of its rows.  16 lanes hold a row's dims;
// where fewer rows are in use than 16, the lanes left over take every second (fourth, ..) run, added up through LDS at the end.  A launch of its own,
// 4 to 5 us for one token's runs, 13 us for those of 772 rows: joined by the last workgroup to arrive, counters would have to be zero when the
// call starts, and the workspace could not be any memory.
// A run's sums of a row, and its maximum and sum of weights
struct KvPartial { const float *o, *ml; };
// rows row0 .. row0 + left - 1 (16 at most) of a sequence and KV head: place(run, r), the run's partial sums of row row0 + r
template <class A, int H, class F> __device__ __forceinline__ void kv_join_rows(const KvAttendArgs& a, const KvSeq& s, int kvh, int row0, int left, int n_runs, F place) {
    using E = typename A::elem;
    constexpr int DL = H / 16, U = 8;                   // dims of a lane, runs in flight
    __shared__ float so[16][H];
    __shared__ float sml[16][2];
    const int tid = threadIdx.x, group = a.kv.group;
    const int lg = left > 8 ? 4 : left > 4 ? 3 : left > 2 ? 2 : left > 1 ? 1 : 0, phases = 16 >> lg;
    const int r = (tid >> 4) & ((1 << lg) - 1), phase = tid >> (4 + lg), d0 = (tid & 15) * DL;
    float acc[DL] = {}, top = -INFINITY, sum = 0.f;
    if (r < left)
        for (int i0 = phase; i0 < n_runs; i0 += U * phases) {
            float x[U][DL];
            float2 ml[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const bool on = i0 + u * phases < n_runs;
                const KvPartial p = place(on ? i0 + u * phases : i0, r);
                ml[u] = *(const float2*)p.ml;
                if (!on) ml[u] = float2{-INFINITY, 0.f};
#pragma unroll
                for (int d = 0; d < DL; d += 2) { const float2 y = *(const float2*)(p.o + d0 + d); x[u][d] = y.x; x[u][d + 1] = y.y; }
            }
            float mn = top;
#pragma unroll
            for (int u = 0; u < U; ++u) mn = fmaxf(mn, ml[u].x);
            const float ref = mn == -INFINITY ? 0.f : mn, alpha = __builtin_amdgcn_exp2f((top - ref) * a.c2);
            top = mn;
            sum *= alpha;
#pragma unroll
            for (int d = 0; d < DL; ++d) acc[d] *= alpha;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (i0 + u * phases >= n_runs) break;
                const float wt = __builtin_amdgcn_exp2f((ml[u].x - ref) * a.c2);
                sum += ml[u].y * wt;
#pragma unroll
                for (int d = 0; d < DL; ++d) acc[d] += x[u][d] * wt;
            }
        }
    if (phases > 1) {
#pragma unroll
        for (int d = 0; d < DL; ++d) so[tid >> 4][d0 + d] = acc[d];
        if ((tid & 15) == 0) { sml[tid >> 4][0] = top; sml[tid >> 4][1] = sum; }
        __syncthreads();
        if (phase) return;
        float mn = -INFINITY;
        for (int q = 0; q < phases; ++q) mn = fmaxf(mn, sml[(q << lg) + r][0]);
        const float ref = mn == -INFINITY ? 0.f : mn;
        sum = 0.f;
#pragma unroll
        for (int d = 0; d < DL; ++d) acc[d] = 0.f;
        for (int q = 0; q < phases; ++q) {
            const float wt = __builtin_amdgcn_exp2f((sml[(q << lg) + r][0] - ref) * a.c2);
            sum += sml[(q << lg) + r][1] * wt;
#pragma unroll
            for (int d = 0; d < DL; ++d) acc[d] += so[(q << lg) + r][d0 + d] * wt;
        }
    }
    if (r >= left) return;
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    const int row = row0 + r, token = row / group, head = kvh * group + row % group;
    E* out = (E*)a.out + (s.r0 + (int64_t)token) * a.out_stride + head * H + d0;
#pragma unroll
    for (int d = 0; d < DL; d += 2) {
        if constexpr (sizeof(E) == 2) *(uint32_t*)(out + d) = bf16_pair(acc[d] * inv, acc[d + 1] * inv);
        else *(float2*)(out + d) = float2{acc[d] * inv, acc[d + 1] * inv};
    }
}

template <class A, int H, int NT>
__global__ __launch_bounds__(256) void kv_join_kernel(const KvAttendArgs a) {
    constexpr int R = 16 * NT;                          // rows of a tile
    const int lane = threadIdx.x & 63, n_kv = a.kv.n_kv, group = a.kv.group;
    int seq, local;
    int64_t first;
    KvSeq s;
    KvLanes all;
    all.load(a.kv, 0, lane, false);
    auto chunks = [](const KvSeq& v) { return (v.len + 63) / 64; };
    const int run = kv_run<NT>(a, all, lane, chunks);
    // (tile, KV head) pairs of the cut sequences
    if (!kv_find(a.kv, all, blockIdx.x, lane, false, [&](const KvSeq& v) { return kv_splits(chunks(v), run) > 1 ? kv_tiles<NT>(a.kv, v) * n_kv : 0; }, &seq, &local, &first, &s)) return;
    // the first work item of the sequence
    int64_t item0 = 0;
    for (int s0 = 0; s0 <= seq; s0 += 64) {
        if (s0) all.load(a.kv, s0, lane, false);
        int64_t c = s0 + lane < seq ? (int64_t)kv_tiles<NT>(a.kv, all.v) * kv_splits(chunks(all.v), run) * n_kv : 0;
        item0 += seq ? wave_sum(c) : 0;
    }
    const int n_splits = kv_splits(chunks(s), run), n_tiles = kv_tiles<NT>(a.kv, s), kvh = local % n_kv, tile = local / n_kv;
    const int row0 = tile * R + blockIdx.y * 16, left = min(s.n * group - row0, 16);
    if (left <= 0) return;
    const int64_t step = (int64_t)n_tiles * n_kv * R, at = (item0 + (int64_t)tile * n_kv + kvh) * R + blockIdx.y * 16;      // a run's place to the next run's
    kv_join_rows<A, H>(a, s, kvh, row0, left, n_splits, [&](int i, int r) { const int64_t p = at + r + i * step; return KvPartial{a.o_part + p * H, a.ml_part + p * 2}; });
}
