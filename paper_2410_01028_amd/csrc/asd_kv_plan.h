// How the attention of a batch is run: which kernel, which tiles, how keys are cut.
#pragma once
#include "asd_kv_host.h"

namespace {

// How attention over a batch of these bounds runs
struct AttendPlan {
    int nt;                        // 16-row column blocks of a tile
    bool rows;                     // kv_rows_kernel
    int32_t target, max_tiles, min_run;
    int64_t grid;                  // most work items
    bool join;                     // some sequence's keys may be cut
    int32_t tail;                  // > 0: only the tiles of the last, partly filled round are, into this many runs at most
    int64_t join_blocks;           // 16-row blocks that may be joined
    size_t o_bytes, bytes;
};
// What differs between the forms of attention.  PLAN_CAUSAL: asd_kv_attend, whose sums stay as they are.  PLAN_EVEN: tiles of a batch walk about as many chunks each (a
// window).  PLAN_BOTH: as causal attention.  PLAN_FRONT: keys that groups share, for the rows of a group.  PLAN_WAVE: an item is a wave's, of 16 rows.
enum PlanForm { PLAN_CAUSAL, PLAN_EVEN, PLAN_BOTH, PLAN_FRONT, PLAN_WAVE };
// walk(R): the chunks that tiles of R rows walk at most
template <class F> AttendPlan attend_plan(const asd_kv_shape* s, const asd_kv_batch* b, F walk, PlanForm form = PLAN_CAUSAL) {
    AttendPlan p{};
    const int group = s->n_heads / s->n_kv_heads;
    const int64_t rows = (int64_t)b->max_new * group;
    int64_t chunks = walk(16);
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
    // Shared keys are read from memory once either way: 128 rows as soon as they are more than two tiles, and the work more than a chunk or two for each compute unit (64 / 8
    // heads, 8 bits, one token of 64 sequences behind 1000 shared ones: 24 us against 30, behind 4000 32 against 48; five of 8 sequences behind 1000: 19.4 against 17.6)
    if (form == PLAN_FRONT) p.rows = bf16 && s->head_dim >= 64 && rows > 32 && work * chunks > 12 * (int64_t)units();
    if (form == PLAN_WAVE) p.rows = false;
    if (p.rows) p.nt = 8;
    if (form == PLAN_WAVE) p.nt = 1;
    p.max_tiles = (int32_t)tiles(p.nt);
    chunks = walk(16 * p.nt);
    // Keys are cut into about four items per compute unit (48 sequences of 500 to 8192 tokens: 90 us, with two 100, with eight 97), but not
    // into runs of fewer than 16 chunks (with 8, five rows of eight sequences of 1031 tokens take 19.1 us, not 16.9), and not where
    // kv_rows_kernel's tiles are as many by themselves: full ones, or, as long as none is long, ones that a token alone may have.  (64 / 8 heads x 128,
    // 8 bits, 128 tokens behind 400, 512 rows behind 3488 and a token behind 4000: 164 us, cut 177; behind 8192: 245 and 178; behind 60000: 1493
    // and 221.  128 tokens behind 400 .. 8192 and the 512 rows: 402 and 428, behind 400 .. 16384 734 and 703)
    p.min_run = 16;
    p.target = 4 * units();
    const int64_t whole = (int64_t)p.max_tiles * s->n_kv_heads;
    // Fewer tiles than compute units: runs of four chunks are worth their join (a token of one sequence of 8192, window 4096, 32 / 32 heads x 128, bf16 pages: 20 us against 23.5)
    if ((form == PLAN_EVEN || form == PLAN_BOTH) && whole < units()) { p.min_run = 4; p.target = units(); }
    // Shared keys: runs of 8 chunks (128 rows: 16), shorter ones as long as there are fewer than compute units (sixteen samples of a prompt of 2048 tokens, 32 / 32 heads, bf16
    // pages: 28.4 us with 16, 25.8 with 8; one token of 16 sequences behind 16000, 64 / 8 heads, 8 bits: 38 with 15, 30 with 8)
    if (form == PLAN_FRONT) {
        const int64_t base = p.rows ? 16 : 8, tile = 16 * p.nt, fill = (rows + tile - 1) / tile * seqs * s->n_kv_heads * chunks / units();
        p.min_run = (int32_t)(fill >= base ? base : fill > 4 ? fill : 4);
    }
    // An item that is a wave's: about eight to a compute unit, two chunks each if they are short (the sixteen samples' own 512 tokens and less: 35 us with 16 chunks, 26 with 2)
    if (form == PLAN_WAVE) { p.min_run = 2; p.target = 8 * units(); }
    const int64_t full = (int64_t)b->n_rows * group / (16 * p.nt) * s->n_kv_heads;
    const int64_t most = (chunks + p.min_run / 2) / p.min_run;      // runs of the longest sequence
    p.join = most > 1 && !(p.rows && (full >= p.target || (whole >= p.target && chunks < 128)));
    // kv_many_rows' tiles are few and long beside the two that a compute unit works on at a time.  Those that fill whole rounds stay whole; the rest are cut so that they fill
    // one more (512 rows behind 8195 tokens and 260 behind 2665, 64 / 8 heads, 8 bits, window 2048, 392 tiles: 110 us with all tiles cut, 92 so; 24 questions behind system
    // prompts of 4000, 2756 and 2976 tokens, 2.2 rounds: 307 us with none cut, 272 so).
    if (p.rows && ((form == PLAN_EVEN && chunks < 128) || ((form == PLAN_EVEN || form == PLAN_BOTH) && !p.join))) {
        p.target = 2 * units();
        p.tail = (int32_t)(chunks / 8 < 1 ? 1 : chunks / 8 < p.target ? chunks / 8 : p.target);
        p.join = p.tail > 1;
        p.grid = whole + (p.join ? p.target : 0);
        p.join_blocks = (whole < p.target / 2 ? whole : p.target / 2) * p.nt;
        if (p.join) {
            p.o_bytes = ((size_t)p.target * 16 * p.nt * s->head_dim * 4 + 255) / 256 * 256;
            p.bytes = p.o_bytes + (size_t)p.target * 16 * p.nt * 8;
        }
        return p;
    }
    p.grid = p.join ? whole + p.target : whole;
    p.join_blocks = tiles(1) * s->n_kv_heads;
    if (p.join && whole * most < p.grid) p.grid = whole * most;
    if (p.join) {
        p.o_bytes = ((size_t)p.grid * 16 * p.nt * s->head_dim * 4 + 255) / 256 * 256;
        p.bytes = p.o_bytes + (size_t)p.grid * 16 * p.nt * 8;
    }
    return p;
}

// causal attention: all that a sequence can have
auto whole_lengths(const asd_kv_shape* s, const asd_kv_batch* b) {
    const int64_t chunks = (kv_args(s, b).cap + 63) / 64;
    return [=](int) { return chunks; };
}

}  // namespace
