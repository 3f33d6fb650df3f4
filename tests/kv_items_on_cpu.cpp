// The kernels of the attention with a window and of shared beginnings on the CPU, with everything but the work on a tile: the lanes of a wave take turns, each running until the next
// exchange between lanes, so that a launch is carried out as it is written, workgroup by workgroup.  What a work item would do, and where it would leave its sums, is noted and checked;
// so is what the join reads.  Built for the host alone by test_kv_items.py, which puts the host side's text (SPANS: launches turned into calls of on_cpu) beside it.
#include <hip/hip_runtime.h>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <string>
#include <type_traits>
#include <unordered_map>
#include <vector>

// ---------------------------------------------------------------- 64 lanes, a stack each
extern "C" void wave_switch(void** from, void* to);
asm(R"(
.text
.type wave_switch, @function
wave_switch:
    pushq %rbp
    pushq %rbx
    pushq %r12
    pushq %r13
    pushq %r14
    pushq %r15
    movq %rsp, (%rdi)
    movq %rsi, %rsp
    popq %r15
    popq %r14
    popq %r13
    popq %r12
    popq %rbx
    popq %rbp
    ret
)");
namespace wave {
constexpr size_t STACK = 256 << 10;
char* stacks;
void *at[64], *home;
int lane, wave_of_group;
unsigned group;
int slot[2][64], turns[64];                             // exchanges that a lane has taken part in
int64_t all_turns, most_turns;                          // of all waves, of the longest
void (*body)(void*);
void* body_of;
std::string fault;
void failed(const char* fmt, ...) {
    if (!fault.empty()) return;
    char buf[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    fault = buf;
}
void to_lane(int to) { const int me = lane; lane = to; wave_switch(&at[me], at[to]); }
void lane_main() {
    body(body_of);
    if (turns[lane] != turns[0]) failed("lane %d takes part in %d exchanges, lane 0 in %d", lane, turns[lane], turns[0]);
    void* gone;
    if (lane == 63) wave_switch(&gone, home);
    ++lane;
    wave_switch(&gone, at[lane]);
}
int* exchange(int x) {                                  // what all lanes have put in
    const int turn = turns[lane]++ & 1;
    slot[turn][lane] = x;
    to_lane((lane + 1) & 63);
    return slot[turn];
}
void run(void (*f)(void*), void* of) {
    if (!stacks) stacks = (char*)aligned_alloc(4096, 64 * STACK);
    body = f; body_of = of;
    for (int i = 0; i < 64; ++i) {
        void** top = (void**)(stacks + (i + 1) * STACK) - 8;
        memset(top, 0, 64);
        top[6] = (void*)lane_main;
        at[i] = top; turns[i] = 0;
    }
    lane = 0;
    wave_switch(&home, at[0]);
    all_turns += turns[0];
    if (turns[0] > most_turns) most_turns = turns[0];
}
int from(int x, int l) { return exchange(x)[l & 63]; }
unsigned long long ballot(bool x) {
    const int* y = exchange(x);
    unsigned long long r = 0;
    for (int i = 0; i < 64; ++i) r |= (unsigned long long)(y[i] != 0) << i;
    return r;
}
int dpp(int old, int x, int ctrl, int rows) {           // row_shr:n, row_bcast:15, row_bcast:31
    const int row = lane / 16, me = lane, src = ctrl < 0x120 ? (lane % 16 >= (ctrl & 15) ? lane - (ctrl & 15) : -1) : ctrl == 0x142 ? row * 16 - 1 : row >= 2 ? 31 : -1;
    const int y = from(x, src < 0 ? me : src);
    return src >= 0 && (rows >> row & 1) ? y : old;
}
struct Place { unsigned x, y, z; };
Place thread() { return Place{(unsigned)(wave_of_group * 64 + lane), 0, 0}; }
}  // namespace wave

#undef __device__
#define __device__
#undef __host__
#define __host__
#undef __global__
#define __global__
#undef __shared__
#define __shared__
#undef __launch_bounds__
#define __launch_bounds__(...)
#undef __forceinline__
#define __forceinline__ inline
#define __syncthreads() ((void)0)
#define threadIdx wave::thread()
#define blockIdx (wave::Place{wave::group, 0, 0})
#define __builtin_amdgcn_readlane(x, l) wave::from(x, l)
#define __builtin_amdgcn_readfirstlane(x) wave::from(x, 0)
#define __builtin_amdgcn_update_dpp(o, x, ctrl, rows, banks, bound) wave::dpp(o, x, ctrl, rows)
#define __builtin_amdgcn_raw_ptr_buffer_load_lds(...) ((void)0)
#define __shfl(x, l) wave::from(x, l)
#define __shfl_up(x, n) wave::from(x, wave::lane >= (n) ? wave::lane - (n) : wave::lane)
#define __shfl_xor(x, n) wave::from(x, wave::lane ^ (n))
#define __ballot(x) wave::ballot(x)
#define __any(x) (wave::ballot(x) != 0)
#define __ffsll(x) __builtin_ffsll((long long)(x))
#define __uint_as_float(x) __builtin_bit_cast(float, (uint32_t)(x))
#define __float_as_uint(x) __builtin_bit_cast(uint32_t, (float)(x))
#define atomicOr(p, b) (*(p) |= (b))
#define hipGetDevice(x) hipErrorNoDevice
#define hipGetLastError() hipSuccess
// (of the wider type, as on the device)
template <class A, class B> inline std::common_type_t<A, B> least(A a, B b) { return b < a ? b : a; }
template <class A, class B> inline std::common_type_t<A, B> greatest(A a, B b) { return a < b ? b : a; }

#include "../include/asd.h"
#define min least
#define max greatest
#include "../paper_2410_01028_amd/csrc/asd_kv_attend.h"
#undef min
#undef max

// ---------------------------------------------------------------- what items do, and what is joined
namespace notebook {
struct Item { int sees, rows, block, wave; KvItem it; int steps; };      // steps: chunks that its tile walks
std::vector<Item> items;
struct Owner { int item, row; };
std::unordered_map<int64_t, Owner> owners;              // partial sums of a row, by their place in the workspace
std::vector<uint8_t> answered;                          // [row][head]
char* ws;
size_t ws_bytes;
int n_rows, n_heads, heads_of_kv, joined;

void answer(const char* who, int64_t global, int kvh) {      // row x head of the group, KV head
    const int64_t row = global / heads_of_kv, head = kvh * heads_of_kv + global % heads_of_kv;
    if (row < 0 || row >= n_rows) return wave::failed("%s: row %lld", who, (long long)row);
    if (answered[row * n_heads + head]++) wave::failed("%s: row %lld, head %lld twice", who, (long long)row, (long long)head);
}
bool same(const KvItem& a, const KvItem& b) {
    return a.seq == b.seq && a.s.r0 == b.s.r0 && a.s.n == b.s.n && a.s.len == b.s.len && a.s.low == b.s.low && a.kvh == b.kvh && a.tile == b.tile && a.split == b.split && a.per == b.per &&
           a.whole == b.whole && (a.whole || a.part == b.part);
}
template <int SEES, class Args> void tile(const Args& a, const KvItem& it, int R, int H, int waves) {
    const int block = (int)wave::group, w = waves == 1 ? wave::wave_of_group : 0;
    if (!items.empty() && items.back().block == block && items.back().wave == w && items.back().sees == SEES) {
        if (!same(items.back().it, it)) wave::failed("workgroup %d: lane %d of wave %d has another item than the first", block, wave::lane, wave::wave_of_group);
        return;
    }
    const int group = a.kv.group, rows = it.s.n * group, base = it.s.len - it.s.n, first = it.tile * R, last_row = std::min(first + R, rows) - 1;
    if (it.seq < 0 || it.seq >= a.kv.n_seqs || first >= rows || it.kvh < 0 || it.kvh >= a.kv.n_kv || it.split < 0 || it.per < 0 || it.s.len > a.kv.cap || it.s.len < 0)
        return wave::failed("workgroup %d: sequence %d, tile %d of %d rows, KV head %d, run %d", block, it.seq, it.tile, rows, it.kvh, it.split);
    const int from = SEES == KV_SHARED ? it.s.len - 1 : base + first / group, last = SEES == KV_SHARED ? it.s.len - 1 : base + last_row / group;
    int low = it.s.low;
    if constexpr (SEES == KV_WINDOW) low = from - a.window + 1;
    const KvSteps steps = kv_steps<SEES>(a, low, 64);
    items.push_back(Item{SEES, R, block, w, it, std::max(0, (last + 64) / 64 - steps.skip)});
    if (it.whole && (it.split || it.per < items.back().steps)) wave::failed("workgroup %d: whole, run %d of %d chunks, the tile has %d", block, it.split, it.per, items.back().steps);
    for (int row = first; row <= last_row; ++row) {
        if (it.whole) { answer("item", (int64_t)it.s.r0 * group + row, it.kvh); continue; }
        const int64_t at = it.part * R + row - first;
        const char *o = (const char*)(a.o_part + at * H), *ml = (const char*)(a.ml_part + at * 2);
        if (it.part < 0 || o < ws || o + H * 4 > (const char*)a.ml_part || ml < ws || ml + 8 > ws + ws_bytes) return wave::failed("workgroup %d: sums of place %lld leave the workspace", block, (long long)it.part);
        if (!owners.emplace(o - ws, Owner{(int)items.size() - 1, row}).second) return wave::failed("workgroup %d: place %lld is taken", block, (long long)it.part);
    }
}
template <class F> void join(const KvSeq& s, int kvh, int row0, int left, int n_runs, F place) {
    if (wave::wave_of_group || wave::lane) return;
    ++joined;
    for (int r = 0; r < left; ++r) {
        const int64_t global = (int64_t)s.r0 * heads_of_kv + row0 + r;
        answer("join", global, kvh);
        std::vector<int> seen[2];                       // runs: of the row's own tile, of the shared keys
        int per[2] = {0, 0}, steps[2] = {0, 0}, low = 0;
        for (int i = 0; i < n_runs; ++i) {
            const auto f = owners.find((const char*)place(i, r).o - ws);
            if (f == owners.end()) return wave::failed("join: sequence at row %d, row %d, run %d: nobody has left these sums", s.r0, row0 + r, i);
            const Item& x = items[f->second.item];
            const int k = x.sees == KV_SHARED;
            if (x.it.kvh != kvh || (int64_t)x.it.s.r0 * heads_of_kv + f->second.row != global) return wave::failed("join: sequence at row %d, row %d, run %d: another row's sums", s.r0, row0 + r, i);
            seen[k].push_back(x.it.split);
            per[k] = x.it.per; steps[k] = x.steps;
            if (!k) low = x.it.s.low * (x.sees == KV_OWN);
            if (k && x.it.s.len != low) return wave::failed("join: sequence at row %d: %d shared tokens, its own begin at %d", s.r0, x.it.s.len, low);
        }
        for (int k = 0; k < 2; ++k) {
            for (int i = 0; i < (int)seen[k].size(); ++i) if (seen[k][i] != i) return wave::failed("join: run %d in place of run %d", seen[k][i], i);
            if ((int64_t)seen[k].size() * per[k] < steps[k]) return wave::failed("join: %zu runs of %d chunks, the tile has %d", seen[k].size(), per[k], steps[k]);
        }
        if (seen[0].empty() || (low > 0) != !seen[1].empty()) return wave::failed("join: sequence at row %d: %zu and %zu runs, own keys from %d", s.r0, seen[0].size(), seen[1].size(), low);
    }
}
}  // namespace notebook
template <class A, class C, int H, int NT, int SEES, int W, class Args> void noted_few_rows(const Args& a, const KvItem& it, KvFewLds<H>&) { notebook::tile<SEES>(a, it, 16 * NT, H, W); }
template <class C, int H, int NT, int NW, int SEES, class Args> void noted_many_rows(const Args& a, const KvItem& it, u32x4 (&)[KV_RING<C, H>]) { notebook::tile<SEES>(a, it, 16 * NT * NW, H, NW); }
template <class A, int H, class F> void noted_join(const KvAttendArgs&, const KvSeq& s, int kvh, int row0, int left, int n_runs, F place) { notebook::join(s, kvh, row0, left, n_runs, place); }
int64_t launches, groups_of[2];                         // workgroups of a call's launches
bool some;                                              // the first two and every eighth part of a launch's workgroups are enough
template <class F> void on_cpu(F kernel, unsigned grid) {
    if (launches < 2) groups_of[launches] = grid;
    ++launches;
    for (wave::group = 0; wave::group < grid; ++wave::group) {
        if (some && wave::group > 1 && wave::group % std::max(grid / 8, 1u)) continue;
        for (wave::wave_of_group = 0; wave::wave_of_group < 4 && wave::fault.empty(); ++wave::wave_of_group)
            wave::run([](void* f) { (*(F*)f)(); }, &kernel);
    }
}
#define kv_few_rows noted_few_rows
#define kv_many_rows noted_many_rows
#define kv_join_rows noted_join
#include "../paper_2410_01028_amd/csrc/asd_kv_host.h"
#define min least
#define max greatest
#include SPANS
#undef min
#undef max
void asd_note_error(const char*) {}
extern "C" size_t asd_kv_page_bytes(const asd_kv_shape* s) {
    size_t n = 0;
    by_shape(s, [&](auto, auto c, auto h) { n = (size_t)KvLayout<decltype(c), h.value>::CHUNK * (s->page_tokens / 64) * s->n_kv_heads; });
    return n;
}

extern "C" {
void cpu_begin(void* ws, size_t bytes, int n_rows, int n_heads, int n_kv, int64_t some_groups) {
    some = some_groups != 0;
    notebook::items.clear(); notebook::owners.clear();
    notebook::answered.assign((size_t)n_rows * n_heads, 0);
    notebook::ws = (char*)ws; notebook::ws_bytes = bytes;
    notebook::n_rows = n_rows; notebook::n_heads = n_heads; notebook::heads_of_kv = n_heads / n_kv; notebook::joined = 0;
    wave::fault.clear();
    wave::all_turns = wave::most_turns = 0; launches = groups_of[0] = groups_of[1] = 0;
}
const char* cpu_fault() { return wave::fault.c_str(); }
const uint8_t* cpu_answered() { return notebook::answered.data(); }
// the first key of its own of every sequence that has items (-1: none)
const int32_t* cpu_lows(int n_seqs) {
    static std::vector<int32_t> low;
    low.assign(n_seqs, -1);
    for (const auto& i : notebook::items) if (i.sees != KV_SHARED) low[i.it.seq] = i.it.s.low;
    return low.data();
}
// items, cut ones, rows of the widest tile, joined blocks, exchanges of the longest wave and of all, workgroups of the two launches, items of shared keys
void cpu_counts(int64_t* x) {
    x[0] = (int64_t)notebook::items.size(); x[1] = x[2] = 0;
    for (const auto& i : notebook::items) { x[1] += i.it.per < i.steps; x[2] = std::max<int64_t>(x[2], i.rows); }
    x[8] = 0;
    for (const auto& i : notebook::items) x[8] += i.sees == KV_SHARED;
    x[3] = notebook::joined; x[4] = wave::most_turns; x[5] = wave::all_turns; x[6] = groups_of[0]; x[7] = groups_of[1];
}
}
