// Operators over a paged cache of several sequences: new rows prepared and written into the pages (asd_kv_append), causal
// attention of the new rows over them (asd_kv_attend), rows read back (asd_kv_read), rotary tables (asd_rope_table).
//
// A page holds, per KV head, page_tokens / 64 chunks of 64 tokens: the chunk's K fragments, then its V^T fragments, in the
// layout of the engine's own cache (asd_common.h), so that for fp32 and bf16 a layer of an engine is such a set of pages.
// The 8-bit cache keeps e4m3 codes in the same scheme with 16 codes to a 16-byte piece, and behind the fragments one byte
// per token for K and one for V: 127 + the exponent of that token's scale.  Scales are powers of two: scaling a value
// before its one rounding is exact, and a code times its scale is exactly a bf16 number, so that what the attention
// multiplies is the stored value itself; a floating-point code loses nothing to a scale that is up to 2x too large.
#pragma once
#include "asd_common.h"
#include <type_traits>

// e4m3 codes (cache only); 16 to a lane's piece
struct FP8 {
    using elem = uint8_t;
    static constexpr int KE = 16;
};
// keys of a score tile as for the other types: the four tiles' registers of lane group g are keys 16g .. 16g + 15
template <> __device__ __forceinline__ int score_key<FP8>(int kt, int r) { return 16 * (r >> 2) + 4 * kt + (r & 3); }
template <> __host__ __device__ __forceinline__ void score_tile_of<FP8>(int key, int* kt, int* r) { *kt = (key >> 2) & 3; *r = 4 * (key >> 4) + (key & 3); }

// Layout of a chunk of cache type C at head dim H
template <class C, int H> struct KvLayout {
    using E = typename C::elem;
    static constexpr bool Q8 = sizeof(E) == 1;
    static constexpr int KV = C::KE;                                     // keys of a V^T piece (16 bytes)
    static constexpr int KK = C::KE < H / 4 ? C::KE : H / 4;             // dims of a K piece (8 bytes for codes at H = 32, else 16)
    static constexpr int HP = H / (4 * KK), HT = H / 16, KST = 64 / (4 * KV);
    static constexpr int K_BYTES = 64 * H * (int)sizeof(E);
    static constexpr int CHUNK = 2 * K_BYTES + (Q8 ? 128 : 0);
    static __device__ __forceinline__ int k_off(int key, int dim) {      // byte offsets of one element (key of the chunk)
        int kt, r;
        score_tile_of<C>(key, &kt, &r);
        return (((kt * HP + dim / (4 * KK)) * 64 + ((dim / KK) & 3) * 16 + r) * KK + dim % KK) * (int)sizeof(E);
    }
    static __device__ __forceinline__ int v_off(int key, int dim) {
        return K_BYTES + (((dim / 16 * KST + key / (4 * KV)) * 64 + ((key / KV) & 3) * 16 + dim % 16) * KV + key % KV) * (int)sizeof(E);
    }
};

struct KvArgs {
    char* pages;
    const int32_t *table, *row_start, *kv_len;
    int32_t* status;
    int32_t n_pages, table_stride, n_seqs, n_rows, max_new, cap;        // cap: most tokens a sequence can have (max_len, the table's reach)
    int32_t n_h, n_kv, group, page_tokens;
};

// One sequence's rows (n of them from row r0 on) and the position behind the last (len; rows in front of position 0 are possible), held inside the
// buffers whatever the arrays say
struct KvSeq { int r0, n, len, low = 0, lead = 0; };      // low: first key of its own, behind those that it shares with sequence `lead`
__device__ __forceinline__ KvSeq kv_seq(const KvArgs& a, int s, bool* bad = nullptr) {
    const int f0 = a.row_start[s], f1 = a.row_start[s + 1], fl = a.kv_len[s];
    KvSeq v;
    v.r0 = min(max(f0, 0), a.n_rows);
    v.n = min(min(max(f1, v.r0), a.n_rows) - v.r0, a.max_new);
    v.len = min(max(fl, 0), a.cap);
    if (bad) *bad = v.r0 != f0 || v.r0 + v.n != f1 || v.len != fl || v.n > v.len;
    return v;
}
__device__ __forceinline__ void kv_flag(const KvArgs& a, int bit) { if (a.status) atomicOr(a.status, bit); }
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int from_lane(int x, int lane) { return __builtin_amdgcn_readlane(x, lane); }      // (the same lane for all)
// Sums and maxima over a wave's lanes in front of a lane and itself, in the vector unit: within rows of 16, then from row to row.  Exchanges through LDS take
// several times as long, and every workgroup waits for a few of these before its first request.
template <int STEP, int ROWS> __device__ __forceinline__ int wave_step(int x) { return __builtin_amdgcn_update_dpp(0, x, STEP, ROWS, 0xf, false); }
template <class F> __device__ __forceinline__ int wave_upto(int x, F join) {      // join(x, 0) is x
    x = join(x, wave_step<0x111, 0xf>(x));
    x = join(x, wave_step<0x112, 0xf>(x));
    x = join(x, wave_step<0x114, 0xf>(x));
    x = join(x, wave_step<0x118, 0xf>(x));
    x = join(x, wave_step<0x142, 0xa>(x));
    return join(x, wave_step<0x143, 0xc>(x));
}
__device__ __forceinline__ int wave_sum_upto(int c) { return wave_upto(c, [](int a, int b) { return a + b; }); }
__device__ __forceinline__ int wave_max_upto(int c) { return wave_upto(c, [](int a, int b) { return max(a, b); }); }      // (of numbers >= 0)
__device__ __forceinline__ int64_t wave_sum(int64_t t) {                          // (0 <= t, all of it below 2^48)
    const int lo = from_lane(wave_sum_upto((int)(t & 0xffffff)), 63), hi = from_lane(wave_sum_upto((int)(t >> 24)), 63);
    return ((int64_t)hi << 24) + lo;
}

// A wave's view of the batch, 64 sequences at a time, in order: the first 64 stay in registers.  check: the wave reports arrays out of range.
// From the first bad sequence on: rows keep the positions that the arrays give them, whatever is cut, and those past cap are left out.  Launches and
// workspaces have room for tiles of n_rows rows, so no row may belong to two sequences: one that begins in front of the end (top) of an earlier one has none.
struct KvLanes {
    KvSeq v;
    int top = -1;                                       // (nothing was bad so far)
    static __device__ __forceinline__ int entries(const KvArgs& a) { return a.n_seqs; }
    __device__ __forceinline__ void load(const KvArgs& a, int s0, int lane, bool check) {
        v = KvSeq{0, 0, 0};
        bool bad = false;
        if (s0 + lane < a.n_seqs) v = kv_seq(a, s0 + lane, &bad);
        if (__any(bad) || top >= 0) mend(a, s0, lane, bad, check);
    }
    __device__ __forceinline__ void mend(const KvArgs& a, int s0, int lane, bool bad, bool check) {
        int end = 0;
        if (s0 + lane < a.n_seqs) {
            const int f1 = a.row_start[s0 + lane + 1];
            end = min(max(f1, v.r0), a.n_rows);
            if (bad) {
                if (check) kv_flag(a, ASD_KV_BAD_ROWS);
                const int64_t first = (int64_t)a.kv_len[s0 + lane] - f1 + v.r0;      // position of row r0
                v.n = (int)max(min((int64_t)v.n, a.cap - first), (int64_t)0);
                v.len = (int)min(max(first + v.n, (int64_t)0), (int64_t)a.cap);
            }
        }
        if (top < 0) top = min(max(a.row_start[s0], 0), a.n_rows);      // (the sequences in front of s0 lie one behind the other)
        end = wave_max_upto(end);
        const int before = __shfl_up(end, 1);
        if (v.r0 < max(top, lane ? before : 0)) v.n = 0;
        top = max(top, from_lane(end, 63));
    }
};
// Work items of all sequences one behind the other: count(sequence) items each.  Finds the sequence of `item`, its
// number within it and the first item of the sequence; each wave counts for itself, so no list has to be built in a launch of its own.
template <class Lanes, class F>
__device__ __forceinline__ bool kv_find(const KvArgs& a, Lanes x, int64_t item, int lane, bool check, F count, int* seq, int* local, int64_t* first, KvSeq* view) {
    const int n = x.entries(a);
    int64_t base = 0;
    for (int s0 = 0;;) {
        const int c = count(x.v);
        if (n == 1) {                                   // (nothing to add up)
            *seq = 0; *first = 0; *local = (int)item;
            *view = KvSeq{uniform(x.v.r0), uniform(x.v.n), uniform(x.v.len), uniform(x.v.low), uniform(x.v.lead)};
            return item < uniform(c);
        }
        const int incl = wave_sum_upto(c), total = from_lane(incl, 63);
        if (item < base + total) {
            const int l = uniform(__ffsll((unsigned long long)__ballot(base + incl > item)) - 1);
            *seq = uniform(s0 + l);
            *first = base + from_lane(incl - c, l);
            *local = uniform((int)(item - *first));
            *view = KvSeq{from_lane(x.v.r0, l), from_lane(x.v.n, l), from_lane(x.v.len, l), from_lane(x.v.low, l), from_lane(x.v.lead, l)};
            if (check) for (s0 += 64; s0 < n; s0 += 64) x.load(a, s0, lane, true);
            return true;
        }
        base += total;
        s0 += 64;
        if (s0 >= n) return false;
        x.load(a, s0, lane, check);
    }
}
// Chunk c of a sequence for one KV head; null where the page table holds no page of the pool
template <class C, int H>
__device__ __forceinline__ const char* kv_chunk(const KvArgs& a, int seq, int c, int kvh) {
    const int per = a.page_tokens / 64, page = a.table[(size_t)seq * a.table_stride + c / per];
    if ((unsigned)page >= (unsigned)a.n_pages) return nullptr;
    return a.pages + (((size_t)page * a.n_kv + kvh) * per + c % per) * KvLayout<C, H>::CHUNK;
}

// ---- 8-bit values
// exponent of the scale: the least e with top * 2^-e <= 448 = 1.75 * 2^8 (0 for top = 0), held in a range whose powers are normal numbers
__device__ __forceinline__ int q8_exponent(float top) {
    const uint32_t u = __float_as_uint(top);
    const int e = (int)(u >> 23) - 127 - ((u & 0x7fffffu) <= 0x600000u ? 8 : 7);
    return top == 0.f ? 0 : min(max(e, -100), 120);
}
__device__ __forceinline__ float q8_scale(uint32_t byte) { return __uint_as_float(byte << 23); }
__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u; }
// four values as codes (the format has no infinity: the caller has made NaN of what is not finite)
__device__ __forceinline__ uint32_t q8_pack(float a, float b, float c, float d) {
    const int p = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, p, true);
}
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;
// two values as a word of bf16
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2));
}

// maximum and sum over the four lane groups (every lane gets them): exchanges of rows and halves in the vector unit, no LDS round trip
__device__ __forceinline__ float groups_max(float x) {
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float groups_sum(float x) {
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// A matrix-core operand register of activation type A out of step u of a piece of cache type C (codes: times `scale`)
template <class A, class C> __device__ __forceinline__ u32x4 kv_operand(const u32x4& piece, int u, float scale) {
    if constexpr (sizeof(typename C::elem) > 1) {
        return piece;
    } else if constexpr (A::KE == 8) {
        u32x4 r;
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            r[2 * w] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(piece[2 * u + w], scale, false));
            r[2 * w + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(piece[2 * u + w], scale, true));
        }
        return r;
    } else {
        const f32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(piece[u], scale, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(piece[u], scale, true);
        return u32x4{__float_as_uint(lo[0]), __float_as_uint(lo[1]), __float_as_uint(hi[0]), __float_as_uint(hi[1])};
    }
}
// four consecutive elements of a row
template <class T> __device__ __forceinline__ void store4(typename T::elem* p, const float (&v)[4]) {
    if constexpr (sizeof(typename T::elem) == 4) *(float4*)p = float4{v[0], v[1], v[2], v[3]};
    else *(uint2*)p = uint2{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
}

// ---------------------------------------------------------------- new rows into the cache
// (token, head) pairs that a workgroup of kv_append_kernel holds: four heads of a tile, but no more than 36 KiB
__host__ __device__ constexpr int APPEND_SLOTS(int tok, int row_bytes) { return 4 * tok * row_bytes <= 32768 ? 4 * tok : 32768 / row_bytes > tok ? 32768 / row_bytes : tok; }
struct KvAppendArgs {
    KvArgs kv;
    const void *q, *k, *v;
    void* q_out;
    int64_t q_stride, k_stride, v_stride, out_stride;
    const float *q_gain, *k_gain, *rope;
    float eps;
    int32_t rope_positions, rot;
    int32_t kv_heads_per, q_heads_per, kv_blocks, blocks;      // heads of a workgroup; of a tile's `blocks` workgroups kv_blocks take K, as many V, the others q
};

// A head's vector lies in H / 2DU lanes, two units of 16 bytes (DU dims) each, chosen so that both partners of every rotated pair
// are in one lane: neighbours (interleaved), or dims p * DU .. and those rot/2 further on (half layout), the dims behind the
// rotated part after them.  The norm's sum of squares runs over the lanes by shuffles.
template <class T, int H, bool INTER> struct HeadVec {
    static constexpr int DU = 16 / (int)sizeof(typename T::elem), LPV = H / (2 * DU);
    float x[2][DU];
    // first dims of lane p's units
    static __device__ __forceinline__ void place(int p, int rot, int (&d)[2]) {
        const bool pair = !INTER && 2 * DU * p < rot;
        d[0] = pair ? DU * p : 2 * DU * p;
        d[1] = pair ? rot / 2 + DU * p : 2 * DU * p + DU;
    }
    __device__ __forceinline__ void load(const typename T::elem* row, const int (&d)[2]) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const u32x4 r = *(const u32x4*)(row + d[i]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (DU == 4) x[i][j] = __uint_as_float(r[j]);
                else { x[i][2 * j] = __uint_as_float(r[j] << 16); x[i][2 * j + 1] = __uint_as_float(r[j] & 0xffff0000u); }
            }
        }
    }
    static __device__ __forceinline__ u32x4 pack(const float (&v)[DU]) {
        u32x4 r;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (DU == 4) r[j] = __float_as_uint(v[j]);
            else r[j] = bf16_pair(v[2 * j], v[2 * j + 1]);
        }
        return r;
    }
    __device__ __forceinline__ void normalise(const float* gain, float eps, const int (&d)[2]) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < DU; ++j) s += x[i][j] * x[i][j];
#pragma unroll
        for (int o = 1; o < LPV; o <<= 1) s += __shfl_xor(s, o);
        const float r = 1.f / sqrtf(s * (1.f / H) + eps);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < DU; j += 4) {
                const float4 g = *(const float4*)(gain + d[i] + j);
                x[i][j] *= r * g.x; x[i][j + 1] *= r * g.y; x[i][j + 2] *= r * g.z; x[i][j + 3] *= r * g.w;
            }
    }
    // cs: (cos, sin) of the angles of the lane's DU pairs
    __device__ __forceinline__ void rotate(const float4 (&cs)[DU / 2]) {
        auto turn = [&](float& a, float& b, int j) {
            const float c = j & 1 ? cs[j / 2].z : cs[j / 2].x, s = j & 1 ? cs[j / 2].w : cs[j / 2].y;
            const float a1 = a * c - b * s, b1 = b * c + a * s;
            a = a1; b = b1;
        };
#pragma unroll
        for (int j = 0; j < DU; ++j) {
            if constexpr (INTER) turn(x[2 * j / DU][2 * j % DU], x[2 * j / DU][2 * j % DU + 1], j);
            else turn(x[0][j], x[1][j], j);
        }
    }
};

// A workgroup takes up to TOK tokens of one sequence (a tile at positions TOK * t ..) and some heads.  Bound by memory: every row is read
// once, 16 bytes a lane, four heads of a token in flight (their angles are read once); what the vector unit does per value is kept short, and
// values that are not finite are looked for by one comparison of the largest magnitude.  The cache's elements go through LDS, K row by
// row and V to be transposed, so that they leave in the layout's own 16-byte pieces, whole lines for whole chunks.  A V^T piece some of whose
// keys are not new is written element by element, so that what the cache holds beside the new rows stays.  Prompts of 6901 tokens, 32 + 32 heads
// x 128, into 8-bit pages: 67 us, 283 MB, 4.2 TB/s; one token of 48 sequences, 64 + 8 heads: 7.0 us, a chain of look-ups (lengths, table, rows).
// (Neighbours turn in a kernel of their own: an array whose elements two branches pair differently stays in memory.)
template <class T, class C, int H, int TOK, bool INTER>
__global__ __launch_bounds__(256) void kv_append_kernel(const KvAppendArgs a) {
    using L = KvLayout<C, H>;
    using E = typename T::elem;
    using CE = typename C::elem;
    using V = HeadVec<T, H, INTER>;
    constexpr int DU = V::DU, LPV = V::LPV, VPP = 256 / LPV, U = 4;       // dims of a unit, lanes of a vector; vectors of a pass, heads in flight
    constexpr int RS = H + 16 / (int)sizeof(CE);                          // an LDS row, 16 bytes longer: its pieces fall on different banks
    constexpr int SLOTS = APPEND_SLOTS(TOK, H * sizeof(CE));              // (token, head) pairs of a workgroup
    __shared__ __align__(16) CE rows[SLOTS][RS];
    __shared__ uint8_t exps[SLOTS];
    const int tid = threadIdx.x, lane = tid & 63;
    int seq, tile;
    int64_t first;
    KvSeq s;
    auto tiles = [](const KvSeq& v) { return v.n > 0 && v.len > 0 ? (v.len + TOK - 1) / TOK - max(v.len - v.n, 0) / TOK : 0; };
    // a tile's workgroups side by side: those that run at a time read whole rows, not the same part of many
    const int item = blockIdx.x / a.blocks, block = blockIdx.x % a.blocks;
    const bool check = blockIdx.x == 0 && tid < 64;
    KvLanes all;
    all.load(a.kv, 0, lane, check);
    if (!kv_find(a.kv, all, item, lane, check, tiles, &seq, &tile, &first, &s)) return;
    const int base = s.len - s.n;                      // position of row 0 (negative: rows in front have no place)
    const int t0 = (max(base, 0) / TOK + tile) * TOK;
    const int lo = max(max(base, 0), t0), nt = min(s.len, t0 + TOK) - lo;
    const int vec = tid / LPV, p = tid % LPV;
    int d[2];
    V::place(p, a.rot, d);
    // heads h0 .. h0 + nh - 1 of the tile's rows of x, prepared, into sink(vector, token of the tile, head of the workgroup)
    auto each = [&](const void* x, int64_t stride, int h0, int nh, bool turn, const float* gain, auto sink) {
        const int uh = nt * nh > VPP ? U : 1, groups = (nh + uh - 1) / uh;      // heads of a lane's turn: one where they would leave lanes idle
        for (int i = vec; i < nt * groups; i += VPP) {                           // (the lanes of a vector take the same turns)
            const int token = groups == 1 ? i : i / groups, g0 = groups == 1 ? 0 : i % groups * uh, left = min(nh - g0, uh), pos = lo + token;
            const E* row = (const E*)x + (s.r0 + (int64_t)(pos - base)) * stride + (h0 + g0) * H;
            V v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) v[u].load(row + min(u, left - 1) * H, d);
            float4 cs[DU / 2];
            turn = turn && 2 * DU * p < a.rot;
            if (turn) {
                if (pos >= a.rope_positions) kv_flag(a.kv, ASD_KV_BAD_POS);
                const float4* at = (const float4*)(a.rope + ((size_t)min(pos, a.rope_positions - 1) * (a.rot / 2) + DU * p) * 2);
#pragma unroll
                for (int j = 0; j < DU / 2; ++j) cs[j] = at[j];
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (gain) v[u].normalise(gain, a.eps, d);
                if (turn) v[u].rotate(cs);
                if (u < left) sink(v[u], token, g0 + u);
            }
        }
    };
    if (block >= 2 * a.kv_blocks) {                    // queries
        const int h0 = (block - 2 * a.kv_blocks) * a.q_heads_per;
        each(a.q, a.q_stride, h0, min(a.q_heads_per, a.kv.n_h - h0), true, a.q_gain, [&](const V& v, int token, int head) {
            E* out = (E*)a.q_out + (s.r0 + (int64_t)(lo + token - base)) * a.out_stride + (h0 + head) * H;
            *(u32x4*)(out + d[0]) = V::pack(v.x[0]);
            *(u32x4*)(out + d[1]) = V::pack(v.x[1]);
        });
        return;
    }
    const bool isv = block >= a.kv_blocks;
    const int h0 = (isv ? block - a.kv_blocks : block) * a.kv_heads_per, nh = min(a.kv_heads_per, a.kv.n_kv - h0);
    const int k0 = lo & 63, k1 = k0 + nt;              // the chunk's new keys; a pair's slot: (key - k0) * nh + head
    auto keep = [&](const V& v, int token, int head) {
        const int slot = token * nh + head;
        CE* row = rows[slot];
        if constexpr (L::Q8) {
            uint32_t top = 0;                          // largest magnitude, as its bits
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < DU; ++j) top = max(top, __float_as_uint(v.x[i][j]) & 0x7fffffffu);
#pragma unroll
            for (int o = 1; o < LPV; o <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
            float y[2][DU];
            // Something is not finite: it becomes NaN, and the scale comes from the rest.  Or a magnitude of 248 * 2^120 and more, whose code would be
            // 256, beyond fp32 with that scale, the largest: 240 (off by 2^-4 of it at most, as a rounding may be)
            constexpr uint32_t MOST = 0x7f780000u;
            const bool odd = top >= MOST;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < DU; ++j) y[i][j] = v.x[i][j];
            if (odd) {
                top = 0;
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < DU; ++j) {
                        const uint32_t u = __float_as_uint(y[i][j]), m = u & 0x7fffffffu;
                        if (m < 0x7f800000u) {
                            top = max(top, m);
                            if (m >= MOST) y[i][j] = __uint_as_float((u & 0x80000000u) | 0x7f700000u);
                        } else {
                            y[i][j] = __uint_as_float(0x7fc00000u);
                        }
                    }
#pragma unroll
                for (int o = 1; o < LPV; o <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
            }
            const int e = q8_exponent(__uint_as_float(top));
            const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < DU; j += 4) *(uint32_t*)(row + d[i] + j) = q8_pack(y[i][j] * inv, y[i][j + 1] * inv, y[i][j + 2] * inv, y[i][j + 3] * inv);
            if (p == 0) exps[slot] = (uint8_t)(e + 127);
        } else {
            *(u32x4*)(row + d[0]) = V::pack(v.x[0]);
            *(u32x4*)(row + d[1]) = V::pack(v.x[1]);
        }
    };
    if (isv) each(a.v, a.v_stride, h0, nh, false, nullptr, keep);
    else each(a.k, a.k_stride, h0, nh, true, a.k_gain, keep);
    char* chunk0 = (char*)kv_chunk<C, H>(a.kv, seq, t0 / 64, h0);
    if (!chunk0) { if (tid == 0) kv_flag(a.kv, ASD_KV_BAD_PAGE); return; }
    const size_t head_bytes = (size_t)(a.kv.page_tokens / 64) * L::CHUNK;
    __syncthreads();
    if constexpr (L::Q8)
        for (int i = tid; i < nh * nt; i += 256) *(uint8_t*)(chunk0 + i % nh * head_bytes + 2 * L::K_BYTES + 64 * isv + k0 + i / nh) = exps[i];
    constexpr int KP = 4 * L::HP * 64, VP = L::HT * L::KST * 64, KV = L::KV;      // pieces of a chunk, in the order in which they lie
    if (TOK == 16 && !isv) {                           // few keys: by rows
        constexpr int PR = H / L::KK;                  // pieces of a row
        for (int i = tid; i < nh * nt * PR; i += 256) {
            const int slot = i / PR, dim = i % PR * L::KK, key = k0 + slot / nh;
            CE* dst = (CE*)(chunk0 + slot % nh * head_bytes + L::k_off(key, dim));
            if constexpr (L::KK * sizeof(CE) == 16) *(u32x4*)dst = *(const u32x4*)&rows[slot][dim];
            else *(uint2*)dst = *(const uint2*)&rows[slot][dim];
        }
        return;
    }
    if (TOK == 16 && nt < KV) {                        // ... and elements
        for (int i = tid; i < nh * nt * H; i += 256) {
            const int slot = i / H, dim = i % H, key = k0 + slot / nh;
            *(CE*)(chunk0 + slot % nh * head_bytes + L::v_off(key, dim)) = rows[slot][dim];
        }
        return;
    }
    for (int hd = 0; hd < nh && !isv; ++hd)
        for (int q = tid; q < KP; q += 256) {
            const int l = q & 63, key = score_key<C>(q / 64 / L::HP, l & 15);
            if (key < k0 || key >= k1) continue;
            const CE* src = &rows[(key - k0) * nh + hd][q / 64 % L::HP * 4 * L::KK + (l >> 4) * L::KK];
            CE* dst = (CE*)(chunk0 + hd * head_bytes) + (size_t)q * L::KK;
            if constexpr (L::KK * sizeof(CE) == 16) *(u32x4*)dst = *(const u32x4*)src;
            else *(uint2*)dst = *(const uint2*)src;
        }
    for (int hd = 0; hd < nh && isv; ++hd)
        for (int q = tid; q < VP; q += 256) {
            const int l = q & 63, dim = q / 64 / L::KST * 16 + (l & 15), first_key = q / 64 % L::KST * 4 * KV + (l >> 4) * KV;
            const int b = max(k0, first_key), e = min(k1, first_key + KV);
            if (b >= e) continue;
            CE* dst = (CE*)(chunk0 + hd * head_bytes + L::K_BYTES) + (size_t)q * KV;
            if (e - b == KV) {
                u32x4 r;
                CE* t = (CE*)&r;
#pragma unroll
                for (int j = 0; j < KV; ++j) t[j] = rows[(first_key + j - k0) * nh + hd][dim];
                *(u32x4*)dst = r;
            } else {
                for (int j = b; j < e; ++j) dst[j - first_key] = rows[(j - k0) * nh + hd][dim];
            }
        }
}

// ---------------------------------------------------------------- rows out of the cache
struct KvReadArgs {
    KvArgs kv;
    void *k_out, *v_out;
    int64_t k_stride, v_stride;
};
// A workgroup takes one chunk of one sequence and KV head, its K or its V: the pieces that hold wanted rows come in as they
// lie, go through LDS as rows, and leave as rows.  Bound by memory: 16 sequences of up to 4096 tokens, 8 heads x 128 in 8 bits, 254 MB,
// 58 us (4.4 TB/s; a large copy reaches 5.0); a few tokens 4.1 us, a chain of look-ups.
template <class T, class C, int H>
__global__ __launch_bounds__(256) void kv_read_kernel(const KvReadArgs a) {
    using L = KvLayout<C, H>;
    using E = typename T::elem;
    using CE = typename C::elem;
    constexpr int PAD = 16 / (int)sizeof(E);
    __shared__ __align__(16) E rows[64][H + PAD];
    const int tid = threadIdx.x, lane = tid & 63, kvh = blockIdx.y;
    const bool isv = blockIdx.z != 0;
    E* out = (E*)(isv ? a.v_out : a.k_out);
    if (!out) return;
    int seq, local;
    int64_t first;
    KvSeq s;
    auto chunks = [](const KvSeq& v) { return v.n > 0 && v.len > 0 ? (v.len + 63) / 64 - max(v.len - v.n, 0) / 64 : 0; };
    const bool check = blockIdx.x == 0 && blockIdx.y == 0 && tid < 64;
    KvLanes all;
    all.load(a.kv, 0, lane, check);
    if (!kv_find(a.kv, all, blockIdx.x, lane, check, chunks, &seq, &local, &first, &s)) return;
    const int base = s.len - s.n, c = max(base, 0) / 64 + local;
    const int lo = max(max(base, 0) - 64 * c, 0), hi = min(s.len - 64 * c, 64);      // keys of the chunk that are wanted
    const char* chunk = kv_chunk<C, H>(a.kv, seq, c, kvh);
    if (!chunk) { if (tid == 0) kv_flag(a.kv, ASD_KV_BAD_PAGE); return; }
    const uint8_t* exps = (const uint8_t*)chunk + 2 * L::K_BYTES + (isv ? 64 : 0);
    auto value = [&](CE code, float scale) -> E {
        if constexpr (!L::Q8) return code;
        else return T::from_f32(__builtin_amdgcn_cvt_f32_fp8(code, 0) * scale);
    };
    auto element = [&](const u32x4& piece, int j) -> CE {                // element j of a piece (j known at compile time)
        if constexpr (sizeof(CE) == 4) return __uint_as_float(piece[j]);
        else return (CE)(piece[j * sizeof(CE) / 4] >> (8 * (j * sizeof(CE) % 4)));
    };
    if (!isv) {
        constexpr int KK = L::KK;
        for (int i = tid; i < 64 * H / KK; i += 256) {
            const int l = i & 63, hp = i / 64 % L::HP, kt = i / (64 * L::HP), key = score_key<C>(kt, l & 15);
            if (key < lo || key >= hi) continue;
            u32x4 piece;
            if constexpr (KK * sizeof(CE) == 16) piece = *(const u32x4*)(chunk + (size_t)i * 16);
            else { const uint2 x = *(const uint2*)(chunk + (size_t)i * 8); piece = u32x4{x.x, x.y, 0u, 0u}; }
            float scale = 1.f;
            if constexpr (L::Q8) scale = q8_scale(exps[key]);
            E* dst = &rows[key][hp * 4 * KK + (l >> 4) * KK];
            if constexpr (sizeof(CE) == 4) { *(u32x4*)dst = piece; }
            else {
#pragma unroll
                for (int j = 0; j < KK; ++j) dst[j] = value(element(piece, j), scale);
            }
        }
    } else {
        constexpr int KV = L::KV;
        for (int i = tid; i < 64 * H / KV; i += 256) {
            const int l = i & 63, ks = i / 64 % L::KST, ht = i / (64 * L::KST), key = ks * 4 * KV + (l >> 4) * KV, dim = ht * 16 + (l & 15);
            if (key + KV <= lo || key >= hi) continue;
            const u32x4 piece = *(const u32x4*)(chunk + L::K_BYTES + (size_t)i * 16);
            u32x4 ex{};
            if constexpr (L::Q8) ex = *(const u32x4*)(exps + key);
#pragma unroll
            for (int j = 0; j < KV; ++j) {
                float scale = 1.f;
                if constexpr (L::Q8) scale = q8_scale((ex[j / 4] >> (8 * (j % 4))) & 255u);
                rows[key + j][dim] = value(element(piece, j), scale);
            }
        }
    }
    __syncthreads();
    const int64_t stride = isv ? a.v_stride : a.k_stride;
    constexpr int PPR = H * (int)sizeof(E) / 16;       // 16-byte pieces of a row
    for (int i = tid; i < (hi - lo) * PPR; i += 256) {
        const int key = lo + i / PPR, pc = i % PPR;
        *(u32x4*)(out + (s.r0 + (int64_t)64 * c + key - base) * stride + kvh * H + pc * PAD) = *(const u32x4*)&rows[key][pc * PAD];
    }
}
