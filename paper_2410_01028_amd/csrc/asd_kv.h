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
struct KvSeq { int r0, n, len; };
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

// A wave's view of the batch, 64 sequences at a time, in order: the first 64 stay in registers.  check: the wave reports arrays out of range.
// From the first bad sequence on: rows keep the positions that the arrays give them, whatever is cut, and those past cap are left out.  Launches and
// workspaces have room for tiles of n_rows rows, so no row may belong to two sequences: one that begins in front of the end (top) of an earlier one has none.
struct KvLanes {
    KvSeq v;
    int top = -1;                                       // (nothing was bad so far)
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
        for (int o = 1; o < 64; o <<= 1) { const int t = __shfl_up(end, o); if (lane >= o) end = max(end, t); }
        const int before = __shfl_up(end, 1);
        if (v.r0 < max(top, lane ? before : 0)) v.n = 0;
        top = max(top, __shfl(end, 63));
    }
};
__device__ __forceinline__ int wave_sum_upto(int c, int lane) {          // inclusive
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) { const int t = __shfl_up(c, o); if (lane >= o) c += t; }
    return c;
}
// Work items of all sequences one behind the other: count(sequence) items each.  Finds the sequence of `item`, its
// number within it and the first item of the sequence; each wave counts for itself, so no list has to be built in a launch of its own.
template <class F>
__device__ __forceinline__ bool kv_find(const KvArgs& a, KvLanes x, int64_t item, int lane, bool check, F count, int* seq, int* local, int64_t* first, KvSeq* view) {
    int64_t base = 0;
    for (int s0 = 0;;) {
        const int c = count(x.v);
        if (a.n_seqs == 1) {                            // (nothing to add up)
            *seq = 0; *first = 0; *local = (int)item;
            *view = KvSeq{uniform(x.v.r0), uniform(x.v.n), uniform(x.v.len)};
            return item < uniform(c);
        }
        const int incl = wave_sum_upto(c, lane), total = uniform(__shfl(incl, 63));
        if (item < base + total) {
            const int l = __ffsll((unsigned long long)__ballot(base + incl > item)) - 1;
            *seq = uniform(s0 + l);
            *first = base + uniform(__shfl(incl - c, l));
            *local = (int)(item - *first);
            *view = KvSeq{uniform(__shfl(x.v.r0, l)), uniform(__shfl(x.v.n, l)), uniform(__shfl(x.v.len, l))};
            if (check) for (s0 += 64; s0 < a.n_seqs; s0 += 64) x.load(a, s0, lane, true);
            return true;
        }
        base += total;
        s0 += 64;
        if (s0 >= a.n_seqs) return false;
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
};
// How a batch is cut.  The rows of a sequence and KV head are its new tokens x the heads of the group; a tile is 16 * NT of
// them.  With `cut`, all tiles' key ranges are cut into runs of `run` chunks, the same for every sequence, so that about `target` items come out
// whatever the lengths are: one long conversation among short ones is spread over the card.  (attend_plan in asd_kv.hip says which batches are cut.)
template <int NT> __device__ __forceinline__ int kv_tiles(const KvArgs& a, const KvSeq& v) { return (int)(((int64_t)v.n * a.group + 16 * NT - 1) / (16 * NT)); }
template <int NT> __device__ __forceinline__ int kv_run(const KvAttendArgs& a, const KvLanes& all, int lane) {
    if (!a.cut) return 1 << 28;
    auto units = [&](const KvSeq& v) { return (int64_t)kv_tiles<NT>(a.kv, v) * ((v.len + 63) / 64); };
    int64_t t = units(all.v);
    for (int s = lane + 64; s < a.kv.n_seqs; s += 64) t += units(kv_seq(a.kv, s));      // (of bad ones no less than they have: longer runs)
    if (a.kv.n_seqs > 1) {
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) t += __shfl_xor(t, o);
    }
    const int run = (int)fminf((float)(t * a.kv.n_kv) / (float)a.target, 1e8f) + 1;
    return uniform(max(run, a.min_run));
}
// runs of a sequence, of equal length: its chunks / run, to the nearest
__device__ __forceinline__ int kv_splits(const KvSeq& v, int run) { return max(1, (int)(((int64_t)(v.len + 63) / 64 + run / 2) / run)); }
__device__ __forceinline__ int kv_per_split(const KvSeq& v, int n_splits) { return ((v.len + 63) / 64 + n_splits - 1) / n_splits; }

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
// their sum over the keys key0 .. last at one dim (0: there are none)
template <class C, int H> __device__ float kv_odd_sum(const KvArgs& a, int seq, int kvh, int key0, int last, int dim) {
    float sum = 0.f;
    for (int key = key0; key <= last; ++key) {
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
// 16 * NT rows against a run of chunks, in units: the keys of one step of V^T pieces (16 fp32, 32 bf16, 64 codes).  Four waves, wave w
// the units w, w + 4, ... of the run with a running maximum and sum per row, merged through LDS at the end.  Scores S[key][row] = K q^T and the output O[dim][row] = V^T P are matrix-core products with the rows as
// columns (see asd_attn.h); a unit's fragments go from memory into registers ahead of their use: memory-bound while the rows are few.
// 8 bits: K is widened with its scale, V without: V's scales go into the probabilities, one value per key.
// One token of 48 sequences of 500 to 8192 tokens, 64 / 8 heads x 128, 8 bits: 85 us, with the join 5.5 TB/s.  A batch too small for memory to
// bound it waits for its loads, 1.7 us for each unit of a wave: five rows of eight sequences of up to 1031 tokens, 40 heads, 16 us.
template <class A, class C, int H, int NT>
__global__ __launch_bounds__(256, A::KE == 4 ? 1 : 2) void kv_attend_kernel(const KvAttendArgs a) {
    using L = KvLayout<C, H>;
    using E = typename A::elem;
    constexpr int AE = A::KE, KK = L::KK, HP = L::HP, US = KK / AE, QS = HP * US;      // operand steps of a K piece, of a row
    constexpr int HT = L::HT, KST = L::KST, VS = L::KV / AE;                           // ... of a V^T piece
    constexpr int UPC = KV_UNITS(C), UK = 64 / UPC, KT = 4 / UPC, KSU = KST / UPC, PS = KSU * VS;      // units of a chunk; keys, score tiles, V^T pieces, steps of a unit
    __shared__ float so[4][16][H];
    __shared__ float sml[4][16][2];
    __shared__ int s_odd;
    const int tid = threadIdx.x, lane = tid & 63, w = uniform(tid >> 6), g = lane >> 4, m = lane & 15;
    int seq, local;
    int64_t first;
    KvSeq s;
    if (tid == 0) s_odd = 0;
    const bool check = blockIdx.x == 0 && w == 0;
    KvLanes all;
    all.load(a.kv, 0, lane, check);
    const int run = kv_run<NT>(a, all, lane), n_kv = a.kv.n_kv;
    if (!kv_find(a.kv, all, blockIdx.x, lane, check, [&](const KvSeq& v) { return kv_tiles<NT>(a.kv, v) * kv_splits(v, run) * n_kv; }, &seq, &local, &first, &s)) return;
    const int n_tiles = kv_tiles<NT>(a.kv, s), n_splits = kv_splits(s, run), per = kv_per_split(s, n_splits);
    const int kvh = local % n_kv, tile = local / n_kv % n_tiles, split = local / n_kv / n_tiles;
    const int rows = s.n * a.kv.group, base = s.len - s.n;
    int pos[NT];                                        // last key of this lane's rows (-1: no such row, or none)
    u32x4 qf[NT][QS];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int row = (tile * NT + t) * 16 + m, token = row / a.kv.group, head = kvh * a.kv.group + row % a.kv.group;
        const bool on = row < rows;
        pos[t] = on ? base + token : -1;
        const E* qp = (const E*)a.q + (s.r0 + (int64_t)token) * a.q_stride + head * H;
#pragma unroll
        for (int i = 0; i < QS; ++i) qf[t][i] = on ? *(const u32x4*)(qp + i / US * 4 * KK + g * KK + i % US * AE) : u32x4{0u, 0u, 0u, 0u};
    }
    const int last = base + (min((tile + 1) * NT * 16, rows) - 1) / a.kv.group, from = base + tile * NT * 16 / a.kv.group;      // positions of the tile's rows
    const int u_end = min((last + UK) / UK, (split + 1) * per * UPC);      // (nothing to do where last is negative)

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
    // The pages of 64 entries of the table lie in the wave's lanes (-1: no page of the pool): a look-up in memory per unit would wait
    // for every fragment asked for before it
    const int cpp = a.kv.page_tokens / 64;
    int page_base = -64, pages = 0;
    // the first unit from u on that has a page, and where it is; one without counts as hidden
    const char *at_k = nullptr, *at_v = nullptr;
    auto next = [&](int u) {
        for (; u < u_end; u += 4) {
            const int c = u / UPC, i = c / cpp;
            if (i - page_base >= 64) {
                page_base = i;
                pages = i + lane < a.kv.table_stride ? a.kv.table[(size_t)seq * a.kv.table_stride + i + lane] : -1;
                if ((unsigned)pages >= (unsigned)a.kv.n_pages) pages = -1;
            }
            const int page = __builtin_amdgcn_readlane(pages, i - page_base);
            const char* p = a.kv.pages + (((size_t)max(page, 0) * n_kv + kvh) * cpp + c % cpp) * L::CHUNK;
            at_k = p + u % UPC * KT * HP * 64 * KK * sizeof(typename C::elem);
            at_v = p + L::K_BYTES + u % UPC * KSU * 1024;
            if (page >= 0) break;
            if (lane == 0) kv_flag(a.kv, ASD_KV_BAD_PAGE);
        }
        return u;
    };
    bool odd = false;
    auto work = [&](Unit& f, const int key0, auto after_scores) {
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
        const bool edge = key0 + UK - 1 > from;
        const int n_keys = s.len - key0;
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
                        if (key0 + score_key<C>(kt, 4 * g + j) > pos[t]) sc[t][kt][j] = -INFINITY;
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
                        if (edge && key0 + score_key<C>(kt, 4 * g + j) > pos[t]) pr[kt][j] = 0.f;
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
            if (n_keys < UK) {                           // what is behind the end is cleared: 0 times whatever lies there must be 0
#pragma unroll
                for (int ks = 0; ks < KSU; ++ks)
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const uint32_t keep = kv_kept<C>(n_keys, ks, g, x);
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
    int unit = next(split * per * UPC + w);
    // One token against bf16 pages: two units in registers, all of the next on its way while one is worked on (one sequence of 8192 tokens,
    // 32 heads: 29.4 -> 28.6 us).  Codes and fp32 rows take more registers per unit or more time per key: with two units, 48 sequences
    // of 8-bit pages took 103 us and not 90, a small fp32 batch 10.6 and not 9.5
    if constexpr (NT == 1 && sizeof(typename C::elem) == 2) {
        Unit f0, f1;
        auto ask = [&](Unit& f) { ask_k(f, at_k); ask_v(f, at_v); };
        auto turn = [&](Unit& now, Unit& then) {
            const int un = next(unit + 4);
            if (un < u_end) ask(then);
            __builtin_amdgcn_sched_barrier(0);
            work(now, unit * UK, [] {});
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
            const int un = next(unit + 4);
            work(f, unit * UK, [&] { if (un < u_end) ask_k(f, at_k); });
            __builtin_amdgcn_sched_barrier(0);
            if (un < u_end) ask_v(f, at_v);
            __builtin_amdgcn_sched_barrier(0);
            unit = un;
        }
    }

    // ---- the waves' results, 16 rows at a time, wave order
    __syncthreads();                                    // (s_odd is cleared)
    if (odd && lane == 0) s_odd = 1;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        if (t) __syncthreads();
        l[t] = groups_sum(l[t]);
        if (g == 0) { sml[w][m][0] = mx[t]; sml[w][m][1] = l[t]; }
#pragma unroll
        for (int ht = 0; ht < HT; ++ht) *(f32x4*)&so[w][m][ht * 16 + 4 * g] = o[t][ht];
        __syncthreads();
        const int r = tid & 15, row = (tile * NT + t) * 16 + r, token = row / a.kv.group, head = kvh * a.kv.group + row % a.kv.group;
        float top = -INFINITY, sum = 0.f, wt[4];
#pragma unroll
        for (int ww = 0; ww < 4; ++ww) top = fmaxf(top, sml[ww][r][0]);
        const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
        for (int ww = 0; ww < 4; ++ww) { wt[ww] = __builtin_amdgcn_exp2f((sml[ww][r][0] - ref) * a.c2); sum += sml[ww][r][1] * wt[ww]; }
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        for (int d = (tid >> 4) * 4; d < H; d += 64) {
            float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ww = 0; ww < 4; ++ww) {
                const f32x4 x = *(const f32x4*)&so[ww][r][d];
                v[0] += x[0] * wt[ww]; v[1] += x[1] * wt[ww]; v[2] += x[2] * wt[ww]; v[3] += x[3] * wt[ww];
            }
            if (row >= rows) continue;
            if (s_odd) {
                const int first_key = max((from + 1) / UK * UK, split * per * 64), last_key = min(base + token, u_end * UK - 1);
                for (int j = 0; j < 4; ++j) v[j] += kv_odd_sum<C, H>(a.kv, seq, kvh, first_key, last_key, d + j);
            }
            if (n_splits == 1) {
                v[0] *= inv; v[1] *= inv; v[2] *= inv; v[3] *= inv;
                store4<A>((E*)a.out + (s.r0 + (int64_t)token) * a.out_stride + head * H + d, v);
            } else {
                const size_t at = (size_t)blockIdx.x * (16 * NT) + t * 16 + r;
                *(float4*)(a.o_part + at * H + d) = float4{v[0], v[1], v[2], v[3]};
                if (d == 0) { a.ml_part[at * 2] = top; a.ml_part[at * 2 + 1] = sum; }
            }
        }
    }
}


// Many rows (bf16): NW waves with 16 * NT rows each walk a run of chunks together, their fragments in LDS once for all of them.  They come by
// direct loads into a ring of five half-chunks (K, V^T, K, ..): one barrier per chunk c, behind which K and V^T of c have landed
// and the slots of c - 1 may be asked for anew (V^T of c + 1, K of c + 2).  A SIMD has two waves.
// (Prompts of 1035 to 2048 tokens, 32 heads x 128, bf16 pages, took 160 us so at the step when four waves of 16 rows took 199 and two waves with the
// next product's fragments in registers 200, both spilling.)  Bound by products and exponentials (in 8 bits the widening, too, which each
// wave does for itself) one after the other: the vector unit issues in 53 % of the busy cycles (8 bits 73), the matrix cores are at work in 38 (37),
// little of it at the same time; and by what each tile takes once.  These prompts now take 137 to 143 us (8-bit pages 156), 720 to 750 TFLOP/s,
// one of 8192 tokens 1001 TFLOP/s (944); 512 rows behind 8195 tokens and 260 behind 2665 in 8 bits, 64 / 8 heads, 214 us with the join.
template <class C, int H, int NT, int NW>
__global__ __launch_bounds__(64 * NW, 2) void kv_rows_kernel(const KvAttendArgs a) {
    using A = BF16;
    using L = KvLayout<C, H>;
    constexpr int AE = A::KE, KK = L::KK, HP = L::HP, US = KK / AE, QS = HP * US, HT = L::HT, KST = L::KST, VS = L::KV / AE, PS = KST * VS;
    constexpr int HF = L::K_BYTES / 1024, LH = HF / NW, SLOTS = 5, SC = 4, X = L::Q8 ? 1 : 0, RT = NW * NT;      // fragments of a half, requests per wave and half; chunks' scales; 16-row blocks of a tile
    static_assert(HF % NW == 0 && HF == 4 * HP && HF == HT * KST, "every wave asks for the same number of fragments");
    __shared__ u32x4 mem[SLOTS * HF * 64 + (L::Q8 ? SC * 8 : 0)];       // (bf16 at head dim 128: two of them are a unit's whole LDS)
    const int tid = threadIdx.x, lane = tid & 63, w = uniform(tid >> 6), g = lane >> 4, m = lane & 15;
    int seq, local;
    int64_t first;
    KvSeq s;
    const bool check = blockIdx.x == 0 && w == 0;
    KvLanes all;
    all.load(a.kv, 0, lane, check);
    const int run = kv_run<RT>(a, all, lane), n_kv = a.kv.n_kv;
    if (!kv_find(a.kv, all, blockIdx.x, lane, check, [&](const KvSeq& v) { return kv_tiles<RT>(a.kv, v) * kv_splits(v, run) * n_kv; }, &seq, &local, &first, &s)) return;
    const int n_tiles = kv_tiles<RT>(a.kv, s), n_splits = kv_splits(s, run), per = kv_per_split(s, n_splits);
    const int kvh = local % n_kv, tile = n_tiles - 1 - local / n_kv % n_tiles, split = local / n_kv / n_tiles;      // longest first
    const int rows = s.n * a.kv.group, base = s.len - s.n, row0 = (tile * NW + w) * NT * 16;
    int pos[NT];
    u32x4 qf[NT][QS];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int row = row0 + t * 16 + m, token = row / a.kv.group, head = kvh * a.kv.group + row % a.kv.group;
        const bool on = row < rows;
        pos[t] = on ? base + token : -1;
        const uint16_t* qp = (const uint16_t*)a.q + (s.r0 + (int64_t)token) * a.q_stride + head * H;
#pragma unroll
        for (int i = 0; i < QS; ++i) qf[t][i] = on ? *(const u32x4*)(qp + i / US * 4 * KK + g * KK + i % US * AE) : u32x4{0u, 0u, 0u, 0u};
    }
    auto chunks_of = [&](int row_end) { return (base + (min(row_end, rows) - 1) / a.kv.group + 64) / 64; };      // chunks that rows up to there see
    const int c0 = split * per, c_end = min(chunks_of((tile + 1) * 16 * RT), c0 + per);                         // ... of the workgroup
    const int c_my = row0 < rows ? min(chunks_of(row0 + 16 * NT), c_end) : 0;                                   // ... of this wave
    const int from = base + row0 / a.kv.group;
    const int c_main = min(c_end, (base + tile * RT * 16 / a.kv.group + 1) / 64);                               // chunks that all its rows see whole
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
        // The page of the chunk asked for next: 64 entries of the table lie in the wave's lanes (-1: no page of the pool)
        const int cpp = a.kv.page_tokens / 64;
        int page_i = c0 / cpp, in_page = c0 % cpp, page_base = page_i, pages = 0;
        auto fetch_pages = [&]() {
            const int i = page_base + lane;
            pages = i < a.kv.table_stride ? a.kv.table[(size_t)seq * a.kv.table_stride + i] : -1;
            if ((unsigned)pages >= (unsigned)a.kv.n_pages) pages = -1;
        };
        fetch_pages();
        uint32_t gone = 0;                               // bit c % 32: chunk c has no page
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
        auto ask_k = [&]() {                             // past the end: the last chunk again
            if (asked < c_end) {
                const int page = __builtin_amdgcn_readlane(pages, page_i - page_base);
                src = a.kv.pages + (((size_t)max(page, 0) * n_kv + kvh) * cpp + in_page) * L::CHUNK;
                n_bytes = page >= 0 ? -1 : 0;
                gone = page >= 0 ? gone & ~(1u << (asked & 31)) : gone | 1u << (asked & 31);
                lost |= page < 0;
                if (++in_page == cpp) { in_page = 0; ++page_i; }
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
        wait_vm<0, true>();                              // from here on only the ring's requests count
        ask_k(); ask_v(src, n_bytes); ask_k();           // K, V^T of the first chunk, K of the next
        auto turn = [&]() {
            if (page_i - page_base >= 62) {              // (once in 62 pages: the ring runs dry for a moment)
                page_base = page_i;
                fetch_pages();
                wait_vm<0, false>();
            }
            wait_vm<LH + X, true>();                     // the K of the next chunk may still be on its way
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
        };
        auto ask = [&]() { ask_v(src, n_bytes); ask_k(); };      // V^T of the next chunk, K of the one behind it
        // a chunk that this wave has products for; edge: some of its rows do not see all of it
        auto work = [&](const int c, auto is_edge) {
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
                for (int kt = 0; kt < 4; ++kt) f[(hp + 1) & 1][kt] = hp + 1 < HP ? kp[(kt * HP + hp + 1) * 64] : vp[kt * 64];
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
                    for (int j = 0; j < 4; ++j) vs[kt][j] = q8_scale((ve[kt] >> (8 * j)) & 255u);
            if constexpr (edge) {
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            if (c * 64 + score_key<C>(kt, 4 * g + j) > pos[t]) sc[t][kt][j] = -INFINITY;
                if constexpr (L::Q8) {                   // (an unwritten scale may be anything)
                    const int n_keys = s.len - c * 64;
#pragma unroll
                    for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                        for (int j = 0; j < 4; ++j) if (score_key<C>(kt, 4 * g + j) >= n_keys) vs[kt][j] = 0.f;
                }
            }
            u32x4 pf[NT][PS];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                float cm = sc[t][0][0];
#pragma unroll
                for (int kt = 0; kt < 4; ++kt)
#pragma unroll
                    for (int j = 0; j < 4; ++j) cm = fmaxf(cm, sc[t][kt][j]);
                cm = groups_max(cm);
                // The reference of a row's exponents need not be its maximum: it moves only when a weight would pass 2^8
                if (__any((cm - mx[t]) * a.c2 > 8.f)) {
                    const float mn = fmaxf(mx[t], cm), alpha = mn == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((mx[t] - mn) * a.c2);
                    mx[t] = mn;
                    l[t] *= alpha;
#pragma unroll
                    for (int ht = 0; ht < HT; ++ht) { o[t][ht][0] *= alpha; o[t][ht][1] *= alpha; o[t][ht][2] *= alpha; o[t][ht][3] *= alpha; }
                }
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
                    pf[t][kt / 2][kt % 2 * 2] = bf16_pair(e[0], e[1]);      // as V is: see kv_attend_kernel
                    pf[t][kt / 2][kt % 2 * 2 + 1] = bf16_pair(e[2], e[3]);
                }
                l[t] += sum[0] + sum[1];
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
        // A chunk with an edge: keys behind the end and values that are not finite leave V^T (see kv_clean); each wave cleans what it has asked for
        auto clean = [&](const int c) {
            const int n_keys = s.len - c * 64;
            uint32_t hit = 0;
#pragma unroll 1
            for (int q = 0; q < LH; ++q) {
                const int j = w + NW * q;
                u32x4* p = mem + (use_v * HF + j) * 64 + lane;
                u32x4 f = *p;
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    f[x] &= kv_kept<C>(n_keys, j % KST, g, x);
                    hit |= kv_odd<C>(f[x]);
                    f[x] = kv_clean<C>(f[x]);
                }
                *p = f;
            }
            odd |= hit != 0;
            asm volatile("" ::: "memory");
            wait_vm<63, true>();                         // (the ring's requests go on)
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
        };
        auto done = [&]() {
            use_k = use_k + 2 >= SLOTS ? use_k + 2 - SLOTS : use_k + 2;
            use_v = use_v + 2 >= SLOTS ? use_v + 2 - SLOTS : use_v + 2;
        };
        // Chunks that all rows of the workgroup see run in a loop of their own, without masks; those with an edge, or without a page, one by one
        int c = c0;
        for (;;) {
            for (; c < c_main && gone == 0; ++c) {
                turn();
                work(c, std::false_type{});
                done();
            }
            if (c >= c_end) break;
            turn();
            if (c >= c_main) clean(c);                   // (beside a missing page: what all rows see goes through the products)
            if (c < c_my && !((gone >> (c & 31)) & 1u)) work(c, std::true_type{}); else ask();
            done();
            gone &= ~(1u << (c & 31));
            ++c;
        }
        if (lost && tid == 0) kv_flag(a.kv, ASD_KV_BAD_PAGE);
        wait_vm<0, true>();                              // no request may outlive the workgroup's LDS
        __syncthreads();
        int* any = (int*)mem;                            // the ring is free: what one lane has taken out concerns all
        if (tid == 0) *any = 0;
        __syncthreads();
        if (odd) *any = 1;
        __syncthreads();
        odd = *any != 0;
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const float z = groups_sum(l[t]);
        const int row = row0 + t * 16 + m, token = row / a.kv.group, head = kvh * a.kv.group + row % a.kv.group;
        if (row >= rows) continue;
        const size_t at = (size_t)(first + (int64_t)(split * n_tiles + tile) * n_kv + kvh) * (16 * RT) + row - tile * 16 * RT;
        uint16_t* out = (uint16_t*)a.out + (s.r0 + (int64_t)token) * a.out_stride + head * H;
        if (n_splits == 1) {
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
                const float x = kv_odd_sum<C, H>(a.kv, seq, kvh, max(c_main, c0) * 64, min(pos[t], c_end * 64 - 1), dim);
                if (finite(x)) continue;                 // (nothing of its own row's to add)
                if (n_splits == 1) out[dim] = BF16::from_f32(BF16::to_f32(out[dim]) + x); else a.o_part[at * H + dim] += x;
            }
        }
    }
}

// Joins the runs of tiles whose keys were cut: a workgroup per tile, KV head and 16 of its rows.  16 lanes hold a row's dims;
// where fewer rows are in use than 16, the lanes left over take every second (fourth, ..) run, added up through LDS at the end.  A launch of its own,
// 4 to 5 us for one token's runs, 13 us for those of 772 rows: joined by the last workgroup to arrive, counters would have to be zero when the
// call starts, and the workspace could not be any memory.
template <class A, int H, int NT>
__global__ __launch_bounds__(256) void kv_join_kernel(const KvAttendArgs a) {
    using E = typename A::elem;
    constexpr int R = 16 * NT, DL = H / 16, U = 8;      // rows of a tile, dims of a lane, runs in flight
    __shared__ float so[16][H];
    __shared__ float sml[16][2];
    const int tid = threadIdx.x, lane = tid & 63, n_kv = a.kv.n_kv, group = a.kv.group;
    int seq, local;
    int64_t first;
    KvSeq s;
    KvLanes all;
    all.load(a.kv, 0, lane, false);
    const int run = kv_run<NT>(a, all, lane);
    // (tile, KV head) pairs of the cut sequences
    if (!kv_find(a.kv, all, blockIdx.x, lane, false, [&](const KvSeq& v) { return kv_splits(v, run) > 1 ? kv_tiles<NT>(a.kv, v) * n_kv : 0; }, &seq, &local, &first, &s)) return;
    // the first work item of the sequence
    int64_t item0 = 0;
    for (int s0 = 0; s0 <= seq; s0 += 64) {
        if (s0) all.load(a.kv, s0, lane, false);
        int64_t c = s0 + lane < seq ? (int64_t)kv_tiles<NT>(a.kv, all.v) * kv_splits(all.v, run) * n_kv : 0;
        if (seq)
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) c += __shfl_xor(c, o);
        item0 += c;
    }
    const int n_splits = kv_splits(s, run), n_tiles = kv_tiles<NT>(a.kv, s), kvh = local % n_kv, tile = local / n_kv;
    const int row0 = tile * R + blockIdx.y * 16, left = min(s.n * group - row0, 16);
    if (left <= 0) return;
    const int lg = left > 8 ? 4 : left > 4 ? 3 : left > 2 ? 2 : left > 1 ? 1 : 0, phases = 16 >> lg;
    const int r = (tid >> 4) & ((1 << lg) - 1), phase = tid >> (4 + lg), d0 = (tid & 15) * DL;
    const int64_t step = (int64_t)n_tiles * n_kv * R, at = (item0 + (int64_t)tile * n_kv + kvh) * R + blockIdx.y * 16 + r;      // a run's place to the next run's
    float acc[DL] = {}, top = -INFINITY, sum = 0.f;
    if (r < left)
        for (int i0 = phase; i0 < n_splits; i0 += U * phases) {
            float x[U][DL];
            float2 ml[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const bool on = i0 + u * phases < n_splits;
                const int64_t p = at + (on ? i0 + u * phases : i0) * step;
                ml[u] = *(const float2*)(a.ml_part + p * 2);
                if (!on) ml[u] = float2{-INFINITY, 0.f};
#pragma unroll
                for (int d = 0; d < DL; d += 2) { const float2 y = *(const float2*)(a.o_part + p * H + d0 + d); x[u][d] = y.x; x[u][d + 1] = y.y; }
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
                if (i0 + u * phases >= n_splits) break;
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
