// What the forward and the backward kernels of attention share: operands of the matrix cores, tiles in LDS, and the
// description of a call.
//
// Element types go through 32 x 32 products whose operands are 16 bytes a lane: eight bf16 (one v_mfma_f32_32x32x16_bf16)
// or four floats (four v_mfma_f32_32x32x2_f32).  Lane l = 32 h + c holds row (column) c of the operand and the contraction
// indices kStep t + (kStep / 2) h + 0, 1, ..; register r of a product holds row 8 (r / 4) + 4 h + r % 4 of column c.  So the
// registers of one product, a step's share at a time, are the second operand of the next one as they stand, if its first operand
// takes the rows in that order: probabilities never pass through LDS.
#pragma once

#include <type_traits>

#include "fs_internal.h"

namespace fs {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

template <typename T> struct Mma;
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// Floats as the sum of two fp16, under a power of two for all of a head's rows (of do: for each) that puts the largest into [2^14, 2^15):
// 22 bits of every element down to 2^-17 of the largest, and never less than 2^-40 of it.  A product takes three products of the pieces
// (the two lower ones' is below 2^-22), three v_mfma_f32_32x32x16_f16 of 32 cycles for sixteen coordinates, where the fp32
// matrix cores take eight of 64.
struct Pair {};
template <> struct Mma<Pair> {
    using Elem = float;
    struct Frag {
        f16x8 h, l;
    };
    static constexpr int kStep = 16;
    static constexpr int kPiece = 8;
    static __device__ inline f32x16 mma(const Frag &a, const Frag &b, f32x16 c)
    {
        c = __builtin_amdgcn_mfma_f32_32x32x16_f16(a.l, b.h, c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x16_f16(a.h, b.l, c, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(a.h, b.h, c, 0, 0, 0);
    }
    // two elements: their upper pieces, and what is left of each
    static __device__ inline void split(float a, float b, f16x2 &h, f16x2 &l)
    {
        // as floats first: where a product is converted, one instruction may round it to fp16 at once, which near a tie is not the
        // upper piece that the lower one was taken off
        asm volatile("" : "+v"(a), "+v"(b));
        h = f16x2{(_Float16)a, (_Float16)b};
        l = f16x2{(_Float16)fmaf((float)h[0], -1.0f, a), (_Float16)fmaf((float)h[1], -1.0f, b)};
    }
    static __device__ inline Frag pack(const f32x16 &v, int t)
    {
        Frag f;
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            f16x2 h, l;
            split(v[8 * t + j], v[8 * t + j + 1], h, l);
            f.h[j] = h[0];
            f.h[j + 1] = h[1];
            f.l[j] = l[0];
            f.l[j + 1] = l[1];
        }
        return f;
    }
};

template <> struct Mma<__bf16> {
    using Elem = __bf16;
    using Frag = bf16x8;
    static constexpr int kStep = 16;    // contraction indices of a fragment
    static constexpr int kPiece = 8;    // elements of 16 bytes
    static __device__ inline f32x16 mma(Frag a, Frag b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
    // registers kStep / 2 * t .. of a product as an operand
    static __device__ inline Frag pack(const f32x16 &v, int t)
    {
        Frag f;
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = (__bf16)v[8 * t + j];
        return f;
    }
    // what pack() rounds off
    static __device__ inline Frag rest(const f32x16 &v, int t)
    {
        Frag f;
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = (__bf16)(v[8 * t + j] - (float)(__bf16)v[8 * t + j]);
        return f;
    }
};

template <> struct Mma<float> {
    using Elem = float;
    using Frag = f32x4;
    static constexpr int kStep = 8;
    static constexpr int kPiece = 4;
    static __device__ inline f32x16 mma(Frag a, Frag b, f32x16 c)
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
        return c;
    }
    static __device__ inline Frag pack(const f32x16 &v, int t)
    {
        Frag f;
#pragma unroll
        for (int j = 0; j < 4; ++j) f[j] = v[4 * t + j];
        return f;
    }
};

// A tile of rows in LDS, DP elements each (zero beyond d).  16-byte pieces are permuted within their row so that the lanes of a
// fragment read, which take one piece each of 32 consecutive rows, meet in as few banks as there are.
using LdsPtr = const __attribute__((address_space(3))) char *;
template <typename T, int DP> struct Tile {
    static constexpr int kRow = DP * (int)sizeof(T);   // bytes
    static constexpr int kPieces = kRow / 16;
    static constexpr bool kWide = kPieces % 8 == 0;
    static __device__ inline int swz(int row) { return kWide ? row & 7 : (row >> 1) & 3; }
    static __device__ inline int at(int row, int piece) { return row * kRow + ((piece ^ swz(row)) << 4); }

    // The permutation touches the lowest two or three bits of a piece's number: fragments that differ in higher bits, and in their
    // first row (a multiple of 32 or of a step), are at constant distances.  What is left for a lane to compute once:
    static constexpr int kRowBases = kWide ? 4 : 2, kColBases = kWide ? 2 : 1;
    struct Lanes {
        int row[kRowBases], col[kColBases];
    };
    static __device__ inline Lanes lanes(int lane)
    {
        Lanes b;
#pragma unroll
        for (int t = 0; t < kRowBases; ++t) b.row[t] = at(lane & 31, 2 * t + (lane >> 5));
        const int i = lane & 15;
#pragma unroll
        for (int q = 0; q < kColBases; ++q) {
            if constexpr (sizeof(T) == 2)
                b.col[q] = at(4 * (lane >> 5) + (i >> 2), 4 * q + ((lane >> 4) & 1) * 2 + ((i & 3) >> 1)) + (i & 1) * 8;
            else
                b.col[q] = 0;
        }
        return b;
    }
    // operand with the tile's rows as rows: step t of the contraction over coordinates
    static __device__ inline typename Mma<T>::Frag rows(LdsPtr lds, const Lanes &b, int row0, int t)
    {
        return *(const __attribute__((address_space(3))) typename Mma<T>::Frag *)(lds + b.row[t % kRowBases] + row0 * kRow +
                                                                                  t / kRowBases * kRowBases * 32);
    }
    // operand with coordinates 32 db .. 32 db + 31 as rows: step t of the contraction over the 32 rows from row0 on, in the order
    // in which a product's registers hold them
    static __device__ inline typename Mma<T>::Frag cols(LdsPtr lds, const Lanes &b, int row0, int t, int db, int lane)
    {
        if constexpr (sizeof(T) == 2) {
            // sixteen lanes read 4 rows x 16 coordinates, eight bytes each, and get a coordinate each: its four rows
            using P = __attribute__((address_space(3))) s16x4 *;
            const LdsPtr at = lds + b.col[db % kColBases] + (row0 + 16 * t) * kRow + db / kColBases * kColBases * 64;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)at);
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(at + 8 * kRow));
            return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            f32x4 f;
            const int c = 32 * db + (lane & 31);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                f[j] = *(const __attribute__((address_space(3))) float *)(lds + at(row0 + 8 * t + 4 * (lane >> 5) + j, c >> 2) + (c & 3) * 4);
            return f;
        }
    }
};
// Pairs: 32 rows of the upper pieces, then of the lower, each like a bf16 tile.
template <int DP> struct Tile<Pair, DP> {
    using B = Tile<__bf16, DP>;
    using Lanes = typename B::Lanes;
    using Frag = Mma<Pair>::Frag;
    static constexpr int kRow = 2 * B::kRow, kPieces = 2 * B::kPieces;
    static constexpr int kSub = 32 * kRow, kLower = 32 * B::kRow;
    static __device__ inline Lanes lanes(int lane) { return B::lanes(lane); }
    static __device__ inline Frag rows(LdsPtr lds, const Lanes &b, int row0, int t)
    {
        const LdsPtr p = lds + row0 / 32 * kSub;
        return {__builtin_bit_cast(f16x8, B::rows(p, b, 0, t)), __builtin_bit_cast(f16x8, B::rows(p + kLower, b, 0, t))};
    }
    static __device__ inline Frag cols(LdsPtr lds, const Lanes &b, int row0, int t, int db, int lane)
    {
        const LdsPtr p = lds + row0 / 32 * kSub;
        return {__builtin_bit_cast(f16x8, B::cols(p, b, 0, t, db, lane)), __builtin_bit_cast(f16x8, B::cols(p + kLower, b, 0, t, db, lane))};
    }
    // a lane's operand from an image (see PairImage): step t of row `row`
    static __device__ inline Frag from_image(const char *img, int row, int t, int half)
    {
        const char *p = img + (int64_t)(row >> 5) * kSub + B::at(row & 31, 2 * t + half);
        return {*(const f16x8 *)p, *(const f16x8 *)(p + kLower)};
    }
};
// tiles of an image lie in memory as in LDS: linear copies
template <int DP, int ROWS, int NT> struct DmaImage {
    static constexpr int kTile = ROWS * Tile<Pair, DP>::kRow, kCount = kTile / 16 / NT;
    static_assert(kTile % (16 * NT) == 0, "");
    static __device__ inline void load(const char *tile, unsigned lds, int tid)
    {
        const unsigned to = __builtin_amdgcn_readfirstlane(lds + (tid >> 6) * 1024);
#pragma unroll
        for (int i = 0; i < kCount; ++i) dma16s(tile + i * NT * 16, tid * 16, to + i * NT * 16);
    }
};
__device__ inline unsigned lds_address(LdsPtr p) { return (unsigned)(uintptr_t)p; }

// How a tile comes to LDS.
//  kDma   straight from memory (direct loads, 16 bytes a lane, no registers): aligned rows whose offsets within a tile fit
//         32 bits
//  kVec   through registers, 16 bytes a load: aligned rows
//  kAny   through registers, an element a load
// What removed keys (bias of minus infinity) hold does not matter, NaN included: the registers' way leaves it out, the direct one
// clears it in LDS (clear_removed).
// (Pairs are always direct; there the two others say how rows of the tensors themselves are read.)
enum Load { kDma, kVec, kAny };

// Direct loads of a tile of ROWS rows by NT threads: LDS takes consecutive 16-byte pieces of consecutive lanes, so a lane fetches the piece
// that the permutation puts there.  Pieces beyond d are left alone (zeroed once).  Where a round of the threads is a whole number of rows
// that the permutation treats alike, a lane's offset is the same in every round, and the rounds differ in their uniform base.
template <typename T, int DP, int ROWS, int NT> struct Dma {
    using TL = Tile<T, DP>;
    static constexpr int kCount = ROWS * TL::kPieces / NT, kTile = ROWS * TL::kRow;
    static constexpr int kRound = NT / TL::kPieces;   // rows
    static constexpr bool kAlike = NT % TL::kPieces == 0 && kRound % 8 == 0;
    static constexpr int kOffsets = kAlike ? 1 : kCount;
    static __device__ inline int row(int tid, int i) { return (tid + i * NT) / TL::kPieces; }
    static __device__ inline int piece(int tid, int i) { return ((tid + i * NT) % TL::kPieces) ^ TL::swz(row(tid, i)); }
    // base: of the tile's first row (uniform); off: bytes from there, of each round or of the first; round: bytes between rounds;
    // rows from `count` on are left alone
    static __device__ inline void load(const char *base, const unsigned (&off)[kOffsets], int64_t round, unsigned lds, int tid, int d, int count)
    {
        const unsigned to = __builtin_amdgcn_readfirstlane(lds + (tid >> 6) * 1024);
        if (d == DP && count >= ROWS) {
#pragma unroll
            for (int i = 0; i < kCount; ++i) {
                // (a workgroup of one wave is alone with its keys: one query over 50021 keys, four sets, eight heads of d = 128,
                // 120 us, and 130 through the caches)
                if constexpr (NT == 64) dma16s_nt(kAlike ? base + i * round : base, off[kAlike ? 0 : i], to + i * NT * 16);
                else dma16s(kAlike ? base + i * round : base, off[kAlike ? 0 : i], to + i * NT * 16);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kCount; ++i)
                if (piece(tid, i) * Mma<T>::kPiece < d && row(tid, i) < count)
                    dma16s(kAlike ? base + i * round : base, off[kAlike ? 0 : i], to + i * NT * 16);
        }
    }
    // What no load writes is zero, or a row of an earlier tile (which no probability counts): zeroed before the first tile where
    // there are pieces beyond d, or where the last tile, of `count` rows, has no tile before it in its buffer.
    static __device__ inline void clear(char *lds, int tid, int d, int count, int tiles)
    {
        if (d == DP && (count >= ROWS || tiles > 2)) return;
        for (int i = tid; i < 4 * kTile / 16; i += NT) *(uint4 *)(lds + 16 * i) = make_uint4(0, 0, 0, 0);
        __syncthreads();
    }
};
// Zeroes the rows of a tile's keys and values whose bias is minus infinity; all of the workgroup's threads call it, after a barrier
// behind which the tile is there.  If there are such rows it ends in another barrier.  Against the registers' way for every tile with a
// bias: forward 410 instead of 497 us (one set of 8192 points, 16 heads of 64, bf16), forward and backward 702 instead of 770 (two sets
// of 4096, 8 heads of 128), the same at 1000 points and in float32.
template <typename T, int DP, int KEYS, int NT> __device__ inline void clear_removed(char *keys, char *values, const float *bias, int tid)
{
    bool any = false;
#pragma unroll
    for (int i = 0; i < KEYS; i += 64)
        if (i + (tid & 63) < KEYS) any = any || bias[i + (tid & 63)] == -INFINITY;
    if (!__any(any)) return;   // (the same for every wave)
    for (int i = tid; i < KEYS * Tile<T, DP>::kPieces; i += NT) {
        const int row = i / Tile<T, DP>::kPieces;
        if (bias[row] == -INFINITY) {
            *(uint4 *)(keys + 16 * i) = make_uint4(0, 0, 0, 0);
            *(uint4 *)(values + 16 * i) = make_uint4(0, 0, 0, 0);
        }
    }
    __syncthreads();
}
__device__ inline void dma_wait() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

// 16 bytes of a row: elements piece * kPiece .. of d, zero beyond.  ALN: rows are 16-byte aligned and d is a multiple of kPiece.
template <typename T, bool ALN> __device__ inline uint4 load_piece(const T *row, int piece, int d)
{
    constexpr int E = Mma<T>::kPiece;
    if constexpr (ALN) {
        return piece * E < d ? *(const uint4 *)(row + piece * E) : make_uint4(0, 0, 0, 0);
    } else {
        union {
            uint4 u;
            T e[E];
        } v;
        v.u = make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int j = 0; j < E; ++j)
            if (piece * E + j < d) v.e[j] = row[piece * E + j];
        return v.u;
    }
}

// four coordinates each of a product's column: coordinates col + 8 u + 0 .. 3 from registers 4 u ..
template <typename T, bool ALN> __device__ inline void store_column(T *row, const f32x16 &v, float f, int col, int d)
{
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        if (ALN) {   // (d is a multiple of four, and so is col)
            if (col + 8 * u < d) {
                typedef T T4 __attribute__((ext_vector_type(4)));
                T4 w;
#pragma unroll
                for (int j = 0; j < 4; ++j) w[j] = (T)(v[4 * u + j] * f);
                *(T4 *)(row + col + 8 * u) = w;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (col + 8 * u + j < d) row[col + 8 * u + j] = (T)(v[4 * u + j] * f);
        }
    }
}

// where the rows of one tensor lie: element strides of sets (batch), rows and heads
struct HeadsAt {
    int64_t batch, row, head;
};

// Pairs of a call in the workspace: per (set, kv head) tiles of 32 packed rows (or keys), padded to 128 rows, zero where nothing is
// admitted; and eight floats: the scales of q, k and v and the smallest of the rows of do (powers of two), the largest row norm of v, and
// that of do over the row's sum of exponentials.
enum { kPairQ, kPairK, kPairV, kPairDo, kPairTensors };
struct PairImage {
    char *img[kPairTensors];
    float *scale;
    f32x4 *row;    // of the rows of do, padded like them: the scale; <do, o> of do times 2^-15 of it; |do| times it; 0
    float *part;   // maxima of chunks of rows
};
constexpr float kPairP = 16.0f;      // probabilities below a reference (up to 2^11: kSlackPair) enter the second product times this
constexpr float kPairN = 32768.0f;   // normalised ones times this (2^15)

__host__ __device__ inline int64_t pair_rows(int64_t rows) { return (rows + 127) / 128 * 128; }

struct AttnCall {
    PairImage pair;
    const void *q, *k, *v;
    HeadsAt sq, sk, sv;
    void *o;                     // forward: written; backward: read
    HeadsAt so;
    float *stat;                 // [batch][heads][n][2]: the row's largest score, and its sum of exponentials below that
    const void *d_o;             // backward
    HeadsAt s_do;
    void *dq, *dk, *dv, *dbias;
    HeadsAt sdq, sdk, sdv;
    int64_t dbias_ld;
    float *row_stat;             // backward: [batch][kv head][3][packed rows, padded]: see k_attn_dq
    const int32_t *q_len, *k_len;
    const float *bias;
    int64_t bias_ld;
    int32_t batch, n, m, kv_heads, group, d, causal;
    float scale;
    // Splits of the streamed side; more than one: partial results, merged afterwards
    int32_t splits;
    float *part, *part_stat;
    float *dbias_part;           // backward: [split][batch][kv head][key]
};

// The heads that share keys are taken together: packed row r of (set, kv head) is query r / group of head kv_head * group + r % group.
struct Packed {
    int q, g;
};
__device__ inline Packed unpack(int r, int group)
{
    if (group == 1) return {r, 0};
    const int q = r / group;
    return {q, r - q * group};
}

// What a workgroup works on.  Workgroups that share an XCD's L2 (ids equal mod 8) take consecutive work of the order (set and kv head;
// block of rows or keys; split).  Under a causal line blocks are of unequal length, and consecutive blocks would give one XCD the
// long half of a head and its neighbour the short one: `rank` counts blocks from the longest, and
//  - where every XCD has whole heads, their blocks come by rank, the longest of all heads first;
//  - where a head has a whole number of XCDs, each takes every so many-th of them;
//  - otherwise the longest of all heads come first everywhere, and XCDs share heads;
// the last also where sets have lengths of their own: an XCD with the longest sets alone would finish after the others.
struct Work {
    int split, rank, hk, b;
};
__device__ inline Work work_of(int id, int total, int splits, int blocks, int kv_heads, bool causal, bool ragged)
{
    const int x = id & 7, per = total >> 3, more = total & 7, heads = total / (splits * blocks);
    const int share = heads < 8 && 8 % heads == 0 && blocks % (8 / heads) == 0 ? 8 / heads : 0;   // XCDs of a head
    const bool mixed = ragged || (causal && heads % 8 != 0 && !share);
    if (!mixed) id = x * per + (x < more ? x : more) + (id >> 3);
    Work w;
    w.split = id % splits;
    id /= splits;
    int j;
    if (mixed) {
        j = id / heads;
        id %= heads;
    } else {
        j = id % blocks;
        id /= blocks;
        if (causal && share) {
            j = j % (blocks / share) * share + j / (blocks / share);
        } else if (causal) {
            const int own = heads / 8, at = id % own * blocks + j;   // heads of an XCD; place in its order
            j = at / own;
            id += at % own - id % own;
        }
    }
    w.rank = j;
    w.hk = id % kv_heads;
    w.b = id / kv_heads;
    return w;
}

// Whether a float32 call goes through pairs, the bytes that they take (each piece rounded up to 256), and their making.
bool pair_worth(const Ctx *c, const AttnCall &a, bool grad);
size_t pair_bytes(const AttnCall &a, bool grad);
void pair_layout(AttnCall *a, char *ws, bool grad);
fs_status launch_pairs(Ctx *c, const AttnCall &a, bool grad, bool aligned);

// how a forward pass is launched
struct AttnPlan {
    int rows = 0, splits = 1, threads = 64;   // packed rows and threads of a workgroup
    bool pairs = false;
    int64_t grid = 0;
    size_t part_bytes = 0, stat_bytes = 0, pair_bytes = 0;
};
AttnPlan attn_plan(const Ctx *c, const AttnCall &a, bool f32);
fs_status launch_attn(Ctx *c, const AttnCall &a, const AttnPlan &p, bool f32, bool aligned);

// ... and a backward pass: rows' side (dq) and keys' side (dk, dv)
struct AttnGradPlan {
    int q_splits = 1, k_splits = 1;
    bool pairs = false;
    int64_t q_grid = 0, k_grid = 0;
    size_t stat_bytes = 0, dq_bytes = 0, dkv_bytes = 0, dbias_bytes = 0, pair_bytes = 0;
};
AttnGradPlan attn_grad_plan(const Ctx *c, const AttnCall &a, bool f32);
// `ws`: the bytes of the plan, each piece rounded up to 256
fs_status launch_attn_grad(Ctx *c, AttnCall a, const AttnGradPlan &p, char *ws, bool f32, bool aligned);

// the power of two that puts `top` into [2^e, 2^(e + 1)), as far as floats go; 1 where there is nothing to scale
__device__ inline float pair_power(float top, int e)
{
    if (!(top > 0.0f && top < INFINITY)) return 1.0f;
    e += 254 - (int)(__builtin_bit_cast(uint32_t, top) >> 23);
    e = e < 1 ? 1 : e > 240 ? 240 : e;
    return __builtin_bit_cast(float, (uint32_t)e << 23);
}
__device__ inline int pair_exponent(float v) { return (int)(__builtin_bit_cast(uint32_t, v) >> 23) - 127; }
__device__ inline float pair_mantissa(float v) { return __builtin_bit_cast(float, (__builtin_bit_cast(uint32_t, v) & 0x7fffffu) | 0x3f800000u); }
__device__ inline float pair_two(int e) { return __builtin_bit_cast(float, (uint32_t)((e < -126 ? -126 : e > 127 ? 127 : e) + 127) << 23); }   // 2^e

// What turns products of pieces into what they stand for.
struct PairScale {
    float score;   // of <q, k>, with the call's own scale
    float v;       // 1 / scale of v
};
__device__ inline PairScale pair_scale(const AttnCall &c, int64_t bh)
{
    const float *s = c.pair.scale + 8 * bh;
    const float q = 1.0f / s[kPairQ], k = 1.0f / s[kPairK];
    PairScale p;
    // (in 64 bits, and inside the normal floats: what is removed is minus infinity times this, also where all scores are as good as zero)
    p.score = (float)fmin(fmax((double)c.scale * q * k, 0x1p-126), 0x1p126);
    p.v = 1.0f / s[kPairV];
    return p;
}
// ... and of the backward pass.  The gradient of a score, p_ij (<do_i, v_j> - D_i), is at most 2 |do_i| |v| / l_i in size: l_i is the sum
// of exponentials that the largest is one of.  It enters the product for dq, a row's own, under a power of two of that row, from its |do_i|
// and l_i, so that it has its 22 bits in every row.  dk and dv are sums over rows: there it is under one for the head, `ds`, from the
// largest |do_i| / l_i, and p_ij under kPairN times the share of the row's do in the head's largest (do has a scale for every row).
struct PairGrad {
    float top;       // the largest |v| in units of its pieces
    float scale_v;
    int v, g, ds;    // exponents: of the scales of v and of the row of do that has the smallest, and of what puts the head's largest
                     // gradient of a score into [2^13, 2^14)
    float dov;       // ds / (scale of v, g, kPairN): of products of pieces of do and v, and of D in their units
};
__device__ inline PairGrad pair_grad(const AttnCall &c, int64_t bh)
{
    const float *s = c.pair.scale + 8 * bh;
    PairGrad p;
    p.scale_v = s[kPairV];
    p.top = s[4] * p.scale_v;
    p.v = pair_exponent(p.scale_v);
    p.g = pair_exponent(s[kPairDo]);
    const float a = s[4], b = s[5];   // (their product need not be a float)
    const int e = pair_exponent(a) + pair_exponent(b);
    const float m = pair_mantissa(a) * pair_mantissa(b);
    p.ds = a > 0.0f && b > 0.0f && a < INFINITY && b < INFINITY ? 13 - 1 - e - (m >= 2.0f) : 0;
    p.dov = pair_two(p.ds - p.v - p.g - 15);
    return p;
}
// f 2^e in two factors: what is of moderate size stays a float between them if it is one after both.
struct PairFactor {
    float a, b;
};
__device__ inline PairFactor pair_factor(float f, int e) { return {pair_two(e / 2), f * pair_two(e - e / 2)}; }

__device__ inline float across_halves_max(float v)
{
    const auto p = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
    return fmaxf(__builtin_bit_cast(float, (unsigned)p[0]), __builtin_bit_cast(float, (unsigned)p[1]));
}
__device__ inline float across_halves_sum(float v)
{
    const auto p = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, v), __builtin_bit_cast(unsigned, v), false, false);
    return __builtin_bit_cast(float, (unsigned)p[0]) + __builtin_bit_cast(float, (unsigned)p[1]);
}

}  // namespace fs
