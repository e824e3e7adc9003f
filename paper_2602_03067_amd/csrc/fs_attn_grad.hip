// Backward pass of attention.  With p_ij recomputed from the row statistics of the forward pass and D_i = <do_i, o_i>,
//   dv_j = sum_i p_ij do_i      ds_ij = p_ij (<do_i, v_j> - D_i)      dq_i = scale sum_j ds_ij k_j
//   dk_j = scale sum_i ds_ij q_i      dbias_j = sum_i ds_ij
// (sums over i run over all heads that share the keys).  Two passes that both recompute the scores, one whose waves hold 32
// rows and stream keys (dq, and D on the way), one whose waves hold 32 keys and stream rows (dk, dv): seven products of
// n m d instead of five, but nothing is added by atomics, so results do not depend on an order, and no n x m matrix is stored.
#include <algorithm>

#include "fs_attn.h"

namespace fs {
namespace {

constexpr float kLog2eF = 1.44269504088896340736f;

// What turns a score into a probability: exp2((s - m) log2 e - off), m the row's largest score (DIFF: the difference first, see
// k_attn), or exp2(s log2 e - off) with m in off.  A row that sees no key has off = infinity.
struct RowStat {
    float m, off;
};
template <bool DIFF> __device__ inline RowStat row_stat(float top, float sum)
{
    if (!(sum > 0.0f) && sum == sum) return {0.0f, INFINITY};
    const float lg = __builtin_amdgcn_logf(sum);
    return DIFF ? RowStat{top, lg} : RowStat{0.0f, fmaf(top, kLog2eF, lg)};
}

constexpr int kRowBlock = 128;   // packed rows of a dq workgroup; the row statistics are padded to whole ones
__device__ inline int64_t round_up_rows(int rows) { return ((int64_t)rows + kRowBlock - 1) / kRowBlock * kRowBlock; }
template <typename T> constexpr int row_tile(int dp) { return std::is_same<T, __bf16>::value || (std::is_same<T, Pair>::value && dp <= 64) ? 64 : 32; }

// waves per SIMD: what registers allow without spills
template <typename T> constexpr int dq_waves(int dp) { return std::is_same<T, __bf16>::value || dp < 96 ? 2 : 1; }
template <typename T> constexpr int dkv_waves(int dp)
{
    return std::is_same<T, __bf16>::value || dp < (std::is_same<T, Pair>::value ? 96 : 64) ? 2 : 1;
}

// Rows in registers, keys streamed, as in k_attn: S^T = K Q^T and dP^T = V dO^T end as a row's ds in the order dQ^T += K^T dS^T takes them.
// Three products a score; bound by LDS and the matrix cores together: 8192 points under a causal line, 16 heads of 128 over 4, bf16:
// 438 us, 940 TFLOP/s, busy 59 % and 44 %; 64 heads of 1024 points, d = 64: 39 us, 650 TFLOP/s, one round of workgroups whose
// beginnings and ends show.
template <typename T, int DP, int KT, int WAVES, bool BIAS, Load LOAD, bool FINE>
__global__ __launch_bounds__(64 * WAVES, dq_waves<T>(DP)) void k_attn_dq(const AttnCall c)
{
    using M = Mma<T>;
    using E = typename M::Elem;
    using Frag = typename M::Frag;
    using TL = Tile<T, DP>;
    using D = Dma<T, DP, KT, 64 * WAVES>;
    constexpr bool ALN = LOAD != kAny, kPair = std::is_same<T, Pair>::value, kDirect = kPair || LOAD == kDma;
    constexpr int NT = 64 * WAVES, NS = DP / M::kStep, NB = KT / 32, NF = 32 / M::kStep, ND = DP / 32;
    constexpr int kTile = D::kTile, NPC = D::kCount;
    constexpr bool kDiff = BIAS || sizeof(E) == 4;
    static_assert(KT * TL::kPieces % NT == 0 && 32 * WAVES == kRowBlock, "");
    __shared__ __align__(16) char lds[4 * kTile];
    __shared__ __align__(16) float lbias[2][BIAS ? KT : 1];

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5;
    const int rows = c.n * c.group, blocks = (rows + 32 * WAVES - 1) / (32 * WAVES);
    const Work w = work_of(blockIdx.x, gridDim.x, c.splits, blocks, c.kv_heads, c.causal, c.batch > 1 && (c.k_len || c.q_len));
    const int split = w.split, blk = blocks - 1 - w.rank, hk = w.hk, b = w.b;

    const int k_len = c.k_len ? min(max(c.k_len[b], 0), c.m) : c.m;
    const int q_len = c.q_len ? min(max(c.q_len[b], 0), c.n) : c.n;
    const int r = blk * 32 * WAVES + wave * 32 + (lane & 31);
    const Packed pk = unpack(r, c.group);
    const bool live = r < rows && pk.q < q_len;
    const int limit = !live ? 0 : c.causal ? min(k_len, max(0, pk.q + k_len - q_len + 1)) : k_len;
    const int last_q = min((min(rows, (blk + 1) * 32 * WAVES) - 1) / c.group, q_len - 1);
    const int hi = last_q < blk * 32 * WAVES / c.group ? 0 : c.causal ? min(k_len, max(0, last_q + k_len - q_len + 1)) : k_len;
    const int tiles = (hi + KT - 1) / KT, per = (tiles + c.splits - 1) / c.splits;
    const int t0 = min(tiles, split * per), t1 = min(tiles, t0 + per);
    // D = <do, o> has o's rounding to bf16 in it, which beside the gradients of a few keys is as large as a rounding of their own.  Rows of
    // at most 128 keys take D from its definition, sum_j p_ij <do_i, v_j>, in a sweep ahead (of all of a row's keys, in every split);
    // further keys shrink o, and with it the error, beside the v_j.
    constexpr bool kExact = std::is_same<T, __bf16>::value;
    const bool few = tiles * KT <= 128;
    int first = kExact && few ? 0 : t0;
    const int last = kExact && few ? tiles : t1;

    const E *kp = (const E *)c.k + b * c.sk.batch + hk * c.sk.head;
    const E *vp = (const E *)c.v + b * c.sv.batch + hk * c.sv.head;
    const int64_t bh = (int64_t)b * c.kv_heads + hk;
    PairGrad pg;
    if constexpr (kPair) pg = pair_grad(c, bh);
    float own = 1.0f;   // pairs: the power of two of the row's gradients of scores, in units of the pieces
    const float scale = kPair ? pair_scale(c, bh).score : c.scale;
    const float *bp = BIAS ? c.bias + b * c.bias_ld : nullptr;
    const LdsPtr base = (LdsPtr)lds;

    // (tiles of keys as in k_attn)
    unsigned ko[D::kOffsets], vo[D::kOffsets];
    uint4 kr[kDirect ? 1 : NPC], vr[kDirect ? 1 : NPC];
    float br = 0.0f;
    if constexpr (!kPair && LOAD == kDma) {
#pragma unroll
        for (int i = 0; i < D::kOffsets; ++i) {
            ko[i] = (unsigned)(D::row(tid, i) * (int)c.sk.row * (int)sizeof(E) + D::piece(tid, i) * 16);
            vo[i] = (unsigned)(D::row(tid, i) * (int)c.sv.row * (int)sizeof(E) + D::piece(tid, i) * 16);
        }
        if (first < last) D::clear(lds, tid, c.d, k_len - (last - 1) * KT, last - first);
    }
    auto fetch = [&](int tile, int buf) {
        if constexpr (kPair) {
            const int64_t at = (bh * pair_rows(c.m) + (int64_t)tile * KT) * TL::kRow;
            const unsigned to = lds_address(base) + 2 * buf * kTile;
            DmaImage<DP, KT, NT>::load(c.pair.img[kPairK] + at, to, tid);
            DmaImage<DP, KT, NT>::load(c.pair.img[kPairV] + at, to + kTile, tid);
        } else if constexpr (LOAD == kDma) {
            const char *kb = (const char *)(kp + (int64_t)tile * KT * c.sk.row), *vb = (const char *)(vp + (int64_t)tile * KT * c.sv.row);
            const unsigned to = lds_address(base) + 2 * buf * kTile;
            D::load(kb, ko, D::kRound * c.sk.row * (int)sizeof(E), to, tid, c.d, k_len - tile * KT);
            D::load(vb, vo, D::kRound * c.sv.row * (int)sizeof(E), to + kTile, tid, c.d, k_len - tile * KT);
        } else {
#pragma unroll
            for (int i = 0; i < NPC; ++i) {
                const int p = tid + i * NT, pc = p % TL::kPieces, key = tile * KT + p / TL::kPieces, at = min(key, k_len - 1);
                kr[i] = load_piece<E, ALN>(kp + (int64_t)at * c.sk.row, pc, c.d);
                vr[i] = load_piece<E, ALN>(vp + (int64_t)at * c.sv.row, pc, c.d);
                if (BIAS && bp[at] == -INFINITY) kr[i] = vr[i] = make_uint4(0, 0, 0, 0);
            }
        }
        if (BIAS && tid < KT) br = bp[min(tile * KT + tid, k_len - 1)];
    };
    auto put = [&](int buf) {
        if constexpr (!kDirect) {
#pragma unroll
            for (int i = 0; i < NPC; ++i) {
                const int p = tid + i * NT, at = TL::at(p / TL::kPieces, p % TL::kPieces);
                *(uint4 *)(lds + (2 * buf) * kTile + at) = kr[i];
                *(uint4 *)(lds + (2 * buf + 1) * kTile + at) = vr[i];
            }
        }
        if (BIAS && tid < KT) lbias[buf][tid] = br;
    };

    if (first < last) fetch(first, 0);
    Frag q[NS], g[NS];
    const int head = hk * c.group + pk.g;
    float delta = 0.0f;
    f32x4 own_row;   // pairs: see PairImage
    {
        if constexpr (kPair) {
            const int64_t at = bh * pair_rows(rows);
#pragma unroll
            for (int t = 0; t < NS; ++t) {
                q[t] = TL::from_image(c.pair.img[kPairQ] + at * TL::kRow, r, t, half);
                g[t] = TL::from_image(c.pair.img[kPairDo] + at * TL::kRow, r, t, half);
            }
            own_row = c.pair.row[at + r];
        } else {
            const E *rq = (const E *)c.q + b * c.sq.batch + (int64_t)pk.q * c.sq.row + head * c.sq.head;
            const E *rg = (const E *)c.d_o + b * c.s_do.batch + (int64_t)pk.q * c.s_do.row + head * c.s_do.head;
            const E *ro = (const E *)c.o + b * c.so.batch + (int64_t)pk.q * c.so.row + head * c.so.head;
            const uint4 z = make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int t = 0; t < NS; ++t) {
                q[t] = __builtin_bit_cast(Frag, live ? load_piece<E, ALN>(rq, 2 * t + half, c.d) : z);
                g[t] = __builtin_bit_cast(Frag, live ? load_piece<E, ALN>(rg, 2 * t + half, c.d) : z);
                const auto ot = __builtin_bit_cast(Frag, live ? load_piece<E, ALN>(ro, 2 * t + half, c.d) : z);
#pragma unroll
                for (int j = 0; j < M::kPiece; ++j) delta = fmaf((float)g[t][j], (float)ot[j], delta);
            }
        }
    }
    delta = kPair ? own_row[1] * pg.scale_v * 0x1p15f : across_halves_sum(delta);
    RowStat st = {0.0f, INFINITY};
    if (live) {
        const float2 v = *(const float2 *)(c.stat + 2 * ((bh * c.group + pk.g) * c.n + pk.q));
        st = row_stat<kDiff>(v.x, v.y);
        if constexpr (kPair) own = pair_power(2.0f * own_row[2] * pg.top * __builtin_amdgcn_rcpf(v.y), 13);
    }
    const float unit = kDiff ? kLog2eF : scale * kLog2eF;
    const typename TL::Lanes ln = TL::lanes(lane);

    constexpr bool kRemoved = BIAS && !kPair && LOAD == kDma;
    auto removed = [&](int buf) {
        if constexpr (kRemoved) clear_removed<T, DP, KT, NT>(lds + 2 * buf * kTile, lds + (2 * buf + 1) * kTile, lbias[buf], tid);
    };
    // what a row's keys of half a tile add to its gradient
    auto terms = [&](int tile, int buf, int nb, bool masked, f32x16 &s) {
        const LdsPtr lk = base + 2 * buf * kTile, lv = lk + kTile;
        f32x16 dp = (f32x16)(0.0f);
        s = (f32x16)(0.0f);
#pragma unroll
        for (int t = 0; t < NS; ++t) {
            s = M::mma(TL::rows(lk, ln, nb * 32, t), q[t], s);
            dp = M::mma(TL::rows(lv, ln, nb * 32, t), g[t], dp);
        }
        if constexpr (BIAS) {
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const f32x4 add = *(const f32x4 *)&lbias[buf][nb * 32 + 8 * u + 4 * half];
#pragma unroll
                for (int j = 0; j < 4; ++j) s[4 * u + j] = fmaf(s[4 * u + j], scale, add[j]);
            }
        }
        if (masked) {
            const int base = tile * KT + nb * 32 + 4 * half;
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = base + 8 * (i / 4) + i % 4 < limit ? s[i] : -INFINITY;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            // (without bias m is taken off in the same fma that scales)
            const float d = BIAS ? s[i] - st.m : kDiff ? fmaf(s[i], scale, -st.m) : s[i];
            const float p = __builtin_amdgcn_exp2f(fmaf(d, unit, -st.off));
            s[i] = p * (kPair ? fmaf(dp[i], own, -delta) : dp[i] - delta);
        }
    };
    auto begin = [&](int to) {
        if (first < to) put(0);
        dma_wait();
        __builtin_amdgcn_s_waitcnt(0x0f70);
        __syncthreads();
        if (kRemoved && first < to) removed(0);
    };
    auto next = [&](int tile, int buf, int to) {
        if ((!kDirect || BIAS) && tile + 1 < to) put(buf ^ 1);
        if (kDirect) dma_wait();
        __syncthreads();
        if (kRemoved && tile + 1 < to) removed(buf ^ 1);
    };
    begin(last);
    if (kExact && few) {
        float sum = 0.0f;
        delta = 0.0f;
        for (int tile = first; tile < last; ++tile) {
            const int buf = (tile - first) & 1;
            if (tile + 1 < last) fetch(tile + 1, buf ^ 1);
            const bool masked = __any(limit < (tile + 1) * KT);
            for (int nb = 0; nb < NB; ++nb) {
                f32x16 s;
                terms(tile, buf, nb, masked, s);
#pragma unroll
                for (int i = 0; i < 16; ++i) sum += s[i];
            }
            next(tile, buf, last);
        }
        delta = across_halves_sum(sum);
        first = t0;
        if (t0 < t1) fetch(t0, 0);
        begin(t1);
    }
    if (split == 0 && half == 0) {   // for the other pass, whole blocks of rows
        const int64_t pad = (int64_t)blocks * 32 * WAVES;
        float *out = c.row_stat + 3 * bh * pad + r;
        if constexpr (kPair) {   // (probabilities times kPairN = 2^15 and the share of the row's do)
            out[0] = st.off + (float)(pair_exponent(own_row[0]) - pg.g - 15);
            out[pad] = delta * pg.dov;
        } else {
            out[0] = st.off;
            out[pad] = delta;
        }
        if (kDiff) out[2 * pad] = st.m;
    }
    if (kPair) delta *= own;
    f32x16 dq[ND];
#pragma unroll
    for (int i = 0; i < ND; ++i) dq[i] = (f32x16)(0.0f);
    for (int tile = t0; tile < t1; ++tile) {
        const int buf = (tile - t0) & 1;
        const LdsPtr lk = base + 2 * buf * kTile;
        if (tile + 1 < t1) fetch(tile + 1, buf ^ 1);
        const bool masked = __any(limit < (tile + 1) * KT);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            f32x16 s;
            terms(tile, buf, nb, masked, s);
#pragma unroll
            for (int t = 0; t < NF; ++t) {
                const Frag ds = M::pack(s, t);
#pragma unroll
                for (int i = 0; i < ND; ++i) dq[i] = M::mma(TL::cols(lk, ln, nb * 32, t, i, lane), ds, dq[i]);
                if constexpr (FINE) {
                    const Frag rest = M::rest(s, t);
#pragma unroll
                    for (int i = 0; i < ND; ++i) dq[i] = M::mma(TL::cols(lk, ln, nb * 32, t, i, lane), rest, dq[i]);
                }
            }
        }
        next(tile, buf, t1);
    }
    if (r >= rows) return;
    if constexpr (kPair) {
        const PairFactor f = pair_factor(c.scale, -(pair_exponent(own) + pair_exponent(own_row[0]) + pg.v + pair_exponent(c.pair.scale[8 * bh + kPairK])));
#pragma unroll
        for (int i = 0; i < ND; ++i) dq[i] = dq[i] * f.a * f.b;
    }
    if (c.splits > 1) {
        float *po = c.part + ((int64_t)split * c.batch * c.kv_heads * rows + bh * rows + r) * DP + 4 * half;
#pragma unroll
        for (int i = 0; i < ND; ++i)
#pragma unroll
            for (int u = 0; u < 4; ++u)
                *(f32x4 *)(po + 32 * i + 8 * u) = f32x4{dq[i][4 * u], dq[i][4 * u + 1], dq[i][4 * u + 2], dq[i][4 * u + 3]};
        return;
    }
    E *out = (E *)c.dq + b * c.sdq.batch + (int64_t)pk.q * c.sdq.row + head * c.sdq.head;
#pragma unroll
    for (int i = 0; i < ND; ++i) store_column<E, ALN>(out, dq[i], kPair ? 1.0f : c.scale, 32 * i + 4 * half, c.d);
}

// Keys in registers, rows streamed: S = Q K^T and dP = dO V^T end as a key's p and ds in the order dV^T += dO^T P and dK^T += Q^T dS take
// them.  Four products a score; bound as k_attn_dq: 603 us, 910 TFLOP/s, and 50 us, 690 TFLOP/s, at the sizes there.  The products come one
// after the other (d = 128 spills otherwise).
template <typename T, int DP, int RT, int WAVES, bool BIAS, Load LOAD, bool FINE>
__global__ __launch_bounds__(64 * WAVES, FINE && DP > 96 ? 1 : dkv_waves<T>(DP)) void k_attn_dkv(const AttnCall c)
{
    using M = Mma<T>;
    using E = typename M::Elem;
    using Frag = typename M::Frag;
    using TL = Tile<T, DP>;
    using D = Dma<T, DP, RT, 64 * WAVES>;
    constexpr bool ALN = LOAD != kAny, kPair = std::is_same<T, Pair>::value, kDirect = kPair || LOAD == kDma;
    constexpr int NT = 64 * WAVES, NS = DP / M::kStep, NB = RT / 32, NF = 32 / M::kStep, ND = DP / 32;
    constexpr int kTile = D::kTile, NPC = D::kCount;
    constexpr bool kDiff = BIAS || sizeof(E) == 4;
    constexpr int kStats = kDiff ? 3 : 2;
    static_assert(RT * TL::kPieces % NT == 0 && RT <= 64, "");
    __shared__ __align__(16) char lds[4 * kTile];
    __shared__ __align__(16) float lstat[2][kStats][RT];   // off, D, m

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5;
    const int rows = c.n * c.group, blocks = (c.m + 32 * WAVES - 1) / (32 * WAVES);
    const Work w = work_of(blockIdx.x, gridDim.x, c.splits, blocks, c.kv_heads, c.causal, c.batch > 1 && (c.k_len || c.q_len));
    const int split = w.split, blk = w.rank, hk = w.hk, b = w.b;
    const int64_t bh = (int64_t)b * c.kv_heads + hk;

    const int k_len = c.k_len ? min(max(c.k_len[b], 0), c.m) : c.m;
    const int q_len = c.q_len ? min(max(c.q_len[b], 0), c.n) : c.n;
    const int key0 = blk * 32 * WAVES, key = key0 + wave * 32 + (lane & 31);
    const float bias = BIAS && key < k_len ? c.bias[b * c.bias_ld + key] : 0.0f;
    const bool live = key < k_len && (!BIAS || bias != -INFINITY);
    // rows that see a key of this block
    const int first = c.causal ? min(q_len, max(0, key0 - (k_len - q_len))) : 0;
    const int begin = first * c.group / RT, end = key0 < k_len ? (q_len * c.group + RT - 1) / RT : begin;
    const int tiles = max(0, end - begin), per = (tiles + c.splits - 1) / c.splits;
    const int t0 = begin + min(tiles, split * per), t1 = min(begin + tiles, t0 + per);
    // the first packed row that sees this lane's key
    const int sees = c.causal ? max(0, key - k_len + q_len) * c.group : 0;

    const E *qp = (const E *)c.q + b * c.sq.batch + (int64_t)hk * c.group * c.sq.head;
    const E *gp = (const E *)c.d_o + b * c.s_do.batch + (int64_t)hk * c.group * c.s_do.head;
    PairGrad pg;
    if constexpr (kPair) pg = pair_grad(c, bh);
    const float scale = kPair ? pair_scale(c, bh).score : c.scale;
    const int64_t pad = round_up_rows(rows);
    const float *sp = c.row_stat + 3 * bh * pad;
    const LdsPtr base = (LdsPtr)lds;

    unsigned qo[D::kOffsets], go[D::kOffsets];
    uint4 qr[kDirect ? 1 : NPC], gr[kDirect ? 1 : NPC];
    float sr[kStats];
    auto offset = [&](int row, const HeadsAt &at, int piece) {   // of a row within its tile, which begins with a whole query
        const Packed pk = unpack(row, c.group);
        return (unsigned)((pk.q * (int)at.row + pk.g * (int)at.head) * (int)sizeof(E) + piece * 16);
    };
    if constexpr (!kPair && LOAD == kDma) {
#pragma unroll
        for (int i = 0; i < D::kOffsets; ++i) {
            qo[i] = offset(D::row(tid, i), c.sq, D::piece(tid, i));
            go[i] = offset(D::row(tid, i), c.s_do, D::piece(tid, i));
        }
        if (t0 < t1) D::clear(lds, tid, c.d, q_len * c.group - (t1 - 1) * RT, t1 - t0);
    }
    auto fetch = [&](int tile, int buf) {
        if constexpr (kPair) {
            const int64_t at = (bh * pair_rows(rows) + (int64_t)tile * RT) * TL::kRow;
            const unsigned to = lds_address(base) + 2 * buf * kTile;
            DmaImage<DP, RT, NT>::load(c.pair.img[kPairQ] + at, to, tid);
            DmaImage<DP, RT, NT>::load(c.pair.img[kPairDo] + at, to + kTile, tid);
        } else if constexpr (LOAD == kDma) {
            const int64_t q0 = tile * RT / c.group;
            const char *qb = (const char *)(qp + q0 * c.sq.row), *gb = (const char *)(gp + q0 * c.s_do.row);
            const unsigned to = lds_address(base) + 2 * buf * kTile;
            const int queries = D::kRound / c.group, left = q_len * c.group - tile * RT;   // (a round is whole queries: see launch_attn_grad)
            D::load(qb, qo, queries * c.sq.row * (int)sizeof(E), to, tid, c.d, left);
            D::load(gb, go, queries * c.s_do.row * (int)sizeof(E), to + kTile, tid, c.d, left);
        } else {
#pragma unroll
            for (int i = 0; i < NPC; ++i) {
                const int p = tid + i * NT, pc = p % TL::kPieces;
                const Packed pk = unpack(min(tile * RT + p / TL::kPieces, q_len * c.group - 1), c.group);
                qr[i] = load_piece<E, ALN>(qp + (int64_t)pk.q * c.sq.row + pk.g * c.sq.head, pc, c.d);
                gr[i] = load_piece<E, ALN>(gp + (int64_t)pk.q * c.s_do.row + pk.g * c.s_do.head, pc, c.d);
            }
            if (tid < RT)
#pragma unroll
                for (int k = 0; k < kStats; ++k) sr[k] = sp[k * pad + tile * RT + tid];
        }
        if constexpr (kDirect) {
            if (__builtin_amdgcn_readfirstlane(wave) == 0 && lane < RT) {
                const unsigned at = __builtin_amdgcn_readfirstlane(lds_address((LdsPtr)(const char *)&lstat[buf][0][0]));
#pragma unroll
                for (int k = 0; k < kStats; ++k) dma4s(sp + k * pad + (int64_t)tile * RT, 4 * lane, at + k * RT * 4);
            }
        }
    };
    auto put = [&](int buf) {
        if constexpr (!kDirect) {
#pragma unroll
            for (int i = 0; i < NPC; ++i) {
                const int p = tid + i * NT, at = TL::at(p / TL::kPieces, p % TL::kPieces);
                *(uint4 *)(lds + (2 * buf) * kTile + at) = qr[i];
                *(uint4 *)(lds + (2 * buf + 1) * kTile + at) = gr[i];
            }
            if (tid < RT)
#pragma unroll
                for (int k = 0; k < kStats; ++k) lstat[buf][k][tid] = sr[k];
        }
    };

    if (t0 < t1) fetch(t0, 0);
    Frag k[NS], v[NS];
    if constexpr (kPair) {
        const int64_t at = bh * pair_rows(c.m) * TL::kRow;
#pragma unroll
        for (int t = 0; t < NS; ++t) {
            k[t] = TL::from_image(c.pair.img[kPairK] + at, key, t, half);
            v[t] = TL::from_image(c.pair.img[kPairV] + at, key, t, half);
        }
    } else {
        const E *rk = (const E *)c.k + b * c.sk.batch + (int64_t)key * c.sk.row + hk * c.sk.head;
        const E *rv = (const E *)c.v + b * c.sv.batch + (int64_t)key * c.sv.row + hk * c.sv.head;
#pragma unroll
        for (int t = 0; t < NS; ++t) {
            const uint4 z = make_uint4(0, 0, 0, 0);
            k[t] = __builtin_bit_cast(Frag, live ? load_piece<E, ALN>(rk, 2 * t + half, c.d) : z);
            v[t] = __builtin_bit_cast(Frag, live ? load_piece<E, ALN>(rv, 2 * t + half, c.d) : z);
        }
    }
    const float unit = kDiff ? kLog2eF : scale * kLog2eF;
    const typename TL::Lanes ln = TL::lanes(lane);

    f32x16 dk[ND], dv[ND];
    float db = 0.0f;
#pragma unroll
    for (int i = 0; i < ND; ++i) dk[i] = dv[i] = (f32x16)(0.0f);
    if (t0 < t1) put(0);
    dma_wait();
    __builtin_amdgcn_s_waitcnt(0x0f70);
    __syncthreads();
    for (int tile = t0; tile < t1; ++tile) {
        const int buf = (tile - t0) & 1;
        const LdsPtr lq = base + 2 * buf * kTile, lg = lq + kTile;
        if (tile + 1 < t1) fetch(tile + 1, buf ^ 1);
        const bool masked = __any(tile * RT < sees);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            // one after the other: 192 registers of keys, values and accumulators at d = 128 leave room for two of the three products
            // that a block is made of
            f32x16 s = (f32x16)(0.0f), dp = (f32x16)(0.0f);
#pragma unroll
            for (int t = 0; t < NS; ++t) s = M::mma(TL::rows(lq, ln, nb * 32, t), k[t], s);
            if constexpr (BIAS) {
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] = fmaf(s[i], scale, bias);
            }
            if (masked) {
                const int base = tile * RT + nb * 32 + 4 * half;
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] = base + 8 * (i / 4) + i % 4 >= sees ? s[i] : -INFINITY;
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int at = nb * 32 + 8 * u + 4 * half;
                const f32x4 off = *(const f32x4 *)&lstat[buf][0][at];
                f32x4 m;
                if (kDiff) m = *(const f32x4 *)&lstat[buf][kStats - 1][at];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int i = 4 * u + j;
                    const float d = BIAS ? s[i] - m[j] : kDiff ? fmaf(s[i], scale, -m[j]) : s[i];
                    s[i] = __builtin_amdgcn_exp2f(fmaf(d, unit, -off[j]));
                }
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < NF; ++t) {
                const Frag pf = M::pack(s, t);
#pragma unroll
                for (int i = 0; i < ND; ++i) dv[i] = M::mma(TL::cols(lg, ln, nb * 32, t, i, lane), pf, dv[i]);
                if constexpr (FINE) {
                    const Frag rest = M::rest(s, t);
#pragma unroll
                    for (int i = 0; i < ND; ++i) dv[i] = M::mma(TL::cols(lg, ln, nb * 32, t, i, lane), rest, dv[i]);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < NS; ++t) dp = M::mma(TL::rows(lg, ln, nb * 32, t), v[t], dp);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const f32x4 dl = *(const f32x4 *)&lstat[buf][1][nb * 32 + 8 * u + 4 * half];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int i = 4 * u + j;
                    s[i] *= kPair ? fmaf(dp[i], pg.dov, -dl[j]) : dp[i] - dl[j];
                    if (BIAS) db += s[i];
                }
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < NF; ++t) {
                const Frag sf = M::pack(s, t);
#pragma unroll
                for (int i = 0; i < ND; ++i) dk[i] = M::mma(TL::cols(lq, ln, nb * 32, t, i, lane), sf, dk[i]);
                if constexpr (FINE) {
                    const Frag rest = M::rest(s, t);
#pragma unroll
                    for (int i = 0; i < ND; ++i) dk[i] = M::mma(TL::cols(lq, ln, nb * 32, t, i, lane), rest, dk[i]);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if (!kDirect && tile + 1 < t1) put(buf ^ 1);
        if (kDirect) dma_wait();
        __syncthreads();
    }
    if (BIAS) db = across_halves_sum(db);
    if (key >= c.m) return;
    if (!live) {   // (what its column computed came from zeros, and may be anything)
#pragma unroll
        for (int i = 0; i < ND; ++i) dk[i] = dv[i] = (f32x16)(0.0f);
        db = 0.0f;
    }
    if constexpr (kPair) {
        const PairFactor f = pair_factor(c.scale, -(pg.ds + pair_exponent(c.pair.scale[8 * bh + kPairQ]))), fb = pair_factor(1.0f, -pg.ds),
                         fv = pair_factor(1.0f, -15 - pg.g);
#pragma unroll
        for (int i = 0; i < ND; ++i) {
            dk[i] = dk[i] * f.a * f.b;
            dv[i] = dv[i] * fv.a * fv.b;
        }
        db = db * fb.a * fb.b;
    }
    const int64_t slot = ((int64_t)split * c.batch * c.kv_heads + bh) * c.m + key;
    if (BIAS && c.dbias && half == 0) c.dbias_part[slot] = db;
    if (c.splits > 1) {
        float *po = c.part + slot * 2 * DP + 4 * half;
#pragma unroll
        for (int i = 0; i < ND; ++i)
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                *(f32x4 *)(po + 32 * i + 8 * u) = f32x4{dk[i][4 * u], dk[i][4 * u + 1], dk[i][4 * u + 2], dk[i][4 * u + 3]};
                *(f32x4 *)(po + DP + 32 * i + 8 * u) = f32x4{dv[i][4 * u], dv[i][4 * u + 1], dv[i][4 * u + 2], dv[i][4 * u + 3]};
            }
        return;
    }
    E *ok = (E *)c.dk + b * c.sdk.batch + (int64_t)key * c.sdk.row + hk * c.sdk.head;
    E *ov = (E *)c.dv + b * c.sdv.batch + (int64_t)key * c.sdv.row + hk * c.sdv.head;
#pragma unroll
    for (int i = 0; i < ND; ++i) {
        store_column<E, ALN>(ok, dk[i], kPair ? 1.0f : c.scale, 32 * i + 4 * half, c.d);
        store_column<E, ALN>(ov, dv[i], 1.0f, 32 * i + 4 * half, c.d);
    }
}

// Sums over the splits, in an order that does not depend on anything else: of dq, or (KV) of dk and dv; dq and dk times the call's scale
// (SCALED: they have it already).  A thread takes four coordinates of a
// row and every G-th split, four splits' loads at a time; G groups of threads share a row and meet in LDS.
template <typename T, int DP, bool KV, bool SCALED, int G>
__global__ __launch_bounds__(256) void k_attn_grad_join(const AttnCall c)
{
    constexpr int W = DP / 4, R = 256 / (W * G);
    __shared__ f32x4 lacc[G > 1 ? 256 : 1];
    const int t = threadIdx.x, x = t % W, g = t / W % G, rows = KV ? c.m : c.n * c.group;
    // (dk and dv of a key are two rows)
    const int64_t total = (int64_t)c.batch * c.kv_heads * rows * (KV ? 2 : 1), at = (int64_t)blockIdx.x * R + t / (W * G);
    const bool there = t < W * G * R && at < total;
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    if (there)
        for (int s0 = g; s0 < c.splits; s0 += 4 * G) {
            f32x4 v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = *(const f32x4 *)(c.part + (min(s0 + k * G, c.splits - 1) * total + at) * DP + 4 * x);
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (s0 + k * G < c.splits) acc += v[k];
        }
    if constexpr (G > 1) {
        lacc[t] = acc;
        __syncthreads();
        if (g != 0) return;
        for (int k = 1; k < G; ++k) acc += lacc[t + k * W];
    }
    if (!there) return;
    const int64_t row = KV ? at / 2 : at, bh = row / rows;
    const int hk = (int)(bh % c.kv_heads), b = (int)(bh / c.kv_heads), r = (int)(row - bh * rows);
    T *out;
    float f = SCALED ? 1.0f : c.scale;
    if constexpr (KV) {
        if (at % 2 == 0) {
            out = (T *)c.dk + b * c.sdk.batch + (int64_t)r * c.sdk.row + hk * c.sdk.head;
        } else {
            out = (T *)c.dv + b * c.sdv.batch + (int64_t)r * c.sdv.row + hk * c.sdv.head;
            f = 1.0f;
        }
    } else {
        const Packed pk = unpack(r, c.group);
        out = (T *)c.dq + b * c.sdq.batch + (int64_t)pk.q * c.sdq.row + (hk * c.group + pk.g) * c.sdq.head;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (4 * x + j < c.d) out[4 * x + j] = (T)(acc[j] * f);
}

template <typename T, int DP, bool KV, bool SCALED> void join(Ctx *c, const AttnCall &a)
{
    const int64_t total = (int64_t)a.batch * a.kv_heads * (KV ? 2 * (int64_t)a.m : (int64_t)a.n * a.group);
    constexpr int W = DP / 4;
    if (a.splits > 16) k_attn_grad_join<T, DP, KV, SCALED, 8><<<(unsigned)ceil_div(total, 256 / (8 * W)), 256, 0, c->stream>>>(a);
    else if (a.splits > 8) k_attn_grad_join<T, DP, KV, SCALED, 4><<<(unsigned)ceil_div(total, 256 / (4 * W)), 256, 0, c->stream>>>(a);
    else k_attn_grad_join<T, DP, KV, SCALED, 1><<<(unsigned)ceil_div(total, 256 / W), 256, 0, c->stream>>>(a);
}

// Sum over the splits and heads that share a bias: sixteen lanes take a key each, sixteen shares side by side.
template <typename T> __global__ __launch_bounds__(256) void k_attn_dbias(const AttnCall c)
{
    __shared__ float lds[16][17];
    const int x = threadIdx.x % 16, g = threadIdx.x / 16, b = blockIdx.y, key = blockIdx.x * 16 + x;
    float acc = 0.0f;
    if (key < c.m)
#pragma unroll 4
        for (int i = g; i < c.splits * c.kv_heads; i += 16) {
            const int s = i / c.kv_heads, h = i - s * c.kv_heads;
            acc += c.dbias_part[(((int64_t)s * c.batch + b) * c.kv_heads + h) * c.m + key];
        }
    lds[g][x] = acc;
    __syncthreads();
    if (g == 0 && key < c.m) {
        for (int i = 1; i < 16; ++i) acc += lds[i][x];
        ((T *)c.dbias)[b * c.dbias_ld + key] = (T)acc;
    }
}

template <typename T, int DP, bool FINE> void dq_pass(Ctx *c, const AttnCall &a, unsigned grid, Load load)
{
    constexpr int N = row_tile<T>(DP);
    constexpr Load kBest = std::is_same<T, Pair>::value ? kVec : kDma;   // (of pairs only their images are direct)
    if (a.bias) {
        if (load == kDma) k_attn_dq<T, DP, N, 4, true, kBest, FINE><<<grid, 256, 0, c->stream>>>(a);
        else if (load == kVec) k_attn_dq<T, DP, N, 4, true, kVec, FINE><<<grid, 256, 0, c->stream>>>(a);
        else k_attn_dq<T, DP, N, 4, true, kAny, FINE><<<grid, 256, 0, c->stream>>>(a);
    } else {
        if (load == kDma) k_attn_dq<T, DP, N, 4, false, kBest, FINE><<<grid, 256, 0, c->stream>>>(a);
        else if (load == kVec) k_attn_dq<T, DP, N, 4, false, kVec, FINE><<<grid, 256, 0, c->stream>>>(a);
        else k_attn_dq<T, DP, N, 4, false, kAny, FINE><<<grid, 256, 0, c->stream>>>(a);
    }
}
template <typename T, int DP, bool FINE> void dkv_pass(Ctx *c, const AttnCall &a, unsigned grid, Load load)
{
    // (32 rows are one tile, where that is a whole number of the threads' loads)
    constexpr int N = FINE && DP % 64 == 0 ? 32 : row_tile<T>(DP);
    constexpr Load kBest = std::is_same<T, Pair>::value ? kVec : kDma;   // (of pairs only their images are direct)
    if (a.bias) {
        if (load == kDma) k_attn_dkv<T, DP, N, 4, true, kBest, FINE><<<grid, 256, 0, c->stream>>>(a);
        else if (load == kVec) k_attn_dkv<T, DP, N, 4, true, kVec, FINE><<<grid, 256, 0, c->stream>>>(a);
        else k_attn_dkv<T, DP, N, 4, true, kAny, FINE><<<grid, 256, 0, c->stream>>>(a);
    } else {
        if (load == kDma) k_attn_dkv<T, DP, N, 4, false, kBest, FINE><<<grid, 256, 0, c->stream>>>(a);
        else if (load == kVec) k_attn_dkv<T, DP, N, 4, false, kVec, FINE><<<grid, 256, 0, c->stream>>>(a);
        else k_attn_dkv<T, DP, N, 4, false, kAny, FINE><<<grid, 256, 0, c->stream>>>(a);
    }
}

template <typename T, int DP>
fs_status run(Ctx *c, AttnCall a, const AttnGradPlan &p, char *ws, Load keys, Load rows_load)
{
    using E = typename Mma<T>::Elem;
    // p and ds as two bf16 where a head of keys has at most 32 rows: what is left of the error is the outputs' own rounding, 1.7e-3 of
    // their norm; with one it is 2.4e-3, for any number of rows.  The line is drawn by what it costs.  Up to 32 rows, one tile, the pass
    // is bound by its keys: one row, 153 keys, 16 heads over 4, d = 32 19 us both, 32 rows, 2000 keys, four sets, 8 heads of 128 39 us with
    // one piece and 44 with two.  Beyond, the products bind: 64 rows there 42 and 51, 128 rows 52 and 62; 8 sets of 1024, 8 heads of 64,
    // 81 and 106; 4096 points, 8 heads of 128, 270 and 390.
    constexpr bool kBf16 = std::is_same<T, __bf16>::value, kPairs = std::is_same<T, Pair>::value;
    const bool fine = kBf16 && (int64_t)a.n * a.group <= 32;
    Arena A;
    a.row_stat = (float *)(ws + A.take(p.stat_bytes));
    float *dq_part = (float *)(ws + A.take(p.dq_bytes)), *dkv_part = (float *)(ws + A.take(p.dkv_bytes));
    a.dbias_part = (float *)(ws + A.take(p.dbias_bytes));
    a.splits = p.q_splits;
    a.part = dq_part;
    if (p.q_grid) {
        if (fine) dq_pass<T, DP, kBf16>(c, a, (unsigned)p.q_grid, keys);
        else dq_pass<T, DP, false>(c, a, (unsigned)p.q_grid, keys);
        if (a.splits > 1) join<E, DP, false, kPairs>(c, a);
    }
    a.splits = p.k_splits;
    a.part = dkv_part;
    if (p.k_grid) {
        if (fine) dkv_pass<T, DP, kBf16>(c, a, (unsigned)p.k_grid, rows_load);
        else dkv_pass<T, DP, false>(c, a, (unsigned)p.k_grid, rows_load);
        if (a.splits > 1) join<E, DP, true, kPairs>(c, a);
        if (a.dbias) k_attn_dbias<E><<<dim3((unsigned)ceil_div(a.m, 16), (unsigned)a.batch), 256, 0, c->stream>>>(a);
    }
    FS_HIP(c, hipGetLastError());
    return FS_OK;
}

template <typename T> fs_status by_width(Ctx *c, const AttnCall &a, const AttnGradPlan &p, char *ws, Load keys, Load rows)
{
    switch ((a.d + 31) / 32) {
    case 1: return run<T, 32>(c, a, p, ws, keys, rows);
    case 2: return run<T, 64>(c, a, p, ws, keys, rows);
    case 3: return run<T, 96>(c, a, p, ws, keys, rows);
    default: return run<T, 128>(c, a, p, ws, keys, rows);
    }
}

}  // namespace

AttnGradPlan attn_grad_plan(const Ctx *c, const AttnCall &a, bool f32)
{
    AttnGradPlan p;
    const int64_t rows = (int64_t)a.n * a.group, heads = (int64_t)a.batch * a.kv_heads, dp = round_up(a.d, 32);
    const int64_t qb = ceil_div(rows, 128) * heads, kb = ceil_div(a.m, 128) * heads;
    p.pairs = f32 && pair_worth(c, a, true);
    const int tile = !f32 || (p.pairs && dp <= 64) ? 64 : 32;
    const int64_t kt = ceil_div(a.m, tile), rt = ceil_div(rows, tile);
    // Workgroups that fill the chip (two of them in a CU's registers, or one), in splits of at least four tiles, in float32, where a tile
    // takes longer beside the merge, two.  Backward with two, three and four, us (heads x rows x keys, d): bf16 4 x 1024 x 1024, 64: 37.2,
    // 36.1, 34.0; 8 x 600 x 900, 128: 55, 48, 52; 8 x 512 x 512 causal, 64: 29.3, 30.0, 31.5; float32 16 x 200 x 200, 64: 39, 45, 51;
    // 8 x 512 x 512, 64: 46, 49, 53; 12 x 1000 x 777, 40: 73, 74, 76.
    const int64_t want = (int64_t)c->num_cu * (f32 && dp > 64 ? 1 : 2), least = f32 ? 2 : 4;
    auto splits = [&](int64_t blocks, int64_t tiles, int64_t most) {
        const int64_t per = std::max<int64_t>(least, ceil_div(tiles, std::max<int64_t>(1, most / std::max<int64_t>(blocks, 1))));
        return (int)std::max<int64_t>(1, ceil_div(tiles, per));
    };
    p.q_splits = splits(qb, kt, want);
    // (blocks that do not fill the chip and are of unequal length, under a causal line, are cut twice as fine: short ones then fill up
    // behind long ones; 8192 points, 16 heads over 4, d = 128: 1008 us, and 1301 otherwise; where they do fill it splits cost 15 us)
    p.k_splits = kb >= want ? 1 : splits(kb, rt, (a.causal ? 2 : 1) * want);
    p.q_grid = qb * p.q_splits;
    p.k_grid = kb * p.k_splits;
    p.stat_bytes = (size_t)(heads * round_up(rows, kRowBlock)) * 12;
    p.dq_bytes = p.q_splits > 1 ? (size_t)(heads * rows * dp * p.q_splits) * 4 : 0;
    p.dkv_bytes = p.k_splits > 1 ? (size_t)(heads * a.m * dp * 2 * p.k_splits) * 4 : 0;
    p.pair_bytes = p.pairs ? pair_bytes(a, true) : 0;
    p.dbias_bytes = a.dbias ? (size_t)(heads * a.m * p.k_splits) * 4 : 0;
    return p;
}

fs_status launch_attn_grad(Ctx *c, AttnCall a, const AttnGradPlan &p, char *ws, bool f32, bool aligned)
{
    const int es = f32 ? 4 : 2;
    const int64_t kmost = std::max(a.sk.row, a.sv.row) * es * 64;
    const Load keys = !aligned ? kAny : kmost < (int64_t(1) << 31) ? kDma : kVec;
    // tiles of rows, and the rounds that load them, begin with a whole query
    const int rt = f32 ? 32 : 64, dp = (int)round_up(a.d, 32), round = dp == 96 ? rt : std::min(rt, 256 * 16 / dp / es);
    const int64_t rmost = (std::max(a.sq.row, a.s_do.row) * rt / a.group + std::max(a.sq.head, a.s_do.head) * a.group) * es;
    const Load rows = !aligned ? kAny : rt % a.group == 0 && round % a.group == 0 && rmost < (int64_t(1) << 31) ? kDma : kVec;
    if (p.pairs) {
        const fs_status st = launch_pairs(c, a, true, aligned);
        return st ? st : by_width<Pair>(c, a, p, ws, aligned ? kVec : kAny, aligned ? kVec : kAny);
    }
    return f32 ? by_width<float>(c, a, p, ws, keys, rows) : by_width<__bf16>(c, a, p, ws, keys, rows);
}

}  // namespace fs
