// Softmax attention, forward:  o_i = sum_j p_ij v_j,  p_ij = exp(s_ij - m_i) / l_i,  s_ij = scale <q_i, k_j> + bias_j,
// over the keys j that row i may see.  One pass over the keys with the running maximum and sum of every row; scores and
// probabilities stay in registers: a wave holds 32 rows as columns, S^T = K Q^T, and its registers are the operand of
// O^T += V^T P^T (fs_attn.h).
#include <algorithm>

#include "fs_attn.h"

namespace fs {
namespace {

constexpr float kLog2eF = 1.44269504088896340736f;
// Probabilities are taken below a reference: the row's maximum over the first tile in which it sees a key.  As long as no later score
// exceeds it by more than 2^kSlack, and that is the rule, nothing is ever rescaled: sums and accumulators are floats, which 2^30 leaves
// room enough, and a bf16 probability has the same relative rounding at any size.  A wave that meets a larger score goes on in a
// second loop, which follows the maximum and rescales in every tile.  (With the rescaling in a branch of one loop the compiler
// keeps two copies of the accumulators and moves them to and fro.)
constexpr float kSlack = 30.0f;
constexpr float kSlackPair = 11.0f;   // (kPairP times a probability is an fp16)

// keys of a tile where a workgroup has 64 rows: 32 or 64 for each of four parts, at most 128 KB of LDS
constexpr int few_keys(int dp) { return dp > 64 ? 128 : 256; }

// waves per SIMD: what registers allow without spills
template <typename T> constexpr int min_waves(int dp) { return std::is_same<T, float>::value && dp >= 96 ? 1 : 2; }

// What a row reports as its largest score: NaN where a score is NaN, which fmaxf leaves out (of infinite scores the sum alone is NaN).
__device__ inline float reported_max(float top, float sum) { return sum != sum && top < INFINITY ? sum : top; }

// Bound by the vector ALU at d = 64 (two operations and an exp2 a score beside 2 d products: 16384 points, 16 heads, bf16: 1.17 to 1.24 ms,
// 890 to 940 TFLOP/s, vector ALU busy 76 %, matrix cores 47 %), by LDS and the matrix cores towards d = 128 (1060 TFLOP/s; 8192 points
// under a causal line: 306 us, 900 TFLOP/s, busy 63 % and 42 %), by memory for one query (50021 keys, 4 sets, 8 heads of 128: 114 us,
// 5.9 TB/s).  S^T rather than S, since its registers are a row's probabilities in the order the next
// product takes them: they never pass through LDS.  32 rows a wave: two blocks of them a wave were slower (d = 64: 837 TFLOP/s and 843,
// d = 128: 782 and 992), for their registers.
// A workgroup has RW KS waves: wave w holds the w % RW-th 32 rows of the workgroup, and takes the w / RW-th part of every tile of KTS
// keys.  With KS > 1 the parts of a row meet in LDS at the end.
template <typename T, int DP, int KTS, int RW, int KS, bool BIAS, Load LOAD>
__global__ __launch_bounds__(64 * RW * KS, min_waves<T>(DP)) void k_attn(const AttnCall c)
{
    using M = Mma<T>;
    using E = typename M::Elem;
    using Frag = typename M::Frag;
    using TL = Tile<T, DP>;
    using D = Dma<T, DP, KTS, 64 * RW * KS>;
    constexpr bool ALN = LOAD != kAny, kPair = std::is_same<T, Pair>::value, kDirect = kPair || LOAD == kDma;
    constexpr int KT = KTS / KS, NT = 64 * RW * KS, NS = DP / M::kStep, NB = KT / 32, NF = 32 / M::kStep, ND = DP / 32;
    constexpr int kTile = D::kTile, NPC = D::kCount;
    static_assert(KTS * TL::kPieces % NT == 0 && (!kPair || RW == 4), "");
    static_assert((KS - 1) * RW * 64 * (16 * ND + 3) * 4 <= 4 * kTile, "");
    __shared__ __align__(16) char lds[4 * kTile];
    __shared__ __align__(16) float lbias[2][BIAS ? KTS : 1];

    const int tid = threadIdx.x, lane = tid & 63, wave = KS == 1 ? tid >> 6 : (tid >> 6) % RW, part_id = KS == 1 ? 0 : (tid >> 6) / RW,
              half = lane >> 5;
    const int rows = c.n * c.group, blocks = (rows + 32 * RW - 1) / (32 * RW);
    const Work w = work_of(blockIdx.x, gridDim.x, c.splits, blocks, c.kv_heads, c.causal, c.batch > 1 && (c.k_len || c.q_len));
    const int split = w.split, blk = blocks - 1 - w.rank, hk = w.hk, b = w.b;

    const int k_len = c.k_len ? min(max(c.k_len[b], 0), c.m) : c.m;
    const int q_len = c.q_len ? min(max(c.q_len[b], 0), c.n) : c.n;
    const int r = blk * 32 * RW + wave * 32 + (lane & 31);
    const Packed pk = unpack(r, c.group);
    const bool live = r < rows && pk.q < q_len;
    // keys that this row sees: 0 .. limit - 1
    const int limit = !live ? 0 : c.causal ? min(k_len, max(0, pk.q + k_len - q_len + 1)) : k_len;
    const int last_q = min((min(rows, (blk + 1) * 32 * RW) - 1) / c.group, q_len - 1);
    const int hi = last_q < blk * 32 * RW / c.group ? 0 : c.causal ? min(k_len, max(0, last_q + k_len - q_len + 1)) : k_len;
    const int tiles = (hi + KTS - 1) / KTS, per = (tiles + c.splits - 1) / c.splits;
    const int t0 = min(tiles, split * per), t1 = min(tiles, t0 + per);

    const E *kp = (const E *)c.k + b * c.sk.batch + hk * c.sk.head;
    const E *vp = (const E *)c.v + b * c.sv.batch + hk * c.sv.head;
    const int64_t bh = (int64_t)b * c.kv_heads + hk;
    PairScale ps;
    if constexpr (kPair) ps = pair_scale(c, bh);
    const float scale = kPair ? ps.score : c.scale;
    const float *bp = BIAS ? c.bias + b * c.bias_ld : nullptr;
    const LdsPtr base = (LdsPtr)lds;

    // what a thread fetches of a tile
    unsigned ko[D::kOffsets], vo[D::kOffsets];
    uint4 kr[kDirect ? 1 : NPC], vr[kDirect ? 1 : NPC];
    float br = 0.0f;
    if constexpr (!kPair && LOAD == kDma) {
#pragma unroll
        for (int i = 0; i < D::kOffsets; ++i) {
            ko[i] = (unsigned)(D::row(tid, i) * (int)c.sk.row * (int)sizeof(E) + D::piece(tid, i) * 16);
            vo[i] = (unsigned)(D::row(tid, i) * (int)c.sv.row * (int)sizeof(E) + D::piece(tid, i) * 16);
        }
        if (t0 < t1) D::clear(lds, tid, c.d, k_len - (t1 - 1) * KTS, t1 - t0);
    }
    // kDma: the whole way; otherwise to registers
    auto fetch = [&](int tile, int buf) {
        if constexpr (kPair) {
            const int64_t at = (bh * pair_rows(c.m) + (int64_t)tile * KTS) * TL::kRow;
            const unsigned to = lds_address(base) + 2 * buf * kTile;
            DmaImage<DP, KTS, NT>::load(c.pair.img[kPairK] + at, to, tid);
            DmaImage<DP, KTS, NT>::load(c.pair.img[kPairV] + at, to + kTile, tid);
        } else if constexpr (LOAD == kDma) {
            const char *kb = (const char *)(kp + (int64_t)tile * KTS * c.sk.row), *vb = (const char *)(vp + (int64_t)tile * KTS * c.sv.row);
            const unsigned to = lds_address(base) + 2 * buf * kTile;
            D::load(kb, ko, D::kRound * c.sk.row * (int)sizeof(E), to, tid, c.d, k_len - tile * KTS);
            D::load(vb, vo, D::kRound * c.sv.row * (int)sizeof(E), to + kTile, tid, c.d, k_len - tile * KTS);
        } else {
#pragma unroll
            for (int i = 0; i < NPC; ++i) {
                const int p = tid + i * NT, pc = p % TL::kPieces, key = tile * KTS + p / TL::kPieces, at = min(key, k_len - 1);
                kr[i] = load_piece<E, ALN>(kp + (int64_t)at * c.sk.row, pc, c.d);
                vr[i] = load_piece<E, ALN>(vp + (int64_t)at * c.sv.row, pc, c.d);
                if (BIAS && bp[at] == -INFINITY) kr[i] = vr[i] = make_uint4(0, 0, 0, 0);   // what removed keys hold does not matter
            }
        }
        if (BIAS && tid < KTS) br = bp[min(tile * KTS + tid, k_len - 1)];
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
        if (BIAS && tid < KTS) lbias[buf][tid] = br;
    };

    if (t0 < t1) fetch(t0, 0);
    Frag q[NS];
    if constexpr (kPair) {
#pragma unroll
        for (int t = 0; t < NS; ++t) q[t] = TL::from_image(c.pair.img[kPairQ] + bh * pair_rows(rows) * TL::kRow, r, t, half);
    } else {
        const E *row = (const E *)c.q + b * c.sq.batch + (int64_t)pk.q * c.sq.row + (hk * c.group + pk.g) * c.sq.head;
#pragma unroll
        for (int t = 0; t < NS; ++t)
            q[t] = __builtin_bit_cast(Frag, live ? load_piece<E, ALN>(row, 2 * t + half, c.d) : make_uint4(0, 0, 0, 0));
    }
    f32x16 o[ND];
#pragma unroll
    for (int i = 0; i < ND; ++i) o[i] = (f32x16)(0.0f);
    // units of the running values: without bias the products <q, k>, with it the scores
    const float unit = BIAS ? kLog2eF : scale * kLog2eF;
    // exp2((s - ref) unit), the difference first: a bias of the type's lowest value times log2 e would leave the type.  Without bias one
    // fma does, whose reference is rounded once for the whole row (the fp32 matrix cores, which wait for nobody, keep the difference:
    // a row of one key then is that key's value to the last bit).
    constexpr bool kDiff = BIAS || std::is_same<T, float>::value;
    float ref = -INFINITY, top = -INFINITY, sum = 0.0f;
    const typename TL::Lanes ln = TL::lanes(lane);

    constexpr bool kRemoved = BIAS && !kPair && LOAD == kDma;
    auto removed = [&](int buf) {
        if constexpr (kRemoved) clear_removed<T, DP, KTS, NT>(lds + 2 * buf * kTile, lds + (2 * buf + 1) * kTile, lbias[buf], tid);
    };
    if (t0 < t1) put(0);
    dma_wait();   // (of q as well: not inside the loop, where it would wait for the next tile)
    __builtin_amdgcn_s_waitcnt(0x0f70);
    __syncthreads();
    if (kRemoved && t0 < t1) removed(0);
    // scores of a tile; returns the row's largest
    auto scores = [&](int tile, f32x16 (&s)[NB]) {
        const int buf = (tile - t0) & 1;
        const LdsPtr lk = base + 2 * buf * kTile + part_id * KT * TL::kRow;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
            s[nb] = (f32x16)(0.0f);
#pragma unroll
            for (int t = 0; t < NS; ++t) s[nb] = M::mma(TL::rows(lk, ln, nb * 32, t), q[t], s[nb]);
        }
        if constexpr (BIAS) {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const f32x4 add = *(const f32x4 *)&lbias[buf][part_id * KT + nb * 32 + 8 * g + 4 * half];
#pragma unroll
                    for (int j = 0; j < 4; ++j) s[nb][4 * g + j] = fmaf(s[nb][4 * g + j], scale, add[j]);
                }
        }
        const int first = tile * KTS + part_id * KT;
        if (__any(limit < first + KT)) {
            const int key0 = first + 4 * half;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    s[nb][i] = key0 + nb * 32 + 8 * (i / 4) + i % 4 < limit ? s[nb][i] : -INFINITY;
        }
        float mx = -INFINITY;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[nb][i]);
        return across_halves_max(mx);
    };
    // their exponentials into the sum and, times the values, into the accumulators
    auto accumulate = [&](int tile, f32x16 (&s)[NB]) {
        const LdsPtr lv = base + 2 * ((tile - t0) & 1) * kTile + kTile + part_id * KT * TL::kRow;
        const float safe = ref == -INFINITY ? 0.0f : ref, off = safe * unit - (kPair ? 4.0f : 0.0f);   // (kPairP = 2^4)
        float part = 0.0f;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float e = kDiff ? __builtin_amdgcn_exp2f(kPair ? fmaf(s[nb][i] - safe, unit, 4.0f) : (s[nb][i] - safe) * unit)
                                      : __builtin_amdgcn_exp2f(fmaf(s[nb][i], unit, -off));
                s[nb][i] = e;
                part += e;
            }
        sum += part;
        // O^T += V^T P^T; a bf16 probability is rounded to 2^-9 of itself, its row's sum takes it unrounded
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int t = 0; t < NF; ++t) {
                const Frag p = M::pack(s[nb], t);
#pragma unroll
                for (int i = 0; i < ND; ++i) o[i] = M::mma(TL::cols(lv, ln, nb * 32, t, i, lane), p, o[i]);
            }
    };
    auto next_tile = [&](int tile) {
        if ((!kDirect || BIAS) && tile + 1 < t1) put((tile + 1 - t0) & 1);
        if (kDirect) dma_wait();
        __syncthreads();
        if (kRemoved && tile + 1 < t1) removed((tile + 1 - t0) & 1);
    };
    int tile = t0;
    bool fetched = false;
    for (; tile < t1; ++tile) {
        if (tile + 1 < t1) fetch(tile + 1, (tile + 1 - t0) & 1);
        f32x16 s[NB];
        const float mx = scores(tile, s);
        ref = ref == -INFINITY ? mx : ref;
        fetched = __any((mx - ref) * unit > (kPair ? kSlackPair : kSlack));
        if (fetched) break;
        top = fmaxf(top, mx);
        accumulate(tile, s);
        next_tile(tile);
    }
    for (; tile < t1; ++tile) {
        if (!fetched && tile + 1 < t1) fetch(tile + 1, (tile + 1 - t0) & 1);
        fetched = false;
        f32x16 s[NB];
        const float mx = scores(tile, s), next = fmaxf(ref, mx);
        const float f = next == ref ? 1.0f : __builtin_amdgcn_exp2f((ref - next) * unit);   // (from minus infinity: 0)
        top = fmaxf(top, mx);
        ref = next;
        sum *= f;
#pragma unroll
        for (int i = 0; i < ND; ++i) o[i] *= f;
        accumulate(tile, s);
        next_tile(tile);
    }

    sum = across_halves_sum(sum);
    if constexpr (KS > 1) {   // (the last tile's barrier has passed: nobody reads keys any more)
        float *at = (float *)lds + ((part_id - 1) * RW + wave) * (16 * ND + 3) * 64 + lane;
        if (part_id > 0) {
#pragma unroll
            for (int i = 0; i < 16 * ND; ++i) at[64 * i] = o[i / 16][i % 16];
            at[64 * 16 * ND] = top;
            at[64 * (16 * ND + 1)] = ref;
            at[64 * (16 * ND + 2)] = sum;
        }
        __syncthreads();
        if (part_id > 0) return;
        for (int k = 1; k < KS; ++k) {
            const float *in = (const float *)lds + ((k - 1) * RW + wave) * (16 * ND + 3) * 64 + lane;
            const float itop = in[64 * 16 * ND], iref = in[64 * (16 * ND + 1)], isum = in[64 * (16 * ND + 2)];
            // below the higher of the two references (from minus infinity: nothing seen yet)
            const float next = fmaxf(ref, iref), f = ref == next ? 1.0f : __builtin_amdgcn_exp2f((ref - next) * unit),
                        g = iref == next ? 1.0f : __builtin_amdgcn_exp2f((iref - next) * unit);
            top = fmaxf(top, itop);
            ref = next;
            sum = fmaf(isum, g, sum * f);
#pragma unroll
            for (int i = 0; i < 16 * ND; ++i) o[i / 16][i % 16] = fmaf(in[64 * i], g, o[i / 16][i % 16] * f);
        }
    }
    if (r >= rows) return;
    const float st = BIAS ? 1.0f : scale;   // the running values as scores
    if constexpr (kPair) {
        sum /= kPairP;
#pragma unroll
        for (int i = 0; i < ND; ++i) o[i] *= ps.v / kPairP;
    }
    if (c.splits > 1) {
        const int64_t at = ((int64_t)split * c.batch * c.kv_heads + bh) * rows + r;
        float *po = c.part + at * DP + 4 * half;
#pragma unroll
        for (int i = 0; i < ND; ++i)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *(f32x4 *)(po + 32 * i + 8 * g) = f32x4{o[i][4 * g], o[i][4 * g + 1], o[i][4 * g + 2], o[i][4 * g + 3]};
        if (half == 0) *(f32x4 *)(c.part_stat + at * 4) = f32x4{top * st, ref * st, sum, 0.0f};
        return;
    }
    const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
    E *out = (E *)c.o + b * c.so.batch + (int64_t)pk.q * c.so.row + (hk * c.group + pk.g) * c.so.head;
#pragma unroll
    for (int i = 0; i < ND; ++i) store_column<E, ALN>(out, o[i], inv, 32 * i + 4 * half, c.d);
    if (half == 0) {
        const int64_t at = (bh * c.group + pk.g) * c.n + pk.q;
        // the sum below the maximum itself
        const float safe = ref == -INFINITY ? 0.0f : ref;
        *(float2 *)(c.stat + 2 * at) = make_float2(reported_max(top * st, sum), sum == 0.0f ? 0.0f : sum * __builtin_amdgcn_exp2f((safe - top) * unit));
    }
}

// Merge of the splits, o = sum_s e^(m_s - m) o_s / sum_s e^(m_s - m) l_s; bound by latency (12000 rows of 40 in five splits: 5.6 us; four
// rows of 128 a head in 32 splits: 4.9 us).  A thread takes four coordinates of a packed row and every G-th split, four splits' loads at a time; G groups of
// threads share a row and meet in LDS: one up to eight splits (five splits of 12000 rows, d = 40 in float32: 40.3 us with the splits'
// own kernel; four groups, whose loads mostly repeat a split: 43.0).
template <typename T, int DP, int G>
__global__ __launch_bounds__(256) void k_attn_join(const AttnCall c)
{
    constexpr int W = DP / 4, R = 256 / (W * G);   // threads of a group, rows of a workgroup
    __shared__ f32x4 lacc[G > 1 ? 256 : 1];
    __shared__ float2 lst[G > 1 ? 256 : 1];
    const int rows = c.n * c.group, t = threadIdx.x, x = t % W, g = t / W % G;
    const int64_t total = (int64_t)c.batch * c.kv_heads * rows, at = (int64_t)blockIdx.x * R + t / (W * G);
    const bool there = t < W * G * R && at < total;
    float top = -INFINITY, sum = 0.0f;   // the largest score of all, and the sum below it
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    auto add = [&](float mx, float ref, float s, f32x4 v) {   // the split's largest score, what it was taken below, its sums
        if (ref == -INFINITY && s == s) return;   // no key of this split (with scores that are all NaN the sum is NaN as well)
        const float next = fmaxf(top, mx), f = __builtin_amdgcn_exp2f((top - next) * kLog2eF), h = __builtin_amdgcn_exp2f((ref - next) * kLog2eF);
        top = next;
        sum = fmaf(sum, f, s * h);
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] = fmaf(acc[j], f, v[j] * h);
    };
    if (there)
        for (int s0 = g; s0 < c.splits; s0 += 4 * G) {
            f32x4 st[4], v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int64_t slot = min(s0 + k * G, c.splits - 1) * total + at;
                st[k] = *(const f32x4 *)(c.part_stat + slot * 4);
                v[k] = *(const f32x4 *)(c.part + slot * DP + 4 * x);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (s0 + k * G < c.splits) add(st[k][0], st[k][1], st[k][2], v[k]);
        }
    if constexpr (G > 1) {
        lacc[t] = acc;
        lst[t] = make_float2(top, sum);
        __syncthreads();
        if (g != 0) return;
        for (int k = 1; k < G; ++k) add(lst[t + k * W].x, lst[t + k * W].x, lst[t + k * W].y, lacc[t + k * W]);
    }
    if (!there) return;
    const int64_t bh = at / rows;
    const Packed pk = unpack((int)(at - bh * rows), c.group);
    const int hk = (int)(bh % c.kv_heads), b = (int)(bh / c.kv_heads);
    const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
    T *out = (T *)c.o + b * c.so.batch + (int64_t)pk.q * c.so.row + (hk * c.group + pk.g) * c.so.head;
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (4 * x + j < c.d) out[4 * x + j] = (T)(acc[j] * inv);
    if (x == 0) *(float2 *)(c.stat + 2 * ((bh * c.group + pk.g) * c.n + pk.q)) = make_float2(reported_max(top, sum), sum);
}

template <typename T, int DP> void join(Ctx *c, const AttnCall &a)
{
    const int64_t total = (int64_t)a.batch * a.kv_heads * a.n * a.group;
    constexpr int W = DP / 4;
    if (a.splits > 16) k_attn_join<T, DP, 8><<<(unsigned)ceil_div(total, 256 / (8 * W)), 256, 0, c->stream>>>(a);
    else if (a.splits > 8) k_attn_join<T, DP, 4><<<(unsigned)ceil_div(total, 256 / (4 * W)), 256, 0, c->stream>>>(a);
    else k_attn_join<T, DP, 1><<<(unsigned)ceil_div(total, 256 / W), 256, 0, c->stream>>>(a);
}

template <typename T, int DP, int KTS, int RW, int KS>
fs_status run(Ctx *c, const AttnCall &a, Load load, int64_t grid)
{
    const unsigned g = (unsigned)grid, nt = 64 * RW * KS;
    if constexpr (std::is_same<T, Pair>::value) {   // (rows of the tensors themselves are only written)
        if (a.bias) {
            if (load != kAny) k_attn<T, DP, KTS, RW, KS, true, kVec><<<g, nt, 0, c->stream>>>(a);
            else k_attn<T, DP, KTS, RW, KS, true, kAny><<<g, nt, 0, c->stream>>>(a);
        } else {
            if (load != kAny) k_attn<T, DP, KTS, RW, KS, false, kVec><<<g, nt, 0, c->stream>>>(a);
            else k_attn<T, DP, KTS, RW, KS, false, kAny><<<g, nt, 0, c->stream>>>(a);
        }
    } else if (a.bias) {
        if (load == kDma) k_attn<T, DP, KTS, RW, KS, true, kDma><<<g, nt, 0, c->stream>>>(a);
        else if (load == kVec) k_attn<T, DP, KTS, RW, KS, true, kVec><<<g, nt, 0, c->stream>>>(a);
        else k_attn<T, DP, KTS, RW, KS, true, kAny><<<g, nt, 0, c->stream>>>(a);
    } else {
        if (load == kDma) k_attn<T, DP, KTS, RW, KS, false, kDma><<<g, nt, 0, c->stream>>>(a);
        else if (load == kVec) k_attn<T, DP, KTS, RW, KS, false, kVec><<<g, nt, 0, c->stream>>>(a);
        else k_attn<T, DP, KTS, RW, KS, false, kAny><<<g, nt, 0, c->stream>>>(a);
    }
    if (a.splits > 1) join<typename Mma<T>::Elem, DP>(c, a);
    FS_HIP(c, hipGetLastError());
    return FS_OK;
}

fs_status pairs_by_width(Ctx *c, const AttnCall &a, Load load, int64_t grid)
{
    switch ((a.d + 31) / 32) {
    case 1: return run<Pair, 32, 64, 4, 1>(c, a, load, grid);
    case 2: return run<Pair, 64, 64, 4, 1>(c, a, load, grid);
    case 3: return run<Pair, 96, 32, 4, 1>(c, a, load, grid);
    default: return run<Pair, 128, 32, 4, 1>(c, a, load, grid);
    }
}

template <typename T, int DP> fs_status by_rows(Ctx *c, const AttnCall &a, Load load, const AttnPlan &p)
{
    constexpr bool f32 = std::is_same<T, float>::value;
    if (p.rows == 32) return run<T, DP, 32, 1, 1>(c, a, load, p.grid);
    if constexpr (!f32)
        if (p.rows == 64) return run<T, DP, few_keys(DP), 2, 4>(c, a, load, p.grid);
    return run<T, DP, f32 ? 32 : 64, 4, 1>(c, a, load, p.grid);
}

template <typename T> fs_status by_width(Ctx *c, const AttnCall &a, Load load, const AttnPlan &p)
{
    switch ((a.d + 31) / 32) {
    case 1: return by_rows<T, 32>(c, a, load, p);
    case 2: return by_rows<T, 64>(c, a, load, p);
    case 3: return by_rows<T, 96>(c, a, load, p);
    default: return by_rows<T, 128>(c, a, load, p);
    }
}

}  // namespace

AttnPlan attn_plan(const Ctx *c, const AttnCall &a, bool f32)
{
    AttnPlan p;
    const int64_t rows = (int64_t)a.n * a.group, heads = (int64_t)a.batch * a.kv_heads;
    p.pairs = f32 && pair_worth(c, a, false);
    // Rows of a workgroup: 128, or, in bf16 where these do not fill the chip, 64 whose keys eight waves share (16 heads of 1024 points,
    // d = 64: 14.5 us; four splits of 128 rows and their merge take 21; float32 in 64-row workgroups is slower), or 32 of one wave for
    // a few queries over long keys, which is bound by memory.
    const int64_t wide = ceil_div(rows, 128) * heads, few = few_keys((int)round_up(a.d, 32));
    p.rows = p.pairs ? 128 : rows <= 32 ? 32 : !f32 && wide < c->num_cu && a.m >= few ? 64 : 128;
    p.threads = p.rows == 32 ? 64 : p.rows == 64 ? 512 : 256;
    const int64_t kt = p.rows == 64 ? few : p.rows == 32 || f32 ? 32 : 64;
    const int64_t blocks = ceil_div(rows, p.rows) * heads, tiles = ceil_div(a.m, kt);
    const int64_t want = (int64_t)c->num_cu * (p.rows == 32 ? 4 : p.rows == 64 ? 1 : 2);
    p.splits = (int)std::max<int64_t>(1, std::min(want / std::max<int64_t>(blocks, 1), tiles / (p.rows == 64 ? 2 : 4)));
    p.grid = blocks * p.splits;
    const int64_t dp = round_up(a.d, 32), total = heads * rows * p.splits;
    p.part_bytes = p.splits > 1 ? (size_t)total * dp * 4 : 0;
    p.pair_bytes = p.pairs ? pair_bytes(a, false) : 0;
    p.stat_bytes = p.splits > 1 ? (size_t)total * 16 : 0;
    return p;
}

fs_status launch_attn(Ctx *c, const AttnCall &a, const AttnPlan &p, bool f32, bool aligned)
{
    // (direct loads: offsets of 128 rows in 32 bits, as many as a round of eight waves or a tile of d = 96 has)
    const int64_t most = std::max(a.sk.row, a.sv.row) * (f32 ? 4 : 2) * 128;
    const Load load = !aligned ? kAny : most < (int64_t(1) << 31) ? kDma : kVec;
    if (p.pairs) {
        const fs_status st = launch_pairs(c, a, false, aligned);
        return st ? st : pairs_by_width(c, a, load, p.grid);
    }
    return f32 ? by_width<float>(c, a, load, p) : by_width<__bf16>(c, a, load, p);
}

}  // namespace fs
