// Floats as pairs of fp16 for attention in full precision (see Pair in fs_attn.h): two passes over q, k, v and do, one for the largest
// magnitude (and row norm) of every head, one that writes the pieces as the attention kernels' LDS tiles, and of do each row's scale, norm
// and product with o, which the backward pass takes up.  Any strides, lengths and removed keys end here: what is not admitted becomes zero.
#include <algorithm>

#include "fs_attn.h"

namespace fs {
namespace {

// rows of a workgroup of the first pass: 32, or so many that a head has at most 512 workgroups
__host__ __device__ inline int chunk_rows(int64_t rows) { return rows <= 512 * 32 ? 32 : (int)((rows + 511) / 512); }
__host__ __device__ inline int chunks(int64_t rows) { return (int)((rows + chunk_rows(rows) - 1) / chunk_rows(rows)); }

struct Rows {
    const float *p;      // row 0 of this (set, kv head), nullptr: not admitted
    HeadsAt at;
    bool keys;
    int count;           // packed rows, or keys
};
constexpr int kPairO = kPairTensors;   // (not kept in pieces)
__device__ inline Rows rows_of(const AttnCall &c, int tensor, int bh)
{
    const int b = bh / c.kv_heads, hk = bh - b * c.kv_heads;
    const HeadsAt at = tensor == kPairQ ? c.sq : tensor == kPairK ? c.sk : tensor == kPairV ? c.sv : tensor == kPairO ? c.so : c.s_do;
    const void *p = tensor == kPairQ ? c.q : tensor == kPairK ? c.k : tensor == kPairV ? c.v : tensor == kPairO ? c.o : c.d_o;
    const bool keys = tensor == kPairK || tensor == kPairV;
    return {(const float *)p + b * at.batch + (int64_t)(keys ? hk : hk * c.group) * at.head, at, keys, keys ? c.m : c.n * c.group};
}
__device__ inline const float *row_at(const AttnCall &c, const Rows &t, int b, int r)
{
    if (t.keys) {
        const int len = c.k_len ? min(max(c.k_len[b], 0), c.m) : c.m;
        if (r >= len || (c.bias && c.bias[b * c.bias_ld + r] == -INFINITY)) return nullptr;
        return t.p + (int64_t)r * t.at.row;
    }
    const Packed pk = unpack(r, c.group);
    const int len = c.q_len ? min(max(c.q_len[b], 0), c.n) : c.n;
    return pk.q < len ? t.p + (int64_t)pk.q * t.at.row + pk.g * t.at.head : nullptr;
}

// what a row's norm counts: of do over the sum of exponentials, the row's largest probability (a row that sees no key: nothing)
__device__ inline float weight_of(const AttnCall &c, int tensor, int bh, int r)
{
    if (tensor != kPairDo) return 1.0f;
    const Packed pk = unpack(r, c.group);
    const float l = c.stat[2 * (((int64_t)bh * c.group + pk.g) * c.n + pk.q) + 1];
    return l > 0.0f ? 1.0f / l : 0.0f;
}

// `count` elements of a row from `col` on, zero beyond d (ALN: aligned to 16 bytes, d a multiple of four)
template <int N> __device__ inline void load_row(const float *row, int col, int d, bool aligned, float (&v)[N])
{
#pragma unroll
    for (int j = 0; j < N; j += 4) {
        f32x4 u = {0.0f, 0.0f, 0.0f, 0.0f};
        if (row && aligned) {
            if (col + j < d) u = *(const f32x4 *)(row + col + j);
        } else if (row) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (col + j + k < d) u[k] = row[col + j + k];
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) v[j + k] = u[k];
    }
}

// Bound by latency at the sizes that gain from pairs (three sets of 1000 and 777 points, 4 heads of 40, four tensors: 6.1 us, and 7.9 for
// the second pass, of which some 2 are each launch's own).
// Eight lanes take a row, each DP / 8 elements of it; a workgroup 32 rows at a time
template <int DP> __global__ __launch_bounds__(256) void k_pair_max(const AttnCall c, bool aligned)
{
    __shared__ float2 lds[4];
    const int bh = blockIdx.y, tensor = blockIdx.z, heads = c.batch * c.kv_heads;
    const Rows t = rows_of(c, tensor, bh);
    const int per = chunk_rows(t.count), r0 = blockIdx.x * per, r1 = min(t.count, r0 + per), x = threadIdx.x & 7;
    if (r0 >= t.count) return;
    float top = 0.0f, norm = 0.0f;
    for (int r = r0 + threadIdx.x / 8; r < r1; r += 32) {
        float v[DP / 8];
        const float weight = weight_of(c, tensor, bh, r);
        load_row<DP / 8>(row_at(c, t, bh / c.kv_heads, r), x * (DP / 8), c.d, aligned, v);
        double s = 0.0;   // (squares leave a float's range before the values do)
#pragma unroll
        for (int j = 0; j < DP / 8; ++j)
            if (fabsf(v[j]) < INFINITY) {   // (what is not finite spreads by itself)
                top = fmaxf(top, fabsf(v[j]));
                s = fma((double)v[j], (double)v[j], s);
            }
#pragma unroll
        for (int m = 1; m < 8; m *= 2) s += __shfl_xor(s, m);
        norm = fmaxf(norm, (float)sqrt(s) * weight);
    }
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
        top = fmaxf(top, __shfl_xor(top, m));
        norm = fmaxf(norm, __shfl_xor(norm, m));
    }
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = make_float2(top, norm);
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 4; ++i) lds[0] = make_float2(fmaxf(lds[0].x, lds[i].x), fmaxf(lds[0].y, lds[i].y));
        ((float2 *)c.pair.part)[((int64_t)tensor * heads + bh) * 512 + blockIdx.x] = lds[0];
    }
}

// A workgroup writes 32 rows as the attention kernels' LDS holds them, so that these fetch tiles with direct loads of whole lines; of do
// every row under its own scale, with what the backward pass needs of it besides.
template <int DP> __global__ __launch_bounds__(256) void k_pair_split(const AttnCall c, bool aligned)
{
    using TL = Tile<Pair, DP>;
    __shared__ float2 lds[4];
    const int bh = blockIdx.y, tensor = blockIdx.z, heads = c.batch * c.kv_heads;
    const Rows t = rows_of(c, tensor, bh);
    const int64_t pad = pair_rows(t.count);
    if ((int64_t)blockIdx.x * 32 >= pad) return;
    constexpr int W = DP / 8, P = 32 * W, N = (P + 255) / 256;   // pieces of eight elements, of a row and of all
    __shared__ float piece_top[P];
    __shared__ float2 piece_sum[P];
    float v[N][8], o[N][8];   // (on their way while the scale is found)
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int p = threadIdx.x + 256 * i, r = blockIdx.x * 32 + p / W;
        load_row<8>(p < P && r < t.count ? row_at(c, t, bh / c.kv_heads, r) : nullptr, p % W * 8, c.d, aligned, v[i]);
        if (tensor == kPairDo)
            load_row<8>(p < P && r < t.count ? row_at(c, rows_of(c, kPairO, bh), bh / c.kv_heads, r) : nullptr, p % W * 8, c.d, aligned, o[i]);
    }
    float top = 0.0f, norm = 0.0f;
    for (int i = threadIdx.x; i < chunks(t.count); i += 256) {
        const float2 v = ((const float2 *)c.pair.part)[((int64_t)tensor * heads + bh) * 512 + i];
        top = fmaxf(top, v.x);
        norm = fmaxf(norm, v.y);
    }
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
        top = fmaxf(top, __shfl_xor(top, m));
        norm = fmaxf(norm, __shfl_xor(norm, m));
    }
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = make_float2(top, norm);
    if (tensor == kPairDo) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int p = threadIdx.x + 256 * i;
            float m = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) m = fabsf(v[i][j]) < INFINITY ? fmaxf(m, fabsf(v[i][j])) : m;
            if (p < P) piece_top[p] = m;
        }
    }
    __syncthreads();
    top = fmaxf(fmaxf(lds[0].x, lds[1].x), fmaxf(lds[2].x, lds[3].x));
    norm = fmaxf(fmaxf(lds[0].y, lds[1].y), fmaxf(lds[2].y, lds[3].y));
    const float scale = pair_power(top, 14);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        c.pair.scale[8 * bh + tensor] = scale;
        if (tensor >= kPairV) c.pair.scale[8 * bh + 4 + tensor - kPairV] = norm;
    }
    float row_own[N];
    char *img = c.pair.img[tensor] + ((int64_t)bh * pad + (int64_t)blockIdx.x * 32) * TL::kRow;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int p = threadIdx.x + 256 * i;
        if (p >= P) break;
        float own = scale;
        if (tensor == kPairDo) {
            float m = 0.0f;
#pragma unroll
            for (int j = 0; j < W; ++j) m = fmaxf(m, piece_top[p / W * W + j]);
            if (m > 0.0f) own = pair_power(m, 14);   // (never below the head's; a row of zeros takes that)
            if (p % W == 0) row_own[i] = own;
            float2 sum = make_float2(0.0f, 0.0f);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float x = v[i][j] * (own * 0x1p-15f);
                sum.x = fmaf(x, o[i][j], sum.x);
                sum.y = fmaf(x, x, sum.y);
            }
            piece_sum[p] = sum;
        }
        f16x8 h, l;
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            f16x2 a, b;
            Mma<Pair>::split(v[i][j] * own, v[i][j + 1] * own, a, b);
            h[j] = a[0];
            h[j + 1] = a[1];
            l[j] = b[0];
            l[j + 1] = b[1];
        }
        const int at = TL::B::at(p / W, p % W);
        *(f16x8 *)(img + at) = h;
        *(f16x8 *)(img + TL::kLower + at) = l;
    }
    if (tensor != kPairDo) return;
    // what dq takes up of each row
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int p = threadIdx.x + 256 * i;
        if (p >= P || p % W) continue;
        float2 sum = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int j = 0; j < W; ++j) {
            sum.x += piece_sum[p + j].x;
            sum.y += piece_sum[p + j].y;
        }
        c.pair.row[bh * pad + blockIdx.x * 32 + p / W] = f32x4{row_own[i], sum.x, sqrtf(sum.y) * 0x1p15f, 0.0f};
    }
}

int64_t image_bytes(const AttnCall &a, int tensor)
{
    const bool keys = tensor == kPairK || tensor == kPairV;
    return (int64_t)a.batch * a.kv_heads * pair_rows(keys ? a.m : (int64_t)a.n * a.group) * round_up(a.d, 32) * 4;
}

}  // namespace

// The two passes and the pieces' way through memory take 8 to 15 us.  What they save grows with the products, which are padded to 32
// coordinates.  Pairs and fp32 matrix cores, us (heads x rows x keys, d, padded operations forward), forward: 16 x 500 x 500, 64 (1.0e9)
// 27.0 and 23.0; 8 x 600 x 600, 96 (1.1e9) 29.4 and 30.1; 4 x 800 x 800, 128 (1.3e9) 32.9 and 37.5; 12 x 700 x 700, 40 (1.5e9) 32.6 and
// 36.8; 16 x 1000 x 777, 40 (3.2e9) 38.9 and 48.2; 8 x 4096 x 4096, 64 (34e9) 153 and 343.  Backward: 16 x 200 x 200, 64 (0.16e9) 43
// and 39; 32 x 200 x 200, 64 (0.33e9) 48 and 45; 8 x 300 x 300, 128 (0.37e9) 57 and 66; 12 x 512 x 512, 32 (0.4e9) 37 and 43;
// 8 x 512 x 512, 40 (0.5e9) 46 and 49; 16 x 500 x 500, 64 (1.0e9) 52 and 67; 8 x 4096 x 4096, 64 430 and 1010.  A few rows, bound by
// memory, gain nothing.
bool pair_worth(const Ctx *c, const AttnCall &a, bool grad)
{
    const int64_t rows = (int64_t)a.n * a.group;
    if (rows == 0 || a.m == 0 || (int64_t)a.batch * a.kv_heads > 65535 || rows > int64_t(1) << 28) return false;   // (what the two passes' grids hold)
    if (c->dbg_attn_pairs) return c->dbg_attn_pairs == 1;
    return rows > 32 && 4.0 * (double)a.batch * a.kv_heads * rows * a.m * round_up(a.d, 32) * (a.causal ? 0.5 : 1.0) >= (grad ? 0.3e9 : 1.3e9);
}

size_t pair_bytes(const AttnCall &a, bool grad)
{
    AttnCall t = a;
    pair_layout(&t, nullptr, grad);
    return (size_t)((char *)t.pair.part - (char *)nullptr) + (size_t)kPairTensors * a.batch * a.kv_heads * 512 * 8;
}

void pair_layout(AttnCall *a, char *ws, bool grad)
{
    size_t at = 0;
    auto take = [&](size_t bytes) {
        char *p = (char *)((uintptr_t)ws + at);
        at += (bytes + 255) & ~size_t(255);
        return p;
    };
    for (int t = 0; t < kPairTensors; ++t) a->pair.img[t] = t < kPairDo || grad ? take((size_t)image_bytes(*a, t)) : nullptr;
    a->pair.scale = (float *)take((size_t)a->batch * a->kv_heads * 32);
    a->pair.row = grad ? (f32x4 *)take((size_t)a->batch * a->kv_heads * pair_rows((int64_t)a->n * a->group) * 16) : nullptr;
    a->pair.part = (float *)take(0);
}

template <int DP> static void make_pairs(Ctx *c, const AttnCall &a, bool grad, bool aligned)
{
    const int64_t rows = (int64_t)a.n * a.group;
    const unsigned heads = (unsigned)(a.batch * a.kv_heads), tensors = grad ? 4 : 3;
    k_pair_max<DP><<<dim3((unsigned)std::max(chunks(a.m), chunks(rows)), heads, tensors), 256, 0, c->stream>>>(a, aligned);
    k_pair_split<DP><<<dim3((unsigned)(pair_rows(std::max<int64_t>(a.m, rows)) / 32), heads, tensors), 256, 0, c->stream>>>(a, aligned);
}

fs_status launch_pairs(Ctx *c, const AttnCall &a, bool grad, bool aligned)
{
    switch ((a.d + 31) / 32) {
    case 1: make_pairs<32>(c, a, grad, aligned); break;
    case 2: make_pairs<64>(c, a, grad, aligned); break;
    case 3: make_pairs<96>(c, a, grad, aligned); break;
    default: make_pairs<128>(c, a, grad, aligned); break;
    }
    FS_HIP(c, hipGetLastError());
    return FS_OK;
}

}  // namespace fs
