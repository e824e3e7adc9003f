// Layer norm over the columns of a row-major matrix, forward and backward.
//   xh = (x - mean) rstd,   y = xh gamma + beta,   rstd = 1 / sqrt(var + eps)
//   w = dy gamma:  dx = rstd (w - mean(w) - xh mean(w xh)),   dgamma = sum over rows of dy xh,   dbeta = sum of dy
// Bound by memory: x read and y written once, x and dy read and dx written once.  TPR threads hold a row in registers, so the
// variance is that of the deviations from the mean, as a formula of two passes has it, at one pass over memory.  The mean itself is a
// float: what it is off by, the mean of the deviations, is taken off them (a row whose spread is small against its mean, or whose few
// elements nearly agree, would carry it as an error of its own size in xh).  The gradients of
// the weights are summed over rows in registers (a thread keeps its columns), then over the threads of a workgroup in LDS,
// then over workgroups by a second kernel, always in one order.
#include <algorithm>

#include "fs_internal.h"

namespace fs {
namespace {

constexpr int kNormThreads = 256;
constexpr int kLongThreads = 1024;   // one row per workgroup

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// VEC consecutive elements (VEC > 1: 16 bytes, aligned)
template <typename T, int VEC> struct Pack {
    T e[VEC];
};
template <typename T, int VEC> __device__ inline void load_vec(const T *p, float (&v)[VEC])
{
    if constexpr (VEC == 1) {
        v[0] = (float)p[0];
    } else {
        union {
            u32x4 u;
            Pack<T, VEC> t;
        } w;
        w.u = *(const u32x4 *)p;
#pragma unroll
        for (int j = 0; j < VEC; ++j) v[j] = (float)w.t.e[j];
    }
}
// PAST: past the caches (not a branch on a value: the compiler makes one ordinary store of the two)
template <typename T, int VEC, bool PAST> __device__ inline void store_vec(T *p, const float (&v)[VEC])
{
    if constexpr (VEC == 1) {
        p[0] = (T)v[0];
    } else {
        union {
            u32x4 u;
            Pack<T, VEC> t;
        } w;
#pragma unroll
        for (int j = 0; j < VEC; ++j) w.t.e[j] = (T)v[j];
        if constexpr (PAST) __builtin_nontemporal_store(w.u, (u32x4 *)p);
        else *(u32x4 *)p = w.u;
    }
}
// (VEC > 1: w is 16-byte aligned, and col a multiple of VEC)
template <typename W, int VEC> __device__ inline void load_weights(const W *w, int64_t col, float none, float (&v)[VEC])
{
    typedef W WV __attribute__((ext_vector_type(VEC), aligned(VEC == 1 ? sizeof(W) : 8)));
    if (w) {
        const WV u = *(const WV *)(w + col);
#pragma unroll
        for (int j = 0; j < VEC; ++j) v[j] = (float)u[j];
    } else {
#pragma unroll
        for (int j = 0; j < VEC; ++j) v[j] = none;
    }
}

// v + another lane's v: row_shr by 1, 2, 4, 8 (0x111 ..), the last lane of a row of 16 to the next (0x142) or of 32 to the other half (0x143)
template <int CTRL, int ROWS> __device__ inline float add_from(float v)
{
    return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, ROWS, 0xf, false));
}

// Sum over the TPR threads of a row; every one of them gets it.
template <int TPR> __device__ inline float row_sum(float v, float *lds)
{
    if constexpr (TPR < 64) {
#pragma unroll
        for (int m = 1; m < TPR; m *= 2) v += __shfl_xor(v, m);
    } else {   // within rows of 16 lanes, then across them: the last lane has it all
        v = add_from<0x111, 0xf>(v);
        v = add_from<0x112, 0xf>(v);
        v = add_from<0x114, 0xf>(v);
        v = add_from<0x118, 0xf>(v);
        v = add_from<0x142, 0xa>(v);
        v = add_from<0x143, 0xc>(v);
        v = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
    }
    if constexpr (TPR > 64) {
        constexpr int W = TPR / 64;
        __syncthreads();   // (what was read from lds before)
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x / 64] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int i = 0; i < W; ++i) v += lds[i];
    }
    return v;
}

// 1 / sqrt(var + eps), where rounding may leave var below zero (fmaxf would make a number of NaN)
__device__ inline float inverse_root(float var, float eps) { return 1.0f / sqrtf((var < 0.0f ? 0.0f : var) + eps); }

struct NormCall {
    const void *x, *dy;
    const void *gamma, *beta;   // nullable
    void *y, *dx;
    float *stat;
    const float *stat_in;
    float *part;                // [workgroups][2][cols]
    float *rest;                // [rows]: where rows are longer than the registers of a workgroup
    float *dgamma, *dbeta;
    int64_t rows, cols, ldx, ldy, lddy, lddx;
    float eps;
    int32_t blocks;
    bool past;                  // outputs that no cache will hold until they are read go past them
};

// 70000 x 784 float: 82 us, 5.4 TB/s; 50000 x 1024 bf16: 33 us, 6.2 TB/s.
template <typename T, typename W, int VEC, int NV, int TPR, bool PAST>
__global__ __launch_bounds__(TPR > kNormThreads ? TPR : kNormThreads) void k_norm(const NormCall c)
{
    constexpr int NT = TPR > kNormThreads ? TPR : kNormThreads, RPB = NT / TPR;
    __shared__ float lds[3][TPR > 64 ? TPR / 64 : 1];
    const int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;
    const int t = threadIdx.x % TPR;
    const bool live = row < c.rows;
    const T *x = (const T *)c.x + row * c.ldx;
    float v[NV][VEC], s = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int64_t col = (int64_t)(i * TPR + t) * VEC;
        if (live && col < c.cols) load_vec<T, VEC>(x + col, v[i]);
        else
#pragma unroll
            for (int j = 0; j < VEC; ++j) v[i][j] = 0.0f;
#pragma unroll
        for (int j = 0; j < VEC; ++j) s += v[i][j];
    }
    const float inv = 1.0f / (float)c.cols, mean = row_sum<TPR>(s, lds[0]) * inv;
    float s2 = 0.0f;
    s = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if ((int64_t)(i * TPR + t) * VEC < c.cols) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                v[i][j] -= mean;
                s += v[i][j];
                s2 = fmaf(v[i][j], v[i][j], s2);
            }
        }
    const float rest = row_sum<TPR>(s, lds[1]) * inv;
    const float rstd = inverse_root(row_sum<TPR>(s2, lds[2]) * inv - rest * rest, c.eps);
    if (!live) return;
    T *y = (T *)c.y + row * c.ldy;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int64_t col = (int64_t)(i * TPR + t) * VEC;
        if (col < c.cols) {
            float g[VEC], b[VEC];
            load_weights<W, VEC>((const W *)c.gamma, col, 1.0f, g);
            load_weights<W, VEC>((const W *)c.beta, col, 0.0f, b);
#pragma unroll
            for (int j = 0; j < VEC; ++j) v[i][j] = fmaf((v[i][j] - rest) * rstd, g[j], b[j]);
            store_vec<T, VEC, PAST>(y + col, v[i]);
        }
    }
    if (t == 0 && c.stat) *(float2 *)(c.stat + 2 * row) = make_float2(mean + rest, rstd);
}

// 70000 x 784 float: 117 us, 5.6 TB/s; 50000 x 1024 bf16: 52 us, 5.9 TB/s; the workgroups' shares of the weights' gradients: k_norm_wsum, 5 us.
template <typename T, typename W, int VEC, int NV, int TPR, bool PAST>
__global__ __launch_bounds__(TPR > kNormThreads ? TPR : kNormThreads) void k_norm_grad(const NormCall c)
{
    constexpr int NT = TPR > kNormThreads ? TPR : kNormThreads, RPB = NT / TPR;
    __shared__ float lds[3][TPR > 64 ? TPR / 64 : 1];
    constexpr int SIDE = TPR < 64 ? NT / 64 : RPB, WIDE = TPR < 64 ? 64 : TPR;   // waves, or rows, side by side
    __shared__ float lsum[SIDE > 1 ? SIDE * TPR * VEC : 1];
    const int t = threadIdx.x % TPR, slot = threadIdx.x / TPR;
    float g[NV][VEC], dg[NV][VEC], db[NV][VEC];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int64_t col = (int64_t)(i * TPR + t) * VEC;
#pragma unroll
        for (int j = 0; j < VEC; ++j) g[i][j] = dg[i][j] = db[i][j] = 0.0f;
        if (col < c.cols) load_weights<W, VEC>((const W *)c.gamma, col, 1.0f, g[i]);
    }
    const float inv = 1.0f / (float)c.cols;
    for (int64_t row0 = (int64_t)blockIdx.x * RPB; row0 < c.rows; row0 += (int64_t)gridDim.x * RPB) {
        const int64_t row = row0 + slot;
        const bool live = row < c.rows;
        const T *x = (const T *)c.x + row * c.ldx, *dy = (const T *)c.dy + row * c.lddy;
        float v[NV][VEC], w[NV][VEC];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int64_t col = (int64_t)(i * TPR + t) * VEC;
            if (live && col < c.cols) {
                load_vec<T, VEC>(x + col, v[i]);
                load_vec<T, VEC>(dy + col, w[i]);
            } else {
#pragma unroll
                for (int j = 0; j < VEC; ++j) v[i][j] = w[i][j] = 0.0f;
            }
        }
        float2 st = make_float2(0.0f, 0.0f);
        if (live) st = *(const float2 *)(c.stat_in + 2 * row);
        float s0 = 0.0f, s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if ((int64_t)(i * TPR + t) * VEC < c.cols) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    v[i][j] -= st.x;
                    const float u = w[i][j] * g[i][j];
                    s0 += v[i][j];
                    s1 += u;
                    s2 = fmaf(u, v[i][j], s2);
                }
            }
        s0 = row_sum<TPR>(s0, lds[0]) * inv;
        s1 = row_sum<TPR>(s1, lds[1]) * inv;
        s2 = (row_sum<TPR>(s2, lds[2]) * inv - s0 * s1) * st.y;
        T *dx = (T *)c.dx + row * c.lddx;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int64_t col = (int64_t)(i * TPR + t) * VEC;
            if (col < c.cols) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    v[i][j] = (v[i][j] - s0) * st.y;
                    dg[i][j] = fmaf(w[i][j], v[i][j], dg[i][j]);
                    db[i][j] += w[i][j];
                    w[i][j] = st.y * (fmaf(w[i][j], g[i][j], -s1) - v[i][j] * s2);
                }
                if (live && c.dx) store_vec<T, VEC, PAST>(dx + col, w[i]);
            }
        }
    }
    if (!c.part) return;
    // over the rows that the workgroup's threads hold side by side
    float *out = c.part + (int64_t)blockIdx.x * 2 * c.cols;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int64_t col = (int64_t)(i * TPR + t) * VEC;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            float a[VEC];
#pragma unroll
            for (int j = 0; j < VEC; ++j) a[j] = k ? db[i][j] : dg[i][j];
            if constexpr (TPR < 64) {   // rows of one wave
#pragma unroll
                for (int m = TPR; m < 64; m *= 2)
#pragma unroll
                    for (int j = 0; j < VEC; ++j) a[j] += __shfl_xor(a[j], m);
            }
            if constexpr (SIDE > 1) {
                const int side = threadIdx.x / WIDE;
                __syncthreads();
                if (threadIdx.x % WIDE < TPR) {
#pragma unroll
                    for (int j = 0; j < VEC; ++j) lsum[(side * VEC + j) * TPR + t] = a[j];
                }
                __syncthreads();
                if (slot == 0) {
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        a[j] = 0.0f;
#pragma unroll
                        for (int q = 0; q < SIDE; ++q) a[j] += lsum[(q * VEC + j) * TPR + t];
                    }
                }
            }
            if (slot == 0 && col < c.cols) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) out[k * c.cols + col + j] = a[j];
            }
        }
    }
}

// Rows longer than the registers of a workgroup: three passes over the row, which the caches hold.
template <typename T, typename W> __global__ __launch_bounds__(kLongThreads) void k_norm_long(const NormCall c)
{
    __shared__ float lds[kLongThreads / 64];
    const int64_t row = blockIdx.x;
    const T *x = (const T *)c.x + row * c.ldx;
    const float inv = 1.0f / (float)c.cols;
    float s = 0.0f;
    for (int64_t i = threadIdx.x; i < c.cols; i += kLongThreads) s += (float)x[i];
    const float mean = row_sum<kLongThreads>(s, lds) * inv;
    float s2 = 0.0f;
    s = 0.0f;
    for (int64_t i = threadIdx.x; i < c.cols; i += kLongThreads) {
        const float v = (float)x[i] - mean;
        s += v;
        s2 = fmaf(v, v, s2);
    }
    const float rest = row_sum<kLongThreads>(s, lds) * inv;
    const float rstd = inverse_root(row_sum<kLongThreads>(s2, lds) * inv - rest * rest, c.eps);
    T *y = (T *)c.y + row * c.ldy;
    for (int64_t i = threadIdx.x; i < c.cols; i += kLongThreads) {
        float g[1], b[1];
        load_weights<W, 1>((const W *)c.gamma, i, 1.0f, g);
        load_weights<W, 1>((const W *)c.beta, i, 0.0f, b);
        y[i] = (T)fmaf(((float)x[i] - mean - rest) * rstd, g[0], b[0]);
    }
    if (threadIdx.x == 0 && c.stat) *(float2 *)(c.stat + 2 * row) = make_float2(mean + rest, rstd);
}

template <typename T, typename W> __global__ __launch_bounds__(kLongThreads) void k_norm_grad_long(const NormCall c)
{
    __shared__ float lds[3][kLongThreads / 64];
    const int64_t row = blockIdx.x;
    const T *x = (const T *)c.x + row * c.ldx, *dy = (const T *)c.dy + row * c.lddy;
    const float2 st = *(const float2 *)(c.stat_in + 2 * row);
    const float inv = 1.0f / (float)c.cols;
    float s0 = 0.0f, s1 = 0.0f, s2 = 0.0f, g[1];
    for (int64_t i = threadIdx.x; i < c.cols; i += kLongThreads) {
        load_weights<W, 1>((const W *)c.gamma, i, 1.0f, g);
        const float w = (float)dy[i] * g[0], v = (float)x[i] - st.x;
        s0 += v;
        s1 += w;
        s2 = fmaf(w, v, s2);
    }
    s0 = row_sum<kLongThreads>(s0, lds[0]) * inv;
    s1 = row_sum<kLongThreads>(s1, lds[1]) * inv;
    if (threadIdx.x == 0 && c.rest) c.rest[row] = s0;
    s2 = (row_sum<kLongThreads>(s2, lds[2]) * inv - s0 * s1) * st.y;
    T *dx = (T *)c.dx + row * c.lddx;
    for (int64_t i = threadIdx.x; i < c.cols; i += kLongThreads) {
        load_weights<W, 1>((const W *)c.gamma, i, 1.0f, g);
        dx[i] = (T)(st.y * ((float)dy[i] * g[0] - s1 - ((float)x[i] - st.x - s0) * st.y * s2));
    }
}

// what the mean of such rows, a float, is off by: the mean of the deviations
template <typename T> __global__ __launch_bounds__(kLongThreads) void k_norm_rest_long(const NormCall c)
{
    __shared__ float lds[kLongThreads / 64];
    const int64_t row = blockIdx.x;
    const T *x = (const T *)c.x + row * c.ldx;
    const float mean = c.stat_in[2 * row];
    float s = 0.0f;
    for (int64_t i = threadIdx.x; i < c.cols; i += kLongThreads) s += (float)x[i] - mean;
    s = row_sum<kLongThreads>(s, lds) * (1.0f / (float)c.cols);
    if (threadIdx.x == 0) c.rest[row] = s;
}

// the weights' gradients of such rows: a thread takes a column, a workgroup every blocks-th row
template <typename T> __global__ __launch_bounds__(kNormThreads) void k_norm_wgrad_long(const NormCall c)
{
    const int64_t col = (int64_t)blockIdx.x * kNormThreads + threadIdx.x;
    if (col >= c.cols) return;
    float dg = 0.0f, db = 0.0f;
    for (int64_t row = blockIdx.y; row < c.rows; row += c.blocks) {
        const float2 st = *(const float2 *)(c.stat_in + 2 * row);
        const float dy = (float)((const T *)c.dy)[row * c.lddy + col];
        dg = fmaf(dy, ((float)((const T *)c.x)[row * c.ldx + col] - st.x - c.rest[row]) * st.y, dg);
        db += dy;
    }
    float *out = c.part + (int64_t)blockIdx.y * 2 * c.cols;
    out[col] = dg;
    out[c.cols + col] = db;
}

// Sum of the workgroups' shares: 16 columns x 64 shares at a time (four threads read a 64-byte line of each share together).
__global__ __launch_bounds__(1024) void k_norm_wsum(const float *part, int64_t cols, int blocks, float *dgamma, float *dbeta)
{
    __shared__ float lds[64][17];
    const int64_t wide = 2 * cols, col = (int64_t)blockIdx.x * 16 + threadIdx.x % 16;
    const int lane = threadIdx.x / 16;
    float s = 0.0f;
    if (col < wide)
#pragma unroll 4
        for (int b = lane; b < blocks; b += 64) s += part[b * wide + col];
    lds[lane][threadIdx.x % 16] = s;
    __syncthreads();
    if (threadIdx.x < 16 && col < wide) {
        s = 0.0f;
        for (int i = 0; i < 64; ++i) s += lds[i][threadIdx.x];
        float *out = col < cols ? dgamma : dbeta;
        if (out) out[col < cols ? col : col - cols] = s;
    }
}

// The rows from r0 on, `rows` of them, of a call whose elements have es bytes.
NormCall rows_from(NormCall a, int64_t r0, int64_t rows, int es)
{
    auto at = [&](const void *p, int64_t ld) { return p ? (char *)p + r0 * ld * es : nullptr; };
    a.x = at(a.x, a.ldx);
    a.y = at(a.y, a.ldy);
    a.dy = at(a.dy, a.lddy);
    a.dx = at(a.dx, a.lddx);
    if (a.stat) a.stat += 2 * r0;
    if (a.stat_in) a.stat_in += 2 * r0;
    if (a.rest) a.rest += r0;
    a.rows = rows;
    return a;
}
// A launch has fewer than 2^32 threads: calls of more rows are several, of at most 2^31.
template <typename F> void in_launches(const NormCall &a, int threads, int es, F launch)
{
    const int64_t most = (int64_t(1) << 31) / threads;
    for (int64_t r0 = 0; r0 < a.rows; r0 += most) launch(rows_from(a, r0, std::min(most, a.rows - r0), es));
}

// Elements of a row that a thread holds at most (four arrays of them in the backward pass: with 32 among 1024 threads, which
// have 128 registers each, they would not fit).
constexpr int kHeld = 32, kHeldLong = 16;

// threads that share a row: as few as hold it in registers, at most one 16-byte load each below a wave
int threads_per_row(int64_t cols, int vec)
{
    for (int t : {8, 16, 32, 64, 256, kLongThreads})
        if (cols <= (int64_t)t * (t < 64 ? vec : t < kLongThreads ? kHeld : kHeldLong)) return t;
    return 0;
}

template <typename T, typename W, int VEC, int NV, int TPR> fs_status run(Ctx *c, const NormCall &a, bool grad)
{
    constexpr int NT = TPR > kNormThreads ? TPR : kNormThreads;
    if (grad) {
        if (VEC > 1 && a.past) k_norm_grad<T, W, VEC, NV, TPR, (VEC > 1)><<<(unsigned)a.blocks, NT, 0, c->stream>>>(a);
        else k_norm_grad<T, W, VEC, NV, TPR, false><<<(unsigned)a.blocks, NT, 0, c->stream>>>(a);
        return FS_OK;
    }
    in_launches(a, TPR, sizeof(T), [&](const NormCall &p) {
        const unsigned grid = (unsigned)ceil_div(p.rows, NT / TPR);
        if (VEC > 1 && p.past) k_norm<T, W, VEC, NV, TPR, (VEC > 1)><<<grid, NT, 0, c->stream>>>(p);
        else k_norm<T, W, VEC, NV, TPR, false><<<grid, NT, 0, c->stream>>>(p);
    });
    return FS_OK;
}

template <typename T, typename W, int VEC> fs_status by_length(Ctx *c, const NormCall &a, bool grad)
{
    const int tpr = threads_per_row(a.cols, VEC);
    const int64_t nv = tpr ? ceil_div(a.cols, (int64_t)tpr * VEC) : 0;
    constexpr int most = kHeld / VEC;
    switch (tpr) {
    case 8: return run<T, W, VEC, 1, 8>(c, a, grad);
    case 16: return run<T, W, VEC, 1, 16>(c, a, grad);
    case 32: return run<T, W, VEC, 1, 32>(c, a, grad);
    case 64:
        if (nv <= 1) return run<T, W, VEC, 1, 64>(c, a, grad);
        if (nv <= 2) return run<T, W, VEC, 2, 64>(c, a, grad);
        if (nv <= 4) return run<T, W, VEC, 4, 64>(c, a, grad);
        if constexpr (most > 8) {
            if (nv <= 8) return run<T, W, VEC, 8, 64>(c, a, grad);
            if constexpr (most > 16)
                if (nv <= 16) return run<T, W, VEC, 16, 64>(c, a, grad);
        }
        return run<T, W, VEC, most, 64>(c, a, grad);
    case 256: return nv <= most / 2 ? run<T, W, VEC, most / 2, 256>(c, a, grad) : run<T, W, VEC, most, 256>(c, a, grad);
    case kLongThreads: return run<T, W, VEC, kHeldLong / VEC, kLongThreads>(c, a, grad);
    }
    if (!grad) {
        in_launches(a, kLongThreads, sizeof(T), [&](const NormCall &p) { k_norm_long<T, W><<<(unsigned)p.rows, kLongThreads, 0, c->stream>>>(p); });
        return FS_OK;
    }
    // (what the means are off by comes with dx, unless that takes dy's place, and the weights' gradients go first, or is not wanted: 4000 x
    // 20001 bf16 383 us, and 467 with a pass of its own)
    const bool first = !a.dx || a.dx == a.dy;
    if (a.part && first)
        in_launches(a, kLongThreads, sizeof(T), [&](const NormCall &p) { k_norm_rest_long<T><<<(unsigned)p.rows, kLongThreads, 0, c->stream>>>(p); });
    auto weights = [&] {
        k_norm_wgrad_long<T><<<dim3((unsigned)ceil_div(a.cols, kNormThreads), (unsigned)a.blocks), kNormThreads, 0, c->stream>>>(a);
    };
    if (a.part && first) weights();
    if (a.dx)
        in_launches(a, kLongThreads, sizeof(T), [&](const NormCall &p) { k_norm_grad_long<T, W><<<(unsigned)p.rows, kLongThreads, 0, c->stream>>>(p); });
    if (a.part && !first) weights();
    return FS_OK;
}

template <typename T, typename W> fs_status by_alignment(Ctx *c, const NormCall &a, bool grad)
{
    constexpr int V = 16 / (int)sizeof(T);
    auto fits = [](const void *p, int64_t ld) { return !p || ((uintptr_t)p % 16 == 0 && ld % V == 0); };
    const bool vec = a.cols % V == 0 && fits(a.x, a.ldx) && fits(a.y, a.ldy) && fits(a.dy, a.lddy) && fits(a.dx, a.lddx) &&
                     fits(a.gamma, 0) && fits(a.beta, 0);
    return vec ? by_length<T, W, V>(c, a, grad) : by_length<T, W, 1>(c, a, grad);
}

fs_status dispatch(Ctx *c, NormCall a, int32_t dtype, int32_t wtype, bool grad)
{
    // An output beyond the 4 MB of L2 of eight XCDs (forward and backward, with and without, us: 70000 x 784 float 205 and 224,
    // 50000 x 1024 bf16 104 and 105; loads past the caches as well: 205 and 106)
    a.past = a.rows * a.cols * (dtype == FS_BF16 ? 2 : 4) > (int64_t(32) << 20);
    if (dtype == FS_F32) return wtype == FS_F32 ? by_alignment<float, float>(c, a, grad) : by_alignment<float, __bf16>(c, a, grad);
    return wtype == FS_F32 ? by_alignment<__bf16, float>(c, a, grad) : by_alignment<__bf16, __bf16>(c, a, grad);
}

}  // namespace

// Workgroups of a backward pass: four per CU, or as many as the rows fill.
static int norm_grad_blocks(const Ctx *c, int64_t rows, int64_t cols, int32_t dtype)
{
    // (rows that a workgroup holds side by side, with 16-byte loads; where these cannot be used it holds no more)
    const int tpr = threads_per_row(cols, dtype == FS_BF16 ? 8 : 4);
    const int64_t fill = ceil_div(rows, tpr && tpr < kNormThreads ? kNormThreads / tpr : 1);
    return (int)std::max<int64_t>(1, std::min<int64_t>(fill, 4 * (int64_t)c->num_cu));
}

// Floats that it needs: the workgroups' shares of the weights' gradients, and of long rows what their means are off by.
int64_t norm_grad_part(const Ctx *c, int64_t rows, int64_t cols, int32_t dtype)
{
    return norm_grad_blocks(c, rows, cols, dtype) * 2 * cols + (threads_per_row(cols, 1) ? 0 : rows);
}

fs_status launch_norm(Ctx *c, const void *x, int32_t dtype, int64_t rows, int64_t cols, int64_t ldx, const void *gamma, const void *beta,
                      int32_t wtype, float eps, void *y, int64_t ldy, float *stat)
{
    NormCall a = {};
    a.x = x;
    a.gamma = gamma;
    a.beta = beta;
    a.y = y;
    a.stat = stat;
    a.rows = rows;
    a.cols = cols;
    a.ldx = ldx;
    a.ldy = ldy;
    a.eps = eps;
    dispatch(c, a, dtype, wtype, false);
    FS_HIP(c, hipGetLastError());
    return FS_OK;
}

fs_status launch_norm_grad(Ctx *c, const void *x, int32_t dtype, int64_t rows, int64_t cols, int64_t ldx, const void *gamma, int32_t wtype,
                           const float *stat, const void *dy, int64_t lddy, void *dx, int64_t lddx, float *dgamma, float *dbeta, float *part)
{
    NormCall a = {};
    a.x = x;
    a.dy = dy;
    a.gamma = gamma;
    a.stat_in = stat;
    a.dx = dx;
    a.part = dgamma || dbeta ? part : nullptr;
    a.rows = rows;
    a.cols = cols;
    a.ldx = ldx;
    a.lddy = lddy;
    a.lddx = lddx;
    a.blocks = norm_grad_blocks(c, rows, cols, dtype);
    a.rest = part ? part + a.blocks * 2 * cols : nullptr;
    dispatch(c, a, dtype, wtype, true);
    if (a.part) k_norm_wsum<<<(unsigned)ceil_div(2 * cols, 16), 1024, 0, c->stream>>>(part, cols, a.blocks, dgamma, dbeta);
    FS_HIP(c, hipGetLastError());
    return FS_OK;
}

}  // namespace fs
