// One AdamW step over many tensors.
//   m = b1 m + (1 - b1) g,   v = b2 v + (1 - b2) g^2,   p = (1 - lr wd) p - (lr / (1 - b1^t)) m / (sqrt(v / (1 - b2^t)) + eps)
// Bound by memory: every weight is read and written once with its gradient and its state (28 bytes a weight in full precision, 16
// with bf16 weights, float masters and 8-bit states).  The tensors' addresses go along as kernel arguments, as many as these hold,
// so a step takes no table in device memory and no copy to it.
//
// State in 8 bits: OCP e4m3 codes of m and of sqrt(v), under a power of two for each block of 256 weights (a wave's share) that puts the
// block's largest into (224, 448].  A decay of 0.1 % a step moves nothing that is rounded to nearest at three bits of mantissa, so codes
// are rounded up or down at random in proportion, by 32 bits that are a function of the weight's number and the step's seed.  A root
// above zero never becomes zero: a momentum over a vanished root would be a step of any size.
#include <algorithm>

#include "fs_internal.h"

namespace fs {
namespace {

constexpr int kAdamBlock = 256;     // weights under one scale; 64 lanes, four each
constexpr int kAdamChunk = 1024;    // weights of a workgroup: four waves, a block each
constexpr int kTableBytes = 3840;   // of a launch's 4 KB of arguments
constexpr int64_t kLaunchChunks = 1 << 23;   // workgroups of a launch, which has fewer than 2^32 threads: what is left of a tensor goes on in the next

enum { kP, kG, kM, kV, kMaster, kMs, kVs, kSlots };

// which addresses a table holds: weights, gradients, m, v, and masters and scales where there are any
template <bool MASTER, bool Q8> struct Slots {
    static constexpr int kCount = 4 + (MASTER ? 1 : 0) + (Q8 ? 2 : 0);
    static constexpr int of(int s) { return s < kMaster ? s : s == kMaster ? 4 : 4 + (MASTER ? 1 : 0) + (s - kMs); }
};
template <bool MASTER, bool Q8> struct Table {
    static constexpr int kMost = kTableBytes / (8 * Slots<MASTER, Q8>::kCount + 8 + 8);
    void *at[kMost][Slots<MASTER, Q8>::kCount];
    int64_t n[kMost];
    int32_t chunk[kMost];    // the first workgroup of each
    uint32_t block[kMost];   // blocks of the call before each
    int32_t count;
};

struct AdamStep {
    float b1, c1, b2, c2;    // 1 - b1, 1 - b2, rounded from 64 bits
    float keep, rate, inv, eps;   // 1 - lr wd, lr / (1 - b1^t), 1 / sqrt(1 - b2^t)
    uint32_t seed;
    const float *grad_scale;
};

template <typename T, int N, bool ALN> __device__ inline void load_n(const T *p, int64_t left, float (&v)[N])
{
    if constexpr (ALN) {
        typedef T V __attribute__((ext_vector_type(N)));
        const V u = __builtin_nontemporal_load((const V *)p);
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = (float)u[j];
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = j < left ? (float)p[j] : 0.0f;
    }
}
template <typename T, int N, bool ALN> __device__ inline void store_n(T *p, int64_t left, const float (&v)[N])
{
    if constexpr (ALN) {
        typedef T V __attribute__((ext_vector_type(N)));
        V u;
#pragma unroll
        for (int j = 0; j < N; ++j) u[j] = (T)v[j];
        __builtin_nontemporal_store(u, (V *)p);
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (j < left) p[j] = (T)v[j];
    }
}
template <bool ALN> __device__ inline uint32_t load_codes(const uint8_t *p, int64_t left)
{
    if constexpr (ALN) return __builtin_nontemporal_load((const uint32_t *)p);
    uint32_t w = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) w |= (j < left ? (uint32_t)p[j] : 0u) << (8 * j);
    return w;
}
template <bool ALN> __device__ inline void store_codes(uint8_t *p, int64_t left, uint32_t w)
{
    if constexpr (ALN) {
        __builtin_nontemporal_store(w, (uint32_t *)p);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < left) p[j] = (uint8_t)(w >> (8 * j));
    }
}
__device__ inline void decode(uint32_t w, float scale, float (&v)[4])
{
    v[0] = __builtin_amdgcn_cvt_f32_fp8((int)w, 0) * scale;
    v[1] = __builtin_amdgcn_cvt_f32_fp8((int)w, 1) * scale;
    v[2] = __builtin_amdgcn_cvt_f32_fp8((int)w, 2) * scale;
    v[3] = __builtin_amdgcn_cvt_f32_fp8((int)w, 3) * scale;
}
// the power of two of a block whose largest magnitude is top: 2^-k top in (224, 448]
__device__ inline float block_scale(float top)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, top);
    if (u >= 0x7f800000u) return __builtin_nanf("");   // something is not finite: all of the block becomes so
    if (top == 0.0f) return 1.0f;
    // top = f 2^e, f in [1, 2): e - 8, and one more above 1.75
    int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
    e = e < -100 ? -100 : e;   // (and whatever is that small)
    return __builtin_bit_cast(float, (uint32_t)(e + 127) << 23);
}
// the code of x / scale (inv = 1 / scale, exact), rounded up where the dropped twenty bits and the dither's sixteen carry
__device__ inline uint32_t encode(float x, float inv, uint32_t half)
{
    const float a = fabsf(x) * inv;
    const uint32_t low = (half << 4) | 8u;
    const uint32_t normal = ((__builtin_bit_cast(uint32_t, a) + low) >> 20) - (120u << 3);
    const uint32_t small = (uint32_t)fmaf(a, 512.0f, (float)low * 0x1p-20f);   // below 2^-6: multiples of 2^-9
    const uint32_t code = a >= 0x1p-6f ? normal : small;
    return (code & 0x7fu) | ((__builtin_bit_cast(uint32_t, x) >> 24) & 0x80u);
}
// 32 bits for weight `at` (numbered over the call's tensors, whole blocks each); constants: digits of the golden ratio, e and pi
__device__ inline uint32_t dither(uint32_t at, uint32_t seed)
{
    uint32_t h = (at * 0x9E3779B1u) ^ (seed * 0xB7E15163u);
    h = (h ^ (h >> 16)) * 0x85A308D3u;
    h = (h ^ (h >> 13)) * 0xB7E15163u;
    return h ^ (h >> 16);
}
// the largest magnitude in a wave; NaN and infinity are above all
__device__ inline float wave_top(float v)
{
    uint32_t u = __builtin_bit_cast(uint32_t, v) & 0x7fffffffu;
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
        const uint32_t w = (uint32_t)__shfl_xor((int)u, m);
        u = w > u ? w : u;
    }
    return __builtin_bit_cast(float, u);
}

template <typename P, typename G, bool MASTER, bool Q8, bool ALN>
__device__ inline void adam_block(void *const *at, int64_t i, int64_t n, uint32_t block, const AdamStep &s, float gs)
{
    using S = Slots<MASTER, Q8>;
    const int64_t left = n - i;   // (may be negative in a block's upper lanes)
    P *pp = (P *)at[S::of(kP)] + i;
    float *pm = MASTER ? (float *)at[S::of(kMaster)] + i : nullptr;
    float p[4], g[4], m[4], v[4], root[4];
    load_n<G, 4, ALN>((const G *)at[S::of(kG)] + i, left, g);
    if constexpr (MASTER) load_n<float, 4, ALN>(pm, left, p);
    else load_n<P, 4, ALN>(pp, left, p);
    float *ms = nullptr, *vs = nullptr;
    if constexpr (Q8) {
        ms = (float *)at[S::of(kMs)] + i / kAdamBlock;
        vs = (float *)at[S::of(kVs)] + i / kAdamBlock;
        decode(load_codes<ALN>((const uint8_t *)at[S::of(kM)] + i, left), *ms, m);
        decode(load_codes<ALN>((const uint8_t *)at[S::of(kV)] + i, left), *vs, v);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] *= v[j];
    } else {
        load_n<float, 4, ALN>((const float *)at[S::of(kM)] + i, left, m);
        load_n<float, 4, ALN>((const float *)at[S::of(kV)] + i, left, v);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float gj = g[j] * gs;
        // (products and sums rounded one by one: the code of a state then does not depend on how they are contracted)
        m[j] = __fadd_rn(__fmul_rn(m[j], s.b1), __fmul_rn(gj, s.c1));
        v[j] = __fadd_rn(__fmul_rn(v[j], s.b2), __fmul_rn(__fmul_rn(gj, gj), s.c2));
        root[j] = __builtin_amdgcn_sqrtf(v[j]);   // within an ulp
        p[j] = fmaf(p[j], s.keep, -(s.rate * m[j]) * __builtin_amdgcn_rcpf(fmaf(root[j], s.inv, s.eps)));   // (rcp: within an ulp)
    }
    if constexpr (MASTER) store_n<float, 4, ALN>(pm, left, p);
    store_n<P, 4, ALN>(pp, left, p);
    if constexpr (Q8) {
        float mt = 0.0f, vt = 0.0f;
        uint32_t um = 0, uv = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t a = __builtin_bit_cast(uint32_t, m[j]) & 0x7fffffffu, b = __builtin_bit_cast(uint32_t, root[j]) & 0x7fffffffu;
            um = j < left && a > um ? a : um;
            uv = j < left && b > uv ? b : uv;
        }
        mt = wave_top(__builtin_bit_cast(float, um));
        vt = wave_top(__builtin_bit_cast(float, uv));
        const float sm = block_scale(mt), sv = block_scale(vt), im = 1.0f / sm, iv = 1.0f / sv;
        uint32_t cm = 0, cv = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t h = dither(block * kAdamBlock + (uint32_t)(i % kAdamBlock) + j, s.seed);
            cm |= encode(m[j], im, h & 0xffffu) << (8 * j);
            uint32_t w = encode(root[j], iv, h >> 16);
            if (w == 0 && root[j] > 0.0f) w = 1;
            cv |= w << (8 * j);
        }
        store_codes<ALN>((uint8_t *)at[S::of(kM)] + i, left, cm);
        store_codes<ALN>((uint8_t *)at[S::of(kV)] + i, left, cv);
        if (i % kAdamBlock == 0 && left > 0) {
            *ms = sm;
            *vs = sv;
        }
    } else {
        store_n<float, 4, ALN>((float *)at[S::of(kM)] + i, left, m);
        store_n<float, 4, ALN>((float *)at[S::of(kV)] + i, left, v);
    }
}

// 1024 weights a workgroup, everything past the caches: an encoder of 31 million float weights 141 us a step (6.1 TB/s at 28 bytes a
// weight; 165 with 4096 weights and through the caches), one of 101 million with bf16 weights, masters and 8-bit state 267 us (6.1 TB/s;
// 320).  Small tensors: 4.5 us, a launch.
template <typename P, typename G, bool MASTER, bool Q8> __global__ __launch_bounds__(256) void k_adamw(const Table<MASTER, Q8> tb, const AdamStep s)
{
    using S = Slots<MASTER, Q8>;
    // the tensor of this workgroup: the last whose first workgroup is not beyond it
    int lo = 0, hi = tb.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (tb.chunk[mid] <= (int)blockIdx.x) lo = mid;
        else hi = mid - 1;
    }
    const int64_t n = tb.n[lo], first = (int64_t)((int)blockIdx.x - tb.chunk[lo]) * kAdamChunk;
    void *at[S::kCount];
    uintptr_t bits = 0;
#pragma unroll
    for (int k = 0; k < S::kCount; ++k) {
        at[k] = tb.at[lo][k];
        // four elements at a time: 16, 8 or 4 bytes
        const int a = k == kP && sizeof(P) == 2 ? 8 : k == kG && sizeof(G) == 2 ? 8 : Q8 && (k == kM || k == kV) ? 4 : 16;
        if (k < 4 || (MASTER && k == S::of(kMaster))) bits |= (uintptr_t)at[k] & (a - 1);
    }
    const float gs = s.grad_scale ? *s.grad_scale : 1.0f;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t block0 = tb.block[lo];
#pragma unroll
    for (int k = 0; k < kAdamChunk / kAdamBlock / 4; ++k) {
        const int64_t b0 = first + (int64_t)(k * 4 + wave) * kAdamBlock, i = b0 + 4 * lane;
        if (b0 >= n) break;
        const uint32_t block = block0 + (uint32_t)(b0 / kAdamBlock);
        if (bits == 0 && b0 + kAdamBlock <= n) adam_block<P, G, MASTER, Q8, true>(at, i, n, block, s, gs);
        else adam_block<P, G, MASTER, Q8, false>(at, i, n, block, s, gs);
    }
}

template <typename P, typename G, bool MASTER, bool Q8>
fs_status run(Ctx *c, const AdamStep &s, const fs_adamw_tensor *t, int32_t count)
{
    using S = Slots<MASTER, Q8>;
    uint32_t block = 0;
    int64_t done = 0;   // weights of tensor k that earlier launches have: whole workgroups
    for (int32_t k = 0; k < count;) {
        Table<MASTER, Q8> tb;
        int64_t chunks = 0;
        tb.count = 0;
        while (k < count && tb.count < Table<MASTER, Q8>::kMost && chunks < kLaunchChunks) {
            const int64_t left = t[k].n - done, n = std::min(left, (kLaunchChunks - chunks) * kAdamChunk), mine = ceil_div(n, kAdamChunk);
            if (mine) {
                const int q = tb.count++;
                void **at = tb.at[q];
                at[S::of(kP)] = (P *)t[k].p + done;
                at[S::of(kG)] = (G *)const_cast<void *>(t[k].g) + done;
                at[S::of(kM)] = (char *)t[k].m + done * (Q8 ? 1 : 4);
                at[S::of(kV)] = (char *)t[k].v + done * (Q8 ? 1 : 4);
                if constexpr (MASTER) at[S::of(kMaster)] = t[k].master + done;
                if constexpr (Q8) {
                    at[S::of(kMs)] = t[k].m_scale + done / kAdamBlock;
                    at[S::of(kVs)] = t[k].v_scale + done / kAdamBlock;
                }
                tb.n[q] = n;
                tb.chunk[q] = (int32_t)chunks;
                tb.block[q] = block;
                chunks += mine;
                block += (uint32_t)ceil_div(n, kAdamBlock);
            }
            done = n < left ? done + n : 0;
            if (n == left) ++k;
        }
        if (tb.count) k_adamw<P, G, MASTER, Q8><<<(unsigned)chunks, 256, 0, c->stream>>>(tb, s);
    }
    FS_HIP(c, hipGetLastError());
    return FS_OK;
}

template <typename P, typename G> fs_status by_state(Ctx *c, const AdamStep &s, const fs_adamw_tensor *t, int32_t count, bool master, bool q8)
{
    if (master) return q8 ? run<P, G, true, true>(c, s, t, count) : run<P, G, true, false>(c, s, t, count);
    return q8 ? run<P, G, false, true>(c, s, t, count) : run<P, G, false, false>(c, s, t, count);
}

}  // namespace

fs_status launch_adamw(Ctx *c, const fs_adamw_args *a, const fs_adamw_tensor *t, int32_t count, bool master)
{
    AdamStep s;
    const double t1 = 1.0 - pow(a->beta1, (double)a->step), t2 = 1.0 - pow(a->beta2, (double)a->step);
    s.b1 = (float)a->beta1;
    s.c1 = (float)(1.0 - a->beta1);
    s.b2 = (float)a->beta2;
    s.c2 = (float)(1.0 - a->beta2);
    s.keep = (float)(1.0 - a->lr * a->weight_decay);
    s.rate = (float)(a->lr / t1);
    s.inv = (float)(1.0 / sqrt(t2));
    s.eps = (float)a->eps;
    s.seed = a->seed;
    s.grad_scale = a->grad_scale;
    const bool q8 = a->state_bits == 8;
    if (a->p_dtype == FS_F32)
        return a->g_dtype == FS_F32 ? by_state<float, float>(c, s, t, count, false, q8) : by_state<float, __bf16>(c, s, t, count, false, q8);
    return a->g_dtype == FS_F32 ? by_state<__bf16, float>(c, s, t, count, master, q8) : by_state<__bf16, __bf16>(c, s, t, count, master, q8);
}

}  // namespace fs
