// Bidirectional attention over a cache of keys and values held in 4 bits (NV format: E2M1 codes, an E4M3 scale per 16 channels).
//
//   s_j = q . k_j / sqrt(head_dim),  j < length of the sequence;   out = sum_j softmax(s)_j v_j,   lse = log sum_j e^(s_j)
//
// What a code and its scale stand for has six significant bits, so every key and value is exact in fp16 (and bf16); the tensors' factors are
// applied to the scores and to the finished rows.  A row without keys is zero, its lse -inf.
//
// kv4_attn_warp_kernel (mma.sync m16n8k16, any type, head_dim 64 or 128): codes go from global memory to registers and become operand fragments
// there, without passing through shared memory.  The order of channels inside a product is free, so a lane takes the fragments of keys from
// consecutive channels of one row, and those of values from one group of 16 channels: its loads are 4 to 16 bytes, and a scale covers all
// that it multiplies.  One pass with a running maximum that moves only when it has been outgrown by 2^8.
#pragma once
#include <cuda_fp16.h>

#include "fp4.cuh"

namespace ps {
namespace kv4 {

constexpr int ROWS = 16;                         // query rows of a CTA: rows of all heads that share a K/V head form one list, head-major
constexpr int WARPS = 4, THREADS = WARPS * 32;
constexpr int CHUNK = 16;                        // keys a warp takes at a time
constexpr int MAX_SPLIT = 64;
constexpr float SLACK = 8.f;                     // log2 of how far the running maximum may lag behind
constexpr float LIFT = 7.f;                      // probabilities are 2^(s - m + LIFT): fp16 then keeps them down to 2^-31 of the largest

struct Args {
    const void* q; void* out; float* lse;        // [batch][R][n_heads * DH], the same, [batch][R][n_heads] (null: not wanted)
    const uint8_t* kc; const uint8_t* ks; const uint8_t* vc; const uint8_t* vs;
    const float* tk; const float* tv;
    const int* lens;                             // [batch] keys of every sequence (null: cap)
    float* part_o; float2* part_ml;              // partial rows: [split][batch * R * n_heads][DH], (maximum, sum)
    int R, cap, n_heads, n_kv, split;
    long long rows_total;                        // batch * R * n_heads
    float scale;
};

__device__ __forceinline__ float ex2(float x) { float y; asm("ex2.approx.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
__device__ __forceinline__ uint32_t h2mul(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// eight codes -> four fp16 pairs (grid values)
__device__ __forceinline__ void codes_to_half(uint32_t w, uint32_t* h) {
    asm("{\n .reg .b8 a, b, c, d;\n mov.b32 {a, b, c, d}, %4;\n cvt.rn.f16x2.e2m1x2 %0, a;\n cvt.rn.f16x2.e2m1x2 %1, b;\n"
        " cvt.rn.f16x2.e2m1x2 %2, c;\n cvt.rn.f16x2.e2m1x2 %3, d;\n}\n" : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(w));
}
// two E4M3 bytes -> fp16 pair
__device__ __forceinline__ uint32_t scales_to_half(uint32_t b) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)b));
    return r;
}
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float2 unpack_half(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }

__device__ __forceinline__ int seq_len(const Args& a, int b) { return a.lens ? min(max(__ldg(a.lens + b), 0), a.cap) : a.cap; }
// keys [lo, hi) of part s of a sequence: whole chunks
__device__ __forceinline__ void key_range(int len, int split, int s, int& lo, int& hi) {
    const int chunks = (len + CHUNK - 1) / CHUNK;
    lo = min(len, (int)((long long)chunks * s / split) * CHUNK);
    hi = min(len, (int)((long long)chunks * (s + 1) / split) * CHUNK);
}

// the fragments' source words of one chunk
template <int DH> struct Codes {
    uint32_t k[2][DH / 32], ksc[2];              // two key rows: DH / 4 channels each, their scale bytes
    uint32_t v[4][DH / 64], vsc[4];              // four value rows: DH / 8 channels each, the scale byte of their group
};
template <int N> __device__ __forceinline__ void load_words(const uint8_t* p, uint32_t (&w)[N]) {
    if constexpr (N == 4) { const uint4 x = __ldg(reinterpret_cast<const uint4*>(p)); w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w; }
    else if constexpr (N == 2) { const uint2 x = __ldg(reinterpret_cast<const uint2*>(p)); w[0] = x.x; w[1] = x.y; }
    else w[0] = __ldg(reinterpret_cast<const uint32_t*>(p));
}
// Lane (g = lane / 4, t = lane % 4): keys g and g + 8, channels t DH/4 ..; values 2t, 2t + 1, 2t + 8, 2t + 9, channels g DH/8 ..
// Rows from `hi` on are zeros (nothing is read there, whatever it holds).
template <int DH>
__device__ __forceinline__ void load_chunk(Codes<DH>& c, const Args& a, size_t row0, int j0, int hi, int g, int t, int kvh) {
    const size_t stride_c = (size_t)a.n_kv * (DH / 2), stride_s = (size_t)a.n_kv * (DH / 16);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int j = j0 + g + 8 * i;
#pragma unroll
        for (int w = 0; w < DH / 32; ++w) c.k[i][w] = 0u;
        c.ksc[i] = 0u;
        if (j < hi) {
            load_words(a.kc + (row0 + j) * stride_c + kvh * (DH / 2) + t * (DH / 8), c.k[i]);
            const uint8_t* s = a.ks + (row0 + j) * stride_s + kvh * (DH / 16) + t * (DH / 64);
            c.ksc[i] = DH == 128 ? (uint32_t)__ldg(reinterpret_cast<const uint16_t*>(s)) : (uint32_t)__ldg(s) * 0x101u;
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int j = j0 + 2 * t + (i & 1) + 8 * (i >> 1);
#pragma unroll
        for (int w = 0; w < DH / 64; ++w) c.v[i][w] = 0u;
        c.vsc[i] = 0u;
        if (j < hi) {
            load_words(a.vc + (row0 + j) * stride_c + kvh * (DH / 2) + g * (DH / 16), c.v[i]);
            c.vsc[i] = __ldg(a.vs + (row0 + j) * stride_s + kvh * (DH / 16) + g * (DH / 8) / 16);
        }
    }
}

template <typename T> struct QPair;
template <> struct QPair<float> { static __device__ __forceinline__ float2 load(const float* p) { return __ldg(reinterpret_cast<const float2*>(p)); } };
template <> struct QPair<__nv_bfloat16> {
    static __device__ __forceinline__ float2 load(const __nv_bfloat16* p) {
        const uint32_t w = __ldg(reinterpret_cast<const uint32_t*>(p));
        return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    }
};

// grid: x = tile of rows x part of the keys, y = K/V head, z = sequence.
// fp32 rows: q and the probabilities are each two fp16 terms (22 bits), with a product per term.
template <typename T, int DH>
__global__ void __launch_bounds__(THREADS) kv4_attn_warp_kernel(const __grid_constant__ Args a) {
    KERNEL_PROLOGUE(23);   // kv4_attn_warp_kernel
    constexpr int TERMS = sizeof(T) == 4 ? 2 : 1, KS = DH / 16, NT = DH / 8;
    __shared__ float so[WARPS][ROWS][DH + 4];
    __shared__ float sm[WARPS][ROWS], sl[WARPS][ROWS];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int tile = (int)blockIdx.x / a.split, part = (int)blockIdx.x - tile * a.split, kvh = blockIdx.y, b = blockIdx.z;
    const int hpg = a.n_heads / a.n_kv;
    const long long vrows = (long long)hpg * a.R, vr0 = (long long)tile * ROWS;
    const int len = seq_len(a, b);
    int lo, hi;
    key_range(len, a.split, part, lo, hi);
    const size_t row0 = (size_t)b * a.cap;
    auto q_row = [&](long long vr) {             // virtual row -> row of [batch * R * n_heads]
        const int h = (int)(vr / a.R), r = (int)(vr - (long long)h * a.R);
        return ((size_t)b * a.R + r) * a.n_heads + kvh * hpg + h;
    };

    // q as operand fragments, every row scaled by a power of two to at most 2
    uint32_t qf[TERMS][KS][4];
    float unit[2];                               // of rows g and g + 8: scores in units of log 2
    const float tk = a.tk ? __ldg(a.tk) : 1.f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const long long vr = vr0 + g + 8 * i;
        const T* q = (const T*)a.q + (vr < vrows ? q_row(vr) : 0) * DH + t * (DH / 4);
        float2 x[DH / 8];
        uint32_t top = 0;
#pragma unroll
        for (int c = 0; c < DH / 8; ++c) {
            x[c] = vr < vrows ? QPair<T>::load(q + 2 * c) : make_float2(0.f, 0.f);
            top = max(top, max(__float_as_uint(x[c].x) & 0x7fffffffu, __float_as_uint(x[c].y) & 0x7fffffffu));
        }
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const int e = min(max((int)(top >> 23), 1), 253);          // biased exponent of the largest magnitude
        const float down = __uint_as_float((uint32_t)(254 - e) << 23), up = __uint_as_float((uint32_t)e << 23);
        unit[i] = up * (a.scale * 1.4426950408889634f * tk);
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const float2 v = make_float2(x[2 * s + p].x * down, x[2 * s + p].y * down);
                const uint32_t w = pack_half(v.x, v.y);
                qf[0][s][2 * p + i] = w;
                if (TERMS == 2) {
                    const float2 r = unpack_half(w);
                    qf[TERMS - 1][s][2 * p + i] = pack_half(v.x - r.x, v.y - r.y);
                }
            }
    }

    float o[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n) { o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f; }
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};       // l: this lane's columns only

    Codes<DH> cur, nxt;
    int j0 = lo + warp * CHUNK;
    if (j0 < hi) load_chunk<DH>(cur, a, row0, j0, hi, g, t, kvh);
    for (; j0 < hi; j0 += WARPS * CHUNK) {
        const int jn = j0 + WARPS * CHUNK;
        if (jn < hi) load_chunk<DH>(nxt, a, row0, jn, hi, g, t, kvh);
        float s[2][4];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            s[i][0] = s[i][1] = s[i][2] = s[i][3] = 0.f;
            const uint32_t sp = scales_to_half(cur.ksc[i]);
            const uint32_t s0 = __byte_perm(sp, 0, 0x1010), s1 = __byte_perm(sp, 0, 0x3232);
#pragma unroll
            for (int w = 0; w < DH / 32; ++w) {
                uint32_t h[4];
                codes_to_half(cur.k[i][w], h);
                const uint32_t sc = w < DH / 64 ? s0 : s1;
#pragma unroll
                for (int x = 0; x < 4; ++x) h[x] = h2mul(h[x], sc);
#pragma unroll
                for (int tm = 0; tm < TERMS; ++tm) {
                    mma16816(s[i], qf[tm][2 * w], h[0], h[1]);
                    mma16816(s[i], qf[tm][2 * w + 1], h[2], h[3]);
                }
            }
        }
        // columns of s[i]: keys j0 + 8 i + 2 t, + 1; [0], [1]: row g, [2], [3]: row g + 8
        float top[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            top[r] = -INFINITY;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    float& v = s[i][2 * r + x];
                    v = j0 + 8 * i + 2 * t + x < hi ? v * unit[r] : -INFINITY;
                    top[r] = fmaxf(top[r], v);
                }
        }
        if (__any_sync(0xffffffffu, top[0] > m[0] + SLACK || top[1] > m[1] + SLACK)) {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                float nm = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], 1));
                nm = fmaxf(nm, __shfl_xor_sync(0xffffffffu, nm, 2));
                nm = nm > m[r] + SLACK ? nm : m[r];
                const float f = m[r] == -INFINITY ? 0.f : ex2(m[r] - nm);
                m[r] = nm;
                l[r] *= f;
#pragma unroll
                for (int n = 0; n < NT; ++n) { o[n][2 * r] *= f; o[n][2 * r + 1] *= f; }
            }
        }
        uint32_t pf[TERMS][4];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const float base = m[r] == -INFINITY ? 0.f : m[r] - LIFT;      // (nothing but -inf so far: p = 0)
                const float p0 = ex2(s[i][2 * r] - base), p1 = ex2(s[i][2 * r + 1] - base);
                l[r] += p0 + p1;
                const uint32_t w = pack_half(p0, p1);
                pf[0][2 * i + r] = w;
                if (TERMS == 2) {
                    const float2 back = unpack_half(w);
                    pf[TERMS - 1][2 * i + r] = pack_half(p0 - back.x, p1 - back.y);
                }
            }
        // values: nibbles of two neighbouring rows side by side, so that one conversion gives a fragment register
        const uint32_t vs0 = scales_to_half(cur.vsc[0] | (cur.vsc[1] << 8)), vs1 = scales_to_half(cur.vsc[2] | (cur.vsc[3] << 8));
#pragma unroll
        for (int w = 0; w < DH / 64; ++w) {
            uint32_t b0[8], b1[8];
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const uint32_t r0 = cur.v[2 * y][w], r1 = cur.v[2 * y + 1][w];
                const uint32_t even = (r0 & 0x0f0f0f0fu) | ((r1 << 4) & 0xf0f0f0f0u), odd = ((r0 >> 4) & 0x0f0f0f0fu) | (r1 & 0xf0f0f0f0u);
                uint32_t he[4], ho[4];
                codes_to_half(even, he);
                codes_to_half(odd, ho);
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    (y ? b1 : b0)[2 * x] = h2mul(he[x], y ? vs1 : vs0);
                    (y ? b1 : b0)[2 * x + 1] = h2mul(ho[x], y ? vs1 : vs0);
                }
            }
#pragma unroll
            for (int x = 0; x < 8; ++x)
#pragma unroll
                for (int tm = 0; tm < TERMS; ++tm) mma16816(o[8 * w + x], pf[tm], b0[x], b1[x]);
        }
        cur = nxt;
    }

    // ---- the warps' parts of the rows together: tile n's column c is channel c DH/8 + n ----
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
        l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
        if (t == 0) { sm[warp][g + 8 * r] = m[r]; sl[warp][g + 8 * r] = l[r]; }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int x = 0; x < 4; ++x) so[warp][g + 8 * (x >> 1)][(2 * t + (x & 1)) * (DH / 8) + n] = o[n][x];
    __syncthreads();
    const float tv = a.tv ? __ldg(a.tv) : 1.f;
    for (int i = threadIdx.x; i < ROWS * (DH / 4); i += THREADS) {
        const int r = i / (DH / 4), c = (i - r * (DH / 4)) * 4;
        const long long vr = vr0 + r;
        if (vr >= vrows) continue;
        float mm = -INFINITY;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) mm = fmaxf(mm, sm[w][r]);
        float ll = 0.f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < WARPS; ++w) {
            const float f = sm[w][r] == -INFINITY ? (sl[w][r] == 0.f ? 0.f : 1.f) : ex2(sm[w][r] - mm);
            const float4 x = *reinterpret_cast<const float4*>(&so[w][r][c]);
            ll += f * sl[w][r];
            acc.x += f * x.x; acc.y += f * x.y; acc.z += f * x.z; acc.w += f * x.w;
        }
        const size_t row = q_row(vr);
        if (a.split > 1) {
            const size_t p = (size_t)part * a.rows_total + row;
            *reinterpret_cast<float4*>(a.part_o + p * DH + c) = acc;
            if (c == 0) a.part_ml[p] = make_float2(mm, ll);
        } else {
            const float inv = ll == 0.f ? 0.f : tv / ll;
            T* out = (T*)a.out + row * DH + c;
            store_pair<T>(out, acc.x * inv, acc.y * inv);
            store_pair<T>(out + 2, acc.z * inv, acc.w * inv);
            if (c == 0 && a.lse) a.lse[row] = ll == 0.f ? -INFINITY : (mm - LIFT + log2f(ll)) * 0.6931471805599453f;
        }
    }
}

// The parts of the rows put together in their order; a warp per row.
template <typename T, int DH>
__global__ void __launch_bounds__(256) kv4_attn_join_kernel(const __grid_constant__ Args a) {
    KERNEL_PROLOGUE(24);   // kv4_attn_join_kernel
    constexpr int PER = DH / 32;
    const int lane = threadIdx.x & 31;
    const long long row = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (row >= a.rows_total) return;
    float2 ml[MAX_SPLIT / 32];
    float mm = -INFINITY;
#pragma unroll
    for (int i = 0; i < MAX_SPLIT / 32; ++i) {
        const int p = i * 32 + lane;
        ml[i] = p < a.split ? __ldcg(a.part_ml + (size_t)p * a.rows_total + row) : make_float2(-INFINITY, 0.f);
        mm = fmaxf(mm, ml[i].x);
    }
    mm = warp_max(mm);
    float ll = 0.f;
#pragma unroll
    for (int i = 0; i < MAX_SPLIT / 32; ++i) {
        ml[i].x = ml[i].x == -INFINITY ? (ml[i].y == 0.f ? 0.f : 1.f) : ex2(ml[i].x - mm);        // (a part of NaN scores keeps its NaN)
        ll += ml[i].x * ml[i].y;
    }
    ll = warp_sum(ll);
    float acc[PER];
#pragma unroll
    for (int c = 0; c < PER; ++c) acc[c] = 0.f;
    for (int p = 0; p < a.split; ++p) {
        const float f = __shfl_sync(0xffffffffu, p < 32 ? ml[0].x : ml[MAX_SPLIT / 32 - 1].x, p & 31);
        const float* src = a.part_o + ((size_t)p * a.rows_total + row) * DH + lane * PER;
#pragma unroll
        for (int c = 0; c < PER; c += 2) {
            const float2 x = __ldcg(reinterpret_cast<const float2*>(src + c));
            acc[c] += f * x.x; acc[c + 1] += f * x.y;
        }
    }
    const float tv = a.tv ? __ldg(a.tv) : 1.f, inv = ll == 0.f ? 0.f : tv / ll;
    T* out = (T*)a.out + (size_t)row * DH + lane * PER;
#pragma unroll
    for (int c = 0; c < PER; c += 2) store_pair<T>(out + c, acc[c] * inv, acc[c + 1] * inv);
    if (lane == 0 && a.lse) a.lse[row] = ll == 0.f ? -INFINITY : (mm - LIFT + log2f(ll)) * 0.6931471805599453f;
}

}  // namespace kv4
}  // namespace ps
