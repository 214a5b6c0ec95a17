// Bidirectional attention over a cache of keys and values held in 4 bits (NV format: E2M1 codes, an E4M3 scale per 16 channels).
//
//   s_j = q . k_j / sqrt(head_dim),  j < length of the sequence;   out = sum_j softmax(s)_j v_j,   lse = log sum_j e^(s_j)
//
// What a code and its scale stand for has six significant bits, so every key and value is exact in fp16 (and bf16); the tensors' factors are
// applied to the scores and to the finished rows.  A row without keys is zero, its lse -inf; one whose scores are all below fp32's range is NaN.
//
// kv4_attn_warp_kernel (mma.sync m16n8k16, any type, head_dim 64 or 128): for few rows, where the stream of the cache and the instructions that
// unpack it are the bound.  Sixteen keys are the 16 rows of the first operand (S^T = K Q^T) and sixteen channels of values are (O^T = V^T P^T), so
// that 8 query rows fill a product.  A warp copies its own keys' codes into a ring of its own (cp.async, no barrier), and they become operand fragments
// in registers: the order of channels inside a product is free, so a lane takes its fragments of keys from consecutive channels of a row and those of
// values from one group of channels, and a scale covers all that it multiplies.  One pass with a running maximum that moves only when it has been
// outgrown by 2^8.  About 420 instructions of a warp for 16 keys, keys and values, and 8 rows (unpacking, scaling and transposing more than products), which
// keep 57 % of the issue slots busy: registers leave 16 warps to an SM, too few to fill the rest.  One row of 28 heads, 4 K/V heads, eight ragged sequences of up to 32768 keys 32 us, joining included (85 MB: 2.6 TB/s); 32 rows
// of 32 heads over 512 keys 10.5 us, a latency chain.  fp32 rows take two terms of q and p, twice the products: the same tokens 56 us for 30000 keys.
#pragma once
#include <cuda_fp16.h>

#include "fp4.cuh"

namespace ps {
namespace kv4 {

constexpr int WARPS = 4, THREADS = WARPS * 32;
constexpr int CHUNK = 16;                        // keys a warp takes at a time
constexpr int DEPTH = 4;                         // chunks of a warp's ring
constexpr int MAX_SPLIT = 128;
constexpr int JOIN_THREADS = 128;
constexpr int MAX_BATCH = 32;                    // sequences whose parts are cut to measure (a lane each)
constexpr float SLACK = 8.f;                     // log2 of how far the running maximum may lag behind
constexpr float TERM = 4096.f;                   // the second of two fp16 terms is stored times this: at most 2^15 beside a first one of 2^15, and steps down to 2^-36
constexpr float LIFT = 7.f;                      // probabilities are 2^(s - m + LIFT): fp16 then keeps them down to 2^-31 of the largest

struct Args {
    const void* q; void* out; float* lse;        // [batch][R][n_heads * DH], the same, [batch][R][n_heads] (null: not wanted)
    const uint8_t* kc; const uint8_t* ks; const uint8_t* vc; const uint8_t* vs;
    const float* tk; const float* tv;
    const int* lens;                             // [batch] keys of every sequence (null: cap)
    float* part_o; float2* part_ml;              // partial rows: [part][batch * R * n_heads][DH], (maximum, sum)
    int* part_n;                                 // [batch] parts of every sequence (null: a part for each, rows are written at once)
    int batch, R, cap, n_heads, n_kv;
    int slots;                                   // parts per row tile and K/V head: up to MAX_BATCH sequences: at most, all of one length; beyond: the same number of each
    long long rows_total;                        // batch * R * n_heads
    double scale;                                // log2(e) / sqrt(head_dim)
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
// The part that slot number `slot` works on: sequence b with `len` keys, its part p, units of KEYS keys [t0, t0 + n).  False: there are more slots than parts.
// `tell`: the thread that writes down how many parts a sequence has.  The whole warp calls.
template <int KEYS>
__device__ __forceinline__ bool find_part(const Args& a, int slot, bool tell, int& b, int& p, int& t0, int& n, int& len) {
    const int lane = threadIdx.x & 31;
    if (a.batch > MAX_BATCH || a.slots == a.batch) {
        const int each = a.slots / a.batch;
        b = slot / each; p = slot - b * each;
        len = seq_len(a, b);
        const int all = (len + KEYS - 1) / KEYS;
        t0 = (int)((long long)all * p / each);
        n = (int)((long long)all * (p + 1) / each) - t0;
        if (tell && p == 0 && a.part_n) a.part_n[b] = each;
        return true;
    }
    // the shortest length that gives no more parts than slots, an empty sequence having one too, and none more than MAX_SPLIT
    const int my_len = lane < a.batch ? seq_len(a, lane) : 0, my = (my_len + KEYS - 1) / KEYS;
    auto parts = [&](int size) { return lane < a.batch ? max(1, (my + size - 1) / size) : 0; };
    const int longest = __reduce_max_sync(0xffffffffu, my);
    int lo = max(max(1, ((int)__reduce_add_sync(0xffffffffu, my) + a.slots - 1) / a.slots), (longest + MAX_SPLIT - 1) / MAX_SPLIT), hi = max(lo, longest);
    while (lo < hi) {
        // (one sequence, or none that ends inside a part: the first length fits)
        if ((int)__reduce_add_sync(0xffffffffu, parts(lo)) <= a.slots) break;
        const int mid = (lo + 1 + hi) >> 1;
        if ((int)__reduce_add_sync(0xffffffffu, parts(mid)) <= a.slots) hi = mid; else lo = mid;
        if (lo + 1 >= hi) { lo = hi; break; }
    }
    const int mine = parts(lo);
    int end = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const int x = __shfl_up_sync(0xffffffffu, end, o); if (lane >= o) end += x; }
    const unsigned hit = __ballot_sync(0xffffffffu, slot >= end - mine && slot < end);
    if (hit == 0) return false;
    b = __ffs(hit) - 1;
    p = slot - __shfl_sync(0xffffffffu, end - mine, b);
    const int cnt = __shfl_sync(0xffffffffu, mine, b);
    len = __shfl_sync(0xffffffffu, my_len, b);
    t0 = p * lo;
    n = min(lo, __shfl_sync(0xffffffffu, my, b) - t0);
    if (tell && p == 0 && a.part_n) a.part_n[b] = cnt;
    return true;
}

template <typename T> struct QPair;
template <> struct QPair<float> { static __device__ __forceinline__ float2 load(const float* p) { return __ldg(reinterpret_cast<const float2*>(p)); } };
template <> struct QPair<__nv_bfloat16> {
    static __device__ __forceinline__ float2 load(const __nv_bfloat16* p) {
        const uint32_t w = __ldg(reinterpret_cast<const uint32_t*>(p));
        return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    }
};

// One warp's chunk in its ring: codes of 16 key rows and 16 value rows, their scales.
template <int DH> struct Stage {
    static constexpr uint32_t K = 0, V = CHUNK * DH / 2, KS = 2 * V, VS = KS + CHUNK * DH / 16, BYTES = VS + CHUNK * DH / 16;
    // Byte offset of 16-byte piece p of a value row: with 128 channels, rows 2t and 2t + 1 share 128 bytes, and where a piece lies in them is such that
    // the lanes' reads of one row parity spread over all banks.
    static __device__ __forceinline__ uint32_t v_piece(int r, int p) {
        if (DH == 64) return (uint32_t)(r * 32 + p * 16);
        return (uint32_t)((r >> 1) * 128 + (((r ^ (r >> 2)) & 1) << 6) + ((p ^ (r & 2)) << 4));
    }
};
template <int DH, int NB> __host__ __device__ constexpr size_t warp_smem_bytes() {
    const size_t ring = (size_t)WARPS * DEPTH * Stage<DH>::BYTES, join = (size_t)WARPS * 8 * NB * (DH + 4) * 4;
    return ring > join ? ring : join;
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t a) {
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
    return d;
}

// grid: x = tile of 8 NB rows x part, y = K/V head.  Lane (g = lane / 4, t = lane % 4).
// fp32 rows: q and the probabilities are each two fp16 terms (22 bits), the second times TERM, with a product per term.  (Without that factor what is below
// 2^-25 is lost: entries of q beside much larger ones, and probabilities below 2^-32 of the largest, 65536 of which weigh 2^-16.)
template <typename T, int DH, int NB>
__global__ void __launch_bounds__(THREADS) kv4_attn_warp_kernel(const __grid_constant__ Args a) {
    pdl_trigger();
    pdl_wait();
    constexpr int TERMS = sizeof(T) == 4 ? 2 : 1, KS = DH / 16, MT = DH / 16, ROWS = 8 * NB;
    using St = Stage<DH>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ float sm[WARPS][ROWS], sl[WARPS][ROWS];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int tile = (int)blockIdx.x / a.slots, slot_no = (int)blockIdx.x - tile * a.slots, kvh = blockIdx.y;
    const int hpg = a.n_heads / a.n_kv;
    const long long vrows = (long long)hpg * a.R, vr0 = (long long)tile * ROWS;
    constexpr int STEP = WARPS * CHUNK;
    int b = 0, part = 0, t0 = 0, units = 0, len = 0;
    if (!find_part<STEP>(a, slot_no, tile == 0 && kvh == 0 && threadIdx.x == 0, b, part, t0, units, len)) return;
    const int lo = t0 * STEP, hi = min(len, lo + units * STEP);
    auto q_row = [&](long long vr) {             // virtual row -> row of [batch * R * n_heads]
        const int h = (int)(vr / a.R), r = (int)(vr - (long long)h * a.R);
        return ((size_t)b * a.R + r) * a.n_heads + kvh * hpg + h;
    };
    // ---- the ring: what this lane copies of a chunk (sixteen-byte pieces of codes, the scales of one row) ----
    constexpr int PIECES = DH / 32, COPIES = CHUNK * PIECES / 32;          // of a row; per lane, keys and values each
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem_raw) + (uint32_t)warp * (DEPTH * St::BYTES);
    const size_t row_c = (size_t)a.n_kv * (DH / 2), row_s = (size_t)a.n_kv * (DH / 16), seq0 = (size_t)b * a.cap;
    int fj = lo + warp * CHUNK;                                            // first key of the next chunk to fetch
    const uint8_t* fk = a.kc + (seq0 + fj) * row_c + kvh * (DH / 2);
    const uint8_t* fv = a.vc + (seq0 + fj) * row_c + kvh * (DH / 2);
    const uint8_t* fs = (lane < 16 ? a.ks : a.vs) + (seq0 + fj + (lane & 15)) * row_s + kvh * (DH / 16);
    size_t off[COPIES];
    uint32_t to_v[COPIES];
#pragma unroll
    for (int i = 0; i < COPIES; ++i) {
        const int x = i * 32 + lane, r = x / PIECES, p = x % PIECES;
        off[i] = (size_t)r * row_c + p * 16;
        to_v[i] = St::V + St::v_piece(r, p);
    }
    auto fetch = [&](int slot) {
        const uint32_t dst = ring + (uint32_t)slot * St::BYTES;
        if (fj + CHUNK <= hi) {
#pragma unroll
            for (int i = 0; i < COPIES; ++i) {
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + St::K + (uint32_t)((i * 32 + lane) * 16)), "l"(fk + off[i]) : "memory");
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + to_v[i]), "l"(fv + off[i]) : "memory");
            }
            if constexpr (DH == 128) asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst + St::KS + (uint32_t)lane * 8u), "l"(fs) : "memory");
            else asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst + St::KS + (uint32_t)lane * 4u), "l"(fs) : "memory");
            fj += WARPS * CHUNK;
            fk += WARPS * CHUNK * row_c; fv += WARPS * CHUNK * row_c; fs += WARPS * CHUNK * row_s;
        } else if (fj < hi) {                    // rows from the end on are zeros and not read
#pragma unroll
            for (int i = 0; i < COPIES; ++i) {
                const bool in = fj + (i * 32 + lane) / PIECES < hi;
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + St::K + (uint32_t)((i * 32 + lane) * 16)), "l"(in ? fk + off[i] : a.kc), "r"(in ? 16u : 0u) : "memory");
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + to_v[i]), "l"(in ? fv + off[i] : a.kc), "r"(in ? 16u : 0u) : "memory");
            }
            const bool in = fj + (lane & 15) < hi;
            const uint8_t* src = in ? fs : a.ks;
            if constexpr (DH == 128) asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst + St::KS + (uint32_t)lane * 8u), "l"(src), "r"(in ? 8u : 0u) : "memory");
            else asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst + St::KS + (uint32_t)lane * 4u), "l"(src), "r"(in ? 4u : 0u) : "memory");
            fj = hi;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int i = 0; i < DEPTH - 1; ++i) fetch(i);

    // ---- q as operand fragments, every row scaled by a power of two to at most 2: row g, channels t DH/4 .. ----
    uint32_t qf[TERMS][NB][KS][2];
    float unit[NB][2];                           // of rows 2t, 2t + 1: scores in units of log 2
    const float tk = a.tk ? __ldg(a.tk) : 1.f;
#pragma unroll
    for (int n = 0; n < NB; ++n) {
        const long long vr = vr0 + 8 * n + g;
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
        // (infinity or NaN in q: every score of the row is NaN, not -inf, which is a key that is not there)
        const float down = top >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : __uint_as_float((uint32_t)(254 - e) << 23), up = __uint_as_float((uint32_t)e << 23);
        const float un = (float)((double)up * (a.scale * (double)tk));
        unit[n][0] = __shfl_sync(0xffffffffu, un, 8 * t);
        unit[n][1] = __shfl_sync(0xffffffffu, un, 8 * t + 4);
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const float2 v = make_float2(x[2 * s + p].x * down, x[2 * s + p].y * down);
                const uint32_t w = pack_half(v.x, v.y);
                qf[0][n][s][p] = w;
                if (TERMS == 2) {
                    const float2 r = unpack_half(w);
                    qf[TERMS - 1][n][s][p] = pack_half((v.x - r.x) * TERM, (v.y - r.y) * TERM);
                }
            }
    }

    float o[MT][NB][4];                          // channel g DH/8 + 2 mt + (x >> 1), row 2t + (x & 1)
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int n = 0; n < NB; ++n) o[i][n][0] = o[i][n][1] = o[i][n][2] = o[i][n][3] = 0.f;
    float m[NB][2], most[NB][2], low[NB][2], l[NB][2];       // most: LIFT + SLACK, low: m - LIFT (-inf and 0 while there is no m), l: this lane's keys only
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int x = 0; x < 2; ++x) { m[n][x] = most[n][x] = -INFINITY; low[n][x] = l[n][x] = 0.f; }

    int slot = 0;
    for (int j0 = lo + warp * CHUNK; j0 < hi; j0 += WARPS * CHUNK) {
        asm volatile("cp.async.wait_group %0;" ::"n"(DEPTH - 2) : "memory");
        __syncwarp();                            // the chunk has landed for every lane, and everybody is done with the slot in front of it
        fetch(slot == 0 ? DEPTH - 1 : slot - 1);
        const uint32_t st = ring + (uint32_t)slot * St::BYTES;
        slot = slot + 1 == DEPTH ? 0 : slot + 1;
        // scores of keys g and g + 8 (rows of the product) against rows 2t, 2t + 1
        // (the tensor core's sums lose their last places towards zero: fp32 rows keep the products of q's second term and of either half of the channels apart)
        constexpr int SUMS = TERMS == 2 ? 3 : 1;
        float s[NB][4], part_s[SUMS][NB][4];
#pragma unroll
        for (int i = 0; i < SUMS; ++i)
#pragma unroll
            for (int n = 0; n < NB; ++n) part_s[i][n][0] = part_s[i][n][1] = part_s[i][n][2] = part_s[i][n][3] = 0.f;
        {
            uint32_t kw[2][DH / 32], ksc[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t row = (uint32_t)(g + 8 * i);
                if constexpr (DH == 128) {
                    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(kw[i][0]), "=r"(kw[i][1]), "=r"(kw[i][2]), "=r"(kw[i][3]) : "r"(st + St::K + row * 64u + (uint32_t)t * 16u) : "memory");
                    asm volatile("ld.shared.u16 %0, [%1];" : "=r"(ksc[i]) : "r"(st + St::KS + row * 8u + (uint32_t)t * 2u) : "memory");
                } else {
                    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(kw[i][0]), "=r"(kw[i][1]) : "r"(st + St::K + row * 32u + (uint32_t)t * 8u) : "memory");
                    asm volatile("ld.shared.u8 %0, [%1];" : "=r"(ksc[i]) : "r"(st + St::KS + row * 4u + (uint32_t)t) : "memory");
                    ksc[i] *= 0x101u;
                }
            }
            const uint32_t sp0 = scales_to_half(ksc[0]), sp1 = scales_to_half(ksc[1]);
#pragma unroll
            for (int w = 0; w < DH / 32; ++w) {
                const uint32_t sel = w < DH / 64 ? 0x1010u : 0x3232u;
                const uint32_t sc0 = __byte_perm(sp0, 0, sel), sc1 = __byte_perm(sp1, 0, sel);
                uint32_t h0[4], h1[4];
                codes_to_half(kw[0][w], h0);
                codes_to_half(kw[1][w], h1);
#pragma unroll
                for (int x = 0; x < 4; ++x) { h0[x] = h2mul(h0[x], sc0); h1[x] = h2mul(h1[x], sc1); }
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const uint32_t fa[4] = {h0[2 * y], h1[2 * y], h0[2 * y + 1], h1[2 * y + 1]};
#pragma unroll
                    for (int n = 0; n < NB; ++n)
#pragma unroll
                        for (int tm = 0; tm < TERMS; ++tm)
                            mma16816(part_s[TERMS == 1 ? 0 : tm ? 2 : (2 * w + y) / (KS / 2)][n], fa, qf[tm][n][2 * w + y][0], qf[tm][n][2 * w + y][1]);
                }
            }
        }
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int x = 0; x < 4; ++x) s[n][x] = SUMS == 1 ? part_s[0][n][x] : fmaf(part_s[SUMS - 1][n][x], 1.f / TERM, part_s[0][n][x] + part_s[SUMS / 2][n][x]);
        bool grow = false;
        float y[NB][4];                          // score - m + LIFT
        if (__builtin_expect(j0 + CHUNK > hi, 0)) {
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                if (j0 + g >= hi) s[n][0] = s[n][1] = -INFINITY;
                if (j0 + g + 8 >= hi) s[n][2] = s[n][3] = -INFINITY;
            }
        }
        auto relative = [&](int n, int x) { return s[n][x] == -INFINITY ? -INFINITY : fmaf(s[n][x], unit[n][x & 1], -low[n][x & 1]); };
#pragma unroll
        for (int n = 0; n < NB; ++n) {
#pragma unroll
            for (int x = 0; x < 4; ++x) y[n][x] = relative(n, x);
            grow |= fmaxf(y[n][0], y[n][2]) > most[n][0] || fmaxf(y[n][1], y[n][3]) > most[n][1];
        }
        if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    float nm = fmaxf(s[n][x], s[n][x + 2]);
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) nm = fmaxf(nm, __shfl_xor_sync(0xffffffffu, nm, d));
                    nm = nm == -INFINITY ? nm : nm * unit[n][x];           // (unit >= 0: the maximum commutes with it)
                    nm = nm > m[n][x] + SLACK ? nm : m[n][x];
                    const float f = m[n][x] == -INFINITY ? 0.f : ex2(m[n][x] - nm);
                    m[n][x] = nm;
                    if (nm > -INFINITY) { most[n][x] = LIFT + SLACK; low[n][x] = nm - LIFT; }
                    l[n][x] *= f;
#pragma unroll
                    for (int i = 0; i < MT; ++i) { o[i][n][x] *= f; o[i][n][x + 2] *= f; }
                    y[n][x] = relative(n, x); y[n][x + 2] = relative(n, x + 2);
                }
        }
        uint32_t pf[TERMS][NB][2];
#pragma unroll
        for (int n = 0; n < NB; ++n) {
            float p[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) p[x] = ex2(y[n][x]);
            l[n][0] += p[0] + p[2];
            l[n][1] += p[1] + p[3];
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const uint32_t w = pack_half(p[2 * y], p[2 * y + 1]);
                pf[0][n][y] = transpose8x8(w);   // keys g (+ 8), rows 2t.. -> keys 2t.. (+ 8), row g
                if (TERMS == 2) {
                    const float2 back = unpack_half(w);
                    pf[TERMS - 1][n][y] = transpose8x8(pack_half((p[2 * y] - back.x) * TERM, (p[2 * y + 1] - back.y) * TERM));
                }
            }
        }
        // values 2t, 2t + 1, 2t + 8, 2t + 9, channels g DH/8 ..: nibbles of two neighbouring rows side by side, so that one conversion gives a register
        uint32_t vw[4][DH / 64], vsc[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = 2 * t + (i & 1) + 8 * (i >> 1);
            if constexpr (DH == 128) {
                asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(vw[i][0]), "=r"(vw[i][1]) : "r"(st + St::V + St::v_piece(row, g >> 1) + (uint32_t)(g & 1) * 8u) : "memory");
                asm volatile("ld.shared.u8 %0, [%1];" : "=r"(vsc[i]) : "r"(st + St::VS + (uint32_t)(row * 8 + g)) : "memory");
            } else {
                asm volatile("ld.shared.b32 %0, [%1];" : "=r"(vw[i][0]) : "r"(st + St::V + (uint32_t)(row * 32 + g * 4)) : "memory");
                asm volatile("ld.shared.u8 %0, [%1];" : "=r"(vsc[i]) : "r"(st + St::VS + (uint32_t)(row * 4 + (g >> 1))) : "memory");
            }
        }
        const uint32_t vs0 = scales_to_half(vsc[0] | (vsc[1] << 8)), vs1 = scales_to_half(vsc[2] | (vsc[3] << 8));
#pragma unroll
        for (int w = 0; w < DH / 64; ++w) {
            uint32_t he[2][4], ho[2][4];         // even and odd channels, keys 2t.. and 2t + 8 ..
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const uint32_t r0 = vw[2 * y][w], r1 = vw[2 * y + 1][w];
                codes_to_half((r0 & 0x0f0f0f0fu) | ((r1 << 4) & 0xf0f0f0f0u), he[y]);
                codes_to_half(((r0 >> 4) & 0x0f0f0f0fu) | (r1 & 0xf0f0f0f0u), ho[y]);
            }
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const uint32_t fa[4] = {h2mul(he[0][x], vs0), h2mul(ho[0][x], vs0), h2mul(he[1][x], vs1), h2mul(ho[1][x], vs1)};
#pragma unroll
                for (int n = 0; n < NB; ++n) {
                    if (TERMS == 1) {
                        mma16816(o[4 * w + x][n], fa, pf[0][n][0], pf[0][n][1]);
                    } else {                     // (a chunk's sums by themselves, then rounded to nearest)
                        float d[4] = {0.f, 0.f, 0.f, 0.f};
                        mma16816(d, fa, pf[TERMS - 1][n][0], pf[TERMS - 1][n][1]);
#pragma unroll
                        for (int z = 0; z < 4; ++z) d[z] *= 1.f / TERM;
                        mma16816(d, fa, pf[0][n][0], pf[0][n][1]);
#pragma unroll
                        for (int z = 0; z < 4; ++z) o[4 * w + x][n][z] += d[z];
                    }
                }
            }
        }
    }

    // ---- the warps' parts of the rows together, in the ring's place ----
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
    float (*so)[ROWS][DH + 4] = reinterpret_cast<float (*)[ROWS][DH + 4]>(smem_raw);
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) l[n][x] += __shfl_xor_sync(0xffffffffu, l[n][x], d);
            if (g == 0) { sm[warp][8 * n + 2 * t + x] = m[n][x]; sl[warp][8 * n + 2 * t + x] = l[n][x]; }
#pragma unroll
            for (int i = 0; i < MT; ++i)
                *reinterpret_cast<float2*>(&so[warp][8 * n + 2 * t + x][g * (DH / 8) + 2 * i]) = make_float2(o[i][n][x], o[i][n][x + 2]);
        }
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
            const float f = sm[w][r] == -INFINITY ? (sl[w][r] == 0.f ? 0.f : 1.f) : ex2(sm[w][r] - mm);      // (nothing but NaN scores: m = -inf, l = NaN)
            const float4 x = *reinterpret_cast<const float4*>(&so[w][r][c]);
            ll += f * sl[w][r];
            acc.x += f * x.x; acc.y += f * x.y; acc.z += f * x.z; acc.w += f * x.w;
        }
        const size_t row = q_row(vr);
        if (a.part_n) {
            const size_t p = (size_t)part * a.rows_total + row;
            *reinterpret_cast<float4*>(a.part_o + p * DH + c) = acc;
            if (c == 0) a.part_ml[p] = make_float2(mm, ll);
        } else {
            if (ll == 0.f && hi > 0) ll = __uint_as_float(0x7fc00000u);       // (keys, but every score -inf; lo is 0 here)
            const float inv = ll == 0.f ? 0.f : tv / ll;
            T* out = (T*)a.out + row * DH + c;
            store_pair<T>(out, acc.x * inv, acc.y * inv);
            store_pair<T>(out + 2, acc.z * inv, acc.w * inv);
            if (c == 0 && a.lse) a.lse[row] = ll == 0.f ? -INFINITY : (mm - LIFT + log2f(ll)) * 0.6931471805599453f;
        }
    }
}

// The parts of the rows put together, a CTA per row: its warps take eight parts at a time in turn, their sums are added in the warps' order.  A latency chain
// (statistics, weights, parts, sums): 2.5 - 3 us behind the attention kernel.
template <typename T, int DH>
__global__ void __launch_bounds__(JOIN_THREADS) kv4_attn_join_kernel(const __grid_constant__ Args a) {
    pdl_trigger();
    pdl_wait();
    constexpr int PER = DH / 32, JW = JOIN_THREADS / 32;
    __shared__ float wgt[MAX_SPLIT], sum[JW][DH];
    __shared__ float red[2][JW];
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    const size_t row = blockIdx.x;
    const int seq = (int)(row / ((size_t)a.R * a.n_heads)), parts = __ldcg(a.part_n + seq);
    float2 ml = make_float2(-INFINITY, 0.f);
    static_assert(MAX_SPLIT <= JOIN_THREADS, "a part per thread");
    if (t < parts) ml = __ldcg(a.part_ml + (size_t)t * a.rows_total + row);
    const float wm = warp_max(ml.x);
    if (lane == 0) red[0][warp] = wm;
    __syncthreads();
    float mm = red[0][0];
#pragma unroll
    for (int i = 1; i < JW; ++i) mm = fmaxf(mm, red[0][i]);
    const float f = ml.x == -INFINITY ? (ml.y == 0.f ? 0.f : 1.f) : ex2(ml.x - mm);        // (a part of NaN scores keeps its NaN)
    if (t < MAX_SPLIT) wgt[t] = f;
    const float ws = warp_sum(f * ml.y);
    if (lane == 0) red[1][warp] = ws;
    __syncthreads();
    float ll = red[1][0];
#pragma unroll
    for (int i = 1; i < JW; ++i) ll += red[1][i];
    if (ll == 0.f && seq_len(a, seq) > 0) ll = __uint_as_float(0x7fc00000u);             // (keys, but every score -inf)
    float acc[PER];
#pragma unroll
    for (int c = 0; c < PER; ++c) acc[c] = 0.f;
    for (int p0 = 8 * warp; p0 < parts; p0 += 8 * JW) {
        float2 x[8][PER / 2];
        float g[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int p = p0 + i;
            g[i] = p < parts ? wgt[p] : 0.f;
            const float* src = a.part_o + ((size_t)p * a.rows_total + row) * DH + lane * PER;
#pragma unroll
            for (int c = 0; c < PER / 2; ++c) x[i][c] = p < parts ? __ldcg(reinterpret_cast<const float2*>(src) + c) : make_float2(0.f, 0.f);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int c = 0; c < PER / 2; ++c) { acc[2 * c] += g[i] * x[i][c].x; acc[2 * c + 1] += g[i] * x[i][c].y; }
    }
#pragma unroll
    for (int c = 0; c < PER; ++c) sum[warp][lane * PER + c] = acc[c];
    __syncthreads();
    const float tv = a.tv ? __ldg(a.tv) : 1.f, inv = ll == 0.f ? 0.f : tv / ll;
    if (t < DH) {
        float o = sum[0][t];
#pragma unroll
        for (int i = 1; i < JW; ++i) o += sum[i][t];
        ((T*)a.out)[row * DH + t] = from_f<T>(o * inv);
    }
    if (t == 0 && a.lse) a.lse[row] = ll == 0.f ? -INFINITY : (mm - LIFT + log2f(ll)) * 0.6931471805599453f;
}

}  // namespace kv4
}  // namespace ps
