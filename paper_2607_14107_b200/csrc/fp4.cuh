// Microscaled 4-bit floating point: rows to E2M1 codes with a scale byte per group, plain rows and rows of a K/V cache.
//
//   nv   groups of 16 channels, s = E4M3(amax / 6t), nearest even, saturating at 448
//   mx   groups of 32 channels, s = 2^(floor(log2(amax / t)) - 2) as an E8M0 byte (exponent + 127)
//   code = the value of {0, .5, 1, 1.5, 2, 3, 4, 6} nearest to |x| / (s t), ties to the even code, saturating, with the sign of x
//   stored value = code s t                          (t: a factor of the whole tensor, 1 where the caller gives none)
//
// A group with an infinity or NaN gets the scale NaN (0x7f / 0xff) and zero codes: what reads it sees NaN in all of the group.  A group
// whose scale rounds to zero is zero.  All decisions are float32 with IEEE division.
//
// Bound by the copy at thousands of rows, by latency at a block of rows.  A lane holds 16 bytes of a row (4 or 8 channels), so every
// load and store of a warp is contiguous whatever the type; the lanes of a group find its maximum by shuffles.
#pragma once
#include <cuda_fp16.h>
#include <climits>

#include "tcgen05.cuh"

namespace ps {
namespace fp4 {

using namespace tc;

enum { NV = 0, MX = 1 };
enum { ROWS = 0, TILED = 1 };
constexpr int THREADS = 256;
constexpr float FAST_LO = 7.888609052210118e-31f, FAST_HI = 1.2676506002282294e30f;     // 2^-100, 2^100
__host__ __device__ constexpr int group(int fmt) { return fmt == NV ? 16 : 32; }

// Bytes of four groups x 128 rows of the tiled scales are one block of 512, what one copy into tensor memory takes: row r, group g at
// block (r / 128) * ceil(groups / 4) + g / 4, byte (r % 32) * 16 + (r % 128 / 32) * 4 + g % 4.
__device__ __forceinline__ size_t tiled_offset(long long r, int g, int g4) {
    return ((size_t)(r >> 7) * g4 + (g >> 2)) * 512 + (size_t)((r & 31) * 16 + ((r >> 5) & 3) * 4 + (g & 3));
}

// Correctly rounded quotients by a divisor b with r = RN(1 / b): q = x r is within an ulp, and one step q + (x - b q) r rounds correctly (Markstein,
// 1990) while nothing overflows or underflows: |b| and |x| within 2^-100 .. 2^100 (x = 0 too).
__device__ __forceinline__ float divide(float x, float b, float r) {
    const float q = x * r;
    return fmaf(fmaf(-b, q, x), r, q);
}
__device__ __forceinline__ bool in_range(float x) { return x >= FAST_LO && x <= FAST_HI; }

// the tensor's factor and what follows from it alone
struct Factor {
    float t, b, r;                               // b: divisor of a group's maximum (6 t or t), r = RN(1 / b)
    bool fast;
};
template <int FMT> __device__ __forceinline__ Factor make_factor(const float* p) {
    Factor f;
    f.t = p ? __ldg(p) : 1.f;
    f.b = FMT == NV ? __fmul_rn(f.t, 6.f) : f.t;
    f.r = __frcp_rn(f.b);
    f.fast = in_range(f.b);
    return f;
}
// scale of a group from the largest magnitude's bits (an integer maximum: NaN and infinity stay on top)
template <int FMT>
__device__ __forceinline__ float group_scale(uint32_t amax, const Factor& f, uint32_t* byte) {
    const float a = __uint_as_float(amax);
    float q = f.fast && in_range(a) ? divide(a, f.b, f.r) : __fdiv_rn(a, f.b);
    if (FMT == NV) {
        if (amax >= 0x7f800000u) q = __uint_as_float(0x7fc00000u);
        uint16_t e;
        uint32_t h;
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(e) : "f"(0.f), "f"(q));
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"(e));
        *byte = e;
        return __half2float(__ushort_as_half((unsigned short)h));
    }
    const int e = (int)(__float_as_uint(q) >> 23);                     // biased; 255: the quotient is beyond fp32
    const uint32_t b = amax >= 0x7f800000u ? 255u : e == 255 ? 254u : (uint32_t)max(e - 2, 0);
    *byte = b;
    return amax >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : b == 0 ? __uint_as_float(0x00400000u) : __uint_as_float(b << 23);
}

template <typename T> struct Vec;                                     // 16 bytes of a row
template <> struct Vec<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ void unpack(const uint4& w, float* v) {
        v[0] = __uint_as_float(w.x); v[1] = __uint_as_float(w.y); v[2] = __uint_as_float(w.z); v[3] = __uint_as_float(w.w);
    }
    static __device__ __forceinline__ uint32_t amax(const uint4& w) {        // bits of the largest magnitude as a float
        return max(max(w.x & 0x7fffffffu, w.y & 0x7fffffffu), max(w.z & 0x7fffffffu, w.w & 0x7fffffffu));
    }
    static __device__ __forceinline__ uint4 pack(const float* v) {
        return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    }
};
template <> struct Vec<__nv_bfloat16> {
    static constexpr int N = 8;
    static __device__ __forceinline__ void unpack(const uint4& w, float* v) {
        const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(x[i] << 16); v[2 * i + 1] = __uint_as_float(x[i] & 0xffff0000u); }
    }
    static __device__ __forceinline__ uint32_t max2(uint32_t x, uint32_t y) { uint32_t z; asm("max.u16x2 %0, %1, %2;" : "=r"(z) : "r"(x), "r"(y)); return z; }
    static __device__ __forceinline__ uint32_t amax(const uint4& w) {
        const uint32_t m = max2(max2(w.x & 0x7fff7fffu, w.y & 0x7fff7fffu), max2(w.z & 0x7fff7fffu, w.w & 0x7fff7fffu));
        return max(m << 16, m & 0xffff0000u);
    }
    static __device__ __forceinline__ uint4 pack(const float* v) {
        uint32_t x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            x[i] = *reinterpret_cast<const uint32_t*>(&b);
        }
        return make_uint4(x[0], x[1], x[2], x[3]);
    }
};

// One lane's 16 bytes of a group (all lanes of the warp take part; the lanes of a group are neighbours): the codes, four bits each, channel
// 0 lowest, the group's scale byte, and the stored values in the row's type.  The conversion to E2M1 rounds to nearest, ties to the even code, and
// saturates; groups whose unit s t is so far out that the division's steps could overflow or underflow divide by the instruction.
template <typename T, int FMT>
__device__ __forceinline__ uint32_t encode(const uint4& w, const Factor& f, uint32_t* byte, uint4* stored) {
    constexpr int N = Vec<T>::N, LANES = group(FMT) / N;
    uint32_t am = Vec<T>::amax(w);
#pragma unroll
    for (int o = 1; o < LANES; o <<= 1) am = max(am, __shfl_xor_sync(0xffffffffu, am, o));
    const float s = group_scale<FMT>(am, f, byte);
    const float u = __fmul_rn(s, f.t);
    float v[N];
    Vec<T>::unpack(w, v);
    uint32_t codes = 0;
    if (__builtin_expect(in_range(u), 1)) {
        const float r = __frcp_rn(u);
        const uint64_t r2 = f2_pack(r, r), nu = f2_pack(-u, -u);
        uint32_t c[4] = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            const uint64_t x = f2_pack(v[2 * i], v[2 * i + 1]), q = f2_mul(x, r2);
            float y0, y1;
            f2_unpack(f2_fma(f2_fma(nu, q, x), r2, q), y0, y1);
            asm("{\n .reg .b8 b;\n cvt.rn.satfinite.e2m1x2.f32 b, %2, %1;\n mov.b32 %0, {b, 0, 0, 0};\n}\n" : "=r"(c[i]) : "f"(y0), "f"(y1));
        }
        codes = c[0] | (c[1] << 8) | (c[2] << 16) | (c[3] << 24);
    } else if (s > 0.f) {
#pragma unroll
        for (int i = 0; i < N; ++i) codes |= e2m1_code(v[i], u) << (4 * i);
    }
    if (stored) {
        uint32_t h[4];
        asm("{\n .reg .b8 a, b, c, d;\n mov.b32 {a, b, c, d}, %4;\n cvt.rn.f16x2.e2m1x2 %0, a;\n cvt.rn.f16x2.e2m1x2 %1, b;\n"
            " cvt.rn.f16x2.e2m1x2 %2, c;\n cvt.rn.f16x2.e2m1x2 %3, d;\n}\n" : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(codes));
        const uint64_t s2 = f2_pack(s, s), t2 = f2_pack(f.t, f.t);
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            const float2 g = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
            f2_unpack(f2_mul(f2_mul(f2_pack(g.x, g.y), s2), t2), v[2 * i], v[2 * i + 1]);
        }
        *stored = Vec<T>::pack(v);
    }
    return codes;
}
template <typename T> __device__ __forceinline__ void store_codes(uint8_t* p, uint32_t c);
template <> __device__ __forceinline__ void store_codes<float>(uint8_t* p, uint32_t c) { *reinterpret_cast<uint16_t*>(p) = (uint16_t)c; }
template <> __device__ __forceinline__ void store_codes<__nv_bfloat16>(uint8_t* p, uint32_t c) { *reinterpret_cast<uint32_t*>(p) = c; }

struct QuantArgs {
    const void* x; long long ld_x;       // rows, elements between them
    void* deq; long long ld_deq;         // stored values (null: not wanted)
    uint8_t* codes; uint8_t* scales;
    const float* t;
    long long rows;
    int d, layout;
};

// Pieces of 16 bytes: piece i of the call is piece i % ppr of row i / ppr.  A block takes PER x THREADS consecutive ones, all loads of a
// thread in flight at once.
template <typename T, int FMT, int PER>
__global__ void __launch_bounds__(THREADS) quantize_kernel(const __grid_constant__ QuantArgs a) {
    KERNEL_PROLOGUE(20);   // fp4 quantize_kernel
    constexpr int N = Vec<T>::N, G = group(FMT);
    const int ppr = a.d / N, groups = a.d / G, g4 = (groups + 3) >> 2;
    const Factor t = make_factor<FMT>(a.t);
    const long long first = (long long)blockIdx.x * (PER * THREADS), total = a.rows * ppr;
    const long long row0 = first / ppr;
    const unsigned rem0 = (unsigned)(first - row0 * ppr);
    uint4 w[PER];
    long long row[PER];
    int c[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const unsigned loc = rem0 + i * THREADS + threadIdx.x;
        const unsigned dr = loc / (unsigned)ppr;
        row[i] = first + i * THREADS + threadIdx.x < total ? row0 + dr : -1;
        c[i] = (int)(loc - dr * ppr);
        w[i] = make_uint4(0u, 0u, 0u, 0u);
        if (row[i] >= 0) w[i] = __ldg(reinterpret_cast<const uint4*>((const T*)a.x + row[i] * a.ld_x) + c[i]);
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        uint32_t byte;
        uint4 stored;
        const uint32_t codes = encode<T, FMT>(w[i], t, &byte, a.deq ? &stored : nullptr);
        if (row[i] < 0) continue;
        store_codes<T>(a.codes + row[i] * (a.d >> 1) + c[i] * (N / 2), codes);
        if (a.deq) reinterpret_cast<uint4*>((T*)a.deq + row[i] * a.ld_deq)[c[i]] = stored;
        const int g = c[i] * N / G;
        if (c[i] * N == g * G) {
            if (a.layout == ROWS) {
                a.scales[row[i] * groups + g] = (uint8_t)byte;
            } else {
                uint8_t* at = a.scales + tiled_offset(row[i], g, g4);
                *at = (uint8_t)byte;
                if (g == groups - 1)
                    for (int z = 1; z < 4 - (g & 3); ++z) at[z] = 0;               // groups that do not exist
            }
        }
    }
    // tiled scales: rows that do not exist, up to the next 128, are zero
    if (a.layout == TILED) {
        const int pad = (int)(-a.rows & 127);
        for (long long i = (long long)blockIdx.x * THREADS + threadIdx.x; i < (long long)pad * g4; i += (long long)gridDim.x * THREADS)
            *reinterpret_cast<uint32_t*>(a.scales + tiled_offset(a.rows + i / g4, 4 * (int)(i % g4), g4)) = 0u;
    }
}

// ---- rows of a K/V cache ---------------------------------------------------------------------------------------------
struct AppendArgs {
    const void* x[2]; void* deq[2];              // K, V rows [batch][R][width], stored values of the same shape (null: not wanted)
    uint8_t* codes[2]; uint8_t* scales[2];       // [batch][cap][width / 2], [batch][cap][width / 16]
    const float* t[2];
    const int* idx; const int* counts;           // [batch][R] positions, [batch] rows listed (null: R)
    int R, cap, width, rows_per_block;
};
constexpr int APPEND_MAX_ROWS = 256;             // rows of a block

// blockIdx: x = rows_per_block rows, y = sequence, z = K or V.  A row that lists a position outside the cache is skipped, and so is one whose
// position a later row lists again: the last one listed stays, whole.
template <typename T>
__global__ void __launch_bounds__(THREADS) kv_append_kernel(const __grid_constant__ AppendArgs a) {
    KERNEL_PROLOGUE(21);   // fp4 kv_append_kernel
    constexpr int N = Vec<T>::N;
    __shared__ int pos[APPEND_MAX_ROWS];
    const int which = blockIdx.z;
    const size_t seq = blockIdx.y;
    const int count = a.counts ? min(max(a.counts[seq], 0), a.R) : a.R;
    const int r0 = (int)blockIdx.x * a.rows_per_block, r1 = min(r0 + a.rows_per_block, count);
    const int* idx = a.idx ? a.idx + seq * a.R : nullptr;
    if (r0 >= r1) {
        // (stored values of rows that are not listed are left as they were)
        return;
    }
    const int live = r1 - r0, ppr = a.width / N, total = live * ppr;
    const uint4* x = reinterpret_cast<const uint4*>((const T*)a.x[which] + (seq * a.R + r0) * a.width);
    constexpr int PER = 4;
    uint4 w[PER];
    auto load = [&](int b) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int at = b + i * THREADS + threadIdx.x;
            w[i] = at < total ? __ldg(x + at) : make_uint4(0u, 0u, 0u, 0u);
        }
    };
    load(0);                                     // (under way while the list is looked through)
    for (int i = threadIdx.x; i < live; i += THREADS) {
        const int p = idx ? idx[r0 + i] : r0 + i;
        pos[i] = p >= 0 && p < a.cap ? p : -1;
    }
    // an ascending rest of the list, as a selection writes it, has nothing twice; any other is compared entry by entry
    bool ascending = true;
    if (idx) {
        constexpr int AHEAD = 8;
        const int lane = threadIdx.x & 31;
        for (int j0 = r0 + (int)(threadIdx.x & ~31u); j0 < count; j0 += AHEAD * THREADS) {
            int v[AHEAD], last[AHEAD];           // entry j, and the entry behind the warp's last one
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const int j = j0 + i * THREADS + lane;
                v[i] = j < count ? __ldg(idx + j) : INT_MAX;
                last[i] = lane == 31 && j + 1 < count ? __ldg(idx + j + 1) : INT_MAX;
            }
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const int down = __shfl_down_sync(0xffffffffu, v[i], 1), next = lane == 31 ? last[i] : down;
                ascending = ascending && (next > v[i] || next == INT_MAX);
            }
        }
    }
    if (!__syncthreads_and(ascending)) {
        for (int j = r0 + 1 + threadIdx.x; j < count; j += THREADS) {
            const int p = __ldg(idx + j);
            for (int i = 0; i < min(live, j - r0); ++i)
                if (pos[i] == p) pos[i] = -1;        // (races only with the same store)
        }
        __syncthreads();
    }
    const Factor t = make_factor<NV>(a.t[which]);
    uint4* deq = a.deq[which] ? reinterpret_cast<uint4*>((T*)a.deq[which] + (seq * a.R + r0) * a.width) : nullptr;
    uint8_t* codes = a.codes[which] + seq * a.cap * (size_t)(a.width >> 1);
    uint8_t* scales = a.scales[which] + seq * a.cap * (size_t)(a.width >> 4);
    for (int b = 0; b < total; b += PER * THREADS) {
        if (b > 0) load(b);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if (b + i * THREADS >= total) break;     // (the same for all threads)
            const int at = b + i * THREADS + threadIdx.x;
            uint32_t byte;
            uint4 stored;
            const uint32_t cd = encode<T, NV>(w[i], t, &byte, deq ? &stored : nullptr);
            if (at >= total) continue;
            const int r = at / ppr, c = at - r * ppr, p = pos[r];
            if (deq) deq[at] = stored;
            if (p < 0) continue;
            store_codes<T>(codes + (size_t)p * (a.width >> 1) + c * (N / 2), cd);
            if ((c * N) % 16 == 0) scales[(size_t)p * (a.width >> 4) + c * N / 16] = (uint8_t)byte;
        }
    }
}

}  // namespace fp4
}  // namespace ps
