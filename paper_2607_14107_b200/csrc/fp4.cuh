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
// Bound by the copy at thousands of rows of fp32, by instructions at thousands of rows of bf16, by latency at a block of rows.  A lane holds 32 bytes of a row
// (8 or 16 channels); the lanes of a group find its maximum by shuffles.  (16 bytes a lane, every piece paying for its group's scale, took 205 instructions for 8
// channels of bf16: 56 us where 40 are needed now.)  24576 x 4096 fp32 to mx 125 us (6.9 TB/s), 16384 x 4096 bf16 to nv 39 us (4.4 TB/s), with the stored
// values too 52 (5.9 TB/s), 32 x 4096 2.0; 8 x 1984 rows of 4096 channels into a cache, keys and values with stored values 105 us (5.7 TB/s).
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
// 1990) while nothing overflows or underflows: |b| and |x| within 2^-100 .. 2^100 (x = 0 too) and the quotient below that, since an infinite q makes NaN of
// the correction.  (A quotient that underflows is a little off, which no scale sees: those below 2^-124 are all one byte.)
__device__ __forceinline__ float divide(float x, float b, float r) {
    const float q = x * r;
    return fmaf(fmaf(-b, q, x), r, q);
}
__device__ __forceinline__ bool in_range(float x) { return x >= FAST_LO && x <= FAST_HI; }

// the tensor's factor and what follows from it alone
struct Factor {
    float t, b, r;                               // b: divisor of a group's maximum (6 t or t), r = RN(1 / b)
    float hi;                                    // maxima up to here have ordinary quotients (-1: none, b is out of range)
};
template <int FMT> __device__ __forceinline__ Factor make_factor(const float* p) {
    Factor f;
    f.t = p ? __ldg(p) : 1.f;
    f.b = FMT == NV ? __fmul_rn(f.t, 6.f) : f.t;
    f.r = __frcp_rn(f.b);
    f.hi = in_range(f.b) ? fminf(FAST_HI, f.b * FAST_HI) : -1.f;
    return f;
}
// scale of a group from the largest magnitude's bits (an integer maximum: NaN and infinity stay on top)
template <int FMT>
__device__ __forceinline__ float group_scale(uint32_t amax, const Factor& f, uint32_t* byte) {
    const float a = __uint_as_float(amax);
    float q = a >= FAST_LO && a <= f.hi ? divide(a, f.b, f.r) : __fdiv_rn(a, f.b);
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

// One lane's piece of a row: 32 bytes of it, a group's worth or less, so that what a group costs once (its maximum, scale and reciprocal) is paid by as few
// lanes as may be.  All lanes of the warp take part; the lanes of a group are neighbours.  Results: the codes, four bits each, channel 0 lowest, the group's
// scale byte, and the stored values in the row's type.  The conversion to E2M1 rounds to nearest, ties to the even code, and saturates.  Groups whose unit
// s t is far out divide by the instruction, and so do those whose maximum is far above the factor: s saturates there, and a quotient beyond fp32 would make NaN
// of the division's last step, which converts to +6 whatever the sign.  (Elsewhere |x| is below 9 s t, the least s of nv being half the wanted one at worst; an |x| so
// small that the steps underflow is below half a code.)
template <typename T> struct Piece {
    static constexpr int N = 2 * Vec<T>::N, WORDS = N / 8;                 // channels, words of codes
    uint4 w[2];
    __device__ __forceinline__ void clear() { w[0] = w[1] = make_uint4(0u, 0u, 0u, 0u); }
    __device__ __forceinline__ void load(const uint4* p) { w[0] = __ldg(p); w[1] = __ldg(p + 1); }
};
template <typename T, int FMT>
__device__ __forceinline__ void encode(const Piece<T>& x, const Factor& f, uint32_t (&codes)[Piece<T>::WORDS], uint32_t* byte, Piece<T>* stored) {
    constexpr int N = Piece<T>::N, LANES = group(FMT) / N, H = Vec<T>::N;
    uint32_t am = max(Vec<T>::amax(x.w[0]), Vec<T>::amax(x.w[1]));
#pragma unroll
    for (int o = 1; o < LANES; o <<= 1) am = max(am, __shfl_xor_sync(0xffffffffu, am, o));
    const float s = group_scale<FMT>(am, f, byte);
    const float u = __fmul_rn(s, f.t);
    float v[N];
    Vec<T>::unpack(x.w[0], v);
    Vec<T>::unpack(x.w[1], v + H);
#pragma unroll
    for (int h = 0; h < Piece<T>::WORDS; ++h) codes[h] = 0u;
    if (__builtin_expect(in_range(u) && __uint_as_float(am) <= f.hi, 1)) {
        const float r = __frcp_rn(u);
        const uint64_t r2 = f2_pack(r, r), nu = f2_pack(-u, -u);
#pragma unroll
        for (int h = 0; h < Piece<T>::WORDS; ++h) {
            float y[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint64_t z = f2_pack(v[8 * h + 2 * i], v[8 * h + 2 * i + 1]), q = f2_mul(z, r2);
                f2_unpack(f2_fma(f2_fma(nu, q, z), r2, q), y[2 * i], y[2 * i + 1]);
            }
            asm("{\n .reg .b8 a, b, c, d;\n cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n"
                " cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n mov.b32 %0, {a, b, c, d};\n}\n"
                : "=r"(codes[h]) : "f"(y[0]), "f"(y[1]), "f"(y[2]), "f"(y[3]), "f"(y[4]), "f"(y[5]), "f"(y[6]), "f"(y[7]));
        }
    } else if (s > 0.f) {
#pragma unroll
        for (int i = 0; i < N; ++i) codes[i >> 3] |= e2m1_code(v[i], u) << (4 * (i & 7));
    }
    if (stored) {
        const uint64_t s2 = f2_pack(s, s), t2 = f2_pack(f.t, f.t);
#pragma unroll
        for (int k = 0; k < Piece<T>::WORDS; ++k) {
            uint32_t h[4];
            asm("{\n .reg .b8 a, b, c, d;\n mov.b32 {a, b, c, d}, %4;\n cvt.rn.f16x2.e2m1x2 %0, a;\n cvt.rn.f16x2.e2m1x2 %1, b;\n"
                " cvt.rn.f16x2.e2m1x2 %2, c;\n cvt.rn.f16x2.e2m1x2 %3, d;\n}\n" : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(codes[k]));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 g = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
                f2_unpack(f2_mul(f2_mul(f2_pack(g.x, g.y), s2), t2), v[8 * k + 2 * i], v[8 * k + 2 * i + 1]);
            }
        }
        stored->w[0] = Vec<T>::pack(v);
        stored->w[1] = Vec<T>::pack(v + H);
    }
}
// (codes are 4-byte aligned)
__device__ __forceinline__ void store_codes(uint8_t* p, const uint32_t (&c)[1]) { *reinterpret_cast<uint32_t*>(p) = c[0]; }
__device__ __forceinline__ void store_codes(uint8_t* p, const uint32_t (&c)[2]) {
    if (((uintptr_t)p & 7) == 0) *reinterpret_cast<uint2*>(p) = make_uint2(c[0], c[1]);
    else { reinterpret_cast<uint32_t*>(p)[0] = c[0]; reinterpret_cast<uint32_t*>(p)[1] = c[1]; }
}

struct QuantArgs {
    const void* x; long long ld_x;       // rows, elements between them
    void* deq;                           // stored values, dense rows (null: not wanted)
    uint8_t* codes; uint8_t* scales;
    const float* t;
    long long rows;
    int d, layout;
};

// Piece i of the call is piece i % ppr of row i / ppr.  A block takes PER x THREADS consecutive ones, all loads of a thread in flight at once.
template <typename T, int FMT, int PER>
__global__ void __launch_bounds__(THREADS) quantize_kernel(const __grid_constant__ QuantArgs a) {
    pdl_trigger();
    pdl_wait();
    constexpr int N = Piece<T>::N, G = group(FMT);
    const int ppr = a.d / N, groups = a.d / G, g4 = (groups + 3) >> 2;
    const Factor t = make_factor<FMT>(a.t);
    const long long first = (long long)blockIdx.x * (PER * THREADS), total = a.rows * ppr;
    const long long row0 = first / ppr;
    const unsigned rem0 = (unsigned)(first - row0 * ppr);
    // quotients of numbers below ppr + PER * THREADS by ppr: 0 or 1 where ppr is that large, else a product with the rounded-up reciprocal (numbers and
    // divisor below 2^12: exact)
    const bool wide = ppr >= PER * THREADS;
    const unsigned inv = 0xffffffffu / (unsigned)ppr + 1u;                 // (ppr is 2 or more)
    Piece<T> x[PER];
    long long row[PER];
    int c[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const unsigned loc = rem0 + i * THREADS + threadIdx.x;
        const unsigned dr = wide ? (loc >= (unsigned)ppr ? 1u : 0u) : __umulhi(loc, inv);
        row[i] = first + i * THREADS + threadIdx.x < total ? row0 + dr : -1;
        c[i] = (int)(loc - dr * ppr);
        x[i].clear();
        if (row[i] >= 0) x[i].load(reinterpret_cast<const uint4*>((const T*)a.x + row[i] * a.ld_x) + 2 * c[i]);
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        uint32_t byte, codes[Piece<T>::WORDS];
        Piece<T> stored;
        encode<T, FMT>(x[i], t, codes, &byte, a.deq ? &stored : nullptr);
        if (row[i] < 0) continue;
        store_codes(a.codes + row[i] * (a.d >> 1) + c[i] * (N / 2), codes);
        if (a.deq) {
            uint4* to = reinterpret_cast<uint4*>((T*)a.deq + row[i] * a.d) + 2 * c[i];
            to[0] = stored.w[0];
            to[1] = stored.w[1];
        }
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
    // tiled scales: rows that do not exist, up to the next 128, are zero.  A warp takes a block, a lane the rows lane, lane + 32, + 64, + 96: 16 bytes
    const int n = (int)(a.rows & 127);
    if (a.layout == TILED && n != 0) {
        const int lane = threadIdx.x & 31, k0 = max(0, (n - lane + 31) >> 5);
        const bool whole = k0 == 0 && ((uintptr_t)a.scales & 15) == 0;
        for (long long q = (long long)blockIdx.x * (THREADS / 32) + (threadIdx.x >> 5); q < g4; q += (long long)gridDim.x * (THREADS / 32)) {
            uint32_t* at = reinterpret_cast<uint32_t*>(a.scales + ((a.rows >> 7) * g4 + q) * 512) + 4 * lane;
            if (whole) *reinterpret_cast<uint4*>(at) = make_uint4(0u, 0u, 0u, 0u);
            else for (int k = k0; k < 4; ++k) at[k] = 0u;
        }
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
    pdl_trigger();
    pdl_wait();
    constexpr int N = Piece<T>::N;
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
    constexpr int PER = 2;
    Piece<T> w[PER];
    auto load = [&](int b) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int at = b + i * THREADS + threadIdx.x;
            w[i].clear();
            if (at < total) w[i].load(x + 2 * at);
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
            uint32_t byte, cd[Piece<T>::WORDS];
            Piece<T> stored;
            encode<T, NV>(w[i], t, cd, &byte, deq ? &stored : nullptr);
            if (at >= total) continue;
            const int r = at / ppr, c = at - r * ppr, p = pos[r];
            if (deq) { deq[2 * at] = stored.w[0]; deq[2 * at + 1] = stored.w[1]; }
            if (p < 0) continue;
            store_codes(codes + (size_t)p * (a.width >> 1) + c * (N / 2), cd);
            if ((c * N) % 16 == 0) scales[(size_t)p * (a.width >> 4) + c * N / 16] = (uint8_t)byte;
        }
    }
}

}  // namespace fp4
}  // namespace ps
