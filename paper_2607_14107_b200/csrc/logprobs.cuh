// Log-probability of a given token, entropy and the most likely alternatives of logits rows, in one launch that reads every logit once from
// global memory (a few of them twice, from L2).
//
//   m = max x,  S = C + s = (entries equal to m) + sum of e^(x - m) over the others,  Q = sum e^(x - m) (x - m)
//   log p(v) = (x_v - m) - log S,   entropy = log S - Q / S
// Relative to m and with the entries that are m counted apart, a nearly certain row keeps its small values: log S = log C + log1p(s / C).
//
// A thread-block cluster of up to eight CTAs per row, as in the confidence kernel; every thread carries (m, C, s, Q) in 32 bits and
// rescales once per batch of loads.  Alternatives: the k-th largest of the maxima of 64 groups of threads is a lower bound of the k-th largest
// logit, so only the pieces of threads whose own maximum reaches it are read again, dealt out over the whole CTA; what reaches the bound goes through a
// buffer in shared memory as (value, index) keys, whose order is total: larger values first, lower indices first among equals.  If the buffer overflows (many equal
// logits), its own k-th key is a higher bound, and the collection runs again; every round drops all but k of a full buffer, so it ends.
//
// Bound by exponentials and instructions together with the copy at hundreds of rows, by latency at a block of rows: a phase that runs once per CTA costs about
// what its instructions cost one warp, 5 cycles and more each.  Plain / with 8 alternatives: 32 x 126464 fp32 9.5 / 12.7 us, 128 rows 16.7 / 20, 512 rows 48 (5.4 TB/s) /
// 55; 1024 x 152064 bf16 68 (4.6 TB/s) / 79, with 20 alternatives 90.  Per-batch maxima kept in shared memory, so that less is read twice: 512 rows with 32 alternatives 76 instead of
// 80, 32 rows with 8 25 instead of 13, dropped.
#pragma once
#include "tcgen05.cuh"

namespace ps {
namespace lpr {

using namespace tc;

constexpr int MAX_CL = 8, MAX_THREADS = 512, MAX_K = 32, SEGMENTS = 64, CAP = 1024, U = 4;

// Sixteen bytes of logits: unpacked as they are, unpacked with -inf as the lowest finite value (NaN stays), their largest (NaN left out), and the number of those
// that are m, which -inf takes the place of.
template <typename T> struct In;
template <> struct In<float> {
    static constexpr int N = 4;
    static constexpr uint32_t PAD = 0xff800000u;       // a piece that is not there: -inf
    static __device__ __forceinline__ void unpack(const uint4& w, float* v) {
        v[0] = __uint_as_float(w.x); v[1] = __uint_as_float(w.y); v[2] = __uint_as_float(w.z); v[3] = __uint_as_float(w.w);
    }
    static __device__ __forceinline__ void finite(const uint4& w, float* v) {
        unpack(w, v);
#pragma unroll
        for (int i = 0; i < 4; ++i) asm("max.NaN.f32 %0, %0, %1;" : "+f"(v[i]) : "f"(-3.4028234663852886e38f));
    }
    static __device__ __forceinline__ int drop1(uint32_t& x, uint32_t m) { const bool hit = x == m; x = hit ? 0xff800000u : x; return hit; }
    static __device__ __forceinline__ int drop(uint4& w, float m) {
        const uint32_t b = __float_as_uint(m);
        return drop1(w.x, b) + drop1(w.y, b) + drop1(w.z, b) + drop1(w.w, b);
    }
    static __device__ __forceinline__ float top(const uint4& w) {
        return fmaxf(fmaxf(__uint_as_float(w.x), __uint_as_float(w.y)), fmaxf(__uint_as_float(w.z), __uint_as_float(w.w)));
    }
};
template <> struct In<__nv_bfloat16> {
    static constexpr int N = 8;
    static constexpr uint32_t PAD = 0xff80ff80u;
    static __device__ __forceinline__ void spread(uint32_t x, float* v) { v[0] = __uint_as_float(x << 16); v[1] = __uint_as_float(x & 0xffff0000u); }
    static __device__ __forceinline__ void unpack(const uint4& w, float* v) { spread(w.x, v); spread(w.y, v + 2); spread(w.z, v + 4); spread(w.w, v + 6); }
    static __device__ __forceinline__ uint32_t low(uint32_t x) { uint32_t y; asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(y) : "r"(x), "r"(0xff7fff7fu)); return y; }
    static __device__ __forceinline__ void finite(const uint4& w, float* v) { spread(low(w.x), v); spread(low(w.y), v + 2); spread(low(w.z), v + 4); spread(low(w.w), v + 6); }
    static __device__ __forceinline__ int drop1(uint32_t& x, uint32_t m) {
        const bool lo = (x << 16) == m, hi = (x & 0xffff0000u) == m;
        x = lo ? (x & 0xffff0000u) | 0xff80u : x;
        x = hi ? (x & 0xffffu) | 0xff800000u : x;
        return (int)lo + (int)hi;
    }
    static __device__ __forceinline__ int drop(uint4& w, float m) {
        const uint32_t b = __float_as_uint(m);
        return drop1(w.x, b) + drop1(w.y, b) + drop1(w.z, b) + drop1(w.w, b);
    }
    static __device__ __forceinline__ uint32_t max2(uint32_t x, uint32_t y) { uint32_t z; asm("max.bf16x2 %0, %1, %2;" : "=r"(z) : "r"(x), "r"(y)); return z; }
    static __device__ __forceinline__ float top(const uint4& w) {
        const uint32_t m = max2(max2(w.x, w.y), max2(w.z, w.w));
        return fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
    }
};

struct Args {
    const void* x; long long ld;
    const int* target;
    float* logprob; float* entropy; int* top_ids; float* top_logprobs;
    int V, mask_id, k, cl;
};

// the value's place in the order of its type, as an integer (0 below all values; NaN's is not used)
__device__ __forceinline__ uint32_t order(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);         // (-0 counts as 0)
    return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
// sums over the sixteen lanes of a half warp, every lane of the warp taking part
__device__ __forceinline__ int sum16(int v) {
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ int above16(const unsigned long long* list, int n, unsigned long long key, int lane16) {
    int c = 0;
    for (int j = lane16; j < n; j += 16) c += list[j] > key;
    return sum16(c);
}
// (value, index) as one integer: larger is earlier.  -0 counts as 0; NaN is never an alternative (key 0).
__device__ __forceinline__ unsigned long long make_key(float x, int v) {
    return x != x ? 0ull : ((unsigned long long)order(x) << 32) | (uint32_t)~v;
}
__device__ __forceinline__ float key_value(unsigned long long k) {
    const uint32_t o = (uint32_t)(k >> 32);
    return __uint_as_float((o & 0x80000000u) ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ int key_index(unsigned long long k) { return (int)~(uint32_t)k; }

__device__ __forceinline__ float ex2(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
__device__ __forceinline__ float redux_max(float v) {
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}
constexpr float L2E = 1.4426950408889634f;

struct Run {
    float m = -INFINITY, c = 0.f, s = 0.f, q = 0.f;
    // another part of the row
    __device__ __forceinline__ void join(float om, float oc, float os, float oq) {
        const float nm = fmaxf(m, om), ref = nm == -INFINITY ? 0.f : nm;
        const float da = fmaxf(m - ref, -1e30f), db = fmaxf(om - ref, -1e30f);        // (an empty part: factor 0, no NaN from 0 * inf)
        const float fa = expf(da), fb = expf(db);
        q = fa * (q + (c + s) * da) + fb * (oq + (oc + os) * db);
        s = (m == nm ? s : fa * (c + s)) + (om == nm ? os : fb * (oc + os));
        c = (m == nm ? c : 0.f) + (om == nm ? oc : 0.f);
        m = nm;
    }
    __device__ __forceinline__ void join_warp() {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
            join(__shfl_xor_sync(0xffffffffu, m, o), __shfl_xor_sync(0xffffffffu, c, o), __shfl_xor_sync(0xffffffffu, s, o), __shfl_xor_sync(0xffffffffu, q, o));
    }
};

template <typename T>
__global__ void __launch_bounds__(MAX_THREADS) token_logprobs_kernel(Args a) {
    pdl_trigger();
    pdl_wait();
    constexpr int N = In<T>::N;
    __shared__ float4 parts[MAX_CL * (MAX_THREADS / 32)];
    __shared__ unsigned long long tops[MAX_CL * MAX_K];
    __shared__ uint32_t seg[SEGMENTS];
    __shared__ unsigned long long buf[CAP];
    __shared__ unsigned long long bound_sh;
    __shared__ int n_sh, own_n;
    __shared__ unsigned short own[MAX_THREADS];
    const int cl = a.cl, row = (int)blockIdx.x / cl, ch = (int)blockIdx.x - row * cl;
    // (the first CTA must run before anything is pushed into its shared memory: the barrier passes under the loads)
    if (cl > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    const int t = threadIdx.x, nt = blockDim.x, lane = t & 31, wid = t >> 5, nw = nt >> 5;
    // the row from its first 16-byte boundary on in 16-byte pieces; what lies in front and behind is the last CTA's, an element per thread
    const T* l = (const T*)a.x + (size_t)row * a.ld;
    const int lead = min(a.V, (int)(((16 - ((uintptr_t)l & 15)) & 15) / sizeof(T)));
    const int np = (a.V - lead) / N, tail = a.V - lead - np * N;
    const int per = (np + cl - 1) / cl, c0 = min(np, ch * per), c1 = min(np, c0 + per);
    const uint4* l4 = reinterpret_cast<const uint4*>(l + lead);
    const int extra = ch == cl - 1 && t < lead + tail ? (t < lead ? t : a.V - tail + (t - lead)) : -1;
    const float x_extra = extra >= 0 ? to_f<T>(l[extra]) : -INFINITY;

    Run r;
    float best = -INFINITY;                              // the largest alternative of this thread
    if (extra >= 0 && extra != a.mask_id) best = fmaxf(best, x_extra);
    for (int i = c0 + t; i - lane < c1; i += U * nt) {   // (a warp goes round together: it shares its running maximum)
        uint4 w[U];
#pragma unroll
        for (int u = 0; u < U; ++u) w[u] = i + u * nt < c1 ? __ldg(l4 + i + u * nt) : make_uint4(In<T>::PAD, In<T>::PAD, In<T>::PAD, In<T>::PAD);
        float bm = In<T>::top(w[0]);
#pragma unroll
        for (int u = 1; u < U; ++u) bm = fmaxf(bm, In<T>::top(w[u]));
        // the mask token is no alternative: only the batch that holds it looks
        float bb = bm;
        const int vm = a.mask_id - lead - i * N;
        if (a.mask_id >= 0 && vm >= 0 && vm < ((U - 1) * nt + 1) * N && vm % (nt * N) < N) {
            bb = -INFINITY;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float v[N];
                In<T>::unpack(w[u], v);
#pragma unroll
                for (int e = 0; e < N; ++e) bb = fmaxf(bb, vm == u * nt * N + e ? -INFINITY : v[e]);
            }
        }
        best = fmaxf(best, bb);
        const float wm = redux_max(bm);
        if (wm > r.m) {                                  // (rare after the first batches)
            const float d = fmaxf(r.m - wm, -1e30f), f = ex2(d * L2E);
            r.q = f * (r.q + (r.c + r.s) * d);
            r.s = f * (r.c + r.s);
            r.c = 0.f;
            r.m = wm;
        }
        if (__builtin_expect(r.m >= -1e38f, 1)) {
            if (wm == r.m) {                             // the entries that are the maximum are counted apart
                int c = 0;
#pragma unroll
                for (int u = 0; u < U; ++u) c += In<T>::drop(w[u], r.m);
                r.c += (float)c;
            }
            // -inf as the lowest finite value: p = 0 all the same, and p z = 0
            const uint64_t nm2 = f2_pack(-r.m, -r.m), l2e = f2_pack(L2E, L2E);
            uint64_t s2[2] = {0ull, 0ull}, q2[2] = {0ull, 0ull};
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float v[N];
                In<T>::finite(w[u], v);
#pragma unroll
                for (int e = 0; e < N; e += 2) {
                    const uint64_t d = f2_add(f2_pack(v[e], v[e + 1]), nm2);
                    float z0, z1;
                    f2_unpack(f2_mul(d, l2e), z0, z1);
                    const uint64_t p = f2_pack(ex2(z0), ex2(z1));
                    s2[(e >> 1) & 1] = f2_add(s2[(e >> 1) & 1], p);
                    q2[(e >> 1) & 1] = f2_fma(p, d, q2[(e >> 1) & 1]);
                }
            }
            r.s += f2_sum(f2_add(s2[0], s2[1]));
            r.q += f2_sum(f2_add(q2[0], q2[1]));
        } else {
            // nothing above the lowest values has come so far: -inf is told from them
            const float ref = r.m == -INFINITY ? 0.f : r.m;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float v[N];
                In<T>::unpack(w[u], v);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float z = fmaxf(v[e] - ref, -1e30f), p = v[e] == v[e] ? (v[e] == -INFINITY ? 0.f : ex2(z * L2E)) : v[e];
                    const bool top = v[e] == r.m && r.m > -INFINITY;
                    r.c += top ? 1.f : 0.f;
                    r.s += top ? 0.f : p;
                    r.q += p * z;
                }
            }
        }
    }
    if (extra >= 0) r.join(x_extra, x_extra > -INFINITY ? 1.f : 0.f, x_extra == x_extra ? 0.f : x_extra, 0.f);
    r.join_warp();

    // ---- the CTA's k largest alternatives: candidates in buf[0 .. n) ----
    int n = 0;
    if (a.k > 0) {
        // lower bound from the maxima of up to 64 groups of neighbouring threads (values only: equal ones are sorted out below)
        const uint32_t mine = c0 + t < c1 || extra >= 0 ? order(best) : 0u;            // (0: a thread without logits)
        uint32_t top = mine;
        const int width = max(1, nt / SEGMENTS);         // 1, 2, 4 or 8 threads
        for (int o = 1; o < width; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
        if (nt < SEGMENTS * width && t < SEGMENTS) seg[t] = 0;
        if (t == 0) { bound_sh = 0; n_sh = 0; own_n = 0; }
        __syncthreads();
        if (t % width == 0) seg[t / width] = top;
        __syncthreads();
        for (int i = t >> 4; i < SEGMENTS; i += nt >> 4) {
            const uint32_t s0 = seg[i];
            int above = 0;
#pragma unroll
            for (int j = 0; j < SEGMENTS; j += 16) { const uint32_t s1 = seg[j + (t & 15)]; above += s1 > s0 || (s1 == s0 && j + (t & 15) < i); }
            if (sum16(above) == a.k - 1 && (t & 15) == 0) bound_sh = (unsigned long long)s0 << 32;       // (values equal to it are candidates)
        }
        __syncthreads();
        unsigned long long bound = bound_sh;
        while (true) {
            auto offer = [&](float x, int v) {
                const unsigned long long k1 = make_key(x, v);
                if (v != a.mask_id && k1 >= bound && k1 != 0) {
                    const int at = atomicAdd(&n_sh, 1);
                    if (at < CAP) buf[at] = k1;
                }
            };
            // the pieces of the threads whose maximum reaches the bound, over all threads of the CTA
            if (c0 + t < c1 && mine >= (uint32_t)(bound >> 32)) own[atomicAdd(&own_n, 1)] = (unsigned short)t;
            __syncthreads();
            const int each = (c1 - c0 + nt - 1) / nt, items = own_n * each;
            constexpr int AHEAD = 4;             // loads in flight: under the stream of other rows each takes thousands of cycles
            for (int i0 = 0; i0 < items; i0 += AHEAD * nt) {
                uint4 w[AHEAD];
                int at[AHEAD];
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) {
                    at[u] = c1;
                    if (i0 + u * nt < items) {
                        const int i = i0 + u * nt + t, o = i / each;
                        if (i < items) at[u] = c0 + own[o] + (i - o * each) * nt;
                        if (at[u] < c1) w[u] = __ldg(l4 + at[u]);
                    }
                }
#pragma unroll 1
                for (int u = 0; u < AHEAD && i0 + u * nt < items; ++u) {
                    if (at[0] < c1 && order(In<T>::top(w[0])) >= (uint32_t)(bound >> 32)) {
                        float v[N];
                        In<T>::unpack(w[0], v);
#pragma unroll
                        for (int e = 0; e < N; ++e) offer(v[e], lead + at[0] * N + e);
                    }
#pragma unroll
                    for (int z = 0; z + 1 < AHEAD; ++z) { w[z] = w[z + 1]; at[z] = at[z + 1]; }
                }
            }
            if (extra >= 0) offer(x_extra, extra);
            __syncthreads();
            n = n_sh;
            if (n <= CAP) break;
            // a full buffer: its k-th key bounds the k-th of the row from below
            for (int i = t >> 4; i < CAP; i += nt >> 4) {
                const unsigned long long k0 = buf[i];
                if (above16(buf, CAP, k0, t & 15) == a.k - 1 && (t & 15) == 0) bound_sh = k0;
            }
            __syncthreads();
            bound = bound_sh;
            if (t == 0) { n_sh = 0; own_n = 0; }
            __syncthreads();
        }
    }

    // parts and alternatives, these in order, into the first CTA's shared memory
    if (cl > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (lane == 0) {
        const uint32_t dst = dsmem_addr((uint32_t)__cvta_generic_to_shared(parts + ch * nw + wid), 0);
        asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "f"(r.m), "f"(r.c), "f"(r.s), "f"(r.q) : "memory");
    }
    if (a.k > 0) {
        const uint32_t list = dsmem_addr((uint32_t)__cvta_generic_to_shared(tops + ch * a.k), 0);
        auto put = [&](int at, unsigned long long key) { asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(list + 8u * (uint32_t)at), "l"(key) : "memory"); };
        for (int i = t >> 4; i < (n + 1) / 2 * 2; i += nt >> 4) {             // (both halves of a warp, or neither)
            const unsigned long long k0 = i < n ? buf[i] : 0ull;
            const int above = above16(buf, n, k0, t & 15);
            if (i < n && above < a.k && (t & 15) == 0) put(above, k0);       // (keys are distinct: every place is taken once)
        }
        if (t >= n && t < a.k) put(t, 0ull);
    }
    if (cl > 1) cluster_sync_all(); else __syncthreads();
    if (ch != 0) return;
    // every warp of the first CTA puts the parts together in the same fixed order
    Run f;
    for (int i = lane; i < cl * nw; i += 32) f.join(parts[i].x, parts[i].y, parts[i].z, parts[i].w);
    f.join_warp();
    if (f.m > 1e30f) f.q = 0.f;          // floats there are 1e22 apart: p is 1 or 0, and Q exactly 0 (p z may have been 0 * inf)
    // (a row without an entry above -inf: C = s = 0; one with NaN: s is NaN.  These rows' results, and those of one with +inf, are all NaN.)
    const float sum = f.m < INFINITY ? f.c + f.s : __uint_as_float(0x7fc00000u), ls = f.c > 1.f ? logf(f.c) + log1pf(f.s / f.c) : log1pf(f.s);
    if (t == 0) {
        if (a.entropy) a.entropy[row] = sum > 0.f ? fmaxf(ls - f.q / sum, 0.f) : __uint_as_float(0x7fc00000u);
        if (a.logprob) {
            const int v = a.target[row];
            float lp = 0.f;
            if (v >= a.V) lp = __uint_as_float(0x7fc00000u);
            else if (v >= 0) lp = sum > 0.f ? (to_f<T>(l[v]) - f.m) - ls : __uint_as_float(0x7fc00000u);
            a.logprob[row] = lp;
        }
    }
    // Places of the CTAs' alternatives among all of them (keys of 0 are places that none took: they come last, in the order of the lists).  Few: each is
    // compared with all, by half warps; many: its own list's are in order, and in each of the others it is looked for by halving.  us, compared / looked for,
    // 32 rows x 126464: 8 x 8 of them 13.0 / 14.2, 8 x 32 23.8 / 15.2.
    const int all = cl * a.k;
    auto place = [&](int above, unsigned long long k0) {
        if (above >= a.k) return;
        const size_t at = (size_t)row * a.k + above;
        a.top_ids[at] = k0 ? key_index(k0) : -1;         // fewer alternatives than asked for
        a.top_logprobs[at] = k0 && sum > 0.f ? (key_value(k0) - f.m) - ls : (k0 ? __uint_as_float(0x7fc00000u) : -INFINITY);
    };
    if (all <= 96) {
        for (int i = t >> 4; i < (all + 1) / 2 * 2; i += nt >> 4) {
            const unsigned long long k0 = i < all ? tops[i] : 0ull;
            int above = 0;
            for (int j = t & 15; j < all; j += 16) above += tops[j] > k0 || (tops[j] == k0 && j < i);
            above = sum16(above);
            if (i < all && (t & 15) == 0) place(above, k0);
        }
    } else if (wid < cl && lane < a.k) {                 // (nt is 32 cl or more: a warp per list)
        const unsigned long long k0 = tops[wid * a.k + lane];
        int above = lane;
#pragma unroll
        for (int o = 0; o < MAX_CL; ++o) {
            if (o == wid || o >= cl) continue;
            int lo = 0;                                  // entries of the list in front of k0
#pragma unroll
            for (int step = MAX_K; step > 0; step >>= 1) {
                const int at = min(lo + step, a.k) - 1;  // (the last of the entries to skip)
                const unsigned long long x = tops[o * a.k + at];
                if (o < wid ? x >= k0 : x > k0) lo = at + 1;
            }
            above += lo;
        }
        place(above, k0);
    }
}

}  // namespace lpr
}  // namespace ps
