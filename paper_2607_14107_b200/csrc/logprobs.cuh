// Log-probability of a given token, entropy and the most likely alternatives of logits rows, in one launch that reads every logit once from
// global memory (a few of them twice, from L2).
//
//   m = max x,  S = sum e^(x - m),  Q = sum e^(x - m) (x - m)
//   log p(v) = (x_v - m) - log S,   entropy = log S - Q / S       (relative to m, so that a nearly certain row keeps its small values)
//
// A thread-block cluster of up to eight CTAs per row, as in the confidence kernel; every thread carries (m, S, Q) in 32 bits and
// rescales once per batch of loads.  Alternatives: the k-th largest of the maxima of 64 groups of threads is a lower bound of the k-th largest
// logit, so only threads whose own maximum reaches it look at their logits again; what reaches the bound goes through a buffer in shared
// memory as (value, index) keys, whose order is total: larger values first, lower indices first among equals.  If the buffer overflows (many equal
// logits), its own k-th key is a higher bound, and the collection runs again; every round drops all but k of a full buffer, so it ends.
#pragma once
#include "common.cuh"

namespace ps {
namespace lpr {

constexpr int MAX_CL = 8, MAX_THREADS = 512, MAX_K = 32, SEGMENTS = 64, CAP = 1024, U = 4;

template <typename T> struct In;
template <> struct In<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ void unpack(const uint4& w, float* v) {
        v[0] = __uint_as_float(w.x); v[1] = __uint_as_float(w.y); v[2] = __uint_as_float(w.z); v[3] = __uint_as_float(w.w);
    }
    static constexpr uint32_t PAD = 0xff800000u;       // a piece that is not there: -inf
};
template <> struct In<__nv_bfloat16> {
    static constexpr int N = 8;
    static __device__ __forceinline__ void unpack(const uint4& w, float* v) {
        const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(x[i] << 16); v[2 * i + 1] = __uint_as_float(x[i] & 0xffff0000u); }
    }
    static constexpr uint32_t PAD = 0xff80ff80u;
};

struct Args {
    const void* x; long long ld;
    const int* target;
    float* logprob; float* entropy; int* top_ids; float* top_logprobs;
    int V, mask_id, k, cl;
};

// (value, index) as one integer: larger is earlier.  -0 counts as 0; NaN is never an alternative (key 0).
__device__ __forceinline__ unsigned long long make_key(float x, int v) {
    if (x != x) return 0ull;
    const uint32_t b = __float_as_uint(x + 0.f);
    const uint32_t o = (b & 0x80000000u) ? ~b : b | 0x80000000u;
    return ((unsigned long long)o << 32) | (uint32_t)~v;
}
__device__ __forceinline__ float key_value(unsigned long long k) {
    const uint32_t o = (uint32_t)(k >> 32);
    return __uint_as_float((o & 0x80000000u) ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ int key_index(unsigned long long k) { return (int)~(uint32_t)k; }

__device__ __forceinline__ float ex2(float x) { float y; asm("ex2.approx.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
constexpr float L2E = 1.4426950408889634f;

struct Run {
    float m = -INFINITY, s = 0.f, q = 0.f;
    // another part of the row
    __device__ __forceinline__ void join(float om, float os, float oq) {
        const float nm = fmaxf(m, om), ref = nm == -INFINITY ? 0.f : nm;
        const float da = fmaxf(m - ref, -1e30f), db = fmaxf(om - ref, -1e30f);        // (an empty part: factor 0, no NaN from 0 * inf)
        const float fa = expf(da), fb = expf(db);
        q = fa * (q + s * da) + fb * (oq + os * db);
        s = fa * s + fb * os;
        m = nm;
    }
};

template <typename T>
__global__ void __launch_bounds__(MAX_THREADS) token_logprobs_kernel(Args a) {
    KERNEL_PROLOGUE(22);   // token_logprobs_kernel
    constexpr int N = In<T>::N;
    __shared__ float4 parts[MAX_CL * (MAX_THREADS / 32)];
    __shared__ unsigned long long tops[MAX_CL * MAX_K];
    __shared__ unsigned long long seg[SEGMENTS];
    __shared__ unsigned long long buf[CAP];
    __shared__ unsigned long long bound_sh;
    __shared__ int n_sh;
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
    for (int i = c0 + t; i < c1; i += U * nt) {
        uint4 w[U];
#pragma unroll
        for (int u = 0; u < U; ++u) w[u] = i + u * nt < c1 ? __ldg(l4 + i + u * nt) : make_uint4(In<T>::PAD, In<T>::PAD, In<T>::PAD, In<T>::PAD);
        float bm = -INFINITY;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float v[N];
            In<T>::unpack(w[u], v);
#pragma unroll
            for (int e = 0; e < N; ++e) bm = fmaxf(bm, v[e]);
        }
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
        const float nm = fmaxf(r.m, bm), ref = nm == -INFINITY ? 0.f : nm;
        const float d = fmaxf(r.m - ref, -1e30f), f = ex2(d * L2E);
        r.q = f * (r.q + r.s * d);
        r.s *= f;
        r.m = nm;
        float s2[2] = {0.f, 0.f}, q2[2] = {0.f, 0.f};
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float v[N];
            In<T>::unpack(w[u], v);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float z = fmaxf(v[e] - ref, -1e30f);           // (-inf: e^z = 0, and 0 * z = 0)
                const float p = ex2(z * L2E);
                const float pn = v[e] == v[e] ? p : v[e];            // (the maximum of NaN and a number is the number)
                s2[e & 1] += pn;
                q2[e & 1] = fmaf(p, z, q2[e & 1]);
            }
        }
        r.s += s2[0] + s2[1];
        r.q += q2[0] + q2[1];
    }
    if (extra >= 0) r.join(x_extra, x_extra == x_extra ? (x_extra > -INFINITY ? 1.f : 0.f) : x_extra, 0.f);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        r.join(__shfl_xor_sync(0xffffffffu, r.m, o), __shfl_xor_sync(0xffffffffu, r.s, o), __shfl_xor_sync(0xffffffffu, r.q, o));

    // ---- the CTA's k largest alternatives, in order, into tops[ch * MAX_K ..] of the first CTA ----
    unsigned long long mine = 0;                         // the key that thread t < k hands on
    if (a.k > 0) {
        // lower bound from the maxima of up to 64 groups of neighbouring threads (values only: equal ones are sorted out below)
        unsigned long long key = make_key(best, 0) | 0xffffffffull;
        if (c0 + t >= c1 && extra < 0) key = 0;          // a thread without logits
        const int width = max(1, nt / SEGMENTS);         // 1, 2, 4 or 8 threads
        for (int o = 1; o < width; o <<= 1) {
            const unsigned long long other = __shfl_xor_sync(0xffffffffu, key, o);
            key = other > key ? other : key;
        }
        if (t < SEGMENTS) seg[t] = 0;
        if (t == 0) bound_sh = 0;
        __syncthreads();
        if (t % width == 0) seg[t / width] = key;
        __syncthreads();
        if (t < SEGMENTS) {
            const unsigned long long k0 = seg[t];
            int above = 0;
            for (int i = 0; i < SEGMENTS; ++i) above += seg[i] > k0 || (seg[i] == k0 && i < t);
            if (above == a.k - 1) bound_sh = k0 & 0xffffffff00000000ull;       // (values equal to it are candidates)
        }
        __syncthreads();
        unsigned long long bound = bound_sh;
        int n;
        while (true) {
            __syncthreads();
            if (t == 0) n_sh = 0;
            __syncthreads();
            auto offer = [&](float x, int v) {
                const unsigned long long k1 = make_key(x, v);
                if (v != a.mask_id && k1 >= bound && k1 != 0) {
                    const int at = atomicAdd(&n_sh, 1);
                    if (at < CAP) buf[at] = k1;
                }
            };
            // a thread whose maximum reaches the bound: its pieces are read by the lanes of its warp side by side
            const bool look = c0 + t < c1 && (make_key(best, 0) | 0xffffffffull) >= bound;
            for (unsigned todo = __ballot_sync(0xffffffffu, look); todo; todo &= todo - 1) {
                const int owner = wid * 32 + __ffs(todo) - 1;
                for (int i = c0 + owner + lane * nt; i < c1; i += 32 * nt) {
                    const uint4 w = __ldg(l4 + i);
                    float v[N];
                    In<T>::unpack(w, v);
#pragma unroll
                    for (int e = 0; e < N; ++e) offer(v[e], lead + i * N + e);
                }
            }
            if (extra >= 0) offer(x_extra, extra);
            __syncthreads();
            n = n_sh;
            if (n <= CAP) break;
            // a full buffer: its k-th key bounds the k-th of the row from below
            for (int i = t; i < CAP; i += nt) {
                const unsigned long long k0 = buf[i];
                int above = 0;
                for (int j = 0; j < CAP; ++j) above += buf[j] > k0;
                if (above == a.k - 1) bound_sh = k0;
            }
            __syncthreads();
            bound = bound_sh;
        }
        for (int i = t; i < n; i += nt) {
            const unsigned long long k0 = buf[i];
            int above = 0;
            for (int j = 0; j < n; ++j) above += buf[j] > k0;
            if (above < a.k) seg[above] = k0;            // (keys are distinct: every place is taken once)
        }
        __syncthreads();
        if (t < a.k) mine = t < n ? seg[t] : 0ull;
    }

    if (cl > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (lane == 0) {
        const uint32_t dst = dsmem_addr((uint32_t)__cvta_generic_to_shared(parts + ch * nw + wid), 0);
        asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "f"(r.m), "f"(r.s), "f"(r.q), "f"(0.f) : "memory");
    }
    if (t < a.k) {
        const uint32_t dst = dsmem_addr((uint32_t)__cvta_generic_to_shared(tops + ch * a.k + t), 0);
        asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(dst), "l"(mine) : "memory");
    }
    if (cl > 1) cluster_sync_all(); else __syncthreads();
    if (ch != 0) return;
    // every warp of the first CTA puts the parts together in the same fixed order
    Run f;
    for (int c = lane; c < cl * nw; c += 32) f.join(parts[c].x, parts[c].y, parts[c].z);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        f.join(__shfl_xor_sync(0xffffffffu, f.m, o), __shfl_xor_sync(0xffffffffu, f.s, o), __shfl_xor_sync(0xffffffffu, f.q, o));
    const float ls = logf(f.s);
    // (a row without an entry above -inf, or with an infinite one: S = 0; one with NaN: S is NaN.  All its results are NaN.)
    if (t == 0) {
        if (a.entropy) a.entropy[row] = f.s > 0.f ? fmaxf(ls - f.q / f.s, 0.f) : __uint_as_float(0x7fc00000u);
        if (a.logprob) {
            const int v = a.target[row];
            float lp = 0.f;
            if (v >= a.V) lp = __uint_as_float(0x7fc00000u);
            else if (v >= 0) lp = f.s > 0.f ? (to_f<T>(l[v]) - f.m) - ls : __uint_as_float(0x7fc00000u);
            a.logprob[row] = lp;
        }
    }
    for (int i = t; i < cl * a.k; i += nt) {
        const unsigned long long k0 = tops[i];
        int above = 0;
        for (int j = 0; j < cl * a.k; ++j) above += tops[j] > k0 || (tops[j] == k0 && j < i);
        if (above >= a.k) continue;
        const size_t at = (size_t)row * a.k + above;
        a.top_ids[at] = k0 ? key_index(k0) : -1;         // fewer alternatives than asked for
        a.top_logprobs[at] = k0 && f.s > 0.f ? (key_value(k0) - f.m) - ls : (k0 ? __uint_as_float(0x7fc00000u) : -INFINITY);
    }
}

}  // namespace lpr
}  // namespace ps
