// The attention of kv4_attn.cuh on 5th-generation tensor cores: bf16 rows, head_dim 128, many rows.
//
//   rows     the query rows of all heads that share a K/V head form one list (head-major), cut into tiles of 128
//   streams  two per CTA, whose softmax and products alternate.  ROW SPLIT: a row tile each, every key tile serves both.  KEY SPLIT (one row
//            tile in all): the streams take the even and the odd key tiles, and their rows are put together at the end
//   codes    four warps turn the codes of a tile of 128 keys into fp16 rows in the operand layout (128-byte swizzle).  A warp has its own 32 keys:
//            it copies their codes and scales into a staging area of its own (cp.async, two tiles ahead, no barrier), so that the work of a tile is
//            16 conversions, 16 products and four 16-byte stores for every 32 channels
//   scores   S = Q K^T in tensor memory; four warps per stream, one thread per row, keep a running maximum m and sum and write p = 2^(s - m + LIFT),
//            rounded to fp16, over the scores, where it is the A operand of O += P V.  m moves only when it has been outgrown by 2^SLACK
//   split    the key tiles of a batch are cut into parts of one length, the shortest that gives no more parts than there are CTAs, so that ragged
//            lengths leave none of them idle; kv4_attn_join_kernel puts a sequence's parts together
//
// Bound by the softmax warps' chain (read a row's scores, maximum, 128 exponentials, write, hand over) next to the tensor core: 128 rows of 28 heads, 4 K/V heads,
// 65536 keys 155 us (775 TFLOP/s), 32768 keys 89 us; 512 rows of 32 heads over 512 keys 13 us.  Without the turning of codes 8 % less.  Dropped: exponentials
// begun with the old maximum before the new one is known (a longer chain); a form with S^T in tensor memory for up to 64 rows (143 us for 58 at 64 rows,
// 8 x 2048 keys, 32 heads: its code is fetched once per CTA, and that alone takes longer than the products).
//
// fp16 on both sides: keys and values are exact in it, q (bf16) is after a power of two per row down to 2^-17 of the row's largest entry (smaller ones are within
// 2^-25 of that), and probabilities keep three more bits than in bf16.
// The method of the two streams and the lagging maximum is that of attn_flash.cuh (published; named there).  Every mbarrier wait is bounded.
#pragma once
#include "kv4_attn.cuh"
#include "tcgen05.cuh"

namespace ps {
namespace kv4 {

using namespace tc;

constexpr int TC_ROWS = 128, TC_KEYS = 128, TC_DH = 128, UMMA_K = 16;
constexpr int TC_THREADS = 512;                  // warp 0: MMA + tensor memory, warps 4..11: softmax, four per stream, warps 12..15: codes
constexpr uint32_t HALF_TILE = 128 * 128, TC_TILE = 2 * HALF_TILE;     // [128][64] fp16 boxes, two of them per tile
constexpr int TC_SLOTS = 4, TC_DEPTH = 3;        // operand ring, staging ring of every code warp
constexpr uint32_t CODE_BYTES = 32 * 64, RAW_BYTES = CODE_BYTES + 32 * 8;       // 32 keys' codes and scales
// Registers of a thread: the block is launched with 128 each, 512 for the threads that share a lane of the four warpgroups; the softmax warps, which hold a
// row's 128 scores, take what the others give up.
constexpr int TC_LAUNCH_REGS = 128, TC_MMA_REGS = 80, TC_SOFTMAX_REGS = 168, TC_CODE_REGS = 96;
static_assert(TC_MMA_REGS + 2 * TC_SOFTMAX_REGS + TC_CODE_REGS <= 4 * TC_LAUNCH_REGS, "setmaxnreg.inc would wait for ever");
constexpr size_t TC_SMEM = 1024 + (2 + TC_SLOTS) * (size_t)TC_TILE + 4 * TC_DEPTH * RAW_BYTES;
static_assert(TC_SMEM <= 227 * 1024, "shared memory");

struct TcArgs {
    Args a;
    int tiles;                                   // CTAs per K/V head and part: row tiles (key split) or pairs of them
    int key_split;
};

// ---- codes -> operand tiles ---------------------------------------------------------------------------------------------
// A part's tiles in the order the tensor core takes them, two units (K and V) per key tile: K_0, V_0, K_1, V_1, ..., or, two key tiles in flight, K_0,
// K_1, V_0, K_2, V_1, K_3, ..., V_{n-2}, V_{n-1}.
struct Units {
    int n, t0, len, two;                         // key tiles, the first one, the sequence's keys, order
    __device__ __forceinline__ int tile(int u, bool& is_v) const {
        if (!two || n == 1) { is_v = (u & 1) != 0; return u >> 1; }
        if (u < 2) { is_v = false; return u; }
        const int w = u - 2;
        if (w < 2 * (n - 2)) { is_v = (w & 1) == 0; return is_v ? w >> 1 : (w >> 1) + 2; }
        is_v = true;
        return n - 2 + (w - 2 * (n - 2));
    }
};
// One warp's share: keys cw * 32 .. of units first, first + step, ...  It copies codes and scales DEPTH - 1 of them ahead into its staging ring at raw0
// and arrives on full0 + 8 slot once its rows are in the unit's slot of the operand ring at ring0, whose release it waits for on free0 + 8 slot.
// A row's 64 bytes of codes lie as four pieces, piece p at row * 64 + ((p ^ (row / 2 & 3)) << 4): the lanes that read one piece of eight rows then
// spread over all banks.  Rows from the sequence's end on are filled with zeros and not read.
template <int SLOTS, int DEPTH>
__device__ __forceinline__ void turn_codes(const Args& a, const Units& un, int b, int kvh, int cw, int first, int step, uint32_t raw0, uint32_t ring0,
                                           uint32_t full0, uint32_t free0, volatile int* abort_flag) {
    const int lane = threadIdx.x & 31, r8 = lane & 7, piece = lane >> 3, units = 2 * un.n;
    const size_t stride_c = (size_t)a.n_kv * 64, stride_s = (size_t)a.n_kv * 8;
    // what this lane copies of a unit: piece lane % 4 of rows lane / 4, + 8, + 16, + 24, and the scales of row `lane`
    const size_t key0 = (size_t)b * a.cap + (size_t)un.t0 * TC_KEYS + cw * 32;
    const size_t at_c = (key0 + (lane >> 2)) * stride_c + kvh * 64 + (lane & 3) * 16, at_s = (key0 + lane) * stride_s + kvh * 8;
    const uint32_t to_c = (uint32_t)((lane >> 2) * 64 + (((lane & 3) ^ ((lane >> 3) & 3)) << 4)), to_s = CODE_BYTES + (uint32_t)lane * 8u;
    const int left0 = un.len - un.t0 * TC_KEYS - cw * 32;                  // keys from this warp's first one on
    auto fetch = [&](int i) {                    // this warp's piece of work number i
        const int u = first + i * step;
        if (u < units) {
            bool is_v;
            const int t = un.tile(u, is_v), left = left0 - t * TC_KEYS;
            const uint8_t* codes = (is_v ? a.vc : a.kc) + at_c + (size_t)t * (TC_KEYS * stride_c);
            const uint8_t* scales = (is_v ? a.vs : a.ks) + at_s + (size_t)t * (TC_KEYS * stride_s);
            const uint32_t dst = raw0 + (uint32_t)(i % DEPTH) * RAW_BYTES;
            if (left >= 32) {
#pragma unroll
                for (int it = 0; it < 4; ++it)
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + to_c + (uint32_t)(it * 512)), "l"(codes + (size_t)(8 * it) * stride_c) : "memory");
                asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst + to_s), "l"(scales) : "memory");
            } else {                             // rows from the end on: zeros, from an address that is not read
#pragma unroll
                for (int it = 0; it < 4; ++it) {
                    const bool in = 8 * it + (lane >> 2) < left;
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + to_c + (uint32_t)(it * 512)), "l"(in ? codes + (size_t)(8 * it) * stride_c : a.kc), "r"(in ? 16 : 0) : "memory");
                }
                asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst + to_s), "l"(lane < left ? scales : a.ks), "r"(lane < left ? 8 : 0) : "memory");
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int i = 0; i < DEPTH - 1; ++i) fetch(i);
    bool ok = true;
    Ring r(first, SLOTS);
    for (int i = 0, u = first; u < units; ++i, u += step) {
        __syncwarp();              // (every lane has read the staging area that is filled next)
        fetch(i + DEPTH - 1);
        asm volatile("cp.async.wait_group %0;" ::"n"(DEPTH - 1) : "memory");
        __syncwarp();
        if (u >= SLOTS) ok = mbar_wait(free0 + 8u * (uint32_t)r.slot, r.phase ^ 1u, abort_flag);
        ok = __all_sync(0xffffffffu, ok) != 0;
        if (!ok) break;
        const uint32_t raw = raw0 + (uint32_t)(i % DEPTH) * RAW_BYTES;
        const uint32_t dst = ring0 + (uint32_t)r.slot * TC_TILE + (uint32_t)(piece >> 1) * HALF_TILE + (uint32_t)(cw * 32) * 128u;
        uint32_t w[4][4], sc[4];
#pragma unroll
        for (int it = 0; it < 4; ++it) {
            const int row = 8 * it + r8;
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[it][0]), "=r"(w[it][1]), "=r"(w[it][2]), "=r"(w[it][3])
                         : "r"(raw + (uint32_t)(row * 64 + ((piece ^ ((row >> 1) & 3)) << 4))) : "memory");
            asm volatile("ld.shared.u16 %0, [%1];" : "=r"(sc[it]) : "r"(raw + CODE_BYTES + (uint32_t)(row * 8 + piece * 2)) : "memory");
        }
#pragma unroll
        for (int it = 0; it < 4; ++it) {
            const uint32_t sp = scales_to_half(sc[it]), s0 = __byte_perm(sp, 0, 0x1010), s1 = __byte_perm(sp, 0, 0x3232);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                uint32_t h[4];
                codes_to_half(w[it][c], h);
#pragma unroll
                for (int x = 0; x < 4; ++x) h[x] = h2mul(h[x], c < 2 ? s0 : s1);
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst + (uint32_t)((8 * it + r8) * 128) + (uint32_t)((((piece & 1) * 4 + c) ^ r8) << 4)),
                             "r"(h[0]), "r"(h[1]), "r"(h[2]), "r"(h[3]) : "memory");
            }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(full0 + 8u * (uint32_t)r.slot);
        for (int x = 0; x < step; ++x) r.next(SLOTS);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
}

// fp16 x fp16 -> fp32, both operands K-major
__device__ __forceinline__ uint32_t instr_desc_f16(int m, int n) { return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24); }

__global__ void __launch_bounds__(TC_THREADS, 1) kv4_attn_tc_kernel(const __grid_constant__ TcArgs f) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t bars[1 + 2 * TC_SLOTS + 6];
    __shared__ float unit_sh[2][TC_ROWS];
    __shared__ uint32_t tmem_base_sh;
    __shared__ int abort_sh;
    const Args& a = f.a;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int tile = (int)blockIdx.x / a.slots, slot_no = (int)blockIdx.x - tile * a.slots, kvh = blockIdx.y;
    const int hpg = a.n_heads / a.n_kv;
    const long long vrows = (long long)hpg * a.R;
    const bool ksplit = f.key_split != 0;
    const long long vr0 = (long long)tile * (ksplit ? TC_ROWS : 2 * TC_ROWS);

    uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    const uint32_t smem_base = smem_u32(smem), bar0 = smem_u32(&bars[0]);
    auto q_s = [&](int g) { return smem_base + (uint32_t)g * TC_TILE; };
    auto ring_s = [&](int s) { return smem_base + (uint32_t)(2 + s) * TC_TILE; };
    const uint32_t bar_q = bar0;
    auto bar_full = [&](int s) { return bar0 + 8u * (uint32_t)(1 + s); };
    auto bar_free = [&](int s) { return bar0 + 8u * (uint32_t)(1 + TC_SLOTS + s); };
    auto bar_s = [&](int g) { return bar0 + 8u * (uint32_t)(1 + 2 * TC_SLOTS + g); };
    auto bar_p = [&](int g) { return bar0 + 8u * (uint32_t)(3 + 2 * TC_SLOTS + g); };
    auto bar_o = [&](int g) { return bar0 + 8u * (uint32_t)(5 + 2 * TC_SLOTS + g); };
    volatile int* abort_flag = &abort_sh;

    if (threadIdx.x == 0) {
        mbar_init(bar_q, 8);
        for (int s = 0; s < TC_SLOTS; ++s) { mbar_init(bar_full(s), 4); mbar_init(bar_free(s), 1); }
        for (int g = 0; g < 2; ++g) { mbar_init(bar_s(g), 1); mbar_init(bar_p(g), 4); mbar_init(bar_o(g), 1); }
        abort_sh = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 0) tmem_alloc(smem_u32(&tmem_base_sh), 512);       // S / P of stream 0 and 1, O of stream 0 and 1: 128 columns each
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_trigger();
    pdl_wait();            // lengths, codes and q may all come from the kernel before
    const uint32_t tmem_base = tmem_base_sh;

    int b = 0, part = 0, t0 = 0, n = 0, len = 0;
    const bool busy = find_part<TC_KEYS>(a, slot_no, tile == 0 && kvh == 0 && threadIdx.x == 0, b, part, t0, n, len);
    const int cnt0 = ksplit ? (n + 1) >> 1 : n;                    // of stream 0 ...
    const int cnt1 = ksplit ? n >> 1 : (vr0 + TC_ROWS < vrows ? n : 0);       // ... and of stream 1

    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(TC_MMA_REGS));
        if (busy && warp == 0 && elect_one()) {
            const uint32_t idesc_s = instr_desc_f16(TC_ROWS, TC_KEYS);
            const uint32_t idesc_o = instr_desc_f16(TC_ROWS, TC_DH) | (1u << 16);       // B (= V) is MN-major
            bool ok = mbar_wait(bar_q, 0, abort_flag);
            Ring r(0, TC_SLOTS);
            auto take = [&]() {
                const int sl = r.slot;
                ok = ok && mbar_wait(bar_full(sl), r.phase, abort_flag);
                r.next(TC_SLOTS);
                tc_fence_after();
                return sl;
            };
            auto mma_s = [&](int g, int sl) {
                if (!ok) return;
                const uint32_t q = q_s(ksplit ? 0 : g);
#pragma unroll
                for (int k = 0; k < TC_DH / UMMA_K; ++k)
                    umma_bf16(tmem_base + (uint32_t)(g * TC_KEYS), smem_desc_sw128(q + (k >> 2) * HALF_TILE) + (uint64_t)((k & 3) * 2),
                              smem_desc_sw128(ring_s(sl) + (k >> 2) * HALF_TILE) + (uint64_t)((k & 3) * 2), idesc_s, k > 0 ? 1u : 0u);
                umma_commit(bar_s(g));
            };
            auto mma_o = [&](int g, int k0, int sl) {
                ok = ok && mbar_wait(bar_p(g), (uint32_t)k0 & 1u, abort_flag);
                if (!ok) return;
                tc_fence_after();
#pragma unroll
                for (int k = 0; k < TC_KEYS / UMMA_K; ++k)
                    umma_bf16_ta(tmem_base + (uint32_t)(2 * TC_KEYS + g * TC_DH), tmem_base + (uint32_t)(g * TC_KEYS + k * (UMMA_K / 2)),
                                 smem_desc_mn_sw128(ring_s(sl) + (uint32_t)k * 2048u, HALF_TILE), idesc_o, (k0 > 0 || k > 0) ? 1u : 0u);
            };
            auto release = [&](int sl) { if (ok) umma_commit(bar_free(sl)); };
            // The scores of tile k + 1 overwrite the probabilities of tile k: issued behind the P V that reads them, products complete in order.
            if (n > 0 && !ksplit) {
                int ks = take();
                mma_s(0, ks);
                if (cnt1 > 0) mma_s(1, ks);
                release(ks);
                for (int k = 0; k < n && ok; ++k) {
                    const int vs = take();
                    mma_o(0, k, vs);
                    if (k + 1 < n) { ks = take(); mma_s(0, ks); }
                    if (cnt1 > 0) {
                        mma_o(1, k, vs);
                        release(vs);
                        if (k + 1 < n) mma_s(1, ks);
                    } else {
                        release(vs);
                    }
                    if (k + 1 < n) release(ks);
                }
            } else if (n > 0) {
                for (int g = 0; g < min(n, 2); ++g) { const int ks = take(); mma_s(g, ks); release(ks); }
                for (int t = 0; t < n && ok; ++t) {
                    const int vs = take();
                    mma_o(t & 1, t >> 1, vs);
                    release(vs);
                    if (t + 2 < n) { const int ks = take(); mma_s(t & 1, ks); release(ks); }
                }
            }
            umma_commit(bar_o(0));       // (also on failure: the other warps then see the abort flag)
            umma_commit(bar_o(1));
        }
    } else if (warp >= 12) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(TC_CODE_REGS));
        const Units un = {n, t0, len, ksplit};
        if (busy) turn_codes<TC_SLOTS, TC_DEPTH>(a, un, b, kvh, warp - 12, 0, 1, smem_base + (2 + TC_SLOTS) * TC_TILE + (uint32_t)(warp - 12) * (TC_DEPTH * RAW_BYTES),
                                                 ring_s(0), bar_full(0), bar_free(0), abort_flag);
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(TC_SOFTMAX_REGS));
        // ---- softmax warps: tensor-memory lane = row ----
        if (busy) {
        const int sw = warp - 4, g = sw >> 2, quarter = warp & 3;
        const int row = quarter * 32 + lane;
        const int cnt = g ? cnt1 : cnt0;
        const uint32_t tS = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(g * TC_KEYS);
        const uint32_t tO = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(2 * TC_KEYS + g * TC_DH);
        const long long vr = vr0 + ((g && !ksplit) ? TC_ROWS : 0) + row;
        auto q_row = [&](long long v) {          // virtual row -> row of [batch * R * n_heads]
            const int h = (int)(v / a.R), r = (int)(v - (long long)h * a.R);
            return ((size_t)b * a.R + r) * a.n_heads + kvh * hpg + h;
        };
        // q rows into shared memory in the operand layout, half a warp per row (the streams of a key split take 16 rows each), every row scaled by a
        // power of two to at most 2
        if (cnt > 0 || ksplit) {
            const int first = quarter * 32 + (ksplit ? 16 * g : 0), pairs = ksplit ? 8 : 16, ch = lane & 15;
            const long long vq0 = vr0 + ((g && !ksplit) ? TC_ROWS : 0) + first + (lane >> 4);
            const uint32_t dst = q_s(ksplit ? 0 : g) + (uint32_t)(ch >> 3) * HALF_TILE;
            for (int i0 = 0; i0 < pairs; i0 += 4) {
                uint4 v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const long long vq = vq0 + 2 * (i0 + i);
                    v[i] = make_uint4(0u, 0u, 0u, 0u);
                    if (vq < vrows) v[i] = __ldg(reinterpret_cast<const uint4*>((const __nv_bfloat16*)a.q + q_row(vq) * TC_DH) + ch);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int lr = first + (lane >> 4) + 2 * (i0 + i);
                    const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
                    uint32_t top = 0;
#pragma unroll
                    for (int x = 0; x < 4; ++x) top = max(top, max(w[x] & 0x7fff0000u, (w[x] << 16) & 0x7fff0000u));
#pragma unroll
                    for (int o = 1; o < 16; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
                    const int e = min(max((int)(top >> 23), 1), 253);
                    // (infinity or NaN in q: every score of the row is NaN, not -inf)
                    const float down = top >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : __uint_as_float((uint32_t)(254 - e) << 23);
                    if (ch == 0) unit_sh[ksplit ? 0 : g][lr] = __uint_as_float((uint32_t)e << 23);
                    uint32_t h[4];
#pragma unroll
                    for (int x = 0; x < 4; ++x) h[x] = pack_half(__uint_as_float(w[x] << 16) * down, __uint_as_float(w[x] & 0xffff0000u) * down);
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst + (uint32_t)lr * 128u + ((uint32_t)((ch ^ lr) & 7) << 4)),
                                 "r"(h[0]), "r"(h[1]), "r"(h[2]), "r"(h[3]) : "memory");
                }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(bar_q);
        asm volatile("bar.sync 1, 256;" ::: "memory");             // the rows' units
        // (a unit of 0, of a row of zeros and a small factor, would make NaN of the -inf of keys that are not there; at the smallest normal one, scores are still
        // nothing: below 2^-100)
        float unit = (float)((double)unit_sh[ksplit ? 0 : g][row] * (a.scale * (double)(a.tk ? __ldg(a.tk) : 1.f)));
        if (fabsf(unit) < 1.17549435e-38f) unit = 1.17549435e-38f;
        const float tv = a.tv ? __ldg(a.tv) : 1.f;

        float m = -INFINITY, l = 0.f;
        bool ok = true;
        for (int k = 0; k < cnt; ++k) {
            ok = mbar_wait(bar_s(g), (uint32_t)k & 1u, abort_flag) && ok && !*abort_flag;
            ok = __all_sync(0xffffffffu, ok) != 0;
            if (!ok) break;
            tc_fence_after();
            const int kb = (t0 + (ksplit ? 2 * k + g : k)) * TC_KEYS;
            const bool edge = kb + TC_KEYS > len;
            auto mask = [&](uint32_t* r, int c0) {
#pragma unroll
                for (int i = 0; i < 32; ++i) if (kb + c0 + i >= len) r[i] = 0xff800000u;      // -inf
            };
            uint32_t sc[4][32];
            float tm4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_ld32_issue(tS + 32u * (uint32_t)c, sc[c]);
#pragma unroll
            for (int c = 0; c < 4; ++c) { tmem_ld_wait16(sc[c]); tmem_ld_wait16(sc[c] + 16); }
            if (__builtin_expect(edge, 0)) {
#pragma unroll
                for (int c = 0; c < 4; ++c) mask(sc[c], 32 * c);
            }
#pragma unroll
            for (int i = 0; i < 32; ++i)
#pragma unroll
                for (int c = 0; c < 4; ++c) tm4[c] = fmaxf(tm4[c], __uint_as_float(sc[c][i]));
            float tm = fmaxf(fmaxf(tm4[0], tm4[1]), fmaxf(tm4[2], tm4[3]));
            tm *= unit;                                            // (unit > 0: the maximum commutes with it)
            if (k == 0) {
                m = tm;
            } else if (__builtin_expect(__any_sync(0xffffffffu, tm > m + SLACK), 0)) {
                // (the P V of the previous tile has completed: it was issued in front of the scores just read)
                const bool up = tm > m + SLACK;
                const float nm = up ? tm : m, al = up ? (m == -INFINITY ? 0.f : ex2(m - nm)) : 1.f;
                l *= al;
                m = nm;
#pragma unroll 1
                for (int c = 0; c < TC_DH; c += 16) {
                    uint32_t o[16];
                    tmem_ld16_issue(tO + (uint32_t)c, o);
                    tmem_ld_wait16(o);
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * al);
                    tmem_st16_issue(tO + (uint32_t)c, o);
                }
                tmem_st_wait();
            }
            const float neg_m = m == -INFINITY ? 0.f : LIFT - m;
            const uint64_t sc2 = f2_pack(unit, unit), nm2 = f2_pack(neg_m, neg_m);
            uint64_t l2[2] = {0ull, 0ull};
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                uint32_t pw[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    float y0, y1;
                    f2_unpack(f2_fma(f2_pack(sc[c][2 * i], sc[c][2 * i + 1]), sc2, nm2), y0, y1);
                    const float p0 = ex2(y0), p1 = ex2(y1);
                    l2[i & 1] = f2_add(l2[i & 1], f2_pack(p0, p1));
                    pw[i] = pack_half(p0, p1);
                }
                tmem_st16_issue(tS + (uint32_t)(16 * c), pw);
            }
            l += f2_sum(f2_add(l2[0], l2[1]));
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar_p(g));
        }

        // ---- output rows ----
        ok = mbar_wait(bar_o(0), 0, abort_flag) && mbar_wait(bar_o(1), 0, abort_flag) && ok && !*abort_flag;
        ok = __all_sync(0xffffffffu, ok) != 0;
        tc_fence_after();
        float w0 = 1.f, w1 = 0.f;                          // weights of the streams' O
        if (ksplit) {
            // the streams' parts of the row meet in the first ring slot's place: every product has completed
            float* ex = reinterpret_cast<float*>(smem + 2 * TC_TILE);
            ex[(2 * g) * TC_ROWS + row] = m; ex[(2 * g + 1) * TC_ROWS + row] = l;
            asm volatile("bar.sync 1, 256;" ::: "memory");
            const float m0 = ex[row], m1 = ex[2 * TC_ROWS + row], l0 = ex[TC_ROWS + row], l1 = ex[3 * TC_ROWS + row];
            m = fmaxf(m0, m1);
            w0 = m0 == -INFINITY ? 1.f : ex2(m0 - m); w1 = m1 == -INFINITY ? 1.f : ex2(m1 - m);       // (nothing but NaN scores: m = -inf, l = NaN)
            l = l0 * w0 + l1 * w1;
        }
        if (l == 0.f && n > 0 && !a.part_n) l = __uint_as_float(0x7fc00000u);       // (keys, but every score -inf)
        const bool none = l == 0.f;                        // no keys: the accumulators hold nothing
        if ((cnt > 0 || ksplit || n == 0) && vr < vrows) {
            const size_t ro = q_row(vr);
            const float inv = none ? 0.f : tv / l;
            if ((g == 0 || !ksplit)) {
                if (a.part_n) a.part_ml[(size_t)part * a.rows_total + ro] = make_float2(m, ok ? l : __uint_as_float(0x7fc00000u));
                else if (a.lse) a.lse[ro] = !ok ? __uint_as_float(0x7fc00000u) : none ? -INFINITY : (m - LIFT + log2f(l)) * 0.6931471805599453f;
            }
            w0 *= a.part_n ? 1.f : inv; w1 *= a.part_n ? 1.f : inv;
        }
        const int c_lo = ksplit ? 64 * g : 0, c_hi = (cnt > 0 || ksplit || n == 0) ? (ksplit ? c_lo + 64 : TC_DH) : 0;
        const uint32_t tO0 = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(2 * TC_KEYS);
        for (int c = c_lo; c < c_hi; c += 32) {
            uint32_t o[32], o1[32];
            tmem_ld32_issue((ksplit ? tO0 : tO) + (uint32_t)c, o);
            if (ksplit && cnt1 > 0) tmem_ld32_issue(tO0 + (uint32_t)(TC_DH + c), o1);
            tmem_ld_wait16(o); tmem_ld_wait16(o + 16);
            if (ksplit && cnt1 > 0) {
                tmem_ld_wait16(o1); tmem_ld_wait16(o1 + 16);
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * w0 + __uint_as_float(o1[i]) * w1);
            } else {
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * w0);
            }
            if (none || !ok) {
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] = ok ? 0u : 0x7fc00000u;
            }
            if (vr < vrows) {
                if (a.part_n) {
                    float* dst = a.part_o + ((size_t)part * a.rows_total + q_row(vr)) * TC_DH + c;
#pragma unroll
                    for (int q = 0; q < 8; ++q) *reinterpret_cast<uint4*>(dst + 4 * q) = make_uint4(o[4 * q], o[4 * q + 1], o[4 * q + 2], o[4 * q + 3]);
                } else {
                    __nv_bfloat16* dst = (__nv_bfloat16*)a.out + q_row(vr) * TC_DH + c;
                    float v[32];
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(o[i]);
                    store16<__nv_bfloat16>(dst, v);
                    store16<__nv_bfloat16>(dst + 16, v + 16);
                }
            }
        }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 0) tmem_dealloc(tmem_base, 512);
}

}  // namespace kv4
}  // namespace ps
