// Product of two microscaled 4-bit matrices on 5th-generation tensor cores:  out[m][n] = ta tb sum_k A[m][k] B[n][k].
//
// tcgen05.mma with block scales multiplies E2M1 codes (64 of K per instruction, 128 bytes of a row are 256 of K) and takes the groups'
// scales from tensor memory: rows of codes come by TMA (128-byte swizzle, as bf16 rows of the same bytes would), 512-byte blocks of
// the tiled scales (128 rows x 4 groups) by plain bulk copies, and tcgen05.cp moves a block into four columns of tensor memory, copied to the
// four lane quarters.  Products of codes and scales are exact, sums are the tensor core's fp32.
#pragma once
#include "fp4.cuh"
#include "tcgen05.cuh"

namespace ps {
namespace fp4 {

constexpr int KB = 256;                          // K of a ring slot: one 128-byte row of codes
constexpr uint32_t BLOCK_BYTES = 512;            // scales of 128 rows x 4 groups
__host__ __device__ constexpr int scale_blocks(int fmt) { return KB / (4 * group(fmt)); }       // per slot and 128 rows: 4 or 2

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
// Shared-memory descriptor of a scale block: 32 rows of 16 bytes, no swizzle, 8-row groups 128 bytes apart.
__device__ __forceinline__ uint64_t smem_desc_scales(uint32_t addr) {
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(128u >> 4) << 32) | ((uint64_t)1 << 46);
}
__device__ __forceinline__ void copy_scales(uint32_t tmem, uint64_t desc) {
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
// Instruction descriptor: E2M1 x E2M1 -> fp32, both K-major; scales E4M3 (nv) or E8M0 (mx).  The latter take two of the four bytes of a
// column per instruction, which two (0 or 2) is part of the descriptor.
template <int FMT>
__device__ __forceinline__ uint32_t instr_desc_fp4(int m, int n, uint32_t byte) {
    return (byte << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((FMT == MX ? 1u : 0u) << 23) | ((uint32_t)(m >> 7) << 27) | (byte << 29);
}
template <int FMT>
__device__ __forceinline__ void umma_fp4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t accumulate) {
    if (FMT == NV)
        asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %6, 0;\n"
                     " tcgen05.mma.cta_group::1.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], %1, %2, %3, [%4], [%5], p;\n}\n"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate) : "memory");
    else
        asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %6, 0;\n"
                     " tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n}\n"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate) : "memory");
}

// The factors ta tb as two multipliers, applied one after the other: x, the product in full wherever it is a normal number (y is 1), and else with what it
// lacks as a power of two in y, so that neither is 0 or infinite where (sum x) y is not.  (Beyond 2^254 y stays at 2^127: only sums below fp32's normal range
// would not be infinite there.)
__device__ __forceinline__ float2 tensor_factors(const float* ta, const float* tb) {
    const double p = (double)(ta ? __ldg(ta) : 1.f) * (double)(tb ? __ldg(tb) : 1.f);
    const int e = ((__double2hiint(p) >> 20) & 0x7ff) - 1023, rest = min(max(e < 0 ? min(e + 126, 0) : max(e - 126, 0), -126), 127);
    return make_float2((float)(p * __hiloint2double((1023 - rest) << 20, 0)), __uint_as_float((uint32_t)(rest + 127) << 23));
}

// After a wait that gave up: the copies of the last slots asked for land before their shared memory goes (bounded).
__device__ __forceinline__ void drain_ring(int issued, int stages, uint32_t full0) {
    for (int u = max(0, issued - stages); u < issued; ++u) {
        const Ring r(u, stages);
        const long long t0 = clock64();
        while (!mbar_try_wait(full0 + 8u * (uint32_t)r.slot, r.phase) && clock64() - t0 < WAIT_LIMIT_CYCLES) {}
    }
}

struct GemmArgs {
    const uint8_t* as; const uint8_t* bs;        // tiled scales
    const float* ta; const float* tb;            // factors of the tensors (null: 1)
    void* out; long long ld;
    int M, N, K;
    int split, stages;                           // few rows: CTAs of a cluster that share the K of a tile, ring slots of a CTA
    int box_out;                                 // output rows, their stride and base are whole 16 bytes: they leave as tensor stores
};

// ---- few rows of A: bound by the stream of B ---------------------------------------------------------------------------
// The wide matrix takes the 128 lanes: D^T = B A^T, a tile is 128 columns of the output x T rows of it, so a few rows cost no padding of the
// stream.  One tile per CTA: with more tiles than SMs two CTAs share one, each with half the slots.  Where tiles are few, the CTAs of a cluster take
// consecutive parts of K; when all of them have finished their products, each writes its partial sums into the ring of the CTA that owns the output rows
// (distributed shared memory, which takes about 13 bytes a cycle, so 128 rows cost three times what 32 do), and that adds them in the order of K.
// 32 rows, bf16 out: 12288 x 4096 9.2 us (3.1 TB/s of weights; start, first loads and epilogue are half of it), 37888 x 3584 14.3 us (5.3 TB/s),
// 126464 x 4096 51 us (5.7 TB/s, 0.87 of the copy rate); 128 rows 64 us.
constexpr int ST_THREADS = 192;                  // TMA, MMA, four epilogue warps
constexpr int ST_MAX_STAGES = 8;
__host__ __device__ constexpr uint32_t st_stage_bytes(int T, int fmt) { return 128 * 128 + T * 128 + 2 * scale_blocks(fmt) * BLOCK_BYTES; }
// ring slots of a CTA, one or two of which share an SM
__host__ __device__ constexpr int st_stages(int T, int fmt, int per_sm) {
    const int n = (int)(((per_sm == 1 ? 225 : 112) * 1024 - 1024) / st_stage_bytes(T, fmt));
    return n < ST_MAX_STAGES ? n : ST_MAX_STAGES;
}
__host__ __device__ constexpr size_t st_smem_bytes(int T, int fmt, int per_sm) { return 1024 + (size_t)st_stages(T, fmt, per_sm) * st_stage_bytes(T, fmt); }
static_assert(st_stages(128, NV, 1) * st_stage_bytes(128, NV) >= 128 * 128 * 4 && st_stages(32, NV, 1) * st_stage_bytes(32, NV) >= 128 * 32 * 4, "the ring takes the partial sums");

template <int T, int FMT, typename OUT>
__global__ void __launch_bounds__(ST_THREADS, 2)
gemm_stream_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ GemmArgs g) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t bars[2 * ST_MAX_STAGES + 2];
    __shared__ uint32_t tmem_base_sh;
    __shared__ int abort_sh;
    constexpr int SB = scale_blocks(FMT);
    const int STAGES = g.stages;
    constexpr uint32_t STAGE = st_stage_bytes(T, FMT);
    constexpr uint32_t A_OFF = 128 * 128, BS_OFF = A_OFF + T * 128, AS_OFF = BS_OFF + SB * BLOCK_BYTES;
    constexpr uint32_t COLS = 256, SF_COL = 128;          // accumulator: columns 0 .. T - 1; two sets of scales from column 128 on
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = g.split > 1 ? (int)cluster_rank() : 0;
    const int tile_n = (int)blockIdx.x / g.split, tile_m = blockIdx.y;
    const int kb_total = (g.K + KB - 1) / KB;
    const int kb0 = (int)((long long)kb_total * rank / g.split), kb1 = (int)((long long)kb_total * (rank + 1) / g.split);
    const int sb_row = (g.K / group(FMT) + 3) / 4;        // scale blocks of 128 rows

    uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    const uint32_t smem_base = smem_u32(smem), bar0 = smem_u32(&bars[0]);
    auto full = [&](int s) { return bar0 + 8u * (uint32_t)s; };
    auto empty = [&](int s) { return bar0 + 8u * (uint32_t)(ST_MAX_STAGES + s); };
    const uint32_t done = bar0 + 16u * ST_MAX_STAGES;
    volatile int* abort_flag = &abort_sh;

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
        mbar_init(done, 1);
        mbar_init(done + 8u, 1);
        abort_sh = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) tmem_alloc(smem_u32(&tmem_base_sh), COLS);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_trigger();
    const uint32_t tmem = tmem_base_sh;

    int issued = 0;                                       // ring slots that this thread has asked for
    if (warp == 0) {
        if (elect_one()) {
            pdl_wait();
            const uint64_t policy = l2_policy_evict_first();
            bool ok = true;
            Ring r(0, STAGES);
            for (int kb = kb0; kb < kb1 && ok; ++kb, r.next(STAGES)) {
                if (kb - kb0 >= STAGES) ok = mbar_wait(empty(r.slot), r.phase ^ 1u, abort_flag);
                if (!ok) break;
                const uint32_t slot = smem_base + (uint32_t)r.slot * STAGE;
                const uint32_t sbytes = (uint32_t)min(SB, sb_row - kb * SB) * BLOCK_BYTES;
                mbar_expect_tx(full(r.slot), 128 * 128 + T * 128 + 2 * sbytes);
                if (gridDim.y == 1) tma_load_2d_hint(slot, &map_b, full(r.slot), kb * 128, tile_n * 128, policy);
                else tma_load_2d(slot, &map_b, full(r.slot), kb * 128, tile_n * 128);
                tma_load_2d(slot + A_OFF, &map_a, full(r.slot), kb * 128, tile_m * T);
                bulk_load(slot + BS_OFF, g.bs + ((size_t)tile_n * sb_row + kb * SB) * BLOCK_BYTES, sbytes, full(r.slot));
                bulk_load(slot + AS_OFF, g.as + ((size_t)(tile_m * T / 128) * sb_row + kb * SB) * BLOCK_BYTES, sbytes, full(r.slot));
                ++issued;
            }
        }
    } else if (warp == 1) {
        if (elect_one()) {
            bool ok = true;
            Ring r(0, STAGES);
            for (int kb = kb0; kb < kb1 && ok; ++kb, r.next(STAGES)) {
                ok = mbar_wait(full(r.slot), r.phase, abort_flag);
                if (!ok) break;
                tc_fence_after();
                const uint32_t slot = smem_base + (uint32_t)r.slot * STAGE;
                const int steps = min(4, (g.K - kb * KB) / 64), blocks = min(SB, sb_row - kb * SB);
                const uint32_t sf_b = tmem + SF_COL + (uint32_t)(kb & 1) * 32u, sf_a = sf_b + 16u;
                for (int c = 0; c < blocks; ++c) {
                    copy_scales(sf_b + 4u * (uint32_t)c, smem_desc_scales(slot + BS_OFF + (uint32_t)c * BLOCK_BYTES));
                    copy_scales(sf_a + 4u * (uint32_t)c, smem_desc_scales(slot + AS_OFF + (uint32_t)c * BLOCK_BYTES));
                }
                const uint64_t db = smem_desc_sw128(slot), da = smem_desc_sw128(slot + A_OFF);
                for (int s = 0; s < steps; ++s) {
                    const uint32_t c = 4u * (uint32_t)(FMT == NV ? s : s >> 1), byte = FMT == NV ? 0u : (uint32_t)(s & 1) * 2u;
                    umma_fp4<FMT>(tmem, db + (uint64_t)(2 * s), da + (uint64_t)(2 * s), instr_desc_fp4<FMT>(128, T, byte), sf_b + c, sf_a + c, kb > kb0 || s > 0 ? 1u : 0u);
                }
                umma_commit(empty(r.slot));
            }
            umma_commit(done);      // (also on failure: the epilogue then sees the abort flag)
        }
    }
    __syncwarp();
    // ---- epilogue: tensor-memory lane = output column, accumulator column = output row ----
    const int quarter = warp & 3;
    const uint32_t lane_base = tmem + ((uint32_t)(quarter * 32) << 16);
    const int rows_each = T / g.split;                    // output rows that this CTA finishes (a power of two)
    const int live = min(T, g.M - tile_m * T);            // rows of the tile that exist
    bool ok = true;
    float2 scale = make_float2(1.f, 1.f);
    if (warp >= 2) {
        pdl_wait();
        scale = tensor_factors(g.ta, g.tb);
        ok = mbar_wait(done, 0, abort_flag) && !*abort_flag;
        ok = __all_sync(0xffffffffu, ok) != 0;
        tc_fence_after();
        if (!ok) scale.x = __uint_as_float(0x7fc00000u);  // a bounded wait gave up: NaN, not a partial sum
    }
    const int n = tile_n * 128 + quarter * 32 + lane;
    auto store = [&](int m, float v) {
        if (m < g.M && n < g.N) ((OUT*)g.out)[(size_t)m * g.ld + n] = from_f<OUT>(v * scale.x * scale.y);
    };
    if (g.split == 1) {
        if (warp >= 2)
#pragma unroll 1
            for (int c = 0; c < live; c += 16) {
                float v[16];
                tmem_ld16(lane_base + (uint32_t)c, v);
#pragma unroll
                for (int i = 0; i < 16; ++i) store(tile_m * T + c + i, v[i]);
            }
    } else {
        // (the products of every CTA have completed: their operands' place is free)
        if (warp == 2 && !ok && lane < g.split) asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(dsmem_addr(smem_u32(&abort_sh), (uint32_t)lane)), "r"(1u) : "memory");
        __syncwarp();
        cluster_sync_all();
        const int col = quarter * 32 + lane;
        if (warp >= 2) {
            const int shift = __ffs(rows_each) - 1;
            const uint32_t mine = smem_base + (uint32_t)((rank * (rows_each >> 2) * 128 + col) * 16);
#pragma unroll 1
            for (int c = 0; c < live; c += 16) {
                float v[16];
                tmem_ld16(lane_base + (uint32_t)c, v);
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const uint32_t dst = dsmem_addr(mine + (uint32_t)((c + i) & (rows_each - 1)) * 512u, (uint32_t)((c + i) >> shift));
                    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "f"(v[i]), "f"(v[i + 1]), "f"(v[i + 2]), "f"(v[i + 3]) : "memory");
                }
            }
        }
        __syncwarp();
        cluster_sync_all();
        if (warp >= 2) {
            if (*abort_flag) scale.x = __uint_as_float(0x7fc00000u);
            OUT* dst = (OUT*)g.out + (size_t)(tile_m * T + rank * rows_each) * g.ld + n;
            const uint32_t from = smem_base + (uint32_t)(col * 16), step = (uint32_t)rows_each * 512u;
            const int rows = min(rows_each, live - rank * rows_each);
            for (int i = 0; i < rows; i += 4) {           // (rows_each is 4 or more)
                float x[8][4];
#pragma unroll
                for (int s = 0; s < 8; ++s) {             // all loads at once; -0: adds nothing
                    x[s][0] = x[s][1] = x[s][2] = x[s][3] = -0.f;
                    if (s < g.split)
                        asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x[s][0]), "=f"(x[s][1]), "=f"(x[s][2]), "=f"(x[s][3])
                                     : "r"(from + (uint32_t)s * step + (uint32_t)i * 512u) : "memory");
                }
#pragma unroll
                for (int s = 1; s < 8; ++s)
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[0][j] += x[s][j];
#pragma unroll
                for (int j = 0; j < 4; ++j, dst += g.ld)
                    if (i + j < rows && n < g.N) *dst = from_f<OUT>(x[0][j] * scale.x * scale.y);
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (abort_sh && issued > 0) drain_ring(issued, STAGES, bar0);
    if (warp == 1) tmem_dealloc(tmem, COLS);
}

// ---- many rows: bound by the tensor cores and by what L2 hands to them ----------------------------------------------------
// A CTA pair (cluster of two, tcgen05 cta_group::2) works on a tile of 256 x 256 outputs: each CTA holds 128 rows of A and half of the tile's rows of B
// in shared memory and its 128 rows x 256 columns of sums in its tensor memory; the even CTA issues the products for both.  Scales come as boxes of
// whole blocks; every CTA needs those of its own rows of A and of all 256 rows of B.  Persistent: pairs take the tiles in an order in which those in
// flight share their operands.  There is one accumulator (two of 256 columns would leave no tensor memory for scales): eight warps drain it into
// registers, 128 columns each, and hand it back before they store.  A lane has a row, so its stores would touch 32 lines per instruction (8192 cycles of
// the load/store unit for a tile of fp32, more than its products take); rows of 128 bytes go through a swizzled box per warp and leave as tensor
// stores.  Those write whole 16 bytes, also behind the last column: where a row's end or its stride is no multiple of that, the warp stores the boxes'
// rows element by element.
// 8192 x 24576 x 4096, bf16 out 357 us (4.6 PFLOP/s), 4096 x 12288 x 4096 97 us (4.3), 997 x 37888 x 3584 fp32 out mx 72 us (3.8), 512 x 126464 x 4096 131.  L2 hands
// the SMs 10 TB/s or so, which is what tiles of this size ask for at that rate, and the tensor pipe waits for them: a fifth ring slot in the place of the second
// output boxes took 79 to 72 us at 997 rows and 137 to 131 at 512.  With four slots, leaving out the stores took 408 to 361, waiting for the accumulator too 334.
constexpr int PR_THREADS = 384;                  // warp 0: TMA, warp 1: MMA + tensor memory, warps 4..11: epilogue
constexpr int PR_TILE = 256;
constexpr int PR_STAGES = 5;
constexpr uint32_t PR_BOX = 32 * 128;            // a box of outputs, one per epilogue warp: 32 rows of 128 bytes
__host__ __device__ constexpr uint32_t pr_stage_bytes(int fmt) { return 2 * 128 * 128 + 3 * scale_blocks(fmt) * BLOCK_BYTES; }
__host__ __device__ constexpr size_t pr_smem_bytes(int fmt) { return 1024 + (size_t)PR_STAGES * ((pr_stage_bytes(fmt) + 1023) / 1024 * 1024) + 8 * PR_BOX; }
static_assert(pr_smem_bytes(NV) <= 227 * 1024, "shared memory");

__device__ __forceinline__ void pack16(uint32_t (&w)[4], const float (&f)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(f[i]);
}
__device__ __forceinline__ void pack16(uint32_t (&w)[4], const float (&f)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&b);
    }
}
__device__ __forceinline__ void copy_scales_pair(uint32_t tmem, uint64_t desc) {
    asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
template <int FMT>
__device__ __forceinline__ void umma_fp4_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t accumulate) {
    if (FMT == NV)
        asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %6, 0;\n"
                     " tcgen05.mma.cta_group::2.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], %1, %2, %3, [%4], [%5], p;\n}\n"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate) : "memory");
    else
        asm volatile("{\n .reg .pred p;\n setp.ne.b32 p, %6, 0;\n"
                     " tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n}\n"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate) : "memory");
}
// Tile number -> (row tile, column tile): chunks of 16 row tiles, inside which the row tile runs fastest, so that the pairs at work at one time cover a
// compact block of the output (8192 x 24576 x 4096: chunks of 4, 8, 16 385, 364, 357 us).
__device__ __forceinline__ void pair_tile(int id, int tiles_m, int tiles_n, int& tm, int& tn) {
    const int per = 16 * tiles_n, chunk = id / per, local = id - chunk * per, rows = min(16, tiles_m - chunk * 16);
    tn = local / rows;
    tm = chunk * 16 + (local - tn * rows);
}

template <int FMT, typename OUT>
__global__ void __launch_bounds__(PR_THREADS, 1)
gemm_pair_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_as,
                 const __grid_constant__ CUtensorMap map_bs, const __grid_constant__ CUtensorMap map_out, const __grid_constant__ GemmArgs g) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t bars[2 * PR_STAGES + 2];
    __shared__ uint32_t tmem_base_sh;
    __shared__ int abort_sh;
    constexpr int SB = scale_blocks(FMT);
    constexpr uint32_t STAGE = (pr_stage_bytes(FMT) + 1023) / 1024 * 1024, B_OFF = 128 * 128, AS_OFF = 2 * B_OFF, BS_OFF = AS_OFF + SB * BLOCK_BYTES;
    constexpr uint32_t SF_COL = 256;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = (int)cluster_rank();
    const int pair = (int)blockIdx.x >> 1, pairs = (int)gridDim.x >> 1;
    const int tiles_m = (g.M + PR_TILE - 1) / PR_TILE, tiles_n = (g.N + PR_TILE - 1) / PR_TILE, tiles = tiles_m * tiles_n;
    const int kbs = (g.K + KB - 1) / KB, sb_row = (g.K / group(FMT) + 3) / 4;

    uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    const uint32_t smem_base = smem_u32(smem), bar0 = smem_u32(&bars[0]);
    auto full = [&](int s) { return bar0 + 8u * (uint32_t)s; };
    auto empty = [&](int s) { return bar0 + 8u * (uint32_t)(PR_STAGES + s); };
    const uint32_t acc_full = bar0 + 16u * PR_STAGES, acc_empty = acc_full + 8u;
    volatile int* abort_flag = &abort_sh;

    if (threadIdx.x == 0) {
        for (int s = 0; s < PR_STAGES; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
        mbar_init(acc_full, 1);
        mbar_init(acc_empty, 16);                // the epilogue warps of both CTAs
        abort_sh = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base_sh)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    cluster_sync_all();                          // the peer's barriers exist before anything arrives on them
    tc_fence_after();
    pdl_trigger();
    const uint32_t tmem = tmem_base_sh;

    int issued = 0;
    if (warp == 0) {
        if (elect_one()) {
            pdl_wait();
            bool ok = true;
            Ring r(0, PR_STAGES);
            for (int id = pair; id < tiles && ok; id += pairs) {
                int tm, tn;
                pair_tile(id, tiles_m, tiles_n, tm, tn);
                for (int kb = 0; kb < kbs && ok; ++kb, r.next(PR_STAGES)) {
                    if (issued >= PR_STAGES) ok = mbar_wait(empty(r.slot), r.phase ^ 1u, abort_flag);
                    if (!ok) break;
                    const uint32_t slot = smem_base + (uint32_t)r.slot * STAGE, bar = mapa_u32(full(r.slot), 0);
                    if (rank == 0) mbar_expect_tx(full(r.slot), 2 * pr_stage_bytes(FMT));      // of both CTAs
                    tma_load_2d_pair(slot, &map_a, bar, kb * 128, (tm * 2 + rank) * 128);
                    tma_load_2d_pair(slot + B_OFF, &map_b, bar, kb * 128, (tn * 2 + rank) * 128);
                    tma_load_2d_pair(slot + AS_OFF, &map_as, bar, 0, (tm * 2 + rank) * sb_row + kb * SB);
                    tma_load_2d_pair(slot + BS_OFF, &map_bs, bar, 0, (tn * 2) * sb_row + kb * SB);
                    tma_load_2d_pair(slot + BS_OFF + SB * BLOCK_BYTES, &map_bs, bar, 0, (tn * 2 + 1) * sb_row + kb * SB);
                    ++issued;
                }
            }
        }
    } else if (warp == 1) {
        if (rank == 0 && elect_one()) {
            bool ok = true;
            Ring r(0, PR_STAGES);
            int n = 0;                           // tiles of this pair
            uint32_t set = 0;
            for (int id = pair; id < tiles && ok; id += pairs, ++n) {
                if (n > 0) ok = mbar_wait(acc_empty, (uint32_t)(n - 1) & 1u, abort_flag);
                tc_fence_after();
                for (int kb = 0; kb < kbs && ok; ++kb, r.next(PR_STAGES), set ^= 1u) {
                    ok = mbar_wait(full(r.slot), r.phase, abort_flag);
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t slot = smem_base + (uint32_t)r.slot * STAGE;
                    const int steps = min(4, (g.K - kb * KB) / 64), blocks = min(SB, sb_row - kb * SB);
                    const uint32_t sf_a = tmem + SF_COL + set * 64u, sf_b = sf_a + 16u;
                    for (int c = 0; c < blocks; ++c) {
                        copy_scales_pair(sf_a + 4u * (uint32_t)c, smem_desc_scales(slot + AS_OFF + (uint32_t)c * BLOCK_BYTES));
                        copy_scales_pair(sf_b + 8u * (uint32_t)c, smem_desc_scales(slot + BS_OFF + (uint32_t)c * BLOCK_BYTES));
                        copy_scales_pair(sf_b + 8u * (uint32_t)c + 4u, smem_desc_scales(slot + BS_OFF + (uint32_t)(SB + c) * BLOCK_BYTES));
                    }
                    const uint64_t da = smem_desc_sw128(slot), db = smem_desc_sw128(slot + B_OFF);
                    for (int s = 0; s < steps; ++s) {
                        const uint32_t c = (uint32_t)(FMT == NV ? s : s >> 1), byte = FMT == NV ? 0u : (uint32_t)(s & 1) * 2u;
                        umma_fp4_pair<FMT>(tmem, da + (uint64_t)(2 * s), db + (uint64_t)(2 * s), instr_desc_fp4<FMT>(PR_TILE, PR_TILE, byte), sf_a + 4u * c,
                                           sf_b + 8u * c, kb > 0 || s > 0 ? 1u : 0u);
                    }
                    umma_commit_pair(empty(r.slot));
                }
                umma_commit_pair(acc_full);      // (also on failure: the epilogue then sees the abort flag, or its own wait runs out)
            }
        }
    } else if (warp >= 4) {
        pdl_wait();
        const float2 scale = tensor_factors(g.ta, g.tb);
        const int quarter = warp & 3, half = (warp - 4) >> 2;
        const uint32_t taddr = tmem + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(half * 128);
        constexpr int PER = 128 / sizeof(OUT), BOXES = 128 / PER;        // columns of a box, boxes of this warp's 128 columns
        const uint32_t box = smem_base + PR_STAGES * STAGE + (uint32_t)(warp - 4) * PR_BOX;
        bool ok = true;
        int n = 0;
        for (int id = pair; id < tiles; id += pairs, ++n) {
            int tm, tn;
            pair_tile(id, tiles_m, tiles_n, tm, tn);
            if (ok) ok = mbar_wait(acc_full, (uint32_t)n & 1u, abort_flag) && !*abort_flag;
            ok = __all_sync(0xffffffffu, ok) != 0;
            tc_fence_after();
            uint32_t v[8][16];
#pragma unroll
            for (int c = 0; c < 8; ++c) tmem_ld16_issue(taddr + (uint32_t)(16 * c), v[c]);
#pragma unroll
            for (int c = 0; c < 8; ++c) tmem_ld_wait16(v[c]);
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(mapa_u32(acc_empty, 0));
            float last = scale.x;                // (one multiplication an output where one is enough: two cost 1.3 % at 8192 x 24576 x 4096)
            if (__builtin_expect(scale.y != 1.f, 0)) {
                last = scale.y;
#pragma unroll
                for (int c = 0; c < 8; ++c)
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[c][i] = __float_as_uint(__uint_as_float(v[c][i]) * scale.x);
            }
            const int m0 = (tm * 2 + rank) * 128 + quarter * 32, n0 = tn * PR_TILE + half * 128;
            const float nan = __uint_as_float(0x7fc00000u);      // a bounded wait gave up: NaN, not a partial sum
#pragma unroll
            for (int x = 0; x < BOXES; ++x) {
                if (m0 >= g.M || n0 + x * PER >= g.N) break;             // (the same for all lanes)
                if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");      // the store before has read the box
                __syncwarp();
#pragma unroll
                for (int c = 0; c < 8; ++c) {                            // sixteen bytes of the lane's row
                    uint32_t w[4];
                    constexpr int E = 16 / sizeof(OUT);
                    float f[E];
#pragma unroll
                    for (int i = 0; i < E; ++i) { const int col = x * PER + c * E + i; f[i] = ok ? __uint_as_float(v[col >> 4][col & 15]) * last : nan; }
                    pack16(w, f);
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(box + (uint32_t)lane * 128u + (uint32_t)((c ^ (lane & 7)) << 4)), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
                }
                if (g.box_out) {
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) {
                        asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];" ::"l"(&map_out), "r"(box), "r"(n0 + x * PER), "r"(m0) : "memory");
                        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                    }
                } else {
                    __syncwarp();
                    const uint8_t* sm = smem + (box - smem_base);
                    const int rows = min(32, g.M - m0), cols = min(PER, g.N - n0 - x * PER);
                    OUT* dst = (OUT*)g.out + (long long)m0 * g.ld + n0 + x * PER;
                    for (int r = 0; r < rows; ++r, dst += g.ld)
                        for (int c = lane; c < cols; c += 32) {
                            const int byte = c * (int)sizeof(OUT);
                            dst[c] = *reinterpret_cast<const OUT*>(sm + r * 128 + (((byte >> 4) ^ (r & 7)) << 4) + (byte & 15));
                        }
                }
            }
            __syncwarp();
        }
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
    tc_fence_before();
    __syncwarp();
    if (abort_sh && issued > 0) {                // (the even CTA's barriers count the loads of both)
        if (rank == 0) drain_ring(issued, PR_STAGES, bar0);
        else for (const long long t0 = clock64(); clock64() - t0 < 4000000;) {}
    }
    cluster_sync_all();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
}

}  // namespace fp4
}  // namespace ps
