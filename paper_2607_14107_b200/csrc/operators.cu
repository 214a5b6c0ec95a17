// Host side of the operators next to the decoding path: 4-bit rows, products and K/V caches, token log-probabilities.
// A translation unit of its own, so that it and the path compile side by side.
#include "../../include/polestar.h"

#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <climits>
#include <cmath>
#include <cstdlib>
#include <mutex>

#include "fp4.cuh"
#include "fp4_gemm.cuh"
#include "kv4_attn_tc.cuh"
#include "logprobs.cuh"

using namespace ps;

#define CK(call) do { if ((call) != cudaSuccess) return POLESTAR_E_CUDA; } while (0)

// Environment switches: read by the first call and by polestar_reload_env, never on the launch path.
//   POLESTAR_KV4_KERNEL (0 = automatic): 1 the warp-level attention kernel, 2 the tensor-core one where it applies (used by the tests)
//   POLESTAR_FP4_KERNEL (0 = automatic): 1 the product's kernel for few rows, 2 the one for many (used by the tests)
static std::atomic<int> g_kv4_kernel{-1}, g_fp4_kernel{-1};
namespace ps {
void reload_operator_switches() {
    const char *kv = getenv("POLESTAR_KV4_KERNEL"), *fp = getenv("POLESTAR_FP4_KERNEL");
    g_kv4_kernel.store(kv ? std::max(0, atoi(kv)) : 0);
    g_fp4_kernel.store(fp ? std::max(0, atoi(fp)) : 0);
}
}
static int read_switch(const std::atomic<int>& s) {
    if (s.load() < 0) reload_operator_switches();
    return s.load();
}

// Facts of the CURRENT device; the first call on a device queries them and raises the shared-memory limits of the kernels that need
// more than the default there (function attributes are per device).
struct DevInfo {
    bool ready = false;
    int sm_count = 0;
    int gemm_pairs = 0;                          // CTA pairs of the product for many rows that are resident at once ...
    int clusters[3] = {};                        // ... and clusters of 2, 4 and 8 CTAs of the one for few
};
static const int MAX_DEVICES = 64;
static std::mutex g_mu;
static DevInfo g_dev[MAX_DEVICES];
namespace ps { void note_sm_count(int n); }               // polestar.cu: what polestar_sm_count() answers
static cudaError_t set_kernel_attributes();
static void resident_clusters(DevInfo* di);
static int device_info(DevInfo* out) {
    int dev = 0;
    CK(cudaGetDevice(&dev));
    if (dev < 0 || dev >= MAX_DEVICES) return POLESTAR_E_INVAL;
    std::lock_guard<std::mutex> lk(g_mu);
    DevInfo& di = g_dev[dev];
    if (!di.ready) {
        CK(cudaDeviceGetAttribute(&di.sm_count, cudaDevAttrMultiProcessorCount, dev));
        CK(set_kernel_attributes());
        resident_clusters(&di);
        di.ready = true;
    }
    note_sm_count(di.sm_count);
    *out = di;
    return POLESTAR_OK;
}

// ------------------------------------------------------------------------------------------
// microscaled 4-bit floating point
// ------------------------------------------------------------------------------------------
static bool fp4_format_ok(int format, int layout) {
    return (format == POLESTAR_FP4_NV || format == POLESTAR_FP4_MX) && (layout == POLESTAR_SCALES_ROWS || layout == POLESTAR_SCALES_TILED);
}

extern "C" size_t polestar_k_fp4_scale_bytes(int64_t rows, int32_t d, int32_t format, int32_t layout) {
    if (!fp4_format_ok(format, layout) || rows < 0 || rows > INT32_MAX || d <= 0 || d % 32) return 0;
    const size_t groups = (size_t)d / fp4::group(format);
    if (layout == POLESTAR_SCALES_ROWS) return (size_t)rows * groups;
    return ((size_t)rows + 127) / 128 * ((groups + 3) / 4) * 512;
}

template <typename T, int FMT>
static cudaError_t launch_quantize(const fp4::QuantArgs& a, int sms, cudaStream_t st) {
    // one piece of 32 bytes per thread for few rows, two where the loads have to be many (us, one / two: 32 x 4096 bf16 2.3 / 2.6, 16384 x 4096 46 / 40, fp32 69 / 62)
    const long long pieces = a.rows * (a.d / fp4::Piece<T>::N);
    const bool deep = pieces >= 2LL * fp4::THREADS * 8 * sms;
    const long long per = fp4::THREADS * (deep ? 2LL : 1LL), blocks = (pieces + per - 1) / per;
    if (blocks > INT32_MAX) return cudaErrorInvalidValue;
    if (deep) return launch_k(fp4::quantize_kernel<T, FMT, 2>, dim3((unsigned)blocks), dim3(fp4::THREADS), 0, st, a);
    return launch_k(fp4::quantize_kernel<T, FMT, 1>, dim3((unsigned)blocks), dim3(fp4::THREADS), 0, st, a);
}

extern "C" int polestar_k_fp4_quantize(const void* x, int64_t ld_x, int32_t rows, int32_t d, int32_t dtype, int32_t format,
                                       int32_t scale_layout, const float* tensor_scale, uint8_t* codes, uint8_t* scales, void* deq,
                                       void* stream) {
    if (rows < 0 || d <= 0 || d % 32 || !fp4_format_ok(format, scale_layout)) return POLESTAR_E_INVAL;
    if (dtype != POLESTAR_F32 && dtype != POLESTAR_BF16) return POLESTAR_E_INVAL;
    const int per16 = dtype == POLESTAR_BF16 ? 8 : 4;
    if (ld_x < d || ld_x % per16) return POLESTAR_E_INVAL;
    if (rows == 0) return POLESTAR_OK;           // no rows: nothing to do (the pointers may be null)
    if (!x || !codes || !scales) return POLESTAR_E_INVAL;
    if ((((uintptr_t)x | (uintptr_t)deq) & 15) || (((uintptr_t)codes | (uintptr_t)tensor_scale) & 3)) return POLESTAR_E_INVAL;
    if (scale_layout == POLESTAR_SCALES_TILED && ((uintptr_t)scales & 3)) return POLESTAR_E_INVAL;
    DevInfo di;
    int rc = device_info(&di);
    if (rc) return rc;
    fp4::QuantArgs a;
    a.x = x; a.ld_x = ld_x; a.deq = deq; a.codes = codes; a.scales = scales; a.t = tensor_scale;
    a.rows = rows; a.d = d; a.layout = scale_layout;
    cudaStream_t st = (cudaStream_t)stream;
    const bool nv = format == POLESTAR_FP4_NV;
    if (dtype == POLESTAR_BF16) CK(nv ? (launch_quantize<__nv_bfloat16, fp4::NV>(a, di.sm_count, st)) : (launch_quantize<__nv_bfloat16, fp4::MX>(a, di.sm_count, st)));
    else CK(nv ? (launch_quantize<float, fp4::NV>(a, di.sm_count, st)) : (launch_quantize<float, fp4::MX>(a, di.sm_count, st)));
    return POLESTAR_OK;
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
static EncodeTiledFn get_encode_fn() {
    static std::atomic<EncodeTiledFn> fn{nullptr};
    EncodeTiledFn f = fn.load();
    if (!f) {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult qres;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &qres) == cudaSuccess && qres == cudaDriverEntryPointSuccess) {
            f = (EncodeTiledFn)p;
            fn.store(f);
        }
    }
    return f;
}
// rows of codes, [rows][bytes] with bytes % 16 == 0: boxes of 128 bytes x box_rows, 128-byte swizzle; what lies outside arrives as zeros
static bool make_code_map(CUtensorMap* out, const void* base, uint64_t rows, uint64_t bytes, uint32_t box_rows) {
    EncodeTiledFn fn = get_encode_fn();
    if (!fn) return false;
    cuuint64_t dims[2] = {bytes, rows};
    cuuint64_t strides[1] = {bytes};
    cuuint32_t box[2] = {128, box_rows};
    cuuint32_t estr[2] = {1, 1};
    return fn(out, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// blocks of 512 bytes of tiled scales: boxes of n blocks
static bool make_scale_map(CUtensorMap* out, const void* base, uint64_t blocks, uint32_t n) {
    EncodeTiledFn fn = get_encode_fn();
    if (!fn) return false;
    cuuint64_t dims[2] = {128, blocks};
    cuuint64_t strides[1] = {fp4::BLOCK_BYTES};
    cuuint32_t box[2] = {128, n};
    cuuint32_t estr[2] = {1, 1};
    return fn(out, CU_TENSOR_MAP_DATA_TYPE_UINT32, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// output rows of whole 16 bytes: boxes of 32 rows x 128 bytes, 128-byte swizzle
static bool make_out_map(CUtensorMap* out, void* base, uint64_t rows, uint64_t cols, uint64_t ld, int es) {
    EncodeTiledFn fn = get_encode_fn();
    if (!fn) return false;
    cuuint64_t dims[2] = {cols, rows};
    cuuint64_t strides[1] = {ld * es};
    cuuint32_t box[2] = {(cuuint32_t)(128 / es), 32};
    cuuint32_t estr[2] = {1, 1};
    return fn(out, es == 2 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 2, base, dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
template <int FMT, typename OUT>
static int launch_gemm_pair(const uint8_t* a, const uint8_t* b, fp4::GemmArgs g, int pairs, cudaStream_t st) {
    const uint64_t sb_row = ((uint64_t)g.K / fp4::group(FMT) + 3) / 4, rows_a = ((uint64_t)g.M + 127) / 128, rows_b = ((uint64_t)g.N + 127) / 128;
    CUtensorMap ma, mb, mas, mbs;
    if (!make_code_map(&ma, a, g.M, g.K / 2, 128) || !make_code_map(&mb, b, g.N, g.K / 2, 128) ||
        !make_scale_map(&mas, g.as, rows_a * sb_row, fp4::scale_blocks(FMT)) || !make_scale_map(&mbs, g.bs, rows_b * sb_row, fp4::scale_blocks(FMT)))
        return POLESTAR_E_CUDA;
    // (strides of a tensor map stay below 2^40)
    CUtensorMap mo = ma;
    g.box_out = (((uintptr_t)g.out | (uintptr_t)(g.ld * (long long)sizeof(OUT)) | (uintptr_t)((size_t)g.N * sizeof(OUT))) & 15) == 0 && g.ld < (1LL << 36);
    if (g.box_out && !make_out_map(&mo, g.out, g.M, g.N, g.ld, (int)sizeof(OUT))) return POLESTAR_E_CUDA;
    const long long tiles = (((long long)g.M + fp4::PR_TILE - 1) / fp4::PR_TILE) * (((long long)g.N + fp4::PR_TILE - 1) / fp4::PR_TILE);
    if (tiles > INT32_MAX / 2) return POLESTAR_E_INVAL;
    const unsigned n = (unsigned)std::min<long long>(tiles, pairs);
    CK(launch_k_cluster(fp4::gemm_pair_kernel<FMT, OUT>, dim3(2 * n), dim3(fp4::PR_THREADS), fp4::pr_smem_bytes(FMT), st, 2u, ma, mb, mas, mbs, mo, g));
    return POLESTAR_OK;
}

template <int T, int FMT, typename OUT>
static int launch_gemm_stream(const uint8_t* a, const uint8_t* b, fp4::GemmArgs g, const DevInfo& di, cudaStream_t st) {
    CUtensorMap ma, mb;
    if (!make_code_map(&ma, a, g.M, g.K / 2, T) || !make_code_map(&mb, b, g.N, g.K / 2, 128)) return POLESTAR_E_CUDA;
    const long long tiles_n = ((long long)g.N + 127) / 128, tiles_m = ((long long)g.M + T - 1) / T;
    const int kbs = (g.K + fp4::KB - 1) / fp4::KB;
    // The CTAs of a cluster share K while all clusters run at once and each has two slots of K: a slot takes 0.4 us, handing the sums over 1.0 us and 0.016 us a row.  (us,
    // not split / split in 2, 4, 8: 1 row, 1024 x 4096 8.5 / 6.3, 4.7, 4.1; 128 rows, 1024 x 4096 9.5 / 9.1, 7.5, 7.3; 128 rows, 512 x 1024 4.5 / 6.6.)
    g.split = 1;
    double least = 0.4 * kbs;
    for (int i = 0; i < 3 && tiles_n * tiles_m <= di.clusters[i] && 4 << i <= kbs; ++i) {
        const double us = 0.4 * kbs / (2 << i) + 1.0 + 0.016 * std::min(T, g.M);
        if (us < least) { least = us; g.split = 2 << i; }
    }
    if (tiles_m > 65535 || tiles_n * g.split > INT32_MAX) return POLESTAR_E_INVAL;
    const dim3 grid((unsigned)(tiles_n * g.split), (unsigned)tiles_m);
    // more tiles than SMs: two CTAs on each, with half the slots, so that one's start and end pass under the other's stream (us, one / two: 32 rows,
    // 37888 x 3584 19.7 / 14.3, 126464 x 4096 69.5 / 51.2; 128 rows, 126464 x 4096 93 / 64)
    const int per_sm = tiles_n * tiles_m > di.sm_count ? 2 : 1;
    const size_t smem = fp4::st_smem_bytes(T, FMT, per_sm);
    g.stages = fp4::st_stages(T, FMT, per_sm);
    if (g.split > 1) CK(launch_k_cluster(fp4::gemm_stream_kernel<T, FMT, OUT>, grid, dim3(fp4::ST_THREADS), smem, st, (unsigned)g.split, ma, mb, g));
    else CK(launch_k(fp4::gemm_stream_kernel<T, FMT, OUT>, grid, dim3(fp4::ST_THREADS), smem, st, ma, mb, g));
    return POLESTAR_OK;
}
// Which kernel: the one for few rows up to 128 of them, and beyond while its tiles of 128 x 128 run at once, one to an SM, or two where the pairs' tiles of
// 256 x 256 would take two rounds.  us, few / many: 128 rows, 37888 x 3584 15.9 / 24.2; 256 rows, 4096 x 12288 16.7 / 24.8; 512 rows, 4096 x 4096 10.4 /
// 11.8 (128 tiles), 1024 rows 12.4 / 12.6 (256); 384 rows, 12288 x 4096 13.0 / 20.4 (288), 512 rows 22.3 / 20.4 (384).
template <int FMT, typename OUT>
static int launch_gemm_fp4(const uint8_t* a, const uint8_t* b, const fp4::GemmArgs& g, const DevInfo& di, cudaStream_t st) {
    auto tiles = [&](long long size) { return ((g.M + size - 1) / size) * ((g.N + size - 1) / size); };
    const int forced = read_switch(g_fp4_kernel);
    const bool few = g.M <= 128 || tiles(128) <= di.sm_count || (tiles(128) <= 2 * di.sm_count && tiles(fp4::PR_TILE) > di.gemm_pairs);
    if (di.gemm_pairs > 0 && (forced ? forced == 2 : !few)) return launch_gemm_pair<FMT, OUT>(a, b, g, di.gemm_pairs, st);
    if (g.M <= 32) return launch_gemm_stream<32, FMT, OUT>(a, b, g, di, st);
    if (g.M <= 64) return launch_gemm_stream<64, FMT, OUT>(a, b, g, di, st);
    return launch_gemm_stream<128, FMT, OUT>(a, b, g, di, st);
}

extern "C" int polestar_k_fp4_matmul(const uint8_t* a_codes, const uint8_t* a_scales, const uint8_t* b_codes, const uint8_t* b_scales,
                                     const float* a_tensor_scale, const float* b_tensor_scale, void* out, int64_t ld_out, int32_t M,
                                     int32_t N, int32_t K, int32_t format, int32_t out_dtype, void* stream) {
    if (M < 0 || N < 0 || K <= 0 || K % 64 || ld_out < N || !fp4_format_ok(format, POLESTAR_SCALES_TILED)) return POLESTAR_E_INVAL;
    static_assert(fp4::KB <= 256 && fp4::PR_TILE <= 256, "sizes are rounded up to these in 32 bits");
    if (std::max(M, std::max(N, K)) > INT32_MAX - 255) return POLESTAR_E_INVAL;
    if (out_dtype != POLESTAR_F32 && out_dtype != POLESTAR_BF16) return POLESTAR_E_INVAL;
    if (M == 0 || N == 0) return POLESTAR_OK;    // nothing to compute (the pointers may be null)
    if (!a_codes || !a_scales || !b_codes || !b_scales || !out) return POLESTAR_E_INVAL;
    if (((uintptr_t)a_codes | (uintptr_t)a_scales | (uintptr_t)b_codes | (uintptr_t)b_scales) & 15) return POLESTAR_E_INVAL;
    if (((uintptr_t)out & (out_dtype == POLESTAR_BF16 ? 1 : 3)) || (((uintptr_t)a_tensor_scale | (uintptr_t)b_tensor_scale) & 3)) return POLESTAR_E_INVAL;
    DevInfo di;
    int rc = device_info(&di);
    if (rc) return rc;
    fp4::GemmArgs g;
    g.as = a_scales; g.bs = b_scales; g.ta = a_tensor_scale; g.tb = b_tensor_scale; g.out = out; g.ld = ld_out;
    g.M = M; g.N = N; g.K = K; g.split = 1; g.box_out = 0;
    cudaStream_t st = (cudaStream_t)stream;
    const bool nv = format == POLESTAR_FP4_NV;
    if (out_dtype == POLESTAR_BF16)
        return nv ? launch_gemm_fp4<fp4::NV, __nv_bfloat16>(a_codes, b_codes, g, di, st) : launch_gemm_fp4<fp4::MX, __nv_bfloat16>(a_codes, b_codes, g, di, st);
    return nv ? launch_gemm_fp4<fp4::NV, float>(a_codes, b_codes, g, di, st) : launch_gemm_fp4<fp4::MX, float>(a_codes, b_codes, g, di, st);
}

// A cache of keys and values in 4 bits: what append and attention accept of its geometry.
static bool kv4_shape_ok(int batch, int R, int cap, int n_kv, int head_dim) {
    return batch >= 0 && batch <= 65535 && R >= 0 && cap > 0 && cap <= 65536 && n_kv > 0 && n_kv <= 1024 && (head_dim == 64 || head_dim == 128);
}

extern "C" int polestar_k_kv4_append(const void* k, const void* v, const int32_t* idx, const int32_t* count, int32_t batch, int32_t R,
                                     int32_t cap, int32_t n_kv, int32_t head_dim, int32_t dtype, const float* k_scale,
                                     const float* v_scale, uint8_t* kc, uint8_t* ks, uint8_t* vc, uint8_t* vs, void* k_deq, void* v_deq,
                                     void* stream) {
    if (!kv4_shape_ok(batch, R, cap, n_kv, head_dim) || R > 65536) return POLESTAR_E_INVAL;
    if (dtype != POLESTAR_F32 && dtype != POLESTAR_BF16) return POLESTAR_E_INVAL;
    if (batch == 0 || R == 0) return POLESTAR_OK;         // no rows: nothing to do (the pointers may be null)
    if (!k || !v || !kc || !ks || !vc || !vs) return POLESTAR_E_INVAL;
    if (((uintptr_t)k | (uintptr_t)v | (uintptr_t)k_deq | (uintptr_t)v_deq) & 15) return POLESTAR_E_INVAL;
    if (((uintptr_t)kc | (uintptr_t)vc | (uintptr_t)idx | (uintptr_t)count | (uintptr_t)k_scale | (uintptr_t)v_scale) & 3) return POLESTAR_E_INVAL;
    DevInfo di;
    int rc = device_info(&di);
    if (rc) return rc;
    fp4::AppendArgs a;
    a.x[0] = k; a.x[1] = v; a.deq[0] = k_deq; a.deq[1] = v_deq; a.codes[0] = kc; a.codes[1] = vc; a.scales[0] = ks; a.scales[1] = vs;
    a.t[0] = k_scale; a.t[1] = v_scale; a.idx = idx; a.counts = count; a.R = R; a.cap = cap; a.width = n_kv * head_dim;
    // rows of a block: two rounds of loads' worth while there are eight blocks for every SM; more, and fewer blocks, where the list is longer than what a block
    // writes, since each looks through the rest of it
    const int pieces = a.width / (dtype == POLESTAR_BF16 ? fp4::Piece<__nv_bfloat16>::N : fp4::Piece<float>::N);
    int rpb = std::max(1, fp4::THREADS / pieces);
    while (rpb * 2 <= fp4::APPEND_MAX_ROWS) {
        const bool longer = idx && R > 2 * rpb * pieces;
        if (!longer && rpb * pieces >= 4 * fp4::THREADS) break;
        if (2LL * batch * ((R + 2 * rpb - 1) / (2 * rpb)) < (longer ? 3LL : 8LL) * di.sm_count) break;
        rpb *= 2;
    }
    a.rows_per_block = std::min(rpb, fp4::APPEND_MAX_ROWS);
    const dim3 grid((R + a.rows_per_block - 1) / a.rows_per_block, batch, 2);
    if (dtype == POLESTAR_BF16) CK(launch_k(fp4::kv_append_kernel<__nv_bfloat16>, grid, dim3(fp4::THREADS), 0, (cudaStream_t)stream, a));
    else CK(launch_k(fp4::kv_append_kernel<float>, grid, dim3(fp4::THREADS), 0, (cudaStream_t)stream, a));
    return POLESTAR_OK;
}

constexpr size_t KV4_PARTS_BYTES = 65536 * sizeof(int);       // front of the scratch: parts of every sequence
// Plans of the attention kernels: functions of the sizes alone, so that a scratch of polestar_k_kv4_scratch_bytes() bytes suffices for every call of
// these sizes.  Parts of the keys: up to MAX_BATCH sequences share `slots` of them, so that ragged lengths leave no SM idle, more have the same number each.
static int kv4_slots(long long batch, long long wanted) {
    wanted = std::max(batch, std::min(wanted, batch * kv4::MAX_SPLIT));
    return (int)(batch > kv4::MAX_BATCH ? wanted / batch * batch : wanted);
}
static int kv4_parts(int batch, int slots) {         // of one sequence, at most
    return batch > kv4::MAX_BATCH ? slots / batch : std::min(kv4::MAX_SPLIT, slots - batch + 1);
}
// What joining rows of c parts takes: a CTA a row, 520 bytes a part written and read.  (us, 128-wide heads: 2048 rows of 4 parts 7, 8192 rows of 2 and 4 parts 12 and 17, 16384
// rows of 4 parts 39.)
static double kv4_join_us(double rows_total, double c) { return 3.0 + rows_total * (c * 1040 / 3e6 + 1.5 / (16 * 148)); }
// The warp-level kernel: tiles of 8 or 16 rows, four CTAs for every SM, no part of a full sequence shorter than 512 keys, and none at all up to 1024 (joining
// takes what it gains).
struct Kv4Warp { int tiles, rows, slots; };
static Kv4Warp kv4_warp_plan(long long batch, long long R, int cap, int n_heads, int n_kv) {
    const long long vrows = R * (n_heads / n_kv);
    Kv4Warp p;
    p.rows = vrows <= 8 ? 8 : 16;
    p.tiles = (int)((vrows + p.rows - 1) / p.rows);
    p.slots = kv4_slots(batch, std::min(4 * 148LL / std::max<long long>(1, (long long)n_kv * p.tiles), cap <= 1024 ? batch : batch * ((cap + 511) / 512)));
    if (p.slots < 2 * batch) p.slots = (int)batch;        // (a few slots more than sequences are not worth joining for)
    return p;
}
// The tensor-core kernel, one CTA per SM: row tiles of 128, one per CTA with its keys split between the streams, or two per CTA.  Two share the turning of
// codes (a pair takes 2.5 us for 128 keys, one tile 2.1, one of up to 64 rows 1.4), one gives more CTAs where there are few.  Whichever needs less time, by those figures, 6 us for
// the start and end of a CTA, which nothing hides on its SM, 2.5 us for the launch and what joining parts takes; a part of a sequence that fills the cache is no shorter than
// four key tiles.  (us, parts of 16, 8, 4 key tiles, 64 rows, 2048 keys, 32 heads: 4 sequences 30, 49, 66; 8 sequences 60, 98, 123; 1 sequence 31, -, 19.)
struct Kv4Tc { int tiles, key_split, slots; double us; };
static Kv4Tc kv4_tc_plan(long long batch, long long R, int cap, int n_heads, int n_kv) {
    const long long vrows = R * (n_heads / n_kv), row_tiles = (vrows + kv4::TC_ROWS - 1) / kv4::TC_ROWS, key_tiles = (cap + kv4::TC_KEYS - 1) / kv4::TC_KEYS;
    Kv4Tc p;
    p.us = 1e30;
    for (int one = 1; one >= 0; --one) {
        if (!one && row_tiles == 1) continue;
        const long long tiles = one ? row_tiles : (row_tiles + 1) / 2, per = (long long)n_kv * tiles;
        const double tile_us = !one ? 2.5 : vrows <= 64 ? 1.4 : 2.1;
        for (int w = 0; w <= 8; ++w) {           // waves of CTAs; 0: a part for each sequence, whatever that takes
            const int slots = w ? kv4_slots(batch, std::min(148LL * w / per, batch * key_tiles / 4)) : (int)batch;
            const long long c = slots / batch;
            if (w && c < 2) continue;
            const double us = (double)((per * slots + 147) / 148) * ((double)((key_tiles + c - 1) / c) * tile_us + 6.0) + 2.5 + (c > 1 ? kv4_join_us((double)batch * R * n_heads, (double)c) : 0.0);
            if (us >= 0.97 * p.us) continue;
            p.us = us; p.key_split = one; p.tiles = (int)tiles; p.slots = slots;
        }
    }
    return p;
}
// Which kernel: the warp-level one turns codes again for every 16 rows, the tensor-core one once for 128 or 256, but it starts slowly and its rows fill whole
// tiles.  The warp-level one's time as measured: 1.0 us for 16 rows x 128 keys on an SM, or, three CTAs per SM at a time, 1.4 us of latency for 128 keys of a
// part while the CTAs have an SM for two of theirs, 3.2 us once they share them (2.4 in long parts), all of it times 0.75 for 8 rows, and 5 us and the joining.  us, warp-level / tensor-core:
// 7 rows a K/V head, eight ragged sequences of up to 32768 keys 36 / 112; 32 heads, 32 rows, 512 keys 12.9 / 12.7, 8 x 2048 keys 78 / 59; 64 rows, 2048 keys 33 / 19, 8 x 2048
// 121 / 60; 63 rows x 4 heads, 2048 keys 14.5 / 17.3, 8 x 2048 32 / 20; 896 rows, 65536 keys x 4 heads 814 / 155.  (Next to the border it can be a tenth off: 63 rows x 4
// heads over 2 x 2048 keys take 15.8 / 17.4, and it picks the second.)
static bool kv4_use_tc(int dtype, int head_dim, const Kv4Warp& w, const Kv4Tc& t, long long batch, long long R, int cap, int n_heads, int n_kv) {
    if (dtype != POLESTAR_BF16 || head_dim != kv4::TC_DH) return false;
    const int forced = read_switch(g_kv4_kernel);
    if (forced) return forced == 2;
    const double ctas = (double)w.slots * n_kv * w.tiles, part = std::ceil((double)((cap + 127) / 128) * batch / w.slots);
    const double all = (double)batch * n_kv * w.tiles * ((cap + 127) / 128);
    double tile = 1.4 + 1.8 * std::min(1.0, std::max(0.0, (ctas - 74) / 100));
    if (part >= 8) tile = std::min(tile, 2.4);
    const double join = w.slots > batch ? kv4_join_us((double)batch * R * n_heads, (double)w.slots / batch) : 0.0;
    return t.us < (w.rows == 8 ? 0.75 : 1.0) * std::max(all / 148, std::max(1.0, ctas / 444) * part * tile) + 5 + join;
}
static bool kv4_attention_shape_ok(int batch, int R, int cap, int n_heads, int n_kv, int head_dim) {
    return kv4_shape_ok(batch, R, cap, n_kv, head_dim) && R <= 65536 && n_heads > 0 && n_heads <= 1024 && n_heads % n_kv == 0;
}

extern "C" size_t polestar_k_kv4_scratch_bytes(int32_t batch, int32_t R, int32_t cap, int32_t n_heads, int32_t n_kv, int32_t head_dim) {
    if (!kv4_attention_shape_ok(batch, R, cap, n_heads, n_kv, head_dim)) return 0;
    const size_t rows = (size_t)batch * R * n_heads;
    if (rows == 0) return 256;
    const int parts = std::max(kv4_parts(batch, kv4_warp_plan(batch, R, cap, n_heads, n_kv).slots), kv4_parts(batch, kv4_tc_plan(batch, R, cap, n_heads, n_kv).slots));
    return 256 + KV4_PARTS_BYTES + (parts > 1 ? parts * rows * ((size_t)head_dim * 4 + 8) : 0);
}

template <typename T, int DH>
static int launch_kv4_join(const kv4::Args& a, cudaStream_t st) {
    if (a.part_n) CK(launch_k(kv4::kv4_attn_join_kernel<T, DH>, dim3((unsigned)a.rows_total), dim3(kv4::JOIN_THREADS), 0, st, a));
    return POLESTAR_OK;
}
static int launch_kv4_tc(const kv4::Args& a, const Kv4Tc& p, cudaStream_t st) {
    kv4::TcArgs f;
    f.a = a; f.tiles = p.tiles; f.key_split = p.key_split;
    if ((long long)p.tiles * p.slots > INT32_MAX) return POLESTAR_E_INVAL;
    CK(launch_k(kv4::kv4_attn_tc_kernel, dim3((unsigned)(p.tiles * p.slots), a.n_kv), dim3(kv4::TC_THREADS), kv4::TC_SMEM, st, f));
    return launch_kv4_join<__nv_bfloat16, 128>(a, st);
}
template <typename T, int DH, int NB>
static int launch_kv4_warp(const kv4::Args& a, const Kv4Warp& p, cudaStream_t st) {
    if ((long long)p.tiles * p.slots > INT32_MAX) return POLESTAR_E_INVAL;
    CK(launch_k(kv4::kv4_attn_warp_kernel<T, DH, NB>, dim3((unsigned)(p.tiles * p.slots), a.n_kv), dim3(kv4::THREADS), kv4::warp_smem_bytes<DH, NB>(), st, a));
    return launch_kv4_join<T, DH>(a, st);
}
template <typename T>
static int launch_kv4_warp(const kv4::Args& a, const Kv4Warp& p, int head_dim, cudaStream_t st) {
    if (head_dim == 128) return p.rows == 8 ? launch_kv4_warp<T, 128, 1>(a, p, st) : launch_kv4_warp<T, 128, 2>(a, p, st);
    return p.rows == 8 ? launch_kv4_warp<T, 64, 1>(a, p, st) : launch_kv4_warp<T, 64, 2>(a, p, st);
}

extern "C" int polestar_k_kv4_attention(const void* q, const uint8_t* kc, const uint8_t* ks, const uint8_t* vc, const uint8_t* vs,
                                        const float* k_scale, const float* v_scale, const int32_t* lens, void* out, float* lse,
                                        int32_t batch, int32_t R, int32_t cap, int32_t n_heads, int32_t n_kv, int32_t head_dim,
                                        int32_t dtype, void* scratch, size_t scratch_bytes, void* stream) {
    if (!kv4_attention_shape_ok(batch, R, cap, n_heads, n_kv, head_dim)) return POLESTAR_E_INVAL;
    if (dtype != POLESTAR_F32 && dtype != POLESTAR_BF16) return POLESTAR_E_INVAL;
    if (batch == 0 || R == 0) return POLESTAR_OK;         // no rows: nothing to do (the pointers may be null)
    if (!q || !kc || !ks || !vc || !vs || !out || !scratch) return POLESTAR_E_INVAL;
    if (((uintptr_t)q | (uintptr_t)out | (uintptr_t)kc | (uintptr_t)vc | (uintptr_t)ks | (uintptr_t)vs | (uintptr_t)scratch) & 15) return POLESTAR_E_INVAL;
    if (((uintptr_t)k_scale | (uintptr_t)v_scale | (uintptr_t)lens | (uintptr_t)lse) & 3) return POLESTAR_E_INVAL;
    if (scratch_bytes < polestar_k_kv4_scratch_bytes(batch, R, cap, n_heads, n_kv, head_dim)) return POLESTAR_E_NOSPACE;
    DevInfo di;
    int rc = device_info(&di);
    if (rc) return rc;
    kv4::Args a;
    a.q = q; a.out = out; a.lse = lse; a.kc = kc; a.ks = ks; a.vc = vc; a.vs = vs; a.tk = k_scale; a.tv = v_scale; a.lens = lens;
    a.batch = batch; a.R = R; a.cap = cap; a.n_heads = n_heads; a.n_kv = n_kv; a.rows_total = (long long)batch * R * n_heads;
    const Kv4Tc plan = kv4_tc_plan(batch, R, cap, n_heads, n_kv);
    const Kv4Warp wplan = kv4_warp_plan(batch, R, cap, n_heads, n_kv);
    const bool tc = kv4_use_tc(dtype, head_dim, wplan, plan, batch, R, cap, n_heads, n_kv);
    a.slots = tc ? plan.slots : wplan.slots;
    const int parts = kv4_parts(batch, a.slots);
    a.part_n = parts > 1 ? (int*)scratch : nullptr;
    a.part_o = (float*)((char*)scratch + KV4_PARTS_BYTES);
    a.part_ml = (float2*)((char*)a.part_o + (size_t)parts * a.rows_total * head_dim * 4);
    a.scale = 1.4426950408889634 / std::sqrt((double)head_dim);
    cudaStream_t st = (cudaStream_t)stream;
    if (tc) return launch_kv4_tc(a, plan, st);
    if (dtype == POLESTAR_BF16) return launch_kv4_warp<__nv_bfloat16>(a, wplan, head_dim, st);
    return launch_kv4_warp<float>(a, wplan, head_dim, st);
}

// ------------------------------------------------------------------------------------------
// token log-probabilities
// ------------------------------------------------------------------------------------------
extern "C" int polestar_k_token_logprobs(const void* logits, int64_t ld, int32_t rows, int32_t vocab, int32_t dtype,
                                         const int32_t* target, int32_t mask_id, int32_t top_k, float* logprob, float* entropy,
                                         int32_t* top_ids, float* top_logprobs, void* stream) {
    if (rows < 0 || vocab <= 0 || top_k < 0 || top_k > POLESTAR_LOGPROBS_MAX_TOP || ld < vocab) return POLESTAR_E_INVAL;
    if (dtype != POLESTAR_F32 && dtype != POLESTAR_BF16) return POLESTAR_E_INVAL;
    if (rows == 0) return POLESTAR_OK;           // no rows: nothing to do (the pointers may be null)
    if (!logits || (logprob && !target) || (top_k > 0 && (!top_ids || !top_logprobs))) return POLESTAR_E_INVAL;
    const int es = dtype == POLESTAR_BF16 ? 2 : 4;
    if (((uintptr_t)logits & (es - 1)) || (((uintptr_t)target | (uintptr_t)logprob | (uintptr_t)entropy | (uintptr_t)top_ids | (uintptr_t)top_logprobs) & 3))
        return POLESTAR_E_INVAL;
    DevInfo di;
    int rc = device_info(&di);
    if (rc) return rc;
    lpr::Args a;
    a.x = logits; a.ld = ld; a.target = target; a.logprob = logprob; a.entropy = entropy; a.top_ids = top_ids; a.top_logprobs = top_logprobs;
    a.V = vocab; a.mask_id = mask_id >= 0 && mask_id < vocab ? mask_id : -1; a.k = top_k;
    // Threads of a row: as many as have a batch of loads each, 256 in any case, up to 2048 while the threads of all rows are resident at once (64 registers: 1024 to an SM),
    // 4096 for a few rows.  us for 126464 fp32 logits without / with 8 alternatives, as many threads as this, half, twice: 64 rows 11 / 14, 14 / 17, 16 / 24; 128 rows
    // 17 / 20, 23 / 26, 20 / 28; 512 rows 48 / 55, 70 / 86, 51 / 60; 1 row 5.2 / 8.1, 6.2 / 8.8.  In CTAs of 512 rather than 256, which leaves less to put together
    // (128 rows, 20 alternatives 21 / 25; none 16.7 / 16.3); the same with and without alternatives, so that sums are.
    const long long fit = vocab * (long long)es / (16 * lpr::U);
    int per_row = 128;
    for (int next = 256; next <= lpr::MAX_CL * lpr::MAX_THREADS && next <= fit; next *= 2) {
        if (next > 256 && (long long)next * rows > 1040LL * di.sm_count) break;
        if (next > 2048 && 16LL * rows > di.sm_count) break;
        per_row = next;
    }
    a.cl = std::min(lpr::MAX_CL, std::max(1, per_row / lpr::MAX_THREADS));
    const int threads = std::min(lpr::MAX_THREADS, per_row / a.cl);
    const long long blocks = (long long)rows * a.cl;
    if (blocks > INT32_MAX) return POLESTAR_E_INVAL;
    cudaStream_t st = (cudaStream_t)stream;
    auto kern = dtype == POLESTAR_BF16 ? lpr::token_logprobs_kernel<__nv_bfloat16> : lpr::token_logprobs_kernel<float>;
    if (a.cl > 1) CK(launch_k_cluster(kern, dim3((unsigned)blocks), dim3(threads), 0, st, (unsigned)a.cl, a));
    else CK(launch_k(kern, dim3((unsigned)blocks), dim3(threads), 0, st, a));
    return POLESTAR_OK;
}

// kernels with more shared memory than the default limit
template <int T, int FMT>
static cudaError_t stream_attributes() {
    const int n = (int)fp4::st_smem_bytes(T, FMT, 1);
    cudaError_t e = cudaFuncSetAttribute(fp4::gemm_stream_kernel<T, FMT, float>, cudaFuncAttributeMaxDynamicSharedMemorySize, n);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(fp4::gemm_stream_kernel<T, FMT, __nv_bfloat16>, cudaFuncAttributeMaxDynamicSharedMemorySize, n);
    return e;
}
template <int FMT>
static cudaError_t pair_attributes() {
    const int n = (int)fp4::pr_smem_bytes(FMT);
    cudaError_t e = cudaFuncSetAttribute(fp4::gemm_pair_kernel<FMT, float>, cudaFuncAttributeMaxDynamicSharedMemorySize, n);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(fp4::gemm_pair_kernel<FMT, __nv_bfloat16>, cudaFuncAttributeMaxDynamicSharedMemorySize, n);
    return e;
}
static int resident(const void* kernel, int cluster, int threads, size_t smem, int sms) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(cluster * sms); cfg.blockDim = dim3(threads); cfg.dynamicSmemBytes = smem;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = cluster; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    cfg.attrs = at; cfg.numAttrs = 1;
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess) { cudaGetLastError(); return 0; }
    return n;
}
static void resident_clusters(DevInfo* di) {
    di->gemm_pairs = resident((const void*)fp4::gemm_pair_kernel<fp4::NV, __nv_bfloat16>, 2, fp4::PR_THREADS, fp4::pr_smem_bytes(fp4::NV), di->sm_count);
    for (int i = 0; i < 3; ++i)
        di->clusters[i] = resident((const void*)fp4::gemm_stream_kernel<128, fp4::NV, __nv_bfloat16>, 2 << i, fp4::ST_THREADS, fp4::st_smem_bytes(128, fp4::NV, 1), di->sm_count);
}
static cudaError_t set_kernel_attributes() {
    cudaError_t e;
    if ((e = pair_attributes<fp4::NV>()) != cudaSuccess || (e = pair_attributes<fp4::MX>()) != cudaSuccess) return e;
    if ((e = cudaFuncSetAttribute(kv4::kv4_attn_tc_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kv4::TC_SMEM)) != cudaSuccess) return e;
    cudaFuncAttributes at;                       // its warpgroups share out the registers that it is launched with
    if ((e = cudaFuncGetAttributes(&at, kv4::kv4_attn_tc_kernel)) != cudaSuccess) return e;
    if (at.numRegs < kv4::TC_LAUNCH_REGS) return cudaErrorInvalidConfiguration;
    if ((e = stream_attributes<32, fp4::NV>()) != cudaSuccess || (e = stream_attributes<64, fp4::NV>()) != cudaSuccess) return e;
    if ((e = stream_attributes<128, fp4::NV>()) != cudaSuccess || (e = stream_attributes<32, fp4::MX>()) != cudaSuccess) return e;
    if ((e = stream_attributes<64, fp4::MX>()) != cudaSuccess || (e = stream_attributes<128, fp4::MX>()) != cudaSuccess) return e;
    return cudaSuccess;
}
