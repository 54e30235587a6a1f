// Host-side dispatch of the float8 product with a scale for each block of 128, plain and grouped by expert.
#include "gemm_f8_block_few_kernel.h"
#include "gemm_f8_block_wide_kernel.h"

#include <atomic>

namespace sb {
namespace {

typedef DirectCfg<32, 32, 4> D32;
typedef DirectCfg<64, 64, 4> D64;
typedef DirectCfg<64, 64, 2> D64H;

typedef BlockWideCfg<256> W256;
typedef BlockWideCfg<128> W128;

struct Rest64 : D64 {};  // D64 on what the tiled kernel leaves
template <class C, int OUT, int FA, int FB>
struct Body {
    static __device__ __forceinline__ void run(const GemmBlockArgs &p) { gemm_f8_block_direct_body<C, OUT, FA, FB>(p); }
};
template <int OUT, int FA, int FB>
struct Body<Rest64, OUT, FA, FB> {
    static __device__ __forceinline__ void run(const GemmBlockArgs &p) { gemm_f8_block_direct_body<D64, OUT, FA, FB, true>(p); }
};
template <int BN, int OUT, int FA, int FB>
struct Body<BlockWideCfg<BN>, OUT, FA, FB> {
    static __device__ __forceinline__ void run(const GemmBlockArgs &p) { gemm_f8_block_wide_body<OUT, FA, FB, BN>(p); }
};
#define SB_BLOCK_ENTRY(name, CFG, OUT, FA, FB)                                                       \
    __global__ __launch_bounds__(CFG::THREADS) WAVES_##CFG void name(GemmBlockArgs p) {              \
        Body<CFG, OUT, FA, FB>::run(p);                                                              \
    }
#define SB_FEW_ENTRY(name, CFG, OUT, FA, FB) \
    __global__ __launch_bounds__(FewCfg::THREADS) void name(GemmFewArgs p) { gemm_f8_block_few_body<OUT, FA, FB>(p); }
#define WAVES_D32
#define WAVES_D64
#define WAVES_D64H
#define WAVES_Rest64
#define WAVES_W256 __attribute__((amdgpu_waves_per_eu(1, 1)))  // one wave per SIMD: all 512 registers are a lane's
#define WAVES_W128 __attribute__((amdgpu_waves_per_eu(1, 1)))
// name suffix: format of the token-side operand, then of the weight-side operand (4 = E4M3, 5 = E5M2)
#define SB_BLOCK_ENTRIES(ENTRY, name, CFG)       \
    ENTRY(name##_a4b4_bf16, CFG, OUT_BF16, 0, 0) \
    ENTRY(name##_a4b4_f32, CFG, OUT_F32, 0, 0)   \
    ENTRY(name##_a5b4_bf16, CFG, OUT_BF16, 1, 0) \
    ENTRY(name##_a5b4_f32, CFG, OUT_F32, 1, 0)   \
    ENTRY(name##_a4b5_bf16, CFG, OUT_BF16, 0, 1) \
    ENTRY(name##_a4b5_f32, CFG, OUT_F32, 0, 1)   \
    ENTRY(name##_a5b5_bf16, CFG, OUT_BF16, 1, 1) \
    ENTRY(name##_a5b5_f32, CFG, OUT_F32, 1, 1)
SB_BLOCK_ENTRIES(SB_BLOCK_ENTRY, gemm_f8b_d32, D32)
SB_BLOCK_ENTRIES(SB_BLOCK_ENTRY, gemm_f8b_d64, D64)
SB_BLOCK_ENTRIES(SB_BLOCK_ENTRY, gemm_f8b_d64h, D64H)
SB_BLOCK_ENTRIES(SB_BLOCK_ENTRY, gemm_f8b_rest, Rest64)
SB_BLOCK_ENTRIES(SB_BLOCK_ENTRY, gemm_f8b_n, W128)
SB_BLOCK_ENTRIES(SB_BLOCK_ENTRY, gemm_f8b_w, W256)
SB_BLOCK_ENTRIES(SB_FEW_ENTRY, gemm_f8b_few, FewCfg)
#undef SB_FEW_ENTRY
#undef SB_BLOCK_ENTRIES
#undef SB_BLOCK_ENTRY

typedef void (*Kernel)(GemmBlockArgs);
typedef void (*FewKernel)(GemmFewArgs);
#define SB_BLOCK_ROW(name)                                                                                          \
    {name##_a4b4_bf16, name##_a4b4_f32, name##_a5b4_bf16, name##_a5b4_f32, name##_a4b5_bf16, name##_a4b5_f32,       \
     name##_a5b5_bf16, name##_a5b5_f32}
enum { K_D32, K_D64, K_D64H, K_REST, K_N, K_W, KERNELS };
const Kernel kernels[KERNELS][8] = {SB_BLOCK_ROW(gemm_f8b_d32), SB_BLOCK_ROW(gemm_f8b_d64), SB_BLOCK_ROW(gemm_f8b_d64h),
                                    SB_BLOCK_ROW(gemm_f8b_rest), SB_BLOCK_ROW(gemm_f8b_n), SB_BLOCK_ROW(gemm_f8b_w)};
const FewKernel few_kernels[8] = SB_BLOCK_ROW(gemm_f8b_few);
#undef SB_BLOCK_ROW
std::atomic<bool> lds_set[KERNELS][8];  // zero-initialized; a racing second set is harmless

hipError_t launch(int row, int which, int grid, int threads, int lds, const GemmBlockArgs &args, hipStream_t stream) {
    const Kernel kernel = kernels[row][which];
    if (!lds_set[row][which].load(std::memory_order_acquire)) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess) return e;
        lds_set[row][which].store(true, std::memory_order_release);
    }
    kernel<<<grid, threads, lds, stream>>>(args);
    return hipGetLastError();
}

// A direct kernel; runs: workgroups for the row blocks of an expert and a column block.
hipError_t launch_direct(int split, int runs, int which, GemmBlockArgs args, hipStream_t stream) {
    args.runs = runs;
    if (split == DIRECT_32)
        return launch(K_D32, which, args.N / D32::COLS * args.experts * runs, D32::THREADS, BlockDirect<D32>::LDS_BYTES, args, stream);
    const int grid = args.N / D64::COLS * args.experts * runs;
    if (split == DIRECT_64) return launch(K_D64, which, grid, D64::THREADS, BlockDirect<D64>::LDS_BYTES, args, stream);
    return launch(K_D64H, which, grid, D64H::THREADS, BlockDirect<D64H>::LDS_BYTES, args, stream);
}

// A tiled kernel; tile_rows: with experts an upper bound, for which the grid is not shrunk to whole rounds (210 tiles of at most
// 258: 18.5 us on 136 workgroups, 12.5 on 256).
hipError_t launch_tiled(TileKind tile, int64_t tile_rows, int which, const GemmBlockArgs &args, hipStream_t stream) {
    const bool wide = tile == TILES_256;
    const int64_t tiles = tile_rows * ((args.N + (wide ? 255 : 127)) / (wide ? 256 : 128));
    const int ncu = num_compute_units();
    const int grid = persistent_grid(args.offsets != nullptr && tiles > ncu ? ncu : tiles, ncu);
    if (wide) return launch(K_W, which, grid, W256::THREADS, W256::LDS_BYTES, args, stream);
    return launch(K_N, which, grid, W128::THREADS, W128::LDS_BYTES, args, stream);
}

// Rows [first, end) of a product without experts.
GemmBlockArgs rows_of(GemmBlockArgs a, int64_t first, int64_t end, int64_t out_bytes) {
    a.a += first * a.K;
    a.sa += first * 4;
    a.sa_bytes -= (int)(first * 4);
    a.out = static_cast<char *>(a.out) + first * a.N * out_bytes;
    a.M = (int)(end - first);
    return a;
}

}  // namespace

bool few_rows(int64_t M, int64_t N, int64_t K, int64_t experts) { return plan_few_rows(M, N, K, experts); }

hipError_t launch_gemm_f8_block_few(const void *x, int64_t cols, int fmt_x, const uint8_t *bq, int fmt_b, const uint8_t *scales_b,
                                    const int32_t *offsets, int64_t experts, int64_t M, int64_t N, void *out, sb_dtype out_dtype,
                                    hipStream_t stream) {
    static std::atomic<bool> few_lds_set[8];
    GemmFewArgs args;
    args.a = static_cast<const uint8_t *>(x);
    args.sa = nullptr;
    args.b = bq;
    args.sb = scales_b;
    args.offsets = offsets;
    args.out = out;
    args.M = (int)M;
    args.N = (int)N;
    args.K = (int)((cols + 127) / 128 * 128);
    args.sa_rows = args.sa_bytes = 0;
    args.runs = plan_few_runs(M, experts);
    args.cut = 0;
    args.experts = (int)experts;
    args.cols = (int)cols;
    const int which = (fmt_b ? 4 : 0) + (fmt_x ? 2 : 0) + (out_dtype == SB_BF16 ? 0 : 1);
    const FewKernel kernel = few_kernels[which];
    if (!few_lds_set[which].load(std::memory_order_acquire)) {
        const hipError_t e =
            hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, FewCfg::LDS_BYTES);
        if (e != hipSuccess) return e;
        few_lds_set[which].store(true, std::memory_order_release);
    }
    kernel<<<(unsigned int)(N / FewCfg::COLS * experts * args.runs), FewCfg::THREADS, FewCfg::LDS_BYTES, stream>>>(args);
    return hipGetLastError();
}

hipError_t launch_gemm_f8_block(const uint8_t *aq, int fmt_a, const uint8_t *scales_a, const uint8_t *bq, int fmt_b,
                                const uint8_t *scales_b, const int32_t *offsets, int64_t experts, int64_t M, int64_t N, int64_t K,
                                void *out, sb_dtype out_dtype, hipStream_t stream) {
    GemmBlockArgs args;
    args.a = aq;
    args.sa = scales_a;
    args.b = bq;
    args.sb = scales_b;
    args.offsets = offsets;
    args.out = out;
    args.M = (int)M;
    args.N = (int)N;
    args.K = (int)K;
    args.sa_rows = (int)M;
    args.sa_bytes = (int)(uint32_t)((K / 128 + 3) / 4 * M * 4);
    args.experts = (int)experts;
    args.runs = args.cut = 0;
    const int which = (fmt_b ? 4 : 0) + (fmt_a ? 2 : 0) + (out_dtype == SB_BF16 ? 0 : 1);
    const int ncu = num_compute_units(), out_bytes = out_dtype == SB_BF16 ? 2 : 4;
    if (offsets != nullptr) {
        const ExpertProductPlan plan = plan_expert_product(M, N, K, experts, out_bytes, ncu);
        if (plan.split != DIRECT_NONE) return launch_direct(plan.split, plan.runs, which, args, stream);
        args.cut = plan.cut;
        const hipError_t e = launch_tiled(plan.rest, M / 256 + experts, which, args, stream);
        if (e != hipSuccess || plan.cut == 0) return e;
        return launch(K_REST, which, ncu, D64::THREADS, BlockDirect<D64>::LDS_BYTES, args, stream);
    }
    const ProductPlan plan = plan_product(M, N, K, PRODUCT_F8, out_bytes, ncu, TILES_256X128);
    if (plan.first_rows > 0) {
        const hipError_t e = launch_tiled(TILES_256, plan.first_rows / 256, which, rows_of(args, 0, plan.first_rows, out_bytes), stream);
        if (e != hipSuccess) return e;
    }
    if (plan.tile_rows > plan.first_rows) {
        const hipError_t e = launch_tiled(plan.rest, (plan.tile_rows - plan.first_rows + 255) / 256, which,
                                          rows_of(args, plan.first_rows, plan.tile_rows, out_bytes), stream);
        if (e != hipSuccess) return e;
    }
    if (plan.split == DIRECT_NONE) return hipSuccess;
    const int64_t rows = plan.split == DIRECT_32 ? 32 : 64;
    return launch_direct(plan.split, (int)((M - plan.tile_rows + rows - 1) / rows), which, rows_of(args, plan.tile_rows, M, out_bytes),
                         stream);
}

}  // namespace sb
