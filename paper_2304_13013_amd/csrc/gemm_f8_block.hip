// Host-side dispatch of the float8 product with a scale for each block of 128, plain and grouped by expert.
#include "gemm_f8_block_wide_kernel.h"

#include <atomic>

namespace sb {
namespace {

typedef DirectCfg<32, 32, 4> D32;
typedef DirectCfg<64, 64, 4> D64;

typedef BlockWideCfg<256> W256;
typedef BlockWideCfg<128> W128;

template <class C, int OUT, int FA, int FB>
struct Body {
    static __device__ __forceinline__ void run(const GemmBlockArgs &p) { gemm_f8_block_direct_body<C, OUT, FA, FB>(p); }
};
template <int BN, int OUT, int FA, int FB>
struct Body<BlockWideCfg<BN>, OUT, FA, FB> {
    static __device__ __forceinline__ void run(const GemmBlockArgs &p) { gemm_f8_block_wide_body<OUT, FA, FB, BN>(p); }
};
#define SB_BLOCK_ENTRY(name, CFG, OUT, FA, FB)                                                       \
    __global__ __launch_bounds__(CFG::THREADS) WAVES_##CFG void name(GemmBlockArgs p) {              \
        Body<CFG, OUT, FA, FB>::run(p);                                                              \
    }
#define WAVES_D32
#define WAVES_D64
#define WAVES_W256 __attribute__((amdgpu_waves_per_eu(1, 1)))  // one wave per SIMD: all 512 registers are a lane's
#define WAVES_W128 __attribute__((amdgpu_waves_per_eu(1, 1)))
// name suffix: format of the token-side operand, then of the weight-side operand (4 = E4M3, 5 = E5M2)
#define SB_BLOCK_ENTRIES(name, CFG)                        \
    SB_BLOCK_ENTRY(name##_a4b4_bf16, CFG, OUT_BF16, 0, 0)  \
    SB_BLOCK_ENTRY(name##_a4b4_f32, CFG, OUT_F32, 0, 0)    \
    SB_BLOCK_ENTRY(name##_a5b4_bf16, CFG, OUT_BF16, 1, 0)  \
    SB_BLOCK_ENTRY(name##_a5b4_f32, CFG, OUT_F32, 1, 0)    \
    SB_BLOCK_ENTRY(name##_a4b5_bf16, CFG, OUT_BF16, 0, 1)  \
    SB_BLOCK_ENTRY(name##_a4b5_f32, CFG, OUT_F32, 0, 1)    \
    SB_BLOCK_ENTRY(name##_a5b5_bf16, CFG, OUT_BF16, 1, 1)  \
    SB_BLOCK_ENTRY(name##_a5b5_f32, CFG, OUT_F32, 1, 1)
SB_BLOCK_ENTRIES(gemm_f8b_d32, D32)
SB_BLOCK_ENTRIES(gemm_f8b_d64, D64)
SB_BLOCK_ENTRIES(gemm_f8b_n, W128)
SB_BLOCK_ENTRIES(gemm_f8b_w, W256)
#undef SB_BLOCK_ENTRIES
#undef SB_BLOCK_ENTRY

typedef void (*Kernel)(GemmBlockArgs);
#define SB_BLOCK_ROW(name)                                                                                          \
    {name##_a4b4_bf16, name##_a4b4_f32, name##_a5b4_bf16, name##_a5b4_f32, name##_a4b5_bf16, name##_a4b5_f32,       \
     name##_a5b5_bf16, name##_a5b5_f32}
const Kernel kernels[4][8] = {SB_BLOCK_ROW(gemm_f8b_d32), SB_BLOCK_ROW(gemm_f8b_d64), SB_BLOCK_ROW(gemm_f8b_n), SB_BLOCK_ROW(gemm_f8b_w)};
#undef SB_BLOCK_ROW
std::atomic<bool> lds_set[4][8];  // zero-initialized; a racing second set is harmless

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

}  // namespace

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
    args.sa_dwords = (int)((K / 128 + 3) / 4);
    args.experts = (int)experts;
    const int which = (fmt_b ? 4 : 0) + (fmt_a ? 2 : 0) + (out_dtype == SB_BF16 ? 0 : 1);
    const int64_t per_expert = (M + experts - 1) / experts;  // rows, in the mean
    if (per_expert <= 32) {
        args.runs = 1;
        return launch(0, which, (int)(N / D32::COLS * experts), D32::THREADS, BlockDirect<D32>::LDS_BYTES, args, stream);
    }
    const int64_t tile_rows = offsets == nullptr ? (M + 255) / 256 : M / 256 + experts;  // at most
    if (tile_rows * ((N + 255) / 256) * 2 > num_compute_units()) {
        args.runs = 0;
        const int wide = tile_rows * ((N + 255) / 256) >= num_compute_units() ? 1 : 0;
        const int grid = persistent_grid(tile_rows * ((N + 255) / 256) * (wide ? 1 : 2), num_compute_units());
        return launch(2 + wide, which, grid, 256, wide ? W256::LDS_BYTES : W128::LDS_BYTES, args, stream);
    }
    const int64_t runs = (per_expert + 63) / 64;
    args.runs = (int)(runs < 64 ? runs : 64);
    return launch(1, which, (int)(N / D64::COLS * experts * args.runs), D64::THREADS, BlockDirect<D64>::LDS_BYTES, args, stream);
}

}  // namespace sb
