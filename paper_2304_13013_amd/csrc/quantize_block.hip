// Quantizers of the float8 layer with a scale for each block of 128, for gfx950.
//
//   e = the least integer >= -127 with absmax(block) <= MAX * 2^e   (MAX 448 for E4M3, 57344 for E5M2)
//   code = float8(x * 2^-e), round to nearest even;  scale byte = e + 127: the block stands for code * 2^e
//
// Token-side matrices have blocks of 1 x 128, weights of 128 x 128, whose transpose then has the same codes and scales.  With
// powers of two nothing but the conversion rounds, and the matrix instruction takes the bytes as they are.  A block that is all
// zero has scale byte 0 and zero codes.  Codes have rows of whole blocks: what lies behind the last column is zero.
//
// What bounds it: memory, 2 bytes read and 1 written per element (weights with their transpose 2 and 2).  A wave owns 512
// columns of a row at a time (1 KiB of input, one dword of scale bytes), four rows in flight; a weight's block is one workgroup's
// tile, transposed through LDS.  Both jobs of a forward pass are one launch.  32896 x 5120 rows: 84 us, 6.0 TB/s; 32896 x 1280 rows
// with a weight of 5120 x 1280 in both layouts: 26.5 us, 5.8 TB/s.
#include "quantize_block.h"

namespace sb {
namespace {

// Largest value of 16 neighbouring lanes, in each of them.
__device__ __forceinline__ unsigned int max_of_16_lanes(unsigned int v) {
    v = max(v, (unsigned int)__builtin_amdgcn_update_dpp(0, (int)v, 0x128, 0xf, 0xf, false));  // row_ror:8
    v = max(v, (unsigned int)__builtin_amdgcn_update_dpp(0, (int)v, 0x124, 0xf, 0xf, false));
    v = max(v, (unsigned int)__builtin_amdgcn_update_dpp(0, (int)v, 0x122, 0xf, 0xf, false));
    return max(v, (unsigned int)__builtin_amdgcn_update_dpp(0, (int)v, 0x121, 0xf, 0xf, false));
}

constexpr int kRowsPerWave = 4, kRowsPerBlock = 4 * kRowsPerWave;

struct BlockRowsJob {
    const v4u *x;
    int rows, chunks;       // 16-byte chunks of a row
    uint8_t *codes;         // [rows, 128 * blocks]
    unsigned int *scales;   // [dwords, rows]
    int blocks, dwords;     // blocks of 128 columns in a row; dwords of scale bytes, one for each 512 columns
    int row_groups, first, count;  // workgroups [first, first + count) of the launch: row_groups for each 512 columns
};
struct BlockWeightJob {
    const v4u *w;           // [experts, m, n]
    int m, n;
    uint8_t *codes, *codes_t;    // [experts, m, 128 * blocks_n], [experts, n, 128 * blocks_m] or null
    uint8_t *scales, *scales_t;  // [experts, blocks_m, blocks_n], [experts, blocks_n, blocks_m]
    int blocks_m, blocks_n;
};

template <int CODE>
__device__ __forceinline__ void quantize_rows(const BlockRowsJob &job, int group) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int part = group / job.row_groups, row0 = (group % job.row_groups) * kRowsPerBlock + wave * kRowsPerWave;
    const int c = part * 64 + lane;  // chunk of the row
    v4u v[kRowsPerWave];
#pragma unroll
    for (int i = 0; i < kRowsPerWave; ++i) {
        v[i] = v4u{0u, 0u, 0u, 0u};
        if (row0 + i < job.rows && c < job.chunks) v[i] = __builtin_nontemporal_load(job.x + (int64_t)(row0 + i) * job.chunks + c);
    }
#pragma unroll
    for (int i = 0; i < kRowsPerWave; ++i) {
        const unsigned int m = absmax_of_chunk(0, v[i]), s = block_scale_byte<CODE>(max_of_16_lanes(max(m & 0xffffu, m >> 16)));
        const v2u codes = quantize_chunk<CODE>(v[i], inverse_of_scale_byte(s));
        if (row0 + i >= job.rows) break;
        if (c < job.blocks * 16) reinterpret_cast<v2u *>(job.codes)[(int64_t)(row0 + i) * job.blocks * 16 + c] = codes;
        const unsigned int bytes = __builtin_amdgcn_readlane(s, 0) | __builtin_amdgcn_readlane(s, 16) << 8 |
                                   __builtin_amdgcn_readlane(s, 32) << 16 | __builtin_amdgcn_readlane(s, 48) << 24;
        if (lane == 0) job.scales[(int64_t)part * job.rows + row0 + i] = bytes;
    }
}

template <int CODE>
__device__ __forceinline__ void quantize_weight_block(const BlockWeightJob &job, int block, unsigned int *tile, unsigned int *wave_max) {
    const int per_expert = job.blocks_m * job.blocks_n;
    const int expert = block / per_expert, rb = block % per_expert / job.blocks_n, cb = block % job.blocks_n;
    const int r0 = rb * kTile, c0 = cb * kTile, pitch = job.blocks_n * kTile, pitch_t = job.blocks_m * kTile;
    const v4u *w = job.w + (int64_t)expert * job.m * (job.n >> 3);
    v4u v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int id = threadIdx.x + 256 * i, r = r0 + (id >> 4), c = c0 + ((id & 15) << 3);
        v[i] = r < job.m && c < job.n ? w[(int64_t)r * (job.n >> 3) + (c >> 3)] : v4u{0u, 0u, 0u, 0u};
    }
    unsigned int m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = absmax_of_chunk(m, v[i]);
    m = wave_max_u32(max(m & 0xffffu, m >> 16));
    if ((threadIdx.x & 63) == 0) wave_max[threadIdx.x >> 6] = m;
    __syncthreads();
    const unsigned int s = block_scale_byte<CODE>(max(max(wave_max[0], wave_max[1]), max(wave_max[2], wave_max[3])));
    const float t = inverse_of_scale_byte(s);
    if (threadIdx.x == 0) {
        job.scales[((int64_t)expert * job.blocks_m + rb) * job.blocks_n + cb] = (uint8_t)s;
        if (job.codes_t != nullptr) job.scales_t[((int64_t)expert * job.blocks_n + cb) * job.blocks_m + rb] = (uint8_t)s;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int id = threadIdx.x + 256 * i, lr = id >> 4, lc = (id & 15) << 3;
        const v2u codes = quantize_chunk<CODE>(v[i], t);
        if (r0 + lr < job.m) *reinterpret_cast<v2u *>(job.codes + ((int64_t)expert * job.m + r0 + lr) * pitch + c0 + lc) = codes;
        tile[tile_dword(lr, lc >> 2)] = codes.x;
        tile[tile_dword(lr, (lc >> 2) + 1)] = codes.y;
    }
    if (job.codes_t == nullptr) return;  // uniform across the grid
    __syncthreads();
    store_tile_transposed(tile, reinterpret_cast<int8_t *>(job.codes_t) + (int64_t)expert * job.n * pitch_t, pitch_t, job.n, r0, c0);
}

// The weight's blocks first: they take longer than a group of rows.
template <int CODE_X, int CODE_W>
__global__ __launch_bounds__(256) void quantize_block_kernel(BlockRowsJob rows, BlockWeightJob weight) {
    __shared__ unsigned int wave_max[4];
    __shared__ unsigned int tile[kTileDwords];
    if ((int)blockIdx.x >= rows.first) quantize_rows<CODE_X>(rows, (int)blockIdx.x - rows.first);
    else quantize_weight_block<CODE_W>(weight, (int)blockIdx.x, tile, wave_max);
}
template <int CODE>
__global__ __launch_bounds__(256) void quantize_rows_block_kernel(BlockRowsJob rows) {
    quantize_rows<CODE>(rows, (int)blockIdx.x);
}

BlockRowsJob rows_job(const void *x, int64_t rows, int64_t cols, uint8_t *codes, uint8_t *scales, int first) {
    BlockRowsJob job;
    job.x = static_cast<const v4u *>(x);
    job.rows = (int)rows;
    job.chunks = (int)(cols / 8);
    job.codes = codes;
    job.scales = reinterpret_cast<unsigned int *>(scales);
    job.blocks = (int)((cols + 127) / 128);
    job.dwords = (job.blocks + 3) / 4;
    job.row_groups = (int)((rows + kRowsPerBlock - 1) / kRowsPerBlock);
    job.first = first;
    job.count = job.row_groups * job.dwords;
    return job;
}

}  // namespace

hipError_t launch_quantize_rows_block(const void *x, int64_t rows, int64_t cols, int fmt, uint8_t *codes, uint8_t *scales,
                                      hipStream_t stream) {
    const BlockRowsJob job = rows_job(x, rows, cols, codes, scales, 0);
    if (fmt) quantize_rows_block_kernel<CODE_E5M2><<<job.count, 256, 0, stream>>>(job);
    else quantize_rows_block_kernel<CODE_E4M3><<<job.count, 256, 0, stream>>>(job);
    return hipGetLastError();
}

hipError_t launch_quantize_block(const void *x, int64_t rows, int fmt_x, uint8_t *xq, uint8_t *scales_x, const void *w,
                                 int64_t experts, int64_t m, int64_t n, int fmt_w, uint8_t *wq, uint8_t *scales_w, uint8_t *wq_t,
                                 uint8_t *scales_wt, hipStream_t stream) {
    BlockWeightJob weight;
    weight.w = static_cast<const v4u *>(w);
    weight.m = (int)m;
    weight.n = (int)n;
    weight.codes = wq;
    weight.codes_t = wq_t;
    weight.scales = scales_w;
    weight.scales_t = scales_wt;
    weight.blocks_m = (int)((m + 127) / 128);
    weight.blocks_n = (int)((n + 127) / 128);
    const int blocks = (int)(experts * weight.blocks_m * weight.blocks_n);
    const BlockRowsJob job = rows_job(x, rows, n, xq, scales_x, blocks);
    const int grid = blocks + job.count;
    if (fmt_x && fmt_w) quantize_block_kernel<CODE_E5M2, CODE_E5M2><<<grid, 256, 0, stream>>>(job, weight);
    else if (fmt_x) quantize_block_kernel<CODE_E5M2, CODE_E4M3><<<grid, 256, 0, stream>>>(job, weight);
    else if (fmt_w) quantize_block_kernel<CODE_E4M3, CODE_E5M2><<<grid, 256, 0, stream>>>(job, weight);
    else quantize_block_kernel<CODE_E4M3, CODE_E4M3><<<grid, 256, 0, stream>>>(job, weight);
    return hipGetLastError();
}

}  // namespace sb
