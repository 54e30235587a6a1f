// The block-scaled float8 layer for a few rows (a token each of a few sequences), plain and by experts: rows in 16 bit, weights
// in codes, hand-written for gfx950.  gemm_f8_block_kernel.h has the definition.
//
// What bounds it: the weights' way from memory, and the launches.  So the rows are not quantized by a launch of their own (3 us
// of 15 for 16 rows through 4096 -> 16384): every wave fetches its blocks of k of the rows as they are and makes their codes and
// scales in registers, in the shadow of the requests in flight.  A workgroup owns 32 columns of one weight, its four waves split
// the contraction, each with an LDS ring of two stages of 128 k (4 KiB of weights, 4 KiB of rows) that it alone fills and reads;
// two workgroups share a compute unit, so that 64 KiB of weights are on their way to each.  Weights are requested as
// non-temporal: nobody reads them again (4 rows, 4096 -> 16384 from memory: 15.4 -> 13.7 us, 4.9 TB/s).  Not kept: 64 columns a
// workgroup, one on a compute unit (32 experts of 1024 x 4096, 48 rows: 31 -> 36 us, though 16 rows, 4096 -> 16384, without
// non-temporal requests, 16.9 -> 15.6); rows straight into registers, four stages ahead (14.1 -> 16.7 us); eight waves where there
// is a workgroup a compute unit (8 rows, 8192 -> 8192: 13.6 -> 16.5, though 16 rows, 16384 -> 4096: 23.7 -> 22.1).
// v_mfma_scale_f32_16x16x128_f8f6f4 takes a block of k at once: 16 rows, the weight's columns as the first operand, so that a
// lane owns one row and four columns.  Rows past the last one are not fetched.  More than 16 rows of a weight are worked off 16 at
// a time, by `runs` workgroups, the weight read again by each: the dispatch sees to it that they are rare, or the product
// small and the launch most of its time.
#pragma once
#include "gemm_f8_block_kernel.h"
#include "quantize_block.h"

namespace sb {

struct FewCfg {
    static constexpr int ROWS = 16, COLS = 32, WAVES = 4, THREADS = 64 * WAVES, BK = 128, STAGES = 2;
    static constexpr int W_BYTES = COLS * BK, X_BYTES = ROWS * BK * 2, SLOT_BYTES = W_BYTES + X_BYTES;
    static constexpr int REQ = SLOT_BYTES / 1024, WAVE_BYTES = STAGES * SLOT_BYTES, LDS_BYTES = WAVES * WAVE_BYTES;
    static constexpr int PITCH = COLS + 4;  // dwords per row of partial sums
    static_assert(2 * LDS_BYTES <= 160 * 1024 && ROWS * PITCH * 4 <= WAVE_BYTES, "LDS");
};

// GemmBlockArgs with the rows themselves, bf16 [M,cols], in a's place (cols <= K: what lies behind is zero), and no scales of theirs.
struct GemmFewArgs : GemmBlockArgs {
    int cols;
};

template <int OUT, int FMT_A, int FMT_B>
__device__ __forceinline__ void gemm_f8_block_few_body(const GemmFewArgs &p) {
    typedef FewCfg C;
    typedef __attribute__((address_space(3))) void lds_void;
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    constexpr int CODE = FMT_A ? CODE_E5M2 : CODE_E4M3;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row = lane & 15, part = lane >> 4;  // of a fragment: part is a quarter of the block of k
    const int cols = p.N / C::COLS, n0 = (int)blockIdx.x % cols * C::COLS, rest = (int)blockIdx.x / cols;
    const int run = rest % p.runs, expert = rest / p.runs;
    int first, end;
    expert_rows(p, expert, &first, &end);
    if (first + run * C::ROWS >= end) return;
    const int KB = p.K / C::BK;
    const int s0 = (int)((long long)wave * KB / C::WAVES), s1 = (int)((long long)(wave + 1) * KB / C::WAVES), n = s1 - s0;

    // Requests.  Weights: LDS slot (row, q) holds 16-byte chunk q ^ (row & 7) of a 128-byte row; rows: q ^ row of 256 bytes (no
    // bank conflicts in the fragment reads).
    const __amdgpu_buffer_rsrc_t rsrc_w = __builtin_amdgcn_make_buffer_rsrc(
        (void *)(p.b + ((int64_t)expert * p.N + n0) * p.K), 0, (unsigned)(C::COLS * p.K), 0x00020000);
    const unsigned w_off = (unsigned)(lane >> 3) * (unsigned)p.K + (((lane ^ (lane >> 3)) & 7) << 4);
    const int64_t sb_row = ((int64_t)expert * ((p.N + 127) / 128) + n0 / 128) * KB;
    unsigned char *ring = smem + wave * C::WAVE_BYTES;
    const unsigned ring_at = (unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)ring;

    for (int m0 = first + run * C::ROWS; m0 < end; m0 += p.runs * C::ROWS) {
        const int rows = min(end - m0, C::ROWS);
        const __amdgpu_buffer_rsrc_t rsrc_x = __builtin_amdgcn_make_buffer_rsrc(
            (void *)(reinterpret_cast<const unsigned short *>(p.a) + (int64_t)m0 * p.cols), 0, (unsigned)(rows * p.cols * 2), 0x00020000);
        auto issue = [&](int i) {  // stage i of this wave's n
            unsigned char *dst = ring + (i % C::STAGES) * C::SLOT_BYTES;
            const unsigned k0 = (unsigned)(s0 + i) * C::BK;
#pragma unroll
            for (int r = 0; r < C::COLS / 8; ++r)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc_w, (lds_void *)(dst + r * 1024), 16, w_off, (unsigned)(8 * r) * (unsigned)p.K + k0, 0, 2);
#pragma unroll
            for (int r = 0; r < C::ROWS / 4; ++r) {
                const int x_row = 4 * r + (lane >> 4), chunk = (lane & 15) ^ x_row;
                const bool in = k0 + (unsigned)chunk * 8 < (unsigned)p.cols;  // behind a row lies the next one
                const unsigned off = in ? ((unsigned)x_row * (unsigned)p.cols + k0 + (unsigned)chunk * 8) * 2 : 0xfffffff0u;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc_x, (lds_void *)(dst + C::W_BYTES + r * 1024), 16, off, 0, 0, 0);
            }
        };
        v4f acc[2];
#pragma unroll
        for (int c = 0; c < 2; ++c) acc[c] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < C::STAGES; ++i)
            if (i < n) issue(i);
        for (int i = 0; i < n; ++i) {
            const unsigned sw = uniform_byte(p.sb, sb_row + s0 + i);
            wait_stage<C::REQ>(min(C::STAGES - 1, n - 1 - i));  // the requests of a wave retire in order
            __builtin_amdgcn_sched_barrier(0);
            const unsigned at = ring_at + (i % C::STAGES) * C::SLOT_BYTES;
            v4i x[4], w[2][2];
#pragma unroll
            for (int q = 0; q < 4; ++q) x[q] = lds_read_b128<0>(at + C::W_BYTES + row * 256 + (((4 * part + q) ^ row) << 4));
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const unsigned w_at = at + row * C::BK + (((2 * part + h) ^ (row & 7)) << 4);
                w[0][h] = lds_read_b128<0>(w_at);
                w[1][h] = lds_read_b128<16 * C::BK>(w_at);
            }
            wait_lgkmcnt<0>();
#pragma unroll
            for (int q = 0; q < 4; ++q) asm volatile("" : "+v"(x[q]));
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                asm volatile("" : "+v"(w[0][h]));
                asm volatile("" : "+v"(w[1][h]));
            }
            __builtin_amdgcn_sched_barrier(0);
            if (i + C::STAGES < n) issue(i + C::STAGES);  // every read of the slot has returned
            __builtin_amdgcn_sched_barrier(0);
            // The row's block of 128 lies in four lanes.
            unsigned m = 0;
#pragma unroll
            for (int q = 0; q < 4; ++q) m = absmax_of_chunk(m, __builtin_bit_cast(v4u, x[q]));
            m = max(m & 0xffffu, m >> 16);
            const auto m16 = __builtin_amdgcn_permlane16_swap(m, m, false, false);
            m = max(m16[0], m16[1]);
            const auto m32 = __builtin_amdgcn_permlane32_swap(m, m, false, false);
            const unsigned sx = block_scale_byte<CODE>(max(m32[0], m32[1]));
            const float t = inverse_of_scale_byte(sx);
            v8i codes;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const v2u c = quantize_chunk<CODE>(__builtin_bit_cast(v4u, x[q]), t);
                codes[2 * q] = (int)c.x;
                codes[2 * q + 1] = (int)c.y;
            }
#pragma unroll
            for (int c = 0; c < 2; ++c)
                acc[c] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(__builtin_shufflevector(w[c][0], w[c][1], 0, 1, 2, 3, 4, 5, 6, 7), codes,
                                                                          acc[c], FMT_B, FMT_A, 0, (int)sw, 0, (int)sx);
        }

        // Partial sums -> the wave's own LDS: a lane holds its row's columns 16 c + 4 part .. + 3.
        float *sums = reinterpret_cast<float *>(smem);
        constexpr int PART_DWORDS = C::WAVE_BYTES / 4;
#pragma unroll
        for (int c = 0; c < 2; ++c) *reinterpret_cast<v4f *>(sums + wave * PART_DWORDS + row * C::PITCH + 16 * c + 4 * part) = acc[c];
        __syncthreads();
        const int out_row = (int)threadIdx.x >> 4, col = ((int)threadIdx.x & 15) * 2;
        float v[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            v[e] = sums[out_row * C::PITCH + col + e];
#pragma unroll
            for (int w = 1; w < C::WAVES; ++w) v[e] += sums[w * PART_DWORDS + out_row * C::PITCH + col + e];
        }
        if (out_row < rows) {
            const int64_t at = (int64_t)(m0 + out_row) * p.N + n0 + col;
            if (OUT == OUT_BF16) {
                typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
                typedef float v2f __attribute__((ext_vector_type(2)));
                *reinterpret_cast<v2bf *>(static_cast<unsigned short *>(p.out) + at) = __builtin_convertvector((v2f{v[0], v[1]}), v2bf);
            } else {
                typedef float v2f __attribute__((ext_vector_type(2)));
                *reinterpret_cast<v2f *>(static_cast<float *>(p.out) + at) = v2f{v[0], v[1]};
            }
        }
        __syncthreads();  // the next rows' requests write where the sums were read
    }
}

}  // namespace sb
