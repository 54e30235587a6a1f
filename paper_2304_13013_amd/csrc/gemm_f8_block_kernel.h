// The float8 product with a scale for each block of 128, and its form grouped by expert: arguments, and the kernel for few
// output rows or elements, hand-written for gfx950.
//
//   out[i,j] = sum_kb 2^(sa[i,kb] - 127) 2^(sb[j / 128,kb] - 127) sum_{k in block kb} a[i,k] b[j,k]
//
// a [M,K] and b [N,K] (or a b and its scales per expert) are float8 codes with k contiguous, K whole blocks of 128.  The scale
// bytes are exponents as v_mfma_scale_f32_32x32x64_f8f6f4 takes them: it scales both operands on their way in, so that the
// blocks of a row add up in the accumulators and no scaling is left for the epilogue.  With arbitrary scales every block's sum
// would have to be taken out of the accumulators and added by the vector unit, half as many cycles again as the matrix
// instructions take.
//
// By experts: rows offsets[e] .. offsets[e+1] - 1 of a go with the e-th b.  Offsets are read on the GPU and clamped to
// 0 .. M, so that no value of theirs leads out of bounds; rows of no expert are not written.
//
// This kernel: a workgroup owns 64 or 32 columns of one b and works through blocks of as many rows, its waves split the
// contraction, each with an LDS ring of its own, and the partial sums meet in LDS (as in gemm_i8_direct_kernel.h, whose
// operand path it shares: swizzled requests of 128-byte row segments straight into LDS).  Few rows are bound by the weights'
// way from memory: 256 rows, 8 experts of 4096 x 4096 25.5 us, 5.3 TB/s of weights.
#pragma once
#include "gemm_i8_direct_kernel.h"

namespace sb {

struct GemmBlockArgs {
    const uint8_t *a, *sa;  // [M,K]; [ceil(K / 512), sa_rows, 4] bytes: a row's blocks of 128, four to a dword
    const uint8_t *b, *sb;  // [experts,N,K]; [experts, ceil(N / 128), K / 128]
    const int *offsets;     // [experts + 1], or null: one b for all rows
    void *out;              // [M,N]
    int M, N, K, sa_rows, sa_bytes, experts;  // sa_bytes: from sa to the end of the scales, below 2^32
    int runs;               // direct kernel: workgroups that share the row blocks of an expert and a column block
    int cut;                // experts, 256x256 tiles: their workgroups, if a last round of few tiles is the direct kernel's; else 0
};

// Rows of an expert: [first, end).
__device__ __forceinline__ void expert_rows(const GemmBlockArgs &p, int e, int *first, int *end) {
    *first = 0;
    *end = p.M;
    if (p.offsets != nullptr) {
        *first = min(max(uniform_load(p.offsets + e), 0), p.M);
        *end = min(max(uniform_load(p.offsets + e + 1), *first), p.M);
    }
}

// The tile rows of all experts, numbered through: `before` this lane's share of the experts, `total` of all.
struct ExpertTiles {
    static constexpr int ROWS = 256;
    int share, before, total;
};
__device__ __forceinline__ ExpertTiles expert_tiles(const GemmBlockArgs &p) {
    ExpertTiles t{(p.experts + 63) / 64, 0, 0};
    const int lane = threadIdx.x & 63;
    int mine = 0;
    for (int i = 0; i < t.share; ++i) {
        const int e = lane * t.share + i;
        if (e < p.experts) {
            const int first = min(max(p.offsets[e], 0), p.M), end = min(max(p.offsets[e + 1], first), p.M);
            mine += (end - first + ExpertTiles::ROWS - 1) / ExpertTiles::ROWS;
        }
    }
    int sum = mine;  // of the lanes up to this one
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int other = __shfl_up(sum, d, 64);
        if (lane >= d) sum += other;
    }
    t.before = sum - mine;
    t.total = __builtin_amdgcn_readlane(sum, 63);
    return t;
}
// Tile row tm < total: its expert, first row and the end of the expert's rows.
__device__ __forceinline__ void find_tile(const GemmBlockArgs &p, const ExpertTiles &t, int tm, int *expert, int *row, int *end) {
    // The last lane that has no more than tm tile rows before its share has the tile's expert in it.
    const int owner = __builtin_popcountll(__builtin_amdgcn_ballot_w64(t.before <= tm)) - 1;
    int at = tm - __builtin_amdgcn_readlane(t.before, owner);
    for (int e = owner * t.share;; ++e) {
        int first;
        expert_rows(p, e, &first, end);
        const int tiles = (*end - first + ExpertTiles::ROWS - 1) / ExpertTiles::ROWS;
        *expert = e;
        *row = first + at * ExpertTiles::ROWS;
        if (at < tiles || e + 1 >= p.experts) return;
        at -= tiles;
    }
}
// Tile rows that the tiled kernel works on, of `total`; the direct kernel has the others: those behind the last whole round, if
// they are at most an eighth of a round, two rounds of its blocks (plan_expert_product; both kernels decide alike).
__device__ __forceinline__ int tiled_rows(const GemmBlockArgs &p, int total, int tiles_n) {
    if (p.cut == 0) return total;
    const int tiles = total * tiles_n, whole = tiles / p.cut * p.cut;
    return whole == 0 || tiles - whole > p.cut / 8 ? total : whole / tiles_n;
}

// Byte i of an array that starts at a multiple of 4, as part of its dword.
__device__ __forceinline__ unsigned uniform_byte(const uint8_t *bytes, int64_t i) {
    const unsigned v = uniform_load(reinterpret_cast<const unsigned *>(bytes + (i & ~(int64_t)3)));
    return v >> ((unsigned)(i & 3) * 8) & 0xffu;
}

template <class C>
struct BlockDirect {  // C: DirectCfg
    static constexpr int SLOT_BYTES = C::STAGE_BYTES + 256;  // of a ring: a stage's codes, then a dword of scale bytes per row
    static constexpr int WAVE_BYTES = C::STAGES * SLOT_BYTES, LDS_BYTES = C::WAVES * WAVE_BYTES, REQ = C::REQ + 1;
    static_assert(LDS_BYTES <= 160 * 1024 && C::ROWS <= 64 && C::ROWS * C::PITCH * 4 <= WAVE_BYTES, "LDS");
};

// REST: the tile rows that tiled_rows leaves, an item for each block of rows and columns.
template <class C, int OUT, int FMT_A, int FMT_B, bool REST = false>
__device__ __forceinline__ void gemm_f8_block_direct_body(const GemmBlockArgs &p) {
    typedef BlockDirect<C> D;
    typedef __attribute__((address_space(3))) void lds_void;
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int frow = lane & 31, fhalf = lane >> 5;
    // Workgroups of one b follow each other, its column blocks fastest: few experts' weights are in flight at a time.
    const int cols = p.N / C::COLS;
    int n0 = 0, end = 0;
    const int KB = p.K / C::BK;
    const int s0 = (int)((long long)wave * KB / C::WAVES), s1 = (int)((long long)(wave + 1) * KB / C::WAVES), n = s1 - s0;

    const __amdgpu_buffer_rsrc_t rsrc_a =
        __builtin_amdgcn_make_buffer_rsrc((void *)p.a, 0, (unsigned)((size_t)p.M * (size_t)p.K), 0x00020000);
    const __amdgpu_buffer_rsrc_t rsrc_sa =
        __builtin_amdgcn_make_buffer_rsrc((void *)p.sa, 0, (unsigned)p.sa_bytes, 0x00020000);
    __amdgpu_buffer_rsrc_t rsrc_b;
    int64_t sb_row = 0;
    auto set_weight = [&](int expert, int block) {
        n0 = block * C::COLS;
        rsrc_b = __builtin_amdgcn_make_buffer_rsrc((void *)(p.b + (int64_t)expert * p.N * p.K), 0, (unsigned)((size_t)p.N * (size_t)p.K),
                                                   0x00020000);
        sb_row = ((int64_t)expert * ((p.N + 127) / 128) + n0 / 128) * KB;
    };
    unsigned voff[2];
#pragma unroll
    for (int v = 0; v < 2; ++v) {
        const int row = 8 * v + (lane >> 3), chunk = (lane & 7) ^ ((row >> 1) & 7);
        voff[v] = (unsigned)(lane >> 3) * (unsigned)p.K + (unsigned)chunk * 16;
    }
    unsigned char *ring = smem + wave * D::WAVE_BYTES;
    const unsigned ring_at = (unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)ring;
    const unsigned req_step = 8u * (unsigned)p.K;
    const unsigned voff_scale = lane < C::ROWS ? (unsigned)lane * 4 : 0xfffffff0u;

    int frag_off[4];
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) frag_off[kk] = frow * C::BK + (((kk * 2 + fhalf) ^ ((frow >> 1) & 7)) << 4);

    auto row_block = [&](int m0) __attribute__((always_inline)) {
        auto issue = [&](int i) {  // stage i of this wave's n: rows past M read as zero; rows of another expert are not stored
            unsigned char *dst = ring + (i % C::STAGES) * D::SLOT_BYTES;
            const unsigned k0 = (unsigned)(s0 + i) * C::BK;
#pragma unroll
            for (int r = 0; r < C::ROWS / 8; ++r)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc_a, (lds_void *)(dst + r * 1024), 16, voff[r & 1],
                                                         (unsigned)m0 * (unsigned)p.K + (unsigned)r * req_step + k0, 0, 0);
#pragma unroll
            for (int r = 0; r < C::COLS / 8; ++r)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc_b, (lds_void *)(dst + C::ROWS * C::BK + r * 1024), 16, voff[r & 1],
                                                         (unsigned)n0 * (unsigned)p.K + (unsigned)r * req_step + k0, 0, 0);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc_sa, (lds_void *)(dst + C::STAGE_BYTES), 4, voff_scale,
                                                     ((unsigned)m0 + ((unsigned)(s0 + i) >> 2) * (unsigned)p.sa_rows) * 4, 0, 0);
        };
        v16f acc[C::RB][C::CB];
#pragma unroll
        for (int r = 0; r < C::RB; ++r)
#pragma unroll
            for (int c = 0; c < C::CB; ++c)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[r][c][e] = 0.0f;

        v8i xf[2][C::RB], wf[2][C::CB];
        unsigned sx[C::RB];
        auto read_group = [&](int buf, int slot, int g) {
            const unsigned at = ring_at + slot * D::SLOT_BYTES + frag_off[g * 2], at2 = ring_at + slot * D::SLOT_BYTES + frag_off[g * 2 + 1];
            auto read = [&](auto off) -> v8i {
                constexpr int OFF = decltype(off)::value;
                const v4i lo = lds_read_b128<OFF>(at);
                const v4i hi = lds_read_b128<OFF>(at2);
                return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            };
            xf[buf][0] = read(std::integral_constant<int, 0>());
            if constexpr (C::RB == 2) xf[buf][1] = read(std::integral_constant<int, 32 * C::BK>());
            wf[buf][0] = read(std::integral_constant<int, C::ROWS * C::BK>());
            if constexpr (C::CB == 2) wf[buf][1] = read(std::integral_constant<int, (C::ROWS + 32) * C::BK>());
        };
#pragma unroll
        for (int i = 0; i < C::STAGES; ++i)
            if (i < n) issue(i);
        for (int i = 0; i < n; ++i) {
            const int slot = i % C::STAGES;
            const unsigned sw = uniform_byte(p.sb, sb_row + s0 + i), shift = ((unsigned)(s0 + i) & 3) * 8;
            wait_stage<D::REQ>(min(C::STAGES - 1, n - 1 - i));  // the requests of a wave retire in order
            __builtin_amdgcn_sched_barrier(0);
            const unsigned scale_at = ring_at + slot * D::SLOT_BYTES + C::STAGE_BYTES + frow * 4;
#pragma unroll
            for (int r = 0; r < C::RB; ++r) asm volatile("ds_read_b32 %0, %1 offset:%2" : "=v"(sx[r]) : "v"(scale_at), "n"(r * 128));
            read_group(0, slot, 0);
            read_group(1, slot, 1);
            wait_lgkmcnt<0>();
#pragma unroll
            for (int r = 0; r < C::RB; ++r) {
                asm volatile("" : "+v"(sx[r]));
                asm volatile("" : "+v"(xf[0][r]));
                asm volatile("" : "+v"(xf[1][r]));
            }
#pragma unroll
            for (int c = 0; c < C::CB; ++c) {
                asm volatile("" : "+v"(wf[0][c]));
                asm volatile("" : "+v"(wf[1][c]));
            }
#pragma unroll
            for (int r = 0; r < C::RB; ++r) sx[r] = sx[r] >> shift;
#pragma unroll
            for (int g = 0; g < 2; ++g)
#pragma unroll
                for (int r = 0; r < C::RB; ++r)
#pragma unroll
                    for (int c = 0; c < C::CB; ++c)
                        acc[r][c] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wf[g][c], xf[g][r], acc[r][c], FMT_B, FMT_A, 0,
                                                                                    (int)sw, 0, (int)sx[r]);
            __builtin_amdgcn_sched_barrier(0);
            if (i + C::STAGES < n) issue(i + C::STAGES);  // every read of the slot has returned
            __builtin_amdgcn_sched_barrier(0);
        }

        // Partial sums -> the wave's own LDS, row-major: a lane holds row frow of a 32-row block and, per quad q, columns
        // 8q + 4*fhalf .. +3.
        constexpr int PART_DWORDS = D::WAVE_BYTES / 4;
        float *part = reinterpret_cast<float *>(smem) + wave * PART_DWORDS;
#pragma unroll
        for (int r = 0; r < C::RB; ++r)
#pragma unroll
            for (int c = 0; c < C::CB; ++c)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    v4f v;
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = acc[r][c][4 * q + e];
                    *reinterpret_cast<v4f *>(part + (32 * r + frow) * C::PITCH + 32 * c + 8 * q + 4 * fhalf) = v;
                }
        __syncthreads();
        constexpr int V = 4 * C::QUADS, ROW_LANES = C::THREADS / (C::COLS / V), ITEMS = C::ROWS / ROW_LANES;
        const int col = ((int)threadIdx.x % (C::COLS / V)) * V, row0 = (int)threadIdx.x / (C::COLS / V);
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int row = row0 + i * ROW_LANES, gr = m0 + row;
            const float *src = reinterpret_cast<const float *>(smem) + row * C::PITCH + col;
            v4f sum[C::QUADS];
#pragma unroll
            for (int h = 0; h < C::QUADS; ++h) {
                sum[h] = *reinterpret_cast<const v4f *>(src + 4 * h);
#pragma unroll
                for (int w = 1; w < C::WAVES; ++w) sum[h] += *reinterpret_cast<const v4f *>(src + w * PART_DWORDS + 4 * h);
            }
            if (gr >= end) continue;
            const int64_t at = (int64_t)gr * p.N + n0 + col;
            if (OUT == OUT_BF16) {
                unsigned short *out = static_cast<unsigned short *>(p.out) + at;
#pragma unroll
                for (int h = 0; h < C::QUADS; ++h)
                    *reinterpret_cast<v2u *>(out + 4 * h) = __builtin_bit_cast(v2u, __builtin_convertvector(sum[h], v4bf));
            } else {
#pragma unroll
                for (int h = 0; h < C::QUADS; ++h) *reinterpret_cast<v4f *>(static_cast<float *>(p.out) + at + 4 * h) = sum[h];
            }
        }
        __syncthreads();  // the next row block's requests write where the sums were read
    };
    if constexpr (REST) {
        constexpr int BLOCKS = ExpertTiles::ROWS / C::ROWS;  // of a tile row
        const ExpertTiles t = expert_tiles(p);
        const int done = tiled_rows(p, t.total, (p.N + 255) / 256), items = (t.total - done) * BLOCKS * cols;
        for (int item = (int)blockIdx.x; item < items; item += (int)gridDim.x) {
            const int q = item / cols;
            int expert, row;
            find_tile(p, t, done + q / BLOCKS, &expert, &row, &end);
            row += q % BLOCKS * C::ROWS;
            if (row >= end) continue;
            set_weight(expert, item % cols);
            row_block(row);
        }
    } else {
        const int rest = (int)blockIdx.x / cols, run = rest % p.runs, expert = rest / p.runs;
        int first;
        expert_rows(p, expert, &first, &end);
        set_weight(expert, (int)blockIdx.x % cols);
        for (int m0 = first + run * C::ROWS; m0 < end; m0 += p.runs * C::ROWS) row_block(m0);
    }
}

}  // namespace sb
