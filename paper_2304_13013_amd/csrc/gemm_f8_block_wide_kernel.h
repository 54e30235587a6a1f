// The float8 product with a scale for each block of 128, plain and by experts (gemm_f8_block_kernel.h says what it computes),
// on 256x256 or 256x128 tiles: four waves of 128x128 or 128x64, one per SIMD.
//
// The pipeline is that of gemm_i8_wide_kernel.h, which explains it: stages of 128 bytes of k, one barrier per stage, requests
// and fragment reads spread between the matrix instructions, accumulators named in the text, a tile's epilogue under the
// first half stage of the next one.  What differs:
//   * A stage is one block of k, so a fragment has one scale per stage.  Token side: the four scale bytes of four blocks are
//     one dword per row, requested into LDS with every stage (one request of 64 rows a wave), read before the next stage's
//     first fragments and shifted to the stage's byte where the matrix instructions have done with the register.  Weight
//     side: a wave's 128 (or 64) columns lie in one block of the weight, whose byte comes through the scalar cache a stage
//     ahead.  The matrix instruction takes both as they are, at the rate of the plain one (3.86 PFLOP/s from registers on
//     codes of normal data, 3.89 without scales).
//   * Tiles belong to experts.  The tile rows of all experts are numbered through; a lane keeps the number of tile rows before
//     its share of the experts (offsets are read once, when the kernel starts), so that the expert of a tile row is a ballot.
//     A tile's rows start where its expert's do: the last one of an expert is cut short by the output's bounds check.
//   * The epilogue has nothing to scale.
// 16384 x 16384, K = 4096: 757-790 us, 2.8-2.9 PFLOP/s; 32896 x 1280, K = 5120: 183-190 us; 4 % above the product with one state
// per row, for the scales' requests and reads.  What bounds it is what bounds that one: the clock under the instructions' power,
// the operands' way into LDS, the tile boundary at short K.
#pragma once
#include "gemm_f8_block_kernel.h"
#include "gemm_i8_wide_kernel.h"

namespace sb {

template <int BN_>
struct BlockWideCfg {
    static constexpr int BM = 256, BN = BN_, BK = 128, THREADS = 256;
    static constexpr int STAGES = BN == 256 ? 2 : 3;
    static constexpr int WTM = 128, WTN = BN / 2;        // wave tile
    static constexpr int A_BYTES = BM * BK, CODE_BYTES = (BM + BN) * BK, STAGE_BYTES = CODE_BYTES + BM * 4;
    static constexpr int REQ_A = BM / 32, REQ_B = BN / 32, REQ = REQ_A + REQ_B;  // 1 KiB requests per wave and stage
    static constexpr int LPW = REQ + 1;                  // and one of scale bytes
    static constexpr int NBM = WTM / 32, NBN = WTN / 32, SLOTS = NBM * NBN;  // matrix instructions per half stage
    static constexpr int NREADS = (NBM + NBN) * 2;       // 16-byte fragment reads per wave and half stage
    static constexpr int REQ_2ND = BN == 256 ? REQ : REQ / 2;  // code requests of a stage in the second half stage, the others in the first
    static constexpr int PATCH_COLS = WTN / 2, PATCH_PITCH = PATCH_COLS * 2 + 16;
    static constexpr int PATCH_BYTES = 32 * PATCH_PITCH, PATCH_SLOTS = PATCH_COLS / 32;
    static constexpr int PPR = PATCH_COLS / 8, PATCH_READS = 32 * PPR / 64;
    static constexpr int LDS_BYTES = STAGES * STAGE_BYTES + 4 * PATCH_BYTES;
    static_assert(LDS_BYTES <= 160 * 1024, "LDS");
};

template <int OUT, int FMT_A, int FMT_B, int BN>
__device__ __forceinline__ void gemm_f8_block_wide_body(const GemmBlockArgs &p) {
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    typedef __attribute__((address_space(3))) void lds_void;
    typedef BlockWideCfg<BN> C;
    constexpr int S = C::STAGES, NBM = C::NBM, NBN = C::NBN;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);  // wave-uniform: what derives from it is scalar
    const int lane = threadIdx.x & 63;
    const int wm0 = (wave >> 1) * C::WTM, wn0 = (wave & 1) * C::WTN;
    const unsigned lds_base = (unsigned)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)smem;
    const int KT = p.K / C::BK;
    const int tiles_n = (p.N + BN - 1) / BN, blocks_n = (p.N + 127) / 128;

    // ---- Tiles.  before: tile rows of the experts before this lane's share; total: of all.  (As in expert_tiles and
    // find_tile, written out: called here, they make the compiler copy fragments that are still on their way.)
    const int share = (p.experts + 63) / 64;
    int before = 0, total = (p.M + C::BM - 1) / C::BM;
    if (p.offsets != nullptr) {
        int mine = 0;
        for (int i = 0; i < share; ++i) {
            const int e = lane * share + i;
            if (e < p.experts) {
                const int first = min(max(p.offsets[e], 0), p.M), end = min(max(p.offsets[e + 1], first), p.M);
                mine += (end - first + C::BM - 1) / C::BM;
            }
        }
        int sum = mine;  // of the lanes up to this one
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int other = __shfl_up(sum, d, 64);
            if (lane >= d) sum += other;
        }
        before = sum - mine;
        total = __builtin_amdgcn_readlane(sum, 63);
        if constexpr (BN == 256) total = tiled_rows(p, total, tiles_n);
    }
    struct Tile {
        int row, end, tn, expert;  // first row; end of the expert's rows
        bool have;
    };
    auto tile_of = [&](int round) -> Tile {
        Tile t;
        int tm = 0;
        t.tn = t.expert = t.row = 0;
        t.end = p.M;
        t.have = gemm_tile_of(blockIdx.x, round, gridDim.x, total, tiles_n, 8, &tm, &t.tn);
        if (p.offsets == nullptr) {
            t.row = tm * C::BM;
        } else if (t.have) {
            // The last lane that has no more than tm tile rows before its share has the tile's expert in it.
            const int owner = __builtin_popcountll(__builtin_amdgcn_ballot_w64(before <= tm)) - 1;
            int at = tm - __builtin_amdgcn_readlane(before, owner);
            for (t.expert = owner * share;; ++t.expert) {
                int first, end;
                expert_rows(p, t.expert, &first, &end);
                const int tiles = (end - first + C::BM - 1) / C::BM;
                t.row = first + at * C::BM;
                t.end = end;
                if (at < tiles || t.expert + 1 >= p.experts) break;
                at -= tiles;
            }
        }
        return t;
    };
    auto weight_scales = [&](const Tile &t) -> int64_t {  // index of the scale byte of the first block of k
        return ((int64_t)t.expert * blocks_n + min((t.tn * BN + wn0) / 128, blocks_n - 1)) * KT;
    };

    // ---- Requests (swizzle as in gemm_i8_wide_kernel.h for blocks of 32 rows).  Rows past M (or N) read as zero; rows of the
    // next expert feed accumulators that are never stored.
    const int l_row = lane >> 3;
    unsigned voff[2];
#pragma unroll
    for (int v = 0; v < 2; ++v) voff[v] = (unsigned)l_row * p.K + (((lane ^ ((v * 8 + l_row) >> 1)) & 7) << 4);
    const unsigned req_step = 8u * p.K;
    int l_round = 0, l_left = 0;
    unsigned l_a = 0, l_b = 0, l_s = 0;                      // offsets of the next stage in the operands and the scales
    unsigned l_a_bytes = 0, l_b_bytes = 0, l_s_bytes = 0;    // their sizes, 0 past the last tile
    const uint8_t *l_b_base = p.b;
    auto next_tile_sources = [&]() {
        const Tile t = tile_of(l_round++);
        l_left = t.have ? KT : 1 << 30;
        l_a_bytes = t.have ? (unsigned)p.M * (unsigned)p.K : 0;
        l_b_bytes = t.have ? (unsigned)p.N * (unsigned)p.K : 0;
        l_s_bytes = t.have ? (unsigned)p.sa_bytes : 0;
        l_a = (unsigned)(t.row + wave * (C::BM / 4)) * (unsigned)p.K;
        l_b = (unsigned)(t.tn * BN + wave * (BN / 4)) * (unsigned)p.K;
        l_s = (unsigned)(t.row + wave * (C::BM / 4)) * 4;
        l_b_base = p.b + (int64_t)t.expert * p.N * p.K;
    };
    auto issue_req = [&](int slot, int i) {
        const bool is_a = i < C::REQ_A;
        const int r = is_a ? i : i - C::REQ_A;
        unsigned char *dst = smem + slot * C::STAGE_BYTES +
                             (is_a ? wave * C::REQ_A * 1024 : C::A_BYTES + wave * C::REQ_B * 1024) + r * 1024;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            __builtin_amdgcn_make_buffer_rsrc((void *)(is_a ? p.a : l_b_base), 0, is_a ? l_a_bytes : l_b_bytes, 0x00020000),
            (lds_void *)dst, 16, voff[r & 1], (is_a ? l_a : l_b) + (unsigned)r * req_step, 0, 0);
    };
    auto issue_scales = [&](int slot) {  // four blocks' bytes per row, of which the stage uses one
        __builtin_amdgcn_raw_ptr_buffer_load_lds(__builtin_amdgcn_make_buffer_rsrc((void *)p.sa, 0, l_s_bytes, 0x00020000),
                                                 (lds_void *)(smem + slot * C::STAGE_BYTES + C::CODE_BYTES + wave * 256), 4, lane * 4,
                                                 l_s + ((unsigned)(KT - l_left) >> 2) * (unsigned)p.sa_rows * 4, 0, 0);
    };
    auto advance = [&]() {
        l_a += C::BK;
        l_b += C::BK;
        if (--l_left == 0) next_tile_sources();
    };
    next_tile_sources();
#pragma unroll
    for (int s = 0; s < S; ++s) {
        issue_scales(s);
#pragma unroll
        for (int i = 0; i < C::REQ; ++i) issue_req(s, i);
        advance();
    }

    // ---- Fragments: 32 bytes of one row a lane, and the dword of its scale bytes.
    typedef v4i Half;
    const int f_r = lane & 31, f_g = lane >> 5;
    const unsigned f_off = f_r * C::BK + (((f_g * 2) ^ ((f_r >> 1) & 7)) << 4);
    const unsigned x_lane = lds_base + wm0 * C::BK + f_off, w_lane = lds_base + C::A_BYTES + wn0 * C::BK + f_off;
    const unsigned s_lane = lds_base + C::CODE_BYTES + (wm0 + f_r) * 4;
    Half xf[2][NBM][2], wf[2][NBN][2];
    unsigned sx_read[NBM], sx[NBM], sw_read = 0, sw = 0;  // as read; for the instructions
    auto issue_read = [&](int i, int buf, int slot) {
        constexpr int STEP = 32 * C::BK;
        const int n = i / 2, h = i % 2;  // fragments in the order w0 x0 w1 x1 ..., then the token side's others
        const bool is_x = n < 2 * NBN ? n & 1 : true;
        const int f = n < 2 * NBN ? n >> 1 : n - NBN;
        const unsigned at = ((is_x ? x_lane : w_lane) ^ (buf << 6 | h << 4)) + slot * C::STAGE_BYTES;
        Half &dst = is_x ? xf[buf][f][h] : wf[buf][f][h];
        switch (f) {
            case 0: dst = lds_read_b128<0>(at); break;
            case 1: dst = lds_read_b128<STEP>(at); break;
            case 2: dst = lds_read_b128<2 * STEP>(at); break;
            default: dst = lds_read_b128<3 * STEP>(at); break;
        }
    };
    auto issue_scale_read = [&](int a, int slot) {
        const unsigned at = s_lane + slot * C::STAGE_BYTES;
        asm volatile("ds_read_b32 %0, %1 offset:%2" : "=v"(sx_read[a]) : "v"(at), "n"(a * 128));
    };
    auto pin_frags = [&](int buf) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int f = 0; f < NBM; ++f) asm volatile("" : "+v"(xf[buf][f][h]));
#pragma unroll
            for (int f = 0; f < NBN; ++f) asm volatile("" : "+v"(wf[buf][f][h]));
        }
    };

    Tile t = tile_of(0);
    wait_vmcnt<(S - 1) * C::LPW>();
    block_barrier();
    if (!t.have) {
        wait_vmcnt<0>();
        return;
    }
    int64_t scales_at = weight_scales(t), next_scale = 0;  // of the tile; of the next stage
    sw_read = uniform_byte(p.sb, scales_at);
#pragma unroll
    for (int a = 0; a < NBM; ++a) issue_scale_read(a, 0);
    wait_lds_reads();
#pragma unroll
    for (int a = 0; a < NBM; ++a) {
        asm volatile("" : "+v"(sx_read[a]));
        sx[a] = sx_read[a];
    }
#pragma unroll
    for (int i = 0; i < C::NREADS; ++i) issue_read(i, 0, 0);

    int slot = 0;   // of the stage in work
    int block = 0;  // of k: the stage that the next half stage 0 works on
    int slack = 0;  // hand-overs whose wait may leave an epilogue's stores outstanding

    // ---- Epilogue of the tile that has just been finished.
    __amdgpu_buffer_rsrc_t rsrc_out;
    unsigned o_voff = 0;
    int cols_in = 0, n_out = p.N;
    constexpr unsigned NOWHERE = 0x80000000u;
    constexpr int OB = OUT == OUT_BF16 ? 2 : 4;
    const unsigned patch = lds_base + S * C::STAGE_BYTES + wave * C::PATCH_BYTES;
    const unsigned patch_w = patch + f_r * C::PATCH_PITCH + f_g * 8;
    constexpr int PPR = C::PPR;
    const unsigned patch_r = patch + (lane / PPR) * C::PATCH_PITCH + (lane % PPR) * 16;
    auto epi_begin = [&](const Tile &t) {
        const int m_base = t.row + wm0, n_base = t.tn * BN + wn0;
        const unsigned rows_in = __builtin_amdgcn_readfirstlane(min(max(t.end - m_base, 0), C::WTM));
        cols_in = p.N - n_base;
        n_out = p.N;
        asm volatile("" : "+s"(n_out));
        rsrc_out = __builtin_amdgcn_make_buffer_rsrc(static_cast<char *>(p.out) + ((int64_t)m_base * p.N + n_base) * OB, 0,
                                                     rows_in * (unsigned)p.N * OB, 0x00020000);
        int lane_e = lane;
        asm volatile("" : "+v"(lane_e));
        if (OUT == OUT_BF16)
            o_voff = (unsigned)((lane_e / PPR) * p.N + (lane_e % PPR) * 8) * 2;
        else
            o_voff = (unsigned)((lane_e & 15) * p.N + (lane_e >> 4 & 1) * 8 + (lane_e >> 5) * 4) * 4;
    };
    v4u val[C::PATCH_READS];
    auto epi_quad = [&](int a, int b, int q, const float *x) {
        v4f y0, y1;
#pragma unroll
        for (int e = 0; e < 4; ++e) y0[e] = x[4 * q + e];
        if (OUT == OUT_F32) {
            // Two quads, exchanged between groups of 16 lanes: 64 bytes of 16 rows a store (gemm_i8_wide_kernel.h).
            if (q & 1) return;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                y1[e] = x[4 * q + 4 + e];
                const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(y0[e]), __float_as_uint(y1[e]), false, false);
                y0[e] = __uint_as_float(s[0]);
                y1[e] = __uint_as_float(s[1]);
            }
            const unsigned at = b * 32 < cols_in ? o_voff : NOWHERE;
            const unsigned soff = (unsigned)(a * 32 * n_out + b * 32 + q * 8) * 4;
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4u, y0), rsrc_out, at, soff, 0);
            __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4u, y1), rsrc_out, at, soff + 16u * n_out * 4, 0);
        } else {
            const v2u pk = __builtin_bit_cast(v2u, __builtin_convertvector(y0, v4bf));
            const int col = (b * 32) % C::PATCH_COLS + q * 8;
            asm volatile("ds_write_b64 %0, %1 offset:%2" ::"v"(patch_w), "v"(pk), "n"(col * 2));
        }
    };
    auto epi_read_patch = [&]() {
#pragma unroll
        for (int j = 0; j < C::PATCH_READS; ++j)
            asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(val[j]) : "v"(patch_r), "n"(j * (64 / PPR) * C::PATCH_PITCH));
    };
    auto epi_store_patch = [&](int a, int col0) {  // after a wait
        const unsigned at = (lane % PPR) * 8 + col0 < cols_in ? o_voff : NOWHERE;
#pragma unroll
        for (int j = 0; j < C::PATCH_READS; ++j) {
            asm volatile("" : "+v"(val[j]));
            __builtin_amdgcn_raw_buffer_store_b128(val[j], rsrc_out, at, (unsigned)((a * 32 + j * (64 / PPR)) * n_out + col0) * 2, 2);
        }
    };
    constexpr int PATCH_SLOTS = C::PATCH_SLOTS;
    constexpr int STORES = OUT == OUT_BF16 ? C::WTM * C::WTN / 512 : C::WTM * C::WTN / 256;  // of an epilogue, per lane, behind its last request

    auto multiply = [](auto fresh, int r0, const Half (&w)[2], const Half (&x)[2], unsigned w_scale, unsigned x_scale) __attribute__((always_inline)) {
        const v8i w8 = __builtin_shufflevector(w[0], w[1], 0, 1, 2, 3, 4, 5, 6, 7);
        const v8i x8 = __builtin_shufflevector(x[0], x[1], 0, 1, 2, 3, 4, 5, 6, 7);
        if constexpr (decltype(fresh)::value)
            asm volatile("v_mfma_scale_f32_32x32x64_f8f6f4 a[%0:%1], %2, %3, 0, %4, %5 op_sel_hi:[0,0,0] cbsz:%6 blgp:%7" ::"n"(r0),
                         "n"(r0 + 15), "v"(w8), "v"(x8), "v"(w_scale), "v"(x_scale), "n"(FMT_B), "n"(FMT_A));
        else
            asm volatile("v_mfma_scale_f32_32x32x64_f8f6f4 a[%0:%1], %2, %3, a[%0:%1], %4, %5 op_sel_hi:[0,0,0] cbsz:%6 blgp:%7" ::"n"(r0),
                         "n"(r0 + 15), "v"(w8), "v"(x8), "v"(w_scale), "v"(x_scale), "n"(FMT_B), "n"(FMT_A));
    };

    // Half a stage, as in gemm_i8_wide_kernel.h: NORMAL; the FIRST of a tile; the same with the epilogue of the tile before; the
    // LAST of the workgroup, with its tile's own epilogue.
    enum { NORMAL, FIRST, FIRST_EPI, LAST };
    auto period = [&](auto cur_c, auto kind_c) __attribute__((always_inline)) {
        constexpr int cur = decltype(cur_c)::value, nxt = cur ^ 1, kind = decltype(kind_c)::value;
        constexpr bool epi = kind == FIRST_EPI || kind == LAST, more = kind != LAST;
        // A result is there 19 wait states after its instruction: the LAST epilogue stays two instructions behind.
        constexpr int LAG = kind == LAST ? 2 : 0;
        const int next_slot = !cur ? slot : slot + 1 == S ? 0 : slot + 1, prev_slot = slot == 0 ? S - 1 : slot - 1;
        keep_out_of_agprs();
        if (cur && more) {
            constexpr int later = (S - 2) * C::LPW, with_stores = later + STORES < 63 ? later + STORES : 63;
            if (slack == 0) {
                wait_vmcnt<later>();
            } else {
                --slack;
                wait_vmcnt<with_stores>();
            }
        }
        wait_lds_reads();
        if (cur && more) block_barrier();
        pin_frags(cur);
        if (!cur) {
            sw = sw_read;
            // Nobody knows of the matrix instructions in the asm: what the vector unit writes is theirs two wait states later.
            asm volatile("s_nop 1" : "+v"(sw));
        }
        const unsigned shift = (unsigned)(block & 3) * 8;
        auto next_x_scale = [&](int a) {  // not before the last instruction that uses the scale at hand
            sx[a] = sx_read[a] >> shift;
            asm volatile("" : "+v"(sx[a]));
        };
#pragma unroll
        for (int idx = 0; idx < C::SLOTS + LAG; ++idx) {
            const int a = idx / NBN, b = idx % NBN;
            const int e = idx - LAG, ea = e / NBN, eb = e % NBN;  // block whose epilogue it is
            float x[16];
            auto read_block = [&]() {
#pragma unroll
                for (int i = 0; i < 16; ++i) asm volatile("v_accvgpr_read_b32 %0, a[%1]" : "=v"(x[i]) : "n"(e * 16 + i));
            };
            auto store_patch_before = [&](int behind) {
                if (behind == 2) wait_lgkmcnt<2>(); else wait_lgkmcnt<0>();
                const int last = e / PATCH_SLOTS * PATCH_SLOTS - 1;
                epi_store_patch(last / NBN, last % NBN / PATCH_SLOTS * C::PATCH_COLS);
            };
            if (kind == FIRST_EPI) read_block();
            if (idx < C::SLOTS)
                multiply(std::integral_constant<bool, kind == FIRST || kind == FIRST_EPI>(), (a * NBN + b) * 16, wf[cur][b], xf[cur][a], sw, sx[a]);
            if constexpr (more) {
                // The next stage's scales come before its fragments: four reads behind them they have landed.
                constexpr int AHEAD = cur ? NBM : 0;
                if (cur && idx == AHEAD) {
                    wait_lgkmcnt<AHEAD>();
#pragma unroll
                    for (int i = 0; i < NBM; ++i) asm volatile("" : "+v"(sx_read[i]));
                }
                if (cur && idx >= AHEAD) {
#pragma unroll
                    for (int i = 0; i < NBM - 1; ++i)
                        if (idx == (NBN * (i + 1) > AHEAD ? NBN * (i + 1) : AHEAD)) next_x_scale(i);
                }
                if (!cur && idx == 0) next_x_scale(NBM - 1);
                if (cur && idx == AHEAD) sw_read = uniform_byte(p.sb, next_scale);
#pragma unroll
                for (int i = 2 * idx; i < 2 * idx + 2; ++i) {
                    if (i < AHEAD) issue_scale_read(i, next_slot);
                    else if (i < AHEAD + C::NREADS) issue_read(i - AHEAD, nxt, next_slot);
                }
                constexpr int N2 = C::REQ_2ND, N1 = C::REQ - N2;
                if constexpr (cur == 1) {
                    constexpr int RQ = C::SLOTS / N2;
                    if (idx == 0) issue_scales(slot);
                    if (idx % RQ == RQ / 2 && idx / RQ < N2) issue_req(slot, idx / RQ);
                } else if constexpr (N1 > 0 && kind != FIRST) {
                    constexpr int RQ = epi ? 1 : C::SLOTS / N1, PER = epi ? N1 : 1;
#pragma unroll
                    for (int i = idx / RQ * PER; i < (idx / RQ + 1) * PER; ++i)
                        if (idx % RQ == RQ / 2 && i < N1) issue_req(prev_slot, N2 + i);
                }
            }
            if (epi && e >= 0) {
                const bool store = OUT == OUT_BF16 && e >= PATCH_SLOTS && e % PATCH_SLOTS == 0;
                if (store) store_patch_before(more && 2 * idx + 2 <= C::NREADS ? 2 : 0);
                if (kind == LAST) read_block();
#pragma unroll
                for (int q = 0; q < 4; ++q) epi_quad(ea, eb, q, x);
                if (OUT == OUT_BF16 && (e + 1) % PATCH_SLOTS == 0) epi_read_patch();
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if (epi && OUT == OUT_BF16) {
            wait_lds_reads();
            epi_store_patch(NBM - 1, C::WTN - C::PATCH_COLS);
        }
        if (C::REQ_2ND == C::REQ ? cur == 1 && more : cur == 0 && (kind == NORMAL || kind == FIRST_EPI)) advance();
        if (cur) slot = next_slot;
        if (epi) slack = S - 1;
        keep_out_of_agprs();
    };
    typedef std::integral_constant<int, 0> I0;
    typedef std::integral_constant<int, 1> I1;
    typedef std::integral_constant<int, NORMAL> KNormal;
    typedef std::integral_constant<int, FIRST> KFirst;
    typedef std::integral_constant<int, FIRST_EPI> KFirstEpi;
    typedef std::integral_constant<int, LAST> KLast;

    period(I0(), KFirst());
    for (int round = 1;; ++round) {
        for (int kt = 1; kt < KT; ++kt) {
            next_scale = scales_at + kt;
            block = kt;
            period(I1(), KNormal());
            period(I0(), KNormal());
        }
        const Tile next = tile_of(round);
        if (!next.have) break;
        next_scale = scales_at = weight_scales(next);
        block = 0;
        period(I1(), KNormal());
        epi_begin(t);
        t = next;
        period(I0(), KFirstEpi());
    }
    epi_begin(t);
    period(I1(), KLast());
    wait_vmcnt<0>();  // the requests past the end write LDS
}

}  // namespace sb
