// Layer norm over the rows of a matrix, forward and backward, for gfx950.
//
//   mu = mean_j x,  r = 1 / sqrt(mean_j (x - mu)^2 + eps),  h = (x - mu) r,  y = h gamma + beta
//   a = dy gamma,   dx = r (a - mean_j a - h mean_j(a h)),  dgamma_j = sum_i dy h,  dbeta_j = sum_i dy
//
// What bounds it: memory.  A row is read once and stays in registers: the mean first, then the squares of the differences from it
// (a variance formed as E x^2 - mu^2 would lose all digits of rows whose mean is large), and the mean of these differences, by which
// the first one was off (29.4 -> 29.9 us at 32896 x 1280 bf16, nothing elsewhere).  Rows of up to 2048 columns belong to a
// wave, short ones to a part of one, up to 8192 to four waves and up to 16384 to eight; a group walks many rows, holds gamma and
// beta (or its shares of both sums) in registers, and requests its next row before it works on this one.  Wider rows are read
// again: from L2 as long as the 64 rows that an XCD's workgroups have in work fit into its 4 MiB (bf16 up to 32768 columns forward
// and 16384 backward, half of that in f32), else from beyond.  Arithmetic is binary32; y and dx are rounded once.
// 32896 x 1280 bf16: forward 29.9 us, 5.6 TB/s (f32 62, 5.4); backward 46 us and 4.8 for the sums' reduction, 5.0 TB/s; f32 11237 x
// 1088 backward 29 + 4.
//
// The sums over the rows: every workgroup adds its rows' terms in registers, its waves' sums meet in LDS and go to the
// workspace, and a second launch adds those in a fixed order.  No atomics: the same inputs give the same bits.
#include "sb_common.h"
#include <type_traits>

namespace sb {
namespace {

typedef unsigned short u16;

template <class T>
__device__ __forceinline__ float widen(T v) {
    if constexpr (sizeof(T) == 2) return bf16_bits_to_float(v);
    else return v;
}
// Element type T is u16 (bf16 bits) or float; a piece is V consecutive elements: 16 bytes, or one element of rows shorter than
// that.  Rows that are not whole pieces (WHOLE false) start anywhere, and their last piece starts early enough to end with the
// row: it shares elements with the one before, which count once in the sums and are stored twice, with the same value.  (With
// loads of single elements instead, 4000 x 1001 bf16: 6.8 us forward, 19.7 backward; 5.9 and 13.8 so.)
template <class T, int V>
struct Piece {
    T e[V];
};
typedef unsigned int v4u_at2 __attribute__((ext_vector_type(4), aligned(2)));
typedef unsigned int v4u_at4 __attribute__((ext_vector_type(4), aligned(4)));
// (Each type by its name: deduced as a template's argument it would lose its alignment.)
template <int ALIGN, bool ONCE>
__device__ __forceinline__ v4u load_quad(const void *at) {
    const v4u_at2 *at2 = static_cast<const v4u_at2 *>(at);
    const v4u_at4 *at4 = static_cast<const v4u_at4 *>(at);
    const v4u *at16 = static_cast<const v4u *>(at);
    if constexpr (ALIGN == 2) return ONCE ? __builtin_nontemporal_load(at2) : *at2;
    else if constexpr (ALIGN == 4) return ONCE ? __builtin_nontemporal_load(at4) : *at4;
    else return ONCE ? __builtin_nontemporal_load(at16) : *at16;
}
template <int ALIGN>
__device__ __forceinline__ void store_quad(void *at, v4u v) {
    if constexpr (ALIGN == 2) *static_cast<v4u_at2 *>(at) = v;
    else if constexpr (ALIGN == 4) *static_cast<v4u_at4 *>(at) = v;
    else *static_cast<v4u *>(at) = v;
}
// ONCE: nobody reads it again.
template <class T, int V, bool WHOLE, bool ONCE = true>
__device__ __forceinline__ Piece<T, V> load_piece(const T *at) {
    if constexpr (V == 1) {
        return Piece<T, 1>{{ONCE ? __builtin_nontemporal_load(at) : *at}};
    } else {
        static_assert(sizeof(T) * V == 16, "16 bytes");
        return __builtin_bit_cast(Piece<T, V>, (load_quad<WHOLE ? 16 : (int)sizeof(T), ONCE>(at)));
    }
}
template <class T, int V, bool WHOLE>
__device__ __forceinline__ void store_piece(T *at, const float (&v)[V]) {
    constexpr int ALIGN = WHOLE ? 16 : (int)sizeof(T);
    if constexpr (V == 1) {
        if constexpr (sizeof(T) == 4) *at = v[0];
        else *at = __builtin_bit_cast(u16, (__bf16)v[0]);
    } else if constexpr (sizeof(T) == 4) {
        store_quad<ALIGN>(at, __builtin_bit_cast(v4u, (v4f{v[0], v[1], v[2], v[3]})));
    } else {
        const v2u lo = __builtin_bit_cast(v2u, __builtin_convertvector(v4f{v[0], v[1], v[2], v[3]}, v4bf));
        const v2u hi = __builtin_bit_cast(v2u, __builtin_convertvector(v4f{v[4], v[5], v[6], v[7]}, v4bf));
        store_quad<ALIGN>(at, v4u{lo.x, lo.y, hi.x, hi.y});
    }
}
// V elements of a binary32 vector.
template <int V, bool WHOLE>
__device__ __forceinline__ void load_vector(const float *v, int at, float (&out)[V]) {
    if constexpr (V == 1) {
        out[0] = v[at];
    } else {
#pragma unroll
        for (int q = 0; q < V; q += 4) {
            const v4f x = __builtin_bit_cast(v4f, (load_quad<WHOLE ? 16 : 4, false>(v + at + q)));
#pragma unroll
            for (int e = 0; e < 4; ++e) out[q + e] = x[e];
        }
    }
}
// The piece whose columns begin at c: its first column in memory, and how many of its elements belong to the one before.
template <int V, bool WHOLE>
__device__ __forceinline__ int piece_at(int c, int cols) {
    return WHOLE || V == 1 ? c : min(c, cols - V);
}

// A row belongs to a group of LANES lanes: part of a wave, a wave, or a workgroup.
template <int LANES_>
struct Group {
    static constexpr int LANES = LANES_, THREADS = LANES <= 64 ? 256 : LANES, PER_BLOCK = THREADS / LANES;
};

// Sums of a group, in every lane of it.  A group of several waves is the workgroup; `turn` alternates, so that one barrier does:
// who writes a buffer again has passed the barrier of the call between.
template <int LANES, int N>
__device__ __forceinline__ void group_sums(float (&v)[N], float (*shared)[2][16], int turn) {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int off = (LANES < 64 ? LANES : 64) / 2; off > 0; off >>= 1) v[i] += __shfl_xor(v[i], off, 64);
    if constexpr (LANES > 64) {
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) shared[turn][i][threadIdx.x >> 6] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = shared[turn][i][0];
#pragma unroll
            for (int w = 1; w < LANES / 64; ++w) v[i] += shared[turn][i][w];
        }
    }
}

// The first mean is off by its sum's roundings, which a row far from zero multiplies by r (1920 columns of 10000: mean 10000.001, y
// -0.3).  The differences d from it are exact there, so their own mean is what it is off by, and the variance is that of d.
__device__ __forceinline__ float reciprocal_deviation(float mean_of_squares, float off, float eps) {
    const float var = mean_of_squares - off * off;
    return 1.0f / sqrtf((var < 0.0f ? 0.0f : var) + eps);  // NaN stays
}

// Rows of up to LANES * V * P columns; P pieces a lane.  mean and rstd may be null, and gamma and beta.
template <class T, int V, int P, int LANES, bool WHOLE>
__global__ __launch_bounds__(Group<LANES>::THREADS) void layer_norm_kernel(const T *__restrict__ x, const float *__restrict__ gamma,
                                                                            const float *__restrict__ beta, float eps,
                                                                            int64_t rows, int cols, T *__restrict__ y,
                                                                            float *__restrict__ mean, float *__restrict__ rstd) {
    typedef Group<LANES> G;
    __shared__ float shared[2][2][16];
    const int lane = threadIdx.x % G::LANES;
    const int64_t first = (int64_t)blockIdx.x * G::PER_BLOCK + threadIdx.x / G::LANES, step = (int64_t)gridDim.x * G::PER_BLOCK;
    float g[P][V], b[P][V];
    int at[P], shared_with[P];  // of a piece: first column; elements of the one before
#pragma unroll
    for (int p = 0; p < P; ++p) {
        const int c = (lane + p * G::LANES) * V;
        at[p] = piece_at<V, WHOLE>(c, cols);
        shared_with[p] = c - at[p];
#pragma unroll
        for (int e = 0; e < V; ++e) g[p][e] = 1.0f, b[p][e] = 0.0f;
        if (c < cols) {
            if (gamma != nullptr) load_vector<V, WHOLE>(gamma, at[p], g[p]);
            if (beta != nullptr) load_vector<V, WHOLE>(beta, at[p], b[p]);
        }
    }
    Piece<T, V> raw[P];
    auto request = [&](int64_t row) {
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int c = (lane + p * G::LANES) * V;
            raw[p] = Piece<T, V>{};
            if (c < cols) raw[p] = load_piece<T, V, WHOLE>(x + row * cols + at[p]);
        }
    };
    const float inv = 1.0f / (float)cols;
    if (first < rows) request(first);
    // All waves of a workgroup make the same number of rounds where they meet at barriers: it has one row then.
    for (int64_t row = first; row < rows; row += step) {
        float v[P][V], s[1] = {0.0f};
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                v[p][e] = widen(raw[p].e[e]);
                s[0] += WHOLE || e >= shared_with[p] ? v[p][e] : 0.0f;
            }
        if (row + step < rows) request(row + step);
        group_sums<LANES, 1>(s, shared, 0);
        const float near = s[0] * inv;
        float t[2] = {0.0f, 0.0f};
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const bool in = (lane + p * G::LANES) * V < cols;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                v[p][e] = in ? v[p][e] - near : 0.0f;
                const float d = WHOLE || e >= shared_with[p] ? v[p][e] : 0.0f;
                t[0] = fmaf(d, d, t[0]);
                t[1] += d;
            }
        }
        group_sums<LANES, 2>(t, shared, 1);
        const float off = t[1] * inv, r = reciprocal_deviation(t[0] * inv, off, eps);
        if (lane == 0) {
            if (mean != nullptr) mean[row] = near + off;
            if (rstd != nullptr) rstd[row] = r;
        }
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int c = (lane + p * G::LANES) * V;
            float out[V];
#pragma unroll
            for (int e = 0; e < V; ++e) out[e] = fmaf((v[p][e] - off) * r, g[p][e], b[p][e]);
            if (c < cols) store_piece<T, V, WHOLE>(y + row * cols + at[p], out);
        }
    }
}

// Rows that do not fit: three passes.
template <class T, int V, bool WHOLE>
__global__ __launch_bounds__(1024) void layer_norm_long_kernel(const T *__restrict__ x, const float *__restrict__ gamma,
                                                               const float *__restrict__ beta, float eps, int64_t rows, int cols,
                                                               T *__restrict__ y, float *__restrict__ mean,
                                                               float *__restrict__ rstd) {
    __shared__ float shared[2][2][16];
    const float inv = 1.0f / (float)cols;
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const T *xr = x + row * cols;
        float s[1] = {0.0f};
        for (int c = threadIdx.x * V; c < cols; c += 1024 * V) {
            const int at = piece_at<V, WHOLE>(c, cols);
            const Piece<T, V> q = load_piece<T, V, WHOLE, false>(xr + at);
#pragma unroll
            for (int e = 0; e < V; ++e) s[0] += at + e >= c ? widen(q.e[e]) : 0.0f;
        }
        group_sums<1024, 1>(s, shared, 0);
        const float near = s[0] * inv;
        float t[2] = {0.0f, 0.0f};
        for (int c = threadIdx.x * V; c < cols; c += 1024 * V) {
            const int at = piece_at<V, WHOLE>(c, cols);
            const Piece<T, V> q = load_piece<T, V, WHOLE, false>(xr + at);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float d = at + e >= c ? widen(q.e[e]) - near : 0.0f;
                t[0] = fmaf(d, d, t[0]);
                t[1] += d;
            }
        }
        group_sums<1024, 2>(t, shared, 1);
        const float off = t[1] * inv, r = reciprocal_deviation(t[0] * inv, off, eps);
        if (threadIdx.x == 0) {
            if (mean != nullptr) mean[row] = near + off;
            if (rstd != nullptr) rstd[row] = r;
        }
        for (int c = threadIdx.x * V; c < cols; c += 1024 * V) {
            const int at = piece_at<V, WHOLE>(c, cols);
            const Piece<T, V> q = load_piece<T, V, WHOLE, false>(xr + at);
            float g[V], b[V], out[V];
#pragma unroll
            for (int e = 0; e < V; ++e) g[e] = 1.0f, b[e] = 0.0f;
            if (gamma != nullptr) load_vector<V, WHOLE>(gamma, at, g);
            if (beta != nullptr) load_vector<V, WHOLE>(beta, at, b);
#pragma unroll
            for (int e = 0; e < V; ++e) out[e] = fmaf((widen(q.e[e]) - near - off) * r, g[e], b[e]);
            store_piece<T, V, WHOLE>(y + row * cols + at, out);
        }
    }
}

// dgamma and dbeta of 16 columns by a workgroup of `threads`: runs of rows in turn, then the runs in pairs.
template <class T, int THREADS>
__device__ __forceinline__ void column_sums(const T *__restrict__ dy, const T *__restrict__ x, const float *__restrict__ mean,
                                            const float *__restrict__ rstd, int rows, int cols, int block, float *__restrict__ dgamma,
                                            float *__restrict__ dbeta) {
    constexpr int COLS = 16, RUNS = THREADS / COLS, AT_ONCE = 8;
    __shared__ float runs[2][RUNS][COLS + 1];
    const int i = threadIdx.x % COLS, run = threadIdx.x / COLS, c = block * COLS + i;
    float s[2] = {0.0f, 0.0f};
    if (c < cols)
        for (int row = run; row < rows; row += RUNS * AT_ONCE) {
            float d[AT_ONCE], h[AT_ONCE];
#pragma unroll
            for (int j = 0; j < AT_ONCE; ++j) {
                const int at = min(row + j * RUNS, rows - 1);
                d[j] = widen(dy[(int64_t)at * cols + c]);
                h[j] = (widen(x[(int64_t)at * cols + c]) - mean[at]) * rstd[at];
            }
#pragma unroll
            for (int j = 0; j < AT_ONCE; ++j)
                if (row + j * RUNS < rows) {
                    s[0] = fmaf(d[j], h[j], s[0]);
                    s[1] += d[j];
                }
        }
    runs[0][run][i] = s[0];
    runs[1][run][i] = s[1];
#pragma unroll
    for (int half = RUNS / 2; half > 0; half >>= 1) {
        __syncthreads();
        if (run < half)
#pragma unroll
            for (int k = 0; k < 2; ++k) runs[k][run][i] = s[k] = s[k] + runs[k][run + half][i];
    }
    if (run == 0 && c < cols) {
        if (dgamma != nullptr) dgamma[c] = s[0];
        if (dbeta != nullptr) dbeta[c] = s[1];
    }
}

// SUMS: the rows' terms of dgamma and dbeta are added up and left in partial[blockIdx.x][2][cols].  Without, workgroups from
// row_blocks on form the sums of 16 columns each from the rows themselves: for few rows, which lie in L2 and are read twice
// sooner than a second launch starts.  gamma lies in LDS, four consecutive elements of a lane at a time and lanes side by side:
// in registers, next to the sums and two rows, it would leave one wave per SIMD.
template <class T, int V, int P, int LANES, bool SUMS, bool WHOLE>
__global__ __launch_bounds__(Group<LANES>::THREADS) void layer_norm_backward_kernel(
    const T *__restrict__ dy, const T *__restrict__ x, const float *__restrict__ mean, const float *__restrict__ rstd,
    const float *__restrict__ gamma, int64_t rows, int cols, T *__restrict__ dx, float *__restrict__ partial, int row_blocks,
    float *__restrict__ dgamma, float *__restrict__ dbeta) {
    typedef Group<LANES> G;
    if (!SUMS && (int)blockIdx.x >= row_blocks) {
        column_sums<T, G::THREADS>(dy, x, mean, rstd, (int)rows, cols, (int)blockIdx.x - row_blocks, dgamma, dbeta);
        return;
    }
    constexpr int Q = V < 4 ? V : 4;
    typedef float Quad __attribute__((ext_vector_type(Q)));
    __shared__ float shared[2][2][16];
    __shared__ Quad weights[P][V / Q][G::LANES];
    const int lane = threadIdx.x % G::LANES;
    const int64_t first = (int64_t)blockIdx.x * G::PER_BLOCK + threadIdx.x / G::LANES, step = (int64_t)(SUMS ? gridDim.x : row_blocks) * G::PER_BLOCK;
    float dg[SUMS ? P : 1][V], db[SUMS ? P : 1][V];
    int at[P], shared_with[P];  // of a piece: first column; elements of the one before
#pragma unroll
    for (int p = 0; p < P; ++p) {
        at[p] = piece_at<V, WHOLE>((lane + p * G::LANES) * V, cols);
        shared_with[p] = (lane + p * G::LANES) * V - at[p];
    }
    if (threadIdx.x < G::LANES) {
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int q = 0; q < V / Q; ++q) {
                float v[Q];
#pragma unroll
                for (int e = 0; e < Q; ++e) v[e] = 1.0f;
                if ((lane + p * G::LANES) * V < cols && gamma != nullptr) load_vector<Q, WHOLE>(gamma, at[p] + q * Q, v);
                Quad g;
#pragma unroll
                for (int e = 0; e < Q; ++e) g[e] = v[e];
                weights[p][q][lane] = g;
            }
    }
    if (SUMS)
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int e = 0; e < V; ++e) dg[p][e] = db[p][e] = 0.0f;
    Piece<T, V> rx[P], rdy[P];
    float mu = 0.0f, r = 0.0f;
    auto request = [&](int64_t row) {
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int c = (lane + p * G::LANES) * V;
            rx[p] = rdy[p] = Piece<T, V>{};
            if (c < cols) {
                rx[p] = load_piece<T, V, WHOLE>(x + row * cols + at[p]);
                rdy[p] = load_piece<T, V, WHOLE>(dy + row * cols + at[p]);
            }
        }
        mu = mean[row];
        r = rstd[row];
    };
    const float inv = 1.0f / (float)cols;
    if (first < rows) request(first);
    __syncthreads();
    int turn = 0;
    for (int64_t row = first; row < rows; row += step, turn ^= 1) {
        float h[P][V], d[P][V], s[2] = {0.0f, 0.0f};
        const float r0 = r;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const bool in = (lane + p * G::LANES) * V < cols;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                d[p][e] = widen(rdy[p].e[e]);  // zero past the last column
                h[p][e] = in ? (widen(rx[p].e[e]) - mu) * r : 0.0f;
                const float own = WHOLE || e >= shared_with[p] ? d[p][e] : 0.0f, a = own * weights[p][e / Q][lane][e % Q];
                s[0] += a;
                s[1] = fmaf(a, h[p][e], s[1]);
                if (SUMS) {
                    dg[p][e] = fmaf(own, h[p][e], dg[p][e]);
                    db[p][e] += own;
                }
            }
        }
        if (row + step < rows) request(row + step);
        group_sums<LANES, 2>(s, shared, turn);
        const float sa = s[0] * inv, sh = s[1] * inv;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const int c = (lane + p * G::LANES) * V;
            float out[V];
#pragma unroll
            for (int e = 0; e < V; ++e) out[e] = r0 * (fmaf(d[p][e], weights[p][e / Q][lane][e % Q], -sa) - h[p][e] * sh);
            if (c < cols) store_piece<T, V, WHOLE>(dx + row * cols + at[p], out);
        }
    }
    if constexpr (SUMS) {
        float *mine = partial + (int64_t)blockIdx.x * 2 * cols;
        if constexpr (G::PER_BLOCK == 1) {
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const int c = at[p] + e;
                    if (c < cols && (WHOLE || ((lane + p * G::LANES) * V < cols && e >= shared_with[p])))
                        mine[c] = dg[p][e], mine[cols + c] = db[p][e];
                }
        } else {
            // The waves' sums of a piece at a time, in wave order.
            constexpr int SLOTS = G::LANES * V;
            __shared__ float meet[G::PER_BLOCK][2][SLOTS];
            const int wave = threadIdx.x / G::LANES;
#pragma unroll
            for (int p = 0; p < P; ++p) {
                __syncthreads();
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    // What is shared with the piece before is zero, and goes behind the last column.
                    const int to = WHOLE ? e : (e - shared_with[p]) & (V - 1);
                    meet[wave][0][to * G::LANES + lane] = dg[p][e];
                    meet[wave][1][to * G::LANES + lane] = db[p][e];
                }
                __syncthreads();
                for (int i = threadIdx.x; i < 2 * SLOTS; i += G::THREADS) {
                    const int which = i / SLOTS, slot = i % SLOTS;
                    // Slot (column order): lane slot / V, element slot % V.
                    const int at = (slot % V) * G::LANES + slot / V, c = p * SLOTS + slot;
                    float sum = meet[0][which][at];
#pragma unroll
                    for (int w = 1; w < G::PER_BLOCK; ++w) sum += meet[w][which][at];
                    if (c < cols) mine[which * cols + c] = sum;
                }
            }
        }
    }
}

// Rows that do not fit: two passes; the sums over the rows are another launch's.
template <class T, int V, bool WHOLE>
__global__ __launch_bounds__(1024) void layer_norm_backward_long_kernel(const T *__restrict__ dy, const T *__restrict__ x,
                                                                        const float *__restrict__ mean,
                                                                        const float *__restrict__ rstd,
                                                                        const float *__restrict__ gamma, int64_t rows, int cols,
                                                                        T *__restrict__ dx) {
    __shared__ float shared[2][2][16];
    const float inv = 1.0f / (float)cols;
    int turn = 0;
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x, turn ^= 1) {
        const T *xr = x + row * cols, *dr = dy + row * cols;
        const float mu = mean[row], r = rstd[row];
        float s[2] = {0.0f, 0.0f};
        for (int c = threadIdx.x * V; c < cols; c += 1024 * V) {
            const int at = piece_at<V, WHOLE>(c, cols);
            const Piece<T, V> q = load_piece<T, V, WHOLE, false>(xr + at), d = load_piece<T, V, WHOLE, false>(dr + at);
            float g[V];
#pragma unroll
            for (int e = 0; e < V; ++e) g[e] = 1.0f;
            if (gamma != nullptr) load_vector<V, WHOLE>(gamma, at, g);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float a = at + e >= c ? widen(d.e[e]) * g[e] : 0.0f;
                s[0] += a;
                s[1] = fmaf(a, (widen(q.e[e]) - mu) * r, s[1]);
            }
        }
        group_sums<1024, 2>(s, shared, turn);
        const float sa = s[0] * inv, sh = s[1] * inv;
        for (int c = threadIdx.x * V; c < cols; c += 1024 * V) {
            const int at = piece_at<V, WHOLE>(c, cols);
            const Piece<T, V> q = load_piece<T, V, WHOLE, false>(xr + at), d = load_piece<T, V, WHOLE, false>(dr + at);
            float g[V], out[V];
#pragma unroll
            for (int e = 0; e < V; ++e) g[e] = 1.0f;
            if (gamma != nullptr) load_vector<V, WHOLE>(gamma, at, g);
#pragma unroll
            for (int e = 0; e < V; ++e) out[e] = r * (widen(d.e[e]) * g[e] - sa - (widen(q.e[e]) - mu) * r * sh);
            store_piece<T, V, WHOLE>(dx + row * cols + at, out);
        }
    }
}
// partial[blockIdx.y][2][cols]: sums over the blockIdx.y-th share of the rows, a column a thread.
template <class T>
__global__ __launch_bounds__(256) void layer_norm_column_sums_kernel(const T *__restrict__ dy, const T *__restrict__ x,
                                                                     const float *__restrict__ mean,
                                                                     const float *__restrict__ rstd, int64_t rows, int cols,
                                                                     float *__restrict__ partial) {
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= cols) return;
    float dg = 0.0f, db = 0.0f;
    for (int64_t row = blockIdx.y; row < rows; row += gridDim.y) {
        const float d = widen(dy[row * cols + c]);
        dg = fmaf(d, (widen(x[row * cols + c]) - mean[row]) * rstd[row], dg);
        db += d;
    }
    float *mine = partial + (int64_t)blockIdx.y * 2 * cols;
    mine[c] = dg;
    mine[cols + c] = db;
}

// dgamma and dbeta from `parts` partial sums [parts][2][cols]: 16 columns a workgroup, whose 64 runs of partial sums are added
// in order, then the runs in pairs.  Either may be null.  512 x 2560: 6.4 us with 32 columns and runs, a load at a time; 4.1 so.
__global__ __launch_bounds__(1024) void layer_norm_reduce_kernel(const float *__restrict__ partial, int parts, int cols,
                                                                 float *__restrict__ dgamma, float *__restrict__ dbeta) {
    constexpr int COLS = 16, RUNS = 1024 / COLS, AT_ONCE = 8;
    __shared__ float runs[RUNS][COLS + 1];
    const int i = threadIdx.x % COLS, run = threadIdx.x / COLS, total = 2 * cols;
    const int at = blockIdx.x * COLS + i;
    const int first = parts * run / RUNS, end = parts * (run + 1) / RUNS;
    float sum = 0.0f;
    if (at < total) {
        for (int k = first; k < end; k += AT_ONCE) {
            float v[AT_ONCE];
#pragma unroll
            for (int j = 0; j < AT_ONCE; ++j) v[j] = k + j < end ? partial[(int64_t)(k + j) * total + at] : 0.0f;
#pragma unroll
            for (int j = 0; j < AT_ONCE; ++j) sum += v[j];
        }
    }
    runs[run][i] = sum;
#pragma unroll
    for (int half = RUNS / 2; half > 0; half >>= 1) {
        __syncthreads();
        if (run < half) runs[run][i] = sum = sum + runs[run + half][i];
    }
    if (run == 0 && at < total) {
        float *out = at < cols ? dgamma : dbeta;
        if (out != nullptr) out[at < cols ? at : at - cols] = sum;
    }
}

constexpr int kLongParts = 256;  // shares of the rows where their sums are a launch of their own, at most

// Workgroups per compute unit that walk the rows: enough loads in flight, few partial sums.
int walkers(int64_t rows, int per_block, int per_cu) {
    const int64_t need = (rows + per_block - 1) / per_block, most = (int64_t)num_compute_units() * per_cu;
    return (int)(need < most ? need : most);
}

// The group and the pieces for rows of `cols` columns, V elements a piece: calls f(integral constants P, LANES), or returns
// false for rows that do not fit.  A lane holds at most 32 elements; eight waves only of whole pieces (the others' columns and
// masks would not fit in its registers).
template <int V, bool WHOLE, class F>
bool with_group(int cols, F f) {
    auto go = [&](auto elements, auto lanes) {
        constexpr int E = decltype(elements)::value, L = decltype(lanes)::value;
        if (cols > L * E) return false;
        f(std::integral_constant<int, E / V>(), lanes);
        return true;
    };
    typedef std::integral_constant<int, 8> E8;
    typedef std::integral_constant<int, 16> E16;
    typedef std::integral_constant<int, 24> E24;
    typedef std::integral_constant<int, 32> E32;
    typedef std::integral_constant<int, 64> Wave;
    typedef std::integral_constant<int, 256> FourWaves;
    typedef std::integral_constant<int, 512> EightWaves;
    if constexpr (V == 1) {
        return go(std::integral_constant<int, 1>(), std::integral_constant<int, 8>());  // shorter than a piece
    } else {
        const bool done = go(E8(), std::integral_constant<int, 8>()) || go(E8(), std::integral_constant<int, 16>()) ||
                          go(E8(), std::integral_constant<int, 32>()) || go(E8(), Wave()) || go(E16(), Wave()) ||
                          go(E24(), Wave()) || go(E32(), Wave()) || go(E16(), FourWaves()) || go(E32(), FourWaves());
        if constexpr (WHOLE) return done || go(E32(), EightWaves());
        return done;
    }
}
int longest_row(bool whole) { return whole ? 16384 : 8192; }  // that fits

// f(pieces of V elements, whether rows are whole pieces)
template <int V, class F>
hipError_t with_pieces(int64_t cols, F f) {
    if (cols % V == 0) return f(std::integral_constant<int, V>(), std::true_type());
    if (cols >= V) return f(std::integral_constant<int, V>(), std::false_type());
    return f(std::integral_constant<int, 1>(), std::true_type());
}

template <class T, int V, bool WHOLE>
hipError_t forward_of(const T *x, const float *gamma, const float *beta, float eps, int64_t rows, int cols, T *y, float *mean,
                      float *rstd, hipStream_t stream) {
    const bool fits = with_group<V, WHOLE>(cols, [&](auto pieces, auto lanes) {
        constexpr int P = decltype(pieces)::value, L = decltype(lanes)::value;
        typedef Group<L> G;
        layer_norm_kernel<T, V, P, L, WHOLE><<<walkers(rows, G::PER_BLOCK, L == 512 ? 4 : 8), G::THREADS, 0, stream>>>(
            x, gamma, beta, eps, rows, cols, y, mean, rstd);
    });
    if (!fits)
        layer_norm_long_kernel<T, V, WHOLE><<<walkers(rows, 1, 2), 1024, 0, stream>>>(x, gamma, beta, eps, rows, cols, y, mean, rstd);
    return hipGetLastError();
}

// Rows that a workgroup works on at a time, of at most 2048 columns.
int rows_per_block(int cols) { return cols > 256 ? 4 : cols > 128 ? 8 : cols > 64 ? 16 : 32; }

// Few rows: the sums over them in the launch of the rows, which are read twice (1200 x 768 bf16: 7.6 us, 9.5 in two launches; 600 x
// 2048 f32 6.5 / 12.2; on the other side 1200 x 4096 f32 22.9 / 22.1, 2500 x 768 bf16 19.7 / 10.8).
bool sums_in_one_launch(int64_t rows, int cols, bool whole) {
    return rows > 0 && rows <= 1024 && rows * cols <= 1 << 22 && cols <= longest_row(whole);
}

// Workgroups of the backward pass, each of which leaves a pair of partial sums: a large part of the traffic where it has few
// rows.  A workgroup a compute unit for rows of several waves (6000 x 8192 bf16: 68.6 us, 78.4 with two; 5000 x 4096 38.4 / 39.5), of
// four rows at least (600 x 16384: 41.2 on 128 workgroups, 47.5 on 256); two for shorter ones unless that leaves a group fewer
// than two rows (32896 x 1280: 50.4, 55.0 with one; 2500 x 2048 f32 27.6 / 21.4).
int backward_blocks(int64_t rows, int cols, bool whole) {
    if (cols > longest_row(whole)) return (int)(rows < kLongParts ? rows : kLongParts);
    if (cols > 2048) {
        const int64_t four = (rows + 3) / 4;
        return (int)(four < num_compute_units() ? four : num_compute_units());
    }
    const int per_block = rows_per_block(cols);
    return walkers(rows, per_block, rows >= (int64_t)4 * per_block * num_compute_units() ? 2 : 1);
}

template <class T, int V, bool WHOLE>
hipError_t backward_of(const T *dy, const T *x, const float *mean, const float *rstd, const float *gamma, int64_t rows, int cols,
                       T *dx, float *dgamma, float *dbeta, float *partial, hipStream_t stream) {
    const bool any = dgamma != nullptr || dbeta != nullptr, one_launch = sums_in_one_launch(rows, cols, WHOLE), sums = any && !one_launch;
    const int blocks = backward_blocks(rows, cols, WHOLE);
    if (rows > 0) {
        const bool fits = with_group<V, WHOLE>(cols, [&](auto pieces, auto lanes) {
            constexpr int P = decltype(pieces)::value, L = decltype(lanes)::value;
            typedef Group<L> G;
            if (sums)
                layer_norm_backward_kernel<T, V, P, L, true, WHOLE><<<blocks, G::THREADS, 0, stream>>>(
                    dy, x, mean, rstd, gamma, rows, cols, dx, partial, 0, nullptr, nullptr);
            else {
                const int row_blocks = walkers(rows, G::PER_BLOCK, 4);
                layer_norm_backward_kernel<T, V, P, L, false, WHOLE><<<row_blocks + (any ? (cols + 15) / 16 : 0), G::THREADS, 0, stream>>>(
                    dy, x, mean, rstd, gamma, rows, cols, dx, nullptr, row_blocks, dgamma, dbeta);
            }
        });
        if (!fits) {
            layer_norm_backward_long_kernel<T, V, WHOLE><<<walkers(rows, 1, 2), 1024, 0, stream>>>(dy, x, mean, rstd, gamma, rows, cols, dx);
            if (sums)
                layer_norm_column_sums_kernel<T><<<dim3((cols + 255) / 256, blocks), 256, 0, stream>>>(dy, x, mean, rstd, rows,
                                                                                                          cols, partial);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (sums)
        layer_norm_reduce_kernel<<<(2 * cols + 15) / 16, 1024, 0, stream>>>(partial, rows > 0 ? blocks : 0, cols, dgamma, dbeta);
    return hipGetLastError();
}

}  // namespace

size_t layer_norm_backward_workspace_bytes(int64_t rows, int64_t cols) {
    if (rows <= 0) return 0;
    // Either type: rows of whole pieces of four elements need not be of whole pieces of eight.
    const int a = sums_in_one_launch(rows, (int)cols, true) ? 0 : backward_blocks(rows, (int)cols, true);
    const int b = cols % 8 == 0 ? 0 : sums_in_one_launch(rows, (int)cols, false) ? 0 : backward_blocks(rows, (int)cols, false);
    return (size_t)(a > b ? a : b) * 2 * (size_t)cols * sizeof(float);
}

hipError_t launch_layer_norm(const void *x, const float *gamma, const float *beta, float eps, int64_t rows, int64_t cols, bool bf16,
                             void *y, float *mean, float *rstd, hipStream_t stream) {
    auto of = [&](auto element, auto v, auto whole) {
        typedef decltype(element) T;
        return forward_of<T, decltype(v)::value, decltype(whole)::value>(static_cast<const T *>(x), gamma, beta, eps, rows, (int)cols,
                                                                         static_cast<T *>(y), mean, rstd, stream);
    };
    if (bf16) return with_pieces<8>(cols, [&](auto v, auto whole) { return of(u16(), v, whole); });
    return with_pieces<4>(cols, [&](auto v, auto whole) { return of(float(), v, whole); });
}

hipError_t launch_layer_norm_backward(const void *dy, const void *x, const float *mean, const float *rstd, const float *gamma,
                                      int64_t rows, int64_t cols, bool bf16, void *dx, float *dgamma, float *dbeta, void *ws,
                                      hipStream_t stream) {
    auto of = [&](auto element, auto v, auto whole) {
        typedef decltype(element) T;
        return backward_of<T, decltype(v)::value, decltype(whole)::value>(static_cast<const T *>(dy), static_cast<const T *>(x), mean, rstd,
                                                                          gamma, rows, (int)cols, static_cast<T *>(dx), dgamma, dbeta,
                                                                          static_cast<float *>(ws), stream);
    };
    if (bf16) return with_pieces<8>(cols, [&](auto v, auto whole) { return of(u16(), v, whole); });
    return with_pieces<4>(cols, [&](auto v, auto whole) { return of(float(), v, whole); });
}

}  // namespace sb
