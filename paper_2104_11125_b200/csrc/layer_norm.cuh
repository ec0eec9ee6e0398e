// Layer norm, forward and backward, with the reduction of gamma's and beta's gradients.
//
// Both passes are bound by HBM: the forward reads and writes a row once, the backward reads two and writes one. A row
// stays in the registers of the threads that loaded it, so the statistics are formed as the definition has them (the mean
// first, then the squares of the differences) from one read.
#pragma once
#include "ops_common.cuh"

namespace sc {

constexpr int LN_THREADS = 256;

// Blocks on a multiprocessor for an estimate of a thread's registers. Where it is short the kernel spills: 24-76 bytes for 16-bit
// forward rows of 257 to 512 elements, 4-60 in several backward forms; a block fewer was not timed.
constexpr int ln_blocks(int regs) { return regs <= 64 ? 4 : regs <= 80 ? 3 : regs <= 128 ? 2 : 1; }

struct LnParams {
    const void *x, *dy;
    void *y, *dx;
    const float *gamma, *beta;
    const float *mean_in, *rstd_in;
    float *mean, *rstd;
    float* partial;                  // backward: [blocks][2][width]
    float *dgamma, *dbeta;
    int64_t ldx, ldy, lddy, lddx;
    int64_t rows;
    int32_t width, nblocks;
    float eps;
};

// Count, mean and sum of squared differences of a set of values; two sets joined (Chan, Golub and LeVeque's pairwise form).
struct LnMoments { float n, mean, m2; };
__device__ __forceinline__ LnMoments ln_merge(const LnMoments& a, const LnMoments& b) {
    const float n = a.n + b.n;
    if (n == 0.0f) return a;
    const float d = b.mean - a.mean, f = b.n / n;
    LnMoments r;
    r.n = n;
    r.mean = a.mean + d * f;
    r.m2 = a.m2 + b.m2 + d * d * a.n * f;
    return r;
}

// Mean and squared differences over the TPR threads of a row (32: a warp, LN_THREADS: the block) from those of each thread's N
// values: pairs of sets of one size, so the pairwise form has constants only. Either partner of a join computes the same sums of the same
// two terms, so every thread of the row gets the same bits. `part` has two arrays used in turn, so that one barrier a row is enough.
template <int TPR, int N>
__device__ __forceinline__ void row_moments(float& mean, float& m2, float2 (*part)[LN_THREADS / 32], int turn) {
    static_assert(TPR == 32 || TPR == 256, "levels");
    auto join = [&](int o, float size) {
        const float other = __shfl_xor_sync(FULL, mean, o), d = other - mean;
        mean = 0.5f * (mean + other);
        const float both = m2 + __shfl_xor_sync(FULL, m2, o);
        m2 = both + d * d * (0.5f * size);
    };
#pragma unroll
    for (int l = 0; l < 5; ++l) join(1 << l, float(N << l));
    if (TPR > 32) {
        if (lane_id() == 0) part[turn][warp_id()] = make_float2(mean, m2);
        __syncthreads();
        const float2 t = part[turn][lane_id() & 7];
        mean = t.x;
        m2 = t.y;
#pragma unroll
        for (int l = 0; l < 3; ++l) join(1 << l, float(N << (5 + l)));
    }
}
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* part) {
    v = warp_sum_f(v);
    if (TPR > 32) {
        if (lane_id() == 0) part[warp_id()] = v;
        __syncthreads();
        v = part[lane_id() & (TPR / 32 - 1)];
#pragma unroll
        for (int o = TPR / 64; o; o >>= 1) v += __shfl_xor_sync(FULL, v, o);
    }
    return v;
}
template <int TPR>
__device__ __forceinline__ float2 row_sum2(float a, float b, float2 (*part)[LN_THREADS / 32], int turn) {
    a = warp_sum_f(a);
    b = warp_sum_f(b);
    if (TPR > 32) {
        if (lane_id() == 0) part[turn][warp_id()] = make_float2(a, b);
        __syncthreads();
        const float2 t = part[turn][lane_id() & (TPR / 32 - 1)];
        a = t.x;
        b = t.y;
#pragma unroll
        for (int o = TPR / 64; o; o >>= 1) {
            a += __shfl_xor_sync(FULL, a, o);
            b += __shfl_xor_sync(FULL, b, o);
        }
    }
    return make_float2(a, b);
}

// A thread's columns of a row as they lie in memory, loaded ahead of their use.
template <typename T, int VEC, int NV> struct LnRow { Pack<T, VEC> p[NV]; };
// MOST: the row reaches into the last of the thread's NV places, so only that one is compared with the width (a limit
// no column reaches stands for the others, and the comparisons are dropped).
constexpr int LN_NO_LIMIT = 1 << 30;
template <typename T, int VEC, int NV, int TPR, bool MOST>
__device__ __forceinline__ void ln_fetch(const T* row, int t, int row_width, LnRow<T, VEC, NV>& r) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int col = (i * TPR + t) * VEC, width = MOST && i + 1 < NV ? LN_NO_LIMIT : row_width;
        if (col + VEC <= width) {
            r.p[i] = *reinterpret_cast<const Pack<T, VEC>*>(row + col);
        } else {
            uint32_t b[VEC];
#pragma unroll
            for (int j = 0; j < VEC; ++j) b[j] = col + j < width ? bits_of<T>(Elem<T>::up(row[col + j])) : 0u;
            if constexpr (sizeof(T) == 4 || VEC == 1) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) set_word(r.p[i], j, b[j]);
            } else {
#pragma unroll
                for (int j = 0; j < VEC; j += 2) set_word(r.p[i], j / 2, b[j] | (b[j + 1] << 16));
            }
        }
    }
}
// a thread's columns of a vector of `width` parameters
template <int VEC, int NV, int TPR>
__device__ __forceinline__ void ln_params(const float* p, float other, int t, int width, float (&v)[NV][VEC]) {
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const int c = (i * TPR + t) * VEC + j;
            v[i][j] = p && c < width ? __ldg(p + c) : other;
        }
}

template <typename T, int VEC>
__device__ __forceinline__ void ln_store(T* p, int col, int width, const float (&v)[VEC]) {
    if (VEC == 1 || col + VEC <= width) {
        if (VEC > 1 || col < width) store_down<T, VEC>(p + col, v);
    } else {
#pragma unroll
        for (int j = 0; j < VEC; ++j)
            if (col + j < width) p[col + j] = Elem<T>::down(v[j]);
    }
}

// The sum of N values (a power of two) by pairs: for equal values every partial sum is a power of two times the value, so it is exact.
template <int N> __device__ __forceinline__ float pair_sum(const float* v) {
    if constexpr (N == 1) return v[0];
    else return pair_sum<N / 2>(v) + pair_sum<N / 2>(v + N / 2);
}

// A row of equal values has to have that value as its mean, to the bit: rstd is then 1 / sqrt(eps), 316 at the usual 1e-5, and makes a unit in
// the last place of 1000 into 0.02. Where the row fills the threads every sum on the way is exact for such a row. Elsewhere the sum
// times the rounded 1 / width is a few units off (for 7 or 13 columns, say), and the mean of what is left corrects it: of
// equal values these are the same few units, so the correction is exact after the addition's rounding. The sum of 16-bit values is exact for
// such a row (13 bits of a count times 11 of a value) and what is left follows from it, sum - width mean, once a row; fp32 sums are
// rounded, so what is left is summed over the row beside the squares. It costs 0 to 1 % at HBM-bound sizes
// (30011 x 2047 bf16 64.1 to 64.6 us, fp32 82.5 to 83.5) and most for short fp32 rows in L2 (60000 x 101: 11.0 to 12.8).
//
// gamma and beta stay in registers over a thread's rows, and two more rows are on their way while this one is reduced.
// WHOLE: the row fills the threads' columns exactly; its moments take one barrier and no comparisons of columns with the width.
// The 16384 x 4096 bf16 case is as close to the issue rate as to HBM: with values converted three times, comparisons and
// quotients in the joins it took 128 us.
template <typename T, int VEC, int NV, int TPR, bool WHOLE, bool MOST>
__global__ void __launch_bounds__(LN_THREADS, ln_blocks(3 * NV * VEC + 2 * NV * VEC * int(sizeof(T)) / 4 + 16)) layer_norm_kernel(const LnParams P) {
    __shared__ float2 part[2][LN_THREADS / 32];
    constexpr int RPB = LN_THREADS / TPR;
    const int t = threadIdx.x % TPR;
    const int64_t step = int64_t(gridDim.x) * RPB;
    int64_t row = int64_t(blockIdx.x) * RPB + threadIdx.x / TPR;
    const float inv = 1.0f / float(P.width);
    const int width = WHOLE ? NV * TPR * VEC : P.width;
    chain_launch();
    chain_wait();
    LnRow<T, VEC, NV> next, after;
    auto fetch = [&](int64_t r, LnRow<T, VEC, NV>& to) {
        if (r < P.rows) ln_fetch<T, VEC, NV, TPR, MOST>(static_cast<const T*>(P.x) + r * P.ldx, t, width, to);
    };
    fetch(row, next);
    fetch(row + step, after);
    float gamma[NV][VEC], beta[NV][VEC];
    ln_params<VEC, NV, TPR>(P.gamma, 1.0f, t, width, gamma);
    ln_params<VEC, NV, TPR>(P.beta, 0.0f, t, width, beta);
    for (int turn = 0; row < P.rows; row += step, turn ^= 1) {
        float v[NV][VEC], mean = 0.0f, m2 = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                v[i][j] = pack_get<T, VEC>(next.p[i], j);          // 0 beyond the row
                if (!WHOLE) mean += v[i][j];
            }
        next = after;
        fetch(row + 2 * step, after);
        if (WHOLE) {
            mean = pair_sum<NV * VEC>(&v[0][0]) * (1.0f / float(NV * VEC));
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < VEC; ++j) m2 += (v[i][j] - mean) * (v[i][j] - mean);
            row_moments<TPR, NV * VEC>(mean, m2, part, turn);
        } else {
            const float sum = row_sum<TPR>(mean, &part[0][0].x);
            mean = sum * inv;
            auto correct = [&](float left) {                       // an infinity in the row stays its mean
                const float off = left * inv;
                if (fabsf(off) < INFINITY) mean += off;
                return off;
            };
            if (sizeof(T) == 2) correct(fmaf(-mean, float(width), sum));
            float left = 0.0f;
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const float d = (MOST && i + 1 < NV) || (i * TPR + t) * VEC + j < width ? v[i][j] - mean : 0.0f;
                    m2 += d * d;
                    if (sizeof(T) == 4) left += d;
                }
            if (sizeof(T) == 4) {
                const float2 s = row_sum2<TPR>(left, m2, part, 1);
                m2 = s.y - s.x * correct(s.x);
                if (m2 < 0.0f) m2 = 0.0f;                          // a NaN stays
            } else {
                m2 = row_sum<TPR>(m2, &part[1][0].x);
            }
        }
        const float rstd = rsqrtf(m2 * inv + P.eps);
        T* y = static_cast<T*>(P.y) + row * P.ldy;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int col = (i * TPR + t) * VEC, limit = MOST && i + 1 < NV ? LN_NO_LIMIT : width;
            if (col < limit) {
                float o[VEC];
#pragma unroll
                for (int j = 0; j < VEC; ++j) o[j] = (v[i][j] - mean) * rstd * gamma[i][j] + beta[i][j];
                ln_store<T, VEC>(y, col, limit, o);
            }
        }
        if (t == 0) {
            if (P.mean) P.mean[row] = mean;
            if (P.rstd) P.rstd[row] = rstd;
        }
    }
}

// Rows too long for registers: one pass forms mean and squared differences with Welford's update, the threads' triples
// are merged pairwise, a second pass (of a row that is then in L2) writes y.
template <typename T>
__global__ void __launch_bounds__(LN_THREADS) layer_norm_wide_kernel(const LnParams P) {
    __shared__ LnMoments part[LN_THREADS / 32];
    chain_launch();
    chain_wait();
    for (int64_t row = blockIdx.x; row < P.rows; row += gridDim.x) {
        const T* x = static_cast<const T*>(P.x) + row * P.ldx;
        LnMoments m = {0.0f, 0.0f, 0.0f};
        for (int c = threadIdx.x; c < P.width; c += LN_THREADS) {
            const float v = Elem<T>::up(x[c]);
            m.n += 1.0f;
            const float d = v - m.mean;
            m.mean += d / m.n;
            m.m2 += d * (v - m.mean);
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) {
            LnMoments b = {__shfl_down_sync(FULL, m.n, o), __shfl_down_sync(FULL, m.mean, o), __shfl_down_sync(FULL, m.m2, o)};
            m = ln_merge(m, b);
        }
        __syncthreads();
        if (lane_id() == 0) part[warp_id()] = m;
        __syncthreads();
        m = part[0];
        for (int w = 1; w < LN_THREADS / 32; ++w) m = ln_merge(m, part[w]);
        const float mean = m.mean, rstd = rsqrtf(m.m2 / float(P.width) + P.eps);
        T* y = static_cast<T*>(P.y) + row * P.ldy;
        for (int c = threadIdx.x; c < P.width; c += LN_THREADS) {
            const float g = P.gamma ? P.gamma[c] : 1.0f, b = P.beta ? P.beta[c] : 0.0f;
            y[c] = Elem<T>::down((Elem<T>::up(x[c]) - mean) * rstd * g + b);
        }
        if (threadIdx.x == 0) {
            if (P.mean) P.mean[row] = mean;
            if (P.rstd) P.rstd[row] = rstd;
        }
    }
}

// Backward. A block walks over rows with a fixed assignment of columns to threads, so each thread keeps its columns' sums for
// dgamma and dbeta in registers; the blocks' sums go to scratch and a second kernel adds them in block order.
template <typename T, int VEC, int NV, int TPR, bool DW, bool MOST>
__global__ void __launch_bounds__(LN_THREADS, ln_blocks(5 * NV * VEC + (NV * VEC <= 16 ? 4 : 2) * NV * VEC * int(sizeof(T)) / 4 + 24)) layer_norm_backward_kernel(const LnParams P) {
    __shared__ float2 part[2][LN_THREADS / 32];
    extern __shared__ float cols[];                       // TPR = 32: [warps][2][width], to join the warps' sums
    constexpr int RPB = LN_THREADS / TPR;
    constexpr bool AHEAD = NV * VEC <= 16;                // room for the next row in registers
    const int t = threadIdx.x % TPR;
    const int64_t step = int64_t(gridDim.x) * RPB;
    int64_t row = int64_t(blockIdx.x) * RPB + threadIdx.x / TPR;
    const float inv = 1.0f / float(P.width);
    float dg[NV][VEC], db[NV][VEC], gamma[NV][VEC];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) dg[i][j] = db[i][j] = 0.0f;
    chain_launch();
    chain_wait();
    if (AHEAD) ln_params<VEC, NV, TPR>(P.gamma, 1.0f, t, P.width, gamma);
    LnRow<T, VEC, NV> x, dy, x2, dy2;
    float mean = 0.0f, rstd = 0.0f, mean2 = 0.0f, rstd2 = 0.0f;
    auto fetch = [&](int64_t r, LnRow<T, VEC, NV>& a, LnRow<T, VEC, NV>& b, float& mu, float& rs) {
        if (r < P.rows) {
            ln_fetch<T, VEC, NV, TPR, MOST>(static_cast<const T*>(P.x) + r * P.ldx, t, P.width, a);
            ln_fetch<T, VEC, NV, TPR, MOST>(static_cast<const T*>(P.dy) + r * P.lddy, t, P.width, b);
            mu = P.mean_in[r];
            rs = P.rstd_in[r];
        }
    };
    if (AHEAD) fetch(row, x, dy, mean, rstd);
    for (int turn = 0; row < P.rows; row += step, turn ^= 1) {
        if (AHEAD) fetch(row + step, x2, dy2, mean2, rstd2);
        else fetch(row, x, dy, mean, rstd);
        if (!AHEAD) ln_params<VEC, NV, TPR>(P.gamma, 1.0f, t, P.width, gamma);
        float xh[NV][VEC], w[NV][VEC];
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const bool in = VEC == 1 || (MOST && i + 1 < NV) || (i * TPR + t) * VEC + j < P.width;
                xh[i][j] = in ? (pack_get<T, VEC>(x.p[i], j) - mean) * rstd : 0.0f;
                w[i][j] = pack_get<T, VEC>(dy.p[i], j);      // 0 beyond the row
                if (DW) {
                    dg[i][j] += w[i][j] * xh[i][j];
                    db[i][j] += w[i][j];
                }
                w[i][j] *= gamma[i][j];
                s1 += w[i][j];
                s2 += w[i][j] * xh[i][j];
            }
        if (P.dx) {
            const float2 s = row_sum2<TPR>(s1, s2, part, turn);
            const float m1 = s.x * inv, m2 = s.y * inv;
            T* dx = static_cast<T*>(P.dx) + row * P.lddx;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int col = (i * TPR + t) * VEC, width = MOST && i + 1 < NV ? LN_NO_LIMIT : P.width;
                if (col < width) {
                    float o[VEC];
#pragma unroll
                    for (int j = 0; j < VEC; ++j) o[j] = rstd * (w[i][j] - m1 - xh[i][j] * m2);
                    ln_store<T, VEC>(dx, col, width, o);
                }
            }
        }
        if (AHEAD) { x = x2; dy = dy2; mean = mean2; rstd = rstd2; }
    }
    if (DW) {
        float* out = P.partial + int64_t(blockIdx.x) * 2 * P.width;
        float* to = TPR == 32 ? cols + warp_id() * 2 * P.width : out;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const int c = (i * TPR + t) * VEC + j;
                if (c < P.width) {
                    to[c] = dg[i][j];
                    to[P.width + c] = db[i][j];
                }
            }
        if (TPR == 32) {                                  // the warps' sums, in their order
            __syncthreads();
            for (int c = threadIdx.x; c < 2 * P.width; c += LN_THREADS) {
                float s = cols[c];
#pragma unroll
                for (int wp = 1; wp < RPB; ++wp) s += cols[wp * 2 * P.width + c];
                out[c] = s;
            }
        }
    }
}

// Rows too long for registers: dx by two passes over the row, the columns' sums by a kernel of their own.
template <typename T>
__global__ void __launch_bounds__(LN_THREADS) layer_norm_backward_wide_kernel(const LnParams P) {
    __shared__ float2 part[2][LN_THREADS / 32];
    chain_launch();
    chain_wait();
    int turn = 0;
    for (int64_t row = blockIdx.x; row < P.rows; row += gridDim.x, turn ^= 1) {
        const T* x = static_cast<const T*>(P.x) + row * P.ldx;
        const T* dy = static_cast<const T*>(P.dy) + row * P.lddy;
        const float mean = P.mean_in[row], rstd = P.rstd_in[row];
        float s1 = 0.0f, s2 = 0.0f;
        for (int c = threadIdx.x; c < P.width; c += LN_THREADS) {
            const float w = Elem<T>::up(dy[c]) * (P.gamma ? P.gamma[c] : 1.0f);
            s1 += w;
            s2 += w * ((Elem<T>::up(x[c]) - mean) * rstd);
        }
        const float2 s = row_sum2<LN_THREADS>(s1, s2, part, turn);
        const float m1 = s.x / float(P.width), m2 = s.y / float(P.width);
        T* dx = static_cast<T*>(P.dx) + row * P.lddx;
        for (int c = threadIdx.x; c < P.width; c += LN_THREADS) {
            const float w = Elem<T>::up(dy[c]) * (P.gamma ? P.gamma[c] : 1.0f);
            dx[c] = Elem<T>::down(rstd * (w - m1 - (Elem<T>::up(x[c]) - mean) * rstd * m2));
        }
    }
}
// partial sums of 256 columns over the rows y, y + gridDim.y, ...
template <typename T>
__global__ void __launch_bounds__(LN_THREADS) layer_norm_columns_kernel(const LnParams P) {
    chain_launch();
    chain_wait();
    const int c = blockIdx.x * LN_THREADS + threadIdx.x;
    if (c >= P.width) return;
    float dg = 0.0f, db = 0.0f;
    for (int64_t row = blockIdx.y; row < P.rows; row += gridDim.y) {
        const float d = Elem<T>::up(static_cast<const T*>(P.dy)[row * P.lddy + c]);
        dg += d * ((Elem<T>::up(static_cast<const T*>(P.x)[row * P.ldx + c]) - P.mean_in[row]) * P.rstd_in[row]);
        db += d;
    }
    float* out = P.partial + int64_t(blockIdx.y) * 2 * P.width;
    out[c] = dg;
    out[P.width + c] = db;
}

// dgamma and dbeta from the blocks' sums: 32 columns a block, eight groups of rows, joined in a fixed order
__global__ void __launch_bounds__(LN_THREADS) layer_norm_reduce_kernel(const LnParams P) {
    __shared__ float part[LN_THREADS / 32][32];
    chain_launch();
    chain_wait();
    const int c = blockIdx.x * 32 + lane_id();            // over [2][width]
    float s = 0.0f;
    if (c < 2 * P.width)
        for (int b = warp_id(); b < P.nblocks; b += LN_THREADS / 32) s += P.partial[int64_t(b) * 2 * P.width + c];
    part[warp_id()][lane_id()] = s;
    __syncthreads();
    if (warp_id() == 0 && c < 2 * P.width) {
        s = 0.0f;
#pragma unroll
        for (int w = 0; w < LN_THREADS / 32; ++w) s += part[w][lane_id()];
        if (c < P.width) { if (P.dgamma) P.dgamma[c] = s; }
        else if (P.dbeta) P.dbeta[c - P.width] = s;
    }
}

}  // namespace sc
