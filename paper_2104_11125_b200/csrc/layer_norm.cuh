// Layer norm, forward and backward, with the reduction of gamma's and beta's gradients.
//
// Both passes are bound by HBM: the forward reads and writes a row once, the backward reads two and writes one. A row
// stays in the registers of the threads that loaded it, so the statistics are formed as the definition has them (the mean
// first, then the squares of the differences) from one read.
#pragma once
#include "ops_common.cuh"

namespace sc {

constexpr int LN_THREADS = 256;

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

// sum over the TPR threads that share a row; TPR = 32: a warp, TPR = LN_THREADS: the block
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* smem) {
    v = warp_sum_f(v);
    if (TPR > 32) {
        __syncthreads();                                 // the array may still be read from the sum before
        if (lane_id() == 0) smem[warp_id()] = v;
        __syncthreads();
        v = smem[lane_id() & (TPR / 32 - 1)];
#pragma unroll
        for (int o = TPR / 64; o; o >>= 1) v += __shfl_xor_sync(FULL, v, o);
    }
    return v;
}
template <int TPR>
__device__ __forceinline__ float2 row_sum2(float a, float b, float2* smem) {
    a = warp_sum_f(a);
    b = warp_sum_f(b);
    if (TPR > 32) {
        __syncthreads();
        if (lane_id() == 0) smem[warp_id()] = make_float2(a, b);
        __syncthreads();
        const float2 t = smem[lane_id() & (TPR / 32 - 1)];
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

template <typename T, int VEC>
__device__ __forceinline__ void ln_load(const T* p, int col, int width, float (&v)[VEC]) {
    if (VEC == 1 || col + VEC <= width) {
        if (VEC > 1 || col < width) load_up<T, VEC>(p + col, v);
        else v[0] = 0.0f;
    } else {
#pragma unroll
        for (int j = 0; j < VEC; ++j) v[j] = col + j < width ? Elem<T>::up(p[col + j]) : 0.0f;
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

template <typename T, int VEC, int NV, int TPR>
__global__ void __launch_bounds__(LN_THREADS) layer_norm_kernel(const LnParams P) {
    __shared__ float red[LN_THREADS / 32];
    constexpr int RPB = LN_THREADS / TPR;
    const int t = threadIdx.x % TPR;
    const float inv = 1.0f / float(P.width);
    chain_launch();
    chain_wait();
    for (int64_t row = int64_t(blockIdx.x) * RPB + threadIdx.x / TPR; row < P.rows; row += int64_t(gridDim.x) * RPB) {
        const T* x = static_cast<const T*>(P.x) + row * P.ldx;
        float v[NV][VEC];
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) ln_load<T, VEC>(x, (i * TPR + t) * VEC, P.width, v[i]);
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < VEC; ++j) s += v[i][j];
        const float mean = row_sum<TPR>(s, red) * inv;
        s = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                v[i][j] -= mean;
                if ((i * TPR + t) * VEC + j < P.width) s += v[i][j] * v[i][j];
            }
        const float rstd = 1.0f / sqrtf(row_sum<TPR>(s, red) * inv + P.eps);
        T* y = static_cast<T*>(P.y) + row * P.ldy;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int col = (i * TPR + t) * VEC;
            if (col < P.width) {
                float o[VEC];
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const int c = min(col + j, P.width - 1);
                    const float g = P.gamma ? __ldg(P.gamma + c) : 1.0f, b = P.beta ? __ldg(P.beta + c) : 0.0f;
                    o[j] = v[i][j] * rstd * g + b;
                }
                ln_store<T, VEC>(y, col, P.width, o);
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
        const float mean = m.mean, rstd = 1.0f / sqrtf(m.m2 / float(P.width) + P.eps);
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
template <typename T, int VEC, int NV, int TPR, bool DW>
__global__ void __launch_bounds__(LN_THREADS) layer_norm_backward_kernel(const LnParams P) {
    __shared__ float2 red[LN_THREADS / 32];
    extern __shared__ float cols[];                       // TPR = 32: [2][width], to join the warps' sums
    constexpr int RPB = LN_THREADS / TPR;
    const int t = threadIdx.x % TPR;
    const float inv = 1.0f / float(P.width);
    float dg[NV][VEC], db[NV][VEC];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) dg[i][j] = db[i][j] = 0.0f;
    chain_launch();
    chain_wait();
    for (int64_t row = int64_t(blockIdx.x) * RPB + threadIdx.x / TPR; row < P.rows; row += int64_t(gridDim.x) * RPB) {
        const T* x = static_cast<const T*>(P.x) + row * P.ldx;
        const T* dy = static_cast<const T*>(P.dy) + row * P.lddy;
        float xh[NV][VEC], w[NV][VEC];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            ln_load<T, VEC>(x, (i * TPR + t) * VEC, P.width, xh[i]);
            ln_load<T, VEC>(dy, (i * TPR + t) * VEC, P.width, w[i]);
        }
        const float mean = P.mean_in[row], rstd = P.rstd_in[row];
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const int c = (i * TPR + t) * VEC + j;
                const bool in = c < P.width;
                xh[i][j] = in ? (xh[i][j] - mean) * rstd : 0.0f;
                if (DW) {
                    dg[i][j] += w[i][j] * xh[i][j];
                    db[i][j] += w[i][j];
                }
                if (P.gamma) w[i][j] *= in ? __ldg(P.gamma + c) : 0.0f;
                s1 += w[i][j];
                s2 += w[i][j] * xh[i][j];
            }
        if (P.dx) {
            const float2 s = row_sum2<TPR>(s1, s2, red);
            const float m1 = s.x * inv, m2 = s.y * inv;
            T* dx = static_cast<T*>(P.dx) + row * P.lddx;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int col = (i * TPR + t) * VEC;
                if (col < P.width) {
                    float o[VEC];
#pragma unroll
                    for (int j = 0; j < VEC; ++j) o[j] = rstd * (w[i][j] - m1 - xh[i][j] * m2);
                    ln_store<T, VEC>(dx, col, P.width, o);
                }
            }
        }
    }
    if (DW) {
        float* out = P.partial + int64_t(blockIdx.x) * 2 * P.width;
        if (TPR == 32) {                                  // the warps in turn: a fixed order of additions
            for (int wp = 0; wp < RPB; ++wp) {
                if (int(warp_id()) == wp) {
#pragma unroll
                    for (int i = 0; i < NV; ++i)
#pragma unroll
                        for (int j = 0; j < VEC; ++j) {
                            const int c = (i * TPR + t) * VEC + j;
                            if (c < P.width) {
                                cols[c] = (wp ? cols[c] : 0.0f) + dg[i][j];
                                cols[P.width + c] = (wp ? cols[P.width + c] : 0.0f) + db[i][j];
                            }
                        }
                }
                __syncthreads();
            }
            for (int c = threadIdx.x; c < 2 * P.width; c += LN_THREADS) out[c] = cols[c];
        } else {
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const int c = (i * TPR + t) * VEC + j;
                    if (c < P.width) {
                        out[c] = dg[i][j];
                        out[P.width + c] = db[i][j];
                    }
                }
        }
    }
}

// Rows too long for registers: dx by two passes over the row, the columns' sums by a kernel of their own.
template <typename T>
__global__ void __launch_bounds__(LN_THREADS) layer_norm_backward_wide_kernel(const LnParams P) {
    __shared__ float2 red[LN_THREADS / 32];
    chain_launch();
    chain_wait();
    for (int64_t row = blockIdx.x; row < P.rows; row += gridDim.x) {
        const T* x = static_cast<const T*>(P.x) + row * P.ldx;
        const T* dy = static_cast<const T*>(P.dy) + row * P.lddy;
        const float mean = P.mean_in[row], rstd = P.rstd_in[row];
        float s1 = 0.0f, s2 = 0.0f;
        for (int c = threadIdx.x; c < P.width; c += LN_THREADS) {
            const float w = Elem<T>::up(dy[c]) * (P.gamma ? P.gamma[c] : 1.0f);
            s1 += w;
            s2 += w * ((Elem<T>::up(x[c]) - mean) * rstd);
        }
        const float2 s = row_sum2<LN_THREADS>(s1, s2, red);
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
