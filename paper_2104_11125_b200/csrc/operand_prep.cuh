// What has to happen to an operand before the tensor cores can read it: fp32 values become two fp16 planes, 16-bit matrices
// whose rows do not start on 16-byte boundaries are laid out anew, updates are normalised.
#pragma once
#include "ops_common.cuh"

namespace sc {

constexpr int PREP_THREADS = 256;
constexpr int PREP_MAX = 6;

// One source matrix [rows][cols]; every kernel here takes a table of them, blockIdx.y picks one.
struct PrepItem {
    const void* src;
    int64_t ld;                 // elements
    int64_t rows, cols;
    void* dst;                  // [rows][dst_ld]
    int64_t dst_ld;
    int64_t lo;                 // fp32 sources: distance of the lo plane
    uint32_t* amax;             // fp32 sources: largest finite magnitude (bits)
};
struct PrepTable {
    PrepItem item[PREP_MAX];
    int type;                   // of the sources
};

// A block covers `ty` rows x all columns at a time, `tx` threads along a row, eight columns each.
__device__ __forceinline__ int prep_tx(int64_t groups) {
    int tx = PREP_THREADS;
    while (tx > 1 && tx / 2 >= groups) tx /= 2;
    return tx;
}

template <typename T>
__device__ __forceinline__ void prep_load8(const T* p, int64_t left, float (&v)[8], bool inside) {
    constexpr int N = 16 / sizeof(T) > 8 ? 8 : 16 / sizeof(T);
    if (left >= 8 && (reinterpret_cast<uintptr_t>(p) & 15u) == 0) {
#pragma unroll
        for (int i = 0; i < 8; i += N) {
            float t[N];
            load_up<T, N>(p + i, t);
#pragma unroll
            for (int j = 0; j < N; ++j) v[i + j] = t[j];
        }
    } else if (sizeof(T) == 2 && left > 8 && inside) {
        // off the grid, with neighbours of the same row on both sides: whole words, shifted by an element where they have to be
        const uint32_t* w = reinterpret_cast<const uint32_t*>(reinterpret_cast<uintptr_t>(p) & ~uintptr_t(3));
        const bool odd = (reinterpret_cast<uintptr_t>(p) & 2u) != 0;
        uint32_t q[5];
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = w[i];
        q[4] = odd ? w[4] : 0u;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t t = odd ? __funnelshift_r(q[i], q[i + 1], 16) : q[i];
            v[2 * i] = pack_get<T, 16 / sizeof(T)>(make_uint4(t, t, t, t), 0);
            v[2 * i + 1] = pack_get<T, 16 / sizeof(T)>(make_uint4(t, t, t, t), 1);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < left ? Elem<T>::up(p[i]) : 0.0f;
    }
}
__device__ __forceinline__ void prep_load8_typed(int type, const void* base, int64_t off, int64_t left, float (&v)[8], bool inside) {
    if (type == SCALECOM_F32) prep_load8(static_cast<const float*>(base) + off, left, v, inside);
    else if (type == SCALECOM_F16) prep_load8(static_cast<const __half*>(base) + off, left, v, inside);
    else prep_load8(static_cast<const __nv_bfloat16*>(base) + off, left, v, inside);
}
template <typename T>
__device__ __forceinline__ void prep_store8(T* p, int64_t left, const float (&v)[8]) {
    constexpr int N = 16 / sizeof(T) > 8 ? 8 : 16 / sizeof(T);
    if (left >= 8 && (reinterpret_cast<uintptr_t>(p) & 15u) == 0) {
#pragma unroll
        for (int i = 0; i < 8; i += N) {
            float t[N];
#pragma unroll
            for (int j = 0; j < N; ++j) t[j] = v[i + j];
            store_down<T, N>(p + i, t);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) p[i] = Elem<T>::down(v[i]);
    }
}

__global__ void __launch_bounds__(PREP_THREADS) prep_amax_kernel(const __grid_constant__ PrepTable T) {
    chain_launch();
    chain_wait();
    const PrepItem& I = T.item[blockIdx.y];
    const int64_t groups = (I.cols + 7) / 8;
    const int tx = prep_tx(groups), ty = PREP_THREADS / tx;
    __shared__ uint32_t block_top;
    if (threadIdx.x == 0) block_top = 0u;
    __syncthreads();
    uint32_t top = 0u;
    for (int64_t r = int64_t(blockIdx.x) * ty + threadIdx.x / tx; r < I.rows; r += int64_t(gridDim.x) * ty)
        for (int64_t g = threadIdx.x % tx; g < groups; g += tx) {
            float v[8];
            prep_load8(static_cast<const float*>(I.src) + r * I.ld + g * 8, I.cols - g * 8, v, g > 0);
#pragma unroll
            for (int i = 0; i < 8; ++i) top = max(top, finite_bits(v[i]));
        }
    top = __reduce_max_sync(FULL, top);
    if (lane_id() == 0) atomicMax(&block_top, top);
    __syncthreads();
    // a maximum: the order does not matter. One word takes an atomic a nanosecond, so only those that raise it are sent.
    if (threadIdx.x == 0 && block_top > ld_relaxed_u32(I.amax)) atomicMax(I.amax, block_top);
}

__global__ void __launch_bounds__(PREP_THREADS) prep_operand_kernel(const __grid_constant__ PrepTable T) {
    chain_launch();
    chain_wait();
    const PrepItem& I = T.item[blockIdx.y];
    const int64_t groups = (I.cols + 7) / 8;
    const int tx = prep_tx(groups), ty = PREP_THREADS / tx;
    const bool planes = T.type == SCALECOM_F32;
    const float scale = planes ? plane_scale(*I.amax) : 1.0f;
    for (int64_t r = int64_t(blockIdx.x) * ty + threadIdx.x / tx; r < I.rows; r += int64_t(gridDim.x) * ty)
        for (int64_t g = threadIdx.x % tx; g < groups; g += tx) {
            float v[8];
            const int64_t left = I.cols - g * 8, at = r * I.dst_ld + g * 8;
            prep_load8_typed(T.type, I.src, r * I.ld + g * 8, left, v, g > 0);
            if (planes) {
                float l[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    __half h, lo;
                    v[i] *= scale;
                    split_planes(v[i], h, lo);
                    l[i] = __half2float(lo);
                }
                prep_store8(static_cast<__half*>(I.dst) + at, left, v);
                prep_store8(static_cast<__half*>(I.dst) + I.lo + at, left, l);
            } else if (T.type == SCALECOM_F16) {
                prep_store8(static_cast<__half*>(I.dst) + at, left, v);
            } else {
                prep_store8(static_cast<__nv_bfloat16*>(I.dst) + at, left, v);
            }
        }
}

// ---- normalisation of the updates ------------------------------------------------------------------------
struct NormParams {
    const void* in;
    int64_t ld, stride;
    int64_t rows, cols;
    int in_type;
    double* partial;            // [batch][gridDim.x]
    int32_t nparts;
    float eps;
    double factor;              // applied after the division by the norm
    __half* planes;             // [batch][1 or 2][rows][planes_ld], or NULL
    int64_t planes_ld, planes_lo, planes_stride;
    void* out;                  // or a typed result
    int out_type;
    int64_t ld_out, out_stride;
};

// Squares in fp64: neither 1e-30 nor 1e30 leaves its range, and the sum of 2^26 squares keeps fp32's accuracy.
__global__ void __launch_bounds__(PREP_THREADS) norm_partial_kernel(const __grid_constant__ NormParams P) {
    __shared__ double red[PREP_THREADS / 32];
    chain_launch();
    chain_wait();
    const int64_t groups = (P.cols + 7) / 8;
    const int tx = prep_tx(groups), ty = PREP_THREADS / tx;
    double s = 0.0;
    for (int64_t r = int64_t(blockIdx.x) * ty + threadIdx.x / tx; r < P.rows; r += int64_t(gridDim.x) * ty)
        for (int64_t g = threadIdx.x % tx; g < groups; g += tx) {
            float v[8];
            prep_load8_typed(P.in_type, P.in, blockIdx.y * P.stride + r * P.ld + g * 8, P.cols - g * 8, v, g > 0);
#pragma unroll
            for (int i = 0; i < 8; ++i) s += double(v[i]) * double(v[i]);
        }
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(FULL, s, o);
    if (lane_id() == 0) red[warp_id()] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        s = 0.0;
        for (int w = 0; w < PREP_THREADS / 32; ++w) s += red[w];
        P.partial[int64_t(blockIdx.y) * P.nparts + blockIdx.x] = s;
    }
}

__global__ void __launch_bounds__(PREP_THREADS) norm_apply_kernel(const __grid_constant__ NormParams P) {
    __shared__ double total;
    chain_launch();
    chain_wait();
    if (threadIdx.x < 32) {
        double s = 0.0;
        for (int i = threadIdx.x; i < P.nparts; i += 32) s += P.partial[int64_t(blockIdx.y) * P.nparts + i];
#pragma unroll
        for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(FULL, s, o);
        if (threadIdx.x == 0) total = s;
    }
    __syncthreads();
    const double f = P.factor / (sqrt(total) + double(P.eps));
    const int64_t groups = (P.cols + 7) / 8;
    const int tx = prep_tx(groups), ty = PREP_THREADS / tx;
    for (int64_t r = int64_t(blockIdx.x) * ty + threadIdx.x / tx; r < P.rows; r += int64_t(gridDim.x) * ty)
        for (int64_t g = threadIdx.x % tx; g < groups; g += tx) {
            float v[8];
            const int64_t left = P.cols - g * 8;
            prep_load8_typed(P.in_type, P.in, blockIdx.y * P.stride + r * P.ld + g * 8, left, v, g > 0);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = float(double(v[i]) * f);
            if (P.planes) {
                __half* o = P.planes + blockIdx.y * P.planes_stride + r * P.planes_ld + g * 8;
                prep_store8(o, left, v);
                if (P.planes_lo) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        __half h, lo;
                        split_planes(v[i], h, lo);
                        v[i] = __half2float(lo);
                    }
                    prep_store8(o + P.planes_lo, left, v);
                }
            } else {
                const int64_t at = blockIdx.y * P.out_stride + r * P.ld_out + g * 8;
                if (P.out_type == SCALECOM_F32) prep_store8(static_cast<float*>(P.out) + at, left, v);
                else if (P.out_type == SCALECOM_F16) prep_store8(static_cast<__half*>(P.out) + at, left, v);
                else prep_store8(static_cast<__nv_bfloat16*>(P.out) + at, left, v);
            }
        }
}

}  // namespace sc
