// Newton-Schulz on a matrix with one side of at most 128: the whole iteration in one launch.
//
// Such a matrix costs microseconds of arithmetic in fifteen dependent products, so launches and fills are what counts: as
// separate products a 64 x 256 matrix took 138 us.  Here a block (or a cluster of up to eight, which share the long side)
// keeps its part of X, the Gram matrix A and the polynomial B = aI + bA + cAA in shared memory for all steps:
//   A = X X^T    one 16 x 16 tile on or below the diagonal a warp, stored with its mirror image; in a cluster the blocks' parts are
//                added in rank order over distributed shared memory
//   B            the same tiles, in every block of the cluster
//   X <- B X     16 columns of X a warp, read into registers before they are overwritten
// The products are warp-level mma with fp32 accumulators in registers: one instruction of tcgen05 would be the whole
// matrix, with the operands' way through TMEM and back between dependent steps. Their rate is what bounds the kernel (measured:
// some 20 cycles for 16 x 8 x 16 on a quarter of an SM, whatever is fetched ahead), so a single matrix is shared by a cluster
// as soon as that is worth its two barriers a step.
// Values are held as a power of two times themselves in one or two fp16 planes, as in the large path.
#pragma once
#include "ops_common.cuh"
#include "tc_product.cuh"

namespace sc {

constexpr int NSS_THREADS = 512, NSS_WARPS = NSS_THREADS / 32;
constexpr int NSS_MAX_R = 128, NSS_MAX_STEPS = 64;
constexpr float NSS_SCALE = 1024.0f;         // of the first X

// What a step's products are multiplied by: A from X X^T, B = aI + bA + cAA, the next X (or the result) from B X.
struct NsStep { float gram, poly_a, poly_b, poly_c, apply; };

struct NsSmallParams {
    const void* in;
    void* out;
    int64_t ld_in, in_stride, ld_out, out_stride;
    int32_t in_type, out_type;
    int32_t r, n;                  // short and long side
    int32_t tall;                  // stored [n][r]
    int32_t rp, nc;                // r rounded up to 16; columns of a block, a multiple of 16
    int32_t steps;
    float eps;
    NsStep step[NSS_MAX_STEPS];
};

inline int64_t nss_smem(int planes, int64_t rp, int64_t nc, int cluster) {
    return planes * 2 * (rp * (nc + 8) + 2 * rp * (rp + 8)) + (cluster > 1 ? rp * rp * 4 : 0);
}

__device__ __forceinline__ void ldm4(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at));
}
__device__ __forceinline__ void ldm4t(uint32_t (&r)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at));
}
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float ld_cluster_f32(uint32_t at) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at));
    return v;
}
__device__ __forceinline__ double ld_cluster_f64(uint32_t at) {
    double v;
    asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(at) : "memory");
    return v;
}

// A 16 x 16 tile of P Q^T over k, P and Q row-major planes in shared memory: c[0] columns 0-7, c[1] columns 8-15.
// Two planes: lo hi, hi lo, hi hi, and every 16 k the accumulators, which the tensor core cuts, are added to sums with correct rounding.
// (Every 64 k: 8 x 64 x 256 fp32 3.2e-6 from the exact result where plain fp32 products are 1.4e-6; every 16 k 1.2e-6, 39.3 to 40.0 us
// for one matrix.)
template <int PL>
__device__ __forceinline__ void tile_nt(float (&c)[2][4], uint32_t p, uint32_t pl_p, uint32_t ld_p, uint32_t q, uint32_t pl_q, uint32_t ld_q, int k) {
    const uint32_t lane = lane_id();
    const uint32_t at_p = p + ((lane & 15u) * ld_p + (lane >> 4) * 8u) * 2u;
    const uint32_t at_q = q + (((lane & 7u) + ((lane >> 4) << 3)) * ld_q + ((lane >> 3) & 1u) * 8u) * 2u;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) c[h][i] = 0.0f;
    if (PL == 1) {
#pragma unroll 4
        for (int kk = 0; kk < k; kk += 16) {
            uint32_t a[4], b[4];
            ldm4(a, at_p + kk * 2);
            ldm4(b, at_q + kk * 2);
            mma16816(c[0], a, b[0], b[1]);
            mma16816(c[1], a, b[2], b[3]);
        }
    } else {
        for (int kk = 0; kk < k; kk += 16) {
            float s[2][4] = {};
            uint32_t a[4], b[4], al[4], bl[4];
            ldm4(al, at_p + pl_p + kk * 2);
            ldm4(b, at_q + kk * 2);
            ldm4(a, at_p + kk * 2);
            ldm4(bl, at_q + pl_q + kk * 2);
            mma16816(s[0], al, b[0], b[1]);
            mma16816(s[1], al, b[2], b[3]);
            mma16816(s[0], a, bl[0], bl[1]);
            mma16816(s[1], a, bl[2], bl[3]);
            mma16816(s[0], a, b[0], b[1]);
            mma16816(s[1], a, b[2], b[3]);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) c[h][i] += s[h][i];
        }
    }
}
// two neighbouring values into the planes
template <int PL>
__device__ __forceinline__ void put2(uint32_t at, int64_t plane, float x, float y) {
    const __half2 h = __floats2half2_rn(x, y);
    asm volatile("st.shared.b32 [%0], %1;" ::"r"(at), "r"(*reinterpret_cast<const uint32_t*>(&h)) : "memory");
    if (PL == 2) {
        __half hx, lx, hy, ly;
        split_planes(x, hx, lx);
        split_planes(y, hy, ly);
        const __half2 l = __halves2half2(lx, ly);
        asm volatile("st.shared.b32 [%0], %1;" ::"r"(at + uint32_t(plane)), "r"(*reinterpret_cast<const uint32_t*>(&l)) : "memory");
    }
}
template <int PL>
__device__ __forceinline__ float2 get2(uint32_t at, int64_t plane) {
    uint32_t w = lds32(at);
    float2 v = __half22float2(*reinterpret_cast<const __half2*>(&w));
    if (PL == 2) {
        w = lds32(at + uint32_t(plane));
        const float2 l = __half22float2(*reinterpret_cast<const __half2*>(&w));
        v.x += l.x;
        v.y += l.y;
    }
    return v;
}
// four neighbours in memory, the first `left` of them valid
template <typename T>
__device__ __forceinline__ void load_four(const T* p, int left, float (&v)[4]) {
    if (left >= 4 && (reinterpret_cast<uintptr_t>(p) & (4 * sizeof(T) - 1)) == 0) {
        load_up<T, 4>(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = i < left ? Elem<T>::up(p[i]) : 0.0f;
    }
}
// f(line, group, values) for every group of four neighbours of a block's part: lines are `lines` rows in memory, ld apart
template <typename T, typename F>
__device__ __forceinline__ void each_four(const T* p, int64_t ld, int lines, int length, F f) {
    const int groups = (length + 3) / 4;
    int tx = NSS_THREADS;
    while (tx > 1 && tx / 2 >= groups) tx /= 2;
    const int ty = NSS_THREADS / tx, x = threadIdx.x % tx;
    // eight groups on their way at a time: one after another, the loads of a 128 x 512 matrix took 100 us
    for (int g = x; g < groups; g += tx)
        for (int l0 = threadIdx.x / tx; l0 < lines; l0 += 8 * ty) {
            float v[8][4];
#pragma unroll
            for (int q = 0; q < 8; ++q)
                if (l0 + q * ty < lines) load_four(p + int64_t(l0 + q * ty) * ld + 4 * g, length - 4 * g, v[q]);
#pragma unroll
            for (int q = 0; q < 8; ++q)
                if (l0 + q * ty < lines) f(l0 + q * ty, 4 * g, v[q]);
        }
}
template <typename F>
__device__ __forceinline__ void each_four_typed(int type, const void* p, int64_t at, int64_t ld, int lines, int length, F f) {
    if (type == SCALECOM_F32) each_four(static_cast<const float*>(p) + at, ld, lines, length, f);
    else if (type == SCALECOM_F16) each_four(static_cast<const __half*>(p) + at, ld, lines, length, f);
    else each_four(static_cast<const __nv_bfloat16*>(p) + at, ld, lines, length, f);
}
__device__ __forceinline__ void store_one(int type, void* p, int64_t at, float v) {
    if (type == SCALECOM_F32) static_cast<float*>(p)[at] = v;
    else if (type == SCALECOM_F16) static_cast<__half*>(p)[at] = __float2half_rn(v);
    else static_cast<__nv_bfloat16*>(p)[at] = __float2bfloat16_rn(v);
}

template <int PL, bool CLUSTER>
__global__ void __launch_bounds__(NSS_THREADS, 1) ns_small_kernel(const __grid_constant__ NsSmallParams P) {
    extern __shared__ __align__(16) uint8_t nss_raw[];
    __shared__ double red[NSS_WARPS];
    __shared__ double part;
    __shared__ NsStep steps[NSS_MAX_STEPS];       // from the parameters the first reads of each step's cost 0.15 us
    const uint32_t warp = warp_id(), lane = lane_id();
    uint32_t blocks = 1, rank = 0;
    if (CLUSTER) {
        asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(blocks));
        asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    }
    const int r = P.r, rp = P.rp, nc = P.nc, first = int(rank) * nc, mine = max(0, min(nc, P.n - first));
    const uint32_t ldx = uint32_t(nc) + 8u, lda = uint32_t(rp) + 8u;
    const int64_t plx = int64_t(rp) * ldx * 2, pla = int64_t(rp) * lda * 2;         // bytes of a plane
    const uint32_t X = smem_u32(nss_raw), A = X + uint32_t(PL * plx), B = A + uint32_t(PL * pla), G = B + uint32_t(PL * pla);
    const int64_t base = int64_t(blockIdx.y) * P.in_stride;
    // element (i, j) of the short-side-first matrix, j counted from this block's first column
    auto where = [&](int i, int j, int64_t ld) { return P.tall ? int64_t(first + j) * ld + i : int64_t(i) * ld + first + j; };
    chain_launch();
    if (int(threadIdx.x) < P.steps) steps[threadIdx.x] = P.step[threadIdx.x];
    chain_wait();

    // |X|^2 in fp64, over the cluster
    const int lines = P.tall ? mine : r, length = P.tall ? r : mine;
    const int64_t start = base + (P.tall ? int64_t(first) * P.ld_in : first);
    for (uint32_t e = threadIdx.x * 16u; e < uint32_t(PL * plx); e += NSS_THREADS * 16u) sts128(X + e, 0u, 0u, 0u, 0u);
    double s = 0.0;
    each_four_typed(P.in_type, P.in, start, P.ld_in, lines, length, [&](int, int, const float (&v)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) s += double(v[i]) * double(v[i]);
    });
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(FULL, s, o);
    if (lane == 0) red[warp] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        s = 0.0;
        for (int w = 0; w < NSS_WARPS; ++w) s += red[w];
        part = s;
    }
    __syncthreads();
    double total = part;
    if (CLUSTER) {
        cluster_sync();
        total = 0.0;
        for (uint32_t b = 0; b < blocks; ++b) total += ld_cluster_f64(in_block(smem_u32(&part), b));
    }
    const double factor = double(NSS_SCALE) / (sqrt(total) + double(P.eps));
    // X, short side first; what pads it to rp x nc is zero already
    each_four_typed(P.in_type, P.in, start, P.ld_in, lines, length, [&](int line, int at, const float (&v)[4]) {
        float w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = float(double(v[i]) * factor);
        if (!P.tall) {
            const uint32_t to = X + (uint32_t(line) * ldx + at) * 2u;
            put2<PL>(to, plx, w[0], w[1]);
            put2<PL>(to + 4u, plx, w[2], w[3]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t to = X + (uint32_t(at + i) * ldx + line) * 2u;
                __half h, l;
                split_planes(w[i], h, l);
                if (at + i < rp) {
                    sts16(to, __half_as_ushort(h));
                    if (PL == 2) sts16(to + uint32_t(plx), __half_as_ushort(l));
                }
            }
        }
    });
    __syncthreads();

    const int side = rp / 16, tiles = side * (side + 1) / 2;
    const uint32_t fr = lane >> 2, fc = (lane & 3u) * 2u;                           // this lane's first row and column of an accumulator tile
    const uint32_t upla = uint32_t(pla), uplx = uint32_t(plx);
    auto place = [](int t, int& ti, int& tj) {                                      // tiles on and below the diagonal, row by row
        ti = 0;
        while (t > ti) t -= ++ti;
        tj = t;
    };
    // a tile of a symmetric matrix into the planes, here and mirrored
    auto put_tile = [&](uint32_t to, int ti, int tj, const float (&c)[2][4]) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const uint32_t row = ti * 16 + fr + 8 * q, col = tj * 16 + fc + 8 * h;
                put2<PL>(to + (row * lda + col) * 2u, pla, c[h][2 * q], c[h][2 * q + 1]);
                if (ti != tj) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        __half hi, lo;
                        split_planes(c[h][2 * q + i], hi, lo);
                        const uint32_t at = to + ((col + i) * lda + row) * 2u;
                        sts16(at, __half_as_ushort(hi));
                        if (PL == 2) sts16(at + upla, __half_as_ushort(lo));
                    }
                }
            }
    };
    for (int step = 0; step < P.steps; ++step) {
        const NsStep by = steps[step];
        const float ca = by.poly_a, cb = by.poly_b, cc = by.poly_c;
        const bool last = step + 1 == P.steps;
        // A = X X^T
        for (int t = warp; t < tiles; t += NSS_WARPS) {
            int ti, tj;
            place(t, ti, tj);
            float c[2][4];
            tile_nt<PL>(c, X + ti * 16 * ldx * 2, uplx, ldx, X + tj * 16 * ldx * 2, uplx, ldx, nc);
            if (CLUSTER) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    asm volatile("st.shared.f32 [%0], %1;" ::"r"(G + ((t * 8 + i) * 32 + lane) * 4u), "f"(c[i / 4][i % 4]) : "memory");
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) c[i / 4][i % 4] *= by.gram;
                put_tile(A, ti, tj, c);
            }
        }
        if (CLUSTER) {
            cluster_sync();
            for (int t = warp; t < tiles; t += NSS_WARPS) {
                int ti, tj;
                place(t, ti, tj);
                float c[2][4] = {};
                for (uint32_t b0 = 0; b0 < blocks; b0 += 4) {            // a load from another block takes about 1,000 cycles: four blocks' at once
                    float got[4][8];
#pragma unroll
                    for (uint32_t b = 0; b < 4; ++b)
                        if (b0 + b < blocks) {
                            const uint32_t g = in_block(G, b0 + b);
#pragma unroll
                            for (int i = 0; i < 8; ++i) got[b][i] = ld_cluster_f32(g + ((t * 8 + i) * 32 + lane) * 4u);
                        }
#pragma unroll
                    for (uint32_t b = 0; b < 4; ++b)
                        if (b0 + b < blocks) {
#pragma unroll
                            for (int i = 0; i < 8; ++i) c[i / 4][i % 4] += got[b][i];
                        }
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) c[i / 4][i % 4] *= by.gram;
                put_tile(A, ti, tj, c);
            }
            cluster_sync();                                  // the parts are read before the next step overwrites them
        } else {
            __syncthreads();
        }
        // B = aI + bA + cAA (A is symmetric)
        for (int t = warp; t < tiles; t += NSS_WARPS) {
            int ti, tj;
            place(t, ti, tj);
            float c[2][4];
            tile_nt<PL>(c, A + ti * 16 * lda * 2, upla, lda, A + tj * 16 * lda * 2, upla, lda, rp);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    const int row = ti * 16 + fr + 8 * q, col = tj * 16 + fc + 8 * h;
                    const float2 a = get2<PL>(A + (row * lda + col) * 2u, pla);
                    c[h][2 * q] = cb * a.x + cc * c[h][2 * q] + (row == col ? ca : 0.0f);
                    c[h][2 * q + 1] = cb * a.y + cc * c[h][2 * q + 1] + (row == col + 1 ? ca : 0.0f);
                }
            put_tile(B, ti, tj, c);
        }
        __syncthreads();
        // X <- B X, sixteen columns a warp
        constexpr int SIDE = NSS_MAX_R / 16;
        for (int j0 = int(warp) * 16; j0 < nc; j0 += NSS_WARPS * 16) {
            uint32_t xb[PL][SIDE][4];
            const uint32_t at_x = X + (((lane & 7u) + ((lane >> 3) & 1u) * 8u) * ldx + j0 + (lane >> 4) * 8u) * 2u;
#pragma unroll
            for (int kk = 0; kk < SIDE; ++kk)
                if (kk < side) {
#pragma unroll
                    for (int pl = 0; pl < PL; ++pl) ldm4t(xb[pl][kk], at_x + pl * uplx + kk * 16 * ldx * 2);
                }
            for (int ti = 0; ti < side; ++ti) {
                float c[2][4] = {};
                const uint32_t at_b = B + ((ti * 16 + (lane & 15u)) * lda + (lane >> 4) * 8u) * 2u;
#pragma unroll
                for (int kk = 0; kk < SIDE; ++kk)
                    if (kk < side) {
                        uint32_t a[4];
                        if (PL == 2) {
                            float s2[2][4] = {};
                            uint32_t al[4];
                            ldm4(al, at_b + upla + kk * 32);
                            ldm4(a, at_b + kk * 32);
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                mma16816(s2[h], al, xb[0][kk][2 * h], xb[0][kk][2 * h + 1]);
                                mma16816(s2[h], a, xb[PL - 1][kk][2 * h], xb[PL - 1][kk][2 * h + 1]);
                                mma16816(s2[h], a, xb[0][kk][2 * h], xb[0][kk][2 * h + 1]);
#pragma unroll
                                for (int i = 0; i < 4; ++i) c[h][i] += s2[h][i];
                            }
                        } else {
                            ldm4(a, at_b + kk * 32);
                            mma16816(c[0], a, xb[0][kk][0], xb[0][kk][1]);
                            mma16816(c[1], a, xb[0][kk][2], xb[0][kk][3]);
                        }
                    }
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        const int row = ti * 16 + fr + 8 * q, col = j0 + fc + 8 * h;
                        if (!last) {
                            put2<PL>(X + (row * ldx + col) * 2u, plx, c[h][2 * q] * by.apply, c[h][2 * q + 1] * by.apply);
                        } else if (row < r) {
                            const int64_t to = int64_t(blockIdx.y) * P.out_stride;
                            if (col < mine) store_one(P.out_type, P.out, to + where(row, col, P.ld_out), c[h][2 * q] * by.apply);
                            if (col + 1 < mine) store_one(P.out_type, P.out, to + where(row, col + 1, P.ld_out), c[h][2 * q + 1] * by.apply);
                        }
                    }
            }
        }
        __syncthreads();
    }
    if (CLUSTER) cluster_sync();                             // no block leaves while another may read its memory
}

}  // namespace sc
