// The gated feed-forward block's forward pass for a few tokens: every weight is read once for at most eight rows, so HBM bounds it
// and the tensor cores' 128-row tiles have nothing to offer (they took 30 us for one token of 1024 x 4096 in bf16).
//
// A warp (or several, where there are few rows) takes one row of the weights: coalesced 16-byte loads, four on their way for
// each matrix, products and sums in fp32, the tokens' values from L1. Two launches: gate and up with the activation, then down. The
// second fetches its first weights before it waits for the first.
#pragma once
#include "ops_common.cuh"
#include "tc_product.cuh"

namespace sc {

constexpr int FT_THREADS = 256, FT_WARPS = FT_THREADS / 32, FT_MOST = 8;

struct FtParams {
    const void *x, *w0, *w1;        // GATE: x, gate, up; else h, down
    void *out, *saved;              // GATE: h and optionally g, u; else y
    int64_t ldx, ldo;
    int32_t tokens, rows, k;        // weights are [rows][k]
    int32_t split;                  // warps that share a row
    int32_t act;
};

template <typename T, int VEC, int TT, bool GATE>
__global__ void __launch_bounds__(FT_THREADS) ffn_tokens_kernel(const FtParams P) {
    constexpr int NM = GATE ? 2 : 1, U = 4;
    __shared__ float part[FT_WARPS][NM * TT];
    const int warp = int(warp_id()), lane = int(lane_id());
    const int share = warp % P.split, row = blockIdx.x * (FT_WARPS / P.split) + warp / P.split;
    const bool real = row < P.rows;
    const T* w[NM];
    w[0] = static_cast<const T*>(P.w0) + int64_t(real ? row : 0) * P.k;
    if (GATE) w[NM - 1] = static_cast<const T*>(P.w1) + int64_t(real ? row : 0) * P.k;
    const int step = 32 * VEC * P.split, begin = (share * 32 + lane) * VEC;
    Pack<T, VEC> q[U][NM];
    auto fetch = [&](int c0) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int m = 0; m < NM; ++m)
                if (c0 + u * step < P.k) q[u][m] = *reinterpret_cast<const Pack<T, VEC>*>(w[m] + c0 + u * step);
    };
    if (GATE) {
        chain_wait();
        chain_launch();             // not before the wait: what the next kernel reads ahead of its own wait is then complete
        fetch(begin);
    } else {
        chain_launch();
        fetch(begin);               // the weights are inputs of the call, not results of the kernel before
        chain_wait();
    }
    float acc[NM][TT];
#pragma unroll
    for (int m = 0; m < NM; ++m)
#pragma unroll
        for (int t = 0; t < TT; ++t) acc[m][t] = 0.0f;
    for (int c0 = begin; c0 < P.k; c0 += U * step) {
        if (c0 != begin) fetch(c0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = c0 + u * step;
            if (c < P.k) {
#pragma unroll
                for (int t = 0; t < TT; ++t)
                    if (t < P.tokens) {
                        float x[VEC];
                        load_up<T, VEC>(static_cast<const T*>(P.x) + t * P.ldx + c, x);
#pragma unroll
                        for (int m = 0; m < NM; ++m)
#pragma unroll
                            for (int i = 0; i < VEC; ++i) acc[m][t] = fmaf(pack_get<T, VEC>(q[u][m], i), x[i], acc[m][t]);
                    }
            }
        }
    }
#pragma unroll
    for (int m = 0; m < NM; ++m)
#pragma unroll
        for (int t = 0; t < TT; ++t) acc[m][t] = warp_sum_f(acc[m][t]);
    if (P.split > 1) {              // the warps of a row in their order
        if (lane == 0) {
#pragma unroll
            for (int m = 0; m < NM; ++m)
#pragma unroll
                for (int t = 0; t < TT; ++t) part[warp][m * TT + t] = acc[m][t];
        }
        __syncthreads();
        if (share == 0) {
            for (int s = 1; s < P.split; ++s)
#pragma unroll
                for (int m = 0; m < NM; ++m)
#pragma unroll
                    for (int t = 0; t < TT; ++t) acc[m][t] += part[warp + s][m * TT + t];
        }
    }
    if (share != 0 || !real) return;
#pragma unroll
    for (int t = 0; t < TT; ++t)
        if (lane == t && t < P.tokens) {
            T* out = static_cast<T*>(P.out) + t * P.ldo + row;
            if (GATE) {
                const float g = acc[0][t], u = acc[NM - 1][t];
                float a = 0.0f, s;
#define SC_CALL(ACT) act_both<ACT>(g, a, s)
                SC_FOR_ACT(P.act, SC_CALL)
#undef SC_CALL
                *out = Elem<T>::down(a * u);
                if (P.saved) {
                    T* sv = static_cast<T*>(P.saved) + int64_t(t) * P.rows + row;
                    sv[0] = Elem<T>::down(g);
                    sv[int64_t(P.tokens) * P.rows] = Elem<T>::down(u);
                }
            } else {
                *out = Elem<T>::down(acc[0][t]);
            }
        }
}

}  // namespace sc
