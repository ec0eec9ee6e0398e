// Matrix products on the 5th-generation tensor cores with fused epilogues.
//
// One persistent kernel computes  acc[m][n] = sum over k of A[m][k] B[n][k]  (or the sum of two such products) in tiles of
// 128 x BN and hands the fp32 accumulators to an epilogue: a store, the gated activation, its backward, or a step of the
// Newton-Schulz iteration.  Either operand may be stored with k contiguous ("K-major") or with its own rows contiguous
// ("MN-major"), so no operand is ever transposed in memory.
//
// Roles (12 warps): warp 0 issues the TMA copies, warp 1 issues tcgen05.mma, warp 2 owns the TMEM allocation, warps 4-11 run
// the epilogue.  Two accumulators in TMEM: the epilogue of a tile runs under the products of the next.
//
// PL = 2, for fp32 values: each operand is two fp16 planes, x = hi + lo, and a block of k contributes lo hi + hi lo + hi hi.
// The tensor core truncates its fp32 accumulator after every 16 k (measured: 2.2e-8 of the result for each, always towards
// zero, so 2048 k are 3e-6 low), which is why the accumulator is not kept there: after each 64 k, small products first, the epilogue
// warps add it to sums in registers with correct rounding.
#pragma once
#include <cuda.h>

#include "ops_common.cuh"

namespace sc {

constexpr int TC_BM = 128;            // rows of a tile: the tensor core's M
constexpr int TC_BK = 64;             // 64 16-bit values = one 128-byte swizzled row
constexpr int TC_THREADS = 384;
constexpr int TC_EPI_WARPS = 8;
constexpr int TC_EPI_THREADS = TC_EPI_WARPS * 32;
constexpr int TC_A_BYTES = TC_BM * TC_BK * 2;

template <int BN, int PL> struct TcShape {
    static constexpr int B_BYTES = BN * TC_BK * 2;
    static constexpr int STAGE_BYTES = PL * (TC_A_BYTES + B_BYTES);  // A planes, then B planes
    static constexpr int STAGES = 196608 / STAGE_BYTES;              // 192 KB of operands in flight
    static constexpr int SMEM = STAGES * STAGE_BYTES + 1024;         // + alignment of the swizzle atoms
    static constexpr int TMEM_COLS = 2 * BN;
};

enum TcEpilogue { EPI_STORE = 0, EPI_GATE = 1, EPI_GATE_BWD = 2, EPI_GRAM = 3, EPI_POLY = 4, EPI_PLANES = 5 };

struct TcParams {
    CUtensorMap a[2], b[2];
    int32_t pairs, kblocks;                   // products that are summed (1 or 2), 64-wide blocks of k in each
    int32_t m, n;                             // extent of the result (EPI_GATE: n counts gate columns)
    int32_t mt, nt, tiles;                    // tiles of one matrix
    int32_t batch, splits;
    int32_t a_mn, b_mn, a_batched, b_batched;
    uint32_t idesc;
    uint32_t* status;
    float* partial;                           // splits > 1: [batch*tiles][splits][128][BN] accumulators
    uint32_t* arrived;                        // splits > 1: [batch*tiles], zero between launches

    // epilogue
    int32_t type;                             // element type of out / h / saved
    int32_t act;
    float alpha;
    const uint32_t *amax_a, *amax_b;          // largest magnitudes behind the operands' scales, NULL: unscaled
    void *out, *out2, *out3;                  // STORE: out; GATE: h, saved; GATE_BWD: dg, du, h
    const void *in1, *in2;                    // GATE_BWD: saved g, u
    int64_t ldo, ostride;                     // row distance and matrix distance of the outputs (elements)
    int64_t ldi;                              // row distance of in1, in2 / of saved
    uint32_t *amax_o, *amax_o2;               // fp32 intermediates: their largest magnitude is collected
    __half* planes_out;                       // Newton-Schulz: [batch][planes][rows][ldo]
    const __half* planes_in;
    int64_t plane_out, plane_in;              // distance of the lo plane (elements); 0: hi only
    float poly_a, poly_b, poly_c;
};

// ---- mbarriers, TMA, tcgen05 -------------------------------------------------------------------------
__device__ __forceinline__ uint32_t smem_u32(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
    asm volatile("{\n\t.reg .b64 t;\n\tmbarrier.arrive.shared::cta.b64 t, [%0];\n\t}" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void mbar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("{\n\t.reg .b64 t;\n\tmbarrier.arrive.expect_tx.shared::cta.b64 t, [%0], %1;\n\t}" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
// Bounded: gives up after about two seconds, or as soon as another role of the block has, and marks the device status.
constexpr unsigned long long TC_WAIT_NS = 2000000000ull;
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, volatile uint32_t* abort, uint32_t* status) {
    unsigned long long t0 = 0;
    for (uint32_t it = 0; it < 0x40000000u; ++it) {
        if (mbar_try(bar, parity)) return true;
        if ((it & 63u) == 63u) {
            if (*abort) return false;
            const unsigned long long t = global_timer_ns();
            if (!t0) t0 = t;
            else if (t - t0 > TC_WAIT_NS) break;
        }
    }
    *abort = 1u;
    atomicCAS(status, DEV_OK, DEV_TIMEOUT);
    return false;
}
// the last wait of a role that gave up: its own copies or products in flight, whatever the others do
__device__ __forceinline__ void mbar_drain(uint32_t bar, uint32_t parity) {
    unsigned long long t0 = 0;
    for (uint32_t it = 0; it < 0x40000000u; ++it) {
        if (mbar_try(bar, parity)) return;
        if ((it & 63u) == 63u) {
            const unsigned long long t = global_timer_ns();
            if (!t0) t0 = t;
            else if (t - t0 > TC_WAIT_NS) return;
        }
    }
}
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, int c3, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
                 ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(bar) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void tc_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tc_ld32(uint32_t addr, float (&v)[32]) {
    uint32_t r[32];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]),
          "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]),
          "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}

// Shared-memory matrix descriptors, 128-byte swizzle (layout code 2, version 1).
//   K-major:  a tile is rows of 128 bytes; 8 rows form an atom, atoms 1024 bytes apart.
//   MN-major: a tile is 64-row-wide panels; in a panel each k is a 128-byte row, 8 k form an atom (1024 bytes
//             apart along k), and panels are 64 k = 8192 bytes apart.
__device__ __forceinline__ uint64_t tc_desc(uint32_t addr, int mn) {
    const uint64_t lead = mn ? (TC_BK * 128) >> 4 : 1;
    return uint64_t((addr & 0x3FFFFu) >> 4) | (lead << 16) | (uint64_t(1024 >> 4) << 32) | (uint64_t(1) << 46) | (uint64_t(2) << 61);
}

// ---- activations --------------------------------------------------------------------------------------
__device__ __forceinline__ float act_value(int act, float g) {
    switch (act) {
        case SCALECOM_ACT_SILU: return g / (1.0f + expf(-g));
        case SCALECOM_ACT_GELU: return 0.5f * g * (1.0f + erff(g * 0.70710678118654752f));
        case SCALECOM_ACT_GELU_TANH: return 0.5f * g * (1.0f + tanhf(0.79788456080286536f * (g + 0.044715f * g * g * g)));
        default: return g > 0.0f ? g : (g == g ? 0.0f : g);
    }
}
// value and derivative
__device__ __forceinline__ void act_both(int act, float g, float& a, float& s) {
    switch (act) {
        case SCALECOM_ACT_SILU: {
            const float p = 1.0f / (1.0f + expf(-g));
            a = g * p;
            s = p * (1.0f + g * (1.0f - p));
            return;
        }
        case SCALECOM_ACT_GELU: {
            const float c = 0.5f * (1.0f + erff(g * 0.70710678118654752f));
            a = g * c;
            s = c + g * expf(-0.5f * g * g) * 0.39894228040143268f;
            return;
        }
        case SCALECOM_ACT_GELU_TANH: {
            if (fabsf(g) > 30.0f) {                 // tanh is +-1 there; the cube below could overflow
                a = g > 0.0f ? g : 0.0f;
                s = g > 0.0f ? 1.0f : 0.0f;
                return;
            }
            const float t = tanhf(0.79788456080286536f * (g + 0.044715f * g * g * g));
            a = 0.5f * g * (1.0f + t);
            s = 0.5f * (1.0f + t) + 0.5f * g * (1.0f - t * t) * 0.79788456080286536f * (1.0f + 0.134145f * g * g);
            return;
        }
        default:
            a = g > 0.0f ? g : (g == g ? 0.0f : g);
            s = g > 0.0f ? 1.0f : 0.0f;
            return;
    }
}

// ---- tile order ----------------------------------------------------------------------------------------
struct TcUnit { int batch, mt, nt, split, tile; };

template <int BN, int EPI>
__device__ __forceinline__ TcUnit tc_unit(const TcParams& P, int u) {
    TcUnit r;
    r.split = u % P.splits;
    u /= P.splits;
    r.tile = u;                                   // over all matrices
    r.batch = u / P.tiles;
    int t = u % P.tiles;
    if (EPI == EPI_GRAM || EPI == EPI_POLY) {     // symmetric result: tiles that touch the lower triangle
        int mt = 0;
        for (;; ++mt) {
            int cols = (mt * TC_BM + TC_BM - 1) / BN + 1;
            if (cols > P.nt) cols = P.nt;
            if (t < cols) break;
            t -= cols;
        }
        r.mt = mt;
        r.nt = t;
    } else {                                      // bands of 16 row tiles, column by column: the band's A stays in L2
        constexpr int BAND = 16;
        const int band = t / (BAND * P.nt), first = band * BAND;
        const int rows = P.mt - first < BAND ? P.mt - first : BAND;
        const int in = t - band * BAND * P.nt;
        r.nt = in / rows;
        r.mt = first + in % rows;
    }
    return r;
}

// ---- epilogues on 32 columns of a row --------------------------------------------------------------------
__device__ __forceinline__ void store_typed(int type, void* base, int64_t off, const float* v, int ncols) {
    if (type == SCALECOM_BF16) store_row32(static_cast<__nv_bfloat16*>(base) + off, v, ncols);
    else if (type == SCALECOM_F16) store_row32(static_cast<__half*>(base) + off, v, ncols);
    else store_row32(static_cast<float*>(base) + off, v, ncols);
}
__device__ __forceinline__ void load_typed(int type, const void* base, int64_t off, float* v, int ncols) {
    if (type == SCALECOM_BF16) load_row32(static_cast<const __nv_bfloat16*>(base) + off, v, ncols);
    else if (type == SCALECOM_F16) load_row32(static_cast<const __half*>(base) + off, v, ncols);
    else load_row32(static_cast<const float*>(base) + off, v, ncols);
}
__device__ __forceinline__ void store_planes(__half* base, int64_t lo, int64_t off, const float* v, int ncols) {
    if (!lo) {
        store_row32(base + off, v, ncols);
        return;
    }
    float l[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        __half h, r;
        split_planes(v[i], h, r);
        l[i] = __half2float(r);
    }
    store_row32(base + off, v, ncols);
    store_row32(base + lo + off, l, ncols);
}

template <int EPI>
__device__ __forceinline__ void tc_epilogue(const TcParams& P, const TcUnit& u, int row, int col, float (&v)[32], float (&w)[32],
                                            float un, uint32_t& top, uint32_t& top2) {
    const int nc = P.n - col;
    if (row >= P.m || nc <= 0) return;
    if (EPI == EPI_STORE) {
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] *= un;
        store_typed(P.type, P.out, int64_t(u.batch) * P.ostride + int64_t(row) * P.ldo + col, v, nc);
    } else if (EPI == EPI_GATE) {
#pragma unroll
        for (int i = 0; i < 32; ++i) { v[i] *= un; w[i] *= un; }
        if (P.out2) {
            const int64_t at = int64_t(row) * P.n + col;
            store_typed(P.type, P.out2, at, v, nc);
            store_typed(P.type, P.out2, at + int64_t(P.m) * P.n, w, nc);
        }
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            v[i] = act_value(P.act, v[i]) * w[i];
            if (i < nc) top = max(top, finite_bits(v[i]));
        }
        store_typed(P.type, P.out, int64_t(row) * P.ldo + col, v, nc);
    } else if (EPI == EPI_GATE_BWD) {
        float g[32];
        const int64_t at = int64_t(row) * P.ldi + col;
        load_typed(P.type, P.in1, at, g, nc);
        load_typed(P.type, P.in2, at, w, nc);
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            float a, s;
            act_both(P.act, g[i], a, s);
            const float dh = v[i] * un, uu = w[i];
            g[i] = dh * uu * s;            // dg
            w[i] = dh * a;                 // du
            v[i] = a * uu;                 // h
            if (i < nc) {
                top = max(top, max(finite_bits(g[i]), finite_bits(w[i])));
                top2 = max(top2, finite_bits(v[i]));
            }
        }
        const int64_t to = int64_t(row) * P.ldo + col;
        store_typed(P.type, P.out, to, g, nc);
        store_typed(P.type, P.out2, to, w, nc);
        store_typed(P.type, P.out3, to, v, nc);
    } else if (EPI == EPI_PLANES) {
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] *= P.alpha;
        store_planes(P.planes_out + int64_t(u.batch) * P.ostride, P.plane_out, int64_t(row) * P.ldo + col, v, nc);
    } else {
        // symmetric result: columns up to the diagonal, stored at (row, col) and at (col, row)
        const int valid = min(nc, row - col + 1);
        if (valid <= 0) return;
        const int64_t at = int64_t(row) * P.ldo + col;
        if (EPI == EPI_POLY) {
            const __half* in = P.planes_in + int64_t(u.batch) * P.ostride + at;
            load_row32(in, w, valid);
            if (P.plane_in) {
                float l[32];
                load_row32(in + P.plane_in, l, valid);
#pragma unroll
                for (int i = 0; i < 32; ++i) w[i] += l[i];
            }
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = P.poly_b * w[i] + P.poly_c * v[i] + (i == row - col ? P.poly_a : 0.0f);
        } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] *= P.alpha;
        }
        __half* o = P.planes_out + int64_t(u.batch) * P.ostride;
        store_planes(o, P.plane_out, at, v, valid);
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            if (i < valid) {                       // lanes hold consecutive rows: the mirrored store is coalesced
                const int64_t mt = int64_t(col + i) * P.ldo + row;
                __half h, l;
                split_planes(v[i], h, l);
                o[mt] = h;
                if (P.plane_out) o[P.plane_out + mt] = l;
            }
        }
    }
}

// whether `ok` holds for all threads of the epilogue warps (a barrier among them)
__device__ __forceinline__ bool epilogue_all(bool ok) {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, 1, 256, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"(uint32_t(ok)) : "memory");
    return r != 0u;
}

template <int BN, int EPI, int PL>
__global__ void __launch_bounds__(TC_THREADS, 1) tc_product_kernel(const __grid_constant__ TcParams P) {
    using S = TcShape<BN, PL>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ alignas(8) uint64_t bars[2 * S::STAGES + 4 + 1];
    __shared__ uint32_t tmem_base, abort_flag, last_flag;

    const uint32_t warp = warp_id(), lane = lane_id();
    const uint32_t tiles0 = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t bar0 = smem_u32(bars);
    auto full = [&](int s) { return bar0 + 8u * s; };
    auto empty = [&](int s) { return bar0 + 8u * (S::STAGES + s); };
    auto tfull = [&](int s) { return bar0 + 8u * (2 * S::STAGES + s); };
    auto tempty = [&](int s) { return bar0 + 8u * (2 * S::STAGES + 2 + s); };
    const uint32_t drain = bar0 + 8u * (2 * S::STAGES + 4);

    if (warp == 0 && lane == 0) {
        for (int s = 0; s < S::STAGES; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
        for (int s = 0; s < 2; ++s) { mbar_init(tfull(s), 1); mbar_init(tempty(s), TC_EPI_WARPS); }
        mbar_init(drain, 1);
        abort_flag = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base)), "n"(S::TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_base;
    chain_launch();
    chain_wait();

    volatile uint32_t* abort = &abort_flag;
    const int units = P.batch * P.tiles * P.splits;
    const int iters = P.pairs * P.kblocks;

    if (warp == 0) {
        if (lane == 0) {
            int n_issued = 0;                       // copies issued so far; stage and phase follow from it
            bool ok = true;
            for (int un = blockIdx.x; ok && un < units; un += gridDim.x) {
                const TcUnit u = tc_unit<BN, EPI>(P, un);
                const int it0 = int(int64_t(iters) * u.split / P.splits), it1 = int(int64_t(iters) * (u.split + 1) / P.splits);
                const int m0 = u.mt * TC_BM, n0 = u.nt * (EPI == EPI_GATE ? BN / 2 : BN);
                const int ba = P.a_batched ? u.batch : 0, bb = P.b_batched ? u.batch : 0;
                for (int it = it0; it < it1; ++it, ++n_issued) {
                    const int s = n_issued % S::STAGES, round = n_issued / S::STAGES;
                    if (!mbar_wait(empty(s), (round & 1) ^ 1, abort, P.status)) { ok = false; break; }
                    const int pair = it >= P.kblocks, k0 = (it - pair * P.kblocks) * TC_BK;
                    const uint32_t a = tiles0 + s * S::STAGE_BYTES, b = a + PL * TC_A_BYTES, bar = full(s);
                    mbar_expect(bar, S::STAGE_BYTES);
#pragma unroll
                    for (int pl = 0; pl < PL; ++pl) {
                        const uint32_t ap = a + pl * TC_A_BYTES, bp = b + pl * S::B_BYTES;
                        if (P.a_mn) {
                            for (int j = 0; j < TC_BM / 64; ++j) tma_load(ap + j * 8192, &P.a[pair], m0 + 64 * j, k0, pl, ba, bar);
                        } else {
                            tma_load(ap, &P.a[pair], k0, m0, pl, ba, bar);
                        }
                        if (EPI == EPI_GATE) {      // gate columns, then the same columns of the up projection
                            tma_load(bp, &P.b[0], k0, n0, pl, bb, bar);
                            tma_load(bp + S::B_BYTES / 2, &P.b[1], k0, n0, pl, bb, bar);
                        } else if (P.b_mn) {
                            for (int j = 0; j < BN / 64; ++j) tma_load(bp + j * 8192, &P.b[pair], n0 + 64 * j, k0, pl, bb, bar);
                        } else {
                            tma_load(bp, &P.b[pair], k0, n0, pl, bb, bar);
                        }
                    }
                }
            }
            if (!ok)                                // the copies still in flight write this block's shared memory
                for (int i = n_issued > S::STAGES ? n_issued - S::STAGES : 0; i < n_issued; ++i)
                    mbar_drain(full(i % S::STAGES), (i / S::STAGES) & 1);
        }
    } else if (warp == 1) {
        if (lane == 0) {
            int n_used = 0, n_acc = 0;
            bool ok = true;
            for (int un = blockIdx.x; ok && un < units; un += gridDim.x, ++n_acc) {
                const TcUnit u = tc_unit<BN, EPI>(P, un);
                const int it0 = int(int64_t(iters) * u.split / P.splits), it1 = int(int64_t(iters) * (u.split + 1) / P.splits);
                if (PL == 1) {
                    if (!mbar_wait(tempty(n_acc & 1), ((n_acc >> 1) & 1) ^ 1, abort, P.status)) { ok = false; break; }
                    tc_fence_after();
                }
                for (int it = it0; it < it1; ++it, ++n_used) {
                    const int s = n_used % S::STAGES;
                    if (PL == 2) {                  // an accumulator for each block of k
                        if (!mbar_wait(tempty(n_used & 1), ((n_used >> 1) & 1) ^ 1, abort, P.status)) { ok = false; break; }
                    }
                    if (!mbar_wait(full(s), (n_used / S::STAGES) & 1, abort, P.status)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t d = tmem + ((PL == 2 ? n_used : n_acc) & 1) * BN;
                    const uint32_t a = tiles0 + s * S::STAGE_BYTES, b = a + PL * TC_A_BYTES;
                    const uint32_t step_a = P.a_mn ? 2048 >> 4 : 32 >> 4, step_b = P.b_mn ? 2048 >> 4 : 32 >> 4;
#pragma unroll
                    for (int t = 0; t < (PL == 2 ? 3 : 1); ++t) {      // lo hi, hi lo, hi hi
                        const uint64_t da = tc_desc(a + (PL == 2 && t == 0 ? TC_A_BYTES : 0), P.a_mn);
                        const uint64_t db = tc_desc(b + (PL == 2 && t == 1 ? S::B_BYTES : 0), P.b_mn);
#pragma unroll
                        for (int k = 0; k < TC_BK / 16; ++k)
                            tc_mma(d, da + k * step_a, db + k * step_b, P.idesc, (t > 0 || k > 0 || (PL == 1 && it > it0)) ? 1u : 0u);
                    }
                    tc_commit(empty(s));
                    if (PL == 2) tc_commit(tfull(n_used & 1));
                }
                if (PL == 1 && ok) tc_commit(tfull(n_acc & 1));
            }
            if (!ok) {                              // products in flight read shared memory and write TMEM
                tc_commit(drain);
                mbar_drain(drain, 0);
            }
        }
    } else if (warp >= 4) {
        const uint32_t quad = warp & 3u, half = (warp - 4u) >> 2;
        const uint32_t lanes = (quad * 32u) << 16;
        const int tid = int(threadIdx.x) - 128;
        // result columns of a tile, and a warp's 32-column chunks of them: GATE works on a gate chunk and the up chunk beside it
        constexpr int WIDTH = EPI == EPI_GATE ? BN / 2 : BN, CHUNKS = WIDTH / 64;
        auto chunk = [&](int c) { return (int(half) * CHUNKS + c) * 32; };
        float un_scale = P.alpha;
        if (P.amax_a) un_scale *= plane_unscale(*P.amax_a) * plane_unscale(*P.amax_b);
        uint32_t top = 0u, top2 = 0u;
        int n_acc = 0;
        for (int un = blockIdx.x; un < units; un += gridDim.x) {
            const TcUnit u = tc_unit<BN, EPI>(P, un);
            const int row = u.mt * TC_BM + quad * 32 + lane;
            float v[32], w[32];
            float sum[PL == 2 ? BN / 64 : 1][32];       // PL = 2: this thread's columns, in the order of `column`
            auto column = [&](int c) {                  // TMEM column of the thread's c-th 32 columns
                if (EPI == EPI_GATE && PL == 2) return (c & 1) * (BN / 2) + (int(half) * (BN / 128) + (c >> 1)) * 32;
                return int(half) * (BN / 2) + c * 32;
            };
            bool ok = true;
            uint32_t acc = 0;
            int q = 0;
            if (PL == 2) {
                const int it0 = int(int64_t(iters) * u.split / P.splits), it1 = int(int64_t(iters) * (u.split + 1) / P.splits);
#pragma unroll
                for (int c = 0; c < BN / 64; ++c)
#pragma unroll
                    for (int i = 0; i < 32; ++i) sum[c][i] = 0.0f;
                for (int it = it0; it < it1; ++it, ++n_acc) {
                    q = n_acc & 1;
                    ok = __all_sync(FULL, mbar_wait(tfull(q), (n_acc >> 1) & 1, abort, P.status));
                    if (!ok) break;
                    tc_fence_after();
                    acc = tmem + q * BN + lanes;
#pragma unroll
                    for (int c = 0; c < BN / 64; ++c) {
                        tc_ld32(acc + column(c), v);
#pragma unroll
                        for (int i = 0; i < 32; ++i) sum[c][i] += v[i];
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(tempty(q));
                }
            } else {
                q = n_acc & 1;
                ok = __all_sync(FULL, mbar_wait(tfull(q), (n_acc >> 1) & 1, abort, P.status));
                ++n_acc;
                acc = tmem + q * BN + lanes;
            }
            if (P.splits > 1) ok = epilogue_all(ok);       // the block barriers below need every epilogue warp
            if (!ok) break;
            tc_fence_after();
            auto release = [&]() {                          // the accumulator is free once its last columns are in registers
                if (PL == 1) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(tempty(q));
                }
            };
            if (P.splits > 1) {
                // this part's accumulators to scratch, [column][row]; the block that arrives last adds the parts up in their order
                float* mine = P.partial + (int64_t(u.tile) * P.splits) * (TC_BM * BN) + quad * 32 + lane;
                float* put = mine + int64_t(u.split) * (TC_BM * BN);
                if (PL == 2) {
#pragma unroll
                    for (int c = 0; c < BN / 64; ++c)
#pragma unroll
                        for (int i = 0; i < 32; ++i) put[(column(c) + i) * TC_BM] = sum[c][i];
                } else {
#pragma unroll 1
                    for (int c = 0; c < BN / 64; ++c) {
                        tc_ld32(acc + column(c), v);
#pragma unroll
                        for (int i = 0; i < 32; ++i) put[(column(c) + i) * TC_BM] = v[i];
                    }
                }
                release();
                __threadfence();
                asm volatile("bar.sync 1, 256;" ::: "memory");
                if (tid == 0) {
                    const uint32_t before = atomicAdd(&P.arrived[u.tile], 1u);
                    last_flag = before + 1u == uint32_t(P.splits);
                    if (before + 1u == uint32_t(P.splits)) P.arrived[u.tile] = 0u;
                    __threadfence();
                }
                asm volatile("bar.sync 1, 256;" ::: "memory");
                const bool last = last_flag != 0u;
                asm volatile("bar.sync 1, 256;" ::: "memory");
                if (!last) continue;
                __threadfence();
                auto gather = [&](int col, float (&x)[32]) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) x[i] = 0.0f;
                    for (int s = 0; s < P.splits; ++s) {
                        const float* get = mine + int64_t(s) * (TC_BM * BN) + col * TC_BM;
#pragma unroll
                        for (int i = 0; i < 32; ++i) x[i] += __ldcg(&get[i * TC_BM]);
                    }
                };
#pragma unroll 1
                for (int c = 0; c < CHUNKS; ++c) {
                    const int at = chunk(c);
                    gather(at, v);
                    if (EPI == EPI_GATE) gather(BN / 2 + at, w);
                    tc_epilogue<EPI>(P, u, row, u.nt * WIDTH + at, v, w, un_scale, top, top2);
                }
            } else if (PL == 2) {
#pragma unroll
                for (int c = 0; c < CHUNKS; ++c) {
                    if (EPI == EPI_GATE) tc_epilogue<EPI>(P, u, row, u.nt * WIDTH + chunk(c), sum[2 * c], sum[2 * c + 1], un_scale, top, top2);
                    else tc_epilogue<EPI>(P, u, row, u.nt * WIDTH + chunk(c), sum[c], w, un_scale, top, top2);
                }
            } else {
#pragma unroll 1
                for (int c = 0; c < CHUNKS; ++c) {
                    const int at = chunk(c);
                    tc_ld32(acc + at, v);
                    if (EPI == EPI_GATE) tc_ld32(acc + BN / 2 + at, w);
                    if (c == CHUNKS - 1) release();
                    tc_epilogue<EPI>(P, u, row, u.nt * WIDTH + at, v, w, un_scale, top, top2);
                }
            }
        }
        if (EPI == EPI_GATE || EPI == EPI_GATE_BWD) {
            if (P.amax_o) {
                top = __reduce_max_sync(FULL, top);
                if (lane == 0 && top) atomicMax(P.amax_o, top);
            }
            if (P.amax_o2) {
                top2 = __reduce_max_sync(FULL, top2);
                if (lane == 0 && top2) atomicMax(P.amax_o2, top2);
            }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 2) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(S::TMEM_COLS) : "memory");
    }
}

}  // namespace sc
