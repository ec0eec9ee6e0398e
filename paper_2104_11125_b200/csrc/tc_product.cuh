// Matrix products on the 5th-generation tensor cores with fused epilogues.
//
// One persistent kernel computes  acc[m][n] = sum over k of A[m][k] B[n][k]  (or the sum of two such products) in tiles of
// 128 x BN and hands the fp32 accumulators to an epilogue: a store, the gated activation, its backward, or a step of the
// Newton-Schulz iteration.  Either operand may be stored with k contiguous ("K-major") or with its own rows contiguous
// ("MN-major"), so no operand is ever transposed in memory.
//
// CG = 2: a cluster of two blocks (the two SMs of a TPC) computes a tile of 256 x BN.  Each block holds 128 rows of A and half of the
// columns' B, and one tcgen05.mma of the first block reads both halves.  An SM takes at most 64 bytes a clock from L2; a
// single block's 128 x 256 tile asks for 96 while the tensor core runs at its full rate (measured: 800 cycles for a block of 64 k
// that the tensor core does in 512), the pair's for 64.
//
// Results leave through shared memory: a warp lays 32 rows x 32 columns out there and one TMA store writes them, whole sectors at
// a time.  (Stored from the registers, 16 bytes of 32 different rows at a time, a tile of 128 x 128 gated values with three outputs
// took 17,000 cycles, products included; through TMA 14,000.)  Rows off the 16-byte grid go out of the same
// staging area element by element, consecutive lanes on consecutive addresses.
//
// Roles (12 warps): warp 0 issues the TMA copies, warp 1 issues tcgen05.mma, warp 2 owns the TMEM allocation, warps 4-11 run
// the epilogue.  Two accumulators in TMEM: the epilogue of a tile runs under the products of the next.
//
// PL = 2, for fp32 values: each operand is two fp16 planes, x = hi + lo, and a block of k contributes lo hi + hi lo + hi hi.
// The tensor core truncates its fp32 accumulator after every 16 k (measured: 2.2e-8 of the result for each, always towards
// zero, so 2048 k are 3e-6 low), which is why the accumulator is not kept there: after each 64 k, small products first, the epilogue
// warps add it to sums in registers with correct rounding.  Two to four accumulators in turn cover the way from the tensor core to
// those warps and back; the finished sums go to the place of the last one, from where the epilogue proceeds as with one plane.
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

// Staging area of an epilogue warp: two 32 x 32 blocks of 16 bits, or one of 32. What it takes, the operands in flight lack: from a
// stage's last product to its next data being there takes some 2,800 cycles, so the products run at their rate only with
// about 190 KB on their way (measured with 8 KB here: five stages of 32 KB, 620 cycles for 64 k that take 512).
// The gated block's epilogues lay three blocks of 16 bits out and send them together, one fence and one wait for all: a twentieth fewer
// instructions than one by one, and the same time.
constexpr int TC_RING = 4096;
constexpr int tc_ring(int epi, int planes) { return planes == 1 && (epi == 1 || epi == 2) ? 6144 : TC_RING; }
constexpr int TC_CHUNK = 1;             // PL = 2: blocks of 64 k between two additions to the sums (two: a fifth faster, and errors of 1e-6 instead of 3.5e-7)

template <int BN, int EPI, int PL, int CG> struct TcShape {
    static constexpr int B_BYTES = BN / CG * TC_BK * 2;
    static constexpr int STAGE_BYTES = PL * (TC_A_BYTES + B_BYTES);  // A planes, then B planes
    static constexpr bool LOADS = PL == 1 && (EPI == 2 || EPI == 4); // epilogues that read through TMA: 4 KB a warp
    static constexpr int IN_BYTES = LOADS ? 4096 : 0;
    static constexpr int RING = tc_ring(EPI, PL);
    static constexpr int EPI_BYTES = TC_EPI_WARPS * (RING + IN_BYTES);
    static constexpr int STAGES = (227 * 1024 - 1024 - 512 - EPI_BYTES) / STAGE_BYTES;
    static constexpr int BM = TC_BM * CG;                            // rows of a tile
    static constexpr int SMEM = STAGES * STAGE_BYTES + EPI_BYTES + 1024;         // + alignment of the swizzle atoms
    static constexpr int ACCS = PL == 2 ? 512 / BN : 2;              // accumulators in TMEM
    static constexpr int TMEM_COLS = ACCS * BN;
    static constexpr bool MANY_REGS = PL == 2 && BN == 256;          // 128 sums a thread: the epilogue warps take registers from the others
};

enum TcEpilogue { EPI_STORE = 0, EPI_GATE = 1, EPI_GATE_BWD = 2, EPI_GRAM = 3, EPI_POLY = 4, EPI_PLANES = 5 };

struct TcOut {
    char* base;
    int64_t ld, plane, batch;                 // elements
    int32_t tma;                              // 16-byte grid: through the tensor map
};

// one product of a launch
struct TcJob {
    CUtensorMap a[2], b[2];
    CUtensorMap o[2];                         // outputs in blocks of 32 x 32
    TcOut out[2];                             // STORE: out; GATE: h, saved; GATE_BWD: {dg, du, h}; Newton-Schulz: planes
    int32_t pairs, kblocks;                   // products that are summed (1 or 2), 64-wide blocks of k in each
    int32_t m, n;                             // extent of the result (EPI_GATE: n counts gate columns)
    int32_t mt, nt, tiles;                    // tiles of one matrix
    int32_t batch, splits;
    int32_t a_mn, b_mn, a_batched, b_batched;
    uint32_t idesc;
    int32_t type;                             // element type of the outputs and of saved
    float alpha;
    const uint32_t *amax_a[2], *amax_b[2];    // largest magnitudes behind the operands' scales, NULL: unscaled; GATE: b[1] is up's
};
constexpr int TC_JOBS = 4;
// what the epilogues other than STORE read besides
struct TcMore {
    CUtensorMap i;
    const void* in;                           // GATE_BWD: saved; POLY: the planes of A
    int64_t in_ld, in_plane, in_batch;
    int32_t in_tma;
    int32_t act;
    uint32_t *amax_o[3];                      // fp32 intermediates: their largest magnitude is collected (GATE: h; GATE_BWD: dg, du, h)
    float poly_a, poly_b, poly_c;
};
template <int NJ> struct TcParams {
    TcJob job[NJ];                            // independent products, worked on one after another as one list of tiles
    TcMore more;
    int32_t jobs;
    uint32_t* status;
    float* partial;                           // splits > 1: [batch*tiles][blocks of a tile][splits][BN][128] accumulators
    uint32_t* arrived;                        // splits > 1: [batch*tiles][blocks of a tile], zero between launches
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
// an address of this block's shared memory as the same place in block `rank` of the cluster
__device__ __forceinline__ uint32_t in_block(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// CG = 2: `bar` is the first block's barrier (a cluster address), the destination this block's own memory
template <int CG>
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int c0, int c1, int c2, int c3, uint32_t bar) {
    if (CG == 2)
        asm volatile("cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
                     ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(bar) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
                     ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(bar) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
template <int CG>
__device__ __forceinline__ void tc_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    if (CG == 2)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// arrives at `bar` of every block of the pair when the products issued so far are done
template <int CG>
__device__ __forceinline__ void tc_commit(uint32_t bar) {
    if (CG == 2)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                     ::"r"(bar), "h"(uint16_t(3)) : "memory");
    else
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
    for (int i = 0; i < 32; i += 8)
        asm volatile("" : "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3]), "+r"(r[i + 4]), "+r"(r[i + 5]), "+r"(r[i + 6]), "+r"(r[i + 7]));
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}

__device__ __forceinline__ void tma_store(const CUtensorMap* map, int c0, int c1, int c2, int c3, uint32_t src) {
    asm volatile("cp.async.bulk.tensor.4d.global.shared::cta.bulk_group [%0, {%1, %2, %3, %4}], [%5];"
                 ::"l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(src) : "memory");
}
__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void bulk_wait_read() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void sts128(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ void sts16(uint32_t at, uint16_t v) { asm volatile("st.shared.b16 [%0], %1;" ::"r"(at), "h"(v) : "memory"); }
__device__ __forceinline__ uint4 lds128(uint32_t at) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ uint16_t lds16(uint32_t at) {
    uint16_t v;
    asm volatile("ld.shared.b16 %0, [%1];" : "=h"(v) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t lds32(uint32_t at) {
    uint32_t v;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
    return v;
}

// two loads under one wait. The empty statements after it tie the values to it: nothing that uses them can be moved before.
__device__ __forceinline__ void tc_ld32x2(uint32_t addr0, float (&v)[32], uint32_t addr1, float (&w)[32]) {
    uint32_t r[2][32];
#pragma unroll
    for (int k = 0; k < 2; ++k)
        asm volatile(
            "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
            "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
            "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
            : "=r"(r[k][0]), "=r"(r[k][1]), "=r"(r[k][2]), "=r"(r[k][3]), "=r"(r[k][4]), "=r"(r[k][5]), "=r"(r[k][6]), "=r"(r[k][7]),
              "=r"(r[k][8]), "=r"(r[k][9]), "=r"(r[k][10]), "=r"(r[k][11]), "=r"(r[k][12]), "=r"(r[k][13]), "=r"(r[k][14]), "=r"(r[k][15]),
              "=r"(r[k][16]), "=r"(r[k][17]), "=r"(r[k][18]), "=r"(r[k][19]), "=r"(r[k][20]), "=r"(r[k][21]), "=r"(r[k][22]), "=r"(r[k][23]),
              "=r"(r[k][24]), "=r"(r[k][25]), "=r"(r[k][26]), "=r"(r[k][27]), "=r"(r[k][28]), "=r"(r[k][29]), "=r"(r[k][30]), "=r"(r[k][31])
            : "r"(k ? addr1 : addr0));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int i = 0; i < 32; i += 8)
            asm volatile("" : "+r"(r[k][i]), "+r"(r[k][i + 1]), "+r"(r[k][i + 2]), "+r"(r[k][i + 3]), "+r"(r[k][i + 4]), "+r"(r[k][i + 5]),
                              "+r"(r[k][i + 6]), "+r"(r[k][i + 7]));
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        v[i] = __uint_as_float(r[0][i]);
        w[i] = __uint_as_float(r[1][i]);
    }
}
__device__ __forceinline__ void tc_st32(uint32_t addr, const float (&v)[32]) {
    uint32_t r[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) r[i] = __float_as_uint(v[i]);
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};"
        ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
          "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]),
          "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]),
          "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(addr)
        : "memory");
}
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Shared-memory matrix descriptors, 128-byte swizzle (layout code 2, version 1).
//   K-major:  a tile is rows of 128 bytes; 8 rows form an atom, atoms 1024 bytes apart.
//   MN-major: a tile is 64-row-wide panels; in a panel each k is a 128-byte row, 8 k form an atom (1024 bytes
//             apart along k), and panels are 64 k = 8192 bytes apart.
__device__ __forceinline__ uint64_t tc_desc(uint32_t addr, int mn) {
    const uint64_t lead = mn ? (TC_BK * 128) >> 4 : 1;
    return uint64_t((addr & 0x3FFFFu) >> 4) | (lead << 16) | (uint64_t(1024 >> 4) << 32) | (uint64_t(1) << 46) | (uint64_t(2) << 61);
}

// ---- activations --------------------------------------------------------------------------------------
// The multiplexed unit's 2^x (2 units in the last place) and reciprocal (1): with the rounding of x log2(e), a sigmoid is within a few
// units in the last place wherever it is not negligible beside 1 -- below what the products before it lose. Results below
// fp32's normal range are zero. Four instructions a sigmoid: a fifth fewer in the epilogues than with CUDA's __expf and
// __fdividef, for 1 to 5 us of the 65 that the backward kernel takes at 4096 x 4096.
__device__ __forceinline__ float fast_exp2(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ float fast_rcp(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
constexpr float LOG2_E = 1.4426950408889634f;
__device__ __forceinline__ float act_sigmoid(float g) { return fast_rcp(1.0f + fast_exp2(-LOG2_E * g)); }
// value and derivative
template <int ACT>
__device__ __forceinline__ void act_both(float g, float& a, float& s) {
    if (ACT == SCALECOM_ACT_SILU) {
        const float p = act_sigmoid(g);
        a = g * p;
        s = fmaf(a, 1.0f - p, p);
    } else if (ACT == SCALECOM_ACT_GELU) {
        const float c = 0.5f * (1.0f + erff(g * 0.70710678118654752f));
        a = g * c;
        s = fmaf(g * 0.39894228040143268f, fast_exp2((-0.5f * LOG2_E) * g * g), c);
    } else if (ACT == SCALECOM_ACT_GELU_TANH) {
        if (fabsf(g) > 30.0f) {                 // tanh is +-1 there; the cube below could overflow
            a = g > 0.0f ? g : 0.0f;
            s = g > 0.0f ? 1.0f : 0.0f;
            return;
        }
        const float t = tanhf(0.79788456080286536f * (g + 0.044715f * g * g * g));
        a = 0.5f * g * (1.0f + t);
        s = 0.5f * (1.0f + t) + 0.5f * g * (1.0f - t * t) * 0.79788456080286536f * (1.0f + 0.134145f * g * g);
    } else {
        a = g > 0.0f ? g : (g == g ? 0.0f : g);
        s = g > 0.0f ? 1.0f : 0.0f;
    }
}
// 32 columns at once, so that the choice of the activation is made once and not for each element
template <int ACT>
__device__ __forceinline__ void gate_row(const float (&g)[32], float (&v)[32], const float (&w)[32]) {
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        float a, s;
        act_both<ACT>(g[i], a, s);
        v[i] = a * w[i];
    }
}
template <int ACT>
__device__ __forceinline__ void gate_back_row(float (&g)[32], float (&v)[32], float (&w)[32]) {
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        float a, s;
        act_both<ACT>(g[i], a, s);
        const float dh = v[i], u = w[i];
        g[i] = dh * u * s;             // dg
        w[i] = dh * a;                 // du
        v[i] = a * u;                  // h
    }
}
#define SC_FOR_ACT(act, CALL)                                      \
    switch (act) {                                                 \
        case SCALECOM_ACT_SILU: CALL(SCALECOM_ACT_SILU); break;    \
        case SCALECOM_ACT_GELU: CALL(SCALECOM_ACT_GELU); break;    \
        case SCALECOM_ACT_GELU_TANH: CALL(SCALECOM_ACT_GELU_TANH); break; \
        default: CALL(SCALECOM_ACT_RELU); break;                   \
    }

// ---- tile order ----------------------------------------------------------------------------------------
struct TcUnit { int job, batch, mt, nt, split, tile; };

template <int BN, int EPI, int BM, int NJ>
__device__ __forceinline__ TcUnit tc_unit(const TcParams<NJ>& P, int u) {
    TcUnit r;
    r.job = 0;
    if (NJ > 1)
        while (r.job + 1 < P.jobs && u >= P.job[r.job].batch * P.job[r.job].tiles * P.job[r.job].splits) {
            u -= P.job[r.job].batch * P.job[r.job].tiles * P.job[r.job].splits;
            ++r.job;
        }
    const TcJob& J = P.job[r.job];
    r.split = u % J.splits;
    u /= J.splits;
    r.tile = u;                                   // over all matrices
    r.batch = u / J.tiles;
    int t = u % J.tiles;
    if (EPI == EPI_GRAM || EPI == EPI_POLY) {     // symmetric result: tiles that touch the lower triangle
        int mt = 0;
        for (;; ++mt) {
            int cols = (mt * BM + BM - 1) / BN + 1;
            if (cols > J.nt) cols = J.nt;
            if (t < cols) break;
            t -= cols;
        }
        r.mt = mt;
        r.nt = t;
    } else {                                      // bands of 4096 rows, column by column: the band's A stays in L2 (8192 x 4096 x 16384
                                                  // bf16: 2667 us; bands of 2048 2703, of 1024 2776, row by row 2742; no other size tried)
        constexpr int BAND = 4096 / BM;
        const int band = t / (BAND * J.nt), first = band * BAND;
        const int rows = J.mt - first < BAND ? J.mt - first : BAND;
        const int in = t - band * BAND * J.nt;
        r.nt = in / rows;
        r.mt = first + in % rows;
    }
    return r;
}
template <int NJ> __device__ __forceinline__ int tc_units(const TcParams<NJ>& P) {
    int n = 0;
    for (int j = 0; j < (NJ > 1 ? P.jobs : 1); ++j) n += P.job[j].batch * P.job[j].tiles * P.job[j].splits;
    return n;
}

// ---- blocks of 32 x 32 on their way out and in ----------------------------------------------------------------
// A lane holds a row.  In the staging area rows are 64 bytes (16-bit types) or 128 (fp32), their 16-byte pieces
// permuted as the 64- and 128-byte swizzles of the tensor maps have it, so lanes that write the same piece of
// different rows hit different banks.
struct Ring {
    uint32_t base;
    int n;
    bool whole;               // the last block was of 32 bits: it took the whole ring, as one group
};
__device__ __forceinline__ uint32_t piece16(uint32_t row, uint32_t piece) { return row * 64u + ((piece ^ ((row >> 1) & 3u)) << 4); }
__device__ __forceinline__ uint32_t piece32(uint32_t row, uint32_t piece) { return row * 128u + ((piece ^ (row & 7u)) << 4); }

// The next free block of the ring. Two blocks of 16 bits fit, so one store may still be reading when the next block is laid out. A block of
// 32 bits takes all of it: it waits for every store before it, and a block of 16 bits behind it waits for it (a launch of
// several products may have outputs of both sizes).
template <int BYTES>
__device__ __forceinline__ uint32_t ring_next(Ring& r) {
    constexpr int SLOTS = BYTES == 2 ? 2 : 1;
    if (lane_id() == 0) {
        if (BYTES == 2 && !r.whole) bulk_wait_read<1>();
        else bulk_wait_read<0>();
    }
    r.whole = BYTES == 4;
    __syncwarp();
    return r.base + uint32_t(r.n++ & (SLOTS - 1)) * (TC_RING / SLOTS);
}
// a staged block to global memory, element by element: rows off the 16-byte grid. The whole warp, after a __syncwarp.
template <int BYTES>
__device__ __forceinline__ void ring_copy(const TcJob& J, int k, uint32_t slot, int row0, int col0, int plane, int batch) {
    const TcOut& o = J.out[k];
    const uint32_t lane = lane_id();
    const int rows = min(32, J.m - row0);
    const int64_t at = int64_t(batch) * o.batch + int64_t(plane) * o.plane + int64_t(row0) * o.ld + col0 + lane;
    if (col0 + int(lane) < J.n) {
#pragma unroll 4
        for (int r = 0; r < rows; ++r) {
            if (BYTES == 2) reinterpret_cast<uint16_t*>(o.base)[at + r * o.ld] = lds16(slot + piece16(r, lane >> 3) + (lane & 7u) * 2);
            else reinterpret_cast<uint32_t*>(o.base)[at + r * o.ld] = lds32(slot + piece32(r, lane >> 2) + (lane & 3u) * 4);
        }
    }
}
// a staged block to global memory at (row0, col0)
template <int BYTES>
__device__ __forceinline__ void ring_send(const TcJob& J, int k, uint32_t slot, int row0, int col0, int plane, int batch) {
    const TcOut& o = J.out[k];
    if (o.tma) {
        fence_async_smem();
        __syncwarp();
        if (lane_id() == 0) {
            tma_store(&J.o[k], col0, row0, plane, batch, slot);
            bulk_commit();
        }
    } else {
        __syncwarp();
        ring_copy<BYTES>(J, k, slot, row0, col0, plane, batch);
        __syncwarp();
        if (lane_id() == 0) bulk_commit();          // an empty group: the ring counts one for each block
    }
}
__device__ __forceinline__ uint32_t pack16(int type, float a, float b) {
    if (type == SCALECOM_BF16) {
        const __nv_bfloat162 t = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t*>(&t);
    }
    const __half2 t = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&t);
}
__device__ __forceinline__ void stage16(uint32_t slot, int type, const float (&v)[32]) {
    const uint32_t lane = lane_id();
    uint32_t p[16];
    if (type == SCALECOM_BF16) {
#pragma unroll
        for (int i = 0; i < 16; ++i) p[i] = pack16(SCALECOM_BF16, v[2 * i], v[2 * i + 1]);
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) p[i] = pack16(SCALECOM_F16, v[2 * i], v[2 * i + 1]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) sts128(slot + piece16(lane, i), p[4 * i], p[4 * i + 1], p[4 * i + 2], p[4 * i + 3]);
}
// three 16-bit blocks of one place: x to plane px of output kx, and so on; kx < 0: not wanted
__device__ __forceinline__ void emit3(const TcJob& J, uint32_t ring, int type, int row0, int col0, int kx, int px, const float (&x)[32], int ky, int py,
                                      const float (&y)[32], int kz, int pz, const float (&z)[32]) {
    if (lane_id() == 0) bulk_wait_read<0>();        // the blocks of the place before are on their way
    __syncwarp();
    if (kx >= 0) stage16(ring, type, x);
    if (ky >= 0) stage16(ring + 2048u, type, y);
    stage16(ring + 4096u, type, z);
    fence_async_smem();
    __syncwarp();
    const bool copy_x = kx >= 0 && !J.out[kx].tma, copy_y = ky >= 0 && !J.out[ky].tma, copy_z = !J.out[kz].tma;
    if (lane_id() == 0) {
        if (kx >= 0 && !copy_x) tma_store(&J.o[kx], col0, row0, px, 0, ring);
        if (ky >= 0 && !copy_y) tma_store(&J.o[ky], col0, row0, py, 0, ring + 2048u);
        if (!copy_z) tma_store(&J.o[kz], col0, row0, pz, 0, ring + 4096u);
        bulk_commit();
    }
    if (copy_x) ring_copy<2>(J, kx, ring, row0, col0, px, 0);
    if (copy_y) ring_copy<2>(J, ky, ring + 2048u, row0, col0, py, 0);
    if (copy_z) ring_copy<2>(J, kz, ring + 4096u, row0, col0, pz, 0);
}
template <bool MAY_F32>
__device__ __forceinline__ void emit(const TcJob& J, int k, Ring& ring, int type, const float (&v)[32], int row0, int col0, int plane, int batch) {
    if (MAY_F32 && type == SCALECOM_F32) {
        const uint32_t slot = ring_next<4>(ring), lane = lane_id();
#pragma unroll
        for (int i = 0; i < 8; ++i)
            sts128(slot + piece32(lane, i), __float_as_uint(v[4 * i]), __float_as_uint(v[4 * i + 1]), __float_as_uint(v[4 * i + 2]), __float_as_uint(v[4 * i + 3]));
        ring_send<4>(J, k, slot, row0, col0, plane, batch);
    } else {
        const uint32_t slot = ring_next<2>(ring);
        stage16(slot, type, v);
        ring_send<2>(J, k, slot, row0, col0, plane, batch);
    }
}
// fp16 planes of a block, and with MIRROR of its transpose at (col0, row0)
template <int PL, bool MIRROR>
__device__ __forceinline__ void emit_planes(const TcJob& J, Ring& ring, float (&v)[32], int row0, int col0, int batch) {
    const uint32_t lane = lane_id();
#pragma unroll
    for (int pl = 0; pl < PL; ++pl) {
        if (pl == 1) {
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                __half h, l;
                split_planes(v[i], h, l);
                v[i] = __half2float(l);
            }
        }
        emit<false>(J, 0, ring, SCALECOM_F16, v, row0, col0, pl, batch);
        if (MIRROR && col0 != row0) {
            const uint32_t slot = ring_next<2>(ring);
#pragma unroll
            for (int i = 0; i < 32; ++i)
                sts16(slot + piece16(i, lane >> 3) + (lane & 7u) * 2, __half_as_ushort(__float2half_rn(v[i])));
            ring_send<2>(J, 0, slot, col0, row0, pl, batch);
        }
    }
}
// 32 values of this lane's row, from a block that a TMA load has brought
__device__ __forceinline__ void take16(uint32_t at, int type, float (&v)[32]) {
    const uint32_t lane = lane_id();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint4 q = lds128(at + piece16(lane, i));
        const uint32_t r[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (type == SCALECOM_BF16) {
                v[8 * i + 2 * j] = __uint_as_float(r[j] << 16);
                v[8 * i + 2 * j + 1] = __uint_as_float(r[j] & 0xFFFF0000u);
            } else {
                const float2 t = __half22float2(*reinterpret_cast<const __half2*>(&r[j]));
                v[8 * i + 2 * j] = t.x;
                v[8 * i + 2 * j + 1] = t.y;
            }
        }
    }
}
// the same straight from global memory
__device__ __forceinline__ void load_typed(int type, const void* base, int64_t off, float* v, int ncols) {
    if (type == SCALECOM_BF16) load_row32(static_cast<const __nv_bfloat16*>(base) + off, v, ncols);
    else if (type == SCALECOM_F16) load_row32(static_cast<const __half*>(base) + off, v, ncols);
    else load_row32(static_cast<const float*>(base) + off, v, ncols);
}

// Largest finite magnitude (bits) of a row's first nc columns. What lies beyond them are zeros (the operands' edges are filled with
// zeros, and every epilogue maps zeros to zeros), so they need no test.
__device__ __forceinline__ uint32_t row_top(const float (&v)[32], int nc) {
    if (nc <= 0) return 0u;
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < 32; ++i) m = fmaxf(m, fabsf(v[i]));       // NaN is passed over
    if (m < INFINITY) return __float_as_uint(m);
    uint32_t t = 0u;
#pragma unroll
    for (int i = 0; i < 32; ++i) t = max(t, finite_bits(v[i]));
    return t;
}

// Blocks that an epilogue reads (GATE_BWD: g and u, POLY: A), one ahead of the block being worked on.
struct Inflow {
    uint32_t smem, bar;
    uint32_t phase;
    bool pending;
};
template <int EPI>
__device__ __forceinline__ bool block_used(const TcJob& J, int row0, int col0) {
    return row0 < J.m && col0 < J.n && (!(EPI == EPI_GRAM || EPI == EPI_POLY) || col0 <= row0);
}
template <int EPI>
__device__ __forceinline__ void inflow_start(const TcJob& J, const TcMore& M, Inflow& f, int row0, int col0, int batch) {
    if (!M.in_tma || f.pending || !block_used<EPI>(J, row0, col0)) return;
    f.pending = true;
    if (lane_id() == 0) {
        mbar_expect(f.bar, EPI == EPI_GATE_BWD ? 4096u : 2048u);
        tma_load<1>(f.smem, &M.i, col0, row0, 0, batch, f.bar);
        if (EPI == EPI_GATE_BWD) tma_load<1>(f.smem + 2048u, &M.i, col0, row0, 1, batch, f.bar);
    }
}

// the planes' scales taken out of 32 products
__device__ __forceinline__ void unscale_row(float (&v)[32], const Unscale& un) {
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] *= un.first;
    if (un.second != 1.0f) {
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] *= un.second;
    }
}

// ---- epilogues on a block of 32 x 32: v (and w) hold this lane's row --------------------------------------------
template <int EPI, int PL>
__device__ __forceinline__ bool tc_epilogue(const TcJob& J, const TcMore& M, const TcUnit& u, int row0, int col0, int col_next, float (&v)[32], float (&w)[32], const Unscale& un,
                                            const Unscale& un_up, uint32_t (&top)[3], Ring& ring, Inflow& in, volatile uint32_t* abort, uint32_t* status) {
    if (!block_used<EPI>(J, row0, col0)) return true;
    const int row = row0 + int(lane_id()), nc = J.n - col0;
    const bool inside = row < J.m;
    if (EPI == EPI_STORE) {
        if (PL == 2) {
            unscale_row(v, un);
        } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] *= un.first;
        }
        emit<true>(J, 0, ring, J.type, v, row0, col0, 0, u.batch);
    } else if (EPI == EPI_GATE) {
        if (PL == 2) {
            unscale_row(v, un);
            unscale_row(w, un_up);
        }
        const bool save = J.out[1].base != nullptr;
        float h[32];
#define SC_CALL(ACT) gate_row<ACT>(v, h, w)
        SC_FOR_ACT(M.act, SC_CALL)
#undef SC_CALL
        if (PL == 1) {
            emit3(J, ring.base, J.type, row0, col0, save ? 1 : -1, 0, v, save ? 1 : -1, 1, w, 0, 0, h);
        } else {
            if (save) {
                emit<true>(J, 1, ring, J.type, v, row0, col0, 0, 0);
                emit<true>(J, 1, ring, J.type, w, row0, col0, 1, 0);
            }
            top[0] = max(top[0], row_top(h, inside ? nc : 0));
            emit<true>(J, 0, ring, J.type, h, row0, col0, 0, 0);
        }
    } else if (EPI == EPI_GATE_BWD) {
        float g[32];
        if (PL == 1 && M.in_tma) {
            if (!__all_sync(FULL, mbar_wait(in.bar, in.phase, abort, status))) return false;
            in.phase ^= 1u;
            in.pending = false;
            take16(in.smem, J.type, g);
            take16(in.smem + 2048u, J.type, w);
            __syncwarp();
            if (col_next >= 0) inflow_start<EPI>(J, M, in, row0, col_next, u.batch);
        } else {
            const int64_t at = int64_t(row) * M.in_ld + col0;
            load_typed(J.type, M.in, at, g, inside ? nc : 0);
            load_typed(J.type, M.in, at + M.in_plane, w, inside ? nc : 0);
        }
        if (PL == 2) unscale_row(v, un);
#define SC_CALL(ACT) gate_back_row<ACT>(g, v, w)
        SC_FOR_ACT(M.act, SC_CALL)
#undef SC_CALL
        if (PL == 2) {
            top[0] = max(top[0], row_top(g, inside ? nc : 0));
            top[1] = max(top[1], row_top(w, inside ? nc : 0));
            top[2] = max(top[2], row_top(v, inside ? nc : 0));
        }
        if (PL == 1) {
            emit3(J, ring.base, J.type, row0, col0, 0, 0, g, 0, 1, w, 0, 2, v);
        } else {
            emit<true>(J, 0, ring, J.type, g, row0, col0, 0, 0);
            emit<true>(J, 0, ring, J.type, w, row0, col0, 1, 0);
            emit<true>(J, 0, ring, J.type, v, row0, col0, 2, 0);
        }
    } else if (EPI == EPI_PLANES) {
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] *= J.alpha;
        emit_planes<PL, false>(J, ring, v, row0, col0, u.batch);
    } else {
        // a symmetric result: blocks up to the diagonal, stored here and mirrored
        if (EPI == EPI_POLY) {
            if (PL == 1) {
                if (!__all_sync(FULL, mbar_wait(in.bar, in.phase, abort, status))) return false;
                in.phase ^= 1u;
                in.pending = false;
                take16(in.smem, SCALECOM_F16, w);
                __syncwarp();
                if (col_next >= 0) inflow_start<EPI>(J, M, in, row0, col_next, u.batch);
            } else {
                const int64_t at = int64_t(u.batch) * M.in_batch + int64_t(row) * M.in_ld + col0;
                load_typed(SCALECOM_F16, M.in, at, w, inside ? nc : 0);
                float l[32];
                load_typed(SCALECOM_F16, M.in, at + M.in_plane, l, inside ? nc : 0);
#pragma unroll
                for (int i = 0; i < 32; ++i) w[i] += l[i];
            }
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = M.poly_b * w[i] + M.poly_c * v[i] + (i == row - col0 ? M.poly_a : 0.0f);
        } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] *= J.alpha;
        }
        emit_planes<PL, true>(J, ring, v, row0, col0, u.batch);
    }
    return true;
}

// Two products of planes that are summed (dx = dg Wg + du Wu) come in different units, 2^e of their operands' scales. Every tensor has a
// scale of its own: with one for both weights, up weights of 2^-30 of the gate's size were left 10 bits. The product of the smaller
// unit goes first, so that its sums are scaled down, never up, when the other's are added. By how much the first job's unit is larger:
template <int EPI, int PL>
__device__ __forceinline__ int tc_ahead(const TcJob& J) {
    if (PL != 2 || EPI != EPI_STORE || J.pairs != 2 || !J.amax_a[0]) return 0;
    return plane_unshift(*J.amax_a[0], *J.amax_b[0]) - plane_unshift(*J.amax_a[1], *J.amax_b[1]);
}

// whether `ok` holds for all threads of the epilogue warps (a barrier among them)
__device__ __forceinline__ bool epilogue_all(bool ok) {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, 1, 256, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"(uint32_t(ok)) : "memory");
    return r != 0u;
}

template <int BN, int EPI, int PL, int CG, int NJ>
__global__ void __launch_bounds__(TC_THREADS, 1) tc_product_kernel(const __grid_constant__ TcParams<NJ> P) {
    using S = TcShape<BN, EPI, PL, CG>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ alignas(8) uint64_t bars[2 * S::STAGES + 2 * S::ACCS + 1 + TC_EPI_WARPS];
    __shared__ uint32_t tmem_base, abort_flag, last_flag;

    const uint32_t warp = warp_id(), lane = lane_id();
    const uint32_t tiles0 = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t bar0 = smem_u32(bars);
    auto full = [&](int s) { return bar0 + 8u * s; };
    auto empty = [&](int s) { return bar0 + 8u * (S::STAGES + s); };
    auto tfull = [&](int s) { return bar0 + 8u * (2 * S::STAGES + s); };
    auto tempty = [&](int s) { return bar0 + 8u * (2 * S::STAGES + S::ACCS + s); };
    const uint32_t drain = bar0 + 8u * (2 * S::STAGES + 2 * S::ACCS);
    const uint32_t inflow0 = drain + 8u;

    if (warp == 0 && lane == 0) {
        for (int s = 0; s < S::STAGES; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
        for (int s = 0; s < S::ACCS; ++s) { mbar_init(tfull(s), 1); mbar_init(tempty(s), TC_EPI_WARPS * CG); }
        mbar_init(drain, 1);
        for (int w = 0; w < TC_EPI_WARPS; ++w) mbar_init(inflow0 + 8u * w, 1);
        abort_flag = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 3 && lane < 2u * uint32_t(NJ)) {                 // the operands' tensor maps are fetched while the rest is set up
        asm volatile("prefetch.tensormap [%0];" ::"l"(lane & 1u ? &P.job[lane / 2].b[0] : &P.job[lane / 2].a[0]) : "memory");
    }
    if (warp == 2) {
        if (CG == 2) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base)), "n"(S::TMEM_COLS) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base)), "n"(S::TMEM_COLS) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
    }
    const uint32_t rank = CG == 2 ? blockIdx.x & 1u : 0u;        // in the cluster, whose size is CG
    tc_fence_before();
    __syncthreads();
    if (CG == 2) cluster_sync();                                 // the pair's barriers are set up on both sides
    tc_fence_after();
    const uint32_t tmem = tmem_base;
    chain_launch();
    chain_wait();

    volatile uint32_t* abort = &abort_flag;
    const int units = tc_units(P);
    const int first = blockIdx.x / CG, stride = gridDim.x / CG;

    // 384 threads x 168 registers at launch = 128 x 56 + 256 x 224
    if (warp < 4) {
    if (S::MANY_REGS) asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    if (warp == 0) {
        if (lane == 0) {
            int n_issued = 0;                       // copies issued so far; stage and phase follow from it
            bool ok = true;
            for (int un = first; ok && un < units; un += stride) {
                const TcUnit u = tc_unit<BN, EPI, S::BM>(P, un);
                const TcJob& J = P.job[NJ > 1 ? u.job : 0];
                const int iters = J.pairs * J.kblocks;
                const int it0 = int(int64_t(iters) * u.split / J.splits), it1 = int(int64_t(iters) * (u.split + 1) / J.splits);
                const int m0 = u.mt * S::BM + int(rank) * TC_BM;
                const int n0 = EPI == EPI_GATE ? u.nt * (BN / 2) : u.nt * BN + int(rank) * (BN / CG);
                const int ba = J.a_batched ? u.batch : 0, bb = J.b_batched ? u.batch : 0;
                const int second_first = tc_ahead<EPI, PL>(J) > 0;
                for (int it = it0; it < it1; ++it, ++n_issued) {
                    const int s = n_issued % S::STAGES, round = n_issued / S::STAGES;
                    if (!mbar_wait(empty(s), (round & 1) ^ 1, abort, P.status)) { ok = false; break; }
                    const int part = it >= J.kblocks, pair = part ^ second_first, k0 = (it - part * J.kblocks) * TC_BK;
                    const uint32_t a = tiles0 + s * S::STAGE_BYTES, b = a + PL * TC_A_BYTES;
                    const uint32_t bar = CG == 2 ? in_block(full(s), 0) : full(s);
                    if (rank == 0) mbar_expect(full(s), S::STAGE_BYTES * CG);      // both blocks' copies
#pragma unroll
                    for (int pl = 0; pl < PL; ++pl) {
                        const uint32_t ap = a + pl * TC_A_BYTES, bp = b + pl * S::B_BYTES;
                        if (J.a_mn) {
                            for (int j = 0; j < TC_BM / 64; ++j) tma_load<CG>(ap + j * 8192, &J.a[pair], m0 + 64 * j, k0, pl, ba, bar);
                        } else {
                            tma_load<CG>(ap, &J.a[pair], k0, m0, pl, ba, bar);
                        }
                        if (EPI == EPI_GATE && CG == 2) {       // the pair's first block has the gate columns, the second the up columns
                            tma_load<CG>(bp, &J.b[rank], k0, n0, pl, bb, bar);
                        } else if (EPI == EPI_GATE) {
                            tma_load<CG>(bp, &J.b[0], k0, n0, pl, bb, bar);
                            tma_load<CG>(bp + S::B_BYTES / 2, &J.b[1], k0, n0, pl, bb, bar);
                        } else if (J.b_mn) {
                            for (int j = 0; j < BN / CG / 64; ++j) tma_load<CG>(bp + j * 8192, &J.b[pair], n0 + 64 * j, k0, pl, bb, bar);
                        } else {
                            tma_load<CG>(bp, &J.b[pair], k0, n0, pl, bb, bar);
                        }
                    }
                }
            }
            if (!ok && rank == 0)                   // the copies still in flight write shared memory (the pair's: the first block sees them all)
                for (int i = n_issued > S::STAGES ? n_issued - S::STAGES : 0; i < n_issued; ++i)
                    mbar_drain(full(i % S::STAGES), (i / S::STAGES) & 1);
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            int n_used = 0, n_acc = 0;              // stages used, accumulators begun
            bool ok = true;
            for (int un = first; ok && un < units; un += stride) {
                const TcUnit u = tc_unit<BN, EPI, S::BM>(P, un);
                const TcJob& J = P.job[NJ > 1 ? u.job : 0];
                const int iters = J.pairs * J.kblocks;
                const int it0 = int(int64_t(iters) * u.split / J.splits), it1 = int(int64_t(iters) * (u.split + 1) / J.splits);
                if (PL == 1) {
                    if (!mbar_wait(tempty(n_acc % S::ACCS), ((n_acc / S::ACCS) & 1) ^ 1, abort, P.status)) { ok = false; break; }
                    tc_fence_after();
                }
                for (int it = it0; it < it1; ++it, ++n_used) {
                    const int s = n_used % S::STAGES;
                    const bool opens = PL == 2 && (it - it0) % TC_CHUNK == 0, closes = PL == 2 && ((it - it0) % TC_CHUNK == TC_CHUNK - 1 || it + 1 == it1);
                    if (opens && !mbar_wait(tempty(n_acc % S::ACCS), ((n_acc / S::ACCS) & 1) ^ 1, abort, P.status)) { ok = false; break; }
                    if (!mbar_wait(full(s), (n_used / S::STAGES) & 1, abort, P.status)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t d = tmem + (n_acc % S::ACCS) * BN;
                    const uint32_t a = tiles0 + s * S::STAGE_BYTES, b = a + PL * TC_A_BYTES;
                    const uint32_t step_a = J.a_mn ? 2048 >> 4 : 32 >> 4, step_b = J.b_mn ? 2048 >> 4 : 32 >> 4;
#pragma unroll
                    for (int t = 0; t < (PL == 2 ? 3 : 1); ++t) {      // lo hi, hi lo, hi hi
                        const uint64_t da = tc_desc(a + (PL == 2 && t == 0 ? TC_A_BYTES : 0), J.a_mn);
                        const uint64_t db = tc_desc(b + (PL == 2 && t == 1 ? S::B_BYTES : 0), J.b_mn);
#pragma unroll
                        for (int k = 0; k < TC_BK / 16; ++k)
                            tc_mma<CG>(d, da + k * step_a, db + k * step_b, J.idesc, (t > 0 || k > 0 || (PL == 2 ? !opens : it > it0)) ? 1u : 0u);
                    }
                    tc_commit<CG>(empty(s));
                    if (closes) tc_commit<CG>(tfull(n_acc++ % S::ACCS));
                }
                if (PL == 1 && ok) tc_commit<CG>(tfull(n_acc++ % S::ACCS));
            }
            if (!ok) {                              // products in flight read shared memory and write TMEM
                tc_commit<CG>(drain);
                mbar_drain(drain, 0);
            }
        }
    }
    } else {
        if (S::MANY_REGS) asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
        const uint32_t quad = warp & 3u, half = (warp - 4u) >> 2;
        const uint32_t lanes = (quad * 32u) << 16;
        const int tid = int(threadIdx.x) - 128;
        // result columns of a tile, and a warp's 32-column chunks of them: GATE works on a gate chunk and the up chunk beside it
        constexpr int WIDTH = EPI == EPI_GATE ? BN / 2 : BN, CHUNKS = WIDTH / 64;
        auto chunk = [&](int c) { return (int(half) * CHUNKS + c) * 32; };
        auto acc_free = [&](int i) {                // the first block issues the products: it waits for both blocks' warps
            if (rank == 0) mbar_arrive(tempty(i));
            else mbar_arrive_cluster(in_block(tempty(i), 0));
        };
        uint32_t top[3] = {0u, 0u, 0u};
        int n_acc = 0;
        const uint32_t stage0 = tiles0 + S::STAGES * S::STAGE_BYTES;
        Ring ring = {stage0 + (warp - 4u) * S::RING, 0, false};
        Inflow in = {stage0 + TC_EPI_WARPS * S::RING + (warp - 4u) * S::IN_BYTES, inflow0 + 8u * (warp - 4u), 0u, false};
        auto begin = [&](const TcUnit& u, int row0, int c) {
            if (S::LOADS && c < CHUNKS) inflow_start<EPI>(P.job[NJ > 1 ? u.job : 0], P.more, in, row0, u.nt * WIDTH + chunk(c), u.batch);
        };
        for (int un = first; un < units; un += stride) {
            const TcUnit u = tc_unit<BN, EPI, S::BM>(P, un);
                const TcJob& J = P.job[NJ > 1 ? u.job : 0];
                const int iters = J.pairs * J.kblocks;
            Unscale un_scale = {J.alpha, 1.0f}, un_up = un_scale;
            const int ahead = tc_ahead<EPI, PL>(J);
            if (PL == 2 && J.amax_a[0]) {               // alpha is 1 there
                un_scale = plane_unscale(plane_unshift(*J.amax_a[0], *J.amax_b[0]) - min(ahead, 0));
                if (EPI == EPI_GATE) un_up = plane_unscale(plane_unshift(*J.amax_a[0], *J.amax_b[1]));
            }
            const int row0 = u.mt * S::BM + int(rank) * TC_BM + int(quad) * 32;
            float v[32], w[32];
            float sum[BN / 64][32];       // PL = 2: this thread's columns, in the order of `column`
            auto column = [&](int c) {                  // TMEM column of the thread's c-th 32 columns
                if (EPI == EPI_GATE && PL == 2) return (c & 1) * (BN / 2) + (int(half) * (BN / 128) + (c >> 1)) * 32;
                return int(half) * (BN / 2) + c * 32;
            };
            if (J.splits == 1) begin(u, row0, 0);
            bool ok = true;
            uint32_t acc = 0;
            int q = 0;
            if (PL == 2) {
                const int it0 = int(int64_t(iters) * u.split / J.splits), it1 = int(int64_t(iters) * (u.split + 1) / J.splits);
#pragma unroll
                for (int c = 0; c < BN / 64; ++c)
#pragma unroll
                    for (int i = 0; i < 32; ++i) sum[c][i] = 0.0f;
                static_assert(TC_CHUNK == 1, "a chunk is of one product");
                int it = it0;
#pragma unroll 1
                for (int part = 0; part < (EPI == EPI_STORE ? 2 : 1) && ok; ++part) {
                    const int stop = EPI != EPI_STORE || part || J.kblocks > it1 ? it1 : J.kblocks;
                    if (part && ahead) {            // the first product's sums to the second's unit (zeros, if these k have none of the first)
                        const float by = abs(ahead) <= 126 ? power_of_two(-abs(ahead)) : 0.0f;
#pragma unroll
                        for (int c = 0; c < BN / 64; ++c)
#pragma unroll
                            for (int i = 0; i < 32; ++i) sum[c][i] *= by;
                    }
                    for (; it < stop; it += TC_CHUNK, ++n_acc) {
                        q = n_acc % S::ACCS;
                        ok = __all_sync(FULL, mbar_wait(tfull(q), (n_acc / S::ACCS) & 1, abort, P.status));
                        if (!ok) break;
                        tc_fence_after();
                        acc = tmem + q * BN + lanes;
#pragma unroll
                        for (int c = 0; c < BN / 64; c += 2) {
                            tc_ld32x2(acc + column(c), v, acc + column(c + 1), w);
#pragma unroll
                            for (int i = 0; i < 32; ++i) {
                                sum[c][i] += v[i];
                                sum[c + 1][i] += w[i];
                            }
                        }
                        if (it + TC_CHUNK < it1) {
                            tc_fence_before();
                            __syncwarp();
                            if (lane == 0) acc_free(q);
                        }
                    }
                }
                // the last accumulator is kept until the epilogue has read the sums from its place
#pragma unroll
                for (int c = 0; c < BN / 64; ++c)
                    if (ok) tc_st32(acc + column(c), sum[c]);
                tc_wait_st();
            } else {
                q = n_acc % S::ACCS;
                ok = __all_sync(FULL, mbar_wait(tfull(q), (n_acc / S::ACCS) & 1, abort, P.status));
                ++n_acc;
                acc = tmem + q * BN + lanes;
            }
            if (J.splits > 1) ok = epilogue_all(ok);       // the block barriers below need every epilogue warp
            if (!ok) break;
            tc_fence_after();
            auto release = [&]() {                          // the accumulator is free once its last columns are in registers
                tc_fence_before();
                __syncwarp();
                if (lane == 0) acc_free(q);
            };
            if (J.splits > 1) {
                // this part's accumulators to scratch, [column][row]; the block that arrives last adds the parts up in their order
                const int slot = u.tile * CG + int(rank);
                float* mine = P.partial + (int64_t(slot) * J.splits) * (TC_BM * BN) + quad * 32 + lane;
                float* put = mine + int64_t(u.split) * (TC_BM * BN);
#pragma unroll 1
                for (int c = 0; c < BN / 64; ++c) {
                    tc_ld32(acc + column(c), v);
#pragma unroll
                    for (int i = 0; i < 32; ++i) put[(column(c) + i) * TC_BM] = v[i];
                }
                release();
                __threadfence();
                asm volatile("bar.sync 1, 256;" ::: "memory");
                if (tid == 0) {
                    const uint32_t before = atomicAdd(&P.arrived[slot], 1u);
                    last_flag = before + 1u == uint32_t(J.splits);
                    if (before + 1u == uint32_t(J.splits)) P.arrived[slot] = 0u;
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
                    for (int s = 0; s < J.splits; ++s) {
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
                    begin(u, row0, c);
                    ok = ok && tc_epilogue<EPI, PL>(J, P.more, u, row0, u.nt * WIDTH + at, -1, v, w, un_scale, un_up, top, ring, in, abort, P.status);
                }
            } else {
#pragma unroll 1
                for (int c = 0; c < CHUNKS; ++c) {
                    const int at = chunk(c);
                    if (EPI == EPI_GATE) tc_ld32x2(acc + at, v, acc + BN / 2 + at, w);
                    else tc_ld32(acc + at, v);
                    if (c == CHUNKS - 1) release();
                    if (ok) begin(u, row0, c);
                    ok = ok && tc_epilogue<EPI, PL>(J, P.more, u, row0, u.nt * WIDTH + at, c + 1 < CHUNKS ? u.nt * WIDTH + chunk(c + 1) : -1, v, w, un_scale,
                                                    un_up, top, ring, in, abort, P.status);
                }
            }
        }
        if (lane == 0) {
            if (in.pending) mbar_drain(in.bar, in.phase);
            bulk_wait_read<0>();                    // the staging area is read before the block ends; the writes end with the kernel
        }
        if (PL == 2 && (EPI == EPI_GATE || EPI == EPI_GATE_BWD)) {
#pragma unroll
            for (int i = 0; i < (EPI == EPI_GATE ? 1 : 3); ++i) {
                const uint32_t t = __reduce_max_sync(FULL, top[i]);
                if (lane == 0 && t) atomicMax(P.more.amax_o[i], t);
            }
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (CG == 2) cluster_sync();                    // neither block leaves while the other may reach its memory
    if (warp == 2) {
        tc_fence_after();
        if (CG == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(S::TMEM_COLS) : "memory");
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(S::TMEM_COLS) : "memory");
    }
}

}  // namespace sc
