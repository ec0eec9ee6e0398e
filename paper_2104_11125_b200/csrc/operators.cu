// C-ABI of the learner-side operators (see include/scalecom_operators.h): argument checks, scratch, launches.
#include "../../include/scalecom_operators.h"

#include <cuda.h>
#include <cudaTypedefs.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <utility>

#include "ffn_tokens.cuh"
#include "layer_norm.cuh"
#include "ns_small.cuh"
#include "operand_prep.cuh"
#include "ops_common.cuh"
#include "tc_product.cuh"

using namespace sc;

struct scalecom_ops {
    int device = 0;
    int sms = 0;
    cudaStream_t stream = nullptr;
    void* ws = nullptr;                 // scratch of the calls, grown on demand
    size_t ws_bytes = 0;
    bool ws_in_graph = false;           // a call that was captured into a graph has its address
    struct Kept { void* p; Kept* next; };
    Kept* kept = nullptr;               // scratch of such graphs that has been outgrown
    uint32_t* ctrl = nullptr;           // device: [0] status, [16..] arrival counters of split products
    PFN_cuTensorMapEncodeTiled encode = nullptr;
    bool poisoned = false;
    // Blocks of a kernel that fit a multiprocessor, looked up once. In the handle, since the answer is its device's.
    struct Fit { const void* kernel; int blocks; };
    static constexpr int FITS = 512;            // more than there are layer norm kernels
    Fit fits[FITS] = {};
};

namespace {

constexpr int CTRL_WORDS = 16 + 4096;
constexpr int MAX_SPLIT_TILES = 4096;

struct DeviceGuard {
    int prev = -1;
    bool ok = false;
    explicit DeviceGuard(int dev) {
        if (cudaGetDevice(&prev) != cudaSuccess) return;
        ok = (prev == dev) || (cudaSetDevice(dev) == cudaSuccess);
    }
    ~DeviceGuard() {
        int cur = -1;
        if (prev >= 0 && cudaGetDevice(&cur) == cudaSuccess && cur != prev) cudaSetDevice(prev);
    }
};

inline int64_t pad8(int64_t x) { return (x + 7) / 8 * 8; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline bool type_ok(int t) { return t == SCALECOM_F32 || t == SCALECOM_F16 || t == SCALECOM_BF16; }
inline int64_t type_size(int t) { return t == SCALECOM_F32 ? 4 : 2; }
inline bool dim_ok(int64_t v, int64_t low) { return v >= low && v <= SCALECOM_OPS_MAX_DIM; }

bool capturing(const scalecom_ops* o) {
    if (!o->stream) return false;               // the legacy default stream cannot be captured
    cudaStreamCaptureStatus status = cudaStreamCaptureStatusNone;
    if (cudaStreamIsCapturing(o->stream, &status) != cudaSuccess) cudaGetLastError();
    return status != cudaStreamCaptureStatusNone;
}

// A graph replays its launches with the scratch they were captured with, so that one lives until the handle goes; and nothing can be
// waited for or allocated while a stream is captured.
int ensure_ws(scalecom_ops* o, size_t bytes) {
    const bool graph = capturing(o);
    if (bytes <= o->ws_bytes) {
        if (graph) o->ws_in_graph = true;
        return SCALECOM_OK;
    }
    if (graph) return SCALECOM_ERR_BAD_STATE;
    if (cudaStreamSynchronize(o->stream) != cudaSuccess) return SCALECOM_ERR_CUDA;
    if (o->ws_in_graph) {
        scalecom_ops::Kept* k = new (std::nothrow) scalecom_ops::Kept{o->ws, o->kept};
        if (!k) return SCALECOM_ERR_ALLOC;
        o->kept = k;
    } else {
        cudaFree(o->ws);
    }
    o->ws = nullptr;
    o->ws_bytes = 0;
    o->ws_in_graph = false;
    if (cudaMalloc(&o->ws, bytes) != cudaSuccess) {
        cudaGetLastError();
        o->ws = nullptr;
        return SCALECOM_ERR_ALLOC;
    }
    o->ws_bytes = bytes;
    return SCALECOM_OK;
}

// Scratch is laid out in two passes of the same code: the first (base NULL) counts, the second hands out addresses.
struct Carver {
    char* base;
    size_t used = 0;
    template <typename T> T* take(int64_t count) {
        T* p = base ? reinterpret_cast<T*>(base + used) : nullptr;
        used = (used + size_t(count) * sizeof(T) + 255) / 256 * 256;
        return p;
    }
};

template <typename... A, typename... B>
cudaError_t launch_cluster(scalecom_ops* o, int cluster, void (*kernel)(A...), dim3 grid, int threads, size_t smem, B&&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = o->stream;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = unsigned(cluster);
    at[1].val.clusterDim.y = 1;
    at[1].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<A>(args)...);
}
template <typename... A, typename... B>
cudaError_t launch(scalecom_ops* o, void (*kernel)(A...), dim3 grid, int threads, size_t smem, B&&... args) {
    return launch_cluster(o, 1, kernel, grid, threads, smem, std::forward<B>(args)...);
}

int enter(scalecom_ops* o) { return !o ? SCALECOM_ERR_NULL_PTR : o->poisoned ? SCALECOM_ERR_BAD_STATE : SCALECOM_OK; }

// ---- layer norm --------------------------------------------------------------------------------------------
constexpr int LN_MOST_BLOCKS = 4;       // of a backward kernel on a multiprocessor: bounds the scratch

// blocks of a kernel that fit the device at once
template <typename K>
int64_t resident(scalecom_ops* o, K kernel, int threads, size_t smem, int most = 32) {
    const void* key = reinterpret_cast<const void*>(kernel);
    size_t at = (reinterpret_cast<uintptr_t>(key) >> 4) % scalecom_ops::FITS;
    for (int i = 0; i < scalecom_ops::FITS && o->fits[at].kernel && o->fits[at].kernel != key; ++i) at = (at + 1) % scalecom_ops::FITS;
    int per = o->fits[at].kernel == key ? o->fits[at].blocks : 0;
    if (!per) {
        if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per, kernel, threads, smem) != cudaSuccess || per < 1) {
            cudaGetLastError();
            return o->sms;                      // not kept: the next call asks again
        }
        if (!o->fits[at].kernel) o->fits[at] = {key, per};
    }
    return int64_t(o->sms) * (per < most ? per : most);
}

template <typename T, int VEC, int NV, int TPR, bool WHOLE = false, bool MOST = false>
cudaError_t ln_launch(scalecom_ops* o, const LnParams& P) {
    if constexpr (!WHOLE && VEC > 1)
        if (P.width == NV * VEC * TPR) return ln_launch<T, VEC, NV, TPR, true, true>(o, P);
    if constexpr (!MOST && NV > 1)
        if (P.width > (NV - 1) * VEC * TPR) return ln_launch<T, VEC, NV, TPR, WHOLE, true>(o, P);
    const auto kernel = layer_norm_kernel<T, VEC, NV, TPR, WHOLE, MOST>;
    const int64_t cap = resident(o, kernel, LN_THREADS, 0);
    const int64_t want = ceil_div(P.rows, LN_THREADS / TPR);
    return launch(o, kernel, dim3(unsigned(want < cap ? want : cap)), LN_THREADS, 0, P);
}
// A warp takes a row of up to 32 elements a lane, without a barrier; wider rows take a block.
template <typename T, int VEC>
cudaError_t ln_forward(scalecom_ops* o, const LnParams& P) {
    const int w = P.width;
    constexpr int W = 32 * VEC, B = LN_THREADS * VEC;
    if (w <= W) return ln_launch<T, VEC, 1, 32>(o, P);
    if (w <= 2 * W) return ln_launch<T, VEC, 2, 32>(o, P);
    if (w <= 4 * W) return ln_launch<T, VEC, 4, 32>(o, P);
    if (VEC <= 4 && w <= 8 * W) return ln_launch<T, VEC, VEC <= 4 ? 8 : 1, 32>(o, P);
    if (w <= B) return ln_launch<T, VEC, 1, LN_THREADS>(o, P);
    if (w <= 2 * B) return ln_launch<T, VEC, 2, LN_THREADS>(o, P);
    if (w <= 4 * B) return ln_launch<T, VEC, 4, LN_THREADS>(o, P);
    if (VEC <= 4 && w <= 8 * B) return ln_launch<T, VEC, VEC <= 4 ? 8 : 1, LN_THREADS>(o, P);
    if (VEC == 1 && w <= 32 * B) return ln_launch<T, VEC, VEC == 1 ? 32 : 1, LN_THREADS>(o, P);
    const int64_t cap = int64_t(o->sms) * 8;
    return launch(o, layer_norm_wide_kernel<T>, dim3(unsigned(P.rows < cap ? P.rows : cap)), LN_THREADS, 0, P);
}
template <typename T>
cudaError_t ln_forward_t(scalecom_ops* o, const LnParams& P) {
    constexpr int V = 16 / sizeof(T);
    const bool vec = ((reinterpret_cast<uintptr_t>(P.x) | reinterpret_cast<uintptr_t>(P.y)) & 15u) == 0 && P.ldx % V == 0 && P.ldy % V == 0;
    return vec ? ln_forward<T, V>(o, P) : ln_forward<T, 1>(o, P);
}

// rows longer than this leave the registers
constexpr int LN_MOST_WIDTH = 8192;
// blocks to a column of the long rows' column sums
int64_t ln_wide_groups(const scalecom_ops* o, int64_t width) { return ceil_div(int64_t(o->sms) * 8, ceil_div(width, LN_THREADS)); }

// shared memory of a backward kernel at its widest: the sums of a block's warps
template <int VEC, int NV, int TPR, bool DW> constexpr size_t ln_backward_smem() {
    return DW && TPR == 32 ? size_t(NV) * VEC * 32 * 8 * (LN_THREADS / 32) : 0;
}
// Above 48 KB a device has to be told, once for each: 32 columns a lane.
template <typename T>
cudaError_t ln_attributes() {
    constexpr int V = 16 / sizeof(T), NV = 32 / V;
    constexpr int most = int(ln_backward_smem<V, NV, 32, true>());
    const cudaError_t e = cudaFuncSetAttribute(layer_norm_backward_kernel<T, V, NV, 32, true, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
    return e != cudaSuccess ? e : cudaFuncSetAttribute(layer_norm_backward_kernel<T, V, NV, 32, true, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
}

template <typename T, int VEC, int NV, int TPR, bool DW, bool MOST = false>
cudaError_t ln_launch_backward_dw(scalecom_ops* o, LnParams& P) {
    if constexpr (!MOST && NV > 1)
        if (P.width > (NV - 1) * VEC * TPR) return ln_launch_backward_dw<T, VEC, NV, TPR, DW, true>(o, P);
    const auto kernel = layer_norm_backward_kernel<T, VEC, NV, TPR, DW, MOST>;
    const size_t smem = DW && TPR == 32 ? size_t(P.width) * 8 * (LN_THREADS / 32) : 0;
    constexpr size_t most = ln_backward_smem<VEC, NV, TPR, DW>();
    static_assert(most <= 48 * 1024 || NV * VEC == 32, "set in ln_attributes");
    const int64_t fit = resident(o, kernel, LN_THREADS, most, LN_MOST_BLOCKS);
    int64_t blocks = ceil_div(P.rows, LN_THREADS / TPR);
    if (blocks > fit) blocks = fit;
    // each block leaves a partial sum that is written and read again: at most an eighth of the rows' own traffic
    const int64_t few = P.rows * 3 * int64_t(sizeof(T)) / 128;
    if (DW && blocks > few) blocks = few > o->sms ? few : blocks < o->sms ? blocks : o->sms;
    P.nblocks = int32_t(blocks);
    return launch(o, kernel, dim3(P.nblocks), LN_THREADS, smem, P);
}
template <typename T, int VEC, int NV, int TPR>
cudaError_t ln_launch_backward(scalecom_ops* o, LnParams& P) {
    if (P.dgamma || P.dbeta) return ln_launch_backward_dw<T, VEC, NV, TPR, true>(o, P);
    return ln_launch_backward_dw<T, VEC, NV, TPR, false>(o, P);
}
template <typename T, int VEC>
cudaError_t ln_backward(scalecom_ops* o, LnParams& P) {
    const int w = P.width;
    constexpr int W = 32 * VEC, B = LN_THREADS * VEC;
    if (w <= W) return ln_launch_backward<T, VEC, 1, 32>(o, P);
    if (w <= 2 * W) return ln_launch_backward<T, VEC, 2, 32>(o, P);
    if (w <= 4 * W) return ln_launch_backward<T, VEC, 4, 32>(o, P);
    if (VEC <= 4 && w <= 8 * W) return ln_launch_backward<T, VEC, VEC <= 4 ? 8 : 1, 32>(o, P);
    if (w <= B) return ln_launch_backward<T, VEC, 1, LN_THREADS>(o, P);
    if (w <= 2 * B) return ln_launch_backward<T, VEC, 2, LN_THREADS>(o, P);
    if (w <= 4 * B) return ln_launch_backward<T, VEC, 4, LN_THREADS>(o, P);
    if (VEC <= 4 && w <= 8 * B) return ln_launch_backward<T, VEC, VEC <= 4 ? 8 : 1, LN_THREADS>(o, P);
    if (VEC == 1 && w <= 32 * B) return ln_launch_backward<T, VEC, VEC == 1 ? 32 : 1, LN_THREADS>(o, P);
    if (P.dgamma || P.dbeta) {                            // before dx, which may overwrite dy
        const int64_t cols = ceil_div(w, LN_THREADS);
        int64_t groups = ln_wide_groups(o, w);
        if (groups > P.rows) groups = P.rows;
        P.nblocks = int32_t(groups);
        const cudaError_t e = launch(o, layer_norm_columns_kernel<T>, dim3(unsigned(cols), unsigned(groups)), LN_THREADS, 0, P);
        if (e != cudaSuccess) return e;
    }
    if (!P.dx) return cudaSuccess;
    const int64_t cap = int64_t(o->sms) * 8;
    return launch(o, layer_norm_backward_wide_kernel<T>, dim3(unsigned(P.rows < cap ? P.rows : cap)), LN_THREADS, 0, P);
}
template <typename T>
cudaError_t ln_backward_t(scalecom_ops* o, LnParams& P) {
    constexpr int V = 16 / sizeof(T);
    const uintptr_t at = reinterpret_cast<uintptr_t>(P.x) | reinterpret_cast<uintptr_t>(P.dy) | reinterpret_cast<uintptr_t>(P.dx);
    const bool vec = (at & 15u) == 0 && P.ldx % V == 0 && P.lddy % V == 0 && (!P.dx || P.lddx % V == 0);
    return vec ? ln_backward<T, V>(o, P) : ln_backward<T, 1>(o, P);
}

// ---- products ------------------------------------------------------------------------------------------------
// A matrix as the tensor cores read it: [batch][planes][rows][ld], 16-bit, 16-byte aligned rows.
struct Operand {
    const void* p = nullptr;
    int64_t rows = 0, cols = 0, ld = 0;
    int planes = 1;
    int64_t plane = 0;             // elements between planes
    int batch = 1;
    int64_t stride = 0;            // elements between matrices
    const uint32_t* amax = nullptr;
};

inline bool tma_ready(const void* p, int64_t ld) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && ld % 8 == 0; }

// mn: the operand's own rows are contiguous (its stored columns are m or n, its stored rows k)
bool encode(scalecom_ops* o, CUtensorMap* map, const Operand& a, bool bf16, bool mn, int box_rows) {
    const int64_t lead = a.rows * a.ld * 2;
    cuuint64_t dims[4] = {cuuint64_t(a.cols), cuuint64_t(a.rows), cuuint64_t(a.planes), cuuint64_t(a.batch)};
    cuuint64_t strides[3] = {cuuint64_t(a.ld * 2), cuuint64_t(a.planes > 1 ? a.plane * 2 : lead),
                             cuuint64_t(a.batch > 1 ? a.stride * 2 : lead)};
    cuuint32_t box[4] = {64, cuuint32_t(mn ? TC_BK : box_rows), 1, 1};
    cuuint32_t el[4] = {1, 1, 1, 1};
    return o->encode(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, const_cast<void*>(a.p),
                     dims, strides, box, el, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                     CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// A matrix that an epilogue reads or writes in blocks of 32 x 32: [batch][planes][rows][ld] of `type`. Through a tensor map
// where its rows start on the 16-byte grid.
struct Surface {
    const void* p = nullptr;
    int type = SCALECOM_F16;
    int64_t rows = 0, cols = 0, ld = 0;
    int planes = 1;
    int64_t plane = 0;
    int batch = 1;
    int64_t stride = 0;
};
Surface surface(const Operand& a) {
    Surface r;
    r.p = a.p; r.rows = a.rows; r.cols = a.cols; r.ld = a.ld; r.planes = a.planes; r.plane = a.plane; r.batch = a.batch; r.stride = a.stride;
    return r;
}
bool block_map(scalecom_ops* o, CUtensorMap* map, const Surface& a, int32_t* tma) {
    const int64_t e = type_size(a.type), grid = 16 / e;
    *tma = (reinterpret_cast<uintptr_t>(a.p) & 15u) == 0 && a.ld % grid == 0 && (a.planes == 1 || a.plane % grid == 0) &&
           (a.batch == 1 || a.stride % grid == 0);
    if (!*tma) return true;
    const int64_t lead = a.rows * a.ld * e;
    cuuint64_t dims[4] = {cuuint64_t(a.cols), cuuint64_t(a.rows), cuuint64_t(a.planes), cuuint64_t(a.batch)};
    cuuint64_t strides[3] = {cuuint64_t(a.ld * e), cuuint64_t(a.planes > 1 ? a.plane * e : lead), cuuint64_t(a.batch > 1 ? a.stride * e : lead)};
    cuuint32_t box[4] = {32, 32, 1, 1}, el[4] = {1, 1, 1, 1};
    const CUtensorMapDataType type = a.type == SCALECOM_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                   : a.type == SCALECOM_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
    return o->encode(map, type, 4, const_cast<void*>(a.p), dims, strides, box, el, CU_TENSOR_MAP_INTERLEAVE_NONE,
                     e == 4 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
bool set_out(scalecom_ops* o, TcJob& P, int k, const Surface& a) {
    P.out[k].base = static_cast<char*>(const_cast<void*>(a.p));
    P.out[k].ld = a.ld;
    P.out[k].plane = a.plane;
    P.out[k].batch = a.stride;
    return block_map(o, &P.o[k], a, &P.out[k].tma);
}
bool set_in(scalecom_ops* o, TcMore& P, const Surface& a) {
    P.in = a.p;
    P.in_ld = a.ld;
    P.in_plane = a.plane;
    P.in_batch = a.stride;
    return block_map(o, &P.i, a, &P.in_tma);
}

struct Product {
    const Operand *a = nullptr, *b = nullptr, *a2 = nullptr, *b2 = nullptr;   // second pair: GATE's up weights (b2), or a second product
    bool a_mn = false, b_mn = false, a_batched = false, b_batched = false, bf16 = false;
    int64_t m = 0, n = 0, k = 0;
    int batch = 1;
};

struct Plan { int bn, cg, splits; int64_t mt, nt, tiles; };

// Tile shape and parts of k: the least estimated time. A tile's 64 k take the tensor core (256 cycles for 128 columns, three
// times that for two planes, which with the sums in registers become 1,900 cycles for 128 columns and some 2,600 for 256) or the 53 bytes a clock that an SM was
// seen to get from L2, whichever is longer; what a tile adds at its end is only
// seen once, behind the last wave; parts of k cost fences and counting (about 6,000 cycles) and their accumulators' way through L2.
Plan make_plan(const scalecom_ops* o, int epi, int planes, int64_t m, int64_t n, int64_t iters, int64_t batch) {
    struct Shape { int bn, cg; };
    static const Shape one[] = {{256, 2}, {128, 2}, {128, 1}}, two[] = {{256, 2}, {128, 2}, {128, 1}};
    Plan best = {};
    double least = 1e300;
    for (int i = 0; i < 3; ++i) {
        const Shape t = planes > 1 ? two[i] : one[i];
        const int bm = TC_BM * t.cg;
        Plan p;
        p.bn = t.bn;
        p.cg = t.cg;
        p.mt = ceil_div(m, bm);
        p.nt = ceil_div(n, epi == EPI_GATE ? t.bn / 2 : t.bn);
        p.tiles = p.mt * p.nt;
        if (epi == EPI_GRAM || epi == EPI_POLY) {
            p.tiles = 0;
            for (int64_t j = 0; j < p.mt; ++j) {
                const int64_t c = (j * bm + bm - 1) / t.bn + 1;
                p.tiles += c < p.nt ? c : p.nt;
            }
        }
        const double math = t.bn * 2.0 * (planes > 1 ? 3.0 : 1.0), bytes = planes * (16384.0 + t.bn / t.cg * 128.0);
        const double block = planes > 1 ? (t.bn == 256 ? 2600.0 : 1900.0) : math > bytes / 53.0 ? math : bytes / 53.0, drain = t.bn * 12.0;
        for (int s = 1; s <= 32 && (s == 1 || s * 2 <= iters); ++s) {
            if (s > 1 && p.tiles * batch * t.cg > MAX_SPLIT_TILES) break;
            const double waves = double(ceil_div(p.tiles * batch * s, o->sms / t.cg));
            const double cost = waves * double(ceil_div(iters, s)) * block + drain + (s > 1 ? (waves * 5.0 + s * 16.0) * t.bn + 6000.0 : 0.0);
            if (cost < least * 0.97) {
                least = cost;
                best = p;
                best.splits = s;
            }
        }
    }
    return best;
}

int64_t product_iters(const Product& p) {
    return ceil_div(p.k, TC_BK) * (p.a2 ? 2 : 1);
}

template <int BN, int EPI, int PL, int CG, int NJ>
cudaError_t tc_launch(scalecom_ops* o, const TcParams<NJ>& P) {
    int64_t units = 0;
    for (int j = 0; j < P.jobs; ++j) units += int64_t(P.job[j].batch) * P.job[j].tiles * P.job[j].splits;
    const int64_t slots = o->sms / CG;
    return launch_cluster(o, CG, tc_product_kernel<BN, EPI, PL, CG, NJ>, dim3(unsigned((units < slots ? units : slots) * CG)), TC_THREADS,
                          TcShape<BN, EPI, PL, CG>::SMEM, P);
}
template <int EPI>
cudaError_t tc_launch_any(scalecom_ops* o, const Plan& pl, int planes, const TcParams<1>& P) {
    if (planes > 1) return pl.bn == 256 ? tc_launch<256, EPI, 2, 2>(o, P) : pl.cg == 2 ? tc_launch<128, EPI, 2, 2>(o, P) : tc_launch<128, EPI, 2, 1>(o, P);
    if (pl.cg == 1) return tc_launch<128, EPI, 1, 1>(o, P);
    return pl.bn == 256 ? tc_launch<256, EPI, 1, 2>(o, P) : tc_launch<128, EPI, 1, 2>(o, P);
}
template <int BN, int EPI, int PL, int CG, int NJ = 1>
cudaError_t tc_attribute() {
    return cudaFuncSetAttribute(tc_product_kernel<BN, EPI, PL, CG, NJ>, cudaFuncAttributeMaxDynamicSharedMemorySize, TcShape<BN, EPI, PL, CG>::SMEM);
}
template <int EPI>
cudaError_t tc_attributes() {
    cudaError_t e = tc_attribute<256, EPI, 1, 2>();
    if (e == cudaSuccess) e = tc_attribute<128, EPI, 1, 2>();
    if (e == cudaSuccess) e = tc_attribute<128, EPI, 1, 1>();
    if (e == cudaSuccess) e = tc_attribute<256, EPI, 2, 2>();
    if (e == cudaSuccess) e = tc_attribute<128, EPI, 2, 2>();
    if (e == cudaSuccess) e = tc_attribute<128, EPI, 2, 1>();
    return e;
}

// Scratch of a split product. Calls run one after another on the stream, so they share it.
size_t split_bytes(const scalecom_ops* o, int epi, const Product& p) {
    const Plan pl = make_plan(o, epi, p.a->planes, p.m, p.n, product_iters(p), p.batch);
    return pl.splits > 1 ? size_t(pl.tiles) * p.batch * pl.splits * pl.cg * TC_BM * pl.bn * 4 : 0;
}

// Everything of a product but its epilogue's fields, which the caller sets.
int set_job(scalecom_ops* o, int epi, const Product& p, const Plan& pl, TcJob& J) {
    if (pl.tiles * p.batch > 0x7FFFFFFFll / 32) return SCALECOM_ERR_INVALID_ARG;
    const int bbox = epi == EPI_GATE ? pl.bn / 2 : pl.bn / pl.cg;      // rows of B that one copy brings
    bool ok = encode(o, &J.a[0], *p.a, p.bf16, p.a_mn, TC_BM) && encode(o, &J.b[0], *p.b, p.bf16, p.b_mn, bbox);
    if (ok && p.a2) ok = encode(o, &J.a[1], *p.a2, p.bf16, p.a_mn, TC_BM);
    if (ok && p.b2) ok = encode(o, &J.b[1], *p.b2, p.bf16, p.b_mn, bbox);
    if (!ok) return SCALECOM_ERR_CUDA;
    J.pairs = p.a2 ? 2 : 1;
    J.kblocks = int32_t(ceil_div(p.k, TC_BK));
    J.m = int32_t(p.m);
    J.n = int32_t(p.n);
    J.mt = int32_t(pl.mt);
    J.nt = int32_t(pl.nt);
    J.tiles = int32_t(pl.tiles);
    J.batch = p.batch;
    J.splits = pl.splits;
    J.a_mn = p.a_mn;
    J.b_mn = p.b_mn;
    J.a_batched = p.a_batched;
    J.b_batched = p.b_batched;
    // fp32 accumulators; both operands fp16 (0) or bf16 (1); majors; N / 8, M / 16
    J.idesc = (1u << 4) | ((p.bf16 ? 1u : 0u) << 7) | ((p.bf16 ? 1u : 0u) << 10) | ((p.a_mn ? 1u : 0u) << 15) |
              ((p.b_mn ? 1u : 0u) << 16) | (uint32_t(pl.bn / 8) << 17) | (uint32_t(TC_BM * pl.cg / 16) << 24);
    J.amax_a[0] = p.a->amax;
    J.amax_b[0] = p.b->amax;
    if (p.a2) J.amax_a[1] = p.a2->amax;
    if (p.b2) J.amax_b[1] = p.b2->amax;
    return SCALECOM_OK;
}

// P: the epilogue's fields are set by the caller
int run_product(scalecom_ops* o, int epi, const Product& p, TcParams<1>& P, float* partial) {
    const Plan pl = make_plan(o, epi, p.a->planes, p.m, p.n, product_iters(p), p.batch);
    const int rc = set_job(o, epi, p, pl, P.job[0]);
    if (rc != SCALECOM_OK) return rc;
    P.jobs = 1;
    P.status = o->ctrl;
    P.partial = partial;
    P.arrived = o->ctrl + 16;
    cudaError_t e;
    const int planes = p.a->planes;
    switch (epi) {
        case EPI_STORE: e = tc_launch_any<EPI_STORE>(o, pl, planes, P); break;
        case EPI_GATE: e = tc_launch_any<EPI_GATE>(o, pl, planes, P); break;
        case EPI_GATE_BWD: e = tc_launch_any<EPI_GATE_BWD>(o, pl, planes, P); break;
        case EPI_GRAM: e = tc_launch_any<EPI_GRAM>(o, pl, planes, P); break;
        case EPI_POLY: e = tc_launch_any<EPI_POLY>(o, pl, planes, P); break;
        default: e = tc_launch_any<EPI_PLANES>(o, pl, planes, P); break;
    }
    if (e != cudaSuccess) {
        cudaGetLastError();
        return SCALECOM_ERR_CUDA;
    }
    return SCALECOM_OK;
}

// Up to four independent stores. Where together they fill the device without parts of k they are one launch, the longest sums
// first: their tiles then leave one ragged last wave instead of four, and three launches and fills fewer.
struct Stored { const Product* p; Surface out; };
int run_stores(scalecom_ops* o, const Stored* list, int n, float* partial) {
    if (!n) return SCALECOM_OK;
    const int planes = list[0].p->a->planes;
    Plan pl[TC_JOBS];
    int64_t tiles = 0;
    int bn = 256;
    for (; bn >= (planes > 1 ? 128 : 256); bn /= 2) {        // with two planes the narrow tiles cost little more
        tiles = 0;
        for (int i = 0; i < n; ++i) {
            const Product& p = *list[i].p;
            pl[i].bn = bn;
            pl[i].cg = 2;
            pl[i].splits = 1;
            pl[i].mt = ceil_div(p.m, 2 * TC_BM);
            pl[i].nt = ceil_div(p.n, bn);
            pl[i].tiles = pl[i].mt * pl[i].nt;
            tiles += pl[i].tiles;
        }
        if (tiles >= o->sms / 2) break;
    }
    if (n > 1 && tiles >= o->sms / 2) {
        TcParams<TC_JOBS> P;
        std::memset(&P, 0, sizeof P);
        for (int i = 0; i < n; ++i) {
            TcJob& J = P.job[i];
            const int rc = set_job(o, EPI_STORE, *list[i].p, pl[i], J);
            if (rc != SCALECOM_OK) return rc;
            J.type = list[i].out.type;
            J.alpha = 1.0f;
            if (!set_out(o, J, 0, list[i].out)) return SCALECOM_ERR_CUDA;
        }
        P.jobs = n;
        P.status = o->ctrl;
        const cudaError_t e = planes == 1 ? tc_launch<256, EPI_STORE, 1, 2>(o, P) : bn == 256 ? tc_launch<256, EPI_STORE, 2, 2>(o, P)
                                                                                             : tc_launch<128, EPI_STORE, 2, 2>(o, P);
        if (e == cudaSuccess) return SCALECOM_OK;
        cudaGetLastError();
        return SCALECOM_ERR_CUDA;
    }
    for (int i = 0; i < n; ++i) {
        TcParams<1> P;
        std::memset(&P, 0, sizeof P);
        P.job[0].type = list[i].out.type;
        P.job[0].alpha = 1.0f;
        if (!set_out(o, P.job[0], 0, list[i].out)) return SCALECOM_ERR_CUDA;
        const int rc = run_product(o, EPI_STORE, *list[i].p, P, partial);
        if (rc != SCALECOM_OK) return rc;
    }
    return SCALECOM_OK;
}

// Operands of one call that need work before the tensor cores can read them: fp32 ones (planes), 16-bit ones off the
// 16-byte grid. In the counting pass it only takes the scratch.
struct Prep {
    PrepTable t;
    int n = 0;
    int64_t most_rows = 0;
    Prep(int type) { t.type = type; }
    Operand add(Carver& c, const void* p, int64_t rows, int64_t cols, int64_t ld, uint32_t* amax) {
        Operand a;
        a.rows = rows;
        a.cols = cols;
        if (t.type != SCALECOM_F32 && tma_ready(p, ld)) {
            a.p = p;
            a.ld = ld;
            return a;
        }
        a.ld = pad8(cols);
        a.planes = t.type == SCALECOM_F32 ? 2 : 1;
        a.plane = a.planes > 1 ? rows * a.ld : 0;
        a.p = c.take<uint16_t>(a.planes * rows * a.ld);
        a.amax = t.type == SCALECOM_F32 ? amax : nullptr;
        t.item[n++] = {p, ld, rows, cols, const_cast<void*>(a.p), a.ld, a.plane, amax};
        if (rows > most_rows) most_rows = rows;
        return a;
    }
    int run(scalecom_ops* o, bool need_amax) {
        if (!n) return SCALECOM_OK;
        const int64_t cap = int64_t(o->sms) * 4;
        const dim3 grid(unsigned(most_rows < cap ? most_rows : cap), unsigned(n));
        if (t.type == SCALECOM_F32 && need_amax && launch(o, prep_amax_kernel, grid, PREP_THREADS, 0, t) != cudaSuccess)
            return SCALECOM_ERR_CUDA;
        return launch(o, prep_operand_kernel, grid, PREP_THREADS, 0, t) == cudaSuccess ? SCALECOM_OK : SCALECOM_ERR_CUDA;
    }
};

// largest-magnitude words of a call's fp32 operands
enum { AM_X = 0, AM_WG, AM_WU, AM_WD, AM_DY, AM_H, AM_DG, AM_DU, AM_WORDS };

struct FfnArgs {
    int type, act;
    int64_t tokens, width, hidden;
    const void *x, *wg, *wu, *wd;
    int64_t ldx;
};

template <typename T, int VEC, bool GATE>
cudaError_t tokens_launch(scalecom_ops* o, FtParams P) {
    // warps to a row: enough for 16 warps a multiprocessor where there are few rows
    P.split = 1;
    while (P.split < FT_WARPS && int64_t(P.rows) * P.split < int64_t(o->sms) * 16 && P.k / (P.split * 2) >= 32 * VEC) P.split *= 2;
    const dim3 grid(unsigned(ceil_div(P.rows, FT_WARPS / P.split)));
    if (P.tokens == 1) return launch(o, ffn_tokens_kernel<T, VEC, 1, GATE>, grid, FT_THREADS, 0, P);
    if (P.tokens == 2) return launch(o, ffn_tokens_kernel<T, VEC, 2, GATE>, grid, FT_THREADS, 0, P);
    if (P.tokens <= 4) return launch(o, ffn_tokens_kernel<T, VEC, 4, GATE>, grid, FT_THREADS, 0, P);
    return launch(o, ffn_tokens_kernel<T, VEC, 8, GATE>, grid, FT_THREADS, 0, P);
}
template <typename T>
int ffn_tokens(scalecom_ops* o, const FfnArgs& A, void* y, int64_t ldy, void* saved) {
    constexpr int V = 16 / sizeof(T);
    const int64_t fp = pad8(A.hidden);
    int rc = ensure_ws(o, size_t(A.tokens) * fp * sizeof(T));
    if (rc != SCALECOM_OK) return rc;
    auto on_grid = [](const void* p, int64_t ld) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && ld % V == 0; };
    FtParams P;
    std::memset(&P, 0, sizeof P);
    P.x = A.x; P.w0 = A.wg; P.w1 = A.wu; P.out = o->ws; P.saved = saved;
    P.ldx = A.ldx; P.ldo = fp;
    P.tokens = int32_t(A.tokens); P.rows = int32_t(A.hidden); P.k = int32_t(A.width); P.act = A.act;
    const bool v1 = on_grid(A.x, A.ldx) && on_grid(A.wg, A.width) && on_grid(A.wu, A.width);
    cudaError_t e = v1 ? tokens_launch<T, V, true>(o, P) : tokens_launch<T, 1, true>(o, P);
    if (e != cudaSuccess) return SCALECOM_ERR_CUDA;
    P.x = o->ws; P.w0 = A.wd; P.w1 = nullptr; P.out = y; P.saved = nullptr;
    P.ldx = fp; P.ldo = ldy;
    P.rows = int32_t(A.width); P.k = int32_t(A.hidden);
    e = on_grid(A.wd, A.hidden) ? tokens_launch<T, V, false>(o, P) : tokens_launch<T, 1, false>(o, P);
    return e == cudaSuccess ? SCALECOM_OK : SCALECOM_ERR_CUDA;
}

// Whether the rows-at-a-time kernels are the faster ones. Beyond what both spend on launches they take, measured in us for a MB of
// weights, 0.07 + 0.13 t (16 bits) or 0.05 + 0.10 t (fp32) for t tokens -- 0.5 t and 0.23 t off the 16-byte grid -- against 0.19 and
// 0.75 of the tensor-core path (0.4 and 0.9), whose launches and fills take some 15 us more (45 with two planes).
bool few_tokens(const FfnArgs& A) {
    if (A.tokens > FT_MOST) return false;
    const bool f32 = A.type == SCALECOM_F32;
    const int64_t grid = f32 ? 4 : 8;
    const bool vec = A.width % grid == 0 && A.hidden % grid == 0 &&
                     ((reinterpret_cast<uintptr_t>(A.wg) | reinterpret_cast<uintptr_t>(A.wu) | reinterpret_cast<uintptr_t>(A.wd)) & 15u) == 0;
    const double mb = 3e-6 * double(A.width) * double(A.hidden) * double(type_size(A.type)), t = double(A.tokens);
    const double rows = f32 ? (vec ? 0.05 + 0.10 * t : 0.23 * t) : (vec ? 0.07 + 0.13 * t : 0.5 * t);
    const double tiles = f32 ? (vec ? 0.75 : 0.9) : (vec ? 0.19 : 0.4);
    return mb * (rows - tiles) < (f32 ? 45.0 : vec ? 15.0 : 25.0);
}

int ffn_forward(scalecom_ops* o, const FfnArgs& A, void* y, int64_t ldy, void* saved) {
    if (few_tokens(A))
        return A.type == SCALECOM_F32 ? ffn_tokens<float>(o, A, y, ldy, saved)
             : A.type == SCALECOM_F16 ? ffn_tokens<__half>(o, A, y, ldy, saved) : ffn_tokens<__nv_bfloat16>(o, A, y, ldy, saved);
    const bool f32 = A.type == SCALECOM_F32, bf16 = A.type == SCALECOM_BF16;
    const int64_t T = A.tokens, d = A.width, f = A.hidden, fp = pad8(f);
    for (int pass = 0; pass < 2; ++pass) {
        Carver c{pass ? static_cast<char*>(o->ws) : nullptr};
        uint32_t* am = c.take<uint32_t>(AM_WORDS);
        Prep prep(A.type), prep_h(A.type);
        const Operand x = prep.add(c, A.x, T, d, A.ldx, am + AM_X);
        const Operand wg = prep.add(c, A.wg, f, d, d, am + AM_WG), wu = prep.add(c, A.wu, f, d, d, am + AM_WU);
        const Operand wd = prep.add(c, A.wd, d, f, f, am + AM_WD);
        void* h = f32 ? static_cast<void*>(c.take<float>(T * fp)) : static_cast<void*>(c.take<uint16_t>(T * fp));
        Operand ho;
        if (f32) {
            ho = prep_h.add(c, h, T, f, fp, am + AM_H);
        } else {
            ho.p = h;
            ho.rows = T;
            ho.cols = f;
            ho.ld = fp;
        }
        Product up, down;
        up.a = &x; up.b = &wg; up.b2 = &wu; up.bf16 = bf16;
        up.m = T; up.n = f; up.k = d;
        down.a = &ho; down.b = &wd; down.bf16 = bf16;
        down.m = T; down.n = d; down.k = f;
        const size_t s1 = split_bytes(o, EPI_GATE, up), s2 = split_bytes(o, EPI_STORE, down);
        float* partial = reinterpret_cast<float*>(c.take<char>(int64_t(s1 > s2 ? s1 : s2)));
        if (!pass) {
            const int rc = ensure_ws(o, c.used);
            if (rc != SCALECOM_OK) return rc;
            continue;
        }
        if (f32 && cudaMemsetAsync(am, 0, AM_WORDS * 4, o->stream) != cudaSuccess) return SCALECOM_ERR_CUDA;
        int rc = prep.run(o, true);
        if (rc != SCALECOM_OK) return rc;
        TcParams<1> P;
        std::memset(&P, 0, sizeof P);
        P.job[0].type = A.type;
        P.more.act = A.act;
        P.job[0].alpha = 1.0f;
        Surface hs, ss;
        hs.p = h; hs.type = A.type; hs.rows = T; hs.cols = f; hs.ld = fp;
        bool ok = set_out(o, P.job[0], 0, hs);
        if (saved) {
            ss.p = saved; ss.type = A.type; ss.rows = T; ss.cols = f; ss.ld = f; ss.planes = 2; ss.plane = T * f;
            ok = ok && set_out(o, P.job[0], 1, ss);
        }
        if (!ok) return SCALECOM_ERR_CUDA;
        P.more.amax_o[0] = f32 ? am + AM_H : nullptr;
        rc = run_product(o, EPI_GATE, up, P, partial);
        if (rc == SCALECOM_OK) rc = prep_h.run(o, false);
        if (rc != SCALECOM_OK) return rc;
        std::memset(&P, 0, sizeof P);
        P.job[0].type = A.type;
        P.job[0].alpha = 1.0f;
        Surface ys;
        ys.p = y; ys.type = A.type; ys.rows = T; ys.cols = d; ys.ld = ldy;
        if (!set_out(o, P.job[0], 0, ys)) return SCALECOM_ERR_CUDA;
        return run_product(o, EPI_STORE, down, P, partial);
    }
    return SCALECOM_ERR_INTERNAL;
}

int ffn_backward(scalecom_ops* o, const FfnArgs& A, int wgrad_type, const void* dy, int64_t lddy, const void* saved, void* dx,
                 int64_t lddx, void* dwg, void* dwu, void* dwd) {
    const bool f32 = A.type == SCALECOM_F32, bf16 = A.type == SCALECOM_BF16;
    const int64_t T = A.tokens, d = A.width, f = A.hidden, fp = pad8(f);
    const int64_t e = type_size(A.type);
    for (int pass = 0; pass < 2; ++pass) {
        Carver c{pass ? static_cast<char*>(o->ws) : nullptr};
        uint32_t* am = c.take<uint32_t>(AM_WORDS);
        Prep prep(A.type), prep_mid(A.type);
        const Operand dyo = prep.add(c, dy, T, d, lddy, am + AM_DY);
        const Operand wd = prep.add(c, A.wd, d, f, f, am + AM_WD);
        Operand x, wg, wu;
        if (dwg || dwu) x = prep.add(c, A.x, T, d, A.ldx, am + AM_X);
        if (dx) {
            wg = prep.add(c, A.wg, f, d, d, am + AM_WG);
            wu = prep.add(c, A.wu, f, d, d, am + AM_WU);
        }
        // dg, du and h: [3][tokens][fp] in the call's type
        char* mid = c.take<char>(3 * T * fp * e);
        Operand dg, du, h;
        if (f32) {
            dg = prep_mid.add(c, mid, T, f, fp, am + AM_DG);
            du = prep_mid.add(c, mid ? mid + T * fp * e : nullptr, T, f, fp, am + AM_DU);
            h = prep_mid.add(c, mid ? mid + 2 * T * fp * e : nullptr, T, f, fp, am + AM_H);
        } else {
            dg.rows = T; dg.cols = f; dg.ld = fp;
            du = dg; h = dg;
            dg.p = mid;
            du.p = mid ? mid + T * fp * e : nullptr;
            h.p = mid ? mid + 2 * T * fp * e : nullptr;
        }
        Product pdh, pdx, pwg, pwu, pwd;
        pdh.a = &dyo; pdh.b = &wd; pdh.b_mn = true; pdh.bf16 = bf16;
        pdh.m = T; pdh.n = f; pdh.k = d;
        pdx.a = &dg; pdx.a2 = &du; pdx.b = &wg; pdx.b2 = &wu; pdx.b_mn = true; pdx.bf16 = bf16;
        pdx.m = T; pdx.n = d; pdx.k = f;
        pwg.a = &dg; pwg.b = &x; pwg.a_mn = pwg.b_mn = true; pwg.bf16 = bf16;
        pwg.m = f; pwg.n = d; pwg.k = T;
        pwu = pwg;
        pwu.a = &du;
        pwd.a = &dyo; pwd.b = &h; pwd.a_mn = pwd.b_mn = true; pwd.bf16 = bf16;
        pwd.m = d; pwd.n = f; pwd.k = T;
        size_t most = split_bytes(o, EPI_GATE_BWD, pdh);
        auto more = [&](size_t s) { if (s > most) most = s; };
        if (dx) more(split_bytes(o, EPI_STORE, pdx));
        if (dwg || dwu) more(split_bytes(o, EPI_STORE, pwg));
        if (dwd) more(split_bytes(o, EPI_STORE, pwd));
        float* partial = reinterpret_cast<float*>(c.take<char>(int64_t(most)));
        if (!pass) {
            const int rc = ensure_ws(o, c.used);
            if (rc != SCALECOM_OK) return rc;
            continue;
        }
        if (f32 && cudaMemsetAsync(am, 0, AM_WORDS * 4, o->stream) != cudaSuccess) return SCALECOM_ERR_CUDA;
        int rc = prep.run(o, true);
        if (rc != SCALECOM_OK) return rc;
        TcParams<1> P;
        std::memset(&P, 0, sizeof P);
        P.job[0].type = A.type;
        P.more.act = A.act;
        P.job[0].alpha = 1.0f;
        Surface ss, ms;
        ss.p = saved; ss.type = A.type; ss.rows = T; ss.cols = f; ss.ld = f; ss.planes = 2; ss.plane = T * f;
        ms.p = mid; ms.type = A.type; ms.rows = T; ms.cols = f; ms.ld = fp; ms.planes = 3; ms.plane = T * fp;
        if (!set_in(o, P.more, ss) || !set_out(o, P.job[0], 0, ms)) return SCALECOM_ERR_CUDA;
        for (int i = 0; i < 3 && f32; ++i) P.more.amax_o[i] = am + (i == 0 ? AM_DG : i == 1 ? AM_DU : AM_H);
        rc = run_product(o, EPI_GATE_BWD, pdh, P, partial);
        if (rc == SCALECOM_OK) rc = prep_mid.run(o, false);
        if (rc != SCALECOM_OK) return rc;
        Stored list[TC_JOBS];
        int n = 0;
        auto add = [&](const Product& p, void* out, int type, int64_t ld) {
            if (!out) return;
            Surface& os = list[n].out;
            os = Surface();
            os.p = out; os.type = type; os.rows = p.m; os.cols = p.n; os.ld = ld;
            list[n++].p = &p;
        };
        add(pdx, dx, A.type, lddx);
        add(pwg, dwg, wgrad_type, d);
        add(pwu, dwu, wgrad_type, d);
        add(pwd, dwd, wgrad_type, f);
        std::stable_sort(list, list + n, [](const Stored& a, const Stored& b) { return product_iters(*a.p) > product_iters(*b.p); });
        return run_stores(o, list, n, partial);
    }
    return SCALECOM_ERR_INTERNAL;
}

// ---- Newton-Schulz -----------------------------------------------------------------------------------------------
// X, A and B = aI + bA + cAA are held as a power of two times themselves in fp16 planes. The scale is 2^10 -- the smallest
// entries that matter (1 / sqrt(rows * cols) of a normalised matrix) stay far above fp16's subnormals -- as long as no entry can pass 32. An
// entry is at most the matrix's largest singular value: 1 at first, and then what the coefficients make of it, which ns_steps
// follows step by step; where that is more, as with coefficients that add up to more than 32, the scale is the power of two that fits.
constexpr double NS_SCALE = NSS_SCALE, NS_TOP = 32768.0, NS_LEAST = 0x1p-60;

struct NsArgs {
    int64_t batch, rows, cols;
    int in_type, out_type;
    const void* in;
    void* out;
    int64_t ld_in, in_stride, ld_out, out_stride;
    int steps, ncoef;
    const float* co;
    float eps, scale;
};

double ns_scale(double bound) {
    double scale = NS_SCALE;
    while (scale > NS_LEAST && !(scale * bound <= NS_TOP)) scale *= 0.5;
    return scale;
}
// What the products of each step are multiplied by, from the scales of what they read and write.
void ns_steps(const NsArgs& A, NsStep* out) {
    double top = 1.0, sx = NS_SCALE;                     // of X: bound of its singular values, scale
    for (int i = 0; i < A.steps; ++i) {
        const float* co = A.co + (A.ncoef > 1 ? 3 * i : 0);
        const double a = co[0], b = co[1], c = co[2];
        // roundings may have raised it a little; past 10^30 nothing can be kept in range
        top = std::fmin(top * 1.01, 1e30);
        const double end = top * top;
        auto q = [&](double l) { return std::fabs(a + b * l + c * l * l); };
        auto p = [&](double l) { return std::sqrt(l) * q(l); };
        double most_q = std::fmax(q(0.0), q(end)), most_p = p(end);
        auto turn_q = [&](double l) { if (l > 0.0 && l < end) most_q = std::fmax(most_q, q(l)); };
        auto turn_p = [&](double l) { if (l > 0.0 && l < end) most_p = std::fmax(most_p, p(l)); };
        if (c != 0.0) {
            turn_q(-b / (2.0 * c));                      // q' = b + 2 c l
            const double d = 9.0 * b * b - 20.0 * a * c; // p' ~ a + 3 b l + 5 c l^2
            if (d >= 0.0) {
                turn_p((-3.0 * b + std::sqrt(d)) / (10.0 * c));
                turn_p((-3.0 * b - std::sqrt(d)) / (10.0 * c));
            }
        } else if (b != 0.0) {
            turn_p(-a / (3.0 * b));
        }
        const double sa = ns_scale(end), sb = ns_scale(most_q), next = ns_scale(most_p);
        out[i].gram = float(sa / (sx * sx));
        out[i].poly_a = float(a * sb);
        out[i].poly_b = float(b * sb / sa);
        out[i].poly_c = float(c * sb / (sa * sa));
        out[i].apply = float((i + 1 < A.steps ? next : double(A.scale)) / (sb * sx));
        top = most_p;
        sx = next;
    }
}

// Blocks of a cluster for the one-launch kernel, 0: the separate products are taken. By the least estimated cycles: a product of
// 16 x 8 x 16 takes 20 on a quarter of an SM, a cluster's barriers and sums some thousands a step; the chain of separate products measured
// 110 us for small matrices (180 with two planes) and then runs at about half the tensor cores' rate on tiles of 256 rows.
int small_cluster(const scalecom_ops* o, int planes, int64_t r, int64_t n, int64_t batch, int steps) {
    if (r > NSS_MAX_R) return 0;
    const int64_t rp = (r + 15) / 16 * 16, side = rp / 16, tiles = side * (side + 1) / 2;
    const double chain = steps / 5.0 * ((planes > 1 ? 330e3 : 200e3) + double(batch) * n * 256.0 * 256.0 * 15.0 * (planes > 1 ? 3 : 1) / (o->sms * 4096.0));
    double least = chain;
    int best = 0;
    for (int c = 1; c <= 8; c *= 2) {
        const int64_t nc = (ceil_div(n, c) + 15) / 16 * 16;
        if (nss_smem(planes, rp, nc, c) > 225 * 1024) continue;
        const double waves = double(ceil_div(batch * c, o->sms));
        const double mma = 2.0 * (tiles * (nc / 16) + tiles * side + (nc / 16) * side * side) * (planes > 1 ? 3 : 1);
        const double cost = waves * (steps * (mma * 20.0 / 4.0 + 1500.0 + (c > 1 ? (planes > 1 ? 12000.0 : 4000.0) + 1500.0 * ceil_div(tiles, NSS_WARPS) * ceil_div(c, 4) : 0.0)) + 4000.0 + double(rp) * nc / 16.0);
        if (cost < least * 0.95) {
            least = cost;
            best = c;
        }
    }
    return best;
}
template <int PL>
cudaError_t small_attribute() {
    const cudaError_t e = cudaFuncSetAttribute(ns_small_kernel<PL, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, 225 * 1024);
    return e != cudaSuccess ? e : cudaFuncSetAttribute(ns_small_kernel<PL, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, 225 * 1024);
}
int orthogonalise_small(scalecom_ops* o, const NsArgs& A, int planes, int cluster) {
    NsSmallParams P;
    std::memset(&P, 0, sizeof P);
    P.tall = A.rows > A.cols;
    P.in = A.in; P.out = A.out;
    P.ld_in = A.ld_in; P.in_stride = A.in_stride; P.ld_out = A.ld_out; P.out_stride = A.out_stride;
    P.in_type = A.in_type; P.out_type = A.out_type;
    P.r = int32_t(P.tall ? A.cols : A.rows);
    P.n = int32_t(P.tall ? A.rows : A.cols);
    P.rp = (P.r + 15) / 16 * 16;
    P.nc = int32_t((ceil_div(P.n, cluster) + 15) / 16 * 16);
    P.steps = A.steps; P.eps = A.eps;
    ns_steps(A, P.step);
    const size_t smem = size_t(nss_smem(planes, P.rp, P.nc, cluster));
    const dim3 grid{unsigned(cluster), unsigned(A.batch)};
    auto go = [&](auto kernel) { return launch_cluster(o, cluster, kernel, grid, NSS_THREADS, smem, P); };
    const cudaError_t e = planes > 1 ? (cluster > 1 ? go(ns_small_kernel<2, true>) : go(ns_small_kernel<2, false>))
                                     : (cluster > 1 ? go(ns_small_kernel<1, true>) : go(ns_small_kernel<1, false>));
    if (e != cudaSuccess) {
        cudaGetLastError();
        return SCALECOM_ERR_CUDA;
    }
    return SCALECOM_OK;
}

int orthogonalise(scalecom_ops* o, const NsArgs& A) {
    const int planes = A.out_type == SCALECOM_F32 ? 2 : 1;
    const bool tall = A.rows > A.cols;
    const int64_t r = tall ? A.cols : A.rows, big = tall ? A.rows : A.cols;
    const int64_t ldx = pad8(A.cols), lda = pad8(r), B = A.batch;
    const int cluster = A.steps ? small_cluster(o, planes, r, big, B, A.steps) : 0;
    if (cluster) return orthogonalise_small(o, A, planes, cluster);
    int64_t nparts = ceil_div(A.rows * A.cols, 1 << 14);
    if (nparts > ceil_div(int64_t(o->sms) * 4, B)) nparts = ceil_div(int64_t(o->sms) * 4, B);
    if (nparts > A.rows) nparts = A.rows;
    NsStep step[NSS_MAX_STEPS];
    ns_steps(A, step);
    for (int pass = 0; pass < 2; ++pass) {
        Carver c{pass ? static_cast<char*>(o->ws) : nullptr};
        double* part = c.take<double>(B * nparts);
        Operand x[2], g, q;
        if (A.steps) {
            for (int i = 0; i < (A.steps > 1 ? 2 : 1); ++i) {
                x[i].rows = A.rows; x[i].cols = A.cols; x[i].ld = ldx;
                x[i].planes = planes;
                x[i].plane = planes > 1 ? A.rows * ldx : 0;
                x[i].batch = int(B);
                x[i].stride = planes * A.rows * ldx;
                x[i].p = c.take<__half>(B * x[i].stride);
            }
            g.rows = g.cols = r;
            g.ld = lda;
            g.planes = planes;
            g.plane = planes > 1 ? r * lda : 0;
            g.batch = int(B);
            g.stride = planes * r * lda;
            q = g;
            g.p = c.take<__half>(B * g.stride);
            q.p = c.take<__half>(B * q.stride);
        }
        Product gram, poly, apply;
        gram.m = gram.n = r; gram.k = big;
        gram.a_mn = gram.b_mn = tall;
        gram.a = gram.b = &x[0];
        gram.a_batched = gram.b_batched = true;
        gram.batch = int(B);
        poly = gram;
        poly.a_mn = poly.b_mn = false;
        poly.k = r;
        poly.a = poly.b = &g;
        apply = gram;
        apply.m = A.rows; apply.n = A.cols; apply.k = r;
        apply.a_mn = false;
        apply.b_mn = !tall;
        apply.a = tall ? &x[0] : &q;
        apply.b = tall ? &q : &x[0];
        size_t most = 0;
        if (A.steps) {
            const size_t s[3] = {split_bytes(o, EPI_GRAM, gram), split_bytes(o, EPI_POLY, poly), split_bytes(o, EPI_PLANES, apply)};
            for (size_t v : s) if (v > most) most = v;
        }
        float* partial = reinterpret_cast<float*>(c.take<char>(int64_t(most)));
        if (!pass) {
            const int rc = ensure_ws(o, c.used);
            if (rc != SCALECOM_OK) return rc;
            continue;
        }
        NormParams N;
        std::memset(&N, 0, sizeof N);
        N.in = A.in; N.ld = A.ld_in; N.stride = A.in_stride;
        N.rows = A.rows; N.cols = A.cols; N.in_type = A.in_type;
        N.partial = part; N.nparts = int32_t(nparts);
        N.eps = A.eps;
        if (A.steps) {
            N.factor = NS_SCALE;
            N.planes = const_cast<__half*>(static_cast<const __half*>(x[0].p));
            N.planes_ld = ldx; N.planes_lo = x[0].plane; N.planes_stride = x[0].stride;
        } else {
            N.factor = A.scale;
            N.out = A.out; N.out_type = A.out_type; N.ld_out = A.ld_out; N.out_stride = A.out_stride;
        }
        const dim3 grid{unsigned(nparts), unsigned(B)};
        if (launch(o, norm_partial_kernel, grid, PREP_THREADS, 0, N) != cudaSuccess ||
            launch(o, norm_apply_kernel, grid, PREP_THREADS, 0, N) != cudaSuccess) {
            cudaGetLastError();
            return SCALECOM_ERR_CUDA;
        }
        for (int s = 0; s < A.steps; ++s) {
            const Operand *now = &x[s & 1], *next = &x[(s & 1) ^ 1];
            TcParams<1> P;
            std::memset(&P, 0, sizeof P);
            gram.a = gram.b = now;
            P.job[0].alpha = step[s].gram;
            if (!set_out(o, P.job[0], 0, surface(g))) return SCALECOM_ERR_CUDA;
            int rc = run_product(o, EPI_GRAM, gram, P, partial);
            if (rc != SCALECOM_OK) return rc;
            std::memset(&P, 0, sizeof P);
            P.more.poly_a = step[s].poly_a; P.more.poly_b = step[s].poly_b; P.more.poly_c = step[s].poly_c;
            if (!set_in(o, P.more, surface(g)) || !set_out(o, P.job[0], 0, surface(q))) return SCALECOM_ERR_CUDA;
            rc = run_product(o, EPI_POLY, poly, P, partial);
            if (rc != SCALECOM_OK) return rc;
            std::memset(&P, 0, sizeof P);
            (tall ? apply.a : apply.b) = now;
            P.job[0].alpha = step[s].apply;
            if (s + 1 < A.steps) {
                if (!set_out(o, P.job[0], 0, surface(*next))) return SCALECOM_ERR_CUDA;
                rc = run_product(o, EPI_PLANES, apply, P, partial);
            } else {
                P.job[0].type = A.out_type;
                Surface os;
                os.p = A.out; os.type = A.out_type; os.rows = A.rows; os.cols = A.cols; os.ld = A.ld_out; os.batch = int(B); os.stride = A.out_stride;
                if (!set_out(o, P.job[0], 0, os)) return SCALECOM_ERR_CUDA;
                rc = run_product(o, EPI_STORE, apply, P, partial);
            }
            if (rc != SCALECOM_OK) return rc;
        }
        return SCALECOM_OK;
    }
    return SCALECOM_ERR_INTERNAL;
}

bool same(const void* a, const void* b) { return a && a == b; }

}  // namespace

extern "C" {

int scalecom_ops_create(scalecom_ops** out) {
    if (!out) return SCALECOM_ERR_NULL_PTR;
    *out = nullptr;
    scalecom_ops* o = new (std::nothrow) scalecom_ops;
    if (!o) return SCALECOM_ERR_ALLOC;
    int major = 0, minor = 0;
    cudaError_t e = cudaGetDevice(&o->device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&o->sms, cudaDevAttrMultiProcessorCount, o->device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, o->device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&minor, cudaDevAttrComputeCapabilityMinor, o->device);
    if (e == cudaSuccess && (major != 10 || minor != 0)) e = cudaErrorNoKernelImageForDevice;
    if (e == cudaSuccess) {
        void* fn = nullptr;
        cudaDriverEntryPointQueryResult found;
        e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found);
        if (e == cudaSuccess && (found != cudaDriverEntryPointSuccess || !fn)) e = cudaErrorSymbolNotFound;
        o->encode = reinterpret_cast<PFN_cuTensorMapEncodeTiled>(fn);
    }
    if (e == cudaSuccess) e = ln_attributes<float>();
    if (e == cudaSuccess) e = ln_attributes<__half>();
    if (e == cudaSuccess) e = ln_attributes<__nv_bfloat16>();
    if (e == cudaSuccess) e = tc_attributes<EPI_STORE>();
    if (e == cudaSuccess) e = tc_attribute<256, EPI_STORE, 1, 2, TC_JOBS>();
    if (e == cudaSuccess) e = tc_attribute<256, EPI_STORE, 2, 2, TC_JOBS>();
    if (e == cudaSuccess) e = tc_attribute<128, EPI_STORE, 2, 2, TC_JOBS>();
    if (e == cudaSuccess) e = tc_attributes<EPI_GATE>();
    if (e == cudaSuccess) e = tc_attributes<EPI_GATE_BWD>();
    if (e == cudaSuccess) e = tc_attributes<EPI_GRAM>();
    if (e == cudaSuccess) e = tc_attributes<EPI_POLY>();
    if (e == cudaSuccess) e = tc_attributes<EPI_PLANES>();
    if (e == cudaSuccess) e = small_attribute<1>();
    if (e == cudaSuccess) e = small_attribute<2>();
    if (e != cudaSuccess) {
        cudaGetLastError();
        delete o;
        return SCALECOM_ERR_CUDA;
    }
    if (cudaMalloc(reinterpret_cast<void**>(&o->ctrl), CTRL_WORDS * 4) != cudaSuccess) {
        cudaGetLastError();
        delete o;
        return SCALECOM_ERR_ALLOC;
    }
    if (cudaMemset(o->ctrl, 0, CTRL_WORDS * 4) != cudaSuccess || cudaStreamSynchronize(nullptr) != cudaSuccess) {
        cudaGetLastError();
        scalecom_ops_destroy(o);
        return SCALECOM_ERR_CUDA;
    }
    *out = o;
    return SCALECOM_OK;
}

void scalecom_ops_destroy(scalecom_ops* o) {
    if (!o) return;
    DeviceGuard guard(o->device);
    cudaStreamSynchronize(o->stream);
    cudaFree(o->ws);
    while (o->kept) {
        scalecom_ops::Kept* k = o->kept;
        o->kept = k->next;
        cudaFree(k->p);
        delete k;
    }
    cudaFree(o->ctrl);
    cudaGetLastError();
    delete o;
}

int scalecom_ops_set_stream(scalecom_ops* o, void* cuda_stream) {
    if (!o) return SCALECOM_ERR_NULL_PTR;
    DeviceGuard guard(o->device);
    if (!guard.ok) return SCALECOM_ERR_CUDA;
    if (cudaStreamSynchronize(o->stream) != cudaSuccess) return SCALECOM_ERR_CUDA;   // scratch is shared between calls
    o->stream = static_cast<cudaStream_t>(cuda_stream);
    return SCALECOM_OK;
}

int scalecom_ops_reserve(scalecom_ops* o, int64_t bytes) {
    if (!o) return SCALECOM_ERR_NULL_PTR;
    if (bytes < 0) return SCALECOM_ERR_INVALID_ARG;
    DeviceGuard guard(o->device);
    if (!guard.ok) return SCALECOM_ERR_CUDA;
    return ensure_ws(o, size_t(bytes));
}

int scalecom_ops_workspace(const scalecom_ops* o, int64_t* bytes) {
    if (!o || !bytes) return SCALECOM_ERR_NULL_PTR;
    *bytes = int64_t(o->ws_bytes);
    return SCALECOM_OK;
}

int scalecom_ops_status(scalecom_ops* o) {
    if (!o) return SCALECOM_ERR_NULL_PTR;
    DeviceGuard guard(o->device);
    uint32_t st = 0;
    if (!guard.ok || cudaStreamSynchronize(o->stream) != cudaSuccess ||
        cudaMemcpy(&st, o->ctrl, 4, cudaMemcpyDeviceToHost) != cudaSuccess) {
        o->poisoned = true;
        return SCALECOM_ERR_CUDA;
    }
    if (st == DEV_OK) return SCALECOM_OK;
    o->poisoned = true;
    return st == DEV_TIMEOUT ? SCALECOM_ERR_TIMEOUT : SCALECOM_ERR_INTERNAL;
}

int scalecom_ops_reset(scalecom_ops* o) {
    if (!o) return SCALECOM_ERR_NULL_PTR;
    DeviceGuard guard(o->device);
    if (!guard.ok || cudaStreamSynchronize(o->stream) != cudaSuccess ||
        cudaMemset(o->ctrl, 0, CTRL_WORDS * 4) != cudaSuccess || cudaStreamSynchronize(nullptr) != cudaSuccess)
        return SCALECOM_ERR_CUDA;
    o->poisoned = false;
    return SCALECOM_OK;
}

int scalecom_layer_norm(scalecom_ops* o, int32_t dtype, int64_t rows, int64_t width, const void* x, int64_t ldx, const float* gamma,
                        const float* beta, float eps, void* y, int64_t ldy, float* mean, float* rstd) {
    int rc = enter(o);
    if (rc != SCALECOM_OK) return rc;
    if (!type_ok(dtype) || !dim_ok(rows, 0) || !dim_ok(width, 1) || ldx < width || ldy < width || !(eps >= 0.0f) || !std::isfinite(eps))
        return SCALECOM_ERR_INVALID_ARG;
    if (rows == 0) return SCALECOM_OK;
    if (!x || !y) return SCALECOM_ERR_NULL_PTR;
    if ((x == y && ldx != ldy) || same(y, gamma) || same(y, beta) || same(y, mean) || same(y, rstd) || same(mean, rstd) ||
        same(x, mean) || same(x, rstd) || same(gamma, mean) || same(gamma, rstd) || same(beta, mean) || same(beta, rstd))
        return SCALECOM_ERR_ALIAS;
    DeviceGuard guard(o->device);
    if (!guard.ok) return SCALECOM_ERR_CUDA;
    LnParams P;
    std::memset(&P, 0, sizeof P);
    P.x = x; P.y = y; P.gamma = gamma; P.beta = beta; P.mean = mean; P.rstd = rstd;
    P.ldx = ldx; P.ldy = ldy; P.rows = rows; P.width = int32_t(width); P.eps = eps;
    cudaError_t e = dtype == SCALECOM_F32 ? ln_forward_t<float>(o, P)
                  : dtype == SCALECOM_F16 ? ln_forward_t<__half>(o, P) : ln_forward_t<__nv_bfloat16>(o, P);
    if (e != cudaSuccess) { cudaGetLastError(); return SCALECOM_ERR_CUDA; }
    return SCALECOM_OK;
}

int scalecom_layer_norm_backward(scalecom_ops* o, int32_t dtype, int64_t rows, int64_t width, const void* dy, int64_t lddy, const void* x,
                                 int64_t ldx, const float* gamma, const float* mean, const float* rstd, void* dx, int64_t lddx,
                                 float* dgamma, float* dbeta) {
    int rc = enter(o);
    if (rc != SCALECOM_OK) return rc;
    if (!type_ok(dtype) || !dim_ok(rows, 0) || !dim_ok(width, 1) || ldx < width || lddy < width || (dx && lddx < width))
        return SCALECOM_ERR_INVALID_ARG;
    DeviceGuard guard(o->device);
    if (!guard.ok) return SCALECOM_ERR_CUDA;
    if (same(dgamma, dbeta) || same(dgamma, gamma) || same(dbeta, gamma)) return SCALECOM_ERR_ALIAS;     // written without rows, too
    if (rows == 0) {
        if ((dgamma && cudaMemsetAsync(dgamma, 0, size_t(width) * 4, o->stream) != cudaSuccess) ||
            (dbeta && cudaMemsetAsync(dbeta, 0, size_t(width) * 4, o->stream) != cudaSuccess))
            return SCALECOM_ERR_CUDA;
        return SCALECOM_OK;
    }
    if (!dy || !x || !mean || !rstd) return SCALECOM_ERR_NULL_PTR;
    if (same(dx, x) || (same(dx, dy) && lddx != lddy) || same(dx, gamma) || same(dx, mean) || same(dx, rstd) || same(dx, dgamma) ||
        same(dx, dbeta) || same(dgamma, dy) || same(dbeta, dy) || same(dgamma, x) || same(dbeta, x) || same(dgamma, mean) ||
        same(dbeta, mean) || same(dgamma, rstd) || same(dbeta, rstd))
        return SCALECOM_ERR_ALIAS;
    if (!dx && !dgamma && !dbeta) return SCALECOM_OK;
    const bool dw = dgamma || dbeta;
    if (dw) {
        rc = ensure_ws(o, size_t(width > LN_MOST_WIDTH ? ln_wide_groups(o, width) : int64_t(o->sms) * LN_MOST_BLOCKS) * 2 * size_t(width) * 4);
        if (rc != SCALECOM_OK) return rc;
    }
    LnParams P;
    std::memset(&P, 0, sizeof P);
    P.x = x; P.dy = dy; P.dx = dx; P.gamma = gamma; P.mean_in = mean; P.rstd_in = rstd;
    P.dgamma = dgamma; P.dbeta = dbeta; P.partial = static_cast<float*>(o->ws);
    P.ldx = ldx; P.lddy = lddy; P.lddx = lddx; P.rows = rows; P.width = int32_t(width);
    cudaError_t e = dtype == SCALECOM_F32 ? ln_backward_t<float>(o, P)
                  : dtype == SCALECOM_F16 ? ln_backward_t<__half>(o, P) : ln_backward_t<__nv_bfloat16>(o, P);
    if (e == cudaSuccess && dw)
        e = launch(o, layer_norm_reduce_kernel, dim3(unsigned(ceil_div(2 * width, 32))), LN_THREADS, 0, P);
    if (e != cudaSuccess) { cudaGetLastError(); return SCALECOM_ERR_CUDA; }
    return SCALECOM_OK;
}

int scalecom_gated_ffn(scalecom_ops* o, int32_t dtype, int32_t act, int64_t tokens, int64_t width, int64_t hidden, const void* x, int64_t ldx,
                       const void* w_gate, const void* w_up, const void* w_down, void* y, int64_t ldy, void* saved) {
    int rc = enter(o);
    if (rc != SCALECOM_OK) return rc;
    if (!type_ok(dtype) || act < SCALECOM_ACT_SILU || act > SCALECOM_ACT_RELU || !dim_ok(tokens, 0) || !dim_ok(width, 1) ||
        !dim_ok(hidden, 1) || ldx < width || ldy < width)
        return SCALECOM_ERR_INVALID_ARG;
    if (tokens == 0) return SCALECOM_OK;
    if (!x || !w_gate || !w_up || !w_down || !y) return SCALECOM_ERR_NULL_PTR;
    for (const void* p : {x, w_gate, w_up, w_down})
        if (same(saved, p) || same(y, p)) return SCALECOM_ERR_ALIAS;
    if (same(saved, y)) return SCALECOM_ERR_ALIAS;
    DeviceGuard guard(o->device);
    if (!guard.ok) return SCALECOM_ERR_CUDA;
    const FfnArgs A = {dtype, act, tokens, width, hidden, x, w_gate, w_up, w_down, ldx};
    rc = ffn_forward(o, A, y, ldy, saved);
    if (rc == SCALECOM_ERR_CUDA) cudaGetLastError();
    return rc;
}

int scalecom_gated_ffn_backward(scalecom_ops* o, int32_t dtype, int32_t wgrad_type, int32_t act, int64_t tokens, int64_t width, int64_t hidden,
                                const void* dy, int64_t lddy, const void* x, int64_t ldx, const void* w_gate, const void* w_up,
                                const void* w_down, const void* saved, void* dx, int64_t lddx, void* dw_gate, void* dw_up, void* dw_down) {
    int rc = enter(o);
    if (rc != SCALECOM_OK) return rc;
    if (!type_ok(dtype) || (wgrad_type != dtype && wgrad_type != SCALECOM_F32) || act < SCALECOM_ACT_SILU || act > SCALECOM_ACT_RELU ||
        !dim_ok(tokens, 0) || !dim_ok(width, 1) || !dim_ok(hidden, 1) || ldx < width || lddy < width || (dx && lddx < width))
        return SCALECOM_ERR_INVALID_ARG;
    DeviceGuard guard(o->device);
    if (!guard.ok) return SCALECOM_ERR_CUDA;
    void* outs[4] = {dx, dw_gate, dw_up, dw_down};
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < i; ++j)
            if (same(outs[i], outs[j])) return SCALECOM_ERR_ALIAS;
    for (const void* p : {w_gate, w_up, w_down})
        for (void* q : {dw_gate, dw_up, dw_down})                 // written without tokens, too
            if (same(q, p)) return SCALECOM_ERR_ALIAS;
    if (tokens == 0) {
        for (int i = 1; i < 4; ++i)
            if (outs[i] && cudaMemsetAsync(outs[i], 0, size_t(width) * hidden * type_size(wgrad_type), o->stream) != cudaSuccess)
                return SCALECOM_ERR_CUDA;
        return SCALECOM_OK;
    }
    if (!dy || !x || !w_gate || !w_up || !w_down || !saved) return SCALECOM_ERR_NULL_PTR;
    for (const void* p : {dy, x, w_gate, w_up, w_down, saved})
        for (void* q : outs)
            if (same(q, p)) return SCALECOM_ERR_ALIAS;
    if (!dx && !dw_gate && !dw_up && !dw_down) return SCALECOM_OK;
    const FfnArgs A = {dtype, act, tokens, width, hidden, x, w_gate, w_up, w_down, ldx};
    rc = ffn_backward(o, A, wgrad_type, dy, lddy, saved, dx, lddx, dw_gate, dw_up, dw_down);
    if (rc == SCALECOM_ERR_CUDA) cudaGetLastError();
    return rc;
}

int scalecom_orthogonalise(scalecom_ops* o, int64_t batch, int64_t rows, int64_t cols, int32_t in_type, const void* in, int64_t ld_in,
                           int64_t in_stride, int32_t out_type, void* out, int64_t ld_out, int64_t out_stride, int32_t steps,
                           const float* coefficients, int32_t ncoef, float eps, float scale) {
    int rc = enter(o);
    if (rc != SCALECOM_OK) return rc;
    if (!type_ok(in_type) || !type_ok(out_type) || !dim_ok(rows, 1) || !dim_ok(cols, 1) || batch < 0 || batch > 65535 || ld_in < cols ||
        ld_out < cols || steps < 0 || steps > 64 || !(eps >= 0.0f) || !std::isfinite(eps) || !std::isfinite(scale))
        return SCALECOM_ERR_INVALID_ARG;
    if (batch > 1 && (in_stride < (rows - 1) * ld_in + cols || out_stride < (rows - 1) * ld_out + cols)) return SCALECOM_ERR_INVALID_ARG;
    if (steps > 0) {
        if (!coefficients) return SCALECOM_ERR_NULL_PTR;
        if (ncoef != 1 && ncoef != steps) return SCALECOM_ERR_INVALID_ARG;
        for (int i = 0; i < 3 * ncoef; ++i)
            if (!(std::fabs(coefficients[i]) <= 63.0f)) return SCALECOM_ERR_INVALID_ARG;
    }
    if (batch == 0) return SCALECOM_OK;
    if (!in || !out) return SCALECOM_ERR_NULL_PTR;
    if (in == out && (in_type != out_type || ld_in != ld_out || (batch > 1 && in_stride != out_stride))) return SCALECOM_ERR_ALIAS;
    DeviceGuard guard(o->device);
    if (!guard.ok) return SCALECOM_ERR_CUDA;
    const NsArgs A = {batch, rows, cols, in_type, out_type, in, out, ld_in, in_stride, ld_out, out_stride, steps, ncoef, coefficients, eps, scale};
    rc = orthogonalise(o, A);
    if (rc == SCALECOM_ERR_CUDA) cudaGetLastError();
    return rc;
}

}  // extern "C"
