// C ABI of the feed-forward block (include/equarx.h): argument checks, tensor maps, launches.
#include <algorithm>
#include <cstdlib>
#include <mutex>

#include "../../include/equarx.h"
#include "equarx_internal.h"
#include "feedforward_kernels.cuh"

namespace {

using namespace equarx;
using namespace equarx::ff;

constexpr size_t kMaxDim = size_t(1) << 30;
constexpr size_t kBigSmem = 227 * 1024;
constexpr size_t kSplitSmem = 224 * 1024;      // dynamic; the kernel's own variables need a few hundred bytes more

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
inline size_t up(size_t v, size_t to) { return (v + to - 1) / to * to; }
inline size_t ceil_div(size_t a, size_t b) { return (a + b - 1) / b; }

// ---------------------------------------------------------------- checks
struct Span {
    const void* p;
    size_t bytes;           // from the first to the last
    size_t width, stride;   // of a row, in bytes; a buffer is one row
    Span(const void* p, size_t bytes) : Span(p, bytes, bytes, 0) {}
    Span(const void* p, size_t bytes, size_t width, size_t stride) : p(p), bytes(bytes), width(width), stride(stride) {}
};
inline Span matrix(const void* p, size_t rows, size_t cols, size_t ld, size_t size) {
    return rows > 1 ? Span(p, ((rows - 1) * ld + cols) * size, cols * size, ld * size) : Span(p, rows * cols * size);
}
// Matrices of one row stride may share its rows, each with columns of its own (the two halves of a wider buffer):
// one's rows then begin after the other's, counted from there, and end before the other's next ones.  Matrices of
// different strides are kept apart as a whole.
inline bool overlap(const Span& a, const Span& b) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
    if (!(a.bytes && b.bytes && a.p && b.p && x < y + b.bytes && y < x + a.bytes)) return false;
    const size_t stride = std::max(a.stride, b.stride);
    if (!stride || (a.stride && b.stride && a.stride != b.stride)) return true;
    const size_t after = y >= x ? (y - x) % stride : (stride - (x - y) % stride) % stride;
    return after < a.width || after + b.width > stride;
}
// no output may meet an input or another output
int check_overlap(std::initializer_list<Span> in, std::initializer_list<Span> out) {
    for (auto o = out.begin(); o != out.end(); ++o) {
        for (const Span& i : in)
            if (overlap(*o, i)) return EQUARX_ERR_ALIAS;
        for (auto q = out.begin(); q != o; ++q)
            if (overlap(*o, *q)) return EQUARX_ERR_ALIAS;
    }
    return EQUARX_OK;
}
inline bool bad_dim(size_t d) { return d == 0 || d > kMaxDim; }
inline bool bad_ld(size_t ld, size_t cols) { return ld < cols || ld > kMaxDim; }
inline bool is_16bit(int dtype) { return dtype == EQUARX_BF16 || dtype == EQUARX_FP16; }
inline bool is_float(int dtype) { return is_16bit(dtype) || dtype == EQUARX_FP32; }
inline bool is_format(int f) { return f == EQUARX_FP4_MX || f == EQUARX_FP4_NV; }
inline bool is_act(int a) { return a == EQUARX_ACT_SILU || a == EQUARX_ACT_GELU_TANH; }
// bytes, at most 32, that a base and a row stride are multiples of
inline int unit_of(const void* p, size_t ld, size_t size) {
    const uintptr_t bits = reinterpret_cast<uintptr_t>(p) | (ld * size) | 32;
    return int(bits & (~bits + 1));
}
inline size_t size_of(int dtype) { return dtype == EQUARX_FP32 ? 4 : 2; }

inline size_t codes_stride(size_t cols) { return ceil_div(cols, 32) * 16; }
inline size_t fp4_stages(size_t cols) { return ceil_div(cols, 256); }

// ---------------------------------------------------------------- device facts, constant for the process
// (kept in arrays of a fixed size: nothing here may throw into a C caller)
constexpr int kMaxDevices = 64, kMaxKernels = 64;

struct DeviceFacts {
    int sms = 0;                 // 0: not looked up yet
    int clusters[9] = {};        // clusters of so many CTAs that run at one time
    bool has_clusters = false;
};
std::mutex g_facts_mutex;
DeviceFacts g_facts[kMaxDevices];

int device_index(int& dev) {
    const cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return cuda_failure(e);
    return dev < kMaxDevices ? EQUARX_OK : cuda_failure(cudaErrorInvalidDevice);
}

int current_device(int& sms) {
    int dev;
    if (const int st = device_index(dev)) return st;
    std::lock_guard<std::mutex> lock(g_facts_mutex);
    if (!g_facts[dev].sms) {
        const cudaError_t e = cudaDeviceGetAttribute(&g_facts[dev].sms, cudaDevAttrMultiProcessorCount, dev);
        if (e != cudaSuccess) return cuda_failure(e);
    }
    sms = g_facts[dev].sms;
    return EQUARX_OK;
}

// Clusters of 1 .. 8 CTAs that run at one time when each CTA has an SM to itself: a cluster stays inside a
// GPC, so this is less than the number of SMs divided by the size.
int resident_clusters(int (&out)[9]) {
    int dev;
    if (const int st = device_index(dev)) return st;
    std::lock_guard<std::mutex> lock(g_facts_mutex);
    DeviceFacts& facts = g_facts[dev];
    if (!facts.has_clusters) {
        const void* const kernel = reinterpret_cast<const void*>(split_kernel<kHalf, kGated, false, false, false>);
        cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(kSplitSmem));
        for (int size = 1; size <= 8 && e == cudaSuccess; ++size) {
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3(size * 256);
            cfg.blockDim = dim3(kSplitThreads);
            cfg.dynamicSmemBytes = kSplitSmem;
            cudaLaunchAttribute attr;
            attr.id = cudaLaunchAttributeClusterDimension;
            attr.val.clusterDim.x = size;
            attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
            cfg.attrs = &attr;
            cfg.numAttrs = 1;
            e = cudaOccupancyMaxActiveClusters(&facts.clusters[size], kernel, &cfg);
        }
        if (e != cudaSuccess) return cuda_failure(e);
        facts.clusters[1] = std::max(1, facts.clusters[1]);
        facts.has_clusters = true;
    }
    std::copy(facts.clusters, facts.clusters + 9, out);
    return EQUARX_OK;
}

// kernels that need more than 48 KB of shared memory ask for it once per device
cudaError_t allow_smem(const void* kernel) {
    struct Entry {
        const void* kernel;
        uint64_t devices;
    };
    static std::mutex mu;
    static Entry seen[kMaxKernels];
    static int count = 0;
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    std::lock_guard<std::mutex> lock(mu);
    int i = 0;
    while (i < count && seen[i].kernel != kernel) ++i;
    const uint64_t bit = dev < kMaxDevices ? uint64_t(1) << dev : 0;
    if (i < count && (seen[i].devices & bit)) return cudaSuccess;
    cudaFuncAttributes fa;
    e = cudaFuncGetAttributes(&fa, kernel);
    if (e == cudaSuccess)
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(kBigSmem - fa.sharedSizeBytes));
    if (e == cudaSuccess && i < kMaxKernels) {
        seen[i].kernel = kernel;
        seen[i].devices |= bit;
        count = std::max(count, i + 1);
    }
    return e;
}

template <typename Args>
int launch(void (*kernel)(Args), dim3 grid, int threads, size_t smem, unsigned cluster, const Args& args,
           cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    unsigned n = 0;
    if (dependent_launches()) {      // every kernel waits for the stream's earlier work before it reads
        attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n++].val.programmaticStreamSerializationAllowed = 1;
    }
    if (cluster > 1) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = cluster;
        attr[n].val.clusterDim.y = attr[n].val.clusterDim.z = 1;
        ++n;
    }
    cfg.attrs = attr;
    cfg.numAttrs = n;
    cudaError_t e = launch_error_to_inject();
    if (e == cudaSuccess && smem > 48 * 1024) e = allow_smem(reinterpret_cast<const void*>(kernel));
    if (e == cudaSuccess) e = cudaLaunchKernelEx(&cfg, kernel, args);
    return e == cudaSuccess ? EQUARX_OK : cuda_failure(e);
}

// ---------------------------------------------------------------- tensor maps
// The driver's encoder is looked up through the runtime, so the library needs no link to the driver.
using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                            const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                            CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
Encode encoder() {
    static Encode fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess) {
            (void)cudaGetLastError();
            p = nullptr;
        }
        return reinterpret_cast<Encode>(p);
    }();
    return fn;
}

// rows x inner elements of 1 or 2 bytes, row stride in bytes; boxes of box_rows x 128 bytes (64 with the
// 64-byte swizzle); elements outside the matrix read as zero
int make_map(CUtensorMap& map, const void* base, size_t elem, size_t inner, size_t rows, size_t stride, size_t box_rows,
             CUtensorMapSwizzle swizzle = CU_TENSOR_MAP_SWIZZLE_128B) {
    const cuuint64_t dims[2] = {inner, rows}, strides[1] = {stride};
    const cuuint32_t box[2] = {cuuint32_t((swizzle == CU_TENSOR_MAP_SWIZZLE_64B ? 64 : kRowBytes) / elem), cuuint32_t(box_rows)},
                     steps[2] = {1, 1};
    const Encode fn = encoder();
    if (!fn) return cuda_failure(cudaErrorNotSupported);
    const CUresult r = fn(&map, elem == 1 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_UINT16, 2,
                          const_cast<void*>(base), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? EQUARX_OK : cuda_failure(cudaErrorInvalidValue);
}

// scales of a 4-bit matrix as rows of 128 bytes, those of one 128-row group and one stage together
int scale_map(CUtensorMap& map, const uint8_t* scales, size_t rows, size_t cols, int format) {
    const size_t box_rows = (format == EQUARX_FP4_MX ? kScaleBytes<kMx> : kScaleBytes<kNv>) / 128;
    return make_map(map, scales, 1, 128, ceil_div(rows, 128) * fp4_stages(cols) * box_rows, 128, box_rows,
                    CU_TENSOR_MAP_SWIZZLE_NONE);
}

#define TRY(call)                              \
    do {                                       \
        if (const int try_status = (call)) return try_status; \
    } while (0)

inline Out out_rows(void* p, size_t ld, int dtype) {
    return Out{p, ld, dtype, unit_of(p, ld, size_of(dtype))};
}

// ---------------------------------------------------------------- 4-bit matrices
struct Fp4 {
    const uint8_t *codes, *scales;
    const float* row_scales;
};
inline size_t scales_bytes(size_t rows, size_t cols, int format) {
    return ceil_div(rows, 128) * fp4_stages(cols) * (format == EQUARX_FP4_MX ? kScaleBytes<kMx> : kScaleBytes<kNv>);
}
int check_fp4(const Fp4& q, int format) {
    if (!q.codes || !q.scales || (format == EQUARX_FP4_NV && !q.row_scales)) return EQUARX_ERR_NULL;
    if (!aligned(q.codes, 16) || !aligned(q.scales, 16) || (format == EQUARX_FP4_NV && !aligned(q.row_scales, 16)))
        return EQUARX_ERR_ALIGN;
    return EQUARX_OK;
}
inline Span codes_span(const Fp4& q, size_t rows, size_t cols) { return Span{q.codes, rows * codes_stride(cols)}; }
inline Span scales_span(const Fp4& q, size_t rows, size_t cols, int format) {
    return Span{q.scales, scales_bytes(rows, cols, format)};
}
inline Span rows_span(const Fp4& q, size_t rows, int format) {
    return Span{format == EQUARX_FP4_NV ? q.row_scales : nullptr, rows * sizeof(float)};
}

// threads of a row's CTA: three groups of 16 elements each, a whole number of warps
inline int row_threads(size_t cols) { return int(std::min<size_t>(512, up(ceil_div(cols, 16 * kRowChunks), 32))); }

template <bool MX, bool ANYWHERE>
int launch_quantize(const QuantArgs& a, cudaStream_t stream) {
    const dim3 grid(a.rows);
    const int threads = row_threads(a.cols);
    if (a.dtype == EQUARX_BF16) return launch(fp4_quantize_kernel<MX, kBf16, ANYWHERE>, grid, threads, 0, 1, a, stream);
    if (a.dtype == EQUARX_FP16) return launch(fp4_quantize_kernel<MX, kFp16, ANYWHERE>, grid, threads, 0, 1, a, stream);
    return launch(fp4_quantize_kernel<MX, kFp32, ANYWHERE>, grid, threads, 0, 1, a, stream);
}
template <bool MX>
int launch_quantize(const QuantArgs& a, cudaStream_t stream) {
    return a.unit < 16 ? launch_quantize<MX, true>(a, stream) : launch_quantize<MX, false>(a, stream);
}
QuantArgs rows_to_quantize(const void* x, int dtype, size_t rows, size_t cols, size_t ld) {
    QuantArgs a = {};
    a.x = x;
    a.ld = ld;
    a.rows = int(rows);
    a.cols = int(cols);
    a.dtype = dtype;
    a.unit = unit_of(x, ld, size_of(dtype));
    return a;
}
int quantize(const void* x, int dtype, size_t rows, size_t cols, size_t ld, int format, const Fp4& q, cudaStream_t stream) {
    QuantArgs a = rows_to_quantize(x, dtype, rows, cols, ld);
    a.codes = const_cast<uint8_t*>(q.codes);
    a.scales = const_cast<uint8_t*>(q.scales);
    a.row_scales = const_cast<float*>(q.row_scales);
    return format == EQUARX_FP4_MX ? launch_quantize<true>(a, stream) : launch_quantize<false>(a, stream);
}

// ---------------------------------------------------------------- launches of the products
// Tokens up to which a product quantizes its own activations, which saves a launch.  Fused / two launches in us, weights
// that change from call to call, as calls from Python and in a CUDA graph (the kernels alone):
//                          2688 -> 5376           gated 5376 -> 2688      1000 -> 1250
//   MX  1 token   calls    6.0 / 8.0              7.4 / 9.0               4.4 / 7.7
//                 graph    5.2 / 6.2              7.0 / 8.1               3.5 / 4.4
//       8 tokens  graph    5.9 / 6.3              7.3 / 8.3               3.6 / 4.7
//       16        graph    7.5 / 6.4              8.8 / 8.5               4.3 / 4.9
//   NV  1 token   calls    8.6 / 9.1              9.9 / 10.7              6.4 / 7.8
//                 graph    7.9 / 7.7              9.4 / 9.7               5.7 / 5.0
//       2 tokens  calls    8.6 / 9.1              9.9 / 10.7              6.3 / 7.8
//                 graph    7.9 / 7.7              9.5 / 9.7               5.5 / 5.1
//       4         calls    9.3 / 9.2              10.7 / 10.7             6.3 / 7.8
//                 graph    8.6 / 7.8              10.3 / 9.7              5.7 / 5.3
// MX wins up to 8 tokens everywhere.  NV's row maxima go round the cluster first: up to 2 tokens it wins as calls, and in
// a graph for the gated block, where a single product loses 0.2 to 0.7 us.
constexpr size_t kFusedMxTokens = 8, kFusedNvTokens = 2;
static_assert(kFusedMxTokens <= kFusedTokens && kFusedNvTokens <= kFusedTokens, "the fused form takes one tile of tokens");

// Columns of a tile, and what the launch is expected to take in cycles of an SM.  The pairs of SMs work
// through whole rounds of tiles.  A stage takes a pair 1.3 cycles for each of the (256 + bn) rows of 128 bytes
// that it loads (the products alone need 2 bn), a tile 3500 to drain (6000 where 256 columns of 4-bit operands go
// through the activation), the launch 8000.  A narrower tile loads more for each product, but may save a round, or give every pair work when
// there is little.  Measured / expected, us: 16-bit gated, 5376 -> 2688, 128 tokens 24.4 / 24.4, 8192 tokens
// 301 / 325; NV product 5376 -> 2688, 128 tokens 12.1 / 11.6.  4-bit operands: their scales come in groups of 128
// columns.
struct TilePlan {
    int bn;
    size_t cost;
};
TilePlan plan_tiles(size_t tiles_m, size_t cols, size_t stages, bool gated, bool fp4, int sms) {
    TilePlan best = {256, ~size_t(0)};
    const int step = fp4 ? 128 : gated ? 64 : 32;
    for (int bn = 256; bn >= (gated && fp4 ? 256 : step); bn -= step) {
        const size_t tiles = tiles_m * ceil_div(cols, gated ? bn / 2 : bn);
        const size_t cost = 8000 + ceil_div(tiles, sms / 2) * (stages * (256 + bn) * 13 / 10 + (gated && fp4 ? 6000 : 3500));
        if (cost < best.cost) best = {bn, cost};
    }
    return best;
}

// sizes, stores and tiles of a product whose operands and outputs are set
int finish_product(Product& g, const TilePlan& plan, size_t m, size_t n, bool gated) {
    g.m = int(m);
    g.n = int(n);
    g.bn = plan.bn;
    g.tiles_m = int(g.two ? ceil_div(m, kRowsM) : ceil_div(m, kTileM));
    g.tiles_n = int(ceil_div(n, gated ? g.bn / 2 : g.bn));
    g.group = 8;
    for (int i = 0; i < 3; ++i)
        if (g.out[i].p && g.out[i].unit >= 16 && g.out[i].dtype != EQUARX_FP32)
            TRY(make_map(g.store[i], g.out[i].p, 2, n, m, g.out[i].ld * 2, 32, CU_TENSOR_MAP_SWIZZLE_64B));
    return EQUARX_OK;
}

template <int KIND, int MODE>
int launch_tiles(const TileArgs<MODE>& a, cudaStream_t stream) {
    int sms;
    TRY(current_device(sms));
    size_t tiles = 0;
    for (const Product& g : a.product) tiles += size_t(g.tiles_m) * g.tiles_n;
    // a pair of CTAs on the two SMs of each TPC; the kernel declares the cluster
    return launch(tile_kernel<KIND, MODE>, dim3(unsigned(2 * std::min<size_t>(tiles, sms / 2))), kTileThreads<KIND>,
                  kTileSmem<KIND>, 1, a, stream);
}

// Shape of a launch of the transposed kernel, and what it is expected to take in cycles of an SM.
struct SplitPlan {
    int nt, ranks, pipe, reuse;
    size_t tiles, smem, cost;
};

template <int KIND, int MODE, bool X_MN>
int plan_split(SplitPlan& plan, size_t features, size_t tokens, int total) {
    // Tiles of at most 128 tokens.  4-bit operands: their scales come in groups of 128 tokens, so more than
    // one tile means tiles of 128; MN-major operands come in pieces of 64.
    const size_t unit = X_MN ? 64 : 16, parts_of = ceil_div(tokens, 128);
    plan.nt = int(KIND != kHalf && tokens > 128 ? 128 : up(ceil_div(tokens, parts_of), unit));
    plan.tiles = ceil_div(features, kRowsM) * ceil_div(tokens, plan.nt) * (MODE == kOut2 ? 2 : 1);
    // The reduction axis is split over as many CTAs as run at one time for all tiles: at most 8, the
    // portable cluster size.  (5376 -> 2688 gated in 16 bits, one token: 21 tiles of 7 CTAs would take two
    // rounds, 23 us; of 6, one, 14 us.)
    int clusters[9];
    TRY(resident_clusters(clusters));
    plan.ranks = 1;
    for (int size = 2; size <= std::min(8, total); ++size)
        if (size_t(clusters[size]) >= plan.tiles) plan.ranks = size;
    const int stage = split_stage_bytes<KIND, MODE>(plan.nt), parts = split_part_bytes<MODE>(plan.nt, plan.ranks);
    const int room = int(kSplitSmem) - kSmemSlack, wanted = std::min(kSplitMaxPipe, int(ceil_div(total, plan.ranks)));
    // parts that would cost stages lie where the stages were
    plan.reuse = room - parts < wanted * stage && plan.nt > kFusedTokens;
    plan.pipe = std::min(wanted, (plan.reuse ? room : room - parts) / stage);
    plan.smem = plan.reuse ? kSplitSmem : size_t(plan.pipe) * stage + parts + kSmemSlack;
    // Fitted to what the kernels take (16 .. 8192 tokens, 256 .. 5376 wide): 8500 cycles to start and end, a
    // stage's loads at 32 bytes a cycle, and for each token of a tile the exchange of its sums.  Measured /
    // expected, us: 16-bit gated, 5376 -> 2688, 128 tokens 21.2 / 21; 1000 -> 700, 64 tokens 8.1 / 8.4; NV product
    // 5376 -> 2688, 128 tokens 11.0 / 10.5; dx, 2688 -> 5376, 128 tokens 17.5 / 24.
    const size_t rounds = ceil_div(plan.tiles, clusters[plan.ranks]);
    const size_t token = MODE == kGated ? 65 + 90 / plan.ranks : 40 + 80 / plan.ranks;
    plan.cost = 8500 + rounds * (ceil_div(total, plan.ranks) * (stage / 32) + plan.nt * token);
    if (ceil_div(tokens, plan.nt) * 2 > 65535) plan.cost = ~size_t(0);      // more than a grid's second dimension
    return EQUARX_OK;
}

template <int KIND, int MODE, bool W_MN, bool X_MN, bool FUSED>
int launch_split(SplitArgs& a, const SplitPlan& plan, size_t features, size_t tokens, cudaStream_t stream) {
    a.features = int(features);
    a.tokens = int(tokens);
    a.nt = plan.nt;
    a.pipe = plan.pipe;
    a.reuse = plan.reuse;
    a.ranks = plan.ranks;
    a.own = int(ceil_div(plan.nt, plan.ranks));
    const int columns = (MODE == kGated ? 2 : 1) * (a.nt + 4 * kScaleTiles<KIND>) + 4 * kScaleTiles<KIND>;
    for (a.columns = 32; a.columns < columns;) a.columns *= 2;
    const dim3 grid(unsigned(plan.ranks * ceil_div(features, kRowsM)),
                    unsigned(ceil_div(tokens, a.nt) * (MODE == kOut2 ? 2 : 1)));
    return launch(split_kernel<KIND, MODE, W_MN, X_MN, FUSED>, grid, kSplitThreads, plan.smem, plan.ranks, a, stream);
}

// weights of the transposed kernel
template <int KIND, int MODE>
int split_weights(SplitArgs& a, const Fp4* w, size_t n, size_t k) {
    const size_t stride = codes_stride(k);
    for (int i = 0; i < (MODE == kGated ? 2 : 1); ++i) {
        TRY(make_map(a.w[i], w[i].codes, 1, stride, n, stride, kRowsM));
        a.scales_w[i] = w[i].scales;
        a.row_w[i] = w[i].row_scales;
    }
    a.stages = int(fp4_stages(k));
    return EQUARX_OK;
}

template <int KIND, int MODE>
int fp4_product(const Fp4& x, const Fp4* w, size_t m, size_t n, size_t k, int act, const Out& out, cudaStream_t stream) {
    const size_t stride = codes_stride(k);
    int sms;
    TRY(current_device(sms));
    const TilePlan tiles = plan_tiles(ceil_div(m, kTileM), n, fp4_stages(k), MODE == kGated, true, sms);
    SplitPlan split;
    TRY((plan_split<KIND, MODE, false>(split, n, m, int(fp4_stages(k)))));
    if (split.cost < tiles.cost) {
        SplitArgs a = {};
        TRY((split_weights<KIND, MODE>(a, w, n, k)));
        TRY(make_map(a.x[0], x.codes, 1, stride, m, stride, split.nt));
        a.scales_x = x.scales;
        a.row_x = x.row_scales;
        a.out[0] = out;
        a.act = act;
        return launch_split<KIND, MODE, false, false, false>(a, split, n, m, stream);
    }
    TileArgs<MODE> a = {};
    Product& g = a.product[0];
    const int format = KIND == kMx ? EQUARX_FP4_MX : EQUARX_FP4_NV;
    TRY(make_map(g.a[0], x.codes, 1, stride, m, stride, kRowsM));
    TRY(scale_map(a.scales_a, x.scales, m, k, format));
    a.row_a = x.row_scales;
    for (int i = 0; i < (MODE == kGated ? 2 : 1); ++i) {
        TRY(make_map(g.b[i], w[i].codes, 1, stride, n, stride, tiles.bn / 2));
        TRY(scale_map(a.scales_b[i], w[i].scales, n, k, format));
        a.row_b[i] = w[i].row_scales;
    }
    g.out[0] = out;
    g.stages = int(fp4_stages(k));
    g.parts = 1;
    a.act = act;
    TRY(finish_product(g, tiles, m, n, MODE == kGated));
    return launch_tiles<KIND, MODE>(a, stream);
}

// the workspace of a quantized activation: scales, row factors, codes
Fp4 carve(void* ws, size_t rows, size_t cols, int format) {
    uint8_t* p = static_cast<uint8_t*>(ws);
    Fp4 q;
    q.scales = p;
    p += up(scales_bytes(rows, cols, format), 256);
    q.row_scales = reinterpret_cast<float*>(p);
    p += up(rows * sizeof(float), 256);
    q.codes = p;
    return q;
}
inline size_t carved_bytes(size_t rows, size_t cols, int format) {
    return up(scales_bytes(rows, cols, format), 256) + up(rows * sizeof(float), 256) + up(rows * codes_stride(cols), 256);
}

inline bool quantizes_itself(size_t m, int format) { return m <= (format == EQUARX_FP4_MX ? kFusedMxTokens : kFusedNvTokens); }

inline size_t product_workspace(size_t m, size_t k, int format) {
    return quantizes_itself(m, format) ? 0 : carved_bytes(m, k, format);
}

// x (16 bits) quantized and multiplied with one or two weights
template <int KIND, int MODE>
int quantized_product(const QuantArgs& x, const Fp4* w, size_t m, size_t n, size_t k, int act, const Out& out, void* workspace,
                      cudaStream_t stream) {
    const int format = KIND == kMx ? EQUARX_FP4_MX : EQUARX_FP4_NV;
    if (quantizes_itself(m, format)) {
        SplitArgs a = {};
        SplitPlan split;
        TRY((plan_split<KIND, MODE, false>(split, n, m, int(fp4_stages(k)))));
        TRY((split_weights<KIND, MODE>(a, w, n, k)));
        a.raw = x;
        a.out[0] = out;
        a.act = act;
        return launch_split<KIND, MODE, false, false, true>(a, split, n, m, stream);
    }
    const Fp4 q = carve(workspace, m, k, format);
    TRY(quantize(x.x, x.dtype, m, k, x.ld, format, q, stream));
    return fp4_product<KIND, MODE>(q, w, m, n, k, act, out, stream);
}

// ---------------------------------------------------------------- 16-bit operands
// TMA reads rows that start on multiples of 16 bytes; others are copied
inline bool needs_copy(const void* p, size_t ld) { return unit_of(p, ld, 2) < 16; }
inline size_t copy_bytes(size_t rows, size_t cols, const void* p, size_t ld) {
    return needs_copy(p, ld) ? up(rows * up(cols, 8) * 2, 256) : 0;
}

struct Operand {
    const void* p;
    size_t ld;
    size_t rows, cols;
};
// copies those that TMA cannot read to the workspace, with one launch
int make_readable(std::initializer_list<Operand*> operands, uint8_t*& ws, cudaStream_t stream) {
    PackArgs a = {};
    size_t rows = 0;
    int jobs = 0, threads = 32;
    for (Operand* o : operands) {
        if (!needs_copy(o->p, o->ld)) continue;
        PackJob& g = a.job[jobs++];
        g.src = static_cast<const uint16_t*>(o->p);
        g.dst = reinterpret_cast<uint16_t*>(ws);
        g.ld_src = o->ld;
        g.ld_dst = up(o->cols, 8);
        g.rows = int(o->rows);
        g.cols = int(o->cols);
        g.unit = unit_of(o->p, o->ld, 2);
        rows += o->rows;
        threads = std::max(threads, int(std::min<size_t>(512, up(ceil_div(g.ld_dst, 4), 32))));
        ws += copy_bytes(o->rows, o->cols, o->p, o->ld);
        o->p = g.dst;
        o->ld = g.ld_dst;
    }
    return jobs ? launch(pack_kernel, dim3(unsigned(rows)), threads, 0, 1, a, stream) : EQUARX_OK;
}
inline int map16(CUtensorMap& map, const Operand& o, size_t box_rows) {
    return make_map(map, o.p, 2, o.cols, o.rows, o.ld * 2, box_rows);
}

}  // namespace

extern "C" {

size_t equarx_fp4_codes_bytes(size_t rows, size_t cols) {
    return rows > kMaxDim || bad_dim(cols) ? 0 : rows * codes_stride(cols);
}

size_t equarx_fp4_scales_bytes(size_t rows, size_t cols, int format) {
    return rows > kMaxDim || bad_dim(cols) || !is_format(format) ? 0 : scales_bytes(rows, cols, format);
}

int equarx_fp4_quantize(const void* x, int dtype, size_t rows, size_t cols, size_t ld, int format, uint8_t* codes,
                        uint8_t* scales, float* row_scales, equarx_stream_t stream) {
    if (!is_float(dtype) || !is_format(format)) return EQUARX_ERR_FORMAT;
    if (rows > kMaxDim || bad_dim(cols) || bad_ld(ld, cols)) return EQUARX_ERR_COUNT;
    if (rows == 0) return EQUARX_OK;
    const Fp4 q{codes, scales, row_scales};
    if (!x) return EQUARX_ERR_NULL;
    TRY(check_fp4(q, format));
    if (!aligned(x, size_of(dtype))) return EQUARX_ERR_ALIGN;
    TRY(check_overlap({matrix(x, rows, cols, ld, size_of(dtype))},
                      {codes_span(q, rows, cols), scales_span(q, rows, cols, format), rows_span(q, rows, format)}));
    return quantize(x, dtype, rows, cols, ld, format, q, stream);
}

int equarx_fp4_dequantize(const uint8_t* codes, const uint8_t* scales, const float* row_scales, size_t rows, size_t cols,
                          int format, void* out, int dtype, size_t ld, equarx_stream_t stream) {
    if (!is_float(dtype) || !is_format(format)) return EQUARX_ERR_FORMAT;
    if (rows > kMaxDim || bad_dim(cols) || bad_ld(ld, cols)) return EQUARX_ERR_COUNT;
    if (rows == 0) return EQUARX_OK;
    const Fp4 q{codes, scales, row_scales};
    if (!out) return EQUARX_ERR_NULL;
    TRY(check_fp4(q, format));
    if (!aligned(out, size_of(dtype))) return EQUARX_ERR_ALIGN;
    TRY(check_overlap({codes_span(q, rows, cols), scales_span(q, rows, cols, format), rows_span(q, rows, format)},
                      {matrix(out, rows, cols, ld, size_of(dtype))}));
    DequantArgs a = {};
    a.codes = codes;
    a.scales = scales;
    a.row_scales = row_scales;
    a.out = out;
    a.ld = ld;
    a.rows = int(rows);
    a.cols = int(cols);
    a.dtype = dtype;
    a.unit = unit_of(out, ld, size_of(dtype));
    const dim3 grid{unsigned(rows)};
    // groups of 16 elements, or of 8 from the first aligned one
    const int threads = a.unit < 16 ? row_threads(2 * cols + 16) : row_threads(cols);
    return format == EQUARX_FP4_MX ? launch(fp4_dequantize_kernel<true>, grid, threads, 0, 1, a, stream)
                                   : launch(fp4_dequantize_kernel<false>, grid, threads, 0, 1, a, stream);
}

int equarx_fp4_matmul(const uint8_t* a_codes, const uint8_t* a_scales, const float* a_row_scales, const uint8_t* b_codes,
                      const uint8_t* b_scales, const float* b_row_scales, size_t m, size_t n, size_t k, int format, void* out,
                      int dtype, size_t ld, equarx_stream_t stream) {
    if (!is_float(dtype) || !is_format(format)) return EQUARX_ERR_FORMAT;
    if (m > kMaxDim || bad_dim(n) || bad_dim(k) || bad_ld(ld, n)) return EQUARX_ERR_COUNT;
    if (m == 0) return EQUARX_OK;
    const Fp4 a{a_codes, a_scales, a_row_scales}, b{b_codes, b_scales, b_row_scales};
    if (!out) return EQUARX_ERR_NULL;
    TRY(check_fp4(a, format));
    TRY(check_fp4(b, format));
    if (!aligned(out, size_of(dtype))) return EQUARX_ERR_ALIGN;
    TRY(check_overlap({codes_span(a, m, k), scales_span(a, m, k, format), rows_span(a, m, format), codes_span(b, n, k),
                       scales_span(b, n, k, format), rows_span(b, n, format)},
                      {matrix(out, m, n, ld, size_of(dtype))}));
    const Out o = out_rows(out, ld, dtype);
    return format == EQUARX_FP4_MX ? fp4_product<kMx, kPlain>(a, &b, m, n, k, 0, o, stream)
                                   : fp4_product<kNv, kPlain>(a, &b, m, n, k, 0, o, stream);
}

size_t equarx_fp4_linear_workspace_bytes(size_t m, size_t k, int format) {
    return m > kMaxDim || bad_dim(k) || !is_format(format) ? 0 : product_workspace(m, k, format);
}

int equarx_fp4_linear(const void* x, int dtype, size_t ldx, const uint8_t* w_codes, const uint8_t* w_scales,
                      const float* w_row_scales, size_t m, size_t n, size_t k, int format, void* out, size_t ld,
                      void* workspace, size_t workspace_bytes, equarx_stream_t stream) {
    if (!is_16bit(dtype) || !is_format(format)) return EQUARX_ERR_FORMAT;
    if (m > kMaxDim || bad_dim(n) || bad_dim(k) || bad_ld(ldx, k) || bad_ld(ld, n)) return EQUARX_ERR_COUNT;
    if (m == 0) return EQUARX_OK;
    const Fp4 w{w_codes, w_scales, w_row_scales};
    const size_t need = product_workspace(m, k, format);
    if (!x || !out || (need && !workspace)) return EQUARX_ERR_NULL;
    TRY(check_fp4(w, format));
    if (workspace_bytes < need) return EQUARX_ERR_WORKSPACE;
    if (!aligned(x, 2) || !aligned(out, 2) || !aligned(workspace, 16)) return EQUARX_ERR_ALIGN;
    TRY(check_overlap({matrix(x, m, k, ldx, 2), codes_span(w, n, k), scales_span(w, n, k, format), rows_span(w, n, format)},
                      {matrix(out, m, n, ld, 2), Span{workspace, need}}));
    const QuantArgs a = rows_to_quantize(x, dtype, m, k, ldx);
    const Out o = out_rows(out, ld, dtype);
    return format == EQUARX_FP4_MX ? quantized_product<kMx, kPlain>(a, &w, m, n, k, 0, o, workspace, stream)
                                   : quantized_product<kNv, kPlain>(a, &w, m, n, k, 0, o, workspace, stream);
}

int equarx_fp4_gated(const void* x, int dtype, size_t ldx, const uint8_t* g_codes, const uint8_t* g_scales,
                     const float* g_row_scales, const uint8_t* u_codes, const uint8_t* u_scales, const float* u_row_scales,
                     size_t m, size_t f, size_t k, int format, int act, void* h, size_t ldh, void* workspace,
                     size_t workspace_bytes, equarx_stream_t stream) {
    if (!is_16bit(dtype) || !is_format(format) || !is_act(act)) return EQUARX_ERR_FORMAT;
    if (m > kMaxDim || bad_dim(f) || bad_dim(k) || bad_ld(ldx, k) || bad_ld(ldh, f)) return EQUARX_ERR_COUNT;
    if (m == 0) return EQUARX_OK;
    const Fp4 w[2] = {{g_codes, g_scales, g_row_scales}, {u_codes, u_scales, u_row_scales}};
    const size_t need = product_workspace(m, k, format);
    if (!x || !h || (need && !workspace)) return EQUARX_ERR_NULL;
    TRY(check_fp4(w[0], format));
    TRY(check_fp4(w[1], format));
    if (workspace_bytes < need) return EQUARX_ERR_WORKSPACE;
    if (!aligned(x, 2) || !aligned(h, 2) || !aligned(workspace, 16)) return EQUARX_ERR_ALIGN;
    TRY(check_overlap({matrix(x, m, k, ldx, 2), codes_span(w[0], f, k), scales_span(w[0], f, k, format),
                       rows_span(w[0], f, format), codes_span(w[1], f, k), scales_span(w[1], f, k, format),
                       rows_span(w[1], f, format)},
                      {matrix(h, m, f, ldh, 2), Span{workspace, need}}));
    const QuantArgs a = rows_to_quantize(x, dtype, m, k, ldx);
    const Out o = out_rows(h, ldh, dtype);
    return format == EQUARX_FP4_MX ? quantized_product<kMx, kGated>(a, w, m, f, k, act, o, workspace, stream)
                                   : quantized_product<kNv, kGated>(a, w, m, f, k, act, o, workspace, stream);
}

size_t equarx_gated_forward_workspace_bytes(size_t m, size_t f, size_t k, const void* x, size_t ldx, const void* wg, size_t ldwg,
                                             const void* wu, size_t ldwu) {
    if (m > kMaxDim || bad_dim(f) || bad_dim(k) || bad_ld(ldx, k) || bad_ld(ldwg, k) || bad_ld(ldwu, k)) return 0;
    return copy_bytes(m, k, x, ldx) + copy_bytes(f, k, wg, ldwg) + copy_bytes(f, k, wu, ldwu);
}

int equarx_gated_forward(const void* x, size_t ldx, const void* wg, size_t ldwg, const void* wu, size_t ldwu, int dtype,
                         size_t m, size_t f, size_t k, int act, void* h, size_t ldh, void* g, void* u, size_t ldgu,
                         void* workspace, size_t workspace_bytes, equarx_stream_t stream) {
    const int kept = dtype & EQUARX_KEPT_FP32 ? EQUARX_FP32 : dtype;            // type of g and u
    dtype &= ~EQUARX_KEPT_FP32;
    if (!is_16bit(dtype) || !is_act(act)) return EQUARX_ERR_FORMAT;
    if (m > kMaxDim || bad_dim(f) || bad_dim(k) || bad_ld(ldx, k) || bad_ld(ldwg, k) || bad_ld(ldwu, k) || bad_ld(ldh, f))
        return EQUARX_ERR_COUNT;
    if (m == 0) return EQUARX_OK;
    if (!x || !wg || !wu || !h || (!g) != (!u)) return EQUARX_ERR_NULL;
    if (g && bad_ld(ldgu, f)) return EQUARX_ERR_COUNT;
    const size_t need = equarx_gated_forward_workspace_bytes(m, f, k, x, ldx, wg, ldwg, wu, ldwu);
    if (need && !workspace) return EQUARX_ERR_NULL;
    if (workspace_bytes < need) return EQUARX_ERR_WORKSPACE;
    for (const void* p : {x, wg, wu, static_cast<const void*>(h)})
        if (!aligned(p, 2)) return EQUARX_ERR_ALIGN;
    if (!aligned(g, size_of(kept)) || !aligned(u, size_of(kept)) || !aligned(workspace, 16)) return EQUARX_ERR_ALIGN;
    TRY(check_overlap({matrix(x, m, k, ldx, 2), matrix(wg, f, k, ldwg, 2), matrix(wu, f, k, ldwu, 2)},
                      {matrix(h, m, f, ldh, 2), matrix(g, m, f, ldgu, size_of(kept)), matrix(u, m, f, ldgu, size_of(kept)),
                       Span{workspace, need}}));

    uint8_t* ws = static_cast<uint8_t*>(workspace);
    Operand ox{x, ldx, m, k}, og{wg, ldwg, f, k}, ou{wu, ldwu, f, k};
    TRY(make_readable({&ox, &og, &ou}, ws, stream));
    const Out oh = out_rows(h, ldh, dtype), sg = out_rows(g, ldgu, kept), su = out_rows(u, ldgu, kept);
    const int stages = int(ceil_div(k, 64));
    int sms;
    TRY(current_device(sms));
    const TilePlan tiles = plan_tiles(ceil_div(m, kTileM), f, stages, true, false, sms);
    SplitPlan split;
    TRY((plan_split<kHalf, kGated, false>(split, f, m, stages)));
    if (split.cost < tiles.cost) {
        SplitArgs a = {};
        TRY(map16(a.w[0], og, kRowsM));
        TRY(map16(a.w[1], ou, kRowsM));
        TRY(map16(a.x[0], ox, split.nt));
        a.out[0] = oh;
        a.out[1] = sg;
        a.out[2] = su;
        a.stages = stages;
        a.act = act;
        a.bf16 = dtype == EQUARX_BF16;
        a.save = g != nullptr;
        return launch_split<kHalf, kGated, false, false, false>(a, split, f, m, stream);
    }
    TileArgs<kGated> a = {};
    Product& p = a.product[0];
    TRY(map16(p.a[0], ox, kRowsM));
    TRY(map16(p.b[0], og, tiles.bn / 2));
    TRY(map16(p.b[1], ou, tiles.bn / 2));
    p.out[0] = oh;
    p.out[1] = sg;
    p.out[2] = su;
    p.stages = stages;
    p.parts = 1;
    a.act = act;
    a.bf16 = dtype == EQUARX_BF16;
    a.save = g != nullptr;
    TRY(finish_product(p, tiles, m, f, true));
    return launch_tiles<kHalf>(a, stream);
}

size_t equarx_gated_backward_workspace_bytes(size_t m, size_t f, size_t k, const void* x, size_t ldx, const void* wg, size_t ldwg,
                                             const void* wu, size_t ldwu) {
    if (m > kMaxDim || bad_dim(f) || bad_dim(k) || bad_ld(ldx, k) || bad_ld(ldwg, k) || bad_ld(ldwu, k)) return 0;
    return copy_bytes(m, k, x, ldx) + copy_bytes(f, k, wg, ldwg) + copy_bytes(f, k, wu, ldwu) + 2 * up(m * up(f, 8) * 2, 256) +
           (m ? up((m + 1) * sizeof(float), 256) : 0);
}

int equarx_gated_backward(const void* dh, size_t lddh, const void* x, size_t ldx, const void* wg, size_t ldwg, const void* wu,
                          size_t ldwu, const void* g, const void* u, size_t ldgu, int dtype, size_t m, size_t f, size_t k,
                          int act, void* dx, size_t lddx, void* dwg, size_t lddwg, void* dwu, size_t lddwu, void* workspace,
                          size_t workspace_bytes, equarx_stream_t stream) {
    const bool wide = dtype & EQUARX_KEPT_FP32;
    const size_t kept = wide ? 4 : 2;                                           // bytes of an element of g and u
    dtype &= ~EQUARX_KEPT_FP32;
    if (!is_16bit(dtype) || !is_act(act)) return EQUARX_ERR_FORMAT;
    if (m > kMaxDim || bad_dim(f) || bad_dim(k) || bad_ld(lddh, f) || bad_ld(ldx, k) || bad_ld(ldwg, k) || bad_ld(ldwu, k) ||
        bad_ld(ldgu, f) || bad_ld(lddx, k) || bad_ld(lddwg, k) || bad_ld(lddwu, k))
        return EQUARX_ERR_COUNT;
    if (!dwg || !dwu || (m && (!dh || !x || !wg || !wu || !g || !u || !dx || !workspace))) return EQUARX_ERR_NULL;
    const size_t need = equarx_gated_backward_workspace_bytes(m, f, k, x, ldx, wg, ldwg, wu, ldwu);
    if (m && workspace_bytes < need) return EQUARX_ERR_WORKSPACE;
    for (const void* p : {dh, x, wg, wu, static_cast<const void*>(dx), static_cast<const void*>(dwg), static_cast<const void*>(dwu)})
        if (!aligned(p, 2)) return EQUARX_ERR_ALIGN;
    if (!aligned(g, kept) || !aligned(u, kept) || !aligned(workspace, 16)) return EQUARX_ERR_ALIGN;
    TRY(check_overlap({matrix(dh, m, f, lddh, 2), matrix(x, m, k, ldx, 2), matrix(wg, f, k, ldwg, 2),
                       matrix(wu, f, k, ldwu, 2), matrix(g, m, f, ldgu, kept), matrix(u, m, f, ldgu, kept)},
                      {matrix(dx, m, k, lddx, 2), matrix(dwg, f, k, lddwg, 2), matrix(dwu, f, k, lddwu, 2),
                       Span{workspace, m ? need : 0}}));
    if (m == 0) {       // sums over no tokens
        cudaError_t e = launch_error_to_inject();
        if (e == cudaSuccess) e = cudaMemset2DAsync(dwg, lddwg * 2, 0, k * 2, f, stream);
        if (e == cudaSuccess) e = cudaMemset2DAsync(dwu, lddwu * 2, 0, k * 2, f, stream);
        return e == cudaSuccess ? EQUARX_OK : cuda_failure(e);
    }

    int sms;
    TRY(current_device(sms));
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    Operand ox{x, ldx, m, k}, og{wg, ldwg, f, k}, ou{wu, ldwu, f, k};
    TRY(make_readable({&ox, &og, &ou}, ws, stream));
    const size_t ldd = up(f, 8);
    const Operand dg{ws, ldd, m, f}, du{ws + up(m * ldd * 2, 256), ldd, m, f};

    GradArgs e = {};
    e.dh = dh;
    e.g = g;
    e.u = u;
    e.dg = const_cast<void*>(dg.p);
    e.du = const_cast<void*>(du.p);
    e.ld_dh = lddh;
    e.ld_gu = ldgu;
    e.ld_out = ldd;
    e.row_top = reinterpret_cast<float*>(ws + 2 * up(m * ldd * 2, 256));
    e.factor = e.row_top + m;
    e.rows = int(m);
    e.cols = int(f);
    e.act = act;
    e.unit = std::min({unit_of(dh, lddh, 2), unit_of(g, ldgu, kept), unit_of(u, ldgu, kept)});
    const int threads = int(std::min<size_t>(512, up(ceil_div(f, 8 * kGradGroups), 32)));
    const auto grad = dtype == EQUARX_BF16 ? (wide ? gate_grad_kernel<kBf16, true> : gate_grad_kernel<kBf16, false>)
                                           : (wide ? gate_grad_kernel<kFp16, true> : gate_grad_kernel<kFp16, false>);
    TRY(launch(grad, dim3(unsigned(m)), threads, 0, 1, e, stream));
    const float* const factor = dtype == EQUARX_FP16 ? e.factor : nullptr;
    if (factor)
        TRY(launch(wide ? grad_range_kernel<true> : grad_range_kernel<false>, dim3(unsigned(std::min<size_t>(m, sms))), 512, 0, 1, e,
                   stream));

    // dx = dG Wg + dU Wu, whose reduction runs over f, twice, and dWg = dG^T x, dWu = dU^T x, whose runs over the
    // tokens.  Neither needs the other's result: where both take tiles they are one launch; else dx goes first and the
    // second begins on the SMs that it leaves idle.
    const int fs = int(ceil_div(f, 64)), ms = int(ceil_div(m, 64)), bf16 = dtype == EQUARX_BF16;
    const Out ox_out = out_rows(dx, lddx, dtype), og_out = out_rows(dwg, lddwg, dtype), ou_out = out_rows(dwu, lddwu, dtype);
    const TilePlan tiles_x = plan_tiles(ceil_div(m, kTileM), k, 2 * fs, false, false, sms);
    const TilePlan tiles_w = plan_tiles(ceil_div(f, kRowsM), k, ms, false, false, sms);
    SplitPlan split_x, split_w;
    TRY((plan_split<kHalf, kSum2, false>(split_x, k, m, 2 * fs)));
    TRY((plan_split<kHalf, kOut2, true>(split_w, k, f, ms)));
    const bool x_splits = split_x.cost < tiles_x.cost, w_splits = split_w.cost < tiles_w.cost;

    TileArgs<kGrads> t = {};
    t.bf16 = bf16;
    t.factor = factor;
    if (!x_splits) {
        Product& p = t.product[0];
        TRY(map16(p.a[0], dg, kRowsM));
        TRY(map16(p.a[1], du, kRowsM));
        TRY(map16(p.b[0], og, 64));
        TRY(map16(p.b[1], ou, 64));
        p.out[0] = ox_out;
        p.stages = fs;
        p.parts = 2;
        TRY(finish_product(p, tiles_x, m, k, false));
    }
    if (!w_splits) {
        Product& p = t.product[1];
        TRY(map16(p.a[0], dg, 64));
        TRY(map16(p.a[1], du, 64));
        TRY(map16(p.b[0], ox, 64));
        p.out[0] = og_out;
        p.out[1] = ou_out;
        p.stages = ms;
        p.parts = p.a_mn = p.two = 1;
        TRY(finish_product(p, tiles_w, f, k, false));
    }
    if (x_splits) {
        SplitArgs a = {};
        TRY(map16(a.w[0], og, 64));
        TRY(map16(a.w[1], ou, 64));
        TRY(map16(a.x[0], dg, split_x.nt));
        TRY(map16(a.x[1], du, split_x.nt));
        a.out[0] = ox_out;
        a.stages = fs;
        a.bf16 = bf16;
        a.factor = factor;
        a.order = kForwarding;
        TRY((launch_split<kHalf, kSum2, true, false, false>(a, split_x, k, m, stream)));
    }
    if (!x_splits || !w_splits) {
        t.order = x_splits ? kBeside : w_splits ? kForwarding : kOrdered;
        TRY(launch_tiles<kHalf>(t, stream));
    }
    if (!w_splits) return EQUARX_OK;
    SplitArgs a = {};
    TRY(map16(a.w[0], ox, 64));
    TRY(map16(a.x[0], dg, 64));
    TRY(map16(a.x[1], du, 64));
    a.out[0] = og_out;
    a.out[1] = ou_out;
    a.stages = ms;
    a.bf16 = bf16;
    a.factor = factor;
    a.order = kBeside;
    return launch_split<kHalf, kOut2, true, true, false>(a, split_w, k, f, stream);
}

int equarx_feedforward_check(void) {
    uint32_t seen = 0;
    cudaError_t e = cudaSuccess;
    if (const char* polls = std::getenv("EQUARX_INJECT_TIMEOUT")) {
        give_up_kernel<<<1, 64>>>(uint32_t(std::min(std::max(std::atoi(polls), 1), int(tc::kWaitLimit))));
        e = cudaGetLastError();
    }
    if (e == cudaSuccess) e = cudaDeviceSynchronize();
    if (e == cudaSuccess) e = cudaMemcpyFromSymbol(&seen, tc::g_gave_up, sizeof(seen));
    const uint32_t zero = 0;
    if (e == cudaSuccess && seen) e = cudaMemcpyToSymbol(tc::g_gave_up, &zero, sizeof(zero));
    if (e != cudaSuccess) return cuda_failure(e);
    return seen ? EQUARX_ERR_TIMEOUT : EQUARX_OK;
}

}  // extern "C"
