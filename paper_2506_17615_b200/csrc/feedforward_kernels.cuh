// Kernels of the tensor-parallel feed-forward block whose partial sums the AllReduce reduces:
// products and gated products of 16-bit and of microscaled 4- and 8-bit operands, their gradients, and the
// quantisers.
//
//   tile_kernel       persistent 256 x bn output tiles on the tensor cores of two SMs
//   split_kernel      few tokens: weights on the 128-row side, the reduction split over a cluster
//   gate_grad_kernel  gradients of the two projections from dh, g and u
//   grad_range_kernel the same scaled, where fp16 cannot hold them
//   pack_kernel       rows that TMA cannot read (a stride that is no multiple of 16 bytes) -> rows it can
//   fp4_quantize_kernel, fp4_dequantize_kernel, fp8_quantize_kernel, fp8_dequantize_kernel
#pragma once
#include <type_traits>

#include "elements.cuh"
#include "tensor_ops.cuh"

namespace equarx {
namespace ff {

using namespace tc;

// 16-bit operands, 4-bit with either scale format, 8-bit
enum Kind { kHalf = 0, kMx = 1, kNv = 2, kMx8 = 3 };
// what a product kernel computes; the gradients are kGrads in tiles, kSum2 (dx) and kOut2 (dWg, dWu) transposed
enum Mode { kPlain = 0, kGated = 1, kSum2 = 2, kOut2 = 3, kGrads = 4 };
enum Act { kSilu = 0, kGeluTanh = 1 };

constexpr int kRowsM = 128;               // rows of a tile: lanes of tensor memory
constexpr int kRowBytes = 128;            // one stage of the reduction axis: 64 16-bit, 128 8-bit or 256 4-bit elements
constexpr int kTileBytes = kRowsM * kRowBytes;
constexpr int kChunkBytes = 64 * kRowBytes;   // MN-major operands: 64 elements x 64 steps of the reduction

// scales of 128 rows for one stage: 512-byte tiles of 128 rows x 4 scales
template <int KIND> constexpr int kScaleTiles = KIND == kNv ? 4 : KIND == kMx ? 2 : KIND == kMx8 ? 1 : 0;
template <int KIND> constexpr int kScaleBytes = 512 * kScaleTiles<KIND>;

// ---------------------------------------------------------------- activation
// silu(g) = g sigma(g);  gelu_tanh(g) = g sigma(z), z = 2 sqrt(2/pi) (g + 0.044715 g^3), which is
// 0.5 g (1 + tanh(z/2)) without the cancellation of 1 + tanh.  sigma in fp32: e^-z overflows to inf
// for z below -88, where 1 / (1 + inf) is the right 0.
constexpr float kGeluC = 1.5957691216057308f, kGeluC3 = kGeluC * 0.044715f;

__device__ __forceinline__ float sigma(float z) { return __fdividef(1.0f, 1.0f + __expf(-z)); }

__device__ __forceinline__ float act(float g, int kind) {
    const float z = kind == kSilu ? g : g * (kGeluC + kGeluC3 * g * g);
    return g * sigma(z);
}
// value and slope: (g s)' = s + g s (1 - s) z'
__device__ __forceinline__ void act_grad(float g, int kind, float& value, float& slope) {
    const float z = kind == kSilu ? g : g * (kGeluC + kGeluC3 * g * g);
    const float dz = kind == kSilu ? 1.0f : kGeluC + 3.0f * kGeluC3 * g * g;
    const float s = sigma(z);
    value = g * s;
    // s (1 - s) is 0 where s is 0 or 1, also where g dz overflows
    const float t = s * (1.0f - s);
    slope = s + (t == 0.0f ? 0.0f : g * dz * t);
}

// ---------------------------------------------------------------- output rows
struct Out {
    void* p;
    size_t ld;
    int dtype;
    int unit;     // bytes that base and row stride are multiples of: 32, 16, 8, 4 or 2
};

// n <= 4 neighbouring columns of one row, the first a multiple of 4
__device__ __forceinline__ void store4(const Out& o, size_t row, int col, int n, const float (&v)[4]) {
    const size_t at = row * o.ld + col;
    if (n == 4 && o.unit >= (o.dtype == kFp32 ? 16 : 8)) {
        if (o.dtype == kFp32)
            *reinterpret_cast<float4*>(static_cast<float*>(o.p) + at) = make_float4(v[0], v[1], v[2], v[3]);
        else
            *reinterpret_cast<uint2*>(static_cast<uint16_t*>(o.p) + at) =
                make_uint2(pack2(v[0], v[1], o.dtype), pack2(v[2], v[3], o.dtype));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n) store1(o.p, at + i, v[i], o.dtype);
    }
}

constexpr int kStageOut = 32 * 32 * 2;        // bytes of a staged 32 x 32 block of 16-bit outputs

// 32 x 32 outputs of a warp, lane t holding row t, as 16-bit rows of 64 bytes in shared memory; 16-byte
// pieces are swizzled (as the 64-byte swizzle of a tensor map), so that the lanes meet no bank twice
__device__ __forceinline__ uint32_t staged_at(uint32_t row, uint32_t byte) {
    return row * 64 + ((((byte >> 4) ^ (row >> 1)) & 3) << 4) + (byte & 15);
}
__device__ __forceinline__ void stage_rows(uint32_t buf, int dtype, const float (&v)[32]) {
    const uint32_t lane = threadIdx.x & 31;
#pragma unroll
    for (int c = 0; c < 4; ++c)
        st_shared_v4(buf + staged_at(lane, 16 * c), pack2(v[8 * c], v[8 * c + 1], dtype), pack2(v[8 * c + 2], v[8 * c + 3], dtype),
                     pack2(v[8 * c + 4], v[8 * c + 5], dtype), pack2(v[8 * c + 6], v[8 * c + 7], dtype));
}

// To an output whose rows TMA can write.  The store is asynchronous; of the warp's two buffers one is
// free again when at most one later store has not been read.
__device__ __forceinline__ void store_staged(const CUtensorMap* map, uint32_t buf, int row0, int col0, int dtype,
                                             const float (&v)[32]) {
    const uint32_t lane = threadIdx.x & 31;
    if (lane == 0) tma_store_wait_read<1>();
    __syncwarp();
    stage_rows(buf, dtype, v);
    fence_async_shared();
    __syncwarp();
    if (lane == 0) tma_store_2d(map, buf, col0, row0);
}

// To any other output, and the last columns of one whose width is no multiple of 16 bytes.  16-bit: neighbouring lanes write a row's
// neighbouring columns, in units of 8, 4 or 2 bytes as base and row stride allow; each lane writing its own row would touch every
// sector many times.  fp32: each lane writes its own row.
__device__ __forceinline__ void store_direct(const Out& o, uint32_t buf, int row0, int col0, int rows, int cols,
                                             const float (&v)[32]) {
    const uint32_t lane = threadIdx.x & 31;
    if (o.dtype == kFp32) {
        float* q = static_cast<float*>(o.p) + size_t(row0 + lane) * o.ld + col0;
        if (row0 + int(lane) >= rows) return;
        if (o.unit >= 16 && col0 + 32 <= cols) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                reinterpret_cast<float4*>(q)[i] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
        } else {
#pragma unroll
            for (int i = 0; i < 32; ++i)
                if (col0 + i < cols) q[i] = v[i];
        }
        return;
    }
    if (lane == 0) tma_store_wait_read<0>();
    __syncwarp();
    stage_rows(buf, o.dtype, v);
    __syncwarp();
    uint16_t* const base = static_cast<uint16_t*>(o.p) + size_t(row0) * o.ld + col0;
    const int height = min(32, rows - row0), width = min(32, cols - col0);
    if (o.unit >= 8) {
        const int c = (lane & 7) * 4;
#pragma unroll 4
        for (int r = lane >> 3; r < height; r += 4) {
            uint32_t a, b;
            ld_shared_v2(buf + staged_at(r, c * 2), a, b);
            uint16_t* q = base + size_t(r) * o.ld + c;
            if (c + 4 <= width) {
                *reinterpret_cast<uint2*>(q) = make_uint2(a, b);
            } else {
                if (c < width) q[0] = uint16_t(a);
                if (c + 1 < width) q[1] = uint16_t(a >> 16);
                if (c + 2 < width) q[2] = uint16_t(b);
            }
        }
    } else if (o.unit == 4) {
        const int c = (lane & 15) * 2;
#pragma unroll 4
        for (int r = lane >> 4; r < height; r += 2) {
            const uint32_t a = ld_shared_u32(buf + staged_at(r, c * 2));
            uint16_t* q = base + size_t(r) * o.ld + c;
            if (c + 2 <= width) *reinterpret_cast<uint32_t*>(q) = a;
            else if (c < width) q[0] = uint16_t(a);
        }
    } else {
#pragma unroll 4
        for (int r = 0; r < height; ++r)
            if (int(lane) < width) base[size_t(r) * o.ld + lane] = uint16_t(ld_shared_u16(buf + staged_at(r, lane * 2)));
    }
    __syncwarp();
}

// v *= row factor * column factors (in shared memory), in that order: the product of two factors alone
// could underflow
__device__ __forceinline__ void scale_columns(float (&v)[32], float row, const float* cols) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float4 c = reinterpret_cast<const float4*>(cols)[j];
        v[4 * j] = v[4 * j] * row * c.x;
        v[4 * j + 1] = v[4 * j + 1] * row * c.y;
        v[4 * j + 2] = v[4 * j + 2] * row * c.z;
        v[4 * j + 3] = v[4 * j + 3] * row * c.w;
    }
}

// ---------------------------------------------------------------- persistent tiles
// One product: out = a b^T, by tiles of 256 x bn.
struct Product {
    CUtensorMap a[2], b[2];
    CUtensorMap store[3];                 // 16-bit outputs with aligned rows: blocks of 32 x 32, inside the columns or ending with them
    Out out[3];                           // gated: h, g, u; two outputs: one each
    int m, n;                             // rows and columns of an output
    int stages;                           // of the reduction axis, in each part
    int parts;                            // 2: out = a0 b0 + a1 b1
    int a_mn;                             // gradients: the other axis of a is the contiguous one
    int two;                              // two outputs, out0 = a0 b0 and out1 = a1 b0
    int tiles_m, tiles_n, bn, group;
};
// Gradients come two products to a launch, all others one.
template <int MODE> struct TileArgs {
    Product product[MODE == kGrads ? 2 : 1];
    CUtensorMap scales_a, scales_b[2];    // 4-bit: the scales of 128 rows and one stage are rows of 128 bytes
    const float* row_a;                   // NV: one factor for each row of a and of b
    const float* row_b[2];
    const float* factor;                  // gradients in fp16: what outputs are multiplied by; else null
    int act, bf16, save, order;
};

constexpr int kTileM = 256;               // rows of a tile: 128 in each CTA of a pair
// shared memory of a stage, in each CTA: its 128 rows of a, its half of the tile's columns of b, and
// the scales of its rows of a and of all columns of b
template <int KIND> constexpr int kStageBytes = 2 * kTileBytes + 3 * kScaleBytes<KIND>;
template <int KIND> constexpr int kPipe = KIND == kHalf ? 6 : 5;
constexpr int kEpilogueWarps = 8;
template <int KIND> constexpr int kTileThreads = 32 * (kEpilogueWarps + (KIND == kHalf ? 2 : 3));
constexpr int kSmemSlack = 1024;          // 128-byte swizzle atoms start on multiples of 1024 bytes
constexpr int kStaging = kEpilogueWarps * 2 * kStageOut;
template <int KIND> constexpr int kTileSmem = kPipe<KIND> * kStageBytes<KIND> + kStaging + kSmemSlack;
// an SM has 227 KB; a kernel's own variables take up to 512 bytes, the column factors of NV 2048 more
static_assert(kTileSmem<kHalf> + 512 <= 227 * 1024 && kTileSmem<kMx> + 512 <= 227 * 1024 && kTileSmem<kNv> + 2560 <= 227 * 1024 &&
              kTileSmem<kMx8> + 512 <= 227 * 1024);

// tile t in an order that walks `group` row tiles before the next column tile: the tiles that run at
// one time share operands in L2
__device__ __forceinline__ void tile_at(const Product& p, int t, int& mt, int& nt) {
    const int per = p.group * p.tiles_n, g = t / per, first = g * p.group;
    const int gm = min(p.group, p.tiles_m - first), r = t - g * per;
    mt = first + r % gm;
    nt = r / gm;
}

// Output tiles of 256 x bn by pairs of CTAs: each holds half of the rows of a and half of the columns of b, the
// tensor cores of both read both halves of b, so a pair loads (256 + bn) rows a stage where two single CTAs would
// load 2 (128 + bn); L2 to SM traffic, not the tensor cores, bounds the single form.  In each CTA one warp starts
// TMA loads through a ring of stages (a second one those of the scales); in the first CTA one warp issues the
// products for both; eight warps move finished accumulators from tensor memory to the output.  Two accumulators let
// the next tile's products run meanwhile.  4-bit operands: the scales need tensor memory too, so of 256 columns the
// second accumulator begins 64 inside the first, and each is drained from that end first.  (Tiles of 192 columns,
// whose accumulators share none, load more for each product: 8192 x 2688 x 5376 in MX 62.0 us, with 256 columns 57.4.)
//
// kGated: columns [0, bn/2) of the tile, the first CTA's half of b, are x Wg^T and [bn/2, bn) the same
// columns of x Wu^T, so a thread finds g and u of one element in its own row and writes act(g) u.
// kGrads: two products one after the other, dx = dG Wg + dU Wu and the weights' gradients dG^T x, dU^T x.  The
// latter's rows lie one below the other in blocks of 128, and a CTA's block belongs to one of them (21 blocks each
// of 2688 rows make 21 tiles, not 2 x 11).
//
// Measured: 16 bits, 8192 x 5376 by 2 x (2688 x 5376): 300 us, 1.57 PFLOP/s, tensor cores active 91 % of a CTA's
// cycles, bound by the power cap (1.3 - 1.6 GHz); single CTAs of 128 x 256 took 442.  4 bits, 8192 x 2688 x 5376, MX 50 us,
// 4.7 PFLOP/s, NV 60: a tile's 11 stages do not hide the 900 cycles between its last product and the next
// tile's first, nor NV's scale copies; longer reductions reach 5.4 and 5.1 PFLOP/s (5376), bound by the loads of a
// stage (36 and 38 KB a CTA in 500 cycles).  8 bits, gated 8192 x 5376 x 2688: 164 us, 2.9 PFLOP/s, tensor cores active 90 %.
template <int KIND, int MODE>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kTileThreads<KIND>, 1)
    tile_kernel(const __grid_constant__ TileArgs<MODE> p) {
    constexpr bool B_MN = MODE == kGrads;
    constexpr bool SCALED = KIND != kHalf;
    constexpr int PIPE = kPipe<KIND>, STAGE = kStageBytes<KIND>, SB = kScaleBytes<KIND>;
    constexpr uint32_t kSecond = SCALED ? 192 : 256;       // first column of the second accumulator
    constexpr uint32_t kScaleCol = 448;                 // scales of a, then of b
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t bars[2 * PIPE + 5];
    __shared__ uint32_t tmem_slot;
    __shared__ volatile uint32_t abort;
    __shared__ __align__(16) float factors[kEpilogueWarps][KIND == kNv ? 64 : 4];      // NV: of a warp's columns

    const uint32_t smem = (smem_addr(smem_raw) + 1023u) & ~1023u;
    const uint32_t full = smem_addr(bars), empty = full + 8 * PIPE, ready = empty + 8 * PIPE, drained = ready + 16,
                   drain = drained + 16;
    const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const int rank = uniform(cluster_rank()), pair = blockIdx.x / 2, pairs = gridDim.x / 2;

    if (threadIdx.x == 0) {
        for (int i = 0; i < PIPE; ++i) {
            barrier_init(full + 8 * i, 1);
            barrier_init(empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            barrier_init(ready + 8 * i, 1);
            barrier_init(drained + 8 * i, 2 * kEpilogueWarps);
        }
        barrier_init(drain, 1);
        abort = 0;
        fence_barrier_init();
    }
    if (warp == kEpilogueWarps) tmem_alloc<2>(smem_addr(&tmem_slot), 512);
    fence_before();
    __syncthreads();
    cluster_sync();                                     // the other CTA's barriers are ready too
    fence_after();
    const uint32_t tmem = uniform(tmem_slot);

    const int first = p.product[0].tiles_m * p.product[0].tiles_n;
    int tiles = first;
    if constexpr (MODE == kGrads) tiles += p.product[1].tiles_m * p.product[1].tiles_n;
    // tile t: its product, its place there, and this CTA's rows with the output they belong to
    auto tile_of = [&](int t, int& mt, int& nt, int& m0, int& which) -> const Product& {
        const bool second = MODE == kGrads && t >= first;
        const Product& g = p.product[second];
        tile_at(g, second ? t - first : t, mt, nt);
        const int block = mt * 2 + rank, blocks = (g.m + kRowsM - 1) / kRowsM;
        which = MODE == kGrads && g.two && block >= blocks;
        m0 = (block - which * blocks) * kRowsM;
        return g;
    };
    grid_begin(p.order);

    if (warp == kEpilogueWarps + 1) {
        // ---------------------------------------------------- loads of a and b
        // (addresses that do not change are kept out of the loops: with five loads a stage this warp
        // needed 690 cycles for each where the products need 512)
        const uint32_t counted = peer_addr(full, 0);       // both CTAs' loads count on the first one's barriers
        uint32_t slot = 0, phase = 1, issued = 0;
        bool ok = true;
        for (int t = pair; t < tiles && ok; t += pairs) {
            int mt, nt, m0, which;
            const Product& g = tile_of(t, mt, nt, m0, which);
            const int half = g.bn / 2;                     // columns of b in each CTA
            const int n0 = MODE == kGated ? nt * half : nt * g.bn + rank * half;
            uint32_t bytes = 2 * kTileBytes + 2 * (B_MN ? (half + 63) / 64 * kChunkBytes : half * kRowBytes);
            if (SCALED) {
                const int width = MODE == kGated ? half : g.bn;
                const int groups_a = (g.m + 127) / 128, nb = min(width / 128, (g.n + 127) / 128 - nt * width / 128);
                bytes += SB * (min(2, groups_a - mt * 2) + 2 * nb * (MODE == kGated ? 2 : 1));
            }
            const int parts = MODE == kGrads ? g.parts : 1;
            for (int part = 0; part < parts; ++part) {
                const CUtensorMap* const ma = &g.a[which | part];      // one of them is 0
                const CUtensorMap* const mb = &g.b[MODE == kGated ? rank : part];
                const bool a_mn = MODE == kGrads && g.a_mn;
                int kc = 0;
                for (int s = 0; s < g.stages; ++s, kc += SCALED ? kRowBytes : 64) {      // 4-bit codes travel as bytes
                    if (!(ok = barrier_wait_warp(empty + 8 * slot, phase, &abort))) break;
                    const uint32_t sa = smem + slot * STAGE, sb = sa + kTileBytes, bar = counted + 8 * slot;
                    if (rank == 0) barrier_expect_warp(full + 8 * slot, bytes);
                    if (a_mn) {
                        tma_load_2d_pair(sa, ma, m0, kc, bar);
                        tma_load_2d_pair(sa + kChunkBytes, ma, m0 + 64, kc, bar);
                    } else {
                        tma_load_2d_pair(sa, ma, kc, m0, bar);
                    }
                    if (B_MN) {
                        for (int c = 0; c < half; c += 64)
                            tma_load_2d_pair(sb + c / 64 * kChunkBytes, mb, n0 + c, kc, bar);
                    } else {
                        tma_load_2d_pair(sb, mb, kc, n0, bar);
                    }
                    ++issued;
                    if (++slot == PIPE) {
                        slot = 0;
                        phase ^= 1;
                    }
                }
                if (!ok) break;
            }
        }
        // Arrivals on this CTA's barriers that the first CTA's products still owe come before its shared memory goes away:
        // one more turn round the ring, whose slots that were never filled are free.  (The output warps' waits
        // for the last product say nothing of them.)
        for (int i = 0; i < PIPE && ok; ++i) {
            ok = barrier_wait_warp(empty + 8 * slot, phase, &abort);
            if (++slot == PIPE) {
                slot = 0;
                phase ^= 1;
            }
        }
        if (gave_up_warp(&abort) && rank == 0)         // what has been started lands before the shared memory goes away
            for (uint32_t i = issued > PIPE ? issued - PIPE : 0; i < issued; ++i)
                barrier_drain(full + 8 * (i % PIPE), i / PIPE & 1);
        __syncwarp();
    } else if (SCALED && warp == kEpilogueWarps + 2) {
        // ---------------------------------------------------- loads of the scales, counted with those
        const uint32_t counted = peer_addr(full, 0);
        uint32_t slot = 0, phase = 1;
        bool ok = true;
        for (int t = pair; t < tiles && ok; t += pairs) {
            int mt, nt, m0, which;
            const Product& g = tile_of(t, mt, nt, m0, which);
            const int width = MODE == kGated ? g.bn / 2 : g.bn;
            // groups of 128 rows: of a this CTA's own (which may not exist), of b all of the tile's
            const int ga = mt * 2 + rank, gb = nt * width / 128, nb = min(width / 128, (g.n + 127) / 128 - gb);
            const bool has_a = ga < (g.m + 127) / 128;
            const int next = g.stages * (SB / 128);
            int ya = ga * next, yb = gb * next;
            for (int s = 0; s < g.stages; ++s, ya += SB / 128, yb += SB / 128) {
                if (!(ok = barrier_wait_warp(empty + 8 * slot, phase, &abort))) break;
                const uint32_t ss = smem + slot * STAGE + 2 * kTileBytes, bar = counted + 8 * slot;
                if (has_a) tma_load_2d_pair(ss, &p.scales_a, 0, ya, bar);
                tma_load_2d_pair(ss + SB, &p.scales_b[0], 0, yb, bar);
                if (MODE == kGated) tma_load_2d_pair(ss + 2 * SB, &p.scales_b[1], 0, yb, bar);
                else if (nb > 1) tma_load_2d_pair(ss + 2 * SB, &p.scales_b[0], 0, yb + next, bar);
                if (++slot == PIPE) {
                    slot = 0;
                    phase ^= 1;
                }
            }
        }
        __syncwarp();
    } else if (warp == kEpilogueWarps) {
        if (rank == 0) {
            // ------------------------------------------------ products
            const uint32_t ta = tmem + kScaleCol, tb = ta + 4 * kScaleTiles<KIND>;
            uint32_t slot = 0, phase = 0, local = 0;
            bool ok = true;
            for (int t = pair; t < tiles && ok; t += pairs, ++local) {
                const uint32_t buf = local & 1, d = tmem + buf * kSecond;
                const Product& g = p.product[MODE == kGrads && t >= first];
                const int stages = g.stages * (MODE == kGrads ? g.parts : 1);
                const bool a_mn = MODE == kGrads && g.a_mn;
                const uint32_t idesc = SCALED ? 0 : desc_16bit(p.bf16, a_mn, B_MN, kTileM, g.bn);
                for (int s = 0; s < stages; ++s) {
                    if (!(ok = barrier_wait_warp(full + 8 * slot, phase, &abort))) break;
                    fence_after();
                    const uint32_t sa = smem + slot * STAGE, sb = sa + kTileBytes, ss = sb + kTileBytes;
                    if (SCALED) {
#pragma unroll
                        for (int j = 0; j < kScaleTiles<KIND>; ++j) {
                            copy_scales<2>(ta + 4 * j, ss + 512 * j);
                            copy_scales<2>(tb + 8 * j, ss + SB + 512 * j);
                            if (g.bn > 128) copy_scales<2>(tb + 8 * j + 4, ss + 2 * SB + 512 * j);
                        }
                    }
                    if (s == 0) {
                        // 4 bits: the tile before has given up the columns that both accumulators use; 16 bits: the
                        // tile before that has given up this accumulator
                        if (SCALED) {
                            if (local && !(ok = barrier_wait_warp<true>(drained, (local - 1) & 1, &abort))) break;
                        } else {
                            if (local > 1 && !(ok = barrier_wait_warp<true>(drained + 8 * buf, (local / 2 - 1) & 1, &abort))) break;
                        }
                        fence_after();
                    }
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk) {
                        const uint32_t da = a_mn ? swizzled_desc(sa + 2048 * kk, kChunkBytes)
                                                 : swizzled_desc(sa + 32 * kk, 16);
                        const uint32_t db = B_MN ? swizzled_desc(sb + 2048 * kk, kChunkBytes)
                                                 : swizzled_desc(sb + 32 * kk, 16);
                        if constexpr (KIND == kMx8) {
                            mma_fp8<2>(d, da, db, desc_fp8(kTileM, g.bn, kk), ta, tb, s | kk);
                        } else if constexpr (SCALED) {
                            const int j = KIND == kNv ? kk : kk / 2, which = KIND == kNv ? 0 : (kk & 1) * 2;
                            mma_fp4<2, KIND == kMx>(d, da, db, desc_fp4(KIND == kMx, kTileM, g.bn, which), ta + 4 * j,
                                                    tb + 8 * j, s | kk);
                        } else {
                            mma_16bit<2>(d, da, db, idesc, s | kk);
                        }
                    }
                    mma_commit<2>(empty + 8 * slot);
                    if (++slot == PIPE) {
                        slot = 0;
                        phase ^= 1;
                    }
                }
                if (ok) mma_commit<2>(ready + 8 * buf);
            }
            if (gave_up_warp(&abort)) {        // products in flight read this shared memory
                mma_commit<2>(drain);
                barrier_drain(drain, 0);
            }
        }
        __syncwarp();
    } else {
        // ---------------------------------------------------- outputs
        const int quarter = warp & 3, side = warp >> 2;
        uint32_t local = 0, flip = 0;
        const float scale = MODE == kGrads && p.factor ? __ldcg(p.factor) : 1.0f;
        const uint32_t staging = smem + PIPE * STAGE + warp * 2 * kStageOut;
        auto store = [&](const Product& g, int i, int row0, int col0, float (&v)[32]) {
            if (row0 >= g.m || col0 >= g.n) return;
            // TMA ends a row with a whole piece of 16 bytes, zeros past the last column: there may be another matrix
            const bool ragged = col0 + 32 > g.n && g.n % 8;
            if (g.out[i].unit >= 16 && g.out[i].dtype != kFp32 && !ragged) {
                store_staged(&g.store[i], staging + flip, row0, col0, g.out[i].dtype, v);
                flip ^= kStageOut;
            } else {
                store_direct(g.out[i], staging, row0, col0, g.m, g.n, v);
            }
        };
        for (int t = pair; t < tiles; t += pairs, ++local) {
            int mt, nt, m0, which;
            const Product& g = tile_of(t, mt, nt, m0, which);
            const int half = g.bn / 2, width = MODE == kGated ? half : g.bn;
            const int units = width / 32;                  // blocks of 32 output columns
            const int row0 = m0 + quarter * 32, n0 = nt * width;
            const uint32_t buf = local & 1, acc = tmem + buf * kSecond + (uint32_t(quarter * 32) << 16);
            const uint32_t done = peer_addr(SCALED ? drained : drained + 8 * buf, 0);
            float ra = 1.0f;
            const int steps = (units + 1) / 2;
            // the shared columns are the last of the first accumulator and the first of the second
            auto unit_of_step = [&](int i) { return buf ? 2 * i + side : units - 1 - (2 * i + side); };
            // NV: the factors of the columns that this warp will write, one in each lane, loaded while the
            // products run
            constexpr int SETS = MODE == kGated ? 2 : 1;
            float factor[4];                               // of each step, gate before up: at most 4 in all
            if (KIND == kNv) {
                if (row0 + lane < g.m) ra = p.row_a[row0 + lane];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int col = n0 + 32 * unit_of_step(i / SETS) + lane;
                    factor[i] = col >= n0 && col < g.n ? p.row_b[i % SETS][col] : 0.0f;
                }
            }
            const uint32_t limit = wait_limit(g.stages * (MODE == kGrads ? g.parts : 1));
            if (!barrier_wait_warp(ready + 8 * buf, local / 2 & 1, &abort, limit)) break;
            fence_after();
#pragma unroll
            for (int i = 0; i < 4 / (SCALED ? SETS : 1); ++i) {
                if (i >= steps) break;
                __syncwarp();
                const int u = unit_of_step(i);
                const bool live = u >= 0 && u < units;
                uint32_t r[32], q[32];
                if (live) {
                    tmem_load32(acc + 32 * u, r);
                    if (MODE == kGated) tmem_load32(acc + half + 32 * u, q);
                    tmem_wait_loads();
                }
                if (i == (SCALED ? 0 : steps - 1)) {
                    fence_before();
                    __syncwarp();
                    if (lane == 0) barrier_arrive_pair(done);
                }
                if (!live) continue;
                if constexpr (KIND == kNv) {
                    __syncwarp();                          // the step before has been scaled
#pragma unroll
                    for (int q = 0; q < SETS; ++q) factors[warp][32 * q + lane] = factor[SETS * i + q];
                    __syncwarp();
                }
                const int col0 = n0 + 32 * u;
                float v[32];
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(r[j]);
                if constexpr (KIND == kNv) scale_columns(v, ra, factors[warp]);
                if constexpr (MODE == kGated) {
                    float w[32];
#pragma unroll
                    for (int j = 0; j < 32; ++j) w[j] = __uint_as_float(q[j]);
                    if constexpr (KIND == kNv) scale_columns(w, ra, factors[warp] + 32);
                    float h[32];
#pragma unroll
                    for (int j = 0; j < 32; ++j) h[j] = act(v[j], p.act) * w[j];
                    store(g, 0, row0, col0, h);
                    if (KIND == kHalf && p.save) {
                        store(g, 1, row0, col0, v);
                        store(g, 2, row0, col0, w);
                    }
                } else {
                    if (MODE == kGrads && scale != 1.0f) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] *= scale;
                    }
                    store(g, which, row0, col0, v);
                }
            }
        }
        if (lane == 0) tma_store_wait_all();
        __syncwarp();
    }
    fence_before();
    __syncthreads();
    cluster_sync();             // the other CTA reads this one's shared memory and arrives on its barriers
    if (warp == kEpilogueWarps) {
        fence_after();
        tmem_free<2>(tmem, 512);
    }
    grid_end(p.order);
}

// ---------------------------------------------------------------- 16-bit rows, element by element
// dU = dh act(g), dG = dh u act'(g) in fp32, rounded to the 16-bit type that the gradients' products
// read (the tensor cores take 16-bit operands; the sums over them stay in fp32).  Bound by DRAM: 8192 x 2688,
// 220 MB in 39 us, 5.6 TB/s.
struct GradArgs {
    const void *dh, *g, *u;
    void *dg, *du;
    size_t ld_dh, ld_gu, ld_out;      // ld_out is a multiple of 8; columns [cols, ld_out) are not read
    float *row_top, *factor;          // fp16: see below
    int rows, cols, act, unit;        // unit: bytes that the rows of dh, g and u start on multiples of
};
constexpr int kGradGroups = 2;        // groups of 8 elements of a thread, loaded together

// One row by one CTA, divided by a power of two (`times`: its inverse); the largest finite magnitude that this
// thread met, before that.
template <int DT, bool WIDE>
__device__ __forceinline__ float gate_grad_row(const GradArgs& p, size_t row, float times) {
    using Kept = typename std::conditional<WIDE, float, uint16_t>::type;
    const int span = blockDim.x * 8;
    const uint16_t* const dh = static_cast<const uint16_t*>(p.dh) + row * p.ld_dh;
    const Kept* const g = static_cast<const Kept*>(p.g) + row * p.ld_gu;
    const Kept* const u = static_cast<const Kept*>(p.u) + row * p.ld_gu;
    auto load = [&](const uint16_t* src, int col) {
        if (p.unit >= 16 && col + 8 <= p.cols) return *reinterpret_cast<const uint4*>(src + col);
        if (p.unit >= 4 && col + 8 <= p.cols) {
            const uint32_t* q = reinterpret_cast<const uint32_t*>(src + col);
            return make_uint4(q[0], q[1], q[2], q[3]);
        }
        uint32_t w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = col + j < p.cols ? src[col + j] : 0;
        return make_uint4(w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16);
    };
    // eight of g or u, as floats where they were kept in fp32
    struct Eight {
        uint4 w[WIDE ? 2 : 1];
    };
    auto load_kept = [&](const Kept* src, int col) {
        Eight v;
        if constexpr (!WIDE) {
            v.w[0] = load(src, col);
        } else if (p.unit >= 16 && col + 8 <= p.cols) {
            v.w[0] = *reinterpret_cast<const uint4*>(src + col);
            v.w[1] = *reinterpret_cast<const uint4*>(src + col + 4);
        } else {
            uint32_t w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = col + j < p.cols ? __float_as_uint(src[col + j]) : 0;
            v.w[0] = make_uint4(w[0], w[1], w[2], w[3]);
            v.w[1] = make_uint4(w[4], w[5], w[6], w[7]);
        }
        return v;
    };
    auto pair = [&](const Eight& v, int j) {
        if constexpr (WIDE) {
            const uint4& q = v.w[j / 2];
            return j & 1 ? make_float2(__uint_as_float(q.z), __uint_as_float(q.w)) : make_float2(__uint_as_float(q.x), __uint_as_float(q.y));
        } else {
            const uint4& q = v.w[0];
            return unpack2(j == 0 ? q.x : j == 1 ? q.y : j == 2 ? q.z : q.w, DT);
        }
    };
    float top = 0.0f;
    auto rounded = [&](float a, float b) {
        if constexpr (DT == kFp16) {
            if (fabsf(a) < __uint_as_float(0x7F800000u)) top = fmaxf(top, fabsf(a));
            if (fabsf(b) < __uint_as_float(0x7F800000u)) top = fmaxf(top, fabsf(b));
            return pack2(a * times, b * times, DT);
        } else {
            return pack2(a, b, DT);
        }
    };
    for (int first = threadIdx.x * 8; first < p.cols; first += span * kGradGroups) {
        uint4 a[kGradGroups];
        Eight b[kGradGroups], c[kGradGroups];
#pragma unroll
        for (int i = 0; i < kGradGroups; ++i) {
            const int col = first + i * span;
            if (col >= p.cols) continue;
            a[i] = load(dh, col);
            b[i] = load_kept(g, col);
            c[i] = load_kept(u, col);
        }
#pragma unroll
        for (int i = 0; i < kGradGroups; ++i) {
            const int col = first + i * span;
            if (col >= p.cols) continue;
            const uint32_t wa[4] = {a[i].x, a[i].y, a[i].z, a[i].w};
            uint32_t og[4], ou[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 fh = unpack2(wa[j], DT), fg = pair(b[i], j), fu = pair(c[i], j);
                float v0, v1, s0, s1;
                act_grad(fg.x, p.act, v0, s0);
                act_grad(fg.y, p.act, v1, s1);
                ou[j] = rounded(fh.x * v0, fh.y * v1);
                og[j] = rounded(fh.x * fu.x * s0, fh.y * fu.y * s1);
            }
            *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.dg) + row * p.ld_out + col) = make_uint4(og[0], og[1], og[2], og[3]);
            *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.du) + row * p.ld_out + col) = make_uint4(ou[0], ou[1], ou[2], ou[3]);
        }
    }
    return top;
}
// the largest of all threads' values, none of them negative; every thread gets it
__device__ __forceinline__ float block_max(float v, uint32_t (&shared)[16]) {
    const int lane = threadIdx.x & 31, warps = blockDim.x / 32;
    uint32_t m = __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(v));
    if (lane == 0) shared[threadIdx.x >> 5] = m;
    __syncthreads();
    m = __reduce_max_sync(0xFFFFFFFFu, lane < warps ? shared[lane] : 0);
    return __uint_as_float(m);
}

// One CTA a row.  WIDE: g and u were kept in fp32.
template <int DT, bool WIDE>
__global__ void __launch_bounds__(512) gate_grad_kernel(const __grid_constant__ GradArgs p) {
    __shared__ uint32_t shared[16];
    grid_launch();
    grid_wait();
    float top = gate_grad_row<DT, WIDE>(p, blockIdx.x, 1.0f);
    if constexpr (DT == kFp16) {
        top = block_max(top, shared);
        if (threadIdx.x == 0) p.row_top[blockIdx.x] = top;
    }
}

// fp16 alone: dU and dG are products of up to three fp16 numbers and may lie outside its range while the gradients,
// sums over them, lie inside.  Where the largest finite one would round to infinity, or is below 2^-4 (above, no
// rounding error exceeds 2^-21 of it, subnormal numbers included), all are computed again, divided by the power of two
// that brings it into [2^14, 2^15); the products' outputs are multiplied by it (*factor, else 1).  One for both,
// because dx adds products with both.  A few CTAs that each find the largest of all rows.  Where all fit it costs 1 us
// (backward pass of 2048 x 3840, 1920: 98.4 -> 99.5 us).
template <bool WIDE>
__global__ void __launch_bounds__(512) grad_range_kernel(const __grid_constant__ GradArgs p) {
    __shared__ uint32_t shared[16];
    grid_launch();
    grid_wait();
    float top = 0.0f;
    for (int row = threadIdx.x; row < p.rows; row += blockDim.x) top = fmaxf(top, p.row_top[row]);
    top = block_max(top, shared);
    const bool fits = top == 0.0f || (top >= 0x1p-4f && top < 65520.0f);
    const int e = fits ? 0 : max(int(__float_as_uint(top) >> 23), 1) - 127 - 14;      // top = 1.f * 2^(e + 14)
    if (blockIdx.x == 0 && threadIdx.x == 0) *p.factor = __uint_as_float(uint32_t(127 + max(e, -100)) << 23);
    if (fits) return;
    const float times = __uint_as_float(uint32_t(127 - max(e, -100)) << 23);
    for (int row = blockIdx.x; row < p.rows; row += gridDim.x) gate_grad_row<kFp16, WIDE>(p, row, times);
}

// 16-bit words to rows whose stride is a multiple of 16 bytes, up to three matrices in a launch
struct PackJob {
    const uint16_t* src;
    uint16_t* dst;
    size_t ld_src, ld_dst;
    int rows, cols, unit;
};
struct PackArgs {
    PackJob job[3];
};
// One CTA a row.  The source is read in words of 4 bytes where its rows start on such, else of 2.
__global__ void __launch_bounds__(512) pack_kernel(const __grid_constant__ PackArgs p) {
    grid_launch();
    grid_wait();
    size_t row = blockIdx.x;
    int i = 0;
    while (i < 2 && row >= size_t(p.job[i].rows)) row -= p.job[i++].rows;
    const PackJob& g = p.job[i];
    const uint16_t* const src = g.src + row * g.ld_src;
    uint16_t* const dst = g.dst + row * g.ld_dst;
    for (int col = threadIdx.x * 2; col < int(g.ld_dst); col += blockDim.x * 2) {
        uint32_t w;
        if (g.unit >= 4 && col + 2 <= g.cols)
            w = *reinterpret_cast<const uint32_t*>(src + col);
        else
            w = (col < g.cols ? src[col] : 0) | uint32_t(col + 1 < g.cols ? src[col + 1] : 0) << 16;
        *reinterpret_cast<uint32_t*>(dst + col) = w;
    }
}

// ---------------------------------------------------------------- microscaled 4-bit floating point
// Scales are stored as the tensor cores take them: tiles of 128 rows x 4 scales, the scale of row r and
// block b at byte (r % 32) * 16 + (r % 128 / 32) * 4 + b % 4 of tile (r / 128, b / 4); the tiles of a
// 128-row group are consecutive and cover a whole number of 256-element stages.
template <bool MX>
__host__ __device__ constexpr int blocks_per_stage() { return MX ? 8 : 16; }
template <bool MX>
__host__ __device__ inline size_t scale_offset(size_t row, size_t block, size_t stages) {
    return (row / 128 * stages * (blocks_per_stage<MX>() / 4) + block / 4) * 512 + (row % 32) * 16 + (row % 128 / 32) * 4 +
           block % 4;
}

struct QuantArgs {
    const void* x;
    uint8_t *codes, *scales;
    float* row_scales;
    size_t ld;
    int rows, cols, dtype, unit;      // unit: bytes that base and row stride are multiples of: 32, 16, 8, 4 or 2
};

// eight codes, the first in the lowest nibble
__device__ __forceinline__ uint32_t encode8(const float* v) {
    uint32_t r;
    asm("{\n .reg .b8 a, b, c, d;\n"
        " cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n"
        " cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n"
        " mov.b32 %0, {a, b, c, d};\n}"
        : "=r"(r)
        : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return r;
}
__device__ __forceinline__ void decode8(uint32_t w, float* v) {
    uint32_t h[4];
    asm("{\n .reg .b8 a, b, c, d;\n mov.b32 {a, b, c, d}, %4;\n"
        " cvt.rn.f16x2.e2m1x2 %0, a;\n cvt.rn.f16x2.e2m1x2 %1, b;\n"
        " cvt.rn.f16x2.e2m1x2 %2, c;\n cvt.rn.f16x2.e2m1x2 %3, d;\n}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
        : "r"(w));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = unpack2(h[i], kFp16);
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}
constexpr int kRowChunks = 3;                    // groups of 16 elements that a thread holds in registers

// 16 neighbouring elements as they are stored: 8 registers of 16-bit pairs or 16 floats
template <int DT> struct Group {
    uint32_t w[DT == kFp32 ? 16 : 8];
};

template <int DT>
__device__ __forceinline__ void load_elements(const QuantArgs& p, size_t row, int col, Group<DT>& g) {
    if constexpr (DT == kFp32) {
        const uint32_t* q = static_cast<const uint32_t*>(p.x) + row * p.ld;
#pragma unroll
        for (int i = 0; i < 16; ++i) g.w[i] = col + i < p.cols ? q[col + i] : 0;
    } else {
        const uint16_t* q = static_cast<const uint16_t*>(p.x) + row * p.ld;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            g.w[i] = (col + 2 * i < p.cols ? q[col + 2 * i] : 0) | uint32_t(col + 2 * i + 1 < p.cols ? q[col + 2 * i + 1] : 0) << 16;
    }
}
// A group that starts anywhere, from the aligned 16-byte words around it; element by element where a word
// would reach outside the matrix or the group outside its row.  One 2- or 4-byte load for each element or
// pair left most of a sector unused: 8192 x 5001 bf16 NV 50.3 us, now 28.6; 8192 x 5002 fp32 84.2, now 49.2; a
// single row of 1250, which has nothing to save, 2.3 and 2.5.
template <int DT>
__device__ __forceinline__ void load_shifted(const QuantArgs& p, size_t row, int col, Group<DT>& g) {
    constexpr int W = DT == kFp32 ? 16 : 8, SIZE = DT == kFp32 ? 4 : 2;
    const uintptr_t first = reinterpret_cast<uintptr_t>(p.x), end = first + ((p.rows - 1) * p.ld + p.cols) * SIZE;
    const uintptr_t at = first + (row * p.ld + col) * SIZE, from = at & ~uintptr_t(15);
    if (col + 16 > p.cols || from < first || from + 4 * W + 16 > end) return load_elements<DT>(p, row, col, g);
    uint32_t w[W + 4];
#pragma unroll
    for (int i = 0; i < W + 4; i += 4) {
        const uint4 v = reinterpret_cast<const uint4*>(from)[i / 4];
        w[i] = v.x; w[i + 1] = v.y; w[i + 2] = v.z; w[i + 3] = v.w;
    }
#pragma unroll
    for (int i = 0; i < W + 2; ++i) w[i] = at & 8 ? w[i + 2] : w[i];
#pragma unroll
    for (int i = 0; i < W + 1; ++i) w[i] = at & 4 ? w[i + 1] : w[i];
#pragma unroll
    for (int i = 0; i < W; ++i) g.w[i] = DT == kFp32 ? w[i] : __funnelshift_r(w[i], w[i + 1], at & 2 ? 16 : 0);
}
// rows on multiples of 16 bytes; WORDS (16-bit types): on any multiples, best on those of 4
template <int DT, bool WORDS>
__device__ __forceinline__ void load_group(const QuantArgs& p, size_t row, int col, Group<DT>& g) {
    constexpr int W = DT == kFp32 ? 16 : 8, PER = 16 / W;
    if (p.unit == 32 && col + 16 <= p.cols) {
        const uint8_t* q = static_cast<const uint8_t*>(p.x) + (row * p.ld + col) * (4 / PER);
#pragma unroll
        for (int i = 0; i < W / 8; ++i) load_256(q + 32 * i, g.w + 8 * i);
    } else if (p.unit == 16 && col + 16 <= p.cols) {
        const uint4* q = reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(p.x) + (row * p.ld + col) * (4 / PER));
#pragma unroll
        for (int i = 0; i < W / 4; ++i) {
            const uint4 v = q[i];
            g.w[4 * i] = v.x; g.w[4 * i + 1] = v.y; g.w[4 * i + 2] = v.z; g.w[4 * i + 3] = v.w;
        }
    } else if (WORDS && p.unit >= 4 && col + 16 <= p.cols) {
        const uint32_t* q = reinterpret_cast<const uint32_t*>(static_cast<const uint16_t*>(p.x) + row * p.ld + col);
#pragma unroll
        for (int i = 0; i < W; ++i) g.w[i] = q[i];
    } else {
        load_elements<DT>(p, row, col, g);
    }
}

// the largest magnitude as fp32 bits; infinity and NaN come out on top.  Magnitudes of one format order
// like their bits: pairs are compared as 16-bit integers, and only the largest is widened.
template <int DT>
__device__ __forceinline__ uint32_t group_amax(const Group<DT>& g) {
    uint32_t m = 0;
    if constexpr (DT == kFp32) {
#pragma unroll
        for (int i = 0; i < 16; ++i) m = max(m, g.w[i] & 0x7FFFFFFFu);
        return m;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) asm("max.u16x2 %0, %0, %1;" : "+r"(m) : "r"(g.w[i] & 0x7FFF7FFFu));
        m = max(m >> 16, m & 0xFFFFu);
        return DT == kBf16 ? m << 16 : __float_as_uint(unpack2(m, kFp16).x) & 0x7FFFFFFFu;
    }
}
template <int DT>
__device__ __forceinline__ void group_values(const Group<DT>& g, float (&v)[16]) {
    if constexpr (DT == kFp32) {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(g.w[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float2 f = unpack2(g.w[i], DT);
            v[2 * i] = f.x;
            v[2 * i + 1] = f.y;
        }
    }
}

// The scale of a block and what its elements are multiplied by, from the block's largest magnitude (as
// fp32 bits).
//   MX: 32 elements share e = max(floor(log2 amax) - 2, -127): the power of two that brings the largest
//       element into [4, 8); code = rn(v / 2^e), above 6 it saturates.  Every step but the rounding is exact.
//   NV: 16 elements share s = e4m3_rn(min(amax * up, 448)), up = 448 / A, A the row's amax; d = s * g, g =
//       A / 2688; code = rn(v * (1 / d)), all zero where s is.  A row below 2^-100 is zero (up = 0).
// A value that is not finite makes its block's scale (MX) or its row's g (NV) NaN.
template <bool MX>
__device__ __forceinline__ void block_scale(uint32_t amax, float up, float g, uint32_t& byte, float& inv) {
    if (MX) {
        const int e = max(int(amax >> 23) - 2, 0);         // the stored byte: exponent + 127
        byte = amax >= kInfBits ? 255u : uint32_t(e);
        inv = amax >= kInfBits ? 0.0f : __uint_as_float(uint32_t(254 - e) << 23);
    } else {
        byte = up > 0.0f ? to_e4m3(fminf(__fmul_rn(__uint_as_float(amax), up), 448.0f)) : 0;
        const float s = from_e4m3(byte);
        inv = s > 0.0f ? __frcp_rn(__fmul_rn(s, g)) : 0.0f;
    }
}
// the row's factor g and up, from the row's largest magnitude
__device__ __forceinline__ void row_factors(uint32_t amax, float& up, float& g) {
    const float a = __uint_as_float(amax);
    up = 0.0f;
    g = 0.0f;
    if (amax >= kInfBits) {
        g = __uint_as_float(0x7FFFFFFFu);
    } else if (a >= 0x1p-100f) {
        g = __fdiv_rn(a, 2688.0f);
        up = __fdiv_rn(448.0f, a);
    }
}
__device__ __forceinline__ uint2 encode_values(float (&v)[16], float inv) {
#pragma unroll
    for (int i = 0; i < 16; i += 2) mul2(v[i], v[i + 1], inv);
    return make_uint2(encode8(v), encode8(v + 8));
}
template <int DT>
__device__ __forceinline__ uint2 encode_group(const Group<DT>& g, float inv) {
    float v[16];
    group_values<DT>(g, v);
    return encode_values(v, inv);
}
// One CTA a row, one thread 16 neighbouring elements at a time.  A thread's three groups are loaded together
// and stay in registers between the row's maximum and the rounding, so a row of up to 48 elements a thread
// is read once; only longer rows (above 24576 elements) are read a second time for the NV form.  Two and four
// groups were no faster (8192 x 5376 NV: 25.1, 24.2 against 24.4 us; 8192 x 2688: 13.3, 16.3 against 14.0).  8192 x
// 5376: MX 19.6 us, 5.8 TB/s of what has to move; NV 24.4 us, 4.6 TB/s, bound by instruction issue (66 %): the
// row's maximum, a division and two conversions for every 16 elements.
//
// ANYWHERE: rows that do not start on multiples of 16 bytes.
template <bool MX, int DT, bool ANYWHERE>
__global__ void __launch_bounds__(512) fp4_quantize_kernel(const __grid_constant__ QuantArgs p) {
    __shared__ uint32_t top[16];
    const int tid = threadIdx.x, threads = blockDim.x, span = threads * 16 * kRowChunks;
    const size_t row = blockIdx.x;
    const size_t stages = (size_t(p.cols) + 255) / 256;
    const int padded = int(stages * 256);
    const int stride = (p.cols + 31) / 32 * 16;            // bytes of a row of codes
    grid_launch();
    grid_wait();

    Group<DT> x[kRowChunks];
    uint32_t peak[kRowChunks];
    auto load = [&](int first) {
#pragma unroll
        for (int c = 0; c < kRowChunks; ++c) {
            const int col = first + (c * threads + tid) * 16;
            if constexpr (ANYWHERE) load_shifted<DT>(p, row, col, x[c]);
            else load_group<DT, false>(p, row, col, x[c]);
        }
#pragma unroll
        for (int c = 0; c < kRowChunks; ++c) peak[c] = group_amax<DT>(x[c]);
    };
    const bool once = span >= padded;
    float up = 0.0f, g = 0.0f;
    if (!MX) {
        uint32_t m = 0;
        for (int first = 0; first < p.cols; first += span) {
            load(first);
#pragma unroll
            for (int c = 0; c < kRowChunks; ++c) m = max(m, peak[c]);
        }
        m = __reduce_max_sync(0xFFFFFFFFu, m);
        if (threads > 32) {
            if ((tid & 31) == 0) top[tid >> 5] = m;
            __syncthreads();
            m = __reduce_max_sync(0xFFFFFFFFu, (tid & 31) < threads / 32 ? top[tid & 31] : 0);
        }
        row_factors(m, up, g);
        if (tid == 0) p.row_scales[row] = g;
    }
    uint8_t* const codes = p.codes + row * size_t(stride) + tid * 8;
    uint8_t* const scales = p.scales + scale_offset<MX>(row, 0, stages);
    for (int first = 0; first < padded; first += span) {
        if (MX || !once) load(first);
#pragma unroll
        for (int c = 0; c < kRowChunks; ++c) {
            const int col = first + (c * threads + tid) * 16;
            constexpr int PER = MX ? 2 : 1;                // threads of a block
            uint32_t m = peak[c], byte;
            if (MX) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
            float inv;
            block_scale<MX>(m, up, g, byte, inv);
            const uint2 code = encode_group<DT>(x[c], inv);
            if (col / 2 + 8 <= stride) *reinterpret_cast<uint2*>(codes + (first + c * threads * 16) / 2) = code;
            const uint32_t word = gather_scales<PER>(byte);
            if (tid % (4 * PER) == 0 && col < padded)      // 4 scales of the row lie together, 512 bytes from the next 4
                *reinterpret_cast<uint32_t*>(scales + size_t(col / (64 * PER)) * 512) = word;
        }
    }
}

struct DequantArgs {
    const uint8_t *codes, *scales;
    const float* row_scales;
    void* out;
    size_t ld;
    int rows, cols, dtype, unit;
};
// An output row that starts anywhere: groups of 8 elements begin where the output is aligned to 16 bytes, and
// a group's codes are cut out of two neighbouring words.  It touches at most two blocks.  Two elements a
// thread with narrow stores took 55 us for 8192 x 5001 bf16 MX; this takes 32.4.
template <bool MX>
__device__ __forceinline__ void dequantize_shifted(const DequantArgs& p, size_t row, float g) {
    constexpr int B = MX ? 32 : 16;
    const int threads = blockDim.x, stride = (p.cols + 31) / 32 * 16;
    const size_t stages = (size_t(p.cols) + 255) / 256;
    const int size = p.dtype == kFp32 ? 4 : 2;
    uint8_t* const out = static_cast<uint8_t*>(p.out) + row * p.ld * size;
    const int head = int((16 - (reinterpret_cast<uintptr_t>(out) & 15)) & 15) / size;
    const uint8_t* const scales = p.scales + scale_offset<MX>(row, 0, stages);
    const uint32_t* const codes = reinterpret_cast<const uint32_t*>(p.codes + row * size_t(stride));
    for (int first = (head ? head - 8 : 0) + int(threadIdx.x) * 8; first < p.cols; first += threads * 8 * kRowChunks) {
        uint32_t w[kRowChunks], b0[kRowChunks], b1[kRowChunks];
#pragma unroll
        for (int c = 0; c < kRowChunks; ++c) {
            const int col = first + c * threads * 8;
            if (col >= p.cols) continue;
            const int word = col >> 3;                     // -1 for the group before the first boundary
            const uint32_t lo = word >= 0 ? codes[word] : 0, hi = (word + 1) * 4 < stride ? codes[word + 1] : 0;
            w[c] = __funnelshift_r(lo, hi, (col & 7) * 4);
            const int i0 = max(col, 0) / B, i1 = min(col + 7, p.cols - 1) / B;
            b0[c] = scales[size_t(i0 / 4) * 512 + i0 % 4];
            b1[c] = scales[size_t(i1 / 4) * 512 + i1 % 4];
        }
#pragma unroll
        for (int c = 0; c < kRowChunks; ++c) {
            const int col = first + c * threads * 8;
            if (col >= p.cols) continue;
            const float d0 = MX ? from_e8m0(b0[c]) : __fmul_rn(from_e4m3(b0[c]), g);
            const float d1 = MX ? from_e8m0(b1[c]) : __fmul_rn(from_e4m3(b1[c]), g);
            const int n = (max(col, 0) / B + 1) * B - col; // elements of the first block
            float v[8];
            decode8(w[c], v);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = __fmul_rn(v[j], j < n ? d0 : d1);
            if (col < 0 || col + 8 > p.cols) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (col + j >= 0 && col + j < p.cols) store1(out, size_t(col + j), v[j], p.dtype);
            } else if (p.dtype == kFp32) {
                float4* const q = reinterpret_cast<float4*>(out + size_t(col) * 4);
                q[0] = make_float4(v[0], v[1], v[2], v[3]);
                q[1] = make_float4(v[4], v[5], v[6], v[7]);
            } else {
                *reinterpret_cast<uint4*>(out + size_t(col) * 2) =
                    make_uint4(pack2(v[0], v[1], p.dtype), pack2(v[2], v[3], p.dtype), pack2(v[4], v[5], p.dtype),
                               pack2(v[6], v[7], p.dtype));
            }
        }
    }
}

// value = code * scale (MX), code * (scale * row factor) (NV) in fp32, rounded once to the output type.
// One CTA a row as above: a thread's three groups are in flight together.  8192 x 5376: MX 18.9 us, 5.9 TB/s, NV
// 22.8 us; bound by DRAM writes.
template <bool MX>
__global__ void __launch_bounds__(512) fp4_dequantize_kernel(const __grid_constant__ DequantArgs p) {
    const int tid = threadIdx.x, threads = blockDim.x, span = threads * 16 * kRowChunks;
    const size_t row = blockIdx.x, stages = (size_t(p.cols) + 255) / 256;
    const int stride = (p.cols + 31) / 32 * 16;
    grid_launch();
    grid_wait();
    const float g = MX ? 1.0f : p.row_scales[row];
    if (p.unit < 16) {
        dequantize_shifted<MX>(p, row, g);
        return;
    }
    for (int first = 0; first < p.cols; first += span) {
        uint2 w[kRowChunks];
        uint32_t b[kRowChunks];
#pragma unroll
        for (int c = 0; c < kRowChunks; ++c) {
            const int col = first + (c * threads + tid) * 16;
            if (col >= p.cols) continue;
            w[c] = *reinterpret_cast<const uint2*>(p.codes + row * size_t(stride) + col / 2);
            b[c] = p.scales[scale_offset<MX>(row, size_t(col) / (MX ? 32 : 16), stages)];
        }
#pragma unroll
        for (int c = 0; c < kRowChunks; ++c) {
            const int col = first + (c * threads + tid) * 16;
            if (col >= p.cols) continue;
            const float d = MX ? from_e8m0(b[c]) : __fmul_rn(from_e4m3(b[c]), g);
            float v[16];
            decode8(w[c].x, v);
            decode8(w[c].y, v + 8);
#pragma unroll
            for (int j = 0; j < 16; ++j) v[j] = __fmul_rn(v[j], d);
            const size_t at = row * p.ld + col;
            if (col + 16 > p.cols) {
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    if (col + j < p.cols) store1(p.out, at + j, v[j], p.dtype);
            } else if (p.dtype == kFp32) {
                float4* q = reinterpret_cast<float4*>(static_cast<float*>(p.out) + at);
#pragma unroll
                for (int j = 0; j < 4; ++j) q[j] = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
            } else {
                uint32_t o[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] = pack2(v[2 * j], v[2 * j + 1], p.dtype);
                if (p.unit == 32) {
                    store_256(static_cast<uint16_t*>(p.out) + at, o);
                } else {
                    uint4* q = reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.out) + at);
                    q[0] = make_uint4(o[0], o[1], o[2], o[3]);
                    q[1] = make_uint4(o[4], o[5], o[6], o[7]);
                }
            }
        }
    }
}

// ---------------------------------------------------------------- microscaled 8-bit floating point
// One CTA a row, a thread three groups of 16 neighbouring elements at a time, loaded together; two threads are a block.
// ANYWHERE as above.  8192 x 5376: 22 us, 6.1 TB/s; bound by DRAM.
template <int DT, bool ANYWHERE>
__global__ void __launch_bounds__(512) fp8_quantize_kernel(const __grid_constant__ QuantArgs p) {
    const int tid = threadIdx.x, threads = blockDim.x;
    const size_t row = blockIdx.x, stages = fp8_stages(p.cols), stride = fp8_stride(p.cols);
    const int padded = int(stages * 128);
    uint8_t* const codes = p.codes + row * stride;
    uint8_t* const scales = p.scales + fp8_scale_offset(row, 0, stages);
    grid_launch();
    grid_wait();
    for (int first = tid * 16; first - tid * 16 < padded; first += threads * 16 * kRowChunks) {
        Group<DT> x[kRowChunks];
#pragma unroll
        for (int c = 0; c < kRowChunks; ++c) {
            const int col = first + c * threads * 16;
            if constexpr (ANYWHERE) load_shifted<DT>(p, row, col, x[c]);
            else load_group<DT, false>(p, row, col, x[c]);
        }
#pragma unroll
        for (int c = 0; c < kRowChunks; ++c) {
            const int col = first + c * threads * 16;
            uint32_t m = group_amax<DT>(x[c]), byte;
            m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
            float inv, v[16];
            fp8_block_scale(m, byte, inv);
            group_values<DT>(x[c], v);
            const uint4 code = encode_e4m3(v, inv);
            if (col < int(stride)) *reinterpret_cast<uint4*>(codes + col) = code;
            const uint32_t word = gather_scales<2>(byte);
            if (tid % 8 == 0 && col < padded) *reinterpret_cast<uint32_t*>(scales + size_t(col / 128) * 512) = word;
        }
    }
}

// value = code * scale in fp32, rounded once to the output type.  One CTA a row; a thread takes 16 neighbouring elements
// where output rows start on multiples of 16 bytes, else (NARROW) two where they do on multiples of a pair, or one, the
// next thread the next ones, so that a warp's stores are whole sectors anyway.  8192 x 5376: 21 us, 6.3 TB/s.
template <int NARROW>
__device__ __forceinline__ void fp8_dequantize_narrow(const DequantArgs& p, size_t row, const uint8_t* codes, const uint8_t* scales) {
    for (int col = threadIdx.x * NARROW; col < p.cols; col += blockDim.x * NARROW) {
        const float d = from_e8m0(scales[size_t(col / 128) * 512 + col / 32 % 4]);
        const float2 v = decode_e4m3(NARROW == 2 ? *reinterpret_cast<const uint16_t*>(codes + col) : codes[col]);
        const size_t at = row * p.ld + col;
        const float a = __fmul_rn(v.x, d), b = __fmul_rn(v.y, d);
        if (NARROW == 1 || col + 1 >= p.cols) store1(p.out, at, a, p.dtype);
        else if (p.dtype == kFp32) *reinterpret_cast<float2*>(static_cast<float*>(p.out) + at) = make_float2(a, b);
        else *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(p.out) + at) = pack2(a, b, p.dtype);
    }
}
__global__ void __launch_bounds__(512) fp8_dequantize_kernel(const __grid_constant__ DequantArgs p) {
    const int tid = threadIdx.x, threads = blockDim.x;
    const size_t row = blockIdx.x;
    const uint8_t* const codes = p.codes + row * fp8_stride(p.cols);
    const uint8_t* const scales = p.scales + fp8_scale_offset(row, 0, fp8_stages(p.cols));
    grid_launch();
    grid_wait();
    if (p.unit < 16) {
        if (p.unit >= (p.dtype == kFp32 ? 8 : 4)) fp8_dequantize_narrow<2>(p, row, codes, scales);
        else fp8_dequantize_narrow<1>(p, row, codes, scales);
        return;
    }
    for (int first = tid * 16; first < p.cols; first += threads * 16 * kRowChunks) {
        uint4 w[kRowChunks];
        uint32_t b[kRowChunks];
#pragma unroll
        for (int c = 0; c < kRowChunks; ++c) {
            const int col = first + c * threads * 16;
            if (col >= p.cols) continue;
            w[c] = *reinterpret_cast<const uint4*>(codes + col);
            b[c] = scales[size_t(col / 128) * 512 + col / 32 % 4];
        }
#pragma unroll
        for (int c = 0; c < kRowChunks; ++c) {
            const int col = first + c * threads * 16;
            if (col >= p.cols) continue;
            const float d = from_e8m0(b[c]);
            const uint32_t word[4] = {w[c].x, w[c].y, w[c].z, w[c].w};
            float v[16];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float2 f = decode_e4m3(word[j / 2] >> (j & 1) * 16);
                v[2 * j] = __fmul_rn(f.x, d);
                v[2 * j + 1] = __fmul_rn(f.y, d);
            }
            const size_t at = row * p.ld + col;
            if (col + 16 > p.cols) {
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    if (col + j < p.cols) store1(p.out, at + j, v[j], p.dtype);
            } else if (p.dtype == kFp32) {
                float4* q = reinterpret_cast<float4*>(static_cast<float*>(p.out) + at);
#pragma unroll
                for (int j = 0; j < 4; ++j) q[j] = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
            } else {
                uint32_t o[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] = pack2(v[2 * j], v[2 * j + 1], p.dtype);
                if (p.unit == 32) {
                    store_256(static_cast<uint16_t*>(p.out) + at, o);
                } else {
                    uint4* q = reinterpret_cast<uint4*>(static_cast<uint16_t*>(p.out) + at);
                    q[0] = make_uint4(o[0], o[1], o[2], o[3]);
                    q[1] = make_uint4(o[4], o[5], o[6], o[7]);
                }
            }
        }
    }
}

// ---------------------------------------------------------------- few tokens
struct SplitArgs {
    CUtensorMap w[2], x[2];
    const uint8_t* scales_w[2];
    const uint8_t* scales_x;
    const float* row_w[2];
    const float* row_x;
    const float* factor;              // as in TileArgs
    QuantArgs raw;                    // fused: x in 16 bits, quantized by the kernel itself
    Out out[3];
    int features, tokens;             // rows of w, rows of x
    int stages;                       // stages of the reduction axis (of each part of kSum2)
    int nt;                           // tokens of a tile: a multiple of 16, at most 128
    int pipe;                         // stages in shared memory
    int columns;                      // of tensor memory: a power of two
    int ranks;                        // CTAs of a cluster: parts of the reduction axis
    int own;                          // tokens of a tile that one CTA of the cluster adds up
    int reuse;                        // the parts lie where the stages were
    int act, bf16, save, order;
};
constexpr int kSplitThreads = 192, kSplitMaxPipe = 12;
constexpr int kFusedTokens = 16;      // tokens of a tile of the fused form
template <int KIND, int MODE>
__host__ __device__ constexpr int split_stage_bytes(int nt) {
    return (MODE == kGated ? 2 : 1) * (kTileBytes + kScaleBytes<KIND>) + nt * kRowBytes + kScaleBytes<KIND>;
}
// bytes of the parts that a CTA receives for the tokens it adds up
template <int MODE>
__host__ __device__ constexpr int split_part_bytes(int nt, int ranks) {
    return ranks * (MODE == kGated ? 2 : 1) * ((nt + ranks - 1) / ranks) * 128 * 4;
}

// A tile kernel's CTA takes all tensor memory before it waits for the launch before.  If that launch had a CTA on the same SM
// that still had to ask for its own, neither would end: the two must never share an SM.  Shared memory sees to it, also
// for the smallest CTA of the split kernel (one stage, 16 tokens).
constexpr int kSmemOfSm = 228 * 1024, kSmemOfCta = 1024;      // of an SM; what every CTA costs beside its own
constexpr int kLeastSplitSmem = split_stage_bytes<kHalf, kPlain>(16) + split_part_bytes<kPlain>(16, 1) + kSmemSlack;
static_assert(split_stage_bytes<kMx, kPlain>(16) >= split_stage_bytes<kHalf, kPlain>(16) &&
              split_stage_bytes<kMx8, kPlain>(16) >= split_stage_bytes<kHalf, kPlain>(16) &&
              split_part_bytes<kPlain>(16, 8) >= split_part_bytes<kPlain>(16, 1));
static_assert(kLeastSplitSmem >= 24 * 1024);       // what the adapters' kernel counts on
static_assert(kTileSmem<kHalf> + kLeastSplitSmem + 2 * kSmemOfCta > kSmemOfSm &&
              kTileSmem<kMx> + kLeastSplitSmem + 2 * kSmemOfCta > kSmemOfSm &&
              kTileSmem<kNv> + kLeastSplitSmem + 2 * kSmemOfCta > kSmemOfSm &&
              kTileSmem<kMx8> + kLeastSplitSmem + 2 * kSmemOfCta > kSmemOfSm);

// The output transposed: 128 features x nt tokens, so that a single token costs one narrow product over
// each weight tile instead of a 256-row one, and the weights, which are all the bytes there are, are
// read once.  The reduction axis is split over the CTAs of a cluster (cluster dimension x) because
// features / 128 tiles alone would leave most SMs without work.  Each CTA sends its partial sums to the
// CTAs that own their tokens, through distributed shared memory, and the owner adds them in rank order, so
// the sum does not depend on timing.  Few tokens: the parts have a place of their own, and a CTA may send
// as soon as the others have started; many: they lie where the stages were (`reuse`), once all are done.
//
// Measured, one token, 5376 -> 2688, warm: MX product 4.8 us, gated 6.1, 16-bit gated 12.6 (58 MB of weights, 4.6
// TB/s); bound by DRAM where the weights are many, else by the chain of start, first loads (2000 cycles),
// products and the exchange of the sums (2500).
//
// Gradients: kSum2 with weights whose other axis is contiguous (W_MN); kOut2 with the tokens as the
// reduction axis (W_MN and X_MN), features = columns of x and "tokens" = rows of a weight, the second half
// of grid.y being the second output.
//
// FUSED (4 and 8 bits, at most 16 tokens): x comes in 16 bits; the warps that write the output later quantize
// the stages of x first, straight into the swizzled rows that the products read, which saves a launch
// and a round trip of x.
template <int KIND, int MODE, bool W_MN, bool X_MN, bool FUSED>
__global__ void __launch_bounds__(kSplitThreads, 1) split_kernel(const __grid_constant__ SplitArgs p) {
    constexpr bool SCALED = KIND != kHalf, MX = KIND == kMx, NV = KIND == kNv;
    constexpr int SB = kScaleBytes<KIND>, NW = MODE == kGated ? 2 : 1;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t bars[2 * kSplitMaxPipe + 2];
    __shared__ uint32_t tmem_slot;
    __shared__ volatile uint32_t abort;
    __shared__ uint32_t row_max[kFusedTokens];          // fused NV: largest magnitudes of the tokens

    const uint32_t smem = (smem_addr(smem_raw) + 1023u) & ~1023u;
    uint8_t* const smem_ptr = smem_raw + (smem - smem_addr(smem_raw));
    const uint32_t full = smem_addr(bars), empty = full + 8 * kSplitMaxPipe, ready = empty + 8 * kSplitMaxPipe,
                   drain = ready + 8;
    const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const uint32_t xb = p.nt * kRowBytes, STAGE = NW * (kTileBytes + SB) + xb + SB;
    const uint32_t parts = p.reuse ? 0 : p.pipe * STAGE;      // offset of [ranks][NW][own][128] sums

    const int ranks = p.ranks, rank = uniform(cluster_rank());
    const int total = p.stages * (MODE == kSum2 ? 2 : 1);
    const int s0 = int(int64_t(total) * rank / ranks), s1 = int(int64_t(total) * (rank + 1) / ranks);
    const int ttiles = MODE == kOut2 ? gridDim.y / 2 : gridDim.y, which = MODE == kOut2 ? blockIdx.y / ttiles : 0;
    const int f0 = int(blockIdx.x / ranks) * kRowsM, t0 = (blockIdx.y - which * ttiles) * p.nt;

    // Tensor memory is waited for when another kernel's CTA still has it.  So that CTAs of two clusters
    // cannot wait for each other's in a circle, no CTA waits for its cluster while it has tensor memory: it
    // says that it has started before it asks, and gives the memory back before it waits for the sums.  (With
    // `reuse` it says so only when its products are done; the launch then takes all of an SM's shared memory,
    // and no other CTA with tensor memory shares the SM.)
    // What the others may write once they have seen this arrival is ready before it: row_max is zero (its
    // threads' own arrivals release the zeros).
    if (FUSED && threadIdx.x < kFusedTokens) row_max[threadIdx.x] = 0;
    __syncwarp();
    if (!p.reuse) cluster_arrive();

    // the loading warp prepares the barriers and starts; everybody else meets it below
    if (warp == 4) {
        if (lane == 0) {
            prefetch_map(&p.w[0]);
            if (NW == 2 || MODE == kSum2) prefetch_map(&p.w[1]);
            if (!FUSED) prefetch_map(&p.x[0]);
            for (int i = 0; i < p.pipe; ++i) {
                barrier_init(full + 8 * i, FUSED ? 1 + p.tokens : 1);
                barrier_init(empty + 8 * i, 1);
            }
            barrier_init(ready, 1);
            barrier_init(drain, 1);
            abort = 0;
            fence_barrier_init();
        }
        __syncwarp();
    }
    auto load_stage = [&](int it) {
        const int slot = it % p.pipe, s = s0 + it;
        const uint32_t sw = smem + slot * STAGE, sx = sw + NW * kTileBytes, ss = sx + xb, bar = full + 8 * slot;
        const int second = MODE == kSum2 ? s >= p.stages : 0, ks = s - second * p.stages;
        const int kc = SCALED ? ks * kRowBytes : ks * 64;
        barrier_expect_warp(bar, NW * kTileBytes + (FUSED ? 0 : xb) + (SCALED ? (NW + (FUSED ? 0 : 1)) * SB : 0));
        for (int q = 0; q < NW; ++q) {
            const CUtensorMap* mw = &p.w[MODE == kSum2 ? second : q];
            if (W_MN) {
                tma_load_2d(sw, mw, f0, kc, bar);
                tma_load_2d(sw + kChunkBytes, mw, f0 + 64, kc, bar);
            } else {
                tma_load_2d(sw + q * kTileBytes, mw, kc, f0, bar);
            }
            if (SCALED) bulk_load(ss + SB * q, p.scales_w[q] + (size_t(f0 / 128) * p.stages + ks) * SB, SB, bar);
        }
        if (!FUSED) {
            if (X_MN) {
                for (int c = 0; c < p.nt; c += 64) tma_load_2d(sx + c / 64 * kChunkBytes, &p.x[which], t0 + c, kc, bar);
            } else {
                tma_load_2d(sx, &p.x[second], kc, t0, bar);
            }
            if (SCALED) bulk_load(ss + SB * NW, p.scales_x + (size_t(t0 / 128) * p.stages + ks) * SB, SB, bar);
        }
    };
    grid_begin(p.order);
    const int early = min(s1 - s0, p.pipe);
    if (warp == 4) {
        for (int it = 0; it < early; ++it) load_stage(it);
    }
    // FUSED.  A unit is one token's part of one stage: 16 groups of 16 elements, half a warp, or, 8 bits, 8 groups.  The first four
    // warps take the units in the order of the stages, the next one's loads under way.  One body for both
    // 16-bit types and no unrolling: what runs a few times costs mostly the fetching of its instructions.
    constexpr int LANES = KIND == kMx8 ? 8 : 16, AT_ONCE = 32 / LANES;
    const int j = lane % LANES;
    auto for_units = [&](auto&& body) {
        const int n = s1 - s0;
        int it = 0, t = warp * AT_ONCE + lane / LANES;
        auto settle = [&] {
            while (t >= p.tokens && it < n) {
                t -= p.tokens;
                ++it;
            }
        };
        settle();
        Group<kBf16> next = {};                          // the bits of either type
        if (it < n) load_group<kBf16, true>(p.raw, t, ((s0 + it) * LANES + j) * 16, next);
#pragma unroll 1
        while (__any_sync(0xFFFFFFFFu, it < n)) {
            const Group<kBf16> g = next;
            const int at = it, row = t;
            t += 4 * AT_ONCE;
            settle();
            if (it < n) load_group<kBf16, true>(p.raw, t, ((s0 + it) * LANES + j) * 16, next);
            float v[16];
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float2 f = unpack2(g.w[i], p.raw.dtype);
                v[2 * i] = f.x;
                v[2 * i + 1] = f.y;
                m = max(m, max(__float_as_uint(f.x) & 0x7FFFFFFFu, __float_as_uint(f.y) & 0x7FFFFFFFu));
            }
            body(at, row, at < n, v, m);
        }
    };
    if constexpr (FUSED && NV) {
        // The rows' maxima: the cluster's CTAs have the whole of each row between them, and each tells all.
        __syncthreads();
        cluster_wait();                                 // every CTA of the cluster has started
        if (warp < 4) {
            for_units([&](int, int row, bool in, float (&)[16], uint32_t m) {
                // a group past the row's end holds zeros, and so does a unit that does not exist
#pragma unroll
                for (int d = 8; d; d >>= 1) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
                if (in && j == 0)
                    for (int r = 0; r < ranks; ++r) max_cluster_u32(peer_addr(smem_addr(&row_max[row]), r), m);
            });
        }
        __syncwarp();
        cluster_sync();
    }
    if (warp == 5) {
        tmem_alloc<1>(smem_addr(&tmem_slot), p.columns);
        fence_before();
    }
    __syncthreads();
    fence_after();
    const uint32_t tmem = uniform(tmem_slot);

    if (warp == 4) {
        bool ok = true;
        int it = early;
        for (; it < s1 - s0; ++it) {
            const int slot = it % p.pipe;
            if (!(ok = barrier_wait_warp(empty + 8 * slot, (it / p.pipe & 1) ^ 1, &abort))) break;
            load_stage(it);
        }
        // arrivals that are still owed come before the shared memory goes away
        for (int i = max(it - p.pipe, 0); i < it && ok; ++i) ok = barrier_wait_warp(empty + 8 * (i % p.pipe), i / p.pipe & 1, &abort);
        if (gave_up_warp(&abort))
            for (int i = it > p.pipe ? it - p.pipe : 0; i < it; ++i) barrier_drain(full + 8 * (i % p.pipe), i / p.pipe & 1);
        __syncwarp();
    } else if (warp == 5) {
        const uint32_t tw = tmem + NW * p.nt, tx = tw + NW * 4 * kScaleTiles<KIND>;
        bool ok = true;
        for (int it = 0; it < s1 - s0; ++it) {
            const int slot = it % p.pipe;
            if (!(ok = barrier_wait_warp(full + 8 * slot, it / p.pipe & 1, &abort))) break;
            fence_after();
            const uint32_t sw = smem + slot * STAGE, sx = sw + NW * kTileBytes, ss = sx + xb;
            if (SCALED) {
#pragma unroll
                for (int j = 0; j < kScaleTiles<KIND>; ++j) {
#pragma unroll
                    for (int q = 0; q < NW; ++q)
                        copy_scales<1>(tw + (q * kScaleTiles<KIND> + j) * 4, ss + SB * q + 512 * j);
                    copy_scales<1>(tx + 4 * j, ss + SB * NW + 512 * j);
                }
            }
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
                const uint32_t dx = X_MN ? swizzled_desc(sx + 2048 * kk, kChunkBytes) : swizzled_desc(sx + 32 * kk, 16);
#pragma unroll
                for (int q = 0; q < NW; ++q) {
                    const uint32_t a = sw + q * kTileBytes;
                    const uint32_t dw = W_MN ? swizzled_desc(a + 2048 * kk, kChunkBytes) : swizzled_desc(a + 32 * kk, 16);
                    if constexpr (KIND == kMx8) {
                        mma_fp8<1>(tmem + q * p.nt, dw, dx, desc_fp8(128, p.nt, kk), tw + 4 * q, tx, it | kk);
                    } else if constexpr (SCALED) {
                        const int j = KIND == kNv ? kk : kk / 2, which = KIND == kNv ? 0 : (kk & 1) * 2;
                        mma_fp4<1, MX>(tmem + q * p.nt, dw, dx, desc_fp4(MX, 128, p.nt, which),
                                       tw + (q * kScaleTiles<KIND> + j) * 4, tx + 4 * j, it | kk);
                    } else {
                        mma_16bit<1>(tmem + q * p.nt, dw, dx, desc_16bit(p.bf16, W_MN, X_MN, 128, p.nt), it | kk);
                    }
                }
            }
            mma_commit<1>(empty + 8 * slot);
        }
        if (ok) mma_commit<1>(ready);
        if (gave_up_warp(&abort)) {
            mma_commit<1>(drain);
            barrier_drain(drain, 0);
        }
        __syncwarp();
    } else if constexpr (FUSED) {
        // each unit arrives on its stage's barrier
        bool ok = true;
        for_units([&](int at, int row, bool in, float (&v)[16], uint32_t m) {
            const int slot = at % p.pipe;
            float up = 0.0f, factor = 0.0f, inv;
            uint32_t byte;
            if (!NV) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
            if (NV && in) row_factors(row_max[row], up, factor);
            if constexpr (KIND == kMx8) fp8_block_scale(m, byte, inv);
            else block_scale<MX>(m, up, factor, byte, inv);
            auto codes = [&] {
                if constexpr (KIND == kMx8) return encode_e4m3(v, inv);
                else return encode_values(v, inv);
            };
            const auto code = codes();
            // the parts of the warp may wait for different stages, and go on together
            bool vacant = ok;
            if (ok && in && at >= p.pipe) vacant = barrier_wait(empty + 8 * slot, (at / p.pipe & 1) ^ 1, &abort, kWaitLimit);
            ok = __all_sync(0xFFFFFFFFu, vacant);
            if (in && ok) {
                uint8_t* const sx = smem_ptr + slot * STAGE + NW * kTileBytes;
                uint8_t* const ss = sx + xb + SB * NW;
                // byte 8 j, or 16 j, of the row's 128: 16-byte pieces are swizzled by the row
                if constexpr (KIND == kMx8) *reinterpret_cast<uint4*>(sx + row * 128 + ((j ^ (row & 7)) << 4)) = code;
                else *reinterpret_cast<uint2*>(sx + row * 128 + (((j >> 1) ^ (row & 7)) << 4) + (j & 1) * 8) = code;
                const int block = NV ? j : j >> 1;
                if (NV || !(j & 1)) ss[(block >> 2) * 512 + row * 16 + (block & 3)] = uint8_t(byte);
                fence_async_shared();
            }
            __syncwarp();
            if (in && ok && j == 0) barrier_arrive(full + 8 * slot);
        });
    }
    // ---------------------------------------------------- partial sums to their owners
    __syncwarp();
    const int cols = min(p.nt, p.tokens - t0);          // tokens that exist
    const uint32_t lanes = uint32_t((warp & 3) * 32) << 16;
    bool good = true;
    if (warp < 4) {
        good = barrier_wait_warp(ready, 0, &abort, wait_limit(s1 - s0));
        fence_after();
    }
    if (p.reuse) cluster_arrive();                      // this CTA's loads and products are done
    if constexpr (!FUSED || !NV) cluster_wait();        // the others' memory may be written
    if (warp < 4 && good) {
        const uint32_t row = warp * 32 + lane;
        for (int q = 0; q < NW; ++q) {
            int owner = 0, local = 0;
            for (int c = 0; c < cols; c += 16) {
                uint32_t r[16];
                tmem_load16(tmem + q * p.nt + c + lanes, r);
                tmem_wait_loads();
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    if (c + j < cols)
                        st_cluster_f32(peer_addr(smem + parts + (((rank * NW + q) * p.own + local) * 128 + row) * 4, owner),
                                       __uint_as_float(r[j]));
                    if (++local == p.own) {
                        local = 0;
                        ++owner;
                    }
                }
            }
        }
    }
    fence_before();
    __syncthreads();
    if (warp == 5) {
        fence_after();
        tmem_free<1>(tmem, p.columns);
    }
    __syncwarp();
    cluster_sync();

    // A thread adds four neighbouring features of a token.  (One at a time, 128 tokens of 2 parts took 9 us.)
    const int first = rank * p.own, count = min(p.own, cols - first) * 32;
    const float4* const sums = reinterpret_cast<const float4*>(smem_ptr + parts);
    for (int e = threadIdx.x; e < count; e += kSplitThreads) {
        const int t = first + (e >> 5), f = f0 + (e & 31) * 4, n = min(4, p.features - f);
        if (n <= 0) continue;
        float v[4] = {}, w[4] = {};
        for (int r = 0; r < ranks; ++r) {
            const float4 a = sums[r * NW * p.own * 32 + e];
            v[0] += a.x; v[1] += a.y; v[2] += a.z; v[3] += a.w;
            if (MODE == kGated) {
                const float4 b = sums[(r * NW + 1) * p.own * 32 + e];
                w[0] += b.x; w[1] += b.y; w[2] += b.z; w[3] += b.w;
            }
        }
        if (KIND == kNv) {
            float up, rx;
            if (FUSED) row_factors(row_max[t], up, rx); else rx = p.row_x[t0 + t];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (i < n) v[i] = v[i] * rx * p.row_w[0][f + i];
                if (MODE == kGated && i < n) w[i] = w[i] * rx * p.row_w[1][f + i];
            }
        }
        if ((MODE == kSum2 || MODE == kOut2) && p.factor) {
            const float scale = __ldcg(p.factor);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] *= scale;
        }
        const size_t row = size_t(t0 + t);
        if (MODE == kGated) {
            if (KIND == kHalf && p.save) {
                store4(p.out[1], row, f, n, v);
                store4(p.out[2], row, f, n, w);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = act(v[i], p.act) * w[i];
            store4(p.out[0], row, f, n, v);
        } else {
            store4(p.out[which], row, f, n, v);
        }
    }
    grid_end(p.order);
}

}  // namespace ff
}  // namespace equarx
