// Residual addition with root-mean-square norm, its 8-bit output and its gradients.
//
//   norm_kernel        sum = x + residual, y = sum / rms(sum) * (offset + weight), y in 16 bits or microscaled 8
//   norm_grad_kernel   dx of one row after another, and each CTA's part of the weight's gradient
//   norm_parts_kernel  the parts' sum
#pragma once
#include "elements.cuh"
#include "tensor_ops.cuh"

namespace equarx {
namespace ff {

using namespace tc;

constexpr int kGradThreads = 224;          // of the backward pass, at most
constexpr int kGradColumns = kGradThreads * 8;
constexpr int kGradGroups = 5;             // groups of 8 columns for each of its threads, at most
constexpr int kGradStages = 2;             // its rows in shared memory
constexpr int kGradGroupThreads = 3 * kGradThreads, kGradMostGroups = kGradGroupThreads / 32;      // of a CTA that has an SM to itself
constexpr int kGradWide = 1024;            // where each CTA has few rows, at most
constexpr int kRowThreads = 1024;          // of the forward pass, at most

// Eight elements of a row in a thread's registers, pairs of neighbours.  W = 8: all neighbours, for rows that start on
// multiples of 16 bytes.  W = 2 or 1: pairs or single elements, the next thread the next ones, for rows that start on multiples of 4
// or 2 bytes: a warp's accesses are then whole sectors all the same.
struct Place {
    int thread, threads;               // among those that have a row
};
__device__ __forceinline__ Place in_block() { return {int(threadIdx.x), int(blockDim.x)}; }
template <int W>
__device__ __forceinline__ int column_of(int first, int e, Place at = in_block()) {
    if (W == 8) return first + at.thread * 8 + e;
    return first + (e / W * at.threads + at.thread) * W + e % W;
}
// as pairs of 16-bit words; zero past the last column
template <int W>
__device__ __forceinline__ void load_row(const void* row, int first, int cols, uint32_t (&v)[4], Place at = in_block()) {
    const uint16_t* const q = static_cast<const uint16_t*>(row);
    const int col = column_of<W>(first, 0, at);
    if (W == 8 && col + 8 <= cols) {
        const uint4 a = *reinterpret_cast<const uint4*>(q + col);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        return;
    }
    if (W < 8 && column_of<W>(first, 7, at) < cols) {      // one test for all, so that the loads go out together
        uint16_t h[8];
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            if (W == 2) {
                v[e / 2] = *reinterpret_cast<const uint32_t*>(q + column_of<W>(first, e, at));
            } else {
                h[e] = q[column_of<W>(first, e, at)];
                h[e + 1] = q[column_of<W>(first, e + 1, at)];
            }
        }
#pragma unroll
        for (int i = 0; i < 4 && W == 1; ++i) v[i] = h[2 * i] | uint32_t(h[2 * i + 1]) << 16;
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c0 = column_of<W>(first, 2 * i, at), c1 = column_of<W>(first, 2 * i + 1, at);
        if (W == 2 && c1 < cols) v[i] = *reinterpret_cast<const uint32_t*>(q + c0);
        else v[i] = (c0 < cols ? q[c0] : 0) | uint32_t(c1 < cols ? q[c1] : 0) << 16;
    }
}
template <int W>
__device__ __forceinline__ void store_row(void* row, int first, int cols, const uint32_t (&v)[4], Place at = in_block()) {
    uint16_t* const q = static_cast<uint16_t*>(row);
    const int col = column_of<W>(first, 0, at);
    if (W == 8 && col + 8 <= cols) {
        *reinterpret_cast<uint4*>(q + col) = make_uint4(v[0], v[1], v[2], v[3]);
        return;
    }
    if (W < 8 && column_of<W>(first, 7, at) < cols) {
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            if (W == 2) {
                *reinterpret_cast<uint32_t*>(q + column_of<W>(first, e, at)) = v[e / 2];
            } else {
                q[column_of<W>(first, e, at)] = uint16_t(v[e / 2]);
                q[column_of<W>(first, e + 1, at)] = uint16_t(v[e / 2] >> 16);
            }
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c0 = column_of<W>(first, 2 * i, at), c1 = column_of<W>(first, 2 * i + 1, at);
        if (W == 2 && c1 < cols) {
            *reinterpret_cast<uint32_t*>(q + c0) = v[i];
        } else {
            if (c0 < cols) q[c0] = uint16_t(v[i]);
            if (c1 < cols) q[c1] = uint16_t(v[i] >> 16);
        }
    }
}
// offset + weight, the weight in 16 bits or fp32
template <int DT, int W>
__device__ __forceinline__ void load_weights(const void* weight, bool fp32, float offset, int first, int cols, float2 (&v)[4],
                                             Place at = in_block()) {
    if (!fp32) {
        uint32_t h[4];
        load_row<W>(weight, first, cols, h, at);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = unpack2(h[i], DT);
    } else {
        const float* const q = static_cast<const float*>(weight);
        const int col = column_of<W>(first, 0, at);
        if (W == 8 && col + 8 <= cols) {
            const float4 a = reinterpret_cast<const float4*>(q + col)[0], b = reinterpret_cast<const float4*>(q + col)[1];
            v[0] = make_float2(a.x, a.y); v[1] = make_float2(a.z, a.w); v[2] = make_float2(b.x, b.y); v[3] = make_float2(b.z, b.w);
        } else if (W < 8 && column_of<W>(first, 7, at) < cols) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = make_float2(q[column_of<W>(first, 2 * i, at)], q[column_of<W>(first, 2 * i + 1, at)]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int c0 = column_of<W>(first, 2 * i, at), c1 = column_of<W>(first, 2 * i + 1, at);
                v[i] = make_float2(c0 < cols ? q[c0] : 0.0f, c1 < cols ? q[c1] : 0.0f);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = add_pair(v[i], twice(offset));
}

// the sum of the values of a group of warps, whose barrier is `id`, in an order that does not depend on timing; every thread gets
// it.  `shared` is not written again before every thread of the group has passed another barrier.
__device__ __forceinline__ float group_sum(float v, float* shared, Place at, int id) {
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    const int warps = at.threads / 32, lane = at.thread & 31;
    if (warps == 1) return v;
    if (lane == 0) shared[at.thread >> 5] = v;
    asm volatile("barrier.cta.sync.aligned %0, %1;" ::"r"(id), "r"(at.threads) : "memory");
    v = lane < warps ? shared[lane] : 0.0f;
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    return v;
}

// 1 / sqrt(m), in fp64 to about 2^-52: one step of third order from an fp32 start, r (1 + e/2 + 3 e^2/8) with e = 1 - m r^2
// below 2^-21; the general function (twice the time) where fp32 does not reach.
__device__ __forceinline__ double inverse_root(double m) {
    const uint32_t exponent = uint32_t(__double2hiint(m)) >> 20;       // with the sign
    if (exponent - (1023u - 100u) > 200u) return rsqrt(m);
    const double r = double(rsqrtf(float(m))), e = fma(-m * r, r, 1.0);
    return fma(r * e, fma(0.375, e, 0.5), r);
}

// ---------------------------------------------------------------- forward
struct NormArgs {
    const void *x, *residual, *weight;     // residual may be null: the sum is x then, and is not written
    void *sum, *y;
    float* factors;                        // r of each row, for the gradients; may be null
    uint8_t *codes, *scales;               // EIGHT: instead of y
    size_t ldx, ldr, lds, ldy;
    double inverse, eps;                   // 1 / columns
    float offset;
    int rows, cols, fp32;                  // fp32: the weight's type
    int stages;                            // EIGHT: of 128 columns
};

// the codes and scales of eight elements of a row, from column `first` on; scales end at column `end`
template <int W>
__device__ __forceinline__ void store_fp8(const NormArgs& p, size_t row, int first, int end, float2 (&v)[4]) {
    const int stride = (p.cols + 31) & ~31;
    uint8_t* const codes = p.codes + row * uint32_t(stride);
    auto scales = [&] { return p.scales + fp8_scale_offset(row, 0, p.stages); };
    // 0 past the last column, also where r is not finite
    if (column_of<W>(first, 7) >= p.cols) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (column_of<W>(first, 2 * i) >= p.cols) v[i].x = 0.0f;
            if (column_of<W>(first, 2 * i + 1) >= p.cols) v[i].y = 0.0f;
        }
    }
    if constexpr (W == 8) {
        const int col = column_of<W>(first, 0);
        uint32_t m = __float_as_uint(max_abs(max_abs(max_abs(v[0].x, v[0].y, v[1].x), v[1].y, v[2].x),
                                             max_abs(v[2].y, v[3].x, v[3].y), 0.0f)), byte;
        m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
        m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 2));
        float inv;
        fp8_block_scale(m, byte, inv);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = mul_pair(v[i], twice(inv));
        if (col < stride)
            *reinterpret_cast<uint2*>(codes + col) = make_uint2(encode_e4m3(v[0].x, v[0].y) | encode_e4m3(v[1].x, v[1].y) << 16,
                                                                encode_e4m3(v[2].x, v[2].y) | encode_e4m3(v[3].x, v[3].y) << 16);
        const uint32_t word = gather_scales<4>(byte);
        if (threadIdx.x % 16 == 0 && col < end) *reinterpret_cast<uint32_t*>(scales() + (col / 128) * size_t(512)) = word;
    } else {
#pragma unroll
        for (int e = 0; e < 8; e += W) {
            const int col = column_of<W>(first, e);
            const float a = e & 1 ? v[e / 2].y : v[e / 2].x, b = W == 2 ? v[e / 2].y : 0.0f;
            uint32_t m = __float_as_uint(max_abs(a, b, 0.0f)), byte;
            float inv;
#pragma unroll
            for (int d = 16 / W; d; d >>= 1) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
            fp8_block_scale(m, byte, inv);
            const uint32_t code = encode_e4m3(__fmul_rn(a, inv), __fmul_rn(b, inv));
            if (col < stride) {
                if (W == 2) *reinterpret_cast<uint16_t*>(codes + col) = uint16_t(code);
                else codes[col] = uint8_t(code);
            }
            if (col % 32 == 0 && col < end) scales()[(col / 128) * size_t(512) + col / 32 % 4] = uint8_t(byte);
        }
    }
}

// sum = rn16(x + residual), r = 1 / sqrt(mean(sum^2) + eps), v = (sum r) (offset + weight), each step rounded to fp32.  The
// squares are added in fp64: rows of thousands of elements then give an r that does not depend on the order of addition
// (but where it lies within 2^-45 of a border), and with r the 8-bit codes are those of the definition, bit for bit.
//
// One CTA a row, 8 elements a thread, kept in registers between the row's sum and its scaling: each input is read once.
// LONG: rows of more than 8192 elements read their sum again.
//
// Bound by DRAM, 16 bits, and by instruction issue beside it, 8 bits (63 % of the slots).  8192 x 5376: 57.0 us for 352 MB, 6.2 TB/s,
// and 57.5 us for 310 MB, 5.4 TB/s.  Other forms of 8192 x 5376, 16 / 8 bits: 16 elements a thread 62 / 67 us; the row's factor found by
// every warp 59 / 67; CTAs that stay, with the next rows copied ahead, 60 / 77, with 24 elements a thread 67 / 64; a warp a row
// 66 / 74, a warp a row with rows copied ahead 85 / 95.  Rows read by pairs (8191 x 5374) take 71 us, by elements (5375) 144.
template <int DT, int W, bool EIGHT, bool LONG>
__global__ void __launch_bounds__(kRowThreads) norm_kernel(const __grid_constant__ NormArgs p) {
    __shared__ double parts[32];
    __shared__ float root;
    const int span = blockDim.x * 8, warps = blockDim.x / 32, lane = threadIdx.x & 31;
    const size_t row = blockIdx.x;
    const int end = EIGHT ? p.stages * 128 : p.cols;
    const bool add = p.residual != nullptr;
    const uint16_t* const x = static_cast<const uint16_t*>(p.x) + row * p.ldx;
    const uint16_t* const residual = static_cast<const uint16_t*>(p.residual) + row * p.ldr;
    uint16_t* const sum = static_cast<uint16_t*>(p.sum) + row * p.lds;
    grid_launch();
    grid_wait();

    uint32_t h[4];
    float2 w[4];
    double even = 0.0, odd = 0.0;
    for (int first = 0; first < (LONG ? p.cols : 1); first += span) {
        uint32_t b[4];
        load_row<W>(x, first, p.cols, h);
        if (add) load_row<W>(residual, first, p.cols, b);
        if (!LONG) load_weights<DT, W>(p.weight, p.fp32, p.offset, first, p.cols, w);
        if (add) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 f = add_pair(unpack2(h[i], DT), unpack2(b[i], DT));
                h[i] = pack2(f.x, f.y, DT);
            }
            store_row<W>(sum, first, p.cols, h);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = unpack2(h[i], DT);
            even = fma(double(f.x), double(f.x), even);
            odd = fma(double(f.y), double(f.y), odd);
        }
    }
    even += odd;
#pragma unroll
    for (int d = 16; d; d >>= 1) even += __shfl_xor_sync(0xFFFFFFFFu, even, d);
    if (lane == 0) parts[threadIdx.x >> 5] = even;
    __syncthreads();
    if (threadIdx.x < 32) {                                // one warp, so that the others' instructions go to elements
        even = lane < warps ? parts[lane] : 0.0;
#pragma unroll
        for (int d = 16; d; d >>= 1) even += __shfl_xor_sync(0xFFFFFFFFu, even, d);
        if (lane == 0) {
            root = float(inverse_root(fma(even, p.inverse, p.eps)));
            if (!EIGHT && p.factors) p.factors[row] = root;
        }
    }
    __syncthreads();
    const float r = root;

    for (int first = 0; first < (LONG ? end : 1); first += span) {
        if (LONG) {
            load_row<W>(add ? sum : x, first, p.cols, h);
            load_weights<DT, W>(p.weight, p.fp32, p.offset, first, p.cols, w);
        }
        float2 v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = mul_pair(mul_pair(unpack2(h[i], DT), twice(r)), w[i]);
        if constexpr (EIGHT) {
            store_fp8<W>(p, row, first, end, v);
        } else {
            uint32_t out[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) out[i] = pack2(v[i].x, v[i].y, DT);
            store_row<W>(static_cast<uint16_t*>(p.y) + row * p.ldy, first, p.cols, out);
        }
    }
}

// ---------------------------------------------------------------- gradients
struct NormGradArgs {
    const void *dy, *dsum, *sum, *weight;  // dsum may be null
    const float* factors;                  // r of each row
    void* dx;
    float* parts;                          // [count][columns to 8], or null
    void* dw;                              // null: no gradient of the weight
    size_t lddy, ldds, lds, lddx;
    float inverse, offset;
    int rows, cols, fp32, count;           // count: CTAs, and their parts
    int groups;                            // of a CTA's threads, with a row each at a time
    int together;                          // the CTAs are one cluster, which adds their parts up itself
};

__host__ __device__ inline size_t part_stride(size_t cols) { return (cols + 7) & ~size_t(7); }

// n = sum r, g = dy (offset + weight):  dx = dsum + r g - (r mean(g n)) n, dweight = sum over rows of dy n.
// The groups of a CTA's threads take rows in turn, a thread the same G pieces of 8 columns of each, whose weight gradients it adds up in
// registers; at the end the groups' are added in shared memory, so that one part for each SM goes to memory.  W = 8: a row is
// copied to shared memory while the one before it is worked on; a thread copies and reads its own elements, so no barrier is
// needed for them, and reads them twice, so that registers hold weights and sums only.  MOST = 1024: up to 8192 columns with one
// piece each, for CTAs of two rows, whose time is mostly the fetching of instructions.  G = 0: rows that this does not hold; sums
// in the CTA's part in memory.  Few rows: the CTAs are a cluster and add their parts of the weight's gradient up through
// distributed shared memory, which saves a launch.
//
// 8192 x 5376: 59 us for 352 MB, 6.0 TB/s, and 6 us for the sum of 444 parts; bound by DRAM and by the wait for the row's sum.  With
// the whole CTA's barrier for that sum 68 us.  With the sum of parts: without copies ahead, 16 columns a thread, 267 us; with copies and
// 8 columns a thread 93; with 24 columns and 384 threads 92; rows read by pairs (8191 x 5374) 146, by elements (5375) 227: as many
// instructions for two bytes or four as for 16.
template <int DT, int W, int G, int MOST>
__global__ void __launch_bounds__(MOST, MOST == kGradThreads && G <= 3 ? 3 : 1) norm_grad_kernel(const __grid_constant__ NormGradArgs p) {
    constexpr bool STAGED = W == 8 && G > 0, HELD = W < 8 && G == 1;      // HELD: in registers from one use to the next
    constexpr int N = G ? G : 1;
    extern __shared__ __align__(16) uint8_t staged[];
    constexpr bool GROUPS = MOST == kGradGroupThreads;
    __shared__ float shared[GROUPS ? kGradMostGroups : 1][2][32];     // one is written again only after the barrier of the row between
    // (a group is whole warps)
    const int groups = GROUPS ? p.groups : 1, threads = blockDim.x / groups, group = uniform(threadIdx.x / threads);
    const Place at = {int(threadIdx.x) - group * threads, threads};
    const int span = threads * 8;
    const size_t first_row = blockIdx.x * groups + group, step = size_t(gridDim.x) * groups;
    const bool add = p.dsum != nullptr;
    float* const part = p.parts ? p.parts + blockIdx.x * part_stride(p.cols) : nullptr;
    grid_launch();
    grid_wait();
    float2 w[N][4], acc[N][4];
#pragma unroll
    for (int g = 0; g < N; ++g) {
        if (G) load_weights<DT, W>(p.weight, p.fp32, p.offset, g * span, p.cols, w[g], at);
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[g][i] = make_float2(0.0f, 0.0f);
    }
    const int per = threads * 16, per_stage = 3 * N * per;
    const uint32_t mine = smem_addr(staged) + group * kGradStages * per_stage + at.thread * 16;
    auto fetch = [&](size_t row, uint32_t to) {
        if (row < size_t(p.rows)) {
            const uint16_t* const dy = static_cast<const uint16_t*>(p.dy) + row * p.lddy;
            const uint16_t* const h = static_cast<const uint16_t*>(p.sum) + row * p.lds;
            const uint16_t* const ds = static_cast<const uint16_t*>(p.dsum) + row * p.ldds;
#pragma unroll
            for (int g = 0; g < N; ++g) {
                const int col = column_of<8>(g * span, 0, at), bytes = min(16, (p.cols - col) * 2);
                if (bytes <= 0) continue;
                copy_async_16(to + 3 * g * per, dy + col, bytes);
                copy_async_16(to + (3 * g + 1) * per, h + col, bytes);
                if (add) copy_async_16(to + (3 * g + 2) * per, ds + col, bytes);
            }
        }
        copy_async_commit();
    };
    if (STAGED)
        for (int i = 0; i < kGradStages; ++i) fetch(first_row + i * step, mine + i * per_stage);

    int turn = 0, stage = 0;
    float next = first_row < size_t(p.rows) ? p.factors[first_row] : 0.0f;
    for (size_t row = first_row; row < size_t(p.rows); row += step, turn ^= 1) {
        const float r = next;
        if (row + step < size_t(p.rows)) next = p.factors[row + step];
        const uint32_t from = mine + stage * per_stage;
        if (STAGED) copy_async_wait<kGradStages - 1>();
        // eight elements of dy, sum and dsum; past the last column the first two are 0
        auto load = [&](int first, int g, uint32_t (&dy)[4], uint32_t (&h)[4], uint32_t* ds) {
            if constexpr (STAGED) {
                if (column_of<W>(first, 0, at) < p.cols) {
                    ld_shared_v4(from + 3 * g * per, dy);
                    ld_shared_v4(from + (3 * g + 1) * per, h);
                    if (ds && add) ld_shared_v4(from + (3 * g + 2) * per, *reinterpret_cast<uint32_t(*)[4]>(ds));
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) dy[i] = h[i] = 0;
                }
            } else {
                load_row<W>(static_cast<const uint16_t*>(p.dy) + row * p.lddy, first, p.cols, dy, at);
                load_row<W>(static_cast<const uint16_t*>(p.sum) + row * p.lds, first, p.cols, h, at);
                if (ds && add)
                    load_row<W>(static_cast<const uint16_t*>(p.dsum) + row * p.ldds, first, p.cols, *reinterpret_cast<uint32_t(*)[4]>(ds),
                                at);
            }
            if (!G) load_weights<DT, W>(p.weight, p.fp32, p.offset, first, p.cols, w[0], at);
        };
        float2 b = make_float2(0.0f, 0.0f);
        uint32_t held[3][4];
        if (HELD) load(0, 0, held[0], held[1], held[2]);
        auto take = [&](int first, int g) {
            uint32_t dy[4], h[4];
            if (!HELD) load(first, g, dy, h, nullptr);
#pragma unroll
            for (int i = 0; i < 4 && HELD; ++i) {
                dy[i] = held[0][i];
                h[i] = held[1][i];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
                b = fma_pair(mul_pair(unpack2(dy[i], DT), w[g][i]), mul_pair(unpack2(h[i], DT), twice(r)), b);
        };
        if (G) {
#pragma unroll
            for (int g = 0; g < N; ++g) take(g * span, g);
        } else {
            for (int first = 0; first < p.cols; first += span) take(first, 0);
        }
        const float c = group_sum(b.x + b.y, shared[GROUPS ? group : 0][turn], at, 1 + group) * p.inverse * r;
        auto give = [&](int first, int g) {
            uint32_t dy[4], h[4], ds[4], dx[4];
            if (!HELD) load(first, g, dy, h, ds);
#pragma unroll
            for (int i = 0; i < 4 && HELD; ++i) {
                dy[i] = held[0][i];
                h[i] = held[1][i];
                ds[i] = held[2][i];
            }
            float2 dw[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 y = unpack2(dy[i], DT), n = mul_pair(unpack2(h[i], DT), twice(r));
                float2 d = add ? unpack2(ds[i], DT) : make_float2(0.0f, 0.0f);
                d = fma_pair(twice(-c), n, fma_pair(twice(r), mul_pair(y, w[g][i]), d));
                dx[i] = pack2(d.x, d.y, DT);
                if (G) acc[g][i] = fma_pair(y, n, acc[g][i]);
                else dw[i] = mul_pair(y, n);
            }
            store_row<W>(static_cast<uint16_t*>(p.dx) + row * p.lddx, first, p.cols, dx, at);
            if (!G && part) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int col = column_of<W>(first, e, at);
                    const float v = e & 1 ? dw[e / 2].y : dw[e / 2].x;
                    if (col < p.cols) part[col] = row == first_row ? v : part[col] + v;
                }
            }
        };
        if (G) {
#pragma unroll
            for (int g = 0; g < N; ++g) give(g * span, g);
        } else {
            for (int first = 0; first < p.cols; first += span) give(first, 0);
        }
        if (STAGED) {
            fetch(row + kGradStages * step, from);
            stage = stage == kGradStages - 1 ? 0 : stage + 1;
        }
    }
    if (G && p.dw) {
        const size_t stride = part_stride(p.cols);
        float* const sums = reinterpret_cast<float*>(staged);
        float* const to = p.together ? sums : groups > 1 ? sums + group * stride : part;
        __syncthreads();                                   // the rows in shared memory have been read
#pragma unroll
        for (int g = 0; g < N; ++g) {
            if constexpr (W == 8) {
                if (column_of<W>(g * span, 0, at) < p.cols) {
                    float4* const q = reinterpret_cast<float4*>(to + column_of<W>(g * span, 0, at));
                    q[0] = make_float4(acc[g][0].x, acc[g][0].y, acc[g][1].x, acc[g][1].y);
                    q[1] = make_float4(acc[g][2].x, acc[g][2].y, acc[g][3].x, acc[g][3].y);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int col = column_of<W>(g * span, 2 * i, at), after = column_of<W>(g * span, 2 * i + 1, at);
                    if (W == 2 && col < p.cols) *reinterpret_cast<float2*>(to + col) = acc[g][i];
                    if (W == 1 && col < p.cols) to[col] = acc[g][i].x;
                    if (W == 1 && after < p.cols) to[after] = acc[g][i].y;
                }
            }
        }
        if (GROUPS && groups > 1) {
            __syncthreads();
            for (int col = threadIdx.x * 4; col < p.cols; col += blockDim.x * 4) {     // up to the part's end, a multiple of 8
                float4 v = *reinterpret_cast<const float4*>(sums + col);
                for (int g = 1; g < groups; ++g) {
                    const float4 a = *reinterpret_cast<const float4*>(sums + g * stride + col);
                    v.x += a.x; v.y += a.y; v.z += a.z; v.w += a.w;
                }
                *reinterpret_cast<float4*>(part + col) = v;
            }
        }
        if (p.together) {
            cluster_sync();
            for (int col = blockIdx.x * blockDim.x + threadIdx.x; col < p.cols; col += gridDim.x * blockDim.x) {
                float v = 0.0f;
                for (int q = 0; q < p.together; ++q) v += ld_cluster_f32(peer_addr(smem_addr(staged) + col * 4, q));
                store1(p.dw, col, v, p.fp32 ? int(kFp32) : DT);
            }
            __syncwarp();
            cluster_sync();                                // the others' parts have been read
        }
    }
}

// The parts of 32 columns, a lane each, split among the warps and added in a fixed order.  Large CTAs: 256 threads are room enough
// beside the launch before, and what waits there costs the launch after (backward pass of 8192 x 5376, one after the other: 108 us,
// with 1024 threads 75).
constexpr int kPartsThreads = 1024;
template <int DT>
__global__ void __launch_bounds__(kPartsThreads) norm_parts_kernel(const __grid_constant__ NormGradArgs p) {
    constexpr int WARPS = kPartsThreads / 32;
    __shared__ float shared[WARPS][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
    grid_launch();
    grid_wait();
    float v = 0.0f;
    if (col < p.cols) {
        const size_t stride = part_stride(p.cols);
        const float* q = p.parts + warp * stride + col;
#pragma unroll 4
        for (int i = warp; i < p.count; i += WARPS, q += WARPS * stride) v += __ldcg(q);
    }
    shared[warp][lane] = v;
    __syncthreads();
    if (warp || col >= p.cols) return;
#pragma unroll
    for (int i = 1; i < WARPS; ++i) v += shared[i][lane];
    store1(p.dw, col, v, p.fp32 ? int(kFp32) : DT);
}

}  // namespace ff
}  // namespace equarx
