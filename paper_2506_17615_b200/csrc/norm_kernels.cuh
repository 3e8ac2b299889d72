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

constexpr int kNormThreads = 1024;         // at most; a thread holds 16 elements

// Sixteen elements of a row in a thread's registers.  W = 16: neighbours, for rows that start on multiples of 16 bytes.
// W = 2 or 1: pairs or single elements, the next thread the next ones, for rows that start on multiples of 4 or 2 bytes: a
// warp's accesses are then whole sectors all the same (with 16 neighbours each access would touch 32 sectors).
template <int W>
__device__ __forceinline__ int column_of(int first, int e) {
    if (W == 16) return first + int(threadIdx.x) * 16 + e;
    return first + (e / W * int(blockDim.x) + int(threadIdx.x)) * W + e % W;
}
// as pairs of 16-bit words; zero past the last column.  `wide`: rows start on multiples of 32 bytes
template <int W>
__device__ __forceinline__ void load_row(const void* row, int first, int cols, bool wide, uint32_t (&v)[8]) {
    const uint16_t* const q = static_cast<const uint16_t*>(row);
    const int col = column_of<W>(first, 0);
    if (W == 16 && col + 16 <= cols) {
        if (wide) {
            load_256(q + col, v);
        } else {
            const uint4 a = reinterpret_cast<const uint4*>(q + col)[0], b = reinterpret_cast<const uint4*>(q + col)[1];
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int c0 = column_of<W>(first, 2 * i), c1 = column_of<W>(first, 2 * i + 1);
        if (W == 2 && c1 < cols) v[i] = *reinterpret_cast<const uint32_t*>(q + c0);
        else v[i] = (c0 < cols ? q[c0] : 0) | uint32_t(c1 < cols ? q[c1] : 0) << 16;
    }
}
template <int W>
__device__ __forceinline__ void store_row(void* row, int first, int cols, bool wide, const uint32_t (&v)[8]) {
    uint16_t* const q = static_cast<uint16_t*>(row);
    const int col = column_of<W>(first, 0);
    if (W == 16 && col + 16 <= cols) {
        if (wide) {
            store_256(q + col, v);
        } else {
            reinterpret_cast<uint4*>(q + col)[0] = make_uint4(v[0], v[1], v[2], v[3]);
            reinterpret_cast<uint4*>(q + col)[1] = make_uint4(v[4], v[5], v[6], v[7]);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int c0 = column_of<W>(first, 2 * i), c1 = column_of<W>(first, 2 * i + 1);
        if (W == 2 && c1 < cols) {
            *reinterpret_cast<uint32_t*>(q + c0) = v[i];
        } else {
            if (c0 < cols) q[c0] = uint16_t(v[i]);
            if (c1 < cols) q[c1] = uint16_t(v[i] >> 16);
        }
    }
}
// the weight, 16 bits or fp32, as it is stored
struct Weights {
    uint32_t w[16];
};
template <int W>
__device__ __forceinline__ void load_weights(const void* weight, bool fp32, int first, int cols, bool wide, Weights& v) {
    if (!fp32) {
        uint32_t h[8];
        load_row<W>(weight, first, cols, wide, h);
#pragma unroll
        for (int i = 0; i < 8; ++i) v.w[i] = h[i];
        return;
    }
    const uint32_t* const q = static_cast<const uint32_t*>(weight);
    const int col = column_of<W>(first, 0);
    if (W == 16 && col + 16 <= cols) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint4 a = reinterpret_cast<const uint4*>(q + col)[i];
            v.w[4 * i] = a.x; v.w[4 * i + 1] = a.y; v.w[4 * i + 2] = a.z; v.w[4 * i + 3] = a.w;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) v.w[i] = column_of<W>(first, i) < cols ? q[column_of<W>(first, i)] : 0;
}
template <int DT>
__device__ __forceinline__ float2 weight_pair(const Weights& v, bool fp32, int i, float offset) {
    float2 f;
    if (fp32) f = make_float2(__uint_as_float(v.w[2 * i]), __uint_as_float(v.w[2 * i + 1]));
    else f = unpack2(v.w[i], DT);
    return make_float2(__fadd_rn(offset, f.x), __fadd_rn(offset, f.y));
}

// the sum of all threads' values in an order that does not depend on timing; every thread gets it.  `shared` is not
// written again before every thread has passed another barrier.
template <typename T>
__device__ __forceinline__ T block_sum(T v, T* shared) {
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    const int warps = blockDim.x / 32, lane = threadIdx.x & 31;
    if (warps == 1) return v;
    if (lane == 0) shared[threadIdx.x >> 5] = v;
    __syncthreads();
    v = lane < warps ? shared[lane] : T(0);
#pragma unroll
    for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    return v;
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
    int cols, wide, fp32;                  // wide: all rows start on multiples of 32 bytes; fp32: the weight's type
};

// sum = rn16(x + residual), r = 1 / sqrt(mean(sum^2) + eps), v = (sum r) (offset + weight), each step rounded to fp32.  The
// squares are added in fp64: rows of thousands of elements then give an r that does not depend on the order of addition
// (but where it lies within 2^-45 of a border), and with r the 8-bit codes are those of the definition, bit for bit.
//
// One CTA a row, 16 elements a thread, kept in registers between the row's sum and its scaling: each input is read once. Rows
// of more than 16384 elements read their sum again.
template <int DT, int W, bool EIGHT>
__global__ void __launch_bounds__(kNormThreads) norm_kernel(const __grid_constant__ NormArgs p) {
    __shared__ double shared[32];
    const int threads = blockDim.x, span = threads * 16;
    const size_t row = blockIdx.x, stages = fp8_stages(p.cols), stride = fp8_stride(p.cols);
    const int end = EIGHT ? int(stages * 128) : p.cols;
    const uint16_t* const x = static_cast<const uint16_t*>(p.x) + row * p.ldx;
    const uint16_t* const residual = static_cast<const uint16_t*>(p.residual) + (p.residual ? row * p.ldr : 0);
    uint16_t* const sum = static_cast<uint16_t*>(p.sum) + (p.residual ? row * p.lds : 0);
    const bool once = span >= end;
    grid_launch();
    grid_wait();

    uint32_t h[8];
    Weights w;
    double squares = 0.0;
    for (int first = 0; first < p.cols; first += span) {
        load_row<W>(x, first, p.cols, p.wide, h);
        if (p.residual) {
            uint32_t b[8];
            load_row<W>(residual, first, p.cols, p.wide, b);
            if (once) load_weights<W>(p.weight, p.fp32, first, p.cols, p.wide, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float2 f = unpack2(h[i], DT), g = unpack2(b[i], DT);
                h[i] = pack2(__fadd_rn(f.x, g.x), __fadd_rn(f.y, g.y), DT);
            }
            store_row<W>(sum, first, p.cols, p.wide, h);
        } else if (once) {
            load_weights<W>(p.weight, p.fp32, first, p.cols, p.wide, w);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float2 f = unpack2(h[i], DT);
            squares = fma(double(f.x), double(f.x), squares);
            squares = fma(double(f.y), double(f.y), squares);
        }
    }
    squares = block_sum(squares, shared);
    const float r = float(rsqrt(fma(squares, p.inverse, p.eps)));
    if (!EIGHT && p.factors && threadIdx.x == 0) p.factors[row] = r;

    for (int first = 0; first < end; first += span) {
        if (!once) {
            load_row<W>(p.residual ? sum : x, first, p.cols, p.wide, h);
            load_weights<W>(p.weight, p.fp32, first, p.cols, p.wide, w);
        }
        float v[16];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float2 f = unpack2(h[i], DT), s = weight_pair<DT>(w, p.fp32, i, p.offset);
            v[2 * i] = __fmul_rn(__fmul_rn(f.x, r), s.x);
            v[2 * i + 1] = __fmul_rn(__fmul_rn(f.y, r), s.y);
        }
        if constexpr (!EIGHT) {
            uint32_t out[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) out[i] = pack2(v[2 * i], v[2 * i + 1], DT);
            store_row<W>(static_cast<uint16_t*>(p.y) + row * p.ldy, first, p.cols, p.wide, out);
        } else {
            // 0 past the last column, also where r is not finite
#pragma unroll
            for (int e = 0; e < 16; ++e)
                if (column_of<W>(first, e) >= p.cols) v[e] = 0.0f;
            uint8_t* const codes = p.codes + row * stride;
            uint8_t* const scales = p.scales + fp8_scale_offset(row, 0, stages);
            if constexpr (W == 16) {
                uint32_t m = 0, byte;
                float inv;
#pragma unroll
                for (int e = 0; e < 16; ++e) m = max(m, __float_as_uint(v[e]) & 0x7FFFFFFFu);
                m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
                fp8_block_scale(m, byte, inv);
                const uint4 code = encode_e4m3(v, inv);
                const int col = column_of<W>(first, 0);
                if (col < int(stride)) *reinterpret_cast<uint4*>(codes + col) = code;
                const uint32_t word = gather_scales<2>(byte);
                if (threadIdx.x % 8 == 0 && col < end) *reinterpret_cast<uint32_t*>(scales + size_t(col / 128) * 512) = word;
            } else {
#pragma unroll
                for (int e = 0; e < 16; e += W) {
                    uint32_t m = __float_as_uint(v[e]) & 0x7FFFFFFFu, byte;
                    if (W == 2) m = max(m, __float_as_uint(v[e + 1]) & 0x7FFFFFFFu);
#pragma unroll
                    for (int d = 16 / W; d; d >>= 1) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
                    float inv;
                    fp8_block_scale(m, byte, inv);
                    const int col = column_of<W>(first, e);
                    const uint32_t code = encode_e4m3(__fmul_rn(v[e], inv), W == 2 ? __fmul_rn(v[e + 1], inv) : 0.0f);
                    if (col < int(stride)) {
                        if (W == 2) *reinterpret_cast<uint16_t*>(codes + col) = uint16_t(code);
                        else codes[col] = uint8_t(code);
                    }
                    if (col % 32 == 0 && col < end) scales[size_t(col / 128) * 512 + col / 32 % 4] = uint8_t(byte);
                }
            }
        }
    }
}

// ---------------------------------------------------------------- gradients
struct NormGradArgs {
    const void *dy, *dsum, *sum, *weight;  // dsum may be null
    const float* factors;                  // r of each row
    void* dx;
    float* parts;                          // [CTAs][columns], null: no gradient of the weight
    void* dw;
    size_t lddy, ldds, lds, lddx;
    float inverse, offset;
    int rows, cols, wide, fp32, count;     // count: parts
};

// n = sum r, g = dy (offset + weight):  dx = dsum + r (g - n mean(g n)), dweight = sum over rows of dy n.
// A CTA takes every gridDim-th row, a thread the same 16 columns of each, whose weight gradients it adds up in registers
// (rows of more than 16384 elements: in its part in memory).
template <int DT, int W>
__global__ void __launch_bounds__(kNormThreads) norm_grad_kernel(const __grid_constant__ NormGradArgs p) {
    __shared__ float shared[2][32];
    const int span = blockDim.x * 16;
    const bool once = span >= p.cols;
    float* const part = p.parts ? p.parts + size_t(blockIdx.x) * p.cols : nullptr;
    grid_launch();
    grid_wait();
    uint32_t dy[8], ds[8], h[8];
    Weights w;
    float acc[16] = {};
    if (once) load_weights<W>(p.weight, p.fp32, 0, p.cols, p.wide, w);
    int turn = 0;
    for (size_t row = blockIdx.x; row < size_t(p.rows); row += gridDim.x, turn ^= 1) {
        const uint16_t* const qy = static_cast<const uint16_t*>(p.dy) + row * p.lddy;
        const uint16_t* const qs = static_cast<const uint16_t*>(p.dsum) + (p.dsum ? row * p.ldds : 0);
        const uint16_t* const qh = static_cast<const uint16_t*>(p.sum) + row * p.lds;
        const float r = p.factors[row];
        float b = 0.0f;
        for (int first = 0; first < p.cols; first += span) {
            load_row<W>(qy, first, p.cols, p.wide, dy);
            load_row<W>(qh, first, p.cols, p.wide, h);
            if (once) {
                if (p.dsum) load_row<W>(qs, first, p.cols, p.wide, ds);
            } else {
                load_weights<W>(p.weight, p.fp32, first, p.cols, p.wide, w);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                // past the last column dy and h are 0
                const float2 fh = unpack2(h[i], DT), fy = unpack2(dy[i], DT), s = weight_pair<DT>(w, p.fp32, i, p.offset);
                b = fmaf(fy.x * s.x, fh.x * r, b);
                b = fmaf(fy.y * s.y, fh.y * r, b);
            }
        }
        // two buffers: a thread writes one again only after the barrier of the row between
        const float c = block_sum(b, shared[turn]) * p.inverse;
        for (int first = 0; first < p.cols; first += span) {
            if (!once) {
                load_row<W>(qy, first, p.cols, p.wide, dy);
                load_row<W>(qh, first, p.cols, p.wide, h);
                if (p.dsum) load_row<W>(qs, first, p.cols, p.wide, ds);
                load_weights<W>(p.weight, p.fp32, first, p.cols, p.wide, w);
            }
            uint32_t out[8];
            float v[16];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float2 fh = unpack2(h[i], DT), fy = unpack2(dy[i], DT), s = weight_pair<DT>(w, p.fp32, i, p.offset);
                const float2 fs = p.dsum ? unpack2(ds[i], DT) : make_float2(0.0f, 0.0f);
                const float nx = fh.x * r, ny = fh.y * r;
                out[i] = pack2(fmaf(r, fmaf(-c, nx, fy.x * s.x), fs.x), fmaf(r, fmaf(-c, ny, fy.y * s.y), fs.y), DT);
                v[2 * i] = fy.x * nx;
                v[2 * i + 1] = fy.y * ny;
            }
            store_row<W>(static_cast<uint16_t*>(p.dx) + row * p.lddx, first, p.cols, p.wide, out);
            if (once) {
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[e] += v[e];
            } else if (part) {
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int col = column_of<W>(first, e);
                    if (col < p.cols) part[col] = row == blockIdx.x ? v[e] : part[col] + v[e];
                }
            }
        }
    }
    if (once && part) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int col = column_of<W>(0, e);
            if (col < p.cols) part[col] = acc[e];
        }
    }
}

// the parts of 32 columns, 8 threads a column, in a fixed order
template <int DT>
__global__ void __launch_bounds__(256) norm_parts_kernel(const __grid_constant__ NormGradArgs p) {
    __shared__ float shared[8][32];
    const int lane = threadIdx.x & 31, which = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
    grid_launch();
    grid_wait();
    float v = 0.0f;
    if (col < p.cols) {
#pragma unroll 8
        for (int i = which; i < p.count; i += 8) v += __ldcg(p.parts + size_t(i) * p.cols + col);
    }
    shared[which][lane] = v;
    __syncthreads();
    if (which || col >= p.cols) return;
#pragma unroll
    for (int i = 1; i < 8; ++i) v += shared[i][lane];
    store1(p.dw, col, v, p.fp32 ? int(kFp32) : DT);
}

}  // namespace ff
}  // namespace equarx
