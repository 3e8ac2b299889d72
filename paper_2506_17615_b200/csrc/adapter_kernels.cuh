// Low-rank adapters of many requests beside a shared projection.
#pragma once
#include "elements.cuh"
#include "tensor_ops.cuh"

namespace equarx {
namespace ff {

using namespace tc;

// out_t = y_t + c_i (x_t A_i^T) B_i^T with i = index[t]; out_t = y_t where there is no such adapter
struct AdapterArgs {
    const void *y, *x, *a, *b;        // a [adapters][rank][k], b [adapters][n][rank]
    const int* index;
    const float* scale;               // c, or null: 1
    void* out;
    size_t ldy, ldx, ldo;
    int tokens, k, n, rank, adapters;
    int tile;                         // tokens of a cluster, at most 64
    int split;                        // ways in which the warps of a CTA split its part of k; they split the tokens 8 / split ways
    int ctas;                         // of a cluster
};
constexpr int kAdapterWarps = 8, kAdapterThreads = 32 * kAdapterWarps, kAdapterTokens = 64;

// ranks are padded to 16 RT
template <int RT> constexpr int kAdapterGroups = RT <= 2 ? 8 : RT == 4 ? 4 : 2;      // groups of 8 tokens that a warp holds sums of
template <int RT> constexpr int kPackedStride = 16 * RT + 4;                          // of a token, in 16-bit elements
// shared memory: the warps' sums (later the packed ones, high and low halves), the CTA's sums
template <int RT>
__host__ __device__ constexpr int adapter_sums(int tile) { return tile * 16 * RT * 4; }
template <int RT>
__host__ __device__ constexpr int adapter_smem(int tile, int split) {
    const int warps = split * adapter_sums<RT>(tile), packed = 2 * ((tile + 15) / 16 * 16) * kPackedStride<RT> * 2;
    return (warps > packed ? warps : packed) + adapter_sums<RT>(tile);
}

template <int DT>
__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (DT == kBf16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// N (4 or 8) neighbouring elements of a row from `col` on, as pairs; zero past `cols`.  VEC: rows start on multiples of 16
// bytes and have a multiple of 8 elements
template <int N, bool VEC>
__device__ __forceinline__ void load_few(const uint16_t* row, int col, int cols, uint32_t* v) {
    if (VEC) {
        if constexpr (N == 8) {
            const uint4 q = col < cols ? __ldg(reinterpret_cast<const uint4*>(row + col)) : make_uint4(0, 0, 0, 0);
            v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
        } else {
            const uint2 q = col < cols ? __ldg(reinterpret_cast<const uint2*>(row + col)) : make_uint2(0, 0);
            v[0] = q.x; v[1] = q.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N / 2; ++i)
            v[i] = (col + 2 * i < cols ? row[col + 2 * i] : 0) | uint32_t(col + 2 * i + 1 < cols ? row[col + 2 * i + 1] : 0) << 16;
    }
}

// the same 8 from a row that this kernel may also write
template <bool VEC>
__device__ __forceinline__ void load_eight(const uint16_t* row, int col, int cols, uint32_t (&v)[4]) {
    if (VEC) {
        if (col >= cols) return;
        const uint4 q = *reinterpret_cast<const uint4*>(row + col);
        v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            v[i] = (col + 2 * i < cols ? row[col + 2 * i] : 0) | uint32_t(col + 2 * i + 1 < cols ? row[col + 2 * i + 1] : 0) << 16;
    }
}
template <bool VEC>
__device__ __forceinline__ void store_eight(uint16_t* row, int col, int cols, const uint32_t (&v)[4]) {
    if (VEC) {
        if (col < cols) *reinterpret_cast<uint4*>(row + col) = make_uint4(v[0], v[1], v[2], v[3]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (col + i < cols) row[col + i] = uint16_t(v[i / 2] >> (i & 1) * 16);
    }
}

// One cluster for `tile` tokens, in two steps: S = x A^T with k split over its CTAs and their warps, then y + S B^T with the
// output's features split over them.  So x, y and out pass once, a token's adapter is read by one cluster, and there is one
// launch.  The reading bounds it: the tensor cores are used by mma.sync on fragments that come straight from memory (the
// reduction axis is permuted alike for both operands, so that a thread's fragments are 16 neighbouring bytes), since a tile
// of 16 to 64 output columns would not feed tcgen05 anyway.
//
// A product runs once for each adapter that the tokens of a group have, with nothing in the other tokens' places, and only
// this adapter's tokens take its result: what is not finite in one request's adapter does not reach another request.
//
// S is rounded as the tensor cores want it, to two numbers of the 16-bit type, high and low, whose sum has 16 bits (bf16) or
// 22: 2^-17 of S.  In fp16 a token's S is scaled by a power of two first, so that its range does not matter.
template <int DT, int RT, bool VEC>
__global__ void __launch_bounds__(kAdapterThreads) adapters_kernel(const __grid_constant__ AdapterArgs p) {
    constexpr int R = 16 * RT, NT = kAdapterGroups<RT>, PS = kPackedStride<RT>;
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ int own[kAdapterTokens];              // each token's adapter, -1: none
    __shared__ float back[kAdapterTokens];           // what a token's S has been divided by
    const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int rank = int(cluster_rank()), T = p.tile;
    const int first = int(blockIdx.x / p.ctas) * T, count = min(T, p.tokens - first);
    const int warps_bytes = adapter_smem<RT>(T, p.split) - adapter_sums<RT>(T);
    float* const sums = reinterpret_cast<float*>(smem);                      // [split][T][R]
    float* const mine = reinterpret_cast<float*>(smem + warps_bytes);        // [T][R]
    uint16_t* const high = reinterpret_cast<uint16_t*>(smem);                // [T to 16][PS]
    uint16_t* const low = high + (T + 15) / 16 * 16 * PS;
    const uint16_t* const a = static_cast<const uint16_t*>(p.a);
    const uint16_t* const b = static_cast<const uint16_t*>(p.b);

    grid_launch();
    grid_wait();
    if (tid < kAdapterTokens) {
        const int i = tid < count ? p.index[first + tid] : -1;
        own[tid] = i >= 0 && i < p.adapters ? i : -1;
    }
    __syncthreads();
    // Of `width` tokens from `at` on: bit j is set where token j is the first of its 32 with its adapter
    auto leaders = [&](int at, int width) {
        uint64_t bits = 0;
        for (int base = 0; base < width; base += 32) {
            const int d = base + lane < width ? own[at + base + lane] : -1;
            const uint32_t alike = __match_any_sync(0xFFFFFFFFu, d);
            bits |= uint64_t(__ballot_sync(0xFFFFFFFFu, d >= 0 && __ffs(alike) == lane + 1)) << base;
        }
        return bits;
    };

    // ---------------------------------------------------- S = x A^T, transposed: 16 ranks x 8 tokens a product
    const int chunks = (p.k + 31) / 32, c0 = int(int64_t(chunks) * rank / p.ctas), c1 = int(int64_t(chunks) * (rank + 1) / p.ctas);
    {
        const int part = warp % p.split, at = warp / p.split * (NT * 8), width = min(NT * 8, kAdapterTokens - at);
        if (at < count) {
            const uint16_t* xrow[NT];
            int adapter[NT];
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                const int token = at + i * 8 + g;
                adapter[i] = own[token];
                xrow[i] = static_cast<const uint16_t*>(p.x) + size_t(first + min(token, count - 1)) * p.ldx;
            }
            for (uint64_t left = leaders(at, width); left; left &= left - 1) {
                const int d = own[at + __ffsll(left) - 1];
                const uint16_t* const arow = a + size_t(d) * p.rank * p.k;
                float acc[RT][NT][4] = {};
                bool any[NT];
#pragma unroll
                for (int i = 0; i < NT; ++i) any[i] = __any_sync(0xFFFFFFFFu, adapter[i] == d);
#pragma unroll 2
                for (int c = c0 + part; c < c1; c += p.split) {
                    const int col = c * 32 + 8 * t;
                    uint32_t fx[NT][4], fa[RT][2][4];
#pragma unroll
                    for (int i = 0; i < NT; ++i) {
                        fx[i][0] = fx[i][1] = fx[i][2] = fx[i][3] = 0;
                        if (adapter[i] == d) load_few<8, VEC>(xrow[i], col, p.k, fx[i]);
                    }
#pragma unroll
                    for (int i = 0; i < RT; ++i)
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            const int r = i * 16 + half * 8 + g;
                            fa[i][half][0] = fa[i][half][1] = fa[i][half][2] = fa[i][half][3] = 0;
                            if (r < p.rank) load_few<8, VEC>(arow + size_t(r) * p.k, col, p.k, fa[i][half]);
                        }
#pragma unroll
                    for (int i = 0; i < RT; ++i)
#pragma unroll
                        for (int s = 0; s < 2; ++s) {
                            const uint32_t f[4] = {fa[i][0][2 * s], fa[i][1][2 * s], fa[i][0][2 * s + 1], fa[i][1][2 * s + 1]};
#pragma unroll
                            for (int j = 0; j < NT; ++j)
                                if (any[j]) mma_16816<DT>(acc[i][j], f, fx[j][2 * s], fx[j][2 * s + 1]);
                        }
                }
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        const int token = at + j * 8 + 2 * t + q;
                        if (token >= count || own[token] != d) continue;
                        float* const to = sums + (size_t(part) * T + token) * R;
#pragma unroll
                        for (int i = 0; i < RT; ++i) {
                            to[i * 16 + g] = acc[i][j][q];
                            to[i * 16 + 8 + g] = acc[i][j][2 + q];
                        }
                    }
            }
        }
    }
    __syncthreads();
    for (int e = tid; e < count * R; e += kAdapterThreads) {
        float v = 0.0f;
        if (own[e / R] >= 0)
            for (int i = 0; i < p.split; ++i) v += sums[i * T * R + e];
        mine[e] = v;
    }
    cluster_sync();
    // ---------------------------------------------------- the cluster's sums, scaled and packed
    for (int token = warp; token < (T + 15) / 16 * 16; token += kAdapterWarps) {
        const int i = token < count ? own[token] : -1;
        constexpr int PER = (R + 31) / 32;
        float v[PER], top = 0.0f;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int r = lane + 32 * j;
            v[j] = 0.0f;
            if (i >= 0 && r < R) {
                const uint32_t from = smem_addr(mine + token * R + r);
                for (int q = 0; q < p.ctas; ++q) v[j] += ld_cluster_f32(peer_addr(from, q));
                if (p.scale) v[j] *= p.scale[i];
            }
            if (fabsf(v[j]) < __uint_as_float(kInfBits)) top = fmaxf(top, fabsf(v[j]));
        }
        float times = 1.0f;
        if constexpr (DT == kFp16) {
            // the largest finite one goes to [2^14, 2^15)
            top = __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(top)));
            const int e = top > 0.0f ? min(max(int(__float_as_uint(top) >> 23) - 127 - 14, -100), 100) : 0;
            times = __uint_as_float(uint32_t(127 - e) << 23);
            if (lane == 0 && token < kAdapterTokens) back[token] = __uint_as_float(uint32_t(127 + e) << 23);
        }
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int r = lane + 32 * j;
            if (r >= R) continue;
            const float s = v[j] * times;
            const uint32_t h = pack2(s, 0.0f, DT);
            const float rest = s - unpack2(h, DT).x;
            high[token * PS + r] = uint16_t(h);
            // nothing is left of what is not finite
            low[token * PS + r] = fabsf(s) < __uint_as_float(kInfBits) ? uint16_t(pack2(rest, 0.0f, DT)) : uint16_t(0);
        }
    }
    __syncwarp();
    cluster_arrive();                       // the others' sums have been read
    __syncthreads();

    // ---------------------------------------------------- y + S B^T, 16 tokens x 32 features at a time
    // Column c of the j-th of four products is feature 8 (c / 2) + 2 j + c % 2, so that a thread ends up with 8 neighbours.
    const int blocks = (p.n + 31) / 32, b0 = int(int64_t(blocks) * rank / p.ctas), b1 = int(int64_t(blocks) * (rank + 1) / p.ctas);
    for (int m0 = 0; m0 < count; m0 += 16) {
        const uint64_t all = leaders(m0, 16);
        const int d0 = own[m0 + g], d1 = own[m0 + g + 8];
        const size_t r0 = size_t(first + m0 + g), r1 = r0 + 8;
        const bool in0 = m0 + g < count, in1 = m0 + g + 8 < count;
        const float back0 = DT == kFp16 ? back[m0 + g] : 1.0f, back1 = DT == kFp16 ? back[m0 + g + 8] : 1.0f;
        for (int block = b0 + warp; block < b1; block += kAdapterWarps) {
            const int f0 = block * 32 + 8 * t;
            uint32_t y0[4] = {}, y1[4] = {};
            if (in0) load_eight<VEC>(static_cast<const uint16_t*>(p.y) + r0 * p.ldy, f0, p.n, y0);
            if (in1) load_eight<VEC>(static_cast<const uint16_t*>(p.y) + r1 * p.ldy, f0, p.n, y1);
            for (uint64_t left = all; left; left &= left - 1) {
                const int d = own[m0 + __ffsll(left) - 1];
                const uint16_t* const brow = b + (size_t(d) * p.n + block * 32) * p.rank;
                float acc[4][4] = {};
                uint32_t fb[4][2 * RT];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int f = 8 * (g >> 1) + 2 * j + (g & 1);
#pragma unroll
                    for (int i = 0; i < 2 * RT; ++i) fb[j][i] = 0;
                    if (block * 32 + f >= p.n) continue;
                    if constexpr (RT == 1) {
                        load_few<4, VEC>(brow + size_t(f) * p.rank, 4 * t, p.rank, fb[j]);
                    } else {
#pragma unroll
                        for (int i = 0; i < RT / 2; ++i)
                            load_few<8, VEC>(brow + size_t(f) * p.rank, 4 * RT * t + 8 * i, p.rank, fb[j] + 4 * i);
                    }
                }
#pragma unroll
                for (int s = 0; s < RT; ++s) {
                    const int at = (m0 + g) * PS + 4 * RT * t + 4 * s;
                    const uint2 h0 = *reinterpret_cast<const uint2*>(high + at), h1 = *reinterpret_cast<const uint2*>(high + at + 8 * PS);
                    const uint2 l0 = *reinterpret_cast<const uint2*>(low + at), l1 = *reinterpret_cast<const uint2*>(low + at + 8 * PS);
                    const uint32_t fh[4] = {h0.x, h1.x, h0.y, h1.y}, fl[4] = {l0.x, l1.x, l0.y, l1.y};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        mma_16816<DT>(acc[j], fh, fb[j][2 * s], fb[j][2 * s + 1]);
                        mma_16816<DT>(acc[j], fl, fb[j][2 * s], fb[j][2 * s + 1]);
                    }
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 v0 = unpack2(y0[j], DT), v1 = unpack2(y1[j], DT);
                    if (d0 == d) y0[j] = pack2(fmaf(acc[j][0], back0, v0.x), fmaf(acc[j][1], back0, v0.y), DT);
                    if (d1 == d) y1[j] = pack2(fmaf(acc[j][2], back1, v1.x), fmaf(acc[j][3], back1, v1.y), DT);
                }
            }
            if (in0) store_eight<VEC>(static_cast<uint16_t*>(p.out) + r0 * p.ldo, f0, p.n, y0);
            if (in1) store_eight<VEC>(static_cast<uint16_t*>(p.out) + r1 * p.ldo, f0, p.n, y1);
        }
    }
    __syncwarp();
    cluster_wait();
}

}  // namespace ff
}  // namespace equarx
