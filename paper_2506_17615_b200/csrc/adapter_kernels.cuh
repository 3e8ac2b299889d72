// Low-rank adapters of many requests beside a shared projection.
//
//   adapter_token_kernel   few tokens: a cluster each, dot products in fp32
//   adapter_down_kernel    many tokens, rows that TMA cannot read: S = x A^T, split into high and low halves of 16 bits
//   adapter_up_kernel      and out = y + S B^T
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
    uint16_t* s;                      // many tokens: [tokens][high, low][ranks]
    float* back;                      // and what a token's S has been divided by
    size_t ldy, ldx, ldo;
    int tokens, k, n, rank, adapters;
    int ctas;                         // of a cluster, which split k (and, for few tokens, n)
    int tiles;                        // many tokens: through TMA
    int copies;                       // and the clusters that a tile of tokens has
    int blocks;                       // of features, that a CTA of the second product takes where TMA does not read rows
};
constexpr int kAdapterWarps = 8, kAdapterThreads = 32 * kAdapterWarps;
// ranks are padded to 16 RT, RT = 1, 2, 4 or 8

// eight neighbouring elements of a row from `col` on, as pairs; zero past `cols`.  VEC: rows start on multiples of 16 bytes and
// have a multiple of 8 elements
template <bool VEC>
__device__ __forceinline__ void load_eight(const uint16_t* row, int col, int cols, uint32_t* v) {
    if (VEC) {
        const uint4 q = col < cols ? *reinterpret_cast<const uint4*>(row + col) : make_uint4(0, 0, 0, 0);
        v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
    } else if (col + 8 <= cols) {                  // one test, so that the loads go out together
        uint16_t h[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) h[i] = row[col + i];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = h[2 * i] | uint32_t(h[2 * i + 1]) << 16;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            v[i] = (col + 2 * i < cols ? row[col + 2 * i] : 0) | uint32_t(col + 2 * i + 1 < cols ? row[col + 2 * i + 1] : 0) << 16;
    }
}
// the adapter of a token, -1: none
__device__ __forceinline__ int adapter_of(const AdapterArgs& p, int token) {
    const int i = p.index[token];
    return i >= 0 && i < p.adapters ? i : -1;
}
template <int DT>
__device__ __forceinline__ float dot_eight(const uint32_t* a, const float2* b, float v) {
    float2 w = make_float2(v, 0.0f);
#pragma unroll
    for (int i = 0; i < 4; ++i) w = fma_pair(unpack2(a[i], DT), b[i], w);
    return w.x + w.y;
}

// ---------------------------------------------------------------- few tokens
// One cluster for a token: its CTAs split k for S, whose parts they exchange through distributed shared memory, and then n.  Every
// CTA has asked for its first rows of B before it waits for S.  A lane takes 8 columns of a row of A at a time, RT lanes share a row
// of B, 16 ranks each: all reads are of neighbouring bytes.  Everything is summed in fp32.  Bound by the chain of start,
// index, loads, exchange and store: 2688 -> 5376, rank 16, 4.3 us for one token, 7.7 for 64 with an adapter each (18 MB, 2.4 TB/s;
// of rank 64 17.6 us, 3.8 TB/s).  Products of tiles of tokens by mma.sync in one launch took 7.4 and 12.9.
template <int DT, int RT, bool VEC>
__global__ void __launch_bounds__(kAdapterThreads, RT < 4 ? 3 : 2) adapter_token_kernel(const __grid_constant__ AdapterArgs p) {
    constexpr int ROWS = 2 * RT;                     // of A, for each warp
    constexpr int AHEAD = 4;                         // parts of B's rows, for each thread
    __shared__ __align__(16) float mine[16 * RT], total[16 * RT];
    const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31, rank = int(cluster_rank());
    const size_t token = blockIdx.x / p.ctas;
    grid_launch();
    grid_wait();
    const int d = adapter_of(p, int(token));
    const uint16_t* const x = static_cast<const uint16_t*>(p.x) + token * p.ldx;
    const uint16_t* const y = static_cast<const uint16_t*>(p.y) + token * p.ldy;
    uint16_t* const out = static_cast<uint16_t*>(p.out) + token * p.ldo;
    const int f0 = int(int64_t(p.n) * rank / p.ctas), f1 = int(int64_t(p.n) * (rank + 1) / p.ctas);
    if (d < 0) {                                     // all CTAs of the cluster alike
        for (int f = f0 + tid; f < f1; f += kAdapterThreads) out[f] = y[f];
        return;
    }
    const uint16_t* const a = static_cast<const uint16_t*>(p.a) + size_t(d) * p.rank * p.k;
    const uint16_t* const b = static_cast<const uint16_t*>(p.b) + size_t(d) * p.n * p.rank;

    // features f0 + tid / RT, and every kAdapterThreads / RT further; ranks 16 (tid % RT) on
    constexpr int STEP = kAdapterThreads / RT;
    const int part = tid % RT * 16, mf = f0 + tid / RT;
    auto load_b = [&](int f, uint32_t (&v)[8]) {
        const bool in = f < f1;
        load_eight<VEC>(b + size_t(f) * p.rank, in ? part : p.rank, p.rank, v);
        load_eight<VEC>(b + size_t(f) * p.rank, in ? part + 8 : p.rank, p.rank, v + 4);
    };
    uint32_t ahead[AHEAD][8];
    uint16_t old[AHEAD];
    auto load_ahead = [&](int f) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            load_b(f + i * STEP, ahead[i]);
            old[i] = f + i * STEP < f1 ? y[f + i * STEP] : uint16_t(0);
        }
    };
    load_ahead(mf);

    const int chunks = (p.k + 7) / 8, c0 = int(int64_t(chunks) * rank / p.ctas), c1 = int(int64_t(chunks) * (rank + 1) / p.ctas);
    float acc[ROWS] = {};
#pragma unroll(RT < 4 ? 2 : 1)
    for (int c = c0 + lane; c < c1; c += 32) {
        uint32_t v[4];
        float2 f[4];
        load_eight<VEC>(x, c * 8, p.k, v);
        uint32_t w[ROWS][4];
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            const int r = warp + i * kAdapterWarps;
            load_eight<VEC>(a + size_t(r) * p.k, r < p.rank ? c * 8 : p.k, p.k, w[i]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = unpack2(v[i], DT);
#pragma unroll
        for (int i = 0; i < ROWS; ++i) acc[i] = dot_eight<DT>(w[i], f, acc[i]);
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
#pragma unroll
        for (int s = 16; s; s >>= 1) acc[i] += __shfl_xor_sync(0xFFFFFFFFu, acc[i], s);
        if (lane == 0) mine[warp + i * kAdapterWarps] = acc[i];
    }
    __syncwarp();
    cluster_sync();
    if (tid < 16 * RT) {
        float v = 0.0f;
        for (int q = 0; q < p.ctas; ++q) v += ld_cluster_f32(peer_addr(smem_addr(mine + tid), q));
        total[tid] = tid < p.rank ? (p.scale ? v * p.scale[d] : v) : 0.0f;
    }
    __syncwarp();
    cluster_arrive();                                // the others' sums have been read
    __syncthreads();
    float2 s[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] = *reinterpret_cast<const float2*>(total + part + 2 * i);
    for (int f = mf; f - tid / RT < f1; f += AHEAD * STEP) {
        if (f != mf) load_ahead(f);
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            float v = dot_eight<DT>(ahead[i], s, 0.0f) + dot_eight<DT>(ahead[i] + 4, s + 4, 0.0f);
#pragma unroll
            for (int q = RT / 2; q; q >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, q);
            if (tid % RT == 0 && f + i * STEP < f1) out[f + i * STEP] = uint16_t(pack2(unpack2(old[i], DT).x + v, 0.0f, DT));
        }
    }
    __syncwarp();
    cluster_wait();
}

// ---------------------------------------------------------------- many tokens
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
// Of up to 32 tokens, one in each lane: bit j is set where token j is the first with its adapter
__device__ __forceinline__ uint32_t first_of_each(int d) {
    const uint32_t alike = __match_any_sync(0xFFFFFFFFu, d);
    return __ballot_sync(0xFFFFFFFFu, d >= 0 && __ffs(alike) == int(threadIdx.x & 31) + 1);
}

// The form for rows that do not start on multiples of 16 bytes, whose elements are read one by one: that bounds it, so it uses
// mma.sync (the reduction axis is permuted alike for both operands, so that a thread's fragments are 16 neighbouring bytes).  4000
// tokens of one request, 1777 -> 3001, rank 64: 101 us, where rows that TMA reads take 18.
//
// A product runs once for each adapter that the tokens of a tile have, and only this adapter's tokens take their rows of its
// result: what is not finite in one request's adapter does not reach another request.
//
// S is rounded as the tensor cores want it, to two numbers of the 16-bit type, high and low, whose sum has 16 bits (bf16) or
// 22: 2^-17 of S.  In fp16 a token's S is scaled by a power of two first, so that its range does not matter.

// fp16: what a token's S is multiplied by, so that its largest finite magnitude goes to [2^14, 2^15), and what by afterwards
__device__ __forceinline__ void range_of(float top, float& times, float& back) {
    const int e = top > 0.0f ? max(int(__float_as_uint(top) >> 23) - 127 - 14, -100) : 0;       // up to 113
    times = __uint_as_float(uint32_t(127 - e) << 23);
    back = __uint_as_float(uint32_t(127 + e) << 23);
}
// Two values as high and low halves; nothing is left of what is not finite.  bf16: fp32 ends a little later, and what would be rounded
// to infinity has the largest finite number as its high half (fp16: 2^15 is inside the range).
template <int DT>
__device__ __forceinline__ void split_pair(float a, float b, uint32_t& high, uint32_t& low) {
    high = pack2(a, b, DT);
    if constexpr (DT == kBf16) {
        if ((high & 0x7FFFu) == 0x7F80u && fabsf(a) < __uint_as_float(kInfBits)) high -= 1;
        if ((high & 0x7FFF0000u) == 0x7F800000u && fabsf(b) < __uint_as_float(kInfBits)) high -= 0x10000u;
    }
    const float2 h = unpack2(high, DT);
    low = pack2(fabsf(a) < __uint_as_float(kInfBits) ? a - h.x : 0.0f, fabsf(b) < __uint_as_float(kInfBits) ? b - h.y : 0.0f, DT);
}
// A token's S, a warp's lanes 32 ranks apart: scaled, split and stored
template <int DT, int R>
__device__ __forceinline__ void store_sums(const AdapterArgs& p, int token, int adapter, float (&v)[(R + 31) / 32]) {
    constexpr int PER = (R + 31) / 32;
    const int lane = threadIdx.x & 31;
    const float c = p.scale ? p.scale[adapter] : 1.0f;
    float top = 0.0f;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        v[j] *= c;
        if (fabsf(v[j]) < __uint_as_float(kInfBits)) top = fmaxf(top, fabsf(v[j]));
    }
    float times = 1.0f;
    if constexpr (DT == kFp16) {
        top = __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(top)));
        float back;
        range_of(top, times, back);
        if (lane == 0) p.back[token] = back;
    }
    uint16_t* const to = p.s + size_t(token) * (2 * R);
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int r = lane + 32 * j;
        if (r >= R) continue;
        uint32_t high, low;
        split_pair<DT>(v[j] * times, 0.0f, high, low);
        to[r] = uint16_t(high);
        to[R + r] = uint16_t(low);
    }
}

// The same into shared memory
__device__ __forceinline__ void stage_eight(uint32_t to, const uint16_t* row, int col, int cols) {
    uint32_t v[4];
    load_eight<false>(row, col, cols, v);
    st_shared_v4(to, v[0], v[1], v[2], v[3]);
}

// S of 32 tokens, transposed: 16 ranks x 8 tokens a product.  Chunks of x and A go through a ring in shared memory.  A warp has 16
// ranks of S, the warps with the same ranks split a chunk, and the CTAs of a cluster split k where there are few tiles.  Rows
// in shared memory are 64 bytes longer than a multiple of 128, so that two rows' 64 bytes meet no bank twice.
constexpr int kDownTokens = 32, kDownStages = 3;
template <int RT> constexpr int kDownChunk = RT == 1 ? 256 : 128;                         // columns
template <int RT> constexpr int kDownRow = kDownChunk<RT> * 2 + 64;                       // bytes
template <int RT> constexpr int kDownSplit = kAdapterWarps / RT;                          // warps with the same ranks
template <int RT> constexpr int kDownStageBytes = (kDownTokens + 16 * RT) * kDownRow<RT>;
template <int RT> constexpr int kDownSmem = kDownStages * kDownStageBytes<RT> + kDownSplit<RT> * kDownTokens * 16 * RT * 4;
template <int DT, int RT>
__global__ void __launch_bounds__(kAdapterThreads, 2) adapter_down_kernel(const __grid_constant__ AdapterArgs p) {
    constexpr int R = 16 * RT, SPLIT = kDownSplit<RT>, NT = kDownTokens / 8, CHUNK = kDownChunk<RT>, ROW = kDownRow<RT>;
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ int own[kDownTokens];
    const uint32_t ring = smem_addr(smem);
    float* const sums = reinterpret_cast<float*>(smem + kDownStages * kDownStageBytes<RT>);      // [SPLIT][tokens][R]
    const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int rank = int(cluster_rank()), first = int(blockIdx.x / p.ctas) * kDownTokens, count = min(kDownTokens, p.tokens - first);
    const uint16_t* const a = static_cast<const uint16_t*>(p.a);
    const uint16_t* const x = static_cast<const uint16_t*>(p.x) + size_t(first) * p.ldx;
    grid_launch();
    grid_wait();
    if (tid < kDownTokens) own[tid] = tid < count ? adapter_of(p, first + tid) : -1;
    __syncthreads();

    const int chunks = (p.k + CHUNK - 1) / CHUNK;
    const int c0 = int(int64_t(chunks) * rank / p.ctas), c1 = int(int64_t(chunks) * (rank + 1) / p.ctas);
    const int part = warp % SPLIT, r0 = warp / SPLIT * 16;
    for (uint32_t left = first_of_each(own[lane]); left; left &= left - 1) {
        const int d = own[__ffs(left) - 1];
        // a thread copies the same piece of every STEP-th row of x and A
        constexpr int PIECES = CHUNK / 8, STEP = kAdapterThreads / PIECES, XS = kDownTokens / STEP, AS = (R + STEP - 1) / STEP;
        const int row0 = tid / PIECES, piece = tid % PIECES;
        const uint16_t* const rows = a + (size_t(d) * p.rank + row0) * p.k;
        const uint16_t* xs[XS];
#pragma unroll
        for (int i = 0; i < XS; ++i) xs[i] = x + size_t(min(row0 + i * STEP, count - 1)) * p.ldx;
        int ahead = 0;
        auto fetch = [&](int c) {
            if (c < c1) {
                const uint32_t to = ring + ahead * kDownStageBytes<RT> + row0 * ROW + piece * 16;
                const int col = c * CHUNK + piece * 8;
#pragma unroll
                for (int i = 0; i < XS; ++i) stage_eight(to + i * STEP * ROW, xs[i], col, p.k);
                const uint16_t* from = rows;
#pragma unroll
                for (int i = 0; i < AS; ++i, from += size_t(STEP) * p.k)
                    if (R % STEP == 0 || row0 + i * STEP < R) {
                        const bool in = row0 + i * STEP < p.rank;
                        stage_eight(to + (kDownTokens + i * STEP) * ROW, in ? from : a, in ? col : p.k, p.k);
                    }
            }
            ahead = ahead == kDownStages - 1 ? 0 : ahead + 1;
        };
        float acc[NT][4] = {};
        for (int i = 0; i < kDownStages - 1; ++i) fetch(c0 + i);
        int stage = 0;
        for (int c = c0; c < c1; ++c) {
            __syncthreads();                               // this chunk is there, the one before it has been used
            fetch(c + kDownStages - 1);
            const uint32_t from = ring + stage * kDownStageBytes<RT>;
            stage = stage == kDownStages - 1 ? 0 : stage + 1;
#pragma unroll
            for (int u = 0; u < CHUNK / 32 / SPLIT; ++u) {
                const uint32_t at = (part + u * SPLIT) * 64 + t * 16;
                uint32_t fx[NT][4], fa[2][4];
#pragma unroll
                for (int j = 0; j < NT; ++j) ld_shared_v4(from + (j * 8 + g) * ROW + at, fx[j]);
#pragma unroll
                for (int half = 0; half < 2; ++half) ld_shared_v4(from + (kDownTokens + r0 + half * 8 + g) * ROW + at, fa[half]);
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const uint32_t f[4] = {fa[0][2 * s], fa[1][2 * s], fa[0][2 * s + 1], fa[1][2 * s + 1]};
#pragma unroll
                    for (int j = 0; j < NT; ++j) mma_16816<DT>(acc[j], f, fx[j][2 * s], fx[j][2 * s + 1]);
                }
            }
        }
        __syncthreads();                                   // the ring is free again
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int token = j * 8 + 2 * t + q;
                if (own[token] != d) continue;
                sums[(part * kDownTokens + token) * R + r0 + g] = acc[j][q];
                sums[(part * kDownTokens + token) * R + r0 + 8 + g] = acc[j][2 + q];
            }
    }
    __syncthreads();
    if (SPLIT > 1)
        for (int e = tid; e < kDownTokens * R; e += kAdapterThreads) {
            if (own[e / R] < 0) continue;
            float v = 0.0f;
#pragma unroll
            for (int i = 0; i < SPLIT; ++i) v += sums[i * kDownTokens * R + e];
            sums[e] = v;
        }
    cluster_sync();
    // the cluster's sums of every ctas-th token, scaled and split
    for (int token = rank + warp * p.ctas; token < count; token += kAdapterWarps * p.ctas) {
        const int i = own[token];
        if (i < 0) continue;
        constexpr int PER = (R + 31) / 32;
        float v[PER];
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int r = lane + 32 * j;
            v[j] = 0.0f;
            if (r >= R) continue;
            const uint32_t from = smem_addr(sums + token * R + r);
            for (int q = 0; q < p.ctas; ++q) v[j] += ld_cluster_f32(peer_addr(from, q));
            if (r >= p.rank) v[j] = 0.0f;            // zeros times x are NaN where x is infinite
        }
        store_sums<DT, R>(p, first + token, i, v);
    }
    __syncwarp();
    cluster_sync();                                  // the others' sums have been read
}

// out = y + S B^T for 64 tokens, 64 features at a time, whose rows of B and y go through rings in shared memory (of y a thread
// writes and reads its own elements).  A warp keeps S of 16 tokens in registers.  Column c of the j-th of four products is
// feature 8 (c / 2) + 2 j + c % 2, so that a thread ends up with 8 neighbours.
constexpr int kUpWarps = 4, kUpTokens = 16 * kUpWarps, kUpFeatures = 64, kUpStages = 3;
constexpr int kUpAtOnce = 4;                     // products whose sums do not wait for one another
template <int RT> constexpr int kUpRow = 32 * RT + (RT >= 4 ? 16 : 0);                   // bytes of a row of B in shared memory
constexpr int kUpY = kUpTokens * kUpFeatures * 2;                                        // bytes of y
template <int RT> constexpr int kUpSmem = kUpStages * (kUpFeatures * kUpRow<RT> + kUpY);
__device__ __forceinline__ void store_eight(uint16_t* row, int col, int cols, const uint32_t (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (col + i < cols) row[col + i] = uint16_t(v[i / 2] >> (i & 1) * 16);
}
template <int DT, int RT>
__global__ void __launch_bounds__(32 * kUpWarps, RT == 8 ? 2 : 4) adapter_up_kernel(const __grid_constant__ AdapterArgs p) {
    constexpr int R = 16 * RT, ROW = kUpRow<RT>;
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ int own[kUpTokens];
    __shared__ uint32_t leaders[2];
    const uint32_t ring = smem_addr(smem);
    const int tid = threadIdx.x, warp = uniform(tid >> 5), lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int first = int(blockIdx.x) * kUpTokens;
    const uint16_t* const b = static_cast<const uint16_t*>(p.b);
    grid_launch();
    grid_wait();
    if (tid < kUpTokens) own[tid] = first + tid < p.tokens ? adapter_of(p, first + tid) : -1;
    __syncthreads();
    if (tid < kUpTokens) {                           // the first token with each adapter
        bool again = own[tid] < 0;
        for (int i = 0; i < kUpTokens; ++i) again |= i < tid && own[i] == own[tid];
        const uint32_t bits = __ballot_sync(0xFFFFFFFFu, !again);
        if (lane == 0) leaders[warp] = bits;
    }
    __syncthreads();
    const uint64_t list = leaders[0] | uint64_t(leaders[1]) << 32;
    const int adapters = __popcll(list);

    const int d0 = own[warp * 16 + g], d1 = own[warp * 16 + g + 8];
    const size_t t0 = first + warp * 16 + g, t1 = t0 + 8;
    const bool in0 = t0 < size_t(p.tokens), in1 = t1 < size_t(p.tokens);
    // a thread's ranks are [4 RT t, 4 RT (t + 1)), four of them in each step of the product
    uint2 high[2][RT], low[2][RT];
    float back[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const bool has = (i ? d1 : d0) >= 0;
        const size_t token = i ? t1 : t0;
        const uint2* const s = reinterpret_cast<const uint2*>(p.s + token * (2 * R)) + t * RT;
#pragma unroll
        for (int j = 0; j < RT; ++j) {
            high[i][j] = has ? __ldcg(s + j) : make_uint2(0, 0);
            low[i][j] = has ? __ldcg(s + R / 4 + j) : make_uint2(0, 0);
        }
        back[i] = DT == kFp16 && has ? __ldcg(p.back + token) : 1.0f;
    }
    const uint16_t* const y0 = static_cast<const uint16_t*>(p.y) + t0 * p.ldy;
    const uint16_t* const y1 = static_cast<const uint16_t*>(p.y) + t1 * p.ldy;
    uint16_t* const o0 = static_cast<uint16_t*>(p.out) + t0 * p.ldo;
    uint16_t* const o1 = static_cast<uint16_t*>(p.out) + t1 * p.ldo;

    // units: blocks of features, and for each the adapters in turn
    const int f0 = int(blockIdx.y) * p.blocks * kUpFeatures, f1 = min(p.n, f0 + p.blocks * kUpFeatures);
    const int per = max(adapters, 1), units = (f1 - f0 + kUpFeatures - 1) / kUpFeatures * per;
    int ahead = 0, ahead_f = f0, slot = 0, used = 0; // the unit that is copied next, its place and that of the one in use
    uint64_t ahead_left = list;
    int y_slot = 0;                                  // of the features that are copied next; one block of them may have many units
    const uint32_t y_ring = ring + kUpStages * kUpFeatures * ROW + tid * 16;
    auto fetch = [&] {
        if (ahead < units && ahead_left == list) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int col = ahead_f + h * 32 + 8 * t;
                stage_eight(y_ring + y_slot * kUpY + h * (kUpY / 2), in0 ? y0 : b, in0 ? col : p.n, p.n);
                stage_eight(y_ring + y_slot * kUpY + h * (kUpY / 2) + kUpY / 4, in1 ? y1 : b, in1 ? col : p.n, p.n);
            }
            y_slot = y_slot == kUpStages - 1 ? 0 : y_slot + 1;
            if (!adapters) ahead_f += kUpFeatures;
        }
        if (ahead < units && adapters) {
            // a thread copies the same piece of every STEP-th row
            constexpr int STEP = 32 * kUpWarps / (R / 8);
            const int f = ahead_f + tid / (R / 8), r = tid % (R / 8) * 8;
            const uint16_t* from = b + (size_t(own[__ffsll(ahead_left) - 1]) * p.n + f) * p.rank;
            const uint32_t to = ring + slot * (kUpFeatures * ROW) + tid / (R / 8) * ROW + r * 2;
#pragma unroll
            for (int i = 0; i < kUpFeatures / STEP; ++i, from += size_t(STEP) * p.rank) {
                const bool in = f + i * STEP < p.n;
                stage_eight(to + i * STEP * ROW, in ? from : b, in ? r : p.rank, p.rank);
            }
            ahead_left &= ahead_left - 1;
            if (!ahead_left) {
                ahead_left = list;
                ahead_f += kUpFeatures;
            }
        }
        ++ahead;
        slot = slot == kUpStages - 1 ? 0 : slot + 1;
    };
    for (int i = 0; i < kUpStages - 1; ++i) fetch();
    uint32_t v[2][2][4];                             // y: two blocks of 32 features, two tokens
    int y_used = 0;
    uint64_t left = 0;
    int f = f0 - kUpFeatures;
    for (int unit = 0; unit < units; ++unit) {
        __syncthreads();
        if (!left) {                                 // the next features
            left = list;
            f += kUpFeatures;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 2; ++i) ld_shared_v4(y_ring + y_used * kUpY + (2 * h + i) * (kUpY / 4), v[h][i]);
            y_used = y_used == kUpStages - 1 ? 0 : y_used + 1;
        }
        fetch();
        used = unit ? (used == kUpStages - 1 ? 0 : used + 1) : 0;
        if (left) {
            const int d = own[__ffsll(left) - 1];
            const uint32_t from = ring + used * (kUpFeatures * ROW) + 8 * RT * t;
            const bool whole = __all_sync(0xFFFFFFFFu, d0 == d && d1 == d);
            if (__any_sync(0xFFFFFFFFu, d0 == d || d1 == d)) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float acc[4][4] = {};
#pragma unroll
                    for (int j = 0; j < 4; j += kUpAtOnce) {
                        uint32_t fb[kUpAtOnce][2 * RT];
#pragma unroll
                        for (int i = 0; i < kUpAtOnce; ++i) {
                            const uint32_t at = from + (h * 32 + 8 * (g >> 1) + 2 * (j + i) + (g & 1)) * ROW;
                            if constexpr (RT == 1) ld_shared_v2(at, fb[i][0], fb[i][1]);
                            else
#pragma unroll
                                for (int q = 0; q < RT / 2; ++q) ld_shared_v4(at + 16 * q, *reinterpret_cast<uint32_t(*)[4]>(fb[i] + 4 * q));
                        }
#pragma unroll
                        for (int s = 0; s < RT; ++s) {
                            const uint32_t fh[4] = {high[0][s].x, high[1][s].x, high[0][s].y, high[1][s].y};
                            const uint32_t fl[4] = {low[0][s].x, low[1][s].x, low[0][s].y, low[1][s].y};
#pragma unroll
                            for (int i = 0; i < kUpAtOnce; ++i) mma_16816<DT>(acc[j + i], fh, fb[i][2 * s], fb[i][2 * s + 1]);
#pragma unroll
                            for (int i = 0; i < kUpAtOnce; ++i) mma_16816<DT>(acc[j + i], fl, fb[i][2 * s], fb[i][2 * s + 1]);
                        }
                    }
                    if (whole) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const float2 w0 = unpack2(v[h][0][j], DT), w1 = unpack2(v[h][1][j], DT);
                            v[h][0][j] = pack2(fmaf(acc[j][0], back[0], w0.x), fmaf(acc[j][1], back[0], w0.y), DT);
                            v[h][1][j] = pack2(fmaf(acc[j][2], back[1], w1.x), fmaf(acc[j][3], back[1], w1.y), DT);
                        }
                        continue;
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float2 w0 = unpack2(v[h][0][j], DT), w1 = unpack2(v[h][1][j], DT);
                        if (d0 == d) v[h][0][j] = pack2(fmaf(acc[j][0], back[0], w0.x), fmaf(acc[j][1], back[0], w0.y), DT);
                        if (d1 == d) v[h][1][j] = pack2(fmaf(acc[j][2], back[1], w1.x), fmaf(acc[j][3], back[1], w1.y), DT);
                    }
                }
            }
            left &= left - 1;
        }
        if (!left) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int col = f + h * 32 + 8 * t;
                if (in0) store_eight(o0, col, p.n, v[h][0]);
                if (in1) store_eight(o1, col, p.n, v[h][1]);
            }
        }
    }
}

}  // namespace ff
}  // namespace equarx
