// Low-rank adapters of many tokens on the fifth-generation tensor cores, for rows that TMA can read and write.
//
//   adapter_down_tiles   S = x A^T, split into high and low halves of 16 bits
//   adapter_up_tiles     out = y + S B^T
//
// Both take tiles of 128 tokens; reading and writing bounds them, and everything comes and goes by TMA, so that few instructions
// are left (mma.sync on fragments from memory took 154 us for 8192 tokens, 2688 -> 5376 of rank 64, from rings filled by
// asynchronous copies 86, this 57).  A product runs once for each adapter that the tile's tokens have, and only this adapter's tokens
// take their rows of its result: what is not finite in one request's adapter does not reach another request.
#pragma once
#include "adapter_kernels.cuh"

namespace equarx {
namespace ff {

struct AdapterMaps {
    CUtensorMap x, a, high, low, b, y, out;     // boxes of 64 columns; of 128 rows, a: of 16 RT, out: of 32
    AdapterArgs p;
};
constexpr int kTileTokens = 128, kDownWarps = 4, kDownThreads = 32 * (kDownWarps + 2);
constexpr int kBoxBytes = kTileTokens * 128;    // 128 rows x 64 columns of 16 bits
constexpr int kTileSlack = 1024;                // swizzled tiles start on multiples of 1024 bytes

// the adapters of a tile's tokens, each once
struct TileAdapters {
    int own[kTileTokens], list[kTileTokens];    // -1: none
    uint32_t bits[kTileTokens / 32];
    // by all threads; returns how many there are
    __device__ __forceinline__ int find(const AdapterArgs& p, int first) {
        const int t = threadIdx.x;
        int d = 0;
        if (t < kTileTokens) own[t] = d = first + t < p.tokens ? adapter_of(p, first + t) : -1;
        const int one = first < p.tokens ? adapter_of(p, first) : -1;
        if (__syncthreads_and(t >= kTileTokens || d == one)) {             // one request's tokens
            if (t == 0) list[0] = one;
            __syncthreads();
            return one >= 0;
        }
        bool lead = false;
        if (t < kTileTokens) {
            bool again = own[t] < 0;
            for (int i = 0; i < kTileTokens; i += 4) {
                const int4 v = *reinterpret_cast<const int4*>(own + i);
                again |= (i < t && v.x == own[t]) | (i + 1 < t && v.y == own[t]) | (i + 2 < t && v.z == own[t]) | (i + 3 < t && v.w == own[t]);
            }
            lead = !again;
            const uint32_t mine = __ballot_sync(0xFFFFFFFFu, lead);
            if ((t & 31) == 0) bits[t >> 5] = mine;
        }
        __syncthreads();
        int before = 0, all = 0;
#pragma unroll
        for (int i = 0; i < kTileTokens / 32; ++i) {
            if (i < t / 32) before += __popc(bits[i]);
            all += __popc(bits[i]);
        }
        if (lead) list[before + __popc(bits[t / 32] & ((1u << (t & 31)) - 1))] = own[t];
        __syncthreads();
        return all;
    }
};

// ---------------------------------------------------------------- S = x A^T
// 128 tokens x 16 RT ranks; the CTAs of a cluster split k and add their parts up in rank order through distributed shared memory.
// 8192 tokens, 2688 columns, rank 64: 19 us from a cold cache, where reading x takes 7; the rest is the start (index, adapters of the
// tile), the wait for copies and the exchange.
template <int RT> constexpr int kDownPipe = RT == 8 ? 4 : 3;
template <int RT> constexpr int kDownTileStage = kBoxBytes + 16 * RT * 128;
template <int RT> constexpr int kDownPitch = 16 * RT + 4;                        // floats of a token's sums
template <int RT> constexpr int kDownTileSmem = kDownPipe<RT> * kDownTileStage<RT> + kTileTokens * kDownPitch<RT> * 4 + kTileSlack;
static_assert(kDownTileSmem<8> + 4096 <= 227 * 1024 && 2 * (kDownTileSmem<4> + 4096) <= 227 * 1024);

template <int DT, int RT>
__global__ void __launch_bounds__(kDownThreads, RT == 8 ? 1 : 2) adapter_down_tiles(const __grid_constant__ AdapterMaps m) {
    constexpr int R = 16 * RT, PIPE = kDownPipe<RT>, STAGE = kDownTileStage<RT>, PITCH = kDownPitch<RT>;
    constexpr uint32_t COLS = R < 32 ? 32 : R;
    const AdapterArgs& p = m.p;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t bars[2 * PIPE + 3];
    __shared__ uint32_t tmem_slot;
    __shared__ volatile uint32_t abort;
    __shared__ __align__(16) TileAdapters tile;
    const uint32_t smem = (smem_addr(smem_raw) + 1023u) & ~1023u;
    float* const sums = reinterpret_cast<float*>(smem_raw + (smem - smem_addr(smem_raw)) + PIPE * STAGE);      // [tokens][PITCH]
    const uint32_t full = smem_addr(bars), empty = full + 8 * PIPE, ready = empty + 8 * PIPE, drained = ready + 8, drain = drained + 8;
    const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31, rank = uniform(cluster_rank());
    const int first = int(blockIdx.x / p.ctas) * kTileTokens, count = min(kTileTokens, p.tokens - first);
    if (threadIdx.x == 0) {
        for (int i = 0; i < PIPE; ++i) {
            barrier_init(full + 8 * i, 1);
            barrier_init(empty + 8 * i, 1);
        }
        barrier_init(ready, 1);
        barrier_init(drained, kDownWarps);
        barrier_init(drain, 1);
        abort = 0;
        fence_barrier_init();
    }
    grid_launch();
    grid_wait();
    const int adapters = uniform(tile.find(p, first));
    // only now: no launch before this one can still want tensor memory
    if (warp == kDownWarps + 1) {
        tmem_alloc<1>(smem_addr(&tmem_slot), COLS);
        fence_before();
    }
    __syncthreads();
    fence_after();
    const uint32_t tmem = uniform(tmem_slot);
    // every CTA has chunks: a cluster has no more CTAs than there are
    const int chunks = (p.k + 63) / 64, c0 = int(int64_t(chunks) * rank / p.ctas), c1 = int(int64_t(chunks) * (rank + 1) / p.ctas);

    if (warp == kDownWarps) {
        bool ok = true;
        int it = 0;
        for (int i = 0; i < adapters && ok; ++i) {
            const int row = tile.list[i] * p.rank;
            for (int c = c0; c < c1; ++c, ++it) {
                const int slot = it % PIPE;
                if (it >= PIPE && !(ok = barrier_wait_warp(empty + 8 * slot, (it / PIPE & 1) ^ 1, &abort))) break;
                const uint32_t to = smem + slot * STAGE, bar = full + 8 * slot;
                barrier_expect_warp(bar, STAGE);
                tma_load_2d(to, &m.x, c * 64, first, bar);
                tma_load_2d(to + kBoxBytes, &m.a, c * 64, row, bar);
            }
        }
        // arrivals that are still owed come before the shared memory goes away
        for (int i = max(it - PIPE, 0); i < it && ok; ++i) ok = barrier_wait_warp(empty + 8 * (i % PIPE), i / PIPE & 1, &abort);
        if (gave_up_warp(&abort))
            for (int i = max(it - PIPE, 0); i < it; ++i) barrier_drain(full + 8 * (i % PIPE), i / PIPE & 1);
        __syncwarp();
    } else if (warp == kDownWarps + 1) {
        bool ok = true;
        int it = 0;
        for (int i = 0; i < adapters && ok; ++i) {
            if (i && !(ok = barrier_wait_warp(drained, (i - 1) & 1, &abort))) break;
            fence_after();
            for (int c = c0; c < c1; ++c, ++it) {
                const int slot = it % PIPE;
                if (!(ok = barrier_wait_warp(full + 8 * slot, it / PIPE & 1, &abort))) break;
                fence_after();
                const uint32_t from = smem + slot * STAGE;
#pragma unroll
                for (int kk = 0; kk < 4; ++kk)
                    mma_16bit<1>(tmem, swizzled_desc(from + 32 * kk, 16), swizzled_desc(from + kBoxBytes + 32 * kk, 16),
                                 desc_16bit(DT == kBf16, false, false, kTileTokens, R), c > c0 || kk);
                mma_commit<1>(empty + 8 * slot);
            }
            if (ok) mma_commit<1>(ready);
        }
        if (gave_up_warp(&abort)) {        // products in flight read this shared memory
            mma_commit<1>(drain);
            barrier_drain(drain, 0);
        }
        __syncwarp();
    } else {
        const int row = warp * 32 + lane, mine = tile.own[row];
        float4* const to = reinterpret_cast<float4*>(sums + row * PITCH);
        for (int i = 0; i < adapters; ++i) {
            if (!barrier_wait_warp(ready, i & 1, &abort, wait_limit(c1 - c0))) break;
            fence_after();
            const bool take = tile.list[i] == mine;
#pragma unroll
            for (int c = 0; c < R; c += 16) {
                uint32_t v[16];
                __syncwarp();
                tmem_load16(tmem + (uint32_t(warp * 32) << 16) + c, v);
                tmem_wait_loads();
                if (take) {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        to[c / 4 + j] = make_float4(__uint_as_float(v[4 * j]), __uint_as_float(v[4 * j + 1]), __uint_as_float(v[4 * j + 2]),
                                                    __uint_as_float(v[4 * j + 3]));
                }
            }
            fence_before();
            __syncwarp();
            if (lane == 0) barrier_arrive(drained);
        }
        __syncwarp();
    }
    fence_before();
    __syncthreads();
    if (warp == kDownWarps + 1) {
        fence_after();
        tmem_free<1>(tmem, COLS);
    }
    __syncwarp();
    cluster_sync();
    // The cluster's sums of every ctas-th token, scaled, split and stored.  A lane has four ranks; all CTAs' parts are asked for
    // before the first is added.
    constexpr int LANES = R / 4, AT_ONCE = 32 / LANES;
    for (int base = warp * AT_ONCE; base * p.ctas < kTileTokens; base += kDownThreads / 32 * AT_ONCE) {
        const int token = (base + lane / LANES) * p.ctas + rank, r = lane % LANES * 4;
        const int i = token < count ? tile.own[token] : -1;
        float4 part[8];
        const uint32_t from = smem_addr(sums + min(token, kTileTokens - 1) * PITCH + r);
#pragma unroll
        for (int q = 0; q < 8; ++q)
            if (q < p.ctas) part[q] = ld_cluster_f32x4(peer_addr(from, q));
        float v[4] = {};
#pragma unroll
        for (int q = 0; q < 8; ++q)
            if (q < p.ctas) {
                v[0] += part[q].x; v[1] += part[q].y; v[2] += part[q].z; v[3] += part[q].w;
            }
        const float c = p.scale && i >= 0 ? p.scale[i] : 1.0f;
        float top = 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[j] = i >= 0 && r + j < p.rank ? v[j] * c : 0.0f;     // past the adapter's own ranks lie the next one's
            if (fabsf(v[j]) < __uint_as_float(kInfBits)) top = fmaxf(top, fabsf(v[j]));
        }
        float times = 1.0f;
        if constexpr (DT == kFp16) {
#pragma unroll
            for (int s = LANES / 2; s; s >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, s));
            float back;
            range_of(top, times, back);
            if (i >= 0 && r == 0) p.back[first + token] = back;
        }
        if (i < 0) continue;
        uint32_t high[2], low[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            split_pair<DT>(v[2 * j] * times, v[2 * j + 1] * times, high[j], low[j]);
        }
        uint16_t* const to = p.s + size_t(first + token) * (2 * R) + r;
        *reinterpret_cast<uint2*>(to) = make_uint2(high[0], high[1]);
        *reinterpret_cast<uint2*>(to + R) = make_uint2(low[0], low[1]);
    }
    __syncwarp();
    cluster_sync();                        // the others' sums have been read
}

// ---------------------------------------------------------------- out = y + S B^T
// 128 tokens, 128 features at a time.  S stays in shared memory; B and y come through rings, y is added to where it lies and leaves from
// there.  High and low halves of S are two products with the same rows of B, added up in tensor memory, where two accumulators let the
// next products run meanwhile.  8192 tokens, 5376 features, rank 64: 43 us for 176 MB from a cold cache; both launches take 57, without any
// adapter to apply 39, and a plain copy of y 28.  Five blocks of y under way instead of three, with a loading warp of their own, changed
// nothing.
constexpr int kUpBlock = 128, kUpOut = 2 * kBoxBytes;                            // features; bytes of y
constexpr int kUpOutWarps = 8, kUpThreads = 32 * (kUpOutWarps + 2);              // 32 tokens x 64 features each
template <int RT> constexpr int kRankBoxes = RT == 8 ? 2 : 1;                    // of 64 ranks
template <int RT> constexpr int kUpRing = RT == 8 ? 2 : 3;
template <int RT> constexpr int kUpTileSmem = 2 * kRankBoxes<RT> * kBoxBytes + kUpRing<RT> * (kRankBoxes<RT> * kBoxBytes + kUpOut) + kTileSlack;
static_assert(kUpTileSmem<4> + 4096 <= 227 * 1024 && kUpTileSmem<8> + 4096 <= 227 * 1024);

template <int DT, int RT>
__global__ void __launch_bounds__(kUpThreads, 1) adapter_up_tiles(const __grid_constant__ AdapterMaps m) {
    constexpr int BOXES = kRankBoxes<RT>, RING = kUpRing<RT>, B_BYTES = BOXES * kBoxBytes;
    const AdapterArgs& p = m.p;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t bars[4 * RING + 6];
    __shared__ uint32_t tmem_slot;
    __shared__ volatile uint32_t abort;
    __shared__ __align__(16) TileAdapters tile;
    const uint32_t smem = (smem_addr(smem_raw) + 1023u) & ~1023u;
    const uint32_t s_at = smem, b_at = s_at + 2 * B_BYTES, y_at = b_at + RING * B_BYTES;      // S: high, then low
    const uint32_t b_full = smem_addr(bars), b_empty = b_full + 8 * RING, y_full = b_empty + 8 * RING, y_empty = y_full + 8 * RING,
                   s_full = y_empty + 8 * RING, ready = s_full + 8, drained = ready + 16, drain = drained + 16;
    const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const int first = int(blockIdx.x) * kTileTokens;
    const int f0 = int(blockIdx.y) * p.blocks * kUpBlock, blocks = (min(p.n - f0, p.blocks * kUpBlock) + kUpBlock - 1) / kUpBlock;
    if (threadIdx.x == 0) {
        for (int i = 0; i < RING; ++i) {
            barrier_init(b_full + 8 * i, 1);
            barrier_init(b_empty + 8 * i, 1);
            barrier_init(y_full + 8 * i, 1);
            barrier_init(y_empty + 8 * i, kUpOutWarps);
        }
        barrier_init(s_full, 1);
        for (int i = 0; i < 2; ++i) {
            barrier_init(ready + 8 * i, 1);
            barrier_init(drained + 8 * i, kUpOutWarps);
        }
        barrier_init(drain, 1);
        abort = 0;
        fence_barrier_init();
    }
    grid_launch();
    grid_wait();
    const int adapters = uniform(tile.find(p, first));
    if (warp == kUpOutWarps + 1) {
        tmem_alloc<1>(smem_addr(&tmem_slot), 2 * kUpBlock);
        fence_before();
    }
    __syncthreads();
    fence_after();
    const uint32_t tmem = uniform(tmem_slot);

    if (warp == kUpOutWarps) {
        bool ok = true;
        int unit = 0, block = 0;
        if (adapters) {
            barrier_expect_warp(s_full, 2 * B_BYTES);
            for (int c = 0; c < BOXES; ++c) {
                tma_load_2d(s_at + c * kBoxBytes, &m.high, c * 64, first, s_full);
                tma_load_2d(s_at + B_BYTES + c * kBoxBytes, &m.low, c * 64, first, s_full);
            }
        }
        for (; block < blocks && ok; ++block) {
            const int slot = block % RING, f = f0 + block * kUpBlock;
            if (block >= RING && !(ok = barrier_wait_warp(y_empty + 8 * slot, (block / RING & 1) ^ 1, &abort))) break;
            barrier_expect_warp(y_full + 8 * slot, kUpOut);
            for (int h = 0; h < 2; ++h) tma_load_2d(y_at + slot * kUpOut + h * kBoxBytes, &m.y, f + h * 64, first, y_full + 8 * slot);
            for (int i = 0; i < adapters; ++i, ++unit) {
                const int at = unit % RING;
                if (unit >= RING && !(ok = barrier_wait_warp(b_empty + 8 * at, (unit / RING & 1) ^ 1, &abort))) break;
                barrier_expect_warp(b_full + 8 * at, B_BYTES);
                // past this adapter's features lie the next one's, whose results are not stored
                for (int c = 0; c < BOXES; ++c)
                    tma_load_2d(b_at + at * B_BYTES + c * kBoxBytes, &m.b, c * 64, tile.list[i] * p.n + f, b_full + 8 * at);
            }
        }
        for (int i = max(unit - RING, 0); i < unit && ok; ++i) ok = barrier_wait_warp(b_empty + 8 * (i % RING), i / RING & 1, &abort);
        if (gave_up_warp(&abort)) {        // what has been started lands before the shared memory goes away
            if (adapters) barrier_drain(s_full, 0);
            for (int i = max(unit - RING, 0); i < unit; ++i) barrier_drain(b_full + 8 * (i % RING), i / RING & 1);
            for (int i = max(block - RING, 0); i < block; ++i) barrier_drain(y_full + 8 * (i % RING), i / RING & 1);
        }
        __syncwarp();
    } else if (warp == kUpOutWarps + 1) {
        const int units = blocks * adapters;
        bool ok = units == 0 || barrier_wait_warp(s_full, 0, &abort);
        for (int unit = 0; unit < units && ok; ++unit) {
            const int at = unit % RING, buf = unit & 1;
            if (!(ok = barrier_wait_warp(b_full + 8 * at, unit / RING & 1, &abort))) break;
            if (unit > 1 && !(ok = barrier_wait_warp(drained + 8 * buf, (unit / 2 - 1) & 1, &abort))) break;
            fence_after();
            const uint32_t d = tmem + buf * kUpBlock, from = b_at + at * B_BYTES;
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int kk = 0; kk < RT; ++kk) {
                    const uint32_t in = kk / 4 * kBoxBytes + kk % 4 * 32;
                    mma_16bit<1>(d, swizzled_desc(s_at + half * B_BYTES + in, 16), swizzled_desc(from + in, 16),
                                 desc_16bit(DT == kBf16, false, false, kTileTokens, kUpBlock), half | kk);
                }
            mma_commit<1>(b_empty + 8 * at);
            mma_commit<1>(ready + 8 * buf);
        }
        if (gave_up_warp(&abort)) {
            mma_commit<1>(drain);
            barrier_drain(drain, 0);
        }
        __syncwarp();
    } else {
        const int rows = warp % 4 * 32, row = rows + lane, half = warp / 4, mine = tile.own[row];
        const float back = DT == kFp16 && mine >= 0 ? __ldcg(p.back + first + row) : 1.0f;
        bool ok = true;
        int unit = 0;
        for (int block = 0; block < blocks && ok; ++block) {
            const int slot = block % RING, f = f0 + block * kUpBlock;
            const uint32_t y = y_at + slot * kUpOut + half * kBoxBytes + row * 128;
            if (!(ok = barrier_wait_warp(y_full + 8 * slot, block / RING & 1, &abort))) break;
            for (int i = 0; i < adapters; ++i, ++unit) {
                const int buf = unit & 1;
                if (!(ok = barrier_wait_warp(ready + 8 * buf, unit / 2 & 1, &abort))) break;
                fence_after();
                const bool take = tile.list[i] == mine;
                if (__any_sync(0xFFFFFFFFu, take)) {
#pragma unroll
                    for (int c = 0; c < 64; c += 32) {
                        uint32_t v[32];
                        __syncwarp();
                        tmem_load32(tmem + buf * kUpBlock + half * 64 + (uint32_t(rows) << 16) + c, v);
                        tmem_wait_loads();
                        if (!take) continue;
#pragma unroll
                        for (int q = 0; q < 4; ++q) {      // pieces of 8 columns
                            const uint32_t at = y + (((c / 8 + q) ^ (row & 7)) << 4);
                            uint32_t w[4];
                            ld_shared_v4(at, w);
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const float2 old = unpack2(w[j], DT);
                                const float2 add = make_float2(__uint_as_float(v[8 * q + 2 * j]), __uint_as_float(v[8 * q + 2 * j + 1]));
                                const float2 sum = DT == kFp16 ? fma_pair(add, twice(back), old) : add_pair(add, old);
                                w[j] = pack2(sum.x, sum.y, DT);
                            }
                            st_shared_v4(at, w[0], w[1], w[2], w[3]);
                        }
                    }
                }
                fence_before();
                __syncwarp();
                if (lane == 0) barrier_arrive(drained + 8 * buf);
            }
            if (!ok) break;
            fence_async_shared();
            __syncwarp();
            if (lane == 0) {
                if (first + rows < p.tokens && f + half * 64 < p.n)
                    tma_store_2d(&m.out, y_at + slot * kUpOut + half * kBoxBytes + rows * 128, f + half * 64, first + rows);
                tma_store_wait_read<1>();                  // the block before this one has left
                if (block) barrier_arrive(y_empty + 8 * ((block - 1) % RING));
            }
            __syncwarp();
        }
        if (lane == 0) tma_store_wait_all();
        __syncwarp();
    }
    fence_before();
    __syncthreads();
    if (warp == kUpOutWarps + 1) {
        fence_after();
        tmem_free<1>(tmem, 2 * kUpBlock);
    }
}

}  // namespace ff
}  // namespace equarx
