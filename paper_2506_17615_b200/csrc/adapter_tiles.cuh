// Low-rank adapters of many tokens on the fifth-generation tensor cores, for rows that TMA can read and write.
//
// A cluster has a tile of 128 tokens.  Its CTAs split k for S = x A^T, exchange their parts, so that each has the whole of S in shared
// memory, split into high and low halves of 16 bits, and then split n for out = y + S B^T.  More than one cluster for a tile: each
// makes S for itself, and they split n.  A product runs once for each adapter that the tile's tokens have, and only this adapter's
// tokens take their rows of its result: what is not finite in one request's adapter does not reach another request.
//
// Everything comes and goes by TMA, so that few instructions are left: x, and A of up to four adapters for it, through a ring; the first
// blocks of y while S is not there yet; y is added to where it lies and leaves from there.  High and low halves of S are two products
// with the same rows of B, added up in tensor memory.
//
// 8192 tokens, 2688 -> 5376, rank 64: 45 us for one request, 48 for 7, 4.9 and 4.6 TB/s (rank 16: 44).  Bound by DRAM in the second part,
// about 31 us of it, and by the chain of start, first part and exchange before.  Two launches with S in memory took 57 and read y
// only in the second; one group of output warps 57; x read once for each adapter of a tile 51; stores by a warp of their own 54; blocks of
// a cluster's CTAs side by side in a row made no difference.  Results held in registers until all adapters of a tile are done, so that y
// is written once: 54, and 512 tokens of 16 requests mixed, rank 16, 31 instead of 35; a form for each 55 and 41, for want of registers.
// Of 128 ranks, which leave room for two blocks of y, 69.
#pragma once
#include "adapter_kernels.cuh"

namespace equarx {
namespace ff {

struct AdapterMaps {
    CUtensorMap x, a, b, y, out;                // boxes of 64 columns; of 128 rows, a: of 16 RT, out: of 32 (columns to a multiple of 8)
    AdapterArgs p;
};
constexpr int kTileTokens = 128;
constexpr int kBoxBytes = kTileTokens * 128;    // 128 rows x 64 columns of 16 bits
constexpr int kTileSlack = 1024;                // swizzled tiles start on multiples of 1024 bytes
constexpr int kTileBlock = 128, kYBytes = 2 * kBoxBytes;                         // features; bytes of y
// Two groups of eight warps put out alternate blocks, 32 tokens x 64 features each, from tensor memory and slots of y of their own.
constexpr int kGroupWarps = 8, kTileOutWarps = 2 * kGroupWarps, kTileAdapterThreads = 32 * (kTileOutWarps + 2);

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

// Shared memory: S high, S low | blocks of y | blocks of B.  Before S is whole, x and A go through a ring in the place of the later blocks
// of y and the earlier ones of B, and the CTA's part of S is behind it (128 ranks: the part in the place of y).
template <int RT> struct TileRoom {
    static constexpr int R = 16 * RT;
    static constexpr int BOXES = RT == 8 ? 2 : 1;                                // of 64 ranks
    static constexpr int B_BYTES = BOXES * kBoxBytes;
    static constexpr int Y_RING = RT == 8 ? 2 : 4, B_RING = RT == 8 ? 2 : 4;     // a slot of y belongs to one group
    static constexpr int EARLY_Y = RT == 8 ? 0 : 2, EARLY_B = 2;                 // slots that nothing else is in before
    static constexpr int AT_ONCE = RT == 8 ? 1 : RT == 1 ? 4 : 2;                // adapters that a pass over x serves
    static constexpr int PIPE = RT < 4 ? 4 : 3, STAGE = kBoxBytes + AT_ONCE * R * 128;
    static constexpr int Y = 2 * B_BYTES, B = Y + Y_RING * kYBytes, X = RT == 8 ? B : Y + EARLY_Y * kYBytes;
    static constexpr int PART = kTileTokens * R * 4, PARTS = RT == 8 ? Y : B + EARLY_B * B_BYTES;
    static constexpr int END = RT == 8 ? X + PIPE * STAGE : B + B_RING * B_BYTES, BYTES = END + kTileSlack;
    static_assert(RT == 8 || (X + PIPE * STAGE <= PARTS && PARTS + PART <= END));
    static_assert(RT != 8 || (B + B_RING * B_BYTES <= END && PARTS + PART <= X));
};
// A CTA here waits for its cluster while it has tensor memory, and asks for it after the launch before, where a CTA of tile_kernel asks
// earlier.  So that none of them waits in a circle, no other CTA that wants tensor memory, 24 KB of shared memory at least, fits on
// the same SM of 228 KB.
template <int RT> constexpr bool kAlone = TileRoom<RT>::BYTES + 24 * 1024 > 228 * 1024;
static_assert(kAlone<1> && kAlone<2> && kAlone<4> && kAlone<8>);
static_assert(TileRoom<1>::BYTES + 2048 <= 227 * 1024 && TileRoom<2>::BYTES + 2048 <= 227 * 1024 && TileRoom<4>::BYTES + 2048 <= 227 * 1024 &&
              TileRoom<8>::BYTES + 2048 <= 227 * 1024);

template <int DT, int RT>
__global__ void __launch_bounds__(kTileAdapterThreads, 1) adapter_tiles_kernel(const __grid_constant__ AdapterMaps m) {
    using Room = TileRoom<RT>;
    constexpr int R = Room::R, PIPE = Room::PIPE, STAGE = Room::STAGE, BOXES = Room::BOXES, AT_ONCE = Room::AT_ONCE, Y_RING = Room::Y_RING,
                  B_RING = Room::B_RING, B_BYTES = Room::B_BYTES;
    constexpr uint32_t COLS = 4 * kTileBlock;
    const AdapterArgs& p = m.p;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t bars[2 * PIPE + 2 * Y_RING + 2 * B_RING + 11];
    __shared__ uint32_t tmem_slot;
    __shared__ volatile uint32_t abort;
    __shared__ float factors[kTileTokens];         // a token's scale, then (fp16) what its S has been divided by
    __shared__ __align__(16) TileAdapters tile;
    const uint32_t smem = (smem_addr(smem_raw) + 1023u) & ~1023u;
    const uint32_t s_at = smem, y_at = smem + Room::Y, part_at = smem + Room::PARTS, x_at = smem + Room::X, b_at = smem + Room::B;
    const uint32_t full = smem_addr(bars), empty = full + 8 * PIPE, b_full = empty + 8 * PIPE, b_empty = b_full + 8 * B_RING,
                   y_full = b_empty + 8 * B_RING, y_empty = y_full + 8 * Y_RING, got = y_empty + 8 * Y_RING, taken = got + 8,
                   ready = taken + 8, drained = ready + 32, drain = drained + 32;      // ready, drained: of two accumulators for each group
    const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31, rank = uniform(cluster_rank());
    const int cluster = int(blockIdx.x / p.ctas), first = cluster / p.copies * kTileTokens;
    if (threadIdx.x == 0) {
        for (int i = 0; i < PIPE; ++i) {
            barrier_init(full + 8 * i, 1);
            barrier_init(empty + 8 * i, 1);
        }
        for (int i = 0; i < B_RING; ++i) {
            barrier_init(b_full + 8 * i, 1);
            barrier_init(b_empty + 8 * i, 1);
        }
        for (int i = 0; i < Y_RING; ++i) {
            barrier_init(y_full + 8 * i, 1);
            barrier_init(y_empty + 8 * i, kGroupWarps);
        }
        barrier_init(got, 1);
        barrier_init(taken, kTileOutWarps);
        for (int i = 0; i < 4; ++i) {
            barrier_init(ready + 8 * i, 1);
            barrier_init(drained + 8 * i, kGroupWarps);
        }
        barrier_init(drain, 1);
        abort = 0;
        fence_barrier_init();
    }
    grid_launch();
    grid_wait();
    const int adapters = uniform(tile.find(p, first));
    if (threadIdx.x < kTileTokens) {
        const int i = tile.own[threadIdx.x];
        factors[threadIdx.x] = p.scale && i >= 0 ? p.scale[i] : 1.0f;
    }
    // only now: no launch before this one can still want tensor memory
    if (warp == kTileOutWarps + 1) {
        tmem_alloc<1>(smem_addr(&tmem_slot), COLS);
        fence_before();
    }
    __syncthreads();
    fence_after();
    const uint32_t tmem = uniform(tmem_slot);
    // chunks of k: the first CTAs of the cluster have one at least
    const int chunks = (p.k + 63) / 64, sharers = min(p.ctas, chunks);
    const int c0 = rank < sharers ? int(int64_t(chunks) * rank / sharers) : 0;
    const int c1 = rank < sharers ? int(int64_t(chunks) * (rank + 1) / sharers) : 0;
    // blocks of n
    const int all = (p.n + kTileBlock - 1) / kTileBlock, place = cluster % p.copies * p.ctas + rank, places = p.copies * p.ctas;
    const int b0 = int(int64_t(all) * place / places), blocks = int(int64_t(all) * (place + 1) / places) - b0, units = blocks * adapters;

    // ------------------------------------------------ this CTA's part of S
    // the loading warp's: chunks, blocks of y and units of B that it has asked for
    int chunk = 0, asked = 0, unit = 0;
    auto ask_y = [&] {
        const uint32_t bar = y_full + 8 * (asked % Y_RING), to = y_at + asked % Y_RING * kYBytes;
        barrier_expect_warp(bar, kYBytes);
        for (int h = 0; h < 2; ++h) tma_load_2d(to + h * kBoxBytes, &m.y, (b0 + asked) * kTileBlock + h * 64, first, bar);
        ++asked;
    };
    // past this adapter's features lie the next one's, whose results are not stored
    auto ask_b = [&](int block, int i) {
        const uint32_t bar = b_full + 8 * (unit % B_RING), to = b_at + unit % B_RING * B_BYTES;
        barrier_expect_warp(bar, B_BYTES);
        for (int c = 0; c < BOXES; ++c) tma_load_2d(to + c * kBoxBytes, &m.b, c * 64, tile.list[i] * p.n + (b0 + block) * kTileBlock, bar);
        ++unit;
    };
    if (warp == kTileOutWarps) {
        bool ok = true;
        auto early_y = [&] {
            while (asked < min(Room::EARLY_Y, blocks)) ask_y();
        };
        for (int i = 0; i < adapters && ok; i += AT_ONCE) {
            const int now = min(AT_ONCE, adapters - i);
            for (int c = c0; c < c1; ++c, ++chunk) {
                const int slot = chunk % PIPE;
                if (chunk == PIPE) early_y();
                if (chunk >= PIPE && !(ok = barrier_wait_warp(empty + 8 * slot, (chunk / PIPE & 1) ^ 1, &abort))) break;
                const uint32_t to = x_at + slot * STAGE, bar = full + 8 * slot;
                barrier_expect_warp(bar, kBoxBytes + now * (R * 128));
                tma_load_2d(to, &m.x, c * 64, first, bar);
                for (int g = 0; g < now; ++g) tma_load_2d(to + kBoxBytes + g * (R * 128), &m.a, c * 64, tile.list[i + g] * p.rank, bar);
            }
        }
        early_y();
        // the ring has been read: B may come
        for (int i = max(chunk - PIPE, 0); i < chunk && ok; ++i) ok = barrier_wait_warp(empty + 8 * (i % PIPE), i / PIPE & 1, &abort);
        if (gave_up_warp(&abort))          // what has been started lands before the shared memory goes away
            for (int i = max(chunk - PIPE, 0); i < chunk; ++i) barrier_drain(full + 8 * (i % PIPE), i / PIPE & 1);
        else
            while (unit < min(Room::EARLY_B, units)) ask_b(unit / adapters, unit % adapters);
        __syncwarp();
    } else if (warp == kTileOutWarps + 1) {
        bool ok = true;
        int it = 0;
        for (int i = 0, pass = 0; i < adapters && c0 < c1 && ok; i += AT_ONCE, ++pass) {
            if (pass && !(ok = barrier_wait_warp(taken, (pass - 1) & 1, &abort))) break;
            fence_after();
            const int now = min(AT_ONCE, adapters - i);
            for (int c = c0; c < c1; ++c, ++it) {
                const int slot = it % PIPE;
                if (!(ok = barrier_wait_warp(full + 8 * slot, it / PIPE & 1, &abort))) break;
                fence_after();
                const uint32_t from = x_at + slot * STAGE;
                for (int g = 0; g < now; ++g)
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk)
                        mma_16bit<1>(tmem + g * R, swizzled_desc(from + 32 * kk, 16),
                                     swizzled_desc(from + kBoxBytes + g * (R * 128) + 32 * kk, 16),
                                     desc_16bit(DT == kBf16, false, false, kTileTokens, R), c > c0 || kk);
                mma_commit<1>(empty + 8 * slot);
            }
            if (ok) mma_commit<1>(got);
        }
        if (gave_up_warp(&abort)) {        // products in flight read this shared memory
            mma_commit<1>(drain);
            barrier_drain(drain, 0);
        }
        __syncwarp();
    } else {
        // [tokens][ranks]; of a row, four ranks change places with others, so that the rows of a warp meet all banks
        const int row = warp % 4 * 32 + lane, mine = tile.own[row];
        for (int i = 0, pass = 0; i < adapters && c0 < c1; i += AT_ONCE, ++pass) {
            if (!barrier_wait_warp(got, pass & 1, &abort, wait_limit(c1 - c0))) break;
            fence_after();
            for (int g = 0; g < min(AT_ONCE, adapters - i); ++g) {
                const bool take = tile.list[i + g] == mine;
                if (!__any_sync(0xFFFFFFFFu, take)) continue;
#pragma unroll
                for (int c = 0; c < R; c += 64) {
                    const int from = c + warp / 4 * 16;
                    if (from >= R) continue;
                    uint32_t v[16];
                    __syncwarp();
                    tmem_load16(tmem + (uint32_t(warp % 4 * 32) << 16) + g * R + from, v);
                    tmem_wait_loads();
                    if (take) {
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            st_shared_v4(part_at + row * (R * 4) + (((from / 4 + j) ^ (row & (R / 4 - 1))) << 4), v[4 * j], v[4 * j + 1],
                                         v[4 * j + 2], v[4 * j + 3]);
                    }
                }
            }
            fence_before();
            __syncwarp();
            if (lane == 0) barrier_arrive(taken);
        }
        __syncwarp();
    }
    // ------------------------------------------------ S, whole
    // Every ctas-th token, scaled, split and sent to all.  A lane has four ranks; all CTAs' parts are asked for before the first
    // is added, and they are added in rank order.
    if (adapters) {                        // all CTAs of the cluster alike
        fence_before();
        cluster_sync();
        fence_after();
        constexpr int LANES = R / 4, TOKENS = 32 / LANES;
        const int count = p.tokens - first;
        for (int base = warp * TOKENS; base * p.ctas < kTileTokens; base += kTileAdapterThreads / 32 * TOKENS) {
            const int token = (base + lane / LANES) * p.ctas + rank, r = lane % LANES * 4, row = min(token, kTileTokens - 1);
            const int i = token < min(count, kTileTokens) ? tile.own[token] : -1;
            const uint32_t from = part_at + row * (R * 4) + (((r / 4) ^ (row & (R / 4 - 1))) << 4);
            float4 part[8];
#pragma unroll
            for (int q = 0; q < 8; ++q)
                if (q < sharers) part[q] = ld_cluster_f32x4(peer_addr(from, q));
            float v[4] = {};
#pragma unroll
            for (int q = 0; q < 8; ++q)
                if (q < sharers) {
                    v[0] += part[q].x; v[1] += part[q].y; v[2] += part[q].z; v[3] += part[q].w;
                }
            const float c = factors[row];
            float top = 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[j] = i >= 0 && r + j < p.rank ? v[j] * c : 0.0f;     // past the adapter's own ranks lie the next one's
                if (fabsf(v[j]) < __uint_as_float(kInfBits)) top = fmaxf(top, fabsf(v[j]));
            }
            float times = 1.0f, back = 1.0f;
            if constexpr (DT == kFp16) {
#pragma unroll
                for (int d = LANES / 2; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
                range_of(top, times, back);
            }
            if (i < 0) continue;
            uint32_t high[2], low[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) split_pair<DT>(v[2 * j] * times, v[2 * j + 1] * times, high[j], low[j]);
            const uint32_t to = s_at + r / 64 * kBoxBytes + token * 128 + (((r % 64 / 8) ^ (token & 7)) << 4) + r % 8 * 2;
            for (int q = 0; q < p.ctas; ++q) {
                st_cluster_v2(peer_addr(to, q), high[0], high[1]);
                st_cluster_v2(peer_addr(to + B_BYTES, q), low[0], low[1]);
                if (DT == kFp16 && r == 0) st_cluster_f32(peer_addr(smem_addr(factors + token), q), back);
            }
        }
        fence_async();                     // the products read S, and y comes to where the parts were
        __syncwarp();
        cluster_sync();
        fence_async();
    }

    // ------------------------------------------------ out = y + S B^T
    bool ok = !gave_up_warp(&abort);
    if (warp == kTileOutWarps) {
        while (ok && asked < min(Y_RING, blocks)) ask_y();
        for (int block = 0; block < blocks && ok; ++block) {
            if (block >= asked) {
                if (!(ok = barrier_wait_warp(y_empty + 8 * (block % Y_RING), (block / Y_RING & 1) ^ 1, &abort))) break;
                ask_y();
            }
            for (int i = max(unit - block * adapters, 0); i < adapters; ++i) {
                if (unit >= B_RING && !(ok = barrier_wait_warp(b_empty + 8 * (unit % B_RING), (unit / B_RING & 1) ^ 1, &abort))) break;
                ask_b(block, i);
            }
        }
        // arrivals that are still owed come before the shared memory goes away
        for (int i = max(unit - B_RING, 0); i < unit && ok; ++i)
            ok = barrier_wait_warp(b_empty + 8 * (i % B_RING), i / B_RING & 1, &abort);
        if (gave_up_warp(&abort)) {
            for (int i = max(unit - B_RING, 0); i < unit; ++i) barrier_drain(b_full + 8 * (i % B_RING), i / B_RING & 1);
            for (int i = max(asked - Y_RING, 0); i < asked; ++i) barrier_drain(y_full + 8 * (i % Y_RING), i / Y_RING & 1);
        }
        __syncwarp();
    } else if (warp == kTileOutWarps + 1) {
        const bool start = ok;
        int u = 0;
        for (int block = 0; block < blocks && ok; ++block)
            for (int i = 0; i < adapters; ++i, ++u) {
                const int at = u % B_RING, turn = block / 2 * adapters + i, buf = block % 2 * 2 + turn % 2;      // turn: of the group
                if (!(ok = barrier_wait_warp(b_full + 8 * at, u / B_RING & 1, &abort))) break;
                if (turn > 1 && !(ok = barrier_wait_warp(drained + 8 * buf, (turn / 2 - 1) & 1, &abort))) break;
                fence_after();
                const uint32_t d = tmem + buf * kTileBlock, from = b_at + at * B_BYTES;
#pragma unroll
                for (int half = 0; half < 2; ++half)
#pragma unroll
                    for (int kk = 0; kk < RT; ++kk) {
                        const uint32_t in = kk / 4 * kBoxBytes + kk % 4 * 32;
                        mma_16bit<1>(d, swizzled_desc(s_at + half * B_BYTES + in, 16), swizzled_desc(from + in, 16),
                                     desc_16bit(DT == kBf16, false, false, kTileTokens, kTileBlock), half | kk);
                    }
                mma_commit<1>(b_empty + 8 * at);
                mma_commit<1>(ready + 8 * buf);
            }
        if (start && gave_up_warp(&abort)) {
            mma_commit<1>(drain);
            barrier_drain(drain, 0);
        }
        __syncwarp();
    } else {
        const int group = warp / kGroupWarps, rows = warp % 4 * 32, row = rows + lane, half = warp / 4 % 2, mine = tile.own[row];
        const float back = DT == kFp16 && mine >= 0 ? factors[row] : 1.0f;
        const int pieces = p.n & ~7;
        int turn = 0;
        for (int block = group; block < blocks && ok; block += 2) {
            const int slot = block % Y_RING, f = (b0 + block) * kTileBlock;
            const uint32_t y = y_at + slot * kYBytes + half * kBoxBytes + row * 128;
            if (!(ok = barrier_wait_warp(y_full + 8 * slot, block / Y_RING & 1, &abort))) break;
            for (int i = 0; i < adapters; ++i, ++turn) {
                const int buf = group * 2 + turn % 2;
                if (!(ok = barrier_wait_warp(ready + 8 * buf, turn / 2 & 1, &abort))) break;
                fence_after();
                const bool take = tile.list[i] == mine;
                if (__any_sync(0xFFFFFFFFu, take)) {
#pragma unroll
                    for (int c = 0; c < 64; c += 32) {
                        uint32_t v[32];
                        __syncwarp();
                        tmem_load32(tmem + buf * kTileBlock + half * 64 + (uint32_t(rows) << 16) + c, v);
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
            // TMA writes whole pieces of 16 bytes (it would fill the last one with zeros); a lane writes what is left of its row
            if (f + half * 64 + 64 > pieces && first + row < p.tokens) {
                uint16_t* const out = static_cast<uint16_t*>(p.out) + size_t(first + row) * p.ldo;
                for (int c = max(pieces - f - half * 64, 0); c < min(64, p.n - f - half * 64); ++c)
                    out[f + half * 64 + c] = uint16_t(ld_shared_u16(y + (((c / 8) ^ (row & 7)) << 4) + c % 8 * 2));
            }
            fence_async_shared();
            __syncwarp();
            if (lane == 0) {
                if (first + rows < p.tokens && f + half * 64 < pieces)
                    tma_store_2d(&m.out, y_at + slot * kYBytes + half * kBoxBytes + rows * 128, f + half * 64, first + rows);
                tma_store_wait_read<0>();                  // the other group works meanwhile
                barrier_arrive(y_empty + 8 * slot);
            }
            __syncwarp();
        }
        if (lane == 0) tma_store_wait_all();
        __syncwarp();
    }
    fence_before();
    __syncthreads();
    if (warp == kTileOutWarps + 1) {
        fence_after();
        tmem_free<1>(tmem, COLS);
    }
}

}  // namespace ff
}  // namespace equarx
