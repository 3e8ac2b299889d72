// C ABI of the low-rank adapters (include/equarx.h): argument checks, launches.
#include "adapter_tiles.cuh"
#include "host_maps.h"

namespace {

using namespace equarx;
using namespace equarx::ff;
using namespace equarx::host;

constexpr size_t kMaxRank = 128;

inline size_t padded_rank(size_t rank) { return rank <= 16 ? 16 : rank <= 32 ? 32 : rank <= 64 ? 64 : 128; }

// Whether each token gets a cluster of its own, which reads the token's adapter again for each token, or tiles of tokens are
// multiplied with each adapter that they have.  Only the device knows how many that are.  us, bf16, tokens / tiles, requests: 2, one after
// the other | 16 mixed | one for each token:
//   2688 -> 5376, rank 16:  64 tokens 6.9 / 9.1 | 7.6 / 27 | 7.6 / 60     256: 14 / 9.8 | 16 / 28 | 21 / 141    512: 15 / 11 | 24 / 36 | 37 / 216
//                 rank 64:  64        12 / 10 | 13 / 34 | 16 / 79         256: 34 / 11 | 37 / 37 | 46 / 193     512: 35 / 12 | 73 / 46 | 90 / 281
//   512 -> 768,   rank 16:  512       4.5 / 8.4 | 6.7 / 19 | 6.9 / 95     2048: 11 / 8.2 | 18 / 22 | 24 / 119   8192: 50 / 12 | 71 / 41 | 84 / 277
//   128 -> 128,   rank 16:  512       3.6 / 7.9 | 5.7 / 19 | 5.8 / 96     2048: 8.8 / 7.7 | 15 / 19 | 15 / 104  8192: 31 / 7.4 | 53 / 20 | 62 / 118
// A token costs 5 ns and its adapter's bytes at 8 TB/s (the L2 has most).  Tokens have their own clusters where that is 13 us at most, and
// where there are adapters for every second token at least up to eight times as much: with that many loaded, tokens are likely
// those of many requests, a batch of single tokens.  That is a guess, wrong both ways (2688 -> 5376, us, this rule / the other form): 512
// tokens of one request with 256 adapters loaded, rank 64, 66 / 12, rank 16, 22 / 11; 512 tokens of 64 requests mixed, rank 64, 159 / 93 at
// most (what as many different adapters take), rank 16, 124 / 29 at most.
inline bool token_form(size_t tokens, size_t n, size_t k, size_t rank, size_t adapters) {
    const double ns = double(tokens) * (5.0 + 2.0 * double(rank) * double(n + k) / 8000.0);
    return ns <= 13e3 || (tokens <= 2 * adapters && ns <= 104e3);
}
// CTAs of a token's cluster: with them all, two for each SM at most, and 32 KB of adapter at least for each
inline int token_ctas(size_t tokens, size_t n, size_t k, size_t rank, size_t sms) {
    int c = 1;
    while (c < 8 && tokens * c * 2 <= 2 * sms && rank * (n + k) * 2 >= size_t(c) * 2 * 32768 * 7 / 8) c *= 2;
    return c;
}

// a token's S, high and low
inline size_t sums_bytes(size_t tokens, size_t rank) { return up(tokens * padded_rank(rank) * 4, 256); }
inline size_t adapter_workspace(size_t tokens, size_t n, size_t k, size_t rank, size_t adapters) {
    return token_form(tokens, n, k, rank, adapters) ? 0 : sums_bytes(tokens, rank) + up(tokens * sizeof(float), 256);
}

template <int DT, int RT>
int launch_tiles(AdapterArgs& a, cudaStream_t stream) {
    const size_t tiles = ceil_div(a.tokens, kTileTokens), chunks = ceil_div(a.k, 64), blocks = ceil_div(a.n, kTileBlock);
    AdapterMaps m = {};
    TRY(make_map(m.x, a.x, 2, a.k, a.tokens, a.ldx * 2, kTileTokens));
    TRY(make_map(m.a, a.a, 2, a.k, size_t(a.adapters) * a.rank, size_t(a.k) * 2, 16 * RT));
    TRY(make_map(m.b, a.b, 2, a.rank, size_t(a.adapters) * a.n, size_t(a.rank) * 2, kTileBlock));
    TRY(make_map(m.y, a.y, 2, a.n, a.tokens, a.ldy * 2, kTileTokens));
    TRY(make_map(m.out, a.out, 2, std::max(8, a.n & ~7), a.tokens, a.ldo * 2, 32));      // of less than 8 columns nothing is stored
    int clusters[9];
    TRY(resident_clusters(clusters));
    // Whole waves of clusters.  ns: a cluster's start and the exchange of sums; chunks of x and blocks of y, which take longer where many
    // CTAs read and write at one time.  Clusters of one size and another, 2688 -> 5376, rank 64, us: 1024 tokens 18 of 6 or 8, two for
    // each tile, 21 of 6, 26 of 4, 40 of 2; 4096 tokens 30 of 4, 33 of 3, 42 of 2; 8192 tokens 48 of 2, 60 of 3, 74 of 1.
    size_t least = ~size_t(0);
    for (size_t c = 1; c <= 8; ++c)
        for (size_t copies = 1; copies == 1 || (copies <= 8 && copies * c <= blocks && tiles * copies <= size_t(clusters[c])); ++copies) {
            const size_t busy = std::min(tiles * copies, size_t(clusters[c])) * c;
            const size_t chunk = std::max<size_t>(200, 27 * busy / 10), block = std::max<size_t>(1300, 25 * busy / 2);
            const size_t cost = ceil_div(tiles * copies, clusters[c]) *
                                (5000 + ceil_div(chunks, c) * chunk + ceil_div(blocks, c * copies) * block);
            if (cost < least) {
                least = cost;
                a.ctas = int(c);
                a.copies = int(copies);
            }
        }
    m.p = a;
    return launch(adapter_tiles_kernel<DT, RT>, dim3(unsigned(tiles * a.copies * a.ctas)), kTileAdapterThreads, TileRoom<RT>::BYTES,
                  unsigned(a.ctas), m, stream, true);
}

template <int DT, int RT>
int launch_adapters(AdapterArgs& a, bool vec, int sms, cudaStream_t stream) {
    if (token_form(a.tokens, a.n, a.k, a.rank, a.adapters)) {
        a.ctas = token_ctas(a.tokens, a.n, a.k, a.rank, sms);
        return launch(vec ? adapter_token_kernel<DT, RT, true> : adapter_token_kernel<DT, RT, false>, dim3(unsigned(a.tokens) * a.ctas),
                      kAdapterThreads, 0, unsigned(a.ctas), a, stream);
    }
    if (a.tiles) return launch_tiles<DT, RT>(a, stream);
    // two CTAs run on an SM (of more than 64 ranks one, for their shared memory): where there are few tiles, up to eight share one
    const size_t tiles = ceil_div(a.tokens, kDownTokens);
    a.ctas = 1;
    while (a.ctas < 8 && tiles * a.ctas * 2 <= size_t(2 * sms)) a.ctas *= 2;
    TRY(launch(adapter_down_kernel<DT, RT>, dim3(unsigned(tiles * a.ctas)), kAdapterThreads, kDownSmem<RT>, unsigned(a.ctas), a, stream, true));
    // four CTAs run on an SM at one time (of more than 64 ranks two); twice as many, so that a tile with two adapters holds up less
    const size_t up_tiles = ceil_div(a.tokens, kUpTokens), all = ceil_div(a.n, kUpFeatures);
    const size_t parts = std::max<size_t>(1, std::min(size_t(8 * sms) / up_tiles, ceil_div(all, 2)));
    a.blocks = int(ceil_div(all, parts));
    return launch(adapter_up_kernel<DT, RT>, dim3(unsigned(up_tiles), unsigned(ceil_div(all, a.blocks))), 32 * kUpWarps, kUpSmem<RT>, 1, a, stream,
                  true);
}
template <int DT>
int launch_adapters(AdapterArgs& a, bool vec, int sms, cudaStream_t stream) {
    if (a.rank <= 16) return launch_adapters<DT, 1>(a, vec, sms, stream);
    if (a.rank <= 32) return launch_adapters<DT, 2>(a, vec, sms, stream);
    if (a.rank <= 64) return launch_adapters<DT, 4>(a, vec, sms, stream);
    return launch_adapters<DT, 8>(a, vec, sms, stream);
}

}  // namespace

namespace equarx {
cudaError_t adapters_give_up(uint32_t polls) {
    tc::give_up_kernel<tc::kAdapterWaits><<<1, 64>>>(polls);
    return cudaGetLastError();
}
cudaError_t adapters_gave_up(uint32_t& seen) {
    const uint32_t zero = 0;
    cudaError_t e = cudaMemcpyFromSymbol(&seen, tc::g_gave_up, sizeof(seen));
    if (e == cudaSuccess && seen) e = cudaMemcpyToSymbol(tc::g_gave_up, &zero, sizeof(zero));
    return e;
}
}  // namespace equarx

extern "C" {

size_t equarx_add_adapters_workspace_bytes(size_t tokens, size_t n, size_t k, size_t rank, size_t adapters) {
    if (tokens > kMaxDim || bad_dim(n) || bad_dim(k) || rank == 0 || rank > kMaxRank || adapters > kMaxDim) return 0;
    return adapter_workspace(tokens, n, k, rank, adapters);
}

int equarx_add_adapters(const void* y, size_t ldy, const void* x, size_t ldx, const void* a, const void* b, const int32_t* index,
                        const float* scale, int dtype, size_t tokens, size_t n, size_t k, size_t rank, size_t adapters, void* out,
                        size_t ldo, void* workspace, size_t workspace_bytes, equarx_stream_t stream) {
    if (!is_16bit(dtype)) return EQUARX_ERR_FORMAT;
    if (tokens > kMaxDim || bad_dim(n) || bad_dim(k) || rank == 0 || rank > kMaxRank || adapters > kMaxDim || bad_ld(ldy, n) ||
        bad_ld(ldx, k) || bad_ld(ldo, n))
        return EQUARX_ERR_COUNT;
    if (tokens == 0) return EQUARX_OK;
    const size_t need = adapter_workspace(tokens, n, k, rank, adapters);
    if (!y || !x || !index || !out || (adapters && (!a || !b)) || (need && !workspace)) return EQUARX_ERR_NULL;
    if (workspace_bytes < need) return EQUARX_ERR_WORKSPACE;
    for (const void* p : {y, x, a, b, static_cast<const void*>(out)})
        if (!aligned(p, 2)) return EQUARX_ERR_ALIGN;
    if (!aligned(index, 4) || !aligned(scale, 4) || !aligned(workspace, 16)) return EQUARX_ERR_ALIGN;
    const Span o = matrix(out, tokens, n, ldo, 2);
    // out may be y: each element is read before the same thread writes it
    const Span ys = matrix(y, tokens, n, ldy, 2), ws{need ? workspace : nullptr, need};
    if ((!(out == y && (ldo == ldy || tokens == 1)) && overlap(o, ys)) || overlap(ws, ys)) return EQUARX_ERR_ALIAS;
    TRY(check_overlap({matrix(x, tokens, k, ldx, 2), Span{a, adapters * rank * k * 2}, Span{b, adapters * rank * n * 2},
                       Span{index, tokens * 4}, Span{scale, adapters * 4}},
                      {o, ws}));
    AdapterArgs p = {};
    p.y = y;
    p.x = x;
    p.a = a;
    p.b = b;
    p.index = index;
    p.scale = scale;
    p.out = out;
    p.s = static_cast<uint16_t*>(workspace);
    p.back = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + sums_bytes(tokens, rank));
    p.ldy = ldy;
    p.ldx = ldx;
    p.ldo = ldo;
    p.tokens = int(tokens);
    p.k = int(k);
    p.n = int(n);
    p.rank = int(rank);
    p.adapters = int(adapters);
    int sms;
    TRY(current_device(sms));
    // rows that start on multiples of 16 bytes; TMA counts the rows of all adapters together
    const bool vec = k % 8 == 0 && rank % 8 == 0 && aligned(a, 16) && aligned(b, 16) && unit_of(x, ldx, 2) >= 16;
    p.tiles = vec && unit_of(y, ldy, 2) >= 16 && unit_of(out, ldo, 2) >= 16 && adapters && adapters * rank <= size_t(INT32_MAX) &&
              adapters * n <= size_t(INT32_MAX);
    return dtype == EQUARX_BF16 ? launch_adapters<kBf16>(p, vec, sms, stream) : launch_adapters<kFp16>(p, vec, sms, stream);
}

}  // extern "C"
