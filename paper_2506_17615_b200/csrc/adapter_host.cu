// C ABI of the low-rank adapters (include/equarx.h): argument checks, launches.
#include "adapter_kernels.cuh"
#include "host_common.h"

namespace {

using namespace equarx;
using namespace equarx::ff;
using namespace equarx::host;

constexpr size_t kMaxRank = 128;

// Tokens of a cluster and CTAs of it.
void plan(AdapterArgs& a, int sms) {
    a.ctas = 4;
    a.tile = 1;
    while (a.tile < kAdapterTokens && ceil_div(a.tokens, a.tile) > size_t(sms)) a.tile *= 2;
    if (a.tile == 1 && a.tokens * 8 <= 2 * sms) a.ctas = 8;
}

template <int DT, int RT>
int launch_rank(AdapterArgs& a, bool vec, cudaStream_t stream) {
    const int groups = int(ceil_div(a.tile, 8 * kAdapterGroups<RT>));
    a.split = kAdapterWarps / (groups > 2 ? 4 : groups);
    const dim3 grid(unsigned(ceil_div(a.tokens, a.tile) * a.ctas));
    const size_t smem = adapter_smem<RT>(a.tile, a.split);
    return launch(vec ? adapters_kernel<DT, RT, true> : adapters_kernel<DT, RT, false>, grid, kAdapterThreads, smem, unsigned(a.ctas), a,
                  stream);
}
template <int DT>
int launch_type(AdapterArgs& a, bool vec, cudaStream_t stream) {
    if (a.rank <= 16) return launch_rank<DT, 1>(a, vec, stream);
    if (a.rank <= 32) return launch_rank<DT, 2>(a, vec, stream);
    if (a.rank <= 64) return launch_rank<DT, 4>(a, vec, stream);
    return launch_rank<DT, 8>(a, vec, stream);
}

}  // namespace

extern "C" {

int equarx_add_adapters(const void* y, size_t ldy, const void* x, size_t ldx, const void* a, const void* b, const int32_t* index,
                        const float* scale, int dtype, size_t tokens, size_t n, size_t k, size_t rank, size_t adapters, void* out,
                        size_t ldo, equarx_stream_t stream) {
    if (!is_16bit(dtype)) return EQUARX_ERR_FORMAT;
    if (tokens > kMaxDim || bad_dim(n) || bad_dim(k) || rank == 0 || rank > kMaxRank || adapters > kMaxDim || bad_ld(ldy, n) ||
        bad_ld(ldx, k) || bad_ld(ldo, n))
        return EQUARX_ERR_COUNT;
    if (tokens == 0) return EQUARX_OK;
    if (!y || !x || !index || !out || (adapters && (!a || !b))) return EQUARX_ERR_NULL;
    for (const void* p : {y, x, a, b, static_cast<const void*>(out)})
        if (!aligned(p, 2)) return EQUARX_ERR_ALIGN;
    if (!aligned(index, 4) || !aligned(scale, 4)) return EQUARX_ERR_ALIGN;
    const Span o = matrix(out, tokens, n, ldo, 2);
    // out may be y: each element is read before the same thread writes it
    if (!(out == y && (ldo == ldy || tokens == 1)) && overlap(o, matrix(y, tokens, n, ldy, 2))) return EQUARX_ERR_ALIAS;
    TRY(check_overlap({matrix(x, tokens, k, ldx, 2), Span{a, adapters * rank * k * 2}, Span{b, adapters * rank * n * 2},
                       Span{index, tokens * 4}, Span{scale, adapters * 4}},
                      {o}));
    AdapterArgs p = {};
    p.y = y;
    p.x = x;
    p.a = a;
    p.b = b;
    p.index = index;
    p.scale = scale;
    p.out = out;
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
    plan(p, sms);
    bool vec = k % 8 == 0 && n % 8 == 0 && rank % 8 == 0 && aligned(a, 16) && aligned(b, 16);
    vec = vec && unit_of(y, ldy, 2) >= 16 && unit_of(x, ldx, 2) >= 16 && unit_of(out, ldo, 2) >= 16;
    return dtype == EQUARX_BF16 ? launch_type<kBf16>(p, vec, stream) : launch_type<kFp16>(p, vec, stream);
}

}  // extern "C"
