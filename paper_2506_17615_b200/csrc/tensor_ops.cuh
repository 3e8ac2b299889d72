// Blackwell (sm_100a) building blocks of the feed-forward kernels: mbarriers with a bounded wait,
// TMA loads, tensor memory, the fifth-generation tensor-core instructions and their descriptors.
#pragma once
#include <cstdint>
#include <cuda.h>
#include <cuda_runtime.h>

namespace equarx {
namespace tc {

// ---------------------------------------------------------------- shared memory addresses, election
__device__ __forceinline__ uint32_t smem_addr(const void* p) { return uint32_t(__cvta_generic_to_shared(p)); }

// ---------------------------------------------------------------- mbarriers
__device__ __forceinline__ void barrier_init(uint32_t bar, uint32_t arrivals) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(arrivals) : "memory");
}
__device__ __forceinline__ void barrier_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool barrier_try(uint32_t bar, uint32_t parity) {
    uint32_t done;
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
        : "=r"(done)
        : "r"(bar), "r"(parity)
        : "memory");
    return done != 0;
}
// the same for arrivals of barrier_arrive_pair; fence_after orders what follows
__device__ __forceinline__ bool barrier_try_pair(uint32_t bar, uint32_t parity) {
    uint32_t done;
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.try_wait.parity.relaxed.cluster.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}"
        : "=r"(done)
        : "r"(bar), "r"(parity)
        : "memory");
    return done != 0;
}

// The waits are on copies and products of this CTA and, in the tile kernel, of the other CTA of the pair, so they end by
// themselves; the limit is there so that a mistake becomes a status instead of a kernel that never returns.  A poll of
// a barrier on which nothing happens lasts 4.0 us (measured), 2^18 of them 1.05 s, where a stage of the
// reduction takes about 1 us.  A wait that spans many stages asks for more.  A CTA that gives up takes all its warps
// out; the other one of its pair, which waits in vain then, comes to its own limit.
constexpr uint32_t kWaitLimit = 1u << 18;
// for a wait on all products of a tile: 16 us more for each stage
__device__ __forceinline__ uint32_t wait_limit(int stages) { return kWaitLimit + 4 * uint32_t(stages); }

// counts the waits that gave up on this device since the library was loaded
__device__ uint32_t g_gave_up = 0;

// false: this wait, or another one of this CTA, gave up (then `abort` is set and every role leaves)
template <bool PAIR = false>
__device__ __forceinline__ bool barrier_wait(uint32_t bar, uint32_t parity, volatile uint32_t* abort, uint32_t limit) {
    auto done = [&] { return PAIR ? barrier_try_pair(bar, parity) : barrier_try(bar, parity); };
    if (done()) return true;
    for (uint32_t i = 0; i < limit; ++i) {
        if (done()) return true;
        if (*abort) return false;
    }
    *abort = 1;
    atomicAdd(&g_gave_up, 1u);
    return false;
}
// the same without the early exit: for what is in flight when a CTA has already given up
__device__ __forceinline__ void barrier_drain(uint32_t bar, uint32_t parity) {
    for (uint32_t i = 0; i < kWaitLimit; ++i)
        if (barrier_try(bar, parity)) return;
}

__device__ __forceinline__ void fence_barrier_init() {
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
}
__device__ __forceinline__ void st_shared_v4(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ void ld_shared_v4(uint32_t addr, uint32_t (&v)[4]) {
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t ld_shared_u32(uint32_t addr) {
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void ld_shared_v2(uint32_t addr, uint32_t& a, uint32_t& b) {
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(a), "=r"(b) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t ld_shared_u16(uint32_t addr) {
    uint16_t v;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void fence_async_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// the same for any memory, another CTA's too
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async;" ::: "memory"); }

// ---------------------------------------------------------------- copies of one thread
// 16 bytes to shared memory, the last 16 - `bytes` of them zeros; both addresses are multiples of 16
__device__ __forceinline__ void copy_async_16(uint32_t dst, const void* src, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// at most PENDING of this thread's groups are still on their way
template <int PENDING>
__device__ __forceinline__ void copy_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(PENDING) : "memory"); }

// ---------------------------------------------------------------- clusters, dependent launches
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// the address of the same shared variable in another CTA of the cluster
__device__ __forceinline__ uint32_t peer_addr(uint32_t addr, uint32_t rank) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(addr), "r"(rank));
    return a;
}
// Says, to a barrier of either CTA of a pair, that this thread's tensor-memory loads are done (fence_before orders
// them before it).  At cluster scope, since the waiter may be in the other CTA, and relaxed: no other memory is passed
// on, and a release at this scope would hold the arrival back by about 1000 cycles.
__device__ __forceinline__ void barrier_arrive_pair(uint32_t cluster_bar) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
__device__ __forceinline__ void st_cluster_f32(uint32_t cluster_addr, float v) {
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(cluster_addr), "f"(v) : "memory");
}
__device__ __forceinline__ void st_cluster_v2(uint32_t cluster_addr, uint32_t a, uint32_t b) {
    asm volatile("st.shared::cluster.v2.b32 [%0], {%1, %2};" ::"r"(cluster_addr), "r"(a), "r"(b) : "memory");
}
__device__ __forceinline__ float ld_cluster_f32(uint32_t cluster_addr) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(cluster_addr) : "memory");
    return v;
}
__device__ __forceinline__ float4 ld_cluster_f32x4(uint32_t cluster_addr) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(cluster_addr) : "memory");
    return v;
}
__device__ __forceinline__ void max_cluster_u32(uint32_t cluster_addr, uint32_t v) {
    asm volatile("red.shared::cluster.max.u32 [%0], %1;" ::"r"(cluster_addr), "r"(v) : "memory");
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void grid_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// A kernel's place in a sequence of dependent launches.
//   kOrdered    reads what the launch before wrote: waits for it before anything else
//   kForwarding the same, and lets the next launch begin only then, so that the next one may count on
//               everything up to the launch before this one
//   kBeside     behind a kForwarding launch whose outputs it does not touch: runs beside it and waits for it
//               only at its end, so that what follows still finds both complete
enum Order { kOrdered = 0, kForwarding = 1, kBeside = 2 };
__device__ __forceinline__ void grid_launch() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

__device__ __forceinline__ void grid_begin(int order) {
    if (order != kForwarding) grid_launch();
    if (order != kBeside) grid_wait();
    if (order == kForwarding) grid_launch();
}
__device__ __forceinline__ void grid_end(int order) {
    if (order == kBeside) grid_wait();
}

// ---------------------------------------------------------------- instructions of one thread
// Loads and products are issued by one lane of a warp whose 32 lanes run the loop together: with uniform
// control flow the addresses and descriptors stay in uniform registers, where these instructions want
// them.  (A loop run by lane 0 alone took 63 cycles for each instruction it issued, more than the
// tensor cores need for a 256 x 256 x 16 product between them.)
#define EQUARX_ELECT "{\n .reg .pred elected;\n elect.sync _|elected, 0xFFFFFFFF;\n @elected "

// a value that all lanes share, as one the compiler knows to be shared
template <typename T>
__device__ __forceinline__ T uniform(T v) { return __shfl_sync(0xFFFFFFFFu, v, 0); }

// Every wait of a kernel is a whole warp's, which goes on or leaves together: false in every lane as soon as one
// lane's wait gave up
template <bool PAIR = false>
__device__ __forceinline__ bool barrier_wait_warp(uint32_t bar, uint32_t parity, volatile uint32_t* abort,
                                                  uint32_t limit = kWaitLimit) {
    return __all_sync(0xFFFFFFFFu, barrier_wait<PAIR>(bar, parity, abort, limit));
}
// whether a wait of this CTA has given up; one answer for the warp, which may have to issue instructions together
__device__ __forceinline__ bool gave_up_warp(volatile uint32_t* abort) { return __any_sync(0xFFFFFFFFu, *abort != 0); }
__device__ __forceinline__ void barrier_expect_warp(uint32_t bar, uint32_t bytes) {
    asm volatile(EQUARX_ELECT "mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n}" ::"r"(bar), "r"(bytes) : "memory");
}

// ---------------------------------------------------------------- TMA
// 2-D tile load; x (the contiguous coordinate) always is a multiple of 16 bytes here.
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    asm volatile(EQUARX_ELECT
                 "cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n}" ::"r"(
                     dst),
                 "l"(map), "r"(x), "r"(y), "r"(bar)
                 : "memory");
}
// the same for a pair of CTAs that work on one tile: into this CTA's memory, counted on a barrier of
// either CTA (a shared::cluster address); no multicast
__device__ __forceinline__ void tma_load_2d_pair(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t cluster_bar) {
    asm volatile(EQUARX_ELECT
                 "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 "
                 "[%0], [%1, {%2, %3}], [%4];\n}" ::"r"(dst),
                 "l"(map), "r"(x), "r"(y), "r"(cluster_bar)
                 : "memory");
}
// 2-D tile store; the part outside the matrix is dropped
__device__ __forceinline__ void tma_store_2d(const CUtensorMap* map, uint32_t src, int x, int y) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%2, %3}], [%1];\n"
                 "cp.async.bulk.commit_group;" ::"l"(map),
                 "r"(src), "r"(x), "r"(y)
                 : "memory");
}
// at most PENDING of this thread's stores still read shared memory
template <int PENDING>
__device__ __forceinline__ void tma_store_wait_read() {
    asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(PENDING) : "memory");
}
__device__ __forceinline__ void tma_store_wait_all() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile(EQUARX_ELECT "cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];\n}" ::"r"(dst),
                 "l"(src), "r"(bytes), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}

// ---------------------------------------------------------------- tensor memory
// CTAS is 1 or 2 throughout a kernel: with 2 the pair of CTAs of a cluster works on one tile, one of
// them issues the products and copies for both.
template <int CTAS>
__device__ __forceinline__ void tmem_alloc(uint32_t smem_dst, uint32_t columns) {
    if constexpr (CTAS == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_dst), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    } else {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_dst), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
}
template <int CTAS>
__device__ __forceinline__ void tmem_free(uint32_t base, uint32_t columns) {
    if constexpr (CTAS == 1)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(columns) : "memory");
    else
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(columns) : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_loads() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// 32 lanes x 32 columns of 32 bits: thread t of the warp gets lane t's 32 columns
__device__ __forceinline__ void tmem_load32(uint32_t addr, uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr)
        : "memory");
}
__device__ __forceinline__ void tmem_load16(uint32_t addr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr)
        : "memory");
}

// ---------------------------------------------------------------- matrix products
// Shared-memory matrix descriptor: 128-byte swizzled rows.  Operands whose reduction axis is contiguous
// ("K-major"): atoms of 8 rows x 128 bytes, `stride` from one group of 8 rows to the next; the leading
// offset is not used.  Operands whose other axis is contiguous ("MN-major"): atoms of 64 elements (128
// bytes) x 8 steps of the reduction axis, `stride` from one group of 8 steps to the next and `leading`
// from one group of 64 elements to the next.
// Only the low word (address and leading offset) changes; the high one is the stride and constants.
__device__ __forceinline__ uint32_t swizzled_desc(uint32_t addr, uint32_t leading) {
    return ((addr >> 4) & 0x3FFF) | (leading >> 4) << 16;
}
constexpr uint32_t kSwizzledHigh = (1024 >> 4) | 1u << 14 | 2u << 29;
// 32 rows x 16 bytes, unswizzled, 128 bytes for each 8 rows: one scale tile
__device__ __forceinline__ uint32_t scale_desc(uint32_t addr) { return (addr >> 4) & 0x3FFF; }
constexpr uint32_t kScaleHigh = (128 >> 4) | 1u << 14;

// Instruction descriptors.  16-bit operands, fp32 accumulation, m x n (m = 128 for each CTA):
__host__ __device__ constexpr uint32_t desc_16bit(bool bf16, bool a_mn, bool b_mn, uint32_t m, uint32_t n) {
    return (1u << 4) | (uint32_t(bf16) << 7) | (uint32_t(bf16) << 10) | (uint32_t(a_mn) << 15) | (uint32_t(b_mn) << 16) |
           ((n >> 3) << 17) | ((m >> 4) << 24);
}
// block-scaled E2M1 operands, fp32 accumulation; `which` selects the scale bytes (0 or 2) of a 32-bit
// cell when one step of the reduction uses only half of them
__host__ __device__ constexpr uint32_t desc_fp4(bool e8m0, uint32_t m, uint32_t n, uint32_t which) {
    return (which << 4) | (1u << 7) | (1u << 10) | ((n >> 3) << 17) | (uint32_t(e8m0) << 23) | ((m >> 7) << 27) | (which << 29);
}
// block-scaled E4M3 operands with E8M0 scales; `which` selects the scale byte of a 32-bit cell, one for each 32 elements
__host__ __device__ constexpr uint32_t desc_fp8(uint32_t m, uint32_t n, uint32_t which) {
    return (which << 4) | ((n >> 3) << 17) | (1u << 23) | ((m >> 7) << 27) | (which << 29);
}

#define EQUARX_MMA_16BIT(GROUP)                                                                             \
    asm volatile("{\n .reg .pred elected, p;\n .reg .b64 a, b;\n mov.b64 a, {%1, %5};\n mov.b64 b, {%2, %5};\n" \
                 " setp.ne.u32 p, %4, 0;\n elect.sync _|elected, 0xFFFFFFFF;\n"                             \
                 " @elected tcgen05.mma.cta_group::" GROUP ".kind::f16 [%0], a, b, %3, p;\n}" ::"r"(d),     \
                 "r"(a), "r"(b), "r"(idesc), "r"(uint32_t(accumulate)), "n"(kSwizzledHigh)                  \
                 : "memory")
#define EQUARX_MMA_SCALED(GROUP, KIND)                                                                       \
    asm volatile("{\n .reg .pred elected, p;\n .reg .b64 a, b;\n mov.b64 a, {%1, %7};\n mov.b64 b, {%2, %7};\n" \
                 " setp.ne.u32 p, %6, 0;\n elect.sync _|elected, 0xFFFFFFFF;\n"                             \
                 " @elected tcgen05.mma.cta_group::" GROUP ".kind::" KIND " [%0], a, b, %3, [%4], [%5], p;\n}" ::"r"(d), \
                 "r"(a), "r"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(uint32_t(accumulate)), "n"(kSwizzledHigh) \
                 : "memory")

// 16 elements of the reduction axis
template <int CTAS>
__device__ __forceinline__ void mma_16bit(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool accumulate) {
    if constexpr (CTAS == 1) EQUARX_MMA_16BIT("1");
    else EQUARX_MMA_16BIT("2");
}
// 64 elements of the reduction axis; one E4M3 scale for each 16 of them (NV) or one E8M0 for each 32 (MX)
template <int CTAS, bool MX>
__device__ __forceinline__ void mma_fp4(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t sa, uint32_t sb,
                                        bool accumulate) {
    if constexpr (CTAS == 1 && MX) EQUARX_MMA_SCALED("1", "mxf4.block_scale.scale_vec::2X");
    else if constexpr (CTAS == 1) EQUARX_MMA_SCALED("1", "mxf4nvf4.block_scale.scale_vec::4X");
    else if constexpr (MX) EQUARX_MMA_SCALED("2", "mxf4.block_scale.scale_vec::2X");
    else EQUARX_MMA_SCALED("2", "mxf4nvf4.block_scale.scale_vec::4X");
}
// 32 elements of the reduction axis in 8 bits, with one E8M0 scale
template <int CTAS>
__device__ __forceinline__ void mma_fp8(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t sa, uint32_t sb,
                                        bool accumulate) {
    if constexpr (CTAS == 1) EQUARX_MMA_SCALED("1", "mxf8f6f4.block_scale.scale_vec::1X");
    else EQUARX_MMA_SCALED("2", "mxf8f6f4.block_scale.scale_vec::1X");
}
#undef EQUARX_MMA_16BIT
#undef EQUARX_MMA_SCALED
// one scale tile (128 rows x 4 scales) from shared to tensor memory, where each quarter of the lanes
// gets its own copy, as the block-scaled product wants it; with two CTAs, in each of them
template <int CTAS>
__device__ __forceinline__ void copy_scales(uint32_t tmem, uint32_t smem) {
#define EQUARX_COPY(GROUP)                                                                            \
    asm volatile("{\n .reg .pred elected;\n .reg .b64 a;\n mov.b64 a, {%1, %2};\n"                   \
                 " elect.sync _|elected, 0xFFFFFFFF;\n"                                               \
                 " @elected tcgen05.cp.cta_group::" GROUP ".32x128b.warpx4 [%0], a;\n}" ::"r"(tmem),   \
                 "r"(scale_desc(smem)), "n"(kScaleHigh)                                               \
                 : "memory")
    if constexpr (CTAS == 1) EQUARX_COPY("1");
    else EQUARX_COPY("2");
#undef EQUARX_COPY
}
// arrives on `bar` (of both CTAs, with two) when everything this warp has issued before is done
template <int CTAS>
__device__ __forceinline__ void mma_commit(uint32_t bar) {
    if constexpr (CTAS == 1)
        asm volatile(EQUARX_ELECT "tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}" ::"r"(bar)
                     : "memory");
    else
        asm volatile(EQUARX_ELECT
                     "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n}" ::"r"(bar),
                     "h"(uint16_t(3))
                     : "memory");
}

// ---------------------------------------------------------------- a wait that runs out
// For tests of what the host is told: one warp waits `polls` times on a barrier on which nobody arrives, and a second
// one, with the full limit, leaves because the first has given up.  Each source file with waits has a count, and by its number a kernel of
// this name, of its own.
enum GiveUpSource { kFeedForwardWaits = 0, kAdapterWaits = 1 };
template <int SOURCE>
__global__ void __launch_bounds__(64) give_up_kernel(uint32_t polls) {
    __shared__ uint64_t bar;
    __shared__ volatile uint32_t abort;
    const uint32_t never = smem_addr(&bar);
    if (threadIdx.x == 0) {
        barrier_init(never, 1);
        abort = 0;
    }
    __syncthreads();
    barrier_wait_warp(never, 0, &abort, threadIdx.x < 32 ? polls : kWaitLimit);
}

}  // namespace tc
}  // namespace equarx
