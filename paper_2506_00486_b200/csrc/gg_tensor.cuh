// Tensor cores, tensor memory and tensor copies of sm_100a: the instructions that the product kernels are built from.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace gg {

__device__ __forceinline__ uint32_t shared_address(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

// ---- barriers in shared memory
__device__ __forceinline__ void barrier_init(uint32_t bar, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void barrier_expect(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// (an address of the cluster's shared memory, such as peer_address gives.  What it says is that the caller has read tensor memory, and
// tmem_before_sync orders that; a release of the whole cluster would also wait for the caller's stores to memory, which took half of
// the time of a product that is mostly stores)
__device__ __forceinline__ void barrier_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ bool barrier_test(uint32_t bar, uint32_t parity)
{
    uint32_t done;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0;
}
// Every wait ends: after so many polls, of half a microsecond or so, the caller gives up.
__device__ __forceinline__ bool barrier_wait(uint32_t bar, uint32_t parity, uint32_t polls)
{
    for (uint32_t i = 0; i < polls; ++i)
        if (barrier_test(bar, parity)) return true;
    return false;
}
// The address of the same variable in CTA `rank` of the cluster.
__device__ __forceinline__ uint32_t peer_address(uint32_t at, uint32_t rank)
{
    uint32_t d;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(d) : "r"(at), "r"(rank));
    return d;
}
__device__ __forceinline__ void cluster_store(uint32_t at, uint32_t value) { asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(at), "r"(value) : "memory"); }
__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// One lane of a whole warp, always the same.
__device__ __forceinline__ bool elect_lane()
{
    uint32_t is;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(is));
    return is != 0;
}
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// ---- tensor copies into shared memory; kCtas 2: the barrier may be that of the pair's other CTA
template <int kCtas>
__device__ __forceinline__ void tensor_copy(uint32_t to, const void *map, int x, int y, uint32_t bar)
{
    if constexpr (kCtas == 1)
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(to), "l"(map), "r"(x),
                     "r"(y), "r"(bar) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(to),
                     "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
__device__ __forceinline__ void prefetch_map(const void *map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }

// ---- tensor memory
template <int kCtas>
__device__ __forceinline__ void tmem_alloc(uint32_t to, uint32_t columns)
{
    if constexpr (kCtas == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(to), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    } else {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(to), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    }
}
template <int kCtas>
__device__ __forceinline__ void tmem_free(uint32_t at, uint32_t columns)
{
    if constexpr (kCtas == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns));
    else asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns));
}
__device__ __forceinline__ void tmem_before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// 32 columns of the warp's 32 lanes: a thread gets those of its own lane.
__device__ __forceinline__ void tmem_read(uint32_t at, float (&v)[32])
{
    uint32_t r[32];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, "
                 "%30, %31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
                   "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
                   "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]),
                   "=r"(r[31])
                 : "r"(at) : "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}
// 16 columns.
__device__ __forceinline__ void tmem_read(uint32_t at, float (&v)[16])
{
    uint32_t r[16];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
                   "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(at) : "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}
// The registers of tmem_read hold their values from here on.
__device__ __forceinline__ void tmem_read_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// ---- products
// bf16 operands, fp32 sums; kAT, kBT: the operand lies with the rows of the product (not the summed axis) side by side; n: a
// multiple of 16 up to 256
template <int kM, bool kAT, bool kBT>
__device__ __forceinline__ uint32_t product_shape(int n)
{
    return 1u << 4 | 1u << 7 | 1u << 10 | (uint32_t)kAT << 15 | (uint32_t)kBT << 16 | (uint32_t)(n >> 3) << 17 | (uint32_t)(kM >> 4) << 24;
}
// A tile in shared memory as 128-byte rows in the 128-byte swizzle, at a multiple of 1024 bytes.  Along the summed axis: a row
// is 64 summed elements of one product row, 8 rows lie 1024 bytes from the next 8.  Otherwise: a row is 64 product rows of
// one summed element, 8 summed elements lie 1024 bytes from the next 8, and 64 product rows 8192 bytes from the next 64.
template <bool kT>
__device__ __forceinline__ uint64_t tile_descriptor(uint32_t at)
{
    constexpr uint64_t lead = kT ? 8192 >> 4 : 1, stride = 1024 >> 4;
    return (uint64_t)(at >> 4 & 0x3FFF) | lead << 16 | stride << 32 | 1ull << 46 | 2ull << 61;
}
// (the 16 summed elements of one instruction, in units of 16 bytes)
template <bool kT> __host__ __device__ constexpr uint64_t tile_step() { return kT ? 2048 >> 4 : 32 >> 4; }

template <int kCtas>
__device__ __forceinline__ void product_issue(uint32_t to, uint64_t a, uint64_t b, uint32_t shape, bool add)
{
    if constexpr (kCtas == 1)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(to), "l"(a), "l"(b),
                     "r"(shape), "r"((uint32_t)add) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(to), "l"(a), "l"(b),
                     "r"(shape), "r"((uint32_t)add) : "memory");
}
// Arrives at the barrier (of both CTAs of a pair) once the products issued so far are done.
template <int kCtas>
__device__ __forceinline__ void product_commit(uint32_t bar)
{
    if constexpr (kCtas == 1)
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3) : "memory");
}

}  // namespace gg
