// blackwell.cuh -- the sm_103a instructions that the weight gradient, the orthogonal
// update and the bulk copies are made of:
// mbarriers, tensor copies (TMA), tensor memory and tcgen05 products.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>

#include <atomic>
#include <climits>
#include <cstdint>

namespace {

__device__ __forceinline__ uint32_t shared_address(const void* p) {
    return static_cast<uint32_t>(__cvta_generic_to_shared(p));
}

// One lane of a whole warp, the same every time.
__device__ __forceinline__ bool elected() {
    uint32_t is;
    asm volatile(
        "{\n"
        ".reg .pred p;\n"
        "elect.sync _|p, 0xffffffff;\n"
        "selp.u32 %0, 1, 0, p;\n"
        "}\n"
        : "=r"(is));
    return is != 0;
}

// ------------------------------------------------------------------ mbarriers

__device__ __forceinline__ void barrier_init(uint32_t bar, uint32_t arrivals) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(arrivals) : "memory");
}

__device__ __forceinline__ void barriers_ready() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }

// The address of the same place in the shared memory of CTA `rank` of the cluster.
__device__ __forceinline__ uint32_t in_cta(uint32_t at, uint32_t rank) {
    uint32_t to;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(at), "r"(rank));
    return to;
}

__device__ __forceinline__ void barrier_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}

// The same at a barrier of another CTA (an address from in_cta).  Not a release to
// the cluster, which would wait for the whole SM's traffic (2,000 cycles measured):
// it says that writes to shared memory have reached it, as fence_async and a local
// barrier have made sure before.
__device__ __forceinline__ void barrier_arrive_there(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

__device__ __forceinline__ void barrier_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}

__device__ __forceinline__ bool barrier_passed(uint32_t bar, uint32_t parity) {
    uint32_t done;
    asm volatile(
        "{\n"
        ".reg .pred p;\n"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n"
        "selp.u32 %0, 1, 0, p;\n"
        "}\n"
        : "=r"(done)
        : "r"(bar), "r"(parity)
        : "memory");
    return done != 0;
}

constexpr long long kPatience = 2000000000ll;  // cycles, about a second

// Waits for the phase of `parity` to end; false after about a second, when the
// caller gives up, so that no wait can hold the GPU.  One thread.
__device__ __forceinline__ bool barrier_wait(uint32_t bar, uint32_t parity) {
    if (barrier_passed(bar, parity)) return true;
    const long long start = clock64();
    do {
        if (barrier_passed(bar, parity)) return true;
    } while (clock64() - start < kPatience);
    return false;
}

// The same for all lanes of a warp, which go on or give up together.
__device__ __forceinline__ bool barrier_wait_warp(uint32_t bar, uint32_t parity) {
    if (__all_sync(0xffffffffu, barrier_passed(bar, parity))) return true;
    const long long start = clock64();
    do {
        if (__all_sync(0xffffffffu, barrier_passed(bar, parity))) return true;
    } while (__all_sync(0xffffffffu, clock64() - start < kPatience));
    return false;
}

// What goes through kStages places of shared memory by copies, number after number from 0 on: a
// barrier a place (one arrival, that of the thread that asks), and the phase in which a number lands.
// In number i's turn the readers of number i - kBehind are done with its place, and one thread asks
// for what comes there next.
template <int kStages, int kBehind>
struct Numbers {
    uint32_t bars;
    int lost = INT_MAX;  // the first number that was waited for in vain
    __device__ __forceinline__ static int place(int i) { return i % kStages; }
    __device__ __forceinline__ uint32_t bar(int i) const { return bars + 8 * place(i); }
    __device__ __forceinline__ static uint32_t parity(int i) { return i / kStages & 1; }
    // Number i is there; false from the first wait on that ran out, after about a second.  All lanes
    // of a warp.
    __device__ __forceinline__ bool wait(int i) {
        if (lost == INT_MAX && !barrier_wait_warp(bar(i), parity(i))) lost = i;
        return lost == INT_MAX;
    }
    // The number to ask for in number i's turn, if there are as many, and whether it may be (the first
    // kStages are asked for before).  Not once a wait has run out: its phase has not ended, and
    // takes no second arrival.
    __device__ __forceinline__ static int next(int i) { return i - kBehind + kStages; }
    __device__ __forceinline__ bool asks(int i) const { return i >= kBehind && lost == INT_MAX; }
    // Before the end: none of the copies is in flight (about a second each at most).  They have been
    // waited for before, unless a wait ran out.  The thread that asks.
    __device__ __forceinline__ void drain(int count) const {
        const int asked = lost == INT_MAX ? count : min(count, max(lost - kBehind, 0) + kStages);
        for (int i = max(0, asked - kStages); i < asked; ++i) barrier_wait(bar(i), parity(i));
    }
};

// A count in shared memory that one thread raises, and another's wait until it is `least` or
// more (false after about a second): what the one has seen before, the other sees after.
__device__ __forceinline__ void count_store(uint32_t at, int count) {
    asm volatile("st.release.cta.shared::cta.s32 [%0], %1;" ::"r"(at), "r"(count) : "memory");
}

__device__ __forceinline__ bool count_wait(uint32_t at, int least) {
    const long long start = clock64();
    do {
        int count;
        asm volatile("ld.acquire.cta.shared::cta.s32 %0, [%1];" : "=r"(count) : "r"(at) : "memory");
        if (count >= least) return true;
    } while (clock64() - start < kPatience);
    return false;
}

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

// All threads of the cluster's CTAs.
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Registers a thread from here on; all warps of a warpgroup.  The warpgroups'
// shares may not pass what the block was launched with.
template <int kRegisters>
__device__ __forceinline__ void more_registers() {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegisters));
}
template <int kRegisters>
__device__ __forceinline__ void fewer_registers() {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegisters));
}

// ------------------------------------------------------------------- copies

// Box at (x, y, z) of the tensor to shared memory; its bytes count towards `bar`.
__device__ __forceinline__ void copy_box(uint32_t to, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(to),
        "l"(map), "r"(bar), "r"(x), "r"(y), "r"(z)
        : "memory");
}

__device__ __forceinline__ void copy_box(uint32_t to, const CUtensorMap* map, int x, int y, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(to),
        "l"(map), "r"(bar), "r"(x), "r"(y)
        : "memory");
}

// `bytes` next to one another, all three a multiple of 16 bytes.
__device__ __forceinline__ void copy_row(uint32_t to, const void* from, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(to), "l"(from),
                 "r"(bytes), "r"(bar)
                 : "memory");
}

// Orders this thread's writes to shared memory before later reads by copies and
// tensor cores.
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// ----------------------------------------------------- tensor memory and products

// The products are those of a pair of CTAs (a cluster of two): CTA r brings rows
// 128 r .. of A and columns kN / 2 r .. of B in its shared memory and gets rows
// 128 r .. of D in its tensor memory.  With kCtas = 1 a CTA works alone, on 128 rows.

// One warp of each CTA, all lanes; the address goes to shared memory.
template <int kColumns, int kCtas = 2>
__device__ __forceinline__ void tensor_alloc(uint32_t to) {
    if constexpr (kCtas == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(to), "n"(kColumns)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    } else {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(to), "n"(kColumns)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
}

template <int kColumns, int kCtas = 2>
__device__ __forceinline__ void tensor_free(uint32_t at) {
    if constexpr (kCtas == 2)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(at), "n"(kColumns));
    else
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "n"(kColumns));
}

__device__ __forceinline__ void tensor_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tensor_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// Operand in shared memory whose fastest axis is M (or N), in the 128-byte
// swizzle: groups of 64 such elements x 8 steps of K are 1024-byte atoms,
// `next_k` bytes apart along K and `next_mn` along M or N.
__device__ __forceinline__ uint64_t operand(uint32_t at, uint32_t next_mn, uint32_t next_k) {
    return static_cast<uint64_t>((at & 0x3FFFFu) >> 4) | static_cast<uint64_t>(next_mn >> 4) << 16 |
           static_cast<uint64_t>(next_k >> 4) << 32 | uint64_t(1) << 46 | uint64_t(2) << 61;
}

// bf16 x bf16 to fp32, both operands with M and N fastest.
template <int kM, int kN>
constexpr uint32_t kProductKind =
    1u << 4 | 1u << 7 | 1u << 10 | 1u << 15 | 1u << 16 | uint32_t(kN / 8) << 17 | uint32_t(kM / 16) << 24;

// D (+)= A B over 16 steps of K; one thread of CTA 0.
template <int kCtas = 2>
__device__ __forceinline__ void product(uint32_t d, uint64_t a, uint64_t b, uint32_t kind, bool add) {
    if constexpr (kCtas == 2)
        asm volatile(
            "{\n"
            ".reg .pred p;\n"
            "setp.ne.u32 p, %4, 0;\n"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n"
            "}\n" ::"r"(d),
            "l"(a), "l"(b), "r"(kind), "r"(static_cast<uint32_t>(add))
            : "memory");
    else
        asm volatile(
            "{\n"
            ".reg .pred p;\n"
            "setp.ne.u32 p, %4, 0;\n"
            "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n"
            "}\n" ::"r"(d),
            "l"(a), "l"(b), "r"(kind), "r"(static_cast<uint32_t>(add))
            : "memory");
}

// The thread's products so far arrive at `bar` (of both CTAs) when they are done.
template <int kCtas = 2>
__device__ __forceinline__ void products_arrive(uint32_t bar) {
    if constexpr (kCtas == 2)
        asm volatile(
            "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
            "h"(static_cast<uint16_t>(3))
            : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// ------------------------------------------------- kernels launched before their time

// A kernel launched as a programmatic dependent starts while the one before it still runs:
// nothing of that one's may be read or overwritten before this.
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// From here on the next one may start.
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// 16 columns of the warp's 32 lanes: v[c] is this lane's column c.
__device__ __forceinline__ void tensor_load(uint32_t at, float (&v)[16]) {
    uint32_t r[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(at)
        : "memory");
#pragma unroll
    for (int c = 0; c < 16; ++c) v[c] = __uint_as_float(r[c]);
}

// ------------------------------------------------------------------ on the host

using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                            const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                            CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// The driver's cuTensorMapEncodeTiled, NULL where it has none.
inline Encode encoder() {
    static const Encode encode = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) !=
                cudaSuccess ||
            found != cudaDriverEntryPointSuccess) {
            (void)cudaGetLastError();
            f = nullptr;
        }
        return reinterpret_cast<Encode>(f);
    }();
    return encode;
}

// Lets Kernel use its shared memory, once per device.
template <auto Kernel>
bool allow_shared(int bytes) {
    static std::atomic<bool> set[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return false;
    if (dev < 64 && set[dev].load()) return true;
    if (cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) {
        (void)cudaGetLastError();
        return false;
    }
    if (dev < 64) set[dev].store(true);
    return true;
}

}  // namespace
