// What the kernels on the fifth-generation tensor cores share: barriers with bounded waits, copies of boxes, descriptors of operands and scales, the
// block-scaled product, and the host's side of the copies.
#pragma once

#include "hpsgd_ops_common.cuh"

#include <cuda.h>
#include <mutex>

namespace hpsgd {
namespace ops {
namespace {

constexpr int kLanes = 128;                // of the accumulator: rows of the operand whose rows lie on them
constexpr int kStageK = 128;               // k of a stage: one scale block, one row of the 128-byte swizzle

// ---------------------------------------------------------------------------- instructions
__device__ __forceinline__ uint32_t smem_address(const void* p) { return shared_address(p); }

__device__ __forceinline__ void barrier_init(uint32_t bar, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void barrier_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void barrier_expect(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// On a barrier of the cluster's first block, from either.
__device__ __forceinline__ uint32_t first_block_address(uint32_t address)
{
    uint32_t x;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(x) : "r"(address));
    return x;
}
__device__ __forceinline__ void barrier_arrive_cluster(uint32_t bar)
{
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool barrier_try(uint32_t bar, uint32_t parity)
{
    uint32_t done;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(done) : "r"(bar), "r"(parity) : "memory");
    return done != 0;
}

__device__ __forceinline__ uint64_t nanoseconds()
{
    uint64_t t;
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    return t;
}

// Wait for a phase, for two seconds at most.  Then, or as soon as another wait of the block has given up, false: the roles leave their
// loops, the block frees its tensor memory and ends, and hpsgd_ops_check reports it.
__device__ __forceinline__ bool barrier_wait(uint32_t bar, uint32_t parity, volatile int* given_up)
{
    if (barrier_try(bar, parity)) return true;
    const uint64_t start = nanoseconds();
    for (uint32_t i = 0;; ++i) {
        if (barrier_try(bar, parity)) return true;
        if ((i & 255u) == 255u) {
            if (*given_up) return false;
            if (nanoseconds() - start > 2000000000ull) {
                *given_up = 1;
                return false;
            }
        }
    }
}

// A box to this block's shared memory; `bar` may be a barrier of the cluster's first block when two blocks work together.
template <bool PAIR>
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar)
{
    if constexpr (PAIR)
        asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
                     "l"(map), "r"(x), "r"(y), "r"(bar)
                     : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
                     "l"(map), "r"(x), "r"(y), "r"(bar)
                     : "memory");
}

// Shared-memory descriptor of an operand whose rows are 128 bytes, swizzled: eight rows make a group of 1024 bytes.
__device__ __forceinline__ uint64_t operand_descriptor(uint32_t address)
{
    return (uint64_t)(address >> 4 & 0x3FFF) | (uint64_t)1 << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// And of 32 rows of 16 bytes, one after the other, without swizzle: 128 rows' scales.
__device__ __forceinline__ uint64_t scale_descriptor(uint32_t address)
{
    return (uint64_t)(address >> 4 & 0x3FFF) | (uint64_t)1 << 16 | (uint64_t)(128 >> 4) << 32 | (uint64_t)1 << 46;
}

// Instruction descriptor: E4M3 operands, both along k, N = BN, M = 128 or 256, E8M0 scales; `id` names the byte of the scale words.
template <int BN, bool PAIR>
__device__ __forceinline__ uint32_t instruction(uint32_t id)
{
    return id << 4 | (uint32_t)(BN >> 3) << 17 | 1u << 23 | (uint32_t)((PAIR ? 2 * kLanes : kLanes) >> 4) << 24 | id << 29;
}

template <bool PAIR>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, bool add)
{
    if constexpr (PAIR)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
                     "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d), "l"(a), "l"(b),
                     "r"(idesc), "r"(sa), "r"(sb), "r"((uint32_t)add)
                     : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
                     "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale.scale_vec::1X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d), "l"(a), "l"(b),
                     "r"(idesc), "r"(sa), "r"(sb), "r"((uint32_t)add)
                     : "memory");
}
template <bool PAIR>
__device__ __forceinline__ void copy_scales(uint32_t tmem, uint64_t desc)
{
    if constexpr (PAIR) asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
    else asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
// When the products issued so far are done: an arrival at the barrier, in both blocks of a pair.
template <bool PAIR>
__device__ __forceinline__ void commit(uint32_t bar)
{
    if constexpr (PAIR)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((unsigned short)3) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// One lane of a whole warp.  The copies' and products' operands live in uniform registers: behind this, rather than behind a comparison of
// the lane's number, the compiler knows that there is one value of each.
__device__ __forceinline__ bool elected()
{
    uint32_t yes;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(yes));
    return yes != 0;
}
__device__ __forceinline__ void cluster_sync()
{
    cluster_arrive();
    cluster_wait();
}

// Four values at this block's address `at`, out of the memory of block `rank` of its cluster.
__device__ __forceinline__ float4 load_from_block(uint32_t at, int rank)
{
    float4 x;
    uint32_t there;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(at), "r"(rank));
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "r"(there) : "memory");
    return x;
}

__device__ __forceinline__ void word_to_block(uint32_t at, int rank, uint32_t x)
{
    uint32_t there;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(at), "r"(rank));
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(there), "r"(x) : "memory");
}

// C accumulator columns of this thread's lane; complete behind loads_done.
template <int C>
__device__ __forceinline__ void load_columns(uint32_t tmem, float* x)
{
    uint32_t* r = reinterpret_cast<uint32_t*>(x);
    if constexpr (C == 4)
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(tmem));
    else if constexpr (C == 8)
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                     : "r"(tmem));
    else
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
                       "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                     : "r"(tmem));
}
// (the registers are named so that nothing that reads them moves in front of the wait)
template <int C>
__device__ __forceinline__ void loads_done(float* x)
{
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int j = 0; j < C; ++j) asm volatile("" : "+f"(x[j]));
}

// ---------------------------------------------------------------------------- host side
typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

int encoder(EncodeTiled* out)
{
    static std::mutex lock;
    static EncodeTiled found = nullptr;
    std::lock_guard<std::mutex> hold(lock);
    if (!found) {
        void* fn = nullptr;
        cudaDriverEntryPointQueryResult state;
        OPS_CUDA(cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &state));
        if (state != cudaDriverEntryPointSuccess || !fn) return report(HPSGD_E_CUDA, "cuTensorMapEncodeTiled is not available");
        found = reinterpret_cast<EncodeTiled>(fn);
    }
    *out = found;
    return HPSGD_OK;
}

// Boxes of `rows` rows of 128 bytes; what lies outside the matrix reads as zeros.
int make_map(const char* what, CUtensorMap* map, const void* q, int64_t ld, int64_t rows, int64_t cols, int box)
{
    EncodeTiled encode;
    OPS_TRY(encoder(&encode));
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld};
    const cuuint32_t boxes[2] = {(cuuint32_t)kStageK, (cuuint32_t)box}, steps[2] = {1, 1};
    const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(q), dims, strides, boxes, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return report(HPSGD_E_CUDA, "%s: cuTensorMapEncodeTiled failed with %d", what, (int)r);
    return HPSGD_OK;
}

}  // namespace
}  // namespace ops
}  // namespace hpsgd
