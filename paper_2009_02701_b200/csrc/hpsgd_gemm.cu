// Matrix product of two matrices in the 8-bit block format on the fifth-generation tensor cores.
//
// D[m, n] = sum over blocks b of 2^(ea[m, b] + eb[n, b]) * sum over the block's 128 k of A[m, k] B[n, k].  The scales are powers
// of two, so they are exactly the scale operands of the block-scaled tcgen05.mma (E8M0, one for each row and 32 k; the four
// instructions of a 128-block name the same one), and the sums stay in tensor memory in binary32 from the first k to the last.
//
// B's rows (a layer's outputs) lie on the accumulator's 128 lanes and A's rows (tokens) on its columns: with one token a tile is
// 128 x 16 and the kernel streams the weights, and in any case 32 lanes hold 32 neighbouring outputs of a token, so results leave in
// coalesced rows whatever N, the stride and the alignment are.  With many tokens two SMs work on one tile of 256 x 256 (cta_group::2):
// each holds its 128 rows of B and half of A's, so a product of 128 x 256 x 128 on an SM takes 32 KB out of L2 in place of 48.
//
// One block per SM works through its tiles: a thread that keeps a ring of stages full by TMA (128 k of both operands a stage,
// 128-byte swizzle), a warp that puts the scales beside them, a thread that issues the products, and eight warps that empty
// one accumulator while the next is filled.  Few tiles are split along k over the SMs: the blocks of a cluster, which add their parts out of
// each other's shared memory, or for very long sums as many as there are SMs, whose parts a second kernel adds, in their order in any case.
#include "hpsgd_ops_common.cuh"

#include <algorithm>
#include <cuda.h>
#include <mutex>

namespace hpsgd {
namespace ops {

HPSGD_HIDDEN int check_fp8(const char* what, const char* name, const void* q, const void* s, int64_t* ld, int64_t* lds, int64_t rows, int64_t cols);

namespace {

constexpr int kSms = 148;                  // what work is divided by
constexpr int kLanes = 128;                // rows of B in a tile
constexpr int kStageK = 128;               // k of a stage: one scale block, one row of the 128-byte swizzle
constexpr int kGemmThreads = 384;          // copies, products, scales, one idle warp; eight warps for results

__device__ unsigned int g_gemm_timeouts;   // blocks whose wait ran out since the last report

// BN: A's rows in a tile.  PAIR: two blocks (a cluster) share a tile of 256 rows of B, each with 128 of them and half of A's rows.
template <int BN, bool PAIR>
struct Shape {
    static constexpr int kStages = BN <= 64 ? 8 : 6;
    static constexpr int kAtoms = BN <= 128 ? 1 : 2;                     // groups of 128 columns' scales
    static constexpr int kRowsA = PAIR ? BN / 2 : BN;                    // of A, in this block's shared memory
    static constexpr int kBytesB = kLanes * kStageK, kBytesA = kRowsA * kStageK, kBytesS = 512 * (1 + kAtoms);
    static constexpr int kStageBytes = kBytesB + kBytesA;
    static constexpr int kAccs = BN <= 128 ? 2 : 1;
    static constexpr int kPlaces = 4;                                    // groups of scales (four k blocks) in shared memory
    static constexpr int kScaleCols = 4 * (1 + kAtoms);                  // tensor-memory columns of one group, of which one more is kept there
    static constexpr int kCols = kAccs * BN + (kPlaces + 1) * kScaleCols;
    static constexpr int kAlloc = kCols <= 64 ? 64 : kCols <= 128 ? 128 : kCols <= 256 ? 256 : 512;
    static constexpr int kSmem = 1024 + kStages * kStageBytes + kPlaces * kBytesS + 256;
};

struct GemmArgs {
    int M, N, K;
    int tiles_n, tiles;
    int splits, per_split, longer;             // parts along k, a part's k blocks, and how many of the first parts have one more
    int wide;                                  // four neighbouring results may be stored at once
    const uint32_t* sa;
    const uint32_t* sb;
    int64_t ldsa, ldsb, ldd;
    void* d;
    int accumulate;
    uint32_t stall, stall_odd;                 // checked build: bytes that a stage's barrier expects and never gets; in blocks of odd numbers only
    float* part;                               // parts that go through memory: [tile][split][column][lane]
};

// ---------------------------------------------------------------------------- instructions
__device__ __forceinline__ uint32_t smem_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

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
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
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
    if constexpr (C == 8)
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

// ---------------------------------------------------------------------------- the kernel
// Unit u of a block's (or pair's) work: tile u / splits, part u % splits of its k blocks (with joined parts, the block's number in its
// cluster).  n0: this block's first row of B.  Pairs' sums are not split.
struct Unit {
    int n0, m0, k0, k1, tile, split;
};
template <int BN, bool PAIR>
__device__ __forceinline__ Unit unit_of(const GemmArgs& a, int u, int rank)
{
    Unit x;
    x.tile = PAIR ? u : u / a.splits;
    x.split = PAIR ? 0 : u % a.splits;
    x.n0 = x.tile % a.tiles_n * (PAIR ? 2 * kLanes : kLanes) + rank * kLanes;
    x.m0 = x.tile / a.tiles_n * BN;
    x.k0 = PAIR ? 0 : x.split * a.per_split + min(x.split, a.longer);
    x.k1 = PAIR ? a.per_split : x.k0 + a.per_split + (x.split < a.longer);
    return x;
}

// What a result is added to is read, added in registers and written: an addition on the memory side returns nothing to wait for, but PTX has it flush
// subnormal operands and results to 0, so that D += 0 would change D.  The loads go out before the sums are there.  Against that addition, D out of
// HBM: 4096 x 4096 x 512 26.3 us (30.9), 1024 x 1025 x 2000 11.4 (12.4), 4096 x 1024 x 4095 22.8 (22.9), 4096 x 4096 x 8192 135 (126); with 16 MB of D
// in L2, 4096 x 1024 x 512 takes 9.0 (6.9).
__device__ __forceinline__ float load_old(const float* p)
{
    float x;
    asm volatile("ld.global.f32 %0, [%1];" : "=f"(x) : "l"(p) : "memory");
    return x;
}

// C columns of one lane out of rows that are ldd apart, `left` of them there.
template <int C>
__device__ __forceinline__ void load_old_columns(const float* p, int64_t ldd, float* x, int left)
{
    if (left >= C) {
#pragma unroll
        for (int j = 0; j < C; ++j, p += ldd) x[j] = load_old(p);
    } else {
#pragma unroll
        for (int j = 0; j < C; ++j, p += ldd) x[j] = j < left ? load_old(p) : 0.f;
    }
}

// Four neighbours in a row of D, `left` of them there; `wide`: aligned to all four.
__device__ __forceinline__ float4 load_old_four(const float* p, int left, int wide)
{
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    if (wide && left >= 4) asm volatile("ld.global.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "l"(p) : "memory");
    else {
        if (left > 0) x.x = load_old(p);
        if (left > 1) x.y = load_old(p + 1);
        if (left > 2) x.z = load_old(p + 2);
        if (left > 3) x.w = load_old(p + 3);
    }
    return x;
}

template <typename D>
__device__ __forceinline__ void store_four(D* p, const float* v, int left, int wide)
{
    if (wide && left >= 4) {
        if constexpr (sizeof(D) == 4) *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
        else {
            __nv_bfloat162 h[2] = {__floats2bfloat162_rn(v[0], v[1]), __floats2bfloat162_rn(v[2], v[3])};
            *reinterpret_cast<uint2*>(p) = *reinterpret_cast<uint2*>(h);
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (j < left) store1(p + j, v[j]);
}

// C columns of one lane to rows of D that are ldd apart, `left` of them there.
template <int C, typename D>
__device__ __forceinline__ void store_columns(D* p, int64_t ldd, const float* x, int left)
{
    if (left >= C) {
#pragma unroll
        for (int j = 0; j < C; ++j, p += ldd) store1(p, x[j]);
    } else {
#pragma unroll
        for (int j = 0; j < C; ++j, p += ldd)
            if (j < left) store1(p, x[j]);
    }
}

// The sum of a tile's P parts, in their order, out of the shared memory of the P blocks that have them ([column][lane] in each): a warp takes
// 16 / P columns of a part's share at a time (half as many with what they are added to), a thread four lanes of each.
template <int P, typename D, bool ADD>
__device__ __forceinline__ void join_parts(const GemmArgs& a, uint32_t parts, const Unit& x, int cols)
{
    constexpr int kWarps = kGemmThreads / 32, kAtOnce = ADD ? 8 / P : 16 / P;
    const int lane4 = (threadIdx.x & 31) * 4, n = x.n0 + lane4, step = kWarps * P;
    if (n >= a.N) return;
    for (int c0 = (threadIdx.x >> 5) * P + x.split; c0 < cols; c0 += step * kAtOnce) {
        float4 t[kAtOnce][P], old[kAtOnce];
        const auto place = [&](int i) { return static_cast<D*>(a.d) + (int64_t)(x.m0 + c0 + i * step) * a.ldd + n; };
        if constexpr (ADD) {
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i)
                if (c0 + i * step < cols) old[i] = load_old_four(place(i), a.N - n, a.wide);
        }
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i)
#pragma unroll
            for (int k = 0; k < P; ++k)
                if (c0 + i * step < cols) t[i][k] = load_from_block(parts + ((c0 + i * step) * kLanes + lane4) * 4, k);
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            if (c0 + i * step >= cols) continue;
            float v[4] = {t[i][0].x, t[i][0].y, t[i][0].z, t[i][0].w};
#pragma unroll
            for (int k = 1; k < P; ++k) {
                v[0] = __fadd_rn(v[0], t[i][k].x), v[1] = __fadd_rn(v[1], t[i][k].y);
                v[2] = __fadd_rn(v[2], t[i][k].z), v[3] = __fadd_rn(v[3], t[i][k].w);
            }
            if (ADD) v[0] = __fadd_rn(old[i].x, v[0]), v[1] = __fadd_rn(old[i].y, v[1]), v[2] = __fadd_rn(old[i].z, v[2]), v[3] = __fadd_rn(old[i].w, v[3]);
            store_four<D>(place(i), v, a.N - n, a.wide);
        }
    }
}

template <typename D, bool ADD>
__device__ __forceinline__ void join_any(const GemmArgs& a, uint32_t parts, const Unit& x, int cols)
{
    if (a.splits == 2) join_parts<2, D, ADD>(a, parts, x, cols);
    else if (a.splits == 4) join_parts<4, D, ADD>(a, parts, x, cols);
    else join_parts<8, D, ADD>(a, parts, x, cols);
}

// JOIN: the blocks of a cluster have a tile's parts, one each.
template <int BN, bool PAIR, bool JOIN, typename D>
__global__ void __launch_bounds__(kGemmThreads, 1)
    gemm_fp8_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ GemmArgs a)
{
    using S = Shape<BN, PAIR>;
    extern __shared__ uint8_t raw[];
    uint8_t* const smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* const scales = smem + S::kStages * S::kStageBytes;
    uint64_t* const bars = reinterpret_cast<uint64_t*>(scales + S::kPlaces * S::kBytesS);
    __shared__ uint32_t tmem_slot;
    __shared__ volatile int given_up;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = PAIR ? (int)(blockIdx.x & 1) : 0, first = PAIR ? (int)(blockIdx.x >> 1) : (int)blockIdx.x,
              stride = PAIR ? (int)(gridDim.x >> 1) : (int)gridDim.x;      // the first block of a pair issues the products of both
    const uint32_t full = smem_address(bars), empty = full + S::kStages * 8, acc_full = empty + S::kStages * 8, acc_empty = acc_full + S::kAccs * 8,
                   scale_full = acc_empty + S::kAccs * 8, scale_empty = scale_full + S::kPlaces * 8, drained = scale_empty + S::kPlaces * 8;
    if (threadIdx.x == 0) {
        for (int s = 0; s < S::kStages; ++s) {
            barrier_init(full + s * 8, 1);
            barrier_init(empty + s * 8, 1);
        }
        for (int s = 0; s < S::kPlaces; ++s) {
            barrier_init(scale_full + s * 8, PAIR ? 2 : 1);          // the scales of each block
            barrier_init(scale_empty + s * 8, 1);
        }
        for (int s = 0; s < S::kAccs; ++s) {
            barrier_init(acc_full + s * 8, 1);
            barrier_init(acc_empty + s * 8, PAIR ? 16 : 8);          // the warps that read it
        }
        barrier_init(drained, 1);
        given_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 3) {
        if constexpr (PAIR) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_address(&tmem_slot)), "n"(S::kAlloc) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_address(&tmem_slot)), "n"(S::kAlloc) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if constexpr (PAIR) cluster_sync();
    if constexpr (JOIN) cluster_arrive();            // given_up is there to be written by the others; waited for at the end
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    after_previous();
    const uint32_t tmem = tmem_slot, tmem_scales = tmem + S::kAccs * BN;
    const int units = PAIR ? a.tiles : a.tiles * a.splits;

    // Copies and products are requested by one thread for the whole of the loop: with the warp in step, a vote after each wait and an election for
    // each stage, 1 x 30000 x 1024 took 8.0 us in place of 6.7 and 1 x 18944 x 8192 29.9 in place of 27.8 (256 tokens and more: the same).
    // The other roles' waits are the whole warp's, so that what they decide is the same for all of its lanes.
    const auto wait_one = [&](uint32_t bar, uint32_t parity) { return barrier_wait(bar, parity, &given_up); };
    const auto wait = [&](uint32_t bar, uint32_t parity) { return (bool)__all_sync(0xFFFFFFFFu, barrier_wait(bar, parity, &given_up)); };
    if (warp == 0 && elected()) {
        int s = 0;
        uint32_t phase = 1;
        bool ok = true;
        for (int u = first; u < units && ok; u += stride) {
            const Unit x = unit_of<BN, PAIR>(a, u, rank);
            for (int kb = x.k0; kb < x.k1; ++kb) {
                if (!(ok = wait_one(empty + s * 8, phase))) break;
                // Both blocks' boxes count at the first block's barrier, which expects the bytes of both.
                const uint32_t dst = smem_address(smem) + s * S::kStageBytes, bar = PAIR ? first_block_address(full + s * 8) : full + s * 8;
#ifdef HPSGD_DEBUG
                const uint32_t stall = a.stall_odd && !(blockIdx.x & 1) ? 0u : a.stall;
#else
                constexpr uint32_t stall = 0;
#endif
                if (rank == 0) barrier_expect(full + s * 8, (PAIR ? 2 : 1) * S::kStageBytes + stall);
                tma_load<PAIR>(dst, &map_b, kb * kStageK, x.n0, bar);
                tma_load<PAIR>(dst + S::kBytesB, &map_a, kb * kStageK, x.m0 + rank * S::kRowsA, bar);
                if (++s == S::kStages) s = 0, phase ^= 1;
            }
        }
        // giving up: the copies in flight still land (a stage whose scales never came completes no phase, so the wait is for time)
        if (!ok) {
            const uint64_t t = nanoseconds();
            while (nanoseconds() - t < 10000000ull) {}
        }
    } else if (warp == 1 && rank == 0 && elected()) {
        const uint64_t desc_b = operand_descriptor(smem_address(smem)), desc_a = operand_descriptor(smem_address(smem) + S::kBytesB),
                       desc_s = scale_descriptor(smem_address(scales));
        int s = 0, place = 0, column = 0, acc = 0;
        uint32_t phase = 0, place_phase = 0, acc_phase = 1;
        bool ok = true;
        for (int u = first; u < units && ok; u += stride) {
            const Unit x = unit_of<BN, PAIR>(a, u, rank);
            if (!(ok = wait_one(acc_empty + acc * 8, acc_phase))) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            uint32_t sb = 0;
            for (int kb = x.k0; kb < x.k1; ++kb) {
                if (!(ok = wait_one(full + s * 8, phase))) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                if (kb == x.k0 || (kb & 3) == 0) {
                    // The next group's scales, to the column group after the last one's.  Those columns were used kPlaces + 1 groups ago.  This
                    // place was refilled behind the commit of kPlaces groups ago, which waited for all products before its own: they are done.
                    if (!(ok = wait_one(scale_full + place * 8, place_phase))) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    sb = tmem_scales + column * S::kScaleCols;
                    const uint64_t src = desc_s + (uint32_t)(place * (S::kBytesS >> 4));
#pragma unroll
                    for (int t = 0; t < 1 + S::kAtoms; ++t) copy_scales<PAIR>(sb + 4 * t, src + 32 * t);
                    commit<PAIR>(scale_empty + place * 8);
                    if (++column == S::kPlaces + 1) column = 0;
                    if (++place == S::kPlaces) place = 0, place_phase ^= 1;
                }
                const uint64_t db = desc_b + (uint32_t)(s * (S::kStageBytes >> 4)), da = desc_a + (uint32_t)(s * (S::kStageBytes >> 4));
                const uint32_t id = instruction<BN, PAIR>(kb & 3);
#pragma unroll
                for (int k = 0; k < 4; ++k) mma<PAIR>(tmem + acc * BN, db + 2 * k, da + 2 * k, id, sb, sb + 4, kb > x.k0 || k > 0);
                commit<PAIR>(empty + s * 8);
                if (kb + 1 == x.k1) commit<PAIR>(acc_full + acc * 8);
                if (++s == S::kStages) s = 0, phase ^= 1;
            }
            if (++acc == S::kAccs) acc = 0, acc_phase ^= 1;
        }
        if (!ok) {                                  // products in flight read shared memory: let them end
            commit<PAIR>(drained);
            const uint64_t t = nanoseconds();
            while (!barrier_try(drained, 0) && nanoseconds() - t < 1000000000ull) {}
        }
    } else if (warp == 2) {
        // Lane l brings the words of rows l, l + 32, l + 64, l + 96: one 16-byte row of what the copy to tensor memory reads.  A group's words are
        // requested before the place of the group before it is waited for.
        uint32_t w[1 + S::kAtoms][4];
        const auto fetch = [&](const Unit& x, int kb) {
            const int64_t g = kb >> 2;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int r = lane + 32 * j;
                w[0][j] = x.n0 + r < a.N ? __ldg(a.sb + g * a.ldsb + x.n0 + r) : 0u;
#pragma unroll
                for (int t = 0; t < S::kAtoms; ++t) w[1 + t][j] = x.m0 + 128 * t + r < a.M ? __ldg(a.sa + g * a.ldsa + x.m0 + 128 * t + r) : 0u;
            }
        };
        int place = 0;
        uint32_t phase = 1;
        bool ok = true;
        for (int u = first; u < units && ok; u += stride) {
            const Unit x = unit_of<BN, PAIR>(a, u, rank);
            for (int kb = x.k0; kb < x.k1; kb = (kb | 3) + 1) {
                fetch(x, kb);
                if (!(ok = wait(scale_empty + place * 8, phase))) break;
                uint4* const dst = reinterpret_cast<uint4*>(scales + place * S::kBytesS);
#pragma unroll
                for (int t = 0; t < 1 + S::kAtoms; ++t) dst[32 * t + lane] = make_uint4(w[t][0], w[t][1], w[t][2], w[t][3]);
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) {
                    // (across the cluster this release takes about a microsecond: once for four k blocks it stays out of the way, once for
                    // each it was what the kernel waited for)
                    if constexpr (PAIR) barrier_arrive_cluster(first_block_address(scale_full + place * 8));
                    else barrier_arrive(scale_full + place * 8);
                }
                if (++place == S::kPlaces) place = 0, phase ^= 1;
            }
        }
    } else if (warp >= 4) {
        // Two warps for each quarter of the lanes, half of the columns each.  A warp has its scheduler nearly to itself, so what counts is
        // that nothing waits: the columns are requested together, and addresses do not depend on one another.
        constexpr int kHalf = BN / 2, kC = kHalf < 16 ? kHalf : 16;
        const int part = warp & 3, c0 = (warp >> 2) - 1 ? kHalf : 0;
        const uint32_t mine = tmem + c0 + ((uint32_t)part << 21);
        const auto accumulator_read = [&](int acc) {
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
                if constexpr (PAIR) barrier_arrive_cluster(first_block_address(acc_empty + acc * 8));
                else barrier_arrive(acc_empty + acc * 8);
            }
        };
        int done = 0;
        const bool adds = sizeof(D) == 4 && !JOIN && a.accumulate && (PAIR || a.splits == 1);
        if constexpr (sizeof(D) == 4 && !JOIN) {
            // What a unit is added to is requested before its products are waited for, as many columns as registers allow (112 of a pair's 128).  Where
            // a second accumulator lets the next unit's products run ahead, its part of D comes to L2 meanwhile (4096 x 4096 x 512: 33.7 us without,
            // 26.3 with; on pairs that gets in the copies' way: 4096 x 4096 x 8192 132 without, 142 with).
            constexpr int kPieces = kHalf / kC, kSlots = kPieces < 7 ? kPieces : 7;
            float old[kSlots][kC];
            struct Place {
                D* d;
                int left;
            };
            const auto place_of = [&](int u) {
                const Unit x = unit_of<BN, PAIR>(a, u, rank);
                const int n = x.n0 + part * 32 + lane;
                return Place{static_cast<D*>(a.d) + (int64_t)(x.m0 + c0) * a.ldd + n, n < a.N ? a.M - x.m0 - c0 : 0};
            };
            for (int u = first; u < units && adds; u += stride, ++done) {
                const int acc = done % S::kAccs;
                const Place x = place_of(u);
#pragma unroll
                for (int k = 0; k < kSlots; ++k) load_old_columns<kC>(x.d + k * kC * a.ldd, a.ldd, old[k], x.left - k * kC);
                if constexpr (!PAIR) {                // a lane a column: the lines that its 32 neighbouring results begin and end in
                    const int next = u + stride;
                    const Unit y = unit_of<BN, PAIR>(a, next, rank);
                    const int n = y.n0 + part * 32;
#pragma unroll
                    for (int j = lane; j < kHalf; j += 32)
                        if (next < units && n < a.N && y.m0 + c0 + j < a.M) {
                            const D* const row = static_cast<D*>(a.d) + (int64_t)(y.m0 + c0 + j) * a.ldd;
                            asm volatile("prefetch.global.L2 [%0];" ::"l"(row + n));
                            asm volatile("prefetch.global.L2 [%0];" ::"l"(row + min(n + 31, a.N - 1)));
                        }
                }
                if (!wait(acc_full + acc * 8, done / S::kAccs & 1)) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
                for (int k = 0; k < kPieces; ++k) {
                    float v[kC], *const o = old[k % kSlots];
                    load_columns<kC>(mine + acc * BN + k * kC, v);
                    loads_done<kC>(v);
                    if (k + 1 == kPieces) accumulator_read(acc);
#pragma unroll
                    for (int q = 0; q < kC; ++q) o[q] = __fadd_rn(o[q], v[q]);
                    if (kPieces > kSlots) {
                        store_columns<kC, D>(x.d + k * kC * a.ldd, a.ldd, o, x.left - k * kC);
                        if (k + kSlots < kPieces) load_old_columns<kC>(x.d + (k + kSlots) * kC * a.ldd, a.ldd, o, x.left - (k + kSlots) * kC);
                    }
                }
                if (kPieces == kSlots) {
#pragma unroll
                    for (int k = 0; k < kPieces; ++k) store_columns<kC, D>(x.d + k * kC * a.ldd, a.ldd, old[k], x.left - k * kC);
                }
                __syncwarp();
            }
        }
        for (int u = first; u < units && !adds; u += stride, ++done) {
            const Unit x = unit_of<BN, PAIR>(a, u, rank);
            const int acc = done % S::kAccs;
            if (!wait(acc_full + acc * 8, done / S::kAccs & 1)) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t src = mine + acc * BN;
            const int n = x.n0 + part * 32 + lane, cols = a.M - x.m0 - c0;
            D* const d = static_cast<D*>(a.d) + (int64_t)(x.m0 + c0) * a.ldd + n;
            // [column][lane]: a part's own place in device memory, or where this block's stages were (its only unit's products have read them)
            float* const sums = (JOIN ? reinterpret_cast<float*>(smem) : a.part + ((int64_t)x.tile * a.splits + x.split) * (kLanes * BN)) + c0 * kLanes +
                                part * 32 + lane;
            // all of them to registers first, so that the accumulator is free while they are stored
            float v[kHalf];
#pragma unroll
            for (int c = 0; c < kHalf; c += kC) load_columns<kC>(src + c, v + c);
            loads_done<kHalf>(v);
            accumulator_read(acc);
#pragma unroll
            for (int c = 0; c < kHalf; c += kC) {
                if (c >= cols) continue;
                if (JOIN || (!PAIR && a.splits > 1)) store_columns<kC, float>(sums + c * kLanes, kLanes, v + c, cols - c);
                else if (n < a.N) store_columns<kC, D>(d + c * a.ldd, a.ldd, v + c, cols - c);
            }
            __syncwarp();
        }
    }
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0 && given_up) atomicAdd(&g_gemm_timeouts, 1u);
    if constexpr (JOIN) {
        // A block that gave up has no part, and then none of the cluster's blocks writes anything of the tile.  (Told by the one that gave up: asked
        // for by all behind the barrier it cost 0.05 to 0.1 us a product.)
        cluster_wait();
        if (given_up && threadIdx.x < a.splits) word_to_block(smem_address(const_cast<const int*>(&given_up)), threadIdx.x, 1u);
        __syncwarp();
        cluster_sync();
        const Unit x = unit_of<BN, PAIR>(a, first, 0);
        const int cols = given_up ? 0 : min(BN, a.M - x.m0);
        if (sizeof(D) == 4 && a.accumulate) join_any<D, sizeof(D) == 4>(a, smem_address(smem), x, cols);
        else join_any<D, false>(a, smem_address(smem), x, cols);
        __syncwarp();
        cluster_sync();                              // this block's memory stays until the others have read it
    }
    if constexpr (PAIR) cluster_sync();              // the other block's arrivals and products reach into this one
    if (warp == 3) {
        if constexpr (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(S::kAlloc));
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(S::kAlloc));
    }
}

// The sum of a tile's parts, in their order, out of device memory: a warp takes one column (128 lanes, four a thread).  Once a block
// has given up, nothing is written until hpsgd_ops_check has reported it.
constexpr int kSumThreads = 256;
template <int BN, typename D>
__global__ void __launch_bounds__(kSumThreads) sum_parts_kernel(const __grid_constant__ GemmArgs a)
{
    after_previous();
    const int64_t i = (int64_t)blockIdx.x * (kSumThreads / 32) + (threadIdx.x >> 5);
    const int tile = (int)(i / BN), col = (int)(i % BN), lane4 = (threadIdx.x & 31) * 4;
    const int m = tile / a.tiles_n * BN + col, n = tile % a.tiles_n * kLanes + lane4;
    if (tile >= a.tiles || m >= a.M || n >= a.N) return;
    D* const d = static_cast<D*>(a.d) + (int64_t)m * a.ldd + n;
    float4 old;
    if constexpr (sizeof(D) == 4)
        if (a.accumulate) old = load_old_four(d, a.N - n, a.wide);
    const unsigned int gave_up = __ldcg(&g_gemm_timeouts);      // requested in front of the parts, looked at behind their sum
    const float4* const p = reinterpret_cast<const float4*>(a.part + ((int64_t)tile * a.splits * BN + col) * kLanes + lane4);
    float4 x = __ldcg(p);
#pragma unroll 4
    for (int k = 1; k < a.splits; ++k) {
        const float4 y = __ldcg(p + (int64_t)k * (BN * kLanes / 4));
        x = make_float4(__fadd_rn(x.x, y.x), __fadd_rn(x.y, y.y), __fadd_rn(x.z, y.z), __fadd_rn(x.w, y.w));
    }
    if (gave_up != 0u) return;
    if (sizeof(D) == 4 && a.accumulate) x = make_float4(__fadd_rn(old.x, x.x), __fadd_rn(old.y, x.y), __fadd_rn(old.z, x.z), __fadd_rn(old.w, x.w));
    const float v[4] = {x.x, x.y, x.z, x.w};
    store_four<D>(d, v, a.N - n, a.wide);
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

int g_stall = 0;                                // hpsgd_ops_debug_stall

struct Plan {
    int bn, pair, tiles_n, tiles, splits, joined, per_split, longer;
};

// A's side of a tile: the least power of two that holds all its rows, 128 at most; or 256 x 256 on pairs of SMs, which takes half as much
// out of L2 but has one accumulator, so that a tile's results are not stored behind the next one's products.  In a round of tiles an SM spent
// 0.25 us for each k block and 0.2 us more on 128 x 128, 0.37 and 1.8 us on its half of 256 x 256 (4096 x 4096 x 1024: 19.3 against 22.3 us;
// 4096 x 4096 x 4096: 54.8 against 52.2; 8192 x 4096 x 4096: 112 against 95): the fewer of these, rounds counted whole.
//
// Splitting along k, where tiles are fewer than half the SMs and there are 16 k blocks (100 x 1000 x 1000 with its 8: 6.7 us whole, 7.5 to
// 7.8 in parts; 32 x 2048 x 2048 with 16: 6.1 in four parts, 6.7 in two): two, four or eight parts of four blocks or more, a cluster's, as
// many as leave every cluster its SMs at once (the device held 33 clusters of four, 15 of eight; 16 of eight take a second round, 17.9 us
// in place of 10.2).  Beyond 128 k blocks, where there is room for 16 parts, these go through memory: with 1 x 128, K = 16384 takes 7.3 us
// in a cluster and 8.2 through memory, K = 32768 10.2 and 8.5.
constexpr int kSplitBlocks = 16, kLeastBlocks = 4, kJoinBlocks = 128, kMemoryParts = 16, kMemoryBlocks = 8;
Plan plan_of(int64_t M, int64_t N, int64_t K)
{
    const auto up = [](int64_t x, int64_t y) { return (x + y - 1) / y; };
    Plan p{};
    const int blocks = (int)up(K, kStageK);
    p.bn = M <= 16 ? 16 : M <= 32 ? 32 : M <= 64 ? 64 : 128;
    int64_t tiles_n = up(N, kLanes), tiles = tiles_n * up(M, p.bn);
    if (M > 128) {
        const int64_t pairs_n = up(N, 2 * kLanes), pairs = pairs_n * up(M, 256);
        if ((double)up(pairs, kSms / 2) * (9.0 * blocks + 44.0) < (double)up(tiles, kSms) * (6.0 * blocks + 4.0)) {
            p.pair = 1;
            p.bn = 256;
            tiles_n = pairs_n;
            tiles = pairs;
        }
    }
    p.tiles_n = (int)tiles_n;
    p.tiles = (int)tiles;
    p.splits = 1;
    if (!p.pair && tiles <= kSms / 2 && blocks >= kSplitBlocks) {
        const int most = (int)std::min<int64_t>(kSms / tiles, blocks / kMemoryBlocks);
        if (blocks > kJoinBlocks && most >= kMemoryParts) p.splits = most;
        else {
            p.joined = 1;
            p.splits = tiles > 32 ? 2 : tiles > 14 || blocks < 8 * kLeastBlocks ? 4 : 8;
        }
    }
    p.per_split = blocks / p.splits;
    p.longer = blocks % p.splits;
    return p;
}

size_t workspace_of(const Plan& p)
{
    return p.splits > 1 && !p.joined ? (size_t)p.tiles * p.splits * kLanes * p.bn * sizeof(float) : 0;
}

template <int BN, bool PAIR, bool JOIN, typename D>
int launch(const CUtensorMap& ma, const CUtensorMap& mb, const GemmArgs& a, int sms, cudaStream_t s)
{
    using S = Shape<BN, PAIR>;
    // Per device: the blocks (or pairs) that it holds at a time.  Pairs need both their SMs in one GPU cluster, so there may be fewer than
    // half the SMs' number, and work given to more would wait for a second round.
    static int workers[64] = {};
    int dev = 0;
    OPS_CUDA(cudaGetDevice(&dev));
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute attr[2] = {};
    cfg.gridDim = dim3(PAIR ? 2 : 1);
    cfg.blockDim = dim3(kGemmThreads);
    cfg.dynamicSmemBytes = S::kSmem;
    cfg.stream = s;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;          // see launch_early
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = PAIR ? 2 : JOIN ? (unsigned)a.splits : 1;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = PAIR || JOIN ? 2 : 1;
    int at_once = dev < 64 ? workers[dev] : 0;
    if (at_once == 0) {
        OPS_CUDA(cudaFuncSetAttribute(gemm_fp8_kernel<BN, PAIR, JOIN, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem));
        at_once = sms;
        if (PAIR) OPS_CUDA(cudaOccupancyMaxActiveClusters(&at_once, gemm_fp8_kernel<BN, PAIR, JOIN, D>, &cfg));
        at_once = std::max(1, at_once);
        if (dev < 64) workers[dev] = at_once;
    }
    const int64_t units = (int64_t)a.tiles * a.splits;
    cfg.gridDim = dim3((PAIR ? 2u : 1u) * (unsigned)(JOIN ? units : std::min<int64_t>(units, at_once)));
    OPS_CUDA(cudaLaunchKernelEx(&cfg, gemm_fp8_kernel<BN, PAIR, JOIN, D>, ma, mb, a));
    OPS_TRY(launched("hpsgd_gemm_fp8"));
    if (PAIR || JOIN || a.splits == 1) return HPSGD_OK;
    if constexpr (!PAIR && !JOIN) {
        const int64_t columns = (int64_t)a.tiles * BN;
        return launch_early("hpsgd_gemm_fp8", sum_parts_kernel<BN, D>, dim3((unsigned)((columns + kSumThreads / 32 - 1) / (kSumThreads / 32))), kSumThreads, 0, s, a);
    }
    return HPSGD_OK;
}

template <bool JOIN, typename D>
int launch_shape(const Plan& p, const CUtensorMap& ma, const CUtensorMap& mb, const GemmArgs& a, int sms, cudaStream_t s)
{
    switch (p.bn) {
    case 16: return launch<16, false, JOIN, D>(ma, mb, a, sms, s);
    case 32: return launch<32, false, JOIN, D>(ma, mb, a, sms, s);
    case 64: return launch<64, false, JOIN, D>(ma, mb, a, sms, s);
    case 128: return launch<128, false, JOIN, D>(ma, mb, a, sms, s);
    default: return launch<256, true, false, D>(ma, mb, a, sms, s);
    }
}

}  // namespace
}  // namespace ops
}  // namespace hpsgd

using namespace hpsgd;
using namespace hpsgd::ops;

extern "C" {

size_t hpsgd_gemm_fp8_bytes(int64_t M, int64_t N, int64_t K)
{
    if (M <= 0 || N <= 0 || K <= 0 || M > 0x7FFFFFFF || N > 0x7FFFFFFF || K > 0x7FFFFFFF) return 0;
    return workspace_of(plan_of(M, N, K));
}

int hpsgd_gemm_fp8(const hpsgd_gemm_fp8_args* args, void* stream)
{
    const char* what = "hpsgd_gemm_fp8";
    if (!args) return report(HPSGD_E_BADARG, "%s: args is NULL", what);
    hpsgd_gemm_fp8_args p = *args;
    if (p.M < 0 || p.N < 0 || p.K < 0) return report(HPSGD_E_BADARG, "%s: a size is negative", what);
    // coordinates of boxes that reach past the end stay below 2^31, tiles below 2^31
    const int64_t most = 0x7FFFFFFF - 4096;
    if (p.M > most || p.N > most || p.K > most || ((p.N + 127) / 128) * ((p.M + 127) / 128) > most)
        return report(HPSGD_E_UNSUPPORTED, "%s: a size is too large", what);
    if (p.d_dtype != HPSGD_F32 && p.d_dtype != HPSGD_BF16) return report(HPSGD_E_BADARG, "%s: unknown d_dtype %d", what, p.d_dtype);
    if (p.accumulate != 0 && (p.accumulate != 1 || p.d_dtype != HPSGD_F32)) return report(HPSGD_E_BADARG, "%s: accumulate must be 0, or 1 with an fp32 result", what);
    if (p.M == 0 || p.N == 0) return HPSGD_OK;
    const size_t esz = p.d_dtype == HPSGD_F32 ? 4 : 2;
    if (p.ldd == 0) p.ldd = p.N;
    if (!p.d || !aligned(p.d, esz) || p.ldd < p.N) return report(HPSGD_E_BADARG, "%s: d is NULL, not aligned to its elements, or its stride is below N", what);
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    int sms = 0;
    if (p.K == 0) {
        OPS_TRY(device_sms(&sms));
        if (!p.accumulate) OPS_CUDA(cudaMemset2DAsync(p.d, (size_t)p.ldd * esz, 0, (size_t)p.N * esz, (size_t)p.M, s));
        return HPSGD_OK;
    }
    if (!p.a || !p.b) return report(HPSGD_E_BADARG, "%s: a or b is NULL", what);
    OPS_TRY(check_fp8(what, "a", p.a, p.a_scale, &p.lda, &p.ldsa, p.M, p.K));
    OPS_TRY(check_fp8(what, "b", p.b, p.b_scale, &p.ldb, &p.ldsb, p.N, p.K));
    const Plan plan = plan_of(p.M, p.N, p.K);
    const size_t need = workspace_of(plan);
    if (need && (!p.workspace || !aligned(p.workspace, 16))) return report(HPSGD_E_BADARG, "%s: workspace is NULL or not 16-byte aligned", what);
    if (need > p.workspace_bytes) return report(HPSGD_E_NOMEM, "%s: workspace of %zu bytes is smaller than the %zu needed", what, p.workspace_bytes, need);
    OPS_TRY(device_sms(&sms));
    CUtensorMap ma, mb;
    OPS_TRY(make_map(what, &ma, p.a, p.lda, p.M, p.K, plan.pair ? plan.bn / 2 : plan.bn));
    OPS_TRY(make_map(what, &mb, p.b, p.ldb, p.N, p.K, kLanes));
    GemmArgs a{};
    a.M = (int)p.M; a.N = (int)p.N; a.K = (int)p.K;
    a.tiles_n = plan.tiles_n; a.tiles = plan.tiles; a.splits = plan.splits; 
    a.per_split = plan.per_split; a.longer = plan.longer;
    a.wide = p.ldd % 4 == 0 && aligned(p.d, 4 * esz);
    a.sa = reinterpret_cast<const uint32_t*>(p.a_scale); a.sb = reinterpret_cast<const uint32_t*>(p.b_scale);
    a.stall = g_stall ? 16 : 0;
    a.stall_odd = g_stall == 2;
    a.ldsa = p.ldsa; a.ldsb = p.ldsb; a.ldd = p.ldd; a.d = p.d; a.accumulate = p.accumulate;
    a.part = static_cast<float*>(p.workspace);
    if (p.d_dtype == HPSGD_F32) return plan.joined ? launch_shape<true, float>(plan, ma, mb, a, sms, s) : launch_shape<false, float>(plan, ma, mb, a, sms, s);
    return plan.joined ? launch_shape<true, __nv_bfloat16>(plan, ma, mb, a, sms, s) : launch_shape<false, __nv_bfloat16>(plan, ma, mb, a, sms, s);
}

int hpsgd_ops_debug_stall(int enable)
{
#ifdef HPSGD_DEBUG
    if (enable < 0 || enable > 2) return report(HPSGD_E_BADARG, "hpsgd_ops_debug_stall: enable must be 0, 1 or 2");
    g_stall = enable;
    return HPSGD_OK;
#else
    (void)enable;
    return report(HPSGD_E_UNSUPPORTED, "hpsgd_ops_debug_stall: only in the checked build");
#endif
}

int hpsgd_ops_check(void* stream)
{
    int sms = 0;
    OPS_TRY(device_sms(&sms));
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    OPS_CUDA(cudaStreamSynchronize(s));
    unsigned int n = 0;
    OPS_CUDA(cudaMemcpyFromSymbol(&n, g_gemm_timeouts, sizeof n));
    if (n != 0) {
        const unsigned int zero = 0;
        OPS_CUDA(cudaDeviceSynchronize());             // a sum of parts on another stream may still have to see the count
        OPS_CUDA(cudaMemcpyFromSymbol(&n, g_gemm_timeouts, sizeof n));
        OPS_CUDA(cudaMemcpyToSymbol(g_gemm_timeouts, &zero, sizeof zero));
        return report(HPSGD_E_TIMEOUT, "hpsgd_gemm_fp8: %u blocks gave up waiting for their own loads or products after two seconds; their tiles were not written", n);
    }
    return HPSGD_OK;
}

}  // extern "C"
