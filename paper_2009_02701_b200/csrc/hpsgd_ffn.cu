// The gated feed-forward layer on matrices in the 8-bit block format: both projections, the activation and the product in one kernel, and
// the gradients of what they are multiplied to.
//
// Forward, z = act(x Wg^T) * (x Wu^T): the product of hpsgd_gemm.cu with two accumulators, whose lanes are the same 128 features: the gate's rows
// of the weights on one, those of what it gates on the other, tokens on the columns of both.  A stage of shared memory has 128 k of both weights and of
// the tokens, so the tokens are read once for the two.  With many tokens two SMs work on one tile of 256 features x 224 tokens (cta_group::2), whose two times 224
// accumulator columns and scales are the whole of tensor memory.
//
// Bound by what feeds the tensor cores out of L2 and by the power cap with long sums (8192 x 8192 x 2048: 219 us, 2.5 PFLOP/s; 265 us when it is run for long and the
// cap has settled), and with short ones by what the sums go through: activation, product, the block's largest magnitude, rounding, 35 instructions for a result and 50
// where its sums are kept.  Sixteen warps do that, from tensor memory to registers in one
// go, so that the accumulator is free for the next products before anything is rounded.  (Eight warps that took eight columns at a time through
// shared memory, for 128 features of a token to a warp, took 443 us.)
#include "hpsgd_quantize.cuh"
#include "hpsgd_tensor_core.cuh"

#include <algorithm>
#include <type_traits>

namespace hpsgd {
namespace ops {

HPSGD_HIDDEN int check_fp8(const char* what, const char* name, const void* q, const void* s, int64_t* ld, int64_t* lds, int64_t rows, int64_t cols);
HPSGD_HIDDEN int stall_mode();

namespace {

constexpr int kSms = 148;
constexpr int kGroups = 4;                 // of warps for results: each has a quarter of the tokens, and its four warps the 128 features of them
constexpr int kFfnThreads = 128 + 128 * kGroups;      // copies, products, scales, one idle warp; and those

__device__ unsigned int g_ffn_timeouts;    // blocks whose wait ran out since the last report

// BN: tokens of a tile.  PAIR: two blocks (a cluster) share a tile of 256 features, each with 128 of them and half of the tokens.
template <int BN, bool PAIR>
struct FfnShape {
    static constexpr int kStages = BN <= 64 ? 5 : 4;
    static constexpr int kAtoms = BN <= 128 ? 1 : 2;                     // groups of 128 tokens' scales
    static constexpr int kRowsX = PAIR ? BN / 2 : BN;                    // tokens in this block's shared memory
    static constexpr int kBytesW = kLanes * kStageK, kBytesX = kRowsX * kStageK;      // of one of the weights, and of the tokens
    static constexpr int kStageBytes = 2 * kBytesW + kBytesX;
    static constexpr int kAccs = BN <= 64 ? 2 : 1;
    static constexpr int kPlaces = PAIR ? 3 : 4;                         // groups of scales (four k blocks) in shared memory
    static constexpr int kParts = 2 + kAtoms;                            // of one group: gate, gated, tokens
    static constexpr int kBytesS = 512 * kParts;
    static constexpr int kScaleCols = 4 * kParts;
    static constexpr int kCols = kAccs * 2 * BN + (kPlaces + 1) * kScaleCols;
    static constexpr int kAlloc = kCols <= 128 ? 128 : kCols <= 256 ? 256 : 512;
    static constexpr int kMine = BN / kGroups;                           // tokens of a group of warps
    static constexpr int kBytesOut = 2 * 2 * kGroups * 4 * kMine * 4;    // largest magnitudes by warp: of two tiles in turn, of all and of the finite
    static constexpr int kSmem = 1024 + kStages * kStageBytes + kPlaces * kBytesS + kBytesOut + 256;
};

// Where a token's results go.
struct FfnOut {
    int N;
    uint8_t* z8;
    uint8_t* zs;
    void* z;
    __nv_bfloat16* gu;
    int64_t ldz8, ldzs, ldz, ldgu;
    int z_bf16, wide_z, wide_gu;               // wide: four neighbours may be stored at once
};

struct FfnArgs {
    FfnOut out;
    int M, K;
    int tiles_n, tiles;
    int splits, per_split, longer;             // parts along k, a part's k blocks, and how many of the first parts have one more
    const uint32_t* sx;
    const uint32_t* sw;
    int64_t ldsx, ldsw;
    uint32_t stall, stall_odd;                 // checked build, as in hpsgd_gemm.cu
};

// ---------------------------------------------------------------------------- the activation
constexpr float kGelu1 = 1.59576912f, kGelu3 = 0.044715f;      // 2 sqrt(2 / pi): (1 + tanh(w / 2)) / 2 = sigmoid(w)

__device__ __forceinline__ float sigmoid(float x) { return reciprocal(__fadd_rn(1.f, exp2_of(__fmul_rn(x, -kLog2e)))); }

template <int ACT>
__device__ __forceinline__ float activation(float g)
{
    const float w = ACT == HPSGD_SILU ? g : __fmul_rn(kGelu1, __fmaf_rn(__fmul_rn(kGelu3, __fmul_rn(g, g)), g, g));
    return __fmul_rn(g, sigmoid(w));
}

// act(g) and its derivative: with s = sigmoid(w), s + g s (1 - s) w'.  A gate is held to where s is 2^-126: below, the products of s with g and w' would grow again,
// since s is not smaller, while both results are 0 next to anything.  Above 10 gelu's slope is s, but a square that overflows would make 0 times infinity of the rest.
template <int ACT>
__device__ __forceinline__ void activation(float g, float& value, float& slope)
{
    asm("max.NaN.f32 %0, %0, %1;" : "+f"(g) : "f"(ACT == HPSGD_SILU ? -87.33f : -10.001f));
    const float g2 = fminf(__fmul_rn(g, g), 101.f);
    const float w = ACT == HPSGD_SILU ? g : __fmul_rn(kGelu1, __fmaf_rn(__fmul_rn(kGelu3, g2), g, g));
    const float e = exp2_of(__fmul_rn(w, -kLog2e)), s = reciprocal(__fadd_rn(1.f, e));
    value = __fmul_rn(g, s);
    const float t = __fmul_rn(value, __fmul_rn(e, s));
    slope = ACT == HPSGD_SILU ? __fadd_rn(t, s) : __fmaf_rn(t, __fmul_rn(kGelu1, __fmaf_rn(3.f * kGelu3, g2, 1.f)), s);
}

// ---------------------------------------------------------------------------- what a warp does with a token's 128 features
__device__ __forceinline__ void store_bf16(__nv_bfloat16* p, const float* v, int left, int wide)
{
    if (wide && left >= 4) *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
    else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (j < left) p[j] = __float2bfloat16_rn(v[j]);
    }
}

// Lane l has the sums g, u of features n0 + 4 l .. + 3 of token m.
template <int ACT>
__device__ __forceinline__ void finish(const FfnOut& a, int m, int n0, float4 g4, float4 u4)
{
    const int lane = threadIdx.x & 31, n = n0 + lane * 4, left = a.N - n;
    const float g[4] = {g4.x, g4.y, g4.z, g4.w}, u[4] = {u4.x, u4.y, u4.z, u4.w};
    if (a.gu) {
        __nv_bfloat16* const p = a.gu + m * a.ldgu + n;
        store_bf16(p, g, left, a.wide_gu);
        store_bf16(p + a.N, u, left, a.wide_gu);
    }
    float z[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) z[j] = j < left ? __fmul_rn(activation<ACT>(g[j]), u[j]) : 0.f;
    if (a.z) {
        if (a.z_bf16) store_bf16(static_cast<__nv_bfloat16*>(a.z) + m * a.ldz + n, z, left, a.wide_z);
        else {
            float* const p = static_cast<float*>(a.z) + m * a.ldz + n;
            if (a.wide_z && left >= 4) *reinterpret_cast<float4*>(p) = make_float4(z[0], z[1], z[2], z[3]);
            else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (j < left) p[j] = z[j];
            }
        }
    }
    if (!a.z8) return;
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) top = max(top, __float_as_uint(fabsf(z[j])));
    top = __reduce_max_sync(0xFFFFFFFFu, top);
    if (top >= 0x7F800000u) {                         // values that are not finite do not count, and become NaN
        top = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (finite(z[j])) top = max(top, __float_as_uint(fabsf(z[j])));
            else z[j] = __uint_as_float(0x7FC00000u);
        }
        top = __reduce_max_sync(0xFFFFFFFFu, top);
    }
    const int byte = scale_byte(__uint_as_float(top));
    const float inv = scale_inverse(byte);
    if (n < (a.N + 15) / 16 * 16)
        *reinterpret_cast<uint32_t*>(a.z8 + m * a.ldz8 + n) = codes4(__fmul_rn(z[0], inv), __fmul_rn(z[1], inv), __fmul_rn(z[2], inv), __fmul_rn(z[3], inv));
    if (lane == 0) {
        const int b = n0 / kBlock;
        uint8_t* const s = a.zs + scale_index(b, m, a.ldzs);
        *s = (uint8_t)byte;
        if (b == (a.N - 1) / kBlock)                  // zeros behind the row's last block
            for (int k = 1; (b + k) & 3; ++k) s[k] = 0;
    }
}

// ---------------------------------------------------------------------------- the kernel
// Unit u of a block's (or pair's) work; n0: this block's first feature.  Pairs' sums are not split.
struct FfnUnit {
    int n0, m0, k0, k1, split;
};
template <int BN, bool PAIR>
__device__ __forceinline__ FfnUnit ffn_unit(const FfnArgs& a, int u, int rank)
{
    FfnUnit x;
    const int tile = PAIR ? u : u / a.splits;
    x.split = PAIR ? 0 : u % a.splits;
    x.n0 = tile % a.tiles_n * (PAIR ? 2 * kLanes : kLanes) + rank * kLanes;
    x.m0 = tile / a.tiles_n * BN;
    x.k0 = PAIR ? 0 : x.split * a.per_split + min(x.split, a.longer);
    x.k1 = PAIR ? a.per_split : x.k0 + a.per_split + (x.split < a.longer);
    return x;
}

// JOIN: the blocks of a cluster have a tile's parts along k, one each, and add them out of each other's shared memory in their order.
template <int BN, bool PAIR, bool JOIN, int ACT>
__global__ void __launch_bounds__(kFfnThreads, 1)
    gated_ffn_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const __grid_constant__ FfnArgs a)
{
    using S = FfnShape<BN, PAIR>;
    extern __shared__ uint8_t raw[];
    uint8_t* const smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* const scales = smem + S::kStages * S::kStageBytes;
    uint32_t* const tops = reinterpret_cast<uint32_t*>(scales + S::kPlaces * S::kBytesS);
    uint64_t* const bars = reinterpret_cast<uint64_t*>(scales + S::kPlaces * S::kBytesS + S::kBytesOut);
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
            barrier_init(acc_empty + s * 8, (PAIR ? 2 : 1) * 4 * kGroups);      // the warps that read it
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
    const uint32_t tmem = tmem_slot, tmem_scales = tmem + S::kAccs * 2 * BN;
    const int units = PAIR ? a.tiles : a.tiles * a.splits;

    const auto wait_one = [&](uint32_t bar, uint32_t parity) { return barrier_wait(bar, parity, &given_up); };
    const auto wait = [&](uint32_t bar, uint32_t parity) { return (bool)__all_sync(0xFFFFFFFFu, barrier_wait(bar, parity, &given_up)); };
    if (warp == 0 && elected()) {
        int s = 0;
        uint32_t phase = 1;
        bool ok = true;
        for (int u = first; u < units && ok; u += stride) {
            const FfnUnit x = ffn_unit<BN, PAIR>(a, u, rank);
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
                // (rows of the gate's box behind its last feature are the other weights'; they come to nothing)
                tma_load<PAIR>(dst, &map_w, kb * kStageK, x.n0, bar);
                tma_load<PAIR>(dst + S::kBytesW, &map_w, kb * kStageK, a.out.N + x.n0, bar);
                tma_load<PAIR>(dst + 2 * S::kBytesW, &map_x, kb * kStageK, x.m0 + rank * S::kRowsX, bar);
                if (++s == S::kStages) s = 0, phase ^= 1;
            }
        }
        if (!ok) {                                   // giving up: the copies in flight still land
            const uint64_t t = nanoseconds();
            while (nanoseconds() - t < 10000000ull) {}
        }
    } else if (warp == 1 && rank == 0 && elected()) {
        const uint64_t desc = operand_descriptor(smem_address(smem)), desc_s = scale_descriptor(smem_address(scales));
        int s = 0, place = 0, column = 0, acc = 0;
        uint32_t phase = 0, place_phase = 0, acc_phase = 1;
        bool ok = true;
        for (int u = first; u < units && ok; u += stride) {
            const FfnUnit x = ffn_unit<BN, PAIR>(a, u, rank);
            if (!(ok = wait_one(acc_empty + acc * 8, acc_phase))) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            uint32_t sc = 0;
            for (int kb = x.k0; kb < x.k1; ++kb) {
                if (!(ok = wait_one(full + s * 8, phase))) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                if (kb == x.k0 || (kb & 3) == 0) {
                    // the next group's scales, to columns that were used kPlaces + 1 groups ago: those products are done (see hpsgd_gemm.cu)
                    if (!(ok = wait_one(scale_full + place * 8, place_phase))) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    sc = tmem_scales + column * S::kScaleCols;
                    const uint64_t src = desc_s + (uint32_t)(place * (S::kBytesS >> 4));
#pragma unroll
                    for (int t = 0; t < S::kParts; ++t) copy_scales<PAIR>(sc + 4 * t, src + 32 * t);
                    commit<PAIR>(scale_empty + place * 8);
                    if (++column == S::kPlaces + 1) column = 0;
                    if (++place == S::kPlaces) place = 0, place_phase ^= 1;
                }
                const uint64_t dg = desc + (uint32_t)(s * (S::kStageBytes >> 4)), du = dg + (uint32_t)(S::kBytesW >> 4), dx = dg + (uint32_t)(2 * S::kBytesW >> 4);
                const uint32_t id = instruction<BN, PAIR>(kb & 3);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    mma<PAIR>(tmem + acc * 2 * BN, dg + 2 * k, dx + 2 * k, id, sc, sc + 8, kb > x.k0 || k > 0);
                    mma<PAIR>(tmem + acc * 2 * BN + BN, du + 2 * k, dx + 2 * k, id, sc + 4, sc + 8, kb > x.k0 || k > 0);
                }
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
        // Lane l brings the words of rows l, l + 32, l + 64, l + 96: one 16-byte row of what the copy to tensor memory reads.
        uint32_t w[S::kParts][4];
        const auto fetch = [&](const FfnUnit& x, int kb) {
            const int64_t g = kb >> 2;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int r = lane + 32 * j;
                const bool in = x.n0 + r < a.out.N;
                w[0][j] = in ? __ldg(a.sw + g * a.ldsw + x.n0 + r) : 0u;
                w[1][j] = in ? __ldg(a.sw + g * a.ldsw + a.out.N + x.n0 + r) : 0u;
#pragma unroll
                for (int t = 0; t < S::kAtoms; ++t) w[2 + t][j] = 128 * t + r < BN && x.m0 + 128 * t + r < a.M ? __ldg(a.sx + g * a.ldsx + x.m0 + 128 * t + r) : 0u;
            }
        };
        int place = 0;
        uint32_t phase = 1;
        bool ok = true;
        for (int u = first; u < units && ok; u += stride) {
            const FfnUnit x = ffn_unit<BN, PAIR>(a, u, rank);
            for (int kb = x.k0; kb < x.k1; kb = (kb | 3) + 1) {
                fetch(x, kb);
                if (!(ok = wait(scale_empty + place * 8, phase))) break;
                uint4* const dst = reinterpret_cast<uint4*>(scales + place * S::kBytesS);
#pragma unroll
                for (int t = 0; t < S::kParts; ++t) dst[32 * t + lane] = make_uint4(w[t][0], w[t][1], w[t][2], w[t][3]);
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) {
                    if constexpr (PAIR) barrier_arrive_cluster(first_block_address(scale_full + place * 8));
                    else barrier_arrive(scale_full + place * 8);
                }
                if (++place == S::kPlaces) place = 0, phase ^= 1;
            }
        }
    } else if (warp >= 4) {
        // A warp has 32 features and a group's tokens.  First all of them go through the activation, to registers, so that the accumulator is free for the next
        // tile's products; then, with the largest magnitudes of the group's four warps, which make a block, through the rounding.
        constexpr int kMine = S::kMine, kC = kMine < 8 ? kMine : 8, kWords = (kMine + 31) / 32;
        const int part = warp & 3, group = __shfl_sync(0xFFFFFFFFu, (warp >> 2) - 1, 0), c0 = group * kMine;
        const uint32_t mine = tmem + c0 + ((uint32_t)part << 21);
        // the four warps of this group
        const auto all_four = [&](bool yes) {
            uint32_t all;
            asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.and.pred q, %2, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                         : "=r"(all)
                         : "r"((uint32_t)yes), "r"(group + 1)
                         : "memory");
            return all != 0;
        };
        const auto accumulator_read = [&](int acc) {
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) {
                if constexpr (PAIR) barrier_arrive_cluster(first_block_address(acc_empty + acc * 8));
                else barrier_arrive(acc_empty + acc * 8);
            }
        };
        int done = 0;
        for (int u = first; u < units; u += stride, ++done) {
            const FfnUnit x = ffn_unit<BN, PAIR>(a, u, rank);
            const int acc = done % S::kAccs;
            // the four warps of a group wait for one another below, so they go on together or not at all
            if (!all_four(wait(acc_full + acc * 8, done / S::kAccs & 1))) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t src = mine + acc * 2 * BN;
            if constexpr (JOIN) {                    // [sum][column][lane], where this block's stages were (its only unit's products have read them)
                float* const to = reinterpret_cast<float*>(smem) + c0 * kLanes + part * 32 + lane;
#pragma unroll
                for (int c = 0; c < kMine; c += kC) {
                    float g[kC], v[kC];
                    load_columns<kC>(src + c, g);
                    load_columns<kC>(src + BN + c, v);
                    loads_done<kC>(g);
                    loads_done<kC>(v);
#pragma unroll
                    for (int j = 0; j < kC; ++j) {
                        to[(c + j) * kLanes] = g[j];
                        to[(c + j) * kLanes + BN * kLanes] = v[j];
                    }
                }
                accumulator_read(acc);
            } else {
                const FfnOut& o = a.out;
                const int n = x.n0 + part * 32 + lane, m0 = x.m0 + c0, cols = a.M - m0;
                const bool in = n < o.N;
                float z[kMine];
                uint32_t top[kWords];                // lane l's: of columns l, l + 32
                // ALL: every token and feature of the tile is there; KEEP: the sums are kept.  (A column's offset is the same in all threads, so it is added on
                // the way to memory.)
                const auto through = [&](auto all, auto keep) {
                    constexpr bool ALL = decltype(all)::value, KEEP = decltype(keep)::value;
                    uint16_t* const to_g = reinterpret_cast<uint16_t*>(o.gu) + m0 * o.ldgu + n;
                    uint16_t* const to_u = to_g + o.N;
#pragma unroll
                    for (int c = 0; c < kMine; c += kC) {
                        float g[kC], v[kC];
                        load_columns<kC>(src + c, g);
                        load_columns<kC>(src + BN + c, v);
                        loads_done<kC>(g);
                        loads_done<kC>(v);
                        if (c + kC == kMine) accumulator_read(acc);
#pragma unroll
                        for (int j = 0; j < kC; j += 2) {
                            if constexpr (KEEP) {
                                const uint32_t gg = pack_bf16(g[j], g[j + 1]), uu = pack_bf16(v[j], v[j + 1]);
                                const int64_t at = (c + j) * o.ldgu, next = (c + j + 1) * o.ldgu;
                                if (ALL || (in && c + j < cols)) to_g[at] = (uint16_t)gg, to_u[at] = (uint16_t)uu;
                                if (ALL || (in && c + j + 1 < cols)) to_g[next] = (uint16_t)(gg >> 16), to_u[next] = (uint16_t)(uu >> 16);
                            }
                        }
#pragma unroll
                        for (int j = 0; j < kC; ++j) {
                            const float y = __fmul_rn(activation<ACT>(g[j]), v[j]);
                            z[c + j] = ALL || in ? y : 0.f;
                            const uint32_t t = __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(fabsf(z[c + j])));
                            if (lane == ((c + j) & 31)) top[(c + j) >> 5] = t;
                        }
                    }
                };
                const bool all = x.m0 + BN <= a.M && x.n0 + kLanes <= o.N;
                using Yes = std::true_type;
                using No = std::false_type;
                if (all) o.gu ? through(Yes{}, Yes{}) : through(Yes{}, No{});
                else o.gu ? through(No{}, Yes{}) : through(No{}, No{});
                if (o.z) {
#pragma unroll
                    for (int j = 0; j < kMine; ++j)
                        if (in && j < cols) {
                            if (o.z_bf16) static_cast<__nv_bfloat16*>(o.z)[(m0 + j) * o.ldz + n] = __float2bfloat16_rn(z[j]);
                            else static_cast<float*>(o.z)[(m0 + j) * o.ldz + n] = z[j];
                        }
                }
                if (!o.z8) continue;
                // [turn][finite][group][warp][column]
                uint32_t* const place = tops + (done & 1) * (2 * kGroups * 4 * kMine) + group * (4 * kMine);
                const auto exchange = [&](uint32_t* at) {
#pragma unroll
                    for (int i = 0; i < kWords; ++i)
                        if (i * 32 + lane < kMine) at[part * kMine + i * 32 + lane] = top[i];
                    all_four(true);
#pragma unroll
                    for (int i = 0; i < kWords; ++i) {
                        const int col = min(i * 32 + lane, kMine - 1);
                        top[i] = max(max(at[col], at[kMine + col]), max(at[2 * kMine + col], at[3 * kMine + col]));
                    }
                };
                exchange(place);
                bool odd = false;
#pragma unroll
                for (int i = 0; i < kWords; ++i) odd = odd || top[i] >= 0x7F800000u;
                if (__any_sync(0xFFFFFFFFu, odd)) {  // (alike in the four warps) values that are not finite do not count, and become NaN
#pragma unroll
                    for (int j = 0; j < kMine; ++j) {
                        const uint32_t t = __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(finite_magnitude(z[j])));
                        if (lane == (j & 31)) top[j >> 5] = t;
                        if (!finite(z[j])) z[j] = __uint_as_float(0x7FC00000u);
                    }
                    exchange(place + kGroups * 4 * kMine);
                }
                float inverse[kWords];
                const int b = x.n0 / kBlock;
#pragma unroll
                for (int i = 0; i < kWords; ++i) {
                    const int byte = scale_byte(__uint_as_float(top[i])), col = i * 32 + lane;
                    inverse[i] = scale_inverse(byte);
                    if (part == 0 && col < kMine && col < cols && x.n0 < o.N) {
                        uint8_t* const s = o.zs + scale_index(b, m0 + col, o.ldzs);
                        *s = (uint8_t)byte;
                        if (b == (o.N - 1) / kBlock)      // zeros behind the row's last block
                            for (int k = 1; (b + k) & 3; ++k) s[k] = 0;
                    }
                }
                const auto two_codes = [&](int j) {  // of columns j, j + 1
                    unsigned short two;
                    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;"
                        : "=h"(two)
                        : "f"(__fmul_rn(z[j + 1], __shfl_sync(0xFFFFFFFFu, inverse[(j + 1) >> 5], (j + 1) & 31))),
                          "f"(__fmul_rn(z[j], __shfl_sync(0xFFFFFFFFu, inverse[j >> 5], j & 31))));
                    return two;
                };
                uint8_t* const to = o.z8 + m0 * o.ldz8 + n;
                const bool stored = n < (o.N + 15) / 16 * 16;
#pragma unroll
                for (int j = 0; j < kMine; j += 2) {
                    const unsigned short two = two_codes(j);
                    if (all || (stored && j < cols)) to[j * o.ldz8] = (uint8_t)two;
                    if (all || (stored && j + 1 < cols)) to[(j + 1) * o.ldz8] = (uint8_t)(two >> 8);
                }
            }
        }
    }
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0 && given_up) atomicAdd(&g_ffn_timeouts, 1u);
    if constexpr (JOIN || PAIR) __syncwarp();
    if constexpr (JOIN) {
        // A block that gave up has no part, and then none of the cluster's blocks writes anything of the tile.
        cluster_wait();
        if (given_up && threadIdx.x < a.splits) word_to_block(smem_address(const_cast<const int*>(&given_up)), threadIdx.x, 1u);
        __syncwarp();
        cluster_sync();
        const FfnUnit x = ffn_unit<BN, PAIR>(a, first, 0);
        const int cols = given_up ? 0 : min(BN, a.M - x.m0);
        for (int c = warp * a.splits + x.split; c < cols; c += kFfnThreads / 32 * a.splits) {
            const uint32_t at = smem_address(smem) + (c * kLanes + lane * 4) * 4;
            float4 g = load_from_block(at, 0), v = load_from_block(at + BN * kLanes * 4, 0);
            for (int k = 1; k < a.splits; ++k) {
                const float4 g1 = load_from_block(at, k), v1 = load_from_block(at + BN * kLanes * 4, k);
                g = make_float4(__fadd_rn(g.x, g1.x), __fadd_rn(g.y, g1.y), __fadd_rn(g.z, g1.z), __fadd_rn(g.w, g1.w));
                v = make_float4(__fadd_rn(v.x, v1.x), __fadd_rn(v.y, v1.y), __fadd_rn(v.z, v1.z), __fadd_rn(v.w, v1.w));
            }
            finish<ACT>(a.out, x.m0 + c, x.n0, g, v);
        }
        __syncwarp();
        cluster_sync();                              // this block's memory stays until the others have read it
    }
    if constexpr (PAIR) cluster_sync();              // the other block's arrivals and products reach into this one
    if (warp == 3) {
        if constexpr (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(S::kAlloc));
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(S::kAlloc));
    }
}

// ---------------------------------------------------------------------------- backward
// dg = dz u act'(g), du = dz act(g), side by side [M x 2 N], to the block format along rows and along columns and / or to bf16.  A block takes a
// tile of 128 x 128 of the result, which is a whole block of each of its rows and columns.
struct FfnBackward {
    QuantOut out;
    int N;
    const __nv_bfloat16* gu;
    const void* dz;
    __nv_bfloat16* dgu;
    int64_t ldgu, lddz, lddgu;
    int wide, wide_out;                        // eight neighbours may be loaded, stored at once
};

// Where N is a multiple of the block, a block of threads takes a tile of dg and the one of du that comes from the same sums: these are read, and the activation
// is computed, once; du waits in shared memory, each thread's own, while dg is written (4096 x 4096 from bf16: 53 us; tile by tile 64).
template <typename T, int ACT>
__global__ void __launch_bounds__(kQThreads, 2) gated_ffn_backward_kernel(const FfnBackward a)
{
    constexpr int kRows = kPatchRows;
    extern __shared__ __align__(16) float4 waiting[];      // [half a row][thread]
    __shared__ QuantRoom room;
    const int lane = threadIdx.x & 15, patch = threadIdx.x >> 4;
    const int tiles_c = a.N / kTile;
    const int br = (int)(blockIdx.x / (unsigned)tiles_c), bc = (int)(blockIdx.x % (unsigned)tiles_c);
    const int row0 = br * kTile + patch * kRows, col0 = bc * kTile + lane * 8, rows = (int)a.out.rows - row0;
    const T* const dz = static_cast<const T*>(a.dz);
    after_previous();
    f8 x[kRows];
    Raw8<__nv_bfloat16> g[kRows], u[kRows];
    Raw8<T> d[kRows];
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
        const int here = k < rows ? 8 : 0;
        const int64_t m = row0 + k;
        g[k].load(a.gu + m * a.ldgu + col0, a.wide && here == 8, here);
        u[k].load(a.gu + m * a.ldgu + a.N + col0, a.wide && here == 8, here);
        d[k].load(dz + m * a.lddz + col0, a.wide && here == 8, here);
    }
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
        const f8 gk = g[k].values(), uk = u[k].values(), dk = d[k].values();
        f8 y;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float value, slope;
            activation<ACT>(gk.v[j], value, slope);
            x[k].v[j] = __fmul_rn(__fmul_rn(dk.v[j], uk.v[j]), slope);
            y.v[j] = __fmul_rn(dk.v[j], value);
        }
        waiting[2 * k * kQThreads + threadIdx.x] = make_float4(y.v[0], y.v[1], y.v[2], y.v[3]);
        waiting[(2 * k + 1) * kQThreads + threadIdx.x] = make_float4(y.v[4], y.v[5], y.v[6], y.v[7]);
    }
    const auto write = [&](int col, int tile) {
        if (a.dgu) {
#pragma unroll
            for (int k = 0; k < kRows; ++k) store_some(a.dgu + (row0 + k) * a.lddgu + col, x[k], a.wide_out && k < rows, k < rows ? 8 : 0);
        }
        if (a.out.q || a.out.qt) quantize_tile<true>(a.out, room, x, br, tile);
    };
    write(col0, bc);
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
        const float4 lo = waiting[2 * k * kQThreads + threadIdx.x], hi = waiting[(2 * k + 1) * kQThreads + threadIdx.x];
        x[k] = f8{{lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w}};
    }
    write(a.N + col0, tiles_c + bc);
}

// Any N: a tile of the result by itself, which may have columns of both.
template <typename T, int ACT>
__global__ void __launch_bounds__(kQThreads, 2) gated_ffn_backward_any_kernel(const FfnBackward a)
{
    constexpr int kRows = kPatchRows;
    __shared__ QuantRoom room;
    const int lane = threadIdx.x & 15, patch = threadIdx.x >> 4;
    const int tiles_c = (int)((a.out.cols + kTile - 1) / kTile);
    const int br = (int)(blockIdx.x / (unsigned)tiles_c), bc = (int)(blockIdx.x % (unsigned)tiles_c);
    const int row0 = br * kTile + patch * kRows, col0 = bc * kTile + lane * 8;
    const int left = max(0, min(8, (int)a.out.cols - col0)), rows = (int)a.out.rows - row0;
    const T* const dz = static_cast<const T*>(a.dz);
    after_previous();
    f8 x[kRows];
    const auto gradient = [&](float g, float u, float d, bool of_gate) {
        float value, slope;
        activation<ACT>(g, value, slope);
        return of_gate ? __fmul_rn(__fmul_rn(d, u), slope) : __fmul_rn(d, value);
    };
    const bool of_gate = col0 < a.N;
    const int n = of_gate ? col0 : col0 - a.N;
    if (a.wide && left == 8 && (!of_gate || n + 8 <= a.N)) {
        Raw8<__nv_bfloat16> g[kRows], u[kRows];
        Raw8<T> d[kRows];
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
            const int here = k < rows ? 8 : 0;
            const int64_t m = row0 + k;
            g[k].load(a.gu + m * a.ldgu + n, here == 8, here);
            u[k].load(a.gu + m * a.ldgu + a.N + n, here == 8 && of_gate, of_gate ? here : 0);
            d[k].load(dz + m * a.lddz + n, here == 8, here);
        }
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
            const f8 gk = g[k].values(), uk = u[k].values(), dk = d[k].values();
#pragma unroll
            for (int j = 0; j < 8; ++j) x[k].v[j] = gradient(gk.v[j], uk.v[j], dk.v[j], of_gate);
        }
    } else {
#pragma unroll
        for (int k = 0; k < kRows; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                x[k].v[j] = 0.f;
                if (k < rows && j < left) {
                    const int64_t m = row0 + k;
                    const bool gate = col0 + j < a.N;
                    const int c = gate ? col0 + j : col0 + j - a.N;
                    x[k].v[j] = gradient(load1(a.gu + m * a.ldgu + c), load1(a.gu + m * a.ldgu + a.N + c), load1(dz + m * a.lddz + c), gate);
                }
            }
    }
    if (a.dgu) {
#pragma unroll
        for (int k = 0; k < kRows; ++k) store_some(a.dgu + (row0 + k) * a.lddgu + col0, x[k], a.wide_out && k < rows && left == 8, k < rows ? left : 0);
    }
    if (a.out.q || a.out.qt) quantize_tile<true>(a.out, room, x, br, bc);
}

template <typename T, int ACT>
int backward_launch(const FfnBackward& a, cudaStream_t s)
{
    const char* what = "hpsgd_gated_ffn_backward";
    const int64_t tiles_r = (a.out.rows + kTile - 1) / kTile;
    if (a.N % kTile != 0) return launch_early(what, gated_ffn_backward_any_kernel<T, ACT>, dim3((unsigned)(tiles_r * ((a.out.cols + kTile - 1) / kTile))), kQThreads, 0, s, a);
    constexpr int kSmem = kTile * kTile * 4;
    static bool ready[64] = {};
    int dev = 0;
    OPS_CUDA(cudaGetDevice(&dev));
    if (dev >= 64 || !ready[dev]) {
        OPS_CUDA(cudaFuncSetAttribute(gated_ffn_backward_kernel<T, ACT>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem));
        if (dev < 64) ready[dev] = true;
    }
    return launch_early(what, gated_ffn_backward_kernel<T, ACT>, dim3((unsigned)(tiles_r * (a.N / kTile))), kQThreads, kSmem, s, a);
}

// ---------------------------------------------------------------------------- host side
struct FfnPlan {
    int bn, pair, tiles_n, tiles, splits, per_split, longer;
};

constexpr int kPairTokens = 224;           // 2 x 224 accumulator columns and four groups' scales are the 512 columns of tensor memory

// The least power of two that holds all tokens, 128 at most; or 224 on pairs of SMs, which takes fewer bytes out of L2 for a product, but keeps both SMs from the
// next tile's products while the sums go through the activation.  In a round of tiles an SM spent 0.47 us for each k block and 1.2 us more (3.4 where the
// sums are kept) on 128 tokens, and 0.78 and 1.2 (6.3) on its half of a pair's: 8192 x 8192 x 2048 242 us on single SMs, 219 on pairs; 4096 x 4096 x 1024 with
// the sums kept 53 and 66.  The fewer of these, rounds counted whole.  (Sizes that it was not made from: 1001 x 2744 x 1000 22.6 us either way and with the sums kept
// 26.6 where single SMs take 24.6; 3000 x 5000 x 3000 90 and 94; from 256 to 2048 tokens x 4096 x 1024 single SMs, which are 6 to 12 us faster.)
//
// Few tiles are split along k over the blocks of a cluster, as in hpsgd_gemm.cu.
FfnPlan plan_of(int64_t M, int64_t N, int64_t K, bool keep)
{
    const auto up = [](int64_t x, int64_t y) { return (x + y - 1) / y; };
    FfnPlan p{};
    const int blocks = (int)up(K, kStageK);
    p.bn = M <= 16 ? 16 : M <= 32 ? 32 : M <= 64 ? 64 : 128;
    int64_t tiles_n = up(N, kLanes), tiles = tiles_n * up(M, p.bn);
    if (M > 128) {
        const int64_t pairs_n = up(N, 2 * kLanes), pairs = pairs_n * up(M, kPairTokens);
        if ((double)up(pairs, kSms / 2) * (78.0 * blocks + (keep ? 630.0 : 120.0)) < (double)up(tiles, kSms) * (47.0 * blocks + (keep ? 340.0 : 120.0))) {
            p.pair = 1;
            p.bn = kPairTokens;
            tiles_n = pairs_n;
            tiles = pairs;
        }
    }
    p.tiles_n = (int)tiles_n;
    p.tiles = (int)tiles;
    p.splits = 1;
    if (!p.pair && p.tiles <= kSms / 2 && blocks >= 8) p.splits = p.tiles > 32 ? 2 : p.tiles > 14 || blocks < 32 ? 4 : 8;
    p.per_split = blocks / p.splits;
    p.longer = blocks % p.splits;
    return p;
}

template <int BN, bool PAIR, bool JOIN, int ACT>
int forward_act(const CUtensorMap& mx, const CUtensorMap& mw, const FfnArgs& a, int sms, cudaStream_t s)
{
    using S = FfnShape<BN, PAIR>;
    const auto kernel = gated_ffn_kernel<BN, PAIR, JOIN, ACT>;
    // Per device: the blocks (or pairs) that it holds at a time; pairs need both their SMs in one GPU cluster, so there may be fewer than half the SMs.
    static int workers[64] = {};
    int dev = 0;
    OPS_CUDA(cudaGetDevice(&dev));
    int at_once = dev < 64 ? workers[dev] : 0;
    if (at_once == 0) {
        OPS_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem));
        at_once = sms;
        if (PAIR) {
            cudaLaunchConfig_t cfg{};
            cudaLaunchAttribute attr{};
            cfg.gridDim = dim3(2);
            cfg.blockDim = dim3(kFfnThreads);
            cfg.dynamicSmemBytes = S::kSmem;
            attr.id = cudaLaunchAttributeClusterDimension;
            attr.val.clusterDim.x = 2;
            attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
            cfg.attrs = &attr;
            cfg.numAttrs = 1;
            OPS_CUDA(cudaOccupancyMaxActiveClusters(&at_once, kernel, &cfg));
        }
        at_once = std::max(1, at_once);
        if (dev < 64) workers[dev] = at_once;
    }
    const int64_t units = (int64_t)a.tiles * a.splits, blocks = JOIN ? units : std::min<int64_t>(units, at_once);
    return launch_clusters("hpsgd_gated_ffn_forward", kernel, dim3((unsigned)((PAIR ? 2 : 1) * blocks)), kFfnThreads, S::kSmem, PAIR ? 2 : JOIN ? a.splits : 1, s, mx, mw, a);
}

template <int BN, bool PAIR, bool JOIN>
int forward_launch(int act, const CUtensorMap& mx, const CUtensorMap& mw, const FfnArgs& a, int sms, cudaStream_t s)
{
    return act == HPSGD_SILU ? forward_act<BN, PAIR, JOIN, HPSGD_SILU>(mx, mw, a, sms, s) : forward_act<BN, PAIR, JOIN, HPSGD_GELU>(mx, mw, a, sms, s);
}

template <bool JOIN>
int forward_shape(const FfnPlan& p, int act, const CUtensorMap& mx, const CUtensorMap& mw, const FfnArgs& a, int sms, cudaStream_t s)
{
    switch (p.bn) {
    case 16: return forward_launch<16, false, JOIN>(act, mx, mw, a, sms, s);
    case 32: return forward_launch<32, false, JOIN>(act, mx, mw, a, sms, s);
    case 64: return forward_launch<64, false, JOIN>(act, mx, mw, a, sms, s);
    case 128: return forward_launch<128, false, JOIN>(act, mx, mw, a, sms, s);
    default: return forward_launch<kPairTokens, true, false>(act, mx, mw, a, sms, s);
    }
}

int check_act(const char* what, int act)
{
    return act == HPSGD_SILU || act == HPSGD_GELU ? HPSGD_OK : report(HPSGD_E_BADARG, "%s: unknown activation %d", what, act);
}

// Rows of a plain matrix; *wide: `unit` elements may be taken at once.
int check_plain(const char* what, const char* name, const void* p, int64_t* ld, int64_t cols, int64_t esz, int64_t unit, bool* wide)
{
    if (*ld == 0) *ld = cols;
    if (!p) return HPSGD_OK;
    if (*ld < cols) return report(HPSGD_E_BADARG, "%s: the stride of %s is below its row's length", what, name);
    if (!aligned(p, esz)) return report(HPSGD_E_BADARG, "%s: %s is not aligned to its elements", what, name);
    *wide = *wide && aligned(p, unit * esz) && *ld % unit == 0;
    return HPSGD_OK;
}

}  // namespace

// Time-outs of this file's kernels since the last report; and the count set to 0, for which the device has to be idle.
HPSGD_HIDDEN int ffn_timeouts(unsigned int* n)
{
    OPS_CUDA(cudaMemcpyFromSymbol(n, g_ffn_timeouts, sizeof *n));
    return HPSGD_OK;
}
HPSGD_HIDDEN int clear_ffn_timeouts()
{
    const unsigned int zero = 0;
    OPS_CUDA(cudaMemcpyToSymbol(g_ffn_timeouts, &zero, sizeof zero));
    return HPSGD_OK;
}

}  // namespace ops
}  // namespace hpsgd

using namespace hpsgd;
using namespace hpsgd::ops;

extern "C" {

int hpsgd_gated_ffn_forward(const hpsgd_gated_ffn_forward_args* args, void* stream)
{
    const char* what = "hpsgd_gated_ffn_forward";
    if (!args) return report(HPSGD_E_BADARG, "%s: args is NULL", what);
    hpsgd_gated_ffn_forward_args p = *args;
    if (p.M < 0 || p.N < 0 || p.K < 0) return report(HPSGD_E_BADARG, "%s: a size is negative", what);
    const int64_t most = 0x7FFFFFFF - 4096;
    if (p.M > most || p.N > most / 2 || p.K > most || ((p.N + 127) / 128) * ((p.M + 15) / 16) > most / 8) return report(HPSGD_E_UNSUPPORTED, "%s: a size is too large", what);
    OPS_TRY(check_act(what, p.act));
    if (p.z_dtype != HPSGD_F32 && p.z_dtype != HPSGD_BF16) return report(HPSGD_E_BADARG, "%s: unknown z_dtype %d", what, p.z_dtype);
    if (p.M == 0 || p.N == 0) return HPSGD_OK;
    if (p.K == 0) return report(HPSGD_E_BADARG, "%s: K is 0", what);
    if (!p.x || !p.w) return report(HPSGD_E_BADARG, "%s: x or w is NULL", what);
    if (!p.z8 && !p.z) return report(HPSGD_E_BADARG, "%s: no output is asked for", what);
    OPS_TRY(check_fp8(what, "x", p.x, p.x_scale, &p.ldx, &p.ldsx, p.M, p.K));
    OPS_TRY(check_fp8(what, "w", p.w, p.w_scale, &p.ldw, &p.ldsw, 2 * p.N, p.K));
    OPS_TRY(check_fp8(what, "z8", p.z8, p.z_scale, &p.ldz8, &p.ldsz, p.M, p.N));
    bool wide_z = true, wide_gu = p.N % 4 == 0;
    OPS_TRY(check_plain(what, "z", p.z, &p.ldz, p.N, p.z_dtype == HPSGD_F32 ? 4 : 2, 4, &wide_z));
    OPS_TRY(check_plain(what, "gu", p.gu, &p.ldgu, 2 * p.N, 2, 4, &wide_gu));
    int sms = 0;
    OPS_TRY(device_sms(&sms));
    const FfnPlan plan = plan_of(p.M, p.N, p.K, p.gu != nullptr);
    CUtensorMap mx, mw;
    OPS_TRY(make_map(what, &mx, p.x, p.ldx, p.M, p.K, plan.pair ? plan.bn / 2 : plan.bn));
    OPS_TRY(make_map(what, &mw, p.w, p.ldw, 2 * p.N, p.K, kLanes));
    FfnArgs a{};
    a.out = FfnOut{(int)p.N, static_cast<uint8_t*>(p.z8), p.z_scale, p.z, static_cast<__nv_bfloat16*>(p.gu), p.ldz8, p.ldsz, p.ldz, p.ldgu,
                   p.z_dtype == HPSGD_BF16, wide_z, wide_gu};
    a.M = (int)p.M; a.K = (int)p.K;
    a.tiles_n = plan.tiles_n; a.tiles = plan.tiles; a.splits = plan.splits; a.per_split = plan.per_split; a.longer = plan.longer;
    a.sx = reinterpret_cast<const uint32_t*>(p.x_scale); a.sw = reinterpret_cast<const uint32_t*>(p.w_scale);
    a.ldsx = p.ldsx; a.ldsw = p.ldsw;
    a.stall = stall_mode() ? 16 : 0;
    a.stall_odd = stall_mode() == 2;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    return plan.splits > 1 ? forward_shape<true>(plan, p.act, mx, mw, a, sms, s) : forward_shape<false>(plan, p.act, mx, mw, a, sms, s);
}

int hpsgd_gated_ffn_backward(const hpsgd_gated_ffn_backward_args* args, void* stream)
{
    const char* what = "hpsgd_gated_ffn_backward";
    if (!args) return report(HPSGD_E_BADARG, "%s: args is NULL", what);
    hpsgd_gated_ffn_backward_args p = *args;
    if (p.M < 0 || p.N < 0) return report(HPSGD_E_BADARG, "%s: a size is negative", what);
    const int64_t most = 0x7FFFFFFF - 4096;
    if (p.M > most || p.N > most / 2 || ((p.M + 127) / 128) * ((2 * p.N + 127) / 128) > most) return report(HPSGD_E_UNSUPPORTED, "%s: a size is too large", what);
    OPS_TRY(check_act(what, p.act));
    if (p.dz_dtype != HPSGD_F32 && p.dz_dtype != HPSGD_BF16) return report(HPSGD_E_BADARG, "%s: unknown dz_dtype %d", what, p.dz_dtype);
    if (p.M == 0 || p.N == 0) return HPSGD_OK;
    if (!p.gu || !p.dz) return report(HPSGD_E_BADARG, "%s: gu or dz is NULL", what);
    if (!p.dq && !p.dqt && !p.dgu) return report(HPSGD_E_BADARG, "%s: no output is asked for", what);
    if (p.dgu == p.gu) return report(HPSGD_E_BADARG, "%s: dgu is gu's memory, which is read more than once", what);
    bool wide = p.N % 8 == 0, wide_out = true;
    OPS_TRY(check_plain(what, "gu", p.gu, &p.ldgu, 2 * p.N, 2, 8, &wide));
    OPS_TRY(check_plain(what, "dz", p.dz, &p.lddz, p.N, p.dz_dtype == HPSGD_F32 ? 4 : 2, 8, &wide));
    OPS_TRY(check_plain(what, "dgu", p.dgu, &p.lddgu, 2 * p.N, 2, 8, &wide_out));
    OPS_TRY(check_fp8(what, "dq", p.dq, p.dq_scale, &p.lddq, &p.ldsdq, p.M, 2 * p.N));
    OPS_TRY(check_fp8(what, "dqt", p.dqt, p.dqt_scale, &p.lddqt, &p.ldsdqt, 2 * p.N, p.M));
    int sms = 0;
    OPS_TRY(device_sms(&sms));
    FfnBackward a{};
    a.out = QuantOut{p.M, 2 * p.N, p.lddq, p.ldsdq, p.lddqt, p.ldsdqt, static_cast<uint8_t*>(p.dq), p.dq_scale, static_cast<uint8_t*>(p.dqt), p.dqt_scale};
    a.N = (int)p.N; a.gu = static_cast<const __nv_bfloat16*>(p.gu); a.dz = p.dz; a.dgu = static_cast<__nv_bfloat16*>(p.dgu);
    a.ldgu = p.ldgu; a.lddz = p.lddz; a.lddgu = p.lddgu; a.wide = wide; a.wide_out = wide_out;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (p.dz_dtype == HPSGD_F32) return p.act == HPSGD_SILU ? backward_launch<float, HPSGD_SILU>(a, s) : backward_launch<float, HPSGD_GELU>(a, s);
    return p.act == HPSGD_SILU ? backward_launch<__nv_bfloat16, HPSGD_SILU>(a, s) : backward_launch<__nv_bfloat16, HPSGD_GELU>(a, s);
}

}  // extern "C"
