// AdamW over many tensors (moments in 32 or in 8 bits) and the global norm of their gradients.
//
// Both are element-wise passes over HBM: a parameter costs 28 bytes a step with everything in 32 bits, 10 with
// bf16 parameters and gradients and moments in 8 bits, against some dozens of instructions.  As in the replica
// kernels the work is organised around the traffic: one 8-element group per thread and array, all loads requested
// before the first is used, many short blocks.  The table of tensors travels in the kernel's parameters, so a
// step needs no copy to the device and no workspace, and any mix of large and tiny tensors is one launch.
#include "hpsgd_ops_common.cuh"

#include <algorithm>
#include <cuda_fp16.h>

namespace hpsgd {
namespace ops {
namespace {

constexpr int kAdamThreads = 128;
constexpr int kChunk = kAdamThreads * 8;       // elements a block handles: eight 8-bit blocks
constexpr int kMaxItems = 360;                 // what 32764 bytes of kernel parameters hold

// Constants of the element's random bits: frac(sqrt 2, 3, 5) * 2^32 with the low bit set.
constexpr uint32_t kN1 = 0x6A09E667u, kN2 = 0xBB67AE85u, kN3 = 0x3C6EF373u;

struct Item {
    void* p;
    const void* g;
    void* m;
    void* v;
    uint8_t* ms;
    uint8_t* vs;
    __nv_bfloat16* copy;
    int64_t n;
    uint64_t rng;
    float keep;            // 1 - lr * weight_decay
    uint32_t first;        // first chunk of this tensor
    uint32_t wide;         // all addresses allow the wide accesses
    uint32_t pad;
};

template <int CAP>
struct Table {
    Item item[CAP];
    int count;
};

struct Hyper {
    float beta1, rest1, beta2, rest2;          // rest = 1 - beta, rounded once from binary64
    float rate;                                // lr / (1 - beta1^step)
    float root;                                // 1 / sqrt(1 - beta2^step)
    float eps;
    uint32_t key0, key1;
    const float* scale;
};

// The tensor that a chunk belongs to: the last whose first chunk is not behind it.
template <int CAP>
__device__ __forceinline__ int find_item(const Table<CAP>& t, uint32_t chunk)
{
    int lo = 0, hi = t.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (t.item[mid].first <= chunk) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

__device__ __forceinline__ uint32_t random_bits(uint32_t q, uint32_t key0, uint32_t key1)
{
    uint32_t x = (q ^ key0) * kN1;
    x ^= x >> 15;
    x = (x + key1) * kN2;
    x ^= x >> 14;
    x *= kN3;
    return x ^ x >> 16;
}

// Eight codes, as stored.
__device__ __forceinline__ uint2 load_codes(const uint8_t* p, bool wide, int left)
{
    if (wide) return *reinterpret_cast<const uint2*>(p);
    uint2 u = make_uint2(0u, 0u);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if (q < left) u.x |= (uint32_t)p[q] << 8 * q;
        if (q + 4 < left) u.y |= (uint32_t)p[q + 4] << 8 * q;
    }
    return u;
}

__device__ __forceinline__ void store_codes(uint8_t* p, uint2 u, bool wide, int left)
{
    if (wide) {
        *reinterpret_cast<uint2*>(p) = u;
        return;
    }
#pragma unroll
    for (int q = 0; q < 8; ++q)
        if (q < left) p[q] = (uint8_t)((q < 4 ? u.x : u.y) >> 8 * (q & 3));
}

// Two codes (the low 16 bits) to two values: the conversion goes through f16, which holds every E4M3 value and its NaN.
__device__ __forceinline__ void decode_pair(uint32_t two, float& lo, float& hi)
{
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((unsigned short)two));
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
    lo = f.x;
    hi = f.y;
}

__device__ __forceinline__ f8 decode8(uint2 u)
{
    f8 x;
    decode_pair(u.x, x.v[0], x.v[1]);
    decode_pair(u.x >> 16, x.v[2], x.v[3]);
    decode_pair(u.y, x.v[4], x.v[5]);
    decode_pair(u.y >> 16, x.v[6], x.v[7]);
    return x;
}

// What multiplies a value of a block with scale 2^(byte - 127) so that the value's E4M3 code comes to stand in bits 20..26 of
// its binary32 pattern: 2^(127 - byte - 120), in one factor as long as that is a normal number.  Blocks above 2^6 * 448, whose
// factor is not, first have their values multiplied by the rest (`excess`).
__device__ __forceinline__ float code_factor(int byte) { return __uint_as_float((uint32_t)(max(254 - 120 - byte, 1)) << 23); }
__device__ __forceinline__ bool has_excess(int byte) { return byte > 133; }
__device__ __forceinline__ float excess(int byte) { return __uint_as_float((uint32_t)(127 - (byte - 133)) << 23); }

// One of the two codes around |x|, such that the expected value is |x|; `x` is already multiplied by its block's code factor.
// 16 random bits, centred, are added below the last bit that is kept, and the carry decides.  An exact code stays.
// The code comes back in the top byte, sign included.
__device__ __forceinline__ uint32_t round_first(float x, uint32_t rnd)
{
    const uint32_t b = __float_as_uint(fabsf(x)) + ((rnd >> 12 & 0xFFFF0u) | 8u);
    return (b << 4 & 0x7F000000u) | (__float_as_uint(x) & 0x80000000u);
}

// One of the two codes a <= x < b, such that the expected square is x^2: b with probability (x^2 - a^2) / (b^2 - a^2), so where
// x^2 > a^2 + u (b^2 - a^2).  0 only for 0.  `t` is x multiplied by its block's code factor.  The code comes back in the top byte.
__device__ __forceinline__ uint32_t round_second(float t, uint32_t rnd)
{
    const uint32_t ab = __float_as_uint(t) & 0xFFF00000u;
    const float x = __fmul_rn(t, 0x1p120f);
    const float a = __fmul_rn(__uint_as_float(ab), 0x1p120f), b = __fmul_rn(__uint_as_float(ab + 0x100000u), 0x1p120f);
    const float u1 = __uint_as_float(0x3F800040u | (rnd << 7 & 0x7FFF80u));          // 1 + u, u = (16 bits + 0.5) / 2^16
    const float d = __fmul_rn(__fsub_rn(b, a), __fadd_rn(b, a));
    const bool up = __fmul_rn(__fsub_rn(x, a), __fadd_rn(x, a)) > __fmul_rn(__fsub_rn(u1, 1.f), d);
    const uint32_t c = (up ? ab + 0x100000u : ab) << 4;
    return max(c, t > 0.f ? 0x1000000u : 0u);
}

// Four codes from their top bytes.
__device__ __forceinline__ uint32_t gather_codes(uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    return __byte_perm(__byte_perm(a, b, 0x0073), __byte_perm(c, d, 0x0073), 0x5410);
}

__device__ __forceinline__ float root_approx(float x)
{
    float y;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// ---------------------------------------------------------------------------- the step
template <int CAP, typename P, typename G, bool B8>
__global__ void __launch_bounds__(kAdamThreads) adamw_kernel(const __grid_constant__ Table<CAP> table, const __grid_constant__ Hyper hy)
{
    const Item& it = table.item[find_item(table, blockIdx.x)];
    const int64_t at = (int64_t)(blockIdx.x - it.first) * kChunk + threadIdx.x * 8;
    const int64_t rest = it.n - at;
    const int left = rest < 0 ? 0 : rest > 8 ? 8 : (int)rest;
    const bool wide = it.wide && left == 8;
    float c = 1.f;
    if (hy.scale) {
        c = *hy.scale;
        if (!finite(c)) return;                   // the whole grid: nothing of the step happens
    }
    if (!B8 && left == 0) return;

    P* const pp = static_cast<P*>(it.p) + at;
    f8 p = load_some(pp, wide, left);
    f8 g = load_some(static_cast<const G*>(it.g) + at, wide, left);
    f8 m, v;
    if constexpr (B8) {
        const uint2 mc = load_codes(static_cast<const uint8_t*>(it.m) + at, wide, left);
        const uint2 vc = load_codes(static_cast<const uint8_t*>(it.v) + at, wide, left);
        int mb = 0, vb = 0;
        if (left > 0) {
            mb = it.ms[at / kBlock];
            vb = it.vs[at / kBlock];
        }
        const float sm = scale_value(mb), sv = scale_value(vb);
        m = decode8(mc);
        v = decode8(vc);
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            m.v[q] = __fmul_rn(m.v[q], sm);
            v.v[q] = __fmul_rn(v.v[q], sv);
            v.v[q] = __fmul_rn(v.v[q], v.v[q]);
        }
    } else {
        m = load_some(static_cast<const float*>(it.m) + at, wide, left);
        v = load_some(static_cast<const float*>(it.v) + at, wide, left);
    }

    // With 32-bit moments HBM is what bounds the kernel, and root and quotient are correctly rounded; with 8-bit moments
    // instructions are, and they are the hardware's approximations (2 units in the last place, of a step that is added to p).
    f8 r;                                          // sqrt(v), which the step divides by and the 8-bit form keeps
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        const float gq = __fmul_rn(g.v[q], c);
        m.v[q] = __fadd_rn(__fmul_rn(hy.beta1, m.v[q]), __fmul_rn(hy.rest1, gq));
        v.v[q] = __fadd_rn(__fmul_rn(hy.beta2, v.v[q]), __fmul_rn(hy.rest2, __fmul_rn(gq, gq)));
        r.v[q] = B8 ? root_approx(v.v[q]) : __fsqrt_rn(v.v[q]);
        const float below = __fmaf_rn(r.v[q], hy.root, hy.eps);
        const float step = B8 ? __fdividef(m.v[q], below) : __fdiv_rn(m.v[q], below);
        p.v[q] = __fmaf_rn(-hy.rate, step, __fmul_rn(p.v[q], it.keep));
    }

    uint32_t rnd[8];
    constexpr bool kPB = sizeof(P) == 2;
    if constexpr (B8 || kPB) {
        const uint64_t q0 = it.rng + (uint64_t)at;
        const uint32_t low = (uint32_t)q0, key1 = hy.key1 + (uint32_t)(q0 >> 32) * kN3;
        if (low <= 0xFFFFFFF8u) {
#pragma unroll
            for (int q = 0; q < 8; ++q) rnd[q] = random_bits(low + q, hy.key0, key1);
        } else {                                   // the position's upper half changes within the eight
#pragma unroll
            for (int q = 0; q < 8; ++q) rnd[q] = random_bits(low + q, hy.key0, low + q < low ? key1 + kN3 : key1);
        }
    }
    if constexpr (kPB) {
#pragma unroll
        for (int q = 0; q < 8; ++q) {              // exact in bf16 afterwards: the store's own rounding does nothing
            const uint32_t b = __float_as_uint(p.v[q]);
            if (finite(p.v[q])) p.v[q] = __uint_as_float(b + (rnd[q] * kN2 >> 16) & 0xFFFF0000u);
        }
    }
    store_some(pp, p, wide, left);
    if (it.copy) store_some(it.copy + at, p, wide, left);

    if constexpr (B8) {
        // Largest magnitudes of the block, as bit patterns: what is not finite comes out on top of every number.  Elements
        // behind the end of the tensor are zeros here (all their inputs are).
        uint32_t tm = 0, tr = 0;
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            tm = max(tm, __float_as_uint(fabsf(m.v[q])));
            tr = max(tr, __float_as_uint(fabsf(r.v[q])));
        }
        const uint32_t half = threadIdx.x & 16 ? 0xFFFF0000u : 0xFFFFu;       // the 16 lanes that hold the block
        uint32_t bm = __reduce_max_sync(half, tm), br = __reduce_max_sync(half, tr);
        const bool odd = max(bm, br) >= 0x7F800000u;
        if (odd) {                                 // rare: the scale is that of the finite values
            tm = tr = 0;
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                tm = max(tm, __float_as_uint(finite_magnitude(m.v[q])));
                tr = max(tr, __float_as_uint(finite_magnitude(r.v[q])));
            }
            bm = __reduce_max_sync(half, tm);
            br = __reduce_max_sync(half, tr);
        }
        const int mb = scale_byte(__uint_as_float(bm)), vb = scale_byte(__uint_as_float(br));
        f8 sm = m, sr = r;
        if (has_excess(mb) || has_excess(vb)) {
            const float em = has_excess(mb) ? excess(mb) : 1.f, er = has_excess(vb) ? excess(vb) : 1.f;
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                sm.v[q] = __fmul_rn(sm.v[q], em);
                sr.v[q] = __fmul_rn(sr.v[q], er);
            }
        }
        const float fm = code_factor(mb), fr = code_factor(vb);
        uint32_t cm[8], cr[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            cm[q] = round_first(__fmul_rn(sm.v[q], fm), rnd[q]);
            cr[q] = round_second(__fmul_rn(sr.v[q], fr), rnd[q]);
        }
        if (odd) {
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                if (!finite(m.v[q])) cm[q] = 0x7F000000u;
                if (!finite(r.v[q])) cr[q] = 0x7F000000u;
            }
        }
        store_codes(static_cast<uint8_t*>(it.m) + at, make_uint2(gather_codes(cm[0], cm[1], cm[2], cm[3]), gather_codes(cm[4], cm[5], cm[6], cm[7])), wide, left);
        store_codes(static_cast<uint8_t*>(it.v) + at, make_uint2(gather_codes(cr[0], cr[1], cr[2], cr[3]), gather_codes(cr[4], cr[5], cr[6], cr[7])), wide, left);
        if (left > 0 && (threadIdx.x & 15) == 0) {
            it.ms[at / kBlock] = (uint8_t)mb;
            it.vs[at / kBlock] = (uint8_t)vb;
        }
    } else {
        store_some(static_cast<float*>(it.m) + at, m, wide, left);
        store_some(static_cast<float*>(it.v) + at, v, wide, left);
    }
}

// ---------------------------------------------------------------------------- the norm
constexpr int kNormThreads = 256;
constexpr int kNormChunk = kNormThreads * 8 * 4;       // four groups of eight in flight per thread
constexpr int kNormPartials = (HPSGD_GRAD_NORM_WORKSPACE - 64) / 8;

struct NormOut {
    double max_norm;
    unsigned int* ticket;      // blocks that have finished; put back to 0 by the last
    double* partial;           // one per block of all launches of the call
    int before, total;         // blocks of earlier launches, blocks of all
    uint32_t chunks;
    float* out;
};

__device__ __forceinline__ double warp_sum(double x)
{
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, d);
    return x;
}

// Each block adds the chunks block, block + grid, ... of its launch; the last block of the call to finish adds the blocks' sums in
// their order, so the result does not depend on which one that is.
template <int CAP, typename G>
__global__ void __launch_bounds__(kNormThreads) grad_norm_kernel(const __grid_constant__ Table<CAP> table, const __grid_constant__ NormOut no)
{
    __shared__ double part[kNormThreads / 32];
    __shared__ bool last;
    double sum = 0.0;
    for (uint32_t chunk = blockIdx.x; chunk < no.chunks; chunk += gridDim.x) {
        const Item& it = table.item[find_item(table, chunk)];
        const G* const gp = static_cast<const G*>(it.g);
        const int64_t base = (int64_t)(chunk - it.first) * kNormChunk + threadIdx.x * 8;
        f8 x[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int64_t at = base + k * (kNormThreads * 8), rest = it.n - at;
            const int left = rest < 0 ? 0 : rest > 8 ? 8 : (int)rest;
            x[k] = load_some(gp + at, it.wide && left == 8, left);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float s = 0.f;
#pragma unroll
            for (int q = 0; q < 8; ++q) s = __fmaf_rn(x[k].v[q], x[k].v[q], s);
            sum += (double)s;
        }
    }
    sum = warp_sum(sum);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        double s = 0.0;
        for (int k = 0; k < kNormThreads / 32; ++k) s += part[k];
        no.partial[no.before + blockIdx.x] = s;
        __threadfence();
        last = atomicAdd(no.ticket, 1u) == (unsigned)(no.total - 1);
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    sum = 0.0;
    for (int k = threadIdx.x; k < no.total; k += kNormThreads) sum += __ldcg(no.partial + k);
    sum = warp_sum(sum);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        double s = 0.0;
        for (int k = 0; k < kNormThreads / 32; ++k) s += part[k];
        const double norm = sqrt(s);
        no.out[0] = (float)norm;
        no.out[1] = !finite((float)norm) ? __uint_as_float(0x7FC00000u) : norm > no.max_norm ? (float)(no.max_norm / norm) : 1.f;
        *no.ticket = 0u;
    }
}

// ---------------------------------------------------------------------------- host side
uint64_t mix(uint64_t x)
{
    x ^= x >> 32; x *= 0x6a09e667f3bcc909ULL;
    x ^= x >> 29; x *= 0xbb67ae8584caa73bULL;
    return x ^ x >> 32;
}

int check_table(const hpsgd_adamw_tensor* t, int n, int grad_dtype, const char* what)
{
    if (n < 0) return report(HPSGD_E_BADARG, "%s: n_tensors is negative", what);
    if (n > 0 && !t) return report(HPSGD_E_BADARG, "%s: tensors is NULL", what);
    if (grad_dtype != HPSGD_F32 && grad_dtype != HPSGD_BF16) return report(HPSGD_E_BADARG, "%s: unknown grad_dtype %d", what, grad_dtype);
    const size_t gs = grad_dtype == HPSGD_F32 ? 4 : 2;
    for (int k = 0; k < n; ++k) {
        if (t[k].n < 0) return report(HPSGD_E_BADARG, "%s: tensor %d has a negative size", what, k);
        if (t[k].n > (int64_t)1 << 40) return report(HPSGD_E_UNSUPPORTED, "%s: tensor %d has more than 2^40 elements", what, k);
        if (t[k].n == 0) continue;
        if (!t[k].grad) return report(HPSGD_E_BADARG, "%s: tensor %d: grad is NULL", what, k);
        if (!aligned(t[k].grad, gs)) return report(HPSGD_E_BADARG, "%s: tensor %d: grad is not aligned to its elements", what, k);
    }
    return HPSGD_OK;
}

// The next launch's worth of tensors starting at *at: fills `out` and returns its number of chunks.  Empty tensors are left out.
template <int CAP, typename Fill>
uint32_t fill_table(const hpsgd_adamw_tensor* t, int n, int* at, int64_t chunk_elems, Table<CAP>* out, Fill fill)
{
    uint64_t chunks = 0;
    out->count = 0;
    for (; *at < n && out->count < CAP; ++*at) {
        if (t[*at].n == 0) continue;
        const uint64_t here = (uint64_t)(t[*at].n + chunk_elems - 1) / chunk_elems;
        if (chunks + here > 0x7FFFFFFFull) break;      // a launch has at most that many blocks; 2^40 elements fit one alone
        Item& it = out->item[out->count++];
        it = Item{};
        it.n = t[*at].n;
        it.g = t[*at].grad;
        it.first = (uint32_t)chunks;
        fill(t[*at], &it);
        chunks += here;
    }
    return (uint32_t)chunks;
}

template <int CAP, typename P, typename G, bool B8>
int step_launches(const hpsgd_adamw_tensor* t, int n, double lr, const Hyper& hy, cudaStream_t s)
{
    const size_t ap = sizeof(P) == 4 ? 32 : 16, ag = sizeof(G) == 4 ? 32 : 16, as = B8 ? 8 : 32;
    int at = 0;
    Table<CAP> table;
    while (at < n) {
        const uint32_t chunks = fill_table(t, n, &at, kChunk, &table, [&](const hpsgd_adamw_tensor& x, Item* it) {
            it->p = x.param; it->m = x.m; it->v = x.v; it->ms = x.m_scale; it->vs = x.v_scale;
            it->copy = static_cast<__nv_bfloat16*>(x.copy);
            it->rng = x.rng_offset;
            it->keep = (float)(1.0 - lr * x.weight_decay);
            it->wide = aligned(x.param, ap) && aligned(x.grad, ag) && aligned(x.m, as) && aligned(x.v, as) && aligned(x.copy, 16);
        });
        if (!chunks) continue;
        adamw_kernel<CAP, P, G, B8><<<chunks, kAdamThreads, 0, s>>>(table, hy);
        OPS_TRY(launched("hpsgd_adamw_step"));
    }
    return HPSGD_OK;
}

template <int CAP>
int step_types(const hpsgd_adamw_tensor* t, int n, int pd, int gd, int bits, double lr, const Hyper& hy, cudaStream_t s)
{
    using bf = __nv_bfloat16;
    if (pd == HPSGD_F32 && gd == HPSGD_F32) return bits == 8 ? step_launches<CAP, float, float, true>(t, n, lr, hy, s) : step_launches<CAP, float, float, false>(t, n, lr, hy, s);
    if (pd == HPSGD_F32) return bits == 8 ? step_launches<CAP, float, bf, true>(t, n, lr, hy, s) : step_launches<CAP, float, bf, false>(t, n, lr, hy, s);
    if (gd == HPSGD_F32) return bits == 8 ? step_launches<CAP, bf, float, true>(t, n, lr, hy, s) : step_launches<CAP, bf, float, false>(t, n, lr, hy, s);
    return bits == 8 ? step_launches<CAP, bf, bf, true>(t, n, lr, hy, s) : step_launches<CAP, bf, bf, false>(t, n, lr, hy, s);
}

template <int CAP, typename G>
int norm_launches(const hpsgd_adamw_tensor* t, int n, int sms, double max_norm, void* ws, float* out, cudaStream_t s)
{
    // blocks of every launch, so that the last block of the last launch knows what it has to wait for
    Table<CAP> table;
    const auto fill = [](const hpsgd_adamw_tensor& x, Item* it) { it->wide = aligned(x.grad, sizeof(G) == 4 ? 32 : 16); };
    int at = 0, total = 0, launches = 0;
    while (at < n) {
        fill_table(t, n, &at, kNormChunk, &table, fill);
        ++launches;
    }
    const int most = std::max(1, std::min(sms * 8, kNormPartials / std::max(1, launches)));
    const auto grid_of = [&](uint32_t chunks) { return (int)std::min<uint32_t>(std::max<uint32_t>(chunks, 1), most); };
    at = 0;
    while (at < n) total += grid_of(fill_table(t, n, &at, kNormChunk, &table, fill));
    if (total == 0) total = 1;                     // no tensors: one block writes the norm of nothing
    NormOut no{max_norm, static_cast<unsigned int*>(ws), reinterpret_cast<double*>(static_cast<char*>(ws) + 64), 0, total, 0, out};
    at = 0;
    do {
        no.chunks = fill_table(t, n, &at, kNormChunk, &table, fill);
        const int grid = grid_of(no.chunks);
        grad_norm_kernel<CAP, G><<<grid, kNormThreads, 0, s>>>(table, no);
        OPS_TRY(launched("hpsgd_grad_norm"));
        no.before += grid;
    } while (at < n);
    return HPSGD_OK;
}

}  // namespace

int device_sms(int* sms)
{
    int dev = 0, major = 0;
    OPS_CUDA(cudaGetDevice(&dev));
    OPS_CUDA(cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev));
    if (major != 10) return report(HPSGD_E_CUDA, "built for sm_100a only; the device has compute capability %d.x", major);
    OPS_CUDA(cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, dev));
    return HPSGD_OK;
}

}  // namespace ops
}  // namespace hpsgd

using namespace hpsgd;
using namespace hpsgd::ops;

extern "C" {

int hpsgd_adamw_step(const hpsgd_adamw_tensor* tensors, int n_tensors, int param_dtype, int grad_dtype, int state_bits,
                     double lr, double beta1, double beta2, double eps, int64_t step, uint64_t seed, const float* grad_scale,
                     void* stream)
{
    const char* what = "hpsgd_adamw_step";
    OPS_TRY(check_table(tensors, n_tensors, grad_dtype, what));
    if (param_dtype != HPSGD_F32 && param_dtype != HPSGD_BF16) return report(HPSGD_E_BADARG, "%s: unknown param_dtype %d", what, param_dtype);
    if (state_bits != 8 && state_bits != 32) return report(HPSGD_E_BADARG, "%s: state_bits must be 8 or 32", what);
    if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0)) return report(HPSGD_E_BADARG, "%s: beta1 and beta2 must be in [0, 1)", what);
    if (!(eps > 0.0) || !std::isfinite(eps) || (float)eps == 0.f) return report(HPSGD_E_BADARG, "%s: eps must be positive in binary32", what);
    if (!(lr >= 0.0) || !std::isfinite(lr)) return report(HPSGD_E_BADARG, "%s: lr must be >= 0", what);
    if (step < 1) return report(HPSGD_E_BADARG, "%s: step counts from 1", what);
    if (!aligned(grad_scale, 4)) return report(HPSGD_E_BADARG, "%s: grad_scale is not 4-byte aligned", what);
    for (int k = 0; k < n_tensors; ++k) {
        const hpsgd_adamw_tensor& t = tensors[k];
        if (!(t.weight_decay >= 0.0) || !std::isfinite(t.weight_decay)) return report(HPSGD_E_BADARG, "%s: tensor %d: weight_decay must be >= 0", what, k);
        if (t.n == 0) continue;
        if (!t.param || !t.m || !t.v) return report(HPSGD_E_BADARG, "%s: tensor %d: param, m or v is NULL", what, k);
        if (state_bits == 8 && (!t.m_scale || !t.v_scale)) return report(HPSGD_E_BADARG, "%s: tensor %d: m_scale or v_scale is NULL", what, k);
        if (!aligned(t.param, param_dtype == HPSGD_F32 ? 4 : 2) || !aligned(t.copy, 2) ||
            (state_bits == 32 && (!aligned(t.m, 4) || !aligned(t.v, 4))))
            return report(HPSGD_E_BADARG, "%s: tensor %d: an address is not aligned to its elements", what, k);
        if (t.copy && param_dtype != HPSGD_F32) return report(HPSGD_E_BADARG, "%s: tensor %d: a bf16 copy goes with fp32 parameters only", what, k);
    }
    int sms = 0;
    OPS_TRY(device_sms(&sms));
    Hyper hy{};
    hy.beta1 = (float)beta1; hy.rest1 = (float)(1.0 - beta1);
    hy.beta2 = (float)beta2; hy.rest2 = (float)(1.0 - beta2);
    hy.rate = (float)(lr / (1.0 - std::pow(beta1, (double)step)));
    hy.root = (float)(1.0 / std::sqrt(1.0 - std::pow(beta2, (double)step)));
    hy.eps = (float)eps;
    const uint64_t key = mix((mix(seed + 0x3c6ef372fe94f82bULL) ^ (uint64_t)step) + 0xa54ff53a5f1d36f1ULL);
    hy.key0 = (uint32_t)key; hy.key1 = (uint32_t)(key >> 32);
    hy.scale = grad_scale;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (n_tensors <= 8) return step_types<8>(tensors, n_tensors, param_dtype, grad_dtype, state_bits, lr, hy, s);
    return step_types<kMaxItems>(tensors, n_tensors, param_dtype, grad_dtype, state_bits, lr, hy, s);
}

int hpsgd_grad_norm(const hpsgd_adamw_tensor* tensors, int n_tensors, int grad_dtype, double max_norm, void* workspace, float* out,
                    void* stream)
{
    const char* what = "hpsgd_grad_norm";
    OPS_TRY(check_table(tensors, n_tensors, grad_dtype, what));
    if (!(max_norm > 0.0)) return report(HPSGD_E_BADARG, "%s: max_norm must be positive", what);
    if (!workspace || !aligned(workspace, 16)) return report(HPSGD_E_BADARG, "%s: workspace is NULL or not 16-byte aligned", what);
    if (!out || !aligned(out, 4)) return report(HPSGD_E_BADARG, "%s: out is NULL or not 4-byte aligned", what);
    int sms = 0;
    OPS_TRY(device_sms(&sms));
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool f = grad_dtype == HPSGD_F32;
    if (n_tensors <= 8)
        return f ? norm_launches<8, float>(tensors, n_tensors, sms, max_norm, workspace, out, s)
                 : norm_launches<8, __nv_bfloat16>(tensors, n_tensors, sms, max_norm, workspace, out, s);
    return f ? norm_launches<kMaxItems, float>(tensors, n_tensors, sms, max_norm, workspace, out, s)
             : norm_launches<kMaxItems, __nv_bfloat16>(tensors, n_tensors, sms, max_norm, workspace, out, s);
}

}  // extern "C"
