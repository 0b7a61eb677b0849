// What the operators share: the 8-bit block format, wide loads and stores, argument and device checks.
#pragma once

#include "../../include/hpsgd_ops.h"

#include <cmath>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "hpsgd_internal.h"

namespace hpsgd {
namespace ops {

#define OPS_CUDA(expr)                                                                             \
    do {                                                                                           \
        cudaError_t e_ = (expr);                                                                   \
        if (e_ != cudaSuccess) {                                                                   \
            cudaGetLastError();                                                                    \
            return report(HPSGD_E_CUDA, "%s failed: %s", #expr, cudaGetErrorString(e_));           \
        }                                                                                          \
    } while (0)

#define OPS_TRY(expr)            \
    do {                         \
        int rc_ = (expr);        \
        if (rc_) return rc_;     \
    } while (0)

// SM count of the current device, after checking that the kernels can run on it.
HPSGD_HIDDEN int device_sms(int* sms);

// What a kernel launch just did, as a status.
inline int launched(const char* what)
{
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return report(HPSGD_E_CUDA, "%s: launch failed: %s", what, cudaGetErrorString(e));
    count_launches(1);
    return HPSGD_OK;
}

// Launch a kernel whose blocks may be set up while the one before it on the stream still runs (programmatic dependent launch): its
// parameters are fetched and its barriers made by the time its input is there.  Such a kernel calls after_previous() before it touches
// global memory, in every thread that does, and that waits for the whole of the kernel before it; so nothing changes for the caller.  Between
// two small kernels it takes 1 to 2 us off.
template <typename Kernel, typename... Args>
inline int launch_early(const char* what, Kernel kernel, dim3 grid, int threads, size_t smem, cudaStream_t s, const Args&... args)
{
    cudaLaunchConfig_t cfg{};
    cudaLaunchAttribute attr{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, args...);
    if (e != cudaSuccess) {
        cudaGetLastError();
        return report(HPSGD_E_CUDA, "%s: launch failed: %s", what, cudaGetErrorString(e));
    }
    return launched(what);
}

__device__ __forceinline__ void after_previous()
{
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");      // the next kernel's blocks may be set up from here on
    asm volatile("griddepcontrol.wait;" ::: "memory");
}

inline bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

// ---------------------------------------------------------------------------- the 8-bit block format
constexpr int kBlock = 128;

// Exponent byte e + 127 of a block whose largest finite magnitude is `top`: 448 = 1.75 * 2^8, so with
// top = 1.f * 2^k the exponent is k - 8, or k - 7 where 1.f > 1.75.
__device__ __forceinline__ int scale_byte(float top)
{
    const uint32_t b = __float_as_uint(top);
    const int k = (int)(b >> 23);                               // k + 127; 0 for subnormal values, whose scale is 2^-127 anyway
    return max(0, k - 8 + ((b & 0x7FFFFFu) > 0x600000u ? 1 : 0));
}

// 2^(byte - 127) and 2^(127 - byte), exactly; bytes up to 247 (those of finite blocks) keep both normal
// but for 2^-127 itself.
__device__ __forceinline__ float scale_value(int byte)
{
    return __uint_as_float(byte > 0 ? (uint32_t)byte << 23 : 0x400000u);
}
__device__ __forceinline__ float scale_inverse(int byte) { return __uint_as_float((uint32_t)(254 - byte) << 23); }

__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7F800000u) != 0x7F800000u; }
__device__ __forceinline__ float finite_magnitude(float x) { return finite(x) ? fabsf(x) : 0.f; }

// ---------------------------------------------------------------------------- eight consecutive values
struct f8 {
    float v[8];
};

__device__ __forceinline__ void widen_pair(uint32_t u, float& lo, float& hi)
{
    lo = __uint_as_float(u << 16);
    hi = __uint_as_float(u & 0xFFFF0000u);
}

__device__ __forceinline__ f8 load8(const float* p)
{
    f8 x;
    asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=f"(x.v[0]), "=f"(x.v[1]), "=f"(x.v[2]), "=f"(x.v[3]), "=f"(x.v[4]), "=f"(x.v[5]), "=f"(x.v[6]), "=f"(x.v[7])
                 : "l"(p));
    return x;
}

__device__ __forceinline__ void store8(float* p, const f8& x)
{
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "f"(x.v[0]), "f"(x.v[1]), "f"(x.v[2]),
                 "f"(x.v[3]), "f"(x.v[4]), "f"(x.v[5]), "f"(x.v[6]), "f"(x.v[7])
                 : "memory");
}

__device__ __forceinline__ f8 load8(const __nv_bfloat16* p)
{
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    f8 x;
    widen_pair(u.x, x.v[0], x.v[1]);
    widen_pair(u.y, x.v[2], x.v[3]);
    widen_pair(u.z, x.v[4], x.v[5]);
    widen_pair(u.w, x.v[6], x.v[7]);
    return x;
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    uint32_t u;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(u) : "f"(hi), "f"(lo));
    return u;
}

__device__ __forceinline__ void store8(__nv_bfloat16* p, const f8& x)
{
    *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16(x.v[0], x.v[1]), pack_bf16(x.v[2], x.v[3]),
                                              pack_bf16(x.v[4], x.v[5]), pack_bf16(x.v[6], x.v[7]));
}

__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void store1(float* p, float x) { *p = x; }
__device__ __forceinline__ void store1(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

// Eight values from p, or the first `left` of them (zeros behind) where p is not aligned for the wide access or
// the tensor ends inside the eight.
template <typename T>
__device__ __forceinline__ f8 load_some(const T* p, bool wide, int left)
{
    if (wide) return load8(p);
    f8 x;
#pragma unroll
    for (int q = 0; q < 8; ++q) x.v[q] = q < left ? load1(p + q) : 0.f;
    return x;
}

// The same for a store.
template <typename T>
__device__ __forceinline__ void store_some(T* p, const f8& x, bool wide, int left)
{
    if (wide) {
        store8(p, x);
        return;
    }
#pragma unroll
    for (int q = 0; q < 8; ++q)
        if (q < left) store1(p + q, x.v[q]);
}

// And for rows that do not allow the wide access: in the widest units that the address does.
__device__ __forceinline__ void store_unaligned(float* p, const f8& x, int left)
{
    const uint32_t at = (uint32_t)reinterpret_cast<uintptr_t>(p);
    if (left == 8 && (at & 15) == 0) {
        reinterpret_cast<float4*>(p)[0] = make_float4(x.v[0], x.v[1], x.v[2], x.v[3]);
        reinterpret_cast<float4*>(p)[1] = make_float4(x.v[4], x.v[5], x.v[6], x.v[7]);
    } else if (left == 8 && (at & 7) == 0) {
#pragma unroll
        for (int q = 0; q < 4; ++q) reinterpret_cast<float2*>(p)[q] = make_float2(x.v[2 * q], x.v[2 * q + 1]);
    } else {
#pragma unroll
        for (int q = 0; q < 8; ++q)
            if (q < left) store1(p + q, x.v[q]);
    }
}

__device__ __forceinline__ void store_unaligned(__nv_bfloat16* p, const f8& x, int left)
{
    const uint32_t at = (uint32_t)reinterpret_cast<uintptr_t>(p);
    if (left == 8 && (at & 3) == 0) {
        uint32_t u[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) u[q] = pack_bf16(x.v[2 * q], x.v[2 * q + 1]);
        if ((at & 7) == 0) {
            reinterpret_cast<uint2*>(p)[0] = make_uint2(u[0], u[1]);
            reinterpret_cast<uint2*>(p)[1] = make_uint2(u[2], u[3]);
        } else {
#pragma unroll
            for (int q = 0; q < 4; ++q) reinterpret_cast<uint32_t*>(p)[q] = u[q];
        }
    } else {
#pragma unroll
        for (int q = 0; q < 8; ++q)
            if (q < left) store1(p + q, x.v[q]);
    }
}

// ---------------------------------------------------------------------------- two values at a time
// The packed binary32 instructions round each half as the scalar ones do and take one issue slot for two results.
typedef unsigned long long pair;

__device__ __forceinline__ pair make_pair(float lo, float hi)
{
    pair x;
    asm("mov.b64 %0, {%1, %2};" : "=l"(x) : "f"(lo), "f"(hi));
    return x;
}
__device__ __forceinline__ void split(pair x, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(x)); }
__device__ __forceinline__ pair add2(pair a, pair b)
{
    pair x;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(x) : "l"(a), "l"(b));
    return x;
}
__device__ __forceinline__ pair fma2(pair a, pair b, pair c)
{
    pair x;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(x) : "l"(a), "l"(b), "l"(c));
    return x;
}
__device__ __forceinline__ pair both(float x) { return make_pair(x, x); }
__device__ __forceinline__ pair mul2(pair a, pair b)
{
    pair x;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(x) : "l"(a), "l"(b));
    return x;
}
struct p4 {
    pair v[4];
};

__device__ __forceinline__ p4 to_pairs(const f8& x)
{
    p4 y;
#pragma unroll
    for (int q = 0; q < 4; ++q) y.v[q] = make_pair(x.v[2 * q], x.v[2 * q + 1]);
    return y;
}
__device__ __forceinline__ f8 to_values(const p4& x)
{
    f8 y;
#pragma unroll
    for (int q = 0; q < 4; ++q) split(x.v[q], y.v[2 * q], y.v[2 * q + 1]);
    return y;
}

// Two codes (the low 16 bits) to two values: the conversion goes through f16, which holds every E4M3 value and its NaN.
__device__ __forceinline__ pair decode_pair(uint32_t two)
{
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((unsigned short)two));
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
    return make_pair(f.x, f.y);
}

__device__ __forceinline__ p4 decode8(uint2 u)
{
    p4 x;
    x.v[0] = decode_pair(u.x);
    x.v[1] = decode_pair(u.x >> 16);
    x.v[2] = decode_pair(u.y);
    x.v[3] = decode_pair(u.y >> 16);
    return x;
}

// WORDS consecutive 32-bit words from an address of any alignment: the 16-byte pieces that hold them, moved down by words and, with 16-bit
// elements, by half a word.  False, and nothing read, where a piece would reach outside [lo, hi), the memory of the tensor.  (What
// the pieces hold beside the words is never used, so it does not matter if another thread is writing it.)
template <int WORDS>
__device__ __forceinline__ bool load_unaligned(const void* p, const void* lo, const void* hi, uint32_t* out)
{
    const uint32_t off = (uint32_t)reinterpret_cast<uintptr_t>(p) & 15u;
    const char* const first = static_cast<const char*>(p) - off;
    if (first < static_cast<const char*>(lo) || first + WORDS * 4 + 16 > static_cast<const char*>(hi)) return false;
    uint32_t w[WORDS + 4];
#pragma unroll
    for (int k = 0; k < WORDS / 4 + 1; ++k)
        asm volatile("ld.global.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(w[4 * k]), "=r"(w[4 * k + 1]), "=r"(w[4 * k + 2]), "=r"(w[4 * k + 3]) : "l"(first + 16 * k));
    const bool two = off & 8u, one = off & 4u;
#pragma unroll
    for (int i = 0; i < WORDS + 2; ++i) w[i] = two ? w[i + 2] : w[i];
#pragma unroll
    for (int i = 0; i < WORDS + 1; ++i) w[i] = one ? w[i + 1] : w[i];
    const uint32_t bits = (off & 2u) * 8u;
#pragma unroll
    for (int i = 0; i < WORDS; ++i) out[i] = __funnelshift_r(w[i], w[i + 1], bits);
    return true;
}

// Eight values as they are stored (half the registers of their binary32 values where they are bf16): requested early, widened when used.
// The second form is for rows that do not allow the wide access (an odd width, a view); [lo, hi) is the tensor's memory.
template <typename T>
struct Raw8;
template <>
struct Raw8<float> {
    f8 x;
    __device__ __forceinline__ void load(const float* p, bool wide, int left) { x = load_some(p, wide, left); }
    __device__ __forceinline__ void load(const float* p, int left, const void* lo, const void* hi)
    {
        uint32_t w[8];
        if (left > 0 && load_unaligned<8>(p, lo, hi, w)) {
#pragma unroll
            for (int q = 0; q < 8; ++q) x.v[q] = q < left ? __uint_as_float(w[q]) : 0.f;
        } else {
            x = load_some(p, false, left);
        }
    }
    __device__ __forceinline__ f8 values() const { return x; }
};
template <>
struct Raw8<__nv_bfloat16> {
    uint4 u;
    __device__ __forceinline__ void load(const __nv_bfloat16* p, bool wide, int left)
    {
        if (wide) {
            asm volatile("ld.global.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "l"(p));
            return;
        }
        const unsigned short* const h = reinterpret_cast<const unsigned short*>(p);
        uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int q = 0; q < 8; ++q)
            if (q < left) w[q >> 1] |= (uint32_t)h[q] << 16 * (q & 1);
        u = make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ __forceinline__ void load(const __nv_bfloat16* p, int left, const void* lo, const void* hi)
    {
        uint32_t w[4];
        if (left > 0 && load_unaligned<4>(p, lo, hi, w)) {
            if (left < 8) {
#pragma unroll
                for (int q = 0; q < 4; ++q) w[q] &= left >= 2 * q + 2 ? 0xFFFFFFFFu : left == 2 * q + 1 ? 0xFFFFu : 0u;
            }
            u = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
            load(p, false, left);
        }
    }
    __device__ __forceinline__ f8 values() const
    {
        f8 x;
        widen_pair(u.x, x.v[0], x.v[1]);
        widen_pair(u.y, x.v[2], x.v[3]);
        widen_pair(u.z, x.v[4], x.v[5]);
        widen_pair(u.w, x.v[6], x.v[7]);
        return x;
    }
};

// ---------------------------------------------------------------------------- blocks of 16 lanes times eight values
// Largest of eight magnitudes; NaN if one of them is.
__device__ __forceinline__ float top8(const f8& x)
{
    float a, b, c;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(a) : "f"(x.v[0]), "f"(x.v[1]), "f"(x.v[2]));
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(b) : "f"(x.v[3]), "f"(x.v[4]), "f"(x.v[5]));
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(c) : "f"(x.v[6]), "f"(x.v[7]), "f"(a));
    asm("max.NaN.abs.f32 %0, %1, %2, %2;" : "=f"(a) : "f"(b), "f"(c));
    return a;
}

// Largest pattern over the 16 lanes that hold a block.  (A redux over each half of the warp costs fewer instructions but splits the
// warp in two for everything that follows: 424 against 402 us on 138 M elements.)
__device__ __forceinline__ uint32_t block_top(uint32_t x, uint32_t lanes)
{
#pragma unroll
    for (int d = 8; d >= 1; d >>= 1) x = max(x, __shfl_xor_sync(lanes, x, d));
    return x;
}

// Scale byte of the block that 16 lanes hold in x, and what its values are to be encoded as: where some are not finite the scale is that of the
// others and they become NaN.  All lanes of the warp come here.
__device__ __forceinline__ int block_scale(f8& x)
{
    const uint32_t top = block_top(__float_as_uint(top8(x)), 0xFFFFFFFFu);
    if (top < 0x7F800000u) return scale_byte(__uint_as_float(top));
    const uint32_t half = threadIdx.x & 16 ? 0xFFFF0000u : 0xFFFFu;       // the whole block is here, the warp need not be
    uint32_t t = 0;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        if (finite(x.v[q])) t = max(t, __float_as_uint(fabsf(x.v[q])));
        else x.v[q] = __uint_as_float(0x7FC00000u);
    }
    return scale_byte(__uint_as_float(block_top(t, half)));
}

// Four codes to nearest even (of magnitudes up to 448, or NaN).
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d)
{
    unsigned short lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
    return lo | (uint32_t)hi << 16;
}

// Codes of eight values of a block with that scale.
__device__ __forceinline__ uint2 encode_nearest(const f8& x, int byte)
{
    const pair inv = both(scale_inverse(byte));
    p4 y = to_pairs(x);
#pragma unroll
    for (int q = 0; q < 4; ++q) y.v[q] = mul2(y.v[q], inv);
    const f8 z = to_values(y);
    return make_uint2(codes4(z.v[0], z.v[1], z.v[2], z.v[3]), codes4(z.v[4], z.v[5], z.v[6], z.v[7]));
}

// Where the scale of block b of row r stands: words of four blocks, the rows' words of one group of four next to one another.
__device__ __forceinline__ int64_t scale_index(int64_t b, int64_t r, int64_t ld) { return ((b >> 2) * ld + r) * 4 + (b & 3); }

}  // namespace ops
}  // namespace hpsgd
