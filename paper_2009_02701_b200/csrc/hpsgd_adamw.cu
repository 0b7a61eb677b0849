// AdamW over many tensors (moments in 32 or in 8 bits) and the global norm of their gradients.
//
// Both are element-wise passes over HBM: a parameter costs 28 bytes a step with everything in 32 bits, 10 with
// bf16 parameters and gradients and moments in 8 bits, against some dozens of instructions.  As in the replica
// kernels the work is organised around the traffic: one 8-element group per thread and array, all loads requested
// before the first is used, many short blocks.  The table of tensors travels in the kernel's parameters, so a
// step needs no copy to the device and no workspace, and any mix of large and tiny tensors is one launch.
#include "hpsgd_ops_common.cuh"

#include <algorithm>

namespace hpsgd {
namespace ops {
namespace {

constexpr int kAdamThreads = 128;
constexpr int kChunk = kAdamThreads * 8;       // elements a block handles: eight 8-bit blocks
constexpr int kSpanChunks = 2;
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
    uint32_t wide;         // all addresses allow the wide accesses
};

template <int CAP>
struct Table {
    int count;
    uint32_t first[CAP];   // first chunk of each tensor (by themselves: a block's search touches few lines of the parameters)
    Item item[CAP];
};

struct Hyper {
    float beta1, rest1, beta2, rest2;          // rest = 1 - beta, rounded once from binary64
    float rate;                                // lr / (1 - beta1^step)
    float root;                                // 1 / sqrt(1 - beta2^step)
    float eps;
    uint32_t key0, key1;
    const float* scale;
    int span;                                  // elements per block
};

// What the norm needs of a tensor is a fifth of that, and the table holds five times as many.
constexpr int kMaxNormItems = 1600;
template <int CAP>
struct NormTable {
    int count;
    uint32_t first[CAP];
    const void* g[CAP];
    int64_t n2[CAP];       // twice the number of elements, and 1 if the address allows the wide accesses
};

// The tensor that a chunk belongs to: the last whose first chunk is not behind it.
template <typename Tab>
__device__ __forceinline__ int find_item(const Tab& t, uint32_t chunk)
{
    int lo = 0, hi = t.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (t.first[mid] <= chunk) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// `turn`: the second key (with the position's upper half) times N2, which the second product then only adds.
__device__ __forceinline__ uint32_t random_bits(uint32_t q, uint32_t key0, uint32_t turn)
{
    uint32_t x = (q ^ key0) * kN1;
    x ^= x >> 15;
    x = x * kN2 + turn;
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

// A sum of products that are each rounded: a packed addition behind packed multiplications was seen to come out with one rounding fewer,
// so this one is scalar.
__device__ __forceinline__ pair sum_of_rounded(pair a, pair b)
{
    float a0, a1, b0, b1;
    split(a, a0, a1);
    split(b, b0, b1);
    return make_pair(__fadd_rn(a0, b0), __fadd_rn(a1, b1));
}

// ---------------------------------------------------------------------------- codes
// What multiplies a value of a block with scale 2^(byte - 127) so that the value's E4M3 code comes to stand in bits 20..26 of
// its binary32 pattern: 2^(127 - byte - 120), in one factor as long as that is a normal number.  Blocks above 2^6 * 448, whose
// factor is not, first have their values multiplied by the rest (`excess`).  The largest patterns of values that are not finite
// give bytes that have excess too.
__device__ __forceinline__ float code_factor(int byte) { return __uint_as_float((uint32_t)(max(254 - 120 - byte, 1)) << 23); }
__device__ __forceinline__ bool has_excess(int byte) { return byte > 133; }
__device__ __forceinline__ float excess(int byte) { return has_excess(byte) ? __uint_as_float((uint32_t)(127 - (byte - 133)) << 23) : 1.f; }

// Both roundings take x already multiplied by its block's code factor and give the code in bits 20..26 with the sign in bit 31
// (what lies below does not count): see gather_codes.

// One of the two codes around |x|, such that the expected value is |x|: 16 random bits, centred, are added below the last bit that
// is kept, and the carry decides.  An exact code stays.
__device__ __forceinline__ uint32_t round_first(float x, uint32_t rnd)
{
    return __float_as_uint(x) + ((rnd >> 12 & 0xFFFF0u) | 8u);
}

// One of the two codes a <= x < b, such that the expected square is x^2: b with probability (x^2 - a^2) / (b^2 - a^2).  With the
// codes' step as the unit, a = n and x = n + f, that is f (2n + f) / (2n + 1); n + f is 8 times the significand of x, or x itself
// over the step where the code is subnormal (there alone 0 is near: the caller lifts what is not 0 to the first code).  Two elements at a time.
template <bool SUBNORMAL>
__device__ __forceinline__ void round_second(float x0, float x1, uint32_t rnd0, uint32_t rnd1, uint32_t& c0, uint32_t& c1)
{
    c0 = __float_as_uint(x0);
    c1 = __float_as_uint(x1);
    pair s = make_pair(__uint_as_float((c0 & 0x7FFFFFu) | 0x41000000u), __uint_as_float((c1 & 0x7FFFFFu) | 0x41000000u));
    pair n = make_pair(__uint_as_float((c0 & 0x700000u) | 0x41000000u), __uint_as_float((c1 & 0x700000u) | 0x41000000u));
    if (SUBNORMAL) {
        const pair less = make_pair(c0 < 0x800000u ? -8.f : 0.f, c1 < 0x800000u ? -8.f : 0.f);
        s = add2(s, less);
        n = add2(n, less);
    }
    // u = (16 random bits + 0.5) / 2^16: the bits below an exponent of 23 are 2^23 + bits, and the sum below is exact
    const pair u = fma2(make_pair(__uint_as_float(__byte_perm(rnd0, 0x4B00u, 0x5410)), __uint_as_float(__byte_perm(rnd1, 0x4B00u, 0x5410))),
                        both(0x1p-16f), both(0x1p-17f - 128.f));
    const pair lhs = mul2(u, fma2(both(2.f), n, both(1.f)));
    const pair rhs = mul2(fma2(both(-1.f), n, s), add2(n, s));
    float l0, l1, r0, r1;
    split(lhs, l0, l1);
    split(rhs, r0, r1);
    if (l0 < r0) c0 += 0x100000u;
    if (l1 < r1) c1 += 0x100000u;
}

// Four codes next to one another: the upper halves pairwise, shifted and cut two at a time.
__device__ __forceinline__ uint32_t gather_codes(uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    const uint32_t ab = __byte_perm(a, b, 0x7632), cd = __byte_perm(c, d, 0x7632);
    const uint32_t x = (ab << 4 & 0x7F007F00u) | (ab & 0x80008000u), y = (cd << 4 & 0x7F007F00u) | (cd & 0x80008000u);
    return __byte_perm(x, y, 0x7531);
}

__device__ __forceinline__ uint2 gather8(const uint32_t* c)
{
    return make_uint2(gather_codes(c[0], c[1], c[2], c[3]), gather_codes(c[4], c[5], c[6], c[7]));
}

// Eight patterns cut to bf16.
__device__ __forceinline__ void store_upper(__nv_bfloat16* p, const f8& x, bool wide, int left)
{
    uint32_t u[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) u[q] = __byte_perm(__float_as_uint(x.v[2 * q]), __float_as_uint(x.v[2 * q + 1]), 0x7632);
    if (wide) {
        *reinterpret_cast<uint4*>(p) = make_uint4(u[0], u[1], u[2], u[3]);
        return;
    }
    unsigned short* const h = reinterpret_cast<unsigned short*>(p);
#pragma unroll
    for (int q = 0; q < 8; ++q)
        if (q < left) h[q] = (unsigned short)(u[q >> 1] >> 16 * (q & 1));
}

// Reciprocal by the hardware's approximation, 1 unit in the last place.
__device__ __forceinline__ float reciprocal_approx(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Smallest of eight numbers >= 0.
__device__ __forceinline__ float bottom8(const f8& x)
{
    float a, b, c;
    asm("min.f32 %0, %1, %2, %3;" : "=f"(a) : "f"(x.v[0]), "f"(x.v[1]), "f"(x.v[2]));
    asm("min.f32 %0, %1, %2, %3;" : "=f"(b) : "f"(x.v[3]), "f"(x.v[4]), "f"(x.v[5]));
    asm("min.f32 %0, %1, %2, %3;" : "=f"(c) : "f"(x.v[6]), "f"(x.v[7]), "f"(a));
    return fminf(b, c);
}

// ---------------------------------------------------------------------------- the step
// Where a block's share of a tensor starts in each of its arrays.
struct Share {
    void* p;
    const void* g;
    void* m;
    void* v;
    uint8_t* ms;
    uint8_t* vs;
    __nv_bfloat16* copy;
    uint64_t rng;
    float keep;
    bool wide;
};

// The block's codes and scales from its new moments m and r = sqrt(v) (zeros behind the end of the tensor).
__device__ __forceinline__ void encode8(const f8& m, const f8& r, const uint32_t* rnd, int& mb, int& vb, uint2& mc, uint2& vc)
{
    mb = scale_byte(__uint_as_float(block_top(__float_as_uint(top8(m)), 0xFFFFFFFFu)));
    vb = scale_byte(__uint_as_float(block_top(__float_as_uint(top8(r)), 0xFFFFFFFFu)));
    uint32_t cm[8], cr[8];
    float low;
    f8 x;
    {
        const pair fm = both(code_factor(mb)), fr = both(code_factor(vb));
        p4 y = to_pairs(m);
#pragma unroll
        for (int q = 0; q < 4; ++q) y.v[q] = mul2(y.v[q], fm);
        x = to_values(y);
#pragma unroll
        for (int q = 0; q < 8; ++q) cm[q] = round_first(x.v[q], rnd[q]);
        y = to_pairs(r);
#pragma unroll
        for (int q = 0; q < 4; ++q) y.v[q] = mul2(y.v[q], fr);
        x = to_values(y);
        low = bottom8(x);
    }
    if (max(mb, vb) <= 133 && __float_as_uint(low) >= 0x800000u) {
#pragma unroll
        for (int q = 0; q < 8; q += 2) round_second<false>(x.v[q], x.v[q + 1], rnd[q], rnd[q + 1], cr[q], cr[q + 1]);
    } else {
        // some second moment far below its block's largest, a very large block, or values that are not finite: the scales are those of
        // the finite values
        if (has_excess(mb) || has_excess(vb)) {
            uint32_t tm = 0, tr = 0;
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                tm = max(tm, __float_as_uint(finite_magnitude(m.v[q])));
                tr = max(tr, __float_as_uint(finite_magnitude(r.v[q])));
            }
            const uint32_t half = threadIdx.x & 16 ? 0xFFFF0000u : 0xFFFFu;       // the whole block is here, the warp need not be
            mb = scale_byte(__uint_as_float(block_top(tm, half)));
            vb = scale_byte(__uint_as_float(block_top(tr, half)));
        }
        const float em = excess(mb), er = excess(vb), fm = code_factor(mb), fr = code_factor(vb);
#pragma unroll
        for (int q = 0; q < 8; q += 2) {
            round_second<true>(__fmul_rn(__fmul_rn(r.v[q], er), fr), __fmul_rn(__fmul_rn(r.v[q + 1], er), fr), rnd[q], rnd[q + 1], cr[q], cr[q + 1]);
#pragma unroll
            for (int k = q; k < q + 2; ++k) {
                cm[k] = finite(m.v[k]) ? round_first(__fmul_rn(__fmul_rn(m.v[k], em), fm), rnd[k]) : 0x7F00000u;
                // r itself decides what is 0: scaled by its block's factor, one 2^39 below the block's largest has vanished
                if (r.v[k] > 0.f) cr[k] = max(cr[k], 0x100000u);
                if (!finite(r.v[k])) cr[k] = 0x7F00000u;
            }
        }
    }
    mc = gather8(cm);
    vc = gather8(cr);
}

// What a thread reads for one group with 8-bit moments.
template <typename P, typename G>
struct Group8 {
    Raw8<P> p;
    Raw8<G> g;
    uint2 mc, vc;
    uint32_t mb, vb;
    __device__ __forceinline__ void load(const Share& it, int o)
    {
        p.load(static_cast<const P*>(it.p) + o, true, 8);
        g.load(static_cast<const G*>(it.g) + o, true, 8);
        const uint8_t *m = static_cast<const uint8_t*>(it.m) + o, *v = static_cast<const uint8_t*>(it.v) + o;
        asm volatile("ld.global.v2.b32 {%0,%1}, [%2];" : "=r"(mc.x), "=r"(mc.y) : "l"(m));
        asm volatile("ld.global.v2.b32 {%0,%1}, [%2];" : "=r"(vc.x), "=r"(vc.y) : "l"(v));
        asm volatile("ld.global.u8 %0, [%1];" : "=r"(mb) : "l"(it.ms + o / kBlock));
        asm volatile("ld.global.u8 %0, [%1];" : "=r"(vb) : "l"(it.vs + o / kBlock));
    }
};

// One group of eight per thread, `left` of them inside the tensor, at elements o.. of the block's share.  All threads of a warp come
// here.  FULL: the whole block has eight elements a thread and wide accesses, which leaves no branch in the way of the loads; with
// 8-bit moments they have been made already (`ready`).
template <typename P, typename G, bool B8, bool FULL>
__device__ __forceinline__ void adamw_group(const Share& it, const Hyper& hy, float c, int o, int left, const Group8<P, G>* ready = nullptr)
{
    const bool wide = FULL || (it.wide && left == 8);
    P* const pp = static_cast<P*>(it.p) + o;
    f8 p, g, m, v, r;                              // r = sqrt(v), which the step divides by and the 8-bit form keeps
    uint2 mc, vc;
    int mb = 0, vb = 0;
    if constexpr (B8 && FULL) {
        p = ready->p.values();
        g = ready->g.values();
        mc = ready->mc;
        vc = ready->vc;
        mb = (int)ready->mb;
        vb = (int)ready->vb;
    } else {
        p = load_some(pp, wide, left);
        g = load_some(static_cast<const G*>(it.g) + o, wide, left);
        if constexpr (B8) {
            mc = load_codes(static_cast<const uint8_t*>(it.m) + o, wide, left);
            vc = load_codes(static_cast<const uint8_t*>(it.v) + o, wide, left);
            if (left > 0) {
                mb = it.ms[o / kBlock];
                vb = it.vs[o / kBlock];
            }
        } else {
            m = load_some(static_cast<const float*>(it.m) + o, wide, left);
            v = load_some(static_cast<const float*>(it.v) + o, wide, left);
        }
    }
    if (!finite(c)) return;                        // the whole grid: nothing of the step happens

    // With 32-bit moments HBM is what bounds the kernel, and the quotient is correctly rounded; with 8-bit moments instructions are, and
    // it is a product with the hardware's reciprocal (of a step that is added to p, where two units in its last place do not count).  The
    // root decides which code is kept and is correctly rounded in both.
    if constexpr (B8) {
        const pair sm = both(scale_value(mb)), sv = both(scale_value(vb));
        p4 pm = decode8(mc), pv = decode8(vc), pg = to_pairs(g), px = to_pairs(p);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            pm.v[q] = mul2(pm.v[q], sm);
            pv.v[q] = mul2(pv.v[q], sv);
            pv.v[q] = mul2(pv.v[q], pv.v[q]);
            pg.v[q] = mul2(pg.v[q], both(c));
            pm.v[q] = sum_of_rounded(mul2(pm.v[q], both(hy.beta1)), mul2(pg.v[q], both(hy.rest1)));
            pv.v[q] = sum_of_rounded(mul2(pv.v[q], both(hy.beta2)), mul2(mul2(pg.v[q], pg.v[q]), both(hy.rest2)));
        }
        m = to_values(pm);
        v = to_values(pv);
#pragma unroll
        for (int q = 0; q < 8; ++q) r.v[q] = __fsqrt_rn(v.v[q]);
        const p4 pr = to_pairs(r);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float b0, b1;
            split(fma2(pr.v[q], both(hy.root), both(hy.eps)), b0, b1);
            const pair step = mul2(pm.v[q], make_pair(reciprocal_approx(b0), reciprocal_approx(b1)));
            px.v[q] = fma2(both(-hy.rate), step, mul2(px.v[q], both(it.keep)));
        }
        p = to_values(px);
    } else {
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const float gq = __fmul_rn(g.v[q], c);
            m.v[q] = __fadd_rn(__fmul_rn(hy.beta1, m.v[q]), __fmul_rn(hy.rest1, gq));
            v.v[q] = __fadd_rn(__fmul_rn(hy.beta2, v.v[q]), __fmul_rn(hy.rest2, __fmul_rn(gq, gq)));
            r.v[q] = __fsqrt_rn(v.v[q]);
            const float step = __fdiv_rn(m.v[q], __fmaf_rn(r.v[q], hy.root, hy.eps));
            p.v[q] = __fmaf_rn(-hy.rate, step, __fmul_rn(p.v[q], it.keep));
        }
    }

    uint32_t rnd[8];
    constexpr bool kPB = sizeof(P) == 2;
    if constexpr (B8 || kPB) {
        const uint64_t q0 = it.rng + (uint64_t)o;
        const uint32_t low = (uint32_t)q0, turn = (hy.key1 + (uint32_t)(q0 >> 32) * kN3) * kN2;
        if ((low & 7u) == 0) {                     // the position is one bit operation away from the first's
#pragma unroll
            for (int q = 0; q < 8; ++q) rnd[q] = random_bits(low ^ hy.key0, q, turn);
        } else {                                   // its upper half may change within the eight
#pragma unroll
            for (int q = 0; q < 8; ++q) rnd[q] = random_bits(low + q, hy.key0, low + q < low ? turn + kN3 * kN2 : turn);
        }
    }
    if constexpr (kPB) {
        const bool all = finite(top8(p));
#pragma unroll
        for (int q = 0; q < 8; ++q)                // the upper half of the pattern is what is kept
            if (all || finite(p.v[q])) p.v[q] = __uint_as_float(__float_as_uint(p.v[q]) + (rnd[q] * kN2 >> 16));
        store_upper(pp, p, wide, left);
    } else {
        store_some(pp, p, wide, left);
        if (it.copy) store_some(it.copy + o, p, wide, left);
    }

    if constexpr (B8) {
        encode8(m, r, rnd, mb, vb, mc, vc);
        store_codes(static_cast<uint8_t*>(it.m) + o, mc, wide, left);
        store_codes(static_cast<uint8_t*>(it.v) + o, vc, wide, left);
        if ((FULL || left > 0) && (threadIdx.x & 15) == 0) {
            it.ms[o / kBlock] = (uint8_t)mb;
            it.vs[o / kBlock] = (uint8_t)vb;
        }
    } else {
        store_some(static_cast<float*>(it.m) + o, m, wide, left);
        store_some(static_cast<float*>(it.v) + o, v, wide, left);
    }
}

// Block b handles `span` elements, a whole number of chunks, of one tensor.
template <int CAP, typename P, typename G, bool B8>
__global__ void __launch_bounds__(kAdamThreads, B8 ? 6 : 7) adamw_kernel(const __grid_constant__ Table<CAP> table, const __grid_constant__ Hyper hy)
{
    const int which = find_item(table, blockIdx.x);
    const Item& it = table.item[which];
    const int64_t at = (int64_t)(blockIdx.x - table.first[which]) * hy.span;
    const int here = (int)min((int64_t)hy.span, it.n - at);
    Share sh;
    sh.p = static_cast<P*>(it.p) + at;
    sh.g = static_cast<const G*>(it.g) + at;
    sh.m = static_cast<char*>(it.m) + at * (B8 ? 1 : 4);
    sh.v = static_cast<char*>(it.v) + at * (B8 ? 1 : 4);
    sh.ms = it.ms + at / kBlock;
    sh.vs = it.vs + at / kBlock;
    sh.copy = it.copy ? it.copy + at : nullptr;
    sh.rng = it.rng + (uint64_t)at;
    sh.keep = it.keep;
    sh.wide = it.wide;
    after_previous();
    const float c = hy.scale ? *hy.scale : 1.f;
    const int tid8 = threadIdx.x * 8;
    if constexpr (B8) {
        if (sh.wide && here == hy.span) {
            Group8<P, G> now, next;
            now.load(sh, tid8);
#pragma unroll 1
            for (int s = tid8; s < here; s += kChunk) {
                if (s + kChunk < here) next.load(sh, s + kChunk);
                adamw_group<P, G, true, true>(sh, hy, c, s, 8, &now);
                now = next;
            }
            return;
        }
    } else if (sh.wide && here == hy.span) {
        adamw_group<P, G, false, true>(sh, hy, c, tid8, 8);
        return;
    }
    for (int s = 0; s < here; s += kChunk) adamw_group<P, G, B8, false>(sh, hy, c, s + tid8, max(0, min(8, here - s - tid8)));
}

// ---------------------------------------------------------------------------- the norm
constexpr int kNormThreads = 256;
constexpr int kNormChunk = kNormThreads * 8 * 4;       // four groups of eight in flight per thread
constexpr int kNormPartials = (HPSGD_GRAD_NORM_WORKSPACE - 64) / 8;

struct NormOut {
    float max_norm;
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
__global__ void __launch_bounds__(kNormThreads) grad_norm_kernel(const __grid_constant__ NormTable<CAP> table, const __grid_constant__ NormOut no)
{
    __shared__ double part[kNormThreads / 32];
    __shared__ bool last;
    double sum = 0.0;
    after_previous();
    for (uint32_t chunk = blockIdx.x; chunk < no.chunks; chunk += gridDim.x) {
        const int which = find_item(table, chunk);
        const G* const gp = static_cast<const G*>(table.g[which]);
        const int64_t n = table.n2[which] >> 1;
        const bool wide = table.n2[which] & 1;
        const int64_t base = (int64_t)(chunk - table.first[which]) * kNormChunk + threadIdx.x * 8;
        f8 x[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int64_t at = base + k * (kNormThreads * 8), rest = n - at;
            const int left = rest < 0 ? 0 : rest > 8 ? 8 : (int)rest;
            x[k] = load_some(gp + at, wide && left == 8, left);
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
        const float norm = __fsqrt_rn((float)s);
        no.out[0] = norm;
        no.out[1] = !finite(norm) ? __uint_as_float(0x7FC00000u) : norm > no.max_norm ? __fdiv_rn(no.max_norm, norm) : 1.f;
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
    if (n > 1 << 20) return report(HPSGD_E_UNSUPPORTED, "%s: more than 2^20 tensors", what);
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

// The next launch's worth of tensors starting at *at, at most `cap`: calls add(tensor, its place, its first chunk) for each and returns their
// number of chunks.  Empty tensors are left out.
template <typename Add>
uint32_t next_launch(const hpsgd_adamw_tensor* t, int n, int* at, int cap, int64_t chunk_elems, Add add)
{
    uint64_t chunks = 0;
    int place = 0;
    for (; *at < n && place < cap; ++*at) {
        if (t[*at].n == 0) continue;
        const uint64_t here = (uint64_t)(t[*at].n + chunk_elems - 1) / chunk_elems;
        if (chunks + here > 0x7FFFFFFFull) break;      // a launch has at most that many blocks; 2^40 elements fit one alone
        add(t[*at], place++, (uint32_t)chunks);
        chunks += here;
    }
    return (uint32_t)chunks;
}

template <int CAP, typename P, typename G, bool B8>
int step_launches(const hpsgd_adamw_tensor* t, int n, double lr, Hyper hy, int sms, cudaStream_t s)
{
    // With 8-bit moments finding the tensor and its addresses is a tenth of a block's instructions if it handles one chunk; with
    // enough chunks to fill the device all the same, a block takes two and requests the second while it works on the first
    // (138 M elements in bf16: two 364, four 399 us; 25.6 M in fp32 with its norm: 112, 121 us).
    // With 32-bit moments the kernel waits for HBM whatever a block takes.
    int64_t total = 0;
    for (int k = 0; k < n; ++k) total += t[k].n;
    hy.span = B8 && total >= (int64_t)kSpanChunks * kChunk * sms * 16 ? kSpanChunks * kChunk : kChunk;
    const size_t ap = sizeof(P) == 4 ? 32 : 16, ag = sizeof(G) == 4 ? 32 : 16, as = B8 ? 8 : 32;
    int at = 0;
    Table<CAP> table;
    while (at < n) {
        table.count = 0;
        const uint32_t chunks = next_launch(t, n, &at, CAP, hy.span, [&](const hpsgd_adamw_tensor& x, int place, uint32_t first) {
            table.count = place + 1;
            table.first[place] = first;
            Item& it = table.item[place];
            it.p = x.param; it.g = x.grad; it.m = x.m; it.v = x.v; it.ms = x.m_scale; it.vs = x.v_scale;
            it.copy = static_cast<__nv_bfloat16*>(x.copy);
            it.n = x.n;
            it.rng = x.rng_offset;
            it.keep = (float)(1.0 - lr * x.weight_decay);
            it.wide = aligned(x.param, ap) && aligned(x.grad, ag) && aligned(x.m, as) && aligned(x.v, as) && aligned(x.copy, 16);
        });
        if (!chunks) continue;
        OPS_TRY(launch_early("hpsgd_adamw_step", adamw_kernel<CAP, P, G, B8>, dim3(chunks), kAdamThreads, 0, s, table, hy));
    }
    return HPSGD_OK;
}

template <int CAP>
int step_types(const hpsgd_adamw_tensor* t, int n, int pd, int gd, int bits, double lr, const Hyper& hy, int sms, cudaStream_t s)
{
    using bf = __nv_bfloat16;
    if (pd == HPSGD_F32 && gd == HPSGD_F32) return bits == 8 ? step_launches<CAP, float, float, true>(t, n, lr, hy, sms, s) : step_launches<CAP, float, float, false>(t, n, lr, hy, sms, s);
    if (pd == HPSGD_F32) return bits == 8 ? step_launches<CAP, float, bf, true>(t, n, lr, hy, sms, s) : step_launches<CAP, float, bf, false>(t, n, lr, hy, sms, s);
    if (gd == HPSGD_F32) return bits == 8 ? step_launches<CAP, bf, float, true>(t, n, lr, hy, sms, s) : step_launches<CAP, bf, float, false>(t, n, lr, hy, sms, s);
    return bits == 8 ? step_launches<CAP, bf, bf, true>(t, n, lr, hy, sms, s) : step_launches<CAP, bf, bf, false>(t, n, lr, hy, sms, s);
}

template <int CAP, typename G>
int norm_launches(const hpsgd_adamw_tensor* t, int n, int sms, double max_norm, void* ws, float* out, cudaStream_t s)
{
    // blocks of every launch, so that the last block of the last launch knows what it has to wait for
    const auto pass = [](const hpsgd_adamw_tensor&, int, uint32_t) {};
    int at = 0, total = 0, launches = 0;
    while (at < n) {
        next_launch(t, n, &at, CAP, kNormChunk, pass);
        ++launches;
    }
    const int most = std::max(1, std::min(sms * 8, kNormPartials / std::max(1, launches)));
    const auto grid_of = [&](uint32_t chunks) { return (int)std::min<uint32_t>(std::max<uint32_t>(chunks, 1), most); };
    at = 0;
    while (at < n) total += grid_of(next_launch(t, n, &at, CAP, kNormChunk, pass));
    if (total == 0) total = 1;                     // no tensors: one block writes the norm of nothing
    NormOut no{(float)max_norm, static_cast<unsigned int*>(ws), reinterpret_cast<double*>(static_cast<char*>(ws) + 64), 0, total, 0, out};
    at = 0;
    NormTable<CAP> table;
    do {
        table.count = 0;
        no.chunks = next_launch(t, n, &at, CAP, kNormChunk, [&](const hpsgd_adamw_tensor& x, int place, uint32_t first) {
            table.count = place + 1;
            table.first[place] = first;
            table.g[place] = x.grad;
            table.n2[place] = x.n * 2 + aligned(x.grad, sizeof(G) == 4 ? 32 : 16);
        });
        const int grid = grid_of(no.chunks);
        OPS_TRY(launch_early("hpsgd_grad_norm", grad_norm_kernel<CAP, G>, dim3(grid), kNormThreads, 0, s, table, no));
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
    if (!(eps >= 0x1p-126) || !std::isfinite((float)eps)) return report(HPSGD_E_BADARG, "%s: eps must be a normal positive number in binary32", what);
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
    // The host copies a kernel's parameters at every launch: 65 small tensors' step takes 8.1 us by the largest table, 5.9 by the third.
    if (n_tensors <= 8) return step_types<8>(tensors, n_tensors, param_dtype, grad_dtype, state_bits, lr, hy, sms, s);
    if (n_tensors <= 64) return step_types<64>(tensors, n_tensors, param_dtype, grad_dtype, state_bits, lr, hy, sms, s);
    if (n_tensors <= 192) return step_types<192>(tensors, n_tensors, param_dtype, grad_dtype, state_bits, lr, hy, sms, s);
    return step_types<kMaxItems>(tensors, n_tensors, param_dtype, grad_dtype, state_bits, lr, hy, sms, s);
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
    if (n_tensors <= 192)
        return f ? norm_launches<192, float>(tensors, n_tensors, sms, max_norm, workspace, out, s)
                 : norm_launches<192, __nv_bfloat16>(tensors, n_tensors, sms, max_norm, workspace, out, s);
    return f ? norm_launches<kMaxNormItems, float>(tensors, n_tensors, sms, max_norm, workspace, out, s)
             : norm_launches<kMaxNormItems, __nv_bfloat16>(tensors, n_tensors, sms, max_norm, workspace, out, s);
}

}  // extern "C"
