// The loss over a label and a teacher's top logits, and its gradient.
//
// Bound by HBM: a row of logits is read once and a row of gradients written once.  A block takes a row in tiles, two of which are in its registers or on
// their way there: first the sums of exponentials, from the first tile to the last, then the gradient, from the last, which is still there, to the
// first; the tiles between come a second time, out of L2.  (Rows held whole, by one block or in the registers of a cluster's blocks, left too little
// under way while their sums were waited for: 4096 x 30000 bf16 at two temperatures 150 and 236 us; clusters of eight 4096 x 131072 1330.)
//
// Sums of exponentials: s = sum 2^(x c - k) with c = log2(e) / temperature and k the largest x c rounded up to a whole number, so that joining two
// sums multiplies by an exact power of two, and x c - k is rounded once; the softmax is then 2^(x c - k) / s without any error of k's.
//
// Powers of two are what the SM does least of (16 a clock; two for each element are three quarters of the time that its bytes take).  With a label and a
// teacher there are two temperatures, and four of them; where the teacher's is 2, 3 or 4, e^z is that power of e^(z / T), by multiplying.
//
// Large logits: x c - k is the product's rounding error where x c has no digits left behind the point, and that can be 2^100 either way.  k is held above
// -kFar, so masked words that are far below add nothing wherever they are, and a row that is far out as a whole, or has its label or a teacher's entry
// there, is done by far_row(): from differences to the largest logit, one element after another.
#include "hpsgd_ops_common.cuh"

#include <algorithm>
#include <cfloat>

namespace hpsgd {
namespace ops {
namespace {

constexpr int kMaxTeacher = 1024;

struct LossArgs {
    int rows, vocab, k, pieces, piece;              // pieces: blocks that share a row (the gradient alone); piece: columns of each
    const void* z;
    const int64_t* labels;
    const int32_t* index;
    const void* teacher;
    float* loss;
    float* lse;
    void* dz;
    const float* dloss;
    const void* z_end;
    int64_t ldz, ldt, lddz;
    float c1, c2;                                   // log2(e) over the temperatures; c2, the teacher's, is only used where there are two
    float ct, wl, wt, temperature, scale;           // wt: with the square of the temperature
    float inverse;                                  // 1 / temperature
    int teacher_bf16;
    int main_is_teacher;                            // c1 is the teacher's temperature
};

// How long a line is wanted in L2: what is read again until it has been, and nothing that has been written.
__device__ __forceinline__ uint64_t keep_long()
{
    uint64_t x;
    asm("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(x));
    return x;
}
__device__ __forceinline__ uint64_t drop_first()
{
    uint64_t x;
    asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(x));
    return x;
}
__device__ __forceinline__ void load8(Raw8<float>& y, const float* p, uint64_t policy)
{
    f8& x = y.x;
    asm volatile("ld.global.L2::cache_hint.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8], %9;"
                 : "=f"(x.v[0]), "=f"(x.v[1]), "=f"(x.v[2]), "=f"(x.v[3]), "=f"(x.v[4]), "=f"(x.v[5]), "=f"(x.v[6]), "=f"(x.v[7])
                 : "l"(p), "l"(policy));
}
__device__ __forceinline__ void load8(Raw8<__nv_bfloat16>& x, const __nv_bfloat16* p, uint64_t policy)
{
    asm volatile("ld.global.L2::cache_hint.v4.b32 {%0,%1,%2,%3}, [%4], %5;" : "=r"(x.u.x), "=r"(x.u.y), "=r"(x.u.z), "=r"(x.u.w) : "l"(p), "l"(policy));
}
__device__ __forceinline__ void store8(float* p, const f8& x, uint64_t policy)
{
    asm volatile("st.global.L2::cache_hint.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8}, %9;" ::"l"(p), "f"(x.v[0]), "f"(x.v[1]), "f"(x.v[2]), "f"(x.v[3]), "f"(x.v[4]),
                 "f"(x.v[5]), "f"(x.v[6]), "f"(x.v[7]), "l"(policy)
                 : "memory");
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const f8& x, uint64_t policy)
{
    asm volatile("st.global.L2::cache_hint.v4.b32 [%0], {%1,%2,%3,%4}, %5;" ::"l"(p), "r"(pack_bf16(x.v[0], x.v[1])), "r"(pack_bf16(x.v[2], x.v[3])),
                 "r"(pack_bf16(x.v[4], x.v[5])), "r"(pack_bf16(x.v[6], x.v[7])), "l"(policy)
                 : "memory");
}

struct Sum {
    float k, s;                                     // s 2^k
    __device__ __forceinline__ void add(float k2, float s2)
    {
        const float top = fmaxf(k, k2);
        s = __fmaf_rn(s, exp2_of(k - top), __fmul_rn(s2, exp2_of(k2 - top)));
        k = top;
    }
};
__device__ __forceinline__ Sum nothing() { return Sum{-FLT_MAX, 0.f}; }

// Exponents x c of this magnitude and more are far.  Below it a product's rounding is at most 2^-5, so x c - k of the largest is in (-1, 2^-5].
constexpr float kFar = 1048576.f;
__device__ __forceinline__ bool is_far(float k) { return k >= kFar || k == -kFar; }      // (k does not go below -kFar)
__device__ __forceinline__ float log2_of(const Sum& x) { return __fadd_rn(x.k, log2f(x.s)); }

// Over the lanes of a warp; every lane has the result.
__device__ __forceinline__ float top_of_lanes(float x)
{
    float y;
    asm volatile("redux.sync.max.f32 %0, %1, 0xFFFFFFFF;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float sum_of_lanes(float x)
{
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) x = __fadd_rn(x, __shfl_xor_sync(0xFFFFFFFFu, x, d));
    return x;
}
__device__ __forceinline__ Sum join_lanes(Sum x)
{
    const float top = top_of_lanes(x.k);
    return Sum{top, sum_of_lanes(__fmul_rn(x.s, exp2_of(x.k - top)))};
}

struct Stats {
    Sum one, two, teacher;
};

__device__ __forceinline__ float teacher_logit(const LossArgs& a, int64_t at)
{
    return a.teacher_bf16 ? load1(static_cast<const __nv_bfloat16*>(a.teacher) + at) : load1(static_cast<const float*>(a.teacher) + at);
}

__device__ __forceinline__ pair exp2_pair(pair x)
{
    float lo, hi;
    split(x, lo, hi);
    return make_pair(exp2_of(lo), exp2_of(hi));
}
template <int N>
__device__ __forceinline__ pair power(pair e)
{
    const pair e2 = mul2(e, e);
    return N == 2 ? e2 : N == 3 ? mul2(e2, e) : mul2(e2, e2);
}

// How many temperatures there are: one; two, each with its own powers; or two of which the first's are the N-th powers of the second's.
constexpr int kOne = 0, kTwo = 1;

template <typename T>
constexpr int kPerSm = sizeof(T) == 4 ? 1024 : 1536;

// The gradient before what is taken off at the label and the teacher's entries: A softmax(z) + B softmax(z / T), with the sums in A and B.
template <int MODE>
struct Softmax {
    float c1, k1, c2, k2, A, B;
    __device__ __forceinline__ pair operator()(pair x) const
    {
        if constexpr (MODE == kOne) return mul2(both(A), exp2_pair(fma2(x, both(c1), both(-k1))));
        else {
            const pair e = exp2_pair(fma2(x, both(c2), both(-k2)));
            const pair f = MODE == kTwo ? exp2_pair(fma2(x, both(c1), both(-k1))) : power<MODE>(e);
            return fma2(both(A), f, mul2(both(B), e));
        }
    }
};

// What a block knows of the teacher's entries, and of the label behind them: index (-1: not there), probability, its logit, the student's, seen twice.
struct Entries {
    int stride;
    int* index;
    float* p;
    float* t_of;
    float* z_of;
    uint8_t* twice;
    __device__ __forceinline__ Entries(float* room, int k)
        : stride((k + 4) / 4 * 4), index(reinterpret_cast<int*>(room)), p(room + stride), t_of(p + stride), z_of(t_of + stride), twice(reinterpret_cast<uint8_t*>(z_of + stride))
    {
    }
};

// What is taken off the gradient at the label and the teacher's entries among the columns [first, last); the same index twice is one element, written with the
// same value.  softmax(x): the gradient before that, of a logit x.
template <int THREADS, typename T, typename F>
__device__ __forceinline__ void take_off(const Entries& e, int k, T* dz, int first, int last, float on_label, float on_teacher, const F& softmax)
{
    const int label = e.index[k];
#pragma unroll 1
    for (int j = threadIdx.x; j <= k; j += THREADS) {
        const int i = e.index[j];
        if (i < first || i >= last) continue;
        const float off = i == label ? on_label : 0.f;
        float sum_p = e.p[j];
        if (k > 0 && e.twice[j]) {
            sum_p = 0.f;
#pragma unroll 1
            for (int m = 0; m < k; ++m)
                if (e.index[m] == i) sum_p = __fadd_rn(sum_p, e.p[m]);
        }
        const float y = softmax(e.z_of[j]);
        store1(dz + i, __fadd_rn(y, -__fmaf_rn(on_teacher, sum_p, off)));
    }
}

// A row that is far out, by the whole block: everything from differences to the largest logit (the largest entry, for the teacher).  Rare, so it is short: one
// element after another (4096 x 30000, all of them such rows: 491 us).  (As a function that is called it took registers from the kernel even where it was not: 4096 x 30000 125 -> 135 us.)  LATER: the
// gradient from the logits, since an lse in binary32 of that magnitude no longer holds the logarithm of the sum; the row's first block does all of it (the row
// may be written in place).
template <typename T, int THREADS, bool LATER>
__device__ __forceinline__ void far_row(const LossArgs& a, const Entries& e, int64_t row, float* of_warp)
{
    const int k = a.k, vocab = a.vocab;
    const T* const z = static_cast<const T*>(a.z) + row * a.ldz;
    const auto over_block = [&](float x, bool largest) {
        x = largest ? top_of_lanes(x) : sum_of_lanes(x);
        __syncthreads();
        if ((threadIdx.x & 31) == 0) of_warp[threadIdx.x >> 5] = x;
        __syncthreads();
        x = of_warp[0];
#pragma unroll 1
        for (int w = 1; w < THREADS / 32; ++w) x = largest ? fmaxf(x, of_warp[w]) : __fadd_rn(x, of_warp[w]);
        return x;
    };
    const auto power_of = [](float far, float c) { return exp2_of(__fmul_rn(far, c)); };
    const float c1 = kLog2e, c2 = a.ct;
    const int64_t label = a.labels ? a.labels[row] : -1;
    bool wrong = label >= vocab;
#pragma unroll 1
    for (int j = threadIdx.x; j < k; j += THREADS) wrong = wrong || (e.t_of[j] != -INFINITY && a.index[row * a.ldt + j] >= vocab);

    // the student's sums
    float top = -INFINITY, s1 = 0.f, s2 = 0.f;
    bool nan = wrong;
#pragma unroll 1
    for (int c = threadIdx.x; c < vocab; c += THREADS) {
        const float x = load1(z + c);
        nan = nan || x != x;
        top = fmaxf(top, x);
    }
    wrong = __syncthreads_or(wrong);
    nan = __syncthreads_or(nan);
    top = over_block(top, true);
#pragma unroll 1
    for (int c0 = threadIdx.x; c0 < vocab; c0 += 32 * THREADS) {
        float part1 = 0.f, part2 = 0.f;              // (32 at a time: few roundings one upon another)
#pragma unroll 1
        for (int c = c0; c < min(vocab, c0 + 32 * THREADS); c += THREADS) {
            const float x = __fadd_rn(load1(z + c), -top);
            part1 = __fadd_rn(part1, power_of(x, c1));
            part2 = __fadd_rn(part2, power_of(x, c2));
        }
        s1 = __fadd_rn(s1, part1);
        s2 = __fadd_rn(s2, part2);
    }
    s1 = over_block(s1, false);
    s2 = over_block(s2, false);
    if (top == -INFINITY) s1 = s2 = 0.f;            // nothing is there: its differences to itself are no numbers
    if (nan) s1 = s2 = __uint_as_float(0x7FC00000u);

    // the teacher's probabilities
    float top_t = -INFINITY, st = 0.f;
    bool entry = false;
#pragma unroll 1
    for (int j = threadIdx.x; j < k; j += THREADS) {
        entry = entry || e.t_of[j] != -INFINITY;
        top_t = fmaxf(top_t, e.t_of[j]);
    }
    const bool has_teacher = __syncthreads_or(entry);
    top_t = over_block(top_t, true);
#pragma unroll 1
    for (int j = threadIdx.x; j < k; j += THREADS)
        if (e.t_of[j] != -INFINITY) st = __fadd_rn(st, power_of(__fadd_rn(e.t_of[j], -top_t), c2));
    st = over_block(st, false);
    constexpr float kLn2 = 0.69314718f;
    const float log_1 = __fmul_rn(kLn2, log2f(s1)), log_2 = __fmul_rn(kLn2, log2f(s2)), log_t = __fmul_rn(kLn2, log2f(st));
    const auto half_of = [](float x, float y) { return __fmaf_rn(0.5f, x, __fmul_rn(-0.5f, y)); };      // of x - y, which may be more than there is
    float loss = 0.f;
#pragma unroll 1
    for (int j = threadIdx.x; j <= k; j += THREADS) {
        float p = 0.f;
        if (j < k && e.t_of[j] != -INFINITY) {
            p = __fdividef(power_of(__fadd_rn(e.t_of[j], -top_t), c2), st);
            if (!LATER && p != 0.f) {                // p wt ((t - top_t - z + top) / T - log_t + log_2)
                const float w = __fmul_rn(p, a.wt), y = __fadd_rn(half_of(e.t_of[j], top_t), -half_of(e.z_of[j], top));
                loss = __fmaf_rn(__fmul_rn(2.f, __fmul_rn(w, a.inverse)), y, __fmaf_rn(w, __fadd_rn(log_2, -log_t), loss));
            }
        } else if (!LATER && j == k && label >= 0) loss = __fmaf_rn(__fmul_rn(-2.f, a.wl), half_of(e.z_of[k], top), __fmaf_rn(a.wl, log_1, loss));
        e.p[j] = p;
    }
    if constexpr (!LATER) {
        loss = over_block(loss, false);
        if (threadIdx.x == 0 && a.loss) a.loss[row] = wrong ? __uint_as_float(0x7FC00000u) : loss;
        if (threadIdx.x == 0 && a.lse) {
            a.lse[2 * row] = __fadd_rn(top, log_1);
            a.lse[2 * row + 1] = __fmaf_rn(top, a.inverse, log_2);
        }
        if (!a.dz) return;
    }

    T* const dz = static_cast<T*>(a.dz) + row * a.lddz;
    const float g = __fmul_rn(a.dloss ? a.dloss[row] : 1.f, a.scale), on_label = label >= 0 ? __fmul_rn(g, a.wl) : 0.f,
                on_teacher = has_teacher ? __fmul_rn(g, __fmul_rn(a.wt, a.inverse)) : 0.f;
    const bool none = on_label == 0.f && on_teacher == 0.f;
    const auto softmax = [&](float x) {
        const float far = __fadd_rn(x, -top);
        float y = on_label != 0.f ? __fmul_rn(on_label, __fdividef(power_of(far, c1), s1)) : 0.f;
        if (on_teacher != 0.f) y = __fmaf_rn(on_teacher, __fdividef(power_of(far, c2), s2), y);
        return y;
    };
#pragma unroll 1
    for (int c = threadIdx.x; c < vocab; c += THREADS) store1(dz + c, none ? 0.f : softmax(load1(z + c)));
    __syncthreads();
    if (!none) take_off<THREADS>(e, k, dz, 0, vocab, on_label, on_teacher, softmax);
}

// THREADS threads with NV groups of eight columns each (a tile); kPerSm threads on an SM.  SHIFT: rows of logits and of the gradient lie alike to the wide boundaries, and columns
// are counted from the boundary in front of the row; else groups begin at column 0 and are taken piece by piece.  LATER: the gradient alone, from lse.
template <typename T, int THREADS, int NV, int MODE, bool SHIFT, bool LATER>
__global__ void __launch_bounds__(THREADS, kPerSm<T> / THREADS) loss_kernel(const LossArgs a)
{
    constexpr int kWarpsHere = THREADS / 32, kTileCols = THREADS * NV * 8;
    constexpr bool kSecond = MODE != kOne;
    extern __shared__ __align__(16) float room[];
    __shared__ Stats of_warp[kWarpsHere];
    __shared__ float part[kWarpsHere];
    const int k = a.k;
    const Entries e(room, k);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int rank = LATER ? (int)(blockIdx.x % (unsigned)a.pieces) : 0;
    const int64_t row = LATER ? blockIdx.x / (unsigned)a.pieces : blockIdx.x;
    const T* const z = static_cast<const T*>(a.z) + row * a.ldz;
    const int shift = SHIFT ? (int)(reinterpret_cast<uintptr_t>(z) / sizeof(T) % 8) : 0;
    const int first = rank * a.piece - shift, last = min(a.vocab, first + a.piece);      // this block's columns, from max(0, first)
    const int tiles = (last - first + kTileCols - 1) / kTileCols;
    after_previous();

    Raw8<T> even[NV], odd[NV];                      // tile t is in the one that its number says
    const auto column = [&](int tile, int v) { return first + tile * kTileCols + (v * THREADS + (int)threadIdx.x) * 8; };
    const T* const mine_z = z + first + (int)threadIdx.x * 8;
    // tiles that are neither the first nor the last are whole, and lie on the wide boundary where rows do (or can be made to)
    constexpr bool kHints = THREADS == 512;          // long rows: what is under way at a time comes near L2's size
    const uint64_t again = keep_long(), done = drop_first();
    const auto request = [&](Raw8<T>(&x)[NV], int tile, bool last_time) {
        if (SHIFT && tile > 0 && tile + 1 < tiles) {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const T* const from = mine_z + (int64_t)tile * kTileCols + v * THREADS * 8;
                if constexpr (kHints) load8(x[v], from, last_time ? done : again);
                else x[v].load(from, true, 8);
            }
            return;
        }
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = column(tile, v), left = max(0, min(8, last - c));
            // what is not a column is -infinity, and adds nothing
            if (SHIFT ? c >= 0 && left == 8 : left == 8) {
                if constexpr (SHIFT) x[v].load(z + c, true, 8);
                else x[v].load(z + c, 8, a.z, a.z_end);
            } else x[v].load_part(z + c, max(0, -c), left);
        }
    };
    request(even, 0, tiles < 3);
    if (tiles > 1) request(odd, 1, tiles < 4);
    // the label and the teacher's entries meanwhile; an index outside the vocabulary makes the row NaN
    const int64_t label64 = a.labels ? a.labels[row] : -1;
    const bool has_label = label64 >= 0;
    const int label = has_label ? (int)min(label64, (int64_t)0x7FFFFFFF) : -1;
    bool wrong = label >= a.vocab;
    Stats mine{Sum{MODE > kTwo ? -kFar * MODE : -kFar, 0.f}, Sum{-kFar, 0.f}, nothing()};
    const float c_most = kSecond ? fmaxf(a.c1, a.c2) : a.c1;
#pragma unroll 1
    for (int j = threadIdx.x; j <= k; j += THREADS) {
        int i = j < k ? a.index[row * a.ldt + j] : label;
        float t = -INFINITY;
        if (j < k && i >= 0) t = teacher_logit(a, row * a.ldt + j);
        const float x = i >= 0 && i < a.vocab ? load1(z + i) : 0.f, tc = __fmul_rn(t, a.ct);
        if (j < k && t == -INFINITY) i = -1;         // not there, whatever the index is
        if (i >= a.vocab) wrong = true, i = -1;
        e.index[j] = i < 0 ? -1 : i;
        e.t_of[j] = t;
        e.z_of[j] = x;
        if (t != -INFINITY) {
            const float kt = fmaxf(ceilf(tc), -kFar);
            mine.teacher.add(kt, exp2_of(__fmaf_rn(t, a.ct, -kt)));
        }
        // a far logit of the student's at the label, or where the teacher's probability is not sure to be 0, makes the row far
        if (!LATER && fabsf(x) * c_most >= kFar && (j == k || tc > -2.f * kFar)) mine.teacher.add(kFar, 0.f);
    }
    if (k > 0) {                                    // entries that share their index with another are rare, and known before they are needed
        __syncthreads();
#pragma unroll 1
        for (int j = threadIdx.x; j <= k; j += THREADS) {
            int same = 0;
            const int i = e.index[j];
#pragma unroll 1
            for (int m = 0; m < k; m += 4) {
                const int4 four = *reinterpret_cast<const int4*>(e.index + m);
                same += (four.x == i) + (m + 1 < k && four.y == i) + (m + 2 < k && four.z == i) + (m + 3 < k && four.w == i);
            }
            e.twice[j] = same > (j < k ? 1 : 0);
        }
    }

    if constexpr (!LATER) {
        const auto add = [&](Raw8<T>(&x)[NV], int tile) {
            float top = x[0].top();
#pragma unroll
            for (int v = 1; v < NV; ++v) top = fmaxf(top, x[v].top());
#pragma unroll
            for (int v = 0; v < NV; ++v) x[v].keep();
            Sum& base = kSecond ? mine.two : mine.one;
            const float kt = __fmul_rn(top, kSecond ? a.c2 : a.c1);
            // a larger value than so far: the whole warp's k moves.  (Of two temperatures each has a step of its own: at a high one logits that differ by
            // hundreds are within one step, at a low one the other's.)
            if (__any_sync(0xFFFFFFFFu, !(kt <= base.k) || (MODE == kTwo && !(__fmul_rn(top, a.c1) <= mine.one.k)))) {
                const float kb = fmaxf(base.k, ceilf(top_of_lanes(kt)));
                base = Sum{kb, __fmul_rn(base.s, exp2_of(base.k - kb))};
                if (kSecond) {
                    const float kf = MODE == kTwo ? fmaxf(mine.one.k, ceilf(__fmul_rn(top_of_lanes(top), a.c1))) : kb * MODE;
                    mine.one = Sum{kf, __fmul_rn(mine.one.s, exp2_of(mine.one.k - kf))};
                }
            }
            const float kb = base.k, kf = mine.one.k;
            const pair cb = both(kSecond ? a.c2 : a.c1), minus_kb = both(-kb), cf = both(a.c1), minus_kf = both(-kf);
            pair sb = both(0.f), sf = both(0.f);
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const p4 y = to_pairs(x[v].values());
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const pair e = exp2_pair(fma2(y.v[q], cb, minus_kb));
                    sb = add2(sb, e);
                    if constexpr (MODE == kTwo) sf = add2(sf, exp2_pair(fma2(y.v[q], cf, minus_kf)));
                    if constexpr (MODE > kTwo) sf = add2(sf, power<MODE>(e));
                }
            }
#pragma unroll
            for (int v = 0; v < NV; ++v) x[v].keep();
            if (tile + 2 < tiles) request(x, tile + 2, tile + 4 >= tiles);      // (the last two stay in registers)
            float lo, hi;
            split(sb, lo, hi);
            base.s = __fadd_rn(base.s, __fadd_rn(lo, hi));
            if (kSecond) {
                split(sf, lo, hi);
                mine.one.s = __fadd_rn(mine.one.s, __fadd_rn(lo, hi));
            }
        };
#pragma unroll 1
        for (int tile = 0; tile < tiles; tile += 2) {
            add(even, tile);
            if (tile + 1 < tiles) add(odd, tile + 1);
        }
    }
    if (wrong) mine.one.s = mine.two.s = mine.teacher.s = __uint_as_float(0x7FC00000u);
    Stats all;
    all.one = Sum{LATER ? 0.f : mine.one.k, sum_of_lanes(mine.one.s)};      // (a warp has one k)
    all.two = kSecond ? Sum{mine.two.k, sum_of_lanes(mine.two.s)} : nothing();
    all.teacher = warp * 32 <= k ? join_lanes(mine.teacher) : nothing();
    if (lane == 0) of_warp[warp] = all;
    __syncthreads();
    {
        const bool has = lane < kWarpsHere;
        const Stats w = of_warp[has ? lane : 0];
        all.one = join_lanes(has ? w.one : nothing());
        if (kSecond) all.two = join_lanes(has ? w.two : nothing());
        all.teacher = join_lanes(has ? w.teacher : nothing());
    }

    const bool has_teacher = k > 0 && !(all.teacher.s == 0.f);
    if constexpr (LATER) {                          // (no sums so far, but NaN where an index is wrong)
        const float l0 = a.lse[2 * row], l1 = a.lse[2 * row + 1], one = all.one.s != all.one.s ? all.one.s : 1.f;
        all.one = Sum{__fmul_rn(a.main_is_teacher ? l1 : l0, kLog2e), one};
        if (kSecond) all.two = Sum{__fmul_rn(l1, kLog2e), one};
    }
    // (all threads of the block are of one mind)
    if (__builtin_expect((LATER ? fabsf(all.one.k) >= kFar || (kSecond && fabsf(all.two.k) >= kFar) || is_far(all.teacher.k)
              : is_far(kSecond ? all.two.k : all.one.k) || (MODE == kTwo && is_far(all.one.k)) || is_far(all.teacher.k)), 0)) {
        if (rank == 0) far_row<T, THREADS, LATER>(a, e, row, part);
        return;
    }
    const Sum& of_teacher = kSecond ? all.two : all.one;      // the student's sum at the teacher's temperature
    const float c_teacher = kSecond ? a.c2 : a.c1;

    // the teacher's probabilities, and the loss
    if (warp * 32 <= k) {
        float sum = 0.f;
        const float log_t = has_teacher ? log2f(all.teacher.s) : 0.f, log_s = LATER ? 0.f : log2f(of_teacher.s);
#pragma unroll 1
        for (int j = threadIdx.x; j <= k; j += THREADS) {
            float pj = 0.f;
            if (j < k && e.t_of[j] != -INFINITY) {
                const float u = __fmaf_rn(e.t_of[j], a.ct, -all.teacher.k);
                pj = __fdividef(exp2_of(u), all.teacher.s);
                if constexpr (!LATER) {
                    const float kl = __fadd_rn(u - log_t, -(__fmaf_rn(e.z_of[j], c_teacher, -of_teacher.k) - log_s));
                    if (pj != 0.f) sum = __fmaf_rn(__fmul_rn(pj, a.wt), kl, sum);
                }
            } else if (!LATER && j == k && has_label) {
                sum = __fmaf_rn(a.wl, log2f(all.one.s) - __fmaf_rn(e.z_of[k], a.c1, -all.one.k), sum);
            }
            e.p[j] = pj;
        }
        if constexpr (!LATER) {
            if (wrong) sum = __uint_as_float(0x7FC00000u);
            if (a.loss) {
                sum = sum_of_lanes(sum);
                if (lane == 0) part[warp] = sum;
            }
        }
    }
    if (!LATER && a.lse && rank == 0 && threadIdx.x == 0) {
        const float one = __fmul_rn(log2_of(all.one), 0.69314718f), two = kSecond ? __fmul_rn(log2_of(all.two), 0.69314718f) : one;
        a.lse[2 * row] = one;
        a.lse[2 * row + 1] = two;
    }

    // the gradient
    float on_label = 0.f, on_teacher = 0.f;
    Softmax<MODE> softmax;
    bool none = true;
    if (a.dz) {
        const float g = __fmul_rn(a.dloss ? a.dloss[row] : 1.f, a.scale);
        on_label = has_label ? __fmul_rn(g, a.wl) : 0.f;
        on_teacher = has_teacher ? __fmul_rn(g, __fdividef(a.wt, a.temperature)) : 0.f;
        const float main = kSecond ? on_label : __fadd_rn(on_label, on_teacher);
        softmax = Softmax<MODE>{a.c1, all.one.k, a.c2, all.two.k, main != 0.f ? __fdividef(main, all.one.s) : 0.f, kSecond && on_teacher != 0.f ? __fdividef(on_teacher, all.two.s) : 0.f};
        none = on_label == 0.f && on_teacher == 0.f;
        T* const dz = static_cast<T*>(a.dz) + row * a.lddz;
        T* const mine_dz = dz + first + (int)threadIdx.x * 8;
        const auto turn = [&](Raw8<T>(&x)[NV], int tile) {
            const bool whole = SHIFT && tile > 0 && tile + 1 < tiles;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                p4 y = to_pairs(x[v].values());
                if (none) y = p4{};
                else {
#pragma unroll
                    for (int q = 0; q < 4; ++q) y.v[q] = softmax(y.v[q]);
                }
                const f8 d = to_values(y);
                if (whole) {
                    T* const to = mine_dz + (int64_t)tile * kTileCols + v * THREADS * 8;
                    if constexpr (kHints) store8(to, d, done);
                    else ops::store8(to, d);
                    continue;
                }
                const int c = column(tile, v), left = max(0, min(8, last - c));
                if constexpr (SHIFT) {
                    if (c >= 0 && left == 8) ops::store8(dz + c, d);
                    else store_part(dz + c, d, max(0, -c), left);
                } else if (left > 0) store_unaligned(dz + c, d, left);
            }
            // (from the gradient's first tile, which holds the last columns, to the row's first: in place, what is read has not been written)
            if (tile > 1) request(x, tile - 2, true);
        };
#pragma unroll 1
        for (int tile = (tiles - 1) | 1; tile > 0; tile -= 2) {
            if (tile < tiles) turn(odd, tile);
            turn(even, tile - 1);
        }
    }
    __syncthreads();
    if (!LATER && a.loss && rank == 0 && threadIdx.x == 0) {
        float s = part[0];
#pragma unroll 1
        for (int w = 1; w < kWarpsHere && w * 32 <= k; ++w) s = __fadd_rn(s, part[w]);
        a.loss[row] = __fmul_rn(s, 0.69314718f);
    }
    if (none) return;
    take_off<THREADS>(e, k, static_cast<T*>(a.dz) + row * a.lddz, max(0, first), last, on_label, on_teacher, [&](float x) {
        float lo, hi;
        split(softmax(both(x)), lo, hi);
        return lo;
    });
}

template <typename T, int THREADS, int NV, bool LATER>
int loss_launch(const char* what, LossArgs& a, int mode, bool shift, cudaStream_t s)
{
    const dim3 grid((unsigned)((int64_t)a.rows * a.pieces));
    const size_t smem = (size_t)((a.k + 4) / 4 * 4) * 17;
    const auto go = [&](auto kernel) { return launch_early(what, kernel, grid, THREADS, smem, s, a); };
    if (mode == kOne) return shift ? go(loss_kernel<T, THREADS, NV, kOne, true, LATER>) : go(loss_kernel<T, THREADS, NV, kOne, false, LATER>);
    if constexpr (!LATER) {
        if (shift && mode == 2) return go(loss_kernel<T, THREADS, NV, 2, true, LATER>);
        if (shift && mode == 3) return go(loss_kernel<T, THREADS, NV, 3, true, LATER>);
        if (shift && mode == 4) return go(loss_kernel<T, THREADS, NV, 4, true, LATER>);
    }
    return shift ? go(loss_kernel<T, THREADS, NV, kTwo, true, LATER>) : go(loss_kernel<T, THREADS, NV, kTwo, false, LATER>);
}

template <typename T, bool LATER>
int loss_types(const char* what, LossArgs& a, int mode, bool shift, cudaStream_t s)
{
    const int64_t cols = (int64_t)a.vocab + (shift ? 7 : 0);      // counted from the boundary in front of the row
    a.pieces = 1;
    a.piece = (int)((cols + 7) / 8 * 8);
    if constexpr (LATER) {                           // nothing is waited for: two tiles a block
        if (cols <= 1024) return loss_launch<T, 128, 1, LATER>(what, a, mode, shift, s);
        a.piece = std::min(a.piece, 2 * 256 * 2 * 8);
        a.pieces = (int)((cols + a.piece - 1) / a.piece);
        return loss_launch<T, 256, 2, LATER>(what, a, mode, shift, s);
    } else {
        // Rows of which six an SM, as blocks of 256 threads are held, do not fit L2 with room for what is written: three blocks of 512 an SM, and L2 is told
        // what will be read again (4096 x 131072 bf16: 428 us; 450 without the hints; 490 with blocks of 256; one block of 1024 an SM 557).  Shorter ones: blocks of
        // 256 (4096 x 30000: 127 us; of 512 139).
        if (cols * (int64_t)sizeof(T) * 148 * 6 > (96 << 20)) return loss_launch<T, 512, 2, LATER>(what, a, mode, shift, s);
        if (cols <= 1024) return loss_launch<T, 128, 1, LATER>(what, a, mode, shift, s);
        return loss_launch<T, 256, 2, LATER>(what, a, mode, shift, s);
    }
}

int run_loss(const char* what, const hpsgd_distill_loss_args* args, bool later, void* stream)
{
    if (!args) return report(HPSGD_E_BADARG, "%s: args is NULL", what);
    hpsgd_distill_loss_args p = *args;
    if (p.rows < 0 || p.vocab < 0 || p.k < 0) return report(HPSGD_E_BADARG, "%s: a size is negative", what);
    if ((p.dtype != HPSGD_F32 && p.dtype != HPSGD_BF16) || (p.teacher_dtype != HPSGD_F32 && p.teacher_dtype != HPSGD_BF16))
        return report(HPSGD_E_BADARG, "%s: unknown dtype", what);
    if (!(p.temperature > 0.0) || !std::isfinite((float)(1.0 / p.temperature)) || !std::isfinite((float)(p.temperature * p.temperature)) || (float)(p.temperature * p.temperature) == 0.f)
        return report(HPSGD_E_BADARG, "%s: temperature must be positive, and its square and its inverse finite in binary32", what);
    if (!(p.label_weight >= 0.0) || !(p.teacher_weight >= 0.0) || !std::isfinite((float)p.label_weight) || !std::isfinite((float)(p.teacher_weight * p.temperature * p.temperature)))
        return report(HPSGD_E_BADARG, "%s: weights must be >= 0 and finite", what);
    if (!std::isfinite((float)p.grad_scale)) return report(HPSGD_E_BADARG, "%s: grad_scale is not finite", what);
    if (p.k > kMaxTeacher) return report(HPSGD_E_UNSUPPORTED, "%s: at most %d teacher entries a row", what, kMaxTeacher);
    if (p.rows > 0x7FFFFFFF || p.vocab > 0x7FFFFFFF - 65536 || p.rows * ((p.vocab + 8191) / 8192 + 1) > 0x7FFFFFFF) return report(HPSGD_E_UNSUPPORTED, "%s: a size is too large", what);
    if (p.rows == 0 || p.vocab == 0) return HPSGD_OK;
    if (!p.logits) return report(HPSGD_E_BADARG, "%s: logits is NULL", what);
    if (later ? !p.dlogits : !p.loss && !p.lse && !p.dlogits) return report(HPSGD_E_BADARG, "%s: no output is asked for", what);
    if (later && !p.lse) return report(HPSGD_E_BADARG, "%s: lse is NULL", what);
    if (p.k > 0 && (!p.teacher_index || !p.teacher_logits)) return report(HPSGD_E_BADARG, "%s: teacher_index or teacher_logits is NULL", what);
    if (p.ldlogits == 0) p.ldlogits = p.vocab;
    if (p.lddlogits == 0) p.lddlogits = p.vocab;
    if (p.ldteacher == 0) p.ldteacher = p.k;
    const int64_t esz = p.dtype == HPSGD_F32 ? 4 : 2, unit = esz * 8;
    if (p.ldlogits < p.vocab || (p.dlogits && p.lddlogits < p.vocab) || p.ldteacher < p.k) return report(HPSGD_E_BADARG, "%s: a stride is below the row's length", what);
    if (p.dlogits == p.logits && p.lddlogits != p.ldlogits) return report(HPSGD_E_BADARG, "%s: logits and dlogits are the same memory with different strides", what);
    if (!aligned(p.logits, esz) || !aligned(p.dlogits, esz) || !aligned(p.labels, 8) || !aligned(p.teacher_index, 4) || !aligned(p.teacher_logits, p.teacher_dtype == HPSGD_F32 ? 4 : 2) ||
        !aligned(p.loss, 4) || !aligned(p.lse, 4) || !aligned(p.dloss, 4))
        return report(HPSGD_E_BADARG, "%s: an address is not aligned to its elements", what);
    int sms = 0;
    OPS_TRY(device_sms(&sms));
    LossArgs a{};
    a.rows = (int)p.rows; a.vocab = (int)p.vocab;
    const bool label = p.labels && p.label_weight > 0.0, teacher = p.k > 0 && p.teacher_weight > 0.0;
    a.k = teacher ? (int)p.k : 0;
    a.z = p.logits; a.labels = label ? p.labels : nullptr; a.index = p.teacher_index; a.teacher = p.teacher_logits;
    a.loss = p.loss; a.lse = p.lse; a.dz = p.dlogits; a.dloss = p.dloss;
    a.ldz = p.ldlogits; a.ldt = p.ldteacher; a.lddz = p.lddlogits;
    a.z_end = static_cast<const char*>(p.logits) + ((p.rows - 1) * p.ldlogits + p.vocab) * esz;
    const double log2e = 1.4426950408889634;
    const bool same = p.temperature == 1.0, two = !same && ((p.lse && !later) || (label && teacher));
    a.main_is_teacher = !same && !two && teacher;
    a.c1 = (float)(a.main_is_teacher ? log2e / p.temperature : log2e);
    a.c2 = a.ct = (float)(log2e / p.temperature);
    a.wl = (float)p.label_weight; a.wt = (float)(p.teacher_weight * p.temperature * p.temperature);
    a.temperature = (float)p.temperature; a.inverse = (float)(1.0 / p.temperature); a.scale = (float)p.grad_scale;
    a.teacher_bf16 = p.teacher_dtype == HPSGD_BF16;
    // rows of both lie alike to the wide boundaries
    const bool shift = !p.dlogits || ((reinterpret_cast<uintptr_t>(p.logits) - reinterpret_cast<uintptr_t>(p.dlogits)) % unit == 0 && (p.ldlogits - p.lddlogits) * esz % unit == 0);
    const bool whole = p.temperature == 2.0 || p.temperature == 3.0 || p.temperature == 4.0;
    const int mode = !two ? kOne : whole && !later ? (int)p.temperature : kTwo;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (later) return p.dtype == HPSGD_F32 ? loss_types<float, true>(what, a, mode, shift, s) : loss_types<__nv_bfloat16, true>(what, a, mode, shift, s);
    return p.dtype == HPSGD_F32 ? loss_types<float, false>(what, a, mode, shift, s) : loss_types<__nv_bfloat16, false>(what, a, mode, shift, s);
}

}  // namespace
}  // namespace ops
}  // namespace hpsgd

using namespace hpsgd;
using namespace hpsgd::ops;

extern "C" {

int hpsgd_distill_loss(const hpsgd_distill_loss_args* args, void* stream) { return run_loss("hpsgd_distill_loss", args, false, stream); }

int hpsgd_distill_loss_backward(const hpsgd_distill_loss_args* args, void* stream) { return run_loss("hpsgd_distill_loss_backward", args, true, stream); }

}  // extern "C"
