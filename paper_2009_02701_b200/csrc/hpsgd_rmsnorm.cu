// Root-mean-square norm: residual addition, normalisation and 8-bit output in one pass; its gradients in one pass and a
// short sum.
//
// Bound by HBM: 7 bytes an element forward (bf16 in, residual in, sum out, codes out), 8 backward.  A row is held in the
// registers of 32 to 512 threads, eight consecutive columns a thread and group, so it is read once; 16 neighbouring threads hold a
// 128-column block of the output, whose scale is then a matter of shuffles.
#include "hpsgd_ops_common.cuh"

namespace hpsgd {
namespace ops {

HPSGD_HIDDEN int check_fp8(const char* what, const char* name, const void* q, const void* s, int64_t* ld, int64_t* lds, int64_t rows, int64_t cols);

namespace {

constexpr int64_t kMaxCols = 16384;

// Sum over the T threads of a row; T <= 32 within the warp, else through shared memory (one value per warp, two buffers in turn, so
// that one barrier a row is enough).
template <int T>
__device__ __forceinline__ float row_sum(float x, float (*buf)[32], int turn)
{
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) x += __shfl_xor_sync(0xFFFFFFFFu, x, d);
    if constexpr (T > 32) {
        constexpr int kWarps = T / 32;
        const int warp = threadIdx.x >> 5, first = warp / kWarps * kWarps;
        if ((threadIdx.x & 31) == 0) buf[turn][warp] = x;
        __syncthreads();
        x = buf[turn][first];
#pragma unroll
        for (int w = 1; w < kWarps; ++w) x += buf[turn][first + w];
    }
    return x;
}

// ---------------------------------------------------------------------------- forward
struct Forward {
    int64_t rows, cols, ldx, ldres, ldh, ldy, ldy8, ldys;
    const void* x;
    const void* res;
    const void* w;
    void* h;
    void* y;
    uint8_t* y8;
    uint8_t* ys;
    float* rstd;
    const void* x_end;
    const void* res_end;
    float eps, inv_cols;
    bool wide, wide_w;
};

// T threads a row, V groups of eight a thread, R = threads of a block / T rows a block.  WIDE: all rows allow the wide accesses; the other
// form is a kernel of its own, so that its code is not in the way (8192 x 2007 bf16 with a residual: 42 us, 2004: 35; value by value both took 55).
template <typename X, typename W, int T, int V, bool WIDE>
__global__ void __launch_bounds__(T < 128 ? 128 : T) rmsnorm_forward_kernel(const Forward a)
{
    __shared__ float buf[1][32];
    constexpr int kRows = T < 128 ? 128 / T : 1;
    const int t = threadIdx.x % T;
    const int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / T;
    const bool in = row < a.rows;
    const auto fetch = [&](Raw8<X>& v, const void* p, const void* end, int64_t ld, int c, int left) {
        if constexpr (WIDE) v.load(static_cast<const X*>(p) + row * ld + c, left == 8, left);
        else v.load(static_cast<const X*>(p) + row * ld + c, left, p, end);
    };
    const auto store = [&](void* p, int64_t ld, int c, const f8& v, int left) {
        if constexpr (WIDE) store_some(static_cast<X*>(p) + row * ld + c, v, left == 8, left);
        else store_unaligned(static_cast<X*>(p) + row * ld + c, v, left);
    };
    f8 f[V];
    Raw8<X> x[V], r[V];
    Raw8<W> w[V];
    after_previous();
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const int c = (k * T + t) * 8, left = in ? max(0, min(8, (int)a.cols - c)) : 0;
        fetch(x[k], a.x, a.x_end, a.ldx, c, left);
        if (a.res) fetch(r[k], a.res, a.res_end, a.ldres, c, left);
    }
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const int c = (k * T + t) * 8, left = in ? max(0, min(8, (int)a.cols - c)) : 0;
        w[k].load(static_cast<const W*>(a.w) + c, a.wide_w && left == 8, left);
    }
    float ss = 0.f;
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const int c = (k * T + t) * 8, left = in ? max(0, min(8, (int)a.cols - c)) : 0;
        f[k] = x[k].values();
        if (a.res) {
            const f8 rk = r[k].values();
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const float s = __fadd_rn(f[k].v[q], rk.v[q]);
                f[k].v[q] = sizeof(X) == 2 ? __bfloat162float(__float2bfloat16_rn(s)) : s;
            }
            store(a.h, a.ldh, c, f[k], left);
        }
#pragma unroll
        for (int q = 0; q < 8; ++q) ss = __fmaf_rn(f[k].v[q], f[k].v[q], ss);
    }
    ss = row_sum<T>(ss, buf, 0);
    const float rstd = __frcp_rn(__fsqrt_rn(__fmaf_rn(ss, a.inv_cols, a.eps)));
    if (in && t == 0 && a.rstd) a.rstd[row] = rstd;
    const int blocks = (int)((a.cols + kBlock - 1) / kBlock), words4 = (blocks + 3) / 4 * 4, pad = (int)((a.cols + 15) / 16 * 16);
#pragma unroll
    for (int k = 0; k < V; ++k) {
        const int c = (k * T + t) * 8, left = in ? max(0, min(8, (int)a.cols - c)) : 0;
        const f8 wk = w[k].values();
        f8 y;
#pragma unroll
        for (int q = 0; q < 8; ++q) y.v[q] = __fmul_rn(__fmul_rn(f[k].v[q], rstd), wk.v[q]);
        if (left < 8) {                               // zeros behind the last column, even in a row whose rstd is NaN
#pragma unroll
            for (int q = 0; q < 8; ++q)
                if (q >= left) y.v[q] = 0.f;
        }
        if (a.y) store(a.y, a.ldy, c, y, left);
        if (a.y8) {
            const int byte = block_scale(y);
            if (in && c < pad) *reinterpret_cast<uint2*>(a.y8 + row * a.ldy8 + c) = encode_nearest(y, byte);
            const int b = c / kBlock;                 // a row's threads cover whole words of four blocks, so the padding comes with them
            const int upper = __shfl_down_sync(0xFFFFFFFFu, byte, 16);
            if (in && (threadIdx.x & 31) == 0 && b < words4)
                *reinterpret_cast<uint16_t*>(a.ys + scale_index(b, row, a.ldys)) = (uint16_t)(byte | upper << 8);
        }
    }
}

template <typename X, typename W, int T, int V>
int forward_launch(const Forward& a, cudaStream_t s)
{
    constexpr int kRows = T < 128 ? 128 / T : 1;
    const int64_t blocks = (a.rows + kRows - 1) / kRows;
    if (blocks > 0x7FFFFFFF) return report(HPSGD_E_UNSUPPORTED, "hpsgd_rmsnorm_forward: too many rows");
    return launch_early("hpsgd_rmsnorm_forward", a.wide ? rmsnorm_forward_kernel<X, W, T, V, true> : rmsnorm_forward_kernel<X, W, T, V, false>, dim3((unsigned)blocks), T < 128 ? 128 : T, 0, s, a);
}

template <typename X, typename W>
int forward_types(const Forward& a, cudaStream_t s)
{
    // A row's threads cover at least 512 columns (whole words of scales).  With rows enough to fill the device a thread takes two groups of
    // a row, and has twice the bytes under way while it waits for the row's sum (16384 x 4096 bf16 with a residual: 83 us, 103 with one);
    // with fewer, a row is finished sooner by more threads.
    const bool many = a.rows >= 8 * 148;
    if (a.cols <= 512) return forward_launch<X, W, 64, 1>(a, s);
    if (a.cols <= 1024) return many ? forward_launch<X, W, 64, 2>(a, s) : forward_launch<X, W, 128, 1>(a, s);
    if (a.cols <= 2048) return many ? forward_launch<X, W, 128, 2>(a, s) : forward_launch<X, W, 256, 1>(a, s);
    if (a.cols <= 4096) return many ? forward_launch<X, W, 256, 2>(a, s) : forward_launch<X, W, 512, 1>(a, s);
    if (a.cols <= 8192) return forward_launch<X, W, 512, 2>(a, s);
    return forward_launch<X, W, 512, 4>(a, s);
}

// ---------------------------------------------------------------------------- backward
struct Backward {
    int64_t rows, cols, ldh, lddy, lddres, lddx;
    const void* h;
    const void* w;
    const float* rstd;
    const void* dy;
    const void* dres;
    void* dx;
    float* part;           // [blocks][cols]
    float inv_cols;
    bool wide, wide_w;
};

constexpr int kBackBlocks = 592;      // most partial sums of dweight: four blocks on each of 148 SMs

// T threads a row; a block of 256 takes 256 / T rows at a time (512 threads take one), and goes through the rows in steps of the grid.  A
// thread's columns stay the same from row to row, so their dweight is added in registers.
// With one group a thread the next row's values are requested before the present row's sum is waited for; with two, the registers
// go to the row itself; with four, the row and the weights are read a second time behind the sum, from L1 and L2.
template <typename X, int T, int V>
struct Back {
    static constexpr int kThreads = T < 256 ? 256 : T;
    static constexpr int kPerSm = V == 1 ? (sizeof(X) == 2 ? 1024 : 768) / kThreads : 1;      // blocks that an SM holds
};

template <typename X, typename W, int T, int V>
__global__ void __launch_bounds__(Back<X, T, V>::kThreads, Back<X, T, V>::kPerSm) rmsnorm_backward_kernel(const Backward a)
{
    __shared__ float buf[2][32];
    constexpr bool kAhead = V == 1, kKeep = V <= 2;
    constexpr int kThreads = Back<X, T, V>::kThreads, kRows = kThreads / T;
    const int t = threadIdx.x % T, group = threadIdx.x / T;
    f8 dw[V];
    Raw8<W> w[V];
    Raw8<X> h[V], dy[V], dres[V];
    const auto left = [&](int k) { return max(0, min(8, (int)a.cols - (k * T + t) * 8)); };
    const auto load_w = [&](int k) { w[k].load(static_cast<const W*>(a.w) + (k * T + t) * 8, a.wide_w && left(k) == 8, left(k)); };
    const auto fetch = [&](Raw8<X>& x, const void* p, int64_t ld, int64_t r, int k) {
        const int here = r < a.rows ? left(k) : 0;
        x.load(static_cast<const X*>(p) + r * ld + (k * T + t) * 8, a.wide && here == 8, here);
    };
    after_previous();
    const auto rstd_of = [&](int64_t r) { return r < a.rows ? a.rstd[r] : 0.f; };
#pragma unroll
    for (int k = 0; k < V; ++k) {
        if (kKeep) load_w(k);
#pragma unroll
        for (int q = 0; q < 8; ++q) dw[k].v[q] = 0.f;
    }
    int64_t first = (int64_t)blockIdx.x * kRows;
    const int64_t step = (int64_t)gridDim.x * kRows;
    Raw8<X> nh = {}, ndy = {}, ndres = {};
    float next_rstd = 0.f;
    const auto ahead = [&](int64_t r) {
        fetch(nh, a.h, a.ldh, r, 0);
        fetch(ndy, a.dy, a.lddy, r, 0);
        if (a.dres) fetch(ndres, a.dres, a.lddres, r, 0);
        next_rstd = rstd_of(r);
    };
    if (kAhead) ahead(first + group);
    for (int turn = 0; first < a.rows; first += step, turn ^= 1) {
        const int64_t row = first + group;
        const float rs = kAhead ? next_rstd : rstd_of(row);
#pragma unroll
        for (int k = 0; k < V; ++k) {
            if (kAhead) {
                h[k] = nh;
                dy[k] = ndy;
                dres[k] = ndres;
            } else if (kKeep) {
                fetch(h[k], a.h, a.ldh, row, k);
                fetch(dy[k], a.dy, a.lddy, row, k);
                if (a.dres) fetch(dres[k], a.dres, a.lddres, row, k);
            }
        }
        if (kAhead && first + step < a.rows) ahead(row + step);
        float dot = 0.f;
#pragma unroll
        for (int k = 0; k < V; ++k) {
            if (!kKeep) {
                load_w(k);
                fetch(h[k], a.h, a.ldh, row, k);
                fetch(dy[k], a.dy, a.lddy, row, k);
            }
            const f8 wk = w[k].values(), hk = h[k].values(), dk = dy[k].values();
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const float xn = __fmul_rn(hk.v[q], rs);
                dw[k].v[q] = __fmaf_rn(dk.v[q], xn, dw[k].v[q]);
                dot = __fmaf_rn(__fmul_rn(dk.v[q], wk.v[q]), xn, dot);
            }
        }
        const float mean = __fmul_rn(row_sum<T>(dot, buf, turn), a.inv_cols);
#pragma unroll
        for (int k = 0; k < V; ++k) {
            if (!kKeep) {
                load_w(k);
                fetch(h[k], a.h, a.ldh, row, k);
                fetch(dy[k], a.dy, a.lddy, row, k);
                if (a.dres) fetch(dres[k], a.dres, a.lddres, row, k);
            }
            const f8 wk = w[k].values(), hk = h[k].values(), dk = dy[k].values(), rk = dres[k].values();
            f8 x;
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const float xn = __fmul_rn(hk.v[q], rs);
                x.v[q] = __fmul_rn(__fmaf_rn(-xn, mean, __fmul_rn(dk.v[q], wk.v[q])), rs);
                if (a.dres) x.v[q] = __fadd_rn(x.v[q], rk.v[q]);
            }
            const int here = row < a.rows ? left(k) : 0;
            store_some(static_cast<X*>(a.dx) + row * a.lddx + (k * T + t) * 8, x, a.wide && here == 8, here);
        }
    }
    // the block's sums: its groups' in their order
    if constexpr (kRows > 1) {
        __shared__ float all[kRows][T * 8];
#pragma unroll
        for (int q = 0; q < 8; ++q) all[group][t * 8 + q] = dw[0].v[q];
        __syncthreads();
        for (int c = threadIdx.x; c < (int)a.cols; c += kThreads) {
            float s = all[0][c];
#pragma unroll
            for (int g = 1; g < kRows; ++g) s += all[g][c];
            a.part[(int64_t)blockIdx.x * a.cols + c] = s;
        }
    } else {
#pragma unroll
        for (int k = 0; k < V; ++k)
#pragma unroll
            for (int q = 0; q < 8; ++q)
                if (q < left(k)) a.part[(int64_t)blockIdx.x * a.cols + (k * T + t) * 8 + q] = dw[k].v[q];
    }
}

// dweight[c] = sum of the blocks' partial sums, in an order that depends on their number alone: 32 threads a column, each adding every
// 32nd block's, then a tree.
__global__ void __launch_bounds__(1024) dweight_kernel(const float* part, float* dweight, int64_t cols, int blocks)
{
    __shared__ float sum[32][33];
    const int lane = threadIdx.x & 31, y = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;
    float s = 0.f;
    after_previous();
    if (c < cols) {
#pragma unroll 10
        for (int b = y; b < blocks; b += 32) s += part[(int64_t)b * cols + c];
    }
    sum[y][lane] = s;
    __syncthreads();
    s = sum[lane][y];                              // now the column is block * 32 + y, and its 32 sums lie along the warp
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
    const int64_t cy = (int64_t)blockIdx.x * 32 + y;
    if (lane == 0 && cy < cols) dweight[cy] = s;
}

template <typename X, typename W, int T, int V>
int backward_launch(const Backward& a, float* dweight, cudaStream_t s)
{
    // as many blocks as are resident at once, of which each has a row to begin with (half a block an SM more, with fp32 on 512 threads, went through
    // the rows behind the others: 8192 x 4096: 101 us, 86 with whole blocks)
    using B = Back<X, T, V>;
    constexpr int kRows = B::kThreads / T, kResident = 148 * B::kPerSm;
    static_assert(kResident <= kBackBlocks, "the workspace holds kBackBlocks partial sums");
    const int64_t need = (a.rows + kRows - 1) / kRows;
    const int blocks = (int)(need < kResident ? need : kResident);
    OPS_TRY(launch_early("hpsgd_rmsnorm_backward", rmsnorm_backward_kernel<X, W, T, V>, dim3(blocks), B::kThreads, 0, s, a));
    return launch_early("hpsgd_rmsnorm_backward", dweight_kernel, dim3((unsigned)((a.cols + 31) / 32)), 1024, 0, s, (const float*)a.part, dweight, a.cols, blocks);
}

template <typename X, typename W>
int backward_types(const Backward& a, float* dweight, cudaStream_t s)
{
    if (a.cols <= 256) return backward_launch<X, W, 32, 1>(a, dweight, s);
    if (a.cols <= 512) return backward_launch<X, W, 64, 1>(a, dweight, s);
    if (a.cols <= 1024) return backward_launch<X, W, 128, 1>(a, dweight, s);
    if (a.cols <= 2048) return backward_launch<X, W, 256, 1>(a, dweight, s);
    if (a.cols <= 4096) return backward_launch<X, W, 512, 1>(a, dweight, s);
    if (a.cols <= 8192) return backward_launch<X, W, 512, 2>(a, dweight, s);
    return backward_launch<X, W, 512, 4>(a, dweight, s);
}

int check_sizes(const char* what, int64_t rows, int64_t cols, int dtype, int weight_dtype)
{
    if (rows < 0 || cols < 0) return report(HPSGD_E_BADARG, "%s: a size is negative", what);
    if ((dtype != HPSGD_F32 && dtype != HPSGD_BF16) || (weight_dtype != HPSGD_F32 && weight_dtype != HPSGD_BF16))
        return report(HPSGD_E_BADARG, "%s: unknown dtype", what);
    if (cols > kMaxCols) return report(HPSGD_E_UNSUPPORTED, "%s: at most %lld columns", what, (long long)kMaxCols);
    if (rows > 0x7FFFFFFF) return report(HPSGD_E_UNSUPPORTED, "%s: too many rows", what);
    return HPSGD_OK;
}

int check_rows(const char* what, const char* name, const void* p, int64_t* ld, int64_t cols, int dtype, bool* wide)
{
    const int64_t esz = dtype == HPSGD_F32 ? 4 : 2, unit = esz * 8;
    if (!p) return HPSGD_OK;
    if (*ld == 0) *ld = cols;
    if (*ld < cols) return report(HPSGD_E_BADARG, "%s: the stride of %s is below cols", what, name);
    if (!aligned(p, esz)) return report(HPSGD_E_BADARG, "%s: %s is not aligned to its elements", what, name);
    *wide = *wide && aligned(p, unit) && *ld * esz % unit == 0;
    return HPSGD_OK;
}

// Behind the last element of a matrix.
const void* end_of(const void* p, int64_t ld, int64_t rows, int64_t cols, int dtype)
{
    return p ? static_cast<const char*>(p) + ((rows - 1) * ld + cols) * (dtype == HPSGD_F32 ? 4 : 2) : nullptr;
}

}  // namespace
}  // namespace ops
}  // namespace hpsgd

using namespace hpsgd;
using namespace hpsgd::ops;

extern "C" {

int hpsgd_rmsnorm_forward(const hpsgd_rmsnorm_forward_args* args, void* stream)
{
    const char* what = "hpsgd_rmsnorm_forward";
    if (!args) return report(HPSGD_E_BADARG, "%s: args is NULL", what);
    hpsgd_rmsnorm_forward_args p = *args;
    OPS_TRY(check_sizes(what, p.rows, p.cols, p.dtype, p.weight_dtype));
    if (!(p.eps >= 0.0) || !std::isfinite((float)p.eps)) return report(HPSGD_E_BADARG, "%s: eps must be >= 0", what);
    if (p.rows == 0 || p.cols == 0) return HPSGD_OK;
    if (!p.x || !p.weight) return report(HPSGD_E_BADARG, "%s: x or weight is NULL", what);
    if (!p.residual != !p.h) return report(HPSGD_E_BADARG, "%s: residual and h go together", what);
    if (!p.y && !p.y8) return report(HPSGD_E_BADARG, "%s: no output is asked for", what);
    if (!aligned(p.weight, p.weight_dtype == HPSGD_F32 ? 4 : 2) || !aligned(p.rstd, 4)) return report(HPSGD_E_BADARG, "%s: weight or rstd is not aligned to its elements", what);
    Forward a{};
    a.wide = true;
    OPS_TRY(check_rows(what, "x", p.x, &p.ldx, p.cols, p.dtype, &a.wide));
    OPS_TRY(check_rows(what, "residual", p.residual, &p.ldres, p.cols, p.dtype, &a.wide));
    OPS_TRY(check_rows(what, "h", p.h, &p.ldh, p.cols, p.dtype, &a.wide));
    OPS_TRY(check_rows(what, "y", p.y, &p.ldy, p.cols, p.dtype, &a.wide));
    OPS_TRY(check_fp8(what, "y8", p.y8, p.y_scale, &p.ldy8, &p.ldys, p.rows, p.cols));
    int sms = 0;
    OPS_TRY(device_sms(&sms));
    a.rows = p.rows; a.cols = p.cols; a.ldx = p.ldx; a.ldres = p.ldres; a.ldh = p.ldh; a.ldy = p.ldy; a.ldy8 = p.ldy8; a.ldys = p.ldys;
    a.x = p.x; a.res = p.residual; a.w = p.weight; a.h = p.h; a.y = p.y; a.y8 = static_cast<uint8_t*>(p.y8); a.ys = p.y_scale; a.rstd = p.rstd;
    a.eps = (float)p.eps;
    a.x_end = end_of(p.x, p.ldx, p.rows, p.cols, p.dtype); a.res_end = end_of(p.residual, p.ldres, p.rows, p.cols, p.dtype);
    a.inv_cols = (float)(1.0 / (double)p.cols);
    a.wide_w = aligned(p.weight, p.weight_dtype == HPSGD_F32 ? 32 : 16);
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (p.dtype == HPSGD_F32) return p.weight_dtype == HPSGD_F32 ? forward_types<float, float>(a, s) : forward_types<float, __nv_bfloat16>(a, s);
    return p.weight_dtype == HPSGD_F32 ? forward_types<__nv_bfloat16, float>(a, s) : forward_types<__nv_bfloat16, __nv_bfloat16>(a, s);
}

size_t hpsgd_rmsnorm_backward_bytes(int64_t rows, int64_t cols)
{
    if (rows <= 0 || cols <= 0 || cols > kMaxCols) return 0;
    return (size_t)(rows < kBackBlocks ? rows : kBackBlocks) * (size_t)cols * sizeof(float);
}

int hpsgd_rmsnorm_backward(const hpsgd_rmsnorm_backward_args* args, void* stream)
{
    const char* what = "hpsgd_rmsnorm_backward";
    if (!args) return report(HPSGD_E_BADARG, "%s: args is NULL", what);
    hpsgd_rmsnorm_backward_args p = *args;
    OPS_TRY(check_sizes(what, p.rows, p.cols, p.dtype, p.weight_dtype));
    if (p.cols == 0) return HPSGD_OK;
    if (!p.dweight || !aligned(p.dweight, 4)) return report(HPSGD_E_BADARG, "%s: dweight is NULL or not 4-byte aligned", what);
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    int sms = 0;
    if (p.rows == 0) {
        OPS_TRY(device_sms(&sms));
        OPS_CUDA(cudaMemsetAsync(p.dweight, 0, (size_t)p.cols * 4, s));
        return HPSGD_OK;
    }
    if (!p.h || !p.weight || !p.rstd || !p.dy || !p.dx) return report(HPSGD_E_BADARG, "%s: h, weight, rstd, dy or dx is NULL", what);
    if (!p.workspace || !aligned(p.workspace, 16)) return report(HPSGD_E_BADARG, "%s: workspace is NULL or not 16-byte aligned", what);
    if (!aligned(p.weight, p.weight_dtype == HPSGD_F32 ? 4 : 2) || !aligned(p.rstd, 4)) return report(HPSGD_E_BADARG, "%s: weight or rstd is not aligned to its elements", what);
    Backward a{};
    a.wide = true;
    OPS_TRY(check_rows(what, "h", p.h, &p.ldh, p.cols, p.dtype, &a.wide));
    OPS_TRY(check_rows(what, "dy", p.dy, &p.lddy, p.cols, p.dtype, &a.wide));
    OPS_TRY(check_rows(what, "dres", p.dres, &p.lddres, p.cols, p.dtype, &a.wide));
    OPS_TRY(check_rows(what, "dx", p.dx, &p.lddx, p.cols, p.dtype, &a.wide));
    OPS_TRY(device_sms(&sms));
    a.rows = p.rows; a.cols = p.cols; a.ldh = p.ldh; a.lddy = p.lddy; a.lddres = p.lddres; a.lddx = p.lddx;
    a.h = p.h; a.w = p.weight; a.rstd = p.rstd; a.dy = p.dy; a.dres = p.dres; a.dx = p.dx; a.part = static_cast<float*>(p.workspace);
    a.inv_cols = (float)(1.0 / (double)p.cols);
    a.wide_w = aligned(p.weight, p.weight_dtype == HPSGD_F32 ? 32 : 16);
    if (p.dtype == HPSGD_F32)
        return p.weight_dtype == HPSGD_F32 ? backward_types<float, float>(a, p.dweight, s) : backward_types<float, __nv_bfloat16>(a, p.dweight, s);
    return p.weight_dtype == HPSGD_F32 ? backward_types<__nv_bfloat16, float>(a, p.dweight, s) : backward_types<__nv_bfloat16, __nv_bfloat16>(a, p.dweight, s);
}

}  // extern "C"
