// The loss over a label and a teacher's top logits, and its gradient.
//
// Bound by HBM: a row of logits is read once and a row of gradients written once.  A row is held in the registers of one block, or of the
// blocks of a cluster where it is longer than 16384 (8192 in fp32): all of it is requested at once, its sums of exponentials are joined over warps
// and blocks, and what is in the registers then becomes the gradient.  Only rows beyond eight times that are read a second time, out of L2.
//
// Sums of exponentials: s = sum 2^(x c - k) with c = log2(e) / temperature and k the largest x c rounded up to a whole number, so that joining two
// sums multiplies by an exact power of two, and x c - k is rounded once; the softmax is then 2^(x c - k) / s without any error of k's.
#include "hpsgd_ops_common.cuh"

#include <cfloat>

namespace hpsgd {
namespace ops {
namespace {

constexpr int kMaxTeacher = 1024;
constexpr int kMaxLossCluster = 8;

struct LossArgs {
    int rows, vocab, k, pieces, piece;              // pieces: blocks that share a row; piece: columns of each
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
    float c1, c2;                                   // log2(e) over the temperatures; c2 is only used where there are two
    float ct, wl, wt, temperature, scale;           // wt: with the square of the temperature
    int teacher_bf16;
    int later;                                      // the gradient alone, from lse
    int main_is_teacher;                            // c1 is the teacher's temperature
};

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
__device__ __forceinline__ float log2_of(const Sum& x) { return __fadd_rn(x.k, log2f(x.s)); }

// Over the lanes of a warp; every lane has the result.
__device__ __forceinline__ Sum join_lanes(Sum x)
{
    float top = x.k;
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
    x.s = __fmul_rn(x.s, exp2_of(x.k - top));
    x.k = top;
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) x.s = __fadd_rn(x.s, __shfl_xor_sync(0xFFFFFFFFu, x.s, d));
    return x;
}

struct Stats {
    Sum one, two, teacher;
};

__device__ __forceinline__ float teacher_logit(const LossArgs& a, int64_t at)
{
    return a.teacher_bf16 ? load1(static_cast<const __nv_bfloat16*>(a.teacher) + at) : load1(static_cast<const float*>(a.teacher) + at);
}

// THREADS threads with NV groups of eight columns each (a tile); TWO: two temperatures; WIDE: rows allow the wide accesses.
template <typename T, int THREADS, int NV, bool TWO, bool WIDE, bool CLUSTER>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) loss_kernel(const LossArgs a)
{
    constexpr int kWarpsHere = THREADS / 32, kTileCols = THREADS * NV * 8;
    extern __shared__ float room[];                 // of each teacher entry, and of the label behind them: index, probability, its logit, the student's
    __shared__ Stats of_warp[kWarpsHere];
    __shared__ alignas(8) Stats of_block[kMaxLossCluster];
    __shared__ float part[kWarpsHere];
    const int k = a.k;
    int* const index = reinterpret_cast<int*>(room);
    float* const p = room + (k + 1);
    float* const t_of = p + (k + 1);
    float* const z_of = t_of + (k + 1);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int rank = CLUSTER ? (int)(blockIdx.x % (unsigned)a.pieces) : 0;
    const int64_t row = CLUSTER ? blockIdx.x / (unsigned)a.pieces : blockIdx.x;
    const T* const z = static_cast<const T*>(a.z) + row * a.ldz;
    const int first = rank * a.piece, cols = min(a.piece, a.vocab - first);      // this block's columns
    if constexpr (CLUSTER) cluster_arrive();        // the others' memory is there to be written; waited for below
    after_previous();

    Raw8<T> x[NV];
    const auto request = [&](int tile) {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = tile + (v * THREADS + (int)threadIdx.x) * 8, left = max(0, min(8, cols - c));
            if constexpr (WIDE) x[v].load(z + first + c, left == 8, left);
            else x[v].load(z + first + c, left, a.z, a.z_end);
        }
    };
    request(0);
    // the label and the teacher's entries meanwhile; an index outside the vocabulary makes the row NaN
    const int64_t label64 = a.labels ? a.labels[row] : -1;
    const bool has_label = label64 >= 0;
    const int label = has_label ? (int)min(label64, (int64_t)0x7FFFFFFF) : -1;
    bool wrong = label >= a.vocab;
    Stats mine{nothing(), nothing(), nothing()};
    for (int j = threadIdx.x; j <= k; j += THREADS) {
        int i = j < k ? a.index[row * a.ldt + j] : label;
        float t = -INFINITY;
        if (j < k && i >= 0) t = teacher_logit(a, row * a.ldt + j);
        if (i >= a.vocab) wrong = true, i = -1;
        index[j] = i < 0 ? -1 : i;
        t_of[j] = t;
        z_of[j] = i >= 0 ? load1(z + i) : 0.f;
        if (t != -INFINITY) {
            const float kt = ceilf(__fmul_rn(t, a.ct));
            mine.teacher.add(kt, exp2_of(__fmaf_rn(t, a.ct, -kt)));
        }
    }

    if (!a.later) {
        for (int tile = 0; tile < cols; tile += kTileCols) {
            if (tile > 0) request(tile);
            float top = -INFINITY;
            f8 y[NV];
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int left = cols - tile - (v * THREADS + (int)threadIdx.x) * 8;
                y[v] = x[v].values();
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    if (q >= left) y[v].v[q] = -INFINITY;
                    top = fmaxf(top, y[v].v[q]);
                }
            }
            const auto sum = [&](Sum& into, float c) {
                const float kk = fmaxf(into.k, ceilf(__fmul_rn(top, c)));
                float s = __fmul_rn(into.s, exp2_of(into.k - kk));
#pragma unroll
                for (int v = 0; v < NV; ++v)
#pragma unroll
                    for (int q = 0; q < 8; ++q) s = __fadd_rn(s, exp2_of(__fmaf_rn(y[v].v[q], c, -kk)));
                into = Sum{kk, s};
            };
            sum(mine.one, a.c1);
            if (TWO) sum(mine.two, a.c2);
        }
    }
    if (wrong) mine.one.s = mine.two.s = mine.teacher.s = __uint_as_float(0x7FC00000u);
    Stats all{join_lanes(mine.one), TWO ? join_lanes(mine.two) : nothing(), k > 0 ? join_lanes(mine.teacher) : nothing()};
    if (lane == 0) of_warp[warp] = all;
    __syncthreads();
    if (!CLUSTER || warp == 0) {
        const bool has = lane < kWarpsHere;
        const Stats w = of_warp[has ? lane : 0];
        all = Stats{join_lanes(has ? w.one : nothing()), TWO ? join_lanes(has ? w.two : nothing()) : nothing(), join_lanes(has ? w.teacher : nothing())};
    }
    if constexpr (CLUSTER) {
        cluster_wait();
        if (warp == 0 && lane < a.pieces) {
            uint32_t there;
            asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(shared_address(&of_block[rank])), "r"(lane));
            asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(there), "f"(all.one.k), "f"(all.one.s) : "memory");
            asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(there + 8), "f"(all.two.k), "f"(all.two.s) : "memory");
            asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(there + 16), "f"(all.teacher.k), "f"(all.teacher.s) : "memory");
        }
        __syncwarp();
        cluster_arrive();
        cluster_wait();
        all = of_block[0];                          // (every block has the whole teacher)
        for (int r = 1; r < a.pieces; ++r) {
            const Stats s = of_block[r];
            all.one.add(s.one.k, s.one.s);
            if (TWO) all.two.add(s.two.k, s.two.s);
            if (s.teacher.s != s.teacher.s) all.teacher.s = s.teacher.s;
        }
    }

    const bool has_teacher = k > 0 && !(all.teacher.s == 0.f);
    if (a.later) {                                  // (no sums so far, but NaN where an index is wrong)
        const float l0 = a.lse[2 * row], l1 = a.lse[2 * row + 1], one = all.one.s != all.one.s ? all.one.s : 1.f;
        all.one = Sum{__fmul_rn(a.main_is_teacher ? l1 : l0, kLog2e), one};
        if (TWO) all.two = Sum{__fmul_rn(l1, kLog2e), one};
    }
    const Sum& of_teacher = TWO ? all.two : all.one;      // the student's sum at the teacher's temperature
    const float c_teacher = TWO ? a.c2 : a.c1;

    // the teacher's probabilities, and the loss
    float sum = 0.f;
    if (has_teacher || has_label) {
        const float log_t = has_teacher ? log2f(all.teacher.s) : 0.f, log_s = log2f(of_teacher.s);
        for (int j = threadIdx.x; j <= k; j += THREADS) {
            float pj = 0.f;
            if (j < k && t_of[j] != -INFINITY) {
                const float u = __fmaf_rn(t_of[j], a.ct, -all.teacher.k);
                pj = __fdividef(exp2_of(u), all.teacher.s);
                const float kl = __fadd_rn(u - log_t, -(__fmaf_rn(z_of[j], c_teacher, -of_teacher.k) - log_s));
                if (pj != 0.f) sum = __fmaf_rn(__fmul_rn(pj, a.wt), kl, sum);
            } else if (j == k && has_label) {
                sum = __fmaf_rn(a.wl, log2f(all.one.s) - __fmaf_rn(z_of[k], a.c1, -all.one.k), sum);
            }
            p[j] = pj;
        }
        if (wrong) sum = __uint_as_float(0x7FC00000u);
    }
    if (a.loss && !a.later) {
#pragma unroll
        for (int d = 16; d >= 1; d >>= 1) sum = __fadd_rn(sum, __shfl_xor_sync(0xFFFFFFFFu, sum, d));
        if (lane == 0) part[warp] = sum;
    }
    if (a.lse && !a.later && rank == 0 && threadIdx.x == 0) {
        const float one = __fmul_rn(log2_of(all.one), 0.69314718f), two = TWO ? __fmul_rn(log2_of(all.two), 0.69314718f) : one;
        a.lse[2 * row] = one;
        a.lse[2 * row + 1] = two;
    }
    __syncthreads();
    if (a.loss && !a.later && rank == 0 && threadIdx.x == 0) {
        float s = part[0];
        for (int w = 1; w < kWarpsHere; ++w) s = __fadd_rn(s, part[w]);
        a.loss[row] = __fmul_rn(s, 0.69314718f);
    }
    if (!a.dz) return;

    // the gradient
    const float g = __fmul_rn(a.dloss ? a.dloss[row] : 1.f, a.scale);
    const float on_label = has_label ? __fmul_rn(g, a.wl) : 0.f, on_teacher = has_teacher ? __fmul_rn(g, __fdividef(a.wt, a.temperature)) : 0.f;
    const float A = on_label == 0.f && (TWO || on_teacher == 0.f) ? 0.f : __fdividef(TWO ? on_label : __fadd_rn(on_label, on_teacher), all.one.s);
    const float B = TWO && on_teacher != 0.f ? __fdividef(on_teacher, all.two.s) : 0.f;
    const bool none = on_label == 0.f && on_teacher == 0.f;
    const auto softmax = [&](float y) {
        float d = __fmul_rn(A, exp2_of(__fmaf_rn(y, a.c1, -all.one.k)));
        if (TWO) d = __fmaf_rn(B, exp2_of(__fmaf_rn(y, a.c2, -all.two.k)), d);
        return none ? 0.f : d;
    };
    T* const dz = static_cast<T*>(a.dz) + row * a.lddz;
    for (int tile = 0; tile < cols; tile += kTileCols) {
        if (cols > kTileCols) request(tile);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = tile + (v * THREADS + (int)threadIdx.x) * 8, left = max(0, min(8, cols - c));
            f8 d = x[v].values();
#pragma unroll
            for (int q = 0; q < 8; ++q) d.v[q] = softmax(d.v[q]);
            if constexpr (WIDE) store_some(dz + first + c, d, left == 8, left);
            else if (left > 0) store_unaligned(dz + first + c, d, left);
        }
    }
    // and what is taken off at the label and the teacher's entries; the same index twice is one element, written with the same value
    __syncthreads();
    if (none) return;
    for (int j = threadIdx.x; j <= k; j += THREADS) {
        const int i = index[j];
        if (i < first || i >= first + cols) continue;
        float off = i == label ? on_label : 0.f, sum_p = 0.f;
        for (int m = 0; m < k; ++m)
            if (index[m] == i) sum_p = __fadd_rn(sum_p, p[m]);
        store1(dz + i, __fadd_rn(softmax(z_of[j]), -__fmaf_rn(on_teacher, sum_p, off)));
    }
}

template <typename T, int THREADS, int NV, bool CLUSTER>
int loss_launch(const char* what, const LossArgs& a, bool two, bool wide, cudaStream_t s)
{
    const dim3 grid((unsigned)((int64_t)a.rows * a.pieces));
    const size_t smem = (size_t)(a.k + 1) * 16;
    const auto go = [&](auto kernel) { return launch_clusters(what, kernel, grid, THREADS, smem, a.pieces, s, a); };
    if (two) return wide ? go(loss_kernel<T, THREADS, NV, true, true, CLUSTER>) : go(loss_kernel<T, THREADS, NV, true, false, CLUSTER>);
    return wide ? go(loss_kernel<T, THREADS, NV, false, true, CLUSTER>) : go(loss_kernel<T, THREADS, NV, false, false, CLUSTER>);
}

template <typename T>
int loss_types(const char* what, LossArgs& a, bool two, bool wide, cudaStream_t s)
{
    const auto up8 = [](int64_t x) { return (int)((x + 7) / 8 * 8); };
    a.pieces = 1;
    a.piece = up8(a.vocab);
    constexpr int kMost = sizeof(T) == 4 ? 2 : 4;    // groups of eight that a thread holds
    if (a.vocab <= 1024) return loss_launch<T, 128, 1, false>(what, a, two, wide, s);
    if (a.vocab <= 4096) return loss_launch<T, 512, 1, false>(what, a, two, wide, s);
    if (a.vocab <= 8192) return loss_launch<T, 512, 2, false>(what, a, two, wide, s);
    if (kMost == 4 && a.vocab <= 16384) return loss_launch<T, 512, kMost, false>(what, a, two, wide, s);
    while (a.pieces < kMaxLossCluster && a.piece > kMost * 4096) {
        a.pieces *= 2;
        a.piece = up8((a.vocab + a.pieces - 1) / a.pieces);
    }
    return loss_launch<T, 512, kMost, true>(what, a, two, wide, s);
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
    if (p.vocab > 0x7FFFFFFF - 65536 || p.rows > 0x7FFFFFFF / kMaxLossCluster) return report(HPSGD_E_UNSUPPORTED, "%s: a size is too large", what);
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
    a.temperature = (float)p.temperature; a.scale = (float)p.grad_scale;
    a.teacher_bf16 = p.teacher_dtype == HPSGD_BF16;
    a.later = later;
    bool wide = aligned(p.logits, unit) && p.ldlogits * esz % unit == 0;
    if (p.dlogits) wide = wide && aligned(p.dlogits, unit) && p.lddlogits * esz % unit == 0;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    return p.dtype == HPSGD_F32 ? loss_types<float>(what, a, two, wide, s) : loss_types<__nv_bfloat16>(what, a, two, wide, s);
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
