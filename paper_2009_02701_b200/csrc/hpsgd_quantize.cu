// To the 8-bit block format along rows and along columns in one pass.
//
// A 128 x 128 tile is a whole block of each of its rows and of each of its columns, so one read of the tile gives both
// matrices and all 256 scales.  Bound by HBM: 6 bytes an element from fp32 with both outputs, 4 from bf16, 2 when a matrix
// in the format is transposed.  A thread holds a patch of 4 rows x 8 columns: the 16 threads of a half warp cover a row, so the row
// maxima are shuffles and a row's codes leave as 128 contiguous bytes; a column's four codes of a patch are one word of the
// transpose, which is put together in 16 KB of shared memory and leaves in rows of 128 bytes as well.  (Patches of 8 x 8 with half the
// threads left too few warps to wait with: 49 us where this takes 39 us for 30000 x 1024 in fp32.)
#include "hpsgd_ops_common.cuh"

namespace hpsgd {
namespace ops {
namespace {

constexpr int kQThreads = 512;
constexpr int kTile = 128;

struct QuantArgs {
    int64_t rows, cols, ldx, ldxs, ldq, lds, ldqt, ldst;
    const void* x;
    const uint8_t* xs;
    uint8_t* q;
    uint8_t* s;
    uint8_t* qt;
    uint8_t* st;
    bool wide;             // x can be read with wide accesses
};

struct Fp8 {};

__device__ __forceinline__ f8 decode_nearest(uint2 u, float scale)
{
    f8 x;
#pragma unroll
    for (int q = 0; q < 8; ++q) x.v[q] = __fmul_rn(e4m3_value((q < 4 ? u.x : u.y) >> 8 * (q & 3) & 0xFFu), scale);
    return x;
}

// The padding behind a row's last block in its last word of scales.
__device__ __forceinline__ void store_scale(uint8_t* s, int64_t b, int64_t blocks, int64_t r, int64_t ld, int byte)
{
    s[scale_index(b, r, ld)] = (uint8_t)byte;
    if (b == blocks - 1)
        for (int64_t k = b + 1; k & 3; ++k) s[scale_index(k, r, ld)] = 0;
}

template <typename T>
__global__ void __launch_bounds__(kQThreads, 2) quantize_kernel(const QuantArgs a)
{
    constexpr int kRows = 4, kWarps = kQThreads / 32;
    __shared__ uint32_t col_top[kWarps][kTile];      // largest magnitudes (patterns) of each warp's eight rows
    __shared__ alignas(16) uint32_t tile[kTile][kTile / 4];      // the transpose: [column][four rows], words permuted by the column's patch
    __shared__ alignas(16) uint8_t col_byte[kTile];
    __shared__ int odd;                              // some column of the tile has values that are not finite
    constexpr bool kCodes = sizeof(T) == 1;
    const int lane = threadIdx.x & 15, patch = threadIdx.x >> 4, warp = threadIdx.x >> 5;
    const int64_t tiles_c = (a.cols + kTile - 1) / kTile;
    const int64_t r0 = (int64_t)(blockIdx.x / tiles_c) * kTile, c0 = (int64_t)(blockIdx.x % tiles_c) * kTile;
    const int64_t row0 = r0 + patch * kRows, col0 = c0 + lane * 8;
    const int left = (int)max((int64_t)0, min((int64_t)8, a.cols - col0));
    if (threadIdx.x == 0) odd = 0;

    f8 x[kRows];
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
        const int here = row0 + k < a.rows ? left : 0;
        if constexpr (kCodes) {
            uint2 u = make_uint2(0u, 0u);
            int byte = 0;
            if (here) {                               // the codes behind the last column, up to 16, can be read: they are masked below
                u = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(a.x) + (row0 + k) * a.ldx + col0);
                byte = a.xs[scale_index(c0 / kTile, row0 + k, a.ldxs)];
            }
            x[k] = decode_nearest(u, scale_value(byte));
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j >= here) x[k].v[j] = 0.f;
        } else {
            x[k] = load_some(static_cast<const T*>(a.x) + (row0 + k) * a.ldx + col0, a.wide && here == 8, here);
        }
    }

    if constexpr (!kCodes) {
        if (a.q) {
            const int64_t b = c0 / kTile, pad = (a.cols + 15) / 16 * 16;
#pragma unroll
            for (int k = 0; k < kRows; ++k) {
                f8 y = x[k];
                const int byte = block_scale(y);
                if (row0 + k < a.rows) {
                    if (col0 < pad) *reinterpret_cast<uint2*>(a.q + (row0 + k) * a.ldq + col0) = encode_nearest(y, byte);
                    if (lane == 0) store_scale(a.s, b, tiles_c, row0 + k, a.lds, byte);
                }
            }
        }
    }
    if (!a.qt) return;

    // column maxima: over the rows of a warp here, over the warps through shared memory
    const auto maxima = [&](bool only_finite) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            uint32_t t = 0;
#pragma unroll
            for (int k = 0; k < kRows; ++k) {
                const uint32_t u = __float_as_uint(fabsf(x[k].v[j]));
                if (!only_finite || u < 0x7F800000u) t = max(t, u);
            }
            t = max(t, __shfl_xor_sync(0xFFFFFFFFu, t, 16));
            if (threadIdx.x & 16 ? j >= 4 : j < 4) col_top[warp][lane * 8 + j] = t;
        }
        __syncthreads();
        if (threadIdx.x < kTile) {
            uint32_t t = 0;
#pragma unroll
            for (int p = 0; p < kWarps; ++p) t = max(t, col_top[p][threadIdx.x]);
            if (t >= 0x7F800000u) odd = 1;
            const int byte = scale_byte(__uint_as_float(t));
            col_byte[threadIdx.x] = (uint8_t)byte;
            if (t < 0x7F800000u && c0 + threadIdx.x < a.cols)
                store_scale(a.st, r0 / kTile, (a.rows + kTile - 1) / kTile, c0 + threadIdx.x, a.ldst, byte);
        }
        __syncthreads();
    };
    maxima(false);
    if (odd) {                                        // rare: the scales are those of the finite values, and the others become NaN
        maxima(true);
#pragma unroll
        for (int k = 0; k < kRows; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (!finite(x[k].v[j])) x[k].v[j] = __uint_as_float(0x7FC00000u);
    }
    const uint2 bytes = *reinterpret_cast<const uint2*>(col_byte + lane * 8);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float inv = scale_inverse((j < 4 ? bytes.x : bytes.y) >> 8 * (j & 3) & 0xFFu);
        unsigned short lo, hi;
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(__fmul_rn(x[1].v[j], inv)), "f"(__fmul_rn(x[0].v[j], inv)));
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(__fmul_rn(x[3].v[j], inv)), "f"(__fmul_rn(x[2].v[j], inv)));
        tile[lane * 8 + j][patch ^ 2 * lane] = lo | (uint32_t)hi << 16;
    }
    __syncthreads();
    const int64_t pad_t = (a.rows + 15) / 16 * 16;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int c = k * 32 + patch;                 // a half warp takes one row of the transpose
        if (c0 + c < a.cols && r0 + lane * 8 < pad_t)
            *reinterpret_cast<uint2*>(a.qt + (c0 + c) * a.ldqt + r0 + lane * 8) = *reinterpret_cast<const uint2*>(&tile[c][2 * lane ^ 2 * (c >> 3)]);
    }
}

int check_matrix(const char* what, const char* name, const void* q, const void* s, int64_t* ld, int64_t* lds, int64_t rows, int64_t cols)
{
    if (!q != !s) return report(HPSGD_E_BADARG, "%s: %s: codes and scales go together", what, name);
    if (!q) return HPSGD_OK;
    if (*ld == 0) *ld = (cols + 15) / 16 * 16;
    if (*lds == 0) *lds = rows;
    if (*ld < cols || *ld % 16 || !aligned(q, 16)) return report(HPSGD_E_BADARG, "%s: %s: rows of codes must start on 16-byte boundaries and not overlap", what, name);
    if (*lds < rows || !aligned(s, 4)) return report(HPSGD_E_BADARG, "%s: %s: scales are not 4-byte aligned or their stride is below the number of rows", what, name);
    return HPSGD_OK;
}

}  // namespace

int check_fp8(const char* what, const char* name, const void* q, const void* s, int64_t* ld, int64_t* lds, int64_t rows, int64_t cols)
{
    return check_matrix(what, name, q, s, ld, lds, rows, cols);
}

}  // namespace ops
}  // namespace hpsgd

using namespace hpsgd;
using namespace hpsgd::ops;

extern "C" int hpsgd_quantize_fp8(const hpsgd_quantize_fp8_args* args, void* stream)
{
    const char* what = "hpsgd_quantize_fp8";
    if (!args) return report(HPSGD_E_BADARG, "%s: args is NULL", what);
    hpsgd_quantize_fp8_args p = *args;
    if (p.rows < 0 || p.cols < 0) return report(HPSGD_E_BADARG, "%s: a size is negative", what);
    if (p.rows > 0x7FFFFFFF || p.cols > 0x7FFFFFFF) return report(HPSGD_E_UNSUPPORTED, "%s: a size is above 2^31 - 1", what);
    if (p.dtype != HPSGD_F32 && p.dtype != HPSGD_BF16 && p.dtype != HPSGD_FP8) return report(HPSGD_E_BADARG, "%s: unknown dtype %d", what, p.dtype);
    if (p.rows == 0 || p.cols == 0) return HPSGD_OK;
    if (!p.x) return report(HPSGD_E_BADARG, "%s: x is NULL", what);
    if (!p.q && !p.qt) return report(HPSGD_E_BADARG, "%s: no output is asked for", what);
    if (p.dtype == HPSGD_FP8) {
        if (p.q) return report(HPSGD_E_BADARG, "%s: a matrix in the block format can only be transposed", what);
        if (!p.x_scale) return report(HPSGD_E_BADARG, "%s: x_scale is NULL", what);
        OPS_TRY(check_fp8(what, "x", p.x, p.x_scale, &p.ldx, &p.ldxs, p.rows, p.cols));
    } else {
        if (p.ldx == 0) p.ldx = p.cols;
        if (p.ldx < p.cols) return report(HPSGD_E_BADARG, "%s: ldx is below cols", what);
        if (!aligned(p.x, p.dtype == HPSGD_F32 ? 4 : 2)) return report(HPSGD_E_BADARG, "%s: x is not aligned to its elements", what);
    }
    OPS_TRY(check_fp8(what, "q", p.q, p.scale, &p.ldq, &p.lds, p.rows, p.cols));
    OPS_TRY(check_fp8(what, "qt", p.qt, p.scale_t, &p.ldqt, &p.ldst, p.cols, p.rows));
    int sms = 0;
    OPS_TRY(device_sms(&sms));
    const int64_t tiles = ((p.rows + kTile - 1) / kTile) * ((p.cols + kTile - 1) / kTile);
    if (tiles > 0x7FFFFFFF) return report(HPSGD_E_UNSUPPORTED, "%s: more than 2^31 - 1 tiles of 128 x 128", what);
    QuantArgs a{p.rows, p.cols, p.ldx, p.ldxs, p.ldq, p.lds, p.ldqt, p.ldst, p.x, p.x_scale, static_cast<uint8_t*>(p.q), p.scale,
                static_cast<uint8_t*>(p.qt), p.scale_t, false};
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int64_t unit = p.dtype == HPSGD_F32 ? 32 : 16, esz = p.dtype == HPSGD_F32 ? 4 : 2;
    a.wide = aligned(p.x, unit) && p.ldx * esz % unit == 0;
    if (p.dtype == HPSGD_F32) quantize_kernel<float><<<(unsigned)tiles, kQThreads, 0, s>>>(a);
    else if (p.dtype == HPSGD_BF16) quantize_kernel<__nv_bfloat16><<<(unsigned)tiles, kQThreads, 0, s>>>(a);
    else quantize_kernel<Fp8><<<(unsigned)tiles, kQThreads, 0, s>>>(a);
    return launched(what);
}
