// To the 8-bit block format along rows and along columns in one pass.
//
// A 128 x 128 tile is a whole block of each of its rows and of each of its columns, so one read of the tile gives both
// matrices and all 256 scales.  Bound by HBM: 6 bytes an element from fp32 with both outputs, 4 from bf16, 2 when a matrix
// in the format is transposed.  A thread holds an 8 x 8 patch: the 16 threads of a half warp cover a row, so the row maxima
// are shuffles and a row's codes leave as 128 contiguous bytes; a column's eight codes of a patch are eight consecutive bytes of the
// transpose, which is put together in 16 KB of shared memory and leaves in rows of 128 bytes as well.
#include "hpsgd_ops_common.cuh"

namespace hpsgd {
namespace ops {
namespace {

constexpr int kQThreads = 256;
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
__global__ void __launch_bounds__(kQThreads) quantize_kernel(const QuantArgs a)
{
    __shared__ uint32_t col_top[16][kTile];          // largest magnitudes (patterns) of each patch's columns
    __shared__ uint2 tile[kTile][16];                // the transpose: [column][eight rows], chunks permuted by the column's patch
    constexpr bool kCodes = sizeof(T) == 1;
    const int lane = threadIdx.x & 15, patch = threadIdx.x >> 4;
    const int64_t tiles_c = (a.cols + kTile - 1) / kTile;
    const int64_t r0 = (int64_t)(blockIdx.x / tiles_c) * kTile, c0 = (int64_t)(blockIdx.x % tiles_c) * kTile;
    const int64_t row0 = r0 + patch * 8, col0 = c0 + lane * 8;
    const int left = (int)max((int64_t)0, min((int64_t)8, a.cols - col0));

    f8 x[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const bool in = row0 + k < a.rows;
        const int here = in ? left : 0;
        if constexpr (kCodes) {
            uint2 u = make_uint2(0u, 0u);
            int byte = 0;
            if (here) {                               // codes behind the last column are zeros and can be read
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
            const int64_t blocks = tiles_c, b = c0 / kTile, pad = (a.cols + 15) / 16 * 16;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                f8 y = x[k];
                const int byte = block_scale(y);
                if (row0 + k < a.rows) {
                    if (col0 < pad) *reinterpret_cast<uint2*>(a.q + (row0 + k) * a.ldq + col0) = encode_nearest(y, byte);
                    if (lane == 0) store_scale(a.s, b, blocks, row0 + k, a.lds, byte);
                }
            }
        }
    }
    if (!a.qt) return;

    // column maxima: over the patch's rows here, over the 16 patches through shared memory
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        f8 y;
#pragma unroll
        for (int k = 0; k < 8; ++k) y.v[k] = x[k].v[j];
        col_top[patch][lane * 8 + j] = __float_as_uint(top8(y));
    }
    __syncthreads();
    if (threadIdx.x < kTile) {
        uint32_t t = 0;
#pragma unroll
        for (int p = 0; p < 16; ++p) t = max(t, col_top[p][threadIdx.x]);
        col_top[0][threadIdx.x] = t;
    }
    __syncthreads();
    bool odd = false;                                 // some column of the tile has values that are not finite
#pragma unroll
    for (int j = 0; j < 8; ++j) odd |= col_top[0][lane * 8 + j] >= 0x7F800000u;
    if (__syncthreads_or(odd)) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            uint32_t t = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if (finite(x[k].v[j])) t = max(t, __float_as_uint(fabsf(x[k].v[j])));
                else x[k].v[j] = __uint_as_float(0x7FC00000u);
            }
            col_top[patch][lane * 8 + j] = t;
        }
        __syncthreads();
        if (threadIdx.x < kTile) {
            uint32_t t = 0;
#pragma unroll
            for (int p = 0; p < 16; ++p) t = max(t, col_top[p][threadIdx.x]);
            col_top[0][threadIdx.x] = t;
        }
        __syncthreads();
    }
    const int64_t blocks_t = (a.rows + kTile - 1) / kTile, bt = r0 / kTile;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        f8 y;
#pragma unroll
        for (int k = 0; k < 8; ++k) y.v[k] = x[k].v[j];
        const int byte = scale_byte(__uint_as_float(col_top[0][lane * 8 + j]));
        tile[lane * 8 + j][patch ^ lane] = encode_nearest(y, byte);
        if (patch == 0 && col0 + j < a.cols) store_scale(a.st, bt, blocks_t, col0 + j, a.ldst, byte);
    }
    __syncthreads();
    const int64_t pad_t = (a.rows + 15) / 16 * 16;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const int c = k * 16 + patch;                 // a half warp takes one row of the transpose
        if (c0 + c < a.cols && r0 + lane * 8 < pad_t)
            *reinterpret_cast<uint2*>(a.qt + (c0 + c) * a.ldqt + r0 + lane * 8) = tile[c][lane ^ (c >> 3)];
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
