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

template <typename T>
__global__ void __launch_bounds__(kQThreads, 2) quantize_kernel(const QuantArgs a)
{
    constexpr int kRows = 4, kWarps = kQThreads / 32;
    __shared__ float col_top[kWarps][kTile];         // largest magnitudes of each warp's eight rows
    __shared__ alignas(16) uint32_t tile[kTile][kTile / 4];      // the transpose: [column][four rows], words permuted by the column's patch
    __shared__ alignas(16) float col_inverse[kTile];
    __shared__ int odd;                              // some column of the tile has values that are not finite
    constexpr bool kCodes = sizeof(T) == 1;
    const int lane = threadIdx.x & 15, patch = threadIdx.x >> 4, warp = threadIdx.x >> 5;
    const int tiles_c = (int)((a.cols + kTile - 1) / kTile), tiles_r = (int)((a.rows + kTile - 1) / kTile);
    const int br = (int)(blockIdx.x / (unsigned)tiles_c), bc = (int)(blockIdx.x % (unsigned)tiles_c);      // the tile, and the blocks' numbers
    const int row0 = br * kTile + patch * kRows, col0 = bc * kTile + lane * 8;
    const int left = max(0, min(8, (int)a.cols - col0)), rows = (int)a.rows - row0;      // of this patch
    if (threadIdx.x == 0) odd = 0;
    after_previous();

    f8 x[kRows];
    if constexpr (kCodes) {
        const uint8_t* p = static_cast<const uint8_t*>(a.x) + row0 * a.ldx + col0;
        const uint8_t* s = a.xs + scale_index(bc, row0, a.ldxs);
        uint2 u[kRows];
        int byte[kRows];
#pragma unroll
        for (int k = 0; k < kRows; ++k) {            // the codes behind the last column, up to 16, can be read: they are masked below
            const bool in = k < rows && left > 0;
            u[k] = in ? *reinterpret_cast<const uint2*>(p + k * a.ldx) : make_uint2(0u, 0u);
            byte[k] = in ? s[4 * k] : 0;
        }
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
            p4 y = decode8(u[k]);
            const pair f = both(scale_value(byte[k]));
#pragma unroll
            for (int q = 0; q < 4; ++q) y.v[q] = mul2(y.v[q], f);
            x[k] = to_values(y);
            if (left < 8) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j >= left) x[k].v[j] = 0.f;
            }
        }
    } else {
        const T* p = static_cast<const T*>(a.x) + row0 * a.ldx + col0;
        Raw8<T> raw[kRows];
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
            const int here = k < rows ? left : 0;
            raw[k].load(p + k * a.ldx, a.wide && here == 8, here);
        }
#pragma unroll
        for (int k = 0; k < kRows; ++k) x[k] = raw[k].values();
    }

    if constexpr (!kCodes) {
        if (a.q) {
            int byte[kRows];
            uint8_t* const q = a.q + row0 * a.ldq + col0;
            const bool inside = col0 < (a.cols + 15) / 16 * 16;
#pragma unroll
            for (int k = 0; k < kRows; ++k) {
                f8 y = x[k];
                byte[k] = block_scale(y);
                const uint2 codes = encode_nearest(y, byte[k]);
                if (inside && k < rows) *reinterpret_cast<uint2*>(q + k * a.ldq) = codes;
            }
            if (lane < min(kRows, rows)) {            // one lane a row
                uint8_t* const s = a.s + scale_index(bc, row0 + lane, a.lds);
                *s = (uint8_t)(lane & 2 ? lane & 1 ? byte[3] : byte[2] : lane & 1 ? byte[1] : byte[0]);
                if (bc == tiles_c - 1)                // zeros behind the row's last block
                    for (int k = 1; (bc + k) & 3; ++k) s[k] = 0;
            }
        }
    }
    if (!a.qt) return;

    // column maxima: over the rows of a warp here, over the warps through shared memory
    const auto maxima = [&]() {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float t;
            asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(t) : "f"(x[0].v[j]), "f"(x[1].v[j]), "f"(x[2].v[j]));
            asm("max.NaN.abs.f32 %0, %1, %2, %2;" : "=f"(t) : "f"(t), "f"(x[3].v[j]));
            const float other = __shfl_xor_sync(0xFFFFFFFFu, t, 16);
            asm("max.NaN.f32 %0, %0, %1;" : "+f"(t) : "f"(other));
            if (threadIdx.x & 16 ? j >= 4 : j < 4) col_top[warp][lane * 8 + j] = t;
        }
        __syncthreads();
        if (threadIdx.x < kTile) {
            float t = 0.f;
#pragma unroll
            for (int p = 0; p < kWarps; ++p) asm("max.NaN.f32 %0, %0, %1;" : "+f"(t) : "f"(col_top[p][threadIdx.x]));
            if (!finite(t)) odd = 1;
            const int byte = scale_byte(t), c = bc * kTile + threadIdx.x;
            col_inverse[threadIdx.x] = scale_inverse(byte);
            if (finite(t) && c < a.cols) {
                uint8_t* const s = a.st + scale_index(br, c, a.ldst);
                *s = (uint8_t)byte;
                if (br == tiles_r - 1)
                    for (int k = 1; (br + k) & 3; ++k) s[k] = 0;
            }
        }
        __syncthreads();
    };
    maxima();
    uint32_t bad = 0;                                 // which of the patch's values become NaN
    if (odd) {                                        // rare: the scales are those of the finite values
#pragma unroll
        for (int k = 0; k < kRows; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (!finite(x[k].v[j])) {
                    bad |= 1u << (k * 8 + j);
                    x[k].v[j] = 0.f;
                }
        maxima();
#pragma unroll
        for (int k = 0; k < kRows; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (bad >> (k * 8 + j) & 1u) x[k].v[j] = __uint_as_float(0x7FC00000u);
    }
    const float4 i0 = *reinterpret_cast<const float4*>(col_inverse + lane * 8), i1 = *reinterpret_cast<const float4*>(col_inverse + lane * 8 + 4);
    const pair inverse[4] = {make_pair(i0.x, i0.y), make_pair(i0.z, i0.w), make_pair(i1.x, i1.y), make_pair(i1.z, i1.w)};
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
        p4 y = to_pairs(x[k]);
#pragma unroll
        for (int q = 0; q < 4; ++q) y.v[q] = mul2(y.v[q], inverse[q]);
        x[k] = to_values(y);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) tile[lane * 8 + j][patch ^ 2 * lane] = codes4(x[0].v[j], x[1].v[j], x[2].v[j], x[3].v[j]);
    __syncthreads();
    // a half warp takes one row of the transpose
    if (br * kTile + lane * 8 < (a.rows + 15) / 16 * 16) {
        uint8_t* const qt = a.qt + (int64_t)(bc * kTile + patch) * a.ldqt + br * kTile + lane * 8;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int c = k * 32 + patch;
            if (bc * kTile + c < a.cols) *reinterpret_cast<uint2*>(qt + k * 32 * a.ldqt) = *reinterpret_cast<const uint2*>(&tile[c][2 * lane ^ 2 * (c >> 3)]);
        }
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
    if (p.dtype == HPSGD_F32) return launch_early(what, quantize_kernel<float>, dim3((unsigned)tiles), kQThreads, 0, s, a);
    if (p.dtype == HPSGD_BF16) return launch_early(what, quantize_kernel<__nv_bfloat16>, dim3((unsigned)tiles), kQThreads, 0, s, a);
    return launch_early(what, quantize_kernel<Fp8>, dim3((unsigned)tiles), kQThreads, 0, s, a);
}
