// To the 8-bit block format along rows and along columns in one pass.
//
// One read of a 128 x 128 tile gives both matrices and all 256 scales.  Bound by HBM: 6 bytes an element from fp32 with both outputs,
// 4 from bf16, 2 when a matrix in the format is transposed.
#include "hpsgd_quantize.cuh"

namespace hpsgd {
namespace ops {
namespace {

struct QuantArgs {
    QuantOut out;
    int64_t ldx, ldxs;
    const void* x;
    const uint8_t* xs;
    bool wide;             // x can be read with wide accesses
};

struct Fp8 {};

template <typename T>
__global__ void __launch_bounds__(kQThreads, 2) quantize_kernel(const QuantArgs a)
{
    constexpr int kRows = kPatchRows;
    __shared__ QuantRoom room;
    constexpr bool kCodes = sizeof(T) == 1;
    const int lane = threadIdx.x & 15, patch = threadIdx.x >> 4;
    const int tiles_c = (int)((a.out.cols + kTile - 1) / kTile);
    const int br = (int)(blockIdx.x / (unsigned)tiles_c), bc = (int)(blockIdx.x % (unsigned)tiles_c);      // the tile, and the blocks' numbers
    const int row0 = br * kTile + patch * kRows, col0 = bc * kTile + lane * 8;
    const int left = max(0, min(8, (int)a.out.cols - col0)), rows = (int)a.out.rows - row0;      // of this patch
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
    quantize_tile<!kCodes>(a.out, room, x, br, bc);
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
    QuantArgs a{{p.rows, p.cols, p.ldq, p.lds, p.ldqt, p.ldst, static_cast<uint8_t*>(p.q), p.scale, static_cast<uint8_t*>(p.qt), p.scale_t},
                p.ldx, p.ldxs, p.x, p.x_scale, false};
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int64_t unit = p.dtype == HPSGD_F32 ? 32 : 16, esz = p.dtype == HPSGD_F32 ? 4 : 2;
    a.wide = aligned(p.x, unit) && p.ldx * esz % unit == 0;
    if (p.dtype == HPSGD_F32) return launch_early(what, quantize_kernel<float>, dim3((unsigned)tiles), kQThreads, 0, s, a);
    if (p.dtype == HPSGD_BF16) return launch_early(what, quantize_kernel<__nv_bfloat16>, dim3((unsigned)tiles), kQThreads, 0, s, a);
    return launch_early(what, quantize_kernel<Fp8>, dim3((unsigned)tiles), kQThreads, 0, s, a);
}
