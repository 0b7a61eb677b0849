// A tile of 128 x 128 values to the 8-bit block format along its rows and along its columns.
//
// A tile is a whole block of each of its rows and of each of its columns.  A thread holds a patch of 4 rows x 8 columns: the 16 threads of a half
// warp cover a row, so the row maxima are shuffles and a row's codes leave as 128 contiguous bytes; a column's four codes of a patch are one word
// of the transpose, which is put together in 16 KB of shared memory and leaves in rows of 128 bytes as well.  (Patches of 8 x 8 with half the
// threads left too few warps to wait with: 49 us where this takes 39 us for 30000 x 1024 in fp32.)
#pragma once

#include "hpsgd_ops_common.cuh"

namespace hpsgd {
namespace ops {
namespace {

constexpr int kQThreads = 512;
constexpr int kTile = 128;
constexpr int kPatchRows = 4;

// Where the codes and scales of a matrix [rows x cols] go: along rows (q) and along columns (qt), either NULL.
struct QuantOut {
    int64_t rows, cols, ldq, lds, ldqt, ldst;
    uint8_t* q;
    uint8_t* s;
    uint8_t* qt;
    uint8_t* st;
};

struct QuantRoom {
    float col_top[kQThreads / 32][kTile];            // largest magnitudes of each warp's eight rows
    alignas(16) uint32_t tile[kTile][kTile / 4];     // the transpose: [column][four rows], words permuted by the column's patch
    alignas(16) float col_inverse[kTile];
    int odd;                                         // some column of the tile has values that are not finite
};

// The tile in row br and column bc of tiles; x: this thread's patch, zeros where the matrix has ended.  All threads of the block come here; ROWS:
// codes along the rows may be asked for.
template <bool ROWS>
__device__ __forceinline__ void quantize_tile(const QuantOut& a, QuantRoom& room, f8 (&x)[kPatchRows], int br, int bc)
{
    constexpr int kRows = kPatchRows, kWarps = kQThreads / 32;
    auto& col_top = room.col_top;
    auto& tile = room.tile;
    auto& col_inverse = room.col_inverse;
    auto& odd = room.odd;
    const int lane = threadIdx.x & 15, patch = threadIdx.x >> 4, warp = threadIdx.x >> 5;
    const int tiles_c = (int)((a.cols + kTile - 1) / kTile), tiles_r = (int)((a.rows + kTile - 1) / kTile);
    const int row0 = br * kTile + patch * kRows, col0 = bc * kTile + lane * 8, rows = (int)a.rows - row0;
    if (threadIdx.x == 0) odd = 0;
    if constexpr (ROWS) {
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

}  // namespace
}  // namespace ops
}  // namespace hpsgd
