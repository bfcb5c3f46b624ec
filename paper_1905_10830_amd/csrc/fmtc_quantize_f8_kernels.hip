// Values to 8-bit floating point with a scale per block of 128 (fmtc_f8_quantize): largest finite magnitude of the block,
// scale, codes.  Memory bound: every value is read once, whichever of the two outputs are wanted.
#include "fmtc_block.h"

namespace fmtc {

namespace {

// 1 x 128 blocks along the rows: 16 lanes hold a block, 8 values each.  8192 x 4096 bf16 19.6 us (5.1 TB/s).
template <class T, int FORMAT, int SCALE, bool RAGGED>
__global__ __launch_bounds__(256) void k_f8_quantize_rows(const T* __restrict__ x, int64_t rows, int64_t cols, int64_t ld_x,
                                                          uint32_t blocks, fmtc_f8 out) {
    const int64_t item = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
    const int64_t row = item / blocks, b = item - row * blocks;
    if (row >= rows) return;  // (whole rows of 16 lanes)
    const int64_t c = b * kF8Block + (threadIdx.x & 15) * 8;
    float v[8];
    load8<RAGGED>(x + row * ld_x, c, cols, v);
    if (c >= cols)
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = 0.f;
    uint32_t held;
    const float inv = block_scale<FORMAT, SCALE>(row16_max(finite_amax(v)), &held);
    const uint2 q = make_uint2(encode4<FORMAT>(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv),
                               encode4<FORMAT>(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv));
    *reinterpret_cast<uint2*>(static_cast<uint8_t*>(out.d_codes) + row * out.ld + c) = q;
    if ((threadIdx.x & 15) == 0) store_scale<SCALE>(out.d_scales, b * out.ld_scales + row, held);
}

// A tile of 128 x 128 values per workgroup, kept in registers (4 rows x 8 columns a lane) between the maxima and the codes:
// the second output costs no second read.  The transposed codes go through LDS, 4 bytes (4 rows of a column) at a time, at
// places exchanged so that the columns' writes and the rows' reads of 16 lanes spread over the banks.  8192 x 4096 bf16, both
// outputs: 24.1 us (5.6 TB/s), 128 x 128 blocks 21.5 us; 8192 x 4095, whose rows begin at odd places, 32.0 us.  With 8 rows a
// lane and half the lanes a tile's own time shows: 1024 x 2048 6.1 us, as here 5.0 us; 8192 x 4096 25.7 us.
constexpr int kTileThreads = 512;

template <class T, int FORMAT, int SCALE, bool WEIGHTS, bool RAGGED>
__global__ __launch_bounds__(kTileThreads) void k_f8_quantize_tiles(const T* __restrict__ x, int64_t rows, int64_t cols, int64_t ld_x,
                                                           uint32_t col_blocks, fmtc_f8 by_rows, fmtc_f8 by_cols,
                                                           float* __restrict__ col_sums) {
    constexpr int R = 4, kLaneRows = kTileThreads / 16;
    static_assert(R * kLaneRows == kF8Block);
    __shared__ float part[kLaneRows][kF8Block];
    __shared__ float col_inv[kF8Block];
    __shared__ __align__(16) uint32_t tile[kF8Block][kF8Block / 4];
    const int t = threadIdx.x, lane_c = t & 15, lane_r = t >> 4;
    const int64_t rb = blockIdx.x / col_blocks, cb = blockIdx.x - rb * col_blocks;
    const int64_t row0 = rb * kF8Block + lane_r * R, c0 = cb * kF8Block + lane_c * 8;
    Raw<T> raw[R];
#pragma unroll
    for (int i = 0; i < R; i++) raw[i].template load<RAGGED>(x + (row0 + i < rows ? row0 + i : rows - 1) * ld_x, c0, cols);
    if constexpr (RAGGED)
#pragma unroll
        for (int i = 0; i < R; i++) raw[i].settle(c0, cols);
    float v[R][8];
#pragma unroll
    for (int i = 0; i < R; i++) {
        raw[i].zero_unless(row0 + i < rows && c0 < cols);
#pragma unroll
        for (int j = 0; j < 8; j++) v[i][j] = raw[i][j];
    }

    float inv_row[R];
    if constexpr (WEIGHTS) {
        float amax = 0.f;
#pragma unroll
        for (int i = 0; i < R; i++) amax = fmaxf(amax, finite_amax(v[i]));
        amax = row16_max(amax);
        if (lane_c == 0) part[0][lane_r] = amax;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kLaneRows; r += 16) amax = fmaxf(amax, part[0][r + lane_c]);
        amax = row16_max(amax);
        uint32_t held;
        const float inv = block_scale<FORMAT, SCALE>(amax, &held);
#pragma unroll
        for (int i = 0; i < R; i++) inv_row[i] = inv;
        if (t < kF8Block) col_inv[t] = inv;
        if (t == 0) {
            if (by_rows.d_codes) store_scale<SCALE>(by_rows.d_scales, cb * by_rows.ld_scales + rb, held);
            if (by_cols.d_codes) store_scale<SCALE>(by_cols.d_scales, rb * by_cols.ld_scales + cb, held);
        }
    } else {
        if (by_rows.d_codes) {
#pragma unroll
            for (int i = 0; i < R; i++) {
                uint32_t held;
                inv_row[i] = block_scale<FORMAT, SCALE>(row16_max(finite_amax(v[i])), &held);
                if (lane_c == 0 && row0 + i < rows) store_scale<SCALE>(by_rows.d_scales, cb * by_rows.ld_scales + row0 + i, held);
            }
        }
        if (by_cols.d_codes) {
#pragma unroll
            for (int j = 0; j < 8; j++) {
                float amax = 0.f;
#pragma unroll
                for (int i = 0; i < R; i++) amax = fmaxf(amax, finite_abs(v[i][j]));
                part[lane_r][lane_c * 8 + j] = amax;
            }
            __syncthreads();
            if (t < kF8Block) {
                float amax = 0.f;
#pragma unroll
                for (int r = 0; r < kLaneRows; r++) amax = fmaxf(amax, part[r][t]);
                uint32_t held;
                col_inv[t] = block_scale<FORMAT, SCALE>(amax, &held);
                if (cb * kF8Block + t < cols) store_scale<SCALE>(by_cols.d_scales, rb * by_cols.ld_scales + cb * kF8Block + t, held);
            }
        }
    }
    if (by_rows.d_codes) {
#pragma unroll
        for (int i = 0; i < R; i++)
            if (row0 + i < rows) {
                const float s = inv_row[i];
                *reinterpret_cast<uint2*>(static_cast<uint8_t*>(by_rows.d_codes) + (row0 + i) * by_rows.ld + c0) =
                    make_uint2(encode4<FORMAT>(v[i][0] * s, v[i][1] * s, v[i][2] * s, v[i][3] * s),
                               encode4<FORMAT>(v[i][4] * s, v[i][5] * s, v[i][6] * s, v[i][7] * s));
            }
    }
    if (!by_cols.d_codes) return;
    __syncthreads();  // col_inv is there, part is free
#pragma unroll
    for (int j = 0; j < 8; j++) {
        const float s = col_inv[lane_c * 8 + j];
        tile[lane_c * 8 + j][2 * (lane_r / 2 ^ lane_c) + lane_r % 2] = encode4<FORMAT>(v[0][j] * s, v[1][j] * s, v[2][j] * s, v[3][j] * s);
        if (col_sums) {
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < R; i++) sum += v[i][j];
            part[lane_r][lane_c * 8 + j] = sum;
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kF8Block * 8 / kTileThreads; i++) {
        const int col = (t >> 3) + kTileThreads / 8 * i, piece = t & 7, turn = (col >> 3) & 15;
        if (cb * kF8Block + col < cols) {
            const uint2 a = *reinterpret_cast<const uint2*>(&tile[col][2 * ((2 * piece) ^ turn)]),
                        b = *reinterpret_cast<const uint2*>(&tile[col][2 * ((2 * piece + 1) ^ turn)]);
            *reinterpret_cast<uint4*>(static_cast<uint8_t*>(by_cols.d_codes) + (cb * kF8Block + col) * by_cols.ld +
                                      rb * kF8Block + piece * 16) = make_uint4(a.x, a.y, b.x, b.y);
        }
    }
    if (col_sums && t < kF8Block && cb * kF8Block + t < cols) {
        float sum = 0.f, other = 0.f;
#pragma unroll
        for (int r = 0; r < kLaneRows / 2; r++) {
            sum += part[r][t];
            other += part[r + kLaneRows / 2][t];
        }
        col_sums[rb * cols + cb * kF8Block + t] = sum + other;
    }
}

// 32 columns a workgroup, 32 slices of the rows, added up in order
__global__ __launch_bounds__(1024) void k_column_sums(const float* __restrict__ part, int64_t n, int64_t cols,
                                                      float* __restrict__ out, int accumulate) {
    __shared__ float slice[32][33];
    const int col = threadIdx.x & 31, k = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + col;
    float sum = 0.f;
    if (c < cols)
#pragma unroll 4
        for (int64_t i = k; i < n; i += 32) sum += part[i * cols + c];
    slice[k][col] = sum;
    __syncthreads();
    if (k == 0 && c < cols) {
#pragma unroll
        for (int i = 1; i < 32; i++) sum += slice[i][col];
        out[c] = accumulate ? out[c] + sum : sum;
    }
}

__global__ __launch_bounds__(256) void k_fill_rows(float* __restrict__ out, int64_t cols, int64_t ld, int64_t n) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i < n) out[i / cols * ld + i % cols] = 0.f;
}

}  // namespace

hipError_t launch_f8_quantize(const void* d_x, int type, int64_t rows, int64_t cols, int64_t ld_x, const fmtc_f8* by_rows,
                              const fmtc_f8* by_cols, float* d_col_sums, hipStream_t s) {
    const fmtc_f8 none{}, a = by_rows ? *by_rows : none, b = by_cols ? *by_cols : none;
    const fmtc_f8& any = by_rows ? a : b;
    const int64_t col_blocks = (cols + kF8Block - 1) / kF8Block, row_blocks = (rows + kF8Block - 1) / kF8Block;
    return with_type(type, [&](auto ty) {
        using T = typename decltype(ty)::type;
        return with_bit(any.format, [&](auto fm) {
            return with_bit(any.scale, [&](auto sc) {
                return with_bit(cols % 8 != 0, [&](auto rg) {
                    constexpr int F = decltype(fm)::value, S = decltype(sc)::value;
                    constexpr bool R = decltype(rg)::value;
                    const T* x = static_cast<const T*>(d_x);
                    if (!by_cols && any.block_rows == 1)
                        return launch(K_F8_QUANTIZE, k_f8_quantize_rows<T, F, S, R>, dim3((unsigned)((rows * col_blocks + 15) / 16)),
                                      dim3(256), 0, s, x, rows, cols, ld_x, (uint32_t)col_blocks, a);
                    const dim3 grid((unsigned)(row_blocks * col_blocks));
                    auto kernel = any.block_rows == 1 ? k_f8_quantize_tiles<T, F, S, false, R> : k_f8_quantize_tiles<T, F, S, true, R>;
                    return launch(K_F8_QUANTIZE, kernel, grid, dim3(kTileThreads), 0, s, x, rows, cols, ld_x, (uint32_t)col_blocks, a, b, d_col_sums);
                });
            });
        });
    });
}

hipError_t launch_column_sums(const float* d_part, int64_t n, int64_t cols, float* d_out, int accumulate, hipStream_t s) {
    return launch(K_F8_QUANTIZE, k_column_sums, dim3((unsigned)((cols + 31) / 32)), dim3(1024), 0, s, d_part, n, cols, d_out,
                  accumulate);
}

hipError_t launch_fill_rows(float* d_out, int64_t rows, int64_t cols, int64_t ld, hipStream_t s) {
    return launch(K_F8_QUANTIZE, k_fill_rows, dim3((unsigned)((rows * cols + 255) / 256)), dim3(256), 0, s, d_out, cols, ld, rows * cols);
}

}  // namespace fmtc
