// Products of 8-bit floating point matrices with a scale per block of 128 (fmtc_f8_matmul):
//   out[m][n] = sum_b sa[b][m] sb[b][n / block_rows] sum_{k in b} a[m][k] b[n][k] (+ bias[n])
// One v_mfma_f32_16x16x128_f8f6f4 is exactly one block of the depth for 16 x 16 results.  b's rows are the instruction's
// first operand and a's its second: a lane then holds four consecutive columns n of one row m of the result, so that sa is
// one number per lane and the results leave in vectors.  Power-of-two scales are operands of the instruction itself; f32
// scales multiply the block's product, which one fma adds to the running f32 sum.
#include "fmtc_block.h"

namespace fmtc {

namespace {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));

// The same order of the depth in both operands is all the instruction asks for: lanes 16 g .. 16 g + 15 hold the bytes
// 16 g .. and 64 + 16 g .. of the block, so that each of the two loads of a wavefront covers 64 bytes of a row at a time.
__device__ __forceinline__ v8i load_operand(const uint8_t* row_at_block, int g) {
    const v4i lo = *reinterpret_cast<const v4i*>(row_at_block + 16 * g);
    const v4i hi = *reinterpret_cast<const v4i*>(row_at_block + 64 + 16 * g);
    return v8i{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
}

template <int FORMAT>
__device__ __forceinline__ v4f mfma_block(v8i b, v8i a, v4f c) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, c, 0, FORMAT, 0, 0, 0, 0);
}
template <int FORMAT>
__device__ __forceinline__ v4f mfma_block_scaled(v8i b, v8i a, v4f c, int sb, int sa) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, c, 0, FORMAT, 0, sb, 0, sa);
}

// The block's product for f32 results.  The 8-bit instruction aligns the products of a group of 8 to the largest of them and
// drops what lies below 2^-13 of it: 1.5e-5 to 2.4e-5 of a result's norm, measured, which no bf16 or f16 output shows but an
// f32 output does.  Codes are exact in f16, and v_mfma_f32_16x16x32_f16 keeps 24 bits below the largest product, at half the
// rate.  Eight bytes of a lane are one step of 32 of the depth; again both operands only need the same order.
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
template <int FORMAT>
__device__ __forceinline__ v8h widen8(int lo, int hi) {
    typedef _Float16 v2h __attribute__((ext_vector_type(2)));
    v2h r[4];
    if constexpr (FORMAT == FMTC_E4M3) {
        r[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, false);
        r[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, true);
        r[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, false);
        r[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, true);
    } else {
        r[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_bf8(lo, 1.f, false);
        r[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_bf8(lo, 1.f, true);
        r[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_bf8(hi, 1.f, false);
        r[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_bf8(hi, 1.f, true);
    }
    return v8h{r[0][0], r[0][1], r[1][0], r[1][1], r[2][0], r[2][1], r[3][0], r[3][1]};
}
template <int FORMAT>
__device__ __forceinline__ v4f mfma_block_wide(v8i b, v8i a, v4f c) {
#pragma unroll
    for (int j = 0; j < 4; j++)
        c = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen8<FMTC_E4M3>(b[2 * j], b[2 * j + 1]), widen8<FORMAT>(a[2 * j], a[2 * j + 1]), c, 0, 0, 0);
    return c;
}

// How a product is computed: f32 scales and the 8-bit instruction, power-of-two scales as its operands, or f16
enum Way { kScaled = 0, kExponents = 1, kWide = 2 };

// out[m][n .. n + 3] = v (+ bias) (+ what is there)
__device__ __forceinline__ void store_out(void* out, int type, int64_t ld, int64_t m, int64_t n, int64_t N, v4f v,
                                          const float* bias, int accumulate) {
    const int64_t at = m * ld + n;
    const int k = N - n < 4 ? (int)(N - n) : 4;
    if (bias)
#pragma unroll
        for (int i = 0; i < 4; i++)
            if (i < k) v[i] += bias[n + i];
    if (type == FMTC_F32) {
        float* p = static_cast<float*>(out) + at;
#pragma unroll
        for (int i = 0; i < 4; i++)
            if (i < k) v[i] = accumulate ? p[i] + v[i] : v[i];
        if (k == 4) __builtin_memcpy(p, &v, 16);
        else
            for (int i = 0; i < k; i++) p[i] = v[i];
    } else {
        uint16_t r[4];
#pragma unroll
        for (int i = 0; i < 4; i++)
            r[i] = type == FMTC_BF16 ? from_f32<bf16>(v[i]).bits : __builtin_bit_cast(uint16_t, from_f32<_Float16>(v[i]));
        uint16_t* p = static_cast<uint16_t*>(out) + at;
        if (k == 4) __builtin_memcpy(p, r, 8);
        else
            for (int i = 0; i < k; i++) p[i] = r[i];
    }
}

// a scale as a float
__device__ __forceinline__ float scale_value(const void* scales, int kind, int64_t at) {
    if (kind == FMTC_SCALE_F32) return static_cast<const float*>(scales)[at];
    const uint32_t e = static_cast<const uint8_t*>(scales)[at];  // 0: 2^-127, 255: not a number
    return __uint_as_float(e == 0 ? 0x00400000u : e == 255 ? 0x7fc00000u : e << 23);
}

struct Product {
    const uint8_t *a, *b;
    const void *sa, *sb;
    int64_t M, N, blocks, ld_a, ld_b, ld_sa, ld_sb, ld_out;
    const float* bias;
    void* out;
    int out_type, accumulate, scale;
};

// Few rows: 16 MT rows x 16 columns per workgroup, operands straight from memory to registers; the workgroup's wavefronts
// take the blocks of the depth in turn and add their sums up in LDS (in the wavefronts' order).
constexpr int kRowsWaves = 8;
template <int FORMAT, int WAY, int B_ROWS, int MT>
__global__ __launch_bounds__(64 * kRowsWaves) void k_f8_matmul_rows(Product p, uint32_t n_tiles) {
    __shared__ v4f sums[kRowsWaves][MT][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, i16 = lane & 15;
    const int64_t mt = blockIdx.x / n_tiles, nt = blockIdx.x - mt * n_tiles;
    const int64_t n = nt * 16 + i16, n_at = n < p.N ? n : p.N - 1;  // rows that do not exist: the last one, never stored
    const uint8_t* b_row = p.b + n_at * p.ld_b;
    const uint8_t* a_row[MT];
    int64_t m_at[MT];
#pragma unroll
    for (int i = 0; i < MT; i++) {
        const int64_t m = (mt * MT + i) * 16 + i16;
        m_at[i] = m < p.M ? m : p.M - 1;
        a_row[i] = p.a + m_at[i] * p.ld_a;
    }
    v4f acc[MT] = {};
    for (int64_t kb = wave; kb < p.blocks; kb += kRowsWaves) {
        const v8i b = load_operand(b_row + kb * kF8Block, g);
        if constexpr (WAY != kExponents) {
            const int kind = WAY == kScaled ? (int)FMTC_SCALE_F32 : p.scale;
            float sb[4];
#pragma unroll
            for (int r = 0; r < 4; r++) {
                const int64_t nr = nt * 16 + g * 4 + r;
                sb[r] = scale_value(p.sb, kind, kb * p.ld_sb + (nr < p.N ? nr : p.N - 1) / B_ROWS);
            }
#pragma unroll
            for (int i = 0; i < MT; i++) {
                const float sa = scale_value(p.sa, kind, kb * p.ld_sa + m_at[i]);
                const v8i a = load_operand(a_row[i] + kb * kF8Block, g);
                const v4f zero = {}, d = WAY == kScaled ? mfma_block<FORMAT>(b, a, zero) : mfma_block_wide<FORMAT>(b, a, zero);
#pragma unroll
                for (int r = 0; r < 4; r++) acc[i][r] = fmaf(d[r], sa * sb[r], acc[i][r]);
            }
        } else {
            const int sb = static_cast<const uint8_t*>(p.sb)[kb * p.ld_sb + n_at / B_ROWS];
#pragma unroll
            for (int i = 0; i < MT; i++)
                acc[i] = mfma_block_scaled<FORMAT>(b, load_operand(a_row[i] + kb * kF8Block, g), acc[i], sb,
                                                   static_cast<const uint8_t*>(p.sa)[kb * p.ld_sa + m_at[i]]);
        }
    }
#pragma unroll
    for (int i = 0; i < MT; i++) sums[wave][i][lane] = acc[i];
    __syncthreads();
    for (int i = wave; i < MT; i += kRowsWaves) {
        v4f v = sums[0][i][lane];
        for (int w = 1; w < kRowsWaves; w++) v += sums[w][i][lane];
        const int64_t m = (mt * MT + i) * 16 + i16, n4 = nt * 16 + g * 4;
        if (m < p.M && n4 < p.N) store_out(p.out, p.out_type, p.ld_out, m, n4, p.N, v, p.bias, p.accumulate);
    }
}

template <class F>
hipError_t with_way(int way, F&& f) {
    return way == kScaled ? f(Int<kScaled>{}) : way == kExponents ? f(Int<kExponents>{}) : f(Int<kWide>{});
}

}  // namespace

size_t matmul_f8_workspace(int64_t, int64_t, int64_t) { return 0; }

hipError_t launch_f8_matmul(const fmtc_f8& a, const fmtc_f8& b, const float* d_bias, void* d_out, int out_type,
                            int64_t ld_out, int accumulate, void*, hipStream_t s) {
    Product p{static_cast<const uint8_t*>(a.d_codes), static_cast<const uint8_t*>(b.d_codes), a.d_scales, b.d_scales,
              a.rows, b.rows, (a.depth + kF8Block - 1) / kF8Block, a.ld, b.ld, a.ld_scales, b.ld_scales, ld_out,
              d_bias, d_out, out_type, accumulate, a.scale};
    const int64_t n_tiles = (p.N + 15) / 16;
    const int way = out_type == FMTC_F32 ? kWide : a.scale == FMTC_SCALE_E8M0 ? kExponents : kScaled;
    return with_bit(a.format, [&](auto fm) {
        return with_way(way, [&](auto wy) {
            return with_bit(b.block_rows == 1, [&](auto one) {
                constexpr int F = decltype(fm)::value, W = decltype(wy)::value, B = decltype(one)::value ? 1 : kF8Block;
                if (p.M <= 16)
                    return launch(K_F8_MATMUL, k_f8_matmul_rows<F, W, B, 1>, dim3((unsigned)n_tiles), dim3(64 * kRowsWaves), 0, s, p,
                                  (uint32_t)n_tiles);
                return launch(K_F8_MATMUL, k_f8_matmul_rows<F, W, B, 4>, dim3((unsigned)(n_tiles * ((p.M + 63) / 64))),
                              dim3(64 * kRowsWaves), 0, s, p, (uint32_t)n_tiles);
            });
        });
    });
}

}  // namespace fmtc
