// Internal declarations of the block operators (fmtc_f8_*, fmtc_block_norm*): what the host side checks and hands to the
// kernels, and the small device helpers that their kernel files share.
#pragma once
#include <math.h>

#include "fmtc_internal.h"

namespace fmtc {

constexpr int kF8Block = FMTC_F8_BLOCK;

// Leaves a text for fmtc_last_error() and returns `st` (fmtc_api.hip).
fmtc_status set_error(fmtc_status st, const char* fmt, ...);

// ---- launchers (fmtc_quantize_f8_kernels.hip, fmtc_matmul_f8_kernels.hip, fmtc_norm_kernels.hip) ----
// values [rows][cols] -> codes and scales; by_rows, by_cols: either may be NULL.  d_col_sums (NULL, or [blocks of 128
// rows][cols] f32, with by_cols): each block's column sums.
hipError_t launch_f8_quantize(const void* d_x, int type, int64_t rows, int64_t cols, int64_t ld_x, const fmtc_f8* by_rows,
                              const fmtc_f8* by_cols, float* d_col_sums, hipStream_t s);
// out[c] (+)= sum over n rows of d_part[row][c]
hipError_t launch_column_sums(const float* d_part, int64_t n, int64_t cols, float* d_out, int accumulate, hipStream_t s);
// zeros in rows x cols floats
hipError_t launch_fill_rows(float* d_out, int64_t rows, int64_t cols, int64_t ld, hipStream_t s);

size_t matmul_f8_workspace(int64_t M, int64_t N, int64_t K);
hipError_t launch_f8_matmul(const fmtc_f8& a, const fmtc_f8& b, const float* d_bias, void* d_out, int out_type,
                            int64_t ld_out, int accumulate, void* d_ws, hipStream_t s);

size_t block_norm_workspace(int64_t rows, int C, int64_t rows_per_gate);
hipError_t launch_block_norm(const fmtc_norm& a, void* d_h_out, int64_t ld_h_out, void* d_n, int64_t ld_n,
                             const fmtc_f8* n_codes, float* d_stats, hipStream_t s);
hipError_t launch_block_norm_backward(const fmtc_norm& a, const float* d_stats, const void* d_dn, int64_t ld_dn,
                                      const void* d_dh, int64_t ld_dh, void* d_dy, int64_t ld_dy, void* d_dh_in,
                                      int64_t ld_dh_in, float* d_dw_post, float* d_dw_pre, float* d_dgate,
                                      void* d_ws, hipStream_t s);

// ---- device helpers ----
struct bf16 { uint16_t bits; };

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(_Float16 v) { return (float)v; }
__device__ __forceinline__ float to_f32(bf16 v) { return __uint_as_float((uint32_t)v.bits << 16); }

template <class T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ _Float16 from_f32<_Float16>(float v) { return (_Float16)v; }
template <>
__device__ __forceinline__ bf16 from_f32<bf16>(float v) {
    const __bf16 r = (__bf16)v;  // to the nearest, ties to even
    return bf16{__builtin_bit_cast(uint16_t, r)};
}

// the first n of 8 consecutive values; rows need not be aligned beyond their own type: the hardware takes wide accesses at
// any address
template <class T>
__device__ __forceinline__ void store8(T* p, int64_t n, const float (&v)[8]) {
    if (n >= 8) {
        T t[8];
#pragma unroll
        for (int i = 0; i < 8; i++) t[i] = from_f32<T>(v[i]);
        __builtin_memcpy(p, t, sizeof t);
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (i < n) p[i] = from_f32<T>(v[i]);
    }
}

// 8 values as they lie in memory, in whole registers
template <class T>
struct Raw {
    static constexpr int kWords = 2 * sizeof(T), kPer = 4 / sizeof(T);
    uint32_t w[kWords];
    // Values c .. c + 7 of a row of C: one load without a branch, so that many can be on their way together.  At the end of a
    // row whose length is no multiple of 8 it takes the row's last 8 values; lanes past the row read its first ones, which
    // their caller has no use for.
    template <bool RAGGED>
    __device__ __forceinline__ void load(const T* row, int64_t c, int64_t C) {
        if constexpr (!RAGGED) {
            __builtin_memcpy(w, row + (c < C ? c : 0), sizeof w);
        } else if (C >= 8) {
            __builtin_memcpy(w, row + (c + 8 <= C ? c : c < C ? C - 8 : 0), sizeof w);
        } else {
#pragma unroll
            for (int i = 0; i < kWords; i++) {
                w[i] = 0;
#pragma unroll
                for (int j = 0; j < kPer; j++)
                    if (c + i * kPer + j < C) {
                        if constexpr (kPer == 2) w[i] |= (uint32_t)__builtin_bit_cast(uint16_t, row[c + i * kPer + j]) << (16 * j);
                        else w[i] = __builtin_bit_cast(uint32_t, row[c + i]);
                    }
            }
        }
    }
    // when the values are there, in rows whose length is no multiple of 8 (kernels are built for either: without the question
    // the loads of aligned rows run up to a tenth faster): those at the end of a row to their places, 0 behind them
    __device__ __forceinline__ void settle(int64_t c, int64_t C) {
        if (C < 8) return;
        const int by = c < C && c + 8 > C ? (int)(c + 8 - C) : 0;
        int step = kWords / 2;
#pragma unroll
        for (int bit = 4; bit * kPer >= kPer * kPer; bit >>= 1, step >>= 1)
#pragma unroll
            for (int i = 0; i < kWords; i++) {
                const uint32_t from = i + step < kWords ? w[i + step] : 0u;
                w[i] = by & bit ? from : w[i];
            }
        if constexpr (kPer == 2) {
#pragma unroll
            for (int i = 0; i < kWords; i++) {
                const uint32_t above = i + 1 < kWords ? w[i + 1] : 0u;
                w[i] = by & 1 ? w[i] >> 16 | above << 16 : w[i];
            }
        }
    }
    __device__ __forceinline__ void zero_unless(bool live) {
#pragma unroll
        for (int i = 0; i < kWords; i++) w[i] = live ? w[i] : 0u;
    }
    __device__ __forceinline__ float operator[](int i) const {
        if constexpr (kPer == 1) return __uint_as_float(w[i]);
        else return to_f32(__builtin_bit_cast(T, (uint16_t)(w[i >> 1] >> (16 * (i & 1)))));
    }
};
template <bool RAGGED, class T>
__device__ __forceinline__ void load8(const T* row, int64_t c, int64_t C, float (&v)[8]) {
    Raw<T> raw;
    raw.template load<RAGGED>(row, c, C);
    if constexpr (RAGGED) raw.settle(c, C);
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = raw[i];
}

// a reduction over a row of 16 lanes; every lane of the row gets the result
template <int CTRL>
__device__ __forceinline__ float dpp_f32(float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float row16_max(float v) {
    v = fmaxf(v, dpp_f32<0x128>(v));  // row_ror:8
    v = fmaxf(v, dpp_f32<0x124>(v));
    v = fmaxf(v, dpp_f32<0x122>(v));
    return fmaxf(v, dpp_f32<0x121>(v));
}
__device__ __forceinline__ float row16_sum(float v) {
    v += dpp_f32<0x128>(v);
    v += dpp_f32<0x124>(v);
    v += dpp_f32<0x122>(v);
    return v + dpp_f32<0x121>(v);
}

// ---- 8-bit floating point with a scale per block ----
// |v|, or 0 where v is infinite or not a number: such a value takes no part in its block's scale
__device__ __forceinline__ float finite_abs(float v) {
    const uint32_t b = __float_as_uint(v) & 0x7fffffffu;
    return b < 0x7f800000u ? __uint_as_float(b) : 0.f;
}
// largest finite magnitude of 8 values; magnitudes compare as their bits do, and only what is not finite (rare) takes the
// longer way
__device__ __forceinline__ float finite_amax(const float (&v)[8]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const uint32_t b = __float_as_uint(v[i]) & 0x7fffffffu;
        m = b > m ? b : m;
    }
    if (m < 0x7f800000u) return __uint_as_float(m);
    float a = 0.f;
#pragma unroll
    for (int i = 0; i < 8; i++) a = fmaxf(a, finite_abs(v[i]));
    return a;
}
// The scale of a block whose largest magnitude is amax.  -> the factor that values are multiplied by; *held: what is
// stored (a float's bits, or the biased exponent).  Both formats' largest number is 1.75 times a power of two, so the
// power-of-two scale is an exact decision on the bits of amax: one more than its exponent where its fraction is over .75.
template <int FORMAT, int SCALE>
__device__ __forceinline__ float block_scale(float amax, uint32_t* held) {
    if constexpr (SCALE == FMTC_SCALE_F32) {
        const float s = fmaxf(amax * (FORMAT == FMTC_E4M3 ? 1.f / 448.f : 1.f / 57344.f), 0x1p-126f);
        *held = __float_as_uint(s);
        return 1.f / s;
    } else {
        int e = (int)((__float_as_uint(amax) + 0x1fffffu) >> 23) - (FORMAT == FMTC_E4M3 ? 8 : 15);
        e = e < 1 ? 1 : e;  // (at most 254 - 8 + 1)
        *held = (uint32_t)e;
        return __uint_as_float((uint32_t)(254 - e) << 23);
    }
}
// four codes, the first in the lowest byte; to the nearest, ties to even; infinities become NaN in E4M3
template <int FORMAT>
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
    int r = 0;
    if constexpr (FORMAT == FMTC_E4M3) {
        r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, r, false);
        r = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
    } else {
        r = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, r, false);
        r = __builtin_amdgcn_cvt_pk_bf8_f32(c, d, r, true);
    }
    return (uint32_t)r;
}
template <int SCALE>
__device__ __forceinline__ void store_scale(void* d_scales, int64_t at, uint32_t held) {
    if constexpr (SCALE == FMTC_SCALE_F32)
        static_cast<uint32_t*>(d_scales)[at] = held;
    else
        static_cast<uint8_t*>(d_scales)[at] = (uint8_t)held;
}

// Calls body(std::integral_constant-like) for a run-time choice: f(Type<float>{}) and so on.
template <class T>
struct Type { using type = T; };
template <class F>
hipError_t with_type(int type, F&& f) {
    switch (type) {
        case FMTC_BF16: return f(Type<bf16>{});
        case FMTC_F16: return f(Type<_Float16>{});
        default: return f(Type<float>{});
    }
}
template <int V>
struct Int { static constexpr int value = V; };
template <class F>
hipError_t with_bit(int v, F&& f) { return v ? f(Int<1>{}) : f(Int<0>{}); }

}  // namespace fmtc
