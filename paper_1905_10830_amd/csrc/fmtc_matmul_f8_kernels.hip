// Products of 8-bit floating point matrices with a scale per block of 128 (fmtc_f8_matmul):
//   out[m][n] = sum_b sa[b][m] sb[b][n / block_rows] sum_{k in b} a[m][k] b[n][k] (+ bias[n])
// One v_mfma_f32_16x16x128_f8f6f4 is exactly one block of the depth for 16 x 16 results.  b's rows are the instruction's
// first operand and a's its second: a lane then holds four consecutive columns n of one row m of the result, so that sa is
// one number per lane and the results leave in vectors.  Power-of-two scales are operands of the instruction itself; f32
// scales multiply the block's product, which one fma adds to the running f32 sum.
#include <type_traits>

#include "fmtc_block.h"
#include "fmtc_device.h"

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
// drops what lies below 2^-13 of it: 1.5e-5 to 2.4e-5 of the results' norm with operands of one size, 5e-5 to 7e-5 with
// channels 100 times the others (2048 to 4096 deep), beside the 2.1e-4 of rounding to f16.  An f32 result would show it.  Codes are exact in f16, and v_mfma_f32_16x16x32_f16 keeps 24 bits below the largest product, at half the
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
struct Wide { v8h v[4]; };
template <int FORMAT>
__device__ __forceinline__ Wide widen(v8i q) {
    Wide w;
#pragma unroll
    for (int j = 0; j < 4; j++) w.v[j] = widen8<FORMAT>(q[2 * j], q[2 * j + 1]);
    return w;
}
__device__ __forceinline__ v4f mfma_block_wide(const Wide& b, const Wide& a, v4f c) {
#pragma unroll
    for (int j = 0; j < 4; j++) c = __builtin_amdgcn_mfma_f32_16x16x32_f16(b.v[j], a.v[j], c, 0, 0, 0);
    return c;
}

// With power-of-two scales the same in bf16, the scale in the conversion: bf16 has f32's exponents, so that the numbers are as
// exact (but for those under 2^-133), and the instruction adds to the running sum itself (4096^3 150 -> 135 us).
typedef __bf16 v8b __attribute__((ext_vector_type(8)));
template <int FORMAT>
__device__ __forceinline__ v8b widen8_scaled(int lo, int hi, float scale) {
    typedef __bf16 v2b __attribute__((ext_vector_type(2)));
    v2b r[4];
    if constexpr (FORMAT == FMTC_E4M3) {
        r[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
        r[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
        r[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
        r[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    } else {
        r[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(lo, scale, false);
        r[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(lo, scale, true);
        r[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(hi, scale, false);
        r[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(hi, scale, true);
    }
    return v8b{r[0][0], r[0][1], r[1][0], r[1][1], r[2][0], r[2][1], r[3][0], r[3][1]};
}
struct Scaled { v8b v[4]; };
template <int FORMAT>
__device__ __forceinline__ Scaled widen_scaled(v8i q, uint32_t scale) {
    Scaled w;
#pragma unroll
    for (int j = 0; j < 4; j++) w.v[j] = widen8_scaled<FORMAT>(q[2 * j], q[2 * j + 1], __uint_as_float(scale));
    return w;
}
__device__ __forceinline__ v4f mfma_block_wide(const Scaled& b, const Scaled& a, v4f c) {
#pragma unroll
    for (int j = 0; j < 4; j++) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b.v[j], a.v[j], c, 0, 0, 0);
    return c;
}

// How a product is computed: f32 scales and the 8-bit instruction, power-of-two scales as its operands, f32 scales and f16, or
// power-of-two scales and bf16
enum Way { kScaled = 0, kExponents = 1, kWide = 2, kWideExponents = 3 };
constexpr bool is_wide(int way) { return way >= kWide; }
constexpr int scale_kind(int way) { return way == kScaled || way == kWide ? FMTC_SCALE_F32 : FMTC_SCALE_E8M0; }

// bias[n .. n + 3], 0 where there is none.  (Columns past the last: the last one's, for results that are not stored.  Loaded
// once, not for every row, where it would wait for the stores before it: 4096^3 76 -> 64 us, 5125 x 4096 x 315 49 -> 30 us.)
__device__ __forceinline__ v4f load_bias(const float* bias, int64_t n, int64_t N) {
    v4f v = {};
    if (bias)
#pragma unroll
        for (int i = 0; i < 4; i++) v[i] = bias[n + i < N ? n + i : N - 1];
    return v;
}

// out[m][n .. n + 3] = v + bias (+ what is there)
__device__ __forceinline__ void store_out(void* out, int type, int64_t ld, int64_t m, int64_t n, int64_t N, v4f v, v4f bias,
                                          int accumulate) {
    const int64_t at = m * ld + n;
    const int k = N - n < 4 ? (int)(N - n) : 4;
    v += bias;
    if (type == FMTC_F32) {
        float* p = static_cast<float*>(out) + at;
        if (k == 4) {
            if (accumulate) {
                v4f there;
                __builtin_memcpy(&there, p, 16);
                v += there;
            }
            __builtin_memcpy(p, &v, 16);
        } else {
            for (int i = 0; i < k; i++) p[i] = accumulate ? p[i] + v[i] : v[i];
        }
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

// a scale as it is held, and as a float
template <int KIND>
__device__ __forceinline__ uint32_t load_scale(const void* scales, int64_t at) {
    if constexpr (KIND == FMTC_SCALE_F32) return static_cast<const uint32_t*>(scales)[at];
    else return static_cast<const uint8_t*>(scales)[at];
}
template <int KIND>
__device__ __forceinline__ uint32_t scale_bits(uint32_t held) {
    if constexpr (KIND == FMTC_SCALE_F32) return held;
    else return held == 0 ? 0x00400000u : held == 255 ? 0x7fc00000u : held << 23;  // 2^-127 and not a number
}
template <int KIND>
__device__ __forceinline__ float scale_value(const void* scales, int64_t at) {
    return __uint_as_float(scale_bits<KIND>(load_scale<KIND>(scales, at)));
}

struct Product {
    const uint8_t *a, *b;
    const void *sa, *sb;
    int64_t M, N, blocks, ld_a, ld_b, ld_sa, ld_sb, ld_out;
    const float* bias;
    void* out;
    int out_type, accumulate;
    int64_t split_blocks;  // tiles: blocks of the depth that a workgroup takes; the sums of split z go to out + z * split_out
    int64_t split_out;     // floats
};

// Few rows: 16 MT rows x 16 NT columns per workgroup, operands straight from memory to registers; the workgroup's wavefronts
// take the blocks of the depth in turn and add their sums up in LDS (in the wavefronts' order).  Bound by the weights' bytes;
// the rows of a come out of the caches once for every workgroup, so beyond 16 of them two tiles of columns share them where
// that leaves a workgroup for every compute unit (64 x 8192 x 2048 12.7 -> 9.7 us; 13 x 8192 x 8192 would lose, 15.7 -> 19.5 us
// with the weights in the memory-side cache).  1 x 8192 x 8192 13.4 us (5.0 TB/s), 1 x 4096 x 4096 5.9 us; loads of two or four
// blocks ahead gain nothing (13.4 -> 14.5 us).
constexpr int kRowsWaves = 8;
template <int FORMAT, int WAY, int B_ROWS, int MT, int NT>
__global__ __launch_bounds__(64 * kRowsWaves) void k_f8_matmul_rows(Product p, uint32_t n_tiles) {
    __shared__ v4f sums[kRowsWaves][MT * NT][64];
    constexpr int kKind = scale_kind(WAY);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, i16 = lane & 15;
    const int64_t mt = blockIdx.x / n_tiles, nt = blockIdx.x - mt * n_tiles;
    const uint8_t *a_row[MT], *b_row[NT];  // (rows that do not exist: the last one, never stored)
    int64_t m_at[MT], n_at[NT][4];         // rows whose scales are wanted
#pragma unroll
    for (int i = 0; i < MT; i++) {
        const int64_t m = (mt * MT + i) * 16 + i16;
        m_at[i] = m < p.M ? m : p.M - 1;
        a_row[i] = p.a + m_at[i] * p.ld_a;
    }
#pragma unroll
    for (int j = 0; j < NT; j++) {
        const int64_t n0 = (nt * NT + j) * 16, n = n0 + i16;
        b_row[j] = p.b + (n < p.N ? n : p.N - 1) * p.ld_b;
#pragma unroll
        for (int r = 0; r < 4; r++) {
            const int64_t nr = WAY == kExponents ? n : n0 + 4 * g + r;
            n_at[j][r] = (nr < p.N ? nr : p.N - 1) / B_ROWS;
        }
    }
    constexpr int kB = WAY != kExponents && B_ROWS == 1 ? 4 : 1;  // scales of b a lane needs
    v4f acc[MT][NT] = {};
    for (int64_t kb = wave; kb < p.blocks; kb += kRowsWaves) {
        v8i b[NT], a[MT];
        uint32_t sb[NT][kB], sa[MT];
#pragma unroll
        for (int j = 0; j < NT; j++) {
            b[j] = load_operand(b_row[j] + kb * kF8Block, g);
#pragma unroll
            for (int r = 0; r < kB; r++) sb[j][r] = load_scale<kKind>(p.sb, kb * p.ld_sb + n_at[j][r]);
        }
#pragma unroll
        for (int i = 0; i < MT; i++) {
            a[i] = load_operand(a_row[i] + kb * kF8Block, g);
            sa[i] = load_scale<kKind>(p.sa, kb * p.ld_sa + m_at[i]);
        }
        __builtin_amdgcn_sched_barrier(0);  // all loads on their way before the first is waited for
#pragma unroll
        for (int i = 0; i < MT; i++)
#pragma unroll
            for (int j = 0; j < NT; j++) {
                if constexpr (WAY == kExponents) {
                    acc[i][j] = mfma_block_scaled<FORMAT>(b[j], a[i], acc[i][j], (int)sb[j][0], (int)sa[i]);
                } else {
                    v4f d;
                    if constexpr (is_wide(WAY)) d = mfma_block_wide(widen<FMTC_E4M3>(b[j]), widen<FORMAT>(a[i]), v4f{0.f, 0.f, 0.f, 0.f});
                    else d = mfma_block<FORMAT>(b[j], a[i], v4f{0.f, 0.f, 0.f, 0.f});
                    const float s = __uint_as_float(scale_bits<kKind>(sa[i]));
#pragma unroll
                    for (int r = 0; r < 4; r++)
                        acc[i][j][r] = fmaf(d[r], s * __uint_as_float(scale_bits<kKind>(sb[j][kB == 4 ? r : 0])), acc[i][j][r]);
                }
            }
    }
#pragma unroll
    for (int i = 0; i < MT; i++)
#pragma unroll
        for (int j = 0; j < NT; j++) sums[wave][i * NT + j][lane] = acc[i][j];
    __syncthreads();
    for (int k = wave; k < MT * NT; k += kRowsWaves) {
        v4f v = sums[0][k][lane];
#pragma unroll
        for (int w = 1; w < kRowsWaves; w++) v += sums[w][k][lane];
        const int64_t m = (mt * MT + k / NT) * 16 + i16, n4 = (nt * NT + k % NT) * 16 + g * 4;
        if (m < p.M && n4 < p.N) store_out(p.out, p.out_type, p.ld_out, m, n4, p.N, v, load_bias(p.bias, n4, p.N), p.accumulate);
    }
}

// Many rows: a tile of BM x BN results per workgroup, operands through LDS, one block of the depth (128 bytes of a row) a
// step, two steps' operands in LDS.  A wavefront has MT x 4 tiles of 16 x 16: b's four tiles of a step stay in registers,
// a's come one after the other, each read while the one before it is multiplied.  The one barrier of a step stands before
// its last tile of a, when everything that is still needed of the step is in registers: behind it the next step's operands
// are read and those of the step after it set out into the place that came free, all under the last tile's products.
//
// Rows of 128 bytes in LDS, the 16-byte pieces of a row exchanged by a key of the row, so that 16 lanes that read the same
// piece of 16 rows touch every bank once.  The results leave through LDS too, 64 columns of a row at a time.
//
// bf16 results, 4096^3 / 8192^3, on the device: f32 scales 64 / 444 to 458 us (an fma for each result and block), power-of-two
// scales 59 to 65 / 437 to 468 us (2350 to 2520 TFLOP/s; the matrix pipes are busy 45 / 60 % of the clocks, at 2.0 to 2.3 GHz).
// f32 results: f32 scales 132 to 166 / 1060 us, power-of-two scales 104 to 114 / 753 to 835 us (widening shares the issue slots).
template <int WM_, int WN_, int MT_, int STAGES_>
struct Tile {
    static constexpr int WM = WM_, WN = WN_, MT = MT_, NT = 4, kStages = STAGES_;
    static constexpr int kThreads = 64 * WM * WN, BM = WM * MT * 16, BN = WN * NT * 16;
    static constexpr int kStage = (BM + BN) * kF8Block, kScales = 4 * kThreads;
    static constexpr int kLoads = (BM + BN) / 8 / (WM * WN);  // loads of 8 rows a wavefront, a's and b's in one range
    static constexpr int kPitch = 68, kOutRows = 64;         // results in LDS: a wavefront's 64 rows x 64 columns at a time
    static constexpr int kLoop = kStages * (kStage + kScales), kOut = WM * WN * kOutRows * kPitch * 4;
    static constexpr int kLds = kLoop > kOut ? kLoop : kOut;
    static_assert((BM + BN) % (8 * WM * WN) == 0 && BM % 64 == 0 && MT % 4 == 0);
    static_assert(BM + BN <= kThreads);  // a lane moves one scale
    static_assert((kStages & (kStages - 1)) == 0);
};
__device__ __forceinline__ int row_key(int row) { return (row >> 1) & 7; }

// 16 bytes, 4 bytes or a byte (as a word) a lane from base + off straight into LDS, lane l to lds_base + 16 l or 4 l; the
// caller counts its loads in flight
template <int BYTES>
__device__ __forceinline__ void load_to_lds_at(const void* base, uint32_t off, uint32_t lds_base) {
    uint32_t keep;
    if constexpr (BYTES == 16)
        asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2\n\ts_mov_b32 m0, %0"
                     : "=&s"(keep) : "v"(off), "s"(base), "s"(lds_base) : "memory");
    else if constexpr (BYTES == 4)
        asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2\n\ts_mov_b32 m0, %0"
                     : "=&s"(keep) : "v"(off), "s"(base), "s"(lds_base) : "memory");
    else
        asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_ubyte %1, %2\n\ts_mov_b32 m0, %0"
                     : "=&s"(keep) : "v"(off), "s"(base), "s"(lds_base) : "memory");
}

template <int FORMAT, int WAY, int B_ROWS, class S>
__global__ __launch_bounds__(S::kThreads, 2) void k_f8_matmul_tiles(Product p, uint32_t tiles_m, uint32_t tiles_n) {
    extern __shared__ __attribute__((aligned(128))) uint8_t lds[];
    constexpr int MT = S::MT, NT = S::NT;
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), g = lane >> 4, i16 = lane & 15;
    const int wm = wave % S::WM, wn = wave / S::WM;

    // Workgroups go to the 8 XCDs in turn: each XCD gets a range of tiles, and within it four rows of tiles at a time, so
    // that the tiles that run on it together share operands in its cache.
    const uint32_t total = gridDim.x, each = total / 8, more = total % 8, xcd = blockIdx.x % 8;
    const uint32_t place = xcd * each + (xcd < more ? xcd : more) + blockIdx.x / 8;
    const uint32_t z = place / (tiles_m * tiles_n), id = place - z * (tiles_m * tiles_n);
    const uint32_t span = 4 * tiles_n, first = id / span * 4, in = id % span, deep = tiles_m - first < 4 ? tiles_m - first : 4;
    const int64_t m0 = (int64_t)(first + in % deep) * S::BM, n0 = (int64_t)(in / deep) * S::BN;
    const int rows_a = p.M - m0 < S::BM ? (int)(p.M - m0) : S::BM, rows_b = p.N - n0 < S::BN ? (int)(p.N - n0) : S::BN;

    // what this lane moves: 16 bytes of kLoads rows (rows that do not exist: the last one, whose results are not stored)
    const int64_t kb0 = z * p.split_blocks, blocks = p.blocks - kb0 < p.split_blocks ? p.blocks - kb0 : p.split_blocks;
    const uint8_t *from_a = p.a + m0 * p.ld_a + kb0 * kF8Block, *from_b = p.b + n0 * p.ld_b + kb0 * kF8Block;
    uint32_t off[S::kLoads];
#pragma unroll
    for (int i = 0; i < S::kLoads; i++) {
        const int row = (wave * S::kLoads + i) * 8 + (lane >> 3);
        const bool of_a = row < S::BM;
        const int r = of_a ? (row < rows_a ? row : rows_a - 1) : (row - S::BM < rows_b ? row - S::BM : rows_b - 1);
        off[i] = (uint32_t)r * (uint32_t)(of_a ? p.ld_a : p.ld_b) + 16 * ((lane & 7) ^ row_key(row));
    }
    const uint32_t lds_at = (uint32_t)(uintptr_t)(lds_void_t*)lds;
    // Scales: a lane moves that of a row of a or of b (past both: the last of b again), as it is straight into LDS, or, for the
    // bf16 way that would make floats of them again and again, through a register in which it becomes one.
    constexpr bool kStraight = WAY != kWideExponents;
    static_assert(kStraight || S::kStages == 2);
    uint32_t mine = 0;
    constexpr int kScaleBytes = scale_kind(WAY) == FMTC_SCALE_F32 ? 4 : 1, kStages = S::kStages;
    uint32_t* const scales = reinterpret_cast<uint32_t*>(lds + kStages * S::kStage);
    const bool scale_of_a = wave * 64 < S::BM;
    const int64_t step_s = scale_of_a ? p.ld_sa : p.ld_sb;
    const uint8_t* const from_s = static_cast<const uint8_t*>(scale_of_a ? p.sa : p.sb) + ((scale_of_a ? m0 : n0 / B_ROWS) + kb0 * step_s) * kScaleBytes;
    uint32_t off_s;
    if (scale_of_a) off_s = t < rows_a ? t : rows_a - 1;
    else off_s = (t - S::BM < rows_b ? t - S::BM : rows_b - 1) / B_ROWS;
    off_s *= kScaleBytes;
    // A quarter of a step's loads, the scales with the first: all at once, the queue of loads is full and the wavefront stands
    // still.  (f16: the products take twice as long and come less dense, the loads are best out of the way: 1112 us in
    // quarters, 1038 us, 8192^3.)  Past the last block: that one again, into a place that is free; not used, and no branch in
    // the loop.
    constexpr bool kQuarters = !is_wide(WAY);
    const int64_t last = blocks - 1;
    auto fetch = [&](int64_t kb, int quarter) {
        const uint32_t stage = (uint32_t)kb & (kStages - 1), to = lds_at + stage * S::kStage + wave * S::kLoads * 1024;
        if (kb > last) kb = last;
        if (quarter == 0) {
            const uint8_t* const from = from_s + kb * step_s * kScaleBytes;
            if constexpr (kStraight) load_to_lds_at<kScaleBytes>(from, off_s, lds_at + kStages * S::kStage + stage * S::kScales + wave * 256);
            else mine = from[off_s];
        }
#pragma unroll
        for (int i = quarter * S::kLoads / 4; i < (quarter + 1) * S::kLoads / 4; i++)
            load_to_lds_at<16>(((wave * S::kLoads + i) * 8 < S::BM ? from_a : from_b) + kb * kF8Block, off[i], to + i * 1024);
    };
    auto put_scale = [&](int64_t kb) {
        if constexpr (!kStraight) scales[((uint32_t)kb & (kStages - 1)) * S::kThreads + t] = scale_bits<FMTC_SCALE_E8M0>(mine);
    };
    constexpr int kEach = S::kLoads + 1, kFirst = 1 + (kQuarters ? S::kLoads / 2 : S::kLoads);  // loads of a step, of its first part

    const int row_a = wm * MT * 16 + i16, row_b = S::BM + wn * 64 + i16, key = row_key(i16);  // (the key of row + 16 i, too)
    auto piece = [&](int64_t kb, int row) {
        const uint8_t* at = lds + ((uint32_t)kb & (kStages - 1)) * S::kStage + row * kF8Block;
        const v4i lo = *reinterpret_cast<const v4i*>(at + 16 * (g ^ key)), hi = *reinterpret_cast<const v4i*>(at + 16 * ((4 + g) ^ key));
        return v8i{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    };

    v4f acc[MT][NT] = {};
    // all blocks' loads that fit, and the first part of those of the last place's; the rest of them in the first step
#pragma unroll
    for (int k = 0; k < kStages; k++) {
#pragma unroll
        for (int q = 0; q < (kQuarters && k == kStages - 1 ? 2 : 4); q++) fetch(k, q);
        if (k == 0) put_scale(0);
    }
    wait_loads<(kStages - 2) * kEach + kFirst>();
    __syncthreads();
    // b's tiles as the way takes them; the products of a tile of a, added to the sums while the next one is multiplied
    using Held = typename std::conditional<WAY == kWideExponents, Scaled, typename std::conditional<WAY == kWide, Wide, v8i>::type>::type;
    constexpr bool kInside = WAY == kExponents || WAY == kWideExponents;  // the scales are in the operands
    Held b[NT];
    v8i a[3];  // tiles i, i + 1 and i + 2: a tile's read has two tiles' products to arrive under
    uint32_t sa[3], sb[NT][4];
    auto read_a = [&](int to, int64_t kb, int i) {
        a[to] = piece(kb, row_a + 16 * i);
        sa[to] = scales[((uint32_t)kb & (kStages - 1)) * S::kThreads + row_a + 16 * i];
    };
    auto read_b = [&](int64_t kb, int j) {
        const uint32_t* s = scales + ((uint32_t)kb & (kStages - 1)) * S::kThreads;
        const v8i raw = piece(kb, row_b + 16 * j);
        if constexpr (WAY == kWideExponents) b[j] = widen_scaled<FMTC_E4M3>(raw, s[row_b + 16 * j]);
        else if constexpr (WAY == kWide) b[j] = widen<FMTC_E4M3>(raw);
        else b[j] = raw;
        if constexpr (WAY == kExponents) {
            sb[j][0] = s[row_b + 16 * j];
        } else if constexpr (WAY == kWideExponents) {
        } else if constexpr (B_ROWS == 1) {
            const uint4 v = *reinterpret_cast<const uint4*>(s + S::BM + wn * 64 + 16 * j + 4 * g);
            sb[j][0] = v.x, sb[j][1] = v.y, sb[j][2] = v.z, sb[j][3] = v.w;
        } else if (j == 0) {
            sb[0][0] = s[S::BM + wn * 64];
        }
    };
    read_a(0, 0, 0);
    read_a(1, 0, 1);
#pragma unroll
    for (int j = 0; j < NT; j++) read_b(0, j);
    v4f d[NT] = {};
    float f[NT][4] = {};

    for (int64_t kb = 0; kb < blocks; kb++) {
#pragma unroll
        for (int i = 0; i < MT; i++) {
            if (i == MT - 2) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the last tiles of a are in registers
                wait_loads<(kStages - 2) * kEach>();                // the next step's operands (this wavefront's) are in LDS
                put_scale(kb + 1);
                __syncthreads();
            }
            if (i == MT - 2 || (kQuarters && i == MT - 1)) {
#pragma unroll
                for (int q = i - (MT - 2); q < (kQuarters ? i - (MT - 2) + 1 : 4); q++) fetch(kb + kStages, q);
            }
            if (kQuarters && i < 2) fetch(kb + kStages - 1, i + 2);
            // (past the last step: what LDS holds, not used)
            if (i < MT - 2) read_a(2, kb, i + 2);
            else read_a(2, kb + 1, i + 2 - MT);
            if constexpr (WAY == kExponents) {
#pragma unroll
                for (int j = 0; j < NT; j++) {
                    acc[i][j] = mfma_block_scaled<FORMAT>(b[j], a[0], acc[i][j], (int)sb[j][0], (int)sa[0]);
                    if (i == MT - 1) read_b(kb + 1, j);
                }
            } else if constexpr (WAY == kWideExponents) {
                const Scaled with = widen_scaled<FORMAT>(a[0], sa[0]);
#pragma unroll
                for (int j = 0; j < NT; j++) acc[i][j] = mfma_block_wide(b[j], with, acc[i][j]);
                if (i == MT - 1)
#pragma unroll
                    for (int j = 0; j < NT; j++) read_b(kb + 1, j);
            } else {
                v4f* const before = acc[i ? i - 1 : MT - 1];
                const auto with = [&] { if constexpr (is_wide(WAY)) return widen<FORMAT>(a[0]); else return a[0]; }();
#pragma unroll
                for (int j = 0; j < NT; j++) {
                    v4f now;
                    if constexpr (is_wide(WAY)) now = mfma_block_wide(b[j], with, v4f{0.f, 0.f, 0.f, 0.f});
                    else now = mfma_block<FORMAT>(b[j], with, v4f{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                    for (int r = 0; r < 4; r++) {
                        before[j][r] = fmaf(d[j][r], f[B_ROWS == 1 ? j : 0][B_ROWS == 1 ? r : 0], before[j][r]);
                        if constexpr (B_ROWS == 1) f[j][r] = __uint_as_float(sa[0]) * __uint_as_float(sb[j][r]);
                    }
                    if constexpr (is_wide(WAY)) asm volatile("" : "+v"(before[j]));  // (else the scheduler gathers the sums)
                    d[j] = now;
                }
                if constexpr (B_ROWS != 1) f[0][0] = __uint_as_float(sa[0]) * __uint_as_float(sb[0][0]);
                if (i == MT - 1)
#pragma unroll
                    for (int j = 0; j < NT; j++) read_b(kb + 1, j);
            }
            a[0] = a[1], a[1] = a[2], sa[0] = sa[1], sa[1] = sa[2];
            if constexpr (WAY == kScaled) {
#pragma unroll
                for (int j = 0; j < NT; j++) {  // the sums of the tile before it between this one's products
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    if constexpr (!kInside) {
#pragma unroll
        for (int j = 0; j < NT; j++)
#pragma unroll
            for (int r = 0; r < 4; r++) acc[MT - 1][j][r] = fmaf(d[j][r], f[B_ROWS == 1 ? j : 0][B_ROWS == 1 ? r : 0], acc[MT - 1][j][r]);
    }
    // 4 tiles of a at a time: 64 rows of 64 columns in the wavefront's own part of LDS, then whole rows to memory
    wait_loads<0>();
    __syncthreads();
    float* const out = reinterpret_cast<float*>(lds) + wave * S::kOutRows * S::kPitch;
    const int64_t n = n0 + wn * 64 + 4 * i16;
    void* const to = p.split_out ? static_cast<float*>(p.out) + z * p.split_out : p.out;
    v4f bias = load_bias(p.bias, n, p.N);
    asm volatile("" : "+v"(bias));  // (waited for here: in the loop a wait for it is one for the stores, too)
#pragma unroll
    for (int i0 = 0; i0 < MT; i0 += 4) {
#pragma unroll
        for (int i = 0; i < 4; i++)
#pragma unroll
            for (int j = 0; j < NT; j++) *reinterpret_cast<v4f*>(out + (16 * i + i16) * S::kPitch + 16 * j + 4 * g) = acc[i0 + i][j];
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll 4
        for (int r = g; r < 64; r += 4) {
            const int64_t m = m0 + wm * MT * 16 + i0 * 16 + r;
            const v4f v = *reinterpret_cast<const v4f*>(out + r * S::kPitch + 4 * i16);
            if (m < p.M && n < p.N) store_out(to, p.out_type, p.ld_out, m, n, p.N, v, bias, p.accumulate);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
}

// out = sum over the splits in order, and what store_out does: four columns of a row a thread
__global__ __launch_bounds__(256) void k_f8_join(Product p, const float* __restrict__ part, int64_t ld, int splits, uint32_t quads) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, m = i / quads, n = (i - m * quads) * 4;
    if (m >= p.M) return;
    v4f v = *reinterpret_cast<const v4f*>(part + m * ld + n);
#pragma unroll 4
    for (int z = 1; z < splits; z++) v += *reinterpret_cast<const v4f*>(part + z * p.split_out + m * ld + n);
    store_out(p.out, p.out_type, p.ld_out, m, n, p.N, v, load_bias(p.bias, n, p.N), p.accumulate);
}

// rows of the large tile: half as many where operands in f16 with their sums apart take the registers.  (bf16 operands with their scales inside: widening is what bounds it, and twice the rows use b's tiles twice as
// often: 4096^3 135 -> 114 us, 8192^3 879 -> 770 us.)
constexpr int kernel256_rows(int way) { return way == kWide ? 128 : 256; }
// f32 scales for every row of b and bf16 or f16 results have no large tile: the scales leave registers for 128 x 256 only, which
// is no better than 128 x 128 (4096^3 91.7 and 94.1 us, 2048 x 4096 x 2048 28.8 and 29.6, 4096 x 8192 x 1024 66.9 and 61.7,
// 8192 x 8192 x 2048 204 and 196, 16384 x 4096 x 128 59.9 and 55.7).
constexpr bool has_tiles256(int way, int b_rows) { return !(way == kScaled && b_rows == 1); }

template <class F>
hipError_t with_way(int way, F&& f) {
    switch (way) {
        case kScaled: return f(Int<kScaled>{});
        case kExponents: return f(Int<kExponents>{});
        case kWide: return f(Int<kWide>{});
        default: return f(Int<kWideExponents>{});
    }
}

}  // namespace

namespace {

// Which kernel, and in how many parts of the depth: the least of the times that a product of these sizes is expected to
// take, in us, from what each kernel takes to start and end and for a block of the depth, alone on a compute unit and with
// all of them busy.  The numbers are fits to measured times over 17 to 4096 rows, 512 to 8192 columns and a depth of 512 to
// 8192 (16384 for power-of-two scales and f32 results: 4096^3 133 us in tiles of 128, 102 of 256; 1024 x 1024 x 16384 125, in 8
// parts 44).  With f32 scales and bf16 results: 128 x 4096 x 4096 rows 23.2, tiles of 128 26.1, in 4 parts 19.8; 1024 x 1024 x 4096
// 41.7, 26.3, 24.1 in 4 parts; 4096 x 1024 x 1024 45.8, 12.8, tiles of 256 21.6; 4096^3 -, 87.4, 65.7; 16384 x 4096 x 128
// -, 52, 47; 5125 x 4096 x 315 -, 28.0, 29.2.  Four steps' operands
// in LDS (one workgroup a compute unit, not two) where that holds all tiles: 1024 x 4096 x 4096 34.4 -> 28.9; beyond,
// 2048 x 4096 x 4096, 45.0 -> 53.7; alone they gain nothing (512 x 512 x 8192 45.1, 43.9), nor in f16.  Up to 16 rows the
// wavefronts of the first kernel waste nothing: always that one.
struct Plan { int kernel, splits; int64_t split_blocks; };
enum { kRows = 0, kTiles128 = 1, kTiles256 = 2, kTiles128Deep = 3 };
constexpr double kCus = 256;

Plan make_plan(int64_t M, int64_t N, int64_t K, int way, int b_rows) {
    const bool wide = is_wide(way), inside = way == kWideExponents;
    const int64_t blocks = (K + kF8Block - 1) / kF8Block;
    Plan best{kRows, 1, blocks};
    if (M <= 16) return best;
    const double row_groups = (double)((M + 63) / 64) * ((N + 15) / 16);
    double least = 2.5 + (wide ? 2.6 : 2.3) * ((blocks + kRowsWaves - 1) / kRowsWaves) * ceil(row_groups / kCus);
    for (int kernel = kTiles128; kernel <= (M > 128 && N > 128 && has_tiles256(way, b_rows) ? kTiles256 : kTiles128); kernel++)
        for (int64_t want = 1; want <= 16 && want <= blocks; want *= 2) {
            const int64_t bm = kernel == kTiles256 ? kernel256_rows(way) : 128, bn = kernel == kTiles256 ? 256 : 128;
            const int64_t per = (blocks + want - 1) / want, splits = (blocks + per - 1) / per;
            const double groups = (double)((M + bm - 1) / bm) * ((N + bn - 1) / bn) * splits;
            const bool deep = kernel == kTiles128 && !wide && groups <= kCus && groups > kCus / 4;
            const double busy = fmin(1.0, groups / kCus), rounds = ceil(groups / kCus);
            double start, step;
            if (kernel == kTiles128) start = wide ? 7.0 : 6.0, step = inside ? 0.93 + 0.07 * busy : wide ? 1.05 + 0.1 * busy : deep ? 0.58 + 0.1 * busy : 0.6 + 0.1 * busy;
            else start = inside ? 13.0 : wide ? 9.0 : 12.0, step = inside ? 2.3 + 0.5 * busy : wide ? 1.68 + 0.35 * busy : 1.14 + 0.5 * busy;
            const bool apart = wide && !inside;
            const double again = kernel == kTiles128 ? (apart ? 3.0 : 2.0) : apart ? 7.0 : 9.0;  // a further tile's start and end
            double t = start + step * per * rounds + again * (rounds - 1);
            if (splits > 1) t += 4.0 + 1e-6 * splits * M * N;  // the parts' sums written and read, 8 bytes at 8 TB/s
            if (t < least) {
                least = t;
                best = {deep ? (int)kTiles128Deep : kernel, (int)splits, per};
            }
        }
    return best;
}

// (first kernel, more than 16 rows) two tiles of columns a workgroup
bool rows_in_pairs(int64_t M, int64_t N) { return M > 16 && (double)((M + 63) / 64) * ((N + 31) / 32) >= kCus; }

int64_t split_ld(int64_t N) { return (N + 3) / 4 * 4; }

}  // namespace

size_t matmul_f8_workspace(int64_t M, int64_t N, int64_t K) {
    size_t most = 0;
    // (all plans that there are: only kScaled asks for b's blocks, and with blocks of 128 rows its plans are those of kExponents)
    const struct { int way, b_rows; } kinds[] = {{kScaled, kF8Block}, {kScaled, 1}, {kWide, 1}, {kWideExponents, 1}};
    for (const auto& kind : kinds) {
        const Plan plan = make_plan(M, N, K, kind.way, kind.b_rows);
        const size_t bytes = plan.splits > 1 ? align_up(sizeof(float) * (size_t)plan.splits * M * split_ld(N), 256) : 0;
        if (bytes > most) most = bytes;
    }
    return most;
}

hipError_t launch_f8_matmul(const fmtc_f8& a, const fmtc_f8& b, const float* d_bias, void* d_out, int out_type,
                            int64_t ld_out, int accumulate, void* d_ws, hipStream_t s) {
    Product p{static_cast<const uint8_t*>(a.d_codes), static_cast<const uint8_t*>(b.d_codes), a.d_scales, b.d_scales,
              a.rows, b.rows, (a.depth + kF8Block - 1) / kF8Block, a.ld, b.ld, a.ld_scales, b.ld_scales, ld_out,
              d_bias, d_out, out_type, accumulate, 0, 0};
    const bool exponents = a.scale == FMTC_SCALE_E8M0;
    const int way = out_type == FMTC_F32 ? (exponents ? kWideExponents : kWide) : exponents ? kExponents : kScaled;
    Plan plan = make_plan(p.M, p.N, a.depth, way, b.block_rows);
    if (p.ld_a >= (1 << 23) || p.ld_b >= (1 << 23)) plan = {kRows, 1, p.blocks};  // (a tile's offsets are 32 bits)
    p.split_blocks = plan.split_blocks;
    Product inner = p;
    if (plan.splits > 1) {
        inner.out = d_ws;
        inner.ld_out = split_ld(p.N);
        inner.split_out = p.split_out = p.M * inner.ld_out;
        inner.out_type = FMTC_F32;
        inner.bias = nullptr;
        inner.accumulate = 0;
    }
    hipError_t e = with_bit(a.format, [&](auto fm) {
        return with_way(way, [&](auto wy) {
            return with_bit(b.block_rows == 1, [&](auto one) {
                constexpr int F = decltype(fm)::value, W = decltype(wy)::value, B = decltype(one)::value ? 1 : kF8Block;
                auto tiles = [&](auto tile) {
                    using S = decltype(tile);
                    const int64_t tm = (p.M + S::BM - 1) / S::BM, tn = (p.N + S::BN - 1) / S::BN;
                    auto kernel = k_f8_matmul_tiles<F, W, B, S>;
                    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, S::kLds);
                    return e != hipSuccess ? e : launch(K_F8_MATMUL, kernel, dim3((unsigned)(tm * tn * plan.splits)), dim3(S::kThreads), S::kLds, s, inner, (uint32_t)tm, (uint32_t)tn);
                };
                if constexpr (has_tiles256(W, B))
                    if (plan.kernel == kTiles256) return tiles(Tile<2, 4, kernel256_rows(W) / 32, 2>{});
                if (plan.kernel == kTiles128) return tiles(Tile<2, 2, 4, 2>{});
                if constexpr (!is_wide(W))
                    if (plan.kernel == kTiles128Deep) return tiles(Tile<2, 2, 4, 4>{});
                auto rows = [&](auto mt, auto nt) {
                    constexpr int MT = decltype(mt)::value, NT = decltype(nt)::value;
                    const int64_t n_tiles = (p.N + 16 * NT - 1) / (16 * NT);
                    return launch(K_F8_MATMUL, k_f8_matmul_rows<F, W, B, MT, NT>, dim3((unsigned)(n_tiles * ((p.M + 16 * MT - 1) / (16 * MT)))),
                                  dim3(64 * kRowsWaves), 0, s, p, (uint32_t)n_tiles);
                };
                if (p.M <= 16) return rows(Int<1>{}, Int<1>{});
                return rows_in_pairs(p.M, p.N) ? rows(Int<4>{}, Int<2>{}) : rows(Int<4>{}, Int<1>{});
            });
        });
    });
    if (e != hipSuccess || plan.splits == 1) return e;
    const int64_t quads = (p.N + 3) / 4;
    return launch(K_F8_MATMUL, k_f8_join, dim3((unsigned)((p.M * quads + 255) / 256)), dim3(256), 0, s, p, static_cast<const float*>(d_ws),
                  inner.ld_out, plan.splits, (uint32_t)quads);
}

}  // namespace fmtc
