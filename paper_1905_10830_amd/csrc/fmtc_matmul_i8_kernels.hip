// Products of 8-bit integer matrices with a scale for each row (fmtc_i8_quantize, fmtc_i8_matmul, fmtc_i8_linear):
//   out[m][n] = (sum_k a[m][k] b[n][k]) sa[m] sb[n] (+ bias[n])
// The sum is exact in 32 bits, whatever its order, so that the depth can be taken by several wavefronts or workgroups
// without a result depending on it.  b's rows are the matrix instruction's first operand and a's its second: a lane then
// holds four consecutive columns n of one row m of the result, and the results leave in vectors.
// Times are the kernels' own, on operands and results that stay where they are.
#include <type_traits>

#include "fmtc_block.h"
#include "fmtc_device.h"

namespace fmtc {

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));

constexpr int kBlock = kF8Block;  // bytes of a row that a step takes; rows are held with zeros up to a multiple of it

// ---- values to codes ----
// TPR lanes hold a row in registers, VPT groups of 8 consecutive values each: one read of the values.  Memory bound: 8192 x 8192
// bf16 39 to 41 us (5.0 TB/s), 4096 x 4096 9.1 us (out of the caches), 3137 x 960 f32 5.1 us.
constexpr int quantize_threads(int TPR) { return TPR < 256 ? 256 : TPR; }
template <class T, int TPR, int VPT, bool RAGGED>
__global__ __launch_bounds__(quantize_threads(TPR)) void k_i8_quantize(const T* __restrict__ x, int64_t rows, int64_t cols, int64_t ld_x, fmtc_i8 out) {
    __shared__ uint32_t part[quantize_threads(TPR) / 64];
    const int64_t row = (int64_t)blockIdx.x * (quantize_threads(TPR) / TPR) + threadIdx.x / TPR, width = (cols + kBlock - 1) / kBlock * kBlock;
    const int lane = threadIdx.x % TPR;
    if (TPR <= 64 && row >= rows) return;  // (whole rows of lanes; wider ones have a workgroup each, and no barrier is passed by)
    const T* const from = x + row * ld_x;
    Raw<T> raw[VPT];
#pragma unroll
    for (int g = 0; g < VPT; g++) raw[g].template load<RAGGED>(from, 8 * (g * TPR + lane), cols);
    uint32_t m = 0;
    float v[VPT][8];
#pragma unroll
    for (int g = 0; g < VPT; g++) {
        const int64_t c = 8 * (g * TPR + lane);
        if constexpr (RAGGED) raw[g].settle(c, cols);
        raw[g].zero_unless(c < cols);
#pragma unroll
        for (int i = 0; i < 8; i++) v[g][i] = raw[g][i];
        const uint32_t b = amax_bits8(v[g]);
        m = b > m ? b : m;
    }
    float held;
    const float inv = i8_row_scale(row_max_bits<TPR>(m, part), &held);
#pragma unroll
    for (int g = 0; g < VPT; g++) {
        const int64_t c = 8 * (g * TPR + lane);
        if (c < width)
            *reinterpret_cast<uint2*>(static_cast<uint8_t*>(out.d_codes) + row * out.ld + c) = make_uint2(i8_encode4(v[g], inv), i8_encode4(v[g] + 4, inv));
    }
    if (lane == 0) out.d_scales[row] = held;
}

// Rows of more than 16384 values: a workgroup reads its row twice, the second time out of the caches.
template <class T>
__global__ __launch_bounds__(1024) void k_i8_quantize_long(const T* __restrict__ x, int64_t cols, int64_t ld_x, fmtc_i8 out) {
    __shared__ uint32_t part[16];
    const int64_t row = blockIdx.x, width = (cols + kBlock - 1) / kBlock * kBlock;
    const T* const from = x + row * ld_x;
    auto load = [&](int64_t c, float (&v)[8]) {
        load8<true>(from, c, cols, v);
        if (c >= cols)
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] = 0.f;
    };
    uint32_t m = 0;
    float v[8];
    for (int64_t c = 8 * threadIdx.x; c < cols; c += 8 * 1024) {
        load(c, v);
        const uint32_t b = amax_bits8(v);
        m = b > m ? b : m;
    }
    float held;
    const float inv = i8_row_scale(row_max_bits<1024>(m, part), &held);
    for (int64_t c = 8 * threadIdx.x; c < width; c += 8 * 1024) {
        load(c, v);
        *reinterpret_cast<uint2*>(static_cast<uint8_t*>(out.d_codes) + row * out.ld + c) = make_uint2(i8_encode4(v, inv), i8_encode4(v + 4, inv));
    }
    if (threadIdx.x == 0) out.d_scales[row] = held;
}

// ---- products ----
struct Product {
    const uint8_t *a, *b;
    const float *sa, *sb, *bias;
    void* out;
    int64_t M, N, blocks, ld_a, ld_b, ld_out;
    int out_type;
    int64_t split_blocks;  // tiles: blocks of the depth that a workgroup takes; the sums of split z go to part + z * split_out
    int64_t split_out, ld_part;
    int* part;
};

// n .. n + 3 of a vector of N, 0 where there is none (columns past the last: the last one's, not stored)
__device__ __forceinline__ v4f load_four(const float* p, int64_t n, int64_t N) {
    v4f v = {};
    if (p)
#pragma unroll
        for (int i = 0; i < 4; i++) v[i] = p[n + i < N ? n + i : N - 1];
    return v;
}

// The factors one after the other: their product alone could leave f32's range.  Each step rounded, as fmtc.h defines it: left to
// itself the compiler fuses the second factor with the bias, and kernels that fused differently would differ in last bits.
__device__ __forceinline__ v4f scaled(v4i sum, float sa, v4f sb, v4f bias) {
#pragma clang fp contract(off)
    v4f v;
#pragma unroll
    for (int i = 0; i < 4; i++) v[i] = (float)sum[i] * sa * sb[i] + bias[i];
    return v;
}
// k of four consecutive results
template <class O>
__device__ __forceinline__ void store_four(O* to, v4f v, int64_t k) {
    O r[4];
#pragma unroll
    for (int i = 0; i < 4; i++) r[i] = from_f32<O>(v[i]);
    if (k >= 4) __builtin_memcpy(to, r, sizeof r);
    else
#pragma unroll
        for (int i = 0; i < 4; i++)
            if (i < k) to[i] = r[i];
}
// f(the outputs as what they are)
template <class F>
__device__ __forceinline__ void with_out(const Product& p, F&& f) {
    if (p.out_type == FMTC_BF16) f(static_cast<bf16*>(p.out));
    else if (p.out_type == FMTC_F16) f(static_cast<_Float16*>(p.out));
    else f(static_cast<float*>(p.out));
}
// out[m][n .. n + 3]
__device__ __forceinline__ void store_out(const Product& p, int64_t m, int64_t n, v4i sum) {
    const v4f v = scaled(sum, p.sa[m], load_four(p.sb, n, p.N), load_four(p.bias, n, p.N));
    with_out(p, [&](auto* out) { store_four(out + m * p.ld_out + n, v, p.N - n); });
}

// 128 bytes of a row for 16 x 16 results: lanes 16 g .. 16 g + 15 hold the bytes 16 g .. and 64 + 16 g .. (the same order of
// the depth in both operands is all that the instruction asks for)
struct Operand { v4i lo, hi; };
__device__ __forceinline__ Operand load_operand(const uint8_t* row_at_block, int g) {
    return {*reinterpret_cast<const v4i*>(row_at_block + 16 * g), *reinterpret_cast<const v4i*>(row_at_block + 64 + 16 * g)};
}
__device__ __forceinline__ v4i mfma_block(const Operand& b, const Operand& a, v4i c) {
    c = __builtin_amdgcn_mfma_i32_16x16x64_i8(b.lo, a.lo, c, 0, 0, 0);
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(b.hi, a.hi, c, 0, 0, 0);
}

// Few rows: 16 MT rows x 16 NT columns per workgroup, operands straight from memory to registers; the workgroup's wavefronts
// take the blocks of the depth in turn and add their sums up in LDS.  Bound by the weights' bytes and the latency of a few
// dependent loads: 64 x 4096 x 4096 12.3 us.
constexpr int kRowsWaves = 8;
template <int MT, int NT>
__global__ __launch_bounds__(64 * kRowsWaves) void k_i8_matmul_rows(Product p, uint32_t n_tiles) {
    __shared__ v4i sums[kRowsWaves][MT * NT][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, i16 = lane & 15;
    const int64_t mt = blockIdx.x / n_tiles, nt = blockIdx.x - mt * n_tiles;
    const uint8_t *a_row[MT], *b_row[NT];  // (rows that do not exist: the last one, never stored)
#pragma unroll
    for (int i = 0; i < MT; i++) {
        const int64_t m = (mt * MT + i) * 16 + i16;
        a_row[i] = p.a + (m < p.M ? m : p.M - 1) * p.ld_a;
    }
#pragma unroll
    for (int j = 0; j < NT; j++) {
        const int64_t n = (nt * NT + j) * 16 + i16;
        b_row[j] = p.b + (n < p.N ? n : p.N - 1) * p.ld_b;
    }
    v4i acc[MT][NT] = {};
    for (int64_t kb = wave; kb < p.blocks; kb += kRowsWaves) {
        Operand b[NT], a[MT];
#pragma unroll
        for (int j = 0; j < NT; j++) b[j] = load_operand(b_row[j] + kb * kBlock, g);
#pragma unroll
        for (int i = 0; i < MT; i++) a[i] = load_operand(a_row[i] + kb * kBlock, g);
        __builtin_amdgcn_sched_barrier(0);  // all loads on their way before the first is waited for
#pragma unroll
        for (int i = 0; i < MT; i++)
#pragma unroll
            for (int j = 0; j < NT; j++) acc[i][j] = mfma_block(b[j], a[i], acc[i][j]);
    }
#pragma unroll
    for (int i = 0; i < MT; i++)
#pragma unroll
        for (int j = 0; j < NT; j++) sums[wave][i * NT + j][lane] = acc[i][j];
    __syncthreads();
    for (int k = wave; k < MT * NT; k += kRowsWaves) {
        v4i v = sums[0][k][lane];
#pragma unroll
        for (int w = 1; w < kRowsWaves; w++) v += sums[w][k][lane];
        const int64_t m = (mt * MT + k / NT) * 16 + i16, n4 = (nt * NT + k % NT) * 16 + g * 4;
        if (m < p.M && n4 < p.N) store_out(p, m, n4, v);
    }
}

// A layer of very few rows in one launch: every workgroup quantizes the rows itself, into LDS, while its first weights are on
// their way.  tpr lanes (whole wavefronts) take a row, up to 4 groups of 8 values each: up to 16384 values in all.  1 x 4096 x 4096
// 6.6 us, of which the weights' bytes are 3.3 (quantizer and product apart 1.8 + 6.5 us and a launch), 8 x 2048 x 4096 6.3 us.
constexpr int kLinearRows = 8, kLinearGroups = 4, kLinearThreads = 64 * kRowsWaves;
constexpr int kLinearCodes = 8 * kLinearGroups * kLinearThreads;  // bytes of codes: of all rows together
bool linear_fits(int64_t M, int64_t K) {
    int64_t lanes = kLinearThreads;
    for (int64_t rows = 1; rows < M; rows *= 2) lanes /= 2;
    return M <= kLinearRows && (K + kBlock - 1) / kBlock * kBlock <= 8 * kLinearGroups * lanes;
}
template <class T, bool RAGGED>
__global__ __launch_bounds__(kLinearThreads) void k_i8_linear_rows(Product p, const T* __restrict__ x, int64_t K, int64_t ld_x, int tpr) {
    __shared__ v4i sums[kRowsWaves][64];
    __shared__ uint32_t part[kRowsWaves];
    __shared__ float scales[kLinearRows];
    __shared__ __attribute__((aligned(16))) uint8_t codes[kLinearCodes + 16 * kLinearRows];  // (rows apart by 16 bytes more: other banks)
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6, g = lane >> 4, i16 = lane & 15;
    const int row = t / tpr, at = t - row * tpr, M = (int)p.M, width = (int)p.blocks * kBlock, pitch = width + 16;
    const int64_t n0 = (int64_t)blockIdx.x * 16, n = n0 + i16;
    const T* const from = x + (row < M ? row : M - 1) * ld_x;
    Raw<T> raw[kLinearGroups];
#pragma unroll
    for (int j = 0; j < kLinearGroups; j++) raw[j].template load<RAGGED>(from, 8 * (j * tpr + at), K);
    // the weights' blocks wave, wave + 8, ..: the first four now (past the last: that one again, not used)
    const uint8_t* const b_row = p.b + (n < p.N ? n : p.N - 1) * p.ld_b;
    const int blocks = (int)p.blocks;
    constexpr int kAhead = 4;
    Operand b[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; i++) {
        const int kb = wave + i * kRowsWaves;
        b[i] = load_operand(b_row + (int64_t)(kb < blocks ? kb : blocks - 1) * kBlock, g);
    }
    __builtin_amdgcn_sched_barrier(0);
    uint32_t m = 0;
    float v[kLinearGroups][8];
#pragma unroll
    for (int j = 0; j < kLinearGroups; j++) {
        const int c = 8 * (j * tpr + at);
        if constexpr (RAGGED) raw[j].settle(c, K);
        raw[j].zero_unless(c < K);
#pragma unroll
        for (int i = 0; i < 8; i++) v[j][i] = raw[j][i];
        const uint32_t bits = amax_bits8(v[j]);
        m = bits > m ? bits : m;
    }
    m = row_max_bits<64>(m, part);
    if (lane == 0) part[wave] = m;
    __syncthreads();
    for (int w = row * (tpr / 64); w < (row + 1) * (tpr / 64); w++) m = part[w] > m ? part[w] : m;
    float held;
    const float inv = i8_row_scale(m, &held);
    if (row < M) {
        if (at == 0) scales[row] = held;
#pragma unroll
        for (int j = 0; j < kLinearGroups; j++) {
            const int c = 8 * (j * tpr + at);
            if (c < width) *reinterpret_cast<uint2*>(codes + row * pitch + c) = make_uint2(i8_encode4(v[j], inv), i8_encode4(v[j] + 4, inv));
        }
    }
    __syncthreads();
    const uint8_t* const a_row = codes + (i16 < M ? i16 : M - 1) * pitch;  // (rows that do not exist: the last one, never stored)
    v4i acc = {};
    for (int kb = wave; kb < blocks; kb += kAhead * kRowsWaves) {
#pragma unroll
        for (int i = 0; i < kAhead; i++) {
            const int k = kb + i * kRowsWaves;
            if (k < blocks) acc = mfma_block(b[i], load_operand(a_row + k * kBlock, g), acc);
            const int next = k + kAhead * kRowsWaves;
            b[i] = load_operand(b_row + (int64_t)(next < blocks ? next : blocks - 1) * kBlock, g);
        }
    }
    sums[wave][lane] = acc;
    __syncthreads();
    if (wave != 0 || i16 >= M) return;
#pragma unroll
    for (int w = 1; w < kRowsWaves; w++) acc += sums[w][lane];
    const int64_t n4 = n0 + g * 4;
    if (n4 >= p.N) return;
    const v4f out = scaled(acc, scales[i16], load_four(p.sb, n4, p.N), load_four(p.bias, n4, p.N));
    with_out(p, [&](auto* to) { store_four(to + i16 * p.ld_out + n4, out, p.N - n4); });
}

// Many rows: a tile of BM x BN results per workgroup, operands through LDS, one block of the depth (128 bytes of a row) a
// step, STAGES steps' operands in LDS.  A wavefront has MT x NT tiles of 16 x 16: b's tiles of a step stay in registers, a's
// come one after the other, each read two tiles before it is multiplied.  The one barrier of a step stands before its last
// two tiles of a, when everything that is still needed of the step is in registers: behind it the next step's operands are
// read and those of the step after it set out into the place that came free, all under the last tiles' products.
//
// Rows of 128 bytes in LDS, the 16-byte pieces of a row exchanged by a key of the row, so that 16 lanes that read the same
// piece of 16 rows touch every bank once.
//
// bf16 results: 4096^3 56 to 58 us (2400 TOPS), 8192^3 445 to 468 us (2350 to 2470), 3137 x 960 x 1000 12.6 us.  The clock falls to 1.95 GHz
// under this load, and the matrix pipes are busy 59 % of it; without the loop's loads 8192^3 takes 340 us, without its LDS reads
// too 318 us.  32 x 32 x 32 instructions with the same tiles: 515 us; one wavefront a SIMD with 128 x 128 results each: 521 us.
template <int WM_, int WN_, int MT_, int NT_, int STAGES_>
struct Tile {
    static constexpr int WM = WM_, WN = WN_, MT = MT_, NT = NT_, kStages = STAGES_;
    static constexpr int kThreads = 64 * WM * WN, BM = WM * MT * 16, BN = WN * NT * 16;
    static constexpr int kStage = (BM + BN) * kBlock;
    static constexpr int kLoads = (BM + BN) / 8 / (WM * WN);  // loads of 8 rows a wavefront, a's and b's in one range
    static constexpr int kLds = kStages * kStage + 4 * (BM + 2 * BN);  // the operands, the scales and the bias
    static_assert((BM + BN) % (8 * WM * WN) == 0 && kLoads % 2 == 0 && BM % 64 == 0 && MT % 4 == 0 && NT % 4 == 0);
    static_assert((kStages & (kStages - 1)) == 0 && kStages >= 2);
    static_assert(WM * WN * MT * 16 * 128 <= kStages * kStage);  // results on their way out
};
__device__ __forceinline__ int row_key(int row) { return (row >> 1) & 7; }

// 16 bytes a lane from base + off straight into LDS, lane l to lds_base + 16 l; the caller counts its loads in flight
__device__ __forceinline__ void load16_to_lds(const void* base, uint32_t off, uint32_t lds_base) {
    uint32_t keep;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2\n\ts_mov_b32 m0, %0"
                 : "=&s"(keep) : "v"(off), "s"(base), "s"(lds_base) : "memory");
}

template <class S>
__global__ __launch_bounds__(S::kThreads, 2) void k_i8_matmul_tiles(Product p, uint32_t tiles_m, uint32_t tiles_n) {
    extern __shared__ __attribute__((aligned(128))) uint8_t lds[];
    constexpr int MT = S::MT, NT = S::NT, kStages = S::kStages;
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
    const uint8_t *from_a = p.a + m0 * p.ld_a + kb0 * kBlock, *from_b = p.b + n0 * p.ld_b + kb0 * kBlock;
    uint32_t off[S::kLoads];
#pragma unroll
    for (int i = 0; i < S::kLoads; i++) {
        const int row = (wave * S::kLoads + i) * 8 + (lane >> 3);
        const bool of_a = row < S::BM;
        const int r = of_a ? (row < rows_a ? row : rows_a - 1) : (row - S::BM < rows_b ? row - S::BM : rows_b - 1);
        off[i] = (uint32_t)r * (uint32_t)(of_a ? p.ld_a : p.ld_b) + 16 * ((lane & 7) ^ row_key(row));
    }
    const uint32_t lds_at = (uint32_t)(uintptr_t)(lds_void_t*)lds;
    // A quarter of a step's loads at a time: all at once, the queue of loads is full and the wavefront stands still.  Past the
    // last block: that one again, into a place that is free; not used, and no branch in the loop.
    const int64_t last = blocks - 1;
    auto fetch = [&](int64_t kb, int quarter) {
        const uint32_t stage = (uint32_t)kb & (kStages - 1), to = lds_at + stage * S::kStage + wave * S::kLoads * 1024;
        if (kb > last) kb = last;
#pragma unroll
        for (int i = quarter * S::kLoads / 4; i < (quarter + 1) * S::kLoads / 4; i++)
            load16_to_lds(((wave * S::kLoads + i) * 8 < S::BM ? from_a : from_b) + kb * kBlock, off[i], to + i * 1024);
    };

    const int row_a = wm * MT * 16 + i16, row_b = S::BM + wn * NT * 16 + i16, key = row_key(i16);  // (the key of row + 16 i, too)
    auto piece = [&](int64_t kb, int row) {
        const uint8_t* at = lds + ((uint32_t)kb & (kStages - 1)) * S::kStage + row * kBlock;
        return Operand{*reinterpret_cast<const v4i*>(at + 16 * (g ^ key)), *reinterpret_cast<const v4i*>(at + 16 * ((4 + g) ^ key))};
    };

    // scales and bias in LDS for the end (those past the last: the last one's, not stored)
    float* const vectors = reinterpret_cast<float*>(lds + kStages * S::kStage);
    if (!p.part) {
        for (int i = t; i < S::BM; i += S::kThreads) vectors[i] = p.sa[m0 + (i < rows_a ? i : rows_a - 1)];
        for (int i = t; i < S::BN; i += S::kThreads) {
            const int64_t n = n0 + (i < rows_b ? i : rows_b - 1);
            vectors[S::BM + i] = p.sb[n];
            vectors[S::BM + S::BN + i] = p.bias ? p.bias[n] : 0.f;
        }
    }

    v4i acc[MT][NT] = {};
    // all blocks' loads that fit, and the first half of those of the last place's; the rest of them in the first step
#pragma unroll
    for (int k = 0; k < kStages; k++)
#pragma unroll
        for (int q = 0; q < (k == kStages - 1 ? 2 : 4); q++) fetch(k, q);
    wait_loads<(kStages - 2) * S::kLoads + S::kLoads / 2>();
    __syncthreads();
    Operand b[NT], a[3];  // tiles i, i + 1 and i + 2: a tile's read has two tiles' products to arrive under
    a[0] = piece(0, row_a);
    a[1] = piece(0, row_a + 16);
#pragma unroll
    for (int j = 0; j < NT; j++) b[j] = piece(0, row_b + 16 * j);

    for (int64_t kb = 0; kb < blocks; kb++) {
#pragma unroll
        for (int i = 0; i < MT; i++) {
            if (i == MT - 2) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the last tiles of a are in registers
                wait_loads<(kStages - 2) * S::kLoads>();            // the next step's operands (this wavefront's) are in LDS
                __syncthreads();
            }
            if (i >= MT - 2) fetch(kb + kStages, i - (MT - 2));
            if (i < 2) fetch(kb + kStages - 1, i + 2);
            // (past the last step: what LDS holds, not used)
            a[2] = i < MT - 2 ? piece(kb, row_a + 16 * (i + 2)) : piece(kb + 1, row_a + 16 * (i + 2 - MT));
#pragma unroll
            for (int j = 0; j < NT; j++) {
                acc[i][j] = mfma_block(b[j], a[0], acc[i][j]);
                if (i == MT - 1) b[j] = piece(kb + 1, row_b + 16 * j);
            }
            a[0] = a[1], a[1] = a[2];
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    // The results leave through LDS, 128 bytes of each of a wavefront's rows at a time, as what they are in memory: then 8 lanes
    // write a line.  (4096^2 results of 2 bytes: 8.6 us, a fill of such an array 7.2; 8 bytes a lane from sums in LDS 13; straight from
    // the registers, 32 bytes of a row at a time, 24.)
    wait_loads<0>();
    __syncthreads();
    uint8_t* const mine = lds + wave * MT * 16 * 128;
    const float *const sa = vectors + wm * MT * 16 + i16, *const sb = vectors + S::BM + wn * NT * 16 + 4 * g, *const bias = sb + S::BN;
    auto leave = [&](auto* out, int64_t ld, auto&& value) {
        using O = typename std::remove_pointer<decltype(out)>::type;
        constexpr int kCols = 128 / sizeof(O), kTiles = kCols / 16, kPiece = 16 / sizeof(O);
        O* const to = out + (m0 + wm * MT * 16 + (lane >> 3)) * ld + n0 + wn * NT * 16 + (lane & 7) * kPiece;
        const int row = wm * MT * 16 + (lane >> 3), col = wn * NT * 16 + (lane & 7) * kPiece;
#pragma unroll
        for (int j0 = 0; j0 < NT; j0 += kTiles) {
#pragma unroll
            for (int j = 0; j < kTiles; j++)
#pragma unroll
                for (int i = 0; i < MT; i++) {
                    O r[4];
                    value(i, j0 + j, r);
                    const int at = (16 * j + 4 * g) * (int)sizeof(O);
                    __builtin_memcpy(mine + (16 * i + i16) * 128 + ((at / 16 ^ key) * 16 | at % 16), r, sizeof r);
                }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            const int left = rows_b - col - j0 * 16;
#pragma unroll
            for (int r = 0; r < MT * 16; r += 8) {
                const int at = r + (lane >> 3);
                const v4i v = *reinterpret_cast<const v4i*>(mine + at * 128 + 16 * ((lane & 7) ^ row_key(at)));
                if (row + r < rows_a) {
                    O* const here = to + r * ld + j0 * 16;
                    if (left >= kPiece) {
                        __builtin_memcpy(here, &v, 16);
                    } else {
                        O one[kPiece];
                        __builtin_memcpy(one, &v, 16);
#pragma unroll
                        for (int k = 0; k < kPiece; k++)
                            if (k < left) here[k] = one[k];
                    }
                }
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        }
    };
    if (p.part) {
        leave(p.part + z * p.split_out, p.ld_part, [&](int i, int j, int (&r)[4]) {
#pragma unroll
            for (int k = 0; k < 4; k++) r[k] = acc[i][j][k];
        });
        return;
    }
    with_out(p, [&](auto* out) {
        using O = typename std::remove_pointer<decltype(out)>::type;
        leave(out, p.ld_out, [&](int i, int j, O (&r)[4]) {
            const v4f v = scaled(acc[i][j], sa[16 * i], *reinterpret_cast<const v4f*>(sb + 16 * j), *reinterpret_cast<const v4f*>(bias + 16 * j));
#pragma unroll
            for (int k = 0; k < 4; k++) r[k] = from_f32<O>(v[k]);
        });
    });
}

// out from the sums of the splits: four columns of a row a thread
__global__ __launch_bounds__(256) void k_i8_join(Product p, int splits, uint32_t quads) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, m = i / quads, n = (i - m * quads) * 4;
    if (m >= p.M) return;
    v4i v = *reinterpret_cast<const v4i*>(p.part + m * p.ld_part + n);
#pragma unroll 4
    for (int z = 1; z < splits; z++) v += *reinterpret_cast<const v4i*>(p.part + z * p.split_out + m * p.ld_part + n);
    store_out(p, m, n, v);
}

// Which kernel, and in how many parts of the depth: the least of the times that a product of these sizes is expected to take,
// in us: fits to 22 sizes of 32 to 16384 rows, 512 to 8192 columns and a depth of 128 to 8192.  bf16 results, in us, few
// rows / 128 x 128 / 128 x 128 with four steps in LDS / 256 x 256: 64 x 8192 x 2048 12.7 / 15.4 / 11.7 / -; 1024 x 1024 x 1024
// 12.5 / 8.9 / 8.5 / 15.3; 1024 x 4096 x 4096 146 / 28.6 / 23.4 / 42.6; 2048 x 4096 x 2048 - / 23.1 / 26.8 / 28.7; 4096 x 8192 x 2048
// - / 85.6 / 102 / 68.4; 16384 x 4096 x 128 - / 51.6 / 77.2 / 47.7.  In parts: 64 x 1024 x 8192 128 x 128 46.6, in 8 parts 13.1; 128 x
// 4096 x 4096 18.7, in 2 parts 15.5.  Four steps' operands in LDS leave room for one workgroup a compute unit, not two: only where
// there are no more.  Up to 16 rows the wavefronts of the first kernel waste nothing: always that one.
struct Plan { int kernel, splits; int64_t split_blocks; };
enum { kRows = 0, kTiles128 = 1, kTiles256 = 2, kTiles128Deep = 3 };
constexpr double kCus = 256;

Plan choose(int64_t M, int64_t N, int64_t K) {
    const int64_t blocks = (K + kBlock - 1) / kBlock;
    Plan best{kRows, 1, blocks};
    if (M <= 16) return best;
    const double row_groups = (double)((M + 63) / 64) * ((N + 15) / 16);
    double least = 2.5 + 2.3 * ((blocks + kRowsWaves - 1) / kRowsWaves) * ceil(row_groups / kCus);
    for (int kernel = kTiles128; kernel <= kTiles256; kernel++)
        for (int64_t want = 1; want <= 16 && want <= blocks; want *= 2) {
            const int64_t side = kernel == kTiles256 ? 256 : 128;
            const int64_t per = (blocks + want - 1) / want, splits = (blocks + per - 1) / per;
            const double groups = (double)((M + side - 1) / side) * ((N + side - 1) / side) * splits;
            const bool deep = kernel == kTiles128 && groups <= kCus;
            const double busy = fmin(1.0, groups / kCus), rounds = ceil(groups / (kernel == kTiles128 ? 2 * kCus : kCus));
            double t;
            if (deep) t = 5.6 + (0.41 + 0.14 * busy) * per;
            else if (kernel == kTiles128) t = 5.4 + 1.05 * per * rounds + 5.0 * (rounds - 1);
            else t = 7.5 + 4.0 * busy + (1.07 + 0.4 * busy) * per * rounds + 6.0 * (rounds - 1);
            if (splits > 1) t += 3.0 + 1.3e-6 * splits * M * N;
            if (t < least) {
                least = t;
                best = {deep ? (int)kTiles128Deep : kernel, (int)splits, per};
            }
        }
    return best;
}

// A call asks three times for the same sizes (for its workspace, for the check of it, for the launch).
Plan make_plan(int64_t M, int64_t N, int64_t K) {
    struct Last { int64_t M, N, K; Plan plan; };
    static thread_local Last last{};
    if (last.M != M || last.N != N || last.K != K) last = {M, N, K, choose(M, N, K)};
    return last.plan;
}

int64_t split_ld(int64_t N) { return (N + 3) / 4 * 4; }

// A grid has less than 2^32 threads: f(first, how many) for ranges of n things that take `threads` each
template <class F>
hipError_t in_launches(int64_t n, int64_t threads, F&& f) {
    const int64_t most = (((int64_t)1 << 32) - 1) / threads;
    if (most == 0) return hipErrorInvalidConfiguration;
    hipError_t e = hipSuccess;
    for (int64_t at = 0; at < n && e == hipSuccess; at += most) e = f(at, n - at < most ? n - at : most);
    return e;
}
// the product with 16 `tiles` columns from the tile `at` on
Product columns_of(Product p, int64_t at, int64_t tiles) {
    const int64_t n = 16 * at;
    p.b += n * p.ld_b;
    p.sb += n;
    if (p.bias) p.bias += n;
    p.out = static_cast<char*>(p.out) + n * (p.out_type == FMTC_F32 ? 4 : 2);
    p.N = p.N - n < 16 * tiles ? p.N - n : 16 * tiles;
    return p;
}

}  // namespace

size_t matmul_i8_workspace(int64_t M, int64_t N, int64_t K) {
    const Plan plan = make_plan(M, N, K);
    return plan.splits > 1 ? align_up(sizeof(int) * (size_t)plan.splits * M * split_ld(N), 256) : 0;
}

hipError_t launch_i8_matmul(const fmtc_i8& a, const fmtc_i8& b, const float* d_bias, void* d_out, int out_type, int64_t ld_out,
                            void* d_ws, hipStream_t s) {
    Plan plan = make_plan(a.rows, b.rows, a.depth);
    Product p{static_cast<const uint8_t*>(a.d_codes), static_cast<const uint8_t*>(b.d_codes), a.d_scales, b.d_scales, d_bias, d_out,
              a.rows, b.rows, (a.depth + kBlock - 1) / kBlock, a.ld, b.ld, ld_out, out_type, 0, 0, 0, nullptr};
    if (p.ld_a >= (1 << 23) || p.ld_b >= (1 << 23)) plan = {kRows, 1, p.blocks};  // (a tile's offsets are 32 bits)
    p.split_blocks = plan.split_blocks;
    if (plan.splits > 1) {
        p.part = static_cast<int*>(d_ws);
        p.ld_part = split_ld(p.N);
        p.split_out = p.M * p.ld_part;
    }
    auto tiles = [&](auto tile) {
        using S = decltype(tile);
        const int64_t tm = (p.M + S::BM - 1) / S::BM, tn = (p.N + S::BN - 1) / S::BN;
        auto kernel = k_i8_matmul_tiles<S>;
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, S::kLds);
        return e != hipSuccess ? e : launch(K_I8_MATMUL, kernel, dim3((unsigned)(tm * tn * plan.splits)), dim3(S::kThreads), S::kLds, s, p, (uint32_t)tm, (uint32_t)tn);
    };
    auto rows = [&](auto mt) {
        constexpr int MT = decltype(mt)::value;
        const int64_t row_tiles = (p.M + 16 * MT - 1) / (16 * MT);
        return in_launches((p.N + 15) / 16, row_tiles * 64 * kRowsWaves, [&](int64_t at, int64_t n_tiles) {
            return launch(K_I8_MATMUL, k_i8_matmul_rows<MT, 1>, dim3((unsigned)(n_tiles * row_tiles)), dim3(64 * kRowsWaves), 0, s,
                          columns_of(p, at, n_tiles), (uint32_t)n_tiles);
        });
    };
    hipError_t e;
    if (plan.kernel == kTiles256) e = tiles(Tile<2, 4, 8, 4, 2>{});
    else if (plan.kernel == kTiles128) e = tiles(Tile<2, 2, 4, 4, 2>{});
    else if (plan.kernel == kTiles128Deep) e = tiles(Tile<2, 2, 4, 4, 4>{});
    else e = p.M <= 16 ? rows(Int<1>{}) : rows(Int<4>{});
    if (e != hipSuccess || plan.splits == 1) return e;
    const int64_t quads = (p.N + 3) / 4;
    return launch(K_I8_MATMUL, k_i8_join, dim3((unsigned)((p.M * quads + 255) / 256)), dim3(256), 0, s, p, plan.splits, (uint32_t)quads);
}

bool i8_linear_is_one(int64_t M, int64_t K) { return linear_fits(M, K); }
hipError_t launch_i8_linear_one(const void* d_x, int type, int64_t rows, int64_t ld_x, const fmtc_i8& w, const float* d_bias, void* d_out,
                                int out_type, int64_t ld_out, hipStream_t s) {
    Product p{nullptr, static_cast<const uint8_t*>(w.d_codes), nullptr, w.d_scales, d_bias, d_out, rows, w.rows,
              (w.depth + kBlock - 1) / kBlock, 0, w.ld, ld_out, out_type, 0, 0, 0, nullptr};
    int tpr = kLinearThreads;
    for (int64_t r = 1; r < rows; r *= 2) tpr /= 2;
    return with_type(type, [&](auto ty) {
        using T = typename decltype(ty)::type;
        return with_bit(w.depth % 8 != 0, [&](auto rg) {
            return in_launches((p.N + 15) / 16, kLinearThreads, [&](int64_t at, int64_t n_tiles) {
                return launch(K_I8_MATMUL, k_i8_linear_rows<T, decltype(rg)::value>, dim3((unsigned)n_tiles), dim3(kLinearThreads), 0, s,
                              columns_of(p, at, n_tiles), static_cast<const T*>(d_x), w.depth, ld_x, tpr);
            });
        });
    });
}

static hipError_t quantize_rows(const void* d_x, int type, int64_t rows, int64_t cols, int64_t ld_x, const fmtc_i8& out, hipStream_t s) {
    return with_type(type, [&](auto ty) {
        using T = typename decltype(ty)::type;
        const T* x = static_cast<const T*>(d_x);
        if (cols > 16384) return launch(K_I8_QUANTIZE, k_i8_quantize_long<T>, dim3((unsigned)rows), dim3(1024), 0, s, x, cols, ld_x, out);
        return with_bit(cols % 8 != 0, [&](auto rg) {
            constexpr bool R = decltype(rg)::value;
            auto go = [&](auto tpr, auto vpt) {
                constexpr int TPR = decltype(tpr)::value, kRows = quantize_threads(TPR) / TPR;
                return launch(K_I8_QUANTIZE, k_i8_quantize<T, TPR, decltype(vpt)::value, R>, dim3((unsigned)((rows + kRows - 1) / kRows)),
                              dim3(quantize_threads(TPR)), 0, s, x, rows, cols, ld_x, out);
            };
            // (the zeros behind a row are written by its lanes: they have to reach a multiple of 128)
            if (cols <= 128) return go(Int<16>{}, Int<1>{});
            if (cols <= 512) return go(Int<64>{}, Int<1>{});
            if (cols <= 1024) return go(Int<64>{}, Int<2>{});
            if (cols <= 2048) return go(Int<256>{}, Int<1>{});
            if (cols <= 4096) return go(Int<256>{}, Int<2>{});
            if (cols <= 8192) return go(Int<1024>{}, Int<1>{});
            return go(Int<1024>{}, Int<2>{});
        });
    });
}

hipError_t launch_i8_quantize(const void* d_x, int type, int64_t rows, int64_t cols, int64_t ld_x, const fmtc_i8& out, hipStream_t s) {
    return in_launches(rows, 1024, [&](int64_t at, int64_t n) {
        fmtc_i8 some = out;
        some.d_codes = static_cast<uint8_t*>(out.d_codes) + at * out.ld;
        some.d_scales = out.d_scales + at;
        return quantize_rows(static_cast<const char*>(d_x) + at * ld_x * (type == FMTC_F32 ? 4 : 2), type, n, cols, ld_x, some, s);
    });
}

}  // namespace fmtc
