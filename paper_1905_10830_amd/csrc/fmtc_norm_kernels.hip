// What lies between two blocks (fmtc_block_norm and its gradients): the norm of a block's output, gate and scale, the
// residual sum, the next block's norm and, where wanted, the quantizer of its operand, in one pass over the rows.
//   forward:   u = w_post y r_y,  h' = skip h + scale gate u,  n = w_pre h' r_h,   r_v = 1 / sqrt(mean(v^2) + eps)
//   backward:  a = w_pre dn,  t = dh + r_h (a - hn mean(a hn)),  hn = h' r_h;   dh_in = skip t;
//              b = scale gate w_post t,  dy = r_y (b - yn mean(b yn)),  yn = y r_y;
//              dw_pre = sum dn hn,  dgate = w_post z,  dw_post = sum over gate rows of gate z,  z = sum of scale t yn over
//              the rows that share a gate row
// Memory bound: 3 arrays read and 1 or 2 written (forward), 4 read and 2 written (backward), each once.  TPR lanes hold a
// row in registers, VPT groups of 8 consecutive values each; group g of a lane starts at column 8 (g TPR + lane), so that
// 16 lanes hold a block of 128.  A workgroup walks several rows: the weights stay in registers, and the next row's loads are
// on their way while a row is worked on.  Forward 16384 x 4096 bf16 105 us (5.1 TB/s), to codes 106 us, 8192 x 8192 100 us, 8192 x 2048
// f32 44 us, 4096 x 16384 105 us; backward 16384 x 4096 168 us (4.8 TB/s), 8192 x 4096 with a gate for 1024 rows 95 us, in f32 167 + 5
// us, 200704 x 64 29 + 5 us, 4096 x 16384 537 us; one row of 4096 4 us and 5.2 + 2 us.  Backward, 128 registers do not hold all of a row
// where a lane has two groups (324 to 704 bytes of scratch memory a lane: 3.5 times the traffic's time); 12 to 116 bytes in f32 and
// up to 128 channels show in no time.  (Forward, two groups: 12 to 380 bytes.)
#include "fmtc_block.h"

namespace fmtc {

namespace {

__host__ __device__ inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// f32 sums over the TPR lanes of a row, in a fixed order, through one of two slots in turn: a wavefront that writes a slot
// again has passed the other one's barrier, before which every wavefront had read this one.
template <int TPR, int N>
struct RowSums {
    static constexpr int kWaves = TPR > 64 ? TPR / 64 : 1;
    struct Slot { float v[N][kWaves]; };
    __device__ static void run(float (&v)[N], Slot* slots, int& turn) {
        Slot& slot = slots[turn];
        turn ^= 1;
#pragma unroll
        for (int k = 0; k < N; k++) {
            v[k] = row16_sum(v[k]);
            if constexpr (TPR >= 64) {
                v[k] += __shfl_xor(v[k], 16, 64);
                v[k] += __shfl_xor(v[k], 32, 64);
            }
        }
        if constexpr (TPR > 64) {
            const int wave = threadIdx.x % TPR >> 6;
            if ((threadIdx.x & 63) == 0)
#pragma unroll
                for (int k = 0; k < N; k++) slot.v[k][wave] = v[k];
            __syncthreads();
#pragma unroll
            for (int k = 0; k < N; k++) {  // 16 lanes read the wavefronts' sums and add them up as above
                const int i = threadIdx.x & 15;
                v[k] = row16_sum(kWaves == 16 || i < kWaves ? slot.v[k][i % kWaves] : 0.f);
            }
        }
    }
};

template <class T>
__device__ __forceinline__ const T* at(const void* p, int64_t i) { return static_cast<const T*>(p) + i; }
template <class T>
__device__ __forceinline__ T* at(void* p, int64_t i) { return static_cast<T*>(p) + i; }

template <class W, int TPR, int VPT, bool RAGGED>
__device__ __forceinline__ void load_params(const void* p, int64_t row, int C, int lane, float (&v)[VPT][8]) {
#pragma unroll
    for (int g = 0; g < VPT; g++) {
        const int c = 8 * (g * TPR + lane);
        load8<RAGGED>(at<W>(p, row * C), c, C, v[g]);
    }
}

struct NormOut {
    void *h, *n;
    int64_t ld_h, ld_n;
    fmtc_f8 codes;
    float* stats;
};

// which of a workgroup's rows a thread belongs to: one for all of a wavefront from 64 lanes on, so that addresses are scalar
template <int TPR>
__device__ __forceinline__ int row_in_group() {
    const int r = threadIdx.x / TPR;
    return TPR >= 64 ? __builtin_amdgcn_readfirstlane(r) : r;
}

constexpr int norm_threads(int TPR) { return TPR < 256 ? 256 : TPR; }

template <int FORMAT, int SCALE>
__device__ __forceinline__ void store_codes(const fmtc_f8& q, int64_t row, int c, const float (&v)[8]) {
    uint32_t held;
    const float inv = block_scale<FORMAT, SCALE>(row16_max(finite_amax(v)), &held);
    if (c / kF8Block * (int64_t)kF8Block >= q.depth) return;
    *reinterpret_cast<uint2*>(static_cast<uint8_t*>(q.d_codes) + row * q.ld + c) =
        make_uint2(encode4<FORMAT>(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv),
                   encode4<FORMAT>(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv));
    if (c % kF8Block == 0) store_scale<SCALE>(q.d_scales, c / kF8Block * q.ld_scales + row, held);
}

template <class T, class W, int TPR, int VPT, bool RAGGED>
__global__ __launch_bounds__(norm_threads(TPR)) void k_block_norm(fmtc_norm p, NormOut out) {
    constexpr int kRows = norm_threads(TPR) / TPR;
    using Sum = RowSums<TPR, 1>;
    __shared__ typename Sum::Slot slots[kRows][2];
    const int lane = threadIdx.x % TPR, C = p.C;
    const int mine = row_in_group<TPR>();
    typename Sum::Slot* const slot = slots[mine];
    int turn = 0;
    const float rC = 1.f / (float)C;
    float w_pre[VPT][8], gate[VPT][8];
    int64_t gate_row = -1;
    if (p.d_w_pre) load_params<W, TPR, VPT, RAGGED>(p.d_w_pre, 0, C, lane, w_pre);
    Raw<T> next_h[VPT], next_y[VPT];
    auto fetch = [&](int64_t row) {
#pragma unroll
        for (int g = 0; g < VPT; g++) {
            const int c = 8 * (g * TPR + lane);
            next_h[g].template load<RAGGED>(at<T>(p.d_h, row * p.ld_h), c, C);
            if (p.d_y) next_y[g].template load<RAGGED>(at<T>(p.d_y, row * p.ld_y), c, C);
        }
    };
    // Rows are dealt to the workgroups in turn, so that all of them read one stretch of memory at a time (8192 x 8192, no gate:
    // 110 us with consecutive rows a workgroup, 100 us); where gates change, consecutive rows, which share them (8192 x 4096, a
    // gate for 1024 rows: 64 us in turn, 49 us), and where rows share lines of memory (4000 x 8191: 75 us, 67 us).  The rows of
    // a pass walk together: past the end their lanes work on the last row and store nothing.
    const bool in_turn = !RAGGED && (!p.d_gate || p.rows_per_gate >= p.rows);
    const int64_t passes = ceil_div(ceil_div(p.rows, kRows), (int64_t)gridDim.x);
    const int64_t step = in_turn ? (int64_t)gridDim.x * kRows : kRows;
    int64_t first = (int64_t)blockIdx.x * (in_turn ? 1 : passes) * kRows;
    const int64_t stop = in_turn || first + passes * kRows > p.rows ? p.rows : first + passes * kRows;
    auto row_of = [&](int64_t f) {
        const int64_t row = f + mine;
        return row < p.rows ? row : p.rows - 1;
    };
    if (first < stop) fetch(row_of(first));
    for (; first < stop; first += step) {
        const int64_t row = row_of(first);
        const bool live = first + mine < p.rows;
        if constexpr (RAGGED)
#pragma unroll
            for (int g = 0; g < VPT; g++) {
                next_h[g].settle(8 * (g * TPR + lane), C);
                if (p.d_y) next_y[g].settle(8 * (g * TPR + lane), C);
            }
        float h[VPT][8], y[VPT][8];
#pragma unroll
        for (int g = 0; g < VPT; g++)
#pragma unroll
            for (int i = 0; i < 8; i++) {
                h[g][i] = next_h[g][i];
                y[g][i] = p.d_y ? next_y[g][i] : 0.f;
            }
        if (first + step < stop) fetch(row_of(first + step));
        __builtin_amdgcn_sched_barrier(0);  // (the loads stay here, a row ahead of their use: 125 -> 115 us, 16384 x 4096)
        float r_y = 1.f;
        if (p.d_y) {
            const int64_t want = p.d_gate ? row / p.rows_per_gate : 0;
            if (want != gate_row) {  // scale gate w_post: what the normalised y is multiplied by
                gate_row = want;
                if (p.d_gate) load_params<W, TPR, VPT, RAGGED>(p.d_gate, want, C, lane, gate);
                float w[VPT][8];
                if (p.d_w_post) load_params<W, TPR, VPT, RAGGED>(p.d_w_post, 0, C, lane, w);
#pragma unroll
                for (int g = 0; g < VPT; g++)
#pragma unroll
                    for (int i = 0; i < 8; i++)
                        gate[g][i] = p.scale * (p.d_gate ? gate[g][i] : 1.f) * (p.d_w_post ? w[g][i] : 1.f);
            }
            if (p.d_w_post) {
                float sum[1] = {0.f};
#pragma unroll
                for (int g = 0; g < VPT; g++) {
                    float s = 0.f;
#pragma unroll
                    for (int i = 0; i < 8; i++) s = fmaf(y[g][i], y[g][i], s);
                    if (8 * (g * TPR + lane) < C) sum[0] += s;  // (lanes past the row hold values that are not theirs)
                }
                Sum::run(sum, slot, turn);
                r_y = 1.f / sqrtf(sum[0] * rC + p.eps);
            }
#pragma unroll
            for (int g = 0; g < VPT; g++)
#pragma unroll
                for (int i = 0; i < 8; i++) h[g][i] = fmaf(y[g][i] * r_y, gate[g][i], p.skip * h[g][i]);
        } else {
#pragma unroll
            for (int g = 0; g < VPT; g++)
#pragma unroll
                for (int i = 0; i < 8; i++) h[g][i] *= p.skip;
        }
        if (out.h && live)
#pragma unroll
            for (int g = 0; g < VPT; g++) {
                const int c = 8 * (g * TPR + lane);
                store8(at<T>(out.h, row * out.ld_h + c), C - c, h[g]);
            }
        float r_h = 1.f;
        if (p.d_w_pre) {
            float sum[1] = {0.f};
#pragma unroll
            for (int g = 0; g < VPT; g++) {
                float s = 0.f;
#pragma unroll
                for (int i = 0; i < 8; i++) s = fmaf(h[g][i], h[g][i], s);
                if (8 * (g * TPR + lane) < C) sum[0] += s;
            }
            Sum::run(sum, slot, turn);
            r_h = 1.f / sqrtf(sum[0] * rC + p.eps);
#pragma unroll
            for (int g = 0; g < VPT; g++) {
                const int c = 8 * (g * TPR + lane);
#pragma unroll
                for (int i = 0; i < 8; i++) h[g][i] = h[g][i] * r_h * w_pre[g][i];
                if (!live) continue;
                if (out.n) store8(at<T>(out.n, row * out.ld_n + c), C - c, h[g]);
                if (out.codes.d_codes) {
                    if (c >= C)
#pragma unroll
                        for (int i = 0; i < 8; i++) h[g][i] = 0.f;
                    if (out.codes.format == FMTC_E4M3) {
                        if (out.codes.scale == FMTC_SCALE_F32) store_codes<FMTC_E4M3, FMTC_SCALE_F32>(out.codes, row, c, h[g]);
                        else store_codes<FMTC_E4M3, FMTC_SCALE_E8M0>(out.codes, row, c, h[g]);
                    } else {
                        if (out.codes.scale == FMTC_SCALE_F32) store_codes<FMTC_E5M2, FMTC_SCALE_F32>(out.codes, row, c, h[g]);
                        else store_codes<FMTC_E5M2, FMTC_SCALE_E8M0>(out.codes, row, c, h[g]);
                    }
                }
            }
        }
        if (out.stats && live && lane == 0) {
            out.stats[row] = r_y;
            out.stats[p.rows + row] = r_h;
        }
    }
}

// ---- backward ----
// Rows are cut into strips; TPR lanes walk a strip and keep the sums over its rows in registers, and a workgroup adds up
// those of its strips.  Where a gate row serves more rows than a strip has, its rows are cut into `per_gate` strips of their
// own, whose sums for the gate are added up afterwards; where it serves fewer, a strip holds whole gate rows and writes
// their gradients itself.
struct Strips {
    int64_t count, rows;   // strips; rows of each (the last of a gate row may have fewer)
    int64_t per_gate;      // strips of a gate row, 0: a strip holds whole gate rows (or there is no gate)
    int64_t gates;
};
// Lanes of a row by its width, one group of 8 values each up to 8192: a row in as few lanes as hold it, whole wavefronts from
// 129 values on.
constexpr int lanes_of(int C) { return C <= 128 ? 16 : C <= 512 ? 64 : C <= 1024 ? 128 : C <= 2048 ? 256 : C <= 4096 ? 512 : 1024; }

// A gate row for more rows than there are serves them all; callers may say any such number (the largest one for "all"), with
// which sums of rows would pass 63 bits.
int64_t rows_served(int64_t rows, int64_t rows_per_gate) { return rows_per_gate < rows ? rows_per_gate : rows; }

Strips make_strips(int64_t rows, int C, int64_t rows_per_gate) {
    rows_per_gate = rows_served(rows, rows_per_gate);
    // as many strips as 256 compute units walk at a time with 16 wavefronts each: the sums of a large tensor's strips are a
    // small part of the traffic, and a small tensor has every row on its way at once (500 x 960, a gate for every row: 17.7 us
    // in strips of 4 rows)
    const int64_t want = 256 * 1024 / lanes_of(C), each = ceil_div(rows, want);
    Strips s{};
    if (rows_per_gate <= 0) {
        s.rows = each;
        s.count = ceil_div(rows, each);
        return s;
    }
    s.gates = ceil_div(rows, rows_per_gate);
    if (rows_per_gate <= each) {
        s.rows = each / rows_per_gate * rows_per_gate;
        s.count = ceil_div(rows, s.rows);
    } else {
        s.per_gate = ceil_div(rows_per_gate, each);
        s.rows = ceil_div(rows_per_gate, s.per_gate);
        s.count = s.gates * s.per_gate;
    }
    return s;
}

struct NormGrads {
    const float* stats;
    const void *dn, *dh;
    void *dy, *dh_in;
    int64_t ld_dn, ld_dh, ld_dy, ld_dh_in;
    float *part_post, *part_pre;  // [workgroups][C]
    float* part_gate;             // [strips][C], where a gate row has several strips
    float* dgate;
    Strips strips;
};

template <class T, class W, int TPR, int VPT, bool RAGGED>
__global__ __launch_bounds__(norm_threads(TPR), 4) void k_block_norm_backward(fmtc_norm p, NormGrads q) {
    constexpr int kThreads = norm_threads(TPR), kRows = kThreads / TPR;
    constexpr bool kHold = VPT == 1;  // the weights stay in registers; else they come from the cache for every row
    using Sum = RowSums<TPR, 3>;
    __shared__ typename Sum::Slot slots[kRows][2];
    __shared__ float joined[kRows > 1 ? kThreads * 8 : 1];
    const int lane = threadIdx.x % TPR, C = p.C;
    const int mine = row_in_group<TPR>();
    typename Sum::Slot* const slot = slots[mine];
    int turn = 0;
    const float rC = 1.f / (float)C;
    const int64_t strip = (int64_t)blockIdx.x * kRows + mine;
    int64_t first, end;
    if (q.strips.per_gate) {
        const int64_t g = strip / q.strips.per_gate, j = strip - g * q.strips.per_gate, last = (g + 1) * p.rows_per_gate;
        first = g * p.rows_per_gate + j * q.strips.rows;
        end = first + q.strips.rows < last ? first + q.strips.rows : last;
    } else {
        first = strip * q.strips.rows;
        end = first + q.strips.rows;
    }
    if (end > p.rows) end = p.rows;
    if (strip >= q.strips.count) end = first;  // (nothing; the workgroup's strips walk together)

    float d_post[VPT][8] = {}, d_pre[VPT][8] = {}, z[VPT][8] = {}, w_pre[VPT][8], gain[VPT][8];
    int64_t gate_row = 0;
    auto load_gain = [&] {  // scale gate w_post
#pragma unroll
        for (int g = 0; g < VPT; g++)
#pragma unroll
            for (int i = 0; i < 8; i++) gain[g][i] = p.scale;
        float v[VPT][8];
        if (p.d_gate) {
            load_params<W, TPR, VPT, RAGGED>(p.d_gate, gate_row, C, lane, v);
#pragma unroll
            for (int g = 0; g < VPT; g++)
#pragma unroll
                for (int i = 0; i < 8; i++) gain[g][i] *= v[g][i];
        }
        if (p.d_w_post) {
            load_params<W, TPR, VPT, RAGGED>(p.d_w_post, 0, C, lane, v);
#pragma unroll
            for (int g = 0; g < VPT; g++)
#pragma unroll
                for (int i = 0; i < 8; i++) gain[g][i] *= v[g][i];
        }
    };
    // what the rows that share a gate row added up in z: the gate's gradient, and their part of w_post's
    auto flush = [&](float* to) {
#pragma unroll
        for (int g = 0; g < VPT; g++) {
            const int c = 8 * (g * TPR + lane);
            float gate[8], w_post[8];
#pragma unroll
            for (int i = 0; i < 8; i++) gate[i] = w_post[i] = 1.f;
            if (p.d_gate) load8<RAGGED>(at<W>(p.d_gate, gate_row * C), c, C, gate);
            if (p.d_w_post) load8<RAGGED>(at<W>(p.d_w_post, 0), c, C, w_post);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                d_post[g][i] = fmaf(gate[i], z[g][i], d_post[g][i]);
                w_post[i] *= z[g][i];
                z[g][i] = 0.f;
            }
            if (to) store8(to + c, C - c, w_post);
        }
    };
    Raw<T> next_t[VPT], next_h[VPT], next_n[VPT], next_y[VPT];
    float next_r_y = 1.f, next_r_h = 1.f;
    auto fetch = [&](int64_t row) {
#pragma unroll
        for (int g = 0; g < VPT; g++) {
            const int c = 8 * (g * TPR + lane);
            if (q.dh) next_t[g].template load<RAGGED>(at<T>(q.dh, row * q.ld_dh), c, C);
            if (q.dn) {
                next_h[g].template load<RAGGED>(at<T>(p.d_h, row * p.ld_h), c, C);
                next_n[g].template load<RAGGED>(at<T>(q.dn, row * q.ld_dn), c, C);
            }
            if (p.d_y) next_y[g].template load<RAGGED>(at<T>(p.d_y, row * p.ld_y), c, C);
        }
        if (p.d_w_post) next_r_y = q.stats[row];
        next_r_h = q.stats[p.rows + row];
    };
    if (first < end) fetch(first);
    if (p.d_gate && first < end) gate_row = first / p.rows_per_gate;
    if constexpr (kHold) {
        if (p.d_w_pre) load_params<W, TPR, VPT, RAGGED>(p.d_w_pre, 0, C, lane, w_pre);
        load_gain();
    }
    for (int64_t k = 0; k < q.strips.rows; k++) {
        const int64_t row = first + k;
        const bool live = row < end;
        if (p.d_gate && live && row / p.rows_per_gate != gate_row) {
            gate_row = row / p.rows_per_gate;
            if constexpr (kHold) load_gain();
        }
        if constexpr (!kHold) {
            if (p.d_w_pre) load_params<W, TPR, VPT, RAGGED>(p.d_w_pre, 0, C, lane, w_pre);
            load_gain();
        }
        if constexpr (RAGGED)
#pragma unroll
            for (int g = 0; g < VPT; g++) {
                const int c = 8 * (g * TPR + lane);
                if (q.dh) next_t[g].settle(c, C);
                if (q.dn) next_h[g].settle(c, C), next_n[g].settle(c, C);
                if (p.d_y) next_y[g].settle(c, C);
            }
        const float r_y = next_r_y, r_h = next_r_h;
        float t[VPT][8], hn[VPT][8], y[VPT][8];  // (dh + r_h a, to become the whole gradient; h' and y normalised)
        float sum[3] = {0.f, 0.f, 0.f};          // <a, hn>, <scale gate w_post yn, t>, <scale gate w_post yn, hn>
#pragma unroll
        for (int g = 0; g < VPT; g++) {
            float part[3] = {0.f, 0.f, 0.f};
            const int c0 = 8 * (g * TPR + lane);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                t[g][i] = q.dh && live ? next_t[g][i] : 0.f;
                hn[g][i] = 0.f;
                if (q.dn && live) {
                    hn[g][i] = next_h[g][i] * r_h;
                    const float dn = next_n[g][i], a = dn * w_pre[g][i];
                    d_pre[g][i] = fmaf(dn, hn[g][i], d_pre[g][i]);
                    part[0] = fmaf(a, hn[g][i], part[0]);
                    t[g][i] = fmaf(r_h, a, t[g][i]);
                }
                y[g][i] = 0.f;
                if (p.d_y && live) {
                    y[g][i] = next_y[g][i] * r_y;
                    const float c = gain[g][i] * y[g][i];
                    part[1] = fmaf(c, t[g][i], part[1]);
                    part[2] = fmaf(c, hn[g][i], part[2]);
                }
            }
            if (c0 < C)  // (lanes past the row hold values that are not theirs)
#pragma unroll
                for (int k = 0; k < 3; k++) sum[k] += part[k];
        }
        if (row + 1 < end) fetch(row + 1);
        Sum::run(sum, slot, turn);
        const float mean_h = r_h * sum[0] * rC, mean_y = p.d_w_post ? (sum[1] - mean_h * sum[2]) * rC : 0.f;
        if (!live) continue;
#pragma unroll
        for (int g = 0; g < VPT; g++) {
            const int c = 8 * (g * TPR + lane);
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; i++) {
                t[g][i] = fmaf(-mean_h, hn[g][i], t[g][i]);
                v[i] = p.skip * t[g][i];
            }
            if (q.dh_in) store8(at<T>(q.dh_in, row * q.ld_dh_in + c), C - c, v);
            if (!p.d_y) continue;
#pragma unroll
            for (int i = 0; i < 8; i++) {
                z[g][i] = fmaf(p.scale * t[g][i], y[g][i], z[g][i]);
                v[i] = r_y * fmaf(-mean_y, y[g][i], t[g][i] * gain[g][i]);
            }
            if (q.dy) store8(at<T>(q.dy, row * q.ld_dy + c), C - c, v);
        }
        if (p.d_gate && !q.strips.per_gate && ((row + 1) % p.rows_per_gate == 0 || row + 1 == end))
            flush(q.dgate ? q.dgate + gate_row * C : nullptr);
    }
    if (q.strips.per_gate || !p.d_gate) {
        float* to = nullptr;
        if (q.dgate && q.strips.per_gate && strip < q.strips.count) {
            if (q.strips.per_gate > 1) to = q.part_gate + strip * C;  // (a strip without rows: zeros)
            else to = q.dgate + strip * C;
        }
        flush(to);
    }
    auto join = [&](float (&v)[VPT][8], float* part) {
        if (!part) return;
        float* const to = part + (int64_t)blockIdx.x * C;
        if constexpr (kRows == 1) {
#pragma unroll
            for (int g = 0; g < VPT; g++) {
                const int c = 8 * (g * TPR + lane);
                store8(to + c, C - c, v[g]);
            }
        } else {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 8; i++) joined[threadIdx.x * 8 + i] = v[0][i];
            __syncthreads();
            for (int c = threadIdx.x; c < C; c += kThreads) {
                float sum = joined[c];
#pragma unroll
                for (int r = 1; r < kRows; r++) sum += joined[r * TPR * 8 + c];
                to[c] = sum;
            }
        }
    };
    join(d_post, q.part_post);
    join(d_pre, q.part_pre);
}

// Sums over the strips' parts, in order: blockIdx.y 0 and 1 the weights' (n parts), from 2 on the gate rows' (n_gate parts
// each).  32 columns a workgroup, 32 slices of the parts.
__global__ __launch_bounds__(1024) void k_strip_sums(const float* __restrict__ part_post, const float* __restrict__ part_pre, int64_t n,
                                                     const float* __restrict__ part_gate, int64_t n_gate, int C,
                                                     float* __restrict__ d_post, float* __restrict__ d_pre,
                                                     float* __restrict__ d_gate) {
    __shared__ float slice[32][33];
    const int col = threadIdx.x & 31, k = threadIdx.x >> 5, c = blockIdx.x * 32 + col, which = blockIdx.y;
    const float* from = which == 0 ? part_post : which == 1 ? part_pre : part_gate + (int64_t)(which - 2) * n_gate * C;
    float* to = which == 0 ? d_post : which == 1 ? d_pre : d_gate + (int64_t)(which - 2) * C;
    if (!to) return;
    const int64_t count = which < 2 ? n : n_gate;
    float sum = 0.f;
    if (c < C)
#pragma unroll 4
        for (int64_t i = k; i < count; i += 32) sum += from[i * C + c];
    slice[k][col] = sum;
    __syncthreads();
    sum = slice[col][k];  // (transposed: a wavefront's half has one column's slices)
    sum = row16_sum(sum);
    sum += __shfl_xor(sum, 16, 64);
    if (col == 0 && blockIdx.x * 32 + k < C) to[blockIdx.x * 32 + k] = sum;
}

template <class F>
hipError_t with_width(int C, F&& f) {
    return with_bit(C % 8 != 0, [&](auto ragged) {
        switch (lanes_of(C)) {
            case 16: return f(Int<16>{}, Int<1>{}, ragged);
            case 64: return f(Int<64>{}, Int<1>{}, ragged);
            case 128: return f(Int<128>{}, Int<1>{}, ragged);
            case 256: return f(Int<256>{}, Int<1>{}, ragged);
            case 512: return f(Int<512>{}, Int<1>{}, ragged);
            default: return C <= 8192 ? f(Int<1024>{}, Int<1>{}, ragged) : f(Int<1024>{}, Int<2>{}, ragged);
        }
    });
}
template <class F>
hipError_t with_types(int type, int weight_type, F&& f) {
    return with_type(type, [&](auto ty) {
        using T = typename decltype(ty)::type;
        return weight_type == FMTC_F32 ? f(ty, Type<float>{}) : f(ty, Type<T>{});
    });
}

}  // namespace

hipError_t launch_block_norm(const fmtc_norm& a, void* d_h_out, int64_t ld_h_out, void* d_n, int64_t ld_n,
                             const fmtc_f8* n_codes, float* d_stats, hipStream_t s) {
    NormOut out{d_h_out, d_n, ld_h_out, ld_n, n_codes ? *n_codes : fmtc_f8{}, d_stats};
    return with_types(a.type, a.weight_type, [&](auto ty, auto wt) {
        return with_width(a.C, [&](auto lanes, auto groups, auto ragged) {
            constexpr int TPR = decltype(lanes)::value, VPT = decltype(groups)::value;
            constexpr bool RAGGED = decltype(ragged)::value;
            constexpr int rows = norm_threads(TPR) / TPR;
            int64_t grid = ceil_div(a.rows, rows);
            const int64_t most = 256 * 1024 / norm_threads(TPR);  // what walks at a time: 16 wavefronts a compute unit
            if (grid > most) grid = most;
            return launch(K_BLOCK_NORM, k_block_norm<typename decltype(ty)::type, typename decltype(wt)::type, TPR, VPT, RAGGED>,
                          dim3((unsigned)grid), dim3(norm_threads(TPR)), 0, s, a, out);
        });
    });
}

size_t block_norm_workspace(int64_t rows, int C, int64_t rows_per_gate) {
    const Strips st = make_strips(rows, C, rows_per_gate);
    const int64_t groups = ceil_div(st.count, norm_threads(lanes_of(C)) / lanes_of(C));
    return 2 * align_up(sizeof(float) * (size_t)groups * C, 256) + (st.per_gate > 1 ? align_up(sizeof(float) * (size_t)st.count * C, 256) : 0);
}

hipError_t launch_block_norm_backward(const fmtc_norm& a, const float* d_stats, const void* d_dn, int64_t ld_dn,
                                      const void* d_dh, int64_t ld_dh, void* d_dy, int64_t ld_dy, void* d_dh_in,
                                      int64_t ld_dh_in, float* d_dw_post, float* d_dw_pre, float* d_dgate,
                                      void* d_ws, hipStream_t s) {
    fmtc_norm args = a;
    args.rows_per_gate = a.d_gate ? rows_served(a.rows, a.rows_per_gate) : 0;
    const Strips st = make_strips(a.rows, a.C, args.rows_per_gate);
    const int64_t groups = ceil_div(st.count, norm_threads(lanes_of(a.C)) / lanes_of(a.C));
    const size_t each = align_up(sizeof(float) * (size_t)groups * a.C, 256);
    char* ws = static_cast<char*>(d_ws);
    float *post = reinterpret_cast<float*>(ws), *pre = reinterpret_cast<float*>(ws + each), *gate = reinterpret_cast<float*>(ws + 2 * each);
    NormGrads q{d_stats, d_dn, d_dh, d_dy, d_dh_in, ld_dn, ld_dh, ld_dy, ld_dh_in,
                d_dw_post ? post : nullptr, d_dw_pre ? pre : nullptr, gate, d_dgate, st};
    hipError_t e = with_types(a.type, a.weight_type, [&](auto ty, auto wt) {
        return with_width(a.C, [&](auto lanes, auto per, auto ragged) {
            constexpr int TPR = decltype(lanes)::value, VPT = decltype(per)::value;
            constexpr bool RAGGED = decltype(ragged)::value;
            return launch(K_BLOCK_NORM_BACKWARD, k_block_norm_backward<typename decltype(ty)::type, typename decltype(wt)::type, TPR, VPT, RAGGED>,
                          dim3((unsigned)groups), dim3(norm_threads(TPR)), 0, s, args, q);
        });
    });
    const bool join_gate = d_dgate && st.per_gate > 1;
    if (e != hipSuccess || (!d_dw_post && !d_dw_pre && !join_gate)) return e;
    return launch(K_BLOCK_NORM_BACKWARD, k_strip_sums, dim3((unsigned)ceil_div(a.C, 32), (unsigned)(join_gate ? 2 + st.gates : 2)), dim3(1024), 0, s,
                  post, pre, groups, gate, st.per_gate, (int)a.C, d_dw_post, d_dw_pre, join_gate ? d_dgate : nullptr);
}

}  // namespace fmtc
