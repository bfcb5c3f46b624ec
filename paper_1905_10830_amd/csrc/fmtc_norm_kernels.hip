// What lies between two blocks (fmtc_block_norm and its gradients): the norm of a block's output, gate and scale, the
// residual sum, the next block's norm and, where wanted, the quantizer of its operand, in one pass over the rows.
//   forward:   u = w_post y r_y,  h' = skip h + scale gate u,  n = w_pre h' r_h,   r_v = 1 / sqrt(mean(v^2) + eps)
//   backward:  a = w_pre dn,  t = dh + r_h (a - hn mean(a hn)),  hn = h' r_h;   dh_in = skip t;
//              b = scale gate w_post t,  dy = r_y (b - yn mean(b yn)),  yn = y r_y;
//              dw_pre = sum dn hn,  dgate = w_post z,  dw_post = sum over gate rows of gate z,  z = sum of scale t yn over
//              the rows that share a gate row
// Memory bound: 3 arrays read and 1 or 2 written (forward), 4 read and 2 written (backward), each once.  TPR lanes hold a
// row in registers, VPT groups of 8 consecutive values each; group g of a lane starts at column 8 (g TPR + lane), so that
// 16 lanes hold a block of 128.
#include "fmtc_block.h"

namespace fmtc {

namespace {

template <int TPR>
struct RowSum {  // f32 sum over the TPR lanes of a row, in a fixed order
    static constexpr int kSlots = TPR > 64 ? TPR / 64 : 1;
    __device__ static float run(float v, float (*slot)[kSlots]) {
        v = row16_sum(v);
        if constexpr (TPR >= 64) {
            v += __shfl_xor(v, 16, 64);
            v += __shfl_xor(v, 32, 64);
        }
        if constexpr (TPR > 64) {
            if ((threadIdx.x & 63) == 0) (*slot)[threadIdx.x >> 6] = v;
            __syncthreads();
            v = 0.f;
#pragma unroll
            for (int i = 0; i < kSlots; i++) v += (*slot)[i];
        }
        return v;
    }
};

template <class T>
__device__ __forceinline__ const T* at(const void* p, int64_t i) { return static_cast<const T*>(p) + i; }
template <class T>
__device__ __forceinline__ T* at(void* p, int64_t i) { return static_cast<T*>(p) + i; }

template <class W, int TPR, int VPT>
__device__ __forceinline__ void load_params(const void* p, int64_t row, int C, int lane, float (&v)[VPT][8]) {
#pragma unroll
    for (int g = 0; g < VPT; g++) {
        const int c = 8 * (g * TPR + lane);
        load8(at<W>(p, row * C + c), C - c, v[g]);
    }
}

struct NormOut {
    void *h, *n;
    int64_t ld_h, ld_n;
    fmtc_f8 codes;
    float* stats;
};

constexpr int norm_threads(int TPR) { return TPR < 256 ? 256 : TPR; }

template <int FORMAT, int SCALE>
__device__ __forceinline__ void store_codes(const fmtc_f8& q, int64_t row, int c, const float (&v)[8]) {
    float amax = 0.f;
#pragma unroll
    for (int i = 0; i < 8; i++) amax = fmaxf(amax, finite_abs(v[i]));
    uint32_t held;
    const float inv = block_scale<FORMAT, SCALE>(row16_max(amax), &held);
    if (c / kF8Block * (int64_t)kF8Block >= q.depth) return;
    *reinterpret_cast<uint2*>(static_cast<uint8_t*>(q.d_codes) + row * q.ld + c) =
        make_uint2(encode4<FORMAT>(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv),
                   encode4<FORMAT>(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv));
    if (c % kF8Block == 0) store_scale<SCALE>(q.d_scales, c / kF8Block * q.ld_scales + row, held);
}

template <class T, class W, int TPR, int VPT>
__global__ __launch_bounds__(norm_threads(TPR)) void k_block_norm(fmtc_norm p, NormOut out) {
    __shared__ float slots[2][RowSum<TPR>::kSlots];
    constexpr int kRows = norm_threads(TPR) / TPR;
    const int lane = threadIdx.x % TPR, C = p.C;
    const float rC = 1.f / (float)C;
    float w_pre[VPT][8], gate[VPT][8];
    int64_t gate_row = -1;
    if (p.d_w_pre) load_params<W, TPR, VPT>(p.d_w_pre, 0, C, lane, w_pre);
    for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR; row < p.rows; row += (int64_t)gridDim.x * kRows) {
        float h[VPT][8], y[VPT][8];
#pragma unroll
        for (int g = 0; g < VPT; g++) {
            const int c = 8 * (g * TPR + lane);
            load8(at<T>(p.d_h, row * p.ld_h + c), C - c, h[g]);
            if (p.d_y) load8(at<T>(p.d_y, row * p.ld_y + c), C - c, y[g]);
        }
        float r_y = 1.f;
        if (p.d_y) {
            const int64_t want = p.d_gate ? row / p.rows_per_gate : 0;
            if (want != gate_row) {  // scale gate w_post: what the normalised y is multiplied by
                gate_row = want;
                if (p.d_gate) load_params<W, TPR, VPT>(p.d_gate, want, C, lane, gate);
                float w[VPT][8];
                if (p.d_w_post) load_params<W, TPR, VPT>(p.d_w_post, 0, C, lane, w);
#pragma unroll
                for (int g = 0; g < VPT; g++)
#pragma unroll
                    for (int i = 0; i < 8; i++)
                        gate[g][i] = p.scale * (p.d_gate ? gate[g][i] : 1.f) * (p.d_w_post ? w[g][i] : 1.f);
            }
            if (p.d_w_post) {
                float sum = 0.f;
#pragma unroll
                for (int g = 0; g < VPT; g++)
#pragma unroll
                    for (int i = 0; i < 8; i++) sum = fmaf(y[g][i], y[g][i], sum);
                r_y = 1.f / sqrtf(RowSum<TPR>::run(sum, &slots[0]) * rC + p.eps);
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
        if (out.h)
#pragma unroll
            for (int g = 0; g < VPT; g++) {
                const int c = 8 * (g * TPR + lane);
                store8(at<T>(out.h, row * out.ld_h + c), C - c, h[g]);
            }
        float r_h = 1.f;
        if (p.d_w_pre) {
            float sum = 0.f;
#pragma unroll
            for (int g = 0; g < VPT; g++)
#pragma unroll
                for (int i = 0; i < 8; i++) sum = fmaf(h[g][i], h[g][i], sum);
            r_h = 1.f / sqrtf(RowSum<TPR>::run(sum, &slots[1]) * rC + p.eps);
#pragma unroll
            for (int g = 0; g < VPT; g++) {
                const int c = 8 * (g * TPR + lane);
#pragma unroll
                for (int i = 0; i < 8; i++) h[g][i] = h[g][i] * r_h * w_pre[g][i];
                if (out.n) store8(at<T>(out.n, row * out.ld_n + c), C - c, h[g]);
                if (out.codes.d_codes) {
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
        if (out.stats && lane == 0) {
            out.stats[row] = r_y;
            out.stats[p.rows + row] = r_h;
        }
    }
}

// ---- backward ----
// Rows are cut into strips; TPR lanes walk a strip and keep the sums over its rows in registers.  Where a gate row serves at
// least a strip's number of rows, its rows are cut into `per_gate` strips of their own and the strips' sums are added up
// by k_strip_sums; where it serves fewer, a strip holds whole gate rows and writes their gradients itself.
struct Strips {
    int64_t count, rows;   // strips; rows of each (the last of a gate row may have fewer)
    int64_t per_gate;      // strips of a gate row, 0: a strip holds whole gate rows (or there is no gate)
    int64_t gates;
};
__host__ __device__ inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

Strips make_strips(int64_t rows, int C, int64_t rows_per_gate) {
    // 1024 strips of wide rows, more of narrow ones (which have fewer lanes each): enough to fill the device, while the
    // strips' sums stay a small part of the traffic
    const int64_t want = C > 512 ? 1024 : C > 128 ? 4096 : 8192;
    Strips s{};
    int64_t each = ceil_div(rows, want);
    if (each < 4) each = 4;
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
        const int64_t span = rows_per_gate < rows ? rows_per_gate : rows;
        s.per_gate = ceil_div(span, each);
        s.rows = ceil_div(span, s.per_gate);
        s.count = s.gates * s.per_gate;
    }
    return s;
}

struct NormGrads {
    const float* stats;
    const void *dn, *dh;
    void *dy, *dh_in;
    int64_t ld_dn, ld_dh, ld_dy, ld_dh_in;
    float *part_post, *part_pre, *part_gate;  // [strips][C] each (gate: where a gate row has several strips)
    float* dgate;
    Strips strips;
};

template <class T, class W, int TPR, int VPT>
__global__ __launch_bounds__(norm_threads(TPR)) void k_block_norm_backward(fmtc_norm p, NormGrads q) {
    __shared__ float slots[2][RowSum<TPR>::kSlots];
    constexpr int kRows = norm_threads(TPR) / TPR;
    const int lane = threadIdx.x % TPR, C = p.C;
    const float rC = 1.f / (float)C;
    const int64_t strip = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR;
    if (strip >= q.strips.count) return;  // (all lanes of a row)
    int64_t row, end;
    if (q.strips.per_gate) {
        const int64_t g = strip / q.strips.per_gate, j = strip - g * q.strips.per_gate;
        const int64_t last = (g + 1) * p.rows_per_gate;
        row = g * p.rows_per_gate + j * q.strips.rows;
        end = row + q.strips.rows < last ? row + q.strips.rows : last;
    } else {
        row = strip * q.strips.rows;
        end = row + q.strips.rows;
    }
    if (end > p.rows) end = p.rows;
    if (row >= end && q.dgate && q.strips.per_gate > 1)  // the last gate row has fewer rows than the others
#pragma unroll
        for (int g = 0; g < VPT; g++) {
            const int c = 8 * (g * TPR + lane);
            const float none[8] = {};
            store8(q.part_gate + strip * C + c, C - c, none);
        }

    float d_post[VPT][8] = {}, d_pre[VPT][8] = {}, z[VPT][8] = {}, w_post[VPT][8], w_pre[VPT][8], gate[VPT][8];
    if (p.d_w_pre) load_params<W, TPR, VPT>(p.d_w_pre, 0, C, lane, w_pre);
    if (p.d_w_post) load_params<W, TPR, VPT>(p.d_w_post, 0, C, lane, w_post);
    else
#pragma unroll
        for (int g = 0; g < VPT; g++)
#pragma unroll
            for (int i = 0; i < 8; i++) w_post[g][i] = 1.f;
#pragma unroll
    for (int g = 0; g < VPT; g++)
#pragma unroll
        for (int i = 0; i < 8; i++) gate[g][i] = 1.f;
    int64_t gate_row = -1;
    for (; row < end; row++) {
        if (p.d_gate) {
            const int64_t want = row / p.rows_per_gate;
            if (want != gate_row) {
                gate_row = want;
                load_params<W, TPR, VPT>(p.d_gate, want, C, lane, gate);
            }
        }
        const float r_y = p.d_y && p.d_w_post ? q.stats[row] : 1.f, r_h = q.stats[p.rows + row];
        float t[VPT][8], hn[VPT][8], dn[VPT][8], y[VPT][8];
        float sum = 0.f;
#pragma unroll
        for (int g = 0; g < VPT; g++) {
            const int c = 8 * (g * TPR + lane);
            if (q.dh) load8(at<T>(q.dh, row * q.ld_dh + c), C - c, t[g]);
            else
#pragma unroll
                for (int i = 0; i < 8; i++) t[g][i] = 0.f;
            if (p.d_y) load8(at<T>(p.d_y, row * p.ld_y + c), C - c, y[g]);
            if (q.dn) {
                load8(at<T>(p.d_h, row * p.ld_h + c), C - c, hn[g]);
                load8(at<T>(q.dn, row * q.ld_dn + c), C - c, dn[g]);
            }
        }
        if (q.dn) {
#pragma unroll
            for (int g = 0; g < VPT; g++)
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    hn[g][i] *= r_h;
                    d_pre[g][i] = fmaf(dn[g][i], hn[g][i], d_pre[g][i]);
                    dn[g][i] *= w_pre[g][i];
                    sum = fmaf(dn[g][i], hn[g][i], sum);
                }
            const float mean = RowSum<TPR>::run(sum, &slots[0]) * rC;
#pragma unroll
            for (int g = 0; g < VPT; g++)
#pragma unroll
                for (int i = 0; i < 8; i++) t[g][i] = fmaf(r_h, fmaf(-mean, hn[g][i], dn[g][i]), t[g][i]);
        }
        if (q.dh_in) {
#pragma unroll
            for (int g = 0; g < VPT; g++) {
                const int c = 8 * (g * TPR + lane);
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; i++) v[i] = p.skip * t[g][i];
                store8(at<T>(q.dh_in, row * q.ld_dh_in + c), C - c, v);
            }
        }
        if (!p.d_y) continue;
        sum = 0.f;
#pragma unroll
        for (int g = 0; g < VPT; g++)
#pragma unroll
            for (int i = 0; i < 8; i++) {
                y[g][i] *= r_y;
                const float st = p.scale * t[g][i];
                z[g][i] = fmaf(st, y[g][i], z[g][i]);
                t[g][i] = st * gate[g][i] * w_post[g][i];
                sum = fmaf(t[g][i], y[g][i], sum);
            }
        if (p.d_w_post) {
            const float mean = RowSum<TPR>::run(sum, &slots[1]) * rC;
#pragma unroll
            for (int g = 0; g < VPT; g++)
#pragma unroll
                for (int i = 0; i < 8; i++) t[g][i] = r_y * fmaf(-mean, y[g][i], t[g][i]);
        }
        if (q.dy)
#pragma unroll
            for (int g = 0; g < VPT; g++) {
                const int c = 8 * (g * TPR + lane);
                store8(at<T>(q.dy, row * q.ld_dy + c), C - c, t[g]);
            }
        if (row + 1 == end || (p.d_gate && !q.strips.per_gate && (row + 1) % p.rows_per_gate == 0)) {
            float* to = q.dgate ? (q.strips.per_gate > 1 ? q.part_gate + strip * C : q.dgate + gate_row * C) : nullptr;
#pragma unroll
            for (int g = 0; g < VPT; g++) {
                const int c = 8 * (g * TPR + lane);
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    d_post[g][i] = fmaf(gate[g][i], z[g][i], d_post[g][i]);
                    v[i] = w_post[g][i] * z[g][i];
                    z[g][i] = 0.f;
                }
                if (to) store8(to + c, C - c, v);
            }
        }
    }
#pragma unroll
    for (int g = 0; g < VPT; g++) {
        const int c = 8 * (g * TPR + lane);
        if (q.part_post) store8(q.part_post + strip * C + c, C - c, d_post[g]);
        if (q.part_pre) store8(q.part_pre + strip * C + c, C - c, d_pre[g]);
    }
}

// out[j][c] = sum over i < n of part[j n + i][c], j = blockIdx.y: 32 columns a workgroup, 8 slices of the rows, added up in
// order
__global__ __launch_bounds__(256) void k_strip_sums(const float* __restrict__ part, int64_t n, int C, float* __restrict__ out) {
    __shared__ float slice[8][32];
    const int col = threadIdx.x & 31, k = threadIdx.x >> 5, c = blockIdx.x * 32 + col;
    const float* from = part + (int64_t)blockIdx.y * n * C;
    float sum = 0.f;
    if (c < C)
        for (int64_t i = k; i < n; i += 8) sum += from[i * C + c];
    slice[k][col] = sum;
    __syncthreads();
    if (k == 0 && c < C) {
#pragma unroll
        for (int i = 1; i < 8; i++) sum += slice[i][col];
        out[(int64_t)blockIdx.y * C + c] = sum;
    }
}

// TPR and VPT by the width alone: a row in as few lanes as hold it with at most 16 values each, whole wavefronts from 256
// values on
template <class F>
hipError_t with_width(int C, F&& f) {
    if (C <= 128) return f(Int<16>{}, Int<1>{});
    if (C <= 512) return f(Int<64>{}, Int<1>{});
    if (C <= 1024) return f(Int<64>{}, Int<2>{});
    if (C <= 2048) return f(Int<256>{}, Int<1>{});
    if (C <= 4096) return f(Int<256>{}, Int<2>{});
    if (C <= 8192) return f(Int<512>{}, Int<2>{});
    return f(Int<1024>{}, Int<2>{});
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
        return with_width(a.C, [&](auto lanes, auto groups) {
            constexpr int TPR = decltype(lanes)::value, VPT = decltype(groups)::value;
            constexpr int rows = norm_threads(TPR) / TPR;
            int64_t grid = ceil_div(a.rows, rows);
            if (grid > 2048) grid = 2048;
            return launch(K_BLOCK_NORM, k_block_norm<typename decltype(ty)::type, typename decltype(wt)::type, TPR, VPT>,
                          dim3((unsigned)grid), dim3(norm_threads(TPR)), 0, s, a, out);
        });
    });
}

size_t block_norm_workspace(int64_t rows, int C, int64_t rows_per_gate) {
    const Strips st = make_strips(rows, C, rows_per_gate);
    return align_up(sizeof(float) * (size_t)st.count * C, 256) * (st.per_gate > 1 ? 3 : 2);
}

hipError_t launch_block_norm_backward(const fmtc_norm& a, const float* d_stats, const void* d_dn, int64_t ld_dn,
                                      const void* d_dh, int64_t ld_dh, void* d_dy, int64_t ld_dy, void* d_dh_in,
                                      int64_t ld_dh_in, float* d_dw_post, float* d_dw_pre, float* d_dgate,
                                      void* d_ws, hipStream_t s) {
    const Strips st = make_strips(a.rows, a.C, a.d_gate ? a.rows_per_gate : 0);
    const size_t each = align_up(sizeof(float) * (size_t)st.count * a.C, 256);
    float* part[3] = {static_cast<float*>(d_ws), reinterpret_cast<float*>(static_cast<char*>(d_ws) + each),
                      reinterpret_cast<float*>(static_cast<char*>(d_ws) + 2 * each)};
    NormGrads q{d_stats, d_dn, d_dh, d_dy, d_dh_in, ld_dn, ld_dh, ld_dy, ld_dh_in,
                d_dw_post ? part[0] : nullptr, d_dw_pre ? part[1] : nullptr, part[2], d_dgate, st};
    hipError_t e = with_types(a.type, a.weight_type, [&](auto ty, auto wt) {
        return with_width(a.C, [&](auto lanes, auto groups) {
            constexpr int TPR = decltype(lanes)::value, VPT = decltype(groups)::value;
            return launch(K_BLOCK_NORM_BACKWARD, k_block_norm_backward<typename decltype(ty)::type, typename decltype(wt)::type, TPR, VPT>,
                          dim3((unsigned)ceil_div(st.count, norm_threads(TPR) / TPR)), dim3(norm_threads(TPR)), 0, s, a, q);
        });
    });
    auto sums = [&](const float* from, int64_t n, int64_t groups, float* to) {
        return launch(K_BLOCK_NORM_BACKWARD, k_strip_sums, dim3((unsigned)ceil_div(a.C, 32), (unsigned)groups), dim3(256), 0, s, from, n,
                      (int)a.C, to);
    };
    if (e == hipSuccess && d_dw_post) e = sums(part[0], st.count, 1, d_dw_post);
    if (e == hipSuccess && d_dw_pre) e = sums(part[1], st.count, 1, d_dw_pre);
    if (e == hipSuccess && d_dgate && st.per_gate > 1) e = sums(part[2], st.per_gate, st.gates, d_dgate);
    return e;
}

}  // namespace fmtc
