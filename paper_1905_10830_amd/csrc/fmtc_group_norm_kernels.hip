// Group norm with an activation of maps held channels last (fmtc_group_norm and its gradients).  Over the S rows and the D
// channels of a sample's group: mean, r = 1 / sqrt(variance + eps), x^ = (x - mean) r;
//   forward:   z = w x^ + b,  y = act(z)
//   backward:  dz = dy act'(z);  db = sum dz,  dw = sum dz x^  (over all rows);
//              dx = r (w dz - A - x^ B),  A = sum of w dz / (S D),  B = sum of w dz x^ / (S D)  (over the sample's group)
// Memory bound.  A thread takes 8 neighbouring channels (a lane of the row's LX) of every LY-th row, so that whole rows are
// read whatever the groups are; the sums meet in LDS by channel and are added up by group there.
#include "fmtc_block.h"

namespace fmtc {

namespace {

struct Maps {
    int64_t samples, S, ld;
    int C, G, D, LX, LY;     // LX lanes a row, LY rows at a time; D channels a group
    const void *x, *w, *b;
    int weight_type;
    int64_t chunks, per;     // parts of a sample's rows, rows of a part
};

template <class F>
__device__ __forceinline__ void with_weights(int type, F&& f) {
    if (type == FMTC_F32) f(Type<float>{});
    else if (type == FMTC_BF16) f(Type<bf16>{});
    else f(Type<_Float16>{});
}
// channels c .. c + 7 of the weight (1 where there is none) or of the bias (0)
__device__ __forceinline__ void load_param(const void* p, int type, int c, int C, float without, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = without;
    if (p)
        with_weights(type, [&](auto ty) {
            using W = typename decltype(ty)::type;
            load8<true>(static_cast<const W*>(p), c, C, v);
        });
}

// e = exp(-|z|) keeps both the sigmoid and what it lacks to 1 exact to a few roundings
template <int ACT>
__device__ __forceinline__ float act(float z) {
    if constexpr (ACT == FMTC_ACT_RELU) return z < 0.f ? 0.f : z;
    if constexpr (ACT == FMTC_ACT_SILU) return z * __builtin_amdgcn_rcpf(1.f + __expf(-z));
    return z;
}
template <int ACT>
__device__ __forceinline__ float act_gradient(float z) {
    if constexpr (ACT == FMTC_ACT_RELU) return z > 0.f ? 1.f : z <= 0.f ? 0.f : z;
    if constexpr (ACT == FMTC_ACT_SILU) {
        const float e = __expf(-fabsf(z)), r = __builtin_amdgcn_rcpf(1.f + e), er = e * r;
        const float p = z >= 0.f ? r : er, q = z >= 0.f ? er : r;
        return p * fmaf(z, q, 1.f);
    }
    return 1.f;
}

// Sums over the rows and channels of each group of what is in `red` ([LY][8 LX]): f(group, sum) by one thread each.  lanes:
// how many work on a group, a power of two up to 64.
template <class V, class F>
__device__ __forceinline__ void group_sums(const V* red, const Maps& p, int lanes, F&& f) {
    const int l = threadIdx.x & (lanes - 1), step = blockDim.x / lanes, n = p.LY * p.D;
    for (int g = threadIdx.x / lanes; g < p.G; g += step) {
        V sum = 0;
        for (int i = l; i < n; i += lanes) {
            const int y = i / p.D, c = i - y * p.D;
            sum += red[y * 8 * p.LX + g * p.D + c];
        }
        for (int o = lanes >> 1; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
        if (l == 0) f(g, sum);
    }
}
__device__ __forceinline__ int group_lanes(int G) {
    int lanes = 64;
    while (lanes > 1 && lanes * G > (int)blockDim.x) lanes >>= 1;
    return lanes;
}

constexpr int kUnroll = 4;  // rows of a thread on their way together

// The sums of the values and of their squares, of each part of a sample's rows and each group: part[sample][chunk][group].
// In f64, so that the variance is right however far the mean is from 0 (f64 runs at the rate of f32 here).
template <class T, bool RAGGED>
__global__ __launch_bounds__(1024) void k_group_norm_sums(Maps p, double2* __restrict__ part) {
    extern __shared__ __attribute__((aligned(16))) double red[];
    const int t = threadIdx.x, ly = t / p.LX, lx = t - ly * p.LX, c = 8 * lx;
    const int64_t n = blockIdx.x / p.chunks, k = blockIdx.x - n * p.chunks;
    const int64_t r0 = k * p.per, r1 = r0 + p.per < p.S ? r0 + p.per : p.S;
    const bool live = ly < p.LY;
    double s[8] = {}, q[8] = {};
    if (live) {
        const T* const x = static_cast<const T*>(p.x) + n * p.S * p.ld;
        for (int64_t r = r0 + ly; r < r1; r += (int64_t)kUnroll * p.LY) {
            Raw<T> raw[kUnroll];
#pragma unroll
            for (int u = 0; u < kUnroll; u++) {
                const int64_t at = r + (int64_t)u * p.LY;
                raw[u].template load<RAGGED>(x + (at < r1 ? at : r) * p.ld, c, p.C);
            }
#pragma unroll
            for (int u = 0; u < kUnroll; u++) {
                if constexpr (RAGGED) raw[u].settle(c, p.C);
                raw[u].zero_unless(r + (int64_t)u * p.LY < r1);
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    const double v = raw[u][i];
                    s[i] += v;
                    q[i] = fma(v, v, q[i]);
                }
            }
        }
    }
    const int lanes = group_lanes(p.G);
    double2* const to = part + (n * p.chunks + k) * p.G;
    double* const mine = red + (ly * p.LX + lx) * 8;
    if (live)
#pragma unroll
        for (int i = 0; i < 8; i++) mine[i] = s[i];
    __syncthreads();
    group_sums(red, p, lanes, [&](int g, double v) { to[g].x = v; });
    __syncthreads();
    if (live)
#pragma unroll
        for (int i = 0; i < 8; i++) mine[i] = q[i];
    __syncthreads();
    group_sums(red, p, lanes, [&](int g, double v) { to[g].y = v; });
}

// mean and r of each group of sample n into LDS, and, by the sample's first workgroup, where the caller wants them
__device__ __forceinline__ void finish_stats(const Maps& p, const double2* part, int64_t n, float eps, float* mean_r, float* stats, bool first) {
    const int lanes = group_lanes(p.G), l = threadIdx.x & (lanes - 1), step = blockDim.x / lanes;
    const double count = (double)p.S * (double)p.D;
    for (int g = threadIdx.x / lanes; g < p.G; g += step) {
        double s = 0.0, q = 0.0;
        for (int64_t k = l; k < p.chunks; k += lanes) {
            const double2 v = part[(n * p.chunks + k) * p.G + g];
            s += v.x;
            q += v.y;
        }
        for (int o = lanes >> 1; o > 0; o >>= 1) {
            s += __shfl_xor(s, o, 64);
            q += __shfl_xor(q, o, 64);
        }
        if (l == 0) {
            const double mean = s / count, var = q / count - mean * mean;
            const float m = (float)mean, r = (float)(1.0 / sqrt((var < 0.0 ? 0.0 : var) + (double)eps));
            mean_r[g] = m;
            mean_r[p.G + g] = r;
            if (stats && first) {
                stats[n * p.G + g] = m;
                stats[(p.samples + n) * p.G + g] = r;
            }
        }
    }
    __syncthreads();
}

template <class T, bool RAGGED, int ACT>
__global__ __launch_bounds__(1024) void k_group_norm_apply(Maps p, const double2* __restrict__ part, int64_t parts, int64_t rows, float eps,
                                                           T* y, int64_t ld_y, float* __restrict__ stats) {
    extern __shared__ __attribute__((aligned(16))) float mean_r[];
    const int64_t n = blockIdx.x / parts, k = blockIdx.x - n * parts;
    finish_stats(p, part, n, eps, mean_r, stats, k == 0);
    if (!y) return;
    const int t = threadIdx.x, ly = t / p.LX, lx = t - ly * p.LX, c = 8 * lx;
    if (ly >= p.LY) return;
    float w[8], b[8], m[8];
    load_param(p.w, p.weight_type, c, p.C, 1.f, w);
    load_param(p.b, p.weight_type, c, p.C, 0.f, b);
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const int g = (c + i < p.C ? c + i : p.C - 1) / p.D;
        m[i] = mean_r[g];
        w[i] *= mean_r[p.G + g];
    }
    const int64_t r0 = k * rows, r1 = r0 + rows < p.S ? r0 + rows : p.S;
    const T* const x = static_cast<const T*>(p.x) + n * p.S * p.ld;
    T* const out = y + n * p.S * ld_y;
    for (int64_t r = r0 + ly; r < r1; r += (int64_t)kUnroll * p.LY) {
        Raw<T> raw[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; u++) {
            const int64_t at = r + (int64_t)u * p.LY;
            raw[u].template load<RAGGED>(x + (at < r1 ? at : r) * p.ld, c, p.C);
        }
#pragma unroll
        for (int u = 0; u < kUnroll; u++) {
            const int64_t at = r + (int64_t)u * p.LY;
            if (at >= r1) break;
            if constexpr (RAGGED) raw[u].settle(c, p.C);
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] = act<ACT>(fmaf(raw[u][i] - m[i], w[i], b[i]));
            store8(out + at * ld_y + c, RAGGED ? p.C - c : 8, v);
        }
    }
}

// To codes with a scale for each row: TPR lanes hold a row; mean, weight and bias of each channel in LDS.
constexpr int codes_threads(int TPR) { return TPR < 256 ? 256 : TPR; }
template <class T, bool RAGGED, int TPR>
__global__ __launch_bounds__(codes_threads(TPR)) void k_group_norm_codes(Maps p, const double2* __restrict__ part, int64_t parts, int64_t rows,
                                                                         float eps, int act_kind, fmtc_i8 out, T* y, int64_t ld_y,
                                                                         float* __restrict__ stats) {
    extern __shared__ __attribute__((aligned(16))) float mean_r[];
    __shared__ uint32_t turns[2][codes_threads(TPR) / 64];
    constexpr int kRows = codes_threads(TPR) / TPR;
    const int64_t n = blockIdx.x / parts, k = blockIdx.x - n * parts;
    finish_stats(p, part, n, eps, mean_r, stats, k == 0);
    const int lane = threadIdx.x % TPR, c = 8 * lane, width = (p.C + kF8Block - 1) / kF8Block * kF8Block;
    float w[8], b[8], m[8];
    load_param(p.w, p.weight_type, c, p.C, 1.f, w);
    load_param(p.b, p.weight_type, c, p.C, 0.f, b);
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const bool there = c + i < p.C;
        const int g = (there ? c + i : p.C - 1) / p.D;
        m[i] = there ? mean_r[g] : 0.f;
        w[i] = there ? w[i] * mean_r[p.G + g] : 0.f;
        b[i] = there ? b[i] : 0.f;
    }
    const int64_t r0 = k * rows, r1 = r0 + rows < p.S ? r0 + rows : p.S;
    const T* const x = static_cast<const T*>(p.x) + n * p.S * p.ld;
    int turn = 0;
    for (int64_t r = r0; r < r1; r += kRows, turn ^= 1) {  // (all threads take every round: there are barriers in it)
        const int64_t mine = r + threadIdx.x / TPR, at = mine < r1 ? mine : r1 - 1;
        Raw<T> raw;
        raw.template load<RAGGED>(x + at * p.ld, c, p.C);
        if constexpr (RAGGED) raw.settle(c, p.C);
        raw.zero_unless(c < p.C);
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = fmaf(raw[i] - m[i], w[i], b[i]);
        if (act_kind == FMTC_ACT_RELU) {
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] = act<FMTC_ACT_RELU>(v[i]);
        } else if (act_kind == FMTC_ACT_SILU) {
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] = act<FMTC_ACT_SILU>(v[i]);
        }
        float held;
        const float inv = i8_row_scale(row_max_bits<TPR>(amax_bits8(v), turns[turn]), &held);
        if (mine >= r1) continue;
        const int64_t row = n * p.S + at;
        if (c < width)
            *reinterpret_cast<uint2*>(static_cast<uint8_t*>(out.d_codes) + row * out.ld + c) = make_uint2(i8_encode4(v, inv), i8_encode4(v + 4, inv));
        if (lane == 0) out.d_scales[row] = held;
        if (y && c < p.C) store8(y + row * ld_y + c, p.C - c, v);
    }
}

// What a thread needs of its 8 channels for the gradients
struct Channels {
    float m[8], r[8], w[8], b[8];
    __device__ __forceinline__ void load(const Maps& p, const float* stats, int64_t n, int c) {
        load_param(p.w, p.weight_type, c, p.C, 1.f, w);
        load_param(p.b, p.weight_type, c, p.C, 0.f, b);
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const int g = (c + i < p.C ? c + i : p.C - 1) / p.D;
            m[i] = stats[n * p.G + g];
            r[i] = stats[(p.samples + n) * p.G + g];
        }
    }
};
template <int ACT>
__device__ __forceinline__ void gradient(const Channels& ch, int i, float x, float dy, float* xh, float* dz) {
    *xh = (x - ch.m[i]) * ch.r[i];
    *dz = ACT == FMTC_ACT_NONE ? dy : dy * act_gradient<ACT>(fmaf(*xh, ch.w[i], ch.b[i]));
}

// The sums of dz and of dz x^ of each part of a sample's rows and each channel: part[sample][chunk][2][C].
template <class T, bool RAGGED, int ACT>
__global__ __launch_bounds__(1024) void k_group_norm_gradient_sums(Maps p, const float* __restrict__ stats, const T* __restrict__ dy,
                                                                   int64_t ld_dy, float* __restrict__ part) {
    extern __shared__ __attribute__((aligned(16))) float red_f[];
    const int t = threadIdx.x, ly = t / p.LX, lx = t - ly * p.LX, c = 8 * lx;
    const int64_t n = blockIdx.x / p.chunks, k = blockIdx.x - n * p.chunks;
    const int64_t r0 = k * p.per, r1 = r0 + p.per < p.S ? r0 + p.per : p.S;
    float s[8] = {}, q[8] = {};
    if (ly < p.LY) {
        Channels ch;
        ch.load(p, stats, n, c);
        const T *const x = static_cast<const T*>(p.x) + n * p.S * p.ld, *const g = dy + n * p.S * ld_dy;
        constexpr int U = kUnroll / 2;
        for (int64_t r = r0 + ly; r < r1; r += (int64_t)U * p.LY) {
            Raw<T> raw[U], raw_g[U];
#pragma unroll
            for (int u = 0; u < U; u++) {
                const int64_t at = r + (int64_t)u * p.LY, from = at < r1 ? at : r;
                raw[u].template load<RAGGED>(x + from * p.ld, c, p.C);
                raw_g[u].template load<RAGGED>(g + from * ld_dy, c, p.C);
            }
#pragma unroll
            for (int u = 0; u < U; u++) {
                if (r + (int64_t)u * p.LY >= r1) break;
                if constexpr (RAGGED) raw[u].settle(c, p.C), raw_g[u].settle(c, p.C);
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    float xh, dz;
                    gradient<ACT>(ch, i, raw[u][i], raw_g[u][i], &xh, &dz);
                    s[i] += dz;
                    q[i] = fmaf(dz, xh, q[i]);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 8; i++) {
            red_f[(ly * p.LX + lx) * 8 + i] = s[i];
            red_f[((p.LY + ly) * p.LX + lx) * 8 + i] = q[i];
        }
    }
    __syncthreads();
    const int64_t base = (n * p.chunks + k) * 2 * p.C;
    for (int i = t; i < 2 * p.C; i += blockDim.x) {
        const int which = i >= p.C, col = i - which * p.C;
        float sum = 0.f;
        for (int y = 0; y < p.LY; y++) sum += red_f[(which * p.LY + y) * 8 * p.LX + col];
        part[base + i] = sum;
    }
}

template <class T, bool RAGGED, int ACT>
__global__ __launch_bounds__(1024) void k_group_norm_dx(Maps p, const float* __restrict__ stats, const float* __restrict__ part, int64_t parts,
                                                        int64_t rows, const T* dy, int64_t ld_dy, T* dx, int64_t ld_dx) {
    extern __shared__ __attribute__((aligned(16))) float red_f[];  // [2][C]: sums by channel, then [2][G]: A and B
    const int t = threadIdx.x, ly = t / p.LX, lx = t - ly * p.LX, c = 8 * lx;
    const int64_t n = blockIdx.x / parts, k = blockIdx.x - n * parts;
    float* const ab = red_f + 2 * p.C;
    for (int i = t; i < 2 * p.C; i += blockDim.x) {
        float sum = 0.f;
        for (int64_t j = 0; j < p.chunks; j++) sum += part[(n * p.chunks + j) * 2 * p.C + i];
        const int col = i < p.C ? i : i - p.C;
        float w = 1.f;
        if (p.w) with_weights(p.weight_type, [&](auto ty) {
            using W = typename decltype(ty)::type;
            w = to_f32(static_cast<const W*>(p.w)[col]);
        });
        red_f[i] = w * sum;
    }
    __syncthreads();
    const float rcount = 1.f / ((float)p.S * (float)p.D);
    for (int i = t; i < 2 * p.G; i += blockDim.x) {
        const int which = i >= p.G, g = i - which * p.G;
        float sum = 0.f;
        for (int j = 0; j < p.D; j++) sum += red_f[which * p.C + g * p.D + j];
        ab[i] = sum * rcount;
    }
    __syncthreads();
    if (ly >= p.LY) return;
    Channels ch;
    ch.load(p, stats, n, c);
    float A[8], B[8];
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const int g = (c + i < p.C ? c + i : p.C - 1) / p.D;
        A[i] = ab[g];
        B[i] = ab[p.G + g];
    }
    const int64_t r0 = k * rows, r1 = r0 + rows < p.S ? r0 + rows : p.S;
    const T *const x = static_cast<const T*>(p.x) + n * p.S * p.ld, *const g = dy + n * p.S * ld_dy;
    T* const out = dx + n * p.S * ld_dx;
    constexpr int U = kUnroll / 2;
    for (int64_t r = r0 + ly; r < r1; r += (int64_t)U * p.LY) {
        Raw<T> raw[U], raw_g[U];
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int64_t at = r + (int64_t)u * p.LY, from = at < r1 ? at : r;
            raw[u].template load<RAGGED>(x + from * p.ld, c, p.C);
            raw_g[u].template load<RAGGED>(g + from * ld_dy, c, p.C);
        }
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int64_t at = r + (int64_t)u * p.LY;
            if (at >= r1) break;
            if constexpr (RAGGED) raw[u].settle(c, p.C), raw_g[u].settle(c, p.C);
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; i++) {
                float xh, dz;
                gradient<ACT>(ch, i, raw[u][i], raw_g[u][i], &xh, &dz);
                v[i] = ch.r[i] * (fmaf(ch.w[i], dz, -A[i]) - xh * B[i]);
            }
            store8(out + at * ld_dx + c, RAGGED ? p.C - c : 8, v);
        }
    }
}

// dbias and dweight: sums over the parts, 32 columns a workgroup, 32 slices of the parts, added up in order
__global__ __launch_bounds__(1024) void k_group_norm_params(const float* __restrict__ part, int64_t n, int C, float* __restrict__ dweight,
                                                            float* __restrict__ dbias) {
    __shared__ float slice[32][33];
    const int col = threadIdx.x & 31, k = threadIdx.x >> 5, c = blockIdx.x * 32 + col;
    float sum = 0.f;
    if (c < 2 * C)
#pragma unroll 4
        for (int64_t i = k; i < n; i += 32) sum += part[i * 2 * C + c];
    slice[k][col] = sum;
    __syncthreads();
    if (k == 0 && c < 2 * C) {
#pragma unroll
        for (int i = 1; i < 32; i++) sum += slice[i][col];
        float* const to = c < C ? dbias : dweight;
        if (to) to[c < C ? c : c - C] = sum;
    }
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

struct Shape { int threads, LX, LY; };
Shape shape_of(int C) {
    const int LX = (C + 7) / 8, threads = LX <= 64 ? 256 : LX <= 128 ? 512 : 1024;
    return {threads, LX, threads / LX};
}
// parts of a sample's rows: `want` workgroups in all, some rows for every thread, and not more than `most`
int64_t parts_of(int64_t samples, int64_t S, int LY, int64_t want, int64_t most) {
    int64_t parts = ceil_div(want, samples), fit = ceil_div(S, (int64_t)kUnroll * LY);
    parts = parts < fit ? parts : fit;
    parts = parts < most ? parts : most;
    return ceil_div(S, ceil_div(S, parts));
}
constexpr int64_t kWorkgroups = 2048;  // of 256 threads: what runs at a time
constexpr int64_t kMostChunks = 256;

Maps maps_of(const fmtc_gnorm& a, const Shape& sh) {
    Maps p{a.samples, a.rows_per_sample, a.ld_x, a.C, a.groups, a.C / a.groups, sh.LX, sh.LY, a.d_x, a.d_weight, a.d_bias, a.weight_type, 0, 0};
    p.chunks = parts_of(p.samples, p.S, sh.LY, kWorkgroups * 256 / sh.threads, kMostChunks);
    p.per = ceil_div(p.S, p.chunks);
    return p;
}
int64_t chunks_of(int64_t samples, int64_t S, int C) {
    const Shape sh = shape_of(C);
    return parts_of(samples, S, sh.LY, kWorkgroups * 256 / sh.threads, kMostChunks);
}
template <class F>
hipError_t with_act(int act, F&& f) {
    return act == FMTC_ACT_NONE ? f(Int<FMTC_ACT_NONE>{}) : act == FMTC_ACT_RELU ? f(Int<FMTC_ACT_RELU>{}) : f(Int<FMTC_ACT_SILU>{});
}
template <class K>
hipError_t allow_lds(K kernel, size_t bytes) {
    return bytes <= 65536 ? hipSuccess : hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
}

}  // namespace

size_t group_norm_workspace(int64_t samples, int64_t S, int C, int groups) {
    return align_up(sizeof(double2) * (size_t)(samples * chunks_of(samples, S, C)) * groups, 256);
}
size_t group_norm_backward_workspace(int64_t samples, int64_t S, int C, int) {
    return align_up(sizeof(float) * (size_t)(samples * chunks_of(samples, S, C)) * 2 * C, 256);
}

hipError_t launch_group_norm(const fmtc_gnorm& a, void* d_y, int64_t ld_y, const fmtc_i8* codes, float* d_stats, void* d_ws, hipStream_t s) {
    const Shape sh = shape_of(a.C);
    const Maps p = maps_of(a, sh);
    double2* const part = static_cast<double2*>(d_ws);
    return with_type(a.type, [&](auto ty) {
        using T = typename decltype(ty)::type;
        return with_bit(a.C % 8 != 0, [&](auto rg) {
            constexpr bool R = decltype(rg)::value;
            auto sums = k_group_norm_sums<T, R>;
            const size_t lds = sizeof(double) * 8 * sh.LX * sh.LY;
            hipError_t e = allow_lds(sums, lds);
            if (e == hipSuccess) e = launch(K_GROUP_NORM, sums, dim3((unsigned)(p.samples * p.chunks)), dim3(sh.threads), lds, s, p, part);
            if (e != hipSuccess) return e;
            const size_t lds_stats = sizeof(float) * 2 * p.G;
            if (codes) {
                auto go = [&](auto tpr) {
                    constexpr int TPR = decltype(tpr)::value, kRows = codes_threads(TPR) / TPR;
                    const int64_t parts = parts_of(p.samples, p.S, kRows, kWorkgroups, p.S), rows = ceil_div(p.S, parts);
                    auto kernel = k_group_norm_codes<T, R, TPR>;
                    const hipError_t e = allow_lds(kernel, lds_stats);
                    return e != hipSuccess ? e : launch(K_GROUP_NORM, kernel, dim3((unsigned)(p.samples * parts)), dim3(codes_threads(TPR)), lds_stats, s, p,
                                                        (const double2*)part, parts, rows, a.eps, a.act, *codes, static_cast<T*>(d_y), ld_y, d_stats);
                };
                return p.C <= 128 ? go(Int<16>{}) : p.C <= 512 ? go(Int<64>{}) : p.C <= 2048 ? go(Int<256>{}) : go(Int<1024>{});
            }
            const int64_t parts = d_y ? parts_of(p.samples, p.S, sh.LY, kWorkgroups * 256 / sh.threads, p.S) : 1, rows = ceil_div(p.S, parts);
            return with_act(a.act, [&](auto ac) {
                auto kernel = k_group_norm_apply<T, R, decltype(ac)::value>;
                const hipError_t e = allow_lds(kernel, lds_stats);
                return e != hipSuccess ? e : launch(K_GROUP_NORM, kernel, dim3((unsigned)(p.samples * parts)), dim3(sh.threads), lds_stats, s, p, (const double2*)part,
                                                    parts, rows, a.eps, static_cast<T*>(d_y), ld_y, d_stats);
            });
        });
    });
}

hipError_t launch_group_norm_backward(const fmtc_gnorm& a, const float* d_stats, const void* d_dy, int64_t ld_dy, void* d_dx, int64_t ld_dx,
                                      float* d_dweight, float* d_dbias, void* d_ws, hipStream_t s) {
    const Shape sh = shape_of(a.C);
    const Maps p = maps_of(a, sh);
    float* const part = static_cast<float*>(d_ws);
    return with_type(a.type, [&](auto ty) {
        using T = typename decltype(ty)::type;
        return with_bit(a.C % 8 != 0, [&](auto rg) {
            return with_act(a.act, [&](auto ac) {
                constexpr bool R = decltype(rg)::value;
                constexpr int A = decltype(ac)::value;
                const T* dy = static_cast<const T*>(d_dy);
                auto sums = k_group_norm_gradient_sums<T, R, A>;
                const size_t lds = sizeof(float) * 16 * sh.LX * sh.LY, lds_dx = sizeof(float) * 2 * (p.C + p.G);
                hipError_t e = allow_lds(sums, lds);
                if (e == hipSuccess)
                    e = launch(K_GROUP_NORM_BACKWARD, sums, dim3((unsigned)(p.samples * p.chunks)), dim3(sh.threads), lds, s, p, d_stats, dy, ld_dy, part);
                if (e == hipSuccess && (d_dweight || d_dbias))
                    e = launch(K_GROUP_NORM_BACKWARD, k_group_norm_params, dim3((unsigned)ceil_div(2 * p.C, 32)), dim3(1024), 0, s, (const float*)part,
                               p.samples * p.chunks, p.C, d_dweight, d_dbias);
                if (e != hipSuccess || !d_dx) return e;
                const int64_t parts = parts_of(p.samples, p.S, sh.LY, kWorkgroups * 256 / sh.threads, p.S), rows = ceil_div(p.S, parts);
                auto kernel = k_group_norm_dx<T, R, A>;
                e = allow_lds(kernel, lds_dx);
                return e != hipSuccess ? e : launch(K_GROUP_NORM_BACKWARD, kernel, dim3((unsigned)(p.samples * parts)), dim3(sh.threads), lds_dx, s, p, d_stats,
                                                    (const float*)part, parts, rows, dy, ld_dy, static_cast<T*>(d_dx), ld_dx);
            });
        });
    });
}

}  // namespace fmtc
