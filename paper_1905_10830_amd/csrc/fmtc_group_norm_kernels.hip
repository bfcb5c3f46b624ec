// Group norm with an activation of maps held channels last (fmtc_group_norm and its gradients).  Over the S rows and the D
// channels of a sample's group: mean, r = 1 / sqrt(variance + eps), x^ = (x - mean) r;
//   forward:   z = w x^ + b,  y = act(z)
//   backward:  dz = dy act'(z);  db = sum dz,  dw = sum dz x^  (over all rows);
//              dx = r (w dz - A - x^ B),  A = sum of w dz / (S D),  B = sum of w dz x^ / (S D)  (over the sample's group)
// Memory bound.  A workgroup works on a slab of a sample's rows: W neighbouring channels, whole groups.  A thread takes 8
// neighbouring ones of them (a lane of the LX of a row) of every LY-th row; the sums meet in LDS and are added up by group
// there.  Where a slab fits the registers of one workgroup, all is done with one read of the values (k_group_norm_once,
// k_group_norm_backward_once); else the rows are cut in chunks, whose sums one kernel leaves in the workspace and the next one
// adds up before it reads the values again.
// Times are the kernels' own, on inputs and results that stay where they are (the memory-side cache serves a part), where not said
// otherwise.
#include <type_traits>

#include "fmtc_block.h"

namespace fmtc {

namespace {

struct Maps {
    int64_t samples, all, S, ld;  // samples of this launch, and those that the statistics are of (from one to the next of their arrays)
    int C, G, D;          // D channels a group
    int W, groups, slabs, LX, LY; // channels and groups of a slab (the last one may have fewer), slabs of a row; lanes of a row, rows at a time
    int pre;                      // sums by group: a thread's 8 channels leave 1 << pre values (see fold)
    const void *x, *w, *b;
    int weight_type;
    int64_t chunks, per;  // parts of a sample's rows, rows of a part
};

// What a workgroup works on.  Workgroups go to the 8 XCDs in turn: each XCD gets a range of them, so that slabs that share
// lines of memory run on one and find them in its cache.
struct Place {
    int64_t n, k;
    int slab, c0, width, g0, groups;  // the slab's first channel, its channels, its first group, its groups
    __device__ __forceinline__ Place(const Maps& p, int64_t parts, uint32_t first) {
        const uint32_t total = gridDim.x - first, b = blockIdx.x - first, each = total / 8, more = total % 8, xcd = b % 8;
        const uint32_t at = xcd * each + (xcd < more ? xcd : more) + b / 8, row = at / (uint32_t)p.slabs;
        slab = (int)(at - row * p.slabs);
        n = row / (uint32_t)parts;
        k = row - n * parts;
        c0 = slab * p.W;
        width = p.C - c0 < p.W ? p.C - c0 : p.W;
        g0 = slab * p.groups;
        groups = p.G - g0 < p.groups ? p.G - g0 : p.groups;
    }
};

// i / d for i up to 2^20, r = 1 / d: what is added keeps the product further from the next whole number than its roundings go
__device__ __forceinline__ int quotient(int i, float r) { return (int)(((float)i + 0.5f) * r); }

// How the rows of a slab lie: multiples of 8 channels at multiples of 8; 8 channels or more; any number of them.  (The question
// whether there are 8, asked at each load, holds the loads apart: sums of 41 x 1716 x
// 522 40.8 -> 35.0 us, gradient sums of 2 x 18281 x 435 21.0 -> 18.4 us; rows that begin at multiples of 16 bytes: 17.8 and 15.8.)
enum Kind { kWhole = 0, kLong = 1, kShort = 2 };  // (of the narrowest slab)
template <int KIND, class T>
__device__ __forceinline__ void load_raw(Raw<T>& raw, const T* row, int64_t c, int64_t C) {
    if constexpr (KIND == kLong) raw.load_long(row, c, C);
    else raw.template load<KIND == kShort>(row, c, C);
}
template <int KIND, class T>
__device__ __forceinline__ void settle_raw(Raw<T>& raw, int64_t c, int64_t C) {
    if constexpr (KIND != kWhole) raw.settle(c, C);  // (rows of fewer than 8 are loaded value by value, with zeros behind them)
}
template <int KIND, class T>
__device__ __forceinline__ void load_values(const T* row, int64_t c, int64_t C, float (&v)[8]) {
    Raw<T> raw;
    load_raw<KIND>(raw, row, c, C);
    settle_raw<KIND>(raw, c, C);
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = raw[i];
}

// channels c .. c + 7 of the weight (1 where there is none) or of the bias (0); f32, or the type of the values
template <class T, int KIND>
__device__ __forceinline__ void load_param(const void* p, int type, int c, int C, float without, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = without;
    if (p) {
        if (type == FMTC_F32) load_values<KIND>(static_cast<const float*>(p), c, C, v);
        else load_values<KIND>(static_cast<const T*>(p), c, C, v);
    }
}
// f(i, group) for each of 8 channels from c on (of a slab of `width`; those past it: the last one's group)
template <class F>
__device__ __forceinline__ void each_group(int c, int width, int D, F&& f) {
    int g = quotient(c, 1.f / (float)D), left = D - (c - g * D);
#pragma unroll
    for (int i = 0; i < 8; i++) {
        f(i, g);
        left--;
        const bool next = left == 0 && c + i + 1 < width;
        g = next ? g + 1 : g;
        left = next ? D : left;
    }
}

template <int ACT>
__device__ __forceinline__ float act(float z) {
    if constexpr (ACT == FMTC_ACT_RELU) return z < 0.f ? 0.f : z;
    if constexpr (ACT == FMTC_ACT_SILU) return z * __builtin_amdgcn_rcpf(1.f + __expf(-z));
    return z;
}
// (silu: p (1 + z (1 - p)); from z = 17 on p is 1 and z (1 - p) is lost, which is less than 17 half steps of it)
template <int ACT>
__device__ __forceinline__ float act_gradient(float z) {
    if constexpr (ACT == FMTC_ACT_RELU) return z > 0.f ? 1.f : z <= 0.f ? 0.f : z;
    if constexpr (ACT == FMTC_ACT_SILU) {
        const float p = __builtin_amdgcn_rcpf(1.f + __expf(-z));
        return p * fmaf(z, 1.f - p, 1.f);
    }
    return 1.f;
}

// f(group, lane, lanes) on `lanes` neighbouring threads for each of n things: a power of two up to 64 of them, such that all
// threads have work.
template <class F>
__device__ __forceinline__ void spread(int n, F&& f) {
    int lanes = 64;
    while (lanes > 1 && lanes * n > (int)blockDim.x) lanes >>= 1;
    for (int i = threadIdx.x / lanes; i < n; i += blockDim.x / lanes) f(i, (int)threadIdx.x & (lanes - 1), lanes);
}
template <class V>
__device__ __forceinline__ V lanes_sum(V v, int lanes) {
    for (int o = lanes >> 1; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// A thread's sums by channel to 1 << pre sums of neighbours of one group: 1 where a group has a multiple of 8 channels, 8 / D
// for 2 and 4 of them, else 8 as they are.
constexpr int fold_of(int D) { return D % 8 == 0 ? 0 : D == 4 ? 1 : D == 2 ? 2 : 3; }
__device__ __forceinline__ void fold(double (&s)[8], int pre) {
    if (pre < 3)
#pragma unroll
        for (int i = 0; i < 4; i++) s[i] = s[2 * i] + s[2 * i + 1];
    if (pre < 2) s[0] += s[1], s[1] = s[2] + s[3];
    if (pre < 1) s[0] += s[1];
}

// The sums s of the values and q of their squares of all threads, by group: f(group of the slab, sum, sum of squares) on one
// thread each.  red: 2 << pre doubles a thread (a thread's values apart by the number of threads, so that neighbours write to
// neighbouring banks).
template <class F>
__device__ __forceinline__ void sums_by_group(const Maps& p, const Place& at, bool live, double (&s)[8], double (&q)[8], double* red, F&& f) {
    const int T = blockDim.x, pre = p.pre, D = p.D << pre >> 3, n = 1 << pre;  // values of a group in a row
    const float rD = 1.f / (float)D;
    fold(s, pre);
    fold(q, pre);
#pragma unroll
    for (int i = 0; i < 8; i++)
        if (i < n) {
            red[i * T + threadIdx.x] = live ? s[i] : 0.0;
            red[(n + i) * T + threadIdx.x] = live ? q[i] : 0.0;
        }
    __syncthreads();
    auto part_of = [&](int g, int first, int step, double* a, double* b) {
#pragma unroll 4
        for (int i = first; i < p.LY * D; i += step) {
            const int y = quotient(i, rD), v = g * D + i - y * D, from = (v & (n - 1)) * T + y * p.LX + (v >> pre);
            *a += red[from];
            *b += red[n * T + from];
        }
    };
    // Few groups: several wavefronts for each, whose sums meet in LDS again (2 x 16 x 448, one group of 14 channels a workgroup of
    // 1024: 15.8 us with one wavefront, 9.4 with sixteen).
    const int waves = T / 64;
    if (2 * at.groups <= waves) {
        __shared__ double few[2][16];
        const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, teams = waves / at.groups, g = wave / teams, team = wave - g * teams;
        double a = 0.0, b = 0.0;
        if (g < at.groups) part_of(g, team * 64 + lane, teams * 64, &a, &b);
        a = lanes_sum(a, 64);
        b = lanes_sum(b, 64);
        if (lane == 0) few[0][wave] = a, few[1][wave] = b;
        __syncthreads();
        if ((int)threadIdx.x < at.groups) {
            a = b = 0.0;
            for (int i = 0; i < teams; i++) {
                a += few[0][threadIdx.x * teams + i];
                b += few[1][threadIdx.x * teams + i];
            }
            f((int)threadIdx.x, a, b);
        }
        return;
    }
    spread(at.groups, [&](int g, int l, int lanes) {
        double a = 0.0, b = 0.0;
        part_of(g, l, lanes, &a, &b);
        a = lanes_sum(a, lanes);
        b = lanes_sum(b, lanes);
        if (l == 0) f(g, a, b);
    });
}
// The variance is right however far the mean is from 0, with sums in f64 (reading 100 MB takes the same time with them as with f32
// ones, 5.1 TB/s):
// * f32: what is summed is the values' distance from an origin, the first value of their sample's group (0 where that is not
//   finite); in f64 that difference is exact unless the two are 2^29 apart.  The origin lies within sqrt(S D) deviations of the
//   mean, so that the variance loses S D of 2^53 at most.  Sums of the values themselves lose (mean / deviation)^2, which was 7e-4
//   of r at a mean of 3e6 deviations.  (The differences cost 0 to 5 % of a norm's time: 1 x 262144 x 64 36.7 -> 37.3 us, 128 x 784 x
//   256 47.8 -> 48.6, 100 x 60 x 960 14.7 -> 15.4.)
// * 16 bits: values of one sign whose magnitudes are within 4 of each other are multiples of 2^-13 of the largest: sums of up to 2^27
//   of them and of their squares are exact, and finish() loses nothing of those either.  Where others are among them, the mean
//   is within 3 sqrt(S D) deviations of 0.
template <class T>
constexpr bool kFromOrigin = sizeof(T) == 4;
// The origins of a thread's 8 channels (ONE: they are of one group): loaded behind the first values, not before them (128 x 784 x 256
// 48.6 us, else 54.5), and looked at when those are on their way.
template <class T, bool ONE>
struct Origins {
    static constexpr int N = !kFromOrigin<T> ? 0 : ONE ? 1 : 8;
    T raw[N ? N : 1];
    double o[N ? N : 1];
    __device__ __forceinline__ void load(const Maps& p, const Place& at, int c) {
        const T* const first = static_cast<const T*>(p.x) + at.n * p.S * p.ld + at.c0;
        if constexpr (N == 1) raw[0] = first[quotient(c, 1.f / (float)p.D) * p.D];
        if constexpr (N == 8) each_group(c, at.width, p.D, [&](int i, int g) { raw[i] = first[g * p.D]; });
    }
    __device__ __forceinline__ float finite(int i) const { return __builtin_isfinite(to_f32(raw[i])) ? to_f32(raw[i]) : 0.f; }
    __device__ __forceinline__ void settle() {
#pragma unroll
        for (int i = 0; i < N; i++) {
            asm volatile("" : "+v"(raw[i]));  // (here, and not before the loop that this stands in)
            o[i] = finite(i);
        }
    }
    // to where finish() looks for them
    __device__ __forceinline__ void keep(const Maps& p, const Place& at, int c, float* to) const {
        if constexpr (N == 1) to[quotient(c, 1.f / (float)p.D)] = finite(0);
        if constexpr (N == 8) each_group(c, at.width, p.D, [&](int i, int g) { to[g] = finite(i); });
    }
    __device__ __forceinline__ void add(Raw<T>& values, bool live, double (&s)[8], double (&q)[8]) const {
        if constexpr (N > 0) {
            if (!live) return;
        } else {
            values.zero_unless(live);
        }
#pragma unroll
        for (int i = 0; i < 8; i++) {
            double v = values[i];
            if constexpr (N > 0) v -= o[ONE ? 0 : i];
            s[i] += v;
            q[i] = fma(v, v, q[i]);
        }
    }
};
// s, q: sums of the distances from the origin and of their squares.  var = (n q - s^2) / n^2, both products with what their
// rounding takes (and not fused with the difference by the compiler).  stats: the caller's, or NULL
__device__ __forceinline__ void finish(const Maps& p, const Place& at, int g, double origin, double s, double q, float eps, float* mean_r, float* stats) {
#pragma clang fp contract(off)
    const double count = (double)p.S * (double)p.D, mean = origin + s / count, nq = count * q, ss = s * s;
    const double var = ((nq - ss) + (fma(count, q, -nq) - fma(s, s, -ss))) / (count * count);
    // (a variance that is not a number stays that)
    const float m = (float)mean, r = (float)(1.0 / sqrt((var < 0.0 ? 0.0 : var) + (double)eps));
    mean_r[g] = m;
    mean_r[at.groups + g] = r;
    if (stats) {
        stats[at.n * p.G + at.g0 + g] = m;
        stats[(p.all + at.n) * p.G + at.g0 + g] = r;
    }
}

// y = act((x - m) w + b) of a thread's 8 channels (c: of the slab's).  The parameters set out before the statistics are there.
struct Scale {
    float m[8], w[8], b[8];
    template <class T, int KIND>
    __device__ __forceinline__ void load(const Maps& p, const Place& at, int c) {
        load_param<T, KIND>(p.w, p.weight_type, at.c0 + c, p.C, 1.f, w);
        load_param<T, KIND>(p.b, p.weight_type, at.c0 + c, p.C, 0.f, b);
    }
    __device__ __forceinline__ void settle(const Maps& p, const Place& at, int c, const float* mean_r) {
        each_group(c < at.width ? c : at.width - 1, at.width, p.D, [&](int i, int g) {
            const bool there = c + i < at.width;
            m[i] = there ? mean_r[g] : 0.f;
            w[i] = there ? w[i] * mean_r[at.groups + g] : 0.f;
            b[i] = there ? b[i] : 0.f;
        });
    }
    template <class T>
    __device__ __forceinline__ void apply(const Raw<T>& raw, int act_kind, float (&v)[8]) const {
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = fmaf(raw[i] - m[i], w[i], b[i]);
        if (act_kind == FMTC_ACT_RELU) {
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] = act<FMTC_ACT_RELU>(v[i]);
        } else if (act_kind == FMTC_ACT_SILU) {
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] = act<FMTC_ACT_SILU>(v[i]);
        }
    }
};

struct Lane { int ly, lx, c; bool live; };
__device__ __forceinline__ Lane lane_of(const Maps& p, const Place& at) {
    const int t = threadIdx.x, ly = quotient(t, 1.f / (float)p.LX), lx = t - ly * p.LX;
    return {ly, lx, 8 * lx, ly < p.LY && 8 * lx < at.width};
}
template <class T>
__device__ __forceinline__ T* slab_of(void* base, int64_t ld, const Maps& p, const Place& at) {
    return static_cast<T*>(base) + at.n * p.S * ld + at.c0;
}
template <class T>
__device__ __forceinline__ const T* slab_of(const void* base, int64_t ld, const Maps& p, const Place& at) {
    return static_cast<const T*>(base) + at.n * p.S * ld + at.c0;
}

constexpr int kUnroll = 4;  // rows of a thread on their way together

// A slab in the registers of a workgroup, R rows a thread.  256 x 3136 x 64 (32 groups, a ReLU) 42 us (in two passes 64), with inputs
// and results in other memory each time 52.8 us, 3.9 TB/s; 128 x 784 x 256 23 us; 196 x 256 5.2 us, latency.
template <class T, int KIND, bool ONE, int R>
__global__ __launch_bounds__(1024) void k_group_norm_once(Maps p, float eps, int act_kind, T* y, int64_t ld_y, float* __restrict__ stats) {
    extern __shared__ __attribute__((aligned(16))) double red[];
    const Place at(p, 1, 0);
    const Lane me = lane_of(p, at);
    float* const mean_r = reinterpret_cast<float*>(red + (2 << p.pre) * blockDim.x);
    const T* const x = slab_of<T>(p.x, p.ld, p, at);
    Raw<T> raw[R];
    Scale scale;
    double s[8] = {}, q[8] = {};
    if (me.live) {
        Origins<T, ONE> origins;
#pragma unroll
        for (int u = 0; u < R; u++) {
            const int64_t r = me.ly + (int64_t)u * p.LY;
            load_raw<KIND>(raw[u], x + (r < p.S ? r : 0) * p.ld, me.c, at.width);
        }
        origins.load(p, at, me.c);
        constexpr bool kLater = kFromOrigin<T> && !ONE;  // (there are no registers for it beside the origins)
        if constexpr (!kLater) scale.load<T, KIND>(p, at, me.c);
        origins.settle();
#pragma unroll
        for (int u = 0; u < R; u++) {
            settle_raw<KIND>(raw[u], me.c, at.width);
            origins.add(raw[u], me.ly + (int64_t)u * p.LY < p.S, s, q);
        }
        if (me.ly == 0) origins.keep(p, at, me.c, mean_r);
        if constexpr (kLater) scale.load<T, KIND>(p, at, me.c);
    }
    sums_by_group(p, at, me.live, s, q, red, [&](int g, double a, double b) {
        finish(p, at, g, kFromOrigin<T> ? mean_r[g] : 0.0, a, b, eps, mean_r, stats);
    });
    __syncthreads();
    if (!me.live || !y) return;
    scale.settle(p, at, me.c, mean_r);
    T* const out = slab_of<T>(y, ld_y, p, at);
#pragma unroll
    for (int u = 0; u < R; u++) {
        const int64_t r = me.ly + (int64_t)u * p.LY;
        if (r >= p.S) break;
        float v[8];
        scale.apply(raw[u], act_kind, v);
        store8(out + r * ld_y + me.c, KIND != kWhole ? at.width - me.c : 8, v);
    }
}

// The sums of the values (f32: of their distances from the origin) and of the squares, of each part of a sample's rows and each
// group: part[sample][chunk][group], and behind them the origins [sample][group]: the next kernel may write over the values.  512 x
// 512 x 128 12.2 to 13.2 us (5.1 to 5.5 TB/s).
template <class T, int KIND, bool ONE>
__global__ __launch_bounds__(1024) void k_group_norm_sums(Maps p, double2* __restrict__ part) {
    extern __shared__ __attribute__((aligned(16))) double red[];
    const Place at(p, p.chunks, 0);
    const Lane me = lane_of(p, at);
    const int64_t r0 = at.k * p.per, r1 = r0 + p.per < p.S ? r0 + p.per : p.S;
    double s[8] = {}, q[8] = {};
    if (me.live) {
        const T* const x = slab_of<T>(p.x, p.ld, p, at);
        Origins<T, ONE> origins;
        origins.load(p, at, me.c);
        for (int64_t r = r0 + me.ly; r < r1; r += (int64_t)kUnroll * p.LY) {
            Raw<T> raw[kUnroll];
#pragma unroll
            for (int u = 0; u < kUnroll; u++) {
                const int64_t from = r + (int64_t)u * p.LY;
                load_raw<KIND>(raw[u], x + (from < r1 ? from : r) * p.ld, me.c, at.width);
            }
            origins.settle();
#pragma unroll
            for (int u = 0; u < kUnroll; u++) {
                settle_raw<KIND>(raw[u], me.c, at.width);
                origins.add(raw[u], r + (int64_t)u * p.LY < r1, s, q);
            }
        }
        if (at.k == 0 && me.ly == 0) origins.keep(p, at, me.c, reinterpret_cast<float*>(part + p.samples * p.chunks * p.G) + at.n * p.G + at.g0);
    }
    double2* const to = part + (at.n * p.chunks + at.k) * p.G + at.g0;
    sums_by_group(p, at, me.live, s, q, red, [&](int g, double a, double b) { to[g] = make_double2(a, b); });
}

// mean and r of each group of a slab into LDS, and, by the first workgroup of a slab, where the caller wants them
template <class T>
__device__ __forceinline__ void finish_parts(const Maps& p, const Place& at, const double2* part, float eps, float* mean_r, float* stats) {
    const float* const origins = reinterpret_cast<const float*>(part + p.samples * p.chunks * p.G) + at.n * p.G + at.g0;
    spread(at.groups, [&](int g, int l, int lanes) {
        double s = 0.0, q = 0.0;
        const double2* const from = part + at.n * p.chunks * p.G + at.g0 + g;
        for (int64_t k = l; k < p.chunks; k += 8 * lanes) {  // (8 loads on their way together)
            double2 v[8];
#pragma unroll
            for (int j = 0; j < 8; j++) v[j] = from[(k + j * lanes < p.chunks ? k + j * lanes : p.chunks - 1) * p.G];
#pragma unroll
            for (int j = 0; j < 8; j++) {
                s += k + j * lanes < p.chunks ? v[j].x : 0.0;
                q += k + j * lanes < p.chunks ? v[j].y : 0.0;
            }
        }
        s = lanes_sum(s, lanes);
        q = lanes_sum(q, lanes);
        if (l == 0) finish(p, at, g, kFromOrigin<T> ? origins[g] : 0.0, s, q, eps, mean_r, at.k == 0 ? stats : nullptr);
    });
    __syncthreads();
}

// The values again, and y.  512 x 512 x 128 23.8 to 25.2 us (5.3 to 5.6 TB/s of both).
template <class T, int KIND>
__global__ __launch_bounds__(1024) void k_group_norm_apply(Maps p, const double2* __restrict__ part, int64_t parts, int64_t rows, float eps,
                                                           int act_kind, T* y, int64_t ld_y, float* __restrict__ stats) {
    extern __shared__ __attribute__((aligned(16))) float mean_r[];
    const Place at(p, parts, 0);
    const Lane me = lane_of(p, at);
    Scale scale;
    scale.load<T, KIND>(p, at, me.c);
    finish_parts<T>(p, at, part, eps, mean_r, stats);
    if (!y || !me.live) return;
    scale.settle(p, at, me.c, mean_r);
    const int64_t r0 = at.k * rows, r1 = r0 + rows < p.S ? r0 + rows : p.S;
    const T* const x = slab_of<T>(p.x, p.ld, p, at);
    T* const out = slab_of<T>(y, ld_y, p, at);
    for (int64_t r = r0 + me.ly; r < r1; r += (int64_t)kUnroll * p.LY) {
        Raw<T> raw[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; u++) {
            const int64_t from = r + (int64_t)u * p.LY;
            load_raw<KIND>(raw[u], x + (from < r1 ? from : r) * p.ld, me.c, at.width);
        }
#pragma unroll
        for (int u = 0; u < kUnroll; u++) {
            const int64_t to = r + (int64_t)u * p.LY;
            if (to >= r1) break;
            settle_raw<KIND>(raw[u], me.c, at.width);
            float v[8];
            scale.apply(raw[u], act_kind, v);
            store8(out + to * ld_y + me.c, KIND != kWhole ? at.width - me.c : 8, v);
        }
    }
}

// To codes with a scale for each row: TPR lanes hold a row, VPT groups of 8 consecutive channels each.  The statistics come from
// the sums of parts, or (part NULL) are there already.  Bound by the activation's and the codes' instructions: 256 x 49 x 960 f16
// 15.3 us (its bytes 7), 65 x 49 x 960 6.9 us.
constexpr int codes_threads(int TPR) { return TPR < 256 ? 256 : TPR; }
template <class T, int KIND, int TPR, int VPT>
__global__ __launch_bounds__(codes_threads(TPR)) void k_group_norm_codes(Maps p, const double2* __restrict__ part, int64_t parts, int64_t rows,
                                                                         float eps, int act_kind, fmtc_i8 out, float* __restrict__ stats) {
    extern __shared__ __attribute__((aligned(16))) float mean_r[];
    __shared__ uint32_t turns[2][codes_threads(TPR) / 64];
    constexpr int kRows = codes_threads(TPR) / TPR;
    const Place at(p, parts, 0);
    const int lane = threadIdx.x % TPR, width = (p.C + kF8Block - 1) / kF8Block * kF8Block;
    const int64_t r0 = at.k * rows, r1 = r0 + rows < p.S ? r0 + rows : p.S;
    const T* const x = slab_of<T>(p.x, p.ld, p, at);
    Raw<T> next[VPT];
    auto fetch = [&](int64_t r) {
        const int64_t mine = r + threadIdx.x / TPR, from = mine < r1 ? mine : r1 - 1;
#pragma unroll
        for (int j = 0; j < VPT; j++) load_raw<KIND>(next[j], x + from * p.ld, 8 * (j * TPR + lane), p.C);
    };
    fetch(r0);
    Scale scale[VPT];
#pragma unroll
    for (int j = 0; j < VPT; j++) scale[j].template load<T, KIND>(p, at, 8 * (j * TPR + lane));
    if (part) {
        finish_parts<T>(p, at, part, eps, mean_r, stats);
    } else {
        for (int g = threadIdx.x; g < p.G; g += blockDim.x) {
            mean_r[g] = stats[at.n * p.G + g];
            mean_r[p.G + g] = stats[(p.all + at.n) * p.G + g];
        }
        __syncthreads();
    }
#pragma unroll
    for (int j = 0; j < VPT; j++) scale[j].settle(p, at, 8 * (j * TPR + lane), mean_r);
    int turn = 0;
    for (int64_t r = r0; r < r1; r += kRows, turn ^= 1) {  // (all threads take every round: there may be barriers in it)
        const int64_t mine = r + threadIdx.x / TPR, from = mine < r1 ? mine : r1 - 1;
        Raw<T> raw[VPT];
        float v[VPT][8];
        uint32_t m = 0;
#pragma unroll
        for (int j = 0; j < VPT; j++) raw[j] = next[j];
        if (r + kRows < r1) fetch(r + kRows);
#pragma unroll
        for (int j = 0; j < VPT; j++) {
            const int c = 8 * (j * TPR + lane);
            settle_raw<KIND>(raw[j], c, p.C);
            raw[j].zero_unless(c < p.C);
            scale[j].apply(raw[j], act_kind, v[j]);
            const uint32_t b = amax_bits8(v[j]);
            m = b > m ? b : m;
        }
        float held;
        const float inv = i8_row_scale(row_max_bits<TPR>(m, turns[turn]), &held);
        if (mine >= r1) continue;
        const int64_t row = at.n * p.S + from;
#pragma unroll
        for (int j = 0; j < VPT; j++) {
            const int c = 8 * (j * TPR + lane);
            if (c < width)
                *reinterpret_cast<uint2*>(static_cast<uint8_t*>(out.d_codes) + row * out.ld + c) = make_uint2(i8_encode4(v[j], inv), i8_encode4(v[j] + 4, inv));
        }
        if (lane == 0) out.d_scales[row] = held;
    }
}

// ---- gradients ----
// What a thread needs of its 8 channels: x^ = (x - m) r, z = (x - m) a + b with a = w r.  (r stays with its x - m: apart from it,
// as a factor of the sums, values of 1e19 and more or 1e-19 and less leave f32.)
struct Channels {
    float m[8], r[8], a[8], b[8];
    template <class T, int KIND>
    __device__ __forceinline__ void load(const Maps& p, const Place& at, const float* stats, int c) {
        load_param<T, KIND>(p.w, p.weight_type, at.c0 + c, p.C, 1.f, a);
        load_param<T, KIND>(p.b, p.weight_type, at.c0 + c, p.C, 0.f, b);
        const float *const mean = stats + at.n * p.G + at.g0, *const rs = mean + p.all * p.G;
        each_group(c, at.width, p.D, [&](int i, int g) {
            m[i] = mean[g];
            r[i] = rs[g];
            a[i] *= rs[g];
        });
    }
    __device__ __forceinline__ float xh(int i, float x) const { return (x - m[i]) * r[i]; }
    template <int ACT>
    __device__ __forceinline__ float dz(int i, float x, float dy) const {
        return ACT == FMTC_ACT_NONE ? dy : dy * act_gradient<ACT>(fmaf(x - m[i], a[i], b[i]));
    }
};

// The sums of dz (s) and of dz x^ (q) of all threads, by channel of the slab: f(0 or 1, channel, sum) on one thread each.  red:
// 16 floats a thread.
template <class F>
__device__ __forceinline__ void sums_by_channel(const Maps& p, const Place& at, bool live, const float (&s)[8], const float (&q)[8], float* red, F&& f) {
    const int T = blockDim.x;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        red[i * T + threadIdx.x] = live ? s[i] : 0.f;
        red[(8 + i) * T + threadIdx.x] = live ? q[i] : 0.f;
    }
    __syncthreads();
    spread(2 * at.width, [&](int i, int l, int lanes) {
        const int which = i >= at.width, c = i - which * at.width;
        const float* const from = red + (8 * which + c % 8) * T + c / 8;
        float sum = 0.f;
#pragma unroll 8
        for (int y = l; y < p.LY; y += lanes) sum += from[y * p.LX];
        sum = lanes_sum(sum, lanes);
        if (l == 0) f(which, c, sum);
    });
}

template <class T>
__device__ __forceinline__ float weight_at(const Maps& p, int c) {
    return !p.w ? 1.f : p.weight_type == FMTC_F32 ? static_cast<const float*>(p.w)[c] : to_f32(static_cast<const T*>(p.w)[c]);
}
// A and B of each group of the slab from the sums by channel, [2][width] with the weights in them, both in LDS
__device__ __forceinline__ void group_terms(const Maps& p, const Place& at, const float* by_channel, float* ab) {
    const float rcount = 1.f / ((float)p.S * (float)p.D);
    spread(2 * at.groups, [&](int i, int l, int lanes) {
        const int which = i >= at.groups, g = i - which * at.groups;
        float sum = 0.f;
#pragma unroll 8
        for (int c = l; c < p.D; c += lanes) sum += by_channel[which * at.width + g * p.D + c];
        sum = lanes_sum(sum, lanes);
        if (l == 0) ab[i] = sum * rcount;
    });
    __syncthreads();
}
// dx = r (w dz - A - x^ B) = a dz + (x^ D + E):  D = -r B, E = -r A
struct Terms {
    float D[8], E[8];
    __device__ __forceinline__ void load(const Maps& p, const Place& at, const Channels& ch, int c, const float* ab) {
        each_group(c, at.width, p.D, [&](int i, int g) {
            E[i] = -ch.r[i] * ab[g];
            D[i] = -ch.r[i] * ab[at.groups + g];
        });
    }
    __device__ __forceinline__ float dx(const Channels& ch, int i, float x, float dz) const {
        return fmaf(dz, ch.a[i], fmaf(ch.xh(i, x), D[i], E[i]));
    }
};

// A slab in the registers of a workgroup, R rows a thread: x as it is and dz in f32 (an activation's gradient is computed
// once: it costs as much as all the rest).  part[sample][2][C]: the sums by channel.  32 x 3136 x 256, 32 groups, silu 44 us (as
// called 47, with other inputs and results each time 60): its bytes take 30, but they come 32 of a row at a time and the activation's gradient is not all under them; 32 x 1568 x 512, 64
// bytes at a time, 39 us.  In two passes 64 us; computing dz twice 73 us.
template <class T, int KIND, int ACT, int R>
__global__ __launch_bounds__(512) void k_group_norm_backward_once(Maps p, const float* __restrict__ stats, const T* dy, int64_t ld_dy, T* dx,
                                                                  int64_t ld_dx, float* __restrict__ part) {
    extern __shared__ __attribute__((aligned(16))) float red_f[];
    const Place at(p, 1, 0);
    const Lane me = lane_of(p, at);
    float *const by_channel = red_f + 16 * blockDim.x, *const ab = by_channel + 2 * at.width;
    const T *const x = slab_of<T>(p.x, p.ld, p, at), *const g = slab_of<T>(dy, ld_dy, p, at);
    Raw<T> raw[R];
    float dz[R][8], s[8] = {}, q[8] = {};
    Channels ch;
    if (me.live) {
        Raw<T> raw_g[R];
#pragma unroll
        for (int u = 0; u < R; u++) {
            const int64_t r = me.ly + (int64_t)u * p.LY, from = r < p.S ? r : 0;
            load_raw<KIND>(raw[u], x + from * p.ld, me.c, at.width);
            load_raw<KIND>(raw_g[u], g + from * ld_dy, me.c, at.width);
        }
        ch.load<T, KIND>(p, at, stats, me.c);
#pragma unroll
        for (int u = 0; u < R; u++) {
            settle_raw<KIND>(raw[u], me.c, at.width), settle_raw<KIND>(raw_g[u], me.c, at.width);
            raw[u].zero_unless(me.ly + (int64_t)u * p.LY < p.S);
            raw_g[u].zero_unless(me.ly + (int64_t)u * p.LY < p.S);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                dz[u][i] = ch.dz<ACT>(i, raw[u][i], raw_g[u][i]);
                s[i] += dz[u][i];
                q[i] = fmaf(dz[u][i], ch.xh(i, raw[u][i]), q[i]);
            }
            __builtin_amdgcn_sched_barrier(0);  // (row by row: all rows widened at a time are more than the registers hold)
        }
    }
    float* const to = part + at.n * 2 * p.C + at.c0;
    sums_by_channel(p, at, me.live, s, q, red_f, [&](int which, int c, float sum) {
        to[which * p.C + c] = sum;
        by_channel[which * at.width + c] = sum * weight_at<T>(p, at.c0 + c);
    });
    __syncthreads();
    group_terms(p, at, by_channel, ab);
    if (!me.live || !dx) return;
    // (x stays as it is: without this it would be kept widened, and there are no registers for that)
#pragma unroll
    for (int u = 0; u < R; u++)
#pragma unroll
        for (int i = 0; i < Raw<T>::kWords; i++) asm volatile("" : "+v"(raw[u].w[i]));
    Terms terms;
    terms.load(p, at, ch, me.c, ab);
    T* const out = slab_of<T>(dx, ld_dx, p, at);
#pragma unroll
    for (int u = 0; u < R; u++) {
        const int64_t r = me.ly + (int64_t)u * p.LY;
        if (r >= p.S) break;
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = terms.dx(ch, i, raw[u][i], dz[u][i]);
        store8(out + r * ld_dx + me.c, KIND != kWhole ? at.width - me.c : 8, v);
    }
}

// The sums of dz and of dz x^ of each part of a sample's rows and each channel: part[sample][chunk][2][C].
template <class T, int KIND, int ACT>
__global__ __launch_bounds__(1024) void k_group_norm_gradient_sums(Maps p, const float* __restrict__ stats, const T* __restrict__ dy,
                                                                   int64_t ld_dy, float* __restrict__ part) {
    extern __shared__ __attribute__((aligned(16))) float red_f[];
    const Place at(p, p.chunks, 0);
    const Lane me = lane_of(p, at);
    const int64_t r0 = at.k * p.per, r1 = r0 + p.per < p.S ? r0 + p.per : p.S;
    float s[8] = {}, q[8] = {};
    if (me.live) {
        Channels ch;
        ch.load<T, KIND>(p, at, stats, me.c);
        const T *const x = slab_of<T>(p.x, p.ld, p, at), *const g = slab_of<T>(dy, ld_dy, p, at);
        constexpr int U = kUnroll / 2;
        for (int64_t r = r0 + me.ly; r < r1; r += (int64_t)U * p.LY) {
            Raw<T> raw[U], raw_g[U];
#pragma unroll
            for (int u = 0; u < U; u++) {
                const int64_t row = r + (int64_t)u * p.LY, from = row < r1 ? row : r;
                load_raw<KIND>(raw[u], x + from * p.ld, me.c, at.width);
                load_raw<KIND>(raw_g[u], g + from * ld_dy, me.c, at.width);
            }
#pragma unroll
            for (int u = 0; u < U; u++) {
                if (r + (int64_t)u * p.LY >= r1) break;
                settle_raw<KIND>(raw[u], me.c, at.width), settle_raw<KIND>(raw_g[u], me.c, at.width);
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    const float dz = ch.dz<ACT>(i, raw[u][i], raw_g[u][i]);
                    s[i] += dz;
                    q[i] = fmaf(dz, ch.xh(i, raw[u][i]), q[i]);
                }
            }
        }
    }
    float* const to = part + (at.n * p.chunks + at.k) * 2 * p.C + at.c0;
    sums_by_channel(p, at, me.live, s, q, red_f, [&](int which, int c, float sum) { to[which * p.C + c] = sum; });
}

// The sum of from[first], from[first + step].. below n, `apart` from each other, 16 loads on their way together (a loop with a
// remainder would wait for each load of that: 0.7 us each).  V: double over samples, of which there are any number; float over the
// parts of one (128 at most): 7 x 1739 x 161 f32 1 us less.
template <class V>
__device__ __forceinline__ V strided_sum(const float* from, int64_t first, int64_t step, int64_t n, int64_t apart) {
    V sum = 0;
    for (int64_t k = first; k < n; k += 16 * step) {
        float v[16];
#pragma unroll
        for (int j = 0; j < 16; j++) v[j] = from[(k + j * step < n ? k + j * step : n - 1) * apart];
#pragma unroll
        for (int j = 0; j < 16; j++) sum += (V)(k + j * step < n ? v[j] : 0.f);
    }
    return sum;
}

// dbias and dweight: sums over n rows of part, 32 columns a workgroup, slices of the rows, added up in order; with those of the
// launches before this one in sums [2][C], where there are several (first: of the first one)
struct Carry { double* sums; int first; };
__device__ __forceinline__ void param_sums(const float* part, int64_t n, int C, float* dweight, float* dbias, Carry carry, double* slice) {
    const int col = threadIdx.x & 31, k = threadIdx.x >> 5, slices = blockDim.x >> 5, c = blockIdx.x * 32 + col;
    double sum = 0.0;
    if (c < 2 * C) sum = strided_sum<double>(part + c, k, slices, n, 2 * C);
    slice[k * 33 + col] = sum;
    __syncthreads();
    if (k == 0 && c < 2 * C) {
        for (int i = 1; i < slices; i++) sum += slice[i * 33 + col];
        if (carry.sums) {
            if (!carry.first) sum += carry.sums[c];
            carry.sums[c] = sum;
        }
        float* const to = c < C ? dbias : dweight;
        if (to) to[c < C ? c : c - C] = (float)sum;
    }
}
// The sums of every `each` parts by channel: those of a sample, where they are too many for every workgroup of the next kernel to
// add up, or of kEach samples, where there are too many for the few workgroups that the channels make.  32 columns a workgroup.
// to[parts / each][2][C]
__global__ __launch_bounds__(1024) void k_group_norm_join(const float* __restrict__ part, int64_t each, int64_t parts, int C, float* __restrict__ to) {
    __shared__ double slice[32 * 33];
    const int64_t n = blockIdx.y, mine = parts - n * each < each ? parts - n * each : each;
    const int col = threadIdx.x & 31, k = threadIdx.x >> 5, c = blockIdx.x * 32 + col;
    double sum = 0.0;
    if (c < 2 * C) sum = strided_sum<double>(part + n * each * 2 * C + c, k, 32, mine, 2 * C);
    slice[k * 33 + col] = sum;
    __syncthreads();
    if (k == 0 && c < 2 * C) {
#pragma unroll
        for (int i = 1; i < 32; i++) sum += slice[i * 33 + col];
        to[n * 2 * C + c] = (float)sum;
    }
}

__global__ __launch_bounds__(1024) void k_group_norm_params(const float* __restrict__ part, int64_t n, int C, float* __restrict__ dweight,
                                                            float* __restrict__ dbias, Carry carry) {
    __shared__ double slice[32 * 33];
    param_sums(part, n, C, dweight, dbias, carry, slice);
}

// dx from the sums of the parts.  The first `before` workgroups do the sums for dbias and dweight.  7 x 1739 x 161 f32 12.8 us, latency:
// its values set out when the sums over the parts are there (setting out before them gained nothing).
template <class T, int KIND, int ACT>
__global__ __launch_bounds__(1024) void k_group_norm_dx(Maps p, const float* __restrict__ stats, const float* __restrict__ part, int64_t parts,
                                                        int64_t rows, uint32_t before, const T* dy, int64_t ld_dy, T* dx, int64_t ld_dx,
                                                        float* __restrict__ dweight, float* __restrict__ dbias, Carry carry) {
    extern __shared__ __attribute__((aligned(16))) float red_f[];  // [slices][2][width] (or the other sums' slices), then [2][groups]: A and B
    if (blockIdx.x < before) return param_sums(part, p.samples * p.chunks, p.C, dweight, dbias, carry, reinterpret_cast<double*>(red_f));
    const Place at(p, parts, before);
    const int wide = 2 * at.width, t = threadIdx.x, slices = (int)blockDim.x / wide < p.chunks ? (int)blockDim.x / wide : (int)p.chunks;
    float* const ab = red_f + (slices > 1 ? slices : 1) * wide;
    // sums over the chunks: neighbouring threads on neighbouring channels, several slices of the chunks where threads are left
    for (int i = t; i < (slices > 1 ? slices : 1) * wide; i += blockDim.x) {
        const int slice = i / wide, j = i - slice * wide, which = j >= at.width, c = at.c0 + j - which * at.width;
        const float sum = strided_sum<float>(part + at.n * p.chunks * 2 * p.C + which * p.C + c, slice, slices > 1 ? slices : 1, p.chunks, 2 * p.C);
        red_f[i] = sum * weight_at<T>(p, c);
    }
    __syncthreads();
    if (slices > 1) {
        for (int i = t; i < wide; i += blockDim.x)
            for (int k = 1; k < slices; k++) red_f[i] += red_f[k * wide + i];
        __syncthreads();
    }
    group_terms(p, at, red_f, ab);
    const Lane me = lane_of(p, at);
    if (!me.live) return;
    Channels ch;
    ch.load<T, KIND>(p, at, stats, me.c);
    Terms terms;
    terms.load(p, at, ch, me.c, ab);
    const int64_t r0 = at.k * rows, r1 = r0 + rows < p.S ? r0 + rows : p.S;
    const T *const x = slab_of<T>(p.x, p.ld, p, at), *const g = slab_of<T>(dy, ld_dy, p, at);
    T* const out = slab_of<T>(dx, ld_dx, p, at);
    constexpr int U = kUnroll / 2;
    for (int64_t r = r0 + me.ly; r < r1; r += (int64_t)U * p.LY) {
        Raw<T> raw[U], raw_g[U];
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int64_t row = r + (int64_t)u * p.LY, from = row < r1 ? row : r;
            load_raw<KIND>(raw[u], x + from * p.ld, me.c, at.width);
            load_raw<KIND>(raw_g[u], g + from * ld_dy, me.c, at.width);
        }
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int64_t to = r + (int64_t)u * p.LY;
            if (to >= r1) break;
            settle_raw<KIND>(raw[u], me.c, at.width), settle_raw<KIND>(raw_g[u], me.c, at.width);
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] = terms.dx(ch, i, raw[u][i], ch.dz<ACT>(i, raw[u][i], raw_g[u][i]));
            store8(out + to * ld_dx + me.c, KIND != kWhole ? at.width - me.c : 8, v);
        }
    }
}

// ---- which way ----
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

struct Plan {
    int threads, W, rows;     // rows: of a thread, in its registers (0: in two passes)
    int64_t chunks;           // two passes: parts of a sample's rows
    int join;                 // gradients: 1 where a kernel between the two joins the parts
};
constexpr double kCus = 256;
// Every workgroup of the second pass reads the sums of all parts of its sample: 512 workgroups and 128 parts of 512 x 512 x 128
// 39 us, 1024 and 256 47 us, 2048 and 256 53 us.
constexpr int64_t kMostChunks = 128, kSecondPass = 512;

int lanes_of(int W) { return (W + 7) / 8; }
// registers of a thread for a slab: its rows go up in these steps
constexpr int kRowSteps16[] = {1, 2, 4, 8, 13}, kRowSteps32[] = {1, 2, 4, 6};
int row_step(int64_t rows, int size) {
    if (size == 2) {
        for (int r : kRowSteps16) if (rows <= r) return r;
    } else {
        for (int r : kRowSteps32) if (rows <= r) return r;
    }
    return 0;
}

// The least of the times that are expected, in us, from the bytes, the lines of memory that a compute unit takes in for them, and the
// rounds of workgroups.  Over 59 drawn sizes the choice costs 3 % more than the best of all choices would, in the mean.  arrays: read
// (1 forward, 2 backward)
Plan choose(int64_t samples, int64_t S, int C, int groups, int size, int arrays) {
    const int D = C / groups;
    const double values = (double)samples * S * C, bytes = values * size * (arrays + 1);
    Plan best{};
    // two passes: whole rows, cut in slabs where a few samples would need many chunks, whose sums are read again and again
    int W = C;
    auto threads_of = [](int W) { return W > 4096 ? 1024 : 512; };
    auto want = [&](int W) { return ceil_div(512 * 1024 / threads_of(W), samples * ceil_div(C, W)); };
    while (want(W) > 32 && W % 2 == 0 && (W / 2) % D == 0 && (W / 2) * size >= 128 && (W / 2) % 8 == 0) W /= 2;
    best.threads = threads_of(W);
    best.W = W;
    const int64_t rows = ceil_div(S, (int64_t)(kUnroll / arrays) * (best.threads / lanes_of(W)));
    best.chunks = want(W) < rows ? want(W) : rows;
    best.chunks = ceil_div(S, ceil_div(S, best.chunks < kMostChunks ? best.chunks : kMostChunks));
    // (a workgroup's time for the sums over the parts: rounds of its threads, each of several rounds of loads, 0.8 us; a kernel 4)
    best.join = arrays == 2 && best.chunks > 1 && ceil_div(best.chunks, 16) * ceil_div(2 * W, best.threads) > 4;
    double least = 9.0 + (bytes + values * size * arrays * (values * size * arrays > 2e8 ? 1.0 : 0.6)) / 5e6 * (C % 8 ? 1.3 : 1.0);
    // (and the rounds of workgroups past the two or three that the parts make, where there are many samples: 16384 x 16 x 64 215 us,
    // gradients 277, in one pass 31 and 48)
    const double two_rounds = ceil((double)samples * ceil_div(C, W) * best.chunks / (kCus * 1024 / best.threads));
    if (two_rounds > 3) least += (arrays == 1 ? 5.5 : 8.0) * (two_rounds - 2);
    for (int gs = 1;; gs = gs * 2 < groups ? gs * 2 : groups) {
        const int W = gs * D, LX = lanes_of(W);
        // (small workgroups only for whole samples of few rows, and more of them than run at a time: 2^20 x 1 x 64 0.82 ms with 64
        // threads, 3.1 with 256, gradients 1.3 and 3.9; 2048 x 1 x 64 in 8 slabs 16.5 us, whole with 256 threads 9.6)
        const bool tiny = W == C && samples > 4096;
        for (int threads = tiny ? 64 : 256; threads <= (arrays == 1 ? 1024 : 512); threads *= 2) {
            if (threads < 256 && S * LX > threads) continue;
            if (LX > threads || (W < 8 && W != C)) continue;
            const size_t lds = arrays == 1 ? sizeof(double) * (2 << fold_of(D)) * threads + sizeof(float) * 2 * gs : 0;
            if (lds > 159 * 1024) continue;
            const int R = row_step(ceil_div(S, threads / LX), size);
            if (!R) continue;
            const double wgs = (double)samples * ceil_div(groups, gs), at_once = kCus * 1024 / threads;
            const double rounds = ceil(wgs / at_once), segment = W * size, crooked = W % 8 && W != C ? 1.5 : 1.0;
            const double slow = (W == C || segment >= 128 ? 1.0 : segment >= 64 ? 1.05 : segment >= 32 ? 1.2 : 1.6) * crooked;
            const double lines = (W == C || segment >= 128 ? 1.0 : 128.0 / segment) * crooked;  // what a compute unit takes in
            const double mine = bytes / wgs * lines * fmax(1.0, wgs / kCus) / 80e3;
            const double t = 4.0 + 2.5 * rounds * threads / 512 + fmax(bytes * slow / 5e6, mine);
            if (t < least) {
                least = t;
                best.threads = threads;
                best.W = W;
                best.rows = R;
            }
        }
        if (gs == groups) break;
    }
    return best;
}

// A call asks three times for the same sizes (for its workspace, for the check of it, for the launch): 0.4 us each.
Plan make_plan(int64_t samples, int64_t S, int C, int groups, int size, int arrays) {
    struct Last { int64_t samples, S; int C, groups, size, arrays; Plan plan; };
    static thread_local Last last{};
    if (last.samples != samples || last.S != S || last.C != C || last.groups != groups || last.size != size || last.arrays != arrays)
        last = {samples, S, C, groups, size, arrays, choose(samples, S, C, groups, size, arrays)};
    return last.plan;
}

// Samples of a launch: workgroups have a sample each, a grid has less than 2^32 threads, and what lies in the workspace for each
// sample shall not grow without end: sums by group (up to 160 MB), the gradients' sums by channel (64 MB).
constexpr int64_t kMostThreads = ((int64_t)1 << 32) - 1;
int64_t least_of(int64_t a, int64_t b) { return a < b ? a : b; }
int64_t samples_forward(int64_t samples, int groups) { return least_of(samples, least_of((int64_t)1 << 20, ((int64_t)1 << 23) / groups)); }
int64_t samples_backward(int64_t samples, int C) { return least_of(samples, ((int64_t)1 << 23) / (C < 8 ? 8 : C)); }
Maps maps_of(const fmtc_gnorm& a, int64_t all, const Plan& plan) {
    const int LX = lanes_of(plan.W), D = a.C / a.groups;
    return {a.samples, all, a.rows_per_sample, a.ld_x, a.C, a.groups, D, plan.W, plan.W / D, (int)ceil_div(a.C, plan.W), LX, plan.threads / LX, fold_of(D),
            a.d_x, a.d_weight, a.d_bias, a.weight_type, plan.chunks, plan.chunks ? ceil_div(a.rows_per_sample, plan.chunks) : 0};
}
// parts of a sample's rows for the second pass: some rows for every thread, about `want` workgroups in all
int64_t parts_of(const Maps& p, int rows_at_a_time, int unroll, int64_t want) {
    const int64_t fit = ceil_div(p.S, (int64_t)unroll * rows_at_a_time), parts = ceil_div(want, p.samples * p.slabs);
    return ceil_div(p.S, ceil_div(p.S, parts < fit ? parts : fit));
}
template <class F>
hipError_t with_kind(const Maps& p, F&& f) {
    if (p.C % 8 == 0 && p.W % 8 == 0) return f(Int<kWhole>{});
    return p.C - (p.slabs - 1) * p.W >= 8 ? f(Int<kLong>{}) : f(Int<kShort>{});  // (the last slab is the narrowest)
}
template <class F>
hipError_t with_act(int act, F&& f) {
    return act == FMTC_ACT_NONE ? f(Int<FMTC_ACT_NONE>{}) : act == FMTC_ACT_RELU ? f(Int<FMTC_ACT_RELU>{}) : f(Int<FMTC_ACT_SILU>{});
}
template <class T, class F>
hipError_t with_rows(int rows, F&& f) {
    if (rows == 1) return f(Int<1>{});
    if (rows == 2) return f(Int<2>{});
    if (rows == 4) return f(Int<4>{});
    if constexpr (sizeof(T) == 2) return rows == 8 ? f(Int<8>{}) : f(Int<13>{});
    else return f(Int<6>{});
}
template <class... A, class... B>
hipError_t go(int id, void (*kernel)(A...), int64_t grid, int threads, size_t lds, hipStream_t s, B... args) {
    if (lds > 65536) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e != hipSuccess) return e;
    }
    return launch(id, kernel, dim3((unsigned)grid), dim3(threads), lds, s, args...);
}
int type_size(int type) { return type == FMTC_F32 ? 4 : 2; }

}  // namespace

size_t group_norm_workspace(int64_t samples, int64_t S, int C, int groups, int type, bool to_codes) {
    samples = samples_forward(samples, groups);
    const Plan plan = make_plan(samples, S, C, groups, type_size(type), 1);
    // (sums, and the groups' origins)
    if (!plan.rows) return align_up((sizeof(double2) * (size_t)plan.chunks + (type == FMTC_F32 ? sizeof(float) : 0)) * (size_t)samples * groups, 256);
    return to_codes ? align_up(sizeof(float) * 2 * (size_t)samples * groups, 256) : 0;  // (statistics that the caller does not want)
}
// More than kMostParts parts are joined by kEach at a time before the few workgroups that the channels make add them up: 32768 x 64 x
// 128 bf16 440 -> 342 us, 16384 x 49 x 256 328 -> 283.
constexpr int64_t kMostParts = 2048, kEach = 256;
int64_t joined_parts(int64_t parts) { return parts > kMostParts ? ceil_div(parts, kEach) : 0; }
static size_t sums_workspace(int64_t samples, int64_t S, int C, int groups, int type) {  // of a launch
    const Plan plan = make_plan(samples, S, C, groups, type_size(type), 2);  // (in one pass there is one part of a sample)
    const int64_t parts = samples * (plan.rows ? 1 : plan.chunks), joined = plan.join && !plan.rows ? samples : 0;
    return align_up(sizeof(float) * (size_t)(parts + (joined > joined_parts(parts) ? joined : joined_parts(parts))) * 2 * C, 256);
}
size_t group_norm_backward_workspace(int64_t samples, int64_t S, int C, int groups, int type) {
    const int64_t some = samples_backward(samples, C);
    return sums_workspace(some, S, C, groups, type) + (some < samples ? align_up(sizeof(double) * 2 * C, 256) : 0);
}

static hipError_t norm_some(const fmtc_gnorm& a, int64_t all, const Plan& plan, void* d_y, int64_t ld_y, const fmtc_i8* codes, float* d_stats,
                            void* d_ws, hipStream_t s) {
    const bool own_stats = codes && plan.rows && !d_stats;  // (in the workspace)
    Maps p = maps_of(a, own_stats ? a.samples : all, plan);
    double2* const part = static_cast<double2*>(d_ws);
    return with_type(a.type, [&](auto ty) {
        using T = typename decltype(ty)::type;
        return with_kind(p, [&](auto kd) {
            constexpr int R = decltype(kd)::value;
            const size_t lds = sizeof(double) * (2 << p.pre) * plan.threads, lds_stats = sizeof(float) * 2 * p.groups;
            float* const stats = own_stats ? static_cast<float*>(d_ws) : d_stats;
            auto first = [&](auto one) {
                constexpr bool ONE = decltype(one)::value;
                if (plan.rows)
                    return with_rows<T>(plan.rows, [&](auto rows) {
                        return go(K_GROUP_NORM, k_group_norm_once<T, R, ONE, decltype(rows)::value>, p.samples * p.slabs, plan.threads, lds + lds_stats, s,
                                  p, a.eps, a.act, codes ? nullptr : static_cast<T*>(d_y), ld_y, stats);
                    });
                return go(K_GROUP_NORM, k_group_norm_sums<T, R, ONE>, p.samples * p.slabs * p.chunks, plan.threads, lds, s, p, part);
            };
            hipError_t e;
            if constexpr (kFromOrigin<T> && R == kWhole) e = p.pre == 0 ? first(Int<1>{}) : first(Int<0>{});  // (a thread's channels are of one group)
            else e = first(Int<0>{});
            if (e != hipSuccess || (plan.rows && !codes)) return e;
            if (codes) {
                p.W = p.C;  // (rows as a whole)
                p.groups = p.G;
                p.slabs = 1;
                return with_kind(p, [&](auto rows_kind) {
                    auto with = [&](auto tpr, auto vpt) {
                        constexpr int TPR = decltype(tpr)::value, VPT = decltype(vpt)::value;
                        const int64_t parts = parts_of(p, codes_threads(TPR) / TPR, 1, 2048), rows = ceil_div(p.S, parts);
                        return go(K_GROUP_NORM, k_group_norm_codes<T, decltype(rows_kind)::value, TPR, VPT>, p.samples * parts, codes_threads(TPR),
                                  sizeof(float) * 2 * p.G, s, p, plan.rows ? nullptr : part, parts, rows, a.eps, a.act, *codes, stats);
                    };
                    if (p.C <= 128) return with(Int<16>{}, Int<1>{});
                    if (p.C <= 512) return with(Int<64>{}, Int<1>{});
                    if (p.C <= 1024) return with(Int<64>{}, Int<2>{});
                    if (p.C <= 2048) return with(Int<256>{}, Int<1>{});
                    return with(Int<1024>{}, Int<1>{});
                });
            }
            const int64_t parts = d_y ? parts_of(p, p.LY, kUnroll, kSecondPass) : 1, rows = ceil_div(p.S, parts);
            return go(K_GROUP_NORM, k_group_norm_apply<T, R>, p.samples * p.slabs * parts, plan.threads, lds_stats, s, p, part, parts, rows, a.eps,
                      a.act, static_cast<T*>(d_y), ld_y, d_stats);
        });
    });
}

template <class P>
static P* from_row(P* values, int type, int64_t row, int64_t ld) {
    using Byte = typename std::conditional<std::is_const<P>::value, const char, char>::type;
    return values ? static_cast<Byte*>(values) + row * ld * type_size(type) : nullptr;
}
// the samples from n on, `most` at most
static fmtc_gnorm samples_from(const fmtc_gnorm& a, int64_t n, int64_t most) {
    fmtc_gnorm b = a;
    b.samples = a.samples - n < most ? a.samples - n : most;
    b.d_x = from_row(a.d_x, a.type, n * a.rows_per_sample, a.ld_x);
    return b;
}
hipError_t launch_group_norm(const fmtc_gnorm& a, void* d_y, int64_t ld_y, const fmtc_i8* codes, float* d_stats, void* d_ws, hipStream_t s) {
    int64_t most = samples_forward(a.samples, a.groups);
    const Plan plan = make_plan(most, a.rows_per_sample, a.C, a.groups, type_size(a.type), 1);
    most = least_of(most, kMostThreads / (plan.threads * ceil_div(a.C, plan.W) * (plan.rows ? 1 : plan.chunks)));
    hipError_t e = hipSuccess;
    for (int64_t n = 0; n < a.samples && e == hipSuccess; n += most) {
        const int64_t row = n * a.rows_per_sample;
        fmtc_i8 q{};
        if (codes) q = {static_cast<uint8_t*>(codes->d_codes) + row * codes->ld, codes->d_scales + row, codes->rows, codes->depth, codes->ld};
        e = norm_some(samples_from(a, n, most), a.samples, plan, from_row(d_y, a.type, row, ld_y), ld_y, codes ? &q : nullptr,
                      d_stats ? d_stats + n * a.groups : nullptr, d_ws, s);
    }
    return e;
}

static hipError_t backward_some(const fmtc_gnorm& a, int64_t all, const Plan& plan, const float* d_stats, const void* d_dy, int64_t ld_dy, void* d_dx,
                                int64_t ld_dx, float* d_dweight, float* d_dbias, void* d_ws, Carry carry, hipStream_t s) {
    const Maps p = maps_of(a, all, plan);
    float* const part = static_cast<float*>(d_ws);
    return with_type(a.type, [&](auto ty) {
        using T = typename decltype(ty)::type;
        return with_kind(p, [&](auto kd) {
            return with_act(a.act, [&](auto ac) {
                constexpr int R = decltype(kd)::value, A = decltype(ac)::value;
                const T* dy = static_cast<const T*>(d_dy);
                const bool params = d_dweight || d_dbias;
                const int64_t param_groups = params ? ceil_div(2 * p.C, 32) : 0;
                const size_t lds = sizeof(float) * 16 * plan.threads, lds_ab = sizeof(float) * 2 * p.groups;
                auto join = [&](int64_t each, int64_t parts, float* to) {
                    return launch(K_GROUP_NORM_BACKWARD, k_group_norm_join, dim3((unsigned)ceil_div(2 * p.C, 32), (unsigned)ceil_div(parts, each)), dim3(1024), 0, s,
                                  part, each, parts, p.C, to);
                };
                auto sum_params = [&](int64_t n) {
                    if (!params) return hipSuccess;
                    const float* from = part;
                    if (const int64_t joined = joined_parts(n)) {
                        float* const to = part + n * 2 * p.C;
                        const hipError_t e = join(kEach, n, to);
                        if (e != hipSuccess) return e;
                        from = to;
                        n = joined;
                    }
                    return go(K_GROUP_NORM_BACKWARD, k_group_norm_params, param_groups, 1024, 0, s, from, n, p.C, d_dweight, d_dbias, carry);
                };
                if (plan.rows) {
                    const hipError_t e = with_rows<T>(plan.rows, [&](auto rows) {
                        return go(K_GROUP_NORM_BACKWARD, k_group_norm_backward_once<T, R, A, decltype(rows)::value>, p.samples * p.slabs, plan.threads,
                                  lds + sizeof(float) * 2 * p.W + lds_ab, s, p, d_stats, dy, ld_dy, static_cast<T*>(d_dx), ld_dx, part);
                    });
                    return e != hipSuccess ? e : sum_params(p.samples);
                }
                const hipError_t e = go(K_GROUP_NORM_BACKWARD, k_group_norm_gradient_sums<T, R, A>, p.samples * p.slabs * p.chunks, plan.threads, lds, s, p,
                                        d_stats, dy, ld_dy, part);
                if (e != hipSuccess) return e;
                const bool before = d_dx && !joined_parts(p.samples * p.chunks);  // (the parameters' sums by workgroups of the last kernel)
                if (!before) {
                    const hipError_t e = sum_params(p.samples * p.chunks);
                    if (e != hipSuccess || !d_dx) return e;
                }
                Maps joined = p;
                const float* sums_at = part;
                if (plan.join) {
                    float* const to = part + p.samples * p.chunks * 2 * p.C;
                    const hipError_t e = join(p.chunks, p.samples * p.chunks, to);
                    if (e != hipSuccess) return e;
                    joined.chunks = 1;
                    sums_at = to;
                }
                const int64_t parts = parts_of(p, p.LY, kUnroll / 2, kSecondPass), rows = ceil_div(p.S, parts);
                size_t lds_dx = sizeof(float) * (2 * p.W > plan.threads ? 2 * p.W : plan.threads) + lds_ab;
                if (lds_dx < sizeof(double) * 33 * (plan.threads / 32)) lds_dx = sizeof(double) * 33 * (plan.threads / 32);
                const int64_t of_params = before ? param_groups : 0;
                return go(K_GROUP_NORM_BACKWARD, k_group_norm_dx<T, R, A>, of_params + p.samples * p.slabs * parts, plan.threads, lds_dx, s, joined, d_stats,
                          sums_at, parts, rows, (uint32_t)of_params, dy, ld_dy, static_cast<T*>(d_dx), ld_dx, d_dweight, d_dbias, carry);
            });
        });
    });
}

hipError_t launch_group_norm_backward(const fmtc_gnorm& a, const float* d_stats, const void* d_dy, int64_t ld_dy, void* d_dx, int64_t ld_dx,
                                      float* d_dweight, float* d_dbias, void* d_ws, hipStream_t s) {
    const int64_t most = samples_backward(a.samples, a.C);  // (times C / 8 slabs of 512 threads: 2^29)
    const Plan plan = make_plan(most, a.rows_per_sample, a.C, a.groups, type_size(a.type), 2);
    const size_t sums = sums_workspace(most, a.rows_per_sample, a.C, a.groups, a.type);
    double* const carry = most < a.samples ? reinterpret_cast<double*>(static_cast<char*>(d_ws) + sums) : nullptr;
    hipError_t e = hipSuccess;
    for (int64_t n = 0; n < a.samples && e == hipSuccess; n += most) {
        const int64_t row = n * a.rows_per_sample;
        e = backward_some(samples_from(a, n, most), a.samples, plan, d_stats + n * a.groups, from_row(d_dy, a.type, row, ld_dy), ld_dy,
                          from_row(d_dx, a.type, row, ld_dx), ld_dx, d_dweight, d_dbias, d_ws, {carry, n == 0}, s);
    }
    return e;
}

}  // namespace fmtc
