// The norm of many arrays together, and their values scaled to at most a given norm (fmtc_clip):
//   norm = scale sqrt(sum v^2),   out = in f,   f = scale min(1, max_norm / (norm + eps))
// Two passes over the values, for f is known behind the last of them: each workgroup of the first takes a piece of an array
// and leaves its sum, each of the second adds up all sums, in the same order, and scales a piece.  Sums are in f64: the
// squares of f32 and bf16 values leave f32's range, and f64 sums run at the rate of f32 ones here.
// Memory bound.  The arrays' addresses travel with the launch, kMost of them at a time: no table has to be kept anywhere.
#include "fmtc_block.h"

namespace fmtc {

namespace {

constexpr int kMost = 128;       // arrays of a launch (kernel arguments are 4096 bytes at most)
constexpr int kThreads = 256;
constexpr int64_t kStep = 8 * kThreads;      // values that a workgroup takes at a time
constexpr int64_t kPieces = 2048;            // about as many pieces as run at a time

struct List {
    const void* in[kMost];
    void* out[kMost];
    int64_t n[kMost];
    uint32_t first[kMost];  // the first piece of each, ~0 behind the last
    uint8_t type[kMost], out_type[kMost];
    int64_t piece;          // values of a piece, a multiple of kStep
    uint32_t base, pieces;  // of this launch: the first sum, how many
};
static_assert(sizeof(List) <= 4000);

__device__ __forceinline__ int find(const List& a, uint32_t piece) {
    const int lane = threadIdx.x & 63;
    const uint64_t lo = __ballot(a.first[lane] <= piece), hi = __ballot(a.first[lane + 64] <= piece);
    return __builtin_amdgcn_readfirstlane(__popcll(lo) + __popcll(hi) - 1);
}

__device__ __forceinline__ double block_sum(double v, double* part) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int i = 1; i < kThreads / 64; i++) v += part[i];
    return v;
}

// values [c0, c1) of an array of n: f(index, values) for 8 at a time, U loads on their way together
template <class T, int U, class F>
__device__ __forceinline__ void walk(const T* in, int64_t c0, int64_t c1, int64_t n, F&& f) {
    int64_t c = c0 + 8 * threadIdx.x;
    for (; c - 8 * threadIdx.x + U * kStep <= c1; c += U * kStep) {
        Raw<T> raw[U];
#pragma unroll
        for (int u = 0; u < U; u++) raw[u].template load<false>(in, c + u * kStep, n);
#pragma unroll
        for (int u = 0; u < U; u++) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] = raw[u][i];
            f(c + u * kStep, v);
        }
    }
    for (; c < c1; c += kStep) {
        float v[8];
        load8<true>(in, c, n, v);
        f(c, v);
    }
}

template <class F>
__device__ __forceinline__ void with_kind(int type, F&& f) {
    if (type == FMTC_F32) f(Type<float>{});
    else if (type == FMTC_BF16) f(Type<bf16>{});
    else f(Type<_Float16>{});
}

__global__ __launch_bounds__(kThreads) void k_clip_squares(List a, double* __restrict__ sums) {
    __shared__ double part[kThreads / 64];
    const uint32_t piece = blockIdx.x;
    const int k = find(a, piece);
    const int64_t n = a.n[k], c0 = (int64_t)(piece - a.first[k]) * a.piece, c1 = c0 + a.piece < n ? c0 + a.piece : n;
    double s0 = 0.0, s1 = 0.0;
    with_kind(a.type[k], [&](auto ty) {
        using T = typename decltype(ty)::type;
        walk<T, 4>(static_cast<const T*>(a.in[k]), c0, c1, n, [&](int64_t, const float (&v)[8]) {
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                s0 = fma((double)v[i], (double)v[i], s0);
                s1 = fma((double)v[i + 1], (double)v[i + 1], s1);
            }
        });
    });
    const double s = block_sum(s0 + s1, part);
    if (threadIdx.x == 0) sums[a.base + piece] = s;
}

// Pieces in the opposite order: what the first pass read last is still in the memory-side cache.
__global__ __launch_bounds__(kThreads) void k_clip_scale(List a, const double* __restrict__ sums, uint32_t n_sums, double max_norm,
                                                         double scale, double eps, float* __restrict__ norm_out) {
    __shared__ double part[kThreads / 64];
    double s = 0.0;
    for (uint32_t i = threadIdx.x; i < n_sums; i += kThreads) s += sums[i];
    const double norm = scale * sqrt(block_sum(s, part));
    if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
    if (blockIdx.x >= a.pieces) return;
    const double r = max_norm / (norm + eps);
    const float f = (float)(scale * (r > 1.0 ? 1.0 : r));  // (not a number stays that)
    const uint32_t piece = a.pieces - 1 - blockIdx.x;
    const int k = find(a, piece);
    if (f == 1.f && a.in[k] == a.out[k]) return;  // (in place, and nothing changes)
    const int64_t n = a.n[k], c0 = (int64_t)(piece - a.first[k]) * a.piece, c1 = c0 + a.piece < n ? c0 + a.piece : n;
    with_kind(a.type[k], [&](auto ty) {
        with_kind(a.out_type[k], [&](auto to) {
            using T = typename decltype(ty)::type;
            using O = typename decltype(to)::type;
            O* const out = static_cast<O*>(a.out[k]);
            walk<T, 4>(static_cast<const T*>(a.in[k]), c0, c1, n, [&](int64_t c, const float (&v)[8]) {
                float w[8];
#pragma unroll
                for (int i = 0; i < 8; i++) w[i] = v[i] * f;
                store8(out + c, n - c, w);
            });
        });
    });
}

int64_t piece_values(const fmtc_tensor* list, int64_t count) {
    int64_t total = 0;
    for (int64_t i = 0; i < count; i++) total += list[i].n;
    const int64_t steps = (total + kStep * kPieces - 1) / (kStep * kPieces);
    return kStep * (steps < 2 ? 2 : steps);
}
int64_t pieces_of(int64_t n, int64_t piece) { return (n + piece - 1) / piece; }

// The arrays from *at on that fit a launch
List take(const fmtc_tensor* list, int64_t count, int64_t piece, int64_t* at, uint32_t base) {
    List a{};
    a.piece = piece;
    a.base = base;
    int k = 0;
    for (; *at < count && k < kMost; ++*at) {
        const fmtc_tensor& t = list[*at];
        if (t.n == 0) continue;
        a.in[k] = t.d_in;
        a.out[k] = t.d_out;
        a.n[k] = t.n;
        a.first[k] = a.pieces;
        a.type[k] = (uint8_t)t.type;
        a.out_type[k] = (uint8_t)t.out_type;
        a.pieces += (uint32_t)pieces_of(t.n, piece);
        k++;
    }
    for (; k < kMost; k++) a.first[k] = ~0u;
    return a;
}

}  // namespace

size_t clip_workspace(const fmtc_tensor* list, int64_t count) {
    const int64_t piece = piece_values(list, count);
    int64_t sums = 0;
    for (int64_t i = 0; i < count; i++) sums += pieces_of(list[i].n, piece);
    return align_up(sizeof(double) * (size_t)sums, 256);
}

hipError_t launch_clip(const fmtc_tensor* list, int64_t count, double max_norm, double scale, double eps, float* d_norm, void* d_ws, hipStream_t s) {
    const int64_t piece = piece_values(list, count);
    double* const sums = static_cast<double*>(d_ws);
    uint32_t n_sums = 0;
    hipError_t e = hipSuccess;
    for (int64_t at = 0; at < count && e == hipSuccess;) {
        const List a = take(list, count, piece, &at, n_sums);
        if (a.pieces) e = launch(K_CLIP, k_clip_squares, dim3(a.pieces), dim3(kThreads), 0, s, a, sums);
        n_sums += a.pieces;
    }
    bool write = false;
    for (int64_t i = 0; i < count; i++) write = write || (list[i].d_out && list[i].n);
    if (e == hipSuccess && d_norm && !write) {
        List none{};
        return launch(K_CLIP, k_clip_scale, dim3(1), dim3(kThreads), 0, s, none, sums, n_sums, max_norm, scale, eps, d_norm);
    }
    if (!write) return e;
    for (int64_t at = 0; at < count && e == hipSuccess;) {
        const List a = take(list, count, piece, &at, 0);
        if (!a.pieces) continue;
        e = launch(K_CLIP, k_clip_scale, dim3(a.pieces), dim3(kThreads), 0, s, a, sums, n_sums, max_norm, scale, eps, d_norm);
        d_norm = nullptr;
    }
    return e;
}

}  // namespace fmtc
