// The norm of many arrays together, and their values scaled to at most a given norm (fmtc_clip):
//   norm = scale sqrt(sum v^2),   out = in f,   f = scale min(1, max_norm / (norm + eps))
// Two passes over the values, for f is known behind the last of them: each workgroup of the first takes a piece of an array
// and leaves its sum, each of the second adds up all sums, in the same order, and scales a piece.  Sums are in f64: the
// squares of f32 and bf16 values leave f32's range, and f64 sums run at the rate of f32 ones here.
// Memory bound: 400e6 values of 2 bytes 142 + 330 us (5.6 and 4.9 TB/s), 1.6e6 of 4 bytes 3.5 + 5 us.  The arrays' addresses travel with the launch, kMost of them at a time: no table has to be kept anywhere.
#include "fmtc_block.h"

namespace fmtc {

namespace {

constexpr int kMost = 128;       // arrays of a launch (kernel arguments are 4096 bytes at most)
constexpr int kThreads = 256;
constexpr int64_t kStep = 8 * kThreads;      // pieces are multiples of it: what a workgroup takes at a time, or twice that
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

// How many values lie before the first one at a multiple of 128 bytes.  Pieces begin at such places: views into one buffer
// begin anywhere, and wide accesses across the lines of the cache cost a third of the rate.
template <class T>
__device__ __forceinline__ int64_t values_before_line(const void* p) {
    return (int64_t)((0 - (uintptr_t)p) % 128 / sizeof(T));
}
// The values of a piece: f(index, values) for V at a time from `lead` on, U loads on their way together, and one(index) for
// each of the few before the first line and behind the last V.
template <class T, int V, int U, class F, class G>
__device__ __forceinline__ void walk(const T* in, int64_t index, int64_t piece, int64_t n, int64_t lead, F&& f, G&& one) {
    constexpr int64_t kEach = V * kThreads;
    const int64_t c1 = lead + (index + 1) * piece < n ? lead + (index + 1) * piece : n;
    int64_t c = lead + index * piece;
    if (index == 0)
        for (int64_t i = threadIdx.x; i < (lead < n ? lead : n); i += kThreads) one(i);
    const int64_t whole = c < c1 ? c + (c1 - c) / V * V : c;
    for (int64_t i = whole + threadIdx.x; i < c1; i += kThreads) one(i);
    c += V * threadIdx.x;
    for (; c + (U - 1) * kEach < whole; c += U * kEach) {
        T raw[U][V];
#pragma unroll
        for (int u = 0; u < U; u++) __builtin_memcpy(raw[u], in + c + u * kEach, sizeof raw[u]);
#pragma unroll
        for (int u = 0; u < U; u++) {
            float v[V];
#pragma unroll
            for (int i = 0; i < V; i++) v[i] = to_f32(raw[u][i]);
            f(c + u * kEach, v);
        }
    }
    for (; c < whole; c += kEach) {
        T raw[V];
        __builtin_memcpy(raw, in + c, sizeof raw);
        float v[V];
#pragma unroll
        for (int i = 0; i < V; i++) v[i] = to_f32(raw[i]);
        f(c, v);
    }
}

// 16 bytes of results, at a multiple of 16 bytes, past the caches, which keep what the first pass read
template <class O, int V>
__device__ __forceinline__ void stream_out(O* p, const float (&v)[V]) {
    typedef uint32_t words __attribute__((ext_vector_type(4)));
    static_assert(V * sizeof(O) == 16);
    O t[V];
#pragma unroll
    for (int i = 0; i < V; i++) t[i] = from_f32<O>(v[i]);
    words w;
    __builtin_memcpy(&w, t, 16);
    __builtin_nontemporal_store(w, reinterpret_cast<words*>(p));
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
    double s0 = 0.0, s1 = 0.0;
    with_kind(a.type[k], [&](auto ty) {
        using T = typename decltype(ty)::type;
        const T* const in = static_cast<const T*>(a.in[k]);
        constexpr int V = 16 / sizeof(T);
        walk<T, V, 4>(in, piece - a.first[k], a.piece, a.n[k], values_before_line<T>(in),
                   [&](int64_t, const float (&v)[V]) {
#pragma unroll
                       for (int i = 0; i < V; i += 2) {
                           s0 = fma((double)v[i], (double)v[i], s0);
                           s1 = fma((double)v[i + 1], (double)v[i + 1], s1);
                       }
                   },
                   [&](int64_t c) {
                       const double v = to_f32(in[c]);
                       s0 = fma(v, v, s0);
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
    // 0 for an infinite norm, whatever max_norm is; 1 where norm + eps is 0 (values of 0, or a scale of 0): not inf / inf and 0 / 0
    const double most = norm + eps, r = most == 0.0 ? 1.0 : __builtin_isinf(norm) ? 0.0 : max_norm / most;
    const float f = (float)(scale * (r > 1.0 ? 1.0 : r));  // (not a number stays that)
    const uint32_t piece = a.pieces - 1 - blockIdx.x;
    const int k = find(a, piece);
    if (f == 1.f && a.in[k] == a.out[k]) return;  // (in place, and nothing changes)
    with_kind(a.type[k], [&](auto ty) {
        with_kind(a.out_type[k], [&](auto to) {
            using T = typename decltype(ty)::type;
            using O = typename decltype(to)::type;
            O* const out = static_cast<O*>(a.out[k]);
            const T* const in = static_cast<const T*>(a.in[k]);
            constexpr int V = 16 / sizeof(O);  // (a wavefront writes whole lines: 200e6 values of 2 bytes to f32 298 -> 225 us)
            walk<T, V, 4>(in, piece - a.first[k], a.piece, a.n[k], values_before_line<O>(out),
                       [&](int64_t c, const float (&v)[V]) {
                           float w[V];
#pragma unroll
                           for (int i = 0; i < V; i++) w[i] = v[i] * f;
                           stream_out(out + c, w);
                       },
                       [&](int64_t c) { out[c] = from_f32<O>(to_f32(in[c]) * f); });
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

// The arrays from *at on that fit a launch, and where the next one begins; base: the pieces of the launches before it
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
    bool write = false;
    hipError_t e = hipSuccess;
    for (int64_t at = 0; at < count && e == hipSuccess;) {
        const List a = take(list, count, piece, &at, n_sums);
        if (a.pieces) e = launch(K_CLIP, k_clip_squares, dim3(a.pieces), dim3(kThreads), 0, s, a, sums);
        n_sums += a.pieces;
        write = write || a.out[0];
    }
    if (e == hipSuccess && d_norm && !write) {
        const List none{};
        return launch(K_CLIP, k_clip_scale, dim3(1), dim3(kThreads), 0, s, none, sums, n_sums, max_norm, scale, eps, d_norm);
    }
    // the last arrays first, whose values were read last
    for (int64_t end = count; end > 0 && write && e == hipSuccess;) {
        int64_t from = end;
        for (int k = 0; from > 0 && k < kMost;) k += list[--from].n != 0;
        int64_t at = from;
        const List a = take(list, end, piece, &at, 0);
        end = from;
        if (!a.pieces) continue;
        e = launch(K_CLIP, k_clip_scale, dim3(a.pieces), dim3(kThreads), 0, s, a, sums, n_sums, max_norm, scale, eps, d_norm);
        d_norm = nullptr;
    }
    return e;
}

}  // namespace fmtc
