// The global norm of a list of gradients, and clipping by it.
//
//   norm = |scale| sqrt(sum over all tensors of g^2);  coef = scale min(1, max_norm / norm);  clip: out = g coef
//
// Squares and sums are in 64 bits: the square of an fp32 gradient need not have one in fp32 (above 2^64, below 2^-75), and of many small terms
// behind a large sum fp32 would lose most.  A first launch leaves one sum for each workgroup, a second of one workgroup adds them in a fixed
// order, so the result is the same from run to run.  Both are bound by memory.
#include <algorithm>
#include <cmath>
#include "kfac_internal.h"
#include "elements.h"

using namespace kfac;

namespace {

constexpr int ITEMS = 100;           // tensors of a launch: the table and the rest of the arguments stay below 4 KB
constexpr int THREADS = 256;
constexpr int BYTES = 16;            // of a vector
constexpr int UNROLL = 4;            // vectors of a thread and chunk
constexpr int MOST = 2048;           // workgroups of a launch that sums

struct GradItem {
    const void *g;
    void *out;
    uint32_t n;                      // elements
    uint32_t first;                  // first chunk
};
struct GradLaunch {
    GradItem item[ITEMS];
    unsigned char gbf[ITEMS], obf[ITEMS];
    int n;
    uint32_t chunks;
    double *part;                    // one sum for each workgroup
    const float *coef;
};
static_assert(sizeof(GradLaunch) <= 4096, "arguments of a launch");

__device__ inline int item_of(const GradLaunch &a, unsigned chunk) {   // the last tensor whose first chunk is not behind this one
    const int lane = threadIdx.x & 63;
    int before = 0;
    for (int i = 0; i < a.n; i += 64) before += __popcll(__ballot(i + lane < a.n && a.item[min(i + lane, ITEMS - 1)].first <= chunk));
    return __builtin_amdgcn_readfirstlane(before - 1);
}

template <typename T> constexpr int64_t chunk_elements() { return (int64_t)THREADS * UNROLL * BYTES / sizeof(T); }

// Elements of a chunk that this thread has, as fp32: UNROLL vectors, zeros behind the tensor's end.
template <typename T, typename F> __device__ inline void each_vector(const void *p, int64_t first, int64_t n, F use) {
    constexpr int N = BYTES / (int)sizeof(T);
    Vec<T, N> r[UNROLL];
    if (first + (int64_t)THREADS * UNROLL * N <= n) {
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) r[u] = load<T, N>(p, first + ((int64_t)u * THREADS + threadIdx.x) * N);
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) use(first + ((int64_t)u * THREADS + threadIdx.x) * N, N, r[u]);
    } else {
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const int64_t i = first + ((int64_t)u * THREADS + threadIdx.x) * N;
            const int in = (int)min((int64_t)N, max(n - i, (int64_t)0));
            r[u] = Vec<T, N>{};
            if (in == N) r[u] = load<T, N>(p, i);
            else
#pragma unroll
                for (int k = 0; k < N; ++k)
                    if (k < in) r[u].x[k] = ((const T *)p)[i + k];
        }
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const int64_t i = first + ((int64_t)u * THREADS + threadIdx.x) * N;
            use(i, (int)min((int64_t)N, max(n - i, (int64_t)0)), r[u]);
        }
    }
}

template <int WAVES> __device__ inline double sum_workgroup(double x, double *shared) {
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) x += __shfl_xor(x, m);
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = x;
    __syncthreads();
    x = 0.0;
    for (int w = 0; w < WAVES; ++w) x += shared[w];
    return x;
}

__global__ __launch_bounds__(THREADS) void norm_kernel(const GradLaunch a) {
    __shared__ double shared[THREADS / 64];
    double sum = 0.0;
    for (unsigned c = blockIdx.x; c < a.chunks; c += gridDim.x) {
        const int id = item_of(a, c);
        const GradItem it = a.item[id];
        const auto square = [&](int64_t, int, const auto &r) {
#pragma unroll
            for (int k = 0; k < (int)(sizeof(r.x) / sizeof(r.x[0])); ++k) {
                const double g = value_of(r.x[k]);
                sum = fma(g, g, sum);
            }
        };
        if (a.gbf[id]) each_vector<unsigned short>(it.g, (int64_t)(c - it.first) * chunk_elements<unsigned short>(), it.n, square);
        else each_vector<float>(it.g, (int64_t)(c - it.first) * chunk_elements<float>(), it.n, square);
    }
    sum = sum_workgroup<THREADS / 64>(sum, shared);
    if (threadIdx.x == 0) a.part[blockIdx.x] = sum;
}

struct NormArgs {
    const double *part;
    int n;
    double max_norm;
    const float *scale;
    float *norm, *coef;
};
constexpr int JOIN = 1024;
__global__ __launch_bounds__(JOIN) void norm_join_kernel(const NormArgs g) {
    __shared__ double shared[JOIN / 64];
    double sum = 0.0;
    for (int i = threadIdx.x; i < g.n; i += JOIN) sum += g.part[i];
    sum = sum_workgroup<JOIN / 64>(sum, shared);
    if (threadIdx.x != 0) return;
    const double scale = g.scale ? (double)*g.scale : 1.0, norm = sqrt(sum) * fabs(scale);
    // (a norm that is NaN makes the coefficient NaN, an infinite one makes it zero)
    const double clip = norm > g.max_norm ? g.max_norm / norm : norm == norm ? 1.0 : norm;
    *g.norm = (float)norm;
    if (g.coef) *g.coef = (float)(scale * clip);
}

template <typename T, typename O> __device__ inline void clip_chunk(const GradItem &it, int64_t first, float coef) {
    each_vector<T>(it.g, first, it.n, [&](int64_t i, int in, const auto &r) {
        constexpr int N = BYTES / (int)sizeof(T);
        Vec<O, N> o;
#pragma unroll
        for (int k = 0; k < N; ++k) o.x[k] = element_of<O>(value_of(r.x[k]) * coef);
        if (in == N) store(it.out, i, o);
        else
#pragma unroll
            for (int k = 0; k < N; ++k)
                if (k < in) ((O *)it.out)[i + k] = o.x[k];
    });
}

// The last chunks first: what the sums read last may still be in the cache.
__global__ __launch_bounds__(THREADS) void clip_kernel(const GradLaunch a) {
    const unsigned c = a.chunks - 1 - blockIdx.x;
    const int id = item_of(a, c);
    const GradItem it = a.item[id];
    const float coef = *a.coef;
    if (coef == 1.f && it.out == it.g) return;
    if (a.gbf[id]) {
        const int64_t first = (int64_t)(c - it.first) * chunk_elements<unsigned short>();
        if (a.obf[id]) clip_chunk<unsigned short, unsigned short>(it, first, coef);
        else clip_chunk<unsigned short, float>(it, first, coef);
    } else {
        const int64_t first = (int64_t)(c - it.first) * chunk_elements<float>();
        if (a.obf[id]) clip_chunk<float, unsigned short>(it, first, coef);
        else clip_chunk<float, float>(it, first, coef);
    }
}

// The launches of a list: up to ITEMS tensors each, tensors longer than 32-bit counts reach in pieces.
constexpr int64_t PIECE = (int64_t)1 << 31;
constexpr unsigned MOST_CHUNKS = 1u << 23;
template <typename F> int each_launch(int n, const kfac_grad_item *items, F launch) {
    GradLaunch a{};
    int64_t elements = 0, bytes = 0, written = 0;
    auto go = [&]() -> int {
        const int rc = a.n > 0 ? launch(a, elements, bytes, written) : KFAC_OK;
        a.n = 0;
        a.chunks = 0;
        elements = bytes = written = 0;
        return rc;
    };
    for (int i = 0; i < n; ++i) {
        const kfac_grad_item &t = items[i];
        const bool bf = t.grad_dtype == KFAC_BF16, obf = t.out_dtype == KFAC_BF16;
        for (int64_t at = 0; at < t.n; at += PIECE) {
            const int64_t len = std::min(PIECE, t.n - at), per = bf ? chunk_elements<unsigned short>() : chunk_elements<float>();
            const unsigned mine = (unsigned)((len + per - 1) / per);
            if (a.n == ITEMS || a.chunks + mine > MOST_CHUNKS) KFAC_CHECK(go());
            a.gbf[a.n] = bf;
            a.obf[a.n] = obf;
            a.item[a.n++] = GradItem{(const char *)t.grad + at * (bf ? 2 : 4), t.out ? (char *)t.out + at * (obf ? 2 : 4) : nullptr, (uint32_t)len, a.chunks};
            a.chunks += mine;
            elements += len;
            bytes += len * (bf ? 2 : 4);
            written += len * (obf ? 2 : 4);
        }
    }
    return go();
}

}  // namespace

size_t kfac_grad_norm_ws_bytes_impl(int n, const kfac_grad_item *items) {
    size_t parts = 0;
    (void)each_launch(n, items, [&](const GradLaunch &a, int64_t, int64_t, int64_t) -> int {
        parts += std::min<size_t>(a.chunks, MOST);
        return KFAC_OK;
    });
    return kfac_align_up(parts * sizeof(double), 256);
}

int kfac_launch_grad_norm_batched(kfac_ctx *ctx, int n, const kfac_grad_item *items, float max_norm, const float *grad_scale, float *norm, float *coef, bool clip) {
    if (kfac_grad_norm_ws_bytes_impl(n, items) > ctx->ws_bytes) return KFAC_EWORKSPACE;
    double *const part = (double *)ctx->ws;
    int parts = 0;
    KFAC_CHECK(each_launch(n, items, [&](GradLaunch &a, int64_t elements, int64_t bytes, int64_t) -> int {
        const unsigned wgs = std::min<unsigned>(a.chunks, MOST);
        a.part = part + parts;
        parts += (int)wgs;
        KfacProfScope prof(ctx, KC_NORM, 2.0 * (double)elements, (double)bytes);
        hipLaunchKernelGGL(norm_kernel, dim3(wgs), dim3(THREADS), 0, ctx->stream, a);
        KFAC_HIP_CHECK(hipGetLastError());
        return KFAC_OK;
    }));
    {
        KfacProfScope prof(ctx, KC_NORM, 0.0, 8.0 * parts);
        hipLaunchKernelGGL(norm_join_kernel, dim3(1), dim3(JOIN), 0, ctx->stream, NormArgs{part, parts, (double)max_norm, grad_scale, norm, coef});
        KFAC_HIP_CHECK(hipGetLastError());
    }
    if (!clip) return KFAC_OK;
    return each_launch(n, items, [&](GradLaunch &a, int64_t elements, int64_t bytes, int64_t written) -> int {
        a.coef = coef;
        KfacProfScope prof(ctx, KC_NORM, (double)elements, (double)(bytes + written));
        hipLaunchKernelGGL(clip_kernel, dim3(a.chunks), dim3(THREADS), 0, ctx->stream, a);
        KFAC_HIP_CHECK(hipGetLastError());
        return KFAC_OK;
    });
}
