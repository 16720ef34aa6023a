// The global norm of a list of gradients, and clipping by it.
//
//   norm = |scale| sqrt(sum over all tensors of g^2);  coef = scale min(1, max_norm / norm);  clip: out = g coef
//
// Squares and sums are in 64 bits: the square of an fp32 gradient need not have one in fp32 (above 2^64, below 2^-75), and of many small terms
// behind a large sum fp32 would lose most.  A first launch leaves one sum for each workgroup; a second adds them in a fixed order, so that the
// result is the same from run to run: one workgroup for the norm alone, every workgroup for itself where it goes on to clip.  Bound by memory; a
// short list by its launches.
#include <algorithm>
#include <cmath>
#include "kfac_internal.h"
#include "elements.h"

using namespace kfac;

namespace {

constexpr int ITEMS = 100;           // tensors of a launch: the table and the rest of the arguments stay below 4 KB
constexpr int THREADS = 256;
constexpr int UNROLL = 4;            // vectors of 16 bytes of a thread and chunk
template <int TH> constexpr int64_t chunk_bytes() { return 16 * TH * UNROLL; }     // of a chunk that TH threads take
constexpr int MOST = 1024;           // workgroups of a launch that sums

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
};
static_assert(sizeof(GradLaunch) <= 4000, "arguments of a launch");

__device__ inline int item_of(const GradLaunch &a, unsigned chunk) {   // the last tensor whose first chunk is not behind this one
    const int lane = threadIdx.x & 63;
    int before = 0;
    for (int i = 0; i < a.n; i += 64) before += __popcll(__ballot(i + lane < a.n && a.item[min(i + lane, ITEMS - 1)].first <= chunk));
    return __builtin_amdgcn_readfirstlane(before - 1);
}

// What a thread has of a chunk: UNROLL vectors as they lie in memory, zeros behind the tensor's end.
struct Raw { Vec<unsigned, 4> v[UNROLL]; };
template <int TH, bool PAST> __device__ inline Raw raw_chunk(const void *p, int64_t first /* byte */, int64_t end, bool bf, int thread) {
    Raw r;
    if (first + chunk_bytes<TH>() <= end) {
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const char *const at = (const char *)p + first + (u * TH + thread) * 16;
            r.v[u] = PAST ? load_past<unsigned, 4>(at, 0) : load<unsigned, 4>(at, 0);
        }
    } else {
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const int64_t at = first + (u * TH + thread) * 16;
            r.v[u] = Vec<unsigned, 4>{};
            if (at + 16 <= end) r.v[u] = load<unsigned, 4>((const char *)p + at, 0);
            else if (bf) {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (at + 2 * k < end) r.v[u].x[k >> 1] |= (unsigned)*(const unsigned short *)((const char *)p + at + 2 * k) << (16 * (k & 1));
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (at + 4 * k < end) r.v[u].x[k] = *(const unsigned *)((const char *)p + at + 4 * k);
            }
        }
    }
    return r;
}
__device__ inline float low_bf16(unsigned x) { return __uint_as_float(x << 16); }
__device__ inline float high_bf16(unsigned x) { return __uint_as_float(x & 0xffff0000u); }

template <int WAVES> __device__ inline double sum_workgroup(double x, double *shared) {
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) x += __shfl_xor(x, m);
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = x;
    __syncthreads();
    x = 0.0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) x += shared[w];
    return x;
}

// The squares of a thread's share of chunks c0, c0 + step, ..  The next chunk is asked for before this one is summed.
template <int TH, bool PAST> __device__ inline double sum_chunks(const GradLaunch &a, unsigned c, unsigned step, int thread) {
    double sum = 0.0;
    if (c >= a.chunks) return sum;
    int id = item_of(a, c);
    const auto ask = [&](unsigned chunk, bool &bf) {
        while (id + 1 < a.n && a.item[id + 1].first <= chunk) ++id;
        const GradItem &it = a.item[id];
        bf = a.gbf[id] != 0;
        return raw_chunk<TH, PAST>(it.g, (chunk - it.first) * chunk_bytes<TH>(), (int64_t)it.n * (bf ? 2 : 4), bf, thread);
    };
    bool bf;
    Raw r = ask(c, bf);
    for (; c < a.chunks; c += step) {
        const Raw now = r;
        const bool now_bf = bf;
        if (c + step < a.chunks) r = ask(c + step, bf);
        if (now_bf) {
#pragma unroll
            for (int u = 0; u < UNROLL; ++u)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const double lo = low_bf16(now.v[u].x[k]), hi = high_bf16(now.v[u].x[k]);
                    sum = fma(lo, lo, sum);
                    sum = fma(hi, hi, sum);
                }
        } else {
#pragma unroll
            for (int u = 0; u < UNROLL; ++u)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const double g = __uint_as_float(now.v[u].x[k]);
                    sum = fma(g, g, sum);
                }
        }
    }
    return sum;
}
// PAST: a list that the cache cannot hold is read past it (537 MB: 79 us instead of 89, 6.8 TB/s); of a shorter one the clipping, or the
// optimizer's step, finds what was read (102 MB: 33 us of clipping instead of 45).
template <bool PAST> __global__ __launch_bounds__(THREADS) void norm_kernel(const GradLaunch a) {
    __shared__ double shared[THREADS / 64];
    const double sum = sum_workgroup<THREADS / 64>(sum_chunks<THREADS, PAST>(a, blockIdx.x, gridDim.x, threadIdx.x), shared);
    if (threadIdx.x == 0) a.part[blockIdx.x] = sum;
}

struct NormArgs {
    const double *part;
    int n;
    double max_norm;
    const float *scale;
    float *norm, *coef;
};
constexpr int EACH = MOST / THREADS;     // sums that a thread asks for together
// The coefficient from the sum of all squares; `writes`: this thread leaves both results.
__device__ inline float finish(const NormArgs &g, double scale, double sum, bool writes) {
    const double norm = sqrt(sum) * fabs(scale);
    // (a norm that is NaN makes the coefficient NaN, an infinite one makes it zero)
    const double clip = norm > g.max_norm ? g.max_norm / norm : norm == norm ? 1.0 : norm;
    const float coef = (float)(scale * clip);
    if (writes) {
        *g.norm = (float)norm;
        if (g.coef) *g.coef = coef;
    }
    return coef;
}
// The same from the workgroups' sums.
__device__ inline float join_sums(const NormArgs &g, bool writes, double *shared) {
    const double scale = g.scale ? (double)*g.scale : 1.0;
    double sum = 0.0;
    for (int i0 = 0; i0 < g.n; i0 += MOST) {
        double x[EACH];
#pragma unroll
        for (int k = 0; k < EACH; ++k) {
            const int i = i0 + k * THREADS + (int)threadIdx.x;
            x[k] = i < g.n ? g.part[i] : 0.0;
        }
#pragma unroll
        for (int k = 0; k < EACH; ++k) sum += x[k];
    }
    return finish(g, scale, sum_workgroup<THREADS / 64>(sum, shared), writes && threadIdx.x == 0);
}
__global__ __launch_bounds__(THREADS) void norm_join_kernel(const NormArgs g) {
    __shared__ double shared[THREADS / 64];
    (void)join_sums(g, true, shared);
}

// N results of a thread from element i on; `in` of them exist.  Stored past the caches, so that what runs next does not wait for them to be written back: 25M gradients in fp32
// into other buffers, one list after another, 53 us, through the caches 69 (the sums after it 35 instead of 20).  What reads the results at once would have found some of
// them there: 63M clipped in place and read again 184 us, through the caches 179.
template <typename O, int N> __device__ inline void put(void *p, int64_t i, int64_t in, const float (&x)[N]) {
    Vec<O, N> o;
#pragma unroll
    for (int k = 0; k < N; ++k) o.x[k] = element_of<O>(x[k]);
    if (in >= N) {
        if constexpr (sizeof(o) == 16) store_past(p, i, o);
        else store(p, i, o);
    } else
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (k < in) ((O *)p)[i + k] = o.x[k];
}

// A thread's share of chunk c of tensor id, times coef.
template <int TH> __device__ inline void clip_chunk(const GradLaunch &a, int id, unsigned c, float coef, int thread) {
    const GradItem &it = a.item[id];
    const bool bf = a.gbf[id] != 0, obf = a.obf[id] != 0;
    const int64_t first = (c - it.first) * chunk_bytes<TH>();
    const Raw r = raw_chunk<TH, true>(it.g, first, (int64_t)it.n * (bf ? 2 : 4), bf, thread);
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
        const int64_t at = first + (u * TH + thread) * 16;
        if (bf) {
            float x[8];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                x[2 * k] = low_bf16(r.v[u].x[k]) * coef;
                x[2 * k + 1] = high_bf16(r.v[u].x[k]) * coef;
            }
            if (obf) put<unsigned short, 8>(it.out, at / 2, it.n - at / 2, x);
            else put<float, 8>(it.out, at / 2, it.n - at / 2, x);
        } else {
            float x[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = __uint_as_float(r.v[u].x[k]) * coef;
            if (obf) put<unsigned short, 4>(it.out, at / 4, it.n - at / 4, x);
            else put<float, 4>(it.out, at / 4, it.n - at / 4, x);
        }
    }
}

// The last chunks first: what was read last may still be in the cache.  Nothing is read a third time here, so the loads go past it.
__global__ __launch_bounds__(THREADS) void clip_kernel(const GradLaunch a, const NormArgs g, bool writes) {
    __shared__ double shared[THREADS / 64];
    const float coef = join_sums(g, writes && blockIdx.x == 0, shared);
    int id = item_of(a, a.chunks - 1 - blockIdx.x);
    for (unsigned q = blockIdx.x; q < a.chunks; q += gridDim.x) {
        const unsigned c = a.chunks - 1 - q;
        while (a.item[id].first > c) --id;
        if (coef == 1.f && a.item[id].out == a.item[id].g) continue;
        clip_chunk<THREADS>(a, id, c, coef, threadIdx.x);
    }
}

// A short list by one workgroup, whose sixteen waves take chunks of 4 KB: two rounds of them for the norm (8 tensors of 16 KB 5.1 us a call instead of 8.4 by two
// launches; a third takes as long, waited for), one where it goes on to clip (4 of them 5.7 instead of 8.9; two rounds 8.3 for 9.0, and no sooner).
constexpr int ALONE = 1024;
constexpr int64_t alone_chunks(bool clip) { return (clip ? 1 : 2) * ALONE / 64; }
template <bool CLIP> __global__ __launch_bounds__(ALONE) void norm_alone_kernel(const GradLaunch a, const NormArgs g) {
    __shared__ double shared[ALONE / 64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const double scale = g.scale ? (double)*g.scale : 1.0;
    const double sum = sum_workgroup<ALONE / 64>(sum_chunks<64, false>(a, wave, ALONE / 64, lane), shared);
    const float coef = finish(g, scale, sum, threadIdx.x == 0);
    if (CLIP)
        for (unsigned c = wave; c < a.chunks; c += ALONE / 64) {
            const int id = item_of(a, c);
            if (coef != 1.f || a.item[id].out != a.item[id].g) clip_chunk<64>(a, id, c, coef, lane);
        }
}

// The launches of a list: up to ITEMS tensors each, tensors longer than 32-bit counts reach in pieces.
constexpr int64_t PIECE = (int64_t)1 << 31;
constexpr unsigned MOST_CHUNKS = 1u << 23;
constexpr double CACHE_BYTES = 256e6;       // of the cache in front of the memory
constexpr unsigned CLIP_WGS = 4096;         // (1024 to 8192 differ by 1 us for 25.6M gradients)
template <typename F> int each_launch(int n, const kfac_grad_item *items, int64_t chunk, F launch) {
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
            const int64_t len = std::min(PIECE, t.n - at), per = chunk / (bf ? 2 : 4);
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
    (void)each_launch(n, items, chunk_bytes<THREADS>(), [&](const GradLaunch &a, int64_t, int64_t, int64_t) -> int {
        parts += std::min<size_t>(a.chunks, MOST);
        return KFAC_OK;
    });
    return kfac_align_up(parts * sizeof(double), 256);
}

int kfac_launch_grad_norm_batched(kfac_ctx *ctx, int n, const kfac_grad_item *items, float max_norm, const float *grad_scale, float *norm, float *coef, bool clip) {
    NormArgs g{(double *)ctx->ws, 0, (double)max_norm, grad_scale, norm, coef};
    double whole = 0.0;
    int64_t shorts = 0;                                   // chunks of a wave
    int tensors = 0;
    for (int i = 0; i < n; ++i) {
        const int64_t bytes = items[i].n * (items[i].grad_dtype == KFAC_BF16 ? 2 : 4);
        whole += (double)bytes;
        shorts += (bytes + chunk_bytes<64>() - 1) / chunk_bytes<64>();
        tensors += bytes > 0;
    }
    if (tensors > 0 && tensors <= ITEMS && shorts <= alone_chunks(clip))
        return each_launch(n, items, chunk_bytes<64>(), [&](GradLaunch &a, int64_t elements, int64_t bytes, int64_t written) -> int {
            KfacProfScope prof(ctx, KC_NORM, (clip ? 3.0 : 2.0) * (double)elements, (double)(bytes + (clip ? written : 0)));
            hipLaunchKernelGGL((clip ? norm_alone_kernel<true> : norm_alone_kernel<false>), dim3(1), dim3(ALONE), 0, ctx->stream, a, g);
            KFAC_HIP_CHECK(hipGetLastError());
            return KFAC_OK;
        });
    if (kfac_grad_norm_ws_bytes_impl(n, items) > ctx->ws_bytes) return KFAC_EWORKSPACE;
    KFAC_CHECK(each_launch(n, items, chunk_bytes<THREADS>(), [&](GradLaunch &a, int64_t elements, int64_t bytes, int64_t) -> int {
        const unsigned wgs = std::min<unsigned>(a.chunks, MOST);
        a.part = (double *)ctx->ws + g.n;
        g.n += (int)wgs;
        KfacProfScope prof(ctx, KC_NORM, 2.0 * (double)elements, (double)bytes);
        hipLaunchKernelGGL((whole > CACHE_BYTES ? norm_kernel<true> : norm_kernel<false>), dim3(wgs), dim3(THREADS), 0, ctx->stream, a);
        KFAC_HIP_CHECK(hipGetLastError());
        return KFAC_OK;
    }));
    if (!clip || g.n == 0) {
        KfacProfScope prof(ctx, KC_NORM, 0.0, 8.0 * g.n);
        hipLaunchKernelGGL(norm_join_kernel, dim3(1), dim3(THREADS), 0, ctx->stream, g);
        KFAC_HIP_CHECK(hipGetLastError());
        return KFAC_OK;
    }
    bool first = true;
    return each_launch(n, items, chunk_bytes<THREADS>(), [&](GradLaunch &a, int64_t elements, int64_t bytes, int64_t written) -> int {
        KfacProfScope prof(ctx, KC_NORM, (double)elements, (double)(bytes + written));
        hipLaunchKernelGGL(clip_kernel, dim3(std::min<unsigned>(a.chunks, CLIP_WGS)), dim3(THREADS), 0, ctx->stream, a, g, first);
        KFAC_HIP_CHECK(hipGetLastError());
        first = false;
        return KFAC_OK;
    });
}
