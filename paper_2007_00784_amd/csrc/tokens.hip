// Tokens to experts and back: the router's choice with its gradient, tokens sorted by expert, the weighted sum of the experts' results
// with its gradients.  Token t has k slots s = t k + j, each for an expert ids[s] or for none, and the sample matrices of the products for
// layers of experts have one row for each slot that has an expert: those of expert 0 first, each expert's in the order of the slots.
//
//   route         ids = the k largest of p = softmax(logits[t]), weights p[ids] (or those over their sum)
//   route_grad    dlogits = p (.) (dw at ids - <p, dw>)
//   dispatch      offsets, rows[s], Xs[rows[s]] = X[t]
//   combine       Y[t] = add[t] + sum_j w[s] Ys[rows[s]]
//   combine_grad  dYs[rows[s]] = w[s] dY[t],  dw[s] = <dY[t], Ys[rows[s]]>
//
// Everything is bound by memory (training batches) or by the length of a launch's chain of loads (single tokens).
#include <algorithm>
#include <climits>
#include <cmath>
#include <type_traits>
#include "kfac_internal.h"
#include "elements.h"

using namespace kfac;

namespace {

constexpr int THREADS = 256;
constexpr unsigned MOST_WGS = 1u << 23;      // of a launch, which has fewer than 2^32 threads: longer batches go in several

// launch(first token, workgroups) for all tokens, `tok` to a workgroup.
template <typename F> int each_launch(int64_t T, int tok, F launch) {
    for (int64_t first = 0; first < T; first += (int64_t)MOST_WGS * tok) {
        launch((int)first, (unsigned)std::min<int64_t>(MOST_WGS, (T - first + tok - 1) / tok));
        KFAC_HIP_CHECK(hipGetLastError());
    }
    return KFAC_OK;
}

// ---------------------------------------------------------------- the router's choice
// A group of L lanes takes a token, each lane V logits, so what has to cross lanes is one value a choice.  A lane's logits lie in vectors of N (16 bytes) that
// follow one another from lane to lane: element v of a lane is number lane N + place(v).  (With V consecutive ones a lane 65536 x 512 in fp32 took
// 43 us, and stores past the caches of the gradient, 16 bytes of every 128, 315.)
template <typename T, int V> constexpr int vector_of() { return V * (int)sizeof(T) < 16 ? V : 16 / (int)sizeof(T); }
template <typename T, int L, int V> __device__ constexpr int place(int v) {
    constexpr int N = vector_of<T, V>();
    return v / N * (L * N) + v % N;
}

// The largest, the smallest, the sum over a group of 4 to 64 lanes, in all of them: inside a row of sixteen by the cross-lane moves.
template <int L, typename F> __device__ inline unsigned group_fold(unsigned x, F fold) {
#define KFAC_GROUP_STEP(ctrl) x = fold(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, ctrl, 0xf, 0xf, true))
    KFAC_GROUP_STEP(0xB1);               // lanes 1 0 3 2
    KFAC_GROUP_STEP(0x4E);               // lanes 2 3 0 1
    if (L >= 8) KFAC_GROUP_STEP(0x141);      // the other four of each eight
    if (L >= 16) KFAC_GROUP_STEP(0x140);     // the other eight of the sixteen
#undef KFAC_GROUP_STEP
#pragma unroll
    for (int m = 16; m < L; m <<= 1) x = fold(x, (unsigned)__shfl_xor((int)x, m));
    return x;
}
template <int L> __device__ inline unsigned group_max(unsigned x) {
    return group_fold<L>(x, [](unsigned a, unsigned b) { return max(a, b); });
}
template <int L> __device__ inline unsigned group_min(unsigned x) {
    return group_fold<L>(x, [](unsigned a, unsigned b) { return min(a, b); });
}
template <int L> __device__ inline float group_sum(float x) {
    return __uint_as_float(group_fold<L>(__float_as_uint(x), [](unsigned a, unsigned b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }));
}

// Logits as unsigned numbers of the same order: a NaN counts as +inf, -0 as 0.
constexpr unsigned MASKED = 0x007fffffu;                  // -inf
__device__ inline unsigned ordered(float x) {
    x = x == x ? x + 0.f : INFINITY;
    const unsigned u = __float_as_uint(x);
    return u ^ ((unsigned)((int)u >> 31) | 0x80000000u);
}
__device__ inline float logit_of(unsigned key) { return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key); }

// exp(d) for d <= 0.  With U = 2^-24 of the result: the product's rounding moves it by |d| U at most, the constant's by 0.23 |d| U, the instruction by 2 U (results
// below 2^-126 are 0; infinity less infinity is NaN).  Of a softmax's sum that is little: the average of |d| over the softmax itself is at most ln E (its entropy
// is that average plus the logarithm of the sum, and at most ln E), so a sum over 128 experts is off by 8 U, of 4096 by 12, as rounding its additions may.
__device__ inline float exp_below(float d) { return __builtin_amdgcn_exp2f(d * 1.44269504f); }
// The same within 3 U however far d is, for what is a result by itself: what the product and its constant leave out is made good behind the instruction.  (A chosen logit
// 80 below the largest had a weight that was off by 100 U.  Infinity, and infinity less infinity, give 0.)
__device__ inline float exp_far(float d) {
    d = fmaxf(d, -150.f);                                 // (infinity has no such rest)
    const float p = d * 1.44269504f, rest = fmaf(d, 1.92596303e-8f, fmaf(d, 1.44269504f, -p)), r = __builtin_amdgcn_exp2f(p);
    return fmaf(r, rest * 0.693147181f, r);
}

// A lane's logits of a token (base: lane N), -inf behind the last.
template <typename T, int L, int V> __device__ inline void logits_of(const void *p, int64_t row, int base, int E, bool in, float (&x)[V]) {
    constexpr int N = vector_of<T, V>();
    if (in && base + (V / N - 1) * L * N + N <= E) {
        Vec<T, N> r[V / N];
#pragma unroll
        for (int u = 0; u < V / N; ++u) r[u] = load<T, N>(p, row + base + u * L * N);
#pragma unroll
        for (int v = 0; v < V; ++v) x[v] = value_of(r[v / N].x[v % N]);
    } else {
#pragma unroll
        for (int u = 0; u < V / N; ++u) {
            const int at = base + u * L * N;
            if (in && at + N <= E) {
                const auto r = load<T, N>(p, row + at);
#pragma unroll
                for (int n = 0; n < N; ++n) x[u * N + n] = value_of(r.x[n]);
            } else {
#pragma unroll
                for (int n = 0; n < N; ++n) x[u * N + n] = in && at + n < E ? value_of(((const T *)p)[row + at + n]) : -INFINITY;
            }
        }
    }
}

struct RouteArgs {
    const void *logits;
    int64_t ldl;
    int T, E, k, normalize;
    int *ids;
    float *weights;
};

// The largest that are left of a group's V L keys, one after another.
// bf16: value and index fit one key, the lower index the larger, so all keys differ and the next one is the largest below the last: the largest
// difference to it modulo 2^32, which is what every key below it has more of than any above.
template <typename T, int L, int V> struct Choice;
template <int L, int V> struct Choice<unsigned short, L, V> {
    unsigned key[V], last;
    __device__ Choice(const float (&x)[V], int base) {
        // the value as a whole number from -inf = 0 on: the bf16's magnitude with its sign, so that -0 is 0, plus that of infinity; NaN is above, and cut to it
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const unsigned u = __float_as_uint(x[v]);
            const int m = (int)u >> 31;
            const unsigned s = (((u & 0x7fff0000u) ^ (unsigned)m) - (unsigned)m) + 0x7f800000u;
            key[v] = min(s, 0xff000000u) | (unsigned)(0xffff - base - place<unsigned short, L, V>(v));
        }
        last = 0;                                         // (the first: the largest difference to 2^32)
    }
    // whether there is one that is not masked; its logit and index
    __device__ bool next(float &logit, int &e) {
        unsigned most = 0;
#pragma unroll
        for (int v = 0; v < V; ++v) most = max(most, key[v] - last);
        const unsigned now = group_max<L>(most) + last;
        const bool some = now > 0xffffu && (last == 0 || now < last);
        last = some ? now : 1;                            // (below every key: nothing is left from here on)
        const int s = (int)((now & 0xffff0000u) - 0x7f800000u);
        logit = __uint_as_float(s < 0 ? (unsigned)-s | 0x80000000u : (unsigned)s);
        e = 0xffff - (int)(now & 0xffffu);
        return some;
    }
};
// fp32: the largest value first, then the lowest index that has it.
template <int L, int V> struct Choice<float, L, V> {
    unsigned key[V];
    int base;
    __device__ Choice(const float (&x)[V], int b) : base(b) {
#pragma unroll
        for (int v = 0; v < V; ++v) key[v] = ordered(x[v]);
    }
    __device__ bool next(float &logit, int &e) {
        unsigned most = 0;
#pragma unroll
        for (int v = 0; v < V; ++v) most = max(most, key[v]);
        most = group_max<L>(most);
        unsigned at = UINT_MAX;
#pragma unroll
        for (int v = V - 1; v >= 0; --v) at = key[v] == most ? (unsigned)place<float, L, V>(v) : at;
        at = group_min<L>(at == UINT_MAX ? at : at + base);
#pragma unroll
        for (int v = 0; v < V; ++v) key[v] = at - base == (unsigned)place<float, L, V>(v) ? 0u : key[v];
        logit = logit_of(most);
        e = (int)at;
        return most > MASKED;
    }
};

// Slots of a token in a lane, lane j % L has slot j: one, where the slots are no more than the lanes, or as many as there can be (k <= 64, and at most E).
template <int L, int V, bool ONE> constexpr int slots_of_lane() { return ONE ? 1 : ((L * V < 64 ? L * V : 64) + L - 1) / L; }

template <typename T, int L, int V, bool ONE> __global__ __launch_bounds__(THREADS) void route_kernel(const RouteArgs g) {
    constexpr int C = slots_of_lane<L, V, ONE>();
    const int lane = threadIdx.x % L, base = lane * vector_of<T, V>();
    const int64_t t = (int64_t)blockIdx.x * (THREADS / L) + threadIdx.x / L;
    const bool in = t < g.T;
    float x[V];
    logits_of<T, L, V>(g.logits, t * g.ldl, base, g.E, in, x);
    Choice<T, L, V> choice(x, base);
    int id[C];
    float w[C], top = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        id[c] = -1;
        w[c] = -INFINITY;
        for (int j = c * L; j < min(g.k, (c + 1) * L); ++j) {
            float logit;
            int e;
            const bool some = choice.next(logit, e);
            if (j == 0) top = some ? logit : 0.f;
            if (j - c * L == lane && some) {
                id[c] = e;
                w[c] = logit;
            }
        }
    }
    float total = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c) w[c] = exp_far(w[c] - top);
    if (g.normalize) {                                    // (top infinite: nothing but zeros, and zero over zero is NaN)
#pragma unroll
        for (int c = 0; c < C; ++c) total += w[c];
    } else {
#pragma unroll
        for (int v = 0; v < V; ++v) total += exp_below(x[v] - top);
    }
    total = group_sum<L>(total);
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int j = c * L + lane;
        if (in && j < g.k) {
            g.ids[t * g.k + j] = id[c];
            g.weights[t * g.k + j] = id[c] >= 0 ? w[c] / total : 0.f;
        }
    }
}

struct RouteGradArgs {
    const void *logits;
    int64_t ldl;
    int T, E, k, normalize;
    const int *ids;
    const float *dw;
    void *out;
    int64_t ldo;
};

// What the slots give to the experts meets in LDS, a row of L V numbers for each token: one slot after another, so that an expert that occurs more than once
// gets its sum in the order of the slots.  Stored past the caches: 65536 x 512 in bf16, normalised, one batch after another, 16 us, through them 24 (fp32 27 and 39); with the
// product that reads the results at once 70 us, through them 59.
template <typename T, int L, int V, bool ONE> __global__ __launch_bounds__(THREADS) void route_grad_kernel(const RouteGradArgs g) {
    constexpr int N = vector_of<T, V>(), C = slots_of_lane<L, V, ONE>();
    __shared__ float rows[THREADS / L][L * V];
    float *const row = rows[threadIdx.x / L];
    const int lane = threadIdx.x % L, base = lane * N;
    const int64_t t = (int64_t)blockIdx.x * (THREADS / L) + threadIdx.x / L;
    const bool in = t < g.T;
    const T *const logits = (const T *)g.logits + t * g.ldl;
#pragma unroll
    for (int v = 0; v < V; ++v) row[base + place<T, L, V>(v)] = 0.f;
    float x[V], d[V], top = 0.f, sum = 0.f;
    bool some = true;
    if (!g.normalize) {
        logits_of<T, L, V>(g.logits, t * g.ldl, base, g.E, in, x);
        unsigned most = 0;
#pragma unroll
        for (int v = 0; v < V; ++v) most = max(most, ordered(x[v]));
        most = group_max<L>(most);
        some = most > MASKED;                            // (all masked: the gradient is zero)
        top = some ? logit_of(most) : 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            x[v] = exp_far(x[v] - top);
            sum += x[v];
        }
        sum = group_sum<L>(sum);
    }
    int id[C];
    float y[C];
    const int chunks = (g.k + L - 1) / L;
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int j = c * L + lane;
        id[c] = -1;
        y[c] = 0.f;
        if (c < chunks && in && j < g.k) {
            const int e = g.ids[t * g.k + j];
            id[c] = (unsigned)e < (unsigned)g.E ? e : -1;
            y[c] = g.dw[t * g.k + j];
        }
    }
    if (g.normalize) {
        // the softmax over the slots
        float p[C], inner = 0.f;
        unsigned most = 0;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            p[c] = c < chunks && id[c] >= 0 ? value_of(logits[id[c]]) : -INFINITY;
            most = max(most, ordered(p[c]));
        }
        most = group_max<L>(most);
        some = most > MASKED;
        top = some ? logit_of(most) : 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            p[c] = exp_far(p[c] - top);
            sum += p[c];
            inner = fmaf(p[c], id[c] >= 0 ? y[c] : 0.f, inner);
        }
        sum = group_sum<L>(sum);
        inner = group_sum<L>(inner) / sum;
#pragma unroll
        for (int c = 0; c < C; ++c) y[c] = some ? p[c] / sum * (y[c] - inner) : 0.f;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");     // (a wave's accesses to LDS keep their order; L lanes of one wave share a row)
#pragma unroll
    for (int c = 0; c < C; ++c) {
        if (c >= chunks) continue;
        for (int j = 0; j < min(L, g.k - c * L); ++j) {
            if (j == lane && id[c] >= 0) row[id[c]] += y[c];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
        }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) d[v] = row[base + place<T, L, V>(v)];
    if (!g.normalize) {
        const float over = some ? 1.f / sum : 0.f;
        float inner = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            x[v] *= over;
            inner = fmaf(x[v], d[v], inner);
        }
        inner = group_sum<L>(inner);
#pragma unroll
        for (int v = 0; v < V; ++v) d[v] = x[v] * (d[v] - inner);
    }
    if (!in) return;
#pragma unroll
    for (int u = 0; u < V / N; ++u) {
        const int at = base + u * L * N;
        if (at + N <= g.E) {
            Vec<T, N> r;
#pragma unroll
            for (int n = 0; n < N; ++n) r.x[n] = element_of<T>(d[u * N + n]);
            if constexpr (sizeof(r) == 16) store_past(g.out, t * g.ldo + at, r);
            else store(g.out, t * g.ldo + at, r);
        } else {
#pragma unroll
            for (int n = 0; n < N; ++n)
                if (at + n < g.E) ((T *)g.out)[t * g.ldo + at + n] = element_of<T>(d[u * N + n]);
        }
    }
}

// ---------------------------------------------------------------- the order of the slots
struct SortArgs {
    const int *ids;
    int S, E, k;             // slots, experts, slots of a token
    int per, runs;           // slots of a run (a workgroup's), runs
    int *offsets;            // [E + 1]
    int *rows;               // [S]
    int *count;              // [runs][E]: slots of the expert in a run
    int *base;               // [runs][E]: the row of the first of them.  (One run: both lie where the offsets do.)
};

__device__ inline int expert_of(int id, int E) { return (unsigned)id < (unsigned)E ? id : E; }

// Sixty-four slots in a wave's order, one a lane: how many of the same expert are in front of it in the run, whose counts so far stand in `seen`.
// The lanes of one expert are found by the ballots of its number's bits.
__device__ inline int rank_in_run(int e, int bits, int *seen) {
    unsigned long long same = ~0ull;
    for (int b = 0; b < bits; ++b) {
        const unsigned long long set = __ballot((e >> b) & 1);
        same &= (e >> b) & 1 ? set : ~set;
    }
    const int before = __popcll(same & ((1ull << (threadIdx.x & 63)) - 1));
    const int had = seen[e];
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // (all lanes have read before one writes: a wave's LDS accesses keep their order)
    if (before == 0) seen[e] = had + __popcll(same);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    return had + before;
}

// Exclusive sums over the lanes of a workgroup of WAVES waves, and the total; `shared`: WAVES ints.
template <int WAVES> __device__ inline int scan_workgroup(int x, int *shared, int &total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int incl = x;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(incl, d);
        if (lane >= d) incl += o;
    }
    if (lane == 63) shared[wave] = incl;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        if (w < wave) before += shared[w];
        total += shared[w];
    }
    __syncthreads();
    return before + incl - x;
}

constexpr int SCAN = 1024;        // threads of a workgroup that sorts, at most
constexpr int STEPS = 4;          // of a wave over its slots that stay in registers
// A run's slots, its waves' one after another: how many of its own expert are in front of each in the run (rows), and of each expert in all (count).
// ALONE: a single run, E <= SCAN: the whole order, offsets and all.
template <bool ALONE> __global__ __launch_bounds__(SCAN) void sort_count_kernel(const SortArgs g) {
    extern __shared__ int shared[];                       // [waves][E + 1]
    __shared__ int sums[SCAN / 64];
    const int n = blockDim.x >> 6, wave = threadIdx.x >> 6, lane = threadIdx.x & 63, pitch = g.E + 1;
    int *const seen = shared + wave * pitch;
    const int span = g.per / n;                           // of a wave, a multiple of 64
    const int64_t first = (int64_t)blockIdx.x * g.per + (int64_t)wave * span;
    const int64_t last = min(first + span, (int64_t)g.S);
    const int bits = 32 - __builtin_clz(g.E);             // of 0 .. E
    int e[STEPS], rank[STEPS];
    if (span <= 64 * STEPS)
#pragma unroll
        for (int a = 0; a < STEPS; ++a) {
            const int64_t s = first + 64 * a + lane;
            e[a] = s < last ? expert_of(g.ids[s], g.E) : g.E;
        }
    for (int i = threadIdx.x; i < n * pitch; i += blockDim.x) shared[i] = 0;
    __syncthreads();
    if (span <= 64 * STEPS) {
#pragma unroll
        for (int a = 0; a < STEPS; ++a)
            if (first + 64 * a < last) rank[a] = rank_in_run(e[a], bits, seen);
    } else
        for (int64_t s0 = first; s0 < last; s0 += 64 * STEPS) {
#pragma unroll
            for (int a = 0; a < STEPS; ++a) {
                const int64_t s = s0 + 64 * a + lane;
                e[a] = s < last ? expert_of(g.ids[s], g.E) : g.E;
            }
#pragma unroll
            for (int a = 0; a < STEPS; ++a) {
                const int64_t s = s0 + 64 * a + lane;
                const int r = rank_in_run(e[a], bits, seen);
                if (s < last) g.rows[s] = e[a] < g.E ? r : -1;
            }
        }
    __syncthreads();
    // what the waves in front of one have of an expert, in the place of what it has itself
    int row = 0;
    if (ALONE) {
        int whole = 0, total;
        if ((int)threadIdx.x < g.E)
            for (int w = 0; w < n; ++w) whole += shared[w * pitch + threadIdx.x];
        row = scan_workgroup<SCAN / 64>(whole, sums, total);
        if (threadIdx.x == 0) g.offsets[g.E] = total;
        if ((int)threadIdx.x < g.E) g.offsets[threadIdx.x] = row;
    }
    for (int c = threadIdx.x; c < g.E; c += blockDim.x) {
        if (!ALONE) row = 0;
        for (int w = 0; w < n; ++w) {
            const int had = shared[w * pitch + c];
            shared[w * pitch + c] = row;
            row += had;
        }
        if (!ALONE) g.count[(int64_t)blockIdx.x * g.E + c] = row;
    }
    __syncthreads();
    if (span <= 64 * STEPS) {
#pragma unroll
        for (int a = 0; a < STEPS; ++a) {
            const int64_t s = first + 64 * a + lane;
            if (s < last) g.rows[s] = e[a] < g.E ? seen[e[a]] + rank[a] : -1;
        }
    } else
        for (int64_t s = first + lane; s < last; s += 64) {
            const int r = g.rows[s];
            if (r >= 0) g.rows[s] = r + seen[g.ids[s]];
        }
}

// The counts of the runs become the rows at which each run's slots of an expert begin.  A workgroup takes SLICE experts, and adds up all counts of those before;
// a single one takes slice after slice (which it has to where the counts lie in the place of the offsets).
constexpr int SLICE = 64, SHARES = SCAN / SLICE;          // sixteen threads share an expert's runs
constexpr int EACH = 8;                                   // counts that a thread asks for together
__global__ __launch_bounds__(SCAN) void sort_scan_kernel(const SortArgs g) {
    __shared__ int part[SHARES][SLICE], sums[SCAN / 64], start[SLICE];
    const int col = threadIdx.x % SLICE, share = threadIdx.x / SLICE;
    const int each = (g.runs + SHARES - 1) / SHARES, r0 = min(share * each, g.runs), r1 = min(r0 + each, g.runs);
    int below = 0;                                        // rows of the experts before the slice
    for (int e0 = blockIdx.x * SLICE; e0 < g.E; e0 += gridDim.x * SLICE) {
        const int e = e0 + col;
        if (gridDim.x > 1) {
            int wide = 16, sum = 0;                       // threads for a run's counts, four each
            while (wide * 4 < e0 && wide < SCAN) wide *= 2;
            const int q = threadIdx.x % wide * 4, step = SCAN / wide;
            for (int r = threadIdx.x / wide; r < g.runs && q < e0; r += EACH * step) {
                Vec<int, 4> c[EACH] = {};
#pragma unroll
                for (int i = 0; i < EACH; ++i)
                    if (r + i * step < g.runs) c[i] = load<int, 4>(g.count, (int64_t)(r + i * step) * g.E + q);
#pragma unroll
                for (int i = 0; i < EACH; ++i) sum += c[i].x[0] + c[i].x[1] + c[i].x[2] + c[i].x[3];
            }
            (void)scan_workgroup<SCAN / 64>(sum, sums, below);
        }
        int c[EACH], whole = 0;                           // this thread's runs of the expert, the first EACH of them
#pragma unroll
        for (int i = 0; i < EACH; ++i) c[i] = e < g.E && r0 + i < r1 ? g.count[(int64_t)(r0 + i) * g.E + e] : 0;
#pragma unroll
        for (int i = 0; i < EACH; ++i) whole += c[i];
        part[share][col] = whole;
        __syncthreads();
        if (threadIdx.x < SLICE) {                        // one wave: the shares in their order, then the experts
            int at = 0;
#pragma unroll
            for (int i = 0; i < SHARES; ++i) {
                const int had = part[i][col];
                part[i][col] = at;
                at += had;
            }
            int incl = at;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const int o = __shfl_up(incl, d);
                if (col >= d) incl += o;
            }
            start[col] = below + incl - at;
            if (e < g.E) g.offsets[e] = below + incl - at;
            if (e == g.E - 1) g.offsets[g.E] = below + incl;
            if (col == SLICE - 1) sums[0] = below + incl;
        }
        __syncthreads();
        int row = start[col] + part[share][col];
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (e < g.E && r0 + i < r1) {
                g.base[(int64_t)(r0 + i) * g.E + e] = row;
                row += c[i];
            }
        below = sums[0];
        __syncthreads();
    }
}

__device__ inline int ranked_row(const SortArgs &g, unsigned s) {
    const int local = g.rows[s];
    return local < 0 ? -1 : g.base[(int64_t)(s / (unsigned)g.per) * g.E + g.ids[s]] + local;
}
__global__ __launch_bounds__(THREADS) void sort_rows_kernel(const SortArgs g) {
    const unsigned s = blockIdx.x * THREADS + threadIdx.x;
    if (s < (unsigned)g.S) g.rows[s] = ranked_row(g, s);
}

// ---------------------------------------------------------------- rows of tokens to rows of experts
struct MoveArgs {
    int T, k, R, d;          // tokens, slots of a token, rows of the experts' matrices, width
    int first;               // the launch's first token
    const int *rows;         // [T][k]
    const float *w;          // [T][k] or NULL
    const void *x;           // the tokens' matrix, or the experts' (combine)
    int64_t ldx;
    const void *y;           // combine: what is added, or NULL; combine_grad: the experts' results
    int64_t ldy;
    void *out;
    int64_t ldo;
    float *dw;               // combine_grad
    int part;                // vectors of a row that a workgroup takes (a launch's second dimension goes over them)
    SortArgs sort;           // dispatch
};

// Where a workgroup gets the rows of its slots from: they are given; or the runs' counts and first rows are; or there are so few slots that
// every workgroup counts those in front of its own, and a launch needs no other before it.
enum { GIVEN = 0, RANKED = 1, COUNTED = 2 };
constexpr int FEW_SLOTS = 2048;      // (512 x 4 tokens of 4096 bf16 8.2 us in one launch, 9.7 to 10.3 in two; 4096 slots: as long in one)

// The offsets from the counts of all slots, by the launch's last workgroup.
__device__ inline void count_offsets(const SortArgs &g, const int *expert /* LDS */, int *count /* LDS, [E] */, int *waves) {
    for (int e = threadIdx.x; e < g.E; e += THREADS) count[e] = 0;
    __syncthreads();
    for (int s = threadIdx.x; s < g.S; s += THREADS)
        if (expert[s] < g.E) atomicAdd(&count[expert[s]], 1);      // (whole numbers: the order changes nothing)
    __syncthreads();
    const int each = (g.E + THREADS - 1) / THREADS, e0 = min((int)threadIdx.x * each, g.E), e1 = min(e0 + each, g.E);
    int sum = 0, total;
    for (int e = e0; e < e1; ++e) sum += count[e];
    int at = scan_workgroup<THREADS / 64>(sum, waves, total);
    for (int e = e0; e < e1; ++e) {
        g.offsets[e] = at;
        at += count[e];
    }
    if (threadIdx.x == 0) g.offsets[g.E] = total;
}

// A row in vectors of N elements that begin anywhere.  What is left at its end, less than a vector, is the end of a vector that begins N in front of the
// row's end, whose first elements are another's.  (Loads are whole vectors then.  With a path of its own for single elements, which a wave went through
// besides the other, the sum of 20000 x 6 rows of 700 bf16 took 69 us instead of 46.)  A row shorter than a vector is one of single elements, N = 1.
template <int N> struct Row {
    int d, whole;
    __device__ explicit Row(int width) : d(width), whole(width / N) {}
    __device__ int vectors() const { return whole + (d % N != 0); }
    __device__ int column(int q) const { return q < whole ? q * N : d - N; }
    __device__ int others(int q) const { return q < whole ? 0 : N - d % N; }
};
template <typename T, int N, bool PAST> __device__ inline Vec<T, N> fetch(const void *p, int64_t i) {
    if constexpr (PAST && N > 1) return load_past<T, N>(p, i);
    else return load<T, N>(p, i);
}
// Stored past the caches, so that nothing that runs next waits for it to be written back, and what was read stays.  Large matrices gain by it also with the product that reads
// them next (134 MB of copies and that product 168 us, through the caches 176; 98 MB 137 and 139), smaller ones lose there (67 MB 92 and 76, 34 MB 79 and 74) what passes over one
// input after another gain.
template <typename T, int N> __device__ inline void put(void *p, int64_t i, const Vec<T, N> &r) {
    if constexpr (N > 1) store_past(p, i, r);
    else store(p, i, r);
}
template <typename T, int N> __device__ inline Vec<T, N> rounded(const float (&x)[N]) {
    Vec<T, N> r;
#pragma unroll
    for (int n = 0; n < N; ++n) r.x[n] = element_of<T>(x[n]);
    return r;
}

// Xs[rows[s]] = X[t]: every token is read once and stored k times, past the caches.  LANES lanes take a token, a vector each at a time; the first is asked for
// before the rows are known.  16384 x 4 rows of 4096 bf16 that no cache holds: 121 us, 5.5 TB/s, as much as a copy with such stores; with two
// vectors a lane 128, with plain stores 124 (and 132 instead of 104 where X is in the cache).
template <typename T, int N, int LANES, int MODE> __global__ __launch_bounds__(THREADS) void scatter_kernel(const MoveArgs g) {
    constexpr int TOK = THREADS / LANES;
    extern __shared__ int shared[];                       // rows of the workgroup's slots [TOK k]; COUNTED: experts of all slots [S], counts [E]
    __shared__ int waves[THREADS / 64];
    const int64_t t0 = g.first + (int64_t)blockIdx.x * TOK, t = t0 + threadIdx.x / LANES;
    const int mine = (int)min((int64_t)TOK, max((int64_t)g.T - t0, (int64_t)0)) * g.k;
    const Row<N> row(g.d);
    const int q0 = blockIdx.y * g.part + (int)(threadIdx.x % LANES), q1 = t < g.T ? min(row.vectors(), ((int)blockIdx.y + 1) * g.part) : 0;
    Vec<T, N> r;
    if (q0 < q1) r = load<T, N>(g.x, t * g.ldx + row.column(q0));
    if (MODE == COUNTED) {
        int *const expert = shared + TOK * g.k;
        for (int s = threadIdx.x; s < g.sort.S; s += THREADS) expert[s] = expert_of(g.sort.ids[s], g.sort.E);
        __syncthreads();
        if (blockIdx.x == gridDim.x - 1) {
            if (blockIdx.y == 0) count_offsets(g.sort, expert, expert + g.sort.S, waves);
            return;
        }
        const int lane = threadIdx.x & 63;
        for (int i = threadIdx.x >> 6; i < mine; i += THREADS / 64) {
            const int s = (int)t0 * g.k + i, e = expert[s];
            int at = 0;
            for (int o = 0; o < g.sort.S; o += 64) {
                const int f = o + lane < g.sort.S ? expert[o + lane] : g.sort.E;
                at += __popcll(__ballot(f < e || (f == e && o + lane < s)));
            }
            if (lane == 0) {
                shared[i] = at = e < g.sort.E ? at : -1;
                if (blockIdx.y == 0) g.sort.rows[s] = at;
            }
        }
    } else {
        for (int i = threadIdx.x; i < mine; i += THREADS) {
            const int64_t s = t0 * g.k + i;
            const int at = MODE == RANKED ? ranked_row(g.sort, (unsigned)s) : g.rows[s];
            if (MODE == RANKED) g.sort.rows[s] = at;
            shared[i] = at;
        }
    }
    __syncthreads();
    const int *const rows = shared + threadIdx.x / LANES * g.k;
    for (int q = q0; q < q1; q += LANES) {
        const Vec<T, N> now = r;
        if (q + LANES < q1) r = load<T, N>(g.x, t * g.ldx + row.column(q + LANES));
        for (int j = 0; j < g.k; ++j) {
            const int at = rows[j];
            if ((unsigned)at < (unsigned)g.R) put<T, N>(g.out, at * g.ldo + row.column(q), now);
        }
    }
}

// Rows and weights of a workgroup's slots in LDS: a row outside the matrix is -1.
__device__ inline void slots_of(const MoveArgs &g, int64_t t0, int mine, int *rows, float *w) {
    for (int i = threadIdx.x; i < mine; i += blockDim.x) {
        const int row = g.rows[t0 * g.k + i];
        rows[i] = (unsigned)row < (unsigned)g.R ? row : -1;
        w[i] = g.w ? g.w[t0 * g.k + i] : 1.f;
    }
    __syncthreads();
}

// Y[t] = add[t] + sum_j w[s] Ys[rows[s]]: sums in fp32 in the order of j, rounded once.  KB rows are asked for at a time, U vectors of each.
template <typename T, int N, int LANES, int KB, bool PAST> __global__ __launch_bounds__(THREADS) void combine_kernel(const MoveArgs g) {
    constexpr int TOK = THREADS / LANES, U = 2;
    extern __shared__ int shared[];
    float *const weights = (float *)(shared + TOK * g.k);
    const int64_t t0 = g.first + (int64_t)blockIdx.x * TOK, t = t0 + threadIdx.x / LANES;
    const Row<N> row(g.d);
    const int q0 = blockIdx.y * g.part + (int)(threadIdx.x % LANES), q1 = t < g.T ? min(row.vectors(), ((int)blockIdx.y + 1) * g.part) : 0;
    slots_of(g, t0, (int)min((int64_t)TOK, (int64_t)g.T - t0) * g.k, shared, weights);
    const int *const rows = shared + threadIdx.x / LANES * g.k;
    const float *const w = weights + threadIdx.x / LANES * g.k;
    for (int q = q0; q < q1; q += LANES * U) {
        Vec<T, N> a[U] = {};
        if (g.y)
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (q + u * LANES < q1) a[u] = fetch<T, N, PAST>(g.y, t * g.ldy + row.column(q + u * LANES));
        float sum[U][N];
        for (int j0 = 0; j0 < g.k; j0 += KB) {
            Vec<T, N> x[KB][U];
#pragma unroll
            for (int j = 0; j < KB; ++j) {
                const int at = rows[min(j0 + j, g.k - 1)];
                if (at >= 0)
#pragma unroll
                    for (int u = 0; u < U; ++u)
                        if (q + u * LANES < q1) x[j][u] = fetch<T, N, PAST>(g.x, at * g.ldx + row.column(q + u * LANES));
            }
            if (j0 == 0)
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int n = 0; n < N; ++n) sum[u][n] = value_of(a[u].x[n]);
#pragma unroll
            for (int j = 0; j < KB; ++j)
                if (j0 + j < g.k && rows[j0 + j] >= 0)
#pragma unroll
                    for (int u = 0; u < U; ++u)
#pragma unroll
                        for (int n = 0; n < N; ++n) sum[u][n] = fmaf(w[j0 + j], value_of(x[j][u].x[n]), sum[u][n]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int v = q + u * LANES;
            if (v >= q1) continue;
            const Vec<T, N> o = rounded<T>(sum[u]);
            const int64_t at = t * g.ldo + row.column(v);
            if (row.others(v) == 0) put<T, N>(g.out, at, o);
            else                                          // (the others' elements may be what is added, not yet read)
#pragma unroll
                for (int n = 0; n < N; ++n)
                    if (n >= row.others(v)) ((T *)g.out)[at + n] = o.x[n];
        }
    }
}

// dYs[rows[s]] = w[s] dY[t] and dw[s] = <dY[t], Ys[rows[s]]>, KB slots of a token at a time.  A lane's share of a product is summed in fp32 in
// the order of the columns, the lanes' then by halves: the same order from run to run.
template <typename T, int N, int LANES, int KB, bool PAST> __global__ __launch_bounds__(std::max(THREADS, LANES)) void combine_grad_kernel(const MoveArgs g) {
    constexpr int BLOCK = std::max(THREADS, LANES), TOK = BLOCK / LANES, WAVES = LANES / 64;
    extern __shared__ int shared[];
    __shared__ float partial[BLOCK / 64][KB];
    float *const weights = (float *)(shared + TOK * g.k);
    const int64_t t0 = g.first + (int64_t)blockIdx.x * TOK, t = t0 + threadIdx.x / LANES;
    const bool there = t < g.T;
    const Row<N> row(g.d);
    const int lane = threadIdx.x % LANES, q1 = there ? row.vectors() : 0;
    Vec<T, N> first;                                      // of dY, asked for before the rows are known
    if (lane < q1) first = fetch<T, N, PAST>(g.x, t * g.ldx + row.column(lane));
    slots_of(g, t0, (int)min((int64_t)TOK, (int64_t)g.T - t0) * g.k, shared, weights);
    const int *const rows = shared + threadIdx.x / LANES * g.k;
    const float *const w = weights + threadIdx.x / LANES * g.k;
    for (int j0 = 0; j0 < g.k; j0 += KB) {
        float dot[KB];
#pragma unroll
        for (int j = 0; j < KB; ++j) dot[j] = 0.f;
        for (int q = lane; q < q1; q += LANES) {
            const int c = row.column(q);
            const Vec<T, N> dy = q == lane ? first : fetch<T, N, PAST>(g.x, t * g.ldx + c);
            Vec<T, N> x[KB];
#pragma unroll
            for (int j = 0; j < KB; ++j)
                if (j0 + j < g.k && rows[j0 + j] >= 0) x[j] = fetch<T, N, PAST>(g.y, rows[j0 + j] * g.ldy + c);
            float v[N];                                   // what is another's has its place in the stored vector, not in the sum
            const int others = row.others(q);
#pragma unroll
            for (int n = 0; n < N; ++n) v[n] = n >= others ? value_of(dy.x[n]) : 0.f;
#pragma unroll
            for (int j = 0; j < KB; ++j)
                if (j0 + j < g.k && rows[j0 + j] >= 0)
#pragma unroll
                    for (int n = 0; n < N; ++n) dot[j] = n >= others ? fmaf(v[n], value_of(x[j].x[n]), dot[j]) : dot[j];
            __builtin_amdgcn_sched_barrier(0);            // (stores between the loads: 229 us instead of 220 for 16384 x 4 rows of 4096 bf16)
#pragma unroll
            for (int j = 0; j < KB; ++j)
                if (j0 + j < g.k && rows[j0 + j] >= 0) {
                    float o[N];
#pragma unroll
                    for (int n = 0; n < N; ++n) o[n] = w[j0 + j] * value_of(dy.x[n]);
                    put<T, N>(g.out, rows[j0 + j] * g.ldo + c, rounded<T>(o));
                }
        }
#pragma unroll
        for (int j = 0; j < KB; ++j) {
            dot[j] = group_sum<(LANES < 64 ? LANES : 64)>(dot[j]);
            if (LANES > 64 && (threadIdx.x & 63) == 0) partial[threadIdx.x >> 6][j] = dot[j];
        }
        if (LANES > 64) __syncthreads();
        if (there && lane < KB && j0 + lane < g.k) {
            float s = 0.f;
            if (LANES > 64) {
                for (int v = 0; v < WAVES; ++v) s += partial[threadIdx.x / LANES * WAVES + v][lane];
            } else {
#pragma unroll
                for (int j = 0; j < KB; ++j) s = j == lane ? dot[j] : s;
            }
            g.dw[t * g.k + j0 + lane] = s;
        }
        if (LANES > 64) __syncthreads();
    }
}

// Lanes for a token: a power of two from 8 to 256, for `each` vectors of its row a lane: two where rows are read (sums of 65536 x 2 rows of 256 bf16 19 us instead of
// 29 with twice the lanes), one where they are stored (65536 x 8 rows of 100 fp32 74 us instead of 92: parts of cache lines go out alone).
int lanes_of(int vectors, int each) {
    int lanes = 8;
    while (lanes < THREADS && lanes * each < vectors) lanes *= 2;
    return lanes;
}
// Vectors of a row that a workgroup takes: a few long rows are cut until 512 workgroups share them, into parts of a vector for each lane at least.
int part_of(int T, int vectors, int lanes) {
    const int tok = THREADS / lanes;
    const int64_t wgs = ((int64_t)T + tok - 1) / tok;
    const int most = (vectors + lanes - 1) / lanes, want = (int)std::max<int64_t>(1, 512 / std::max<int64_t>(wgs, 1));
    const int parts = std::max(1, std::min(most, want)), steps = std::max(1, (most + parts - 1) / parts);
    return steps * lanes;
}

template <typename T, int N, int MODE> auto scatter_of(int lanes) {
    if constexpr (MODE == COUNTED) return scatter_kernel<T, N, THREADS, MODE>;
    else if constexpr (N == 1) return scatter_kernel<T, 1, 8, MODE>;
    else return lanes == 8 ? scatter_kernel<T, N, 8, MODE> : lanes == 16 ? scatter_kernel<T, N, 16, MODE> : lanes == 32 ? scatter_kernel<T, N, 32, MODE>
              : lanes == 64 ? scatter_kernel<T, N, 64, MODE> : lanes == 128 ? scatter_kernel<T, N, 128, MODE> : scatter_kernel<T, N, 256, MODE>;
}
template <typename T, int N, int MODE> int launch_scatter(kfac_ctx *ctx, MoveArgs g, double bytes) {
    // (counting takes longer than copying, so a workgroup has the slots of one token: 256 x 4 of 512 bf16 4.7 us, with four tokens 8.6)
    const int vectors = (g.d + N - 1) / N, lanes = MODE == COUNTED ? THREADS : lanes_of(vectors, 1), tok = THREADS / lanes;
    g.part = MODE == RANKED ? 1 << 30 : part_of(g.T, vectors, lanes);     // (a second workgroup of a slot would find its rank replaced)
    const unsigned parts = MODE == RANKED ? 1 : std::max(1, (vectors + g.part - 1) / g.part);     // (no columns: the order of the slots alone)
    const size_t lds = 4 * ((size_t)tok * g.k + (MODE == COUNTED ? g.sort.S + g.sort.E : 0));
    const auto kernel = scatter_of<T, N, MODE>(lanes);
    KfacProfScope prof(ctx, KC_TOKENS, 0.0, bytes);
    if (MODE == COUNTED) {                                // (one workgroup more, for the offsets)
        hipLaunchKernelGGL(kernel, dim3((g.T + tok - 1) / tok + 1, parts), dim3(THREADS), lds, ctx->stream, g);
        KFAC_HIP_CHECK(hipGetLastError());
        return KFAC_OK;
    }
    return each_launch(g.T, tok, [&](int first, unsigned wgs) {
        g.first = first;
        hipLaunchKernelGGL(kernel, dim3(wgs, parts), dim3(THREADS), lds, ctx->stream, g);
    });
}
template <typename T, int MODE> int launch_scatter(kfac_ctx *ctx, const MoveArgs &g, double bytes) {
    constexpr int N = 16 / (int)sizeof(T);
    return g.d < N ? launch_scatter<T, 1, MODE>(ctx, g, bytes) : launch_scatter<T, N, MODE>(ctx, g, bytes);
}

// A token's products are one workgroup's, so the gradient of a few tokens of long rows leaves most of the card idle: there a row is shared by more lanes.
// bf16, 1024 lanes against 256: 2 x 2 rows of 65536 11.4 us and 27.6, 14 x 8 of 3272 fp32 6.6 and 11.5, 1 x 8 of 4096 7.0 and 9.7, 256 x 8 of 4096 10 and 13.7;
// 512 x 8 of 4096 17.2 and 16.3, 2048 x 4 of 4096 35 and 24.
constexpr int FEW_TOKENS = 256, FEW_LANES = 1024;
template <typename T, int N, int KB, bool PAST> auto combine_of(int lanes, bool grad) {
    if constexpr (N == 1) return grad ? combine_grad_kernel<T, 1, 8, KB, PAST> : combine_kernel<T, 1, 8, KB, PAST>;
    else if (grad) return lanes == 8 ? combine_grad_kernel<T, N, 8, KB, PAST> : lanes == 16 ? combine_grad_kernel<T, N, 16, KB, PAST> : lanes == 32 ? combine_grad_kernel<T, N, 32, KB, PAST>
                   : lanes == 64 ? combine_grad_kernel<T, N, 64, KB, PAST> : lanes == 128 ? combine_grad_kernel<T, N, 128, KB, PAST>
                   : lanes == 256 ? combine_grad_kernel<T, N, 256, KB, PAST> : combine_grad_kernel<T, N, FEW_LANES, KB, PAST>;
    else return lanes == 8 ? combine_kernel<T, N, 8, KB, PAST> : lanes == 16 ? combine_kernel<T, N, 16, KB, PAST> : lanes == 32 ? combine_kernel<T, N, 32, KB, PAST>
              : lanes == 64 ? combine_kernel<T, N, 64, KB, PAST> : lanes == 128 ? combine_kernel<T, N, 128, KB, PAST> : combine_kernel<T, N, 256, KB, PAST>;
}
template <typename T, int N, int KB, bool PAST> int launch_combine(kfac_ctx *ctx, MoveArgs g, double flops, double bytes) {
    const bool grad = g.dw != nullptr;
    const int vectors = (g.d + N - 1) / N;
    int lanes = lanes_of(vectors, grad ? 1 : 2);
    if (grad && g.T <= FEW_TOKENS && vectors > THREADS) lanes = FEW_LANES;
    const int threads = std::max(lanes, THREADS), tok = threads / lanes;
    const size_t lds = 8 * (size_t)tok * g.k;
    g.part = grad ? vectors : part_of(g.T, vectors, lanes);
    const unsigned parts = (vectors + g.part - 1) / g.part;
    const auto kernel = combine_of<T, N, KB, PAST>(lanes, grad);
    KfacProfScope prof(ctx, KC_TOKENS, flops, bytes);
    return each_launch(g.T, tok, [&](int first, unsigned wgs) {
        g.first = first;
        hipLaunchKernelGGL(kernel, dim3(wgs, parts), dim3(threads), lds, ctx->stream, g);
    });
}
// The experts' rows are read past the caches where it is likely that they are not there any more.  Rows that nothing has touched for long are sooner read past them at any
// size (4 x 4096 bf16 a token: sums of 128 MB 35 us instead of 58, gradients 62 instead of 80; of 32 MB 12 instead of 18 and 20 instead of 24), rows that were just written
// up to the caches' size through them (sums of 64 MB 18 us, past them 21, 128 MB 31 and 36, 256 MB 60 and 63; 384 MB 96 and 88; gradients of 64 MB 28 and 31, 128 MB 59 and
// 64, 192 MB 83 and 90, 256 MB 117 and 114).  Sums follow the product that writes their rows, gradients the whole rest of a step: from half of the caches on the
// most that is lost is less than what is gained.
constexpr double PAST_BYTES = 128e6;
template <typename T, int KB> int launch_combine(kfac_ctx *ctx, const MoveArgs &g, double flops, double bytes) {
    constexpr int N = 16 / (int)sizeof(T);
    if (g.d < N) return launch_combine<T, 1, KB, false>(ctx, g, flops, bytes);
    return (double)sizeof(T) * g.d * g.T * g.k > PAST_BYTES ? launch_combine<T, N, KB, true>(ctx, g, flops, bytes) : launch_combine<T, N, KB, false>(ctx, g, flops, bytes);
}
template <typename T> int launch_combine(kfac_ctx *ctx, const MoveArgs &g, double flops, double bytes) {
    return g.k == 1 ? launch_combine<T, 1>(ctx, g, flops, bytes) : g.k == 2 ? launch_combine<T, 2>(ctx, g, flops, bytes) : launch_combine<T, 4>(ctx, g, flops, bytes);
}

template <typename T, int L, int V> int launch_route(kfac_ctx *ctx, const RouteArgs &all) {
    return each_launch(all.T, THREADS / L, [&](int first, unsigned wgs) {
        RouteArgs g = all;
        g.logits = (const T *)g.logits + first * g.ldl;
        g.T -= first;
        g.ids += (int64_t)first * g.k;
        g.weights += (int64_t)first * g.k;
        hipLaunchKernelGGL((g.k <= L ? route_kernel<T, L, V, true> : route_kernel<T, L, V, false>), dim3(wgs), dim3(THREADS), 0, ctx->stream, g);
    });
}
template <typename T, int L, int V> int launch_route(kfac_ctx *ctx, const RouteGradArgs &all) {
    return each_launch(all.T, THREADS / L, [&](int first, unsigned wgs) {
        RouteGradArgs g = all;
        g.logits = (const T *)g.logits + first * g.ldl;
        g.T -= first;
        g.ids += (int64_t)first * g.k;
        g.dw += (int64_t)first * g.k;
        g.out = (T *)g.out + first * g.ldo;
        hipLaunchKernelGGL((g.k <= L ? route_grad_kernel<T, L, V, true> : route_grad_kernel<T, L, V, false>), dim3(wgs), dim3(THREADS), 0, ctx->stream, g);
    });
}
// The smallest group of lanes that holds the logits of a token.  A choice among up to 128 experts for many tokens is bound by its operations, and groups of
// eight lanes have fewer for each; for few tokens sixteen are sooner done (64 experts, 8 choices: 65536 tokens 8.2 us instead of 10.5, 16 tokens 3.5 instead of 3.0).
template <typename T, typename Args> int launch_route(kfac_ctx *ctx, const Args &g) {
    if constexpr (std::is_same_v<Args, RouteArgs>)
        if (g.E > 16 && g.E <= 128 && g.T >= 4096) return g.E <= 64 ? launch_route<T, 8, 8>(ctx, g) : launch_route<T, 8, 16>(ctx, g);
    if (g.E <= 16) return launch_route<T, 4, 4>(ctx, g);
    if (g.E <= 64) return launch_route<T, 16, 4>(ctx, g);
    if (g.E <= 128) return launch_route<T, 16, 8>(ctx, g);
    if (g.E <= 256) return launch_route<T, 16, 16>(ctx, g);
    if (g.E <= 512) return launch_route<T, 16, 32>(ctx, g);
    if (g.E <= 1024) return launch_route<T, 64, 16>(ctx, g);
    return launch_route<T, 64, 64>(ctx, g);
}

// Waves of a workgroup that sorts, for its counts in LDS.
int sort_waves(int E) { return E <= 512 ? 16 : E <= 1024 ? 8 : E <= 2048 ? 4 : 2; }
constexpr int ONE_SLOTS = 64 * STEPS * SCAN / 64, ONE_EXPERTS = 512;     // what one workgroup sorts alone
// Runs of a sort: as many as the workspace holds, up to as many as a workgroup of the scan has places for.  With a single one its counts become the
// offsets themselves, where they are.
int runs_of(int64_t S, int E, size_t ws_bytes) {
    const int64_t step = 64 * sort_waves(E), most = std::min<int64_t>((S + step - 1) / step, SHARES * EACH);
    return (int)std::max<int64_t>(1, std::min<int64_t>(most, (int64_t)(std::min<size_t>(ws_bytes, (size_t)1 << 40) / (2 * (size_t)E * sizeof(int)))));
}

}  // namespace

size_t kfac_experts_dispatch_ws_bytes_impl(int tokens, int topk, int experts) {
    const int64_t S = (int64_t)tokens * topk;
    if (S <= FEW_SLOTS || (S <= ONE_SLOTS && experts <= ONE_EXPERTS)) return 0;
    return kfac_align_up(2 * (size_t)runs_of(S, experts, SIZE_MAX) * experts * sizeof(int), 256);
}

int kfac_launch_experts_route(kfac_ctx *ctx, int tokens, int experts, int topk, const void *logits, int dtype, int64_t ldl, int normalize, int *ids, float *weights) {
    const RouteArgs g{logits, ldl, tokens, experts, topk, normalize, ids, weights};
    const double n = (double)tokens * experts, es = dtype == KFAC_BF16 ? 2.0 : 4.0;
    KfacProfScope prof(ctx, KC_ROUTE, n * (4 + topk), n * es + 8.0 * tokens * topk);
    return dtype == KFAC_BF16 ? launch_route<unsigned short>(ctx, g) : launch_route<float>(ctx, g);
}

int kfac_launch_experts_route_grad(kfac_ctx *ctx, int tokens, int experts, int topk, const void *logits, int dtype, int64_t ldl, const int *ids, const float *dweights,
                                   int normalize, void *dlogits, int64_t ldd) {
    const RouteGradArgs g{logits, ldl, tokens, experts, topk, normalize, ids, dweights, dlogits, ldd};
    const double n = (double)tokens * experts, s = (double)tokens * topk, es = dtype == KFAC_BF16 ? 2.0 : 4.0;
    KfacProfScope prof(ctx, KC_ROUTE, normalize ? 4.0 * s : 6.0 * n, es * (n + (normalize ? s : n)) + 8.0 * s);
    return dtype == KFAC_BF16 ? launch_route<unsigned short>(ctx, g) : launch_route<float>(ctx, g);
}

int kfac_launch_experts_dispatch(kfac_ctx *ctx, const kfac_slot_desc *d, int experts, const int *ids, const void *X, int64_t ldx, int *offsets, int *rows, void *Xs,
                                 int64_t lds) {
    const int64_t S = (int64_t)d->tokens * d->topk;
    const bool bf = d->dtype == KFAC_BF16;
    const double bytes = 8.0 * (double)S + 4.0 * experts + (X ? (bf ? 2.0 : 4.0) * d->d * ((double)d->tokens + (double)S) : 0.0);
    MoveArgs g{};
    g.T = d->tokens;
    g.k = d->topk;
    g.R = d->rows;
    g.d = X ? d->d : 0;
    g.rows = rows;
    g.x = X;
    g.ldx = ldx;
    g.out = Xs;
    g.ldo = lds;
    SortArgs &s = g.sort;
    s.ids = ids;
    s.S = (int)S;
    s.E = experts;
    s.k = d->topk;
    s.offsets = offsets;
    s.rows = rows;
    if (S <= FEW_SLOTS) return bf ? launch_scatter<unsigned short, COUNTED>(ctx, g, bytes) : launch_scatter<float, COUNTED>(ctx, g, bytes);
    const int waves = sort_waves(experts), step = 64 * waves;
    const size_t counts = (size_t)waves * sizeof(int) * (experts + 1);
    const bool alone = S <= ONE_SLOTS && experts <= ONE_EXPERTS;
    s.runs = alone ? 1 : runs_of(S, experts, ctx->ws_bytes);
    s.per = (int)(((S + s.runs - 1) / s.runs + step - 1) / step * step);
    s.runs = (int)((S + s.per - 1) / s.per);
    s.count = s.runs > 1 ? (int *)ctx->ws : offsets;
    s.base = s.runs > 1 ? s.count + (int64_t)s.runs * experts : offsets;
    {
        KfacProfScope prof(ctx, KC_TOKENS, 0.0, 8.0 * (double)S);
        hipLaunchKernelGGL((alone ? sort_count_kernel<true> : sort_count_kernel<false>), dim3(s.runs), dim3(64 * waves), counts, ctx->stream, s);
        if (!alone) hipLaunchKernelGGL(sort_scan_kernel, dim3(s.runs > 1 ? (experts + SLICE - 1) / SLICE : 1), dim3(SCAN), 0, ctx->stream, s);
    }
    if (alone) {
        KFAC_HIP_CHECK(hipGetLastError());
        if (!X) return KFAC_OK;
        return bf ? launch_scatter<unsigned short, GIVEN>(ctx, g, bytes) : launch_scatter<float, GIVEN>(ctx, g, bytes);
    }
    KFAC_HIP_CHECK(hipGetLastError());
    if (X) return bf ? launch_scatter<unsigned short, RANKED>(ctx, g, bytes) : launch_scatter<float, RANKED>(ctx, g, bytes);
    KfacProfScope prof(ctx, KC_TOKENS, 0.0, 12.0 * (double)S);
    hipLaunchKernelGGL(sort_rows_kernel, dim3((unsigned)((S + THREADS - 1) / THREADS)), dim3(THREADS), 0, ctx->stream, s);
    KFAC_HIP_CHECK(hipGetLastError());
    return KFAC_OK;
}

int kfac_launch_experts_gather(kfac_ctx *ctx, const kfac_slot_desc *d, const int *rows, const void *X, int64_t ldx, void *Xs, int64_t lds) {
    MoveArgs g{};
    g.T = d->tokens;
    g.k = d->topk;
    g.R = d->rows;
    g.d = d->d;
    g.rows = rows;
    g.x = X;
    g.ldx = ldx;
    g.out = Xs;
    g.ldo = lds;
    const double S = (double)d->tokens * d->topk, bytes = 4.0 * S + (d->dtype == KFAC_BF16 ? 2.0 : 4.0) * d->d * (d->tokens + S);
    return d->dtype == KFAC_BF16 ? launch_scatter<unsigned short, GIVEN>(ctx, g, bytes) : launch_scatter<float, GIVEN>(ctx, g, bytes);
}

int kfac_launch_experts_combine(kfac_ctx *ctx, const kfac_slot_desc *d, const int *rows, const float *weights, const void *Ys, int64_t ldys, const void *add, int64_t lda,
                                void *Y, int64_t ldy) {
    MoveArgs g{};
    g.T = d->tokens;
    g.k = d->topk;
    g.R = d->rows;
    g.d = d->d;
    g.rows = rows;
    g.w = weights;
    g.x = Ys;
    g.ldx = ldys;
    g.y = add;
    g.ldy = lda;
    g.out = Y;
    g.ldo = ldy;
    const double S = (double)d->tokens * d->topk, es = d->dtype == KFAC_BF16 ? 2.0 : 4.0;
    const double bytes = (weights ? 8.0 : 4.0) * S + es * d->d * (S + d->tokens * (add ? 2.0 : 1.0)), flops = 2.0 * S * d->d;
    return d->dtype == KFAC_BF16 ? launch_combine<unsigned short>(ctx, g, flops, bytes) : launch_combine<float>(ctx, g, flops, bytes);
}

int kfac_launch_experts_combine_grad(kfac_ctx *ctx, const kfac_slot_desc *d, const int *rows, const float *weights, const void *dY, int64_t lddy, const void *Ys,
                                     int64_t ldys, void *dYs, int64_t lddys, float *dweights) {
    MoveArgs g{};
    g.T = d->tokens;
    g.k = d->topk;
    g.R = d->rows;
    g.d = d->d;
    g.rows = rows;
    g.w = weights;
    g.x = dY;
    g.ldx = lddy;
    g.y = Ys;
    g.ldy = ldys;
    g.out = dYs;
    g.ldo = lddys;
    g.dw = dweights;
    const double S = (double)d->tokens * d->topk, es = d->dtype == KFAC_BF16 ? 2.0 : 4.0;
    const double bytes = 12.0 * S + es * d->d * (2.0 * S + d->tokens), flops = 3.0 * S * d->d;
    return d->dtype == KFAC_BF16 ? launch_combine<unsigned short>(ctx, g, flops, bytes) : launch_combine<float>(ctx, g, flops, bytes);
}
