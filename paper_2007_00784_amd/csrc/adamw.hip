// AdamW over a list of tensors: what follows the preconditioner, which leaves the gradient to take in place (Listing 1 of
// the paper: any optimizer may follow).
//
//   g = grad * grad_scale;  m <- beta1 m + (1 - beta1) g;  v <- beta2 v + (1 - beta2) g^2
//   p <- p - lr weight_decay p - lr (m / (1 - beta1^t)) / (sqrt(v) / sqrt(1 - beta2^t) + eps)
//
// The step is bound by memory: a parameter with fp32 state is 28 bytes (gradient, parameter and both moments in,
// parameter and moments out) for some 30 operations, with 8-bit state and bf16 gradients 16 with the bf16 copy.  So it is one pass:
// each workgroup takes consecutive elements of one tensor, and each thread one vector of them, 4 elements or with 8-bit state 8 (a
// byte each of m and sqrt(v)), all of whose loads are in flight before it computes.  The table of tensors travels in the kernel's
// arguments, so a call copies nothing, needs no workspace and can be captured into a graph; a list of up to ITEMS tensors is one launch
// (two where both kinds of state occur). Measured: the 25.6M parameters of ResNet-50 with fp32 state 131 us, 5.5 TB/s (a copy: 4.9); 268M
// with 8-bit state, bf16 gradients and copies 809 us, 5.3 TB/s, and with their state read back 1066.  With two and four vectors a thread
// the first takes 139 and 144 us, with two the last 1079, and 0.47M with 8-bit state 9.2 instead of 6.2.
//
// 8-bit state: m and sqrt(v) as e4m3 codes times 2^s, one s (a byte, biased by 127) for each BLOCK consecutive elements of
// the tensor, the smallest from -127 to 119 for which the block's largest magnitude is at most 448 * 2^s (what is above 448 * 2^119, seven eighths
// of fp32's range, is held as that: twice the scale would have codes that are not finite).  With a power of two the scaling
// is exact and the code is the only rounding (half to even, at most 2^-4 of the value, or 2^-10 * 2^s below 2^-6 * 2^s); moments are
// computed in fp32, and the parameter is updated with the moments before they are rounded.  sqrt(v) is kept instead of v because v spans
// twice as many binades as the 18 that a block's codes do; and a sqrt(v) above zero never becomes a code of zero (it is held as
// 2^-9 * 2^s at least), since a first moment that outlives its second would be divided by eps.  What is not finite is held as NaN
// and does not count for the scale of its block.
//
// Codes of a running average.  A step moves sqrt(v) by (1 - beta2) / 2 of (g^2 / v - 1), with beta2 = 0.999 mostly by less than 0.1 %, and
// half the distance of two codes is 3 to 6 %.  Rounded half to even such a step is lost: with normal gradients from a state of zero sqrt(v)
// is held at 0.76 of what it should be after 100 steps and at 0.40 after 1000, and once large it never falls.  So with a seed a code is
// rounded up with the probability of its distance from the code below (v_cvt_sr_fp8_f32, which takes 20 bits of a random word: what
// it leaves of an fp32 significand, so for codes from 2^-6 on the expectation is the value itself, below it within 2^-20 of a step).  The
// expectation of m then follows the formula exactly.  That of sqrt(v) does too but for second order: a step's variance, at most |step| times the
// distance of the codes, goes into v, which with normal gradients is 4 % of v, and its spread takes from the mean root: together 1 % of sqrt(v).
// The words come from a hash of element, tensor, step and seed, so a call is the same from run to run and a graph whose step is in
// device memory draws anew at every replay.  268M parameters take 815 us with a seed and 794 without.
#include <algorithm>
#include <cmath>
#include "kfac_internal.h"

namespace {

constexpr int ITEMS = 54;            // tensors of a launch: the table and the rest of the arguments stay below 4 KB
constexpr int BLOCK = 128;           // elements that share a scale
constexpr int THREADS = 256;
constexpr int N32 = 4, N8 = 8;       // elements of a thread

struct AdamItem {
    void *p;
    const void *g;
    void *m, *v;
    unsigned char *ms, *vs;
    unsigned short *copy;            // bf16, or NULL
    uint32_t n;                      // elements
    uint32_t first;                  // first workgroup
};
struct AdamLaunch {
    AdamItem item[ITEMS];
    unsigned char pbf[ITEMS], gbf[ITEMS];   // parameter, gradient in bf16
    int n;
    float b1, c1, b2, c2;            // beta, 1 - beta
    float eps, lr, wd;
    float ibc1, isbc2;               // 1 / (1 - beta1^t), 1 / sqrt(1 - beta2^t) (step_dev: not used)
    double db1, db2;
    const float *gscale, *lr_dev;
    const int64_t *step_dev;
    uint64_t seed;                   // 0: codes are rounded half to even
    int64_t step;                    // (step_dev: not used)
    uint32_t base;                   // of the call's tensors in 8 bits, in pieces: the number of item[0]
};
static_assert(sizeof(AdamLaunch) <= 4096, "arguments of a launch");

struct Hyper { float b1, c1, b2, c2, eps, lr, decay, ibc1, isbc2, gs; };

__device__ inline double int_power(double b, int64_t t) {
    double r = 1.0;
    for (; t > 0; t >>= 1) {
        if (t & 1) r *= b;
        b *= b;
    }
    return r;
}

__device__ inline Hyper hyper_of(const AdamLaunch &a) {
    Hyper h{a.b1, a.c1, a.b2, a.c2, a.eps, a.lr, 0.f, a.ibc1, a.isbc2, 1.f};
    if (a.lr_dev) h.lr = *a.lr_dev;
    if (a.gscale) h.gs = *a.gscale;
    if (a.step_dev) {
        const int64_t t = max(*a.step_dev, (int64_t)1);
        h.ibc1 = (float)(1.0 / (1.0 - int_power(a.db1, t)));
        h.isbc2 = (float)(1.0 / sqrt(1.0 - int_power(a.db2, t)));
    }
    h.decay = h.lr * a.wd;
    return h;
}

// One element: the first moment and the parameter, from the scaled gradient and sqrt(v) of this step.
__device__ inline void adam(const Hyper &h, float g, float root, float &m, float &p) {
    m = fmaf(h.b1, m, h.c1 * g);
    const float step = (m * h.ibc1) / fmaf(root, h.isbc2, h.eps);
    p = fmaf(-h.lr, step, fmaf(-h.decay, p, p));
}
__device__ inline float next_v(const Hyper &h, float g, float v) { return fmaf(h.b2, v, h.c2 * g * g); }
// sqrt(v) of this step from that of the last, which need not have a square in fp32 (below 2^-75, from 2^64 on): both terms are brought to a size
// near one by a power of two first, which changes no bit of what can be squared.  (With beta2 = 0 the last root does not count: 0, or NaN.)
__device__ inline float next_root(const Hyper &h, float g, float root) {
    root = h.b2 > 0.f ? root : root - root;
    const int e = __builtin_amdgcn_frexp_expf(fmaxf(fabsf(g), fabsf(root)));      // (0 for a zero and what is not finite)
    const float x = ldexpf(root, -e);
    return ldexpf(sqrtf(next_v(h, ldexpf(g, -e), x * x)), e);
}

// N consecutive elements from anywhere: tensors may start at any element, and the loads are as wide as N allows all the same (global memory
// takes unaligned vectors).
template <typename T, int N> struct Vec { T x[N]; };
template <typename T, int N> __device__ inline Vec<T, N> load(const void *p, int64_t i) {
    Vec<T, N> r;
    __builtin_memcpy(&r, (const char *)p + i * (int64_t)sizeof(T), sizeof(r));
    return r;
}
template <typename T, int N> __device__ inline void store(void *p, int64_t i, const Vec<T, N> &r) {
    __builtin_memcpy((char *)p + i * (int64_t)sizeof(T), &r, sizeof(r));
}
__device__ inline float widen(unsigned short b) { return __uint_as_float((unsigned)b << 16); }
__device__ inline unsigned short round_bf16(float x) {   // half to even; NaN stays NaN
    const unsigned u = __float_as_uint(x);
    if ((u & 0x7fffffffu) > 0x7f800000u) return (unsigned short)((u >> 16) | 0x40u);
    return (unsigned short)((u + 0x7fffu + ((u >> 16) & 1u)) >> 16);
}

// N elements from i on as fp32, or in bf16; `in` of them exist (N: all, as one vector).
template <int N> __device__ inline void fetch(const void *p, bool bf, int64_t i, int in, float (&x)[N]) {
    if (in == N) {
        if (bf) {
            const auto r = load<unsigned short, N>(p, i);
#pragma unroll
            for (int k = 0; k < N; ++k) x[k] = widen(r.x[k]);
        } else {
            const auto r = load<float, N>(p, i);
#pragma unroll
            for (int k = 0; k < N; ++k) x[k] = r.x[k];
        }
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k) x[k] = k >= in ? 0.f : bf ? widen(((const unsigned short *)p)[i + k]) : ((const float *)p)[i + k];
    }
}
template <int N> __device__ inline void put(void *p, bool bf, int64_t i, int in, const float (&x)[N]) {
    if (in == N) {
        if (bf) {
            Vec<unsigned short, N> r;
#pragma unroll
            for (int k = 0; k < N; ++k) r.x[k] = round_bf16(x[k]);
            store(p, i, r);
        } else {
            Vec<float, N> r;
#pragma unroll
            for (int k = 0; k < N; ++k) r.x[k] = x[k];
            store(p, i, r);
        }
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (k < in) {
                if (bf) ((unsigned short *)p)[i + k] = round_bf16(x[k]);
                else ((float *)p)[i + k] = x[k];
            }
    }
}

// ---- 8-bit state: eight elements a thread, so sixteen lanes (one row of the cross-lane moves) hold a block ----
__device__ inline float row_max(float x) {
#define KFAC_ROW_STEP(ctrl) x = fmaxf(x, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), ctrl, 0xf, 0xf, true)))
    KFAC_ROW_STEP(0xB1);     // lanes 1 0 3 2
    KFAC_ROW_STEP(0x4E);     // lanes 2 3 0 1
    KFAC_ROW_STEP(0x141);    // the other four of each eight
    KFAC_ROW_STEP(0x140);    // the other eight of the sixteen
#undef KFAC_ROW_STEP
    return x;
}
__device__ inline void decode8(const Vec<unsigned, 2> &c, int s, float (&x)[8]) {
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        typedef float float2v __attribute__((ext_vector_type(2)));
        const float2v lo = __builtin_amdgcn_cvt_pk_f32_fp8(c.x[w], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(c.x[w], true);
        x[4 * w] = ldexpf(lo.x, s);
        x[4 * w + 1] = ldexpf(lo.y, s);
        x[4 * w + 2] = ldexpf(hi.x, s);
        x[4 * w + 3] = ldexpf(hi.y, s);
    }
}
// A bijection of 32 bits that spreads every bit over all of them (the multipliers are the fractions of the roots of 2 and 3).
__device__ inline unsigned scatter(unsigned x) {
    x = (x ^ x >> 16) * 0x6a09e667u;
    x = (x ^ x >> 15) * 0xbb67ae85u;
    return x ^ x >> 16;
}
// Where the words of a tensor's elements begin, at this step.
__device__ inline unsigned words_of(const AdamLaunch &a, int id) {
    const uint64_t t = (uint64_t)(a.step_dev ? max(*a.step_dev, (int64_t)1) : a.step);
    unsigned k = scatter((unsigned)a.seed);
    k = scatter(k ^ (unsigned)(a.seed >> 32));
    k = scatter(k ^ (unsigned)t);
    k = scatter(k ^ (unsigned)(t >> 32));
    return scatter(k ^ (a.base + (unsigned)id));
}
// The block's exponent s from the values of its sixteen lanes, and this lane's codes.  `least`: the smallest code of a value above zero.
// `word`: DITHER: random words, of which the upper 20 bits count.
template <bool DITHER> __device__ inline Vec<unsigned, 2> encode8(const float (&x)[8], float least, int &s, const unsigned (&word)[8]) {
    float big = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const float a = fabsf(x[k]);
        big = fmaxf(big, a < INFINITY ? a : 0.f);
    }
    big = row_max(big);
    s = big > 0.f ? min(max(__builtin_amdgcn_frexp_expf(big) - 9 + (__builtin_amdgcn_frexp_mantf(big) > 0.875f ? 1 : 0), -127), 119) : -127;
    Vec<unsigned, 2> c;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        float y[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            y[k] = ldexpf(x[4 * w + k], -s);
            // (448 is passed only where s is at its limit: what is above 448 * 2^119 would be infinite as the next code)
            y[k] = fabsf(y[k]) < INFINITY ? (y[k] > 0.f ? __builtin_amdgcn_fmed3f(y[k], least, 448.f) : fmaxf(y[k], -448.f)) : NAN;
        }
        if (DITHER) {
            int r = __builtin_amdgcn_cvt_sr_fp8_f32(y[0], word[4 * w], 0, 0);
            r = __builtin_amdgcn_cvt_sr_fp8_f32(y[1], word[4 * w + 1], r, 1);
            r = __builtin_amdgcn_cvt_sr_fp8_f32(y[2], word[4 * w + 2], r, 2);
            c.x[w] = __builtin_amdgcn_cvt_sr_fp8_f32(y[3], word[4 * w + 3], r, 3);
        } else {
            unsigned r = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
            c.x[w] = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], r, true);
        }
    }
    return c;
}

__device__ inline int item_of(const AdamLaunch &a, unsigned wg) {   // the last tensor whose first workgroup is not behind this one
    const int lane = threadIdx.x & 63;
    const bool mine = lane < a.n && a.item[lane < ITEMS ? lane : 0].first <= wg;
    return __builtin_amdgcn_readfirstlane(__popcll(__ballot(mine)) - 1);
}

__global__ __launch_bounds__(THREADS) void adamw_kernel(const AdamLaunch a) {
    const int id = item_of(a, blockIdx.x);
    const AdamItem it = a.item[id];
    const bool pbf = a.pbf[id], gbf = a.gbf[id];
    const int64_t i = ((int64_t)(blockIdx.x - it.first) * THREADS + threadIdx.x) * N32;
    const int in = (int)min((int64_t)N32, max((int64_t)it.n - i, (int64_t)0));
    float g[N32], p[N32], m[N32], v[N32];
    fetch(it.g, gbf, i, in, g);
    fetch(it.p, pbf, i, in, p);
    fetch(it.m, false, i, in, m);
    fetch(it.v, false, i, in, v);
    const Hyper h = hyper_of(a);       // (under the loads: with the step in device memory its powers take 64-bit operations)
#pragma unroll
    for (int k = 0; k < N32; ++k) {
        g[k] *= h.gs;
        v[k] = next_v(h, g[k], v[k]);
        adam(h, g[k], sqrtf(v[k]), m[k], p[k]);
    }
    put(it.p, pbf, i, in, p);
    put(it.m, false, i, in, m);
    put(it.v, false, i, in, v);
    if (it.copy) put(it.copy, true, i, in, p);
}

__device__ inline Vec<unsigned, 2> fetch_codes(const void *p, int64_t i, int in) {
    if (in == 8) return load<unsigned, 2>((const char *)p + i, 0);
    Vec<unsigned, 2> c{};
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (k < in) c.x[k >> 2] |= (unsigned)((const unsigned char *)p)[i + k] << (8 * (k & 3));
    return c;
}
__device__ inline void put_codes(void *p, int64_t i, int in, const Vec<unsigned, 2> &c) {
    if (in == 8) {
        store((char *)p + i, 0, c);
        return;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
        if (k < in) ((unsigned char *)p)[i + k] = (unsigned char)(c.x[k >> 2] >> (8 * (k & 3)));
}

template <bool DITHER> __global__ __launch_bounds__(THREADS) void adamw8_kernel(const AdamLaunch a) {
    const int id = item_of(a, blockIdx.x);
    const AdamItem it = a.item[id];
    const bool pbf = a.pbf[id], gbf = a.gbf[id];
    const int64_t i = ((int64_t)(blockIdx.x - it.first) * THREADS + threadIdx.x) * N8;
    const int in = (int)min((int64_t)N8, max((int64_t)it.n - i, (int64_t)0));
    float g[N8], p[N8], m[N8], r[N8];
    const Vec<unsigned, 2> mc = fetch_codes(it.m, i, in), vc = fetch_codes(it.v, i, in);
    const int ms = in > 0 ? it.ms[i / BLOCK] : 0, vs = in > 0 ? it.vs[i / BLOCK] : 0;
    fetch(it.g, gbf, i, in, g);
    fetch(it.p, pbf, i, in, p);
    const Hyper h = hyper_of(a);       // (25.6M parameters, the step in device memory: in front of the loads 83 us, here 79)
    decode8(mc, ms - 127, m);
    decode8(vc, vs - 127, r);
#pragma unroll
    for (int k = 0; k < N8; ++k) {
        g[k] *= h.gs;
        r[k] = next_root(h, g[k], r[k]);
        adam(h, g[k], r[k], m[k], p[k]);
        if (k >= in) m[k] = r[k] = 0.f;       // (a gradient scale that is not finite must not reach the block from behind the tensor's end)
    }
    // one word an element: m takes its upper 20 bits, sqrt(v) its lower 20 (the eight that both have are the last of m's)
    unsigned wm[N8] = {}, wv[N8] = {};
    if (DITHER) {
        const unsigned k0 = words_of(a, id) + (unsigned)i * 0x9e3779b1u;
#pragma unroll
        for (int k = 0; k < N8; ++k) {
            wm[k] = scatter(k0 + (unsigned)k * 0x9e3779b1u);
            wv[k] = wm[k] << 12;
        }
    }
    int s, t;
    const Vec<unsigned, 2> nm = encode8<DITHER>(m, 0.f, s, wm), nv = encode8<DITHER>(r, 0x1p-9f, t, wv);
    put_codes(it.m, i, in, nm);
    put_codes(it.v, i, in, nv);
    if ((threadIdx.x & (BLOCK / N8 - 1)) == 0 && in > 0) {
        it.ms[i / BLOCK] = (unsigned char)(s + 127);
        it.vs[i / BLOCK] = (unsigned char)(t + 127);
    }
    put(it.p, pbf, i, in, p);
    if (it.copy) put(it.copy, true, i, in, p);
}

// What the 8-bit codes stand for, in fp32 or in bf16 (four significant bits, so exactly as long as the last is not below 2^-133: scales from 3 on).
__global__ __launch_bounds__(THREADS) void adamw_values_kernel(const unsigned char *code, const unsigned char *scale, int64_t n, void *out, int bf) {
    const int64_t i = ((int64_t)blockIdx.x * THREADS + threadIdx.x) * 8;
    const int in = (int)min((int64_t)8, max(n - i, (int64_t)0));
    if (in == 0) return;
    float x[8];
    decode8(fetch_codes(code, i, in), (int)scale[i / BLOCK] - 127, x);
    put(out, bf != 0, i, in, x);
}

int launch(kfac_ctx *ctx, const AdamLaunch &a, unsigned wgs, bool eight, double flops, double bytes) {
    KfacProfScope prof(ctx, KC_ADAMW, flops, bytes);
    hipLaunchKernelGGL(!eight ? adamw_kernel : a.seed ? adamw8_kernel<true> : adamw8_kernel<false>, dim3(wgs), dim3(THREADS), 0, ctx->stream, a);
    KFAC_HIP_CHECK(hipGetLastError());
    return KFAC_OK;
}

}  // namespace

int kfac_launch_adamw_batched(kfac_ctx *ctx, int n, const kfac_adamw_item *items, const kfac_adamw_opts *o) {
    AdamLaunch a{};
    a.b1 = (float)o->beta1;
    a.c1 = (float)(1.0 - o->beta1);
    a.b2 = (float)o->beta2;
    a.c2 = (float)(1.0 - o->beta2);
    a.eps = o->eps;
    a.lr = o->lr;
    a.wd = o->weight_decay;
    if (!o->step_dev) {
        a.ibc1 = (float)(1.0 / (1.0 - std::pow(o->beta1, (double)o->step)));
        a.isbc2 = (float)(1.0 / std::sqrt(1.0 - std::pow(o->beta2, (double)o->step)));
    }
    a.db1 = o->beta1;
    a.db2 = o->beta2;
    a.gscale = o->grad_scale;
    a.lr_dev = o->lr_dev;
    a.step_dev = o->step_dev;
    a.seed = o->seed;
    a.step = o->step;
    // a tensor longer than 32-bit offsets and grids reach goes in pieces (a multiple of BLOCK each)
    constexpr int64_t PIECE = (int64_t)1 << 31;
    constexpr unsigned MOST_WGS = 1u << 23;
    for (int eight = 0; eight < 2; ++eight) {
        const int64_t share = THREADS * (eight ? N8 : N32);      // elements of a workgroup
        unsigned wgs = 0;
        double flops = 0.0, bytes = 0.0;
        a.n = 0;
        a.base = 0;
        for (int i = 0; i < n; ++i) {
            const kfac_adamw_item &t = items[i];
            if ((t.m_scale != nullptr) != (eight != 0)) continue;
            const int64_t sp = t.param_dtype == KFAC_BF16 ? 2 : 4, sg = t.grad_dtype == KFAC_BF16 ? 2 : 4, ss = eight ? 1 : 4;
            for (int64_t at = 0; at < t.n; at += PIECE) {
                const int64_t len = std::min(PIECE, t.n - at);
                const unsigned mine = (unsigned)((len + share - 1) / share);
                if (a.n == ITEMS || wgs + mine > MOST_WGS) {
                    KFAC_CHECK(launch(ctx, a, wgs, eight != 0, flops, bytes));
                    a.base += (uint32_t)a.n;
                    a.n = 0;
                    wgs = 0;
                    flops = bytes = 0.0;
                }
                AdamItem &d = a.item[a.n];
                d.p = (char *)t.param + at * sp;
                d.g = (const char *)t.grad + at * sg;
                d.m = (char *)t.m + at * ss;
                d.v = (char *)t.v + at * ss;
                d.ms = eight ? t.m_scale + at / BLOCK : nullptr;
                d.vs = eight ? t.v_scale + at / BLOCK : nullptr;
                d.copy = t.copy ? (unsigned short *)t.copy + at : nullptr;
                d.n = (uint32_t)len;
                d.first = wgs;
                a.pbf[a.n] = t.param_dtype == KFAC_BF16;
                a.gbf[a.n] = t.grad_dtype == KFAC_BF16;
                ++a.n;
                wgs += mine;
                flops += 16.0 * (double)len;
                bytes += (double)len * ((double)(2 * sp + sg + 4 * ss) + (t.copy ? 2.0 : 0.0) + (eight ? 4.0 / BLOCK : 0.0));
            }
        }
        if (wgs > 0) KFAC_CHECK(launch(ctx, a, wgs, eight != 0, flops, bytes));
    }
    return KFAC_OK;
}

int kfac_launch_adamw_state_values(kfac_ctx *ctx, const void *codes, const unsigned char *scale, int64_t n, void *out, int dtype) {
    constexpr int64_t PIECE = (int64_t)1 << 34;      // a grid of 2^23 workgroups
    for (int64_t at = 0; at < n; at += PIECE) {
        const int64_t len = std::min(PIECE, n - at), per = 8 * THREADS;
        KfacProfScope prof(ctx, KC_ADAMW, 0.0, (double)len * (dtype == KFAC_BF16 ? 3.0 : 5.0));
        hipLaunchKernelGGL(adamw_values_kernel, dim3((unsigned)((len + per - 1) / per)), dim3(THREADS), 0, ctx->stream, (const unsigned char *)codes + at,
                           scale + at / BLOCK, len, (char *)out + at * (dtype == KFAC_BF16 ? 2 : 4), dtype == KFAC_BF16 ? 1 : 0);
        KFAC_HIP_CHECK(hipGetLastError());
    }
    return KFAC_OK;
}
