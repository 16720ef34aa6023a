// Products and Kronecker factors of a layer of experts: E weight matrices of one shape, every sample row belongs to one of them, and the
// rows are sorted by expert (offsets in device memory, as a router leaves them).
//
//   forward       Y[r] = X[r] W_e^T (+ bias)                     rows ragged, contraction d_in
//   input_grad    dX[r] = G[r] W_e                               rows ragged, contraction d_out
//   weight_grad   dW_e = sum_r G[r]^T [X[r] | 1]                  contraction ragged (Listing 1's gradient as the preconditioner takes it)
//   factors       F_e <- decay F_e + (1 - decay) scale / R_e sum_r [X[r] | 1]^T [X[r] | 1]    (Sec. II-C, Sec. IV-B, over an expert's rows)
//
// The host does not know the offsets, so a launch has as many workgroups as any offsets could need, and each finds its tile from
// them (a prefix sum over the experts' tiles by one wave); surplus workgroups end at once.  Nothing is copied from the host: all arguments
// travel with the launch, so the calls can be captured into a graph and replayed with other offsets.
#include <algorithm>
#include <cmath>
#include <type_traits>
#include "kfac_internal.h"
#include "mfma_gemm.h"
#include "mfma_gemm_wide.h"

using namespace kfac;

namespace {

enum { FORWARD = 0, INPUT_GRAD = 1, WEIGHT_GRAD = 2, FACTORS = 3 };

struct ExpertArgs {
    const int *offsets;      // [E + 1], device
    int E, R;                // experts; rows of the sample matrices
    const void *a;           // X (forward, factors), G
    int64_t lda;
    const void *b;           // W (forward, input_grad), X (weight_grad)
    int64_t ldb;             // its pitch inside one expert
    int64_t estride;         // W: elements of one expert's matrix
    void *out;               // Y, dX, dW, F
    int64_t ldo;
    int64_t ostride;         // dW, F: elements of one expert's matrix
    int rows, cols;          // outputs per expert (cols without the bias column); rows: d_out (weight_grad), d (factors)
    int K;                   // contraction (forward, input_grad)
    int ones;
    int out_bf16, accumulate;
    int mean;
    float scale, decay;
};

struct Range { int beg, end; };
// Rows of expert e.  Whatever the offsets hold, the range lies inside the sample matrices.
__device__ inline Range range_of(const ExpertArgs &g, int e) {
    const int beg = min(max(g.offsets[e], 0), g.R);
    return Range{beg, min(max(g.offsets[e + 1], beg), g.R)};
}

// Where the workgroup's tile lies: expert, row tile and column tile.
struct Place { int e, m, n; Range r; };

// Rows ragged: expert e has ceil(rows / EXT) row tiles times `nt` column tiles.  The tiles of all experts, in order, are dealt to the eight XCDs
// in equal consecutive parts (workgroup b runs on XCD b % 8), so that tiles that share operands share an L2; inside an expert the
// order goes over BAND row tiles before it takes the next column tile.
constexpr int BAND = 4;
template <int EXT>
__device__ inline bool place_ragged(const ExpertArgs &g, int nt, Place &p) {
    const int lane = threadIdx.x & 63;
    int64_t total = 0;
    for (int e0 = 0; e0 < g.E; e0 += 64) {
        const int e = e0 + lane;
        int mt = 0;
        if (e < g.E) {
            const Range r = range_of(g, e);
            mt = (r.end - r.beg + EXT - 1) / EXT;
        }
#pragma unroll
        for (int d = 32; d; d >>= 1) mt += __shfl_xor(mt, d);
        total += __builtin_amdgcn_readfirstlane(mt);
    }
    total *= nt;
    const int64_t per = (total + 7) / 8, t = (int64_t)(blockIdx.x & 7) * per + (blockIdx.x >> 3);
    if ((int64_t)(blockIdx.x >> 3) >= per || t >= total) return false;
    int64_t before = 0;
    for (int e0 = 0; e0 < g.E; e0 += 64) {
        const int e = e0 + lane;
        Range r{0, 0};
        int mt = 0;
        if (e < g.E) {
            r = range_of(g, e);
            mt = (r.end - r.beg + EXT - 1) / EXT;
        }
        int incl = mt;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(incl, d);
            if (lane >= d) incl += o;
        }
        const int64_t last = before + (int64_t)incl * nt;
        const uint64_t past = __ballot(last > t);
        if (past) {
            const int l = __builtin_ctzll(past);
            p.e = e0 + l;
            p.r = Range{__builtin_amdgcn_readlane(r.beg, l), __builtin_amdgcn_readlane(r.end, l)};
            const int mine = __builtin_amdgcn_readlane(mt, l);
            const int local = (int)(t - (before + (int64_t)(__builtin_amdgcn_readlane(incl, l) - mine) * nt));
            const int band = local / (BAND * nt), in = local - band * BAND * nt, high = min(BAND, mine - band * BAND);
            p.n = in / high;
            p.m = band * BAND + (in - p.n * high);
            return true;
        }
        before += (int64_t)__builtin_amdgcn_readlane(incl, 63) * nt;
    }
    return false;
}

// Outputs fixed per expert: mt x nt tiles each (lower triangular ones of mt x mt where TRI), whose work goes with the expert's rows.  Experts are taken in
// the order of their rows, the longest first (where one wave can hold them: 64 at most), so that no long one is left for the end; and each RUN
// consecutive tiles of that order go to the next XCD, so that every XCD has the same share of every expert and the tiles of a run share its L2.
constexpr int RUN = 8;
template <bool TRI>
__device__ inline bool place_fixed(const ExpertArgs &g, int mt, int nt, Place &p) {
    const int each = TRI ? mt * (mt + 1) / 2 : mt * nt;
    const int64_t i = blockIdx.x >> 3, t = ((i / RUN) * 8 + (blockIdx.x & 7)) * RUN + i % RUN;
    if (t >= (int64_t)each * g.E) return false;
    const int place = (int)(t / each);
    int e = place;
    if (g.E <= 64) {
        const int lane = threadIdx.x & 63;
        int rows = -1;
        if (lane < g.E) {
            const Range r = range_of(g, lane);
            rows = r.end - r.beg;
        }
        int rank = 0;       // how many are longer, or as long and in front
        for (int o = 0; o < g.E; ++o) {
            const int other = __builtin_amdgcn_readlane(rows, o);
            rank += other > rows || (other == rows && o < lane) ? 1 : 0;
        }
        e = __builtin_ctzll(__ballot(lane < g.E && rank == place));
    }
    p.e = e;
    const int local = (int)(t - (int64_t)place * each);
    if (TRI) {
        int i = (int)((sqrtf(8.f * (float)local + 1.f) - 1.f) * 0.5f);
        while ((i + 1) * (i + 2) / 2 <= local) ++i;
        while (i * (i + 1) / 2 > local) --i;
        p.m = i;
        p.n = local - i * (i + 1) / 2;
    } else {
        const int band = local / (BAND * nt), in = local - band * BAND * nt, high = min(BAND, mt - band * BAND);
        p.n = in / high;
        p.m = band * BAND + (in - p.n * high);
    }
    p.r = range_of(g, p.e);
    return true;
}

// ---- what becomes of a finished sum ----
__device__ inline unsigned short to_bf16(float x) {   // half to even
    const __bf16 b = (__bf16)x;
    unsigned short u;
    __builtin_memcpy(&u, &b, 2);
    return u;
}
// Factor weights of an expert: F <- keep F + alpha sum.  With `mean`, an expert without rows keeps its factor as it is.
struct Average { float alpha, keep; };
__device__ inline Average average_of(const ExpertArgs &g, int count) {
    if (!g.mean) return Average{(1.f - g.decay) * g.scale, g.decay};
    return Average{(1.f - g.decay) * g.scale / (float)max(count, 1), g.decay};
}

typedef __bf16 wide_bf16x4 __attribute__((ext_vector_type(4)));

// out(r, c) for one element; r counts the rows of Y / dX (from the matrix' first on) or of an expert's dW / F.
template <int MODE>
__device__ inline void finish(const ExpertArgs &g, int e, int r, int c, float v, const Average &w) {
    if (MODE == FORWARD || MODE == INPUT_GRAD) {
        const int64_t o = (int64_t)r * g.ldo + c;
        if (g.out_bf16) ((unsigned short *)g.out)[o] = to_bf16(v);
        else ((float *)g.out)[o] = v;
    } else if (MODE == WEIGHT_GRAD) {
        const int64_t o = e * g.ostride + (int64_t)r * g.ldo + c;
        if (g.out_bf16) {
            unsigned short *d = (unsigned short *)g.out + o;
            *d = to_bf16(g.accumulate ? v + to_float(*d) : v);
        } else {
            float *d = (float *)g.out + o;
            *d = g.accumulate ? v + *d : v;
        }
    } else {
        float *F = (float *)g.out + e * g.ostride;
        float *d = F + (int64_t)r * g.ldo + c;
        const float x = w.keep != 0.f ? fmaf(w.alpha, v, w.keep * *d) : w.alpha * v;
        *d = x;
        if (r != c) F[(int64_t)c * g.ldo + r] = x;
    }
}

// ---- bf16: the wide engine ----
template <int MODE, int FR, int FC, int WR, int WC, int RING>
__global__ __launch_bounds__(64 * WR * WC) void expert_wide_kernel(const ExpertArgs g) {
    extern __shared__ __align__(16) char smem[];
    constexpr int ROWS = 16 * FR * WR, COLS = 16 * FC * WC, NW = WR * WC;
    constexpr bool RAGGED = MODE == FORWARD || MODE == INPUT_GRAD, ONES = !RAGGED;
    const int nt = (g.cols + COLS - 1) / COLS;
    Place p;
    if (RAGGED ? !place_ragged<ROWS>(g, nt, p) : !place_fixed<MODE == FACTORS>(g, (g.rows + ROWS - 1) / ROWS, nt, p)) return;
    const int count = p.r.end - p.r.beg;
    if (MODE == FACTORS && count == 0 && (g.mean || g.decay == 1.f)) return;
    if (MODE == WEIGHT_GRAD && count == 0 && g.accumulate) return;
    const unsigned short *a = (const unsigned short *)g.a + p.r.beg * g.lda;
    floatx4 acc[FC][FR], one[FR / WC];
    using Row = std::conditional_t<RAGGED, OpAlong<ROWS, NW>, OpAcross<ROWS, NW, false>>;
    using Col = std::conditional_t<MODE == FORWARD, OpAlong<COLS, NW>, OpAcross<COLS, NW, MODE == INPUT_GRAD>>;
    Row row;
    Col col;
    const int K = RAGGED ? g.K : count;
    const bool sums = ONES && g.ones && p.n == 0;
    if constexpr (RAGGED) row.start(a, g.lda, p.m * ROWS, count, K);
    else row.start(a, g.lda, p.m * ROWS, g.rows, K);
    if constexpr (MODE == FORWARD) col.start((const unsigned short *)g.b + p.e * g.estride, g.ldb, p.n * COLS, g.cols, K);
    else if constexpr (MODE == INPUT_GRAD) col.start((const unsigned short *)g.b + p.e * g.estride, g.ldb, p.n * COLS, g.cols, K);
    else if constexpr (MODE == WEIGHT_GRAD) col.start((const unsigned short *)g.b + p.r.beg * g.ldb, g.ldb, p.n * COLS, g.cols, K);
    else col.start(a, g.lda, p.n * COLS, g.cols, K);
    wide_tile<Row, Col, FR, FC, WR, WC, RING, ONES>(row, col, K, smem, acc, one, sums);

    // Each wave turns its 64 columns round in LDS, 32 rows at a time, so that a store covers whole rows of them (128 or 256 bytes side
    // by side; the accumulators' own layout has 32 or 64).
    static_assert(FC == 4 && FR % 2 == 0, "64 columns of a wave");
    constexpr int PITCH = 64 + 4;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wr = wave / WC, wc = wave % WC;
    float *const turn = reinterpret_cast<float *>(smem) + wave * 32 * PITCH;
    const Average w = MODE == FACTORS ? average_of(g, count) : Average{};
    const int c0 = p.n * COLS + 64 * wc + 4 * (lane & 15);                      // four places side by side
    const bool whole = c0 + 4 <= (MODE == FORWARD ? g.cols : g.cols & ~7) && (MODE != FACTORS || p.m * ROWS >= (p.n + 1) * COLS);
    float bias[4] = {0.f, 0.f, 0.f, 0.f};
    if (MODE == FORWARD && g.ones) {
        const unsigned short *W = (const unsigned short *)g.b + p.e * g.estride + g.K;
#pragma unroll
        for (int x = 0; x < 4; ++x) bias[x] = to_float(W[(int64_t)min(c0 + x, g.cols - 1) * g.ldb]);
    }
    __syncthreads();
#pragma unroll
    for (int part = 0; part < FR / 2; ++part) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int i = 0; i < FC; ++i)
                *reinterpret_cast<floatx4 *>(turn + (16 * j + (lane & 15)) * PITCH + 16 * i + 4 * (lane >> 4)) = acc[i][2 * part + j];
        const int r0 = p.m * ROWS + 16 * (wr * FR + 2 * part);
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            const int at = 4 * t + (lane >> 4), r = row.side(r0 + at);
            if (r < 0 || r >= (RAGGED ? count : g.rows)) continue;
            floatx4 v = *reinterpret_cast<const floatx4 *>(turn + at * PITCH + 4 * (lane & 15));
            if (MODE == FORWARD)
#pragma unroll
                for (int x = 0; x < 4; ++x) v[x] += bias[x];
            if (!whole) {
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int c = col.side(c0 + x);
                    if (c < 0 || c >= g.cols || (MODE == FACTORS && c > r)) continue;
                    finish<MODE>(g, p.e, RAGGED ? p.r.beg + r : r, c, v[x], w);
                }
                continue;
            }
            const int64_t o = RAGGED ? (int64_t)(p.r.beg + r) * g.ldo + c0 : p.e * g.ostride + (int64_t)r * g.ldo + c0;
            if (MODE == FACTORS) {
                float *d = (float *)g.out + o;
                floatx4 old = {0.f, 0.f, 0.f, 0.f};
                if (w.keep != 0.f) __builtin_memcpy(&old, d, 16);
#pragma unroll
                for (int x = 0; x < 4; ++x) v[x] = w.keep != 0.f ? fmaf(w.alpha, v[x], w.keep * old[x]) : w.alpha * v[x];
                __builtin_memcpy(d, &v, 16);
                *reinterpret_cast<floatx4 *>(turn + at * PITCH + 4 * (lane & 15)) = v;
            } else if (RAGGED || g.out_bf16) {
                unsigned short *d = (unsigned short *)g.out + o;
                if (MODE == WEIGHT_GRAD && g.accumulate) {
                    unsigned short old[4];
                    __builtin_memcpy(old, d, 8);
#pragma unroll
                    for (int x = 0; x < 4; ++x) v[x] += to_float(old[x]);
                }
                const wide_bf16x4 b = __builtin_convertvector(v, wide_bf16x4);   // half to even
                __builtin_memcpy(d, &b, 8);
            } else {
                float *d = (float *)g.out + o;
                if (MODE == WEIGHT_GRAD && g.accumulate) {
                    floatx4 old;
                    __builtin_memcpy(&old, d, 16);
                    v += old;
                }
                __builtin_memcpy(d, &v, 16);
            }
        }
        if (MODE == FACTORS && p.m * ROWS >= (p.n + 1) * COLS) {
            // the mirrored part: lane l takes rows 4 (l % 8).. of column l / 8, which lie side by side there
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                const int place = 8 * t + (lane >> 3), c = col.side(p.n * COLS + 64 * wc + place);
                if (c < 0 || c >= (g.cols & ~7)) continue;      // (places of a shifted group have stored theirs)
                floatx4 v;
#pragma unroll
                for (int x = 0; x < 4; ++x) v[x] = turn[(4 * (lane & 7) + x) * PITCH + place];
                const int first = r0 + 4 * (lane & 7);
                float *d = (float *)g.out + p.e * g.ostride + (int64_t)c * g.ldo;
                if (first + 4 <= (g.rows & ~7)) __builtin_memcpy(d + first, &v, 16);
                else
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const int r = row.side(first + x);
                        if (r >= 0 && r < g.rows) d[r] = v[x];
                    }
            }
        }
    }
    if (sums && lane < 16) {
#pragma unroll
        for (int j = 0; j < FR / WC; ++j) {
            const int r = row.side(p.m * ROWS + 16 * (wr * FR + wc * (FR / WC) + j) + lane);
            if (r < 0 || r >= g.rows) continue;
            if (MODE == WEIGHT_GRAD) finish<MODE>(g, p.e, r, g.cols, one[j][0], w);
            else finish<MODE>(g, p.e, g.rows, r, one[j][0], w);
        }
        if (MODE == FACTORS && p.m == 0 && wave == 0 && lane == 0) finish<MODE>(g, p.e, g.rows, g.rows, (float)count, w);
    }
}

// ---- fp32, and bf16 with a side shorter than the wide engine's groups: the element-wise engine (fp32 matrix instructions) ----
template <int MODE, typename E>
__global__ __launch_bounds__(NTHREADS) __attribute__((amdgpu_waves_per_eu(2))) void expert_tile_kernel(const ExpertArgs g) {
    __shared__ TileSmem sm;
    __shared__ float cs[BM];
    constexpr bool RAGGED = MODE == FORWARD || MODE == INPUT_GRAD;
    const int nt = (g.cols + BM - 1) / BM;
    Place p;
    if (RAGGED ? !place_ragged<BM>(g, nt, p) : !place_fixed<MODE == FACTORS>(g, (g.rows + BM - 1) / BM, nt, p)) return;
    const int count = p.r.end - p.r.beg;
    if (MODE == FACTORS && count == 0 && (g.mean || g.decay == 1.f)) return;
    if (MODE == WEIGHT_GRAD && count == 0 && g.accumulate) return;
    const E *a = (const E *)uniform_ptr((const E *)g.a + p.r.beg * g.lda);
    const int rows = RAGGED ? count : g.rows, K = RAGGED ? g.K : count;
    const int i0 = p.m * BM, j0 = p.n * BM;
    const bool sums = !RAGGED && g.ones && p.n == 0;
    floatx16 acc[2][2];
    const WaveMap map = wave_map_edge(min(rows - i0, BM), min(g.cols - j0, BM));
    using Row = OpStrided<E, RAGGED>;
    using Col = OpStrided<E, MODE == FORWARD>;
    Row A{a, RAGGED ? g.lda : 1, RAGGED ? 1 : g.lda, rows, K, -1};
    const E *b = (const E *)uniform_ptr(MODE == FORWARD || MODE == INPUT_GRAD ? (const E *)g.b + p.e * g.estride
                                        : MODE == WEIGHT_GRAD ? (const E *)g.b + p.r.beg * g.ldb : a);
    const int64_t ldb = MODE == FACTORS ? g.lda : g.ldb;
    Col B{b, MODE == FORWARD ? ldb : 1, MODE == FORWARD ? 1 : ldb, g.cols, K, -1};
    A.seg_k = B.seg_k = 0;
    if (sums) {
        float csum[EPT];
#pragma unroll
        for (int s = 0; s < EPT; ++s) csum[s] = 0.f;
        gemm_tile<Row, Col, true, true>(A, B, i0, j0, 0, K, sm, acc, csum, true, map);
        // (across: every slot of a thread is row tid & 127; two threads share it)
        float t = 0.f;
#pragma unroll
        for (int s = 0; s < EPT; ++s) t += csum[s];
        float *scratch = &sm.a[0][0][0];
        __syncthreads();
        scratch[threadIdx.x] = t;
        __syncthreads();
        if (threadIdx.x < BM) cs[threadIdx.x] = scratch[threadIdx.x] + scratch[threadIdx.x + BM];
        __syncthreads();
    } else {
        gemm_tile<Row, Col, false, true>(A, B, i0, j0, 0, K, sm, acc, nullptr, true, map);
    }
    const Average w = MODE == FACTORS ? average_of(g, count) : Average{};
    const E *W = (const E *)g.b + p.e * g.estride + g.K;
    for_each_acc(acc, map, [&](int r, int c, float v) {
        r += i0;
        c += j0;
        if (r >= rows || c >= g.cols || (MODE == FACTORS && c > r)) return;
        if (MODE == FORWARD && g.ones) v += to_float(W[(int64_t)c * g.ldb]);
        finish<MODE>(g, p.e, RAGGED ? p.r.beg + r : r, c, v, w);
    });
    if (sums) {
        const int r = i0 + threadIdx.x;
        if (threadIdx.x < BM && r < rows) {
            if (MODE == WEIGHT_GRAD) finish<MODE>(g, p.e, r, g.cols, cs[threadIdx.x], w);
            else finish<MODE>(g, p.e, g.rows, r, cs[threadIdx.x], w);
        }
        if (MODE == FACTORS && p.m == 0 && threadIdx.x == 0) finish<MODE>(g, p.e, g.rows, g.rows, (float)count, w);
    }
}

// ---- launches ----
unsigned grid_of(const ExpertArgs &g, int mode, int ext_r, int ext_c) {
    const int64_t nt = (g.cols + ext_c - 1) / ext_c;
    int64_t tiles;
    if (mode == FORWARD || mode == INPUT_GRAD) tiles = ((int64_t)g.R / ext_r + std::min<int64_t>(g.E, g.R)) * nt;
    else {
        const int64_t mt = (g.rows + ext_r - 1) / ext_r;
        tiles = (mode == FACTORS ? mt * (mt + 1) / 2 : mt * nt) * g.E;
    }
    const int64_t unit = mode == FORWARD || mode == INPUT_GRAD ? 8 : 8 * RUN;
    return (unsigned)std::min<int64_t>((tiles + unit - 1) / unit * unit, (int64_t)1 << 31);
}

template <int MODE, int FR, int FC, int WR, int WC, int RING>
int launch_wide(kfac_ctx *ctx, const ExpertArgs &g) {
    constexpr int lds = ((RING + 1) * 16 * FR * WR + RING * 16 * FC * WC) * WK * 2;
    const auto kernel = expert_wide_kernel<MODE, FR, FC, WR, WC, RING>;
    if (lds > ctx->max_lds) return KFAC_EHIP;
    KFAC_HIP_CHECK(hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds));
    hipLaunchKernelGGL(kernel, dim3(grid_of(g, MODE, 16 * FR * WR, 16 * FC * WC)), dim3(64 * WR * WC), lds, ctx->stream, g);
    KFAC_HIP_CHECK(hipGetLastError());
    return KFAC_OK;
}

template <int MODE>
int launch_mode(kfac_ctx *ctx, const ExpertArgs &g, int dtype) {
    const int es = dtype == KFAC_BF16 ? 2 : 4;
    const bool ragged = MODE == FORWARD || MODE == INPUT_GRAD;
    const double R = g.R, busy = std::min(g.E, g.R), all = g.cols + (ragged ? 0 : g.ones);
    double flops, bytes;   // by the rows handed over, as if every one had an expert and every expert rows
    if (ragged) {
        flops = 2.0 * R * g.K * g.cols;
        bytes = es * (R * (g.K + g.cols) + busy * g.K * g.cols);
    } else if (MODE == WEIGHT_GRAD) {
        flops = 2.0 * R * g.rows * all;
        bytes = es * R * (g.rows + g.cols) + (g.out_bf16 ? 2.0 : 4.0) * g.E * g.rows * all * (g.accumulate ? 2 : 1);
    } else {
        flops = R * all * (all + 1.0);
        bytes = es * R * g.cols + (g.decay != 0.f ? 8.0 : 4.0) * busy * all * all;
    }
    KfacProfScope prof(ctx, dtype == KFAC_BF16 ? KC_EXPERTS_B16 : KC_EXPERTS, flops, bytes);
    const bool wide = dtype == KFAC_BF16 && g.cols >= WIDE_MIN && (ragged ? g.K : g.rows) >= WIDE_MIN;
    if (wide) return launch_wide<MODE, 8, 4, 2, 4, 2>(ctx, g);
    const dim3 grid(grid_of(g, MODE, BM, BM));
    if (dtype == KFAC_BF16) hipLaunchKernelGGL((expert_tile_kernel<MODE, unsigned short>), grid, dim3(NTHREADS), 0, ctx->stream, g);
    else hipLaunchKernelGGL((expert_tile_kernel<MODE, float>), grid, dim3(NTHREADS), 0, ctx->stream, g);
    KFAC_HIP_CHECK(hipGetLastError());
    return KFAC_OK;
}

}  // namespace

int kfac_launch_experts_forward(kfac_ctx *ctx, const kfac_expert_desc *d, const void *X, int64_t ldx, const void *W, void *Y, int64_t ldy) {
    ExpertArgs g{};
    g.offsets = d->offsets;
    g.E = d->experts;
    g.R = d->rows;
    g.a = X;
    g.lda = ldx;
    g.b = W;
    g.ldb = d->d_in + d->append_ones;
    g.estride = (int64_t)d->d_out * g.ldb;
    g.out = Y;
    g.ldo = ldy;
    g.cols = d->d_out;
    g.K = d->d_in;
    g.ones = d->append_ones;
    g.out_bf16 = d->dtype == KFAC_BF16;
    return launch_mode<FORWARD>(ctx, g, d->dtype);
}

int kfac_launch_experts_input_grad(kfac_ctx *ctx, const kfac_expert_desc *d, const void *G, int64_t ldg, const void *W, void *dX, int64_t ldx) {
    ExpertArgs g{};
    g.offsets = d->offsets;
    g.E = d->experts;
    g.R = d->rows;
    g.a = G;
    g.lda = ldg;
    g.b = W;
    g.ldb = d->d_in + d->append_ones;
    g.estride = (int64_t)d->d_out * g.ldb;
    g.out = dX;
    g.ldo = ldx;
    g.cols = d->d_in;
    g.K = d->d_out;
    g.out_bf16 = d->dtype == KFAC_BF16;
    return launch_mode<INPUT_GRAD>(ctx, g, d->dtype);
}

int kfac_launch_experts_weight_grad(kfac_ctx *ctx, const kfac_expert_desc *d, const void *G, int64_t ldg, const void *X, int64_t ldx, int accumulate,
                                    void *dW, int grad_dtype) {
    ExpertArgs g{};
    g.offsets = d->offsets;
    g.E = d->experts;
    g.R = d->rows;
    g.a = G;
    g.lda = ldg;
    g.b = X;
    g.ldb = ldx;
    g.out = dW;
    g.ldo = d->d_in + d->append_ones;
    g.ostride = (int64_t)d->d_out * g.ldo;
    g.rows = d->d_out;
    g.cols = d->d_in;
    g.ones = d->append_ones;
    g.out_bf16 = grad_dtype == KFAC_BF16;
    g.accumulate = accumulate;
    return launch_mode<WEIGHT_GRAD>(ctx, g, d->dtype);
}

int kfac_launch_update_factors_experts(kfac_ctx *ctx, int experts, int rows, const int *offsets, const void *X, int dtype, int64_t ldx, int d, int append_ones,
                                       int mean, float scale, float decay, float *F) {
    ExpertArgs g{};
    g.offsets = offsets;
    g.E = experts;
    g.R = rows;
    g.a = X;
    g.lda = ldx;
    g.out = F;
    g.ldo = d + append_ones;
    g.ostride = g.ldo * g.ldo;
    g.rows = g.cols = d;
    g.ones = append_ones;
    g.mean = mean;
    g.scale = scale;
    g.decay = decay;
    return launch_mode<FACTORS>(ctx, g, dtype);
}
