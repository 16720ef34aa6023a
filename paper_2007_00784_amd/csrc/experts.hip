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
    int splits;              // parts of the contraction, each a workgroup's
    float *part;             // their sums, [tile][splits][..]
};

// A tile's contraction in parts: a first launch leaves the sums of each part in the workspace, a second one adds them in their order
// and goes on as a whole tile does.
enum { WHOLE = 0, PART = 1, JOIN = 2 };

struct Range { int beg, end; };
// Rows of expert e.  Whatever the offsets hold, the range lies inside the sample matrices.
__device__ inline Range range_of(const ExpertArgs &g, int e) {
    const int beg = min(max(g.offsets[e], 0), g.R);
    return Range{beg, min(max(g.offsets[e + 1], beg), g.R)};
}

// Where the workgroup's tile lies: expert, row tile and column tile.
struct Place { int e, m, n; Range r; int64_t t; };       // t: its number, for its parts in the workspace

// Rows ragged: expert e has ceil(rows / EXT) row tiles times `nt` column tiles.  The tiles of all experts, in order, are dealt to the eight XCDs
// in equal consecutive parts (workgroup b runs on XCD b % 8; the parts of a split contraction go round them), so that tiles that share
// operands share an L2; inside an expert the order goes over BAND row tiles before it takes the next column tile.
constexpr int BAND = 4;
template <int EXT>
__device__ inline bool place_ragged(const ExpertArgs &g, int nt, Place &p) {
    const int lane = threadIdx.x & 63;
    Range r{0, 0};          // of expert e0 + lane
    int mt = 0, incl = 0;   // its row tiles; those of the experts from e0 on, up to it
    auto look = [&](int e0) {
        const int e = e0 + lane;
        mt = 0;
        if (e < g.E) {
            r = range_of(g, e);
            mt = (r.end - r.beg + EXT - 1) / EXT;
        }
        incl = mt;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(incl, d);
            if (lane >= d) incl += o;
        }
        return __builtin_amdgcn_readlane(incl, 63);
    };
    int64_t total = 0;
    for (int e0 = 0; e0 < g.E; e0 += 64) total += look(e0);
    total = min(total * nt, (int64_t)gridDim.x);     // (descending offsets could ask for more tiles than there are workgroups, and places for their parts)
    const int64_t per = (total + 7) / 8, t = (int64_t)((blockIdx.x + blockIdx.y) & 7) * per + (blockIdx.x >> 3);
    if ((int64_t)(blockIdx.x >> 3) >= per || t >= total) return false;
    p.t = t;
    int64_t before = 0;
    for (int e0 = 0; e0 < g.E; e0 += 64) {
        if (g.E > 64) look(e0);
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

// Outputs fixed per expert: mt x nt tiles each (lower triangular ones of mt x mt where TRI), whose work goes with the expert's rows.
// Experts are taken in the order of their rows, the longest first (where one wave can hold them: 64 at most), so that no long one is left
// for the end; and each run of consecutive tiles of that order goes to the next XCD, so that every XCD has the same share of every expert
// and the tiles of a run share its L2.  (Runs of 4, 8, 16 and 32: weight gradient of 32 experts 2048 x 2048 over 32768 rows 357, 355, 359,
// 379 us, factors of 16 experts 283, 282, 295, 352; with few tiles the runs are shorter, so that all XCDs have some.)
__host__ __device__ inline int run_of(int64_t tiles) { return tiles >= 512 ? 8 : tiles >= 64 ? (int)(tiles / 64) : 1; }
__host__ __device__ inline int tiles_each(bool tri, int mt, int nt) { return tri ? mt * (mt + 1) / 2 : mt * nt; }
template <bool TRI>
__device__ inline bool place_fixed(const ExpertArgs &g, int mt, int nt, Place &p) {
    const int each = tiles_each(TRI, mt, nt);
    const int run = run_of((int64_t)each * g.E);
    const int64_t i = blockIdx.x >> 3, t = ((i / run) * 8 + ((blockIdx.x + blockIdx.y) & 7)) * run + i % run;
    if (t >= (int64_t)each * g.E) return false;
    p.t = t;
    const int place = (int)(t / each);
    int e = place;
    if (g.E <= 64) {
        const int lane = threadIdx.x & 63;
        int rows = -1;
        Range r{0, 0};
        if (lane < g.E) {
            r = range_of(g, lane);
            rows = r.end - r.beg;
        }
        // the row count in that place, bit by bit from the top: the largest that more than `place` experts reach; then the expert among its
        // equals (comparing all with all took 2.7 us a workgroup)
        int rows_at = 0;
        for (int bit = 31 - __builtin_clz(max(g.R, 1)); bit >= 0; --bit) {
            const int tried = rows_at | 1 << bit;
            if (__popcll(__ballot(rows >= tried)) > place) rows_at = tried;
        }
        const uint64_t equals = __ballot(rows == rows_at);
        const int behind = place - __popcll(__ballot(rows > rows_at));
        const int mine = __builtin_amdgcn_mbcnt_hi((unsigned)(equals >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)equals, 0));
        e = __builtin_ctzll(__ballot(rows == rows_at && mine == behind));
        p.r = Range{__builtin_amdgcn_readlane(r.beg, e), __builtin_amdgcn_readlane(r.end, e)};
    } else {
        p.r = range_of(g, e);
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

// A vector into memory at any element.  Results are not read again before the L2 has long been through other things; they go past it.
template <typename V, int ALIGN> __device__ inline void store_past(void *p, const V &v) {
    typedef V Anywhere __attribute__((aligned(ALIGN)));
    __builtin_nontemporal_store(v, reinterpret_cast<Anywhere *>(p));
}

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

// Between the lanes of a wave LDS goes in program order; this keeps the compiler to that order as well (it may move a lane's load past
// another address' store).  No instruction comes of it.
__device__ inline void wave_order() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
}

// ---- bf16: the wide engine ----
//
// Bound by the matrix core and LDS together where the sums are long (see mfma_gemm_wide.h), by what is written where they are short: 32
// weight gradients 2048 x 2048 over 32768 rows 322 us, of which 111 are the 537 MB of results at 4.8 TB/s; 16 factors 2049 wide over 32768
// rows 258 us, 137 of them with one slab of rows.
template <int FR, int FC, int WR, int WC> constexpr int wide_part() { return (FC * FR + FR / WC) * 64 * WR * WC * 4; }   // floats of one part

template <int MODE, int FR, int FC, int WR, int WC, int RING, int PHASE>
__global__ __launch_bounds__(64 * WR * WC, 2) void expert_wide_kernel(const ExpertArgs g) {
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
    constexpr int THREADS = 64 * WR * WC;
    constexpr bool AHEAD = RAGGED && NW == 8;
    const int nslab = (K + WK - 1) / WK;
    floatx4 *const part = reinterpret_cast<floatx4 *>(g.part + p.t * g.splits * wide_part<FR, FC, WR, WC>()) + threadIdx.x;
    constexpr int PART4 = wide_part<FR, FC, WR, WC>() / 4;
    // a join's workgroup adds two row fragments of every wave's (and the first one the sums), four parts' loads at a time
    auto joined = [&](int f) {
        const floatx4 *q = part + (int64_t)f * THREADS;
        floatx4 v = q[0];
        int u = 1;
        for (; u + 4 <= g.splits; u += 4) {
            floatx4 x[4];
#pragma unroll
            for (int y = 0; y < 4; ++y) x[y] = q[(int64_t)(u + y) * PART4];
#pragma unroll
            for (int y = 0; y < 4; ++y) v += x[y];
        }
        for (; u < g.splits; ++u) v += q[(int64_t)u * PART4];
        return v;
    };
    if constexpr (PHASE == JOIN) {
#pragma unroll
        for (int i = 0; i < FC; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) acc[i][j] = joined(i * FR + 2 * blockIdx.y + j);
        if (sums && blockIdx.y == 0)
#pragma unroll
            for (int j = 0; j < FR / WC; ++j) one[j] = joined(FC * FR + j);
    } else if constexpr (PHASE == PART) {
        const int per = (nslab + g.splits - 1) / g.splits, s0 = min((int)blockIdx.y * per, nslab), s1 = min(s0 + per, nslab);
        wide_tile<Row, Col, FR, FC, WR, WC, RING, ONES, AHEAD>(row, col, K, s0, s1, smem, acc, one, sums);
        floatx4 *const q = part + (int64_t)blockIdx.y * PART4;
#pragma unroll
        for (int i = 0; i < FC; ++i)
#pragma unroll
            for (int j = 0; j < FR; ++j) q[(i * FR + j) * THREADS] = acc[i][j];
#pragma unroll
        for (int j = 0; j < FR / WC; ++j) q[(FC * FR + j) * THREADS] = ONES ? one[j] : floatx4{0.f, 0.f, 0.f, 0.f};
        return;
    } else {
        if (RAGGED && count - p.m * ROWS <= ROWS - 16) wide_tile<Row, Col, FR, FC, WR, WC, RING, ONES, AHEAD, RAGGED>(row, col, K, 0, nslab, smem, acc, one, sums, count - p.m * ROWS);
        else wide_tile<Row, Col, FR, FC, WR, WC, RING, ONES, AHEAD>(row, col, K, 0, nslab, smem, acc, one, sums);
    }

    // Each wave turns its 64 columns round in LDS, 32 rows at a time, so that a store covers whole rows of them (128 or 256 bytes side
    // by side; the accumulators' own layout has 32 or 64).
    static_assert(FC == 4 && FR % 2 == 0, "64 columns of a wave");
    constexpr int PITCH = 64 + 4;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wr = wave / WC, wc = wave % WC;
    float *const turn = reinterpret_cast<float *>(smem) + wave * 32 * PITCH;
    const Average w = MODE == FACTORS ? average_of(g, count) : Average{};
    const int c0 = p.n * COLS + 64 * wc + 4 * (lane & 15);                      // four places side by side
    const bool whole = c0 + 4 <= (MODE == FORWARD ? g.cols : g.cols & ~7);
    float bias[4] = {0.f, 0.f, 0.f, 0.f};
    if (MODE == FORWARD && g.ones) {
        const unsigned short *W = (const unsigned short *)g.b + p.e * g.estride + g.K;
#pragma unroll
        for (int x = 0; x < 4; ++x) bias[x] = to_float(W[(int64_t)min(c0 + x, g.cols - 1) * g.ldb]);
    }
    __syncthreads();
#pragma unroll
    for (int pair = 0; pair < (PHASE == JOIN ? 1 : FR / 2); ++pair) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int i = 0; i < FC; ++i)
                *reinterpret_cast<floatx4 *>(turn + (16 * j + (lane & 15)) * PITCH + 16 * i + 4 * (lane >> 4)) = acc[i][2 * pair + j];
        wave_order();
        const int r0 = p.m * ROWS + 16 * (wr * FR + 2 * (PHASE == JOIN ? (int)blockIdx.y : pair));
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
                if (c0 + 3 <= r) {
                    floatx4 old = {0.f, 0.f, 0.f, 0.f};
                    if (w.keep != 0.f) __builtin_memcpy(&old, d, 16);
#pragma unroll
                    for (int x = 0; x < 4; ++x) v[x] = w.keep != 0.f ? fmaf(w.alpha, v[x], w.keep * old[x]) : w.alpha * v[x];
                    store_past<floatx4, 4>(d, v);
                } else {
#pragma unroll
                    for (int x = 0; x < 4; ++x)
                        if (c0 + x <= r) d[x] = v[x] = w.keep != 0.f ? fmaf(w.alpha, v[x], w.keep * d[x]) : w.alpha * v[x];
                }
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
                store_past<wide_bf16x4, 2>(d, b);
            } else {
                float *d = (float *)g.out + o;
                if (MODE == WEIGHT_GRAD && g.accumulate) {
                    floatx4 old;
                    __builtin_memcpy(&old, d, 16);
                    v += old;
                }
                store_past<floatx4, 4>(d, v);
            }
        }
        if (MODE == FACTORS) {
            wave_order();
            // the mirrored part: lane l takes rows 4 (l % 8).. of column l / 8, which lie side by side there
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                const int place = 8 * t + (lane >> 3), c = p.n * COLS + 64 * wc + place;
                if (c >= (g.cols & ~7)) continue;      // (places of a shifted group have stored theirs)
                floatx4 v;
#pragma unroll
                for (int x = 0; x < 4; ++x) v[x] = turn[(4 * (lane & 7) + x) * PITCH + place];
                const int first = r0 + 4 * (lane & 7);
                float *d = (float *)g.out + p.e * g.ostride + (int64_t)c * g.ldo;
                if (first + 4 <= (g.rows & ~7) && first > c) store_past<floatx4, 4>(d + first, v);
                else
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const int r = row.side(first + x);
                        if (r > c && r < g.rows) d[r] = v[x];
                    }
            }
        }
        wave_order();
    }
    if (sums && lane < 16 && (PHASE != JOIN || blockIdx.y == 0)) {
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

// ---- few rows (bf16 forward), small layers (fp32): operands straight from memory to the matrix core's registers ----
//
// A workgroup's waves share one tile of (16 RT) x (16 CT) outputs and take turns along the contraction, STEP indices each; their sums are
// added in a fixed order through LDS.  Nothing is staged: each lane loads what are its own operands of one or several matrix instructions,
// DEPTH steps of them in flight, so that a tile with a handful of rows streams its weights at the memory's rate, and many small tiles fill
// the chip.  (8 rows on seven of 8 experts 2048 x 2048: 12.7 us, 59 MB at 4.6 TB/s, a copy runs at 4.9.  fp32: what the call waits for
// are operands and the fullest compute unit: the input gradient of 577 x 512 over 1568 rows, 17.7 us, has its matrix cores busy for 7 and reads 4 to
// 7 TB/s from the L2, which gives 20 and more.)
//
// An operand along the contraction (X, G; W forward): lane l holds index 16 f + l % 16 of fragment f at k = V (l / 16).., V = 16 /
// sizeof(E) (one v_mfma_f32_16x16x32_bf16, or four v_mfma_f32_16x16x4_f32 of which number t takes element t).  An operand across it (fp32):
// F consecutive outputs of one row for each t, so that lane l holds index F (l % 16) + f of fragment f.
template <typename E> struct DirectTraits;
template <> struct DirectTraits<unsigned short> {
    static constexpr int V = 8, STEP = 32;
    typedef wide_bf16x8 Reg;
    typedef wide_bf16x8 Anywhere __attribute__((aligned(2)));   // in memory, at any element
};
template <> struct DirectTraits<float> {
    static constexpr int V = 4, STEP = 16;
    typedef floatx4 Reg;
    typedef floatx4 Anywhere __attribute__((aligned(4)));
};
template <typename E> __device__ inline typename DirectTraits<E>::Reg load16(const E *p) {
    return *as_global(reinterpret_cast<const typename DirectTraits<E>::Anywhere *>(p));
}

template <typename E, int F>
struct DirectAlong {
    static constexpr int V = DirectTraits<E>::V, STEP = DirectTraits<E>::STEP, REGS = F;
    using Reg = typename DirectTraits<E>::Reg;
    const E *p[F];
    int K;
    __device__ void start(const E *base, int64_t ld, int i0, int n, int K_) {
        const int lane = threadIdx.x & 63;
        K = K_;
#pragma unroll
        for (int f = 0; f < F; ++f) p[f] = base + (int64_t)min(i0 + 16 * f + (lane & 15), n - 1) * ld;
    }
    __device__ void fetch(int k0, Reg (&x)[REGS]) const {
        const int k = k0 + V * ((threadIdx.x & 63) >> 4);
        if (k0 + STEP <= K) {
#pragma unroll
            for (int f = 0; f < F; ++f) x[f] = load16<E>(p[f] + k);
        } else {     // the last V of the row, without those that the group before has; nothing behind that
            const int over = min(max(k + V - K, 0), V);
#pragma unroll
            for (int f = 0; f < F; ++f) {
                E e[V];
                const Reg last = load16<E>(p[f] + min(k, K - V));
                __builtin_memcpy(e, &last, 16);
#pragma unroll
                for (int v = 0; v < V; ++v) e[v] = v < over ? (E)0 : e[v];
                __builtin_memcpy(&x[f], e, 16);
            }
        }
    }
    __device__ static float part(const Reg (&x)[REGS], int f, int t) { return x[f][t]; }
    __device__ static constexpr int at(int f, int i) { return 16 * f + i; }
    __device__ int side(int place, int) const { return place; }
};

// MAPPED: the other operand is a DirectAlong, whose last group is shifted where K is no multiple of four.
template <int F, bool MAPPED>
struct DirectAcross {     // fp32
    static constexpr int STEP = 16, REGS = 4;
    typedef float Reg __attribute__((ext_vector_type(F)));
    typedef Reg Anywhere __attribute__((aligned(4)));
    const float *p;
    int64_t ld;
    int K;
    __device__ void start(const float *base, int64_t ld_, int i0, int n, int K_) {
        const int lane = threadIdx.x & 63, i = i0 + F * (lane & 15);
        K = K_;
        ld = ld_;
        p = base + min(i, n - F) + (int64_t)(4 * (lane >> 4)) * ld;
    }
    __device__ Reg load(int k) const { return *as_global(reinterpret_cast<const Anywhere *>(p + (int64_t)k * ld)); }
    __device__ void fetch(int k0, Reg (&x)[REGS]) const {
        const int k = k0 + 4 * ((threadIdx.x & 63) >> 4);
        if (k0 + STEP <= K) {
#pragma unroll
            for (int t = 0; t < 4; ++t) x[t] = load(k0 + t);
        } else {
            const int over = MAPPED ? min(max(k + 4 - K, 0), 4) : 0;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int back = over + max(k + t - over - (K - 1), 0);
                x[t] = load(k0 + t - back);
                if (t < over || k + t - over >= K) x[t] = 0.f;
            }
        }
    }
    __device__ static float part(const Reg (&x)[REGS], int f, int t) { return x[t][f]; }
    __device__ static constexpr int at(int f, int i) { return F * i + f; }
    __device__ int side(int place, int n) const { return across_side<F>(place, n); }
};

template <int RT, int CT> constexpr int direct_part() { return 16 * RT * (16 * CT + 4 + 1); }     // floats of one wave's sums

template <int MODE, typename E, int RT, int CT, int WAVES, int DEPTH>
__global__ __launch_bounds__(64 * WAVES) void expert_direct_kernel(const ExpertArgs g) {
    constexpr bool RAGGED = MODE == FORWARD || MODE == INPUT_GRAD, BF = sizeof(E) == 2;
    constexpr int ROWS = 16 * RT, COLS = 16 * CT, STEP = DirectTraits<E>::STEP, PITCH = COLS + 4;
    extern __shared__ __align__(16) float parts[];      // of each wave: [ROWS][PITCH], then [ROWS] sums of the row operand
    constexpr int SIZE = direct_part<RT, CT>();
    const int nt = (g.cols + COLS - 1) / COLS;
    Place p;
    if (RAGGED ? !place_ragged<ROWS>(g, nt, p) : !place_fixed<MODE == FACTORS>(g, (g.rows + ROWS - 1) / ROWS, nt, p)) return;
    const int count = p.r.end - p.r.beg;
    if (MODE == FACTORS && count == 0 && (g.mean || g.decay == 1.f)) return;
    if (MODE == WEIGHT_GRAD && count == 0 && g.accumulate) return;
    const E *a = (const E *)g.a + p.r.beg * g.lda;
    const int K = RAGGED ? g.K : count, rows = RAGGED ? count : g.rows;
    const bool sums = !RAGGED && g.ones && p.n == 0;
    using Row = std::conditional_t<RAGGED, DirectAlong<E, RT>, DirectAcross<RT, false>>;
    using Col = std::conditional_t<MODE == FORWARD, DirectAlong<E, CT>, DirectAcross<CT, MODE == INPUT_GRAD>>;
    Row row;
    Col col;
    row.start(a, g.lda, p.m * ROWS, rows, K);
    if constexpr (RAGGED) col.start((const E *)g.b + p.e * g.estride, g.ldb, p.n * COLS, g.cols, K);
    else if constexpr (MODE == WEIGHT_GRAD) col.start((const E *)g.b + p.r.beg * g.ldb, g.ldb, p.n * COLS, g.cols, K);
    else col.start(a, g.lda, p.n * COLS, g.cols, K);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    floatx4 acc[CT][RT];
#pragma unroll
    for (int i = 0; i < CT; ++i)
#pragma unroll
        for (int j = 0; j < RT; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
    float total[RT];
#pragma unroll
    for (int j = 0; j < RT; ++j) total[j] = 0.f;
    typename Row::Reg x[DEPTH][Row::REGS];
    typename Col::Reg y[DEPTH][Col::REGS];
    constexpr int ROUND = STEP * WAVES;
    const int k_first = wave * STEP;
    auto multiply = [&](int d) {
        if constexpr (BF) {
#pragma unroll
            for (int j = 0; j < RT; ++j)
#pragma unroll
                for (int i = 0; i < CT; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y[d][i], x[d][j], acc[i][j], 0, 0, 0);
        } else {
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int j = 0; j < RT; ++j) {
                    const float r = Row::part(x[d], j, t);
                    if (!RAGGED) total[j] += r;
#pragma unroll
                    for (int i = 0; i < CT; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(Col::part(y[d], i, t), r, acc[i][j], 0, 0, 0);
                }
        }
    };
    if (K > 0) {
#pragma unroll
        for (int d = 0; d < DEPTH; ++d)
            if (k_first + d * ROUND < K) {
                row.fetch(k_first + d * ROUND, x[d]);
                col.fetch(k_first + d * ROUND, y[d]);
            }
        for (int k = k_first; k < K; k += DEPTH * ROUND) {
#pragma unroll
            for (int d = 0; d < DEPTH; ++d) {
                if (k + d * ROUND < K) multiply(d);
                const int next = k + (d + DEPTH) * ROUND;
                if (next < K) {
                    row.fetch(next, x[d]);
                    col.fetch(next, y[d]);
                }
            }
        }
    }
    {    // every wave's sums into LDS, consecutive columns at a time
        float *const mine = parts + wave * SIZE;
#pragma unroll
        for (int j = 0; j < RT; ++j) {
            const int r = Row::at(j, lane & 15);
            if constexpr (MODE != FORWARD) {
#pragma unroll
                for (int x4 = 0; x4 < 4; ++x4)
#pragma unroll
                    for (int i = 0; i < CT; ++i) mine[r * PITCH + CT * (4 * (lane >> 4) + x4) + i] = acc[i][j][x4];
            } else {
#pragma unroll
                for (int i = 0; i < CT; ++i) *reinterpret_cast<floatx4 *>(mine + r * PITCH + 16 * i + 4 * (lane >> 4)) = acc[i][j];
            }
        }
        if (!RAGGED && sums) {
#pragma unroll
            for (int j = 0; j < RT; ++j) {
                total[j] += __shfl_xor(total[j], 16);
                total[j] += __shfl_xor(total[j], 32);
                if (lane < 16) mine[ROWS * PITCH + Row::at(j, lane)] = total[j];
            }
        }
        __syncthreads();
    }
    const Average w = MODE == FACTORS ? average_of(g, count) : Average{};
    for (int q = threadIdx.x; q < ROWS * COLS / 4; q += 64 * WAVES) {
        const int at = q / (COLS / 4), c_at = 4 * (q % (COLS / 4)), c0 = p.n * COLS + c_at;
        const int r = row.side(p.m * ROWS + at, rows);
        if (r < 0 || r >= rows) continue;
        floatx4 v = *reinterpret_cast<const floatx4 *>(parts + at * PITCH + c_at);
#pragma unroll
        for (int u = 1; u < WAVES; ++u) v += *reinterpret_cast<const floatx4 *>(parts + u * SIZE + at * PITCH + c_at);
#pragma unroll
        for (int x4 = 0; x4 < 4; ++x4) {
            const int c = col.side(c0 + x4, g.cols);
            if (c < 0 || c >= g.cols || (MODE == FACTORS && c > r)) continue;
            float z = v[x4];
            if (MODE == FORWARD && g.ones) z += to_float(((const E *)g.b)[p.e * g.estride + (int64_t)c * g.ldb + g.K]);
            finish<MODE>(g, p.e, RAGGED ? p.r.beg + r : r, c, z, w);
        }
    }
    if (!RAGGED && sums) {
        for (int at = threadIdx.x; at < ROWS; at += 64 * WAVES) {
            const int r = row.side(p.m * ROWS + at, rows);
            if (r < 0 || r >= rows) continue;
            float t = parts[ROWS * PITCH + at];
#pragma unroll
            for (int u = 1; u < WAVES; ++u) t += parts[u * SIZE + ROWS * PITCH + at];
            if (MODE == WEIGHT_GRAD) finish<MODE>(g, p.e, r, g.cols, t, w);
            else finish<MODE>(g, p.e, g.rows, r, t, w);
        }
        if (MODE == FACTORS && p.m == 0 && threadIdx.x == 0) finish<MODE>(g, p.e, g.rows, g.rows, (float)count, w);
    }
}

// ---- fp32, and bf16 with a side shorter than the wide engine's groups: the element-wise engine (fp32 matrix instructions) ----
constexpr int TILE_PART = BM * BM + BM;     // floats of one part: the accumulators, then the sums of the row operand
template <int MODE, typename E, int PHASE>
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
    WaveMap map = wave_map_edge(min(rows - i0, BM), min(g.cols - j0, BM));
    using Row = OpStrided<E, RAGGED>;
    using Col = OpStrided<E, MODE == FORWARD>;
    // (a part ends at k1: what is behind it belongs to the next one, and slabs end where BK does)
    Row A{a, RAGGED ? g.lda : 1, RAGGED ? 1 : g.lda, rows, K, -1};
    const E *b = (const E *)uniform_ptr(MODE == FORWARD || MODE == INPUT_GRAD ? (const E *)g.b + p.e * g.estride
                                        : MODE == WEIGHT_GRAD ? (const E *)g.b + p.r.beg * g.ldb : a);
    const int64_t ldb = MODE == FACTORS ? g.lda : g.ldb;
    Col B{b, MODE == FORWARD ? ldb : 1, MODE == FORWARD ? 1 : ldb, g.cols, K, -1};
    A.seg_k = B.seg_k = 0;
    const int slabs = (K + BK - 1) / BK, per = PHASE == PART ? (slabs + g.splits - 1) / g.splits : slabs;
    const int k0 = PHASE == PART ? min((int)blockIdx.y * per, slabs) * BK : 0, k1 = PHASE == PART ? min(k0 + per * BK, K) : K;
    float *const stored = g.part + p.t * g.splits * TILE_PART;
    if (PHASE == JOIN) {     // a workgroup adds one 32 x 32 block of every wave's (and the first one the sums)
        const int block = blockIdx.y;
        map = WaveMap{map.wm + 32 * (block >> 1), map.wn + 32 * (block & 1), (map.blocks >> block) & 1u};
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[0][0][r] = 0.f;
        for (int u = 0; u < g.splits; ++u) {
            const float *q = stored + (int64_t)u * TILE_PART + block * 16 * NTHREADS + threadIdx.x;
            float x[16];
#pragma unroll
            for (int r = 0; r < 16; ++r) x[r] = q[r * NTHREADS];
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[0][0][r] += x[r];
        }
        if (sums && threadIdx.x < BM) {
            float t = 0.f;
            for (int u = 0; u < g.splits; ++u) t += stored[(int64_t)u * TILE_PART + BM * BM + threadIdx.x];
            cs[threadIdx.x] = t;
        }
    } else if (sums) {
        float csum[EPT];
#pragma unroll
        for (int s = 0; s < EPT; ++s) csum[s] = 0.f;
        gemm_tile<Row, Col, true, true>(A, B, i0, j0, k0, k1, sm, acc, csum, true, map);
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
        gemm_tile<Row, Col, false, true>(A, B, i0, j0, k0, k1, sm, acc, nullptr, true, map);
    }
    if (PHASE == PART) {
        float *const q = stored + (int64_t)blockIdx.y * TILE_PART;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) q[((i * 2 + j) * 16 + r) * NTHREADS + threadIdx.x] = acc[i][j][r];
        if (sums && threadIdx.x < BM) q[BM * BM + threadIdx.x] = cs[threadIdx.x];
        return;
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
    if (sums && (PHASE != JOIN || blockIdx.y == 0)) {
        const int r = i0 + threadIdx.x;
        if (threadIdx.x < BM && r < rows) {
            if (MODE == WEIGHT_GRAD) finish<MODE>(g, p.e, r, g.cols, cs[threadIdx.x], w);
            else finish<MODE>(g, p.e, g.rows, r, cs[threadIdx.x], w);
        }
        if (MODE == FACTORS && p.m == 0 && threadIdx.x == 0) finish<MODE>(g, p.e, g.rows, g.rows, (float)count, w);
    }
}

// ---- launches ----
int64_t grid_of(const ExpertArgs &g, int mode, int ext_r, int ext_c) {
    const int64_t nt = (g.cols + ext_c - 1) / ext_c;
    int64_t tiles;
    if (mode == FORWARD || mode == INPUT_GRAD) tiles = ((int64_t)g.R / ext_r + std::min<int64_t>(g.E, g.R)) * nt;
    else {
        const int64_t mt = (g.rows + ext_r - 1) / ext_r;
        tiles = (int64_t)tiles_each(mode == FACTORS, (int)mt, (int)nt) * g.E;
    }
    const int64_t unit = mode == FORWARD || mode == INPUT_GRAD ? 8 : 8 * run_of(tiles);
    return (tiles + unit - 1) / unit * unit;
}

bool fits_launch(int64_t tiles, int threads) { return tiles * threads < (int64_t)1 << 32; }     // what a launch can have

template <typename F> int launch_one(kfac_ctx *ctx, F kernel, int64_t tiles, int parts, int threads, int lds, const ExpertArgs &g) {
    if (!fits_launch(tiles, threads)) return KFAC_EINVAL;     // (not in the largest tiles either: no such layer fits the memory)
    const dim3 grid((unsigned)tiles, (unsigned)parts);
    if (lds > ctx->max_lds) return KFAC_EHIP;
    if (lds > 65536) KFAC_HIP_CHECK(hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds));
    hipLaunchKernelGGL(kernel, grid, dim3(threads), lds, ctx->stream, g);
    KFAC_HIP_CHECK(hipGetLastError());
    return KFAC_OK;
}

template <int MODE, int FR, int FC, int WR, int WC, int RING, bool SPLIT>
int launch_wide(kfac_ctx *ctx, ExpertArgs g, int splits) {
    constexpr int lds = ((RING + 1) * 16 * FR * WR + RING * 16 * FC * WC) * WK * 2, threads = 64 * WR * WC;
    const int64_t tiles = grid_of(g, MODE, 16 * FR * WR, 16 * FC * WC);
    if constexpr (SPLIT) {
        if (splits > 1) {
            g.splits = splits;
            g.part = (float *)ctx->ws;
            KFAC_CHECK(launch_one(ctx, expert_wide_kernel<MODE, FR, FC, WR, WC, RING, PART>, tiles, splits, threads, lds, g));
            return launch_one(ctx, expert_wide_kernel<MODE, FR, FC, WR, WC, RING, JOIN>, tiles, FR / 2, threads, threads / 64 * 32 * 68 * 4, g);
        }
    }
    return launch_one(ctx, expert_wide_kernel<MODE, FR, FC, WR, WC, RING, WHOLE>, tiles, 1, threads, lds, g);
}

template <int MODE, typename E, int RT, int CT, int WAVES, int DEPTH>
int launch_direct(kfac_ctx *ctx, const ExpertArgs &g) {
    return launch_one(ctx, expert_direct_kernel<MODE, E, RT, CT, WAVES, DEPTH>, grid_of(g, MODE, 16 * RT, 16 * CT), 1, 64 * WAVES, WAVES * direct_part<RT, CT>() * 4, g);
}

template <int MODE, typename E>
int launch_tiles(kfac_ctx *ctx, ExpertArgs g, int splits) {
    const int64_t tiles = grid_of(g, MODE, BM, BM);
    if (splits > 1) {
        g.splits = splits;
        g.part = (float *)ctx->ws;
        KFAC_CHECK(launch_one(ctx, expert_tile_kernel<MODE, E, PART>, tiles, splits, NTHREADS, 0, g));
        return launch_one(ctx, expert_tile_kernel<MODE, E, JOIN>, tiles, 4, NTHREADS, 0, g);
    }
    return launch_one(ctx, expert_tile_kernel<MODE, E, WHOLE>, tiles, 1, NTHREADS, 0, g);
}

// ---- which kernel a call takes ----
enum Engine { DIRECT_FEW = 0, DIRECT_SOME, DIRECT_SMALL, WIDE, WIDE_SMALL, TILES, DIRECT_MEDIUM };
struct Plan { Engine engine; int splits; };
struct Shape { int rows, cols, threads; };      // of an engine's tile, and its workgroup
Shape shape_of(Engine e) {
    switch (e) {
        case DIRECT_FEW: return {16, 32, 256};
        case DIRECT_SOME: return {32, 64, 256};
        case DIRECT_SMALL: return {32, 32, 256};
        case DIRECT_MEDIUM: return {32, 64, 256};
        case WIDE: return {256, 256, 512};
        case WIDE_SMALL: return {128, 128, 256};
        case TILES: break;
    }
    return {BM, BM, NTHREADS};
}
constexpr int MOST_SPLITS = 32;

// The engines that a call can take are priced in us from its sizes alone (the offsets are on the device: every expert is taken to have rows
// / experts of them), and the cheapest one runs.
Plan plan_of(const ExpertArgs &g, int mode, int dtype, size_t ws) {
    const bool ragged = mode == FORWARD || mode == INPUT_GRAD;
    const int shortest = std::min(g.cols, ragged ? g.K : g.rows);
    const double busy = std::min(g.E, std::max(g.R, 1)), each = std::max(1.0, g.R / busy), K = ragged ? g.K : each;
    const double es = dtype == KFAC_BF16 ? 2.0 : 4.0;
    const double weights = ragged ? busy * g.K * g.cols * es : mode == WEIGHT_GRAD ? 4.0 * g.E * g.rows * g.cols : 8.0 * busy * g.cols * g.cols;
    const double hbm = (weights + es * g.R * (double)(ragged ? g.K + g.cols : g.rows + (mode == FACTORS ? 0 : g.cols))) / 4.5e6;
    auto tiles = [&](double ext_r, double ext_c) {
        const double nt = std::ceil(g.cols / ext_c);
        if (ragged && g.E == 1) return std::ceil(each / ext_r) * nt;
        if (ragged) return busy * std::max(1.0, each / ext_r + 0.6) * nt;     // (half a tile is lost behind each expert's rows, and they differ)
        const double mt = std::ceil(g.rows / ext_r);
        return (mode == FACTORS ? mt * (mt + 1) / 2 : mt * nt) * busy;
    };
    // of sums over rows, the longest expert's takes the most, and where there is a compute unit for every tile it is what the call takes
    const double longest = !ragged && g.E > 1 ? 1.5 : 1.0;
    Plan best{TILES, 1};
    double least = 1e300;
    auto offer = [&](Engine e, int splits, double cost) {
        const Shape t = shape_of(e);
        if (cost < least && fits_launch(grid_of(g, mode, t.rows, t.cols), t.threads)) {
            least = cost;
            best = Plan{e, splits};
        }
    };
    // an engine whose sums can go in up to `most` parts: `slots` workgroups run at once; a step of the contraction takes `alone` in a workgroup that has its compute unit to itself
    // and `full` where all slots are taken; parts cost the way to memory and back, and a second launch; `stream`: what
    // reading and writing what the call cannot do without takes, over the rate of a copy
    auto offer_split = [&](Engine e, int most, double t, double slots, double steps, double alone, double full, double fixed, double stream, size_t part_bytes, size_t grid) {
        for (int s = 1; s <= most && (s == 1 || steps / s >= 4.0); s *= 2) {
            if (s > 1 && (size_t)s * part_bytes * grid > ws) break;
            const double wgs = t * s, units = slots / 256.0, there = std::min(units, std::ceil(wgs / 256.0));     // on the fullest compute unit
            const double step = units > 1.0 ? alone + (full - alone) * (there - 1.0) / (units - 1.0) : alone + (full - alone) * std::min(1.0, wgs / 256.0);
            const double n = std::ceil(steps / s), run = std::max({std::ceil(wgs / slots) * (fixed + n * step), longest * (fixed + n * alone), stream * hbm});
            offer(e, s, 3.0 + run + (s > 1 ? 5.0 + 2.0 * (double)part_bytes * t * s / 2.5e6 + 0.3 * s : 0.0));
        }
    };
    if (dtype == KFAC_BF16 && shortest >= WIDE_MIN) {
        if (mode == FORWARD) {
            // the weights are streamed past 16 or 32 rows at a time; us: 8 experts of 2048 x 2048 with 8 rows each 15.1, 15.7 and
            // (WIDE_SMALL) 21.4, with 32 26.6, 17.5 and 22.2; 64 of 1024 x 2048 with 16 each 74.0, 67.2 and 70.5, with 64 each 194, 111 and
            // 75.4
            const double few = tiles(16, 32), some = tiles(32, 64);
            offer(DIRECT_FEW, 1, 5.0 + std::max({0.28 * K / 128 * std::max(1.0, few / 1024), hbm, few * 48.0 * 2.0 * K / 9.4e6}));
            offer(DIRECT_SOME, 1, 5.0 + std::max({0.62 * K / 128 * std::max(1.0, some / 512), hbm, some * 96.0 * 2.0 * K / 9.4e6}));
        }
        // us: one 1024 x 1024 layer forward over 4096 rows 27.5 and 15.9; 8 of 4096 x 4096 over 32768 872 and 1175; weight gradient 512 x 512
        // over 32768 rows 654 and 337, in 16 parts 60
        const double slabs = K / WK;
        offer_split(WIDE, 1, tiles(256, 256), 256, slabs, 1.1, 1.55, 4.0, 1.25, 0, 0);
        offer_split(WIDE_SMALL, MOST_SPLITS, tiles(128, 128), 512, slabs, 0.72, 1.25, 3.0, 1.15, wide_part<4, 4, 2, 2>() * 4, grid_of(g, mode, 128, 128));
        return best;
    }
    // us, in tiles of 32 x 32, of 32 x 64 and (TILES) of 128 x 128: forward 512 x 512 of 8 experts over 64 rows 8.8, 10.0, 26; input
    // gradient 577 x 512 of 8 over 1568 23.3, 19.7, 52.5; weight gradient 1001 x 512 of 10 over 1000 40, 31.4, 44; 512 x 512 of 16 over
    // 16384 (32 x 64, TILES) 107 and 174; one 1024 x 1024 forward over 4096 138, 125, 97
    if (dtype == KFAC_F32 && shortest >= 4) {
        offer(DIRECT_SMALL, 1, 6.0 + std::max(hbm, std::max(longest, tiles(32, 32) / 256.0) * K * 0.0085));
        if (mode != FACTORS) offer(DIRECT_MEDIUM, 1, 6.0 + std::max(hbm, std::max(longest, tiles(32, 64) / 256.0) * K * (mode == FORWARD ? 0.0145 : 0.012)));
    }
    offer_split(TILES, MOST_SPLITS, tiles(128, 128), 768, K / BK, 1.36, 3.6, 3.0, 1.0, TILE_PART * 4, grid_of(g, mode, BM, BM));
    return best;
}

template <int MODE>
int launch_mode(kfac_ctx *ctx, const ExpertArgs &g, int dtype) {
    const int es = dtype == KFAC_BF16 ? 2 : 4;
    constexpr bool ragged = MODE == FORWARD || MODE == INPUT_GRAD;
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
    const Plan plan = plan_of(g, MODE, dtype, ctx->ws_bytes);
    switch (plan.engine) {
        case DIRECT_FEW:
            if constexpr (MODE == FORWARD) return launch_direct<MODE, unsigned short, 1, 2, 4, 8>(ctx, g);
            break;
        case DIRECT_SOME:
            if constexpr (MODE == FORWARD) return launch_direct<MODE, unsigned short, 2, 4, 4, 2>(ctx, g);
            break;
        case DIRECT_SMALL: return launch_direct<MODE, float, 2, 2, 4, ragged ? 2 : 6>(ctx, g);
        case DIRECT_MEDIUM:
            // (steps in flight: 1, 2, 4: forward 577 x 512 of 8 experts over 1568 rows 24.1, 23.4, 23.7 us, input gradient of 1024 x 1024
            // over 512 18.4, 16.8, 16.1, weight gradient of the table above 31.4, 34.4, 40.1)
            if constexpr (MODE != FACTORS) return launch_direct<MODE, float, 2, 4, 4, MODE == FORWARD ? 2 : MODE == INPUT_GRAD ? 4 : 1>(ctx, g);
            break;
        case WIDE: return launch_wide<MODE, 8, 4, 2, 4, 2, false>(ctx, g, 1);
        case WIDE_SMALL: return launch_wide<MODE, 4, 4, 2, 2, 2, true>(ctx, g, plan.splits);
        case TILES: break;
    }
    return dtype == KFAC_BF16 ? launch_tiles<MODE, unsigned short>(ctx, g, plan.splits) : launch_tiles<MODE, float>(ctx, g, plan.splits);
}

}  // namespace

namespace {

ExpertArgs args_of(int mode, const kfac_expert_desc *d) {
    ExpertArgs g{};
    g.offsets = d->offsets;
    g.E = d->experts;
    g.R = d->rows;
    g.ones = mode == INPUT_GRAD ? 0 : d->append_ones;
    const int64_t wide = d->d_in + d->append_ones;      // row of an expert's matrix
    if (mode == FORWARD || mode == INPUT_GRAD) {
        g.cols = mode == FORWARD ? d->d_out : d->d_in;
        g.K = mode == FORWARD ? d->d_in : d->d_out;
        g.ldb = wide;
        g.estride = d->d_out * wide;
        g.out_bf16 = d->dtype == KFAC_BF16;
    } else {
        g.rows = mode == FACTORS ? d->d_in : d->d_out;
        g.cols = d->d_in;
        g.ldo = wide;
        g.ostride = (mode == FACTORS ? wide : d->d_out) * wide;
    }
    return g;
}

size_t part_bytes(Engine e) { return e == WIDE_SMALL ? wide_part<4, 4, 2, 2>() * sizeof(float) : TILE_PART * sizeof(float); }

}  // namespace

extern "C" int kfac_experts_plan(int mode, const kfac_expert_desc *d, size_t workspace_bytes) {
    const Plan p = plan_of(args_of(mode, d), mode, d->dtype, workspace_bytes);
    return 100 * p.engine + p.splits;
}

size_t kfac_experts_ws_bytes_impl(const kfac_expert_desc *d) {
    size_t need = 0;
    kfac_expert_desc turned = *d;       // the factor of the output gradients
    turned.d_in = d->d_out;
    turned.append_ones = 0;
    for (int mode = FORWARD; mode <= FACTORS + 1; ++mode) {
        const int m = std::min<int>(mode, FACTORS);
        const ExpertArgs g = args_of(m, mode > FACTORS ? &turned : d);
        const Plan p = plan_of(g, m, d->dtype, SIZE_MAX / 2);
        if (p.splits > 1) need = std::max(need, (size_t)p.splits * part_bytes(p.engine) * grid_of(g, m, BM, BM));
    }
    return kfac_align_up(need, 256);
}

int kfac_launch_experts_forward(kfac_ctx *ctx, const kfac_expert_desc *d, const void *X, int64_t ldx, const void *W, void *Y, int64_t ldy) {
    ExpertArgs g = args_of(FORWARD, d);
    g.a = X;
    g.lda = ldx;
    g.b = W;
    g.out = Y;
    g.ldo = ldy;
    return launch_mode<FORWARD>(ctx, g, d->dtype);
}

int kfac_launch_experts_input_grad(kfac_ctx *ctx, const kfac_expert_desc *d, const void *G, int64_t ldg, const void *W, void *dX, int64_t ldx) {
    ExpertArgs g = args_of(INPUT_GRAD, d);
    g.a = G;
    g.lda = ldg;
    g.b = W;
    g.out = dX;
    g.ldo = ldx;
    return launch_mode<INPUT_GRAD>(ctx, g, d->dtype);
}

int kfac_launch_experts_weight_grad(kfac_ctx *ctx, const kfac_expert_desc *d, const void *G, int64_t ldg, const void *X, int64_t ldx, int accumulate,
                                    void *dW, int grad_dtype) {
    ExpertArgs g = args_of(WEIGHT_GRAD, d);
    g.a = G;
    g.lda = ldg;
    g.b = X;
    g.ldb = ldx;
    g.out = dW;
    g.out_bf16 = grad_dtype == KFAC_BF16;
    g.accumulate = accumulate;
    return launch_mode<WEIGHT_GRAD>(ctx, g, d->dtype);
}

int kfac_launch_update_factors_experts(kfac_ctx *ctx, int experts, int rows, const int *offsets, const void *X, int dtype, int64_t ldx, int d, int append_ones,
                                       int mean, float scale, float decay, float *F) {
    const kfac_expert_desc desc{experts, rows, d, d, append_ones, dtype, offsets};
    ExpertArgs g = args_of(FACTORS, &desc);
    g.a = X;
    g.lda = ldx;
    g.out = F;
    g.mean = mean;
    g.scale = scale;
    g.decay = decay;
    return launch_mode<FACTORS>(ctx, g, dtype);
}
