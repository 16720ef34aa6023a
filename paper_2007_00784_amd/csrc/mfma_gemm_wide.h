// bf16 MFMA tile engine for operands in rows ([rows][d], d contiguous): one workgroup computes C = sum_k R(r, k) Q(c, k) for a
// tile of ROWS x COLS outputs, K in slabs of 64 through a ring of LDS buffers for each operand.  An operand lies in memory in one of two ways:
//   OpAlong   the contraction index is the contiguous one (rows of X against rows of W)
//   OpAcross  the output index is the contiguous one (columns of W, of G or of X; the contraction walks over rows)
// Both are moved by 16-byte loads that land in LDS (no registers, no LDS stores), and both end as the same operand registers of
// v_mfma_f32_16x16x32_bf16: eight consecutive k of one output index per lane.  OpAlong reads them as one 16-byte LDS read; OpAcross
// reads four k of sixteen columns at a time with the transposing LDS read (ds_read_b64_tr_b16: of a group of sixteen lanes, lane i
// names the 8 bytes at row i / 4, columns 4 (i % 4)..; it is given column i of the four rows).
//
// Measured (8192 x 8192 x 8192): 774 us, 1420 TFLOP/s; without the loads 1654, with all of them hits in the L2 1427.  A slab of a 256 x 256
// tile is 2048 cycles of matrix instructions for each SIMD, 192 KB of LDS reads (1536 cycles) and 64 KB that land in LDS (512): both pipes
// are full at once.
//
// The matrix core's first operand is the COLUMN side, so a lane's four accumulator registers are four consecutive columns of one
// output row, which it stores as one vector.
//
// No load leaves its row: a group of eight that runs past the end of a row is taken from the row's last eight elements instead.  Along the
// contraction the elements that the group before had already are cleared once they have landed; across it, the tile simply has them twice
// and side() says which column a place stands for.  So an extent of 8 at least is assumed, and any pitch.  What is outside an
// operand (rows behind the last, k behind the end) is loaded with an offset that the buffer's range check turns into zeros.
#pragma once
#include <type_traits>
#include "mfma_gemm.h"

namespace kfac {

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef __bf16 wide_bf16x8 __attribute__((ext_vector_type(8)));
typedef short wide_s16x4 __attribute__((ext_vector_type(4)));

constexpr int WK = 64;                      // contraction indices of a slab: 128 bytes of a row, a whole cache line
constexpr int WIDE_MIN = 8;                 // smallest extent of any side

__device__ inline const void *uniform_ptr(const void *p) {
    const uint64_t a = (uint64_t)p;
    return (const void *)(((uint64_t)(unsigned)__builtin_amdgcn_readfirstlane((int)(a >> 32)) << 32) | (unsigned)__builtin_amdgcn_readfirstlane((int)a));
}

// 64 x 16 bytes from `off` bytes behind the descriptor's base into 1 KB of LDS at `lds` (the same for the whole wave), lane l at 16 l.
// The compiler would make every later LDS read wait for it, whatever part of LDS it reads; the waits stand in the loop.
typedef int wide_rsrc __attribute__((ext_vector_type(4)));
__device__ inline wide_rsrc wide_buffer(const void *base, unsigned extent) {
    const uint64_t a = (uint64_t)uniform_ptr(base);
    return wide_rsrc{(int)a, (int)(a >> 32) & 0xffff, __builtin_amdgcn_readfirstlane((int)extent), 0x00020000};
}
__device__ inline void load_to_lds(wide_rsrc rs, unsigned off, unsigned lds) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(off), "s"(rs), "s"(lds) : "memory", "m0");
}
__device__ inline unsigned lds_address(const void *p) {
    return (unsigned)(uintptr_t)(const __attribute__((address_space(3))) char *)p;
}

// Which output index the place `at` (from the matrix' first on) of an operand that is read in groups of G along its `n` outputs stands for,
// or -1: the group of places that begins at n - r, 0 < r < G left over, holds the last G outputs, of which the first G - r are already
// there.
template <int G>
__device__ inline int across_side(int at, int n) {
    const int r = n % G, last = n - r;
    if (at < last) return at;
    if (r == 0 || at >= last + G) return -1;
    return at - last >= G - r ? at - (G - r) : -1;
}

// elem(i, k) = p[i * ld + k], i < rows, k < K; K >= 8.  EXT output indices from `i0` on; NW waves.
template <int EXT, int NW>
struct OpAlong {
    static constexpr int LOADS = EXT / 8 / NW, BYTES = EXT * WK * 2;
    const unsigned short *p;      // row i0
    int64_t ld;
    int K;
    unsigned extent, off[LOADS];
    int g;                        // group of eight k of this thread, the same for its loads
    unsigned place;               // LDS offset of the wave's first load in a slab
    __device__ void start(const unsigned short *base, int64_t ld_, int i0, int rows, int K_) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        ld = ld_;
        K = K_;
        p = (const unsigned short *)uniform_ptr(base + (int64_t)i0 * ld);
        extent = (unsigned)((int64_t)min(rows - i0, EXT) * ld * 2);
        place = __builtin_amdgcn_readfirstlane(wave * 1024);
        g = (lane & 7) ^ (lane >> 3);
#pragma unroll
        for (int u = 0; u < LOADS; ++u) off[u] = (unsigned)((wave * 8 + (lane >> 3) + u * 8 * NW) * ld * 2 + g * 16);
    }
    __device__ int over(int k0) const { return min(max(k0 + 8 * g + 8 - K, 0), 8); }    // of the group's eight, how many are behind the end
    // load u of a slab that ends before K
    __device__ void issue_inside(unsigned slab, int k0, int u) const { load_to_lds(wide_buffer(p + k0, extent - 2u * k0), off[u], slab + place + u * NW * 1024); }
    __device__ void issue(unsigned slab, int k0) const {
        slab += place;
        if (k0 + WK <= K) {
#pragma unroll
            for (int u = 0; u < LOADS; ++u) issue_inside(slab - place, k0, u);
        } else {
            const auto rs = wide_buffer(p, extent);
            const int o = over(k0);
#pragma unroll
            for (int u = 0; u < LOADS; ++u)
                load_to_lds(rs, o < 8 ? off[u] + 2u * k0 - 2u * o : BUF_OUTSIDE, slab + u * NW * 1024);
        }
    }
    // Once the slab's loads have landed: clear what the last, shifted group holds of the one before.
    __device__ void patch(char *slab, int k0) const {
        const int o = over(k0);
        if (o == 0 || o == 8) return;
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        unsigned keep[4];
#pragma unroll
        for (int w = 0; w < 4; ++w) keep[w] = (2 * w >= o ? 0xffffu : 0u) | (2 * w + 1 >= o ? 0xffff0000u : 0u);
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
            uint4 *x = reinterpret_cast<uint4 *>(slab + (wave + u * NW) * 1024 + lane * 16);
            uint4 v = *x;
            v.x &= keep[0]; v.y &= keep[1]; v.z &= keep[2]; v.w &= keep[3];
            *x = v;
        }
    }
    // The registers of output indices i .. i + 15 (i a multiple of 16, in the tile) and of half `ks` of the slab.
    __device__ static wide_bf16x8 fragment(const char *slab, int i, int ks) {
        const int lane = threadIdx.x & 63;
        wide_bf16x8 x;
        __builtin_memcpy(&x, __builtin_assume_aligned(slab + (i + (lane & 15)) * (WK * 2) + (((4 * ks + (lane >> 4)) ^ (lane & 7)) * 16), 16), 16);
        return x;
    }
    __device__ int side(int at) const { return at; }      // (the caller knows how many there are)
};

// elem(i, k) = p[k * ld + i], i < n, k < K; n >= 8.  MAPPED: the other operand is an OpAlong with the same K, whose last group is shifted.
template <int EXT, int NW, bool MAPPED>
struct OpAcross {
    static constexpr int PITCH = EXT * 2, PER = 1024 / PITCH, LOADS = WK / PER / NW, BYTES = EXT * WK * 2;
    const unsigned short *p;      // row 0
    int64_t ld;
    int K, n;
    unsigned off[LOADS], place;
    int k_of[MAPPED ? LOADS : 1];
    // 32-byte units of a row of LDS are permuted by k, so that the four rows of a transposing read (and the four eight rows on, which the
    // next sixteen lanes read) lie on different banks
    __device__ static int swizzle(int k) { return (k & 3) | ((k >> 1) & 4); }
    __device__ void start(const unsigned short *base, int64_t ld_, int i0, int n_, int K_) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        ld = ld_;
        K = K_;
        n = n_;
        p = (const unsigned short *)uniform_ptr(base);
        place = __builtin_amdgcn_readfirstlane(wave * 1024);
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
            const int k = (wave + u * NW) * PER + lane / (EXT / 8), slot = lane % (EXT / 8);
            const int at = i0 + 8 * (2 * ((slot >> 1) ^ swizzle(k)) + (slot & 1));
            off[u] = at >= n ? BUF_OUTSIDE : (unsigned)(((int64_t)k * ld + min(at, n - 8)) * 2);
            if (MAPPED) k_of[u] = k;
        }
    }
    __device__ void issue_inside(unsigned slab, int k0, int u) const {
        load_to_lds(wide_buffer(p + (int64_t)k0 * ld, (unsigned)min((int64_t)(K - k0) * ld * 2, (int64_t)BUF_EXTENT)), off[u], slab + place + u * NW * 1024);
    }
    __device__ void issue(unsigned slab, int k0) const {
        slab += place;
        if (!MAPPED || k0 + WK <= K) {
#pragma unroll
            for (int u = 0; u < LOADS; ++u) issue_inside(slab - place, k0, u);
        } else {
            const int back = min(k0, 8), r = K & 7, k8 = K & ~7;
            const auto rs = wide_buffer(p + (int64_t)(k0 - back) * ld, (unsigned)min((int64_t)(K - k0 + back) * ld * 2, (int64_t)BUF_EXTENT));
#pragma unroll
            for (int u = 0; u < LOADS; ++u) {
                const int k = k0 + k_of[u], shift = k < k8 ? 0 : 8 - r;
                const bool in = off[u] != BUF_OUTSIDE && (k < k8 || (r != 0 && k < k8 + 8 && k - k8 >= 8 - r));
                load_to_lds(rs, in ? off[u] + (unsigned)((back - shift) * ld * 2) : BUF_OUTSIDE, slab + u * NW * 1024);
            }
        }
    }
    __device__ void patch(char *, int) const {}
    __device__ static wide_bf16x8 fragment(const char *slab, int i, int ks) {
        const int lane = threadIdx.x & 63, sixteenth = lane & 15, q = lane >> 4;
        const int k = 32 * ks + 8 * q + (sixteenth >> 2);
        const char *a = slab + k * PITCH + (((i >> 4) ^ swizzle(k)) << 5) + (sixteenth & 3) * 8;
        typedef __attribute__((address_space(3))) wide_s16x4 *lds4;
        const wide_s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(__attribute__((address_space(3))) char *)a);
        const wide_s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(__attribute__((address_space(3))) char *)(a + 4 * PITCH));
        wide_bf16x8 x;
        __builtin_memcpy(&x, &lo, 8);
        __builtin_memcpy((char *)&x + 8, &hi, 8);
        return x;
    }
    __device__ int side(int at) const { return across_side<8>(at, n); }
};

// Tile of (16 FR WR) rows x (16 FC WC) columns for WR x WC waves, over the slabs s0 .. s1 - 1 of the contraction.  acc[i][j]: columns 16
// i.., rows 16 j.. of the wave's part.  ONES: with `sums`, one[] of the wave whose column is wc takes the sums over k of row fragments wc
// FR / WC .. (in every register the same).
//
// The row side has RING + 1 buffers, the column side RING: 3 and 2 slabs of 256 places fill the 160 KB of LDS.  A slab is multiplied in two
// halves.  While one half is multiplied out of registers the next one's registers are read, each as soon as its last use is issued; so all
// of a slab has been read when its second half begins.  There stands the only barrier of a slab: behind it everybody has the next slab
// complete.  Columns of slab s + RING are loaded during the second half of slab s, rows of it during the first, a load behind one
// group of matrix instructions and the next (together they would queue up behind one another, and behind those of all the chip).  AHEAD:
// rows half a slab earlier, during the second half of the slab before: where experts' rows differ and many tiles have few, 4096 x 4096
// forward 892 us instead of 916, input gradients 291 instead of 300; without, weight gradients 320 instead of 324. SHORT: of a tile whose
// rows end inside it, only the fragments with some of its `height` rows are multiplied (the others' accumulators stay zero).
template <class R, class Q, int FR, int FC, int WR, int WC, int RING, bool ONES, bool AHEAD, bool SHORT = false>
__device__ inline void wide_tile(const R &row, const Q &col, int K, int s0, int s1, char *smem, floatx4 (&acc)[FC][FR], floatx4 (&one)[FR / WC], bool sums,
                                 int height = 0) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wr = wave / WC, wc = wave % WC;
    const int mine = __builtin_amdgcn_readfirstlane((height + 15) / 16 - wr * FR);      // row fragments of this wave
#pragma unroll
    for (int i = 0; i < FC; ++i)
#pragma unroll
        for (int j = 0; j < FR; ++j) acc[i][j] = floatx4{0.f, 0.f, 0.f, 0.f};
    if (ONES)
#pragma unroll
        for (int j = 0; j < FR / WC; ++j) one[j] = floatx4{0.f, 0.f, 0.f, 0.f};
    if (s0 >= s1) return;
    wide_bf16x8 unit;
#pragma unroll
    for (int e = 0; e < 8; ++e) unit[e] = (__bf16)1.0f;
    constexpr int RB = R::BYTES, QB = Q::BYTES;
    char *const rows = smem, *const cols = smem + (RING + 1) * RB;
    const unsigned rows_at = lds_address(rows), cols_at = lds_address(cols);
    wide_bf16x8 a[2][FC], b[FR];
    int rb = 0, cb = 0;                                       // buffers of slab s
    // Multiplies one half (registers `half`) and reads the other one's from (rslab, cslab); at the end of the contraction that is a
    // buffer nobody has filled, and what is read is not used.
    auto multiply = [&](auto half_, const char *rslab, const char *cslab, auto between) {
        constexpr int half = decltype(half_)::value;
#pragma unroll
        for (int j = 0; j < FR; ++j) {
            __builtin_amdgcn_sched_barrier(0);
            if (!SHORT || j < mine)
#pragma unroll
                for (int i = 0; i < FC; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[half][i], b[j], acc[i][j], 0, 0, 0);
            if (ONES && sums && j / (FR / WC) == wc) one[j % (FR / WC)] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(unit, b[j], one[j % (FR / WC)], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
            if (j < FC) a[half ^ 1][j] = Q::fragment(cslab, 16 * (wc * FC + j), half ^ 1);
            b[j] = R::fragment(rslab, 16 * (wr * FR + j), half ^ 1);
            between(j);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    constexpr std::integral_constant<int, 0> first;
    constexpr std::integral_constant<int, 1> second;
    // `inside`: the slabs that are issued exist and end before K
    auto slab = [&](int s, auto inside) {
        constexpr bool INSIDE = decltype(inside)::value;
        const int rn = rb == RING ? 0 : rb + 1, cn = cb == RING - 1 ? 0 : cb + 1;
        const int rp = rb == 0 ? RING : rb - 1;                // what slab s - 1 was in
        const unsigned to_c = cols_at + cb * QB, to_r = rows_at + (AHEAD ? rb : rp) * RB;
        if (!INSIDE && !AHEAD && s + RING < s1) row.issue(to_r, (s + RING) * WK);
        multiply(first, rows + rb * RB, cols + cb * QB, [&](int j) {
            if (INSIDE && !AHEAD)
#pragma unroll
                for (int x = j * R::LOADS / FR; x < (j + 1) * R::LOADS / FR; ++x) row.issue_inside(to_r, (s + RING) * WK, x);
        });
        if (INSIDE) {                                          // (rows of slab s + RING may still be on their way)
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(R::LOADS) : "memory");
        } else {
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            if (s + 2 == s1) {
                row.patch(rows + rn * RB, (s + 1) * WK);
                col.patch(cols + cn * QB, (s + 1) * WK);
            }
            __syncthreads();
        }
        if (!INSIDE && s + RING < s1) col.issue(to_c, (s + RING) * WK);
        if (!INSIDE && AHEAD && s + RING + 1 < s1) row.issue(to_r, (s + RING + 1) * WK);
        multiply(second, rows + rn * RB, cols + cn * QB, [&](int j) {
            if (!INSIDE) return;
            constexpr int TOTAL = Q::LOADS + (AHEAD ? R::LOADS : 0);
#pragma unroll
            for (int x = j * TOTAL / FR; x < (j + 1) * TOTAL / FR; ++x) {
                if (x < Q::LOADS) col.issue_inside(to_c, (s + RING) * WK, x);
                else row.issue_inside(to_r, (s + RING + 1) * WK, x - Q::LOADS);
            }
        });
        rb = rn;
        cb = cn;
    };
#pragma unroll
    for (int u = 0; u < RING; ++u)
        if (s0 + u < s1) {
            row.issue(rows_at + u * RB, (s0 + u) * WK);
            col.issue(cols_at + u * QB, (s0 + u) * WK);
        }
    if (AHEAD && s0 + RING < s1) row.issue(rows_at + RING * RB, (s0 + RING) * WK);
    if (s0 + RING + AHEAD <= s1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"((RING - 1) * (R::LOADS + Q::LOADS) + AHEAD * R::LOADS) : "memory");   // the first slab
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if (s0 + 1 == s1) {
        row.patch(rows, s0 * WK);
        col.patch(cols, s0 * WK);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < FC; ++i) a[0][i] = Q::fragment(cols, 16 * (wc * FC + i), 0);
#pragma unroll
    for (int j = 0; j < FR; ++j) b[j] = R::fragment(rows, 16 * (wr * FR + j), 0);
    int s = s0;
    constexpr int TOUCHED = RING + 1 + AHEAD;      // slabs of a step
    for (; s + TOUCHED <= s1 && (s + TOUCHED) * WK <= K; ++s) slab(s, std::true_type());
    for (; s < s1; ++s) slab(s, std::false_type());
}

}  // namespace kfac
