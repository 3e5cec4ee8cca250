// The SwiGLU experts on 8-bit integers: rows of tokens with one scale each, weights with one scale for each output column.
//
//   G[r,n] = xs[r] sg[n] sum_k xq[r,k] wgq[n,k],  U likewise;  A = silu(G) U;  A -> integers aq with one scale as for each row;
//   Y[r,n] = as[r] sd[n] sum_k aq[r,k] wdq[n,k]
//
// The integer sums are exact (v_mfma_i32_32x32x32_i8, twice the rate of bf16), so no order of them shows in a result.
// Both operands of both products lie K-contiguous in rows of a multiple of 128 bytes, zeros behind the last value: a unit of
// 128 k is one cache line of each row, and widths that are no multiple of anything have no special case but the edge of an
// output tile.
//
// A row's scale is known when all columns of A are.  The product therefore leaves A in float32 with the maximum of every 32
// columns, and a pass over it (q8_rows_kernel) makes the 8-bit rows: the row's maximum is the largest of the 32-column ones, so
// this pass reads A once.
#include "xmoe_ffn.h"

namespace xmoe {
namespace {

typedef __attribute__((ext_vector_type(4))) int q8_i32x4_t;
typedef __attribute__((ext_vector_type(16))) int q8_i32x16_t;

constexpr int kQ8Group = 32;       // columns of A that share a maximum

__device__ __forceinline__ void q8_load16(const int8_t* p, char* lds) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)p,
                                     (__attribute__((address_space(3))) void*)lds, 16, 0, 0);
}
// at most N of the wave's loads on their way, its LDS reads returned; then the barrier.  (As asm: __syncthreads() would wait
// for every direct-to-LDS load.)
template <int N>
__device__ __forceinline__ void q8_wait_and_barrier() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// The thread's number, anew: what follows from it inside a loop over tiles is computed there, not held in registers over the
// products
__device__ __forceinline__ int q8_tid() {
    int t = threadIdx.x;
    asm volatile("" : "+v"(t));
    return t;
}

// A lane's pieces of the wave's share of an operand unit ([rows][128 bytes of k]): 8 rows per load, piece (lane % 8) XOR-ed
// with (row / 2) % 8, so that a fragment read falls on all banks.  Units are requested in order; behind the last one of K
// that one is fetched again, which keeps the wait counts uniform, and not used.
template <int LOADS>
struct Q8Rows {
    const int8_t* p[LOADS];
    // row r of the operand is at base + source(r) * pitch
    template <class Source>
    __device__ __forceinline__ void init(const int8_t* base, size_t pitch, int first, Source source) {
        const int lane = q8_tid() & 63;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int r = first + i * 8 + (lane >> 3);
            p[i] = base + (size_t)source(r) * pitch + (((lane & 7) ^ ((r >> 1) & 7)) << 4);
        }
    }
    // unit: LDS of the operand's unit; more: another unit follows
    __device__ __forceinline__ void issue(char* __restrict__ unit, int first, bool more) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            q8_load16(p[i], unit + (first + i * 8) * 128);
            p[i] += more ? 128 : 0;
        }
    }
};
// 16 bytes of k (32 ks + 16 (lane / 32) ..) of row base + lane % 32
__device__ __forceinline__ q8_i32x4_t q8_frag(const char* unit, int base, int ks) {
    const int lane = threadIdx.x & 63, r = base + (lane & 31), c = 2 * ks + (lane >> 5);
    return *reinterpret_cast<const q8_i32x4_t*>(unit + r * 128 + ((c ^ ((r >> 1) & 7)) << 4));
}

// The weights come first in the instruction: accumulator register v of lane l is row l % 32 and column
// 8 (v / 4) + 4 (l / 32) + v % 4 of its 32 x 32 block.
template <int MI, int NI>
struct Q8Frags {
    q8_i32x4_t a[MI], b[NI];
};
// four values from an address that is aligned to one
struct __attribute__((packed, aligned(4))) Q8F4 {
    float v[4];
};
__device__ __forceinline__ void q8_scales(const float* __restrict__ scale, int col, int N, float (&s)[4]) {
    if (col + 4 <= N) {
        const Q8F4 q = *reinterpret_cast<const Q8F4*>(scale + col);
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = q.v[i];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = col + i < N ? scale[col + i] : 0.f;   // columns past N: zero
    }
}
// A row's 32 columns of gate and up sums (this lane: 16 of them) -> A, four columns after the other at out, out + 8, ..; the
// maximum of all 32.  gs: the gate columns' scales times log2 e, us: the up columns' divided by it.
__device__ __forceinline__ float q8_activation(const q8_i32x16_t& g, const q8_i32x16_t& u, float xs,
                                               const float (&gs)[4][4], const float (&us)[4][4], float* out, bool store) {
    float a[16], m = 0.f;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
        const float gv = (float)g[v] * xs * gs[v / 4][v % 4], uv = (float)u[v] * xs * us[v / 4][v % 4];
        a[v] = gv * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-gv)) * uv;
        m = __builtin_elementwise_maximum(m, fabsf(a[v]));   // a NaN stays
    }
    if (store) {
#pragma unroll
        for (int q = 0; q < 4; ++q)
            *reinterpret_cast<float4*>(out + 8 * q) = make_float4(a[4 * q], a[4 * q + 1], a[4 * q + 2], a[4 * q + 3]);
    }
    return __builtin_elementwise_maximum(m, __shfl_xor(m, 32, 64));
}
constexpr float kLog2e = 1.44269504088896341f;

// eight bf16 from col on (of N) at an address that is aligned to one
struct __attribute__((packed, aligned(2))) Q8B8 {
    uint32_t v[4];
};
__device__ __forceinline__ void q8_store8(bf16_t* __restrict__ row, int col, int N, const uint4& q) {
    if (col + 8 <= N) {
        *reinterpret_cast<Q8B8*>(row + col) = Q8B8{{q.x, q.y, q.z, q.w}};
        return;
    }
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (col + i < N) row[col + i] = bf16_t{(uint16_t)(w[i / 2] >> (16 * (i & 1)))};
}
__device__ __forceinline__ void q8_store4(float* __restrict__ row, int col, int N, const float (&s)[4]) {
    if (col + 4 <= N) {
        *reinterpret_cast<Q8F4*>(row + col) = Q8F4{{s[0], s[1], s[2], s[3]}};
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (col + i < N) row[col + i] = s[i];
}

struct __attribute__((packed, aligned(2))) Q8B4 {
    uint32_t v[2];
};
__device__ __forceinline__ void q8_store4(bf16_t* __restrict__ row, int col, int N, const float (&s)[4]) {
    if (col + 4 <= N) {
        *reinterpret_cast<Q8B4*>(row + col) = Q8B4{{pack_bf16x2(s[0], s[1]), pack_bf16x2(s[2], s[3])}};
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (col + i < N) row[col + i] = from_float<bf16_t>(s[i]);
}

struct Q8Args {
    const int8_t* x;            // rows, pitch bytes each
    const float* x_scale;       // of a row
    const int32_t* row_index;   // or NULL
    const int32_t *off, *map;
    const int8_t *w0, *w1;      // [E, N, pitch]; w1: up
    const float *s0, *s1;       // [E, N]
    int pitch, N, tile_rows;    // tile_rows: the tile map's
    int group;                  // row tiles that go through the column tiles together
    float* a32;                 // gate/up: [rows][a_pitch]
    float* gmax;                // [rows][a_pitch / 32]
    int a_pitch;
    void* y;                    // down: [rows][N]
};

// Row tiles that go through the column tiles together.  The 32 CUs of an XCD then read 4 + 8 operand tiles at a time, not 1 + 32
// (d 4096, f 14336, 8 experts with 512 rows each: 1038 us, in fours 969; 33 experts, f 1024, 1241 mean rows: 663 either way; 66
// experts, d 2048, f 1408, 993 mean rows: 814 and 821).
constexpr int kQ8RowTiles = 4;
// Tile L: row tiles x column tiles, in groups of `group` row tiles (those of a column tile, then the next column tile), dealt to
// the XCDs in eight runs of equal length (workgroup L goes to XCD L % 8): tiles in flight together share their weights
// and rows in one L2.
struct Q8Tile {
    int e, row0, rows, n0;
    __device__ __forceinline__ bool place(const Q8Args& a, int cols, int group, long L) {
        const int nt = (a.N + cols - 1) / cols;
        const long total = (long)a.map[0] * nt, run = (total + 7) / 8, slot = L >> 3, t = (L & 7) * run + slot;
        if (slot >= run || t >= total) return false;
        const int g0 = (int)(t / ((long)nt * group)) * group, in = (int)(t - (long)g0 * nt);
        const int rows_of_group = a.map[0] - g0 < group ? a.map[0] - g0 : group;
        const int tile = g0 + in % rows_of_group;
        n0 = in / rows_of_group * cols;
        e = a.map[4 + 2 * tile];
        row0 = a.map[4 + 2 * tile + 1];
        rows = a.off[e + 1] - row0;
        rows = rows < a.tile_rows ? rows : a.tile_rows;
        return true;
    }
};

long q8_blocks(int N, int cols, int max_tiles) { return ((long)max_tiles * ((N + cols - 1) / cols) + 7) / 8 * 8; }

// =========================================================================================================
// Tiles of MT x MT (gate/up: the same MT / 2 columns of both).  Units A(0) B(0) A(1) B(1) .. of MT rows x 128 k run through
// five slots, two to three of them on their way.
//   256: 8 waves (2 x 4) of 128 x 64 each, 160 KiB, one block per CU: the most products per byte of LDS.  A block takes tile
//        after tile, and the units of the next one follow those of this one without a pause (66 experts, d 2048, f 1408, 993
//        mean rows: a block per tile 496 us for gate/up, 256 for down, this way 478 and 245: 1.57 POP/s, where a large library
//        product has 2.08).  Matrix cores are busy 41 % of it.  LDS does not hold it up, by its counter: active 15 % of the
//        clocks; waves wait 3 % of their time for its issue, 32 % for loads and barriers and 45 % for the issue of an
//        instruction of any kind.  (Waves of higher priority in their matrix instructions: 1 to 2 % slower.)
//   128: 4 waves (2 x 2) of 64 x 64 each, 80 KiB, two blocks per CU: where the weights' bytes are the bound, or 256 rows few
// =========================================================================================================
template <int MT, int WAVES>
struct Tile8 {
    static constexpr int kWaves = WAVES, kThreads = 64 * WAVES, kWn = WAVES / 2, kMi = MT / 64, kNi = MT / 32 / kWn,
                         kLoads = MT / 8 / WAVES, kUnit = MT * 128, kLds = 5 * kUnit;
    static constexpr bool kRoll = MT == 256;
    static constexpr int kCols = MT / 2, kPieces = kCols / 8;   // columns of a 32-column block of all waves; 16-byte pieces
    typedef q8_i32x16_t Acc[kMi][kNi];
    __device__ __forceinline__ static int wave() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }
    __device__ __forceinline__ static int wm() { return wave() / kWn; }
    __device__ __forceinline__ static int wn() { return wave() % kWn; }
    __device__ __forceinline__ static int first() { return wave() * 8 * kLoads; }   // row of the wave's share of a unit
    // first column of the wave's ni-th 32, first row of its mi-th
    __device__ __forceinline__ static int col(int ni) { return ni * kCols + wn() * 32; }
    __device__ __forceinline__ static int row(int mi) { return wm() * (MT / 2) + mi * 32; }
};
template <class W, int MI>
__device__ __forceinline__ void tile8_read(Q8Frags<MI, W::kNi>& f, const char* ua, const char* ub, int ks) {
#pragma unroll
    for (int ni = 0; ni < W::kNi; ++ni) f.b[ni] = q8_frag(ub, W::col(ni), ks);
#pragma unroll
    for (int mi = 0; mi < MI; ++mi) f.a[mi] = q8_frag(ua, W::row(mi), ks);
}
template <int MI, int NI, int N>
__device__ __forceinline__ void q8_mma(q8_i32x16_t (&acc)[N][NI], const Q8Frags<MI, NI>& f) {
#pragma unroll
    for (int mi = 0; mi < MI; ++mi)
#pragma unroll
        for (int ni = 0; ni < NI; ++ni)
            acc[mi][ni] = __builtin_amdgcn_mfma_i32_32x32x32_i8(f.b[ni], f.a[mi], acc[mi][ni], 0, 0, 0);
}
// One pass: the four steps on A(p) = ua, B(p) = ub.  On entry both have landed, every wave has left the units of pass p - 1
// (fill1, fill2), and f1 holds that pass's last step.  The slots are distinct, and saying so matters: an LDS read that may
// observe a direct-to-LDS load in flight makes the compiler wait for all of them.
template <class W, int MI>
__device__ __forceinline__ void tile8_pass(typename W::Acc& acc, Q8Frags<MI, W::kNi>& f0, Q8Frags<MI, W::kNi>& f1,
                                           Q8Rows<W::kLoads>& a, Q8Rows<W::kLoads>& b, bool more_a, bool more_b,
                                           char* __restrict__ fill1, char* __restrict__ fill2,
                                           const char* __restrict__ ua, const char* __restrict__ ub) {
    b.issue(fill1, W::first(), more_b);  // B(p+1)
    __builtin_amdgcn_sched_barrier(0);   // the requests stay where they stand: sunk to the end of the pass they are late
    tile8_read<W, MI>(f0, ua, ub, 0);
    q8_mma(acc, f1);
    tile8_read<W, MI>(f1, ua, ub, 1);
    q8_mma(acc, f0);
    __builtin_amdgcn_sched_barrier(0);
    a.issue(fill2, W::first(), more_a);  // A(p+2)
    __builtin_amdgcn_sched_barrier(0);
    tile8_read<W, MI>(f0, ua, ub, 2);
    q8_mma(acc, f1);
    tile8_read<W, MI>(f1, ua, ub, 3);
    q8_mma(acc, f0);
}
__device__ __forceinline__ int q8_slot(int s) { return s < 5 ? s : s - 5; }
// MI: the wave's 32-row blocks that hold rows (0: it only takes part in the loads).  sa: slot of A(0), then of the pass.
// Where tiles follow one another (W::kRoll) the units behind the last one are the next tile's first: next_a() and next_b()
// turn to it.
template <class W, int MI, class NextA, class NextB>
__device__ __forceinline__ void tile8_loop(typename W::Acc& acc, Q8Rows<W::kLoads>& a, Q8Rows<W::kLoads>& b, int np, char* smem,
                                           int& sa, NextA next_a, NextB next_b) {
    constexpr int kUnit = W::kUnit, M = MI > 0 ? MI : 1;
    const q8_i32x4_t z = {0, 0, 0, 0};
    Q8Frags<M, W::kNi> f0, f1;
#pragma unroll
    for (int mi = 0; mi < M; ++mi) f1.a[mi] = z;
#pragma unroll
    for (int ni = 0; ni < W::kNi; ++ni) f1.b[ni] = z;
#pragma nounroll
    for (int p = 0; p < np; ++p) {
        const int sb = q8_slot(sa + 1), s3 = q8_slot(sa + 3), s4 = q8_slot(sa + 4);
        if (W::kRoll && p + 2 == np) next_a();
        if (W::kRoll && p + 1 == np) next_b();
        __builtin_amdgcn_sched_barrier(0);
        const bool more_a = W::kRoll || p + 3 < np, more_b = W::kRoll || p + 2 < np;
        if (MI > 0) {
            tile8_pass<W, M>(acc, f0, f1, a, b, more_a, more_b, smem + s3 * kUnit, smem + s4 * kUnit, smem + sa * kUnit,
                             smem + sb * kUnit);
        } else {
            b.issue(smem + s3 * kUnit, W::first(), more_b);
            a.issue(smem + s4 * kUnit, W::first(), more_a);
        }
        q8_wait_and_barrier<W::kLoads>();
        sa = q8_slot(sa + 2);
    }
    if (MI > 0) q8_mma(acc, f1);
}
// The tile's sums.  rows: valid ones of the tile, which may exceed it
template <class W, class NextA, class NextB>
__device__ __forceinline__ void tile8_product(typename W::Acc& acc, Q8Rows<W::kLoads>& a, Q8Rows<W::kLoads>& b, int np, int rows,
                                              char* smem, int& sa, NextA next_a, NextB next_b) {
#pragma unroll
    for (int mi = 0; mi < W::kMi; ++mi)
#pragma unroll
        for (int ni = 0; ni < W::kNi; ++ni)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[mi][ni][v] = 0;
    const int left = rows - W::row(0);
    if (left <= 0)
        tile8_loop<W, 0>(acc, a, b, np, smem, sa, next_a, next_b);
    else if (W::kMi == 2 && left <= 32)
        tile8_loop<W, 1>(acc, a, b, np, smem, sa, next_a, next_b);
    else
        tile8_loop<W, W::kMi>(acc, a, b, np, smem, sa, next_a, next_b);
    if (!W::kRoll) q8_wait_and_barrier<0>();   // nothing may land in this LDS any more: it becomes the results'
}
// The block's tiles: one, or (kRoll) every gridDim-th.  rows_of(t, i): row of g.x of the tile's i-th;  weights(t, i): the tile's
// i-th row of weights;  results(t, acc, at): at(r) is row r of MT / 2 columns of 16 bits in LDS that is free: the two units of
// the last pass, those behind hold the next tile's.
template <class W, class RowIndex, class Weights, class Ahead, class Results>
__device__ __forceinline__ void tile8_run(const Q8Args& g, int cols, char* smem, RowIndex row_index, Weights weights, Ahead ahead,
                                          Results results) {
    Q8Tile t, next;
    long L = blockIdx.x;
    if (!t.place(g, cols, g.group, L)) return;
    const int np = g.pitch / 128;
    Q8Rows<W::kLoads> a, b;
    int src[W::kLoads];   // rows of the A units to come
    auto fetch_rows = [&](const Q8Tile& u) {
        const int r0 = W::first() + ((q8_tid() & 63) >> 3);
#pragma unroll
        for (int i = 0; i < W::kLoads; ++i) src[i] = row_index(u, r0 + 8 * i);
    };
    auto turn_a = [&] {
        int i = 0;
        a.init(g.x, g.pitch, W::first(), [&](int) { return src[i++]; });
    };
    fetch_rows(t);
    turn_a();
    weights(t, b);
    a.issue(smem, W::first(), np > 1);
    b.issue(smem + W::kUnit, W::first(), np > 1 || W::kRoll);
    a.issue(smem + 2 * W::kUnit, W::first(), np > 2 || W::kRoll);
    // at the top of pass p everything up to B(p) has landed for every thread, A(p+1) may be on its way
    q8_wait_and_barrier<W::kLoads>();
    int sa = 0;
    for (;;) {
        L += gridDim.x;
        const bool more = W::kRoll && next.place(g, cols, g.group, L);
        if (!more) next = t;   // its units are requested again, and not used
        if (W::kRoll) fetch_rows(next);
        ahead(t);
        typename W::Acc acc;
        tile8_product<W>(acc, a, b, np, t.rows, smem, sa, turn_a, [&] { weights(next, b); });
        char *res0 = smem + (W::kRoll ? q8_slot(sa + 3) : 0) * W::kUnit, *res1 = smem + (W::kRoll ? q8_slot(sa + 4) : 1) * W::kUnit;
        __builtin_amdgcn_sched_barrier(0);
        results(t, acc, res0, res1);
        if (!more) break;
        t = next;
    }
    if (W::kRoll) q8_wait_and_barrier<0>();
}
// LDS writes done and seen, or LDS reads returned: direct-to-LDS loads go on
__device__ __forceinline__ void q8_lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// A 16-byte piece c of row r of results, pieces XOR-ed with the row.  u0, u1: units of 128 rows of 256 bytes, or of 128 of 128
template <class W>
__device__ __forceinline__ char* tile8_at(char* u0, char* u1, int r, int c) {
    return (r < 128 ? u0 : u1) + (r & 127) * (2 * W::kCols) + ((c ^ (r & (W::kPieces - 1))) << 4);
}
// store(r, c, piece c of row r) for the pieces in LDS of all rows below `rows`
template <class W, class Store>
__device__ __forceinline__ void tile8_store(char* u0, char* u1, int rows, Store store) {
    constexpr int kStep = W::kThreads / W::kPieces, kRows = W::kMi * 64;
    const int tid = q8_tid();
#pragma unroll 4
    for (int i = 0; i < kRows / kStep; ++i) {
        const int r = i * kStep + tid / W::kPieces, c = tid % W::kPieces;
        const uint4 v = *reinterpret_cast<const uint4*>(tile8_at<W>(u0, u1, r, c));
        if (r < rows) store(r, c, v);
    }
}

template <int MT, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void q8_gateup_kernel(Q8Args g) {
    typedef Tile8<MT, WAVES> W;
    constexpr int kCols = W::kCols;
    __shared__ __align__(16) char smem[W::kLds];
    float xs[W::kMi], gs[4][4], us[4][4];
    auto scales = [&](const Q8Tile& t) {
        const int lane = q8_tid() & 63;
#pragma unroll
        for (int mi = 0; mi < W::kMi; ++mi) {
            const int r = W::row(mi) + (lane & 31), row = t.row0 + (r < t.rows ? r : t.rows - 1);
            xs[mi] = g.x_scale[g.row_index ? g.row_index[row] : row];
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int c = t.n0 + W::col(0) + 4 * (lane >> 5) + 8 * q;
            q8_scales(g.s0 + (size_t)t.e * g.N, c, g.N, gs[q]);
            q8_scales(g.s1 + (size_t)t.e * g.N, c, g.N, us[q]);
        }
    };
    tile8_run<W>(
        g, kCols, smem,
        [&](const Q8Tile& t, int r) {
            r = t.row0 + (r < t.rows ? r : t.rows - 1);   // rows past the last one repeat it; what they give is not stored
            return g.row_index ? g.row_index[r] : r;
        },
        [&](const Q8Tile& t, Q8Rows<W::kLoads>& b) {
            b.init(W::wave() < WAVES / 2 ? g.w0 : g.w1, g.pitch, W::first(), [&](int r) {
                const int n = t.n0 + (r & (kCols - 1));
                return (size_t)t.e * g.N + (n < g.N ? n : g.N - 1);
            });
        },
        [&](const Q8Tile& t) {
            if (!W::kRoll) scales(t);   // ahead of the loop, where the registers allow it
        },
        [&](const Q8Tile& t, typename W::Acc& acc, char*, char*) {
            if (W::kRoll) scales(t);
            const int lane = q8_tid() & 63;
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                gs[v / 4][v % 4] *= kLog2e;
                us[v / 4][v % 4] *= 1.0f / kLog2e;
            }
            const int c0 = W::col(0);
#pragma unroll
            for (int mi = 0; mi < W::kMi; ++mi) {
                const int r = W::row(mi) + (lane & 31);
                const size_t row = t.row0 + r;
                // a wave writes whole cache lines of its rows, 32 bytes of each at a time
                const float m = q8_activation(acc[mi][0], acc[mi][1], xs[mi], gs, us,
                                              g.a32 + row * g.a_pitch + t.n0 + c0 + 4 * (lane >> 5), r < t.rows);
                if (lane < 32 && r < t.rows) g.gmax[row * (g.a_pitch / kQ8Group) + (t.n0 + c0) / kQ8Group] = m;
            }
        });
}

template <int MT, int WAVES, typename T>
__global__ __launch_bounds__(64 * WAVES, 2) void q8_down_kernel(Q8Args g) {
    typedef Tile8<MT, WAVES> W;
    __shared__ __align__(16) char smem[W::kLds];
    float as[W::kMi];
    auto scales = [&](const Q8Tile& t) {
        const int lane = q8_tid() & 63;
#pragma unroll
        for (int mi = 0; mi < W::kMi; ++mi) {
            const int r = W::row(mi) + (lane & 31);
            as[mi] = g.x_scale[t.row0 + (r < t.rows ? r : t.rows - 1)];
        }
    };
    tile8_run<W>(
        g, MT, smem, [&](const Q8Tile& t, int r) { return t.row0 + (r < t.rows ? r : t.rows - 1); },
        [&](const Q8Tile& t, Q8Rows<W::kLoads>& b) {
            b.init(g.w0, g.pitch, W::first(), [&](int r) {
                const int n = t.n0 + r;
                return (size_t)t.e * g.N + (n < g.N ? n : g.N - 1);
            });
        },
        [&](const Q8Tile& t) {
            if (!W::kRoll) scales(t);
        },
        [&](const Q8Tile& t, typename W::Acc& acc, char* u0, char* u1) {
            if (W::kRoll) scales(t);
            const int lane = q8_tid() & 63;
#pragma unroll
            for (int ni = 0; ni < W::kNi; ++ni) {   // MT / 2 columns of all waves
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int c = W::wn() * 32 + 8 * q + 4 * (lane >> 5), col = t.n0 + ni * W::kCols + c;
                    float s[4];
                    q8_scales(g.s0 + (size_t)t.e * g.N, col, g.N, s);
#pragma unroll
                    for (int mi = 0; mi < W::kMi; ++mi) {
                        const int r = W::row(mi) + (lane & 31);
                        float o[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[i] = (float)acc[mi][ni][4 * q + i] * (as[mi] * s[i]);
                        if (sizeof(T) == 4) {
                            if (r < t.rows) q8_store4((float*)g.y + (size_t)(t.row0 + r) * g.N, col, g.N, o);
                        } else {
                            *reinterpret_cast<uint2*>(tile8_at<W>(u0, u1, r, c / 8) + 8 * (lane >> 5)) =
                                make_uint2(pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3]));
                        }
                    }
                }
                if (sizeof(T) == 4) continue;
                q8_lds_barrier();
                tile8_store<W>(u0, u1, t.rows, [&](int r, int c, const uint4& v) {
                    q8_store8((bf16_t*)g.y + (size_t)(t.row0 + r) * g.N, t.n0 + ni * W::kCols + 8 * c, g.N, v);
                });
                if (W::kRoll || ni + 1 < W::kNi) q8_lds_barrier();
            }
        });
}

// blocks of the persistent kernels: one per CU
constexpr long kQ8RollBlocks = 256;

template <int MT, int WAVES>
int launch_q8_gateup(const Q8Args& a, int max_tiles, hipStream_t s) {
    typedef Tile8<MT, WAVES> W;
    long blocks = q8_blocks(a.N, MT / 2, max_tiles);
    if (W::kRoll && blocks > kQ8RollBlocks) blocks = kQ8RollBlocks;
    XMOE_LAUNCH(K_Q8_GATEUP, s,
                hipLaunchKernelGGL((q8_gateup_kernel<MT, WAVES>), dim3((unsigned)blocks), dim3(64 * WAVES), 0, s, a));
    return XMOE_OK;
}
template <int MT, int WAVES>
int launch_q8_down(const Q8Args& a, int max_tiles, int dt, hipStream_t s) {
    typedef Tile8<MT, WAVES> W;
    long blocks = q8_blocks(a.N, MT, max_tiles);
    if (W::kRoll && blocks > kQ8RollBlocks) blocks = kQ8RollBlocks;
    const dim3 grid((unsigned)blocks), block(64 * WAVES);
    if (dt == XMOE_F32)
        XMOE_LAUNCH(K_Q8_DOWN, s, hipLaunchKernelGGL((q8_down_kernel<MT, WAVES, float>), grid, block, 0, s, a));
    else
        XMOE_LAUNCH(K_Q8_DOWN, s, hipLaunchKernelGGL((q8_down_kernel<MT, WAVES, bf16_t>), grid, block, 0, s, a));
    return XMOE_OK;
}

// =========================================================================================================
// Few rows (a decoding step): the weights' bytes are the bound.  32 rows and 64 columns (gate/up: of either matrix) per block
// of 4 waves.  A stage is 256 k, two cache lines of each row (one line of each costs memory a tenth of its rate); two stages,
// the second on its way while the first is multiplied, 40 KiB each for gate/up (two blocks per CU), 24 for down (three).
// Waves 0, 1 and 2, 3 take half of a stage's k each, and their sums, which are integers, are added in LDS.  Tried: straight
// from memory to registers, 32 bytes of 32 rows at a time (slower by a quarter, the loads' addresses take the L1 cache too
// long); 128 columns for down (37 experts, d 2048, f 1408: 30 us for 25, too few blocks for an even load); 32 for gate/up (48
// for 45); 64 rows (one block per CU: 95 for 76).  Measured, d 2048, f 1408, 37 of 66 experts with one or two rows each:
// gate/up 45 us (4.7 TB/s), down 25 (4.3); all 66: 72 (5.3) and 39 (4.9).
// =========================================================================================================
__device__ __align__(16) const uint32_t kQ8Zero[4] = {0u, 0u, 0u, 0u};

// A lane's pieces of the wave's share of an operand's stage ([rows][256 bytes]), 4 rows per load, piece (lane % 16) XOR-ed with
// row % 16; those behind the end of K in the last stage come from a block of zeros
template <int LOADS>
struct Few8Rows {
    const int8_t* p[LOADS];
    uint32_t upper;   // bit i: the i-th piece lies in the stage's second half
    template <class Source>
    __device__ __forceinline__ void init(const int8_t* base, size_t pitch, int first, Source source) {
        const int lane = threadIdx.x & 63;
        upper = 0u;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int r = first + i * 4 + (lane >> 4), c = (lane & 15) ^ (r & 15);
            p[i] = base + (size_t)source(r) * pitch + (c << 4);
            upper |= (uint32_t)(c >> 3) << i;
        }
    }
    // half: K ends in the middle.  Four rows none of which is below `rows` are left out.
    __device__ __forceinline__ void issue(char* __restrict__ unit, int first, int rows, bool half) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            if (first + i * 4 >= rows) break;
            const bool out = half && ((upper >> i) & 1u);
            q8_load16(out ? reinterpret_cast<const int8_t*>(kQ8Zero) : p[i], unit + (first + i * 4) * 256);
            p[i] += 256;
        }
    }
};
__device__ __forceinline__ q8_i32x4_t few8_frag(const char* unit, int base, int ks) {
    const int lane = threadIdx.x & 63, r = base + (lane & 31), c = 2 * ks + (lane >> 5);
    return *reinterpret_cast<const q8_i32x4_t*>(unit + r * 256 + ((c ^ (r & 15)) << 4));
}
// Stages of 64 NB weight rows and 32 rows of x.  Wave (wn = wave % 2, wk = wave / 2): weight rows 64 n + 32 wn .. + 31 of every
// n < NB, all of x, half wk of a stage's k.
template <int NB>
struct Few8 {
    static constexpr int kW = NB * 64 * 256, kStage = kW + 32 * 256;
    Few8Rows<4 * NB> w;
    Few8Rows<2> x;
    q8_i32x16_t acc[NB];
    __device__ __forceinline__ static int wave() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }
    __device__ __forceinline__ void issue(char* __restrict__ stage, int rows, bool half) {
        w.issue(stage, wave() * 16 * NB, 64 * NB, half);
        x.issue(stage + kW, wave() * 8, rows, half);
    }
    __device__ __forceinline__ void stage(int rows, bool more, bool half, char* __restrict__ next, const char* __restrict__ cur) {
        const int wn = wave() & 1, wk = wave() >> 1;
        if (more) issue(next, rows, half);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int ks = 4 * wk + i;
            const q8_i32x4_t a = few8_frag(cur + kW, 0, ks);
#pragma unroll
            for (int n = 0; n < NB; ++n)
                acc[n] = __builtin_amdgcn_mfma_i32_32x32x32_i8(few8_frag(cur, 64 * n + 32 * wn, ks), a, acc[n], 0, 0, 0);
        }
    }
    // Rows of x from `rows` on hold anything.  The waves' sums of half of k, in LDS, are added by sum().
    __device__ __forceinline__ void product(int pitch, int rows, char* smem) {
        const int stages = (pitch + 255) / 256;
        const bool tail = pitch % 256 != 0;
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[n][v] = 0;
        issue(smem, rows, tail && stages == 1);
        for (int s = 0; s < stages; ++s) {
            q8_wait_and_barrier<0>();   // stage s has landed for every thread, and every wave is done with stage s - 1
            stage(rows, s + 1 < stages, tail && s + 2 == stages, smem + ((s + 1) & 1) * kStage, smem + (s & 1) * kStage);
        }
        __syncthreads();
        int* red = reinterpret_cast<int*>(smem) + wave() * (NB * 1024) + (threadIdx.x & 63);
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int v = 0; v < 16; ++v) red[(n * 16 + v) * 64] = acc[n][v];
        __syncthreads();
    }
    // weight rows 64 n + 32 wn ..
    __device__ __forceinline__ static q8_i32x16_t sum(const char* smem, int n, int wn) {
        const int* red = reinterpret_cast<const int*>(smem) + (wn * NB + n) * 1024 + (threadIdx.x & 63);
        q8_i32x16_t a;
#pragma unroll
        for (int v = 0; v < 16; ++v) a[v] = red[v * 64] + red[2 * NB * 1024 + v * 64];
        return a;
    }
};

__global__ __launch_bounds__(256, 2) void q8_gateup_few_kernel(Q8Args g) {
    typedef Few8<2> F;
    __shared__ __align__(16) char smem[2 * F::kStage];
    Q8Tile t;
    if (!t.place(g, 64, 1, blockIdx.x)) return;
    const int lane = threadIdx.x & 63, wave = F::wave(), half = lane >> 5;
    F p;
    p.w.init(wave < 2 ? g.w0 : g.w1, g.pitch, wave * 32, [&](int c) {
        const int n = t.n0 + (c & 63);
        return (size_t)t.e * g.N + (n < g.N ? n : g.N - 1);
    });
    p.x.init(g.x, g.pitch, wave * 8, [&](int i) {
        i = t.row0 + (i < t.rows ? i : t.rows - 1);
        return g.row_index ? g.row_index[i] : i;
    });
    const int r = lane & 31, row = t.row0 + (r < t.rows ? r : t.rows - 1), c0 = t.n0 + 32 * (wave & 1);
    float xs = g.x_scale[g.row_index ? g.row_index[row] : row], gs[4][4], us[4][4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        q8_scales(g.s0 + (size_t)t.e * g.N, c0 + 4 * half + 8 * q, g.N, gs[q]);
        q8_scales(g.s1 + (size_t)t.e * g.N, c0 + 4 * half + 8 * q, g.N, us[q]);
    }
    p.product(g.pitch, t.rows, smem);
    if (wave >= 2) return;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
        gs[v / 4][v % 4] *= kLog2e;
        us[v / 4][v % 4] *= 1.0f / kLog2e;
    }
    const float m = q8_activation(F::sum(smem, 0, wave & 1), F::sum(smem, 1, wave & 1), xs, gs, us,
                                  g.a32 + (size_t)row * g.a_pitch + c0 + 4 * half, r < t.rows);
    if (half == 0 && r < t.rows) g.gmax[(size_t)row * (g.a_pitch / kQ8Group) + c0 / kQ8Group] = m;
}

template <typename T>
__global__ __launch_bounds__(256, 2) void q8_down_few_kernel(Q8Args g) {
    typedef Few8<1> F;
    __shared__ __align__(16) char smem[2 * F::kStage];
    Q8Tile t;
    if (!t.place(g, 64, 1, blockIdx.x)) return;
    const int lane = threadIdx.x & 63, wave = F::wave();
    F p;
    p.w.init(g.w0, g.pitch, wave * 16, [&](int c) {
        const int n = t.n0 + c;
        return (size_t)t.e * g.N + (n < g.N ? n : g.N - 1);
    });
    p.x.init(g.x, g.pitch, wave * 8, [&](int i) { return t.row0 + (i < t.rows ? i : t.rows - 1); });
    const int r = lane & 31, row = t.row0 + (r < t.rows ? r : t.rows - 1);
    const float as = g.x_scale[row];
    p.product(g.pitch, t.rows, smem);
    if (wave >= 2 || r >= t.rows) return;
    const q8_i32x16_t sum = F::sum(smem, 0, wave & 1);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int col = t.n0 + 32 * wave + 8 * q + 4 * (lane >> 5);
        float s[4], o[4];
        q8_scales(g.s0 + (size_t)t.e * g.N, col, g.N, s);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = (float)sum[4 * q + i] * (as * s[i]);
        q8_store4((T*)g.y + (size_t)row * g.N, col, g.N, o);
    }
}

int launch_q8_gateup_few(const Q8Args& a, int max_tiles, hipStream_t s) {
    XMOE_LAUNCH(K_Q8_GATEUP_FEW, s, hipLaunchKernelGGL(q8_gateup_few_kernel, dim3((unsigned)q8_blocks(a.N, 64, max_tiles)),
                                                       dim3(256), 0, s, a));
    return XMOE_OK;
}
int launch_q8_down_few(const Q8Args& a, int max_tiles, int dt, hipStream_t s) {
    const dim3 grid((unsigned)q8_blocks(a.N, 64, max_tiles)), block(256);
    if (dt == XMOE_F32)
        XMOE_LAUNCH(K_Q8_DOWN_FEW, s, hipLaunchKernelGGL(q8_down_few_kernel<float>, grid, block, 0, s, a));
    else
        XMOE_LAUNCH(K_Q8_DOWN_FEW, s, hipLaunchKernelGGL(q8_down_few_kernel<bf16_t>, grid, block, 0, s, a));
    return XMOE_OK;
}

// =========================================================================================================
// A's 8-bit rows: one wave per row.  HBM-bound: 65536 rows, f 1408, 85 us, 5.4 TB/s.
// =========================================================================================================
__global__ __launch_bounds__(256) void q8_rows_kernel(const float* __restrict__ a32, const float* __restrict__ gmax,
                                                      const int32_t* __restrict__ off, int E, int f, int pitch,
                                                      int8_t* __restrict__ aq, float* __restrict__ as) {
    const int lane = threadIdx.x & 63, row = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= off[E]) return;
    const float* gm = gmax + (size_t)row * (pitch / kQ8Group);
    const int groups = (f + kQ8Group - 1) / kQ8Group;
    uint32_t mx = 0u;
    for (int i = lane; i < groups; i += 64) {
        const uint32_t b = __float_as_uint(gm[i]);
        mx = b > mx ? b : mx;
    }
#pragma unroll
    for (int w = 32; w >= 1; w >>= 1) {
        const uint32_t o = (uint32_t)__shfl_xor((int)mx, w, 64);
        mx = o > mx ? o : mx;
    }
    // as xmoe_add_rmsnorm: below 2^-120 the quotient would overflow, such a row counts as zero
    const bool none = mx < 0x03800000u;
    const float m = __uint_as_float(mx), inv = none ? 0.f : 127.f / m;
    if (lane == 0) as[row] = none ? 0.f : m / 127.f;
    const float* src = a32 + (size_t)row * pitch;
    int8_t* dst = aq + (size_t)row * pitch;
    for (int c = lane; c < pitch / 8; c += 64) {
        uint2 o = make_uint2(0u, 0u);
        if (8 * c < f) {   // columns past f are zeros already, whole pieces of them were not written
            const float4 lo = *reinterpret_cast<const float4*>(src + 8 * c);
            const float4 hi = *reinterpret_cast<const float4*>(src + 8 * c + 4);
            const float v[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
            uint32_t p[2] = {0u, 0u};
#pragma unroll
            for (int i = 0; i < 8; ++i)
                p[i / 4] |= ((uint32_t)(int)rintf(fminf(fmaxf(v[i] * inv, -127.f), 127.f)) & 0xffu) << (8 * (i & 3));
            o = make_uint2(p[0], p[1]);
        }
        *reinterpret_cast<uint2*>(dst + 8 * c) = o;
    }
}

// =========================================================================================================
// Weights [K, N] ("in x out") of an expert -> [N, pitch] integers and one scale per column.  Done once for a model's weights,
// so it is simple: a block owns 64 columns, reads them twice (maximum, then integers) and turns 64 x 64 pieces over in LDS.
// 66 matrices of 2048 x 1408 in bf16: 407 us, 2.3 TB/s of what it reads and writes; read once, they would take 96 at memory's
// rate.
// =========================================================================================================
template <typename T>
__global__ __launch_bounds__(256) void quantize_weights_kernel(const T* __restrict__ w, int K, int N, int pitch,
                                                               int8_t* __restrict__ wq, float* __restrict__ scale) {
    __shared__ uint32_t part[4][64];
    __shared__ __align__(16) int8_t tile[64][80];
    const int c = threadIdx.x & 63, g = threadIdx.x >> 6, n = blockIdx.x * 64 + c;
    const T* src = w + (size_t)blockIdx.y * K * N + n;
    uint32_t mx = 0u;
    if (n < N) {
#pragma unroll 8
        for (int k = g; k < K; k += 4) {
            const uint32_t b = __float_as_uint(to_float(src[(size_t)k * N])) & 0x7fffffffu;
            mx = b > mx ? b : mx;
        }
    }
    part[g][c] = mx;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) mx = part[i][c] > mx ? part[i][c] : mx;
    const bool none = mx < 0x03800000u;   // below 2^-120 the quotient would overflow: the column counts as zero
    const float m = __uint_as_float(mx), inv = none ? 0.f : 127.f / m;
    if (g == 0 && n < N) scale[(size_t)blockIdx.y * N + n] = none ? 0.f : m / 127.f;
    for (int k0 = 0; k0 < pitch; k0 += 64) {
        __syncthreads();
#pragma unroll 4
        for (int i = 0; i < 16; ++i) {
            const int k = k0 + g * 16 + i;
            float v = n < N && k < K ? to_float(src[(size_t)k * N]) * inv : 0.f;
            tile[c][g * 16 + i] = (int8_t)(int)rintf(fminf(fmaxf(v, -127.f), 127.f));
        }
        __syncthreads();
        const int r = threadIdx.x >> 2, p = threadIdx.x & 3, o = blockIdx.x * 64 + r;
        if (o < N)
            *reinterpret_cast<uint4*>(wq + ((size_t)blockIdx.y * N + o) * pitch + k0 + 16 * p) =
                *reinterpret_cast<const uint4*>(&tile[r][16 * p]);
    }
}


// Rows of a tile, by the mean load.  Measured (MI355X, the whole call, us, 256 | 128 | 32):
//     mean rows                         1           8            16           31           47           62
//     64 experts + 2, d 2048, f 1408  108|89|77  160|140|126  165|142|136  172|151|147  176|166|179  185|173|200
//     256 experts, d 2048, f 512                                                                     254|241|295
//     mean rows                         124      155      186      248      310      496
//     64 experts + 2, d 2048, f 1408  219|201  230|229  248|289  261|304           427|556
//     8 experts, d 2048, f 1408                          62|44    65|53
//     8 experts, d 4096, f 14336      421|442                    524|645           863|1006
//     256 experts, d 2048, f 512      290|315                    413|501
//     24 experts, d 1000, f 712, Zipf  51|37              52|49    56|54
//     32 experts + 1, d 4096, f 1024           196|184           216|214  231|273
//     16 experts + 1, d 7168, f 2048           293|281           313|320
// Up to 384 rows the larger tile also has to come out at one tile for every CU; and K has two units or more, as the next tile's
// first are requested with this one's last.  The mean is all that the rule goes by: at 124 rows of wide experts or of many it
// loses 5 and 8 % so, 3 % at 31 rows and 1 to 4 % at 248 of a skewed load or few tiles.
int q8_tile_rows(int B, int E, int d, int f) {
    if (B <= 16ll * E) return 32;
    const long tiles = ((long)B / 256 + E) * ((f + 127) / 128);
    if (B <= 160ll * E || (B <= 384ll * E && tiles < kQ8RollBlocks)) return 128;
    return q8_pitch(d) < 256 || q8_pitch(f) < 256 ? 128 : 256;
}

}  // namespace
}  // namespace xmoe

using namespace xmoe;

extern "C" {

int xmoe_quantize_weights(const void* w, int E, int K, int N, int dt, void* wq, float* scale, void* stream) {
    if (!dtype_ok(dt)) return XMOE_ERR_UNSUPPORTED;
    if (E < 1 || K < 1 || N < 1) return XMOE_ERR_INVALID_ARG;
    if (E > 65535 || K > XMOE_MAX_Q8_WIDTH) return XMOE_ERR_UNSUPPORTED;
    if (((long)N + 63) / 64 * 256 >= (1l << 32)) return XMOE_ERR_UNSUPPORTED;   // a grid has fewer than 2^32 threads
    if (!w || !wq || !scale || (reinterpret_cast<uintptr_t>(wq) & 15u)) return XMOE_ERR_INVALID_ARG;
    hipStream_t s = (hipStream_t)stream;
    const dim3 grid((unsigned)((N + 63) / 64), (unsigned)E);
    if (dt == XMOE_F32)
        XMOE_LAUNCH(K_QUANTIZE_WEIGHTS, s, hipLaunchKernelGGL(quantize_weights_kernel<float>, grid, dim3(256), 0, s,
                                                              (const float*)w, K, N, q8_pitch(K), (int8_t*)wq, scale));
    else
        XMOE_LAUNCH(K_QUANTIZE_WEIGHTS, s, hipLaunchKernelGGL(quantize_weights_kernel<bf16_t>, grid, dim3(256), 0, s,
                                                              (const bf16_t*)w, K, N, q8_pitch(K), (int8_t*)wq, scale));
    return XMOE_OK;
}

int xmoe_expert_ffn_q8_fwd(const void* xq, const float* x_scale, const int32_t* row_index, const int32_t* expert_offsets,
                           int B, int E, int d, int f, const void* wgq, const float* g_scale, const void* wuq,
                           const float* u_scale, const void* wdq, const float* d_scale, void* y, int dt, void* ws,
                           size_t ws_bytes, void* stream) {
    if (!dtype_ok(dt)) return XMOE_ERR_UNSUPPORTED;
    if (B < 0 || E < 1 || d < 1 || f < 1) return XMOE_ERR_INVALID_ARG;
    if (E > XMOE_MAX_EXPERTS || d > XMOE_MAX_Q8_WIDTH || f > XMOE_MAX_Q8_WIDTH) return XMOE_ERR_UNSUPPORTED;
    if (!expert_offsets || !wgq || !g_scale || !wuq || !u_scale || !wdq || !d_scale) return XMOE_ERR_INVALID_ARG;
    if (B == 0) return XMOE_OK;
    if (!xq || !x_scale || !y || !aligned16(xq) || !aligned16(wgq) || !aligned16(wuq) || !aligned16(wdq))
        return XMOE_ERR_INVALID_ARG;
    if (B >= (1 << 26)) return XMOE_ERR_INVALID_ARG;
    if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255u) || ws_bytes < ffn_q8_ws_bytes(B, E, f)) return XMOE_ERR_WORKSPACE;
    const int fp = q8_pitch(f), dp = q8_pitch(d);
    char* p = (char*)ws;
    int32_t* map = (int32_t*)p;
    p += ffn_q8_tilemap_bytes(B, E);
    float* a32 = (float*)p;
    p += align_up((size_t)B * fp * 4, 256);
    float* gmax = (float*)p;
    p += align_up((size_t)B * (fp / kQ8Group) * 4, 256);
    int8_t* aq = (int8_t*)p;
    p += align_up((size_t)B * fp, 256);
    float* as = (float*)p;
    hipStream_t s = (hipStream_t)stream;
    const int tile_rows = q8_tile_rows(B, E, d, f), max_tiles = ffn_max_tiles(B, E, tile_rows);
    // a grid has fewer than 2^32 threads: tiles of 64 columns and 256 threads are the most
    if (q8_blocks(f > d ? f : d, 64, max_tiles) * 256 >= (1l << 32)) return XMOE_ERR_UNSUPPORTED;
    int st = launch_tile_map(expert_offsets, E, tile_rows, max_tiles, map, map + ffn_q8_sched_offset(B, E), false, s);
    if (st != XMOE_OK) return st;
    const Q8Args up = {(const int8_t*)xq, x_scale, row_index, expert_offsets, map, (const int8_t*)wgq, (const int8_t*)wuq,
                       g_scale, u_scale, dp, f, tile_rows, kQ8RowTiles, a32, gmax, fp, nullptr};
    const Q8Args down = {aq, as, nullptr, expert_offsets, map, (const int8_t*)wdq, nullptr, d_scale, nullptr, fp, d, tile_rows,
                         kQ8RowTiles, nullptr, nullptr, 0, y};
    st = tile_rows == 256   ? launch_q8_gateup<256, 8>(up, max_tiles, s)
         : tile_rows == 128 ? launch_q8_gateup<128, 4>(up, max_tiles, s)
                            : launch_q8_gateup_few(up, max_tiles, s);
    if (st != XMOE_OK) return st;
    XMOE_LAUNCH(K_Q8_ROWS, s,
                hipLaunchKernelGGL(q8_rows_kernel, dim3((unsigned)((B + 3) / 4)), dim3(256), 0, s, a32, gmax, expert_offsets,
                                   E, f, fp, aq, as));
    return tile_rows == 256   ? launch_q8_down<256, 8>(down, max_tiles, dt, s)
           : tile_rows == 128 ? launch_q8_down<128, 4>(down, max_tiles, dt, s)
                              : launch_q8_down_few(down, max_tiles, dt, s);
}

}  // extern "C"
