// A whole MoE layer for a few tokens (a decoding step): gate, top-k, the experts' SwiGLU, the weighted sum, in few launches.
//
//   out[t] = sum_j p[t, e_j] FFN_{e_j}(x[t]) + sum_s FFN_{E+s}(x[t]) (+ addend[t]),   FFN_e(x) = (silu(x Wg) * (x Wu)) Wd
//
// Bound by the weights of the experts that some token picked: each is read once, for all of its tokens.  Nothing of the
// routing goes through tables in memory: a token's choice is a few integers, and every block finds the active experts and
// their tokens (a 32-bit mask per expert) in LDS by itself.
//
//   route   one block per token: logits in the fixed order of xmoe_gate_logits (a lane is one of the 64 partial sums), top-k.
//   up      A = silu(x Wg) * (x Wu) of an active expert and 64 of its columns
//   down    A Wd of an active expert and 128 columns, float32, one row for each (token, expert); the block that finishes a
//           tile of columns last adds the tokens' rows up, in the order of the slots: the result does not depend on which.
//
// Two families of products: bf16 with widths that are multiples of 64 on the matrix cores (the ring of xmoe_few_tile.h),
// everything else on the vector ALUs, where 16 groups of threads share a tile's K and read the weights straight to registers.
#include "xmoe_few_tile.h"
#include "xmoe_route.h"

namespace xmoe {
namespace {

struct LayerArgs {
    const void *x, *w_router, *wg, *wu, *wd, *addend;
    const float* bias;
    int T, d, E, E_s, k, f;
    float* logits;
    int32_t* topk_idx;
    float* topk_w;
    void* out;
    int32_t* done;   // [column tiles of down]: blocks that have finished one
    void* act;       // A, one row of f for each (token, expert)
    float* y;        // the experts' outputs, one row of y_pitch for each (token, expert)
    int y_pitch;
};

// ---------------------------------------------------------------------------------------------------------
// route: one block of 8 waves per token.  Wave w takes the experts 8 w .., 8 (w + 8) ..
// ---------------------------------------------------------------------------------------------------------
// elements at an address that is aligned to one
template <typename T, int N>
struct __attribute__((packed, aligned(sizeof(T)))) LayerVec {
    T v[N];
};

template <typename T, int PER_LANE>
__global__ __launch_bounds__(512) void layer_route_kernel(LayerArgs g) {
    __shared__ float row[XMOE_MAX_EXPERTS];
    const int t = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const T* x = (const T*)g.x + (size_t)t * g.d;
    const T* w = (const T*)g.w_router;
    for (int e0 = wave * 8; e0 < g.E; e0 += 64) {
        float p[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (e0 + 8 <= g.E) {
#pragma unroll 8
            for (int i = lane; i < g.d; i += 64) {
                const float a = to_float(x[i]);
                const LayerVec<T, 8> q = *reinterpret_cast<const LayerVec<T, 8>*>(w + (size_t)i * g.E + e0);
#pragma unroll
                for (int j = 0; j < 8; ++j) p[j] = fmaf(a, to_float(q.v[j]), p[j]);
            }
        } else {
            for (int i = lane; i < g.d; i += 64) {
                const float a = to_float(x[i]);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (e0 + j < g.E) p[j] = fmaf(a, to_float(w[(size_t)i * g.E + e0 + j]), p[j]);
            }
        }
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1)
#pragma unroll
            for (int j = 0; j < 8; ++j) p[j] += __shfl_xor(p[j], off, 64);
        if (lane == 0) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (e0 + j < g.E) {
                    const float v = g.bias ? p[j] + g.bias[e0 + j] : p[j];
                    row[e0 + j] = v;
                    g.logits[(size_t)t * g.E + e0 + j] = v;
                }
        }
    }
    __syncthreads();
    if (wave > 0) return;
    int idx;
    float wt;
    route_token<PER_LANE>(row, g.E, g.k, idx, wt);
    if (lane < g.k) {
        g.topk_idx[(size_t)t * g.k + lane] = idx;
        g.topk_w[(size_t)t * g.k + lane] = wt;
    }
}

// ---------------------------------------------------------------------------------------------------------
// the active experts, in LDS: mask[e] the tokens of expert e, row0[e] the row of its first one, list[i] the i-th active one.
// Every thread of the block (256) calls it.
// ---------------------------------------------------------------------------------------------------------
struct LayerPlan {
    uint32_t mask[XMOE_MAX_EXPERTS];
    int row0[XMOE_MAX_EXPERTS];
    int list[XMOE_MAX_EXPERTS];
    int wave_sum[4];
    int tok[32];   // the tokens of the block's expert
    int n;         // active experts
    int last;
};
__device__ __forceinline__ uint32_t layer_all(int T) { return T < 32 ? (1u << T) - 1u : ~0u; }
__device__ __forceinline__ void layer_plan(LayerPlan& pl, const LayerArgs& g) {
    const int tid = threadIdx.x, Ea = g.E + g.E_s;
#pragma unroll
    for (int i = 0; i < XMOE_MAX_EXPERTS / 256; ++i) {
        const int e = tid + 256 * i;
        pl.mask[e] = e >= g.E && e < Ea ? layer_all(g.T) : 0u;
    }
    __syncthreads();
    for (int i = tid; i < g.T * g.k; i += 256) atomicOr(&pl.mask[g.topk_idx[i]], 1u << (i / g.k));
    __syncthreads();
    // experts 2 tid and 2 tid + 1: how many are active, how many rows they have (packed: up to 512 and up to 32 * 575)
    const uint32_t m0 = pl.mask[2 * tid], m1 = pl.mask[2 * tid + 1];
    const int c = (m0 != 0) + (m1 != 0), r = __popc(m0) + __popc(m1);
    int v = c | (r << 16);
    const int own = v;
#pragma unroll
    for (int w = 1; w < 64; w *= 2) {
        const int o = __shfl_up(v, w, 64);
        if ((tid & 63) >= w) v += o;
    }
    if ((tid & 63) == 63) pl.wave_sum[tid >> 6] = v;
    __syncthreads();
    int before = v - own, all = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if (w < (tid >> 6)) before += pl.wave_sum[w];
        all += pl.wave_sum[w];
    }
    int at = before & 0xffff, row = before >> 16;
    pl.row0[2 * tid] = row;
    pl.row0[2 * tid + 1] = row + __popc(m0);
    if (m0) pl.list[at++] = 2 * tid;
    if (m1) pl.list[at] = 2 * tid + 1;
    if (tid == 0) pl.n = all & 0xffff;
    __syncthreads();
}
// the block's expert (of the plan's list), its tokens in pl.tok; returns how many
__device__ __forceinline__ int layer_tokens(LayerPlan& pl, int e) {
    const uint32_t m = pl.mask[e];
    if (threadIdx.x < 32 && ((m >> threadIdx.x) & 1u)) pl.tok[__popc(m & ((1u << threadIdx.x) - 1u))] = threadIdx.x;
    __syncthreads();
    return __popc(m);
}

// The rows of the tokens in columns [n0, n0 + cols) are complete: out = their weighted sum.  Every thread of the last block.
template <typename T>
__device__ __forceinline__ void layer_sum(const LayerPlan& pl, const LayerArgs& g, int n0, int cols) {
    const int groups = cols / 4;   // of four columns
    for (int i = threadIdx.x; i < g.T * groups; i += 256) {
        const int t = i / groups, col = n0 + 4 * (i - t * groups);
        if (col >= g.d) continue;
        const uint32_t below = (1u << t) - 1u;
        float s[4] = {0.f, 0.f, 0.f, 0.f};
        for (int j = 0; j < g.k; ++j) {
            const int e = g.topk_idx[t * g.k + j];
            const float w = g.topk_w[t * g.k + j];
            const float4 v = *reinterpret_cast<const float4*>(g.y + (size_t)(pl.row0[e] + __popc(pl.mask[e] & below)) * g.y_pitch + col);
            s[0] = fmaf(w, v.x, s[0]);
            s[1] = fmaf(w, v.y, s[1]);
            s[2] = fmaf(w, v.z, s[2]);
            s[3] = fmaf(w, v.w, s[3]);
        }
        for (int e = g.E; e < g.E + g.E_s; ++e) {
            const float4 v = *reinterpret_cast<const float4*>(g.y + (size_t)(pl.row0[e] + t) * g.y_pitch + col);
            s[0] += v.x;
            s[1] += v.y;
            s[2] += v.z;
            s[3] += v.w;
        }
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (col + q < g.d) {
                const size_t at = (size_t)t * g.d + col + q;
                ((T*)g.out)[at] = from_float<T>(g.addend ? s[q] + to_float(((const T*)g.addend)[at]) : s[q]);
            }
    }
}
// Behind the block's rows of y for column tile `tile`: the block that comes last of the n adds the tile up.
template <typename T>
__device__ __forceinline__ void layer_finish(LayerPlan& pl, const LayerArgs& g, int tile, int cols) {
    __threadfence();   // this thread's rows are visible to the device
    __syncthreads();
    if (threadIdx.x == 0) pl.last = atomicAdd(&g.done[tile], 1) == pl.n - 1;
    __syncthreads();
    if (!pl.last) return;
    __threadfence();   // and the others' to this block
    layer_sum<T>(pl, g, tile * cols, cols);
}
__device__ __forceinline__ void layer_clear(const LayerArgs& g, int tiles) {
    if (blockIdx.x == 0)
        for (int i = threadIdx.x; i < tiles; i += 256) g.done[i] = 0;
}

// ---------------------------------------------------------------------------------------------------------
// matrix cores (bf16, d % 64 == 0, f % 64 == 0, 16-byte aligned)
// ---------------------------------------------------------------------------------------------------------
template <int MODE>
__device__ __forceinline__ void layer_loader(FewLoader& ld, const bf16_t* x, size_t ldx, const int* tok, int row0, int rows,
                                             const bf16_t* w0, const bf16_t* w1, int K, int N, int n0) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    {
        int r = wave * 16 + (lane >> 2);   // rows past the last one repeat it; what they give is not stored
        const int c = (lane & 3) ^ ((r >> 2) & 3);
        r = r < rows ? r : rows - 1;
        ld.x = x + (size_t)(tok ? tok[r] : row0 + r) * ldx + 8 * c;
    }
    const int c = (lane & 15) ^ ((lane >> 4) << 2);
    const bf16_t* w = MODE == FEW_GATEUP && c >= 8 ? w1 : w0;
    int col = n0 + 8 * (MODE == FEW_GATEUP ? c & 7 : c);
    if (col >= N) col = n0;   // the second half of a tile at the edge: not stored
    w += (size_t)(wave * 8 + (lane >> 4)) * N + col;
    ld.w[0] = w;
    ld.w[1] = w + (size_t)4 * N;
    ld.step = (size_t)kFewK * N;
    ld.left = K / kFewK;
}

__global__ __launch_bounds__(256, 2) void layer_up_few_kernel(LayerArgs g, int down_tiles) {
    __shared__ __align__(16) char smem[kFewStages * kFewStageBytes];
    __shared__ LayerPlan pl;
    layer_clear(g, down_tiles);
    layer_plan(pl, g);
    const int nt = (g.f + 63) / 64, i = blockIdx.x / nt, n0 = (blockIdx.x - i * nt) * 64;
    if (i >= pl.n) return;
    const int e = pl.list[i], rows = layer_tokens(pl, e);
    const size_t we = (size_t)e * g.d * g.f;
    FewLoader ld;
    layer_loader<FEW_GATEUP>(ld, (const bf16_t*)g.x, g.d, pl.tok, 0, rows, (const bf16_t*)g.wg + we, (const bf16_t*)g.wu + we,
                             g.d, g.f, n0);
    few_f32x16_t acc[1];
    few_loop<FEW_GATEUP, 1>(acc, ld, smem, g.d / kFewK);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 31, col = n0 + 16 * wave + 4 * (lane >> 5);
    if (r >= rows) return;
    bf16_t* o = (bf16_t*)g.act + (size_t)(pl.row0[e] + r) * g.f + col;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        float a[4];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const float gv = acc[0][4 * q + v];
            a[v] = gv * fast_sigmoid(gv) * acc[0][8 + 4 * q + v];
        }
        *reinterpret_cast<uint2*>(o + 8 * q) = make_uint2(pack_bf16x2(a[0], a[1]), pack_bf16x2(a[2], a[3]));
    }
}

__global__ __launch_bounds__(256, 2) void layer_down_few_kernel(LayerArgs g) {
    __shared__ __align__(16) char smem[kFewStages * kFewStageBytes];
    __shared__ LayerPlan pl;
    layer_plan(pl, g);
    const int nt = (g.d + kFewCols - 1) / kFewCols, i = blockIdx.x / nt, tile = blockIdx.x - i * nt, n0 = tile * kFewCols;
    if (i >= pl.n) return;
    const int e = pl.list[i], rows = __popc(pl.mask[e]), row0 = pl.row0[e];
    FewLoader ld;
    layer_loader<FEW_PLAIN>(ld, (const bf16_t*)g.act, g.f, nullptr, row0, rows, (const bf16_t*)g.wd + (size_t)e * g.f * g.d,
                            nullptr, g.f, g.d, n0);
    few_f32x16_t acc[1];
    few_loop<FEW_PLAIN, 1>(acc, ld, smem, g.f / kFewK);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 31, col = n0 + 32 * wave + 4 * (lane >> 5);
    if (r < rows && col < g.d) {
        float* o = g.y + (size_t)(row0 + r) * g.y_pitch + col;
#pragma unroll
        for (int q = 0; q < 4; ++q)
            *reinterpret_cast<float4*>(o + 8 * q) = make_float4(acc[0][4 * q], acc[0][4 * q + 1], acc[0][4 * q + 2], acc[0][4 * q + 3]);
    }
    layer_finish<bf16_t>(pl, g, tile, kFewCols);
}

// ---------------------------------------------------------------------------------------------------------
// vector ALUs: float32, and bf16 widths that are no multiple of 64
// ---------------------------------------------------------------------------------------------------------
// Thread (k-group of 16, column group c of 16): four consecutive k of every 64 and EV columns (16 bytes; one where N is less
// than 16 bytes).  A column group that would pass N starts at N - EV instead: the columns it shares with its neighbour come
// out the same twice.
constexpr int kAluRows = 4;   // rows multiplied at a time

template <typename T, int M, int EV>
__device__ __forceinline__ void alu_tile(const T* x, size_t ldx, const int (&src)[kAluRows], int K, const T* w0, const T* w1, int N,
                                         int col, float (&acc)[M][kAluRows][EV]) {
    const int kg = threadIdx.x >> 4;
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
        for (int r = 0; r < kAluRows; ++r)
#pragma unroll
            for (int j = 0; j < EV; ++j) acc[m][r][j] = 0.f;
    const T* xr[kAluRows];
#pragma unroll
    for (int r = 0; r < kAluRows; ++r) xr[r] = x + (size_t)src[r] * ldx;
    auto step = [&](int k0, auto part) {   // k0 .. k0 + 3, part: those below K
        constexpr bool kPart = decltype(part)::value;
        LayerVec<T, EV> w[M][4];
        float a[kAluRows][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int k = kPart && k0 + i >= K ? K - 1 : k0 + i;
#pragma unroll
            for (int m = 0; m < M; ++m) {
                w[m][i] = *reinterpret_cast<const LayerVec<T, EV>*>((m == 0 ? w0 : w1) + (size_t)k * N + col);
            }
        }
#pragma unroll
        for (int r = 0; r < kAluRows; ++r) {
            if (kPart) {
#pragma unroll
                for (int i = 0; i < 4; ++i) a[r][i] = to_float(xr[r][k0 + i < K ? k0 + i : K - 1]);
            } else {
                const LayerVec<T, 4> q = *reinterpret_cast<const LayerVec<T, 4>*>(xr[r] + k0);
#pragma unroll
                for (int i = 0; i < 4; ++i) a[r][i] = to_float(q.v[i]);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (kPart && k0 + i >= K) break;
#pragma unroll
            for (int m = 0; m < M; ++m)
#pragma unroll
                for (int r = 0; r < kAluRows; ++r)
#pragma unroll
                    for (int j = 0; j < EV; ++j) acc[m][r][j] = fmaf(a[r][i], to_float(w[m][i].v[j]), acc[m][r][j]);
        }
    };
    int k0 = 4 * kg;
#pragma unroll 2
    for (; k0 + 4 <= K; k0 += 64) step(k0, std::false_type{});
    if (k0 < K) step(k0, std::true_type{});
}

// The block's tile of `cols` = 16 EV columns from n0 on: result(r, column, value of matrix 0, value of matrix 1) for every
// row r < rows and column < N.  source(r): row r of x.
template <typename T, int M, int EV, class Source, class Result>
__device__ __forceinline__ void alu_product(const T* x, size_t ldx, int rows, int K, const T* w0, const T* w1, int N, int n0,
                                            float* red, Source source, Result result) {
    constexpr int C = 16 * EV;
    const int c = threadIdx.x & 15, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    int col = n0 + c * EV;
    if (col + EV > N) col = N - EV;
    for (int r0 = 0; r0 < rows; r0 += kAluRows) {
        int src[kAluRows];
#pragma unroll
        for (int r = 0; r < kAluRows; ++r) src[r] = source(r0 + r < rows ? r0 + r : rows - 1);
        float acc[M][kAluRows][EV];
        alu_tile<T, M, EV>(x, ldx, src, K, w0, w1, N, col, acc);
        // the sixteen groups' sums: four of a wave, then the waves in order
#pragma unroll
        for (int m = 0; m < M; ++m)
#pragma unroll
            for (int r = 0; r < kAluRows; ++r)
#pragma unroll
                for (int j = 0; j < EV; ++j) {
                    float v = acc[m][r][j];
                    v += __shfl_xor(v, 16, 64);
                    v += __shfl_xor(v, 32, 64);
                    if (lane < 16) red[((wave * M + m) * kAluRows + r) * C + c * EV + j] = v;
                }
        __syncthreads();
        for (int i = threadIdx.x; i < kAluRows * C; i += 256) {
            const int r = i / C, cc = i - r * C;
            int at = n0 + cc / EV * EV;   // where the column group of this sum starts
            if (at + EV > N) at = N - EV;
            at += cc % EV;
            float v[2] = {0.f, 0.f};
#pragma unroll
            for (int m = 0; m < M; ++m)
#pragma unroll
                for (int w = 0; w < 4; ++w) v[m] += red[((w * M + m) * kAluRows + r) * C + cc];
            if (r0 + r < rows && at < N) result(r0 + r, at, v[0], v[1]);
        }
        __syncthreads();
    }
}

template <typename T, int EV>
__global__ __launch_bounds__(256) void layer_up_alu_kernel(LayerArgs g, int down_tiles) {
    constexpr int C = 16 * EV;
    __shared__ float red[4 * 2 * kAluRows * C];
    __shared__ LayerPlan pl;
    layer_clear(g, down_tiles);
    layer_plan(pl, g);
    const int nt = (g.f + C - 1) / C, i = blockIdx.x / nt, n0 = (blockIdx.x - i * nt) * C;
    if (i >= pl.n) return;
    const int e = pl.list[i], rows = layer_tokens(pl, e), row0 = pl.row0[e];
    const size_t we = (size_t)e * g.d * g.f;
    T* o = (T*)g.act;
    alu_product<T, 2, EV>((const T*)g.x, g.d, rows, g.d, (const T*)g.wg + we, (const T*)g.wu + we, g.f, n0, red,
                            [&](int r) { return pl.tok[r]; },
                            [&](int r, int c, float gv, float uv) {
                                o[(size_t)(row0 + r) * g.f + c] = from_float<T>(siluf_(gv) * uv);
                            });
}
template <typename T, int EV>
__global__ __launch_bounds__(256) void layer_down_alu_kernel(LayerArgs g) {
    constexpr int C = 16 * EV;
    __shared__ float red[4 * kAluRows * C];
    __shared__ LayerPlan pl;
    layer_plan(pl, g);
    const int nt = (g.d + C - 1) / C, i = blockIdx.x / nt, tile = blockIdx.x - i * nt;
    if (i >= pl.n) return;
    const int e = pl.list[i], rows = __popc(pl.mask[e]), row0 = pl.row0[e];
    alu_product<T, 1, EV>((const T*)g.act, g.f, rows, g.f, (const T*)g.wd + (size_t)e * g.f * g.d, (const T*)nullptr, g.d,
                            tile * C, red, [&](int r) { return row0 + r; },
                            [&](int r, int c, float v, float) { g.y[(size_t)(row0 + r) * g.y_pitch + c] = v; });
    layer_finish<T>(pl, g, tile, C);
}

template <typename T>
int launch_alu(const LayerArgs& a, int active, hipStream_t s) {
    constexpr int EV = 16 / (int)sizeof(T);
    const int cu = a.f < EV ? 16 : 16 * EV, cd = a.d < EV ? 16 : 16 * EV, up = (a.f + cu - 1) / cu, down = (a.d + cd - 1) / cd;
    const dim3 g1((unsigned)(active * up)), g2((unsigned)(active * down));
    if (a.f < EV)
        XMOE_LAUNCH(K_LAYER_UP_ALU, s, hipLaunchKernelGGL((layer_up_alu_kernel<T, 1>), g1, dim3(256), 0, s, a, down));
    else
        XMOE_LAUNCH(K_LAYER_UP_ALU, s, hipLaunchKernelGGL((layer_up_alu_kernel<T, EV>), g1, dim3(256), 0, s, a, down));
    if (a.d < EV)
        XMOE_LAUNCH(K_LAYER_DOWN_ALU, s, hipLaunchKernelGGL((layer_down_alu_kernel<T, 1>), g2, dim3(256), 0, s, a));
    else
        XMOE_LAUNCH(K_LAYER_DOWN_ALU, s, hipLaunchKernelGGL((layer_down_alu_kernel<T, EV>), g2, dim3(256), 0, s, a));
    return XMOE_OK;
}

template <typename T>
int launch_layer_route(const LayerArgs& a, hipStream_t s) {
    const dim3 grid((unsigned)a.T);
#define XMOE_CALL(PL) \
    XMOE_LAUNCH(K_LAYER_ROUTE, s, hipLaunchKernelGGL((layer_route_kernel<T, PL>), grid, dim3(512), 0, s, a))
    if (a.E <= 64) XMOE_CALL(1);
    else if (a.E <= 128) XMOE_CALL(2);
    else if (a.E <= 256) XMOE_CALL(4);
    else XMOE_CALL(8);
#undef XMOE_CALL
    return XMOE_OK;
}

// A block per token reads the whole router: up to this many bytes of it
constexpr size_t kRouteBytes = 512 << 10;

}  // namespace
}  // namespace xmoe

using namespace xmoe;

extern "C" int xmoe_layer_few_fwd(const void* x, const void* w_router, const float* bias, const void* wg, const void* wu,
                                  const void* wd, const void* addend, int T, int d, int E, int E_s, int k, int f, int dt,
                                  float* logits, int32_t* topk_idx, float* topk_w, void* out, void* ws, size_t ws_bytes,
                                  void* stream) {
    if (!dtype_ok(dt)) return XMOE_ERR_UNSUPPORTED;
    if (T < 0 || d < 1 || E < 1 || E_s < 0 || k < 1 || k > E || f < 1) return XMOE_ERR_INVALID_ARG;
    if (T > XMOE_FEW_TOKENS || E > XMOE_MAX_EXPERTS || E_s > XMOE_MAX_EXPERTS - E || k > 64 || d > XMOE_MAX_FEW_WIDTH ||
        f > XMOE_MAX_FEW_WIDTH)
        return XMOE_ERR_UNSUPPORTED;
    if (!w_router || !wg || !wu || !wd) return XMOE_ERR_INVALID_ARG;
    if (T == 0) return XMOE_OK;
    if (!x || !logits || !topk_idx || !topk_w || !out) return XMOE_ERR_INVALID_ARG;
    if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255u) || ws_bytes < layer_few_ws_bytes(T, d, k + E_s, f, dt))
        return XMOE_ERR_WORKSPACE;
    hipStream_t s = (hipStream_t)stream;
    const size_t rows = (size_t)T * (k + E_s);
    LayerArgs a{x, w_router, wg, wu, wd, addend, bias, T, d, E, E_s, k, f, logits, topk_idx, topk_w, out};
    char* p = (char*)ws;
    a.done = (int32_t*)p;
    p += layer_few_done_bytes(d);
    a.act = p;
    p += align_up(rows * f * dtype_size(dt), 256);
    a.y = (float*)p;
    a.y_pitch = layer_few_y_pitch(d);
    int st;
    if ((size_t)d * E * dtype_size(dt) <= kRouteBytes) {
        st = dt == XMOE_F32 ? launch_layer_route<float>(a, s) : launch_layer_route<bf16_t>(a, s);
    } else {
        st = xmoe_gate_logits(x, w_router, bias, logits, T, d, E, dt, stream);
        if (st == XMOE_OK) st = xmoe_route(logits, T, E, k, topk_idx, topk_w, stream);
    }
    if (st != XMOE_OK) return st;
    const int active = (T * k < E ? T * k : E) + E_s;
    if (dt == XMOE_F32) return launch_alu<float>(a, active, s);
    if (d % 64 || f % 64 || !aligned16(x) || !aligned16(wg) || !aligned16(wu) || !aligned16(wd))
        return launch_alu<bf16_t>(a, active, s);
    const int up = f / 64, down = (d + kFewCols - 1) / kFewCols;
    XMOE_LAUNCH(K_LAYER_UP_FEW, s,
                hipLaunchKernelGGL(layer_up_few_kernel, dim3((unsigned)(active * up)), dim3(256), 0, s, a, down));
    XMOE_LAUNCH(K_LAYER_DOWN_FEW, s,
                hipLaunchKernelGGL(layer_down_few_kernel, dim3((unsigned)(active * down)), dim3(256), 0, s, a));
    return XMOE_OK;
}
