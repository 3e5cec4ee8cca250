// A whole MoE layer for a few tokens (a decoding step): gate, top-k, the experts' SwiGLU, the weighted sum, in few launches.
//
//   out[t] = sum_j p[t, e_j] FFN_{e_j}(x[t]) + sum_s FFN_{E+s}(x[t]) (+ addend[t]),   FFN_e(x) = (silu(x Wg) * (x Wu)) Wd
//
// Bound by the weights of the experts that some token picked: on the matrix cores each is read once, for all of its tokens, on
// the vector ALUs once for every 8 of them (float32) or 4 (bf16).  Nothing of the routing goes through tables in memory: a
// token's choice is a few integers, and every block finds the active experts and their tokens (a 32-bit mask per expert) in LDS
// by itself.
//
//   route   one block per token: logits in the fixed order of xmoe_gate_logits, top-k (large routers: that call and xmoe_route)
//   up      A = silu(x Wg) * (x Wu) of an active expert and 64 or 128 of its columns
//   down    A Wd of an active expert, 256 columns and a slab of f, float32, one row for each (token, expert) and slab
//   sum     the tokens' rows, slabs and slots in order
//
// Two families of products: bf16 with widths that are multiples of 8 on the matrix cores, weights on a ring of direct-to-LDS
// stages; everything else on the vector ALUs, where 16 groups of threads share a tile's K and read the weights straight to
// registers.  A is an operand of the matrix cores and so rounded to bf16, as in the layer for many tokens; sums are float32 up to
// the result (its distance from 64-bit arithmetic: 0.0018, of which the result's own rounding is 0.0017).
// d 2048, f 1408, 6 of 64 experts + 2, bf16: one token 48 us (12 + 20.6 + 10.8 + 4.9; 139 MB in up and down at 4.4 TB/s), 16
// tokens 189 (12 + 113 + 58 + 5.4; 5.2 TB/s).
// Tried: a launch less, the last block of a column's down tiles adding the rows (a fence by every block: slower), and one
// launch for all of it with a ticket per item (an atomic on one address takes 60 to 75 ns: 71 us for one token).
#include "xmoe_ffn.h"
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
    void* act;       // A, one row of f for each (token, expert)
    float* y;        // the experts' outputs, slabs x (one row of y_pitch for each (token, expert))
    int32_t* row_of;   // [T][k + E_s]: the row of a token's j-th expert
    int y_pitch, slabs;
};

// ---------------------------------------------------------------------------------------------------------
// route: one block of 8 waves per token.  64 rows of the router are contiguous, and a thread takes 16 bytes of them (EV
// experts of one row: one of the 64 partial sums of each; EV = 1 where rows are no whole 16-byte pieces), those of the next 64
// rows, and so on: whole lines, every load independent of every other.  The partial sums are folded in LDS, and the first
// wave picks the experts.  Latency: a router of 256 KiB is on its way to one CU at once, in registers.
// ---------------------------------------------------------------------------------------------------------
// elements at an address that is aligned to one
template <typename T, int N>
struct __attribute__((packed, aligned(sizeof(T)))) LayerVec {
    T v[N];
};
constexpr int kRouteExperts = 128, kRouteX = 4096;   // experts at most; values of x in LDS at a time
constexpr int kRouteSteps = 16;                      // of 64 rows, whose loads are in flight together

template <typename T, int EV>
__global__ __launch_bounds__(512) void layer_route_kernel(LayerArgs g) {
    __shared__ float xs[kRouteX], part[64 * kRouteExperts];   // part: [partial sum][expert]
    const int t = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const T* x = (const T*)g.x + (size_t)t * g.d;
    const T* w = (const T*)g.w_router;
    const int per_row = g.E / EV, chunk = 64 * per_row;   // pieces of a row, of 64 rows
    // every thread has the same number of pieces but for the last round
    for (int n0 = 0; n0 < chunk; n0 += 512) {
        const int n = n0 + threadIdx.x < chunk ? n0 + threadIdx.x : chunk - 1, l = n / per_row;   // past the last: not stored
        float p[EV];
#pragma unroll
        for (int j = 0; j < EV; ++j) p[j] = 0.f;
        for (int i0 = 0; i0 < g.d; i0 += kRouteX) {
            const int len = g.d - i0 < kRouteX ? g.d - i0 : kRouteX;
            const T* src = w + (size_t)i0 * g.E + (size_t)n * EV;
            LayerVec<T, EV> q[kRouteSteps];
            auto fetch = [&](int m) {   // rows i0 + 64 m + l ..; one past the end: row 64 m0 + l of the chunk again, not used
#pragma unroll
                for (int u = 0; u < kRouteSteps; ++u)
                    q[u] = *reinterpret_cast<const LayerVec<T, EV>*>(src + (size_t)(64 * (m + u) + l < len ? m + u : 0) * chunk * EV);
            };
            // the row l itself may be past the end of a short router: its first piece stands in
            if (l >= len) src = w;
            fetch(0);
            if (n0 > 0 || i0 > 0) __syncthreads();
            for (int i = threadIdx.x; i < len; i += 512) xs[i] = to_float(x[i0 + i]);
            __syncthreads();
            for (int m = 0; 64 * m < len; m += kRouteSteps) {
#pragma unroll
                for (int u = 0; u < kRouteSteps; ++u) {
                    const int i = 64 * (m + u) + l;
                    if (i < len) {
                        const float a = xs[i];
#pragma unroll
                        for (int j = 0; j < EV; ++j) p[j] = fmaf(a, to_float(q[u].v[j]), p[j]);
                    }
                }
                if (64 * (m + kRouteSteps) < len) fetch(m + kRouteSteps);
            }
        }
        if (n0 + (int)threadIdx.x < chunk) {
#pragma unroll
            for (int j = 0; j < EV; ++j) part[n * EV + j] = p[j];   // [l][expert]: the pieces' own order
        }
    }
    __syncthreads();
    for (int off = 32; off >= 1; off /= 2) {
        for (int i = threadIdx.x; i < off * g.E; i += 512) part[i] += part[i + off * g.E];
        __syncthreads();
    }
    for (int e = threadIdx.x; e < g.E; e += 512) {
        const float v = g.bias ? part[e] + g.bias[e] : part[e];
        g.logits[(size_t)t * g.E + e] = v;
        xs[e] = v;
    }
    __syncthreads();
    if (wave > 0) return;
    int idx;
    float wt;
    if (g.E <= 64)
        route_token<1>(xs, g.E, g.k, idx, wt);
    else
        route_token<kRouteExperts / 64>(xs, g.E, g.k, idx, wt);
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
// the rows of the tokens' experts, for the sums (by one block of up)
__device__ __forceinline__ void layer_rows(const LayerPlan& pl, const LayerArgs& g) {
    const int n = g.k + g.E_s;
    for (int i = threadIdx.x; i < g.T * n; i += 256) {
        const int t = i / n, j = i - t * n, e = j < g.k ? g.topk_idx[t * g.k + j] : g.E + j - g.k;
        g.row_of[i] = pl.row0[e] + __popc(pl.mask[e] & ((1u << t) - 1u));
    }
}
// the block's expert (of the plan's list), its tokens in pl.tok; returns how many
__device__ __forceinline__ int layer_tokens(LayerPlan& pl, int e) {
    const uint32_t m = pl.mask[e];
    if (threadIdx.x < 32 && ((m >> threadIdx.x) & 1u)) pl.tok[__popc(m & ((1u << threadIdx.x) - 1u))] = threadIdx.x;
    __syncthreads();
    return __popc(m);
}

// ---------------------------------------------------------------------------------------------------------
// matrix cores (bf16, d % 8 == 0, f % 8 == 0, 16-byte aligned: rows are whole 16-byte pieces)
// ---------------------------------------------------------------------------------------------------------
// A block of 4 waves multiplies up to 32 rows with COLS columns, KS k to a stage, on a ring of direct-to-LDS stages.
// LDS of a stage: KS k-rows of COLS columns, whose 16-byte pieces are XOR-ed with 4 * (k-row % 4), then 32 rows of x with 2 KS
// bytes each, pieces XOR-ed with (row / 4) % 4 or (row / 2) % 8: the fragment reads fall on all banks.
// The plan lies behind the ring in the same array: LDS reads of an object of its own would make the compiler wait for every
// direct-to-LDS load in flight at each of the ring's reads.
typedef __attribute__((ext_vector_type(8))) __bf16 layer_bf16x8_t;
typedef __attribute__((ext_vector_type(16))) float layer_f32x16_t;
typedef __attribute__((ext_vector_type(4))) short layer_s16x4_t;
typedef __attribute__((ext_vector_type(8))) short layer_s16x8_t;

__device__ __align__(16) const uint32_t kRingZero[4] = {0u, 0u, 0u, 0u};
__device__ __forceinline__ void ring_load16(const bf16_t* p, char* lds) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)p,
                                     (__attribute__((address_space(3))) void*)lds, 16, 0, 0);
}
// DUAL: the columns are COLS / 2 of two matrices each
template <int COLS, bool DUAL, int KS, int STAGES>
struct Ring {
    static constexpr int kW = KS * COLS * 2, kStage = kW + 32 * KS * 2, kBytes = STAGES * kStage;
    static constexpr int kLoads = kW / 4096;       // of weights, per wave and stage
    static constexpr int kPieces = KS / 8;         // of a row of x; with 64 k every wave fetches 8 rows, with 32 waves 0 and 1 16
    static constexpr bool kAllX = KS == 64;
    static constexpr int kBlocks = COLS / 128;     // of 32 columns, per wave
    static constexpr int kRows = 1024 / (2 * COLS);   // k-rows of a load
    const bf16_t *w[kLoads], *x;   // of the stage issued next
    size_t step;                   // elements between the weights of two stages
    int left;                      // stages behind the one issued next
    uint32_t out;                  // bit i: the i-th piece of weights (bit kLoads: of x) lies behind K in the last stage

    __host__ __device__ static int stages(int K) { return (K + KS - 1) / KS; }
    __device__ __forceinline__ static int x_piece(int r, int c) { return c ^ (kAllX ? (r >> 1) & 7 : (r >> 2) & 3); }
    // rows: source(r) is row r's first element; w0, w1: element (first k, n0) of the matrices, N columns of which cols exist
    template <class Source>
    __device__ __forceinline__ void init(Source source, int rows, const bf16_t* w0, const bf16_t* w1, int N, int cols, int K) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = stages(K), tail = K - KS * (n - 1);
        out = 0u;
        {
            const int r = (kAllX ? wave : wave & 1) * (64 / kPieces) + lane / kPieces, c = x_piece(r, lane % kPieces);
            x = source(r < rows ? r : rows - 1) + 8 * c;   // rows past the last one repeat it; what they give is not stored
            if (8 * c >= tail) out |= 1u << kLoads;
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int kr = wave * (KS / 4) + i * kRows + lane * 8 / COLS;
            if (kr >= tail) out |= 1u << i;
            int col = 8 * ((lane & (COLS / 8 - 1)) ^ ((kr & 3) << 2));
            const bf16_t* b = w0;
            if (DUAL && col >= COLS / 2) {
                b = w1;
                col -= COLS / 2;
            }
            if (col >= cols) col = 0;   // past the edge: not stored
            w[i] = b + (size_t)kr * N + col;
        }
        step = (size_t)KS * N;
        left = n - 1;
    }
    // pieces behind K come from a block of zeros; behind the last stage that one is fetched again, so that the counts stay
    // uniform, and not used
    __device__ __forceinline__ void issue(char* __restrict__ stage) {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        if (left == 0) {   // the last stage: from now on
            const bf16_t* zero = reinterpret_cast<const bf16_t*>(kRingZero);
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
                if ((out >> i) & 1u) w[i] = zero;
            if ((out >> kLoads) & 1u) x = zero;
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            ring_load16(w[i], stage + wave * (kW / 4) + i * 1024);
            w[i] += left > 0 ? step : 0;
        }
        if (kAllX || wave < 2) ring_load16(x, stage + kW + wave * 1024);
        x += left > 0 ? KS : 0;
        --left;
    }
    // at most N stages of the wave's loads on their way, its LDS reads returned
    template <int N>
    __device__ __forceinline__ static void wait() {
        if (kAllX || __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) < 2)
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N * (kLoads + 1)) : "memory");
        else
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(N * kLoads) : "memory");
    }
    // the wave's b-th 32 columns (DUAL with one block: 16 of either matrix), 8 k (16 ks + 8 (lane / 32) ..): in a group of 16
    // lanes, lane s addresses 4 consecutive columns (s % 4) of k-row s / 4, and the transposing read hands every lane one
    // column with 4 consecutive k
    __device__ __forceinline__ static layer_bf16x8_t frag_w(const char* stage, int b, int ks) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, G = lane >> 4, s = lane & 15;
        const int col = (DUAL ? (kBlocks == 1 ? 64 * (G & 1) + 16 * wave : 128 * b + 32 * wave + 16 * (G & 1))
                              : 32 * kBlocks * wave + 32 * b + 16 * (G & 1)) + 4 * (s & 3);
        layer_s16x4_t h[2];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int kr = 16 * ks + 8 * (G >> 1) + (s >> 2) + 4 * q;
            const char* a = stage + kr * (2 * COLS) + (((col >> 3) ^ ((kr & 3) << 2)) << 4) + (col & 7) * 2;
            h[q] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) layer_s16x4_t*)(
                (__attribute__((address_space(3))) void*)a));
        }
        const layer_s16x8_t v = {h[0][0], h[0][1], h[0][2], h[0][3], h[1][0], h[1][1], h[1][2], h[1][3]};
        return __builtin_bit_cast(layer_bf16x8_t, v);
    }
    __device__ __forceinline__ static layer_bf16x8_t frag_x(const char* stage, int ks) {
        const int lane = threadIdx.x & 63, r = lane & 31, c = 2 * ks + (lane >> 5);
        return *reinterpret_cast<const layer_bf16x8_t*>(stage + kW + r * (2 * KS) + (x_piece(r, c) << 4));
    }
    // Refills the stage read before the last barrier and multiplies `cur`.  The two are distinct, and saying so matters: an
    // LDS read that may observe a direct-to-LDS load in flight makes the compiler wait for all of them.
    __device__ __forceinline__ void step_on(layer_f32x16_t (&acc)[kBlocks], char* __restrict__ next,
                                            const char* __restrict__ cur) {
        issue(next);
#pragma unroll
        for (int ks = 0; ks < KS / 16; ++ks) {
            const layer_bf16x8_t a = frag_x(cur, ks);
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
                acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag_w(cur, b, ks), a, acc[b], 0, 0, 0);
        }
    }
    // acc[b], register v of lane l: row l % 32, column 8 (v/4) + 4 (l/32) + v%4 of the wave's b-th 32
    __device__ __forceinline__ void run(layer_f32x16_t (&acc)[kBlocks], char* smem, int n) {
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[b][v] = 0.f;
#pragma unroll
        for (int s = 0; s < STAGES - 1; ++s) issue(smem + s * kStage);
        int cur = 0, next = STAGES - 1;
        for (int i = 0; i < n; ++i) {
            // stage i has landed for every thread, and every wave is done with stage i - 1, which is refilled now
            wait<STAGES - 2>();
            asm volatile("s_barrier" ::: "memory");
            step_on(acc, smem + next * kStage, smem + cur * kStage);
            next = cur;
            cur = cur + 1 < STAGES ? cur + 1 : 0;
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // nothing may land in this LDS once the block has left it
    }
};

__device__ __forceinline__ void layer_store_act(const LayerArgs& g, int row, int col, const float (&gv)[4], const float (&uv)[4]) {
    float a[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = gv[i] * fast_sigmoid(gv[i]) * uv[i];
    *reinterpret_cast<uint2*>((bf16_t*)g.act + (size_t)row * g.f + col) = make_uint2(pack_bf16x2(a[0], a[1]), pack_bf16x2(a[2], a[3]));
}

// COLS / 2 columns of A of one expert
template <int COLS, int KS, int STAGES>
__global__ __launch_bounds__(256, 2) void layer_up_few_kernel(LayerArgs g) {
    typedef Ring<COLS, true, KS, STAGES> R;
    __shared__ __align__(16) char smem[R::kBytes + sizeof(LayerPlan)];
    LayerPlan& pl = *reinterpret_cast<LayerPlan*>(smem + R::kBytes);
    layer_plan(pl, g);
    if (blockIdx.x == 0) layer_rows(pl, g);
    const int nt = (g.f + COLS / 2 - 1) / (COLS / 2), i = blockIdx.x / nt, n0 = (blockIdx.x - i * nt) * (COLS / 2);
    if (i >= pl.n) return;
    const int e = pl.list[i], rows = layer_tokens(pl, e), row0 = pl.row0[e];
    const size_t we = (size_t)e * g.d * g.f + n0;
    R ring;
    ring.init([&](int r) { return (const bf16_t*)g.x + (size_t)pl.tok[r] * g.d; }, rows, (const bf16_t*)g.wg + we,
              (const bf16_t*)g.wu + we, g.f, g.f - n0, g.d);
    layer_f32x16_t acc[R::kBlocks];
    ring.run(acc, smem, R::stages(g.d));
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 31;
    if (r >= rows) return;
    const int col = n0 + COLS / 8 * wave + 4 * (lane >> 5);
#pragma unroll
    for (int q = 0; q < COLS / 64; ++q) {
        float gv[4], uv[4];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            gv[v] = acc[0][4 * q + v];
            uv[v] = COLS == 128 ? acc[0][(8 + 4 * q + v) & 15] : acc[R::kBlocks - 1][4 * q + v];
        }
        if (col + 8 * q < g.f) layer_store_act(g, row0 + r, col + 8 * q, gv, uv);
    }
}

// 256 columns of an expert's output, over a slab of f
constexpr int kDownCols = 256, kDownK = 32, kDownStages = 4;
__global__ __launch_bounds__(256, 2) void layer_down_few_kernel(LayerArgs g) {
    typedef Ring<kDownCols, false, kDownK, kDownStages> R;
    __shared__ __align__(16) char smem[R::kBytes + sizeof(LayerPlan)];
    LayerPlan& pl = *reinterpret_cast<LayerPlan*>(smem + R::kBytes);
    layer_plan(pl, g);
    const int nt = (g.d + kDownCols - 1) / kDownCols, per = nt * g.slabs, i = blockIdx.x / per;
    if (i >= pl.n) return;
    const int slab = (blockIdx.x - i * per) / nt, n0 = (blockIdx.x - i * per - slab * nt) * kDownCols;
    const int all = R::stages(g.f), s0 = all * slab / g.slabs, s1 = all * (slab + 1) / g.slabs;   // slabs <= all
    const int K = (s1 < all ? kDownK * s1 : g.f) - kDownK * s0;
    const int e = pl.list[i], rows = __popc(pl.mask[e]), row0 = pl.row0[e];
    R ring;
    ring.init([&](int r) { return (const bf16_t*)g.act + (size_t)(row0 + r) * g.f + s0 * kDownK; }, rows,
              (const bf16_t*)g.wd + ((size_t)e * g.f + s0 * kDownK) * g.d + n0, nullptr, g.d, g.d - n0, K);
    layer_f32x16_t acc[R::kBlocks];
    ring.run(acc, smem, s1 - s0);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 31;
    if (r >= rows) return;
    const int col = n0 + 64 * wave + 4 * (lane >> 5);
    float* o = g.y + ((size_t)slab * g.T * (g.k + g.E_s) + row0 + r) * g.y_pitch + col;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (col + 32 * b + 8 * q < g.d)
                *reinterpret_cast<float4*>(o + 32 * b + 8 * q) =
                    make_float4(acc[b][4 * q], acc[b][4 * q + 1], acc[b][4 * q + 2], acc[b][4 * q + 3]);
}

// out = the weighted sum of the tokens' rows: slots in order, then the shared experts, then the addend; a row's slabs in order.
// Latency: a thread fetches sixteen pieces at a time.  One wave per token and 256 columns, as one CU fetches 47 GB/s (1 token, 8
// rows of 4 slabs, d 2048: 5.4 us with blocks of 1024 columns and eight pieces, 4.1 so).
template <typename T, int SLABS>
__global__ __launch_bounds__(64) void layer_sum_kernel(LayerArgs g) {
    const int t = blockIdx.x, col = (blockIdx.y * 64 + threadIdx.x) * 4, n = g.k + g.E_s;
    if (col >= g.d) return;
    const size_t slab = (size_t)g.T * n * g.y_pitch;
    constexpr int N = SLABS == 1 ? 8 : 16 / SLABS;   // rows at a time (float32 and 5 of them, 16 at a time: 6.3 us for 3.6)
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    for (int j0 = 0; j0 < n; j0 += N) {
        float4 v[N][SLABS];
        float w[N];
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const int j = j0 + u < n ? j0 + u : n - 1;   // past the last one: fetched again, not added
            const float* p = g.y + (size_t)g.row_of[t * n + j] * g.y_pitch + col;
            w[u] = j < g.k ? g.topk_w[t * g.k + j] : 1.0f;
#pragma unroll
            for (int i = 0; i < SLABS; ++i) v[u][i] = *reinterpret_cast<const float4*>(p + i * slab);
        }
#pragma unroll
        for (int u = 0; u < N; ++u) {
            if (j0 + u >= n) break;
            float4 a = v[u][0];
#pragma unroll
            for (int i = 1; i < SLABS; ++i)
                a = make_float4(a.x + v[u][i].x, a.y + v[u][i].y, a.z + v[u][i].z, a.w + v[u][i].w);
            s[0] = fmaf(w[u], a.x, s[0]);
            s[1] = fmaf(w[u], a.y, s[1]);
            s[2] = fmaf(w[u], a.z, s[2]);
            s[3] = fmaf(w[u], a.w, s[3]);
        }
    }
#pragma unroll
    for (int q = 0; q < 4; ++q)
        if (col + q < g.d) {
            const size_t at = (size_t)t * g.d + col + q;
            ((T*)g.out)[at] = from_float<T>(g.addend ? s[q] + to_float(((const T*)g.addend)[at]) : s[q]);
        }
}
template <typename T>
int launch_layer_sum(const LayerArgs& a, hipStream_t s) {
    const dim3 grid((unsigned)a.T, (unsigned)((a.d + 255) / 256));
#define XMOE_CALL(N) XMOE_LAUNCH(K_LAYER_SUM, s, hipLaunchKernelGGL((layer_sum_kernel<T, N>), grid, dim3(64), 0, s, a))
    if (a.slabs == 1) XMOE_CALL(1);
    else if (a.slabs == 2) XMOE_CALL(2);
    else XMOE_CALL(4);
#undef XMOE_CALL
    return XMOE_OK;
}

// ---------------------------------------------------------------------------------------------------------
// vector ALUs: float32, and bf16 widths that are no multiple of 8
// ---------------------------------------------------------------------------------------------------------
// Thread (k-group of 16, column group c of 16): four consecutive k of every 64 and EV columns (16 bytes; one where N is less
// than 16 bytes).  A column group that would pass N starts at N - EV instead: the columns it shares with its neighbour come
// out the same twice.
// Rows multiplied at a time (R): 4, or 8 for the experts with more where EV is 4 (float32: acc holds 2 x 8 x 4 values; bf16's
// EV = 8 would need 256 registers for it).
template <int EV>
constexpr int kAluRows = EV <= 4 ? 8 : 4;

template <typename T, int M, int EV, int R>
__device__ __forceinline__ void alu_tile(const T* x, size_t ldx, const int (&src)[R], int K, const T* w0, const T* w1, int N,
                                         int col, float (&acc)[M][R][EV]) {
    const int kg = threadIdx.x >> 4;
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int j = 0; j < EV; ++j) acc[m][r][j] = 0.f;
    const T* xr[R];
#pragma unroll
    for (int r = 0; r < R; ++r) xr[r] = x + (size_t)src[r] * ldx;
    auto step = [&](int k0, auto part) {   // k0 .. k0 + 3, part: those below K
        constexpr bool kPart = decltype(part)::value;
        LayerVec<T, EV> w[M][4];
        float a[R][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int k = kPart && k0 + i >= K ? K - 1 : k0 + i;
#pragma unroll
            for (int m = 0; m < M; ++m) {
                w[m][i] = *reinterpret_cast<const LayerVec<T, EV>*>((m == 0 ? w0 : w1) + (size_t)k * N + col);
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
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
                for (int r = 0; r < R; ++r)
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
template <typename T, int M, int EV, int R, class Source, class Result>
__device__ __forceinline__ void alu_rows(const T* x, size_t ldx, int rows, int K, const T* w0, const T* w1, int N, int n0,
                                            float* red, Source source, Result result) {
    constexpr int C = 16 * EV;
    const int c = threadIdx.x & 15, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    int col = n0 + c * EV;
    if (col + EV > N) col = N - EV;
    for (int r0 = 0; r0 < rows; r0 += R) {
        int src[R];
#pragma unroll
        for (int r = 0; r < R; ++r) src[r] = source(r0 + r < rows ? r0 + r : rows - 1);
        float acc[M][R][EV];
        alu_tile<T, M, EV, R>(x, ldx, src, K, w0, w1, N, col, acc);
        // the sixteen groups' sums: four of a wave, then the waves in order
#pragma unroll
        for (int m = 0; m < M; ++m)
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int j = 0; j < EV; ++j) {
                    float v = acc[m][r][j];
                    v += __shfl_xor(v, 16, 64);
                    v += __shfl_xor(v, 32, 64);
                    if (lane < 16) red[((wave * M + m) * R + r) * C + c * EV + j] = v;
                }
        __syncthreads();
        for (int i = threadIdx.x; i < R * C; i += 256) {
            const int r = i / C, cc = i - r * C;
            int at = n0 + cc / EV * EV;   // where the column group of this sum starts
            if (at + EV > N) at = N - EV;
            at += cc % EV;
            float v[2] = {0.f, 0.f};
#pragma unroll
            for (int m = 0; m < M; ++m)
#pragma unroll
                for (int w = 0; w < 4; ++w) v[m] += red[((w * M + m) * R + r) * C + cc];
            if (r0 + r < rows && at < N) result(r0 + r, at, v[0], v[1]);
        }
        __syncthreads();
    }
}
template <typename T, int M, int EV, class Source, class Result>
__device__ __forceinline__ void alu_product(const T* x, size_t ldx, int rows, int K, const T* w0, const T* w1, int N, int n0,
                                            float* red, Source source, Result result) {
    if (kAluRows<EV> > 4 && rows > 4)
        alu_rows<T, M, EV, kAluRows<EV>>(x, ldx, rows, K, w0, w1, N, n0, red, source, result);
    else
        alu_rows<T, M, EV, 4>(x, ldx, rows, K, w0, w1, N, n0, red, source, result);
}

template <typename T, int EV>
__global__ __launch_bounds__(256) void layer_up_alu_kernel(LayerArgs g) {
    constexpr int C = 16 * EV;
    __shared__ float red[4 * 2 * kAluRows<EV> * C];
    __shared__ LayerPlan pl;
    layer_plan(pl, g);
    if (blockIdx.x == 0) layer_rows(pl, g);
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
    __shared__ float red[4 * kAluRows<EV> * C];
    __shared__ LayerPlan pl;
    layer_plan(pl, g);
    const int nt = (g.d + C - 1) / C, i = blockIdx.x / nt, tile = blockIdx.x - i * nt;
    if (i >= pl.n) return;
    const int e = pl.list[i], rows = __popc(pl.mask[e]), row0 = pl.row0[e];
    alu_product<T, 1, EV>((const T*)g.act, g.f, rows, g.f, (const T*)g.wd + (size_t)e * g.f * g.d, (const T*)nullptr, g.d,
                            tile * C, red, [&](int r) { return row0 + r; },
                            [&](int r, int c, float v, float) { g.y[(size_t)(row0 + r) * g.y_pitch + c] = v; });
}

template <typename T>
int launch_alu(const LayerArgs& a, int active, hipStream_t s) {
    constexpr int EV = 16 / (int)sizeof(T);
    const int cu = a.f < EV ? 16 : 16 * EV, cd = a.d < EV ? 16 : 16 * EV, up = (a.f + cu - 1) / cu, down = (a.d + cd - 1) / cd;
    const dim3 g1((unsigned)(active * up)), g2((unsigned)(active * down));
    if (a.f < EV)
        XMOE_LAUNCH(K_LAYER_UP_ALU, s, hipLaunchKernelGGL((layer_up_alu_kernel<T, 1>), g1, dim3(256), 0, s, a));
    else
        XMOE_LAUNCH(K_LAYER_UP_ALU, s, hipLaunchKernelGGL((layer_up_alu_kernel<T, EV>), g1, dim3(256), 0, s, a));
    if (a.d < EV)
        XMOE_LAUNCH(K_LAYER_DOWN_ALU, s, hipLaunchKernelGGL((layer_down_alu_kernel<T, 1>), g2, dim3(256), 0, s, a));
    else
        XMOE_LAUNCH(K_LAYER_DOWN_ALU, s, hipLaunchKernelGGL((layer_down_alu_kernel<T, EV>), g2, dim3(256), 0, s, a));
    return launch_layer_sum<T>(a, s);
}

template <typename T>
int launch_layer_route(const LayerArgs& a, hipStream_t s) {
    constexpr int EV = 16 / (int)sizeof(T);
    if (a.E % EV == 0 && aligned16(a.w_router))
        XMOE_LAUNCH(K_LAYER_ROUTE, s, hipLaunchKernelGGL((layer_route_kernel<T, EV>), dim3((unsigned)a.T), dim3(512), 0, s, a));
    else
        XMOE_LAUNCH(K_LAYER_ROUTE, s, hipLaunchKernelGGL((layer_route_kernel<T, 1>), dim3((unsigned)a.T), dim3(512), 0, s, a));
    return XMOE_OK;
}

// A block per token reads the whole router through one CU: up to this many bytes of it.  The whole call, us, so | by
// xmoe_gate_logits and xmoe_route: 256 KiB (d 2048, 64 experts) 1 token 27.8|28.8, 8 tokens 31.1|30.9, 32 tokens 39.9|40.5;
// 512 KiB (d 2048, 128 experts) 33.5|29.1 and 63.2|58.2 for 1 and 32, (d 4096, 64) 41.6|41.5 and 72.4|73.0; 1 MiB 50.5|41.6.
constexpr size_t kRouteBytes = 256 << 10;
// From this many tiles of 128 columns on, up takes them (rows of 256 bytes of either matrix) instead of 64.  The whole call, us,
// 128 | 64 columns, d 2048, f 1408: 88 tiles 55.5|48.7, 154 65.4|71.1, 286 97.9|96.8, 550 137|143, 726 189|184; d 4096, f 14336:
// 224 tiles 148|160, 896 326|337; d 4096, f 1024: 264 tiles 134|148; d 1024, f 512: 64 tiles 28.1|24.0, 256 50.5|54.8.  (At 286
// and 726 tiles 64 columns are 1 and 3 % better: no line in the number of tiles tells those from their neighbours.)
constexpr long kWideTiles = 128;

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
    a.slabs = 1;
    a.y_pitch = layer_few_y_pitch(d);
    char* p = (char*)ws;
    a.row_of = (int32_t*)p;
    p += align_up(rows * sizeof(int32_t), 256);
    a.act = p;
    p += align_up(rows * f * dtype_size(dt), 256);
    a.y = (float*)p;
    int st;
    if (E <= kRouteExperts && (size_t)d * E * dtype_size(dt) <= kRouteBytes) {
        st = dt == XMOE_F32 ? launch_layer_route<float>(a, s) : launch_layer_route<bf16_t>(a, s);
    } else {
        st = xmoe_gate_logits(x, w_router, bias, logits, T, d, E, dt, stream);
        if (st == XMOE_OK) st = xmoe_route(logits, T, E, k, topk_idx, topk_w, stream);
    }
    if (st != XMOE_OK) return st;
    const int active = (T * k < E ? T * k : E) + E_s;
    if (dt == XMOE_F32) return launch_alu<float>(a, active, s);
    if (d % 8 || f % 8 || !aligned16(x) || !aligned16(wg) || !aligned16(wu) || !aligned16(wd))
        return launch_alu<bf16_t>(a, active, s);
    // slabs of at least 8 stages until a token's experts alone give two blocks to every CU (the number of tokens has no say:
    // a token's bits are the same in every call)
    int down = (d + kDownCols - 1) / kDownCols;
    while (a.slabs < kLayerSlabs && (k + E_s) * down * a.slabs < 512 && f >= 16 * kDownK * a.slabs) a.slabs *= 2;
    down *= a.slabs;
    if ((long)active * ((f + 127) / 128) >= kWideTiles)
        XMOE_LAUNCH(K_LAYER_UP_FEW, s, hipLaunchKernelGGL((layer_up_few_kernel<256, 32, 4>), dim3((unsigned)(active * ((f + 127) / 128))),
                                                          dim3(256), 0, s, a));
    else
        XMOE_LAUNCH(K_LAYER_UP_FEW, s, hipLaunchKernelGGL((layer_up_few_kernel<128, 64, 3>), dim3((unsigned)(active * ((f + 63) / 64))),
                                                          dim3(256), 0, s, a));
    XMOE_LAUNCH(K_LAYER_DOWN_FEW, s, hipLaunchKernelGGL(layer_down_few_kernel, dim3((unsigned)(active * down)), dim3(256), 0, s, a));
    return launch_layer_sum<bf16_t>(a, s);
}
