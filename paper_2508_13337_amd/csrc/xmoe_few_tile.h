// The ring of direct-to-LDS stages behind the products of experts with few rows (bf16): a block of 4 waves multiplies up to
// 64 rows with 128 columns (gate/up: the same 64 columns of two matrices), 32 k to a stage.  Used by xmoe_ffn_few.hip and
// xmoe_layer_few.hip.
#pragma once

#include "xmoe_ffn.h"

namespace xmoe {

typedef __attribute__((ext_vector_type(8))) __bf16 few_bf16x8_t;
typedef __attribute__((ext_vector_type(16))) float few_f32x16_t;
typedef __attribute__((ext_vector_type(4))) short few_s16x4_t;
typedef __attribute__((ext_vector_type(8))) short few_s16x8_t;

constexpr int kFewRows = 64, kFewCols = 128, kFewK = 32, kFewStages = 6;
constexpr int kFewWBytes = kFewK * kFewCols * 2;              // [32 k][128 columns]
constexpr int kFewStageBytes = kFewWBytes + kFewRows * kFewK * 2;   // and [64 rows][32 k]
constexpr int kFewLoads = 3;                                  // per wave and stage: two of weights, one of rows
static __device__ __align__(16) const unsigned int kFewZero[4] = {0u, 0u, 0u, 0u};

// what becomes of a product
enum FewMode { FEW_PLAIN = 0, FEW_GATEUP = 1, FEW_MLP2 = 2 };

__device__ __forceinline__ void few_load16(const bf16_t* p, char* lds) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)p,
                                     (__attribute__((address_space(3))) void*)lds, 16, 0, 0);
}

// A lane's share of the loads: 16 bytes of k-rows kr and kr + 4 of the weights and of one row of X per stage.
struct FewLoader {
    const bf16_t *w[2], *x;   // of the stage issued next
    size_t step;              // elements between the weights of two stages
    int left;                 // stages of K not yet issued; behind them the block of zeros, so that the counts stay uniform
    __device__ __forceinline__ void issue(char* __restrict__ stage) {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const bool in = left > 0;
        const bf16_t* z = reinterpret_cast<const bf16_t*>(kFewZero);
        few_load16(in ? w[0] : z, stage + wave * 2048);
        few_load16(in ? w[1] : z, stage + wave * 2048 + 1024);
        few_load16(in ? x : z, stage + kFewWBytes + wave * 1024);
        w[0] += step;
        w[1] += step;
        x += kFewK;
        --left;
    }
};

// LDS layout: k-rows of 256 bytes whose 16-byte pieces are XOR-swizzled with 4 * (k-row % 4), rows of X of 64 bytes with
// pieces XOR-swizzled with (row / 4) % 4: the fragment reads fall on all banks.
// Columns of the wave, 8 k (16 ks + 8 (lane/32) ..): in a group of 16 lanes, lane s addresses 4 consecutive columns (s%4)
// of k-row s/4, and the transposing read hands every lane one column with 4 consecutive k.
template <int MODE>
__device__ __forceinline__ few_bf16x8_t few_frag_w(const char* stage, int ks) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, G = lane >> 4, s = lane & 15;
    const int col = (MODE == FEW_GATEUP ? 64 * (G & 1) + 16 * wave : 32 * wave + 16 * (G & 1)) + 4 * (s & 3);
    few_s16x4_t h[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const int kr = 16 * ks + 8 * (G >> 1) + (s >> 2) + 4 * q;
        const char* a = stage + kr * 256 + (((col >> 3) ^ ((kr & 3) << 2)) << 4) + (col & 7) * 2;
        h[q] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) few_s16x4_t*)(
            (__attribute__((address_space(3))) void*)a));
    }
    const few_s16x8_t v = {h[0][0], h[0][1], h[0][2], h[0][3], h[1][0], h[1][1], h[1][2], h[1][3]};
    return __builtin_bit_cast(few_bf16x8_t, v);
}
__device__ __forceinline__ few_bf16x8_t few_frag_x(const char* stage, int mb, int ks) {
    const int lane = threadIdx.x & 63, r = mb * 32 + (lane & 31), c = 2 * ks + (lane >> 5);
    return *reinterpret_cast<const few_bf16x8_t*>(stage + kFewWBytes + r * 64 + ((c ^ ((r >> 2) & 3)) << 4));
}

// Refills the stage read before the last barrier and multiplies `cur`.  The two are distinct, and saying so matters: an
// LDS read that may observe a direct-to-LDS load in flight makes the compiler wait for all of them.
template <int MODE, int MB>
__device__ __forceinline__ void few_step(few_f32x16_t (&acc)[MB], FewLoader& ld, char* __restrict__ next,
                                         const char* __restrict__ cur) {
    ld.issue(next);
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
        const few_bf16x8_t w = few_frag_w<MODE>(cur, ks);
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
            acc[mb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(w, few_frag_x(cur, mb, ks), acc[mb], 0, 0, 0);
    }
}

// acc = the product over n stages of the block's rows (32 MB of them) and columns.  Every thread of the block calls it.
// acc[mb], register v of lane l: row 32 mb + l % 32, column 8 (v/4) + 4 (l/32) + v%4 of the wave's 32 (GATEUP: 16 gate, then
// 16 up)
template <int MODE, int MB>
__device__ __forceinline__ void few_loop(few_f32x16_t (&acc)[MB], FewLoader& ld, char* smem, int n) {
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[mb][v] = 0.f;
#pragma unroll
    for (int s = 0; s < kFewStages - 1; ++s) ld.issue(smem + s * kFewStageBytes);
    int cur = 0, next = kFewStages - 1;
    for (int i = 0; i < n; ++i) {
        // stage i has landed for every thread, and every wave is done with stage i - 1, which is refilled now
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(kFewLoads * (kFewStages - 2)) : "memory");
        few_step<MODE, MB>(acc, ld, smem + next * kFewStageBytes, smem + cur * kFewStageBytes);
        next = cur;
        cur = cur + 1 < kFewStages ? cur + 1 : 0;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // nothing may land in this LDS once the block has left it
}

}  // namespace xmoe
