// Softmax and top-k of one token's logits by one wave (xmoe_route; xmoe_layer_few.hip routes its tokens itself).
#pragma once

#include <type_traits>

#include "xmoe_internal.h"

namespace xmoe {

constexpr int kMaxPerLane = XMOE_MAX_EXPERTS / 64;   // 8

// order-preserving bit pattern of a float; -0.0 and +0.0 compare equal as numbers, so both map to +0.0's key and
// the lower expert index decides between them like any other tie
__device__ __forceinline__ uint32_t order_key(float v) {
    uint32_t u = __float_as_uint(v);
    if (u == 0x80000000u) u = 0u;
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) v = fmaxf(v, __shfl_xor(v, off, 64));
    return v;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off, 64);
    return v;
}
// the largest of the wave's values, wave-uniform: lane moves of the vector ALU, which cost no LDS traffic
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
    auto step = [&](auto ctrl, auto rows) {
        const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, decltype(rows)::value, 0xf,
                                                                 false);
        v = o > v ? o : v;
    };
    typedef std::integral_constant<int, 0xf> all;
    step(std::integral_constant<int, 0x111>{}, all{});   // row_shr 1, 2, 4, 8: lane 15 of a row holds the row's maximum
    step(std::integral_constant<int, 0x112>{}, all{});
    step(std::integral_constant<int, 0x114>{}, all{});
    step(std::integral_constant<int, 0x118>{}, all{});
    step(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});   // row_bcast 15 into rows 1 and 3
    step(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});   // row_bcast 31 into rows 2 and 3
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

// Lane j < k receives slot j: the expert of the j-th largest of the E logits at `row` (the lower index among equals) and its
// probability.  E <= 64 PER_LANE, k <= 64.
template <int PER_LANE>
__device__ __forceinline__ void route_token(const float* row, int E, int k, int& my_idx, float& my_w) {
    const int lane = threadIdx.x & 63;
    float l[PER_LANE];
    // order-preserving bits of the logits; 0 stands for a column that does not exist or has been selected, and is the key of
    // one logit, the NaN of all ones.  The largest key wins, and among equal ones the lowest expert, i.e. the first lane of
    // the first j.
    uint32_t key[PER_LANE];
#pragma unroll
    for (int j = 0; j < PER_LANE; ++j) {
        const int e = lane + 64 * j;
        l[j] = e < E ? row[e] : -INFINITY;
        key[j] = e < E ? order_key(l[j]) : 0u;
    }
    auto wave_best = [&] {
        uint32_t best = 0u;
#pragma unroll
        for (int j = 0; j < PER_LANE; ++j) best = key[j] > best ? key[j] : best;
        return wave_max_u32(best);
    };
    auto logit_of = [](uint32_t ob) { return __uint_as_float((ob & 0x80000000u) ? (ob & 0x7fffffffu) : ~ob); };
    uint32_t best = wave_best();
    const float m = logit_of(best);
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < PER_LANE; ++j) s += (lane + 64 * j < E) ? expf(l[j] - m) : 0.f;
    s = wave_sum(s);
    const float inv = 1.0f / s;

    my_idx = 0;
    my_w = 0.f;
    int slot = 0;
    for (; slot < k; ++slot) {
        if (best == 0u) break;   // wave-uniform, as `best` is
        int e = 0;
        bool found = false;
#pragma unroll
        for (int j = 0; j < PER_LANE; ++j) {
            const unsigned long long who = __ballot(key[j] == best);
            if (!found && who) {   // wave-uniform
                found = true;
                const int winner = __ffsll((long long)who) - 1;
                e = winner + 64 * j;
                if (lane == winner) key[j] = 0u;   // retired
            }
        }
        if (lane == slot) {
            my_idx = e;
            my_w = expf(logit_of(best) - m) * inv;
        }
        if (slot + 1 < k) best = wave_best();
    }
    // only NaNs of all ones are left: by ascending expert
    for (int last = -1; slot < k; ++slot) {
        int e = E;
#pragma unroll
        for (int j = PER_LANE - 1; j >= 0; --j) {
            const unsigned long long who = __ballot(__float_as_uint(l[j]) == 0xffffffffu && lane + 64 * j > last);
            if (who) e = __ffsll((long long)who) - 1 + 64 * j;
        }
        last = e;
        if (lane == slot) {
            my_idx = e;
            my_w = logit_of(0u);
        }
    }
}

}  // namespace xmoe
