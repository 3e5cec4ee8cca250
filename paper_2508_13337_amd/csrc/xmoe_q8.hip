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
// A row's scale is known when all columns of A are.  The product therefore leaves A as 16-bit integers relative to the
// maximum of every 32 columns (half a step: 2^-16 of that maximum, 1/500 of a step of the 8 bits that follow) with those
// maxima in float32, and a pass over them (q8_rows_kernel) makes the 8-bit rows: the row's maximum is the largest of the 32-column
// ones, so this pass reads A once, at half of float32's bytes.
#include "xmoe_ffn.h"

namespace xmoe {
namespace {

typedef __attribute__((ext_vector_type(4))) int q8_i32x4_t;
typedef __attribute__((ext_vector_type(16))) int q8_i32x16_t;

constexpr int kQ8Group = 32;       // columns of A that share a 16-bit scale
constexpr float kQ8Tiny = 0x1p-112f;   // a maximum below counts as zero: 32767 / it would overflow
constexpr uint32_t kQ8TinyBits = (127 - 112) << 23;

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

// A lane's pieces of the wave's share of an operand unit ([rows][128 bytes of k]): 8 rows per load, piece (lane % 8) XOR-ed
// with (row / 2) % 8, so that a fragment read falls on all banks.  Units are requested in order; behind the last one of K
// that one is fetched again, which keeps the wait counts uniform, and not used.
template <int LOADS>
struct Q8Rows {
    const int8_t* p[LOADS];
    // row r of the operand is at base + source(r) * pitch
    template <class Source>
    __device__ __forceinline__ void init(const int8_t* base, size_t pitch, int first, Source source) {
        const int lane = threadIdx.x & 63;
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
template <int MI>
struct Q8Frags {
    q8_i32x4_t a[MI], b[2];
};
template <int MI>
__device__ __forceinline__ void q8_mma(q8_i32x16_t (&acc)[MI][2], const Q8Frags<MI>& f) {
#pragma unroll
    for (int mi = 0; mi < MI; ++mi)
#pragma unroll
        for (int ni = 0; ni < 2; ++ni)
            acc[mi][ni] = __builtin_amdgcn_mfma_i32_32x32x32_i8(f.b[ni], f.a[mi], acc[mi][ni], 0, 0, 0);
}

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
__device__ __forceinline__ int q8_round16(float v, float inv) {
    return (int)rintf(fminf(fmaxf(v * inv, -32767.f), 32767.f));
}

// A row's 32 columns of gate and up sums (this lane: 16 of them) -> 16-bit integers, packed in the order of the registers'
// column quadruples, and the maximum of all 32.  gs, us: the columns' scales
__device__ __forceinline__ float q8_activation(const q8_i32x16_t& g, const q8_i32x16_t& u, float xs,
                                               const float (&gs)[4][4], const float (&us)[4][4], uint2 (&out)[4]) {
    float a[16];
    uint32_t mx = 0u;
#pragma unroll
    for (int v = 0; v < 16; ++v) {
        const float gv = (float)g[v] * (xs * gs[v / 4][v % 4]), uv = (float)u[v] * (xs * us[v / 4][v % 4]);
        a[v] = gv * fast_sigmoid(gv) * uv;
        const uint32_t b = __float_as_uint(a[v]) & 0x7fffffffu;   // ordered as the numbers are, a NaN above them all
        mx = b > mx ? b : mx;
    }
    const uint32_t o = (uint32_t)__shfl_xor((int)mx, 32, 64);
    mx = o > mx ? o : mx;
    const float m = __uint_as_float(mx), inv = mx < kQ8TinyBits ? 0.f : 32767.f * __builtin_amdgcn_rcpf(m);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        uint32_t w[2];
#pragma unroll
        for (int i = 0; i < 2; ++i)
            w[i] = ((uint32_t)q8_round16(a[4 * q + 2 * i], inv) & 0xffffu) |
                   ((uint32_t)q8_round16(a[4 * q + 2 * i + 1], inv) << 16);
        out[q] = make_uint2(w[0], w[1]);
    }
    return m;
}

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

struct Q8Args {
    const int8_t* x;            // rows, pitch bytes each
    const float* x_scale;       // of a row
    const int32_t* row_index;   // or NULL
    const int32_t *off, *map;
    const int8_t *w0, *w1;      // [E, N, pitch]; w1: up
    const float *s0, *s1;       // [E, N]
    int pitch, N;
    int16_t* a16;               // gate/up: [rows][a_pitch]
    float* gmax;                // [rows][a_pitch / 32]
    int a_pitch;
    void* y;                    // down: [rows][N]
};

// The block's tile: row tiles x column tiles, column tiles of a row tile in a run, the runs dealt to the XCDs in eight parts
// of equal length (workgroup L goes to XCD L % 8): the tiles of an expert share their weights and rows in one L2.
struct Q8Tile {
    int e, row0, rows, n0;
    __device__ __forceinline__ bool place(const Q8Args& a, int cols) {
        const int nt = (a.N + cols - 1) / cols;
        const long total = (long)a.map[0] * nt, run = (total + 7) / 8, slot = blockIdx.x >> 3, t = (blockIdx.x & 7) * run + slot;
        if (slot >= run || t >= total) return false;
        const int tile = (int)(t / nt);
        n0 = (int)(t - (long)tile * nt) * cols;
        e = a.map[4 + 2 * tile];
        row0 = a.map[4 + 2 * tile + 1];
        rows = a.off[e + 1] - row0;
        return true;
    }
};

// =========================================================================================================
// Many rows: 256 x 256 tiles (gate/up: the same 128 columns of both), 8 waves (2 x 4) of 128 x 64 each, one block per CU.
// Units A(0) B(0) A(1) B(1) .. of 256 rows x 128 k run through five slots of 32 KiB, two to three of them on their way.
// =========================================================================================================
constexpr int kBigUnit = 256 * 128, kBigLds = 5 * kBigUnit;

template <bool DUAL>
__device__ __forceinline__ int big_col(int ni) {
    const int wn = (threadIdx.x >> 6) & 3;
    return DUAL ? ni * 128 + wn * 32 : wn * 64 + ni * 32;
}
template <bool DUAL>
__device__ __forceinline__ void big_read(Q8Frags<4>& f, const char* ua, const char* ub, int ks) {
    const int wm = threadIdx.x >> 8;
#pragma unroll
    for (int ni = 0; ni < 2; ++ni) f.b[ni] = q8_frag(ub, big_col<DUAL>(ni), ks);
#pragma unroll
    for (int mi = 0; mi < 4; ++mi) f.a[mi] = q8_frag(ua, wm * 128 + mi * 32, ks);
}
// One pass: the four steps on A(p) = ua, B(p) = ub.  On entry both have landed, every wave has left the units of pass p - 1
// (fill1, fill2), and f1 holds that pass's last step.  The slots are distinct, and saying so matters: an LDS read that may
// observe a direct-to-LDS load in flight makes the compiler wait for all of them.
template <bool DUAL>
__device__ __forceinline__ void big_pass(q8_i32x16_t (&acc)[4][2], Q8Frags<4>& f0, Q8Frags<4>& f1, Q8Rows<4>& a,
                                         Q8Rows<4>& b, bool more_a, bool more_b, char* __restrict__ fill1,
                                         char* __restrict__ fill2, const char* __restrict__ ua,
                                         const char* __restrict__ ub) {
    const int first = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * 32;
    b.issue(fill1, first, more_b);       // B(p+1)
    __builtin_amdgcn_sched_barrier(0);   // the requests stay where they stand: sunk to the end of the pass they are late
    big_read<DUAL>(f0, ua, ub, 0);
    q8_mma<4>(acc, f1);
    big_read<DUAL>(f1, ua, ub, 1);
    q8_mma<4>(acc, f0);
    __builtin_amdgcn_sched_barrier(0);
    a.issue(fill2, first, more_a);       // A(p+2)
    __builtin_amdgcn_sched_barrier(0);
    big_read<DUAL>(f0, ua, ub, 2);
    q8_mma<4>(acc, f1);
    big_read<DUAL>(f1, ua, ub, 3);
    q8_mma<4>(acc, f0);
}
template <bool DUAL>
__device__ __forceinline__ void big_mainloop(q8_i32x16_t (&acc)[4][2], Q8Rows<4>& a, Q8Rows<4>& b, int np, char* smem) {
    const int first = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * 32;
    const q8_i32x4_t z = {0, 0, 0, 0};
    Q8Frags<4> f0, f1;
#pragma unroll
    for (int mi = 0; mi < 4; ++mi) {
        f1.a[mi] = z;
        f1.b[mi & 1] = z;
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[mi][0][v] = acc[mi][1][v] = 0;
    }
    a.issue(smem, first, np > 1);
    b.issue(smem + kBigUnit, first, np > 1);
    a.issue(smem + 2 * kBigUnit, first, np > 2);
    // at the top of pass p everything up to B(p) has landed for every thread, A(p+1) may be on its way
    q8_wait_and_barrier<4>();
    int sa = 0;   // slot of A(p) = 2p % 5
    for (int p = 0; p < np; ++p) {
        const int sb = sa + 1 < 5 ? sa + 1 : sa - 4, s3 = sa + 3 < 5 ? sa + 3 : sa - 2, s4 = sa + 4 < 5 ? sa + 4 : sa - 1;
        big_pass<DUAL>(acc, f0, f1, a, b, p + 3 < np, p + 2 < np, smem + s3 * kBigUnit, smem + s4 * kBigUnit,
                       smem + sa * kBigUnit, smem + sb * kBigUnit);
        q8_wait_and_barrier<4>();
        sa = sa + 2 < 5 ? sa + 2 : sa - 3;
    }
    q8_mma<4>(acc, f1);
    q8_wait_and_barrier<0>();   // nothing may land in this LDS any more: it becomes the results'
}

__global__ __launch_bounds__(512) void q8_gateup_kernel(Q8Args g) {
    __shared__ __align__(16) char smem[kBigLds];
    Q8Tile t;
    if (!t.place(g, 128)) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave >> 2, wn = wave & 3;
    Q8Rows<4> a, b;
    a.init(g.x, g.pitch, wave * 32, [&](int r) {
        r = t.row0 + (r < t.rows ? r : t.rows - 1);   // rows past the last one repeat it; what they give is not stored
        return g.row_index ? g.row_index[r] : r;
    });
    b.init(wave < 4 ? g.w0 : g.w1, g.pitch, wave * 32, [&](int r) {
        const int n = t.n0 + (r & 127);
        return (size_t)t.e * g.N + (n < g.N ? n : g.N - 1);
    });
    q8_i32x16_t acc[4][2];
    big_mainloop<true>(acc, a, b, g.pitch / 128, smem);
    float gs[4][4], us[4][4];
    const int c0 = t.n0 + wn * 32 + 4 * (lane >> 5);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        q8_scales(g.s0 + (size_t)t.e * g.N, c0 + 8 * q, g.N, gs[q]);
        q8_scales(g.s1 + (size_t)t.e * g.N, c0 + 8 * q, g.N, us[q]);
    }
    // results: rows of 128 columns, 16-byte pieces XOR-ed with the row
#pragma unroll
    for (int mi = 0; mi < 4; ++mi) {
        const int r = wm * 128 + mi * 32 + (lane & 31), row = t.row0 + (r < t.rows ? r : t.rows - 1);
        const float xs = g.x_scale[g.row_index ? g.row_index[row] : row];
        uint2 o[4];
        const float m = q8_activation(acc[mi][0], acc[mi][1], xs, gs, us, o);
        if (lane < 32 && r < t.rows) g.gmax[(size_t)row * (g.a_pitch / kQ8Group) + (t.n0 / kQ8Group + wn)] = m;
#pragma unroll
        for (int q = 0; q < 4; ++q)
            *reinterpret_cast<uint2*>(smem + r * 256 + (((wn * 4 + q) ^ (r & 15)) << 4) + 8 * (lane >> 5)) = o[q];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = i * 32 + (threadIdx.x >> 4), c = threadIdx.x & 15;
        const uint4 v = *reinterpret_cast<const uint4*>(smem + r * 256 + ((c ^ (r & 15)) << 4));
        if (r < t.rows) *reinterpret_cast<uint4*>(g.a16 + (size_t)(t.row0 + r) * g.a_pitch + t.n0 + 8 * c) = v;
    }
}

template <typename T>
__global__ __launch_bounds__(512) void q8_down_kernel(Q8Args g) {
    __shared__ __align__(16) char smem[kBigLds];
    Q8Tile t;
    if (!t.place(g, 256)) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave >> 2, wn = wave & 3;
    Q8Rows<4> a, b;
    a.init(g.x, g.pitch, wave * 32, [&](int r) { return t.row0 + (r < t.rows ? r : t.rows - 1); });
    b.init(g.w0, g.pitch, wave * 32, [&](int r) {
        const int n = t.n0 + r;
        return (size_t)t.e * g.N + (n < g.N ? n : g.N - 1);
    });
    q8_i32x16_t acc[4][2];
    big_mainloop<false>(acc, a, b, g.pitch / 128, smem);
    float as[4];
#pragma unroll
    for (int mi = 0; mi < 4; ++mi) {
        const int r = wm * 128 + mi * 32 + (lane & 31);
        as[mi] = g.x_scale[t.row0 + (r < t.rows ? r : t.rows - 1)];
    }
#pragma unroll
    for (int ni = 0; ni < 2; ++ni)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int col = wn * 64 + ni * 32 + 8 * q + 4 * (lane >> 5);
            float s[4];
            q8_scales(g.s0 + (size_t)t.e * g.N, t.n0 + col, g.N, s);
#pragma unroll
            for (int mi = 0; mi < 4; ++mi) {
                const int r = wm * 128 + mi * 32 + (lane & 31);
                float o[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) o[i] = (float)acc[mi][ni][4 * q + i] * (as[mi] * s[i]);
                if (sizeof(T) == 4) {
                    if (r < t.rows) q8_store4((float*)g.y + (size_t)(t.row0 + r) * g.N, t.n0 + col, g.N, o);
                } else {   // rows of 256 columns, 16-byte pieces XOR-ed with the row
                    *reinterpret_cast<uint2*>(smem + r * 512 + (((wn * 8 + ni * 4 + q) ^ (r & 31)) << 4) + 8 * (lane >> 5)) =
                        make_uint2(pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3]));
                }
            }
        }
    if (sizeof(T) == 4) return;
    __syncthreads();
#pragma unroll 4
    for (int i = 0; i < 16; ++i) {
        const int r = i * 16 + (threadIdx.x >> 5), c = threadIdx.x & 31;
        const uint4 v = *reinterpret_cast<const uint4*>(smem + r * 512 + ((c ^ (r & 31)) << 4));
        if (r < t.rows) q8_store8((bf16_t*)g.y + (size_t)(t.row0 + r) * g.N, t.n0 + 8 * c, g.N, v);
    }
}

// =========================================================================================================
// A's 8-bit rows: one wave per row.  HBM-bound.
// =========================================================================================================
__global__ __launch_bounds__(256) void q8_rows_kernel(const int16_t* __restrict__ a16, const float* __restrict__ gmax,
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
    const float m = __uint_as_float(mx), inv = mx < kQ8TinyBits ? 0.f : 127.f / m;
    if (lane == 0) as[row] = mx < kQ8TinyBits ? 0.f : m / 127.f;
    const int16_t* src = a16 + (size_t)row * pitch;
    int8_t* dst = aq + (size_t)row * pitch;
    for (int c = lane; c < pitch / 8; c += 64) {
        uint2 o = make_uint2(0u, 0u);
        if (8 * c < f) {   // columns past f are zeros already, whole pieces of them were not written
            const uint4 v = *reinterpret_cast<const uint4*>(src + 8 * c);
            const float k = gm[c / 4] * inv * (1.0f / 32767.f);
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
            uint32_t p[2] = {0u, 0u};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float a = (float)(int16_t)(w[i / 2] >> (16 * (i & 1))) * k;
                p[i / 4] |= ((uint32_t)(int)rintf(fminf(fmaxf(a, -127.f), 127.f)) & 0xffu) << (8 * (i & 3));
            }
            o = make_uint2(p[0], p[1]);
        }
        *reinterpret_cast<uint2*>(dst + 8 * c) = o;
    }
}

// =========================================================================================================
// Weights [K, N] ("in x out") of an expert -> [N, pitch] integers and one scale per column.  Done once for a model's weights:
// a block owns 64 columns, reads them twice (maximum, then integers) and turns 64 x 64 pieces over in LDS.
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

long q8_blocks(int N, int cols, int max_tiles) { return ((long)max_tiles * ((N + cols - 1) / cols) + 7) / 8 * 8; }

}  // namespace
}  // namespace xmoe

using namespace xmoe;

extern "C" {

int xmoe_quantize_weights(const void* w, int E, int K, int N, int dt, void* wq, float* scale, void* stream) {
    if (!dtype_ok(dt)) return XMOE_ERR_UNSUPPORTED;
    if (E < 1 || K < 1 || N < 1) return XMOE_ERR_INVALID_ARG;
    if (E > 65535 || K > XMOE_MAX_Q8_WIDTH || N > (1 << 30)) return XMOE_ERR_UNSUPPORTED;
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
    p += ffn_tilemap_bytes(B, E);
    int16_t* a16 = (int16_t*)p;
    p += align_up((size_t)B * fp * 2, 256);
    float* gmax = (float*)p;
    p += align_up((size_t)B * (fp / kQ8Group) * 4, 256);
    int8_t* aq = (int8_t*)p;
    p += align_up((size_t)B * fp, 256);
    float* as = (float*)p;
    hipStream_t s = (hipStream_t)stream;
    const int tile_rows = 256, max_tiles = ffn_max_tiles(B, E, tile_rows);
    const long up_blocks = q8_blocks(f, 128, max_tiles), down_blocks = q8_blocks(d, 256, max_tiles);
    if ((up_blocks > down_blocks ? up_blocks : down_blocks) * 512 >= (1l << 32)) return XMOE_ERR_UNSUPPORTED;   // a grid's threads
    int st = launch_tile_map(expert_offsets, E, tile_rows, max_tiles, map, map + ffn_sched_offset(B, E), false, s);
    if (st != XMOE_OK) return st;
    const Q8Args up = {(const int8_t*)xq, x_scale, row_index, expert_offsets, map, (const int8_t*)wgq, (const int8_t*)wuq,
                       g_scale, u_scale, dp, f, a16, gmax, fp, nullptr};
    const Q8Args down = {aq, as, nullptr, expert_offsets, map, (const int8_t*)wdq, nullptr, d_scale, nullptr, fp, d, nullptr,
                         nullptr, 0, y};
    XMOE_LAUNCH(K_Q8_GATEUP, s,
                hipLaunchKernelGGL(q8_gateup_kernel, dim3((unsigned)up_blocks), dim3(512), 0, s, up));
    XMOE_LAUNCH(K_Q8_ROWS, s,
                hipLaunchKernelGGL(q8_rows_kernel, dim3((unsigned)((B + 3) / 4)), dim3(256), 0, s, a16, gmax, expert_offsets,
                                   E, f, fp, aq, as));
    if (dt == XMOE_F32)
        XMOE_LAUNCH(K_Q8_DOWN, s,
                    hipLaunchKernelGGL(q8_down_kernel<float>, dim3((unsigned)down_blocks), dim3(512), 0, s, down));
    else
        XMOE_LAUNCH(K_Q8_DOWN, s,
                    hipLaunchKernelGGL(q8_down_kernel<bf16_t>, dim3((unsigned)down_blocks), dim3(512), 0, s, down));
    return XMOE_OK;
}

}  // extern "C"
