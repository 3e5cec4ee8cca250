// Root-mean-square norm in front of the MoE layer: the residual's addition, the norm, its output in the storage type or as
// 8-bit rows, and the backward.
//
//   h = round(x + residual);  r = 1 / sqrt(mean_i h_i^2 + eps);  y = round(h r gain)
//   8-bit rows: q_i = rint(h_i gain_i * 127 / m), m = max_i |h_i gain_i|, and scale = m r / 127.  The factor r scales a row
//   and its maximum alike, so the integers follow from products and a maximum, which are the same in any order.
//   backward, n = h r and v = dy gain:  dx_i = r (v_i - n_i mean_j v_j n_j) + dh_i,   dgain_i = sum_t dy_ti n_ti
//
// HBM-bound: a row is read once and lives in registers from the first load to the last store.  TPR threads share a row
// (64: four rows per block and no barrier; 256, 1024: sums over the waves through LDS), each with NV vectors of 16 bytes,
// thread t on the vectors t, t + TPR, ...  Rows whose width is no multiple of a vector are read and written by the same
// vectors from addresses aligned to one element, and the last one element by element.
// Sums are float32: of a thread's elements in ascending order, then by halving over the wave, then over the waves in
// order; dgain over a block's rows in order, then over the blocks' partial rows.  Nothing depends on which block is first, and
// a row's bits not on the number of rows, by which the threads of a row are chosen up to 256 vectors: 64 vectors are a sum of
// their own whether one wave has all of them or four have 64 each.
#include "xmoe_internal.h"
#include "xmoe_sizes.h"

namespace xmoe {
namespace {

template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) NormVec {
    uint32_t v[4];
};
struct __attribute__((packed, aligned(4))) NormF4 {
    float v[4];
};

// elements [i, i + N) of a row as floats; those past d are 0 (as raw words, widened when they are used)
template <typename T>
struct NormRow {
    static constexpr int N = 16 / (int)sizeof(T);
    uint32_t w[4];
    __device__ __forceinline__ void load(const T* __restrict__ p, int i, int d) {
        if (i + N <= d) {
            const NormVec<T> q = *reinterpret_cast<const NormVec<T>*>(p + i);
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = q.v[j];
            return;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = 0u;
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (i + j < d) set(j, p[i + j]);
    }
    __device__ __forceinline__ void store(T* __restrict__ p, int i, int d) const {
        if (i + N <= d) {
            NormVec<T> q;
#pragma unroll
            for (int j = 0; j < 4; ++j) q.v[j] = w[j];
            *reinterpret_cast<NormVec<T>*>(p + i) = q;
            return;
        }
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (i + j < d) p[i + j] = element(j);
    }
    __device__ __forceinline__ void set(int j, float v) { w[j] = __float_as_uint(v); }
    __device__ __forceinline__ void set(int j, bf16_t v) { w[j / 2] |= (uint32_t)v.bits << (16 * (j & 1)); }
    __device__ __forceinline__ T element(int j) const;
    __device__ __forceinline__ float at(int j) const {
        if (N == 4) return __uint_as_float(w[j]);
        return __uint_as_float(j & 1 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16);
    }
    // from here on nothing is known of the words
    __device__ __forceinline__ void renew() {
#pragma unroll
        for (int j = 0; j < 4; ++j) asm volatile("" : "+v"(w[j]));
    }
    // the values rounded to the storage type
    __device__ __forceinline__ void round(const float (&f)[N]) {
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = N == 4 ? __float_as_uint(f[j]) : pack_bf16x2(f[(2 * j) % N], f[(2 * j + 1) % N]);
    }
};
template <>
__device__ __forceinline__ float NormRow<float>::element(int j) const {
    return __uint_as_float(w[j]);
}
template <>
__device__ __forceinline__ bf16_t NormRow<bf16_t>::element(int j) const {
    return bf16_t{(uint16_t)(w[j / 2] >> (16 * (j & 1)))};
}

// Sums that a thread keeps of its NV vectors: of each where a wave has the row, so that 64 vectors are one sum as they are
// where a wave has no more; else one.
constexpr int norm_sums(int tpr, int nv) { return tpr == 64 ? nv : 1; }

// The row's sum (and the largest of `mx`), the same in all of its TPR threads.  Every thread of the block calls it; the
// LDS is free again for a call with another `part`.
// A wave's S sums are halved together: a lane hands over those that its partner keeps, until it has one, the lane's bits 5 and
// 4 telling which; every sum's tree is that of S = 1.
template <int TPR, int S>
__device__ __forceinline__ float norm_row_reduce(const float (&sums)[S], uint32_t& mx, float* part_s, uint32_t* part_m) {
    static_assert(S == 1 || S == 2 || S == 4, "a lane's bits 5 and 4");
    float v[S];
#pragma unroll
    for (int n = 0; n < S; ++n) v[n] = sums[n];
    int off = 32;
#pragma unroll
    for (int s = S / 2; s >= 1; s /= 2, off /= 2) {
        const bool upper = (threadIdx.x & off) != 0;
#pragma unroll
        for (int n = 0; n < s; ++n) {
            const float keep = upper ? v[n + s] : v[n], give = upper ? v[n] : v[n + s];
            v[n] = keep + __shfl_xor(give, off, 64);
        }
    }
#pragma unroll
    for (; off >= 1; off >>= 1) v[0] += __shfl_xor(v[0], off, 64);
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
        const uint32_t m = (uint32_t)__shfl_xor((int)mx, o, 64);
        mx = m > mx ? m : mx;
    }
    float sum = 0.f;
    if (TPR == 64) {
#pragma unroll
        for (int n = 0; n < S; ++n)
            sum += __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v[0]), n * (64 / S)));
        return sum;
    }
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) {
        part_s[wave] = v[0];
        part_m[wave] = mx;
    }
    __syncthreads();
    mx = 0u;
#pragma unroll
    for (int w = 0; w < TPR / 64; ++w) {
        sum += part_s[w];
        mx = part_m[w] > mx ? part_m[w] : mx;
    }
    return sum;
}

constexpr int norm_block(int tpr) { return tpr > 256 ? tpr : 256; }

// q: rows of `pitch` bytes, zeros behind the first d.  h may be x or residual: a thread has read its elements of both
// before it writes.
template <typename T, int TPR, int NV>
__global__ __launch_bounds__(norm_block(TPR)) void add_rmsnorm_kernel(
    const T* x, const T* residual, const T* __restrict__ gain, int Tn, int d, float eps, T* h, T* __restrict__ y,
    int8_t* __restrict__ q, int pitch, float* __restrict__ q_scale, float* __restrict__ rstd) {
    typedef NormRow<T> Row;
    constexpr int N = Row::N, RPB = norm_block(TPR) / TPR;
    __shared__ float part_s[norm_block(TPR) / 64];
    __shared__ uint32_t part_m[norm_block(TPR) / 64];
    const int t = blockIdx.x * RPB + (int)threadIdx.x / TPR, i0 = ((int)threadIdx.x % TPR) * N;
    if (TPR == 64 && t >= Tn) return;   // a wave of its own; wider rows are a block's
    const size_t at = (size_t)t * d;
    Row v[NV], g[NV];
#pragma unroll
    for (int n = 0; n < NV; ++n) v[n].load(x + at, i0 + n * TPR * N, d);
    if (residual) {
        Row b[NV];
#pragma unroll
        for (int n = 0; n < NV; ++n) b[n].load(residual + at, i0 + n * TPR * N, d);
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            float f[N];
#pragma unroll
            for (int j = 0; j < N; ++j) f[j] = v[n].at(j) + b[n].at(j);
            v[n].round(f);
        }
    }
#pragma unroll
    for (int n = 0; n < NV; ++n) g[n].load(gain, i0 + n * TPR * N, d);
    if (h) {
#pragma unroll
        for (int n = 0; n < NV; ++n) v[n].store(h + at, i0 + n * TPR * N, d);
    }
    // the maximum of the bit patterns without the sign: as of the numbers, and a NaN is above them all
    constexpr int S = norm_sums(TPR, NV);
    float sums[S];
#pragma unroll
    for (int n = 0; n < S; ++n) sums[n] = 0.f;
    uint32_t mx = 0u;
#pragma unroll
    for (int n = 0; n < NV; ++n)
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float a = v[n].at(j);
            sums[n % S] = fmaf(a, a, sums[n % S]);
            const uint32_t b = __float_as_uint(a * g[n].at(j)) & 0x7fffffffu;
            mx = b > mx ? b : mx;
        }
    const float sum = norm_row_reduce<TPR>(sums, mx, part_s, part_m);
    // the elements are widened again below: as floats, held over the sum, they would take twice the registers
#pragma unroll
    for (int n = 0; n < NV; ++n) {
        v[n].renew();
        g[n].renew();
    }
    const float r = 1.0f / sqrtf(sum / (float)d + eps);
    if (rstd && i0 == 0) rstd[t] = r;
    if (y) {
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            float f[N];
#pragma unroll
            for (int j = 0; j < N; ++j) f[j] = v[n].at(j) * r * g[n].at(j);
            Row o;
            o.round(f);
            o.store(y + at, i0 + n * TPR * N, d);
        }
    }
    if (q) {
        // below 2^-120 the quotient would overflow: such a row counts as zero
        const float m = __uint_as_float(mx);
        const bool none = mx < 0x03800000u;
        // a maximum that is no number: 0 keeps the zeros past d (and 127 / inf does)
        const float inv = none || mx > 0x7f800000u ? 0.f : 127.0f / m;
        if (i0 == 0) q_scale[t] = none ? 0.f : m * r / 127.0f;
        int8_t* row = q + (size_t)t * pitch;
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            const int i = i0 + n * TPR * N;
            uint32_t w[2] = {0u, 0u};
#pragma unroll
            for (int j = 0; j < N; ++j) {   // elements past d are 0; one that is no number has a scale that is none either
                const float c = fminf(fmaxf(v[n].at(j) * g[n].at(j) * inv, -127.f), 127.f);
                w[j / 4] |= (uint32_t)((int)rintf(c) & 0xff) << (8 * (j & 3));
            }
            if (i < pitch) {
                *reinterpret_cast<uint32_t*>(row + i) = w[0];
                if (N == 8) *reinterpret_cast<uint32_t*>(row + i + 4) = w[1];
            }
        }
    }
}

// Backward.  A block takes the rows blockIdx.x * RPB + .., stepping by the grid, keeps its threads' columns of dgain in
// registers and leaves one partial row of them, [block][d] in `partial`.
template <typename T, int TPR, int NV>
__global__ __launch_bounds__(norm_block(TPR)) void add_rmsnorm_bwd_kernel(const T* __restrict__ dy, const T* __restrict__ dh,
                                                                          const T* __restrict__ h, const T* __restrict__ gain,
                                                                          const float* __restrict__ rstd, int Tn, int d,
                                                                          T* __restrict__ dx, float* __restrict__ partial) {
    typedef NormRow<T> Row;
    constexpr int N = Row::N, RPB = norm_block(TPR) / TPR;
    __shared__ float part_s[2][norm_block(TPR) / 64];
    __shared__ uint32_t part_m[2][norm_block(TPR) / 64];
    // RPB > 1: the waves' sums of a column, one vector of each lane at a time
    __shared__ float fold[RPB > 1 ? RPB : 1][RPB > 1 ? 64 * N : 1];
    const int i0 = ((int)threadIdx.x % TPR) * N;
    float acc[NV][N];
    Row g[NV];
#pragma unroll
    for (int n = 0; n < NV; ++n) {
        g[n].load(gain, i0 + n * TPR * N, d);
#pragma unroll
        for (int j = 0; j < N; ++j) acc[n][j] = 0.f;
    }
    int turn = 0;
    for (long t = (long)blockIdx.x * RPB + (int)threadIdx.x / TPR; t < Tn; t += (long)gridDim.x * RPB, turn ^= 1) {
        const size_t at = (size_t)t * d;
        Row a[NV], b[NV], c[NV];
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            a[n].load(h + at, i0 + n * TPR * N, d);
            b[n].load(dy + at, i0 + n * TPR * N, d);
        }
        auto load_dh = [&] {
            if (dh) {
#pragma unroll
                for (int n = 0; n < NV; ++n) c[n].load(dh + at, i0 + n * TPR * N, d);
            }
        };
        constexpr bool kLate = TPR * NV > 2048;   // the widest rows: 128 registers do not hold all three at once
        if (!kLate) load_dh();
        const float r = rstd[t];
        constexpr int S = norm_sums(TPR, NV);
        float sums[S];
#pragma unroll
        for (int n = 0; n < S; ++n) sums[n] = 0.f;
        uint32_t none = 0u;
#pragma unroll
        for (int n = 0; n < NV; ++n)
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float nrm = a[n].at(j) * r, v = b[n].at(j);
                sums[n % S] = fmaf(v * g[n].at(j), nrm, sums[n % S]);
                acc[n][j] = fmaf(v, nrm, acc[n][j]);
            }
        const float mean = norm_row_reduce<TPR>(sums, none, part_s[turn], part_m[turn]) / (float)d;
        if (kLate) load_dh();
#pragma unroll
        for (int n = 0; n < NV; ++n) {
            float f[N];
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float nrm = a[n].at(j) * r;
                f[j] = r * (b[n].at(j) * g[n].at(j) - nrm * mean);
                if (dh) f[j] += c[n].at(j);
            }
            Row o;
            o.round(f);
            o.store(dx + at, i0 + n * TPR * N, d);
        }
    }
    float* row = partial + (size_t)blockIdx.x * d;
#pragma unroll
    for (int n = 0; n < NV; ++n) {
        const int i = i0 + n * TPR * N;
        if (RPB > 1) {
            const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
            __syncthreads();
#pragma unroll
            for (int j = 0; j < N; ++j) fold[w][lane * N + j] = acc[n][j];
            __syncthreads();
            for (int c = threadIdx.x; c < 64 * N; c += 256) {
                float s = 0.f;
#pragma unroll
                for (int k = 0; k < RPB; ++k) s += fold[k][c];
                if (n * 64 * N + c < d) row[n * 64 * N + c] = s;
            }
        } else if (i + N <= d) {
#pragma unroll
            for (int k = 0; k < N; k += 4) {
                NormF4 o = {{acc[n][k], acc[n][k + 1], acc[n][k + 2], acc[n][k + 3]}};
                *reinterpret_cast<NormF4*>(row + i + k) = o;
            }
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (i + j < d) row[i + j] = acc[n][j];
        }
    }
}

// dgain[i] = sum of the partial rows, rows r = w, w + 16, ... by thread row w in ascending order, then the sixteen in order.
// 64 columns a block: whole cache lines of a partial row.
template <typename T>
__global__ __launch_bounds__(1024) void norm_dgain_kernel(const float* __restrict__ partial, int rows, int d,
                                                          T* __restrict__ dgain) {
    __shared__ float part[16][64];
    const int c = threadIdx.x & 63, w = threadIdx.x >> 6, i = blockIdx.x * 64 + c;
    float s = 0.f;
    if (i < d) {
#pragma unroll 8
        for (int r = w; r < rows; r += 16) s += partial[(size_t)r * d + i];
    }
    part[w][c] = s;
    __syncthreads();
    if (w == 0 && i < d) {
#pragma unroll
        for (int k = 1; k < 16; ++k) s += part[k][c];
        dgain[i] = from_float<T>(s);
    }
}

// Threads of a row and vectors of a thread, for `vecs` 16-byte vectors of a row (CALL(threads, vectors)).  Few rows are
// spread over more threads: a launch of few blocks waits for its loads, and more of them are in flight at once.  wide: rows of
// up to 1024 vectors by as many threads (the backward, whose columns of dgain stay in registers).
#define XMOE_NORM_SHAPE(vecs, few, wide, CALL)                   \
    do {                                                         \
        if ((vecs) <= 64) { CALL(64, 1); }                       \
        else if (!(few) && (vecs) <= 128) { CALL(64, 2); }       \
        else if (!(few) && (vecs) <= 256) { CALL(64, 4); }       \
        else if ((vecs) <= 256) { CALL(256, 1); }                \
        else if ((vecs) <= 512) { CALL(256, 2); }                \
        else if (!(wide) && (vecs) <= 1024) { CALL(256, 4); }    \
        else if ((vecs) <= 1024) { CALL(1024, 1); }              \
        else if ((vecs) <= 2048) { CALL(1024, 2); }              \
        else if constexpr (sizeof(T) == 4) { CALL(1024, 4); }    \
    } while (0)
constexpr int kNormFewRows = 1024;

template <typename T>
int launch_norm(const void* x, const void* residual, const void* gain, int Tn, int d, float eps, void* h, void* y, void* q,
                float* q_scale, float* rstd, hipStream_t s) {
    const int vecs = (d + NormRow<T>::N - 1) / NormRow<T>::N, pitch = q8_pitch(d);
    // 8-bit rows are filled up to their pitch: by the vectors that cover it
    const int cover = q ? pitch / NormRow<T>::N : vecs;
#define XMOE_CALL(TPR, NV)                                                                                             \
    XMOE_LAUNCH(K_ADD_RMSNORM, s,                                                                                      \
                hipLaunchKernelGGL((add_rmsnorm_kernel<T, TPR, NV>),                                                   \
                                   dim3((unsigned)((Tn + norm_block(TPR) / TPR - 1) / (norm_block(TPR) / TPR))),       \
                                   dim3(norm_block(TPR)), 0, s, (const T*)x, (const T*)residual, (const T*)gain, Tn, d, \
                                   eps, (T*)h, (T*)y, (int8_t*)q, pitch, q_scale, rstd))
    XMOE_NORM_SHAPE(cover, Tn <= kNormFewRows, false, XMOE_CALL);
#undef XMOE_CALL
    return XMOE_OK;
}

template <typename T>
int launch_norm_bwd(const void* dy, const void* dh, const void* h, const void* gain, const float* rstd, int Tn, int d,
                    void* dx, void* dgain, float* partial, hipStream_t s) {
    const int vecs = (d + NormRow<T>::N - 1) / NormRow<T>::N, blocks = norm_bwd_blocks(Tn, d);
    if (blocks > 0) {
#define XMOE_CALL(TPR, NV)                                                                                              \
    XMOE_LAUNCH(K_ADD_RMSNORM_BWD, s,                                                                                   \
                hipLaunchKernelGGL((add_rmsnorm_bwd_kernel<T, TPR, NV>), dim3((unsigned)blocks), dim3(norm_block(TPR)), 0, s, \
                                   (const T*)dy, (const T*)dh, (const T*)h, (const T*)gain, rstd, Tn, d, (T*)dx, partial))
        XMOE_NORM_SHAPE(vecs, Tn <= kNormFewRows, true, XMOE_CALL);
#undef XMOE_CALL
    }
    XMOE_LAUNCH(K_NORM_DGAIN, s,
                hipLaunchKernelGGL(norm_dgain_kernel<T>, dim3((unsigned)((d + 63) / 64)), dim3(1024), 0, s, partial, blocks,
                                   d, (T*)dgain));
    return XMOE_OK;
}

int check_norm(int T, int d, int dt) {
    if (!dtype_ok(dt)) return XMOE_ERR_UNSUPPORTED;
    if (T < 0 || d < 1 || T >= (1 << 22)) return XMOE_ERR_INVALID_ARG;   // a grid has fewer than 2^32 threads
    if (d > XMOE_MAX_NORM_WIDTH) return XMOE_ERR_UNSUPPORTED;
    return XMOE_OK;
}

}  // namespace
}  // namespace xmoe

using namespace xmoe;

extern "C" {

int xmoe_add_rmsnorm(const void* x, const void* residual, const void* gain, int T, int d, float eps, int dt, void* h,
                     void* y, void* q, float* q_scale, float* rstd, void* stream) {
    int st = check_norm(T, d, dt);
    if (st != XMOE_OK) return st;
    if (!(eps > 0.f) || !(eps < INFINITY)) return XMOE_ERR_INVALID_ARG;
    if (T == 0) return XMOE_OK;
    if ((!y && !q) || !q != !q_scale || (residual && !h)) return XMOE_ERR_INVALID_ARG;
    if (!x || !gain || (reinterpret_cast<uintptr_t>(q) & 15u)) return XMOE_ERR_INVALID_ARG;
    hipStream_t s = (hipStream_t)stream;
    return dt == XMOE_F32 ? launch_norm<float>(x, residual, gain, T, d, eps, h, y, q, q_scale, rstd, s)
                          : launch_norm<bf16_t>(x, residual, gain, T, d, eps, h, y, q, q_scale, rstd, s);
}

int xmoe_add_rmsnorm_bwd(const void* dy, const void* dh, const void* h, const void* gain, const float* rstd, int T, int d,
                         int dt, void* dx, void* dgain, void* ws, size_t ws_bytes, void* stream) {
    int st = check_norm(T, d, dt);
    if (st != XMOE_OK) return st;
    if (!gain || !dgain) return XMOE_ERR_INVALID_ARG;
    if (T > 0 && (!dy || !h || !rstd || !dx)) return XMOE_ERR_INVALID_ARG;
    if (!ws || (reinterpret_cast<uintptr_t>(ws) & 255u) || ws_bytes < norm_bwd_ws_bytes(T, d)) return XMOE_ERR_WORKSPACE;
    hipStream_t s = (hipStream_t)stream;
    return dt == XMOE_F32 ? launch_norm_bwd<float>(dy, dh, h, gain, rstd, T, d, dx, dgain, (float*)ws, s)
                          : launch_norm_bwd<bf16_t>(dy, dh, h, gain, rstd, T, d, dx, dgain, (float*)ws, s);
}

}  // extern "C"
