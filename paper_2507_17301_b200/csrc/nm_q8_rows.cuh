// Activations to 8-bit integers with a scale for each row (token), fused with what stands in front of it.
//
//   p_j = s_j w_j with s = x + r held in the activations' type (rmsnorm), u_j g_j / (1 + exp(-g_j)) (silu_mul), x_j (rows)
//   a = max |p_j|,   q_j = nearest integer to 127 p_j / a (ties to even),   scale = a / 127, times 1 / sqrt(mean s^2 + eps) for rmsnorm
//
// The norm's factor cancels out of q, so one reduction over the row gives both the sum of squares and the maximum, and a row is
// read once: its p stay in registers (rows of more than 16384 columns are read again, out of the L2).
//
// q is the integer that exact arithmetic gives, whatever the kernel's shape: p is worked out in 32 bits, and where 127 p / a lies so
// near a border between two integers that their error could decide, it is worked out again in 64; the maximum is taken in 64
// bits over the elements that 32 bits cannot tell from it.  (Products of two 16-bit values are exact in 32 bits, so these norms
// need neither.)  Rows whose maximum or sum leaves the range in which the error bounds hold (NaN, infinities, zeros, overflow)
// are done in 64 bits altogether: zeros give q = 0 and scale 0, a row that is not finite gives q = 0 and scale NaN.
//
// Bound by memory: reading and writing each element once, 16 bytes a load, with at least four loads a thread in flight.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cmath>

#include "nm_ptx.cuh"
#include "nm_q8.h"

namespace q8rows {

template <typename T>
__device__ __forceinline__ float to_float(T v);
template <>
__device__ __forceinline__ float to_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ float to_float<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <>
__device__ __forceinline__ float to_float<__half>(__half v) { return __half2float(v); }
template <typename T>
__device__ __forceinline__ T from_float(float v);
template <>
__device__ __forceinline__ float from_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }

template <typename T>
struct alignas(sizeof(T) * 8 < 16 ? sizeof(T) * 8 : 16) Eight {
    T v[8];
};

// Eight consecutive elements, the `n` first of which exist (zeros for the others); VEC: `p` is 16-byte aligned.
template <typename T, bool VEC>
__device__ __forceinline__ Eight<T> load8(const T* p, int n)
{
    Eight<T> e;
    if (VEC && n >= 8) {
        if constexpr (sizeof(T) == 2) {
            *reinterpret_cast<uint4*>(&e) = *reinterpret_cast<const uint4*>(p);
        } else {
            reinterpret_cast<uint4*>(&e)[0] = reinterpret_cast<const uint4*>(p)[0];
            reinterpret_cast<uint4*>(&e)[1] = reinterpret_cast<const uint4*>(p)[1];
        }
        return e;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) e.v[i] = i < n ? p[i] : from_float<T>(0.f);
    return e;
}
template <typename T, bool VEC>
__device__ __forceinline__ void store8(T* p, const Eight<T>& e, int n)
{
    if (VEC && n >= 8) {
        if constexpr (sizeof(T) == 2) {
            *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(&e);
        } else {
            reinterpret_cast<uint4*>(p)[0] = reinterpret_cast<const uint4*>(&e)[0];
            reinterpret_cast<uint4*>(p)[1] = reinterpret_cast<const uint4*>(&e)[1];
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) p[i] = e.v[i];
}

// Relative error of p times 127 / a in 32 bits, with room: four roundings (2.4e-7); for silu_mul the exponential's (at most
// 2 + 1.173 |g| units of 2^-23, |g| <= 80), the division's (2 units) and three roundings, 1.2e-5.
template <Q8RowOp OP>
constexpr float kError = OP == Q8_SILU_MUL ? 1.5e-5f : 4e-7f;

// p of one column in 64 bits, from memory.
template <Q8RowOp OP, typename T, typename W>
__device__ double exact_value(const Q8Rows& a, size_t row, int col, double* s_out = nullptr)
{
    if constexpr (OP == Q8_SILU_MUL) {
        const double g = to_float(static_cast<const T*>(a.x)[row * a.x_ld + col]), u = to_float(static_cast<const T*>(a.r)[row * a.r_ld + col]);
        return g / (1.0 + exp(-g)) * u;
    } else if constexpr (OP == Q8_ROWS) {
        return to_float(static_cast<const T*>(a.x)[row * a.x_ld + col]);
    } else {
        // (a thread reads back what it has written itself)
        const double s = a.r ? to_float(static_cast<const T*>(a.s)[row * a.s_ld + col]) : to_float(static_cast<const T*>(a.x)[row * a.x_ld + col]);
        if (s_out) *s_out = s;
        return s * static_cast<double>(to_float(static_cast<const W*>(a.weight)[col]));
    }
}

template <Q8RowOp OP, typename T, typename W>
__device__ __noinline__ double exact_again(const Q8Rows& a, size_t row, int col)
{
    return exact_value<OP, T, W>(a, row, col);
}

// u * SiLU(g) where 32 bits do not reach.
__device__ __noinline__ inline float gated_in_64(float g, float u)
{
    const double d = g;
    return static_cast<float>(d / (1.0 + exp(-d)) * static_cast<double>(u));
}

struct Scratch {
    float sum[32];
    uint32_t top[32];
    double a[32], sum64[32];
    int bad[32];
};

// Maximum of non-negative doubles (their bits are ordered like them) and sum over the TPR threads of a row.
__device__ __forceinline__ double warp_max(double v)
{
    for (int d = 16; d > 0; d >>= 1) v = fmax(v, __shfl_xor_sync(0xFFFFFFFFu, v, d));
    return v;
}
template <int TPR>
__device__ __forceinline__ double row_max(double v, double* part)
{
    v = warp_max(v);
    if constexpr (TPR > 32) {
        if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
        __syncthreads();
        const int lane = threadIdx.x & 31;
        v = warp_max(lane < TPR / 32 ? part[lane] : 0.0);
    }
    return v;
}

// The whole row in 64 bits (its thread `t` of TPR; all of them come here together).
template <Q8RowOp OP, typename T, typename W, int TPR>
__device__ __noinline__ void row_in_64(const Q8Rows& a, size_t row, int t, Scratch* sc)
{
    double top = 0.0, sum = 0.0;
    int bad = 0;
    for (int v = t; v * 8 < a.h; v += TPR)
        for (int c = v * 8; c < min(v * 8 + 8, a.h); ++c) {
            double s = 0.0;
            const double p = exact_value<OP, T, W>(a, row, c, &s);
            bad |= !(fabs(p) <= 1e300) || !(fabs(s) <= 1e300);
            top = fmax(top, fabs(p));
            sum += s * s;
        }
    for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
    bad = __any_sync(0xFFFFFFFFu, bad);
    if constexpr (TPR > 32) {
        __syncthreads();   // (the scratch may still be read)
        if ((t & 31) == 0) {
            sc->sum64[t >> 5] = sum;
            sc->bad[t >> 5] = bad;
        }
    }
    top = row_max<TPR>(top, sc->a);
    if constexpr (TPR > 32) {
        sum = 0.0;
        bad = 0;
        for (int i = 0; i < TPR / 32; ++i) {
            sum += sc->sum64[i];
            bad |= sc->bad[i];
        }
    }
    double scale = top / 127.0;
    if constexpr (OP == Q8_RMSNORM) scale = top / sqrt(sum / a.h + static_cast<double>(a.eps)) / 127.0;
    const float stored = static_cast<float>(scale);
    const bool good = !bad && stored < INFINITY;
    if (t == 0) a.scale[row] = good ? stored : NAN;
    for (int v = t; v * 8 < a.h; v += TPR)
        for (int c = v * 8; c < min(v * 8 + 8, a.h); ++c)
            a.q[row * a.q_ld + c] =
                good && top > 0.0 ? static_cast<int8_t>(rint(127.0 * exact_value<OP, T, W>(a, row, c) / top)) : static_cast<int8_t>(0);
}

// TPR threads take a row, each NV groups of eight columns, in steps of TPR groups.  KEEP: the row's p stay in registers (8 * NV * TPR >= h).
template <Q8RowOp OP, typename T, typename W, int TPR, int NV, bool KEEP, bool VEC>
__global__ void __launch_bounds__(TPR < 128 ? 128 : TPR) k_q8_rows(const __grid_constant__ Q8Rows a)
{
    constexpr int ROWS = TPR < 128 ? 128 / TPR : 1;
    static_assert(TPR == 32 || ROWS == 1, "a row is a warp's or a block's");
    // products of two 16-bit values fit 32 bits, an input is itself
    constexpr bool EXACT = OP == Q8_ROWS || (OP == Q8_RMSNORM && sizeof(T) == 2 && sizeof(W) == 2);
    __shared__ Scratch scratch[ROWS];
    const int t = threadIdx.x % TPR;
    const size_t row = static_cast<size_t>(blockIdx.x) * ROWS + threadIdx.x / TPR;
    nmk::pdl_launch_dependents();
    nmk::pdl_wait();
    if (row >= static_cast<size_t>(a.tokens)) return;   // (whole rows: ROWS > 1 has no barrier across warps)
    Scratch* sc = scratch + threadIdx.x / TPR;
    const T* x = static_cast<const T*>(a.x) + row * a.x_ld;
    const T* r = a.r ? static_cast<const T*>(a.r) + row * a.r_ld : nullptr;
    T* s_row = a.s ? static_cast<T*>(a.s) + row * a.s_ld : nullptr;
    const W* weight = static_cast<const W*>(a.weight);

    float p[KEEP ? NV : 1][8];
    float sum = 0.f;
    uint32_t top = 0u;   // bits of max |p|: NaN above infinity above numbers
    // p of the groups at `base` on; `first`: sums, and the residual's addition is written
    auto values = [&](int v, float (&out)[8], const Eight<T>& ex, const Eight<T>& er, const Eight<W>& ew, bool first) {
        const int n = a.h - v * 8;
        if constexpr (OP == Q8_RMSNORM) {
            Eight<T> es = ex;
            if (r && first) {
#pragma unroll
                for (int i = 0; i < 8; ++i) es.v[i] = from_float<T>(to_float(ex.v[i]) + to_float(er.v[i]));
                store8<T, VEC>(s_row + v * 8, es, n);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float s = to_float(es.v[i]);
                if (first) sum = fmaf(s, s, sum);
                out[i] = s * to_float(ew.v[i]);
            }
        } else if constexpr (OP == Q8_SILU_MUL) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float g = to_float(ex.v[i]), u = to_float(er.v[i]);
                out[i] = __fdividef(g, 1.f + __expf(-g)) * u;
                // outside the range of the error bound: exp(-g) overflows, or g is next to the least number
                if (g < -80.f || (fabsf(g) < 1e-30f && g != 0.f)) out[i] = gated_in_64(g, u);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) out[i] = to_float(ex.v[i]);
        }
        if (first) {
#pragma unroll
            for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(out[i]) & 0x7FFFFFFFu);   // (columns past the end are zeros)
        }
    };
    auto pass = [&](int base, bool first, auto&& use) {
        Eight<T> ex[NV], er[NV];
        Eight<W> ew[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = base + i * TPR, n = a.h - v * 8;
            if (n <= 0) continue;
            // the second reading of a norm's row finds the sum in memory
            const T* from = OP == Q8_RMSNORM && r && !first ? s_row : x;
            ex[i] = load8<T, VEC>(from + v * 8, n);
            if (OP == Q8_SILU_MUL || (OP == Q8_RMSNORM && r && first)) er[i] = load8<T, VEC>(r + v * 8, n);
            if (OP == Q8_RMSNORM) ew[i] = load8<W, VEC>(weight + v * 8, n);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = base + i * TPR;
            if (v * 8 >= a.h) continue;
            float tmp[8];
            values(v, tmp, ex[i], er[i], ew[i], first);
            use(i, v, tmp);
        }
    };
    if constexpr (KEEP) {
        pass(t, true, [&](int i, int, float (&f)[8]) {
#pragma unroll
            for (int e = 0; e < 8; ++e) p[i][e] = f[e];
        });
    } else {
        for (int base = t; base * 8 < a.h; base += NV * TPR) pass(base, true, [](int, int, float (&)[8]) {});
    }

    if constexpr (OP == Q8_RMSNORM) {
        for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
    }
    top = __reduce_max_sync(0xFFFFFFFFu, top);
    if constexpr (TPR > 32) {
        if ((t & 31) == 0) {
            sc->sum[t >> 5] = sum;
            sc->top[t >> 5] = top;
        }
        __syncthreads();
        const int lane = t & 31;
        top = __reduce_max_sync(0xFFFFFFFFu, lane < TPR / 32 ? sc->top[lane] : 0u);
        if constexpr (OP == Q8_RMSNORM) {
            sum = lane < TPR / 32 ? sc->sum[lane] : 0.f;
            for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
        }
    }
    const float a32 = __uint_as_float(top);
    // 2^-60: products that 32 bits lose below 2^-126 are then less than a step by far
    if (!(a32 >= 0x1p-60f && a32 < INFINITY && sum < INFINITY)) {
        row_in_64<OP, T, W, TPR>(a, row, t, sc);
        return;
    }
    double a64 = a32;
    if constexpr (!EXACT) {
        double mine = 0.0;
        const float near_top = a32 * (1.f - 2.f * kError<OP>);
        auto look = [&](int, int v, float (&f)[8]) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (fabsf(f[e]) >= near_top) mine = fmax(mine, fabs(exact_again<OP, T, W>(a, row, v * 8 + e)));
        };
        if constexpr (KEEP) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if ((t + i * TPR) * 8 < a.h) look(i, t + i * TPR, p[i]);
        } else {
            for (int base = t; base * 8 < a.h; base += NV * TPR) pass(base, false, look);
        }
        a64 = row_max<TPR>(mine, sc->a);
    }
    if (t == 0) {
        float scale = static_cast<float>(a64 / 127.0);
        if constexpr (OP == Q8_RMSNORM) scale *= 1.f / sqrtf(sum / static_cast<float>(a.h) + a.eps);
        a.scale[row] = scale < INFINITY ? scale : NAN;
    }
    const float inv = 127.f / static_cast<float>(a64);
    int8_t* q_row = a.q + row * a.q_ld;
    auto quantise = [&](int, int v, float (&f)[8]) {
        int k[8];
        bool again = false;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float y = f[e] * inv, n = rintf(y);
            k[e] = static_cast<int>(n);
            again |= fabsf(y - n) > 0.5f - fabsf(y) * kError<OP>;
        }
        if (again) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float y = f[e] * inv;
                if (fabsf(y - rintf(y)) > 0.5f - fabsf(y) * kError<OP>) {
                    const double d = EXACT ? static_cast<double>(f[e]) : exact_again<OP, T, W>(a, row, v * 8 + e);
                    k[e] = static_cast<int>(rint(127.0 * d / a64));
                }
            }
        }
        uint32_t lo = 0u, hi = 0u;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            lo |= (static_cast<uint32_t>(k[e]) & 0xFFu) << (8 * e);
            hi |= (static_cast<uint32_t>(k[e + 4]) & 0xFFu) << (8 * e);
        }
        const int n = a.h - v * 8;
        if (n >= 8) {
            *reinterpret_cast<uint2*>(q_row + v * 8) = make_uint2(lo, hi);
        } else {
            for (int e = 0; e < n; ++e) q_row[v * 8 + e] = static_cast<int8_t>((e < 4 ? lo >> (8 * e) : hi >> (8 * (e - 4))) & 0xFFu);
        }
    };
    if constexpr (KEEP) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if ((t + i * TPR) * 8 < a.h) quantise(i, t + i * TPR, p[i]);
    } else {
        for (int base = t; base * 8 < a.h; base += NV * TPR) pass(base, false, quantise);
    }
}

template <Q8RowOp OP, typename T, typename W, int TPR, int NV, bool KEEP, bool VEC>
cudaError_t launch_one(const Q8Rows& a, cudaStream_t st)
{
    constexpr int rows = TPR < 128 ? 128 / TPR : 1;
    return nmhost::launch_pdl(k_q8_rows<OP, T, W, TPR, NV, KEEP, VEC>, static_cast<unsigned>((a.tokens + rows - 1) / rows), TPR < 128 ? 128u : TPR, 0,
                              st, a);
}

// Threads for a row: four groups of eight columns each, one or two where there are too few rows to fill the GPU.
template <Q8RowOp OP, typename T, typename W>
cudaError_t launch_shape(const Q8Rows& a, bool vec, cudaStream_t st)
{
    if (!vec) {
        if (a.h <= 1024) return launch_one<OP, T, W, 32, 4, true, false>(a, st);
        if (a.h <= 8192) return launch_one<OP, T, W, 256, 4, true, false>(a, st);
        return launch_one<OP, T, W, 512, 4, false, false>(a, st);
    }
    const bool few = a.tokens <= 2 * nmhost::sm_count();
    if (a.h <= 1024 && !few) return launch_one<OP, T, W, 32, 4, true, true>(a, st);
    if (a.h <= 4096) return few ? launch_one<OP, T, W, 512, 1, true, true>(a, st) : launch_one<OP, T, W, 128, 4, true, true>(a, st);
    if (a.h <= 8192 && !few) return launch_one<OP, T, W, 256, 4, true, true>(a, st);
    if (a.h <= 16384) return few ? launch_one<OP, T, W, 1024, 2, true, true>(a, st) : launch_one<OP, T, W, 512, 4, true, true>(a, st);
    return launch_one<OP, T, W, 512, 4, false, true>(a, st);
}

template <typename T>
nm_status_t launch(Q8RowOp op, const Q8Rows& a, nm_dtype_t weight_type, bool vec, cudaStream_t st)
{
    cudaError_t e;
    if (op == Q8_SILU_MUL) e = launch_shape<Q8_SILU_MUL, T, T>(a, vec, st);
    else if (op == Q8_ROWS) e = launch_shape<Q8_ROWS, T, T>(a, vec, st);
    else if (sizeof(T) == 2 && weight_type == NM_F32) e = launch_shape<Q8_RMSNORM, T, float>(a, vec, st);
    else e = launch_shape<Q8_RMSNORM, T, T>(a, vec, st);
    nmhost::count_launch(1);
    if (e == cudaSuccess) e = cudaGetLastError();
    if (e != cudaSuccess) return nmhost::fail(NM_ERR_CUDA, "8-bit row kernel launch: %s", cudaGetErrorString(e));
    return NM_OK;
}

}  // namespace q8rows
