// Activations to 8-bit integers with a scale for each row (token), fused with what stands in front of it.
//
//   p_j = s_j w_j with s = x + r held in the activations' type (rmsnorm), u_j g_j / (1 + exp(-g_j)) (silu_mul), x_j (rows)
//   a = max |p_j|,   q_j = nearest integer to 127 p_j / a (ties to even),   scale = a / 127, times 1 / sqrt(mean s^2 + eps) for rmsnorm
//
// The norm's factor cancels out of q, so one reduction over the row gives both the sum of squares and the maximum, and a row is
// read once: its p stay in registers (rows of more than 32768 columns, 16384 of 32 bits or off the 16-byte boundaries, are read again,
// out of the L2).
//
// q is the integer that exact arithmetic gives, whatever the kernel's shape: p is worked out in 32 bits, and where 127 p / a lies so
// near a border between two integers that their error could decide, it is worked out again in 64; the maximum is taken in 64
// bits over the elements that 32 bits cannot tell from it.  (Products of two 16-bit values are exact in 32 bits, and of bfloat16
// values so small that a corrected division tells every quotient's side: those need neither.)  Rows whose maximum or sum leaves the range in which the error bounds hold (NaN, infinities, zeros, overflow)
// are done in 64 bits altogether: zeros give q = 0 and scale 0, a row that is not finite gives q = 0 and scale NaN.
//
// Each element is read and written once.  Persistent blocks: a thread has its part of the next row on its way to shared memory (16 bytes a
// copy, places of its own, no barrier) while the row before is reduced and written.  8192 x 8192 bf16 with residual 86.5 us, 83 % of the
// copy rate; gated 4096 x 12288 bf16 63 us, 61 %, with 61 % of the issue slots used and 35 % of the warps active (why no more is not known);
// 4096 x 8192 fp32 with residual 135 us, 50 %, gated 4096 x 12288 fp32 143 us, 48 %.  Rows that do not start on 16 bytes go without the
// copies, an element at a time: 4096 x 1001 bf16 plain 9.7 us, 19 %, gated 16.8.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cmath>
#include <type_traits>

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

// The columns of a group: eight consecutive ones where rows can be read 16 bytes at a time, else every TPR-th, so that neighbouring
// threads read neighbouring columns (4096 x 1001 bf16 with eight consecutive ones everywhere 21.6 us).
template <int TPR, bool VEC>
struct Group {
    int first, count;   // of them; may be more than eight, or none
    static constexpr int step = VEC ? 1 : TPR;
    __device__ __forceinline__ Group(int v, int h)
    {
        first = VEC ? v * 8 : v / TPR * 8 * TPR + v % TPR;
        count = VEC ? h - first : (h - first + TPR - 1) / TPR;
    }
};

// Eight elements `STEP` apart, the `n` first of which exist (zeros for the others); VEC: consecutive, and `p` is 16-byte aligned.
template <typename T, bool VEC, int STEP>
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
    for (int i = 0; i < 8; ++i) e.v[i] = i < n ? p[i * STEP] : from_float<T>(0.f);
    return e;
}
template <typename T, bool VEC, int STEP>
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
        if (i < n) p[i * STEP] = e.v[i];
}

// x + r, rounded once: for 16-bit types the two-way addition, which gives what a sum in 32 bits rounded to 16 gives (where that
// sum is not exact the lesser number is below a quarter of the greater's last place, and both round to the greater).
template <typename T>
__device__ __forceinline__ Eight<T> add8(const Eight<T>& x, const Eight<T>& r)
{
    Eight<T> s;
    if constexpr (sizeof(T) == 2) {
        using T2 = std::conditional_t<std::is_same_v<T, __half>, __half2, __nv_bfloat162>;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            reinterpret_cast<T2*>(&s)[i] = __hadd2_rn(reinterpret_cast<const T2*>(&x)[i], reinterpret_cast<const T2*>(&r)[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) s.v[i] = x.v[i] + r.v[i];
    }
    return s;
}

// Two fp32 numbers in a 64-bit register, for the instructions that work on both.
using Pair = unsigned long long;
__device__ __forceinline__ Pair pair(float lo, float hi)
{
    Pair d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi));
    return d;
}
__device__ __forceinline__ void split(Pair p, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(p)); }
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c)
{
    Pair d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ Pair mul2(Pair a, Pair b)
{
    Pair d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ Pair add2(Pair a, Pair b)
{
    Pair d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
// max(|a|, |b|, |c|), NaN if one is.
__device__ __forceinline__ float top3(float a, float b, float c)
{
    float m;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(a), "f"(b), "f"(c));
    return m;
}
// Elements 2i and 2i + 1.
template <typename T>
__device__ __forceinline__ Pair two_of(const Eight<T>& e, int i)
{
    if constexpr (std::is_same_v<T, __nv_bfloat16>) {
        const uint32_t u = reinterpret_cast<const uint32_t*>(&e)[i];
        return pair(__uint_as_float(u << 16), __uint_as_float(u & 0xFFFF0000u));
    } else {
        return pair(to_float(e.v[2 * i]), to_float(e.v[2 * i + 1]));
    }
}

// Relative error of p times 127 / a in 32 bits, with room: five roundings (3e-7); for silu_mul beside them the exponent's two
// roundings of up to 126 * 2^-24 each (1.04e-5 in all, g >= -87), 2^-22 and 2^-23 of the exponential and the reciprocal, and three more.
template <Q8RowOp OP>
constexpr float kError = OP == Q8_SILU_MUL ? 1.5e-5f : 4e-7f;
// silu_mul beyond g = -87: less than kMostProduct * 2^-125 * 88, which is nothing beside kLeastTop
constexpr float kMostProduct = 0x1p40f, kLeastTop = 0x1p-60f;
constexpr float kMostTop = 0x1p100f;   // (127 p and 1 / a stay normal numbers)
constexpr float kMostSum = 0x1p120f;
// How near 127 p / a may come to a border between two integers before 64 bits decide.  Its error is that of p and that of the maximum, both
// relative to the quotient, which is up to a half more than the integer: border_of counts the integer's share, and the half's stands
// here (all there is where the integer is 0), beside the roundings of 127 / a.
template <Q8RowOp OP>
constexpr float kBorder = 0.5f - kError<OP> - 1e-7f;

// The products g u and g u / (1 + exp(-g)): (g u) first, whose underflow cannot matter beside kLeastTop.  Where the exponential
// or its reciprocal leaves 32 bits (g < -87) the result is 0.  (Making good the exponent's rounding leaves a twentieth of the quotients
// to 64 bits and costs more than it saves: 4096 x 12288 bf16 72 us instead of 69.)
__device__ __forceinline__ void gated(Pair g, Pair u, Pair* product, Pair* p)
{
    float a, b;
    split(g, a, b);
    a *= -1.44269504f;
    b *= -1.44269504f;
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(a));
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(b));
    a += 1.f;
    b += 1.f;
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(a));
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(b));
    *product = mul2(g, u);
    *p = mul2(*product, pair(a, b));
}

__device__ __forceinline__ double gated_in_64(double g, double u) { return g / (1.0 + exp(-g)) * u; }
template <typename T>
__device__ __forceinline__ T shared_element(uint32_t at)
{
    T v;
    if constexpr (sizeof(T) == 4) {
        asm volatile("ld.shared.f32 %0, [%1];" : "=f"(reinterpret_cast<float&>(v)) : "r"(at) : "memory");
    } else {
        asm volatile("ld.shared.u16 %0, [%1];" : "=h"(reinterpret_cast<uint16_t&>(v)) : "r"(at) : "memory");
    }
    return v;
}

// p of one column in 64 bits, from memory.
template <Q8RowOp OP, typename T, typename W>
__device__ double exact_value(const Q8Rows& a, size_t row, int col, double* s_out = nullptr)
{
    if constexpr (OP == Q8_SILU_MUL) {
        const double g = to_float(static_cast<const T*>(a.x)[row * a.x_ld + col]), u = to_float(static_cast<const T*>(a.r)[row * a.r_ld + col]);
        return gated_in_64(g, u);
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
__device__ __forceinline__ bool product_of_non_zeros(const Q8Rows& a, size_t row, int col)
{
    const float x = to_float(OP == Q8_RMSNORM && a.r ? static_cast<const T*>(a.s)[row * a.s_ld + col] : static_cast<const T*>(a.x)[row * a.x_ld + col]);
    if constexpr (OP == Q8_SILU_MUL) return x != 0.f && to_float(static_cast<const T*>(a.r)[row * a.r_ld + col]) != 0.f;
    if constexpr (OP == Q8_RMSNORM) return x != 0.f && to_float(static_cast<const W*>(a.weight)[col]) != 0.f;
    return x != 0.f;
}

constexpr float kRound = 12582912.f;   // adding 1.5 * 2^23 rounds to an integer, whose low byte is then the sum's

// Distance of p * inv to the nearest integer plus the error that goes with the integer (see kBorder); the low byte of *k is the integer's.
template <Q8RowOp OP>
__device__ __forceinline__ float border_of(float p, float inv, uint32_t* k)
{
    const float n = fmaf(p, inv, kRound), whole = n - kRound;
    *k = __float_as_uint(n);
    return fmaf(fabsf(whole), 2.f * kError<OP>, fabsf(fmaf(p, inv, -whole)));   // (the maximum's error beside p's)
}
// One column's integer, which 32 bits left open, in 64 bits; top = 0: |p| itself instead.  x_at, r_at: where the column's inputs
// lie in shared memory (0: read them from global memory, which takes longer).
template <Q8RowOp OP, typename T, typename W>
__device__ __noinline__ double again(const Q8Rows& a, size_t row, int col, uint32_t x_at, uint32_t r_at, double top)
{
    double p;
    if (x_at == 0u) {
        p = exact_value<OP, T, W>(a, row, col);
    } else {
        const T x = shared_element<T>(x_at);
        if constexpr (OP == Q8_RMSNORM) {
            const T s = a.r ? from_float<T>(to_float(x) + to_float(shared_element<T>(r_at))) : x;
            p = static_cast<double>(to_float(s)) * static_cast<double>(to_float(static_cast<const W*>(a.weight)[col]));
        } else if constexpr (OP == Q8_SILU_MUL) {
            p = gated_in_64(to_float(x), to_float(shared_element<T>(r_at)));
        } else {
            p = to_float(x);
        }
    }
    if (top == 0.0) return fabs(p);
    a.q[row * a.q_ld + col] = static_cast<int8_t>(rint(127.0 * p / top));
    return 0.0;
}
// Elements of a group for which `f` holds, a bit each.
template <typename F>
__device__ __forceinline__ uint32_t which(const Pair (&p)[4], F&& f)
{
    uint32_t bits = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float lo, hi;
        split(p[i], lo, hi);
        bits |= (f(lo) ? 1u : 0u) << (2 * i) | (f(hi) ? 2u : 0u) << (2 * i);
    }
    return bits;
}

// (a multiple of 128 bytes: the copied pieces lie behind it, and off a 128-byte boundary a warp's 512 bytes take a pass more: 8192 x 8192
// bf16 with residual 104 us instead of 90)
struct alignas(128) Scratch {
    unsigned long long top64;   // bits of the maximum in 64 bits
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
template <Q8RowOp OP, typename T, typename W, int TPR, bool VEC>
__device__ __noinline__ void row_in_64(const Q8Rows& a, size_t row, int t, bool zero, Scratch* sc)
{
    using G = Group<TPR, VEC>;
    if (zero) {
        // every product is 0 in 32 bits: usually a row of padding.  It is one of zeros if every product has a factor 0
        int some = 0;
        for (int v = t;; v += TPR) {
            const G g(v, a.h);
            if (g.count <= 0) break;
            for (int e = 0; e < min(g.count, 8); ++e) some |= product_of_non_zeros<OP, T, W>(a, row, g.first + e * G::step);
        }
        if constexpr (TPR > 32) some = __syncthreads_or(some);
        else some = __any_sync(0xFFFFFFFFu, some);
        if (!some) {
            if (t == 0) a.scale[row] = 0.f;
            for (int v = t;; v += TPR) {
                const G g(v, a.h);
                if (g.count <= 0) break;
                int8_t* q = a.q + row * a.q_ld + g.first;
                if (VEC && g.count >= 8) *reinterpret_cast<uint2*>(q) = make_uint2(0u, 0u);
                else for (int e = 0; e < min(g.count, 8); ++e) q[e * G::step] = 0;
            }
            return;
        }
    }
    double top = 0.0, sum = 0.0;
    int bad = 0;
    for (int v = t;; v += TPR) {
        const G g(v, a.h);
        if (g.count <= 0) break;
        for (int e = 0; e < min(g.count, 8); ++e) {
            double s = 0.0;
            const double p = exact_value<OP, T, W>(a, row, g.first + e * G::step, &s);
            bad |= !(fabs(p) <= 1e300) || !(fabs(s) <= 1e300);
            top = fmax(top, fabs(p));
            sum += s * s;
        }
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
    for (int v = t;; v += TPR) {
        const G g(v, a.h);
        if (g.count <= 0) break;
        for (int e = 0; e < min(g.count, 8); ++e) {
            const int c = g.first + e * G::step;
            a.q[row * a.q_ld + c] =
                good && top > 0.0 ? static_cast<int8_t>(rint(127.0 * exact_value<OP, T, W>(a, row, c) / top)) : static_cast<int8_t>(0);
        }
    }
}

// TPR threads take a row, each NV groups of eight columns, in steps of TPR groups.  KEEP: the row's p stay in registers (8 * NV * TPR >= h).
// (at least 768 threads an SM)
// TWO: two tensors are read (silu_mul, rmsnorm with a residual).  SLOTS: rows in shared memory at a time (0: none, straight to registers).
template <Q8RowOp OP, bool TWO, typename T, typename W, int TPR, int NV, bool KEEP, bool VEC, int SLOTS>
__global__ void __launch_bounds__(TPR < 128 ? 128 : TPR, TPR < 128 ? 6 : TPR > 768 ? 1 : 768 / TPR) k_q8_rows(const __grid_constant__ Q8Rows a)
{
    constexpr int ROWS = TPR < 128 ? 128 / TPR : 1;
    static_assert(TPR == 32 || ROWS == 1, "a row is a warp's or a block's");
    // products of two 16-bit values fit 32 bits, an input is itself
    constexpr bool EXACT = OP == Q8_ROWS || (OP == Q8_RMSNORM && sizeof(T) == 2 && sizeof(W) == 2);
    // p of at most 16 bits: 127 p is exact in 32, and 127 p / a is a half or further from it than fp32's half a place: 254 p - (2k + 1) a
    // is a multiple of p's last place, more than 2^-16 p, and that over 2 a is more than 2^-24 of the quotient
    constexpr bool DIVIDE = sizeof(T) == 2 && (OP == Q8_ROWS || (OP == Q8_RMSNORM && std::is_same_v<T, __nv_bfloat16> && sizeof(W) == 2));
    constexpr bool ASYNC = SLOTS > 0;
    using G = Group<TPR, VEC>;
    static_assert(!ASYNC || (KEEP && VEC), "copied pieces are read once, 16 bytes at a time");
    extern __shared__ uint4 smem[];
    __shared__ Scratch scratch[2];   // rows take turns: a row's is written after the barrier behind the last reading of it
    const int t = threadIdx.x % TPR;
    const size_t tokens = static_cast<size_t>(a.tokens), step = static_cast<size_t>(gridDim.x) * ROWS;
    const W* weight = static_cast<const W*>(a.weight);
    nmk::pdl_launch_dependents();
    nmk::pdl_wait();
    // ASYNC: a thread copies its part of the next row into places of its own in shared memory while this row is reduced and written
    // (no barrier, no registers; two sets of places taken in turn, one where a row is too long for two)
    constexpr int PIECES = sizeof(T) / 2, THREADS = TPR < 128 ? 128 : TPR;
    uint4* const places = smem + threadIdx.x;
    auto place = [&](int turn, int tensor, int i, int piece) {
        return places + (((SLOTS == 2 ? turn : 0) * (TWO ? 2 : 1) + tensor) * NV * PIECES + i * PIECES + piece) * THREADS;
    };
    const int left = a.h - t * 8;   // columns from this thread's first group on
    auto fetch = [&](size_t row, int turn) {
        const T* x = static_cast<const T*>(a.x) + row * a.x_ld + t * 8;
        const T* r = static_cast<const T*>(a.r) + (TWO ? row * a.r_ld + t * 8 : 0);
        const uint32_t to = nmk::smem_u32(place(turn, 0, 0, 0));
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (left <= i * TPR * 8) continue;
#pragma unroll
            for (int piece = 0; piece < PIECES; ++piece) {
                // zeros behind the last column (of a group of fp32 numbers the second piece may be all behind it: nothing is read then)
                const int bytes = (left - i * TPR * 8) * static_cast<int>(sizeof(T)) - piece * 16;
                const uint32_t some = PIECES == 1 ? min(bytes, 16) : max(min(bytes, 16), 0);
                const int from = PIECES == 1 || some ? i * TPR * 8 + piece * (16 / static_cast<int>(sizeof(T))) : 0;
                nmk::cp_async16(to + (i * PIECES + piece) * THREADS * 16, x + from, some);
                if (TWO) nmk::cp_async16(to + ((NV + i) * PIECES + piece) * THREADS * 16, r + from, some);
            }
        }
    };
    auto fetched = [&](int turn, int tensor, int i) {
        Eight<T> e;
#pragma unroll
        for (int piece = 0; piece < PIECES; ++piece) {
            reinterpret_cast<uint4*>(&e)[piece] = *place(turn, tensor, i, piece);
        }
        return e;
    };
    // 16-bit weights stay in registers from row to row
    constexpr bool HELD = ASYNC && OP == Q8_RMSNORM && sizeof(W) == 2 && TPR < 1024;
    Eight<W> held[HELD ? NV : 1];
    if constexpr (HELD) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (left > i * TPR * 8) held[i] = load8<W, VEC, 1>(weight + t * 8 + i * TPR * 8, left - i * TPR * 8);
    }
    // (whole rows leave: ROWS > 1 has no barrier across warps)
    size_t row = static_cast<size_t>(blockIdx.x) * ROWS + threadIdx.x / TPR;
    if constexpr (SLOTS == 2) {
        if (row < tokens) fetch(row, 0);
        nmk::cp_async_commit();
    }
    const size_t first_row = row;
    bool set_aside = false;
    for (int turn = 0; row < tokens; row += step, turn ^= 1) {
    Scratch* sc = scratch + turn;
    const T* x = static_cast<const T*>(a.x) + row * a.x_ld;
    const T* r = TWO ? static_cast<const T*>(a.r) + row * a.r_ld : nullptr;
    T* s_row = OP == Q8_RMSNORM && TWO ? static_cast<T*>(a.s) + row * a.s_ld : nullptr;

    Pair p[KEEP ? NV : 1][4];
    Pair sum2 = 0;
    float top = 0.f;   // max |p|, NaN if one is
    // p of the group `v`; `first`: sums, and the residual's addition is written
    auto values = [&](int v, Pair (&out)[4], const Eight<T>& ex, const Eight<T>& er, const Eight<W>& ew, bool first) {
        if constexpr (OP == Q8_RMSNORM) {
            Eight<T> es = ex;
            if (TWO && first) {
                es = add8<T>(ex, er);
                const G g(v, a.h);
                store8<T, VEC, G::step>(s_row + g.first, es, g.count);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const Pair s = two_of(es, i);
                if (first) sum2 = fma2(s, s, sum2);
                out[i] = mul2(s, two_of(ew, i));
            }
        } else if constexpr (OP == Q8_SILU_MUL) {
            float most = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                Pair product;
                gated(two_of(ex, i), two_of(er, i), &product, &out[i]);
                float lo, hi;
                split(product, lo, hi);
                most = top3(most, lo, hi);
            }
            if (!(most <= kMostProduct)) top = NAN;   // (the row goes to 64 bits)
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) out[i] = two_of(ex, i);
        }
        if (first) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {   // (columns past the end are zeros)
                float lo, hi;
                split(out[i], lo, hi);
                top = top3(top, lo, hi);
            }
        }
    };
    auto pass = [&](int base, bool first, auto&& use) {
        Eight<T> ex[NV], er[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const G g(base + i * TPR, a.h);
            if (g.count <= 0) continue;
            // the second reading of a norm's row finds the sum in memory
            const T* from = OP == Q8_RMSNORM && TWO && !first ? s_row : x;
            ex[i] = load8<T, VEC, G::step>(from + g.first, g.count);
            if (TWO && (OP == Q8_SILU_MUL || first)) er[i] = load8<T, VEC, G::step>(r + g.first, g.count);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = base + i * TPR;
            const G g(v, a.h);
            if (g.count <= 0) continue;
            Eight<W> ew;
            if (OP == Q8_RMSNORM) ew = load8<W, VEC, G::step>(weight + g.first, g.count);   // (out of the L1: every row reads them)
            Pair tmp[4];
            values(v, tmp, ex[i], er[i], ew, first);
            use(i, v, tmp);
        }
    };
    // groups of a row that is read again: this thread's `base`, base + NV * TPR, ...
    auto begins = [&](int base) { return G(base, a.h).count > 0; };
    if constexpr (ASYNC) {
        if constexpr (SLOTS == 2) {
            if (row + step < tokens) fetch(row + step, turn ^ 1);
        } else {
            fetch(row, 0);
        }
        nmk::cp_async_commit();
        nmk::cp_async_wait<SLOTS - 1>();
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            Eight<T> er = {};
            Eight<W> ew = {};
            if (left <= i * TPR * 8) continue;
            if (HELD) ew = held[HELD ? i : 0];
            else if (OP == Q8_RMSNORM) ew = load8<W, VEC, 1>(weight + t * 8 + i * TPR * 8, left - i * TPR * 8);   // (out of the L1: every row reads them)
            if (TWO) er = fetched(turn, 1, i);
            values(t + i * TPR, p[i], fetched(turn, 0, i), er, ew, true);
        }
    } else if constexpr (KEEP) {
        pass(t, true, [&](int i, int, Pair (&f)[4]) {
#pragma unroll
            for (int e = 0; e < 4; ++e) p[i][e] = f[e];
        });
    } else {
        for (int base = t; begins(base); base += NV * TPR) pass(base, true, [](int, int, Pair (&)[4]) {});
    }

    float sum = 0.f;
    if constexpr (OP == Q8_RMSNORM) {
        float lo, hi;
        split(sum2, lo, hi);
        sum = lo + hi;
        for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
        if (!(sum <= kMostSum)) top = NAN;   // (the row goes to 64 bits; 32 sums below the bound do not overflow)
    }
    // as bits: NaN above infinity above numbers
    uint32_t top_bits = __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(top) & 0x7FFFFFFFu);
    if constexpr (TPR > 32) {
        if ((t & 31) == 0) {
            sc->sum[t >> 5] = sum;
            sc->top[t >> 5] = top_bits;
        }
        if (!EXACT && t == 0) sc->top64 = 0ull;
        __syncthreads();
        const int lane = t & 31;
        top_bits = __reduce_max_sync(0xFFFFFFFFu, lane < TPR / 32 ? sc->top[lane] : 0u);
        if (OP == Q8_RMSNORM && t < 32) {   // (only the first thread wants it)
            sum = lane < TPR / 32 ? sc->sum[lane] : 0.f;
            for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
        }
    }
    const float a32 = __uint_as_float(top_bits);
    // kLeastTop: what 32 bits lose below 2^-126 is then less than a step by far
    if (!(a32 >= kLeastTop && a32 <= kMostTop)) {
        // (after the others: a call in here would cost the loop registers)
        set_aside = true;
        if (t == 0) a.scale[row] = a32 == 0.f ? -2.f : -1.f;
        continue;
    }
    // (element `at` of this thread's part: group at / 8, column at % 8 of it)
    auto column_of = [&](int v0, int at) { return G(v0 + at / 8 * TPR, a.h).first + at % 8 * G::step; };
    auto input_at = [&](int tensor, int at) {
        return ASYNC ? nmk::smem_u32(place(turn, TWO ? tensor : 0, at / 8, at % 8 / (8 / PIECES))) + static_cast<uint32_t>(at % (8 / PIECES) * sizeof(T)) : 0u;
    };
    double a64 = a32;
    if constexpr (!EXACT) {
        const float near_top = a32 * (1.f - 2.f * kError<OP>);
        double mine = 0.0;
        auto is_near = [&](float v) { return fabsf(v) >= near_top; };
        // (KEEP: one loop over all groups' bits, so that there is one call; a lane or two of the row have any)
        auto look = [&](uint32_t bits, int v0) {
            for (; bits; bits &= bits - 1u) {
                const int at = __ffs(bits) - 1;
                mine = fmax(mine, again<OP, T, W>(a, row, column_of(v0, at), input_at(0, at), input_at(1, at), 0.0));
            }
        };
        if (top < near_top) {
            // none of this thread's
        } else if constexpr (KEEP) {
            uint32_t bits = 0u;
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (begins(t + i * TPR)) bits |= which(p[i], is_near) << (8 * i);
            look(bits, t);
        } else {
            for (int base = t; begins(base); base += NV * TPR)
                pass(base, false, [&](int, int v, Pair (&f)[4]) { look(which(f, is_near), v); });
        }
        // The maximum in 64 bits decides only where 32 leave a quotient open: it is collected while all threads go on with the one in 32
        // (of a row that is read again at once, for the decisions are made on the way)
        if constexpr (TPR == 32) {
            a64 = warp_max(mine);
        } else {
            if (mine > 0.0) atomicMax(&sc->top64, static_cast<unsigned long long>(__double_as_longlong(mine)));
            if constexpr (!KEEP) {
                __syncthreads();
                a64 = __longlong_as_double(static_cast<long long>(sc->top64));
            }
        }
    }
    auto write_scale = [&] {
        if (t != 0) return;
        float scale = EXACT ? a32 / 127.f : static_cast<float>(a64 / 127.0);
        if constexpr (OP == Q8_RMSNORM) scale *= 1.f / sqrtf(sum / static_cast<float>(a.h) + a.eps);
        a.scale[row] = scale < INFINITY ? scale : NAN;
    };
    if (EXACT) write_scale();
    const float rcp = __frcp_rn(a32), inv = 127.f * rcp;
    int8_t* q_row = a.q + row * a.q_ld;
    // q of the group `v`; a bit for each that 64 bits have to decide
    auto quantise = [&](int v, Pair (&f)[4]) {
        uint32_t k[8];
        float border = 0.f;
        if constexpr (DIVIDE) {
            // 127 p / a, rounded correctly (Markstein: a quotient from the reciprocal, its remainder by fma, one correction), and
            // that to an integer: a quotient between two halves keeps its side, a tie is exact (see DIVIDE)
            const Pair r = pair(rcp, rcp), minus_a = pair(-a32, -a32);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float lo, hi;
                split(f[i], lo, hi);
                const Pair t = pair(127.f * lo, 127.f * hi), y = mul2(t, r);
                split(fma2(fma2(y, minus_a, t), r, y), lo, hi);
                k[2 * i] = __float_as_uint(lo + kRound);
                k[2 * i + 1] = __float_as_uint(hi + kRound);
            }
        } else {
            // the nearest integer to p * inv, and how far off that is: within the error bound of a half, 64 bits decide
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float lo, hi;
                split(f[i], lo, hi);
                border = top3(border, border_of<OP>(lo, inv, &k[2 * i]), border_of<OP>(hi, inv, &k[2 * i + 1]));
            }
        }
        const uint32_t lo = __byte_perm(__byte_perm(k[0], k[1], 0x0040), __byte_perm(k[2], k[3], 0x0040), 0x5410);
        const uint32_t hi = __byte_perm(__byte_perm(k[4], k[5], 0x0040), __byte_perm(k[6], k[7], 0x0040), 0x5410);
        const G g(v, a.h);
        if (VEC && g.count >= 8) {
            *reinterpret_cast<uint2*>(q_row + g.first) = make_uint2(lo, hi);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < g.count) q_row[g.first + e * G::step] = static_cast<int8_t>((e < 4 ? lo >> (8 * e) : hi >> (8 * (e - 4))) & 0xFFu);
        }
        return border > kBorder<OP> ? which(f, [&](float p) {
            uint32_t unused;
            return border_of<OP>(p, inv, &unused) > kBorder<OP>;
        }) : 0u;
    };
    auto decide = [&](uint32_t bits, int v0) {
        for (; bits; bits &= bits - 1u) {
            const int at = __ffs(bits) - 1, col = column_of(v0, at);
            if (col < a.h) again<OP, T, W>(a, row, col, input_at(0, at), input_at(1, at), a64);
        }
    };
    if constexpr (KEEP) {
        uint32_t open = 0u;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (begins(t + i * TPR)) open |= quantise(t + i * TPR, p[i]) << (8 * i);
        if constexpr (!EXACT && TPR > 32) {
            __syncthreads();
            a64 = __longlong_as_double(static_cast<long long>(sc->top64));
        }
        if constexpr (!DIVIDE) decide(open, t);
    } else {
        for (int base = t; begins(base); base += NV * TPR)
            pass(base, false, [&](int, int v, Pair (&f)[4]) {
                const uint32_t open = quantise(v, f);
                if constexpr (!DIVIDE) decide(open, v);
            });
    }
    if (!EXACT) write_scale();
    }
    if (!set_aside) return;
    if constexpr (TPR > 32) __syncthreads();
    else __syncwarp();
    for (row = first_row; row < tokens; row += step) {
        const float mark = *reinterpret_cast<volatile float*>(a.scale + row);
        if constexpr (TPR > 32) __syncthreads();   // (its first thread replaces the mark, and the scratch is used again)
        else __syncwarp();
        if (mark < 0.f) row_in_64<OP, T, W, TPR, VEC>(a, row, t, mark == -2.f, scratch);
    }
}

template <Q8RowOp OP, bool TWO, typename T, typename W, int TPR, int NV, bool KEEP, bool VEC, int SLOTS>
cudaError_t launch_one(const Q8Rows& a, cudaStream_t st)
{
    constexpr int rows = TPR < 128 ? 128 / TPR : 1, threads = TPR < 128 ? 128 : TPR;
    const int blocks = (a.tokens + rows - 1) / rows;
    // as many blocks as an SM holds for certain (768 threads, 227 KB)
    constexpr size_t smem = static_cast<size_t>(threads) * NV * 8 * sizeof(T) * SLOTS * (TWO ? 2 : 1);
    int resident = threads > 768 ? 1 : 768 / threads;
    if (smem && 225 * 1024 / (smem + 3 * 1024) < static_cast<size_t>(resident)) resident = static_cast<int>(225 * 1024 / (smem + 3 * 1024));
    resident *= nmhost::sm_count();
    auto kernel = k_q8_rows<OP, TWO, T, W, TPR, NV, KEEP, VEC, SLOTS>;
    const cudaError_t e = nmhost::ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), smem);
    if (e != cudaSuccess) return e;
    return nmhost::launch_pdl(kernel, static_cast<unsigned>(blocks < resident ? blocks : resident), static_cast<unsigned>(threads), smem, st, a);
}

// Threads for a row, four groups of eight columns each (two of 32-bit numbers); fewer groups, of more threads, where there are too few rows
// to fill the GPU: 333 x 1001 fp32 (rows off the 16-byte boundaries) a block of 256 to a row 3.2 us, a warp 7.8; 4096 x 1001 bf16 21 and 16.5.
template <Q8RowOp OP, bool TWO, typename T, typename W>
cudaError_t launch_shape(const Q8Rows& a, bool vec, cudaStream_t st)
{
#define NM_ROWS(TPR, NV, KEEP, VEC, SLOTS) launch_one<OP, TWO, T, W, TPR, NV, KEEP, VEC, SLOTS>(a, st)
    const bool few = a.tokens <= 2 * nmhost::sm_count();
    if (!vec) {
        if (a.h <= 512) return NM_ROWS(32, 2, true, false, 0);
        if (a.h <= 4096 && a.tokens <= 6 * nmhost::sm_count()) return NM_ROWS(256, 2, true, false, 0);
        if (a.h <= 1024) return NM_ROWS(32, 4, true, false, 0);
        if (a.h <= 4096) return NM_ROWS(128, 4, true, false, 0);
        if (a.h <= 8192) return NM_ROWS(256, 4, true, false, 0);
        if (a.h <= 16384) return NM_ROWS(512, 4, true, false, 0);
        return NM_ROWS(512, 2, false, false, 0);
    }
    if (a.h <= 512) return NM_ROWS(32, 2, true, true, 2);
    if (a.h <= 2048 && !few) return NM_ROWS(128, 2, true, true, 2);
    if (few) {
        if (a.h <= 4096) return NM_ROWS(512, 1, true, true, 2);
        if (a.h <= 8192) return NM_ROWS(1024, 1, true, true, 2);
    }
    if constexpr (sizeof(T) == 4) {
        if (a.h <= 4096) return NM_ROWS(256, 2, true, true, 2);
        if (a.h <= 8192) return NM_ROWS(512, 2, true, true, 2);
        if (a.h <= 12288) return NM_ROWS(768, 2, true, true, 2);
        if (a.h <= 16384) return NM_ROWS(1024, 2, true, true, 1);
    } else {
        if (few && a.h <= 16384) return NM_ROWS(1024, 2, true, true, 2);
        if (a.h <= 4096) return NM_ROWS(128, 4, true, true, 2);
        if (a.h <= 8192) return NM_ROWS(256, 4, true, true, 2);
        if (a.h <= 12288) return NM_ROWS(384, 4, true, true, 2);
        if (a.h <= 16384) return NM_ROWS(512, 4, true, true, 2);
        if (a.h <= 32768) return NM_ROWS(1024, 4, true, true, 1);
    }
    return NM_ROWS(512, 2, false, true, 0);
#undef NM_ROWS
}

template <typename T>
nm_status_t launch(Q8RowOp op, const Q8Rows& a, nm_dtype_t weight_type, bool vec, cudaStream_t st)
{
    cudaError_t e;
    const bool wide = sizeof(T) == 2 && weight_type == NM_F32;
    if (op == Q8_SILU_MUL) e = launch_shape<Q8_SILU_MUL, true, T, T>(a, vec, st);
    else if (op == Q8_ROWS) e = launch_shape<Q8_ROWS, false, T, T>(a, vec, st);
    else if (a.r) e = wide ? launch_shape<Q8_RMSNORM, true, T, float>(a, vec, st) : launch_shape<Q8_RMSNORM, true, T, T>(a, vec, st);
    else e = wide ? launch_shape<Q8_RMSNORM, false, T, float>(a, vec, st) : launch_shape<Q8_RMSNORM, false, T, T>(a, vec, st);
    nmhost::count_launch(1);
    if (e == cudaSuccess) e = cudaGetLastError();
    if (e != cudaSuccess) return nmhost::fail(NM_ERR_CUDA, "8-bit row kernel launch: %s", cudaGetErrorString(e));
    return NM_OK;
}

}  // namespace q8rows
