// Product of a few tokens (up to 8) with column-wise N:M pruned 8-bit weights: only the retained weights are read, once.
//
// A layer's retained weights are c_out * kk bytes, a microsecond or two of memory traffic, and a call is bound by what else stands
// in series with them: launch, gather, sums, store.  So a block is short: 16 or 32 rows of one pruning tile, whose columns they
// share, all columns (no second block to wait for), eight warps that share the columns.  It
//   - has a warp's first four loads of weights on their way before the kernel before has ended (they do not depend on it),
//   - gathers the activations of the tile's columns into shared memory, four columns of a token at a time, by byte permutations of
//     aligned eights where the four lie in one or two (1:4, 2:4, 3:4, 2:8, 4:8), and
//   - adds the products up as integers, per warp, then over the warps, in a fixed order.
// Up to four tokens by dp4a; more by mma.sync on fp16 numbers, 16 rows x 8 tokens x 16 columns: 8-bit integers are exact in fp16,
// and so is the sum of 1024 products in fp32 (1024 * 2^14 = 2^24), after which a warp adds it to its integers.  (On 8-bit integers
// mma.sync runs at a fraction of that rate.)
#include <algorithm>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "nm_ptx.cuh"
#include "nm_q8.h"

namespace {

using namespace nmk;

constexpr int WARPS = 8, THREADS = 32 * WARPS;
constexpr int CHUNK = 64;   // columns a warp takes at a time: 16 bytes a lane, four lanes a row

struct FewArgs {
    const int8_t* packed;
    const uint16_t* indices;
    const float* w_scale;
    const int8_t* x;
    long long x_ld;
    const float* x_scale;
    const float* bias;
    void* y;
    long long y_ld;
    int y_type;
    int tokens, c_out, k, kk_ld, tile_t, units;
    int groups;     // blocks of rows in a tile
    int pitch;      // bytes of a token's row in shared memory
};

__device__ __forceinline__ uint4 load_weights(const int8_t* p)
{
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
// Four 8-bit integers as fp16 numbers: a byte with the sign bit turned over, under the exponent of 1024, is 1024 + 128 + the integer.
__device__ __forceinline__ void halves_of(uint32_t v, uint32_t& lo, uint32_t& hi)
{
    const uint32_t u = v ^ 0x80808080u, bias = 0x64806480u;   // 1152, twice
    const uint32_t a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(lo) : "r"(a), "r"(bias));
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(hi) : "r"(b), "r"(bias));
}
__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint4 load_shared16(uint32_t at)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}

// Columns 4 quad .. 4 quad + 3 of the tile's retained ones, of all tokens, to `store(token, four bytes)`; BATCH tokens on their
// way at a time.  `from`: their places (unused where every column is retained).
template <bool DENSE, int BATCH, typename S>
__device__ __forceinline__ void gather_quad(const FewArgs& g, int quad, uint2 from, S&& store)
{
    const int8_t* x = g.x;
    auto take = [&](auto&& load) {
        for (int token = 0; token < g.tokens; token += BATCH, x += BATCH * g.x_ld) {
            uint32_t v[BATCH];
#pragma unroll
            for (int i = 0; i < BATCH; ++i)
                if (i == 0 || token + i < g.tokens) v[i] = load(x + i * g.x_ld);
#pragma unroll
            for (int i = 0; i < BATCH; ++i)
                if (i == 0 || token + i < g.tokens) store(token + i, v[i]);
        }
    };
    if constexpr (DENSE) {
        const int col = quad * 4;
        if (col + 4 <= g.k) {
            take([&](const int8_t* p) { return *reinterpret_cast<const uint32_t*>(p + col); });
        } else {
            take([&](const int8_t* p) {
                uint32_t v = 0u;
                for (int b = 0; b < 4; ++b)
                    if (col + b < g.k) v |= (static_cast<uint32_t>(p[col + b]) & 0xFFu) << (8 * b);
                return v;
            });
        }
    } else {
        // (column 0 behind the last one: its weights are zeros)
        const uint32_t c[4] = {from.x & 0xFFFFu, from.x >> 16, from.y & 0xFFFFu, from.y >> 16};
        const bool inside = static_cast<int>(max(max(c[0], c[1]), max(c[2], c[3])) | 7u) < g.k;   // (whole aligned eights are read)
        const uint32_t a_sel = (c[0] & 7u) | (c[1] & 7u) << 4, b_sel = (c[2] & 7u) | (c[3] & 7u) << 4;
        const bool a_one = c[0] >> 3 == c[1] >> 3, b_one = c[2] >> 3 == c[3] >> 3;
        if (inside && a_one && b_one && c[0] >> 3 == c[2] >> 3) {   // 2:4, 4:8
            const uint32_t at = c[0] & ~7u, sel = a_sel | b_sel << 8;
            take([&](const int8_t* p) {
                const uint2 w = *reinterpret_cast<const uint2*>(p + at);
                return __byte_perm(w.x, w.y, sel);
            });
        } else if (inside && a_one && b_one) {   // 1:4, 3:4, 2:8
            const uint32_t at = c[0] & ~7u, bt = c[2] & ~7u;
            take([&](const int8_t* p) {
                const uint2 w = *reinterpret_cast<const uint2*>(p + at), z = *reinterpret_cast<const uint2*>(p + bt);
                return __byte_perm(__byte_perm(w.x, w.y, a_sel), __byte_perm(z.x, z.y, b_sel), 0x5410);
            });
        } else {
            take([&](const int8_t* p) {
                return (static_cast<uint32_t>(p[c[0]]) & 0xFFu) | (static_cast<uint32_t>(p[c[1]]) & 0xFFu) << 8 |
                       (static_cast<uint32_t>(p[c[2]]) & 0xFFu) << 16 | static_cast<uint32_t>(p[c[3]]) << 24;
            });
        }
    }
}

// TOKENS: 1, 2, 4 by dp4a; 8 by mma.sync.  UNITS: groups of eight rows, 2 or 4.  DENSE: every column is retained.
// Two or three blocks an SM: with the registers of two and all four loads ahead 4096 -> 4096 at 2:4 takes 3.5 us for four tokens and 4.2 for
// eight, with those of three 4.3 and 5.8; the wide form, which runs many blocks, wants three of them and fewer loads ahead
// (4096 -> 12288: 6.7 and 7.5 against 9.4 and 11).
template <int TOKENS, int UNITS, bool DENSE>
__global__ void __launch_bounds__(THREADS, TOKENS > 2 && UNITS == 2 ? 2 : 3) k_q8_few(const FewArgs g)
{
    constexpr bool MMA = TOKENS >= 8;
    constexpr int ROWS = 8 * UNITS, DEPTH = UNITS == 2 ? 4 : TOKENS <= 2 ? 2 : 1;
    constexpr int EXACT_CHUNKS = 16;  // columns whose products fp32 adds up exactly, in chunks
    extern __shared__ uint4 smem[];   // activations of the tile's columns [tokens][pitch]: 8-bit for dp4a, fp16 for mma.sync
    __shared__ int s_sum[WARPS][TOKENS][ROWS];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int tile = static_cast<int>(blockIdx.x) / g.groups, unit0 = static_cast<int>(blockIdx.x) % g.groups * UNITS;
    const int n_units = min(UNITS, g.units - unit0);
    const int row0 = tile * g.tile_t + unit0 * 8, row_end = min(g.c_out, (tile + 1) * g.tile_t);
    const int chunks = g.kk_ld / CHUNK;
    const int r = lane >> 2, t = lane & 3;   // row of a unit (of the weights), or token of a group; quarter of a chunk

    const int8_t* w = g.packed + static_cast<size_t>(tile * g.units + unit0) * chunks * 512 + lane * 16;
    const size_t unit_bytes = static_cast<size_t>(chunks) * 512;
    uint4 ring[DEPTH][UNITS];
    auto fetch = [&](uint4 (&to)[UNITS], int c) {
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            to[u] = make_uint4(0u, 0u, 0u, 0u);
            if (c < chunks && u < n_units) to[u] = load_weights(w + u * unit_bytes + static_cast<size_t>(c) * 512);
        }
    };
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) fetch(ring[d], warp + d * WARPS);
    const int quads = chunks * (CHUNK / 4);
    const uint32_t xs = smem_u32(smem);
    const uint2* idx = reinterpret_cast<const uint2*>(g.indices + static_cast<size_t>(tile) * g.kk_ld);
    uint2 from[2];   // (of the handle too)
#pragma unroll
    for (int i = 0; i < 2; ++i) from[i] = !DENSE && tid + i * THREADS < quads ? __ldg(idx + tid + i * THREADS) : make_uint2(0u, 0u);
    pdl_launch_dependents();
    pdl_wait();

    // scales of the output this thread writes first
    const int out_token = tid / ROWS, out_row = row0 + tid % ROWS;
    const bool writes = out_token < g.tokens && out_row < row_end;
    const float xs0 = writes ? __ldg(g.x_scale + out_token) : 0.f, ws0 = writes ? __ldg(g.w_scale + out_row) : 0.f;
    const float bias0 = writes && g.bias ? __ldg(g.bias + out_row) : 0.f;
    auto gather = [&](int quad, uint2 places) {
        gather_quad<DENSE, TOKENS < 4 ? TOKENS : 4>(g, quad, places, [&](int token, uint32_t v) {
            if constexpr (MMA) {
                uint32_t lo, hi;
                halves_of(v, lo, hi);
                asm volatile("st.shared.v2.u32 [%0], {%1, %2};" ::"r"(xs + token * g.pitch + quad * 8), "r"(lo), "r"(hi) : "memory");
            } else {
                asm volatile("st.shared.u32 [%0], %1;" ::"r"(xs + token * g.pitch + quad * 4), "r"(v) : "memory");
            }
        });
    };
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if (tid + i * THREADS < quads) gather(tid + i * THREADS, from[i]);
    for (int quad = tid + 2 * THREADS; quad < quads; quad += THREADS) gather(quad, DENSE ? make_uint2(0u, 0u) : __ldg(idx + quad));
    __syncthreads();

    if constexpr (!MMA) {
        int acc[TOKENS][UNITS] = {};
        for (int c = warp; c < chunks; c += WARPS) {
            uint4 cur[UNITS];
#pragma unroll
            for (int u = 0; u < UNITS; ++u) {
                cur[u] = ring[0][u];
#pragma unroll
                for (int d = 0; d + 1 < DEPTH; ++d) ring[d][u] = ring[d + 1][u];
            }
            fetch(ring[DEPTH - 1], c + DEPTH * WARPS);
#pragma unroll
            for (int n = 0; n < TOKENS; ++n) {
                if (n > 0 && n >= g.tokens) break;
                const uint4 b = load_shared16(xs + n * g.pitch + c * CHUNK + t * 16);
#pragma unroll
                for (int u = 0; u < UNITS; ++u) {
                    int v = __dp4a(static_cast<int>(cur[u].x), static_cast<int>(b.x), acc[n][u]);
                    v = __dp4a(static_cast<int>(cur[u].y), static_cast<int>(b.y), v);
                    v = __dp4a(static_cast<int>(cur[u].z), static_cast<int>(b.z), v);
                    acc[n][u] = __dp4a(static_cast<int>(cur[u].w), static_cast<int>(b.w), v);
                }
            }
        }
#pragma unroll
        for (int n = 0; n < TOKENS; ++n)
#pragma unroll
            for (int u = 0; u < UNITS; ++u) {
                int v = acc[n][u];
                v += __shfl_xor_sync(0xFFFFFFFFu, v, 1);
                v += __shfl_xor_sync(0xFFFFFFFFu, v, 2);
                if (t == 0) s_sum[warp][n][u * 8 + r] = v;
            }
    } else {
        constexpr int MT = UNITS / 2;
        float acc[MT][4] = {};
        bool before = false;   // there are sums in s_sum
        auto add_up = [&] {
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    int& sum = s_sum[warp][t * 2 + (e & 1)][m * 16 + (e >> 1) * 8 + r];
                    sum = (before ? sum : 0) + __float2int_rn(acc[m][e]);
                    acc[m][e] = 0.f;
                }
            before = true;
        };
        int added = 0;
        for (int c = warp; c < chunks; c += WARPS) {
            uint4 cur[UNITS];
#pragma unroll
            for (int u = 0; u < UNITS; ++u) {
                cur[u] = ring[0][u];
#pragma unroll
                for (int d = 0; d + 1 < DEPTH; ++d) ring[d][u] = ring[d + 1][u];
            }
            fetch(ring[DEPTH - 1], c + DEPTH * WARPS);
            const uint32_t at = xs + r * g.pitch + (c * CHUNK + t * 16) * 2;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const uint4 b = r < g.tokens ? load_shared16(at + half * 16) : make_uint4(0u, 0u, 0u, 0u);
                __syncwarp();
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    uint32_t a0, a1, a2, a3;
                    halves_of(half ? cur[2 * m].z : cur[2 * m].x, a0, a2);
                    halves_of(half ? cur[2 * m + 1].z : cur[2 * m + 1].x, a1, a3);
                    mma_f16(acc[m], a0, a1, a2, a3, b.x, b.y);
                    halves_of(half ? cur[2 * m].w : cur[2 * m].y, a0, a2);
                    halves_of(half ? cur[2 * m + 1].w : cur[2 * m + 1].y, a1, a3);
                    mma_f16(acc[m], a0, a1, a2, a3, b.z, b.w);
                }
            }
            if (++added == EXACT_CHUNKS) {
                add_up();
                added = 0;
            }
        }
        add_up();
    }
    __syncthreads();
    for (int i = tid; i < g.tokens * ROWS; i += THREADS) {
        const int token = i / ROWS, row = row0 + i % ROWS;
        if (row >= row_end) continue;
        int sum = 0;
#pragma unroll
        for (int k = 0; k < WARPS; ++k) sum += s_sum[k][token][i % ROWS];
        const bool first = i == tid;
        const float v = fmaf(static_cast<float>(sum) * (first ? xs0 : __ldg(g.x_scale + token)), first ? ws0 : __ldg(g.w_scale + row),
                             first ? bias0 : g.bias ? __ldg(g.bias + row) : 0.f);
        const size_t place = static_cast<size_t>(token) * g.y_ld + row;
        if (g.y_type == NM_F32) static_cast<float*>(g.y)[place] = v;
        else if (g.y_type == NM_BF16) static_cast<__nv_bfloat16*>(g.y)[place] = __float2bfloat16_rn(v);
        else static_cast<__half*>(g.y)[place] = __float2half_rn(v);
    }
}

struct FewPlan {
    int tokens, units, groups, blocks, pitch;
    size_t smem;
};

// Which calls the kernel takes, and its rows a block.  Every block gathers all columns for its rows, so that the tokens it pays for go by
// its rows; against the tensor-memory kernel, us: 4096 -> 4096 at 2:4 in tiles of 64, one token 3.2 / 5.2, eight 4.4 / 5.2; in tiles of 8
// one token 5.9 / 5.1, but 1000 -> 1001 at 2:8 in tiles of 8 1.8 / 2.8; dense 4096 -> 4096, four tokens 5.5 / 6.8, eight 7.9 / 6.9;
// 8192 -> 2048 at 1:4, eight tokens 4.7 / 4.6.
// Blocks of 32 rows where 16 would be more than two an SM (4096 -> 12288 at 2:4: one token 5.5 us against 7.1, eight 7.5 against 12).
bool plan(const Q8Linear& p, FewPlan* f)
{
    const nm_q8_weights* w = p.w;
    const bool dense = w->n_keep == w->m_group;
    if (!w->packed || p.tokens > (dense || w->units < 2 ? 4 : 8)) return false;
    if (w->units < 2 && w->sparse && w->n_tiles > 2 * nmhost::sm_count()) return false;
    f->tokens = p.tokens <= 2 ? p.tokens : p.tokens <= 4 ? 4 : 8;
    const int tiles = dense ? 1 : w->n_tiles;
    f->units = w->units >= 4 && static_cast<long long>(tiles) * ((w->units + 1) / 2) > 2 * nmhost::sm_count() ? 4 : 2;
    f->groups = (w->units + f->units - 1) / f->units;
    if (static_cast<long long>(tiles) * f->groups > (1 << 24)) return false;
    f->blocks = tiles * f->groups;
    // (16 bytes more: a quarter warp's loads of fp16 numbers meet no bank twice)
    f->pitch = f->tokens >= 8 ? w->kk_ld * 2 + 16 : w->kk_ld;
    f->smem = static_cast<size_t>(p.tokens) * f->pitch;
    return f->smem <= 180 * 1024;
}

using Kernel = void (*)(FewArgs);
template <bool DENSE, int UNITS>
Kernel kernel_of(int tokens)
{
    switch (tokens) {
        case 1: return k_q8_few<1, UNITS, DENSE>;
        case 2: return k_q8_few<2, UNITS, DENSE>;
        case 4: return k_q8_few<4, UNITS, DENSE>;
        default: return k_q8_few<8, UNITS, DENSE>;
    }
}

}  // namespace

namespace nmhost {

bool q8_few_takes(const Q8Linear& p)
{
    FewPlan f;
    return plan(p, &f);
}

nm_status_t launch_q8_few(const Q8Linear& p, cudaStream_t st)
{
    const nm_q8_weights* w = p.w;
    FewPlan f;
    if (!plan(p, &f)) return fail(NM_ERR_UNSUPPORTED, "nm_q8_linear: too many tokens for the few-token kernel");
    const bool dense = w->n_keep == w->m_group;
    FewArgs g = {};
    g.packed = w->packed; g.units = w->units; g.indices = w->indices; g.w_scale = w->scales; g.x = p.x; g.x_ld = p.x_ld; g.x_scale = p.x_scale;
    g.bias = p.bias; g.y = p.y; g.y_ld = p.y_ld; g.y_type = p.y_type; g.tokens = p.tokens; g.c_out = w->c_out; g.k = w->k; g.kk_ld = w->kk_ld;
    g.tile_t = dense ? w->c_out : w->tile_t;
    g.groups = f.groups; g.pitch = f.pitch;
    const Kernel kernel = dense ? (f.units == 4 ? kernel_of<true, 4>(f.tokens) : kernel_of<true, 2>(f.tokens))
                                : (f.units == 4 ? kernel_of<false, 4>(f.tokens) : kernel_of<false, 2>(f.tokens));
    cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), f.smem);
    if (e != cudaSuccess) return fail(NM_ERR_CUDA, "nm_q8_linear: cudaFuncSetAttribute: %s", cudaGetErrorString(e));
    e = launch_pdl(kernel, static_cast<unsigned>(f.blocks), THREADS, f.smem, st, g);
    count_launch(1);
    if (e == cudaSuccess) e = cudaGetLastError();
    if (e != cudaSuccess) return fail(NM_ERR_CUDA, "nm_q8_linear launch (few tokens): %s", cudaGetErrorString(e));
    return NM_OK;
}

}  // namespace nmhost
