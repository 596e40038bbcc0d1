// Product of 8-bit activations with column-wise N:M pruned 8-bit weights on the tensor core (kind::i8, exact 32-bit sums).
//
//   D[channel][token] = sum over blocks of columns of  W[128 channels x block] * X[BN tokens x block]^T
//
// Weights are the M side (128 channels a tile), tokens the N side (16 to 128), so that a few tokens fill an instruction as well as
// many.  A block is 128 columns of the expanded weights, whose pruned columns are zeros, or, where a pattern keeps at most two of
// four aligned columns, 256 columns of the sparse form: the same 16 KB and 4 KB of places, which go to tensor memory, for the sparse
// instruction.  Either lies in memory as the shared-memory image, one bulk copy; activations come by TMA, zeros past the last
// column and token.
// Where there are far fewer tiles than SMs the reduction axis is split over the 2 or 4 CTAs of a cluster: each sends the runs of tokens
// that another finishes as one bulk copy into that CTA's shared memory.  Sums are integers: the result does not depend on the split.
//
//   producer (1 thread), MMA issuer (1 thread), epilogue (4 warps): sums through shared memory to rows of tokens, y = (sum * x_scale) * w_scale + bias
#include <algorithm>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "nm_ptx.cuh"
#include "nm_q8.h"
#include "nm_tmap.cuh"

namespace {

using namespace nmk;

constexpr int THREADS = 192;   // warps: 0 producer, 1 MMA issuer and tensor memory, 2-5 epilogue
constexpr int NSTAGE_MAX = 8;
constexpr int A_BYTES = 128 * 128;
constexpr int MOST_TOKENS = 128;   // of a tile; more than a round of such tiles is the pair kernel's
constexpr int PLACES = 4096;   // bytes of a sparse stage's places
constexpr int RING_ALONE = 224 * 1024 - 1024 - 2048, RING_SHARED = 112 * 1024 - 1024 - 2048;   // bytes for a CTA's ring, alone on its SM and beside another
// A tile's sums go through the ring, 512 bytes a token.  Two stages hold them, at any width, and every ring has two (a stage of sparse
// weights is the longer one; a cluster's CTA alone on its SM also holds the sums it receives).
static_assert(2 * (A_BYTES + MOST_TOKENS * 128) >= MOST_TOKENS * 512, "two stages hold a tile's sums");
static_assert(2 * (A_BYTES + PLACES + 2 * MOST_TOKENS * 128) <= RING_SHARED && RING_SHARED <= RING_ALONE - MOST_TOKENS * 512, "two stages fit");

struct GemmArgs {
    const int8_t* weights;     // expanded or sparse
    const uint8_t* places;
    const float* w_scale;
    const float* x_scale;
    const float* bias;
    void* y;
    long long y_ld;
    int* status;
    int tokens, c_out, rows;
    int blocks;   // of the reduction axis: 128 columns, 256 of sparse weights
    int c_tiles;
    int bn;
    int ks;       // CTAs of a cluster = ranges of the reduction axis
    int stages, stage_bytes;
    int tmem;     // columns of tensor memory
    int never_loaded;   // block from which on nothing is loaded, so that the wait for it expires (self-test); -1: none
};

template <typename T>
__device__ __forceinline__ T narrow(float v);
template <>
__device__ __forceinline__ float narrow<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 narrow<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ __half narrow<__half>(float v) { return __float2half_rn(v); }

template <typename T>
struct alignas(4 * sizeof(T)) Four {
    T v[4];
};
// Four channels of a token, the first `n` of which exist.
template <typename T>
__device__ __forceinline__ void put4(T* y, const float (&v)[4], int n, bool aligned)
{
    Four<T> f;
#pragma unroll
    for (int i = 0; i < 4; ++i) f.v[i] = narrow<T>(v[i]);
    if (aligned && n >= 4) {
        *reinterpret_cast<Four<T>*>(y) = f;
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < n) y[i] = f.v[i];
}
__device__ __forceinline__ int4 load_int4(uint32_t at)
{
    int4 v;
    asm volatile("ld.shared.v4.s32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
    return v;
}

template <typename T, bool SPARSE>
__global__ void __launch_bounds__(THREADS, 2) k_q8_gemm(const GemmArgs g, const __grid_constant__ CUtensorMap tm_x)
{
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t s_full[NSTAGE_MAX], s_free[NSTAGE_MAX], s_acc, s_recv;
    __shared__ uint32_t s_tmem;
    __shared__ int s_abort;
    __shared__ float s_scale[MOST_TOKENS];   // of the tile's tokens

    const int tid = threadIdx.x, warp = warp_index(), lane = tid & 31;
    const uint32_t rank = g.ks > 1 ? cluster_ctarank() : 0u;
    const int item = static_cast<int>(blockIdx.x) / g.ks;
    const int c0 = item % g.c_tiles * 128;                 // consecutive items share their tokens
    const int t0 = item / g.c_tiles * g.bn;
    const int kb0 = static_cast<int>(static_cast<long long>(g.blocks) * rank / g.ks), kb1 = static_cast<int>(static_cast<long long>(g.blocks) * (rank + 1) / g.ks);
    const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t recv = ring + g.stages * g.stage_bytes;   // [ks][bn / ks tokens][128 channels] (ks > 1)
    volatile int* abort_flag = &s_abort;

    if (warp == 1) tmem_alloc(smem_u32(&s_tmem), g.tmem);
    if (tid == 0) {
        for (int i = 0; i < NSTAGE_MAX; ++i) {
            mbar_init(smem_u32(&s_full[i]), 1);
            mbar_init(smem_u32(&s_free[i]), 1);
        }
        mbar_init(smem_u32(&s_acc), 1);
        mbar_init(smem_u32(&s_recv), 1);
        mbar_fence_init();
        if (g.ks > 1) mbar_arrive_expect_tx(smem_u32(&s_recv), static_cast<uint32_t>(g.bn) * 512u);
        s_abort = 0;
        tma_prefetch_desc(&tm_x);
    }
    tc_fence_before();
    if (g.ks > 1) cluster_sync_all();   // the other CTAs' barriers are initialised before anything is sent to them
    else __syncthreads();
    tc_fence_after();
    const uint32_t tmem = s_tmem;
    pdl_launch_dependents();            // (after the allocation: what starts now cannot take tensor memory that this launch still wants)

    if (warp == 0) {
        if (elect_one()) {
            const int8_t* src = g.weights + (static_cast<size_t>(kb0) * g.rows + c0) * 128;
            const uint8_t* places = SPARSE ? g.places + (static_cast<size_t>(kb0) * g.rows + c0) * 32 : nullptr;
            RingPos rp;
            int issued = 0;
            bool after = false;   // the kernel before has ended
            const int end = g.never_loaded >= kb0 && g.never_loaded < kb1 ? g.never_loaded : kb1;
            for (int kb = kb0; kb < end; ++kb) {
                if (rp.wrapped && !mbar_wait_lone(smem_u32(&s_free[rp.s]), rp.parity ^ 1u)) { *abort_flag = 1; break; }
                const uint32_t at = ring + rp.s * g.stage_bytes, bar = smem_u32(&s_full[rp.s]);
                mbar_arrive_expect_tx(bar, static_cast<uint32_t>(g.stage_bytes));
                bulk_load_1d(at, src, A_BYTES, bar);   // weights: no kernel of the stream writes them
                if constexpr (SPARSE) {
                    bulk_load_1d(at + A_BYTES, places, PLACES, bar);
                    places += static_cast<size_t>(g.rows) * 32;
                }
                if (!after) pdl_wait();
                after = true;
                if constexpr (SPARSE) {   // (past the last column: zeros)
                    tma_load_2d(at + A_BYTES + PLACES, &tm_x, bar, kb * 256, t0);
                    tma_load_2d(at + A_BYTES + PLACES + g.bn * 128, &tm_x, bar, kb * 256 + 128, t0);
                } else {
                    tma_load_2d(at + A_BYTES, &tm_x, bar, kb * 128, t0);
                }
                src += static_cast<size_t>(g.rows) * 128;
                rp.advance(g.stages);
                ++issued;
            }
            if (!after) pdl_wait();
            (void)mbar_wait(smem_u32(&s_acc), 0);   // the issuer is through with the stages, or has given up and said so
            if (*abort_flag != 0) {
                // let the loads in flight land
                for (int back = 0; back < g.stages && back < issued; ++back) {
                    if (rp.s == 0) { rp.s = g.stages; rp.parity ^= 1u; }
                    --rp.s;
                    (void)mbar_wait(smem_u32(&s_full[rp.s]), rp.parity);
                }
            }
        }
    } else if (warp == 1) {
        if (elect_one()) {
            const uint32_t idesc = umma_idesc_s8(128, g.bn) | (SPARSE ? kSparseA : 0u);
            RingPos rp;
            pdl_wait();   // (its waits are bounded: the time that the kernel before still takes is no part of them)
            int kb = kb0;
            for (; kb < kb1; ++kb) {
                if (!mbar_wait_lone(smem_u32(&s_full[rp.s]), rp.parity)) { *abort_flag = 2; break; }
                tc_fence_after();
                const uint32_t at = ring + rp.s * g.stage_bytes;
                const uint64_t adesc = umma_desc_k_sw128(at, 1024);
                if constexpr (SPARSE) {
                    // (in order with the MMAs behind it; a stage's columns are free again when its shared memory is)
                    const uint32_t places = tmem + g.bn + 8 * rp.s;
                    tmem_cp_128x256b(places, umma_desc_k_plain(at + A_BYTES, 128, 256));
#pragma unroll
                    for (int kq = 0; kq < 4; ++kq)
                        umma_s8_sparse(tmem, adesc + 2 * kq, umma_desc_k_sw128(at + A_BYTES + PLACES + kq / 2 * g.bn * 128, 1024) + 4 * (kq % 2), places + 2 * kq, idesc,
                                       (kb > kb0 || kq > 0) ? 1u : 0u);
                } else {
                    const uint64_t bdesc = umma_desc_k_sw128(at + A_BYTES, 1024);
#pragma unroll
                    for (int kq = 0; kq < 4; ++kq) umma_s8_ss(tmem, adesc + 2 * kq, bdesc + 2 * kq, idesc, (kb > kb0 || kq > 0) ? 1u : 0u);
                }
                umma_commit(smem_u32(&s_free[rp.s]));
                rp.advance(g.stages);
            }
            if (kb < kb1) __threadfence_block();   // the flag is seen by whoever sees the commit, which waits for the MMAs issued so far
            umma_commit(smem_u32(&s_acc));
        }
    } else {
        pdl_wait();
        const int e = tid - 64;   // 0 to 127
        for (int i = e; i < g.bn; i += 128) s_scale[i] = t0 + i < g.tokens ? __ldg(g.x_scale + t0 + i) : 0.f;
        // a lane stores four channels of a token at a time (every fourth token is this warp's)
        const int row = (warp & 3) * 32 + lane, ch = c0 + lane * 4, n_ch = g.c_out - ch;
        float ws[4], bias[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            ws[i] = i < n_ch ? __ldg(g.w_scale + ch + i) : 0.f;
            bias[i] = g.bias && i < n_ch ? __ldg(g.bias + ch + i) : 0.f;
        }
        const bool aligned = g.y_ld % 4 == 0 && reinterpret_cast<uintptr_t>(g.y) % (4 * sizeof(T)) == 0;
        const bool ok = mbar_wait(smem_u32(&s_acc), 0);
        if (!ok) *abort_flag = 3;
        const int given_up = *abort_flag;   // the issuer: its sums are written nowhere (asked below, so that nobody waits for the load)
        tc_fence_after();
        // sums by token into the ring, whose loads have all been used: a lane holds a channel of 32 tokens, a row of the ring is a token
        const uint32_t mine = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
        for (int b = 0; b < g.bn; b += 16) {
            uint32_t v[16];
            tmem_ld16(mine + b, v);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 16; ++i)
                asm volatile("st.shared.b32 [%0], %1;" ::"r"(ring + static_cast<uint32_t>((b + i) * 128 + row) * 4u), "r"(v[i]) : "memory");
        }
        const int run = g.bn / g.ks;   // tokens that this CTA finishes
        uint32_t parts = ring;
        bool complete = ok && given_up == 0;
        if (g.ks > 1) {
            // each CTA's run of tokens to that CTA (one that has given up sends nothing, and the waits of all of them expire)
            fence_proxy_async();
            asm volatile("bar.sync 1, 128;" ::: "memory");
            if (e == 0 && complete) {
                for (int d = 0; d < g.ks; ++d)
                    bulk_copy_cluster(mapa_shared(recv + rank * run * 512u, d), ring + static_cast<uint32_t>(d * run) * 512u, static_cast<uint32_t>(run) * 512u,
                                      mapa_shared(smem_u32(&s_recv), d));
            }
            if (!mbar_wait_cluster(smem_u32(&s_recv), 0)) {
                *abort_flag = 4;
                complete = false;
            }
            parts = recv;
        } else {
            asm volatile("bar.sync 1, 128;" ::: "memory");
        }
        if (complete) {
            const int first = static_cast<int>(rank) * run;
#pragma unroll 2
            for (int i = warp - 2; i < run; i += 4) {
                const int token = t0 + first + i;
                if (token >= g.tokens) break;
                int4 sum = load_int4(parts + static_cast<uint32_t>(i * 128 + lane * 4) * 4u);
                for (int s = 1; s < g.ks; ++s) {
                    const int4 v = load_int4(parts + static_cast<uint32_t>((s * run + i) * 128 + lane * 4) * 4u);
                    sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
                }
                const float xs = s_scale[first + i];
                const float v[4] = {fmaf(static_cast<float>(sum.x) * xs, ws[0], bias[0]), fmaf(static_cast<float>(sum.y) * xs, ws[1], bias[1]),
                                    fmaf(static_cast<float>(sum.z) * xs, ws[2], bias[2]), fmaf(static_cast<float>(sum.w) * xs, ws[3], bias[3])};
                put4<T>(static_cast<T*>(g.y) + static_cast<size_t>(token) * g.y_ld + ch, v, n_ch, aligned);
            }
        }
    }

    tc_fence_before();
    if (g.ks > 1) cluster_sync_all();   // nobody leaves while its shared memory is read or written by another CTA
    else __syncthreads();
    if (tid == 0 && s_abort != 0) {
        atomicExch(g.status + 0, static_cast<int>(NM_ERR_TIMEOUT));
        atomicExch(g.status + 1, 200 + s_abort);
        atomicExch(g.status + 2, static_cast<int>(blockIdx.x));
    }
    if (warp == 1) tmem_dealloc(tmem, g.tmem);
}

using Kernel = void (*)(GemmArgs, CUtensorMap);
template <bool SPARSE>
Kernel kernel_of(nm_dtype_t t)
{
    return t == NM_F32 ? k_q8_gemm<float, SPARSE> : t == NM_BF16 ? k_q8_gemm<__nv_bfloat16, SPARSE> : k_q8_gemm<__half, SPARSE>;
}

}  // namespace

namespace nmhost {

bool q8_encode_x(const Q8Linear& p, int rows, void* tensor_map)
{
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(p.w->k), static_cast<cuuint64_t>(p.tokens)};
    const cuuint64_t strides[1] = {static_cast<cuuint64_t>(p.x_ld)};
    const cuuint32_t box[2] = {128, static_cast<cuuint32_t>(rows)}, es[2] = {1, 1};
    return nmtm::available() &&
           nmtm::encoders().tiled(static_cast<CUtensorMap*>(tensor_map), CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<int8_t*>(p.x), dims, strides, box, es,
                                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

nm_status_t launch_q8_gemm(const Q8Linear& p, cudaStream_t st)
{
    const nm_q8_weights* w = p.w;
    GemmArgs g = {};
    const bool sparse = w->sparse != nullptr;
    g.weights = sparse ? w->sparse : w->expanded; g.places = w->places; g.w_scale = w->scales; g.x_scale = p.x_scale; g.bias = p.bias; g.y = p.y; g.y_ld = p.y_ld; g.status = w->status;
    g.tokens = p.tokens; g.c_out = w->c_out; g.rows = w->rows;
    g.blocks = sparse ? w->s_blocks : w->k_blocks;
    g.never_loaded = p.never_loaded;
    g.c_tiles = (w->c_out + 127) / 128;
    // The narrowest tiles (in sixteens) that still are one round, us: 4096 -> 4096, 128 tokens in tiles of 16 / 32 / 64 / 128: 16.0 / 8.7 / 9.2 /
    // 11.1; 512 tokens: 56 / 34 / 19 / 12.2.  A split of the reduction axis pays where half the SMs would idle (16 tokens, 2048 -> 2048: 5.0
    // whole, 3.8 in four), not in eight (7.9).  (Figures of dense weights.)
    const int columns = std::max(1, sm_count() / g.c_tiles);   // tiles along the tokens
    g.bn = static_cast<int>(std::min<long long>(MOST_TOKENS, ((static_cast<long long>(p.tokens) + columns - 1) / columns + 15) / 16 * 16));
    const long long items = static_cast<long long>(g.c_tiles) * ((p.tokens + g.bn - 1) / g.bn);
    if (items > (1ll << 27)) return fail(NM_ERR_UNSUPPORTED, "nm_q8_linear: too many tiles");
    g.ks = 1;
    while (g.ks < 4 && items * g.ks * 2 <= sm_count() && g.blocks * (sparse ? 2 : 1) >= g.ks * 4) g.ks *= 2;
    // More than a round of CTAs: two on an SM, one sets up and loads while the other finishes (in one round the deeper ring is faster:
    // 4096 -> 4096, 512 tokens 12.2 us against 16.9)
    const bool half = items > sm_count();
    g.stage_bytes = sparse ? A_BYTES + PLACES + 2 * g.bn * 128 : A_BYTES + g.bn * 128;
    const int budget = (half ? RING_SHARED : RING_ALONE) - (g.ks > 1 ? g.bn * 512 : 0);
    g.stages = std::min(NSTAGE_MAX, budget / g.stage_bytes);
    g.tmem = 32;
    while (g.tmem < g.bn + (sparse ? 8 * g.stages : 0)) g.tmem *= 2;
    alignas(64) CUtensorMap tm;
    if (!q8_encode_x(p, g.bn, &tm)) return fail(NM_ERR_CUDA, "nm_q8_linear: tensor-map encoding failed");
    size_t smem = 1024 + static_cast<size_t>(g.stages) * g.stage_bytes + (g.ks > 1 ? g.bn * 512 : 0);
    // Alone on its SM: CTAs of a cluster wait for each other while they hold tensor memory.  The others need more than what the kernels
    // that take all of it leave free.
    if (!half && smem < NM_EXCLUSIVE_SMEM) smem = NM_EXCLUSIVE_SMEM;
    if (half && smem < 76 * 1024) smem = 76 * 1024;   // (at most two on an SM, of 256 columns of tensor memory at most)
    const Kernel kernel = sparse ? kernel_of<true>(p.y_type) : kernel_of<false>(p.y_type);
    cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), smem);
    if (e != cudaSuccess) return fail(NM_ERR_CUDA, "nm_q8_linear: cudaFuncSetAttribute: %s", cudaGetErrorString(e));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(items * g.ks));
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = static_cast<unsigned>(g.ks);
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = pdl_enabled() ? 2 : 1;
    e = cudaLaunchKernelEx(&cfg, kernel, g, tm);
    count_launch(1);
    if (e == cudaSuccess) e = cudaGetLastError();
    if (e != cudaSuccess) return fail(NM_ERR_CUDA, "nm_q8_linear launch: %s", cudaGetErrorString(e));
    return NM_OK;
}

}  // namespace nmhost
