// Product of many 8-bit activations with column-wise N:M pruned 8-bit weights: pairs of CTAs (tcgen05 cta_group::2, kind::i8).
//
//   D[256 channels][256 tokens] += W[256 x 128] * X[256 x 128]^T   a stage
//
// Weights are the M side of the instruction, tokens the N side.  In the expanded form (pruned columns are zeros):  A pair's MMA is 256 x
// 256 x 32: each CTA holds the weights of its own 128 channels and the activations of HALF the tokens (the hardware exchanges the
// halves), so that a stage of 128 columns is 32 KB written to and 32 KB read from a CTA's shared memory for 512 tensor cycles; a CTA by
// itself would need 48 KB of each, which is more than shared memory moves in that time.  Sums of a CTA's channels stay in its own tensor
// memory, two tiles of 256 columns in turn, so that one is written out while the next is added up.
// In the sparse form (patterns that keep at most two of four aligned columns) a stage is 256 columns, 16 KB of weights, 4 KB of their places,
// which go to tensor memory ahead of the MMAs, and 28 KB of activations: 224 tokens a tile, so that the places of four stages fit beside
// the sums.  4096 -> 12288 at 2:4, 8192 tokens: 242 us expanded, 183 sparse (2.2 POP/s on the retained weights) at 1.65 GHz or more; in a
// run of a second or longer the power limit takes the clock to 1.3 GHz and a call to 218.  A stage takes 690 cycles, not the 448 of the
// sparse rate: without the loads of activations it still takes 605 (480 with 128 tokens a tile, 570 with 192: an instruction of 128, 192
// and 224 tokens 120, 142 and 151 cycles, where its rate is 64, 96 and 112), and the copy of the places is no more than 10 of them.  What
// the rest is has not been found.  Stages of the expanded form take 520 of 512.
//
//   producer (1 thread per CTA)   a bulk copy of the weights' swizzled image and a TMA load of the activations per stage
//   relay (1 thread, second CTA)  forwards "stage landed" to the first CTA's barrier
//   MMA issuer (1 thread, first CTA)
//   epilogue (8 warps per CTA)    a lane has a channel of 16 tokens: y = (sum * x_scale) * w_scale + bias, transposed through shared
//                                 memory to rows of 32 channels
// A work item is 256 channels x 256 tokens (224 in the sparse form), items of one token block follow one another; pairs walk them in a
// static persistent schedule.  Every wait is bounded; the two cluster-wide barriers at start and end are reached by all threads unconditionally.
#include <atomic>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "nm_ptx.cuh"
#include "nm_q8.h"
#include "nm_tmap.cuh"

namespace {

using namespace nmk;

constexpr int THREADS = 384;             // 4 service warps + 8 epilogue warps
constexpr int EPI_TOKENS = 16;           // of an epilogue step
constexpr int STAGING = EPI_TOKENS * 32 * 4;   // bytes of a warp's box

// Tokens of a tile; columns and bytes of a stage.
template <bool SPARSE>
struct Shape {
    static constexpr int BN = SPARSE ? 224 : 256, COLUMNS = SPARSE ? 256 : 128, STAGES = SPARSE ? 4 : 6;
    static constexpr int A_BYTES = 128 * 128, PLACES = SPARSE ? 4096 : 0, B_BLOCK = BN / 2 * 128, B_BLOCKS = SPARSE ? 2 : 1;
    static constexpr int B_AT = A_BYTES + PLACES, STAGE_BYTES = B_AT + B_BLOCKS * B_BLOCK;
    static constexpr size_t SMEM = 1024 + STAGES * STAGE_BYTES + 8 * STAGING;
};
// places in tensor memory: eight columns of each stage behind the first accumulator (the second begins at 256)
static_assert(Shape<true>::BN + 8 * Shape<true>::STAGES <= 256, "");

struct PairArgs {
    const int8_t* weights;     // expanded or sparse
    const uint8_t* places;
    const float* w_scale;
    const float* x_scale;
    const float* bias;
    void* y;
    long long y_ld;
    int* status;
    int tokens, c_out, rows, blocks;   // blocks: stages of a work item
    uint32_t c_tiles, n_work;
};

__device__ __forceinline__ bool aborted(volatile int* flag) { return *flag != 0; }

template <typename T>
__device__ __forceinline__ uint32_t bits_of(float v)
{
    if constexpr (sizeof(T) == 4) return __float_as_uint(v);
    else if constexpr (std::is_same_v<T, __half>) return __half_as_ushort(__float2half_rn(v));
    else return __bfloat16_as_ushort(__float2bfloat16_rn(v));
}

template <typename T, bool SPARSE>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(THREADS, 1) k_q8_pair(const PairArgs g, const __grid_constant__ CUtensorMap tm_x)
{
    using S = Shape<SPARSE>;
    constexpr int BN = S::BN, STAGES = S::STAGES, STAGE_BYTES = S::STAGE_BYTES, A_BYTES = S::A_BYTES;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t s_full[STAGES], s_free[STAGES], s_accfull[2], s_accfree[2];
    __shared__ uint32_t s_tmem;
    __shared__ int s_abort;

    const int tid = threadIdx.x, warp = warp_index(), lane = tid & 31;
    const uint32_t rank = cluster_ctarank();                  // 0: issues the MMAs
    const uint32_t pair = blockIdx.x >> 1, n_pairs = gridDim.x >> 1;
    const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;
    volatile int* abort_flag = &s_abort;

    if (warp == 2) tmem_alloc_pair(smem_u32(&s_tmem), 512);
    if (tid == 0) {
        for (int i = 0; i < STAGES; ++i) {
            mbar_init(smem_u32(&s_full[i]), rank == 0 ? 2 : 1);   // first CTA: its producer's arrival and the relay's
            mbar_init(smem_u32(&s_free[i]), 1);                   // multicast MMA commit
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&s_accfull[i]), 1);    // multicast MMA commit
            mbar_init(smem_u32(&s_accfree[i]), 16);   // the epilogue warps of both CTAs (used in the first CTA)
        }
        mbar_fence_init();
        s_abort = 0;
        tma_prefetch_desc(&tm_x);
    }
    tc_fence_before();
    cluster_sync_all();   // barriers of both CTAs are initialised before either CTA signals the other
    tc_fence_after();
    const uint32_t tmem = s_tmem;
    pdl_launch_dependents();
    pdl_wait();

    if (warp == 0) {
        // =========================== producer (both CTAs) ===========================
        if (elect_one()) {
            int issued = 0;
            RingPos rp;
            for (uint32_t work = pair; work < g.n_work && !aborted(abort_flag); work += n_pairs) {
                const uint32_t c_tile = work % g.c_tiles, t_tile = work / g.c_tiles;
                const int8_t* src = g.weights + (static_cast<size_t>(c_tile) * 256 + rank * 128) * 128;
                const uint8_t* places = SPARSE ? g.places + static_cast<size_t>(c_tile * 2 + rank) * 4096 : nullptr;
                const int t0 = static_cast<int>(t_tile * BN + rank * (BN / 2));
                for (int kb = 0; kb < g.blocks; ++kb) {
                    if (rp.wrapped && !mbar_wait_lone(smem_u32(&s_free[rp.s]), rp.parity ^ 1u)) *abort_flag = 2;
                    if (aborted(abort_flag)) break;
                    const uint32_t at = ring + rp.s * STAGE_BYTES, bar = smem_u32(&s_full[rp.s]);
                    mbar_arrive_expect_tx(bar, STAGE_BYTES);
                    bulk_load_1d(at, src, A_BYTES, bar);
                    if constexpr (SPARSE) {
                        bulk_load_1d(at + A_BYTES, places, S::PLACES, bar);
                        places += static_cast<size_t>(g.rows) * 32;
                    }
#pragma unroll
                    for (int b = 0; b < S::B_BLOCKS; ++b)   // (past the last column: zeros)
                        tma_load_2d(at + S::B_AT + b * S::B_BLOCK, &tm_x, bar, kb * S::COLUMNS + b * 128, t0);
                    src += static_cast<size_t>(g.rows) * 128;
                    rp.advance(STAGES);
                    ++issued;
                }
            }
            // Back over the stages still in use: on the normal path until the pair's MMAs have released them, so that no multicast
            // arrival is still on its way to this CTA when it leaves; after an abort until the loads in flight have landed.
            const bool bad = aborted(abort_flag);
            for (int back = 0; back < STAGES && back < issued; ++back) {
                if (rp.s == 0) { rp.s = STAGES; rp.parity ^= 1u; }
                --rp.s;
                if (bad) (void)mbar_wait(smem_u32(&s_full[rp.s]), rp.parity);
                else if (!mbar_wait(smem_u32(&s_free[rp.s]), rp.parity)) { *abort_flag = 3; break; }
            }
        }
    } else if (warp == 1 && rank == 1) {
        // =========================== relay (second CTA) ===========================
        if (elect_one()) {
            RingPos rp;
            for (uint32_t work = pair; work < g.n_work && !aborted(abort_flag); work += n_pairs) {
                for (int kb = 0; kb < g.blocks; ++kb) {
                    if (!mbar_wait_lone(smem_u32(&s_full[rp.s]), rp.parity)) { *abort_flag = 4; break; }
                    mbar_arrive_cluster_relaxed(mapa_shared(smem_u32(&s_full[rp.s]), 0));
                    rp.advance(STAGES);
                }
            }
        }
    } else if (warp == 1) {
        // =========================== MMA issuer (first CTA) ===========================
        if (elect_one()) {
            constexpr uint32_t idesc = umma_idesc_s8(256, BN) | (SPARSE ? kSparseA : 0u);
            RingPos rp;
            uint32_t ab = 0, acc_par = 0;
            bool acc_wrapped = false;
            for (uint32_t work = pair; work < g.n_work && !aborted(abort_flag); work += n_pairs) {
                if (acc_wrapped && !mbar_wait_cluster(smem_u32(&s_accfree[ab]), acc_par ^ 1u)) {
                    *abort_flag = 5;
                    break;
                }
                tc_fence_after();
                const uint32_t acc = tmem + ab * 256;
                for (int kb = 0; kb < g.blocks; ++kb) {
                    if (!mbar_wait_lone(smem_u32(&s_full[rp.s]), rp.parity)) { *abort_flag = 6; break; }
                    tc_fence_after();
                    const uint32_t at = ring + rp.s * STAGE_BYTES;
                    const uint64_t adesc = umma_desc_k_sw128(at, 1024);
                    if constexpr (SPARSE) {
                        // (in order with the MMAs behind it; a stage's columns are free again when its shared memory is)
                        const uint32_t places = tmem + BN + 8 * rp.s;
                        tmem_cp_128x256b_pair(places, umma_desc_k_plain(at + A_BYTES, 128, 256));
#pragma unroll
                        for (int kq = 0; kq < 4; ++kq)
                            umma_s8_sparse_pair(acc, adesc + 2 * kq, umma_desc_k_sw128(at + S::B_AT + kq / 2 * S::B_BLOCK, 1024) + 4 * (kq % 2), places + 2 * kq, idesc,
                                                (kb > 0 || kq > 0) ? 1u : 0u);
                    } else {
                        const uint64_t bdesc = umma_desc_k_sw128(at + S::B_AT, 1024);
#pragma unroll
                        for (int kq = 0; kq < 4; ++kq) umma_s8_ss_pair(acc, adesc + 2 * kq, bdesc + 2 * kq, idesc, (kb > 0 || kq > 0) ? 1u : 0u);
                    }
                    umma_commit_pair(smem_u32(&s_free[rp.s]));
                    rp.advance(STAGES);
                }
                if (aborted(abort_flag)) break;
                umma_commit_pair(smem_u32(&s_accfull[ab]));
                if (ab == 1) { acc_par ^= 1u; acc_wrapped = true; }
                ab ^= 1u;
            }
        }
    } else if (warp >= 4) {
        // =========================== epilogue (both CTAs) ===========================
        const int q = warp & 3, half = (warp - 4) >> 2;
        const uint32_t mine = tmem + (static_cast<uint32_t>(q * 32) << 16);
        const uint32_t box = ring + STAGES * STAGE_BYTES + (warp - 4) * STAGING;
        constexpr int PER = 16 / sizeof(T), LANES = 32 / PER, ROWS = 32 / LANES;   // channels of 16 bytes; lanes and rows of a store
        const bool aligned = g.y_ld % PER == 0 && reinterpret_cast<uintptr_t>(g.y) % 16 == 0;
        T* const y = static_cast<T*>(g.y);
        uint32_t turn = 0;
        for (uint32_t work = pair; work < g.n_work; work += n_pairs, ++turn) {
            const int c_first = static_cast<int>(work % g.c_tiles * 256 + rank * 128) + q * 32, t_first = static_cast<int>(work / g.c_tiles * BN);
            const int ch = c_first + lane;
            const float ws = ch < g.c_out ? __ldg(g.w_scale + ch) : 0.f, bias = g.bias && ch < g.c_out ? __ldg(g.bias + ch) : 0.f;
            const uint32_t ab = turn & 1u;
            auto scale_of = [&](int blk) {   // of token `lane` of a step
                const int t = t_first + blk * EPI_TOKENS + (lane & 15);
                return t < g.tokens ? __ldg(g.x_scale + t) : 0.f;
            };
            float xs_next = scale_of(half);
            const bool ok = aborted(abort_flag) || mbar_wait(smem_u32(&s_accfull[ab]), (turn >> 1) & 1u);
            if (!__all_sync(0xFFFFFFFFu, ok)) *abort_flag = 8;
            if (__any_sync(0xFFFFFFFFu, aborted(abort_flag))) break;
            tc_fence_after();
            for (int blk = half; blk < BN / EPI_TOKENS; blk += 2) {
                uint32_t v[16];
                tmem_ld16(mine + ab * 256 + blk * EPI_TOKENS, v);
                const float xs = xs_next;
                if (blk + 2 < BN / EPI_TOKENS) xs_next = scale_of(blk + 2);
                tmem_ld_wait();
                if (blk + 2 >= BN / EPI_TOKENS) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_cluster(mapa_shared(smem_u32(&s_accfree[ab]), 0));
                }
                const int token0 = t_first + blk * EPI_TOKENS;
                if (token0 >= g.tokens || c_first >= g.c_out) continue;
                uint32_t out[EPI_TOKENS];
#pragma unroll
                for (int i = 0; i < EPI_TOKENS; ++i)
                    out[i] = bits_of<T>(fmaf(static_cast<float>(static_cast<int>(v[i])) * __shfl_sync(0xFFFFFFFFu, xs, i), ws, bias));
                if (!aligned) {   // a token's 32 channels at a time (through the box a lane would write eight numbers one by one)
#pragma unroll
                    for (int i = 0; i < EPI_TOKENS; ++i) {
                        if (token0 + i >= g.tokens || ch >= g.c_out) continue;
                        T* to = y + static_cast<size_t>(token0 + i) * g.y_ld + ch;
                        if constexpr (sizeof(T) == 4) *reinterpret_cast<uint32_t*>(to) = out[i];
                        else *reinterpret_cast<uint16_t*>(to) = static_cast<uint16_t>(out[i]);
                    }
                    continue;
                }
#pragma unroll
                for (int i = 0; i < EPI_TOKENS; ++i) {
                    const uint32_t at = box + static_cast<uint32_t>((i * 32 + lane) * sizeof(T));
                    if constexpr (sizeof(T) == 4) asm volatile("st.shared.b32 [%0], %1;" ::"r"(at), "r"(out[i]) : "memory");
                    else asm volatile("st.shared.b16 [%0], %1;" ::"r"(at), "h"(static_cast<uint16_t>(out[i])) : "memory");
                }
                __syncwarp();
                const int col = lane % LANES * PER, n_ch = g.c_out - c_first - col;
#pragma unroll
                for (int i = 0; i < EPI_TOKENS / ROWS; ++i) {
                    const int r = i * ROWS + lane / LANES, token = token0 + r;
                    uint4 u;
                    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                                 : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w)
                                 : "r"(box + static_cast<uint32_t>((r * 32 + col) * sizeof(T)))
                                 : "memory");
                    if (token >= g.tokens) continue;
                    T* to = y + static_cast<size_t>(token) * g.y_ld + c_first + col;
                    if (n_ch >= PER) {
                        *reinterpret_cast<uint4*>(to) = u;
                    } else {
                        const T* f = reinterpret_cast<const T*>(&u);
#pragma unroll
                        for (int k = 0; k < PER; ++k)
                            if (k < n_ch) to[k] = f[k];
                    }
                }
                __syncwarp();
            }
        }
    }

    tc_fence_before();
    cluster_sync_all();   // neither CTA leaves (or frees tensor memory) while the other may still signal it
    if (tid == 0 && s_abort != 0) {
        atomicExch(g.status + 0, static_cast<int>(NM_ERR_TIMEOUT));
        atomicExch(g.status + 1, 220 + s_abort);
        atomicExch(g.status + 2, static_cast<int>(blockIdx.x));
    }
    if (warp == 2) tmem_dealloc_pair(tmem, 512);
}

using Kernel = void (*)(PairArgs, CUtensorMap);
template <bool SPARSE>
Kernel kernel_of(nm_dtype_t t)
{
    return t == NM_F32 ? k_q8_pair<float, SPARSE> : t == NM_BF16 ? k_q8_pair<__nv_bfloat16, SPARSE> : k_q8_pair<__half, SPARSE>;
}

// Pairs of SMs that can hold one cluster each at the same time (0 = clusters unavailable).
int max_pairs()
{
    static std::atomic<int> known[64];   // + 1
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
    int n = known[dev].load();
    if (n == 0) {
        const Kernel kernel = kernel_of<false>(NM_BF16);
        constexpr size_t SMEM = Shape<false>::SMEM;   // (either takes a whole SM)
        cudaLaunchConfig_t lc = {};
        lc.gridDim = dim3(2);
        lc.blockDim = dim3(THREADS);
        lc.dynamicSmemBytes = SMEM;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = 2;
        attr[0].val.clusterDim.y = 1;
        attr[0].val.clusterDim.z = 1;
        lc.attrs = attr;
        lc.numAttrs = 1;
        if (nmhost::ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), SMEM) != cudaSuccess || cudaOccupancyMaxActiveClusters(&n, kernel, &lc) != cudaSuccess) {
            (void)cudaGetLastError();
            n = 0;
        }
        known[dev].store(++n);
    }
    return n - 1;
}

}  // namespace

namespace nmhost {

bool q8_pair_takes(const Q8Linear& p)
{
    // One round of the other kernel's tiles of 128 x 128 or less is faster, us (this / the other) at 2:4: 4096 -> 4096, 512 tokens 12.5 / 11.6, 640
    // tokens 12.6 / 20.0; 2048 -> 2048, 1024 tokens 9.5 / 8.9, 1500 tokens 10.1 / 14.5; 4096 -> 12288, 96 tokens 11.7 / 11.7, 160 tokens
    // 12.9 / 19.2; 4096 -> 1001, 2048 tokens 15.7 / 12.3.
    const long long small = static_cast<long long>((p.w->c_out + 127) / 128) * ((static_cast<long long>(p.tokens) + 127) / 128);
    const long long work = static_cast<long long>(p.w->rows / 256) * ((static_cast<long long>(p.tokens) + 223) / 224);
    return p.tokens > 128 && small > sm_count() && work < (1ll << 30) && max_pairs() > 0;
}

nm_status_t launch_q8_pair(const Q8Linear& p, cudaStream_t st)
{
    const nm_q8_weights* w = p.w;
    const bool sparse = w->sparse != nullptr;
    const int bn = sparse ? Shape<true>::BN : Shape<false>::BN;
    const size_t smem = sparse ? Shape<true>::SMEM : Shape<false>::SMEM;
    PairArgs g = {};
    g.weights = sparse ? w->sparse : w->expanded; g.places = w->places; g.w_scale = w->scales; g.x_scale = p.x_scale; g.bias = p.bias; g.y = p.y;
    g.y_ld = p.y_ld; g.status = w->status; g.tokens = p.tokens; g.c_out = w->c_out; g.rows = w->rows;
    g.blocks = sparse ? w->s_blocks : w->k_blocks;
    g.c_tiles = static_cast<uint32_t>(w->rows / 256);
    g.n_work = g.c_tiles * static_cast<uint32_t>((static_cast<long long>(p.tokens) + bn - 1) / bn);
    alignas(64) CUtensorMap tm;
    if (!q8_encode_x(p, bn / 2, &tm)) return fail(NM_ERR_CUDA, "nm_q8_linear: tensor-map encoding failed (pairs)");
    const Kernel kernel = sparse ? kernel_of<true>(p.y_type) : kernel_of<false>(p.y_type);
    cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), smem);
    if (e != cudaSuccess) return fail(NM_ERR_CUDA, "nm_q8_linear: cudaFuncSetAttribute: %s", cudaGetErrorString(e));
    const unsigned pairs_max = static_cast<unsigned>(max_pairs());
    if (pairs_max < 1) return fail(NM_ERR_UNSUPPORTED, "nm_q8_linear: this device runs no clusters of two CTAs");
    const unsigned pairs = g.n_work < pairs_max ? g.n_work : pairs_max;
    e = launch_pdl(kernel, 2 * pairs, THREADS, smem, st, g, tm);
    count_launch(1);
    if (e == cudaSuccess) e = cudaGetLastError();
    if (e != cudaSuccess) return fail(NM_ERR_CUDA, "nm_q8_linear launch (pairs): %s", cudaGetErrorString(e));
    return NM_OK;
}

}  // namespace nmhost
