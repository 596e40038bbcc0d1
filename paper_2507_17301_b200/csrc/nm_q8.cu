// Host side of the 8-bit operators: argument checks, the weight handle and the kernels that build it.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>

#include "nm_q8.h"

namespace {

using nmhost::fail;

constexpr int kMostTokens = 1 << 30;

size_t size_of(nm_dtype_t t) { return t == NM_F32 ? 4 : 2; }
bool known(nm_dtype_t t) { return t == NM_F32 || t == NM_BF16 || t == NM_F16; }
uintptr_t at(const void* p) { return reinterpret_cast<uintptr_t>(p); }

// A [rows][cols] tensor of `size`-byte elements whose rows are `ld` elements apart.
struct Span {
    const void* p;
    long long ld;
    long long cols;
    size_t size;
};
bool overlap(const Span& a, const Span& b, long long rows)
{
    if (!a.p || !b.p || rows < 1) return false;
    const uintptr_t a0 = at(a.p), b0 = at(b.p);
    const uintptr_t a_row = static_cast<uintptr_t>(a.cols) * a.size, b_row = static_cast<uintptr_t>(b.cols) * b.size;
    const uintptr_t a_ld = static_cast<uintptr_t>(a.ld) * a.size, b_ld = static_cast<uintptr_t>(b.ld) * b.size;
    if (a0 + (rows - 1) * a_ld + a_row <= b0 || b0 + (rows - 1) * b_ld + b_row <= a0) return false;
    if (rows > 1 && a_ld == b_ld) {   // columns of one buffer, side by side
        const uintptr_t d = b0 >= a0 ? (b0 - a0) % a_ld : (a_ld - (a0 - b0) % a_ld) % a_ld;
        return d < a_row || a_ld - d < b_row;
    }
    return true;
}
bool same(const Span& a, const Span& b, long long rows) { return a.p == b.p && a.size == b.size && (rows < 2 || a.ld == b.ld); }

nm_status_t run_rows(const char* who, Q8RowOp op, Q8Rows a, nm_dtype_t type, nm_dtype_t weight_type, cudaStream_t st)
{
    if (!known(type) || !known(weight_type)) return fail(NM_ERR_INVALID_ARG, "%s: unknown type", who);
    if (a.tokens < 0 || a.h < 1) return fail(NM_ERR_INVALID_ARG, "%s: need tokens >= 0 and h >= 1", who);
    if (a.h > 65535) return fail(NM_ERR_UNSUPPORTED, "%s: h = %d exceeds 65535", who, a.h);
    if (a.tokens > kMostTokens) return fail(NM_ERR_UNSUPPORTED, "%s: more than 2^30 tokens", who);
    if (a.tokens == 0) return NM_OK;
    if (!a.x || !a.q || !a.scale) return fail(NM_ERR_INVALID_ARG, "%s: a tensor is NULL", who);
    const size_t size = size_of(type);
    const long long h16 = (static_cast<long long>(a.h) + 15) / 16 * 16;
    if (a.tokens == 1) {   // no second row: pitches that pass the checks below
        a.x_ld = a.r_ld = a.s_ld = a.q_ld = h16;
    }
    if (a.x_ld < a.h || (a.r && a.r_ld < a.h) || (a.s && a.s_ld < a.h) || a.q_ld < a.h)
        return fail(NM_ERR_INVALID_ARG, "%s: rows are closer than h = %d elements", who, a.h);
    if ((at(a.x) | at(a.r) | at(a.s)) % size || at(a.weight) % size_of(weight_type) || at(a.scale) % 4)
        return fail(NM_ERR_INVALID_ARG, "%s: a tensor is not aligned to its elements", who);
    if (at(a.q) % 16 || a.q_ld % 16) return fail(NM_ERR_INVALID_ARG, "%s: q must be 16-byte aligned with rows a multiple of 16 bytes apart", who);
    const Span x = {a.x, a.x_ld, a.h, size}, r = {a.r, a.r_ld, a.h, size}, s = {a.s, a.s_ld, a.h, size}, q = {a.q, a.q_ld, a.h, 1},
               w = {a.weight, 0, a.h, size_of(weight_type)}, sc = {a.scale, 0, a.tokens, 4};
    // one-dimensional tensors against whole two-dimensional ones: as one row of everything
    auto whole = [&](const Span& t) { return Span{t.p, 0, (a.tokens - 1) * t.ld + t.cols, t.size}; };
    bool bad = overlap(q, x, a.tokens) || overlap(q, r, a.tokens) || overlap(q, s, a.tokens);
    for (const Span& t : {x, r, s, q}) bad = bad || overlap(sc, whole(t), 1);
    bad = bad || overlap(w, whole(q), 1) || overlap(w, whole(s), 1) || overlap(w, sc, 1);
    if (a.s) bad = bad || (!same(s, x, a.tokens) && overlap(s, x, a.tokens)) || (!same(s, r, a.tokens) && overlap(s, r, a.tokens));
    if (bad) return fail(NM_ERR_INVALID_ARG, "%s: an output overlaps another tensor", who);
    bool vec = true;   // rows that can be read 16 bytes at a time
    for (const Span& t : {x, r, s}) vec = vec && (!t.p || (at(t.p) % 16 == 0 && (a.tokens == 1 || t.ld * static_cast<long long>(size) % 16 == 0)));
    vec = vec && at(a.weight) % 16 == 0;
    switch (type) {
        case NM_F32: return nmhost::launch_q8_rows_f32(op, a, weight_type, vec, st);
        case NM_BF16: return nmhost::launch_q8_rows_bf16(op, a, weight_type, vec, st);
        default: return nmhost::launch_q8_rows_f16(op, a, weight_type, vec, st);
    }
}

bool valid(const nm_q8_weights* w) { return w && w->magic == NM_Q8_MAGIC; }

struct OnDevice {   // makes a handle's device the current one for as long as the object lives
    int before = -1;
    explicit OnDevice(int device)
    {
        int dev = device;
        if (cudaGetDevice(&dev) == cudaSuccess && dev != device && cudaSetDevice(device) == cudaSuccess) before = dev;
    }
    ~OnDevice()
    {
        if (before >= 0) cudaSetDevice(before);
    }
    OnDevice(const OnDevice&) = delete;
    OnDevice& operator=(const OnDevice&) = delete;
};

// One row's retained weights to 8 bits: values [c_out][kk].
__global__ void __launch_bounds__(256) k_q8_quantise(const float* __restrict__ w, int k, int kk, int kk_ld, int tile_t, const uint16_t* __restrict__ idx,
                                                     int8_t* __restrict__ values, float* __restrict__ scales)
{
    __shared__ uint32_t part[8];
    const int o = blockIdx.x;
    const float* row = w + static_cast<size_t>(o) * k;
    const uint16_t* col = idx + static_cast<size_t>(o / tile_t) * kk_ld;
    uint32_t top = 0u;   // bits of the largest magnitude: NaN above infinity above numbers
    for (int j = threadIdx.x; j < kk; j += 256) top = max(top, __float_as_uint(row[col[j]]) & 0x7FFFFFFFu);
    top = __reduce_max_sync(0xFFFFFFFFu, top);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = top;
    __syncthreads();
    for (int i = 0; i < 8; ++i) top = max(top, part[i]);
    const bool good = top < 0x7F800000u;
    const double a = __uint_as_float(top);
    if (threadIdx.x == 0) scales[o] = good ? static_cast<float>(a / 127.0) : NAN;
    for (int j = threadIdx.x; j < kk; j += 256)
        values[static_cast<size_t>(o) * kk + j] = good && top ? static_cast<int8_t>(rint(127.0 * static_cast<double>(row[col[j]]) / a)) : static_cast<int8_t>(0);
}

// The handle's copy of given index rows.  `bad` is set for one that is not strictly ascending below k with N columns per group; such a
// handle is thrown away.
__global__ void __launch_bounds__(256) k_q8_indices(const uint16_t* __restrict__ idx, const nm_q8_weights h, int* __restrict__ bad)
{
    const int j = blockIdx.x * 256 + threadIdx.x;
    if (j >= h.kk_ld) return;
    for (int tile = blockIdx.y; tile < h.n_tiles; tile += gridDim.y) {
        const uint16_t* row = idx + static_cast<size_t>(tile) * h.kk;
        const int c = j < h.kk ? row[j] : 0;
        if (j < h.kk && (c >= h.k || (j > 0 && c <= row[j - 1]) || c / h.m_group != j / h.n_keep)) *bad = 1;
        h.indices[static_cast<size_t>(tile) * h.kk_ld + j] = static_cast<uint16_t>(c);
    }
}

// 32 columns of a row in the sparse form: 16 bytes and a word of places.  Of four columns the two that are not zero, or as many as there
// are and the first others.
__device__ __forceinline__ void store_sparse(const nm_q8_weights& h, int kb, int r, int quarter, const uint32_t (&in)[8])
{
    uint32_t out[4] = {0u, 0u, 0u, 0u}, places = 0u;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        uint32_t set = 0u;   // columns that are not zero
        for (int b = 0; b < 4; ++b)
            if (in[q] >> (8 * b) & 0xFFu) set |= 1u << b;
        for (int b = 0; b < 4 && __popc(set) < 2; ++b) set |= 1u << b;
        const int first = __ffs(set) - 1, second = __ffs(set & (set - 1u)) - 1;
        places |= static_cast<uint32_t>(first | second << 2) << (4 * q);
        const uint32_t two = (in[q] >> (8 * first) & 0xFFu) | (in[q] >> (8 * second) & 0xFFu) << 8;
        out[q / 2] |= two << (16 * (q % 2));
    }
    const int sb = kb / 2, eighth = kb % 2 * 4 + quarter;
    uint8_t* dst = reinterpret_cast<uint8_t*>(h.sparse) + (static_cast<size_t>(sb) * h.rows + r) * 128;
    *reinterpret_cast<uint4*>(dst + ((eighth ^ (r & 7)) << 4)) = make_uint4(out[0], out[1], out[2], out[3]);
    uint8_t* to = h.places + (static_cast<size_t>(sb) * (h.rows / 128) + r / 128) * 4096;
    *reinterpret_cast<uint32_t*>(to + r % 128 / 8 * 256 + eighth / 4 * 128 + r % 8 * 16 + eighth % 4 * 4) = places;
}

// The form that the tensor core reads, sparse or expanded, from the handle's indices and values [c_out][kk]: a block writes 64 rows of
// 128 columns, a thread 16 bytes of a row.  (Index rows out of order give a wrong place, never one outside a row.)
template <bool SPARSE>
__global__ void __launch_bounds__(256) k_q8_expand(const int8_t* __restrict__ values, const nm_q8_weights h)
{
    constexpr int COLS = SPARSE ? 32 : 16, PIECES = 128 / COLS;
    __shared__ int s_pos[128];   // place of a column among the tile's retained ones, -1: pruned
    const int kb = blockIdx.x, row0 = blockIdx.y * 64;
    for (int r0 = row0; r0 < row0 + 64 && r0 < h.rows;) {
        // rows of one tile at a time
        const int tile = r0 < h.c_out ? r0 / h.tile_t : -1;
        const int r1 = r0 < h.c_out ? min(min((tile + 1) * h.tile_t, h.c_out), row0 + 64) : row0 + 64;
        __syncthreads();
        if (threadIdx.x < 128) {
            const int c = kb * 128 + threadIdx.x;
            int pos = -1;
            if (tile >= 0 && c < h.k) {
                const uint16_t* row = h.indices + static_cast<size_t>(tile) * h.kk_ld;
                int lo = 0, hi = h.kk;
                while (lo < hi) {
                    const int mid = (lo + hi) / 2;
                    if (row[mid] < c) lo = mid + 1;
                    else hi = mid;
                }
                if (lo < h.kk && row[lo] == c) pos = lo;
            }
            s_pos[threadIdx.x] = pos;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < (r1 - r0) * PIECES; i += 256) {
            const int r = r0 + i / PIECES, piece = i % PIECES;
            uint32_t word[COLS / 4] = {};
            if (r < h.c_out) {
#pragma unroll
                for (int b = 0; b < COLS; ++b) {
                    const int pos = s_pos[piece * COLS + b];
                    if (pos >= 0) word[b / 4] |= (static_cast<uint32_t>(values[static_cast<size_t>(r) * h.kk + pos]) & 0xFFu) << (8 * (b % 4));
                }
            }
            if constexpr (SPARSE) {
                store_sparse(h, kb, r, piece, word);
            } else {
                uint8_t* dst = reinterpret_cast<uint8_t*>(h.expanded) + (static_cast<size_t>(kb) * h.rows + r) * 128 + ((piece ^ (r & 7)) << 4);
                *reinterpret_cast<uint4*>(dst) = make_uint4(word[0], word[1], word[2], word[3]);
            }
        }
        r0 = r1;
    }
}

// Most columns that an N:M pattern can keep of four aligned ones of k.
int most_of_four(int n_keep, int m_group, int k)
{
    int most = 0;
    for (int i = 0; i < m_group && 4 * i < k; ++i) {   // (the pattern repeats after m_group fours)
        int kept = 0;
        for (int c = 4 * i, end = 4 * i + 4; c < end;) {
            const int in_group = std::min(m_group - c % m_group, end - c);
            kept += std::min(n_keep, in_group);
            c += in_group;
        }
        most = std::max(most, kept);
    }
    return most;
}

int packed_tile(const nm_q8_weights& h) { return h.n_keep == h.m_group ? h.c_out : h.tile_t; }

// Packed form from values [c_out][kk]: a warp writes a unit's 512 bytes of 64 columns.
__global__ void __launch_bounds__(256) k_q8_pack(const int8_t* __restrict__ values, const nm_q8_weights h, int tile_t)
{
    const int chunks = h.kk_ld / 64, c = blockIdx.x * 8 + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (c >= chunks) return;
    const int n_units = (h.c_out + tile_t - 1) / tile_t * h.units;
    for (int u = blockIdx.y; u < n_units; u += gridDim.y) {
        const int in_tile = u % h.units * 8 + (lane >> 2), o = u / h.units * tile_t + in_tile, j0 = c * 64 + (lane & 3) * 16;
        uint32_t word[4] = {0u, 0u, 0u, 0u};
        if (in_tile < tile_t && o < h.c_out) {
#pragma unroll
            for (int b = 0; b < 16; ++b)
                if (j0 + b < h.kk) word[b / 4] |= (static_cast<uint32_t>(values[static_cast<size_t>(o) * h.kk + j0 + b]) & 0xFFu) << (8 * (b % 4));
        }
        reinterpret_cast<uint4*>(h.packed)[(static_cast<size_t>(u) * chunks + c) * 32 + lane] = make_uint4(word[0], word[1], word[2], word[3]);
    }
}

// values [c_out][kk] out of the sparse or the expanded form.
__global__ void __launch_bounds__(256) k_q8_values(const nm_q8_weights h, int8_t* __restrict__ values)
{
    const int j = blockIdx.x * 256 + threadIdx.x;
    if (j >= h.kk) return;
    for (int o = blockIdx.y; o < h.c_out; o += gridDim.y) {
        const int c = h.indices[static_cast<size_t>(o / h.tile_t) * h.kk_ld + j];
        int8_t value;
        if (h.sparse) {   // (see store_sparse; a column that is in neither place is a zero)
            const int sb = c / 256, eighth = c % 256 / 32, four = c % 32 / 4;
            const uint8_t* from = h.places + (static_cast<size_t>(sb) * (h.rows / 128) + o / 128) * 4096;
            const uint32_t two = *reinterpret_cast<const uint32_t*>(from + o % 128 / 8 * 256 + eighth / 4 * 128 + o % 8 * 16 + eighth % 4 * 4) >> (4 * four);
            const int8_t* at = h.sparse + (static_cast<size_t>(sb) * h.rows + o) * 128 + ((eighth ^ (o & 7)) << 4) + 2 * four;
            value = (two & 3u) == c % 4u ? at[0] : (two >> 2 & 3u) == c % 4u ? at[1] : static_cast<int8_t>(0);
        } else {
            const int piece = c % 128 / 16;
            value = h.expanded[(static_cast<size_t>(c / 128) * h.rows + o) * 128 + ((piece ^ (o & 7)) << 4) + c % 16];
        }
        values[static_cast<size_t>(o) * h.kk + j] = value;
    }
}

// Checks and an empty handle.
nm_status_t make(const char* who, int c_out, int k, int n_keep, int m_group, int tile_t, nm_q8_weights** out)
{
    if (c_out < 1 || k < 1) return fail(NM_ERR_INVALID_ARG, "%s: c_out and k must be >= 1", who);
    if (n_keep < 1 || m_group < 1 || n_keep > m_group) return fail(NM_ERR_INVALID_ARG, "%s: need 1 <= n_keep <= m_group (got %d:%d)", who, n_keep, m_group);
    if (tile_t < 1) return fail(NM_ERR_INVALID_ARG, "%s: tile_t must be >= 1", who);
    if (k > 65535) return fail(NM_ERR_UNSUPPORTED, "%s: K = %d exceeds the uint16 index range", who, k);
    if (tile_t > 256) return fail(NM_ERR_UNSUPPORTED, "%s: tile_t above 256", who);
    if (c_out > (1 << 22) - 256 || (c_out + tile_t - 1) / tile_t > 65535) return fail(NM_ERR_UNSUPPORTED, "%s: more than 65535 tiles", who);
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return fail(NM_ERR_CUDA, "%s: cudaGetDevice: %s", who, cudaGetErrorString(e));
    nm_q8_weights* h = new (std::nothrow) nm_q8_weights();
    if (!h) return fail(NM_ERR_ALLOC, "%s: out of host memory", who);
    std::memset(h, 0, sizeof(*h));
    h->magic = NM_Q8_MAGIC;
    h->device = dev;
    h->c_out = c_out; h->k = k; h->n_keep = n_keep; h->m_group = m_group; h->tile_t = tile_t;
    h->kk = k / m_group * n_keep + std::min(k % m_group, n_keep);
    h->kk_ld = (h->kk + 63) / 64 * 64;
    h->n_tiles = (c_out + tile_t - 1) / tile_t;
    h->k_blocks = (k + 127) / 128;
    h->rows = (c_out + 255) / 256 * 256;
    if (most_of_four(n_keep, m_group, k) <= 2) h->s_blocks = (k + 255) / 256;
    if (packed_tile(*h) >= 8) h->units = (packed_tile(*h) + 7) / 8;
    size_t total = 0;
    auto place = [&total](size_t bytes) {
        const size_t here = total;
        total += (bytes + 1023) / 1024 * 1024;
        return here;
    };
    const size_t at_expanded = place(h->s_blocks ? 0 : static_cast<size_t>(h->k_blocks) * h->rows * 128);
    const size_t tiles = n_keep == m_group ? 1 : h->n_tiles;
    const size_t at_packed = place(tiles * h->units * 8 * h->kk_ld);
    const size_t at_sparse = place(static_cast<size_t>(h->s_blocks) * h->rows * 128), at_places = place(static_cast<size_t>(h->s_blocks) * h->rows * 32);
    const size_t at_indices = place(static_cast<size_t>(h->n_tiles) * h->kk_ld * 2);
    const size_t at_scales = place(static_cast<size_t>(c_out) * 4);
    const size_t at_status = place(16);
    h->block = static_cast<uint8_t*>(nmhost::device_block_alloc(total, dev, &h->block_bytes));
    if (!h->block) {
        delete h;
        return fail(NM_ERR_ALLOC, "%s: cannot allocate %zu bytes on the device", who, total);
    }
    if (!h->s_blocks) h->expanded = reinterpret_cast<int8_t*>(h->block + at_expanded);
    h->packed = h->units ? reinterpret_cast<int8_t*>(h->block + at_packed) : nullptr;
    h->indices = reinterpret_cast<uint16_t*>(h->block + at_indices);
    if (h->s_blocks) {
        h->sparse = reinterpret_cast<int8_t*>(h->block + at_sparse);
        h->places = h->block + at_places;
    }
    h->scales = reinterpret_cast<float*>(h->block + at_scales);
    h->status = reinterpret_cast<int*>(h->block + at_status);
    *out = h;
    return NM_OK;
}

void discard(nm_q8_weights* h, bool idle)
{
    nmhost::device_block_free(h->block, h->block_bytes, h->device, idle);
    h->magic = 0;
    delete h;
}

// Layouts from values [c_out][kk] and index rows (`idx` NULL: the handle has its own), and the one synchronisation: the handle is
// complete when the call returns, whatever stream uses it next.
nm_status_t finish(const char* who, nm_q8_weights* h, const int8_t* values, const uint16_t* idx, cudaStream_t st)
{
    cudaError_t e = cudaMemsetAsync(h->status, 0, 16, st);
    int* bad = h->status + 3;
    if (idx) k_q8_indices<<<dim3((h->kk_ld + 255) / 256, h->n_tiles), 256, 0, st>>>(idx, *h, bad);
    if (h->sparse) k_q8_expand<true><<<dim3(2 * h->s_blocks, h->rows / 64), 256, 0, st>>>(values, *h);
    else k_q8_expand<false><<<dim3(h->k_blocks, h->rows / 64), 256, 0, st>>>(values, *h);
    nmhost::count_launch(idx ? 2 : 1);
    if (h->packed) {
        const int tile = packed_tile(*h), n_units = (h->c_out + tile - 1) / tile * h->units;
        k_q8_pack<<<dim3((h->kk_ld / 64 + 7) / 8, std::min(n_units, 65535)), 256, 0, st>>>(values, *h, tile);
        nmhost::count_launch(1);
    }
    if (e == cudaSuccess) e = cudaGetLastError();
    int found = 0;
    if (e == cudaSuccess) e = cudaMemcpyAsync(&found, bad, sizeof(int), cudaMemcpyDeviceToHost, st);
    const cudaError_t e2 = cudaStreamSynchronize(st);
    if (e == cudaSuccess) e = e2;
    if (e != cudaSuccess) return fail(NM_ERR_CUDA, "%s: %s", who, cudaGetErrorString(e));
    if (found) return fail(NM_ERR_INVALID_ARG, "%s: an index row is not strictly ascending below K, or does not hold N columns per group of M", who);
    return NM_OK;
}

}  // namespace

// nm_q8_linear, and its self-test (never_loaded >= 0), whose calls all go to the kernel of middling token counts.
static nm_status_t linear(const char* who, const nm_q8_weights_t* w, const int8_t* x, long long x_ld, const float* x_scale, int tokens, const float* bias,
                          void* y, long long y_ld, nm_dtype_t y_dtype, int never_loaded, void* cuda_stream)
{
    if (!valid(w)) return fail(NM_ERR_INVALID_ARG, "%s: bad weights handle", who);
    if (!known(y_dtype)) return fail(NM_ERR_INVALID_ARG, "%s: unknown type", who);
    if (tokens < 0) return fail(NM_ERR_INVALID_ARG, "%s: tokens must be >= 0", who);
    if (tokens > kMostTokens) return fail(NM_ERR_UNSUPPORTED, "%s: more than 2^30 tokens", who);
    if (tokens == 0) return NM_OK;
    if (!x || !x_scale || !y) return fail(NM_ERR_INVALID_ARG, "%s: x, x_scale or y is NULL", who);
    if (tokens == 1) {
        x_ld = (w->k + 15) / 16 * 16;
        y_ld = w->c_out;
    }
    if (x_ld < w->k || y_ld < w->c_out) return fail(NM_ERR_INVALID_ARG, "%s: rows are closer than their length", who);
    if (x_ld > (1ll << 38)) return fail(NM_ERR_UNSUPPORTED, "%s: rows of x are too far apart", who);
    if (at(x) % 16 || x_ld % 16) return fail(NM_ERR_INVALID_ARG, "%s: x must be 16-byte aligned with rows a multiple of 16 bytes apart", who);
    if (at(y) % size_of(y_dtype) || at(x_scale) % 4 || at(bias) % 4)
        return fail(NM_ERR_INVALID_ARG, "%s: a tensor is not aligned to its elements", who);
    const Span ys = {y, y_ld, w->c_out, size_of(y_dtype)}, all = {y, 0, (tokens - 1) * y_ld + w->c_out, size_of(y_dtype)};
    if (overlap(ys, {x, x_ld, w->k, 1}, tokens) || overlap(all, {x_scale, 0, tokens, 4}, 1) || overlap(all, {bias, 0, w->c_out, 4}, 1))
        return fail(NM_ERR_INVALID_ARG, "%s: y overlaps an input", who);
    int dev = 0;
    const cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return fail(NM_ERR_CUDA, "%s: cudaGetDevice: %s", who, cudaGetErrorString(e));
    if (dev != w->device) return fail(NM_ERR_INVALID_ARG, "%s: the handle belongs to device %d, current is %d", who, w->device, dev);
    const Q8Linear p = {w, x, x_ld, x_scale, bias, y, y_ld, tokens, y_dtype, never_loaded};
    if (never_loaded >= 0) return nmhost::launch_q8_gemm(p, static_cast<cudaStream_t>(cuda_stream));
    if (nmhost::q8_few_takes(p)) return nmhost::launch_q8_few(p, static_cast<cudaStream_t>(cuda_stream));
    if (nmhost::q8_pair_takes(p)) return nmhost::launch_q8_pair(p, static_cast<cudaStream_t>(cuda_stream));
    return nmhost::launch_q8_gemm(p, static_cast<cudaStream_t>(cuda_stream));
}

extern "C" {

nm_status_t nm_q8_rows(const void* x, long long x_ld, nm_dtype_t dtype, int tokens, int h, int8_t* q, long long q_ld, float* scale,
                       void* cuda_stream)
{
    Q8Rows a = {};
    a.x = x; a.x_ld = x_ld; a.tokens = tokens; a.h = h; a.q = q; a.q_ld = q_ld; a.scale = scale;
    return run_rows("nm_q8_rows", Q8_ROWS, a, dtype, dtype, static_cast<cudaStream_t>(cuda_stream));
}

nm_status_t nm_q8_silu_mul(const void* gate, long long gate_ld, const void* up, long long up_ld, nm_dtype_t dtype, int tokens, int h, int8_t* q,
                           long long q_ld, float* scale, void* cuda_stream)
{
    if (!up && tokens > 0) return fail(NM_ERR_INVALID_ARG, "nm_q8_silu_mul: up is NULL");
    Q8Rows a = {};
    a.x = gate; a.x_ld = gate_ld; a.r = up; a.r_ld = up_ld; a.tokens = tokens; a.h = h; a.q = q; a.q_ld = q_ld; a.scale = scale;
    return run_rows("nm_q8_silu_mul", Q8_SILU_MUL, a, dtype, dtype, static_cast<cudaStream_t>(cuda_stream));
}

nm_status_t nm_q8_rmsnorm(const void* x, long long x_ld, const void* residual, long long residual_ld, void* residual_out, long long residual_out_ld,
                          const void* weight, nm_dtype_t dtype, nm_dtype_t weight_dtype, int tokens, int h, float eps, int8_t* q, long long q_ld,
                          float* scale, void* cuda_stream)
{
    if (!(eps >= 1e-12f && eps <= 1.f)) return fail(NM_ERR_INVALID_ARG, "nm_q8_rmsnorm: eps must lie between 1e-12 and 1");
    if (tokens > 0 && !weight) return fail(NM_ERR_INVALID_ARG, "nm_q8_rmsnorm: weight is NULL");
    if (tokens > 0 && (residual == nullptr) != (residual_out == nullptr))
        return fail(NM_ERR_INVALID_ARG, "nm_q8_rmsnorm: residual and residual_out are given together");
    if (weight_dtype != dtype && weight_dtype != NM_F32) return fail(NM_ERR_INVALID_ARG, "nm_q8_rmsnorm: weight must be of x's type or fp32");
    Q8Rows a = {};
    a.x = x; a.x_ld = x_ld; a.r = residual; a.r_ld = residual_ld; a.s = residual_out; a.s_ld = residual_out_ld; a.weight = weight;
    a.tokens = tokens; a.h = h; a.eps = eps; a.q = q; a.q_ld = q_ld; a.scale = scale;
    return run_rows("nm_q8_rmsnorm", Q8_RMSNORM, a, dtype, weight_dtype, static_cast<cudaStream_t>(cuda_stream));
}

nm_status_t nm_q8_prune(const float* w_dense, int c_out, int k, int n_keep, int m_group, int tile_t, void* cuda_stream, nm_q8_weights_t** out)
{
    if (!w_dense || !out) return fail(NM_ERR_INVALID_ARG, "nm_q8_prune: w_dense or out is NULL");
    *out = nullptr;
    if (at(w_dense) % 4) return fail(NM_ERR_INVALID_ARG, "nm_q8_prune: w_dense is not aligned to its elements");
    const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    nm_q8_weights* h = nullptr;
    nm_status_t s = make("nm_q8_prune", c_out, k, n_keep, m_group, tile_t, &h);
    if (s != NM_OK) return s;
    if (!nmhost::kernel_may_touch(w_dense, w_dense, h->device)) {
        discard(h, true);
        return fail(NM_ERR_INVALID_ARG, "nm_q8_prune: w_dense must lie on the current device");
    }
    // scores (fp64) and keep flags of every (tile, column), values
    const size_t cells = static_cast<size_t>(h->n_tiles) * k, want = cells * 9 + static_cast<size_t>(c_out) * h->kk;
    size_t scratch_bytes = 0;
    uint8_t* scratch = static_cast<uint8_t*>(nmhost::device_block_alloc(want, h->device, &scratch_bytes));
    if (!scratch) {
        discard(h, true);
        return fail(NM_ERR_ALLOC, "nm_q8_prune: cannot allocate %zu bytes of scratch", want);
    }
    int8_t* values = reinterpret_cast<int8_t*>(scratch + cells * 9);
    cudaError_t e = cudaMemsetAsync(h->indices, 0, static_cast<size_t>(h->n_tiles) * h->kk_ld * 2, st);
    nmhost::select_columns(w_dense, c_out, k, h->kk, h->kk_ld, n_keep, m_group, tile_t, reinterpret_cast<double*>(scratch), scratch + cells * 8,
                           h->indices, st);
    k_q8_quantise<<<c_out, 256, 0, st>>>(w_dense, k, h->kk, h->kk_ld, tile_t, h->indices, values, h->scales);
    nmhost::count_launch(1);
    if (e == cudaSuccess) e = cudaGetLastError();
    s = e == cudaSuccess ? finish("nm_q8_prune", h, values, nullptr, st) : fail(NM_ERR_CUDA, "nm_q8_prune: %s", cudaGetErrorString(e));
    nmhost::device_block_free(scratch, scratch_bytes, h->device, s == NM_OK);
    if (s != NM_OK) {
        discard(h, false);
        return s;
    }
    *out = h;
    return NM_OK;
}

nm_status_t nm_q8_weights_import(const int8_t* values, const float* scales, const uint16_t* indices, int c_out, int k, int n_keep, int m_group,
                                 int tile_t, void* cuda_stream, nm_q8_weights_t** out)
{
    if (!values || !scales || !indices || !out) return fail(NM_ERR_INVALID_ARG, "nm_q8_weights_import: values, scales, indices or out is NULL");
    *out = nullptr;
    if (at(scales) % 4 || at(indices) % 2) return fail(NM_ERR_INVALID_ARG, "nm_q8_weights_import: a tensor is not aligned to its elements");
    const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    nm_q8_weights* h = nullptr;
    nm_status_t s = make("nm_q8_weights_import", c_out, k, n_keep, m_group, tile_t, &h);
    if (s != NM_OK) return s;
    if (!nmhost::kernel_may_touch(values, indices, h->device) || !nmhost::kernel_may_touch(scales, scales, h->device)) {
        discard(h, true);
        return fail(NM_ERR_INVALID_ARG, "nm_q8_weights_import: values, scales and indices must lie on the current device");
    }
    const cudaError_t e = cudaMemcpyAsync(h->scales, scales, static_cast<size_t>(c_out) * 4, cudaMemcpyDeviceToDevice, st);
    s = e == cudaSuccess ? finish("nm_q8_weights_import", h, values, indices, st) : fail(NM_ERR_CUDA, "nm_q8_weights_import: %s", cudaGetErrorString(e));
    if (s != NM_OK) {
        discard(h, false);
        return s;
    }
    *out = h;
    return NM_OK;
}

nm_status_t nm_q8_weights_export(const nm_q8_weights_t* w, int8_t* values, float* scales, uint16_t* indices, void* cuda_stream)
{
    if (!valid(w)) return fail(NM_ERR_INVALID_ARG, "nm_q8_weights_export: bad weights handle");
    const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    cudaError_t e = cudaSuccess;
    if (values) {
        if (!nmhost::kernel_may_touch(values, w->scales, w->device))
            return fail(NM_ERR_INVALID_ARG, "nm_q8_weights_export: values must lie on the handle's device, which is the current one");
        k_q8_values<<<dim3((w->kk + 255) / 256, std::min(w->c_out, 65535)), 256, 0, st>>>(*w, values);
        nmhost::count_launch(1);
        e = cudaGetLastError();
    }
    if (e == cudaSuccess && scales) e = cudaMemcpyAsync(scales, w->scales, static_cast<size_t>(w->c_out) * 4, cudaMemcpyDeviceToDevice, st);
    if (e == cudaSuccess && indices)
        e = cudaMemcpy2DAsync(indices, w->kk * 2, w->indices, w->kk_ld * 2, w->kk * 2, w->n_tiles, cudaMemcpyDeviceToDevice, st);
    if (e != cudaSuccess) return fail(NM_ERR_CUDA, "nm_q8_weights_export: %s", cudaGetErrorString(e));
    return NM_OK;
}

nm_status_t nm_q8_weights_dims(const nm_q8_weights_t* w, int* c_out, int* k, int* kk, int* n_tiles, int* tile_t)
{
    if (!valid(w)) return fail(NM_ERR_INVALID_ARG, "nm_q8_weights_dims: bad weights handle");
    if (c_out) *c_out = w->c_out;
    if (k) *k = w->k;
    if (kk) *kk = w->kk;
    if (n_tiles) *n_tiles = w->n_tiles;
    if (tile_t) *tile_t = w->tile_t;
    return NM_OK;
}

nm_status_t nm_q8_weights_check(const nm_q8_weights_t* w, void* cuda_stream)
{
    if (!valid(w)) return fail(NM_ERR_INVALID_ARG, "nm_q8_weights_check: bad weights handle");
    const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    int host[4] = {0, 0, 0, 0};
    cudaError_t e = cudaMemcpyAsync(host, w->status, sizeof(host), cudaMemcpyDeviceToHost, st);
    if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    if (e != cudaSuccess) return fail(NM_ERR_CUDA, "nm_q8_weights_check: %s", cudaGetErrorString(e));
    if (host[0] != 0) {
        cudaMemsetAsync(w->status, 0, sizeof(host), st);
        cudaStreamSynchronize(st);
        return fail(static_cast<nm_status_t>(host[0]), "device-side wait expired (site %d, block %d)", host[1], host[2]);
    }
    return NM_OK;
}

nm_status_t nm_q8_weights_free(nm_q8_weights_t* w)
{
    if (!w) return NM_OK;
    if (!valid(w)) return fail(NM_ERR_INVALID_ARG, "nm_q8_weights_free: bad weights handle");
    const OnDevice on(w->device);
    const bool idle = cudaDeviceSynchronize() == cudaSuccess;
    discard(w, idle);
    return NM_OK;
}

nm_status_t nm_q8_linear(const nm_q8_weights_t* w, const int8_t* x, long long x_ld, const float* x_scale, int tokens, const float* bias, void* y,
                         long long y_ld, nm_dtype_t y_dtype, void* cuda_stream)
{
    return linear("nm_q8_linear", w, x, x_ld, x_scale, tokens, bias, y, y_ld, y_dtype, -1, cuda_stream);
}

nm_status_t nm_selftest_q8_wait_expiry(const nm_q8_weights_t* w, const int8_t* x, long long x_ld, const float* x_scale, int tokens, float* y,
                                       long long y_ld, int block, void* cuda_stream)
{
    if (block < 0) return fail(NM_ERR_INVALID_ARG, "nm_selftest_q8_wait_expiry: block must be >= 0");
    return linear("nm_selftest_q8_wait_expiry", w, x, x_ld, x_scale, tokens, nullptr, y, y_ld, NM_F32, block, cuda_stream);
}

}  // extern "C"
