// Declarations shared by the translation units of the 8-bit operators.
#pragma once
#include <cstdint>
#include <cuda_runtime.h>

#include "nm_internal.h"

constexpr uint32_t NM_Q8_MAGIC = 0x4E4D5138u;   // "NMQ8"

// Compressed 8-bit weights of one linear layer.
struct nm_q8_weights {
    uint32_t magic;
    int device;
    uint8_t* block;        // the handle's device memory: one allocation that every array below lies in
    size_t block_bytes;
    int c_out, k, kk, n_keep, m_group, tile_t, n_tiles;
    int kk_ld;             // row pitch of `indices`: kk rounded up to a multiple of 64 (column 0 in between)
    int k_blocks, rows;    // of `expanded`: ceil(k / 128) blocks, c_out rounded up to a multiple of 256
    int units;             // of `packed` in a tile (a dense layer is one tile): its rows in eights; 0: no packed form
    int s_blocks;          // of `sparse`: ceil(k / 256) blocks; 0: a pattern that keeps more than two of four aligned columns
    float* scales;         // [c_out]
    uint16_t* indices;     // [n_tiles][kk_ld]
    int8_t* packed;        // [tile][unit][kk_ld / 64][8 rows x 4 quarters][16]: retained weights, zeros behind the last column and row; the 512
                           // bytes of a unit and 64 columns are one warp's load, row and quarter by lane.  NULL for tiles of less than 8 rows
    int8_t* expanded;      // [k_blocks][rows][128]: pruned columns are zeros; a row's eight 16-byte pieces stand in the order of the
                           // tensor core's 128-byte swizzle (piece i of row r at i ^ (r & 7)).  NULL where there is a sparse form, which every
                           // product reads instead (4096 -> 12288 at 2:4: 1.2 bytes a dense weight in all, 2.2 with both)
    int8_t* sparse;        // [s_blocks][rows][128]: two of every four columns, the others are zeros; pieces as in `expanded`
    uint8_t* places;       // [s_blocks][rows / 128][4096]: which two, four bits for four columns, 32 bytes a row, as the image that
                           // tmem_cp_128x256b reads: 8-row groups of two 128-byte halves, 16 bytes of each row in a half
    int* status;           // device int[4], as in nm_weights
};

// One call of a row operator (strides in elements).
struct Q8Rows {
    const void* x;         // rmsnorm, rows: input; silu_mul: gate
    long long x_ld;
    const void* r;         // rmsnorm: residual or NULL; silu_mul: up
    long long r_ld;
    void* s;               // rmsnorm with a residual: x + r
    long long s_ld;
    const void* weight;    // rmsnorm
    int tokens, h;
    float eps;
    int8_t* q;
    long long q_ld;
    float* scale;
};
enum Q8RowOp { Q8_RMSNORM = 0, Q8_SILU_MUL = 1, Q8_ROWS = 2 };

// One call of the product.
struct Q8Linear {
    const nm_q8_weights* w;
    const int8_t* x;       // [tokens][x_ld]
    long long x_ld;
    const float* x_scale;
    const float* bias;     // or NULL
    void* y;               // [tokens][y_ld]
    long long y_ld;
    int tokens;
    nm_dtype_t y_type;
    int never_loaded;      // nm_q8_gemm.cu: block of columns from which on nothing is loaded (self-test), -1: none
};

namespace nmhost {
// nm_q8_rows_*.cu, one per type of the activations
nm_status_t launch_q8_rows_f32(Q8RowOp op, const Q8Rows& a, nm_dtype_t weight_type, bool vec, cudaStream_t st);
nm_status_t launch_q8_rows_bf16(Q8RowOp op, const Q8Rows& a, nm_dtype_t weight_type, bool vec, cudaStream_t st);
nm_status_t launch_q8_rows_f16(Q8RowOp op, const Q8Rows& a, nm_dtype_t weight_type, bool vec, cudaStream_t st);

// nm_q8_few.cu: few tokens (8 at most, 4 of a dense layer or one of narrow tiles); false where the kernel does not take the call
bool q8_few_takes(const Q8Linear& p);
nm_status_t launch_q8_few(const Q8Linear& p, cudaStream_t st);

// nm_q8_gemm.cu
nm_status_t launch_q8_gemm(const Q8Linear& p, cudaStream_t st);

// nm_q8_pair.cu: many tokens
bool q8_pair_takes(const Q8Linear& p);
nm_status_t launch_q8_pair(const Q8Linear& p, cudaStream_t st);

// Activations [tokens][x_ld] as a tiled tensor map with a 128-column x `rows` box, 128-byte swizzle.
bool q8_encode_x(const Q8Linear& p, int rows, void* tensor_map);

// nm_prune.cu: retained columns of every tile by their L1 norms; `score` and `keep`: scratch of n_tiles * k entries each
void select_columns(const float* w_dense, int c_out, int k, int kk, int kk_ld, int n_keep, int m_group, int tile_t, double* score,
                    uint8_t* keep, uint16_t* indices, cudaStream_t st);
}  // namespace nmhost
