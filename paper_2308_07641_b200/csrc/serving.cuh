// Definitions shared by the serving operators (include/tsvd_serving.h): 8-bit linear layers and the 4-bit
// key/value cache.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "tsvd_internal.cuh"
#include "tsvd_serving.h"

// ---- 8-bit operands in tensor-core order ---------------------------------------------------------------------------
// Both operands of the 8-bit product are kept as rows of 128 contraction bytes in the K-major 128-byte-swizzle order:
// eight rows make a group of 1 KiB in which the 16-byte unit u of row r lies at unit u ^ (r & 7).
//   weights      [row tile of 128][block of 128 columns][16 groups]
//   activations  [block of 128 columns][token group of 8]
// so that one row tile's blocks, and any run of token groups of a block, are contiguous (one bulk copy each).
__host__ __device__ inline size_t i8_group_offset(int row_in_group, int col_in_block)
{
    return (size_t)row_in_group * 128 + (size_t)((((col_in_block >> 4) ^ row_in_group) << 4) | (col_in_block & 15));
}

struct tsvd_i8_s {
    int device = 0;
    int sms = 0;
    int M = 0, N = 0;
    int row_tiles = 0, col_blocks = 0;   // 128 each
    int clusters[9] = {};                // [2, 4, 8]: clusters of so many blocks that run at a time
    int8_t* W = nullptr;                 // device, row_tiles * col_blocks * 16 KiB
    float* w_scale = nullptr;            // device, [row_tiles * 128], zero padded
    float* bias = nullptr;               // device, the same, or null
    uint8_t* ws = nullptr;               // scratch: activations in tensor-core order, then their scales
    size_t ws_bytes = 0;
    int* dev_status = nullptr;
};

// i8_mma.cu: the product of B tokens in tensor-core order (x, then their scales) with the handle's weights
tsvd_status_t i8_product(const tsvd_i8_s* h, const uint8_t* x, const float* x_scale, int B, void* y, long long ldy, bool y_bf16, bool test_stall,
                         cudaStream_t st);
tsvd_status_t i8_product_prepare(tsvd_i8_s* h);   // once for a handle, on its device, before its first product

// ---- the 4-bit cache ------------------------------------------------------------------------------------------------
// A page is [kv head][block of 16 positions], a block 20 * head_dim bytes:
//   key codes    [16][head_dim / 2]      a position's row: for j = 0..3 the words w = 0 .. head_dim/32-1, word (j, w) the
//                                        codes of numbers 32 w + 8 j .. + 7 (one word of every group for each j)
//   key scales   [16][head_dim / 32]     (step, base) as two fp16
//   value codes  [16][head_dim / 2]      a position's row: words of eight consecutive numbers, in order
//   value scales [16][head_dim / 32]
// Inside a word number e lies at nibble (e >> 1) + 4 (e & 1): nibbles p and p + 4 -- the pair that one mask leaves in the
// two halves of a word -- are the neighbours 2 p and 2 p + 1.
constexpr int KV4_BLOCK = 16;
constexpr int KV4_GROUP = 32;

struct Kv4Geom {
    uint8_t* pool;
    int heads, dim, page_tokens;
    int n_pages;
    unsigned block_bytes, head_bytes;   // of a block of 16 positions; of one head's blocks in a page
    size_t page_bytes;
    // the block that holds position `at` of page `page`, for one head
    __host__ __device__ uint8_t* block(int page, int head, int at) const
    {
        return pool + (size_t)page * page_bytes + (size_t)head * head_bytes + ((unsigned)at / KV4_BLOCK) * block_bytes;
    }
};

constexpr int KV4_DEV_TIMEOUT = 1;   // bits of the device status word
constexpr int KV4_DEV_INDEX = 2;

// Which rows belong to which sequence, and where their pages are (all device memory of the caller).
struct Kv4Batch {
    const int* table;      // [n_seq][max_pages]
    int max_pages;
    const int* seq_len;    // [n_seq]
    const int* q_start;    // [n_seq + 1] or null: one row per sequence
    int n_seq, n_rows;
};

struct tsvd_kv4_s {
    int device = 0;
    Kv4Geom g{};
    int sms = 0;
    size_t pool_bytes = 0;
    int* dev_status = nullptr;
    float* parts = nullptr;        // partial results of split rows
    unsigned* tickets = nullptr;   // one per group of split rows: how many of its parts are done (0 between calls)
};

#ifdef __CUDACC__
__device__ __forceinline__ int kv4_first_row(const Kv4Batch& b, int s) { return b.q_start ? b.q_start[s] : s; }

// The sequence that row `i` belongs to: the number of sequences that end at or before it.  Whole warp.
__device__ __forceinline__ int kv4_seq_of_row(const Kv4Batch& b, int i)
{
    if (!b.q_start) return i;
    int n = 0;
    for (int s0 = 0; s0 < b.n_seq; s0 += 32) {
        const int s = s0 + (int)(threadIdx.x & 31);
        n += __popc(__ballot_sync(0xffffffffu, s < b.n_seq && b.q_start[s + 1] <= i));
    }
    return n;
}

template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
#endif

// Columns, rows and sequences are counted in 32 bits, some beyond the last one (up to a block's share of them); calls whose counts
// would not fit are refused.
constexpr int TSVD_COUNT_MOST = 0x7fffffff - 0xffff;

// A handle's memory lies on one device; its calls launch on the current one.
inline tsvd_status_t on_current_device(int device)
{
    int now = 0;
    TSVD_CUDA_OK(cudaGetDevice(&now));
    return now == device ? TSVD_OK : TSVD_E_CUDA;
}

struct AttendArgs {
    tsvd_kv4_s* h;
    Kv4Batch b;
    const void* q;
    long long ldq;
    void* out;
    long long ldo;
    int n_heads;
    tsvd_dtype_t dtype;
    int max_q, max_kv;
    float scale;
    int window;
    int sinks;             // first positions that the window does not hide; 0 without a window
    bool causal;
    bool test_stall;       // TSVD_FLAG_TEST_STALL
    cudaStream_t stream;
};
tsvd_status_t kv4_attend_simple(const AttendArgs& a);   // kv4_simple.cu
tsvd_status_t kv4_attend_decode(const AttendArgs& a);   // kv4_decode.cu: few rows, bf16
tsvd_status_t kv4_decode_prepare();                     // once for the current device
tsvd_status_t kv4_attend_prefill(const AttendArgs& a);  // kv4_prefill.cu: many rows, bf16
tsvd_status_t kv4_prefill_prepare();
size_t kv4_prefill_parts_bytes(int sms, int dim);
size_t kv4_decode_parts_bytes(int sms, int dim);        // its scratch
size_t kv4_decode_tickets(int sms);
