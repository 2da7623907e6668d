// 8-bit integers with a scale for each token and channel: quantisation of rows, and the linear layer on them.
#include <new>

#include "serving.cuh"

namespace {

constexpr float kSmallest = 7.888609e-31f;   // 2^-100: below it 127 / a is no longer safely finite

// q = rint(x * (127 / a)); 0 for a row without values of any size, the (poisoned) scale says when a is not finite
__device__ __forceinline__ float inverse_step(float a) { return a >= kSmallest ? __fdiv_rn(127.0f, a) : 0.0f; }
__device__ __forceinline__ int quantised(float x, float inv) { return __float2int_rn(__fmul_rn(x, inv)); }

// |a| and |b| compared as integers: the larger magnitude, and a NaN (whose bits exceed infinity's) wins over everything
__device__ __forceinline__ uint32_t max_magnitude(uint32_t m, float v) { return max(m, __float_as_uint(v) & 0x7fffffffu); }

__device__ __forceinline__ uint32_t block_max(uint32_t m, uint32_t* slots)
{
    m = __reduce_max_sync(0xffffffffu, m);
    if ((threadIdx.x & 31) == 0) slots[threadIdx.x >> 5] = m;
    __syncthreads();
    const unsigned n = blockDim.x >> 5;
    m = __reduce_max_sync(0xffffffffu, (threadIdx.x & 31) < n ? slots[threadIdx.x & 31] : 0u);
    __syncthreads();
    return m;
}

// A block per row; the row is read twice (the second time from cache).
template <typename T>
__global__ void quantize_rows_kernel(const T* __restrict__ x, int cols, long long ldx, int8_t* __restrict__ q, long long ldq,
                                     float* __restrict__ scale)
{
    __shared__ uint32_t slots[32];
    const T* row = x + (long long)blockIdx.x * ldx;
    uint32_t m = 0;
    for (int c = threadIdx.x; c < cols; c += blockDim.x) m = max_magnitude(m, to_f32(row[c]));
    const float a = __uint_as_float(block_max(m, slots));
    const float inv = inverse_step(a);
    for (int c = threadIdx.x; c < cols; c += blockDim.x) q[(long long)blockIdx.x * ldq + c] = (int8_t)quantised(to_f32(row[c]), inv);
    if (threadIdx.x == 0) scale[blockIdx.x] = __fdiv_rn(a, 127.0f);
}

template <typename T>
__global__ void dequantize_rows_kernel(const int8_t* __restrict__ q, long long ldq, const float* __restrict__ scale, int cols,
                                       T* __restrict__ y, long long ldy)
{
    const float s = scale[blockIdx.x];
    for (int c = threadIdx.x; c < cols; c += blockDim.x)
        y[(long long)blockIdx.x * ldy + c] = from_f32<T>((float)q[(long long)blockIdx.x * ldq + c] * s);
}

// Activations into tensor-core order: [block of 128 columns][token group of 8], zeros beyond the last column.
template <typename T>
__global__ void stage_rows_kernel(const T* __restrict__ x, int cols, long long ldx, const float* __restrict__ x_scale,
                                  int col_blocks, int groups, uint8_t* __restrict__ tiles, float* __restrict__ scale)
{
    __shared__ uint32_t slots[32];
    const int b = blockIdx.x;
    const T* row = x + (long long)b * ldx;
    float inv = 1.0f, step = 1.0f;
    if constexpr (sizeof(T) > 1) {
        uint32_t m = 0;
        for (int c = threadIdx.x; c < cols; c += blockDim.x) m = max_magnitude(m, to_f32(row[c]));
        const float a = __uint_as_float(block_max(m, slots));
        inv = inverse_step(a);
        step = __fdiv_rn(a, 127.0f);
    } else {
        if (x_scale) step = x_scale[b];
    }
    for (int c = threadIdx.x; c < col_blocks * 128; c += blockDim.x) {
        int v = 0;
        if (c < cols) {
            if constexpr (sizeof(T) > 1) v = quantised(to_f32(row[c]), inv);
            else v = row[c];
        }
        tiles[((size_t)(c >> 7) * groups + (b >> 3)) * 1024 + i8_group_offset(b & 7, c & 127)] = (uint8_t)(int8_t)v;
    }
    if (threadIdx.x == 0) scale[b] = step;
}

// Simple product: a block takes 32 channels x 8 tokens, a thread one of each.
__global__ void i8_product_simple_kernel(const int8_t* __restrict__ W, const uint8_t* __restrict__ xt, const float* __restrict__ xs,
                                         const float* __restrict__ ws, const float* __restrict__ bias, int M, int B, int col_blocks,
                                         int groups, void* y, long long ldy, int out_bf16)
{
    const int m = blockIdx.x * 32 + threadIdx.x, b = blockIdx.y * 8 + threadIdx.y;
    if (m >= M || b >= B) return;
    int sum = 0;
    for (int kb = 0; kb < col_blocks; ++kb) {
        const int8_t* w = W + ((size_t)(m >> 7) * col_blocks + kb) * 16384 + (size_t)((m & 127) >> 3) * 1024;
        const uint8_t* x = xt + ((size_t)kb * groups + (b >> 3)) * 1024;
        for (int c = 0; c < 128; c += 4)
            sum = __dp4a(*reinterpret_cast<const int*>(w + i8_group_offset(m & 7, c)),
                         *reinterpret_cast<const int*>(x + i8_group_offset(b & 7, c)), sum);
    }
    float v = (float)sum * xs[b] * ws[m];
    if (bias) v += bias[m];
    if (out_bf16) reinterpret_cast<__nv_bfloat16*>(y)[(long long)b * ldy + m] = __float2bfloat16_rn(v);
    else reinterpret_cast<float*>(y)[(long long)b * ldy + m] = v;
}

__global__ void i8_tile_weights_kernel(const int8_t* __restrict__ W, long long ldw, int rows, int N, int col_blocks,
                                       int8_t* __restrict__ out, int row0)
{
    const int r = blockIdx.x;              // row of this chunk
    const int row = row0 + r;
    for (int c = threadIdx.x; c < col_blocks * 128; c += blockDim.x)
        out[((size_t)(row >> 7) * col_blocks + (c >> 7)) * 16384 + (size_t)((row & 127) >> 3) * 1024 + i8_group_offset(row & 7, c & 127)] =
            (r < rows && c < N) ? W[(long long)r * ldw + c] : (int8_t)0;
}

bool misaligned(const void* p, size_t size) { return ((uintptr_t)p & (size - 1)) != 0; }

unsigned row_threads(long long cols) { return cols >= 2048 ? 256u : cols >= 512 ? 128u : 64u; }

}  // namespace

extern "C" tsvd_status_t tsvd_quantize(const void* x, tsvd_dtype_t dtype, long long rows, int cols, long long ldx, int8_t* q,
                                       long long ldq, float* scale, void* stream)
{
    if (rows < 0 || rows > 0x7fffffffLL || cols < 1 || ldx < cols || ldq < cols) return TSVD_E_SHAPE;
    if (dtype != TSVD_F32 && dtype != TSVD_BF16) return TSVD_E_DTYPE;
    if (rows == 0) return TSVD_OK;
    if (!x || !q || !scale) return TSVD_E_NULL;
    if (misaligned(x, dtype == TSVD_F32 ? 4 : 2) || misaligned(scale, 4)) return TSVD_E_ALIGN;
    cudaStream_t st = (cudaStream_t)stream;
    if (dtype == TSVD_F32)
        quantize_rows_kernel<float><<<(unsigned)rows, row_threads(cols), 0, st>>>((const float*)x, cols, ldx, q, ldq, scale);
    else
        quantize_rows_kernel<__nv_bfloat16><<<(unsigned)rows, row_threads(cols), 0, st>>>((const __nv_bfloat16*)x, cols, ldx, q, ldq, scale);
    TSVD_CUDA_OK(cudaGetLastError());
    tsvd_count_launch();
    return TSVD_OK;
}

extern "C" tsvd_status_t tsvd_dequantize(const int8_t* q, long long ldq, const float* scale, long long rows, int cols, void* y,
                                         tsvd_dtype_t dtype, long long ldy, void* stream)
{
    if (rows < 0 || rows > 0x7fffffffLL || cols < 1 || ldy < cols || ldq < cols) return TSVD_E_SHAPE;
    if (dtype != TSVD_F32 && dtype != TSVD_BF16) return TSVD_E_DTYPE;
    if (rows == 0) return TSVD_OK;
    if (!q || !scale || !y) return TSVD_E_NULL;
    if (misaligned(y, dtype == TSVD_F32 ? 4 : 2) || misaligned(scale, 4)) return TSVD_E_ALIGN;
    cudaStream_t st = (cudaStream_t)stream;
    if (dtype == TSVD_F32)
        dequantize_rows_kernel<float><<<(unsigned)rows, row_threads(cols), 0, st>>>(q, ldq, scale, cols, (float*)y, ldy);
    else
        dequantize_rows_kernel<__nv_bfloat16><<<(unsigned)rows, row_threads(cols), 0, st>>>(q, ldq, scale, cols, (__nv_bfloat16*)y, ldy);
    TSVD_CUDA_OK(cudaGetLastError());
    tsvd_count_launch();
    return TSVD_OK;
}

// ---- the layer --------------------------------------------------------------------------------------------------------

static void i8_free(tsvd_i8_s* h)
{
    if (!h) return;
    if (h->W) cudaFree(h->W);
    if (h->w_scale) cudaFree(h->w_scale);
    if (h->bias) cudaFree(h->bias);
    if (h->ws) cudaFree(h->ws);
    if (h->dev_status) cudaFree(h->dev_status);
    (void)cudaGetLastError();
    delete h;
}

static tsvd_status_t i8_fill(tsvd_i8_s* h, const int8_t* W, long long ldw, const float* w_scale, const float* bias)
{
    const size_t rows_pad = (size_t)h->row_tiles * 128;
    TSVD_CUDA_OK(cudaMalloc(&h->dev_status, sizeof(int)));
    TSVD_CUDA_OK(cudaMemset(h->dev_status, 0, sizeof(int)));
    TSVD_CUDA_OK(cudaMalloc(&h->W, rows_pad * h->col_blocks * 128));
    TSVD_CUDA_OK(cudaMalloc(&h->w_scale, rows_pad * sizeof(float)));
    TSVD_CUDA_OK(cudaMemset(h->w_scale, 0, rows_pad * sizeof(float)));
    TSVD_CUDA_OK(cudaMemcpy(h->w_scale, w_scale, (size_t)h->M * sizeof(float), cudaMemcpyDefault));
    if (bias) {
        TSVD_CUDA_OK(cudaMalloc(&h->bias, rows_pad * sizeof(float)));
        TSVD_CUDA_OK(cudaMemset(h->bias, 0, rows_pad * sizeof(float)));
        TSVD_CUDA_OK(cudaMemcpy(h->bias, bias, (size_t)h->M * sizeof(float), cudaMemcpyDefault));
    }
    // The weights come over row by row into a staging buffer (host or device source alike), a chunk of row tiles at a time.
    const int tiles_at_once = (int)(((size_t)64 << 20) / ((size_t)128 * h->N) + 1);
    int8_t* staging = nullptr;
    const int chunk = (tiles_at_once < h->row_tiles ? tiles_at_once : h->row_tiles) * 128;
    TSVD_CUDA_OK(cudaMalloc(&staging, (size_t)chunk * h->N));
    cudaError_t e = cudaSuccess;
    for (int r0 = 0; r0 < (int)rows_pad && e == cudaSuccess; r0 += chunk) {
        const int pad = (int)rows_pad - r0 < chunk ? (int)rows_pad - r0 : chunk;
        const int rows = h->M - r0 < pad ? h->M - r0 : pad;
        e = cudaMemcpy2D(staging, (size_t)h->N, W + (long long)r0 * ldw, (size_t)ldw, (size_t)h->N, (size_t)rows, cudaMemcpyDefault);
        if (e != cudaSuccess) break;
        i8_tile_weights_kernel<<<(unsigned)pad, 256>>>(staging, h->N, rows, h->N, h->col_blocks, h->W, r0);
        tsvd_count_launch();
        e = cudaGetLastError();
        if (e == cudaSuccess) e = cudaDeviceSynchronize();   // the staging buffer is used again
    }
    cudaFree(staging);
    TSVD_CUDA_OK(e);
    return TSVD_OK;
}

extern "C" tsvd_status_t tsvd_i8_pack(const int8_t* W, long long ldw, const float* w_scale, const float* bias, int M, int N,
                                      unsigned flags, tsvd_i8_t* out)
{
    if (!out) return TSVD_E_NULL;
    *out = nullptr;
    if (!W || !w_scale) return TSVD_E_NULL;
    if (M < 1 || N < 1 || ldw < N) return TSVD_E_SHAPE;
    if (flags) return TSVD_E_DTYPE;
    if (N > TSVD_I8_MAX_N) return TSVD_E_TOOBIG;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) { (void)cudaGetLastError(); return TSVD_E_CUDA; }
    tsvd_i8_s* h = new (std::nothrow) tsvd_i8_s();
    if (!h) return TSVD_E_NOMEM;
    h->device = dev;
    h->M = M;
    h->N = N;
    h->row_tiles = (M + 127) / 128;
    h->col_blocks = (N + 127) / 128;
    const tsvd_status_t st = i8_fill(h, W, ldw, w_scale, bias);
    if (st != TSVD_OK) { i8_free(h); return st; }
    *out = h;
    return TSVD_OK;
}

static size_t i8_ws_bytes(const tsvd_i8_s* h, int B)
{
    const size_t padded = ((size_t)B + 255) / 256 * 256;
    return padded * ((size_t)h->col_blocks * 128 + sizeof(float));
}

static tsvd_status_t i8_grow(tsvd_i8_s* h, int B)
{
    const size_t need = i8_ws_bytes(h, B);
    if (need <= h->ws_bytes) return TSVD_OK;
    TSVD_CUDA_OK(cudaDeviceSynchronize());
    if (h->ws) { cudaFree(h->ws); h->ws = nullptr; h->ws_bytes = 0; }
    TSVD_CUDA_OK(cudaMalloc(&h->ws, need));
    TSVD_CUDA_OK(cudaMemset(h->ws, 0, need));
    h->ws_bytes = need;
    return TSVD_OK;
}

extern "C" tsvd_status_t tsvd_i8_reserve(tsvd_i8_t h, int B_max, tsvd_dtype_t dtype)
{
    if (!h) return TSVD_E_NULL;
    if (B_max < 1) return TSVD_E_SHAPE;
    if (dtype != TSVD_F32 && dtype != TSVD_BF16 && dtype != TSVD_I8) return TSVD_E_DTYPE;
    return i8_grow(h, B_max);
}

extern "C" tsvd_status_t tsvd_i8_forward(tsvd_i8_t h, const void* x, long long ldx, const float* x_scale, void* y, long long ldy,
                                         int B, tsvd_dtype_t dtype, unsigned flags, void* stream)
{
    if (!h) return TSVD_E_NULL;
    if (B < 0 || ldx < h->N || ldy < h->M) return TSVD_E_SHAPE;
    if (dtype != TSVD_F32 && dtype != TSVD_BF16 && dtype != TSVD_I8) return TSVD_E_DTYPE;
    if ((flags & ~(TSVD_FLAG_OUT_F32 | TSVD_FLAG_OUT_BF16)) || flags == (TSVD_FLAG_OUT_F32 | TSVD_FLAG_OUT_BF16)) return TSVD_E_DTYPE;
    if (x_scale && dtype != TSVD_I8) return TSVD_E_DTYPE;
    if (B == 0) return TSVD_OK;
    if (!x || !y) return TSVD_E_NULL;
    const bool y_bf16 = flags ? flags == TSVD_FLAG_OUT_BF16 : dtype == TSVD_BF16;
    if (misaligned(x, dtype == TSVD_F32 ? 4 : dtype == TSVD_BF16 ? 2 : 1) || misaligned(y, y_bf16 ? 2 : 4) || misaligned(x_scale, 4))
        return TSVD_E_ALIGN;
    const tsvd_status_t grown = i8_grow(h, B);
    if (grown != TSVD_OK) return grown;
    cudaStream_t st = (cudaStream_t)stream;
    const int groups = (B + 255) / 256 * 32;
    float* xs = reinterpret_cast<float*>(h->ws + (size_t)groups * 8 * h->col_blocks * 128);
    const unsigned threads = row_threads((long long)h->col_blocks * 128);
    if (dtype == TSVD_F32)
        stage_rows_kernel<float><<<(unsigned)B, threads, 0, st>>>((const float*)x, h->N, ldx, nullptr, h->col_blocks, groups, h->ws, xs);
    else if (dtype == TSVD_BF16)
        stage_rows_kernel<__nv_bfloat16><<<(unsigned)B, threads, 0, st>>>((const __nv_bfloat16*)x, h->N, ldx, nullptr, h->col_blocks, groups, h->ws, xs);
    else
        stage_rows_kernel<int8_t><<<(unsigned)B, threads, 0, st>>>((const int8_t*)x, h->N, ldx, x_scale, h->col_blocks, groups, h->ws, xs);
    TSVD_CUDA_OK(cudaGetLastError());
    i8_product_simple_kernel<<<dim3((unsigned)(h->M + 31) / 32, (unsigned)(B + 7) / 8), dim3(32, 8), 0, st>>>(
        h->W, h->ws, xs, h->w_scale, h->bias, h->M, B, h->col_blocks, groups, y, ldy, y_bf16);
    TSVD_CUDA_OK(cudaGetLastError());
    tsvd_count_launch(2);
    return TSVD_OK;
}

extern "C" tsvd_status_t tsvd_i8_info(tsvd_i8_t h, int* M, int* N, size_t* packed_bytes)
{
    if (!h) return TSVD_E_NULL;
    if (M) *M = h->M;
    if (N) *N = h->N;
    if (packed_bytes) *packed_bytes = (size_t)h->row_tiles * 128 * ((size_t)h->col_blocks * 128 + sizeof(float) * (h->bias ? 2 : 1));
    return TSVD_OK;
}

extern "C" tsvd_status_t tsvd_i8_last_status(tsvd_i8_t h)
{
    if (!h) return TSVD_E_NULL;
    int word = 0;
    TSVD_CUDA_OK(cudaMemcpy(&word, h->dev_status, sizeof(int), cudaMemcpyDeviceToHost));
    if (word) TSVD_CUDA_OK(cudaMemset(h->dev_status, 0, sizeof(int)));
    return (word & TSVD_DEV_TIMEOUT) ? TSVD_E_TIMEOUT : TSVD_OK;
}

extern "C" void tsvd_i8_destroy(tsvd_i8_t h)
{
    if (!h) return;
    const int dev = h->device;
    int prev = dev;
    if (cudaGetDevice(&prev) == cudaSuccess && prev != dev) cudaSetDevice(dev);
    cudaDeviceSynchronize();
    i8_free(h);
    if (prev != dev) cudaSetDevice(prev);
}
