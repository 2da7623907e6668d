// 8-bit integers with a scale for each token and channel: quantisation of rows, and the linear layer on them.
#include <new>

#include "rows8.cuh"
#include "serving.cuh"

namespace {

// A thread takes 16 bytes of y at a time (4 or 8 columns), `per_row` threads (a power of two) a row, so that a warp's loads
// and stores are whole lines: with 16 columns a thread, and its stores 64 bytes apart, 2048 x 4096 took 14 us.
// Bound by its stores: 2048 x 4096 to fp32, 42 MB, 6.2 us with q in L2 (the copy bandwidth gives 6.5 from DRAM); 333 x 1001 2.9.
template <typename T>
__global__ void __launch_bounds__(256)
dequantize_rows_kernel(const int8_t* q, long long ldq, const float* scale, int rows, int cols, T* __restrict__ y,
                       long long ldy, int per_row_log, bool wide)
{
    constexpr int N = 16 / (int)sizeof(T);
    pdl_launch_dependents();
    pdl_wait();
    const unsigned row = blockIdx.x * (256u >> per_row_log) + (threadIdx.x >> per_row_log);
    if (row >= (unsigned)rows) return;
    const float s = scale[row];
    const int8_t* src = q + (long long)row * ldq;
    T* dst = y + (long long)row * ldy;
    const int step = N << per_row_log;
#pragma unroll 4
    for (int c = (int)(threadIdx.x & ((1u << per_row_log) - 1)) * N; c < cols; c += step) {
        if (wide && c + N <= cols) {
            alignas(16) int8_t b[N];
            if constexpr (N == 4) *reinterpret_cast<uint32_t*>(b) = *reinterpret_cast<const uint32_t*>(src + c);
            else *reinterpret_cast<uint2*>(b) = *reinterpret_cast<const uint2*>(src + c);
            alignas(16) T t[N];
#pragma unroll
            for (int e = 0; e < N; ++e) t[e] = from_f32<T>((float)b[e] * s);
            *reinterpret_cast<uint4*>(dst + c) = *reinterpret_cast<uint4*>(t);
        } else {
            for (int e = 0; e < N && c + e < cols; ++e) dst[c + e] = from_f32<T>((float)src[c + e] * s);
        }
    }
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

constexpr long long TSVD_ROWS_MOST = 0x7fffffff;
bool misaligned(const void* p, size_t size) { return ((uintptr_t)p & (size - 1)) != 0; }

}  // namespace

extern "C" tsvd_status_t tsvd_quantize(const void* x, tsvd_dtype_t dtype, long long rows, int cols, long long ldx, int8_t* q,
                                       long long ldq, float* scale, void* stream)
{
    if (rows < 0 || rows > TSVD_ROWS_MOST || cols < 1 || ldx < cols || ldq < cols) return TSVD_E_SHAPE;
    if (cols > TSVD_COUNT_MOST) return TSVD_E_TOOBIG;
    if (dtype != TSVD_F32 && dtype != TSVD_BF16) return TSVD_E_DTYPE;
    if (rows == 0) return TSVD_OK;
    if (!x || !q || !scale) return TSVD_E_NULL;
    if (misaligned(x, dtype == TSVD_F32 ? 4 : 2) || misaligned(scale, 4)) return TSVD_E_ALIGN;
    const rows8::RowMajor out{q, ldq, (((uintptr_t)q) & 15) == 0 && (rows == 1 || ldq % 16 == 0)};
    TSVD_CUDA_OK(rows8::quantize(x, dtype, (int)rows, cols, ldx, nullptr, out, scale, (cudaStream_t)stream));
    tsvd_count_launch();
    return TSVD_OK;
}

extern "C" tsvd_status_t tsvd_dequantize(const int8_t* q, long long ldq, const float* scale, long long rows, int cols, void* y,
                                         tsvd_dtype_t dtype, long long ldy, void* stream)
{
    if (rows < 0 || rows > TSVD_ROWS_MOST || cols < 1 || ldy < cols || ldq < cols) return TSVD_E_SHAPE;
    if (cols > TSVD_COUNT_MOST) return TSVD_E_TOOBIG;
    if (dtype != TSVD_F32 && dtype != TSVD_BF16) return TSVD_E_DTYPE;
    if (rows == 0) return TSVD_OK;
    if (!q || !scale || !y) return TSVD_E_NULL;
    if (misaligned(y, dtype == TSVD_F32 ? 4 : 2) || misaligned(scale, 4)) return TSVD_E_ALIGN;
    cudaStream_t st = (cudaStream_t)stream;
    const bool wide = (((uintptr_t)q | (uintptr_t)y) & 15) == 0 && (rows == 1 || (ldq % 8 == 0 && ldy * (dtype == TSVD_F32 ? 4 : 2) % 16 == 0));
    const int pieces = (cols + (dtype == TSVD_F32 ? 3 : 7)) / (dtype == TSVD_F32 ? 4 : 8);
    int log = 8;                                              // threads a row: a block's 256, fewer for short rows
    while (log > 0 && (1 << (log - 1)) >= pieces) --log;
    PdlLaunch l((unsigned)(((rows << log) + 255) / 256), 256, 0, st);
    if (dtype == TSVD_F32)
        TSVD_CUDA_OK(cudaLaunchKernelEx(&l.cfg, dequantize_rows_kernel<float>, q, ldq, scale, (int)rows, cols, (float*)y, ldy, log, wide));
    else
        TSVD_CUDA_OK(cudaLaunchKernelEx(&l.cfg, dequantize_rows_kernel<__nv_bfloat16>, q, ldq, scale, (int)rows, cols, (__nv_bfloat16*)y, ldy, log, wide));
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
    if (cudaDeviceGetAttribute(&h->sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) { (void)cudaGetLastError(); delete h; return TSVD_E_CUDA; }
    h->row_tiles = (M + 127) / 128;
    h->col_blocks = (N + 127) / 128;
    tsvd_status_t st = i8_fill(h, W, ldw, w_scale, bias);
    if (st == TSVD_OK) st = i8_product_prepare(h);
    if (st != TSVD_OK) { i8_free(h); return st; }
    *out = h;
    return TSVD_OK;
}

static size_t i8_ws_bytes(const tsvd_i8_s* h, int B)
{
    const size_t groups = ((size_t)B + 7) / 8;
    return groups * 8 * ((size_t)h->col_blocks * 128 + sizeof(float)) + 64;   // scales are read 16 at a time
}

static tsvd_status_t i8_grow(tsvd_i8_s* h, int B)
{
    const size_t need = i8_ws_bytes(h, B);
    if (need <= h->ws_bytes) return TSVD_OK;
    TSVD_CUDA_OK(cudaDeviceSynchronize());
    if (h->ws) { cudaFree(h->ws); h->ws = nullptr; h->ws_bytes = 0; }
    TSVD_CUDA_OK(cudaMalloc(&h->ws, need));
    h->ws_bytes = need;
    return TSVD_OK;
}

extern "C" tsvd_status_t tsvd_i8_reserve(tsvd_i8_t h, int B_max, tsvd_dtype_t dtype)
{
    if (!h) return TSVD_E_NULL;
    if (B_max < 1) return TSVD_E_SHAPE;
    if (dtype != TSVD_F32 && dtype != TSVD_BF16 && dtype != TSVD_I8) return TSVD_E_DTYPE;
    if (const tsvd_status_t on = on_current_device(h->device); on != TSVD_OK) return on;
    return i8_grow(h, B_max);
}

extern "C" tsvd_status_t tsvd_i8_forward(tsvd_i8_t h, const void* x, long long ldx, const float* x_scale, void* y, long long ldy,
                                         int B, tsvd_dtype_t dtype, unsigned flags, void* stream)
{
    if (!h) return TSVD_E_NULL;
    if (B < 0 || ldx < h->N || ldy < h->M) return TSVD_E_SHAPE;
    if (dtype != TSVD_F32 && dtype != TSVD_BF16 && dtype != TSVD_I8) return TSVD_E_DTYPE;
    const unsigned as = flags & (TSVD_FLAG_OUT_F32 | TSVD_FLAG_OUT_BF16);
    if ((flags & ~(as | TSVD_FLAG_TEST_STALL)) || as == (TSVD_FLAG_OUT_F32 | TSVD_FLAG_OUT_BF16)) return TSVD_E_DTYPE;
    if (x_scale && dtype != TSVD_I8) return TSVD_E_DTYPE;
    if (B == 0) return TSVD_OK;
    if (!x || !y) return TSVD_E_NULL;
    const bool y_bf16 = as ? as == TSVD_FLAG_OUT_BF16 : dtype == TSVD_BF16;
    if (misaligned(x, dtype == TSVD_F32 ? 4 : dtype == TSVD_BF16 ? 2 : 1) || misaligned(y, y_bf16 ? 2 : 4) || misaligned(x_scale, 4))
        return TSVD_E_ALIGN;
    if (const tsvd_status_t on = on_current_device(h->device); on != TSVD_OK) return on;
    const tsvd_status_t grown = i8_grow(h, B);
    if (grown != TSVD_OK) return grown;
    const int groups = (B + 7) / 8;
    float* xs = reinterpret_cast<float*>(h->ws + (size_t)groups * 1024 * h->col_blocks);
    const rows8::Tiles out{h->ws, groups};
    TSVD_CUDA_OK(rows8::quantize(x, dtype, B, h->N, ldx, x_scale, out, xs, (cudaStream_t)stream));
    tsvd_count_launch();
    return i8_product(h, h->ws, xs, B, y, ldy, y_bf16, flags & TSVD_FLAG_TEST_STALL, (cudaStream_t)stream);
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
    if (const tsvd_status_t on = on_current_device(h->device); on != TSVD_OK) return on;
    int word = 0;
    TSVD_CUDA_OK(cudaMemcpy(&word, h->dev_status, sizeof(int), cudaMemcpyDeviceToHost));
    if (word) TSVD_CUDA_OK(cudaMemset(h->dev_status, 0, sizeof(int)));
    if (word) TSVD_CUDA_OK(cudaStreamSynchronize(nullptr));      // other streams do not wait for the memset
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
